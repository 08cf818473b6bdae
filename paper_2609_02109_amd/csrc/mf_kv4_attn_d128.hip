// Attention over the 4-bit cache, heads of 128 (mf_kv4_attn.h).
#include "mf_kv4_attn.h"

namespace mfs {

hipError_t launch_attn_d128(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s)
{
    if (a.g.group == 32) return f16 ? pick_attn<true, 128, 32>(a, p, s) : pick_attn<false, 128, 32>(a, p, s);
    if (a.g.group == 64) return f16 ? pick_attn<true, 128, 64>(a, p, s) : pick_attn<false, 128, 64>(a, p, s);
    return f16 ? pick_attn<true, 128, 128>(a, p, s) : pick_attn<false, 128, 128>(a, p, s);
}

}  // namespace mfs
