// Attention over the 4-bit cache, heads of 64 (mf_kv4_attn.h).
#include "mf_kv4_attn.h"

namespace mfs {

hipError_t launch_attn_d64(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s)
{
    if (a.g.group == 32) return f16 ? pick_attn<true, 64, 32>(a, p, s) : pick_attn<false, 64, 32>(a, p, s);
    return f16 ? pick_attn<true, 64, 64>(a, p, s) : pick_attn<false, 64, 64>(a, p, s);
}

}  // namespace mfs
