// Attention over the 8-bit cache, heads of 128.
#include "mf_kv8_attn.h"

namespace mfs {

hipError_t launch_attn8_d128(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s) { return f16 ? pick_attn8<true, 128>(a, p, s) : pick_attn8<false, 128>(a, p, s); }

}  // namespace mfs
