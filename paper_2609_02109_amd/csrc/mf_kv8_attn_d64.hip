// Attention over the 8-bit cache, heads of 64.
#include "mf_kv8_attn.h"

namespace mfs {

hipError_t launch_attn8_d64(const KvAttnArgs &a, const KvPlan &p, bool f16, hipStream_t s) { return f16 ? pick_attn8<true, 64>(a, p, s) : pick_attn8<false, 64>(a, p, s); }

}  // namespace mfs
