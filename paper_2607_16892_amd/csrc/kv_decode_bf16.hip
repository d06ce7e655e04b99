// Decode attention with bf16 queries.
#include "kv_decode.h"

namespace dro {
template void launch_kv_decode<bf16>(const KvAttnArgs &, const KvCut &, const KvPlan &, int, int, uint32_t,
                                     uint32_t, bool, float *, float2 *, hipStream_t);
}  // namespace dro
