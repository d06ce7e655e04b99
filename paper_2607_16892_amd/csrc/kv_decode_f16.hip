// Attention of few rows a request, f16 queries.
#include "kv_decode.h"

namespace dro {
template void launch_kv_decode<f16>(const KvAttnArgs &, const KvCut &, const uint64_t *, int, int, bool, float *,
                                   float2 *, KvJoin *, hipStream_t);
}  // namespace dro
