// Attention of few rows a request, bf16 queries.
#include "kv_decode.h"

namespace dro {
template void launch_kv_decode<bf16>(const KvAttnArgs &, const KvCut &, const uint64_t *, int, int, bool, float *,
                                   float2 *, KvJoin *, hipStream_t);
int kv_decode_waves(int cache_dtype, int DP) { return decode_waves(DP, cache_dtype == DRO_FP8_E4M3 ? 1 : 2); }
}  // namespace dro
