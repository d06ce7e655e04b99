// Attention of few rows a request, bf16 queries.
#include "kv_decode.h"

namespace dro {
template void launch_kv_decode<bf16>(const KvMxArgs &, const KvCut &, const uint64_t *, int, int, bool, float *,
                                   float2 *, KvJoin *, hipStream_t);
int kv_decode_waves(int cache_dtype, int DP)
{
    return cache_dtype == DRO_MXFP4      ? decode_waves_of<mx4>(DP)
           : cache_dtype == DRO_MXFP8    ? decode_waves_of<mx8>(DP)
           : cache_dtype == DRO_FP8_E4M3 ? decode_waves_of<fp8>(DP)
                                         : decode_waves_of<bf16>(DP);
}
}  // namespace dro
