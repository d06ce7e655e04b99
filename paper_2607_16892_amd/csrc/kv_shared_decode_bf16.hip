// Attention of few rows a request behind shared prefixes, bf16 queries.
#include "kv_decode.h"

namespace dro {
template void launch_kv_decode<bf16>(const KvSharedArgs &, const KvCut &, const uint64_t *, int, int, bool, float *,
                                   float2 *, KvJoin *, hipStream_t);
template void launch_kv_decode<bf16>(const KvJoinedArgs &, const KvCut &, const uint64_t *, int, int, bool, float *,
                                   float2 *, KvJoin *, hipStream_t);
}  // namespace dro
