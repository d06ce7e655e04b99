// Attention of many rows a request, f16 queries.
#include "kv_prefill.h"

namespace dro {
template void launch_kv_prefill<f16>(const KvAttnArgs &, const KvCut &, const KvTiles &, unsigned, int, int, bool, float *,
                                    float2 *, KvJoin *, hipStream_t);
}  // namespace dro
