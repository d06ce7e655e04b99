// Attention of many rows a request, bf16 queries.
#include "kv_prefill.h"

namespace dro {
template void launch_kv_prefill<bf16>(const KvMxArgs &, const KvCut &, const KvTiles &, unsigned, int, int, bool, float *,
                                    float2 *, KvJoin *, hipStream_t);
int kv_prefill_groups(int DP) { return prefill_groups(DP); }
int kv_prefill_rows(int DP) { return prefill_rows(DP); }
int kv_prefill_keys(int DP) { return prefill_keys(DP); }
}  // namespace dro
