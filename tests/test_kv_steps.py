"""The comparison of test_kv_steps_gpu.py sees a lost step: mistakes planted in the oracle."""
import numpy as np
import pytest

import kv_steps


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("L,D", [(300, 64), (5000, 128), (20_000, 64), (60_000, 128), (131_000, 256)])
def test_the_bound_sees_one_step_lost_or_misjoined(L, D, dtype):
    r = np.random.default_rng(L + D)
    k, q = r.standard_normal((L, D)), r.standard_normal(D)
    w, ds = kv_steps.weights(q, k, D ** -0.5, L - 1)
    ref = kv_steps.masses(w, 16, D)
    tol = kv_steps.bound(ref, L, ds, dtype)
    seen = 0
    starts = r.integers(0, L // 32, 200) * 32
    for a in starts:
        for wrong in (lambda x: 0 * x, lambda x: 2 * x, lambda x: x / 2):      # lost, twice, a factor
            bad = w.copy()
            bad[a:a + 32] = wrong(bad[a:a + 32])
            seen += bool((np.abs(kv_steps.masses(bad, 16, D) - ref) > tol).any())
    # (steps whose keys hardly weigh may be lost unseen)
    assert seen >= 0.95 * 3 * len(starts)
