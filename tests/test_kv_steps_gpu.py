"""No step of keys is lost, read twice or joined with a wrong factor (kv_steps.py; that the bounds
see such mistakes is tested on the CPU)."""
import numpy as np
import pytest

import kv_steps
from kv_cases import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(dev):
    import paper_2607_16892_amd as dro
    c = dro.Context(dev.index or 0)
    yield c
    c.close()


def _name_blocks(c):
    """v of block i of every request: the unit vector i % D (times the head's scale)."""
    import torch
    eye = torch.eye(c.D, device=c.dev).to(c.v.dtype)
    bits = torch.uint8 if c.cache_type == "fp8" else torch.int16
    for r, L in enumerate(c.ctx):
        n = -(-L // c.block)
        if n:
            rows = eye.view(bits)[torch.arange(n, device=c.dev) % c.D]
            c.v.view(bits)[c.table[r, :n].long()] = rows[:, None, None, :]


def _check(c, got, window=0, softcap=0.0):
    out = got["out"].double().cpu().numpy()
    G = c.Hq // c.H
    worst = 0.0
    for r in range(0, len(c.ctx), 1 + len(c.ctx) // 9):
        L, n, a = c.ctx[r], c.new[r], sum(c.new[:r])
        if not n:
            continue
        ids = c.table_h[r, : -(-L // c.block)].long()
        for hq in sorted({0, c.Hq - 1}):
            h = hq // G
            k = c.k_h[ids, :, h].float().double().numpy().reshape(-1, c.D)[:L]
            k = k if c.ks is None else k * float(c.ks[h])
            unit = 1.0 if c.vs is None else float(c.vs[h])
            for i in sorted({0, n // 2, n - 1}):
                p = L - n + i
                q = c.q_h[a + i, hq].double().numpy()
                w, ds = kv_steps.weights(q, k, c.D ** -0.5, p, window, softcap)
                m = kv_steps.masses(w, c.block, c.D)
                tol = kv_steps.bound(m, L, ds, c.dtype) * unit + 2.0 ** -25 * (c.dtype == "f16")
                err = np.abs(out[a + i, hq] - m * unit)
                worst = max(worst, float((err / tol).max()))
                assert (err <= tol).all(), (f"request {r} (context {L}, rows {n}) row {i} head {hq}: component "
                                            f"{np.argmax(err / tol)}, {np.max(err / tol):.3g} of the bound")
    print(f"[gpu] kv steps: worst {worst:.3g} of the bound", flush=True)


@pytest.mark.parametrize("Hq,H,D,dtype,cache,lens,new,kw", [
    # single tokens: long ones cut many times, short ones whole, two tiles of heads
    (8, 1, 128, "bf16", None, [100_000, 20_000, 77], [1, 1, 1], dict()),
    (8, 2, 128, "bf16", "fp8", [60_000, 500, 33], [1, 1, 1], dict()),
    (4, 1, 64, "f16", None, [90_000], [1], dict()),
    (6, 2, 64, "f16", "fp8", [40_000, 9], [1, 1], dict(softcap=20.0)),
    (4, 1, 256, "bf16", None, [30_000, 4000], [1, 1], dict()),
    (2, 1, 256, "f16", "fp8", [30_000, 4000], [1, 1], dict()),
    (40, 1, 64, "bf16", None, [20_000, 1000], [1, 1], dict()),
    (5, 1, 80, "bf16", None, [30_000, 70], [1, 1], dict(window=12_000)),
    (8, 2, 128, "bf16", None, [500 + 61 * i for i in range(130)], [1] * 130, dict()),       # listed by a launch
    (8, 1, 64, "bf16", None, [300 + 211 * i for i in range(32)], [2] * 32, dict()),
    (4, 1, 128, "f16", None, [9000], [5], dict()),
    # chunks: tiles cut and joined, whole, beside single tokens
    (8, 1, 128, "bf16", None, [60_000], [100], dict()),
    (8, 1, 128, "f16", None, [60_000, 300], [64, 300], dict()),
    (8, 2, 256, "bf16", "fp8", [20_000, 50], [70, 50], dict(softcap=10.0)),
    (4, 2, 256, "f16", None, [9000, 2000], [50, 9], dict()),
    (7, 1, 80, "f16", None, [30_000, 3], [100, 3], dict(window=12_000)),
    (4, 2, 64, "bf16", "fp8", [30_000, 700], [200, 700], dict()),
    (3, 1, 192, "bf16", None, [20_000, 90], [90, 33], dict()),
    (16, 16, 64, "bf16", None, [3000], [3000], dict()),
    (16, 2, 128, "bf16", None, [60 + 61 * i for i in range(69)] + [30_000],
     [1] * 69 + [200], dict()),                                                             # both kernels
    (8, 8, 64, "f16", None, [90 + i % 9 for i in range(1100)], [60 if i % 92 == 0 else 1 for i in range(1100)], dict()),
])
def test_every_step_counts_once(ctx, dev, Hq, H, D, dtype, cache, lens, new, kw):
    print(f"[gpu] kv steps Hq={Hq} H={H} D={D} {dtype}/{cache} requests {len(lens)}", flush=True)
    c = Case(dev, lens, new, Hq, H, D, dtype, cache, seed=Hq + D + len(lens))
    _name_blocks(c)
    _check(c, c.run(ctx, **kw), **kw)


@pytest.mark.parametrize("most", [1, 3, 20, 500])
def test_every_step_counts_once_whatever_the_bound(ctx, dev, most):
    c = Case(dev, [20_000, 300, 900], [1, 20, 130], 8, 2, 128, "bf16", seed=most)
    _name_blocks(c)
    _check(c, c.run(ctx, max_new=most))
