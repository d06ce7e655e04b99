"""The bias by distance of kv_attention by another way of computing it."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(dev):
    import paper_2607_16892_amd as dro
    c = dro.Context(dev.index or 0)
    yield c
    c.close()


@pytest.mark.parametrize("new", [1, 9, 200])
@pytest.mark.parametrize("Hq,H,D,dtype,cap", [(6, 2, 128, "bf16", 0.0), (12, 12, 64, "f16", 0.0), (4, 2, 256, "bf16", 15.0)])
def test_a_bias_by_distance_is_one_by_the_key(ctx, dev, new, Hq, H, D, dtype, cap):
    """slope (j - p) differs from slope j by what is the same for all keys of a row, ahead of it
    (in a prefix) or behind, so the softmax is that of s_j + slope j, and lse lies slope p below.
    (Tolerances as in kv_cases, for scores and biases up to `tops`.)"""
    import torch
    from kv_cases import Case
    print(f"[gpu] kv slopes Hq={Hq} D={D} new={new}", flush=True)
    L = [new + 120, new + 7]
    c = Case(dev, L, [new] * 2, Hq, H, D, dtype, seed=D + new)
    slopes = 0.2 * torch.arange(1, Hq + 1, dtype=torch.float32) / Hq
    prefix = torch.tensor([new + 100, 3], dtype=torch.int32, device=dev)
    got = c.run(ctx, slopes=slopes.to(dev), prefix=prefix, softcap=cap)
    u = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11
    for r in range(2):
        k, v = (torch.from_numpy(x) for x in c.keys(r))
        j, p = torch.arange(L[r]), L[r] - new + torch.arange(new)[:, None]
        see = (j <= p) | (j < int(prefix[r]))
        for hq in range(Hq):
            kk, vv, q = k[:, hq // (Hq // H)], v[:, hq // (Hq // H)], c.q_h[r * new:(r + 1) * new, hq].double()
            s = q @ kk.T * D ** -0.5
            dots = (q.abs() @ kk.abs().T).max() * D ** -0.5
            if cap:
                s = cap * torch.tanh(s / cap)
            slope = float(slopes[hq])
            tops = (s.abs() + slope * (j - p).abs()).max()
            s = (s + slope * j).masked_fill(~see, -torch.inf)
            w = torch.softmax(s, 1)
            A = w @ vv.abs()
            ds = float((D + 4) * 2.0 ** -24 * dots + 2.0 ** -21 * cap + 4 * 2.0 ** -23 * (tops + 1))
            tol = (2 * u + np.expm1(2 * ds) + (L[r] + 8) * 2.0 ** -24) * A + 2.0 ** -24
            err = (got["out"][r * new:(r + 1) * new, hq].double().cpu() - w @ vv).abs()
            assert (err <= tol).all(), f"request {r} head {hq}: {float((err / tol).max()):.3g} of the bound"
            lse = torch.logsumexp(s, 1) - slope * p[:, 0]
            e = (got["lse"][r * new:(r + 1) * new, hq].double().cpu() - lse).abs()
            assert (e <= ds + (L[r] + 8) * 2.0 ** -24 + 2.0 ** -21 * (1 + tops)).all()
