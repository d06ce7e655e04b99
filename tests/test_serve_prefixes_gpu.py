"""What the serving loop holds of its shared prefixes, step by step."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("serve_step", os.path.join(ROOT, "examples", "serve_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("policy,slots,blocks", [("dro", 18, 900), ("mean", 18, 900), ("dro", 48, 3600), ("dro", 2, 900)])
def test_prefixes_keep_their_tokens(dev, monkeypatch, policy, slots, blocks):
    """Once a class's prefix holds its L_pre tokens it holds them in every step after, also where the
    pool is short, brings no rows, and no request of the class has rows before.  (Two slots: steps in
    which nobody has rows.)"""
    import paper_2607_16892_amd as dro
    from workloads.configs import serving_workload
    w, svc = serving_workload(C=6, N=5000, K=513, M=64, L=1024, seed=0)
    steps, attention = [], dro.kv_shared_attention

    def watched(ctx, cache, q, table, start, context, max_new, shared, **kw):
        steps.append([x.tolist() for x in (start, shared.first, shared.context)] + [max_new, shared.max_new])
        return attention(ctx, cache, q, table, start, context, max_new, shared, **kw)

    monkeypatch.setattr(dro, "kv_shared_attention", watched)
    m = _example()
    out = m.serve(str(dev), steps=60, policy=policy, slots=slots, blocks=blocks, share=True)
    print(f"[gpu] serve {out}", flush=True)
    assert len(steps) == 60 * m.LAYERS and out["free"] + out["in_use"] == blocks
    filled = [False] * w.C
    for start, first, context, max_new, group_new in steps[::m.LAYERS]:
        rows = [b - a for a, b in zip(start, start[1:])]
        assert first[0] == 0 and first[-1] == slots and max(rows) <= max_new
        for g, most in enumerate(svc.Lpre.tolist()):
            mine = sum(rows[first[g]:first[g + 1]])
            assert mine <= group_new
            assert not filled[g] or (context[g] == most and rows[slots + g] == 0), (g, context[g], most)
            assert filled[g] or mine == 0
            filled[g] |= context[g] == most
    assert all(filled)
