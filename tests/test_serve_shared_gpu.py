"""The serving loop behind shared prefixes and over caches in shared scales, and the calls together:
tables, store, attention behind prefixes, and what kv_load reads back."""
import importlib.util
import os

import numpy as np
import pytest

from kv_cases import Case

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("serve_step", os.path.join(ROOT, "examples", "serve_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("cache,share", [("mxfp4", False), ("mxfp8", False), ("bf16", True), ("mxfp4", True), ("fp8", True)])
def test_the_loop(dev, cache, share):
    import torch
    seen = []
    out = _example().serve(str(dev), steps=60, cache=cache, slots=18, blocks=900, share=share,
                           collect=lambda step, x: seen.append(bool(torch.isfinite(x).all())))
    print(f"[gpu] serve {out}", flush=True)
    assert out["tokens"] > 500 and all(seen) and len(seen) == 60
    assert out["free"] + out["in_use"] == out["blocks"]


@pytest.mark.parametrize("cache,dtype", [("bf16", "bf16"), ("mxfp4", "bf16"), ("mxfp8", "f16"), ("fp8", "f16")])
def test_steps_of_a_service(dev, cache, dtype):
    """Two prefixes and five requests through chunks and single tokens: every row agrees with fp64
    attention over what kv_load reads back of its prefix and its own tokens."""
    import torch
    import paper_2607_16892_amd as dro
    Hq, H, D, block = 8, 2, 64, 16
    t16 = torch.bfloat16 if dtype == "bf16" else torch.float16
    first_h, R = [0, 3, 5], 7                                     # requests 5 and 6 are the prefixes
    g = torch.Generator().manual_seed(3)
    i32 = dict(dtype=torch.int32, device=dev)
    with dro.Context(dev.index or 0) as ctx:
        kind = {"bf16": torch.bfloat16, "fp8": torch.float8_e4m3fn}.get(cache, cache)
        c = dro.KvCache.empty(40, block, H, D, kind, dev)
        pool = dro.BlockPool.empty(R, 20, 40, block, dev)
        held = np.zeros(R, int)
        for step, add in enumerate(([0, 0, 0, 0, 0, 70, 33], [9, 1, 30, 5, 2, 40, 0], [1, 1, 1, 300, 1, 0, 0],
                                    [1, 1, 40, 1, 1, 0, 1], [-1, 1, 1, 1, 1, 0, 0], [20, 1, 1, -1, 1, 0, 0])):
            length, adds = (torch.tensor(list(x), **i32) for x in (np.where(held < 0, 0, held), add))
            T = int(sum(max(x, 0) for x in add))
            plan = pool.take(dro.kv_block_tables(ctx, pool, length, adds, T))
            qkv = torch.randn((T, Hq + 2 * H, D), generator=g).to(t16).to(dev)
            dro.kv_store(ctx, c, qkv[:, Hq:Hq + H], qkv[:, Hq + H:], plan["slot"])
            new = [max(x, 0) for x in add]
            shared = dro.SharedPrefixes(torch.tensor(first_h, **i32), plan["context"][5:], pool.table[5:],
                                        max(sum(new[:3]), sum(new[3:5])))
            got = dro.kv_shared_attention(ctx, c, qkv[:, :Hq], pool.table, plan["start"], plan["context"],
                                          max(new), shared)
            granted = plan["granted"].tolist()
            held = np.where(np.array(add) < 0, 0, held + np.where(granted, new, 0))
            ctx_h = plan["context"].tolist()

            def tokens(r, n):
                p = torch.arange(n, device=dev)
                slot = pool.table[r].long()[p // block] * block + p % block
                back = dro.kv_load(ctx, c, slot, dtype=t16)
                return [back[x].double().cpu().numpy() for x in "kv"]

            for r in range(R):
                if new[r] == 0:
                    continue
                if not granted[r] or add[r] < 0:
                    continue                                      # its rows have no tokens
                pre = 5 if r < 3 else 6 if r < 5 else None
                S = 0 if pre is None else ctx_h[pre]
                own = tokens(r, ctx_h[r])
                keys = own if not S else [np.concatenate(x) for x in zip(tokens(pre, S), own)]
                view = Case.__new__(Case)
                view.dtype, view.D, view.start = dtype, D, plan["start"]
                view.ctx, view.new = [S + ctx_h[r]] * R, new
                view.q_h, view.keys = qkv[:, :Hq].cpu(), lambda _: keys
                view.check(got, prefix=[S] * R, rows=[r])
        assert int(pool.free) + int(pool.held.sum()) == 40
