"""Ways through kv_shared_attention that small calls of chunks do not take: single tokens whose requests
read their prefixes themselves, beside the same by groups, on bad data, between rows of no request and
captured; and steps beyond what a workgroup of the plan holds at once."""
import math

import numpy as np
import pytest

from shared_cases import Shared

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(dev):
    import paper_2607_16892_amd as dro
    c = dro.Context(dev.index or 0)
    yield c
    c.close()


def same(a, b):
    import torch
    return torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])


TYPES = [("bf16", None), ("f16", "fp8"), ("bf16", "mxfp4"), ("f16", "mxfp8")]
ways = pytest.mark.parametrize("wide", [False, True], ids=["itself", "groups"])


@ways
@pytest.mark.parametrize("dtype,cache", TYPES)
def test_bad_data_of_single_tokens(ctx, dev, monkeypatch, wide, dtype, cache):
    """Blocks outside the pool are its nearest ones, lengths are cut to the table and to none, and
    requests that no group names have no prefix, however its ends lie."""
    import torch
    monkeypatch.setattr(Shared, "wide", wide)
    c = Shared(dev, [50, 60, 7], [1, 1, 1], [2], [100], 4, 2, 128, dtype, cache, seed=3)
    k, nb = c.case, c.case.k.shape[0]
    print(f"[gpu] kv shared bad data {dtype}/{cache} wide={wide}", flush=True)
    good = c.shared.table
    table = c.shared.table = good.clone()
    table[0, 1], table[0, 3] = 0, nb - 1
    ref = c.run(ctx)
    table[0, 1], table[0, 3] = -7, 2 ** 31 - 1
    assert same(c.run(ctx), ref)
    c.shared.table, most = k.table[3:], k.table.shape[1] * 16
    c.shared.context = torch.tensor([2 ** 31 - 1], dtype=torch.int32, device=dev)
    full = c.run(ctx)
    c.shared.context = torch.tensor([most], dtype=torch.int32, device=dev)
    assert same(c.run(ctx), full)
    c.shared.table, c.shared.context = good, torch.tensor([100], dtype=torch.int32, device=dev)
    for first, of in (([0, 2], [0, 0, -1]), ([-5, 2 ** 31 - 1], [0, 0, 0]), ([-2 ** 31, 0], [-1] * 3), ([7, 9], [-1] * 3),
                      ([2, 1], [-1] * 3), ([2 ** 31 - 1, -2 ** 31], [-1] * 3), ([1, 2], [-1, 0, -1])):
        c.shared.first, c.of = torch.tensor(first, dtype=torch.int32, device=dev), of
        for kw in (dict(), dict(slopes=torch.tensor([0.1, 0.2, 0.3, 0.4], device=dev)), dict(softcap=20.0)):
            c.check(c.run(ctx, **kw), **kw)
    c.shared.first, c.of = torch.tensor([0, 2], dtype=torch.int32, device=dev), [-1] * 3
    for context in (-3, 0, -2 ** 31):
        c.shared.context = torch.tensor([context], dtype=torch.int32, device=dev)
        c.check(c.run(ctx))


@ways
@pytest.mark.parametrize("dtype,cache", TYPES)
def test_rows_of_no_request_beside_single_tokens(ctx, dev, monkeypatch, wide, dtype, cache):
    import torch
    import paper_2607_16892_amd as dro
    monkeypatch.setattr(Shared, "wide", wide)
    c = Shared(dev, [50, 60, 7, 0], [1, 1, 1, 1], [2], [100], 4, 2, 64, dtype, cache, seed=4)
    k, t16 = c.case, c.case.q.dtype
    ref = c.run(ctx)
    c.check(ref)
    assert (ref["out"][3] == 0).all() and (ref["lse"][3] == -math.inf).all()
    q = torch.zeros((40, 4, 64), dtype=t16, device=dev)
    q[3:7] = k.q
    buf = torch.full((40, 4, 80), 5.0, dtype=t16, device=dev)
    lse = torch.full((40, 4), 5.0, device=dev)
    got = dro.kv_shared_attention(ctx, k.cache, q, k.table[:4], k.start[:5] + 3, k.context[:4], 1, c.shared,
                                  out=buf[..., :64], lse=lse)
    assert got["out"].data_ptr() == buf.data_ptr() and got["lse"] is lse
    assert torch.equal(buf[3:7, :, :64], ref["out"]) and torch.equal(lse[3:7], ref["lse"])
    for part in (slice(0, 3), slice(7, 40)):
        assert (buf[part, :, :64] == 0).all() and (lse[part] == -math.inf).all()
    assert (buf[..., 64:] == 5).all()


@ways
@pytest.mark.parametrize("cache", [None, "mxfp4"])
def test_captured_single_tokens(dev, monkeypatch, wide, cache):
    """Captured without a window, replayed over new queries, longer own contexts and other prefixes
    while larger calls on the same context outgrow the workspace between the replays."""
    import torch
    import paper_2607_16892_amd as dro
    with dro.Context(dev.index or 0) as ctx:
        monkeypatch.setattr(Shared, "wide", wide)
        c = Shared(dev, [50, 60, 7, 300], [1, 1, 1, 1], [3], [500], 8, 2, 128, cache=cache, seed=5)
        ref = c.run(ctx)
        out, lse = torch.zeros_like(ref["out"]), torch.zeros_like(ref["lse"])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream(dev)):
            c.run(ctx, out=out, lse=lse)
        for n in range(4):
            big = Shared(dev, [900 * (n + 1)], [900], [1], [1000], 8, 2, 128, seed=6)
            first = big.run(ctx)
            c.case.q.copy_(torch.randn(c.case.q.shape, generator=torch.Generator().manual_seed(n)))
            c.case.context[:4] = torch.tensor([50 - n, 60, 7 - 2 * n, 300 - 90 * n])
            c.shared.context.fill_(500 - 130 * n)
            out.fill_(9), lse.fill_(9)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert same(dict(out=out, lse=lse), c.run(ctx))
            assert same(big.run(ctx), first)


def _groups(r, R, groups):
    # (group 3 is the widest, group 5 empty)
    sizes = r.multinomial(R - R // 9, np.full(groups, 1.0 / groups))
    sizes[3] += sizes[5]
    sizes[5] = 0
    return sizes.tolist(), r.integers(0, 120, groups).tolist()


@pytest.mark.parametrize("groups", [40, 1300])
def test_single_tokens_of_thousands(ctx, dev, groups):
    """2,100 requests behind few or many prefixes: the plan's searches in memory, tiles of the wide
    groups among more sources than it has threads."""
    r = np.random.default_rng(groups)
    sizes, pre = _groups(r, 2100, groups)
    c = Shared(dev, r.integers(1, 90, 2100).tolist(), [1] * 2100, sizes, pre, 4, 2, 64, seed=groups, before=5)
    print(f"[gpu] kv shared {groups} groups of 2100", flush=True)
    # (each request's oracle takes ten milliseconds: the ends, the widest group's and some others)
    wide, end = c.first_h[3], c.first_h[4]
    rows = sorted({0, 4, 5, 6, 2098, 2099, wide, end - 1, end, *r.integers(0, 2100, 120).tolist()})
    got = c.run(ctx)
    c.check(got, rows=rows)
    assert same(c.run(ctx), got)
    kw = dict(window=70)
    c.check(c.run(ctx, **kw), rows=rows, **kw)


def test_chunks_of_thousands(ctx, dev):
    """2,200 chunks of 123 tokens, 270,600 rows: more tiles than the plan sorts, and more rows than its
    workgroups take at once."""
    import torch
    r = np.random.default_rng(1)
    R, new = 2200, 123
    sizes, pre = _groups(r, R, 700)
    own = (new + r.integers(0, 60, R)).tolist()
    print("[gpu] kv shared 2200 chunks", flush=True)
    c = Shared(dev, own, [new] * R, sizes, pre, 2, 1, 64, seed=1, before=7, fused=False)
    rows = sorted({0, 6, 7, 8, R - 1, R - 2, *r.integers(0, R, 20).tolist()})
    got = c.run(ctx)
    c.check(got, rows=rows)
    kw = dict(window=90, slopes=torch.tensor([0.05, 0.1], device=dev))
    c.check(c.run(ctx, **kw), rows=rows, **kw)
    # the others: as kv_attention, where a request has no prefix, up to two calls' rounding
    got, ref = c.run(ctx), c.case.run(ctx)
    alone = torch.tensor([x < 0 or not c.pre[x] for x in c.of], device=dev).repeat_interleave(new)
    vmax = float(c.case.v.float().abs().max())
    assert int(alone.sum()) > new * 100
    assert float((got["out"] - ref["out"])[alone].abs().max()) <= 4 * 2.0 ** -8 * vmax
    assert float((got["lse"] - ref["lse"])[alone].abs().max()) <= 1e-4
