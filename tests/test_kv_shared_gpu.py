"""kv_shared_attention against the definition in fp64 over each request's prefix and own keys."""
import ctypes as ct
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


@pytest.fixture(params=[False, True], ids=["narrow", "wide"], autouse=True)
def wide(request, monkeypatch):
    """Both ways of a call of single tokens: requests that read their prefixes themselves, and groups."""
    monkeypatch.setattr(Shared, "wide", request.param)


def same(a, b):
    import torch
    return torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])


TYPES = [("bf16", None), ("f16", None), ("bf16", "fp8"), ("f16", "fp8"), ("bf16", "mxfp4"), ("f16", "mxfp4"),
         ("bf16", "mxfp8"), ("f16", "mxfp8")]
SHAPES = [(8, 1, 128, 16), (14, 2, 128, 32), (3, 3, 64, 16), (6, 2, 96, 64), (4, 2, 256, 16), (5, 5, 160, 16)]
OWN = [1, 17, 33, 64, 5, 200, 1, 90, 128, 31, 2, 300]


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("Hq,H,D,block", SHAPES)
def test_single_tokens(ctx, dev, dtype, cache, Hq, H, D, block):
    """Groups of 1 to 5 requests, one of none, one of no shared tokens, and requests without a group
    before and behind them."""
    print(f"[gpu] kv shared decode {dtype}/{cache} Hq={Hq} H={H} D={D} block={block}", flush=True)
    c = Shared(dev, OWN, [1] * 12, [1, 5, 0, 2, 2], [65, 130, 40, 0, 1], Hq, H, D, dtype, cache, before=1,
               block=block, seed=D + Hq)
    c.check(c.run(ctx))


@pytest.mark.parametrize("dtype,cache", TYPES)
@pytest.mark.parametrize("Hq,H,D,block", SHAPES[:5])
def test_chunks(ctx, dev, dtype, cache, Hq, H, D, block):
    """Chunks, whole own prompts, single tokens and no tokens; group rows of one tile and several."""
    print(f"[gpu] kv shared chunks {dtype}/{cache} Hq={Hq} H={H} D={D} block={block}", flush=True)
    c = Shared(dev, [300, 17, 1, 129, 64, 90, 0, 33, 150], [45, 17, 1, 0, 2, 90, 0, 1, 130], [4, 1, 2], [257, 31, 700],
               Hq, H, D, dtype, cache, block=block, seed=D + Hq, layout="tokens")
    c.check(c.run(ctx))


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("opts", [dict(softcap=5.0), dict(window=1), dict(window=33), dict(window=170), dict(window=400),
                                  dict(slopes=0.3), dict(slopes=0.3, window=150), dict(prefix=True),
                                  dict(prefix=True, window=90), dict(scale=-0.1), dict(scale=0.0),
                                  dict(softcap=30.0, slopes=0.1, window=120, prefix=True, scale=0.2)])
@pytest.mark.parametrize("D,dtype,cache", [(128, "bf16", None), (64, "f16", None), (128, "bf16", "mxfp4")])
def test_scores_and_masks(ctx, dev, new, opts, D, dtype, cache):
    """Caps, biases by the positions behind the prefix, and windows that end before, in and behind it,
    for each request elsewhere."""
    import torch
    print(f"[gpu] kv shared options {opts} new={new} D={D}", flush=True)
    lens = [new, new + 1, new + 30, new + 64, new + 150, new + 5, new + 90]
    c = Shared(dev, lens, [new] * 7, [4, 2], [200, 77], 6, 2, D, dtype, cache, seed=new + D, scale_q=2.0)
    kw = dict(opts)
    if "slopes" in kw:
        kw["slopes"] = (kw["slopes"] * torch.arange(1, 7, dtype=torch.float32) / 6).to(dev)
    if "prefix" in kw:
        kw["prefix"] = torch.tensor([0, 5, new + 30, new + 500, 40, 0, 7], dtype=torch.int32, device=dev)
    c.check(c.run(ctx, **kw), **kw)


@pytest.mark.parametrize("max_new", [None, 0, 10 ** 9])
@pytest.mark.parametrize("D,dtype,cache", [(128, "bf16", None), (64, "f16", "fp8")])
def test_many(ctx, dev, D, dtype, cache, max_new):
    """More requests and more groups than a wave has lanes, and a long prefix split over workgroups;
    bounds of the rows that do not hold lose no row."""
    r = np.random.default_rng(3)
    R, G = 180, 70
    lens = r.integers(1, 60, R).tolist()
    sizes = r.multinomial(R - 5, np.full(G, 1 / G)).tolist()
    pre = r.integers(0, 150, G).tolist()
    pre[7] = 6001
    c = Shared(dev, lens, [1] * R, sizes, pre, 4, 2, D, dtype, cache, seed=D)
    if max_new is not None:
        c.shared.max_new = max_new
    got = c.run(ctx)
    c.check(got)
    assert same(c.run(ctx), got)


@pytest.mark.parametrize("R", [3, 90])
def test_one_group(ctx, dev, R):
    """Everybody behind one long prefix."""
    r = np.random.default_rng(R)
    c = Shared(dev, r.integers(1, 300, R).tolist(), [1] * R, [R], [3000], 8, 2, 128, seed=R)
    c.check(c.run(ctx))


def test_rows_that_see_nothing(ctx, dev):
    """No shared token and no own one, or fewer own tokens than rows; beside a prefix the rows before
    the first own token see that alone, and below a window of one token nothing."""
    import torch
    c = Shared(dev, [4, 0, 9, 3], [9, 2, 9, 1], [2, 1], [0, 50], 4, 2, 128, seed=2)
    got = c.run(ctx)
    c.check(got)
    assert (got["out"][:5] == 0).all() and (got["lse"][:5] == -math.inf).all()
    assert (got["out"][9:11] == 0).all() and (got["lse"][9:11] == -math.inf).all()
    c = Shared(dev, [2, 0], [5, 3], [2], [50], 4, 2, 128, seed=2)
    for window in (0, 4, 2, 1):
        c.check(c.run(ctx, window=window), window=window)
    none = Shared(dev, [40, 3], [5, 1], [], [], 4, 2, 128, seed=2)       # no group at all
    assert same(none.run(ctx), none.case.run(ctx))


@pytest.mark.parametrize("new", [1, 50])
@pytest.mark.parametrize("dtype,cache,D", [("bf16", None, 128), ("f16", "fp8", 64), ("bf16", "mxfp4", 128), ("f16", None, 256)])
def test_hidden_places_may_hold_anything(ctx, dev, new, dtype, cache, D):
    """NaN behind the prefixes' ends, in blocks of nobody, and before the windows; and in a token of
    the prefix that only one request's window reaches."""
    import torch
    lens = [new + 2, new + 40, new + 90]
    c = Shared(dev, lens, [new] * 3, [3], [101], 4, 2, D, dtype, cache, seed=D + new)
    k = c.case
    nan = {"fp8": 0x7f, None: {"bf16": 0x7fc0, "f16": 0x7e00}[dtype]}.get(cache)

    def spoil(b, i, keys=True):
        if cache == "mxfp4":
            for t in ((k.cache.k_power, k.cache.v_power) if keys else (k.cache.v_power,)):
                t[b, i] = 255
        else:
            for t in ((k.k, k.v) if keys else (k.v,)):
                t.view(torch.uint8 if cache else torch.int16)[b, i] = nan

    ref, used = c.run(ctx), torch.zeros(k.k.shape[:2], dtype=torch.bool)
    win = c.run(ctx, window=new + 60)
    c.check(win, window=new + 60)
    for r, L in enumerate(lens + [101]):
        p = torch.arange(L)
        used[k.table_h[r, p // 16].long(), p % 16] = True
    b, i = (x.to(dev) for x in torch.nonzero(~used, as_tuple=True))
    spoil(b, i)
    assert same(c.run(ctx), ref)
    # request 0's first row is at 101 + 2 and sees from 101 + 2 - (new + 60) + 1 on, later ones the same (from
    # the beginning) or less
    first = max(104 - (new + 60), 0)
    p = torch.arange(first)
    b, i = k.table_h[3, p // 16].long().to(dev), (p % 16).to(dev)
    spoil(b, i)
    assert same(c.run(ctx, window=new + 60), win)
    spoil(k.table_h[3, first // 16].long().to(dev)[None], torch.tensor([first % 16], device=dev), keys=False)
    got = c.run(ctx, window=new + 60)
    hit = torch.zeros_like(win["out"], dtype=torch.bool)
    hit[: min(new, new + 60 + first - 103)] = True   # rows i with 103 + i - first < new + 60
    assert torch.isnan(got["out"][hit]).all()
    assert torch.equal(got["out"][~hit], win["out"][~hit]) and torch.equal(got["lse"], win["lse"])


def test_bad_data_stays_inside(ctx, dev):
    """Blocks outside the pool are its nearest ones, lengths are cut to the table, groups beyond the
    requests to them."""
    import torch
    c = Shared(dev, [50, 60, 7], [1, 20, 1], [2], [100], 4, 2, 128, seed=3)
    k, nb = c.case, c.case.k.shape[0]
    table = c.shared.table.clone()
    table[0, 1], table[0, 3] = 0, nb - 1
    c.shared.table = table
    ref = c.run(ctx)
    table[0, 1], table[0, 3] = -7, 2 ** 31 - 1
    assert same(c.run(ctx), ref)
    c.shared.table, c.shared.context = k.table[3:], torch.tensor([2 ** 31 - 1], dtype=torch.int32, device=dev)
    full = c.run(ctx)
    c.shared.context = torch.tensor([k.table.shape[1] * 16], dtype=torch.int32, device=dev)
    assert same(c.run(ctx), full)
    if Shared.wide:
        c.shared.table = table
    for first in ([-5, 2 ** 31 - 1], [-2 ** 31, 0], [7, 9], [2, 1], [2 ** 31 - 1, -2 ** 31]):
        c.shared.first = torch.tensor(first, dtype=torch.int32, device=dev)
        c.run(ctx, window=30)
        c.run(ctx, slopes=torch.ones(4, device=dev))
    torch.cuda.synchronize()
    c.shared.first = torch.tensor([0, 2], dtype=torch.int32, device=dev)
    c.shared.context = torch.tensor([-3], dtype=torch.int32, device=dev)       # counts as none
    got = c.run(ctx)
    c.shared.context = torch.zeros(1, dtype=torch.int32, device=dev)
    assert same(c.run(ctx), got)


def test_rows_of_no_request_and_strides(ctx, dev):
    """Rows before and behind the requests' are zero; out and lse may be given, rows strided."""
    import torch
    import paper_2607_16892_amd as dro
    c = Shared(dev, [50, 60, 7], [1, 20, 1], [2], [100], 4, 2, 64, "f16", seed=4)
    k = c.case
    ref = c.run(ctx)
    q = torch.zeros((40, 4, 64), dtype=torch.float16, device=dev)
    q[3:25] = k.q
    buf = torch.full((40, 4, 80), 5.0, dtype=torch.float16, device=dev)
    lse = torch.full((40, 4), 5.0, device=dev)
    got = dro.kv_shared_attention(ctx, k.cache, q, k.table[:3], k.start[:4] + 3, k.context[:3], 20, c.shared,
                                  out=buf[..., :64], lse=lse)
    assert got["out"].data_ptr() == buf.data_ptr() and got["lse"] is lse
    assert torch.equal(buf[3:25, :, :64], ref["out"]) and torch.equal(lse[3:25], ref["lse"])
    for part in (slice(0, 3), slice(25, 40)):
        assert (buf[part, :, :64] == 0).all() and (lse[part] == -math.inf).all()
    assert (buf[..., 64:] == 5).all()
    none = dro.kv_shared_attention(ctx, k.cache, q[:0], k.table[:3], k.start[:4], k.context[:3], 1, c.shared)
    assert none["out"].shape == (0, 4, 64)


@pytest.mark.parametrize("new", [1, 30])
def test_against_attention_over_joined_tables(ctx, dev, new):
    """Where prefixes fill whole blocks, as kv_attention over tables that name them for each request,
    up to the rounding of the weights and of the output: two calls' errors of 2 u of sum w |v|."""
    import torch
    c = Shared(dev, [new + 9, new + 70, new + 16], [new] * 3, [3], [96], 8, 2, 128, seed=new)
    k = c.case
    got = c.run(ctx)
    c.check(got)
    table = torch.cat([k.table[3:, :6].expand(3, -1), k.table[:3]], 1).contiguous()
    import paper_2607_16892_amd as dro
    ref = dro.kv_attention(ctx, k.cache, k.q, table, k.start[:4], k.context[:3] + 96, new)
    vmax = float(k.v.float().abs().max())
    assert float((got["out"].float() - ref["out"].float()).abs().max()) <= 4 * 2.0 ** -8 * vmax
    assert float((got["lse"] - ref["lse"]).abs().max()) <= 1e-4


def test_a_captured_step_between_other_calls(dev):
    """Captured once, replayed after larger calls have outgrown the workspace and over new inputs."""
    import torch
    with __import__("paper_2607_16892_amd").Context(dev.index or 0) as ctx:
        c = Shared(dev, [50, 60, 7, 300], [1, 1, 1, 1], [3], [500], 8, 2, 128, seed=5)
        ref = c.run(ctx, window=400)
        out, lse = torch.zeros_like(ref["out"]), torch.zeros_like(ref["lse"])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream(dev)):
            c.run(ctx, window=400, out=out, lse=lse)
        big = Shared(dev, [900], [900], [1], [1000], 8, 2, 128, seed=6)
        for seed in range(3):
            first = big.run(ctx)
            g = torch.Generator().manual_seed(seed)
            c.case.q.copy_(torch.randn(c.case.q.shape, generator=g))
            out.fill_(9), lse.fill_(9)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert same(dict(out=out, lse=lse), c.run(ctx, window=400))
            assert same(big.run(ctx), first)


def test_two_streams_in_turn(dev):
    """Contexts of their own on two streams at once, and one context on a side stream."""
    import torch
    import paper_2607_16892_amd as dro
    with dro.Context(dev.index or 0) as one, dro.Context(dev.index or 0) as two:
        a = Shared(dev, [50, 600], [1, 1], [2], [900], 8, 2, 128, seed=5)
        b = Shared(dev, [70, 40, 3], [30, 1, 1], [3], [400], 8, 2, 128, seed=6)
        ra, rb = a.run(one), b.run(one)
        torch.cuda.synchronize()
        s, t = torch.cuda.Stream(dev), torch.cuda.Stream(dev)
        got = [(a.run(one, stream=s), b.run(two, stream=t)) for _ in range(5)]
        torch.cuda.synchronize()
        assert all(same(x, ra) and same(y, rb) for x, y in got)


def test_refusals(ctx, dev):
    import torch
    import paper_2607_16892_amd as dro
    from paper_2607_16892_amd import _native
    c = Shared(dev, [50, 60], [1, 1], [2], [100], 4, 2, 128, seed=3)
    k, s = c.case, c.shared

    def shared(**kw):
        return dro.SharedPrefixes(**{**dict(first=s.first, context=s.context, table=s.table, max_new=2), **kw})

    for bad, error in ((None, TypeError), (shared(first=s.first[:1]), ValueError), (shared(first=s.first.long()), TypeError),
                       (shared(context=s.context.cpu()), TypeError), (shared(context=s.first), ValueError),
                       (shared(table=s.table.long()), ValueError), (shared(table=s.table.cpu()), TypeError),
                       (shared(max_new=-1), dro.DroError), (shared(table=s.table[0]), ValueError)):
        with pytest.raises(error):
            c.run(ctx, shared=bad)
    with pytest.raises(dro.DroError):
        c.run(ctx, window=-1)
    q = k.q
    k.q = q.clone().requires_grad_()
    with pytest.raises(RuntimeError, match="kv_shared_attention has no backward"):
        c.run(ctx)
    k.q = q
    # the C entry: no shared, a table too narrow for its stride, limits
    cs = k.cache.struct()
    out = torch.zeros((2, 4, 128), dtype=torch.bfloat16, device=dev)
    rows = _native.KvRowsStruct(0, 2, 4, 2, q.data_ptr(), q.stride(0), 128, out.data_ptr(), 512, 128, None,
                                k.start.data_ptr(), k.context.data_ptr(), k.table.data_ptr(), k.table.stride(0),
                                k.table.shape[1], 1, 0.1, 0.0, 0, None, None)
    call = ctx._lib.kv_shared_attention
    assert call(ctx.handle, ct.byref(cs), ct.byref(rows), None, None) == -1
    assert call(None, ct.byref(cs), ct.byref(rows), None, None) == -1
    good = s.struct(dev)
    for change, code in ((dict(groups=-1), -1), (dict(first=None), -1), (dict(context=None), -1), (dict(table=None), -1),
                         (dict(max_blocks=0), -1), (dict(table_stride=1), -1), (dict(max_blocks=1 << 27, table_stride=1 << 27), -5),
                         (dict(groups=(1 << 20) + 1), -5)):
        bad = _native.KvSharedStruct.from_buffer_copy(good)
        for name, value in change.items():
            setattr(bad, name, value)
        assert call(ctx.handle, ct.byref(cs), ct.byref(rows), ct.byref(bad), None) == code, change
    assert call(ctx.handle, ct.byref(cs), ct.byref(rows), ct.byref(good), None) == 0
    torch.cuda.synchronize()
