"""kv_attention against its definition in fp64 (oracle/kv.py)."""
import math

import numpy as np
import pytest

from kv_cases import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(dev):
    import paper_2607_16892_amd as dro
    c = dro.Context(dev.index or 0)
    yield c
    c.close()


EDGES = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 513, 0, 1023]


@pytest.mark.parametrize("dtype,cache", [("bf16", None), ("f16", None), ("bf16", "fp8"), ("f16", "fp8")])
@pytest.mark.parametrize("Hq,H,D,block", [(8, 1, 128, 16), (14, 2, 128, 32), (3, 3, 64, 16),
                                          (32, 2, 80, 16), (4, 2, 256, 64), (40, 1, 8, 128),
                                          (2, 1, 192, 16), (5, 5, 104, 1024)])
def test_single_tokens(ctx, dev, dtype, cache, Hq, H, D, block):
    print(f"[gpu] kv decode {dtype}/{cache} Hq={Hq} H={H} D={D} block={block}", flush=True)
    c = Case(dev, EDGES, [1] * len(EDGES), Hq, H, D, dtype, cache, block, seed=D + Hq)
    c.check(c.run(ctx))


@pytest.mark.parametrize("dtype,cache", [("bf16", None), ("f16", None), ("bf16", "fp8"), ("f16", "fp8")])
@pytest.mark.parametrize("Hq,H,D,block", [(8, 2, 128, 16), (7, 1, 128, 32), (2, 2, 64, 16),
                                          (6, 2, 80, 64), (4, 2, 256, 16)])
def test_chunks(ctx, dev, dtype, cache, Hq, H, D, block):
    # chunks over what is cached, whole prompts, single tokens and no tokens in one call
    print(f"[gpu] kv chunks {dtype}/{cache} Hq={Hq} H={H} D={D} block={block}", flush=True)
    c = Case(dev, [300, 17, 1, 129, 64, 400, 0, 33, 250, 90], [45, 17, 1, 0, 2, 130, 0, 1, 250, 33],
             Hq, H, D, dtype, cache, block, seed=D + Hq, layout="tokens")
    c.check(c.run(ctx))


@pytest.mark.parametrize("new", [1, 9, 70, 200])
@pytest.mark.parametrize("opts", [dict(softcap=5.0), dict(window=1), dict(window=16), dict(window=33),
                                  dict(window=100, softcap=20.0), dict(slopes=0.5), dict(slopes=-0.01),
                                  dict(prefix=True), dict(prefix=True, window=20), dict(scale=0.7),
                                  dict(scale=-0.1), dict(scale=0.0),
                                  dict(softcap=30.0, slopes=0.1, window=64, prefix=True, scale=0.2)])
@pytest.mark.parametrize("D,dtype", [(128, "bf16"), (64, "f16")])
def test_scores_and_masks(ctx, dev, new, opts, D, dtype):
    import torch
    print(f"[gpu] kv options {opts} new={new} D={D}", flush=True)
    lens = [new, new + 1, new + 30, new + 64, new + 333]
    c = Case(dev, lens, [new] * 5, 6, 2, D, dtype, seed=new + D, scale_q=2.0)
    kw = dict(opts)
    if "slopes" in kw:
        kw["slopes"] = (kw["slopes"] * torch.arange(1, 7, dtype=torch.float32) / 6).to(dev)
    if "prefix" in kw:
        kw["prefix"] = torch.tensor([0, 5, new + 30, new + 500, 40], dtype=torch.int32, device=dev)
    got = c.run(ctx, **kw)
    c.check(got, **kw)


@pytest.mark.parametrize("new", [1, 40])
def test_rows_that_see_nothing(ctx, dev, new):
    import torch
    # fewer tokens in the cache than rows (the first rows lie before it), none at all, and a
    # window that a prefix does not reach into
    c = Case(dev, [new // 2, 0, new], [new] * 3, 4, 2, 128, seed=5)
    got = c.run(ctx)
    c.check(got)
    gone = new - new // 2
    assert (got["out"][:gone] == 0).all() and (got["lse"][:gone] == -math.inf).all()
    assert (got["out"][new:2 * new] == 0).all() and (got["lse"][new:2 * new] == -math.inf).all()
    pre = torch.tensor([3, 0, 3], dtype=torch.int32, device=dev)
    got = c.run(ctx, prefix=pre, window=7)
    c.check(got, prefix=pre, window=7)


@pytest.mark.parametrize("Hq,H,D,dtype,cache", [(8, 1, 128, "bf16", None), (14, 2, 128, "f16", "fp8"),
                                                (3, 3, 64, "f16", None), (4, 4, 256, "bf16", None)])
@pytest.mark.parametrize("new", [1, 50])
def test_long_contexts(ctx, dev, Hq, H, D, dtype, cache, new):
    # a long axis split over workgroups, beside short requests
    print(f"[gpu] kv long Hq={Hq} H={H} D={D} {dtype}/{cache} new={new}", flush=True)
    c = Case(dev, [20_011, 70, 3001, 5], [new, new, 1, 1], Hq, H, D, dtype, cache, seed=D)
    c.check(c.run(ctx))


@pytest.mark.parametrize("R,most,new", [(65, 300, 1), (130, 120, 5), (700, 40, 1), (64, 900, 2), (200, 3000, 1),
                                        (1500, 9, 2)])
def test_many_requests(ctx, dev, R, most, new):
    # more requests than a wave has lanes, some without tokens, one long among short ones
    r = np.random.default_rng(R)
    lens = r.integers(0, most + 1, R).tolist()
    lens[R // 3] = 4 * most
    news = [int(min(x, n)) for x, n in zip(lens, r.integers(0, new + 1, R))]
    print(f"[gpu] kv many R={R}", flush=True)
    c = Case(dev, lens, news, 4, 2, 64, "f16", seed=R)
    c.check(c.run(ctx))


@pytest.mark.parametrize("new", [1, 3, 60])
@pytest.mark.parametrize("dtype,D", [("bf16", 128), ("f16", 64), ("bf16", 256)])
def test_hidden_places_may_hold_anything(ctx, dev, new, dtype, D):
    """NaN and infinities beyond the context, in blocks of no request, and in tokens that some
    rows of a chunk see and others do not."""
    import torch
    lens = [new + 5, new + 40, 64 + new]
    c = Case(dev, lens, [new] * 3, 4, 2, D, dtype, seed=new + D)
    ref = c.run(ctx)
    c.check(ref)
    used = torch.zeros(c.k.shape[:2], dtype=torch.bool)
    for r, L in enumerate(lens):
        p = torch.arange(L)
        used[c.table_h[r, p // 16].long(), p % 16] = True
    for bad in (float("nan"), float("inf")):
        hide = (~used).to(dev)
        c.k[hide], c.v[hide] = bad, -bad
        got = c.run(ctx)
        assert torch.equal(got["out"], ref["out"]) and torch.equal(got["lse"], ref["lse"])
    if new == 1:
        return
    # the last token of request 1 is seen by its own last row alone
    L = lens[1]
    b = int(c.table_h[1, (L - 1) // 16])
    for x in (c.v, c.k):
        x[b, (L - 1) % 16] = float("nan")
        got = c.run(ctx)
        last = 2 * new - 1
        keep = [t for t in range(3 * new) if t != last]
        assert torch.isnan(got["out"][last]).all()
        assert torch.equal(got["out"][keep], ref["out"][keep])
        assert torch.equal(got["lse"][keep], ref["lse"][keep])


def test_infinite_value_of_one_component(ctx, dev):
    """An infinity among the values reaches only the rows that see it, and only its component."""
    import torch
    n = 40
    c = Case(dev, [n + 30], [n], 4, 2, 128, "bf16", seed=3)
    ref = c.run(ctx)
    j = n + 30 - 10                          # seen by the last ten rows
    b = int(c.table_h[0, j // 16])
    c.v[b, j % 16, 1, 77] = float("inf")
    got = c.run(ctx)
    hit = torch.zeros_like(ref["out"], dtype=torch.bool)
    hit[n - 10:, 2:, 77] = True              # key head 1 serves query heads 2 and 3
    assert (got["out"][hit] == float("inf")).all()
    assert torch.equal(got["out"][~hit], ref["out"][~hit])


def test_table_entries_outside_the_pool_are_not_followed(ctx, dev):
    """Entries beyond the context are never used; bad ones within it read inside the pool."""
    import torch
    c = Case(dev, [40, 90], [1, 20], 4, 2, 128, seed=9)
    ref = c.run(ctx)
    t = c.table.clone()
    t[0, 3:], t[1, 6:] = 2 ** 30, -5
    c.table = t
    got = c.run(ctx)
    assert torch.equal(got["out"], ref["out"])
    c.table[0, 0], c.table[1, 2] = 2 ** 31 - 1, -2 ** 31
    c.run(ctx)
    torch.cuda.synchronize()
    # a context beyond the table is cut to the table
    c.context = torch.tensor([10 ** 9, 90], dtype=torch.int32, device=dev)
    c.run(ctx)
    torch.cuda.synchronize()


@pytest.mark.parametrize("new", [1, 30])
def test_starts_outside_the_rows_are_cut(ctx, dev, new):
    """Starts below 0 and beyond T count as 0 and T; requests whose end is not behind their start
    have no rows."""
    import torch
    c = Case(dev, [50, 60, 70], [new] * 3, 4, 2, 128, seed=2)
    ref = c.run(ctx)
    c.start = torch.tensor([-7, new, 2 * new, 2 ** 31 - 1], dtype=torch.int32, device=dev)
    got = c.run(ctx)
    assert torch.equal(got["out"], ref["out"]) and torch.equal(got["lse"], ref["lse"])
    c.start = torch.tensor([0, new, new - 1, 3 * new], dtype=torch.int32, device=dev)
    got = c.run(ctx)
    assert torch.equal(got["out"][:new - 1], ref["out"][:new - 1])
    c.start = torch.tensor([2 ** 31 - 1, -2 ** 31, 5, 0], dtype=torch.int32, device=dev)
    c.run(ctx)
    torch.cuda.synchronize()


@pytest.mark.parametrize("new", [1, 30])
def test_rows_of_no_request_are_zero(ctx, dev, new):
    import torch
    c = Case(dev, [50, 60], [new, new], 4, 2, 128, seed=2)
    ref = c.run(ctx)
    T = 2 * new + 37
    q = torch.randn((T, 4, 128), dtype=torch.bfloat16, device=dev)
    q[: 2 * new] = c.q
    c.q = q
    out = torch.full_like(q, 7.0)
    lse = torch.full((T, 4), 7.0, device=dev)
    got = c.run(ctx, out=out, lse=lse)
    assert torch.equal(got["out"][: 2 * new], ref["out"])
    assert (out[2 * new:] == 0).all() and (lse[2 * new:] == -math.inf).all()


def test_strided_outputs_and_no_lse(ctx, dev):
    import torch
    c = Case(dev, [50, 61], [1, 33], 4, 2, 128, seed=4)
    ref = c.run(ctx)
    big = torch.full((34, 7, 136), 3.0, dtype=torch.bfloat16, device=dev)
    got = c.run(ctx, out=big[:, 2:6, :128], want_lse=False)
    assert got["lse"] is None
    assert torch.equal(big[:, 2:6, :128], ref["out"])
    assert (big[:, :2] == 3).all() and (big[:, 6:] == 3).all() and (big[:, :, 128:] == 3).all()


@pytest.mark.parametrize("lens,new", [([5000, 3000, 70], [1, 1, 1]), ([9000, 400], [3, 300]),
                                      ([700], [700])])
def test_two_calls_agree_and_max_new_changes_no_meaning(ctx, dev, lens, new):
    import torch
    c = Case(dev, lens, new, 8, 2, 128, seed=6)
    a, b = c.run(ctx), c.run(ctx)
    assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])
    for most in (0, 1, 2, 64, 100_000):      # a bound that does not hold costs time only
        c.check(c.run(ctx, max_new=most))


def test_cache_beyond_32_bit_offsets(ctx, dev):
    """A cache of 9.7 GB (2^32 elements and more), the request's blocks at both of its ends."""
    import torch
    import paper_2607_16892_amd as dro
    H, D, B, nb = 8, 128, 16, 148_000
    g = torch.Generator(device=dev).manual_seed(1)
    k, v = (torch.empty((nb, B, H, D), dtype=torch.float16, device=dev) for _ in range(2))
    assert k.numel() > 2 ** 31 and k.numel() * 2 > 2 ** 32
    small = Case(dev, [100, 160], [1, 30], 16, H, D, "f16", seed=8, layout="tokens")
    ids = [nb - 1, 0, nb - 2, 140_000, 5, 131_072, 131_071, nb - 3, 7, 65_536, 9, 11, 12, 13, 14, 15, 16, 17]
    table = small.table.clone()
    for r, L in enumerate(small.ctx):
        for b in range(-(-L // B)):
            new = ids.pop(0)
            old = int(small.table_h[r, b])
            k[new], v[new] = small.k[old], small.v[old]
            table[r, b] = new
    cache = dro.KvCache(k, v)
    got = dro.kv_attention(ctx, cache, small.q, table, small.start, small.context, 30)
    ref = small.run(ctx)
    assert torch.equal(got["out"], ref["out"]) and torch.equal(got["lse"], ref["lse"])
    # and the store into its last blocks
    kn = torch.randn((4, H, D), dtype=torch.float16, device=dev, generator=g)
    slot = torch.tensor([nb * B - 1, 3, -1, (nb - 2) * B], device=dev)
    dro.kv_store(ctx, cache, kn, kn, slot)
    assert torch.equal(k[nb - 1, B - 1], kn[0]) and torch.equal(v[nb - 2, 0], kn[3])
    assert torch.equal(k[0, 3], kn[1])


def test_large_scores_and_flat_weights(ctx, dev):
    """Scores of hundreds (one weight takes all) and equal keys (every weight the same)."""
    import torch
    c = Case(dev, [700, 200], [1, 90], 4, 2, 128, "f16", seed=7, scale_q=40.0)
    c.check(c.run(ctx))
    c.k.zero_()
    c.k_h.zero_()
    c.check(c.run(ctx))


@pytest.mark.parametrize("new", [1, 60])
@pytest.mark.parametrize("scale", [1e-30, -1e-30])
def test_scores_that_vanish(ctx, dev, new, scale):
    """A scale and a key scale whose product is below the smallest float: every key seen weighs
    the same, and hidden ones nothing."""
    import torch
    import paper_2607_16892_amd as dro
    c = Case(dev, [new + 70, new], [new, new], 4, 2, 128, "bf16", "fp8", seed=11)
    c.ks = torch.full((2,), 1e-20)
    c.cache = dro.KvCache(c.k, c.v, c.ks.to(dev), c.vs.to(dev))
    c.check(c.run(ctx, scale=scale), scale=scale)


def test_side_stream_and_graph(dev):
    """On a stream of its own, and captured: replays follow new inputs in place."""
    import torch
    import paper_2607_16892_amd as dro
    with dro.Context(dev.index or 0) as ctx:
        cases = [Case(dev, [5000, 33, 900], [1, 1, 1], 8, 2, 128, seed=s) for s in (1, 2)]
        chunk = Case(dev, [900, 300], [70, 200], 8, 2, 128, seed=3)
        refs = [c.run(ctx) for c in cases + [chunk]]
        torch.cuda.synchronize()
        s = torch.cuda.Stream(dev)
        got = [c.run(ctx, stream=s) for c in cases + [chunk]]
        s.synchronize()
        for g, r in zip(got, refs):
            assert torch.equal(g["out"], r["out"]) and torch.equal(g["lse"], r["lse"])
        c = cases[0]
        out, lse = torch.zeros_like(refs[0]["out"]), torch.zeros_like(refs[0]["lse"])
        o2, l2 = torch.zeros_like(refs[2]["out"]), torch.zeros_like(refs[2]["lse"])
        with torch.cuda.stream(s):
            c.run(ctx, out=out, lse=lse)
            chunk.run(ctx, out=o2, lse=l2)
        s.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            c.run(ctx, out=out, lse=lse)
            chunk.run(ctx, out=o2, lse=l2)
        for src, ref in ((cases[1], refs[1]), (cases[0], refs[0]), (cases[1], refs[1])):
            c.q.copy_(src.q)
            for a, b in ((c.k, src.k), (c.v, src.v)):
                a.copy_(b) if src is not c else None
            c.table.copy_(src.table)
            if src is c:                     # the first case's own data again
                c2 = Case(dev, [5000, 33, 900], [1, 1, 1], 8, 2, 128, seed=1)
                c.q.copy_(c2.q), c.k.copy_(c2.k), c.v.copy_(c2.v), c.table.copy_(c2.table)
            out.fill_(9), lse.fill_(9), o2.fill_(9), l2.fill_(9)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, ref["out"]) and torch.equal(lse, ref["lse"])
            assert torch.equal(o2, refs[2]["out"]) and torch.equal(l2, refs[2]["lse"])


def test_refusals(ctx, dev):
    import torch
    import paper_2607_16892_amd as dro
    c = Case(dev, [50, 60], [1, 2], 4, 2, 128, seed=2)
    out = torch.full((3, 4, 128), 7.0, dtype=torch.bfloat16, device=dev)

    def code(**kw):
        with pytest.raises(dro.DroError) as e:
            c.run(ctx, out=out, **kw)
        return e.value.code

    assert code(softcap=-1.0) == -1
    assert code(softcap=math.nan) == -1
    assert code(scale=math.inf) == -1
    assert code(window=-3) == -1
    assert code(max_new=-1) == -1
    good = c.q
    c.q = good.repeat(1, 1, 1)[:, :3]
    with pytest.raises((dro.DroError, ValueError)):      # 3 query heads over 2 key heads
        c.run(ctx)
    c.q = good.half()
    with pytest.raises(dro.DroError):                    # not the cache's type
        c.run(ctx)
    c.q = good.float()
    with pytest.raises(TypeError):
        c.run(ctx)
    odd = torch.empty(3 * 4 * 128 + 8, dtype=torch.bfloat16, device=dev)
    c.q = odd[1:1 + 3 * 4 * 128].view(3, 4, 128)
    with pytest.raises(dro.DroError):                    # not aligned
        c.run(ctx)
    c.q = good
    for name, bad in (("start", c.start[:2]), ("context", c.context.long()), ("table", c.table.long())):
        keep = getattr(c, name)
        setattr(c, name, bad)
        with pytest.raises((TypeError, ValueError)):
            c.run(ctx)
        setattr(c, name, keep)
    with pytest.raises(ValueError):
        c.run(ctx, slopes=torch.ones(3, device=dev))
    k = torch.zeros((4, 24, 2, 128), dtype=torch.bfloat16, device=dev)
    with pytest.raises(dro.DroError):                    # a block of 24 tokens
        dro.kv_attention(ctx, dro.KvCache(k, k), c.q, c.table, c.start, c.context, 2)
    k = torch.zeros((4, 16, 2, 264), dtype=torch.bfloat16, device=dev)
    with pytest.raises(dro.DroError):                    # 264 components
        dro.kv_attention(ctx, dro.KvCache(k, k), torch.zeros((3, 4, 264), dtype=torch.bfloat16,
                                                             device=dev),
                         c.table, c.start, c.context, 2)
    k = torch.zeros((4, 16, 2, 128), dtype=torch.float8_e4m3fn, device=dev)
    with pytest.raises(dro.DroError):                    # 8 bits without scales
        dro.kv_attention(ctx, dro.KvCache(k, k), c.q, c.table, c.start, c.context, 2)
    torch.cuda.synchronize()
    assert (out == 7).all()
    # no rows: nothing to do
    e = dro.kv_attention(ctx, c.cache, c.q[:0], c.table, torch.zeros(3, dtype=torch.int32, device=dev),
                         c.context, 0)
    assert e["out"].shape == (0, 4, 128)


def _reference(c, r, rows, softcap=0.0, window=0, prefix=0):
    """Rows `rows` of request r in fp64 on the GPU: (out, lse)."""
    import torch
    k, v = (torch.from_numpy(x).to(c.dev) for x in c.keys(r))
    L, n, a = c.ctx[r], c.new[r], int(c.start[r])
    q = c.q[a:a + n][rows].double()
    G = c.Hq // c.H
    p = (L - n + torch.as_tensor(rows, device=c.dev)).double()[:, None]
    j = torch.arange(L, device=c.dev, dtype=torch.float64)[None, :]
    see = (j <= p) | (j < prefix)
    if window:
        see &= p - j < window
    out = torch.empty((len(rows), c.Hq, c.D), dtype=torch.float64, device=c.dev)
    mass, lse = torch.empty_like(out), torch.empty((len(rows), c.Hq), dtype=torch.float64, device=c.dev)
    for h in range(c.Hq):
        s = q[:, h].contiguous() @ k[:, h // G].T.contiguous() * c.D ** -0.5
        if softcap:
            s = softcap * torch.tanh(s / softcap)
        s = s.masked_fill(~see, -math.inf)
        lse[:, h] = torch.logsumexp(s, -1)
        w = torch.softmax(s, -1)
        out[:, h], mass[:, h] = w @ v[:, h // G].contiguous(), w @ v[:, h // G].abs().contiguous()
    return out, lse, mass


@pytest.mark.parametrize("Hq,H,D,dtype,cache,lens,new,kw", [
    # enough tiles that each workgroup takes one, all of a prompt
    (64, 32, 128, "bf16", None, [4500], [4500], dict()),
    (48, 48, 64, "f16", "fp8", [2900, 700, 33], [2900, 700, 33], dict(window=500)),
    # many tiles beside one long request, whose tiles are cut into chunks
    (64, 64, 64, "bf16", None, [60_000] + [40] * 70, [150] + [40] * 70, dict()),
    (48, 16, 128, "f16", None, [45_000, 3000, 1500], [200, 3000, 1], dict(softcap=20.0)),
    # few tiles over long contexts: runs
    (8, 2, 256, "bf16", "fp8", [30_000, 50], [70, 50], dict(softcap=10.0)),
    (8, 1, 80, "f16", None, [50_000, 3], [100, 3], dict(window=20_000)),
])
def test_many_tiles(ctx, dev, Hq, H, D, dtype, cache, lens, new, kw):
    """Large calls, some of their rows against fp64 (sums of weights times |v| as in
    kv_cases; scores of unit variance, so 2^-17 bounds what fp32 adds)."""
    import torch
    from kv_cases import UNIT
    print(f"[gpu] kv tiles Hq={Hq} H={H} D={D} {dtype}/{cache} requests {len(lens)}", flush=True)
    c = Case(dev, lens, new, Hq, H, D, dtype, cache, seed=Hq + D)
    got = c.run(ctx, **kw)
    again = c.run(ctx, **kw)
    assert torch.equal(got["out"], again["out"]) and torch.equal(got["lse"], again["lse"])
    u = UNIT[dtype]
    for r in {0, 1 % len(lens), len(lens) - 1}:
        n, a = new[r], int(c.start[r])
        rows = sorted({0, 1, n // 3, n // 2, n - 2, n - 1} & set(range(n)))
        out, lse, mass = _reference(c, r, rows, **kw)
        err = (got["out"][a:a + n][rows].double() - out).abs()
        tol = (2 * u + 2.0 ** -17 * (1 + 4 * (kw.get("softcap", 0) > 0))) * mass + lens[r] * 2.0 ** -25 * 8 + 2.0 ** -24
        assert (err <= tol).all(), f"request {r}: {(err / tol).max().item():.3g} of the bound"
        assert ((got["lse"][a:a + n][rows].double() - lse).abs() <= 2.0 ** -16 * (1 + lse.abs())).all()


def test_a_bound_that_does_not_hold_loses_no_request(ctx, dev):
    """max_new below a request's rows, with so many rows that every other one seems long."""
    c = Case(dev, [400, 90, 7], [1, 300, 7], 8, 2, 128, seed=12)
    for most in (1, 5, 100, 150, 299):
        c.check(c.run(ctx, max_new=most))


@pytest.mark.parametrize("Hq,H,D,lens,new", [
    (8, 1, 64, [300 + i % 7 for i in range(61)], [300] * 61),             # more tiles than a pass lists
    (24, 12, 64, [1500, 40, 900, 2100], [1500, 40, 900, 700]),            # heads that no die has whole
    (10, 5, 128, [700, 3000, 90, 5], [300, 64, 90, 1]),
    (32, 16, 80, [2500, 800, 33], [65, 800, 33]),
    (16, 8, 256, [4000, 100, 2000, 900, 1], [50, 9, 33, 60, 1]),          # a tile each, of unequal length
    (16, 2, 128, [60 + 31 * i % 900 for i in range(70)],                  # both kernels
     [1 if i % 7 else min(100, 60 + 31 * i % 900) for i in range(70)]),
    (64, 8, 128, [500 + 17 * i for i in range(70)], [3] * 70),
    (4, 2, 64, [90 + i % 9 for i in range(1100)], [60 if i % 92 == 0 else 1 for i in range(1100)]),  # a list in passes
])
def test_orders_of_tiles(ctx, dev, Hq, H, D, lens, new):
    """Tiles listed longest first, dealt to the dies by heads or in turn, cut and whole: rows of
    every request against fp64 (bounds as in test_many_tiles)."""
    import torch
    from kv_cases import UNIT
    print(f"[gpu] kv orders Hq={Hq} H={H} D={D} requests {len(lens)}", flush=True)
    c = Case(dev, lens, new, Hq, H, D, "bf16", seed=Hq + D)
    got = c.run(ctx)
    for r in range(0, len(lens), 1 + len(lens) // 12):
        n, a = new[r], int(c.start[r])
        rows = sorted({0, n // 2, n - 1})
        out, lse, mass = _reference(c, r, rows)
        err = (got["out"][a:a + n][rows].double() - out).abs()
        tol = (2 * UNIT["bf16"] + 2.0 ** -17) * mass + lens[r] * 2.0 ** -25 * 8 + 2.0 ** -24
        assert (err <= tol).all(), f"request {r}: {(err / tol).max().item():.3g} of the bound"
        assert ((got["lse"][a:a + n][rows].double() - lse).abs() <= 2.0 ** -16 * (1 + lse.abs())).all()


@pytest.mark.parametrize("lens,new", [([20_000, 70], [40, 70]), ([20_000], [1]), ([300, 300], [90, 1])])
def test_infinities_in_long_and_cut_requests(ctx, dev, lens, new):
    """An infinity and a NaN in the last token of a request: its last row alone has them, in
    their components, whether the request is whole or cut."""
    import torch
    c = Case(dev, lens, new, 4, 2, 128, "bf16", seed=21)
    ref = c.run(ctx)
    L = lens[0]
    b = int(c.table_h[0, (L - 1) // 16])
    c.v[b, (L - 1) % 16, 0, 5] = float("inf")
    c.v[b, (L - 1) % 16, 1, 9] = float("nan")
    got = c.run(ctx)
    hit = torch.zeros_like(ref["out"], dtype=torch.bool)
    hit[new[0] - 1, :2, 5] = True
    hit[new[0] - 1, 2:, 9] = True
    assert not torch.isfinite(got["out"][hit]).any()
    assert torch.equal(got["out"][~hit], ref["out"][~hit]) and torch.equal(got["lse"], ref["lse"])
