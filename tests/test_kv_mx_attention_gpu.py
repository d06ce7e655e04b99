"""kv_attention over caches in shared scales against its definition in fp64 on the values held: these
are exact in q's type, so the bound is that of a 16-bit cache."""
import math

import numpy as np
import pytest

from mx_cases import mx_case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(dev):
    import paper_2607_16892_amd as dro
    c = dro.Context(dev.index or 0)
    yield c
    c.close()


EDGES = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 100, 127, 128, 129, 255, 256, 257, 513, 0, 1023]
KINDS = [(k, t) for k in ("mxfp4", "mxfp8") for t in ("bf16", "f16")]
SHAPES = [(8, 1, 128, 16), (14, 2, 128, 32), (3, 3, 64, 16), (32, 2, 96, 16), (4, 2, 256, 64), (40, 1, 32, 128),
          (2, 1, 192, 16), (5, 5, 160, 1024)]


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("Hq,H,D,block", SHAPES)
@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_single_tokens(ctx, dev, kind, dtype, Hq, H, D, block, layout):
    print(f"[gpu] kv mx decode {dtype}/{kind} Hq={Hq} H={H} D={D} block={block}", flush=True)
    c = mx_case(dev, kind, EDGES, [1] * len(EDGES), Hq, H, D, dtype, layout, block=block, seed=D + Hq)
    c.check(c.run(ctx))


@pytest.mark.parametrize("kind,dtype", KINDS)
@pytest.mark.parametrize("Hq,H,D,block,layout", [(8, 2, 128, 16, "tokens"), (7, 1, 128, 32, "heads"), (2, 2, 64, 16, "heads"),
                                                 (6, 2, 96, 64, "tokens"), (4, 2, 256, 16, "heads"), (3, 1, 224, 16, "heads")])
def test_chunks(ctx, dev, kind, dtype, Hq, H, D, block, layout):
    # chunks over what is cached, whole prompts, single tokens and no tokens in one call
    print(f"[gpu] kv mx chunks {dtype}/{kind} Hq={Hq} H={H} D={D} block={block}", flush=True)
    c = mx_case(dev, kind, [300, 17, 1, 129, 64, 400, 0, 33, 250, 90], [45, 17, 1, 0, 2, 130, 0, 1, 250, 33],
                Hq, H, D, dtype, layout, block=block, seed=D + Hq)
    c.check(c.run(ctx))


@pytest.mark.parametrize("new", [1, 9, 200])
@pytest.mark.parametrize("opts", [dict(softcap=5.0), dict(window=1), dict(window=33), dict(slopes=0.5),
                                  dict(prefix=True, window=20), dict(scale=-0.1), dict(scale=0.0),
                                  dict(softcap=30.0, slopes=0.1, window=64, prefix=True, scale=0.2)])
@pytest.mark.parametrize("D,kind,dtype", [(128, "mxfp4", "bf16"), (64, "mxfp4", "f16"), (128, "mxfp8", "f16"),
                                          (256, "mxfp8", "bf16")])
def test_scores_and_masks(ctx, dev, new, opts, D, kind, dtype):
    import torch
    print(f"[gpu] kv mx options {opts} new={new} D={D}", flush=True)
    lens = [new, new + 1, new + 30, new + 64, new + 333]
    c = mx_case(dev, kind, lens, [new] * 5, 6, 2, D, dtype, seed=new + D, scale_q=2.0)
    kw = dict(opts)
    if "slopes" in kw:
        kw["slopes"] = (kw["slopes"] * torch.arange(1, 7, dtype=torch.float32) / 6).to(dev)
    if "prefix" in kw:
        kw["prefix"] = torch.tensor([0, 5, new + 30, new + 500, 40], dtype=torch.int32, device=dev)
    c.check(c.run(ctx, **kw), **kw)


@pytest.mark.parametrize("kind", ["mxfp4", "mxfp8"])
@pytest.mark.parametrize("new", [1, 40])
def test_long_and_many(ctx, dev, kind, new):
    """A long axis split over workgroups beside short requests, rows that see nothing, and more
    requests than a wave has lanes."""
    c = mx_case(dev, kind, [20_011, 70, 3001, 5, new // 2, 0], [new, new, 1, 1, new, new], 8, 2, 128, seed=1)
    c.check(c.run(ctx))
    r = np.random.default_rng(5)
    lens = r.integers(0, 121, 130).tolist()
    lens[40] = 480
    news = [int(min(x, n)) for x, n in zip(lens, r.integers(0, new + 1, 130))]
    c = mx_case(dev, kind, lens, news, 4, 2, 64, "f16", seed=2)
    got = c.run(ctx)
    c.check(got)
    again = c.run(ctx)
    assert torch_equal(got, again)


def torch_equal(a, b):
    import torch
    return torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])


def _powers(c):
    return c.cache.k_power, c.cache.v_power


@pytest.mark.parametrize("new", [1, 3, 60])
@pytest.mark.parametrize("kind,dtype,D", [("mxfp4", "bf16", 128), ("mxfp4", "f16", 64), ("mxfp8", "bf16", 256),
                                          ("mxfp8", "f16", 96), ("mxfp4", "bf16", 192), ("mxfp8", "bf16", 128)])
def test_unused_places_may_hold_anything(ctx, dev, new, kind, dtype, D):
    """Blocks of no request and tokens beyond the contexts: any codes under any powers, those of NaN
    and of values beyond the types' ranges among them."""
    import torch
    print(f"[gpu] kv mx hidden {kind}/{dtype} D={D} new={new}", flush=True)
    lens = [new + 5, new + 40, 64 + new, new]
    c = mx_case(dev, kind, lens, [new] * 4, 4, 2, D, dtype, seed=new + D)
    ref = c.run(ctx)
    c.check(ref)
    used = torch.zeros(c.k.shape[:2], dtype=torch.bool)
    for r, L in enumerate(lens):
        p = torch.arange(L)
        used[c.table_h[r, p // 16].long(), p % 16] = True
    hide = (~used).to(dev)
    for byte, code in ((255, 0x11), (254, 0x77), (253, 0x7e), (0, 0xff), (145, 0x7f)):
        for t in _powers(c):
            t[hide] = byte
        for t in (c.k, c.v):
            t.view(torch.uint8)[hide] = code
        assert torch_equal(c.run(ctx), ref), (byte, code)


@pytest.mark.parametrize("new", [2, 3, 60])
@pytest.mark.parametrize("kind,dtype,D", [("mxfp4", "bf16", 128), ("mxfp4", "f16", 64), ("mxfp8", "bf16", 256),
                                          ("mxfp8", "f16", 96), ("mxfp4", "f16", 160)])
def test_a_token_that_one_row_sees(ctx, dev, new, kind, dtype, D):
    """A group of NaN in a request's last value: its last row has them, in the group's components, and
    no other row changes; then in its key: that row is NaN."""
    import torch
    lens = [new + 5, new + 40]
    c = mx_case(dev, kind, lens, [new] * 2, 4, 2, D, dtype, seed=new + D)
    ref = c.run(ctx)
    p = lens[1] - 1
    b, i = int(c.table_h[1, p // 16]), p % 16
    g = D // 32 - 1
    c.cache.v_power[b, i, 0, g] = 255
    got = c.run(ctx)
    hit = torch.zeros_like(ref["out"], dtype=torch.bool)
    hit[2 * new - 1, :2, 32 * g:] = True
    assert torch.isnan(got["out"][hit]).all()
    assert torch.equal(got["out"][~hit], ref["out"][~hit]) and torch.equal(got["lse"], ref["lse"])
    c.cache.k_power[b, i, 1, 0] = 255
    got = c.run(ctx)
    hit[2 * new - 1, 2:] = True
    assert torch.isnan(got["out"][hit]).all() and torch.isnan(got["lse"][2 * new - 1, 2:]).all()
    assert torch.equal(got["out"][~hit], ref["out"][~hit])
    assert torch.equal(got["lse"][: 2 * new - 1], ref["lse"][: 2 * new - 1])


@pytest.mark.parametrize("new", [1, 50])
def test_bad_tables_stay_inside(ctx, dev, new):
    """Blocks outside the pool are read as its nearest ones."""
    import torch
    c = mx_case(dev, "mxfp4", [200, 90], [new] * 2, 4, 2, 128, seed=3)
    nb = c.k.shape[0]
    ref_table = c.table.clone()
    ref_table[0, 2], ref_table[1, 1] = 0, nb - 1
    bad = ref_table.clone()
    bad[0, 2], bad[1, 1] = -(2 ** 31), 2 ** 31 - 1
    c.table = ref_table
    ref = c.run(ctx)
    c.table = bad
    assert torch_equal(c.run(ctx), ref)


def test_stored_then_attended(ctx, dev):
    """A prompt stored by kv_store and attended: as over the values that kv_load gives, kept in 16
    bits, up to the order of the sums."""
    import torch
    import paper_2607_16892_amd as dro
    T, Hq, H, D = 150, 8, 2, 128
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn((T, h, D), generator=g).bfloat16().to(dev) for h in (Hq, H, H))
    i32 = dict(dtype=torch.int32, device=dev)
    table = torch.arange(10, **i32).flip(0)[None].contiguous()
    p = torch.arange(T, device=dev)
    slot = table[0, p // 16].long() * 16 + p % 16
    start, context = torch.tensor([0, T], **i32), torch.tensor([T], **i32)
    for kind in ("mxfp4", "mxfp8"):
        c = dro.KvCache.empty(10, 16, H, D, kind, dev)
        dro.kv_store(ctx, c, k, v, slot)
        got = dro.kv_attention(ctx, c, q, table, start, context, T)
        wide = dro.KvCache.empty(10, 16, H, D, torch.bfloat16, dev)
        back = dro.kv_load(ctx, c, slot)
        dro.kv_store(ctx, wide, back["k"], back["v"], slot)
        ref = dro.kv_attention(ctx, wide, q, table, start, context, T)
        assert torch_equal(got, ref)     # the same kernel on the same values in 16 bits


def test_a_captured_step(dev):
    """Store and attention of a decode step in a graph, replayed over other inputs."""
    import torch
    import paper_2607_16892_amd as dro
    with dro.Context(dev.index or 0) as ctx:
        c = mx_case(dev, "mxfp4", [700, 33, 1], [1, 1, 1], 8, 2, 128, seed=4)
        p = torch.tensor([699, 32, 0], device=dev)
        slot = c.table[torch.arange(3, device=dev), p // 16].long() * 16 + p % 16
        k = torch.zeros((3, 2, 128), dtype=torch.bfloat16, device=dev)
        v = torch.zeros_like(k)

        def step(**kw):
            dro.kv_store(ctx, c.cache, k, v, slot)
            return c.run(ctx, **kw)

        ref = step()
        out, lse = torch.zeros_like(ref["out"]), torch.zeros_like(ref["lse"])
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=torch.cuda.Stream(dev)):
            step(out=out, lse=lse)
        for seed in range(3):
            g = torch.Generator().manual_seed(seed)
            k.copy_(torch.randn(k.shape, generator=g))
            v.copy_(torch.randn(k.shape, generator=g))
            out.fill_(9)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch_equal(dict(out=out, lse=lse), step())


@pytest.mark.parametrize("new", [2, 60])
@pytest.mark.parametrize("kind,dtype,D,byte", [("mxfp4", "bf16", 128, 253), ("mxfp4", "f16", 64, 141), ("mxfp8", "bf16", 96, 250),
                                               ("mxfp8", "f16", 128, 139)])
def test_values_beyond_the_range(ctx, dev, new, kind, dtype, D, byte):
    """Codes whose values are infinite in q's type, as no store leaves them: the row that sees them has
    them, infinite or NaN, in their components, and the others are as they were."""
    import torch
    lens = [new + 5, new + 40]
    c = mx_case(dev, kind, lens, [new] * 2, 4, 2, D, dtype, seed=new + D)
    ref = c.run(ctx)
    p = lens[1] - 1
    b, i = int(c.table_h[1, p // 16]), p % 16
    c.cache.v_power[b, i, 0, 1] = byte
    c.v.view(torch.uint8)[b, i, 0, 16 if kind == "mxfp4" else 32] = 0x07 if kind == "mxfp4" else 0x7e   # component 32
    got = c.run(ctx)
    hit = torch.zeros_like(ref["out"], dtype=torch.bool)
    hit[2 * new - 1, :2, 32:64] = True
    assert not torch.isfinite(got["out"][2 * new - 1, :2, 32]).any()
    assert torch.equal(got["out"][~hit], ref["out"][~hit]) and torch.equal(got["lse"], ref["lse"])


@pytest.mark.parametrize("kind", ["mxfp4", "mxfp8"])
def test_places_beyond_32_bits(ctx, dev, kind):
    """Requests, and a shared prefix, at the end of a cache of more than 2^32 bytes: as in a small one."""
    import torch
    import paper_2607_16892_amd as dro
    H, D, block = 8, 128, 1024
    nb = 9000 if kind == "mxfp4" else 5000                             # 4.7 and 5.2 GB of codes each
    g = torch.Generator().manual_seed(1)
    i32 = dict(dtype=torch.int32, device=dev)
    k, v = (torch.randn((3 * block, H, D), generator=g).bfloat16().to(dev) for _ in range(2))
    q = torch.randn((61, 32, D), generator=g).bfloat16().to(dev)
    start, context = torch.tensor([0, 1, 61], **i32), torch.tensor([1500, 900], **i32)
    out = []
    for blocks in (nb, 3):
        c = dro.KvCache.empty(blocks, block, H, D, kind, dev)
        dro.kv_store(ctx, c, k, v, torch.arange((blocks - 3) * block, blocks * block, device=dev))
        table = torch.tensor([[blocks - 1, blocks - 3], [blocks - 2, 0]], **i32)
        both = dro.kv_attention(ctx, c, q, table, start, context, 60)
        one = dro.kv_attention(ctx, c, q[:1], table[:1], start[:2], context[:1], 1)
        shared = dro.SharedPrefixes(torch.tensor([0, 2], **i32), torch.tensor([700], **i32),
                                    torch.tensor([[blocks - 3]], **i32), 61)
        out.append((both, one, dro.kv_shared_attention(ctx, c, q, table, start, context, 60, shared),
                    dro.kv_shared_attention(ctx, c, q[:1], table, start[:2].repeat_interleave(torch.tensor([1, 2], device=dev)),
                                            context, 1, shared)))
        del c
    assert all(torch_equal(a, b) for a, b in zip(*out))
