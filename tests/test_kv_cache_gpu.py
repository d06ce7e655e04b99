"""kv_block_tables and kv_store against their definitions (oracle/kv.py, torch in fp32)."""
import numpy as np
import pytest

from oracle import kv as okv

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(dev):
    import paper_2607_16892_amd as dro
    c = dro.Context(dev.index or 0)
    yield c
    c.close()


def _i32(a, dev):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(dev)


def _random(seed, R, W, block, free, chunk=40, ended=0.2, reserve=True, wide=0.0):
    """A pool in mid-service: unequal lengths, requests that hold their reservation or not."""
    r = np.random.default_rng(seed)
    top = W * block
    add = r.integers(0, chunk + 1, R)
    add[r.random(R) < 0.5] = 1
    add[r.random(R) < ended] = -1
    length = np.minimum(r.integers(0, top + 1, R), top - np.maximum(add, 0))
    length = np.maximum(np.where(r.random(R) < 0.3, 0, length), 0)
    want = np.minimum(length + r.integers(0, 4 * block, R), top) if reserve else None
    if wide:
        length[r.random(R) < wide] = top + 5
    held = np.minimum(-(-length // block) + (r.random(R) < 0.4) * r.integers(0, 3, R), W)
    nb = int(held.sum()) + free + 5
    order = r.permutation(nb).astype(np.int32)
    table = np.full((R, W), -1, np.int32)
    at = 0
    for i in range(R):
        table[i, : held[i]] = order[at:at + held[i]]
        at += held[i]
    stack = np.full(nb, -7, np.int32)
    stack[:free] = order[at:at + free]
    return dict(block=block, table=table, held=held, free_list=stack, free=free, length=length, add=add,
                reserve=want, tokens=int(np.maximum(add, 0).sum()))


def _step(ctx, dev, c, in_place=False, tokens=None, wide_rows=0, **kw):
    import torch
    import paper_2607_16892_amd as dro
    R, W = c["table"].shape
    table = torch.full((R, W + wide_rows), -3, dtype=torch.int32, device=dev)
    table[:, :W] = _i32(c["table"], dev)
    pool = dro.BlockPool(block=c["block"], table=table[:, :W], held=_i32(c["held"], dev),
                         free_list=_i32(c["free_list"], dev), free=_i32([c["free"]], dev))
    out = dict(held=pool.held, free=pool.free) if in_place else None
    r = dro.kv_block_tables(ctx, pool, _i32(c["length"], dev), _i32(c["add"], dev),
                            c["tokens"] if tokens is None else tokens,
                            reserve=None if c["reserve"] is None else _i32(c["reserve"], dev), out=out, **kw)
    return dict(r, table=pool.table, free_list=pool.free_list), pool


def _same(got, ref):
    for k, v in ref.items():
        a, b = got[k].cpu().numpy().reshape(-1), np.asarray(v).reshape(-1)
        assert np.array_equal(a, b), f"{k}: {np.flatnonzero(a != b)[:8]} of {a.size}"


@pytest.mark.parametrize("R,W,block,chunk", [(1, 1, 16, 16), (1, 40, 16, 300), (5, 4, 16, 3), (64, 12, 16, 20),
                                             (65, 9, 32, 50), (300, 30, 16, 40), (1025, 17, 64, 9),
                                             (5000, 6, 16, 5), (40, 3, 1024, 700)])
@pytest.mark.parametrize("free", [0, 7, 100_000])
@pytest.mark.parametrize("reserve", [True, False])
def test_one_step(ctx, dev, R, W, block, chunk, free, reserve):
    print(f"[gpu] kv tables R={R} W={W} block={block} free={free}", flush=True)
    for seed in range(3):
        c = _random(seed, R, W, block, free, chunk, reserve=reserve, ended=(0.2, 0.0, 1.0)[seed],
                    wide=0.1 if seed == 1 else 0.0)
        if seed == 1:
            c["held"] = np.minimum(c["held"], W)
        got, _ = _step(ctx, dev, c, in_place=seed == 2, wide_rows=seed)
        _same(got, okv.block_tables(**c))


def test_first_come_first_served(ctx, dev):
    """After the first request that has to wait no later one grows, and those that need no block
    go on."""
    table = np.full((5, 8), -1, np.int32)
    table[3, 0] = 9
    c = dict(block=16, table=table, held=np.array([0, 0, 0, 1, 0]), free_list=np.arange(12, dtype=np.int32),
             free=5, length=np.array([0, 0, 0, 3, 0]), add=np.array([33, 49, 1, 2, 0]), reserve=None,
             tokens=85)
    got, _ = _step(ctx, dev, c)
    _same(got, okv.block_tables(**c))
    assert got["granted"].tolist() == [1, 0, 0, 1, 1]
    assert got["free"].item() == 2


def test_tokens_beyond_the_batch_and_padding(ctx, dev):
    c = _random(4, 30, 20, 16, 1000)
    n = c["tokens"]
    for T in (0, 1, n // 2, n + 100):
        c["tokens"] = T
        got, _ = _step(ctx, dev, c)
        _same(got, okv.block_tables(**c))


def test_a_service_of_many_steps(ctx, dev):
    """A loop in place: requests come, grow and end; no block is ever held twice or lost."""
    import torch
    import paper_2607_16892_amd as dro
    r = np.random.default_rng(3)
    R, W, B, nb = 48, 10, 16, 200
    pool = dro.BlockPool.empty(R, W, nb, B, dev)
    length = np.zeros(R, np.int64)
    for step in range(40):
        add = np.where(length == 0, r.integers(0, 60, R), 1)
        add[(length > 0) & ((r.random(R) < 0.15) | (length >= W * B))] = -1
        want = np.minimum(length + 30, W * B)
        ref = okv.block_tables(B, pool.table.cpu().numpy(), pool.held.cpu().numpy(),
                               pool.free_list.cpu().numpy(), pool.free.item(), length, add, want,
                               int(np.maximum(add, 0).sum()))
        got = dro.kv_block_tables(ctx, pool, _i32(length, dev), _i32(add, dev),
                                  int(np.maximum(add, 0).sum()), reserve=_i32(want, dev))
        pool.take(got)
        _same(dict(got, table=pool.table, free_list=pool.free_list), ref)
        length = np.where(add < 0, 0, np.where(np.array(ref["granted"]) == 1, length + np.maximum(add, 0), length))
        held, table = pool.held.cpu().numpy(), pool.table.cpu().numpy()
        mine = np.concatenate([table[i, : held[i]] for i in range(R)] + [pool.free_list.cpu().numpy()[: pool.free.item()]])
        assert sorted(mine.tolist()) == list(range(nb))


def test_tables_bad_data_stays_inside(ctx, dev):
    """Counts and lengths outside their ranges: cut, and nothing outside the arrays is touched."""
    import torch
    import paper_2607_16892_amd as dro
    R, W, nb = 6, 4, 20
    whole = torch.full((R + 2, W), 77, dtype=torch.int32, device=dev)
    pool = dro.BlockPool(16, whole[1:-1], _i32([-5, 2 ** 31 - 1, 1, 4, 0, 4], dev),
                         torch.arange(nb, dtype=torch.int32, device=dev), _i32([10 ** 6], dev))
    add = _i32([5, -1, -1, 2 ** 31 - 1, 64, -1], dev)
    got = dro.kv_block_tables(ctx, pool, _i32([-9, 3, 5, 2 ** 31 - 1, 0, 64], dev), add, 50,
                              reserve=_i32([-1, 0, 0, 0, 2 ** 31 - 1, 0], dev))
    torch.cuda.synchronize()
    assert (whole[0] == 77).all() and (whole[-1] == 77).all()
    assert 0 <= got["free"].item() <= nb
    assert got["granted"].tolist() == [1, 0, 0, 0, 0, 0]


def test_tables_on_a_side_stream_and_in_a_graph(dev):
    import torch
    import paper_2607_16892_amd as dro
    with dro.Context(dev.index or 0) as ctx:
        c = _random(9, 200, 20, 16, 500)
        ref = okv.block_tables(**c)
        s = torch.cuda.Stream(dev)
        torch.cuda.synchronize()
        got, pool = _step(ctx, dev, c)
        table, stack = _i32(c["table"], dev), _i32(c["free_list"], dev)
        args = (_i32(c["length"], dev), _i32(c["add"], dev), c["tokens"])
        res = _i32(c["reserve"], dev)
        torch.cuda.synchronize()
        out = dro.kv_block_tables(ctx, pool, *args, reserve=res, stream=s)
        s.synchronize()
        _same(out, {k: ref[k] for k in out})
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            dro.kv_block_tables(ctx, pool, *args, reserve=res, out=out)
        for _ in range(3):
            pool.table.copy_(table), pool.free_list.copy_(stack)
            for v in out.values():
                v.fill_(3)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            _same(dict(out, table=pool.table, free_list=pool.free_list), ref)


def test_tables_refusals(ctx, dev):
    import torch
    import paper_2607_16892_amd as dro
    c = _random(1, 4, 6, 16, 10)
    _, pool = _step(ctx, dev, c)
    before = pool.table.clone()
    a = (_i32(c["length"], dev), _i32(c["add"], dev), c["tokens"])
    for field, bad, err in (("block", 8, dro.DroError), ("block", 24, dro.DroError), ("block", 2048, dro.DroError),
                            ("held", pool.held[:2], ValueError), ("free_list", pool.free_list.long(), TypeError),
                            ("table", pool.table.cpu(), TypeError), ("table", pool.table.t(), ValueError)):
        keep = getattr(pool, field)
        setattr(pool, field, bad)
        with pytest.raises(err):
            dro.kv_block_tables(ctx, pool, *a)
        setattr(pool, field, keep)
    with pytest.raises(ValueError):
        dro.kv_block_tables(ctx, pool, a[0][:2], a[1], a[2])
    with pytest.raises(ValueError):
        dro.kv_block_tables(ctx, pool, a[0], a[1], -1)
    with pytest.raises(dro.DroError):
        dro.kv_block_tables(ctx, pool, a[0], a[1], (1 << 24) + 1, out=dict(
            slot=torch.empty(((1 << 24) + 1,), dtype=torch.int64, device=dev)))
    torch.cuda.synchronize()
    assert torch.equal(pool.table, before)


# ------------------------------------------------------------------ store ----

@pytest.mark.parametrize("dtype,cache", [("bf16", "bf16"), ("f16", "f16"), ("bf16", "fp8"), ("f16", "fp8")])
@pytest.mark.parametrize("T,H,D,block", [(1, 1, 8, 16), (1, 8, 128, 16), (7, 5, 80, 32), (300, 2, 256, 16),
                                         (65, 3, 104, 64), (1000, 1, 64, 128)])
@pytest.mark.parametrize("layout", ["heads", "tokens"])
def test_store(ctx, dev, dtype, cache, T, H, D, block, layout):
    import torch
    import paper_2607_16892_amd as dro
    from kv_cases import dtypes
    print(f"[gpu] kv store {dtype}->{cache} T={T} H={H} D={D} block={block} {layout}", flush=True)
    dt = dtypes()
    g = torch.Generator(device=dev).manual_seed(T + D)
    nb = -(-T // block) + 2
    shape = (nb, H, block, D) if layout == "heads" else (nb, block, H, D)
    caches = []
    for _ in range(2):
        x = torch.randn(shape, device=dev, generator=g).to(dt[cache])
        caches.append(x.permute(0, 2, 1, 3) if layout == "heads" else x)
    x = torch.randn((T, 3 * H, D), device=dev, generator=g).to(dt[dtype]) * 3
    x[0, 0, :4] = torch.tensor([0.0, 1e4, -1e4, 2.0 ** -9], device=dev).to(dt[dtype])
    k, v = x[:, H:2 * H], x[:, 2 * H:]
    k[0, 0, :8] = torch.tensor([0.0, -0.0, 1e4, -1e4, 2.0 ** -9, float("inf"), float("-inf"), float("nan")],
                               device=dev).to(dt[dtype])
    slot = torch.randperm(nb * block, generator=g, device=dev)[:T]
    slot[T // 2::5] = -1
    if T > 20:
        slot[3], slot[4] = nb * block, 2 ** 40
    scales = [None, None]
    if cache == "fp8":
        scales = [torch.rand(H, device=dev, generator=g) + 0.1 for _ in range(2)]
    want = []
    for y, old, sc in ((k, caches[0], scales[0]), (v, caches[1], scales[1])):
        f = y.float()
        if sc is not None:
            f = (f / sc[None, :, None]).clamp(-448.0, 448.0)
        w = old.clone()
        keep = (slot >= 0) & (slot < nb * block)
        s = slot[keep]
        w.view(torch.uint8)[s // block, s % block] = f.to(dt[cache])[keep].view(torch.uint8)
        want.append(w)
    c = dro.KvCache(*caches, *scales)
    dro.kv_store(ctx, c, k, v, slot)
    torch.cuda.synchronize()
    for got, w in zip(caches, want):
        a, b = got.float(), w.float()
        assert torch.equal(torch.isnan(a), torch.isnan(b))
        assert torch.equal(a.nan_to_num(9e9), b.nan_to_num(9e9))


def test_every_fp8_value_survives_the_cache(ctx, dev):
    """All 256 codes (both NaN as NaN) stored with scale 1 come back as themselves, and halfway
    values round to even."""
    import torch
    import paper_2607_16892_amd as dro
    codes = torch.arange(256, dtype=torch.uint8, device=dev).view(torch.float8_e4m3fn)
    x = codes.to(torch.float16).view(1, 2, 128)
    c = dro.KvCache.empty(1, 16, 2, 128, torch.float8_e4m3fn, dev)
    dro.kv_store(ctx, c, x, x, torch.tensor([5], device=dev))
    got = c.k[0, 5].float().reshape(-1)
    assert torch.equal(got.nan_to_num(999.0), codes.float().nan_to_num(999.0))
    f = codes.float()[:127]
    half = torch.zeros(128, device=dev)
    half[:126] = (f[:-1] + f[1:]) / 2
    y = half.to(torch.float16).view(1, 1, 128).repeat(1, 2, 1)
    dro.kv_store(ctx, c, y, y, torch.tensor([6], device=dev))
    assert torch.equal(c.v[0, 6].float(), y[0].to(torch.float8_e4m3fn).float())


def test_store_refusals(ctx, dev):
    import torch
    import paper_2607_16892_amd as dro
    c = dro.KvCache.empty(4, 16, 2, 128, torch.bfloat16, dev)
    x = torch.ones((3, 2, 128), dtype=torch.bfloat16, device=dev)
    slot = torch.tensor([0, 1, 2], device=dev)
    with pytest.raises(dro.DroError):
        dro.kv_store(ctx, c, x.half(), x.half(), slot)
    with pytest.raises(TypeError):
        dro.kv_store(ctx, c, x.float(), x.float(), slot)
    with pytest.raises(ValueError):
        dro.kv_store(ctx, c, x[:, :1], x[:, :1], slot)
    with pytest.raises(ValueError):
        dro.kv_store(ctx, c, x, x, slot[:2])
    with pytest.raises(TypeError):
        dro.kv_store(ctx, c, x, x, slot.int())
    odd = torch.empty(3 * 256 + 8, dtype=torch.bfloat16, device=dev)[4:4 + 3 * 256].view(3, 2, 128)
    with pytest.raises(dro.DroError):
        dro.kv_store(ctx, c, odd, odd, slot)
    torch.cuda.synchronize()
    assert (c.k == 0).all() and (c.v == 0).all()
    dro.kv_store(ctx, c, x[:0], x[:0], slot[:0])
