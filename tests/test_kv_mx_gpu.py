"""Store into and load from caches in shared scales, bit for bit against the oracle."""
import numpy as np
import pytest

from mx_cases import as_np, cache, codes, encode, put, rows, same
from oracle import kv as okv

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(dev):
    import paper_2607_16892_amd as dro
    c = dro.Context(dev.index or 0)
    yield c
    c.close()


def _slots(T, nb, block, seed, refused=True):
    r = np.random.RandomState(seed)
    slot = r.permutation(nb * block)[:T].astype(np.int64)
    if refused and T > 3:
        slot[1], slot[T // 2] = -1, nb * block
        slot[T - 1] = 2 ** 62
    return slot


CASES = [("mxfp4", "bf16", 1, 1, 32, 16, "heads"), ("mxfp4", "bf16", 64, 8, 128, 16, "heads"),
         ("mxfp4", "f16", 131, 3, 96, 32, "tokens"), ("mxfp4", "f16", 13, 5, 256, 64, "heads"),
         ("mxfp8", "bf16", 12, 2, 64, 16, "tokens"), ("mxfp8", "f16", 301, 8, 128, 16, "heads"),
         ("mxfp8", "bf16", 33, 1, 224, 1024, "heads"), ("mxfp4", "bf16", 40, 70, 32, 16, "tokens"),
         ("mxfp8", "f16", 20, 9, 256, 16, "heads")]


@pytest.mark.parametrize("kind,dtype,T,H,D,block,layout", CASES)
def test_store_and_load(ctx, dev, kind, dtype, T, H, D, block, layout):
    """Codes and powers are the oracle's, places of no token stay as they were, and what is read
    back is what the codes stand for, with zeros for slots outside."""
    import torch
    import paper_2607_16892_amd as dro
    nb = -(-T // block) + 2
    c = cache(dev, kind, nb, block, H, D, layout)
    k, v = rows(T, H, D, dtype, 3), rows(T, H, D, dtype, 4, special=False)
    both = torch.cat([k, k, v], 1).to(dev)                        # views of a joint projection
    slot = _slots(T, nb, block, 5)
    want = codes(c)
    print(f"[gpu] kv mx {kind} {dtype} T={T} H={H} D={D} block={block}", flush=True)
    dro.kv_store(ctx, c, both[:, :H], both[:, 2 * H:], torch.from_numpy(slot).to(dev))
    torch.cuda.synchronize()
    at = np.flatnonzero((slot >= 0) & (slot < nb * block))
    values = []
    for (code, byte), (have, power), x in zip(want, codes(c), (k, v)):
        wc, wb = encode(x[at], kind, dtype)
        code[slot[at] // block, slot[at] % block] = wc
        byte[slot[at] // block, slot[at] % block] = wb
        assert np.array_equal(power, byte), "powers"
        finite = np.repeat(byte != 255, code.shape[-1] // byte.shape[-1], -1)
        if kind == "mxfp8":                                         # (NaN has two codes, by its sign)
            have[(have & 0x7f) == 0x7f] = 0x7f
        assert np.array_equal(have[finite], code[finite]), "codes"   # (a NaN group's codes: any)
        y = np.zeros((T, H, D))
        y[at] = okv.mx_decode(wc, wb, kind)
        values.append(y)
    t16 = torch.bfloat16 if dtype == "bf16" else torch.float16
    got = dro.kv_load(ctx, c, torch.from_numpy(slot).to(dev), dtype=t16)
    for y, name in zip(values, "kv"):
        z = torch.from_numpy(y).to(t16)
        assert same(as_np(got[name].cpu()), as_np(z)), name
        assert (y[at][np.isfinite(y[at])] == as_np(z)[at][np.isfinite(y[at])]).all() or dtype == "f16"


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("kind", ["mxfp4", "mxfp8"])
def test_every_code_and_power(ctx, dev, kind, dtype):
    """Every code under every byte of the powers reads as its value rounded to the type once."""
    import torch
    import paper_2607_16892_amd as dro
    D, block = 256, 16
    T = 256
    code = np.tile(np.arange(D // 2 if kind == "mxfp4" else D, dtype=np.uint8), (T, 1, 1))
    if kind == "mxfp4":
        code = np.concatenate([code, code + 128], 1)              # two heads: all bytes
    byte = np.broadcast_to(np.arange(256, dtype=np.uint8)[:, None, None], (T, code.shape[1], D // 32)).copy()
    c = cache(dev, kind, T // block, block, code.shape[1], D)
    slot = np.arange(T)
    put(c, slot, block, (code, byte), (code[:, :, ::-1].copy(), byte))
    t16 = torch.bfloat16 if dtype == "bf16" else torch.float16
    got = dro.kv_load(ctx, c, torch.from_numpy(slot).to(dev), dtype=t16)
    for name, cc in (("k", code), ("v", code[:, :, ::-1])):
        want = torch.from_numpy(okv.mx_decode(np.ascontiguousarray(cc), byte, kind)).float().to(t16)
        assert same(as_np(got[name].cpu()), as_np(want)), name


@pytest.mark.parametrize("cache_type,dtype", [("bf16", "bf16"), ("f16", "f16"), ("fp8", "bf16"), ("fp8", "f16")])
def test_load_of_the_other_types(ctx, dev, cache_type, dtype):
    """16-bit caches give their bits, 8-bit ones code times scale rounded once; rows may be strided
    and out of their own tensors, and slots may repeat."""
    import torch
    import paper_2607_16892_amd as dro
    from kv_cases import dtypes
    T, H, D, nb, block = 77, 3, 80, 9, 16
    g = torch.Generator().manual_seed(1)
    dt = dtypes()
    k, v = (torch.randn((nb, block, H, D), generator=g).to(dt[cache_type]) for _ in range(2))
    scales = [torch.rand(H, generator=g) + 0.3 for _ in range(2)] if cache_type == "fp8" else [None, None]
    c = dro.KvCache(k.to(dev), v.to(dev), *(None if s is None else s.to(dev) for s in scales))
    slot = torch.randint(0, nb * block, (T,), generator=g)
    slot[3], slot[9], slot[10] = -5, nb * block, slot[11]
    buf = torch.full((T, 2 * H + 1, D + 8), 9.0, dtype=dt[dtype], device=dev)
    got = dro.kv_load(ctx, c, slot.to(dev), k=buf[:, :H, :D], v=buf[:, H:2 * H, :D])
    keep = (slot >= 0) & (slot < nb * block)
    for name, x, s in (("k", k, scales[0]), ("v", v, scales[1])):
        y = x.float().reshape(-1, H, D)[slot.clamp(0, nb * block - 1)]
        y = torch.where(keep[:, None, None], y if s is None else y * s[None, :, None], 0.0).to(dt[dtype])
        assert torch.equal(got[name].cpu(), y), name
    assert (buf[:, 2 * H] == 9).all() and (buf[:, :, D:] == 9).all()
    assert dro.kv_load(ctx, c, slot[:0].to(dev))["k"].shape == (0, H, D)


def test_a_prefix_moves_between_types(ctx, dev):
    """bf16 to MXFP8 to MXFP4 and on to a cache of another block size: what each holds is what its
    format makes of what it was given."""
    import torch
    import paper_2607_16892_amd as dro
    T, H, D = 100, 2, 64
    x, y = rows(T, H, D, "bf16", 8, special=False), rows(T, H, D, "bf16", 9, special=False)
    slot = torch.arange(T, device=dev)
    at = [dro.KvCache.empty(7, 16, H, D, torch.bfloat16, dev), dro.KvCache.empty(2, 64, H, D, "mxfp8", dev),
          dro.KvCache.empty(7, 16, H, D, "mxfp4", dev), dro.KvCache.empty(4, 32, H, D, torch.bfloat16, dev)]
    k, v = x.to(dev), y.to(dev)
    for c in at:
        dro.kv_store(ctx, c, k, v, slot)
        got = dro.kv_load(ctx, c, slot)
        k, v = got["k"], got["v"]
    for got, z in ((k, x), (v, y)):
        z8 = okv.mx_decode(*encode(z, "mxfp8", "bf16"), "mxfp8")
        z4 = okv.mx_decode(*okv.mx_encode(z8, "mxfp4", "bf16"), "mxfp4")
        assert same(as_np(got.cpu()), z4)


def test_places_beyond_32_bits(ctx, dev):
    """A cache of 6 GB: codes and powers at its end."""
    import torch
    import paper_2607_16892_amd as dro
    H, D, block = 8, 128, 1024
    nb = 6000                                                      # 3.1 GB of codes each
    c = dro.KvCache.empty(nb, block, H, D, "mxfp4", dev)
    x = rows(50, H, D, "bf16", 2, special=False)
    slot = torch.arange(nb * block - 50, nb * block, device=dev)
    dro.kv_store(ctx, c, x.to(dev), x.to(dev), slot)
    got = dro.kv_load(ctx, c, slot)
    want = okv.mx_decode(*encode(x, "mxfp4", "bf16"), "mxfp4")
    assert same(as_np(got["k"].cpu()), want) and same(as_np(got["v"].cpu()), want)
    assert int(torch.count_nonzero(c.k[: nb - 1])) == 0


def test_side_stream_and_graph(dev):
    """On another stream and captured: the replays write and read the inputs of their time."""
    import torch
    import paper_2607_16892_amd as dro
    T, H, D = 40, 4, 128
    with dro.Context(dev.index or 0) as ctx:
        c = dro.KvCache.empty(4, 16, H, D, "mxfp4", dev)
        x = rows(T, H, D, "bf16", 1, special=False).to(dev)
        slot = torch.arange(T, device=dev)
        out = dict(k=torch.zeros_like(x), v=torch.zeros_like(x))
        s = torch.cuda.Stream(dev)
        s.wait_stream(torch.cuda.current_stream(dev))
        dro.kv_store(ctx, c, x, x, slot, stream=s)
        dro.kv_load(ctx, c, slot, **out, stream=s)
        torch.cuda.current_stream(dev).wait_stream(s)
        assert same(as_np(out["k"].cpu()), okv.mx_decode(*encode(x.cpu(), "mxfp4", "bf16"), "mxfp4"))
        graph = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=s):
            dro.kv_store(ctx, c, x, x, slot)
            dro.kv_load(ctx, c, slot, **out)
        for seed in (5, 6, 7):
            x.copy_(rows(T, H, D, "bf16", seed, special=False))
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            want = okv.mx_decode(*encode(x.cpu(), "mxfp4", "bf16"), "mxfp4")
            assert same(as_np(out["k"].cpu()), want) and same(as_np(out["v"].cpu()), want)


def test_refusals(ctx, dev):
    import torch
    import paper_2607_16892_amd as dro
    from paper_2607_16892_amd import _native
    c = dro.KvCache.empty(2, 16, 2, 64, "mxfp4", dev)
    x = torch.zeros((3, 2, 64), dtype=torch.bfloat16, device=dev)
    slot = torch.arange(3, device=dev)
    for bad in (dict(k_power=c.k_power), dict(v_power=c.v_power),
                dict(k_power=c.k_power, v_power=c.v_power.cpu()),
                dict(k_power=c.k_power.float(), v_power=c.v_power)):
        with pytest.raises(TypeError):
            dro.KvCache(c.k, c.v, **bad)
    with pytest.raises(ValueError):
        dro.KvCache(c.k, c.v, k_power=c.k_power[:1], v_power=c.v_power)
    apart = torch.zeros((2, 16, 2, 2), dtype=torch.uint8, device=dev)   # tokens of a head apart
    with pytest.raises(ValueError):
        dro.KvCache(c.k, c.v, k_power=apart, v_power=c.v_power)
    with pytest.raises(TypeError):
        dro.KvCache(c.k, c.v)                                      # bytes without powers
    with pytest.raises(TypeError):
        dro.KvCache(x[None, :2], x[None, :2], k_power=c.k_power, v_power=c.v_power)
    one = torch.ones(2, device=dev)
    with pytest.raises(dro.DroError):                              # scales beside powers
        dro.kv_store(ctx, dro.KvCache(c.k, c.v, one, one, c.k_power, c.v_power), x, x, slot)
    wide = torch.zeros((2, 16, 2, 40), dtype=torch.uint8, device=dev)
    with pytest.raises(dro.DroError):                              # rows of 40 bytes: not aligned
        dro.kv_store(ctx, dro.KvCache(wide[..., :32], wide[..., :32], k_power=c.k_power, v_power=c.v_power), x, x, slot)
    with pytest.raises(TypeError):
        dro.kv_load(ctx, c, slot, dtype=torch.float32)
    with pytest.raises(ValueError):
        dro.kv_load(ctx, c, slot, k=x[:2])
    with pytest.raises(ValueError):
        dro.kv_load(ctx, c, slot, dtype=torch.float16, k=x)
    with pytest.raises(TypeError):
        dro.kv_load(ctx, c, slot.int())
    with pytest.raises(TypeError):
        dro.kv_load(ctx, c, slot, k=[1, 2, 3])
    with pytest.raises(dro.DroError):                              # a 16-bit cache gives its own type
        dro.kv_load(ctx, dro.KvCache.empty(2, 16, 2, 64, torch.float16, dev), slot, dtype=torch.bfloat16)
    with pytest.raises(dro.DroError):                              # rows of 68 elements: not aligned
        dro.kv_load(ctx, c, slot, k=torch.zeros((3, 2, 68), dtype=torch.bfloat16, device=dev)[..., :64])
    grad = x.clone().requires_grad_()
    with pytest.raises(RuntimeError, match="no backward"):
        dro.kv_store(ctx, c, grad, x, slot)
    with pytest.raises(RuntimeError, match="no backward"):
        dro.kv_load(ctx, c, slot, k=grad, v=x)
    s = c.struct()
    lib = ctx._lib
    import ctypes as ct

    def load(cache, T=3, dtype=0):
        return lib.kv_load(ctx.handle, ct.byref(cache), dtype, T, x.data_ptr(), 128, 64, x.data_ptr(), 128, 64,
                           slot.data_ptr(), None)

    for change, code in ((dict(dtype=5), -1), (dict(k_power=None), -1),
                         (dict(v_power_block=-16), -5), (dict(v_power_block=-1), -1),
                         (dict(k_power_head=1 << 39), -5), (dict(k_power_head=8), -1), (dict(v_power=s.v_power + 4), -1),
                         (dict(dim=48), -5),
                         (dict(k_head=16), -1), (dict(k=s.k + 8), -1), (dict(dim=288), -5)):
        bad = _native.KvCacheStruct.from_buffer_copy(s)
        for name, value in change.items():
            setattr(bad, name, value)
        assert load(bad) == code, change
    assert load(s, T=-1) == -1 and load(s, dtype=3) == -1 and load(s, T=1 << 25) == -5
    assert int(torch.count_nonzero(c.k)) == 0 and int(torch.count_nonzero(c.k_power)) == 0
