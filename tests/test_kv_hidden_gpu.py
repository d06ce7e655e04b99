"""What rows do not see, in caches of 8 bits, below windows and under other layouts."""
import math

import numpy as np
import pytest

from kv_cases import Case, dtypes

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(dev):
    import paper_2607_16892_amd as dro
    c = dro.Context(dev.index or 0)
    yield c
    c.close()


def _bits(x):
    import torch
    return x.view(torch.uint8 if x.element_size() == 1 else torch.int16)


def _codes(c):
    """NaN (both signs) and, where the type has them, infinities, as bits."""
    return {"fp8": (0x7f, -1 & 0xff), "bf16": (0x7fc0, 0x7f80, 0xff80 - 0x10000),
            "f16": (0x7e00, 0x7c00, 0xfc00 - 0x10000)}[c.cache_type]


def _places(c, r, keys):
    import torch
    keys = torch.as_tensor(keys, dtype=torch.long)
    return c.table_h[r, keys // c.block].long().to(c.dev), (keys % c.block).to(c.dev)


CASES = [("bf16", "fp8", 128), ("f16", "fp8", 64), ("bf16", "fp8", 256), ("f16", "fp8", 80), ("bf16", "fp8", 192),
         ("bf16", None, 128), ("f16", None, 256), ("bf16", None, 104)]


@pytest.mark.parametrize("new", [1, 3, 60])
@pytest.mark.parametrize("dtype,cache,D", CASES)
def test_unused_places_may_hold_anything(ctx, dev, new, dtype, cache, D):
    """Blocks of no request and tokens beyond the contexts, as fresh memory leaves them."""
    import torch
    print(f"[gpu] kv hidden {dtype}/{cache} D={D} new={new}", flush=True)
    lens = [new + 5, new + 40, 64 + new, new]
    c = Case(dev, lens, [new] * 4, 4, 2, D, dtype, cache, seed=new + D)
    ref = c.run(ctx)
    c.check(ref)
    used = torch.zeros(c.k.shape[:2], dtype=torch.bool)
    for r, L in enumerate(lens):
        p = torch.arange(L)
        used[c.table_h[r, p // 16].long(), p % 16] = True
    hide = (~used).to(dev)
    for code in _codes(c):
        _bits(c.k)[hide], _bits(c.v)[hide] = code, code
        got = c.run(ctx)
        assert torch.equal(got["out"], ref["out"]) and torch.equal(got["lse"], ref["lse"])


@pytest.mark.parametrize("new", [2, 3, 60])
@pytest.mark.parametrize("dtype,cache,D", CASES)
def test_a_token_that_one_row_sees(ctx, dev, new, dtype, cache, D):
    """NaN in a request's last value and then key: its last row has them, in the values' components,
    and no other row changes."""
    import torch
    lens = [new + 5, new + 40]
    c = Case(dev, lens, [new] * 2, 4, 2, D, dtype, cache, seed=new + D)
    ref = c.run(ctx)
    b, i = _places(c, 1, [lens[1] - 1])
    nan = _codes(c)[0]
    _bits(c.v)[b, i, 0, D - 3] = nan
    got = c.run(ctx)
    hit = torch.zeros_like(ref["out"], dtype=torch.bool)
    hit[2 * new - 1, :2, D - 3] = True
    assert torch.isnan(got["out"][hit]).all()
    assert torch.equal(got["out"][~hit], ref["out"][~hit]) and torch.equal(got["lse"], ref["lse"])
    _bits(c.k)[b, i, 1] = nan
    got = c.run(ctx)
    hit[2 * new - 1, 2:] = True
    assert torch.isnan(got["out"][hit]).all() and torch.isnan(got["lse"][2 * new - 1, 2:]).all()
    assert torch.equal(got["out"][~hit], ref["out"][~hit])
    assert torch.equal(got["lse"][: 2 * new - 1], ref["lse"][: 2 * new - 1])


@pytest.mark.parametrize("new", [1, 3, 60])
@pytest.mark.parametrize("window", [1, 16, 33, 100])
@pytest.mark.parametrize("dtype,cache,D", CASES)
def test_below_a_window(ctx, dev, new, window, dtype, cache, D):
    """NaN and infinities in the keys and values that no row's window reaches, as a service leaves
    the blocks that it has handed on; and in one that only the first row's does."""
    import torch
    lens = [new + 300, new + 77]
    c = Case(dev, lens, [new] * 2, 4, 2, D, dtype, cache, seed=window + D)
    ref = c.run(ctx, window=window)
    c.check(ref, window=window)
    for code in _codes(c):
        for r, L in enumerate(lens):
            below = max(L - new - window + 1, 0)         # the first row's window begins there
            b, i = _places(c, r, list(range(below)))
            _bits(c.k)[b, i], _bits(c.v)[b, i] = code, code
        got = c.run(ctx, window=window)
        assert torch.equal(got["out"], ref["out"]) and torch.equal(got["lse"], ref["lse"])
    if new == 1:
        return
    b, i = _places(c, 0, [lens[0] - new - window + 1])
    _bits(c.v)[b, i, 0, 5] = _codes(c)[0]
    got = c.run(ctx, window=window)
    hit = torch.zeros_like(ref["out"], dtype=torch.bool)
    hit[0, :2, 5] = True
    assert torch.isnan(got["out"][hit]).all()
    assert torch.equal(got["out"][~hit], ref["out"][~hit]) and torch.equal(got["lse"], ref["lse"])


def _relaid(c, k_order, v_order, pad):
    """The case's cache with keys and values in layouts of their own: [blocks, heads, tokens] or
    [blocks, tokens, heads], rows of `pad` components more."""
    import torch
    import paper_2607_16892_amd as dro
    kv = []
    for x, order, more in ((c.k, k_order, 0), (c.v, v_order, pad)):
        nb, B, H, D = x.shape
        shape = {"heads": (nb, H, B), "tokens": (nb, B, H), "outer": (H, nb, B)}[order]
        y = _bits(torch.empty((*shape, D + more), dtype=x.dtype, device=x.device))
        y.fill_(0x7f if x.element_size() == 1 else 0x7fff)
        y = y[..., :D].permute({"heads": (0, 2, 1, 3), "tokens": (0, 1, 2, 3), "outer": (1, 2, 0, 3)}[order])
        y.copy_(_bits(x))
        kv.append(y.view(x.dtype))
    return dro.KvCache(*kv, *(None if s is None else s.to(c.dev) for s in (c.ks, c.vs)))


@pytest.mark.parametrize("new", [1, 50])
@pytest.mark.parametrize("dtype,cache,D", CASES)
@pytest.mark.parametrize("k_order,v_order", [("tokens", "heads"), ("heads", "tokens"), ("outer", "heads"),
                                             ("tokens", "outer")])
def test_keys_and_values_of_different_strides(ctx, dev, new, dtype, cache, D, k_order, v_order):
    import torch
    import paper_2607_16892_amd as dro
    c = Case(dev, [new + 150, new + 3], [new] * 2, 6, 3, D, dtype, cache, seed=D)
    ref = c.run(ctx)
    other = _relaid(c, k_order, v_order, 16)
    c.cache = other
    got = c.run(ctx)
    assert torch.equal(got["out"], ref["out"]) and torch.equal(got["lse"], ref["lse"])
    # the store into both: the same bits in the same places, nothing beside them
    g = torch.Generator(device=dev).manual_seed(D)
    x = torch.randn((40, 6, D), generator=g, device=dev).to(dtypes()[dtype])
    slot = torch.randperm(c.k.shape[0] * c.block, generator=g, device=dev)[:40]
    slot[3] = -1
    plain = dro.KvCache(c.k, c.v, *(None if s is None else s.to(dev) for s in (c.ks, c.vs)))
    for cache_ in (plain, other):
        dro.kv_store(ctx, cache_, x[:, :3], x[:, 3:], slot)
    assert torch.equal(_bits(other.k), _bits(c.k)) and torch.equal(_bits(other.v), _bits(c.v))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("most", [1, 40, 600])
def test_an_infinite_value_of_a_small_weight(ctx, dev, dtype, most):
    """In the middle of a context, under weights that 16 bits may not hold: the component is
    infinite or NaN in the rows that see it, and everything else as it was."""
    import torch
    new, L = [40, 1], [900, 700]
    c = Case(dev, L, new, 4, 2, 64, dtype, seed=17)
    b, i = _places(c, 0, [10])
    c.k[b, i] = 4.0                                      # a key that takes nearly all of the weight
    c.q[:] = 1.0
    ref = c.run(ctx, max_new=most)
    assert torch.isfinite(ref["out"]).all()
    hit = torch.zeros_like(ref["out"], dtype=torch.bool)
    for r, key, a in ((0, 400, 0), (1, 333, 40)):
        b, i = _places(c, r, [key])
        c.v[b, i, 1, 33] = math.inf
        hit[a:a + new[r], 2:, 33] = True
    got = c.run(ctx, max_new=most)
    x = got["out"][hit]
    print(f"[gpu] kv infinity {dtype} most={most}: {int(torch.isnan(x).sum())} of {x.numel()} NaN", flush=True)
    assert (torch.isnan(x) | (x == math.inf)).all()
    assert torch.equal(got["out"][~hit], ref["out"][~hit]) and torch.equal(got["lse"], ref["lse"])
    assert np.isfinite(got["lse"].cpu().numpy()).all()
