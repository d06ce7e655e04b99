"""The oracle of shared scales against the format's rules, and the binding's checks (CPU)."""
import ctypes as ct

import numpy as np
import pytest

from mx_cases import as_np, encode, rows, same
from oracle import kv as okv


@pytest.mark.parametrize("kind,dtype", [(k, t) for k in ("mxfp4", "mxfp8") for t in ("bf16", "f16")])
def test_nearest_values(kind, dtype):
    """Every component becomes the nearest value of its group's power (ties to even), the power is
    the least that cuts nothing by more than half a step, and a second time changes nothing."""
    x = rows(40, 2, 96, dtype, 1)
    code, byte = encode(x, kind, dtype)
    y, g = okv.mx_decode(code, byte, kind).reshape(-1, 32), as_np(x).reshape(-1, 32)
    top = np.array(okv.MX_CODES[kind])
    lowest, highest = okv.MX_POWERS[kind, dtype]
    half = (top[-1] - top[-2]) / 2
    values = np.concatenate([-top[::-1], top])
    for row, got, b in zip(g, y, byte.reshape(-1)):
        nan = np.isnan(row)
        if nan.any() and kind == "mxfp4":
            assert b == 255 and np.isnan(got).all()
            continue
        assert np.array_equal(np.isnan(got), nan)
        e = int(b) - 127
        size = np.minimum(np.abs(row[~nan]), okv.FINITE[dtype])
        most = size.max() if len(size) else 0.0
        assert lowest <= e <= highest
        assert most <= (top[-1] + half) * 2.0 ** e or e == highest
        assert e == lowest or most > (top[-1] + half) * 2.0 ** (e - 1)
        a = np.copysign(size, row[~nan])
        near = np.abs(a[:, None] - values[None] * 2.0 ** e).min(1)
        assert np.array_equal(np.abs(a - got[~nan]), near)
    again = okv.mx_encode(np.where(np.isnan(okv.mx_decode(code, byte, kind)), 0.0, okv.mx_decode(code, byte, kind)), kind, dtype)
    y2 = okv.mx_decode(*again, kind).reshape(-1, 32)
    keep = ~np.isnan(y).any(1)
    assert same(y[keep], y2[keep])


def test_codes():
    """The list of codes is the format's: 4 bits 1 + 2 exponent + 1 fraction bits, 8 bits e4m3."""
    torch = pytest.importorskip("torch")
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    byte = np.full((1, 8), 127, np.uint8)
    got = okv.mx_decode(np.arange(256, dtype=np.uint8)[None], byte, "mxfp8")[0]
    assert same(got, every)
    four = okv.mx_decode((np.arange(16, dtype=np.uint8) * 17)[None], byte[:, :1], "mxfp4")[0]
    for c in range(16):
        e, m = c >> 1 & 3, c & 1
        want = (m / 2 if e == 0 else (1 + m / 2) * 2.0 ** (e - 1)) * (-1 if c & 8 else 1)
        assert four[2 * c] == want and four[2 * c + 1] == want
    nan = okv.mx_decode(np.zeros((1, 16), np.uint8), np.full((1, 1), 255, np.uint8), "mxfp4")
    assert np.isnan(nan).all()


def test_caches_on_the_host_are_refused():
    import torch
    import paper_2607_16892_amd as dro
    code, power = torch.zeros((2, 16, 1, 32), dtype=torch.uint8), torch.zeros((2, 16, 1, 2), dtype=torch.uint8)
    with pytest.raises(TypeError, match="CUDA"):
        dro.KvCache(code, code, k_power=power, v_power=power)
    with pytest.raises(ValueError, match="multiple of 32"):
        dro.KvCache.empty(2, 16, 1, 48, "mxfp4", "cpu")
    with pytest.raises(ValueError, match="no k_scale"):
        dro.KvCache.empty(2, 16, 1, 64, "mxfp8", "cpu", k_scale=torch.ones(1))


def test_calls_without_a_context_are_refused():
    from paper_2607_16892_amd import _native
    lib = _native.load()
    c = _native.KvCacheStruct()
    assert lib.kv_load(None, ct.byref(c), 0, 1, None, 8, 8, None, 8, 8, None, None) == -1
    assert lib.kv_store(None, ct.byref(c), 0, 1, None, 8, 8, None, 8, 8, None, None) == -1
