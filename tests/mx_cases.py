"""Caches in shared scales for the tests: rows that meet every rule of the format, and caches whose
codes the oracle made."""
from __future__ import annotations

import numpy as np

from oracle import kv as okv


def rows(T, H, D, dtype, seed, special=True):
    """[T, H, D] values of a 16-bit type (host tensor): sizes over the whole range, and among the
    first rows zeros, infinities, NaN, the ends of the range and values between two codes."""
    import torch
    g = torch.Generator().manual_seed(seed)
    t = torch.bfloat16 if dtype == "bf16" else torch.float16
    lo, hi = (-140, 128) if dtype == "bf16" else (-24, 16)
    x = torch.randn((T, H, D), generator=g, dtype=torch.float64)
    x *= torch.exp2(torch.randint(lo, hi, (T, H, D // 32, 1), generator=g).double()).expand(-1, -1, -1, 32).reshape(T, H, D)
    x[T // 2:] = torch.randn((T - T // 2, H, D), generator=g, dtype=torch.float64)
    big = torch.finfo(t).max
    x = x.clamp(-big, big).to(t)
    if special and T >= 12:
        x[0] = 0.0
        x[1, :, ::3] = 0.0
        x[2, 0, 1] = float("inf")
        x[3, -1, D - 1] = float("-inf")
        x[4, 0, 5] = float("nan")
        x[5, -1, 32 * (D // 32) - 7] = float("nan")
        x[5, -1, 32 * (D // 32) - 8] = float("inf")
        x[6, 0, :] = big
        x[7, 0, :] = torch.finfo(t).tiny
        # every multiple of an eighth up to 8, the middles of the codes among them, and the tops
        n = torch.arange(D) % 64
        x[8, 0] = ((n + 1) / 8.0 * (1 - 2 * (n % 2))).to(t)
        x[9, 0] = (7.0 if dtype == "bf16" else 3.5) * 4       # exactly the largest that keeps its power
        x[10, 0] = 7.03125 * 4                                # the next bf16 number beyond
        x[11, 0] = 464.0
        x[11, -1] = 466.0 if dtype == "bf16" else 464.25      # the same for 8 bits
    return x


def as_np(x):
    return x.double().numpy()


def cache(dev, kind, nb, block, heads, D, layout="heads", seed=0, fill=0x5a):
    """A KvCache whose codes and powers are `fill`."""
    import torch
    import paper_2607_16892_amd as dro
    out = []
    for width in (D // 2 if kind == "mxfp4" else D, D // 32):
        for _ in range(2):
            heads_first = layout == "heads" or width == D // 32
            shape = (nb, heads, block, width) if heads_first else (nb, block, heads, width)
            x = torch.full(shape, fill, dtype=torch.uint8, device=dev)
            out.append(x.permute(0, 2, 1, 3) if heads_first else x)
    k, v, kp, vp = out
    if kind == "mxfp8":
        k, v = k.view(torch.float8_e4m3fn), v.view(torch.float8_e4m3fn)
    return dro.KvCache(k, v, k_power=kp, v_power=vp)


def put(c, slot, block, k, v):
    """Codes and powers (numpy, from the oracle) into the slots of a cache."""
    import torch
    at = torch.from_numpy(slot // block), torch.from_numpy(slot % block)
    for t, x in ((c.k, k[0]), (c.k_power, k[1]), (c.v, v[0]), (c.v_power, v[1])):
        t.view(torch.uint8)[at[0].to(t.device), at[1].to(t.device)] = torch.from_numpy(x).to(t.device)


def codes(c):
    """Codes and powers of a cache as numpy, keys then values."""
    import torch
    return [tuple(t.view(torch.uint8).cpu().numpy() for t in pair) for pair in ((c.k, c.k_power), (c.v, c.v_power))]


def encode(x, kind, dtype):
    return okv.mx_encode(as_np(x), kind, dtype)


def same(a, b):
    """Equal values, NaN in the same places."""
    return np.array_equal(np.isnan(a), np.isnan(b)) and np.array_equal(np.nan_to_num(a, nan=0.0, posinf=np.inf, neginf=-np.inf),
                                                                       np.nan_to_num(b, nan=0.0, posinf=np.inf, neginf=-np.inf))


def mx_case(dev, kind, ctx, new, Hq, H, D, dtype="bf16", layout="heads", **kw):
    """A Case whose cache is in shared scales: the oracle's codes of normal keys and values, some
    groups of them many times as large."""
    import torch
    import paper_2607_16892_amd as dro
    from kv_cases import Case
    c = Case(dev, ctx, new, Hq, H, D, dtype, layout=layout, **kw)
    out = []
    for n, x in enumerate((c.k_h, c.v_h)):
        y = x.double().numpy().copy()
        y[..., : 32] *= 4.0 if n else 0.25
        code, byte = okv.mx_encode(y, kind, dtype)
        held = torch.from_numpy(okv.mx_decode(code, byte, kind)).float()
        t = [torch.from_numpy(z).to(dev) for z in (code, byte)]
        if layout == "heads":            # laid out as blocks of one head's tokens
            t[0] = t[0].permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
            t[1] = t[1].permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3)
        else:                            # the powers by heads, with some bytes between the blocks'
            nb, blk = t[1].shape[:2]
            size = H * blk * (D // 32)
            wide = torch.full((nb, size + 16), 200, dtype=torch.uint8, device=dev)
            mine = wide[:, :size].unflatten(1, (H, blk, D // 32)).permute(0, 2, 1, 3)
            mine.copy_(t[1])
            t[1] = mine
        if kind == "mxfp8":
            t[0] = t[0].view(torch.float8_e4m3fn)
        out.append((held, *t))
    c.k_h, c.v_h = out[0][0], out[1][0]
    c.k, c.v = out[0][1], out[1][1]
    c.cache = dro.KvCache(c.k, c.v, k_power=out[0][2], v_power=out[1][2])
    c.cache_type = kind
    return c
