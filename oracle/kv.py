"""The paged-cache operators by their definitions, in Python integers and fp64 (CPU).

block_tables   one scheduling step, request by request, with the free blocks as a list
mx_encode      rows into shared scales (a power of two for 32 components), by search
mx_decode      the values that such codes stand for
attention      one request's rows, key by key visible to each, with an fp64 softmax, and
               the quantities that the tests' error bounds are made of
"""
from __future__ import annotations

import numpy as np


def block_tables(block, table, held, free_list, free, length, add, reserve, tokens):
    table, stack = table.copy(), [int(x) for x in free_list[:free]]
    R, W = table.shape
    words = [int(x) for x in free_list]
    new_held = [int(x) for x in held]
    for r in range(R):
        if add[r] < 0:
            stack += [int(x) for x in table[r, : held[r]]]
            new_held[r] = 0
    words[: len(stack)] = stack
    left, waits = len(stack), False
    context, granted, start = [], [], [0]
    slot, pos = [-1] * tokens, [-1] * tokens
    for r in range(R):
        n = max(int(add[r]), 0)
        most = int(length[r]) + n
        if reserve is not None:
            most = max(most, int(reserve[r]))
        blocks = -(-most // block)
        ok = add[r] >= 0 and blocks <= W
        if ok and blocks > held[r]:
            waits = waits or blocks - held[r] > left
            ok = not waits
            if ok:
                for b in range(held[r], blocks):
                    left -= 1
                    table[r, b] = stack[left]
                new_held[r] = blocks
        if ok:
            for i in range(n):
                if start[-1] + i < tokens:
                    p = int(length[r]) + i
                    pos[start[-1] + i] = p
                    slot[start[-1] + i] = int(table[r, p // block]) * block + p % block
        granted.append(int(ok))
        context.append(int(length[r]) + n if ok else 0)
        start.append(start[-1] + n)
    return dict(table=table, free_list=words, held=new_held, free=[left], context=context,
                granted=granted, start=start, slot=slot, pos=pos)


def attention(q, k, v, context, scale, softcap=0.0, window=0, slopes=None, prefix=0):
    """q [n, Hq, D]; k, v [context, H, D] (fp64).  Returns out [n, Hq, D], lse [n, Hq],
    mass = sum of the weights times |v| (same shape as out), and per row the largest
    scale sum |q k| and |s| over the keys seen."""
    n, Hq, D = q.shape
    G = Hq // k.shape[1]
    out, mass = np.zeros((n, Hq, D)), np.zeros((n, Hq, D))
    lse = np.full((n, Hq), -np.inf)
    dots, tops = np.zeros((n, Hq)), np.zeros((n, Hq))
    for i in range(n):
        p = context - n + i
        j = np.arange(context)
        see = (j <= p) | (j < prefix)
        if window:
            see &= p - j < window
        j = j[see]
        if not len(j):
            continue
        for h in range(Hq):
            kk, vv = k[j, h // G], v[j, h // G]
            s = scale * (kk @ q[i, h])
            dots[i, h] = abs(scale) * (np.abs(kk) @ np.abs(q[i, h])).max()
            if softcap:
                s = softcap * np.tanh(s / softcap)
            if slopes is not None:
                s = s + float(slopes[h]) * (j - p)
            m = s.max()
            e = np.exp(s - m)
            lse[i, h] = m + np.log(e.sum())
            out[i, h] = (e @ vv) / e.sum()
            mass[i, h] = (e @ np.abs(vv)) / e.sum()
            tops[i, h] = np.abs(s).max()
    return dict(out=out, lse=lse, mass=mass, dots=dots, tops=tops)


MX_CODES = {
    "mxfp4": [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0],
    "mxfp8": [m * 2.0 ** -9 for m in range(8)]
             + [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:-1],
}
# powers that may be written from bf16 and from f16
MX_POWERS = {("mxfp4", "bf16"): (-125, 125), ("mxfp4", "f16"): (-125, 13),
             ("mxfp8", "bf16"): (-117, 119), ("mxfp8", "f16"): (-117, 7)}
FINITE = {"bf16": (2.0 - 2.0 ** -7) * 2.0 ** 127, "f16": 65504.0}


def mx_encode(x, kind, dtype):
    """Rows x [.., D] (fp64, values of `dtype`) into codes and powers' bytes: uint8 [.., D / 2]
    (mxfp4) or [.., D] (mxfp8), and uint8 [.., D / 32]."""
    values = np.array(MX_CODES[kind])
    lowest, highest = MX_POWERS[kind, dtype]
    half = (values[-1] - values[-2]) / 2
    g = x.reshape(-1, 32)
    bad = np.isnan(g)
    size = np.minimum(np.abs(np.where(bad, 0.0, g)), FINITE[dtype])
    top = size.max(1)
    # from below up until the largest is not above half a step too much
    e = np.clip(np.floor(np.log2(np.maximum(top, 2.0 ** -200))) - 12, lowest, highest).astype(np.int64)
    while True:
        small = (top > (values[-1] + half) * 2.0 ** e) & (e < highest)
        if not small.any():
            break
        e[small] += 1
    a = size / 2.0 ** e[:, None]
    # the nearest value, of two the one with the even code: count those whose upper neighbour is
    # not further away
    middle = (values[1:] + values[:-1]) / 2
    code = np.zeros(a.shape, np.int64)
    for n, m in enumerate(middle):
        code += (a > m) | ((a == m) & (n % 2 == 1))
    byte = (e + 127).astype(np.int64)
    neg = np.signbit(g) & ~bad
    if kind == "mxfp8":
        code = np.where(bad, 0x7f, code) + 128 * neg
        return code.astype(np.uint8).reshape(x.shape), byte.astype(np.uint8).reshape(*x.shape[:-1], -1)
    byte[bad.any(1)] = 255
    code = (code + 8 * neg).reshape(*x.shape[:-1], -1, 2)
    return ((code[..., 0] + 16 * code[..., 1]).astype(np.uint8),
            byte.astype(np.uint8).reshape(*x.shape[:-1], -1))


def mx_decode(code, byte, kind):
    """The values (fp64) of codes and powers' bytes as mx_encode gives them."""
    values = np.array(MX_CODES[kind])
    if kind == "mxfp4":
        code = np.stack([code & 15, code >> 4], -1).reshape(*code.shape[:-1], -1)
        table = np.concatenate([values, -values])
    else:
        table = np.concatenate([values, [np.nan], -values, [np.nan]])
    power = np.where(byte == 255, np.nan, 2.0 ** (byte.astype(np.float64) - 127))
    return table[code] * np.repeat(power, 32, axis=-1)
