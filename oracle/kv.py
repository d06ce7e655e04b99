"""The paged-cache operators by their definitions, in Python integers and fp64 (CPU).

block_tables   one scheduling step, request by request, with the free blocks as a list
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
