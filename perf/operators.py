"""Cases of the paged-cache operators: block tables, the store into the cache, attention over it.

  tables   kv_block_tables: one scheduling step of a serving loop.  Requests grow by
           their new tokens or to their reservation, ended ones give their blocks back,
           and every new token gets its slot
  store    kv_store: the new tokens' keys and values into the cache
  attn     kv_attention: the new tokens' attention over the cache, single tokens
           (decode), chunks of a prompt over what is cached already, and whole prompts

Sizes follow the package's own: blocks of 16 tokens, inputs of 50 to 2,000 tokens, lengths
up to 8192 and 32768, heavy-tailed output lengths; heads as one GPU of a tensor-parallel
group holds them (head dimensions 64 to 256).  The requests' lengths follow from the case
("mix"), the values and the order of the blocks in the pool from the seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.float8_e4m3fn}
SIZE = {"bf16": 2, "f16": 2, "fp8": 1}
FP8_MAX = 448.0


# ------------------------------------------------------------------- cases ----

def _tables(name=None, *, R, T, width, mix, ended=0, tight=False, reserve=True, block=16):
    c = dict(kind="tables", R=R, T=T, width=width, mix=mix, ended=ended, tight=tight,
             reserve=reserve, block=block)
    return dict(c, name=name) if name else c


def _store(name=None, *, T, H, D, dtype="bf16", cache="bf16", block=16, fused=True):
    c = dict(kind="store", T=T, H=H, D=D, dtype=dtype, cache=cache, block=block, fused=fused)
    return dict(c, name=name) if name else c


def _attn(name=None, *, R, lo, hi, new_lo=1, new_hi=1, chunks=-1, Hq, H, D=128, dtype="bf16",
          cache="", mix, block=16, cap=0.0, window=0, slopes=False, prefix=0):
    c = dict(kind="attn", R=R, lo=lo, hi=hi, new_lo=new_lo, new_hi=new_hi,
             chunks=R if chunks < 0 else chunks, Hq=Hq, H=H, D=D, dtype=dtype,
             cache=cache or dtype, mix=mix, block=block, cap=cap, window=window, slopes=slopes,
             prefix=prefix)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decode step of a small service: 64 requests, one token each
        _tables("tables-64-decode", R=64, T=64, width=512, mix=1),
        # a large service at a busy moment: some of 4,096 requests end, some bring chunks of
        # their prompts, the pool is nearly full, a table row covers 32,768 tokens
        _tables("tables-4096-busy", R=4096, T=65_536, width=2048, mix=2, ended=400, tight=True),
        # one layer of a decode step: 64 tokens' heads out of a fused projection
        _store("store-64-decode", T=64, H=8, D=128),
        # one layer of a step full of prompts, kept in 8 bits
        _store("store-8001-fp8", T=8001, H=8, D=128, cache="fp8"),
        # one request of about a thousand tokens on one of eight tensor-parallel GPUs: latency
        _attn("decode-1x1k", R=1, lo=1000, hi=1000, Hq=8, H=1, mix=3),
        # an ordinary decode step: 64 requests of unequal lengths
        _attn("decode-64-ragged", R=64, lo=50, hi=8192, Hq=32, H=8, mix=4),
        # a large decode step over an 8-bit cache
        _attn("decode-128-fp8", R=128, lo=1000, hi=16_384, Hq=64, H=8, cache="fp8", mix=5),
        # few very long requests, seven query heads to a key head
        _attn("decode-3-long", R=3, lo=100_001, hi=131_071, Hq=28, H=4, dtype="f16", mix=6),
        # chunks of 512 prompt tokens over the tokens cached before
        _attn("chunk-4x512", R=4, lo=4000, hi=8192, new_lo=512, new_hi=512, Hq=32, H=8, mix=7),
        # a whole prompt of 8,192 tokens
        _attn("prompt-8192", R=1, lo=8192, hi=8192, new_lo=8192, new_hi=8192, Hq=64, H=8, mix=8),
        # a mixed step (decode and odd chunks) of a model with capped scores and a window
        _attn("mixed-cap-window", R=40, lo=100, hi=4096, new_lo=33, new_hi=300, chunks=9, Hq=8,
              H=4, D=256, cap=50.0, window=1024, mix=9),
        # prompts with a prefix that all of their tokens see, biased by distance, one head to a
        # key head
        _attn("prefix-bias", R=6, lo=300, hi=2000, new_lo=300, new_hi=2000, Hq=12, H=12, D=64,
              dtype="f16", slopes=True, prefix=200, mix=10),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    mix = rng.randrange(1, 1 << 20)
    kind = rng.choice(("tables", "store", "attn", "attn", "attn"))
    if kind == "tables":
        R = log(1, 4096)
        return _tables(R=R, T=log(R, max(R, min(65_536, 400 * R))), width=rng.choice((512, 700, 2048)),
                       mix=mix, ended=rng.randrange(R // 4 + 1), tight=rng.random() < 0.4,
                       reserve=rng.random() < 0.7, block=rng.choice((16, 32, 64)))
    if kind == "store":
        return _store(T=log(1, 8192), H=rng.choice((1, 2, 4, 5, 8)), D=rng.choice((64, 80, 128, 256)),
                      **rng.choice((dict(), dict(dtype="f16", cache="f16"), dict(cache="fp8"),
                                    dict(dtype="f16", cache="fp8"))),
                      block=rng.choice((16, 32, 64)), fused=rng.random() < 0.6)
    H, G = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 4, 7, 8))
    D = rng.choice((64, 80, 128, 128, 256))
    if D == 256:
        G = min(G, 4)
    dtype = rng.choice(("bf16", "bf16", "f16"))
    more = dict(Hq=H * G, H=H, D=D, dtype=dtype, mix=mix, block=rng.choice((16, 16, 32, 128)))
    if rng.random() < 0.3:
        more["cache"] = "fp8"
    x = rng.random()
    if x < 0.3:
        more["cap"] = rng.choice((20.0, 50.0))
    elif x < 0.5:
        more["slopes"] = True
    if rng.random() < 0.3:
        more["window"] = log(16, 4096)
    form = rng.choice(("decode", "long", "chunks", "prompts", "mixed"))
    if form == "decode":
        hi = log(64, 16_384)
        return _attn(R=log(1, 128), lo=max(1, hi // 16), hi=hi, **more)
    if form == "long":
        hi = log(20_000, 131_072)
        return _attn(R=log(1, 3), lo=hi // 2, hi=hi, **more)
    if rng.random() < 0.3:
        more["prefix"] = log(16, 1000)
    if form == "chunks":
        n = log(2, 512)
        return _attn(R=log(1, 4), lo=max(n, 500), hi=log(max(n, 500), 8192), new_lo=n, new_hi=n, **more)
    if form == "prompts":
        hi = log(1, 2000)
        return _attn(R=log(1, 6), lo=(hi + 2) // 3, hi=hi, new_lo=hi, new_hi=hi, **more)
    R = log(2, 40)
    n = log(2, 300)
    return _attn(R=R, lo=100, hi=log(400, 4096), new_lo=max(1, n // 3), new_hi=n,
                 chunks=rng.randrange(R), **more)


# ----------------------------------------------------------------- lengths ----

def _spread(r, lo, hi, n):
    """n heavy-tailed lengths in [lo, hi]; the first is hi."""
    x = np.exp(r.uniform(math.log(lo), math.log(hi + 1), n)).astype(np.int64)
    x[0] = hi
    return np.clip(x, lo, hi)


def _attn_lengths(c):
    """Context (new tokens included), new tokens and prefix of every request."""
    r = np.random.RandomState(c["mix"])
    ctx = _spread(r, c["lo"], c["hi"], c["R"])
    new = np.ones(c["R"], np.int64)
    at = r.permutation(c["R"])[: c["chunks"]]
    new[at] = r.randint(c["new_lo"], c["new_hi"] + 1, c["R"])[at]
    new = np.minimum(new, ctx)
    return ctx, new, np.minimum(c["prefix"], ctx)


def _tables_lengths(c):
    """Tokens held, new tokens (-1: ends), reservation and blocks held of every request, and
    the blocks free in the pool."""
    r = np.random.RandomState(c["mix"])
    R, B = c["R"], c["block"]
    top = c["width"] * B
    add = np.ones(R, np.int64)
    gone = r.permutation(R)[: c["ended"]]
    add[gone] = -1
    left = c["T"] - int((add > 0).sum())
    if left > 0:                         # chunks of prompts for one request in eight
        live = np.flatnonzero(add > 0)
        if len(live):
            at = live[r.permutation(len(live))[: max(1, len(live) // 8)]]
            share = r.multinomial(left, np.full(len(at), 1.0 / len(at)))
            add[at] += np.minimum(share, top // 2)
    length = np.minimum(_spread(r, 50, top // 4, R), top - np.maximum(add, 0))
    length[r.rand(R) < 0.15] = 0         # requests that start with this step
    want = np.zeros(R, np.int64)
    if c["reserve"]:                     # the input and a reservation for the answer
        want = np.minimum(length + np.exp(r.normal(5.0, 1.0, R)).astype(np.int64), top)
    held = -(-length // B)
    grown = r.rand(R) < 0.7              # most hold their reservation already
    held = np.where(grown & (length > 0), np.maximum(held, -(-want // B)), held)
    need = np.maximum(-(-np.maximum(length + np.maximum(add, 0), want) // B) - held, 0)
    need = int(need[add >= 0].sum())
    free = max(0, need - need // 8 - int(held[add < 0].sum())) if c["tight"] else need + 100
    return length, add, want, held, free


# ----------------------------------------------------------------- prepare ----

_CTX = None


def _context():
    global _CTX
    if _CTX is None:
        import paper_2607_16892_amd as dro
        _CTX = dro.Context(0)
    return _CTX


def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _pool(g, used, block, H, D, cache, filled):
    """A cache of `used` blocks and a tenth more, [blocks, block, heads, dim] seen from blocks
    that hold one head's tokens together, and the order its blocks are handed out in."""
    nb = used + used // 10 + 1
    dt = TYPES[cache]
    kv = []
    for _ in range(2):
        m = torch.empty((nb, H, block, D), dtype=torch.bfloat16 if cache == "fp8" else dt, device=DEV)
        m = m.normal_(generator=g) if filled else m.zero_()
        kv.append((m.to(dt) if cache == "fp8" else m).permute(0, 2, 1, 3))
    scales = [torch.empty(H, device=DEV).uniform_(0.6, 1.6, generator=g) for _ in range(2)] \
        if cache == "fp8" else [None, None]
    order = torch.randperm(nb, generator=g, device=DEV).to(torch.int32)
    return kv, scales, order


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    s = dict(case=c)
    if c["kind"] == "tables":
        length, add, want, held, free = _tables_lengths(c)
        nb = int(held.sum()) + free + 64
        order = torch.randperm(nb, generator=g, device=DEV).to(torch.int32)
        R, W = c["R"], c["width"]
        s.update(length=_i32(length), add=_i32(add), want=_i32(want) if c["reserve"] else None,
                 held=_i32(held), T=c["T"], block=c["block"], num_blocks=nb)
        start = np.concatenate([[0], np.cumsum(held)])
        at = torch.arange(W, device=DEV)[None, :]
        idx = (_i32(start[:-1])[:, None] + at).clamp(max=nb - 1)
        s["table"] = torch.where(at < s["held"][:, None], order[idx.long()], -1).to(torch.int32)
        # the free blocks lie at the bottom of the stack, what is above is old
        stack = torch.full((nb,), -1, dtype=torch.int32, device=DEV)
        stack[:free] = order[int(start[-1]):int(start[-1]) + free]
        s.update(free_list=stack, free=_i32([free]), free_h=free)
    elif c["kind"] == "store":
        T, H, D = c["T"], c["H"], c["D"]
        kv, scales, order = _pool(g, -(-T // c["block"]) + 3, c["block"], H, D, c["cache"], False)
        dt = TYPES[c["dtype"]]
        if c["fused"]:                   # keys and values out of one projection's rows
            x = torch.empty((T, 6 * H, D), dtype=dt, device=DEV).normal_(0, 1.5, generator=g)
            k, v = x[:, 4 * H:5 * H], x[:, 5 * H:]
        else:
            k, v = (torch.empty((T, H, D), dtype=dt, device=DEV).normal_(0, 1.5, generator=g)
                    for _ in range(2))
        # tokens of one chunk in order from the middle of a block on, one in fifty refused
        p = torch.arange(T, device=DEV) + c["block"] // 3
        slot = order[p // c["block"]].long() * c["block"] + p % c["block"]
        slot[torch.rand(T, generator=g, device=DEV) < 0.02] = -1
        s.update(k=k, v=v, kc=kv[0], vc=kv[1], ks=scales[0], vs=scales[1], slot=slot)
    else:
        ctx, new, pre = _attn_lengths(c)
        B = c["block"]
        nblk = -(-ctx // B)
        start = np.concatenate([[0], np.cumsum(nblk)])
        kv, scales, order = _pool(g, int(nblk.sum()), B, c["H"], c["D"], c["cache"], True)
        W = int(nblk.max()) + 3
        at = torch.arange(W, device=DEV)[None, :]
        idx = (_i32(start[:-1])[:, None] + at).clamp(max=order.numel() - 1)
        table = torch.where(at < _i32(nblk)[:, None], order[idx.long()], -1).to(torch.int32)
        cu = np.concatenate([[0], np.cumsum(new)])
        T = int(cu[-1])
        dt = TYPES[c["dtype"]]
        q = torch.empty((T, c["Hq"] + 2 * c["H"], c["D"]), dtype=dt, device=DEV)
        q = q.normal_(generator=g)[:, : c["Hq"]]
        s.update(q=q, kc=kv[0], vc=kv[1], ks=scales[0], vs=scales[1], table=table, start=_i32(cu),
                 context=_i32(ctx), prefix=_i32(pre) if c["prefix"] else None, T=T,
                 max_new=int(new.max()), max_ctx=int(ctx.max()))
        s["slopes"] = (2.0 ** (-8.0 * torch.arange(1, c["Hq"] + 1, device=DEV) / c["Hq"])).float() \
            if c["slopes"] else None
    if own:
        import paper_2607_16892_amd as dro
        s["ctx"] = _context()
        if c["kind"] == "tables":
            s["pool"] = dro.BlockPool(block=s["block"], table=s["table"], held=s["held"],
                                      free_list=s["free_list"], free=s["free"])
        else:
            s["cache"] = dro.KvCache(k=s["kc"], v=s["vc"], k_scale=s["ks"], v_scale=s["vs"])
    return s


# --------------------------------------------------------------------- run ----

def run(state):
    s = state
    kind = s["case"]["kind"]
    if not own:
        return {"tables": _plain_tables, "store": _plain_store, "attn": _plain_attn}[kind](s)
    import paper_2607_16892_amd as dro
    c = s["case"]
    if kind == "tables":
        r = dro.kv_block_tables(s["ctx"], s["pool"], s["length"], s["add"], s["T"], reserve=s["want"])
        return dict(table=s["table"], free_list=s["free_list"], **r)
    if kind == "store":
        dro.kv_store(s["ctx"], s["cache"], s["k"], s["v"], s["slot"])
        return dict(k=s["kc"], v=s["vc"])
    return dro.kv_attention(s["ctx"], s["cache"], s["q"], s["table"], s["start"], s["context"],
                            s["max_new"], softcap=c["cap"], window=c["window"], slopes=s["slopes"],
                            prefix=s["prefix"])


def _plain_tables(s):
    B, W, nb, T = s["block"], s["table"].shape[1], s["num_blocks"], s["T"]
    table, stack = s["table"].clone(), torch.cat([s["free_list"], s["free_list"][:1]])
    length, add, held = s["length"].long(), s["add"].long(), s["held"].long()
    ended = add < 0
    n = add.clamp(min=0)
    after = length + n
    most = after if s["want"] is None else torch.maximum(after, s["want"].long())
    blocks = (most + B - 1) // B
    live = ~ended & (blocks <= W)
    grow = torch.where(live, (blocks - held).clamp(min=0), 0)
    back = torch.where(ended, held, 0)
    free = s["free"].long()
    top = free + back.sum()
    cum = grow.cumsum(0)
    granted = live & ((grow == 0) | (cum <= top))
    j = torch.arange(W, device=DEV)[None, :]
    # blocks given back, above the free ones
    first = (free + back.cumsum(0) - back)[:, None]
    at = torch.where(j < back[:, None], first + j, nb)
    stack[at.reshape(-1)] = table.reshape(-1)
    # blocks handed out, from the top down
    took = granted[:, None] & (j >= held[:, None]) & (j < blocks[:, None])
    at = top - 1 - (cum - grow)[:, None] - (j - held[:, None])
    table = torch.where(took, stack[at.clamp(0, nb)], table)
    start = torch.cat([torch.zeros(1, dtype=torch.long, device=DEV), n.cumsum(0)])
    t = torch.arange(T, device=DEV)
    r = torch.searchsorted(start[1:], t, right=True).clamp(max=held.numel() - 1)
    pos = length[r] + t - start[r]
    here = (t < start[-1]) & granted[r]
    blk = table.reshape(-1)[(r * W + (pos // B).clamp(0, W - 1))].long()
    return dict(table=table, free_list=stack[:nb], context=torch.where(granted, after, 0).int(),
                free=(top - torch.where(granted, grow, 0).sum()).int(), granted=granted.to(torch.uint8),
                held=torch.where(ended, 0, torch.where(granted, torch.maximum(held, blocks), held)).int(),
                pos=torch.where(here, pos, -1).int(), slot=torch.where(here, blk * B + pos % B, -1),
                start=start.int())


def _plain_store(s):
    B = s["kc"].shape[1]
    out = {}
    keep = (s["slot"] >= 0)
    slot = s["slot"].clamp(min=0)
    for name, x, cache, scale in (("k", s["k"], s["kc"], s["ks"]), ("v", s["v"], s["vc"], s["vs"])):
        y = x.float()
        if scale is not None:
            y = (y / scale[None, :, None]).clamp(-FP8_MAX, FP8_MAX)
        y = y.to(cache.dtype)
        # refused tokens write back what the slot 0 of the pool gets from its own token, if any
        bits = cache.view(torch.uint8)
        yb = y.view(torch.uint8)
        mine = (keep & (slot == 0))
        zero = torch.where(mine[:, None, None], yb.int(), 0).sum(0).to(torch.uint8)
        zero = torch.where(mine.any(), zero, bits[0, 0])
        yb = torch.where(keep[:, None, None], yb, zero[None])
        bits[slot // B, slot % B] = yb
        out[name] = cache
    return out


def _plain_attn(s):
    c = s["case"]
    R, H, Hq, D, N, L, B = c["R"], c["H"], c["Hq"], c["D"], s["max_new"], s["max_ctx"], c["block"]
    G = Hq // H
    start, ctx = s["start"].long(), s["context"].long()
    new = start[1:] - start[:-1]
    i = torch.arange(N, device=DEV)
    j = torch.arange(L, device=DEV)
    tok = (start[:-1, None] + i[None, :]).clamp(max=s["T"] - 1)              # [R, N]
    q = s["q"].float()[tok]                                                 # [R, N, Hq, D]
    q = q.reshape(R, N, H, G, D).permute(0, 2, 3, 1, 4).reshape(R, H, G * N, D)
    blk = s["table"].long().clamp(min=0)[:, j // B]                          # [R, L]
    k, v = (x.to(torch.float32)[blk, (j % B)[None, :]].permute(0, 2, 1, 3) for x in (s["kc"], s["vc"]))
    if s["ks"] is not None:
        k, v = k * s["ks"][None, :, None, None], v * s["vs"][None, :, None, None]
    x = torch.matmul(q, k.transpose(-1, -2)).reshape(R, Hq, N, L) * (1.0 / math.sqrt(D))
    del k
    if c["cap"]:
        x = torch.tanh(x / c["cap"]) * c["cap"]
    p = (ctx - new)[:, None] + i[None, :]                                   # [R, N]
    d = j[None, None, :] - p[:, :, None]                                    # [R, N, L]
    if s["slopes"] is not None:
        x = x + s["slopes"][None, :, None, None] * d[:, None].float()
    see = d <= 0
    if s["prefix"] is not None:
        see = see | (j[None, None, :] < s["prefix"].long()[:, None, None])
    if c["window"]:
        see = see & (d > -c["window"])
    see = see & (j[None, None, :] < ctx[:, None, None])
    x = torch.where(see[:, None], x, -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)
    x = torch.exp(x - top)
    sums = x.sum(-1, keepdim=True)
    lse = (torch.log(sums) + top).squeeze(-1)                               # [R, Hq, N]
    o = torch.matmul(x.reshape(R, H, G * N, L), v).reshape(R, Hq, N, D)
    o = o / torch.where(sums > 0, sums, 1.0)
    # back to the tokens' rows
    row = torch.searchsorted(start[1:], torch.arange(s["T"], device=DEV), right=True)
    n = torch.arange(s["T"], device=DEV) - start[row]
    return dict(lse=lse[row, :, n], out=o[row, :, n].to(s["q"].dtype))


# -------------------------------------------------------------------- work ----

def _visible(c):
    """Per request: keys that some row sees, and (row, key) pairs of one head."""
    ctx, new, pre = _attn_lengths(c)
    keys = pairs = 0
    for L, n, f in zip(ctx.tolist(), new.tolist(), pre.tolist()):
        p = np.arange(L - n, L)
        hi = np.minimum(np.maximum(p + 1, f), L)
        lo = np.maximum(p - c["window"] + 1, 0) if c["window"] else np.zeros_like(p)
        keys += int(hi.max() - lo.min())
        pairs += int((hi - lo).sum())
    return keys, pairs


def work(case):
    c = case
    if c["kind"] == "tables":
        length, add, want, held, free = _tables_lengths(c)
        B = c["block"]
        blocks = -(-np.maximum(length + np.maximum(add, 0), want) // B)
        grow = np.maximum(blocks - held, 0)[add >= 0].sum()
        back = held[add < 0].sum()
        R, T = c["R"], int(np.maximum(add, 0).sum())
        reads = 4 * R * (4 if c["reserve"] else 3) + 4 * grow + 4 * back + 4
        return {"bytes": float(reads + 4 * grow + 4 * back + 4 * R * 3 + R + 8 + 12 * c["T"]),
                "flops": float(4 * R + 4 * T)}
    if c["kind"] == "store":
        n = 2 * c["T"] * c["H"] * c["D"]
        return {"bytes": float(n * (SIZE[c["dtype"]] + SIZE[c["cache"]]) + 8 * c["T"]), "flops": float(n)}
    keys, pairs = _visible(c)
    T = int(_attn_lengths(c)[1].sum())
    kv = 2 * keys * c["H"] * c["D"] * SIZE[c["cache"]]
    io = T * c["Hq"] * (2 * c["D"] * SIZE[c["dtype"]] + 4)
    return {"bytes": float(kv + io + 4 * keys // c["block"]), "flops": 4.0 * c["D"] * c["Hq"] * pairs}


# ------------------------------------------------------------------- exact ----

def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["kind"] == "tables":
        return _exact_tables(s)
    if c["kind"] == "store":
        return _exact_store(s)
    if _visible(c)[1] * c["Hq"] * c["D"] > 3e12:
        return None
    return _exact_attn(s)


def _exact_tables(s):
    """Request by request, with the free blocks as a list."""
    B, T = s["block"], s["T"]
    length, add, held = (s[k].cpu().tolist() for k in ("length", "add", "held"))
    want = [0] * len(length) if s["want"] is None else s["want"].cpu().tolist()
    table, words = s["table"].cpu().numpy().copy(), s["free_list"].cpu().tolist()
    W = table.shape[1]
    stack = words[: s["free_h"]]
    new_held, granted, context, start = list(held), [], [], [0]
    for r in range(len(length)):
        if add[r] < 0:
            stack += table[r, : held[r]].tolist()
            new_held[r] = 0
    words = stack + words[len(stack):]
    left, shut = len(stack), False
    slot, pos = np.full(T, -1, np.int64), np.full(T, -1, np.int32)
    for r in range(len(length)):
        n = max(add[r], 0)
        blocks = -(-max(length[r] + n, want[r]) // B)
        ok = add[r] >= 0 and blocks <= W
        if ok and blocks > held[r]:
            shut = shut or blocks - held[r] > left
            ok = not shut
            if ok:
                for b in range(held[r], blocks):
                    left -= 1
                    table[r, b] = words[left]
                new_held[r] = blocks
        granted.append(int(ok))
        context.append(length[r] + n if ok else 0)
        if ok:
            p = np.arange(length[r], length[r] + n)[: max(0, T - start[-1])]
            pos[start[-1]:start[-1] + len(p)] = p
            slot[start[-1]:start[-1] + len(p)] = table[r, p // B].astype(np.int64) * B + p % B
        start.append(start[-1] + n)
    i32 = lambda a: np.asarray(a, np.int32)  # noqa: E731
    return dict(table=i32(table), free_list=i32(words), context=i32(context), free=i32([left]),
                granted=np.asarray(granted, np.uint8), held=i32(new_held), pos=pos, slot=slot,
                start=i32(start))


def _exact_store(s):
    out = {}
    B = s["kc"].shape[1]
    at = torch.nonzero(s["slot"] >= 0)[:, 0]
    slot = s["slot"][at]
    for name, x, cache, scale in (("k", s["k"], s["kc"], s["ks"]), ("v", s["v"], s["vc"], s["vs"])):
        y = x[at].double()
        if scale is not None:
            y = (y / scale.double()[None, :, None]).clamp(-FP8_MAX, FP8_MAX)
        full = cache.double()
        full[slot // B, slot % B] = y
        out[name] = full
    return out


def _exact_attn(s):
    """Request by request and head by head of the keys, on the tokens the request has."""
    c = s["case"]
    G, B, D = c["Hq"] // c["H"], c["block"], c["D"]
    start, ctx = s["start"].cpu().tolist(), s["context"].cpu().tolist()
    out = torch.zeros((s["T"], c["Hq"], D), dtype=torch.float64, device=DEV)
    lse = torch.zeros((s["T"], c["Hq"]), dtype=torch.float64, device=DEV)
    for r, L in enumerate(ctx):
        a, b = start[r], start[r + 1]
        n = b - a
        p = torch.arange(L - n, L, device=DEV, dtype=torch.float64)[:, None]
        j = torch.arange(L, device=DEV, dtype=torch.float64)[None, :]
        hidden = j > p
        if s["prefix"] is not None:
            hidden &= j >= int(s["prefix"][r])
        if c["window"]:
            hidden |= p - j >= c["window"]
        ids = s["table"][r, : -(-L // B)].long()
        for h in range(c["H"]):
            k, v = (x[ids, :, h].to(torch.float64).reshape(-1, D)[:L] for x in (s["kc"], s["vc"]))
            if s["ks"] is not None:
                k, v = k * s["ks"][h].double(), v * s["vs"][h].double()
            for g in range(G):
                head = h * G + g
                z = s["q"][a:b, head].double() @ k.T / math.sqrt(D)
                if c["cap"]:
                    z = c["cap"] * torch.tanh(z / c["cap"])
                if s["slopes"] is not None:
                    z = z - s["slopes"][head].double() * (p - j)
                z.masked_fill_(hidden, -math.inf)
                lse[a:b, head] = torch.logsumexp(z, -1)
                out[a:b, head] = torch.softmax(z, -1) @ v
    return dict(lse=lse, out=out)
