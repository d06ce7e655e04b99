"""Cases of the paged cache in shared scales and of shared prefixes.

  swap     kv_store, then kv_load: tokens' keys and values quantised into the cache as they are
           written, and read back as the values it holds
  load     kv_load: the keys and values of tokens out of the cache, in 16 bits
  attn     kv_attention over a cache in shared scales: single tokens, chunks and prompts
  shared   kv_shared_attention: groups of requests whose tokens follow a prefix that the cache
           holds once for each group

Caches in shared scales hold a row's components in groups of 32, each group as a power of two
(a byte, 2^(byte - 127)) and 32 codes: "mx4" of 4 bits (values 0, .5, 1, 1.5, 2, 3, 4, 6 and a
sign; byte i of a row holds the codes of components 2i, its low half, and 2i + 1) or "mx8" of 8
(e4m3).  The power is the least that leaves the group's largest value nearest to the format's
largest or below it, within the powers whose codes are all normal and finite in the type written.

Sizes follow the package's own: blocks of 16 tokens, inputs of 50 to 2,000 tokens of which a
part is shared, lengths up to 8192, 16,384 and 32,768; heads as one GPU of a tensor-parallel
group holds them.  The lengths follow from the case ("mix"), the values and the order of the
blocks in the pool from the seed.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.float8_e4m3fn}
GROUP = 32
# bytes of a component, the powers of the groups among them
SIZE = {"bf16": 2.0, "f16": 2.0, "fp8": 1.0, "mx8": 1.0 + 1.0 / GROUP, "mx4": 0.5 + 1.0 / GROUP}
MX = ("mx4", "mx8")


# ------------------------------------------------------------------- cases ----

def _tokens(kind, name=None, *, T, H, D=128, dtype="bf16", cache, block=16, fused=True, long=0):
    c = dict(kind=kind, T=T, H=H, D=D, dtype=dtype, cache=cache, block=block, fused=fused, long=long)
    return dict(c, name=name) if name else c


def _attn(name=None, *, R, lo, hi, new_lo=1, new_hi=1, chunks=-1, groups=0, loose=0, pre_lo=0,
          pre_hi=0, Hq, H, D=128, dtype="bf16", cache="", mix, block=16, cap=0.0, window=0,
          slopes=False, prefix=0):
    """lo..hi: the tokens of a request (with a shared prefix: those after it)."""
    c = dict(kind="shared" if groups else "attn", R=R, lo=lo, hi=hi, new_lo=new_lo, new_hi=new_hi,
             chunks=R if chunks < 0 else chunks, groups=groups, loose=loose, pre_lo=pre_lo,
             pre_hi=pre_hi, Hq=Hq, H=H, D=D, dtype=dtype, cache=cache or dtype, mix=mix,
             block=block, cap=cap, window=window, slopes=slopes, prefix=prefix)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one layer of a decode step kept in 4 bits: 64 tokens' heads out of a fused projection
        _tokens("swap", "swap-64-mx4", T=64, H=8, cache="mx4"),
        # one layer of a step full of prompts, kept in 8 bits of f16
        _tokens("swap", "swap-8001-mx8", T=8001, H=8, dtype="f16", cache="mx8", fused=False),
        # one request's tokens move to another place: latency
        _tokens("load", "load-500-mx8", T=500, H=2, cache="mx8"),
        # a long prompt out of a 4-bit cache, for a copy elsewhere
        _tokens("load", "load-32768-mx4", T=32_768, H=8, cache="mx4", long=40_000),
        # one request of about a thousand tokens on one of eight tensor-parallel GPUs: latency
        _attn("decode-1x1k-mx4", R=1, lo=1000, hi=1000, Hq=8, H=1, cache="mx4", mix=21),
        # an ordinary decode step of 64 requests of unequal lengths
        _attn("decode-64-mx8", R=64, lo=50, hi=8192, Hq=32, H=8, cache="mx8", mix=22),
        # a large decode step over a 4-bit cache
        _attn("decode-128-mx4", R=128, lo=1000, hi=16_384, Hq=64, H=8, cache="mx4", mix=23),
        # chunks of 512 prompt tokens over the tokens cached before
        _attn("chunk-4x512-mx4", R=4, lo=4000, hi=8192, new_lo=512, new_hi=512, Hq=32, H=8,
              cache="mx4", mix=24),
        # a small decode step: eight requests behind one instruction of a thousand tokens
        _attn("shared-8x1k", R=8, lo=20, hi=300, groups=1, pre_lo=1000, pre_hi=1000, Hq=8, H=1,
              mix=25),
        # a decode step of 64 requests about one document of 8,192 tokens
        _attn("shared-64x8k", R=64, lo=50, hi=2000, groups=1, pre_lo=8192, pre_hi=8192, Hq=32, H=8,
              mix=26),
        # a large decode step over a 4-bit cache: 116 requests in groups behind 12 prefixes, and
        # 12 that share nothing
        _attn("shared-12-mx4", R=128, lo=50, hi=4000, groups=12, loose=12, pre_lo=500, pre_hi=6001,
              Hq=64, H=8, cache="mx4", mix=27),
        # a step of odd chunks and single tokens behind two prefixes, f16, a cap and a window
        # that ends inside the prefixes
        _attn("shared-chunks-window", R=20, lo=100, hi=1500, new_lo=33, new_hi=300, chunks=7,
              groups=2, pre_lo=1801, pre_hi=3500, Hq=12, H=12, D=64, dtype="f16", cap=30.0,
              window=2048, mix=28),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(("swap", "load", "attn", "attn", "shared", "shared"))
    dtype = rng.choice(("bf16", "bf16", "f16"))
    block = rng.choice((16, 16, 32, 64))
    cache = rng.choice(MX)
    if kind in ("swap", "load"):
        return _tokens(kind, T=log(1, 20_000), H=rng.choice((1, 2, 4, 5, 8)),
                       D=rng.choice((64, 96, 128, 256)), dtype=dtype,
                       cache=cache if kind == "swap" or rng.random() < 0.6 else rng.choice((dtype, "fp8")),
                       block=block, fused=rng.random() < 0.6)
    H, G, D = rng.choice((1, 2, 4, 8)), rng.choice((1, 2, 4, 7, 8)), rng.choice((64, 96, 128, 128, 256))
    if D == 256:
        H, G = min(H, 4), min(G, 4)
    more = dict(Hq=H * G, H=H, D=D, dtype=dtype, cache=cache, block=block, mix=rng.randrange(1, 1 << 20))
    x = rng.random()
    if x < 0.2:
        more["cap"] = rng.choice((20.0, 50.0))
    elif x < 0.4:
        more["slopes"] = True
    if rng.random() < 0.25:
        more["window"] = log(16, 4096)
    if kind == "attn":
        form = rng.choice(("decode", "decode", "long", "chunks", "prompts", "mixed"))
        if form == "decode":
            hi = log(64, 16_384)
            return _attn(R=log(1, 128), lo=max(1, hi // 16), hi=hi, **more)
        if form == "long":
            hi = log(20_000, 100_000)
            return _attn(R=log(1, 3), lo=hi // 2, hi=hi, **more)
        if form == "chunks":
            n = log(2, 512)
            return _attn(R=log(1, 4), lo=max(n, 500), hi=log(max(n, 500), 8192), new_lo=n, new_hi=n, **more)
        if form == "prompts":
            hi = log(1, 2000)
            return _attn(R=log(1, 6), lo=(hi + 2) // 3, hi=hi, new_lo=hi, new_hi=hi,
                         prefix=rng.choice((0, 0, 100)), **more)
        R, n = log(2, 40), log(2, 300)
        return _attn(R=R, lo=100, hi=log(400, 4096), new_lo=max(1, n // 3), new_hi=n,
                     chunks=rng.randrange(R), **more)
    if rng.random() < 0.6:
        more["cache"] = rng.choice((dtype, dtype, "fp8"))
    chunks = rng.random() < 0.4
    R = log(1, 24 if chunks else 128)
    groups = min(R, log(1, 16))
    hi, pre = log(1, 2000), log(16, 8192)
    more.update(R=R, groups=groups, loose=rng.randrange(R - groups + 1) if rng.random() < 0.3 else 0,
                lo=(hi + 9) // 10, hi=hi, pre_lo=(pre + 5) // 6, pre_hi=pre)
    if not chunks:
        return _attn(**more)
    n = log(2, 256)
    return _attn(new_lo=max(1, n // 3), new_hi=n, chunks=rng.randrange(min(R, 8) + 1), **more)


# ----------------------------------------------------------------- lengths ----

def _spread(r, lo, hi, n):
    """n heavy-tailed lengths in [lo, hi]; the first is hi."""
    x = np.exp(r.uniform(math.log(lo), math.log(hi + 1), n)).astype(np.int64)
    x[0] = hi
    return np.clip(x, lo, hi)


def _lengths(c):
    """Per request its tokens (new ones included, a shared prefix not), new tokens, prefix that all
    its rows see; per group its first request (and the end) and its shared tokens."""
    r = np.random.RandomState(c["mix"])
    ctx = _spread(r, c["lo"], c["hi"], c["R"])
    new = np.ones(c["R"], np.int64)
    at = r.permutation(c["R"])[: c["chunks"]]
    new[at] = r.randint(c["new_lo"], c["new_hi"] + 1, c["R"])[at]
    new = np.minimum(new, ctx)
    first, pre = np.zeros(1, np.int64), np.zeros(0, np.int64)
    if c["groups"]:
        rest = c["R"] - c["loose"] - c["groups"]
        size = 1 + r.multinomial(rest, np.full(c["groups"], 1.0 / c["groups"]))
        first = np.concatenate([[0], np.cumsum(size)])
        pre = _spread(r, c["pre_lo"], c["pre_hi"], c["groups"])
    return ctx, new, np.minimum(c["prefix"], ctx), first, pre


# ----------------------------------------------------------------- formats ----

def _power(e):
    """2^e of whole e from -126 to 127."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _powers(dtype, four):
    """The least and the largest power of a group: the format's smallest value is a normal bf16
    number there, its largest one finite in `dtype`."""
    wide = dtype != torch.float16
    return (-125, 125 if wide else 13) if four else (-117, 119 if wide else 7)


def _encode(x, kind):
    """Codes (mx4: two a byte; mx8: e4m3) and powers' bytes of rows x [.., D]."""
    g = x.float().unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1)
    m, e = torch.frexp(top)
    four = kind == "mx4"
    e = e - 3 + (m > 0.875).int() if four else e - 9 + (m > 0.90625).int()
    least, most = _powers(x.dtype, four)
    e = torch.where(top > 0, e, least).clamp(least, most)
    y = (g * _power(-e)[..., None]).flatten(-2)
    byte = (e + 127).to(torch.uint8)
    if not four:
        return y.clamp(-448.0, 448.0).to(torch.float8_e4m3fn), byte
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5)
            + (a > 5.0) + (y < 0).to(torch.uint8) * 8).to(torch.uint8)
    return code[..., 0::2] | (code[..., 1::2] << 4), byte


def _decode(code, byte, kind):
    """The values of rows of codes, in 32 bits."""
    if kind == "mx8":
        y = code.float()
    else:
        v = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0], device=code.device)
        v = torch.cat([v, -v])
        y = torch.stack([v[(code & 15).int()], v[(code >> 4).int()]], -1).flatten(-2)
    return (y.unflatten(-1, (-1, GROUP)) * _power(byte.int() - 127)[..., None]).flatten(-2)


def _values(s, name, at, off):
    """Keys ("k") or values ("v") at places (block, token) of the cache, in 32 bits."""
    kind = s["case"]["cache"]
    x = s[name + "c"][at, off]
    if kind in MX:
        return _decode(x, s[name + "e"][at, off], kind)
    x = x.float()
    return x if s[name + "s"] is None else x * s[name + "s"][:, None]


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


def _cache(g, c, used, filled, s):
    """A cache of `used` blocks and a tenth more, [blocks, block, heads, ..] seen from blocks that
    hold one head's tokens together, and the order its blocks are handed out in."""
    nb, H, B, D, kind = used + used // 10 + 2, c["H"], c["block"], c["D"], c["cache"]
    for name in "kv":
        s[name + "e"] = s[name + "s"] = None
        wide = torch.bfloat16 if kind not in ("bf16", "f16") else TYPES[kind]
        m = torch.empty((nb, H, B, D), dtype=wide, device=DEV)
        if filled:
            m.normal_(generator=g)
            # some components of keys are several times as large as the others
            m *= 1.0 + 3.0 * (torch.rand((H, 1, D), generator=g, device=DEV) < 0.05) * (name == "k")
        else:
            m.zero_()
        if kind in MX:
            parts = [_encode(x, kind) for x in m.split(4096)]
            x, e = (torch.cat([p[i] for p in parts]) for i in range(2))
            s[name + "c"], s[name + "e"] = x.permute(0, 2, 1, 3), e.permute(0, 2, 1, 3)
        else:
            s[name + "c"] = m.to(TYPES[kind]).permute(0, 2, 1, 3)
            if kind == "fp8":
                s[name + "s"] = torch.empty(H, device=DEV).uniform_(0.6, 1.6, generator=g)
    return torch.randperm(nb - 1, generator=g, device=DEV).to(torch.int32)   # (the last one: nobody's)


def _tables(order, at, counts):
    """Rows that name counts[r] blocks each, from place `at` of the order on; -1 behind them."""
    start = np.concatenate([[0], np.cumsum(counts)])
    j = torch.arange(int(counts.max()) + 3, device=DEV)[None, :]
    idx = (_i32(at + start[:-1])[:, None] + j).clamp(max=order.numel() - 1)
    return torch.where(j < _i32(counts)[:, None], order[idx.long()], -1).to(torch.int32)


def prepare(case, seed):
    c = case
    g = torch.Generator(device=DEV).manual_seed(int(seed))
    s, dt, B = dict(case=c), TYPES[c["dtype"]], c["block"]
    if c["kind"] in ("swap", "load"):
        T, H, D = c["T"], c["H"], c["D"]
        order = _cache(g, c, -(-max(T, c["long"]) // B) + 3, c["kind"] == "load", s)
        p = torch.arange(T, device=DEV) + B // 3
        slot = order[p // B].long() * B + p % B
        slot[torch.rand(T, generator=g, device=DEV) < 0.02] = -1     # one in fifty refused
        s["slot"] = slot
        if c["kind"] == "swap":
            if c["fused"]:                # keys and values out of one projection's rows
                x = torch.empty((T, 6 * H, D), dtype=dt, device=DEV).normal_(0, 1.5, generator=g)
                s.update(k=x[:, 4 * H:5 * H], v=x[:, 5 * H:])
            else:
                s.update({n: torch.empty((T, H, D), dtype=dt, device=DEV).normal_(0, 1.5, generator=g)
                          for n in "kv"})
    else:
        ctx, new, see, first, pre = _lengths(c)
        nblk, nshare = -(-ctx // B), -(-pre // B)
        order = _cache(g, c, int(nblk.sum() + nshare.sum()), True, s)
        s["table"] = _tables(order, 0, nblk)
        cu = np.concatenate([[0], np.cumsum(new)])
        T = int(cu[-1])
        q = torch.empty((T, c["Hq"] + 2 * c["H"], c["D"]), dtype=dt, device=DEV)
        s.update(q=q.normal_(generator=g)[:, : c["Hq"]], start=_i32(cu), context=_i32(ctx), T=T,
                 see=_i32(see) if c["prefix"] else None, max_new=int(new.max()))
        s["slopes"] = (2.0 ** (-8.0 * torch.arange(1, c["Hq"] + 1, device=DEV) / c["Hq"])).float() \
            if c["slopes"] else None
        # of each request its group, for the plain form; none: an empty group at the end
        of = np.repeat(np.arange(len(pre) + 1), np.diff(np.concatenate([first, [c["R"]]])))
        s["of"] = torch.from_numpy(of).to(DEV)
        total = np.concatenate([pre, [0]])[of] + ctx
        s.update(longest=int(total.max()))
        s["pre"] = _i32(np.concatenate([pre, [0]]))
        if c["groups"]:
            s.update(shared_table=_tables(order, int(nblk.sum()), nshare), first=_i32(first),
                     shared_new=int(np.diff(cu[first]).max()))
        else:
            s["shared_table"] = s["table"][:1]
    if own:
        import paper_2607_16892_amd as dro
        s["ctx"] = _context()
        s["cache"] = dro.KvCache(k=s["kc"], v=s["vc"], k_scale=s["ks"], v_scale=s["vs"],
                                 k_power=s["ke"], v_power=s["ve"])
        if c["kind"] == "shared":
            s["shared"] = dro.SharedPrefixes(first=s["first"], context=s["pre"][:-1],
                                             table=s["shared_table"], max_new=s["shared_new"])
    return s


# --------------------------------------------------------------------- run ----

def run(state):
    s = state
    c = s["case"]
    if not own:
        return {"swap": _plain_swap, "load": _plain_load, "attn": _plain_attn,
                "shared": _plain_attn}[c["kind"]](s)
    import paper_2607_16892_amd as dro
    if c["kind"] in ("swap", "load"):
        if c["kind"] == "swap":
            dro.kv_store(s["ctx"], s["cache"], s["k"], s["v"], s["slot"])
        return dro.kv_load(s["ctx"], s["cache"], s["slot"], dtype=TYPES[c["dtype"]])
    args = [s["ctx"], s["cache"], s["q"], s["table"], s["start"], s["context"], s["max_new"]]
    more = dict(softcap=c["cap"], window=c["window"], slopes=s["slopes"], prefix=s["see"])
    if c["kind"] == "attn":
        return dro.kv_attention(*args, **more)
    return dro.kv_shared_attention(*args, s["shared"], **more)


def _plain_load(s):
    B, slot = s["case"]["block"], s["slot"]
    at, keep = slot.clamp(min=0), (slot >= 0)[:, None, None]
    k, v = (torch.where(keep, _values(s, n, at // B, at % B), 0.0).to(TYPES[s["case"]["dtype"]]) for n in "kv")
    return dict(k=k, v=v)


def _plain_swap(s):
    B, slot = s["case"]["block"], s["slot"]
    at = torch.where(slot >= 0, slot, s["kc"].shape[0] * B - 1)      # refused: into nobody's block
    kcode, kbyte = _encode(s["k"], s["case"]["cache"])
    vcode, vbyte = _encode(s["v"], s["case"]["cache"])
    s["kc"].view(torch.uint8)[at // B, at % B] = kcode.view(torch.uint8)
    s["vc"].view(torch.uint8)[at // B, at % B] = vcode.view(torch.uint8)
    s["ke"][at // B, at % B] = kbyte
    s["ve"][at // B, at % B] = vbyte
    return _plain_load(s)


def _plain_attn(s):
    c = s["case"]
    R, H, Hq, D, N, L, B = c["R"], c["H"], c["Hq"], c["D"], s["max_new"], s["longest"], c["block"]
    G = Hq // H
    start = s["start"].long()
    pre = s["pre"].long()[s["of"]]                                          # [R]
    ctx = pre + s["context"].long()
    new = start[1:] - start[:-1]
    i = torch.arange(N, device=DEV)
    j = torch.arange(L, device=DEV)
    tok = (start[:-1, None] + i[None, :]).clamp(max=s["T"] - 1)              # [R, N]
    q = s["q"].float()[tok]                                                 # [R, N, Hq, D]
    q = q.reshape(R, N, H, G, D).permute(0, 2, 3, 1, 4).reshape(R, H, G * N, D)
    # key j of a request: of its group's prefix, or its own
    shared = j[None, :] < pre[:, None]
    jo = (j[None, :] - pre[:, None]).clamp(min=0)
    mine = s["table"].long().gather(1, (jo // B).clamp(max=s["table"].shape[1] - 1))
    theirs = s["shared_table"].long()[s["of"].clamp(max=s["shared_table"].shape[0] - 1)[:, None],
                                      (j // B).clamp(max=s["shared_table"].shape[1] - 1)[None, :]]
    blk = torch.where(shared, theirs, mine).clamp(min=0)                     # [R, L]
    off = torch.where(shared, j[None, :], jo) % B
    x = torch.matmul(q, _values(s, "k", blk, off).permute(0, 2, 3, 1)).reshape(R, Hq, N, L)
    x = x * (1.0 / math.sqrt(D))
    if c["cap"]:
        x = torch.tanh(x / c["cap"]) * c["cap"]
    p = (ctx - new)[:, None] + i[None, :]                                   # [R, N]
    d = j[None, None, :] - p[:, :, None]                                    # [R, N, L]
    if s["slopes"] is not None:
        x = x + s["slopes"][None, :, None, None] * d[:, None].float()
    see = d <= 0
    if s["see"] is not None:
        see = see | (j[None, None, :] < (pre + s["see"].long())[:, None, None])
    if c["window"]:
        see = see & (d > -c["window"])
    see = see & (j[None, None, :] < ctx[:, None, None])
    x = torch.where(see[:, None], x, -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)
    x = torch.exp(x - top)
    sums = x.sum(-1, keepdim=True)
    lse = (torch.log(sums) + top).squeeze(-1)                               # [R, Hq, N]
    v = _values(s, "v", blk, off).permute(0, 2, 1, 3)
    o = torch.matmul(x.reshape(R, H, G * N, L), v).reshape(R, Hq, N, D)
    o = o / torch.where(sums > 0, sums, 1.0)
    # back to the tokens' rows
    row = torch.searchsorted(start[1:], torch.arange(s["T"], device=DEV), right=True)
    n = torch.arange(s["T"], device=DEV) - start[row]
    return dict(lse=lse[row, :, n], out=o[row, :, n].to(s["q"].dtype))


# -------------------------------------------------------------------- work ----

def work(case):
    c = case
    if c["kind"] in ("swap", "load"):
        n = 2 * c["T"] * c["H"] * c["D"]
        if c["kind"] == "load":
            return {"bytes": n * (SIZE[c["cache"]] + 2) + 8 * c["T"], "flops": float(n)}
        # written, and read back
        return {"bytes": n * (2 + 2 * SIZE[c["cache"]] + 2) + 16 * c["T"], "flops": 3.0 * n}
    ctx, new, see, first, pre = _lengths(c)
    of = np.repeat(np.arange(len(pre) + 1), np.diff(np.concatenate([first, [c["R"]]])))
    keys = pairs = 0
    least = pre.copy()                       # per group: the first shared key that a row sees
    for r, (L, n, f) in enumerate(zip(ctx.tolist(), new.tolist(), see.tolist())):
        S = int(np.concatenate([pre, [0]])[of[r]])
        p = S + np.arange(L - n, L)
        hi = np.minimum(np.maximum(p + 1, S + f), S + L)
        lo = np.maximum(p - c["window"] + 1, 0) if c["window"] else np.zeros_like(p)
        pairs += int((hi - lo).sum())
        keys += int(hi.max() - max(lo.min(), S))
        if S:
            least[of[r]] = min(least[of[r]], lo.min())
    keys += int((pre - least).sum())
    kv = 2 * keys * c["H"] * c["D"] * SIZE[c["cache"]]
    io = int(new.sum()) * c["Hq"] * (4 * c["D"] + 4)
    return {"bytes": float(kv + io + 4 * keys // c["block"]), "flops": 4.0 * c["D"] * c["Hq"] * pairs}


# ------------------------------------------------------------------- exact ----

def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "swap":
        keep = (s["slot"] >= 0)[:, None, None]
        return {n: torch.where(keep, _exact_nearest(s[n], case["cache"]), 0.0) for n in "kv"}
    if case["kind"] == "load":
        return _exact_load(s)
    if work(case)["flops"] > 1.2e13:
        return None
    return _exact_attn(s)


def _exact_nearest(x, kind):
    """Every component's nearest value (ties to the even code) in its group's power, in 64 bits."""
    g = x.double().unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1, keepdim=True)
    big, half = (6.0, 1.0) if kind == "mx4" else (448.0, 16.0)
    least, most = _powers(x.dtype, kind == "mx4")
    # the least power whose largest value is half a step away at most
    e = torch.ceil(torch.log2(top / (big + half)))
    e = torch.where(top > (big + half) * torch.exp2(e), e + 1, e)
    e = torch.where(top <= (big + half) * torch.exp2(e - 1), e - 1, e).clamp(least, most)
    a = g / torch.exp2(e)
    # steps: of a value in [2^n, 2^(n + 1)) 2^(n - mantissa bits), n at least the smallest normal's
    bits, low = (1, 0) if kind == "mx4" else (3, -6)
    n = torch.frexp(a)[1] - 1
    step = torch.exp2((n.clamp(min=low) - bits).double())
    return (torch.round(a / step) * step).clamp(-big, big).mul(torch.exp2(e)).flatten(-2)


def _exact_values(s, name, blocks, offs, h):
    """Head h's components at places of the cache, in 64 bits, from the bits of the codes."""
    kind = s["case"]["cache"]
    x = s[name + "c"][blocks, offs, h]
    if kind in ("bf16", "f16"):
        return x.double()
    if kind == "fp8":
        return x.double() * s[name + "s"][h].double()
    b = x.view(torch.uint8).int()
    if kind == "mx4":
        b = torch.stack([b % 16, b // 16], -1).flatten(-2)
        sign, exponent, mantissa, bias, bits = b // 8, b // 2 % 4, b % 2, 1, 1
    else:
        sign, exponent, mantissa, bias, bits = b // 128, b // 8 % 16, b % 8, 7, 3
    m = mantissa.double() / 2 ** bits + (exponent > 0)
    y = m * torch.exp2((exponent.clamp(min=1) - bias).double()) * (1 - 2 * sign)
    power = torch.exp2(s[name + "e"][blocks, offs, h].double() - 127.0)
    return (y.unflatten(-1, (-1, GROUP)) * power[..., None]).flatten(-2)


def _exact_load(s):
    B, slot = s["case"]["block"], s["slot"]
    out = {}
    for name in "kv":
        rows = []
        for h in range(s["case"]["H"]):
            y = _exact_values(s, name, slot.clamp(min=0) // B, slot.clamp(min=0) % B, h)
            y[slot < 0] = 0.0
            rows.append(y)
        out[name] = torch.stack(rows, 1)
    return out


def _exact_attn(s):
    """Request by request and head by head of the keys, on the tokens the request has."""
    c = s["case"]
    G, B, D = c["Hq"] // c["H"], c["block"], c["D"]
    start, own_ctx, of, pre = (s[k].cpu().tolist() for k in ("start", "context", "of", "pre"))
    out = torch.zeros((s["T"], c["Hq"], D), dtype=torch.float64, device=DEV)
    lse = torch.zeros((s["T"], c["Hq"]), dtype=torch.float64, device=DEV)
    for r, L in enumerate(own_ctx):
        a, b, S = start[r], start[r + 1], pre[of[r]]
        j = torch.arange(S + L, device=DEV)
        ids = s["table"][r, : -(-L // B)].long()
        blocks = ids[torch.arange(L, device=DEV) // B]
        if S:
            ids = s["shared_table"][of[r], : -(-S // B)].long()
            blocks = torch.cat([ids[j[:S] // B], blocks])
        offs = torch.where(j < S, j, j - S) % B
        j = j.double()[None, :]
        p = torch.arange(S + L - (b - a), S + L, device=DEV, dtype=torch.float64)[:, None]
        hidden = j > p
        if s["see"] is not None:
            hidden &= j >= S + int(s["see"][r])
        if c["window"]:
            hidden |= p - j >= c["window"]
        for h in range(c["H"]):
            k, v = (_exact_values(s, n, blocks, offs, h) for n in "kv")
            z = torch.matmul(s["q"][a:b, h * G:(h + 1) * G].double().transpose(0, 1), k.T) / math.sqrt(D)
            if c["cap"]:
                z = c["cap"] * torch.tanh(z / c["cap"])
            if s["slopes"] is not None:
                z = z - s["slopes"][h * G:(h + 1) * G].double()[:, None, None] * (p - j)
            z = z.masked_fill(hidden, -math.inf)
            lse[a:b, h * G:(h + 1) * G] = torch.logsumexp(z, -1).T
            out[a:b, h * G:(h + 1) * G] = torch.matmul(torch.softmax(z, -1), v).transpose(0, 1)
    return dict(lse=lse, out=out)
