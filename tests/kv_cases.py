"""Small paged caches with requests of given lengths, and the comparison with the oracle."""
from __future__ import annotations

import math

import numpy as np

from oracle import kv as okv

UNIT = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}      # unit roundoff of the 16-bit types


def dtypes():
    import torch
    return {"bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.float8_e4m3fn}


class Case:
    """Requests of context ctx[r] tokens whose last new[r] are the rows, blocks in random order."""

    def __init__(self, dev, ctx, new, Hq, H, D, dtype="bf16", cache=None, block=16, seed=0,
                 layout="heads", fused=True, spare=2, scale_q=1.0):
        import torch
        import paper_2607_16892_amd as dro
        cache = cache or dtype
        g = torch.Generator().manual_seed(seed)
        self.dev, self.dtype, self.cache_type, self.block = dev, dtype, cache, block
        self.ctx, self.new, self.Hq, self.H, self.D = list(ctx), list(new), Hq, H, D
        R = len(self.ctx)
        nblk = [-(-c // block) for c in self.ctx]
        nb = sum(nblk) + 3
        W = max(nblk) + spare
        order = torch.randperm(nb, generator=g).to(torch.int32)
        table = torch.full((R, W + 3), -1, dtype=torch.int32)      # wider rows: strided table
        at = 0
        for r, n in enumerate(nblk):
            table[r, :n] = order[at:at + n]
            at += n
        dt = dtypes()
        kv = []
        for _ in range(2):
            shape = (nb, H, block, D) if layout == "heads" else (nb, block, H, D)
            x = torch.randn(shape, generator=g)
            x = x.permute(0, 2, 1, 3) if layout == "heads" else x
            kv.append(x.to(dt[cache]) if cache != "fp8" else (x * 20).to(dt[cache]))
        self.ks = self.vs = None
        if cache == "fp8":
            self.ks, self.vs = (torch.rand(H, generator=g) * 0.05 + 0.02 for _ in range(2))
        T = sum(self.new)
        self.T = T
        q = (torch.randn((T + 1, Hq + (2 * H if fused else 0), D), generator=g) * scale_q).to(dt[dtype])
        self.k_h, self.v_h, self.q_h, self.table_h = kv[0], kv[1], q[:T, :Hq], table[:, :W]
        self.k, self.v = (self._put(x) for x in kv)
        self.q = q.to(dev)[:T, :Hq]
        self.table = table.to(dev)[:, :W]
        self.start = torch.tensor(np.concatenate([[0], np.cumsum(self.new)]), dtype=torch.int32).to(dev)
        self.context = torch.tensor(self.ctx, dtype=torch.int32).to(dev)
        self.cache = dro.KvCache(self.k, self.v, *(None if s is None else s.to(dev)
                                                   for s in (self.ks, self.vs)))

    def _put(self, x):
        # keeps the strides of the host tensor
        import torch
        y = torch.empty_strided(x.shape, x.stride(), dtype=x.dtype, device=self.dev)
        y.copy_(x.to(self.dev))
        return y

    def keys(self, r):
        """The request's keys and values in fp64, as the cache holds them."""
        ids = self.table_h[r, : -(-self.ctx[r] // self.block)].long()
        out = []
        for x, s in ((self.k_h, self.ks), (self.v_h, self.vs)):
            y = x.float()[ids].reshape(-1, self.H, self.D)[: self.ctx[r]].double().numpy()
            out.append(y if s is None else y * s.double().numpy()[None, :, None])
        return out

    def run(self, ctx, **kw):
        import paper_2607_16892_amd as dro
        kw.setdefault("max_new", max(self.new + [0]))
        return dro.kv_attention(ctx, self.cache, self.q, self.table, self.start, self.context, **kw)

    def check(self, got, softcap=0.0, window=0, slopes=None, prefix=None, scale=None, rows=None):
        """Element by element within the bound that the formats and fp32 sums allow.

        u: unit roundoff of the 16-bit type; A = sum of weights times |v|.
          weights rounded to 16 bits, and the output: 2 u A (f16 weights below 2^-14 of the
            largest lose at most 2^-25 each: L 2^-25 max |v|)
          scores: fp32 products and sums of D terms, at most (D + 4) 2^-24 sum |q k| scale;
            the cap's tanh 2^-21 cap; the bias and the exponent's argument, rounded in fp32
            to 2^-23 of the largest |s| each: ds in all, which moves a weight by e^(2 ds) - 1
          sums of L weights and products in fp32: (L + 8) 2^-24 A
        """
        u = UNIT[self.dtype]
        out, lse = got["out"].float().cpu().double().numpy(), got["lse"].double().cpu().numpy()
        scale = self.D ** -0.5 if scale is None else scale
        s_h = None if slopes is None else slopes.cpu().numpy()
        for r in range(len(self.ctx)) if rows is None else rows:
            a, n, L = int(self.start[r]), self.new[r], self.ctx[r]
            if n == 0:
                continue
            k, v = self.keys(r)
            ref = okv.attention(self.q_h[a:a + n].double().numpy(), k, v, L, scale, softcap, window,
                                s_h, 0 if prefix is None else int(prefix[r]))
            ds = ((self.D + 4) * 2.0 ** -24 * ref["dots"] + 2.0 ** -21 * softcap
                  + 4 * 2.0 ** -23 * (ref["tops"] + 1))
            A = ref["mass"]
            vmax = np.abs(v[np.isfinite(v)]).max() if L else 0.0
            tol = (2 * u + np.expm1(2 * ds)[..., None] + (L + 8) * 2.0 ** -24) * A \
                + L * 2.0 ** -25 * vmax + 2.0 ** -24
            err = np.abs(out[a:a + n] - ref["out"])
            assert np.isfinite(out[a:a + n]).all(), f"request {r}: not finite"
            bad = err > tol
            assert not bad.any(), (f"request {r} (context {L}, rows {n}): {bad.sum()} of {bad.size} "
                                   f"beyond the bound, worst {np.max(err / tol):.3g} of it at "
                                   f"{np.unravel_index(np.argmax(err / tol), err.shape)}")
            empty = ~np.isfinite(ref["lse"])
            assert (lse[a:a + n][empty] == -math.inf).all() and (out[a:a + n][empty] == 0).all()
            e = np.abs(lse[a:a + n][~empty] - ref["lse"][~empty])
            lim = (ds + (L + 8) * 2.0 ** -24 + 2.0 ** -21 * (1 + ref["tops"]))[~empty]
            assert (e <= lim).all(), f"request {r}: lse off by {np.max(e / lim):.3g} of the bound"
