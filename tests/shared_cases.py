"""Requests behind shared prefixes: a Case whose last "requests" are the groups' prefixes."""
from __future__ import annotations

import copy

import numpy as np


class Shared:
    """sizes[g] requests of group g behind pre[g] shared tokens, after `before` requests without a
    group and before the rest.  `wide`: the prefixes' table has columns for a million tokens, so that
    small calls of single tokens are planned like large ones too."""

    wide = False

    def __init__(self, dev, ctx, new, sizes, pre, Hq, H, D, dtype="bf16", cache=None, before=0, **kw):
        import torch
        import paper_2607_16892_amd as dro
        from kv_cases import Case
        from mx_cases import mx_case
        all_ctx, all_new = list(ctx) + list(pre), list(new) + [0] * len(pre)
        if cache in ("mxfp4", "mxfp8"):
            c = mx_case(dev, cache, all_ctx, all_new, Hq, H, D, dtype, **kw)
        else:
            c = Case(dev, all_ctx, all_new, Hq, H, D, dtype, cache, **kw)
        R = self.R = len(ctx)
        self.case, self.pre, self.new = c, list(pre), list(new)
        self.first_h = before + np.concatenate([[0], np.cumsum(sizes)]).astype(int)
        assert self.first_h[-1] <= R
        self.of = [-1] * R
        for g in range(len(pre)):
            for r in range(self.first_h[g], self.first_h[g + 1]):
                self.of[r] = g
        first = torch.tensor(self.first_h, dtype=torch.int32, device=dev)
        most = max([sum(self.new[self.first_h[g]:self.first_h[g + 1]]) for g in range(len(pre))] + [0])
        table = c.table[R:]
        if self.wide:
            table = torch.full((len(pre), (1 << 20) // c.block), -1, dtype=torch.int32, device=dev)
            table[:, : c.table.shape[1]] = c.table[R:]
        self.shared = dro.SharedPrefixes(first, c.context[R:], table, most)

    def run(self, ctx, **kw):
        import paper_2607_16892_amd as dro
        c, R = self.case, self.R
        kw.setdefault("max_new", max(self.new + [0]))
        kw.setdefault("shared", self.shared)
        return dro.kv_shared_attention(ctx, c.cache, c.q, c.table[:R], c.start[: R + 1], c.context[:R], **kw)

    def total(self, r):
        return self.case.ctx[r] + (self.pre[self.of[r]] if self.of[r] >= 0 else 0)

    def check(self, got, prefix=None, **kw):
        """As Case.check, each request's keys being its prefix's, which all its rows see, and its own."""
        c, R = self.case, self.R
        view = copy.copy(c)
        view.ctx, view.new = [self.total(r) for r in range(R)], self.new

        def keys(r):
            own, g = c.keys(r), self.of[r]
            if g < 0:
                return own
            return [np.concatenate([s, o]) for s, o in zip(c.keys(R + g), own)]

        view.keys = keys
        prefix = [self.total(r) - c.ctx[r] + (0 if prefix is None else max(int(prefix[r]), 0)) for r in range(R)]
        view.check(got, prefix=prefix, **kw)
