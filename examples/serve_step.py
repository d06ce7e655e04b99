"""A serving loop on the reservations: blocks, cache and attention of every step.

Requests of the synthetic serving workload's classes arrive with their inputs, reserve
L_in + eta* tokens each (eta* of the worst-case table, or the class mean), bring their
prompts in chunks, decode a token a step and end at their output length.  Each step is
one kv_block_tables for the batch and, per layer, kv_store and kv_attention.  The model
around them is two random layers of projections, so the tokens mean nothing; what it
shows is how the calls fit together, and how often a policy's requests have to wait for
blocks.

With --share the L_pre shared tokens of each class are held once: a row of the table of their
own brings them like a request, and the class's requests, which lie next to one another in the
batch, follow them by kv_shared_attention.

    python examples/serve_step.py [--steps 200] [--policy dro|mean] [--cache bf16|fp8|mxfp8|mxfp4] [--share]
"""
from __future__ import annotations

import argparse
import os
import sys

import numpy as np
import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2607_16892_amd as dro  # noqa: E402
from workloads.configs import serving_workload  # noqa: E402

HEADS, KV_HEADS, DIM, LAYERS, CHUNK = 32, 8, 128, 2, 512


class Layers:
    """Random projections of a residual stream: q, k, v out of one product, and back."""

    def __init__(self, dev, dtype, seed):
        g = torch.Generator(device=dev).manual_seed(seed)
        width = HEADS * DIM

        def weight(*shape):
            return (torch.randn(shape, generator=g, device=dev) * width ** -0.5).to(dtype)

        self.qkv = [weight(width, (HEADS + 2 * KV_HEADS) * DIM) for _ in range(LAYERS)]
        self.back = [weight(width, width) for _ in range(LAYERS)]
        self.embed = weight(4096, width) * width ** 0.5

    def step(self, ctx, caches, x, pool, plan, max_new, shared=None):
        for cache, qkv, back in zip(caches, self.qkv, self.back):
            y = (x @ qkv).view(-1, HEADS + 2 * KV_HEADS, DIM)
            dro.kv_store(ctx, cache, y[:, HEADS:HEADS + KV_HEADS], y[:, HEADS + KV_HEADS:], plan["slot"])
            rows = (ctx, cache, y[:, :HEADS], pool.table, plan["start"], plan["context"], max_new)
            o = (dro.kv_attention(*rows, want_lse=False) if shared is None else
                 dro.kv_shared_attention(*rows, shared, want_lse=False))["out"]
            x = x + o.flatten(1) @ back
        return x


def reservations(ctx, w, dev, policy):
    """Tokens reserved beyond the input, per class."""
    prob = dro.Problem.from_workload(w, dev)
    if policy == "mean":
        m = dro.class_moments(ctx, prob)
        return dro.dro_baseline_reservations(ctx, m, prob.L)["mean"].cpu().numpy()
    eps = torch.from_numpy(np.ascontiguousarray(w.eps[: w.C], np.float32)).to(dev)
    k = dro.dro_exact_table(ctx, prob, eps)["k_star"][0]
    return prob.eta[k.long()].cpu().numpy()


def serve(dev="cuda:0", steps=200, policy="dro", cache="bf16", slots=48, blocks=3600, block=16, seed=0,
          collect=None, share=False):
    """Runs the loop; returns counts.  collect(step, x): called with the rows' outputs."""
    r = np.random.default_rng(seed)
    dev = torch.device(dev)
    w, svc = serving_workload(C=6, N=5000, K=513, M=64, L=1024, seed=seed)
    most = -(-(int(svc.Lin.max()) + 1024) // block)
    dtype = torch.bfloat16
    done = waits = tokens = 0
    with dro.Context(dev.index or 0) as ctx:
        eta = reservations(ctx, w, dev, policy)
        layers = Layers(dev, dtype, seed)
        kind = {"fp8": torch.float8_e4m3fn, "bf16": dtype}.get(cache, cache)
        scale = torch.full((KV_HEADS,), 0.05, device=dev)
        caches = [dro.KvCache.empty(blocks, block, KV_HEADS, DIM, kind, dev,
                                    *((scale, scale) if cache == "fp8" else ()))
                  for _ in range(LAYERS)]
        # a row of the table for each slot, and behind them one for each prefix that is shared
        groups = w.C if share else 0
        rows = slots + groups
        pool = dro.BlockPool.empty(rows, most, blocks, block, dev)
        held, target, prompt, want = (np.zeros(rows, np.int64) for _ in range(4))
        live = np.zeros(rows, bool)
        edges = np.arange(groups + 1) * slots // max(groups, 1)  # the slots of each group
        first = torch.from_numpy(edges.astype(np.int32)).to(dev)
        if share:
            live[slots:], target[slots:] = True, 1 << 40
            prompt[slots:] = want[slots:] = svc.Lpre
        for step in range(steps):
            for i in np.flatnonzero(~live)[: 1 + step % 3]:      # arrivals
                c = int(r.integers(w.C))
                own = svc.Lin[c]
                if share:                                        # a slot of its class, behind its prefix
                    free_slots = np.flatnonzero(~live[edges[c]:edges[c + 1]])
                    if held[slots + c] < prompt[slots + c] or not len(free_slots):
                        continue
                    i, own = edges[c] + free_slots[0], svc.Lin[c] - svc.Lpre[c]
                live[i], held[i], prompt[i] = True, 0, own
                target[i] = own + r.choice(w.samples_of(c))
                want[i] = own + eta[c]
            over = live & (held >= target)                       # ended: their blocks go back
            add = np.where(live, np.where(held < prompt, np.minimum(prompt - held, CHUNK), 1), 0)
            add[slots:][held[slots:] >= prompt[slots:]] = 0      # a prefix that is whole brings nothing more
            add[over] = -1
            T = int(np.maximum(add, 0).sum())
            i32 = [torch.from_numpy(x.astype(np.int32)).to(dev) for x in (held, add, want)]
            plan = pool.take(dro.kv_block_tables(ctx, pool, i32[0], i32[1], T, reserve=i32[2]))
            x = layers.embed[torch.from_numpy(r.integers(0, 4096, T)).to(dev)]
            new = np.maximum(add, 0)
            shared = dro.SharedPrefixes(first, plan["context"][slots:], pool.table[slots:],
                                        int(max(new[a:b].sum() for a, b in zip(edges, edges[1:])))) if share else None
            x = layers.step(ctx, caches, x, pool, plan, int(add.max(initial=0)), shared)
            if collect:
                collect(step, x)
            granted = plan["granted"].cpu().numpy().astype(bool)
            waits += int((live & ~over & ~granted).sum())
            tokens += int(new[granted].sum())
            done += int(over.sum())
            held = np.where(over, 0, held + np.where(granted, new, 0))
            live &= ~over
        free = int(pool.free.item())
        in_use = int(pool.held.sum().item())
    return dict(policy=policy, steps=steps, tokens=tokens, ended=done, waits=waits, free=free, in_use=in_use,
                blocks=blocks)


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--policy", choices=("dro", "mean"), default="dro")
    ap.add_argument("--cache", choices=("bf16", "fp8", "mxfp8", "mxfp4"), default="bf16")
    ap.add_argument("--share", action="store_true", help="hold each class's shared prefix once")
    a = ap.parse_args()
    out = serve(steps=a.steps, policy=a.policy, cache=a.cache, share=a.share)
    print("{policy}: {tokens} tokens in {steps} steps, {ended} requests ended, {waits} waits for blocks, "
          "{in_use} of {blocks} blocks in use".format(**out))
