"""The serving loop of examples/serve_step.py: every step's rows against fp64 attention over
the tokens that its requests have stored, and the pool's accounting."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _example():
    spec = importlib.util.spec_from_file_location("serve_step", os.path.join(ROOT, "examples", "serve_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("policy", ["dro", "mean"])
@pytest.mark.parametrize("cache", ["bf16", "fp8"])
def test_the_loop_keeps_its_blocks(dev, policy, cache):
    import torch
    m = _example()
    seen = []
    out = m.serve(str(dev), steps=60, policy=policy, cache=cache, slots=16, blocks=700,
                  collect=lambda step, x: seen.append(bool(torch.isfinite(x).all())))
    print(f"[gpu] serve {out}", flush=True)
    assert out["tokens"] > 500 and all(seen) and len(seen) == 60
    assert out["free"] + out["in_use"] == out["blocks"]


def test_a_loop_whose_pool_is_small_waits(dev):
    out = _example().serve(str(dev), steps=60, slots=16, blocks=150)
    assert out["waits"] > 0 and out["free"] + out["in_use"] == 150


def test_layers_equal_plain_attention(dev):
    """Three requests through chunks and single tokens: the second layer's rows agree with
    attention over each request's own keys and values, kept apart in fp32."""
    import torch
    import paper_2607_16892_amd as dro
    m = _example()
    H, K, D = m.HEADS, m.KV_HEADS, m.DIM
    layers = m.Layers(dev, torch.bfloat16, 3)
    with dro.Context(dev.index or 0) as ctx:
        caches = [dro.KvCache.empty(64, 16, K, D, device=dev) for _ in range(m.LAYERS)]
        pool = dro.BlockPool.empty(3, 20, 64, 16, dev)
        kept = [[([], []) for _ in range(3)] for _ in range(m.LAYERS)]
        held = [0, 0, 0]
        g = torch.Generator(device=dev).manual_seed(1)
        for add in ([40, 7, 0], [33, 1, 100], [1, 1, 1], [1, 1, 1], [5, 0, 1]):
            i32 = [torch.tensor(x, dtype=torch.int32, device=dev) for x in (held, add)]
            T = sum(add)
            plan = pool.take(dro.kv_block_tables(ctx, pool, i32[0], i32[1], T))
            assert plan["granted"].tolist() == [1, 1, 1]
            x = torch.randn((T, H * D), generator=g, device=dev).to(torch.bfloat16)
            y = layers.step(ctx, caches, x, pool, plan, max(add))
            z = x
            for li in range(m.LAYERS):
                p = (z @ layers.qkv[li]).view(T, H + 2 * K, D)
                outs = []
                at = 0
                for r, n in enumerate(add):
                    q = p[at:at + n, :H].float()
                    kept[li][r][0].append(p[at:at + n, H:H + K].float())
                    kept[li][r][1].append(p[at:at + n, H + K:].float())
                    at += n
                    k, v = (torch.cat(s).repeat_interleave(H // K, 1) for s in kept[li][r])
                    L = len(k)
                    s = torch.einsum("qhd,khd->hqk", q, k) * D ** -0.5
                    i = torch.arange(L - n, L, device=dev)
                    s = s.masked_fill(torch.arange(L, device=dev)[None, None, :] > i[None, :, None], -torch.inf)
                    outs.append(torch.einsum("hqk,khd->qhd", torch.softmax(s, -1), v))
                z = z + torch.cat(outs).reshape(T, -1).to(torch.bfloat16) @ layers.back[li]
            # two bf16 attentions and four bf16 roundings of values of order one apart
            assert (y.float() - z.float()).abs().max() <= 0.06
            held = [h + n for h, n in zip(held, add)]
