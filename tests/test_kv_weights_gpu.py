"""The 16-bit weights of kv_attention where most of them are small."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(dev):
    import paper_2607_16892_amd as dro
    c = dro.Context(dev.index or 0)
    yield c
    c.close()


@pytest.mark.parametrize("R,new", [(3072, 1), (512, 128)])      # both kernels, no item cut
@pytest.mark.parametrize("L,nats", [(131_072, 14.5), (131_072, 17.3), (60_000, 16.0), (60_000, 12.0)])
def test_f16_a_long_flat_tail_beside_one_key(ctx, dev, R, new, L, nats):
    """The first key's score lies `nats` above those of a long, nearly flat tail whose values have
    a mean: the tail's weights, small as they are, count in the values' sum as in the weights'.

    With A = sum of weights times |v|: weights and outputs rounded to f16 2 u A; a lane adds at
    most L / 4 weights, and a value's sum takes as many products one after the other, (L / 4 + 8)
    2^-24 of each; scores as in kv_cases; a weight below f16's normal numbers is off by 2^-25 of
    its unit, and the largest is at least 2^7 units: L 2^-32 max |v|."""
    import torch
    import paper_2607_16892_amd as dro
    D, B = 64, 16
    print(f"[gpu] kv weights R={R} new={new} L={L} nats={nats}", flush=True)
    g = torch.Generator().manual_seed(L + int(10 * nats))
    k = torch.randn((L, D), generator=g)
    k[:, 0] = 0.0
    k[0] = 0.0
    k[0, 0] = nats
    v = 1.0 + 0.1 * torch.randn((L, D), generator=g)
    v[0] = 0.0
    T = R * new
    q = 0.05 * torch.randn((T, D), generator=g)
    q[:, 0] = 8.0                                       # scale 1 / 8: the first key's score is nats
    k, v, q = k.half(), v.half(), q.half()
    nb = -(-L // B)
    pool = [torch.zeros((nb * B, D), dtype=torch.float16) for _ in range(2)]
    pool[0][:L], pool[1][:L] = k, v
    cache = dro.KvCache(*(x.view(nb, B, 1, D).to(dev) for x in pool))
    table = torch.arange(nb, dtype=torch.int32, device=dev).repeat(R, 1)      # all read the same blocks
    start = torch.arange(0, T + 1, new, dtype=torch.int32, device=dev)
    context = torch.full((R,), L, dtype=torch.int32, device=dev)
    got = dro.kv_attention(ctx, cache, q.view(T, 1, D).to(dev), table, start, context, new)
    torch.cuda.synchronize()
    u = 2.0 ** -11
    kd, vd = k.double(), v.double()
    for t in sorted({0, 1, new - 1, T // 2, T - new, T - 1}):
        see = L - new + t % new + 1
        s = kd[:see] @ q[t].double() * 0.125
        w = torch.softmax(s, 0)
        ref, A = w @ vd[:see], w @ vd[:see].abs()
        ds = (D + 4) * 2.0 ** -24 * 0.125 * (kd[:see].abs() @ q[t].double().abs()).max() \
            + 4 * 2.0 ** -23 * (s.abs().max() + 1)
        tol = (2 * u + torch.expm1(2 * ds) + 2 * (L / 4 + 8) * 2.0 ** -24) * A + L * 2.0 ** -32 * vd.abs().max()
        err = (got["out"][t, 0].double().cpu() - ref).abs()
        assert (err <= tol).all(), f"row {t}: {(err / tol).max().item():.3g} of the bound"
        lse = torch.logsumexp(s, 0).item()
        assert abs(got["lse"][t, 0].item() - lse) <= float(ds) + (L / 4 + 8) * 2.0 ** -24 + 2.0 ** -21 * (1 + abs(lse))


@pytest.mark.parametrize("new", [1, 40])
@pytest.mark.parametrize("exponent", [10, 20, 23, 24, 26])
def test_f16_weights_of_large_scores_stay_in_range(ctx, dev, new, exponent):
    """Scores up to 2^exponent, whose last places are many units wide then, ascending with the
    key: no weight passes f16's largest number.  From 2^20 on neighbours are 2^10 and more apart,
    so a row's last key takes it (weight and output rounded: 2 u |v|)."""
    import torch
    from kv_cases import Case
    N = new + 300
    c = Case(dev, [N], [new], 4, 2, 64, "f16", seed=exponent)
    j = torch.arange(N)
    ids, at = c.table_h[0, j // 16].long(), j % 16
    c.k_h[ids, at] = 0.0
    c.k_h[ids, at, :, 0] = ((0.5 + j / 1024.0) * 2.0 ** (exponent // 2)).half()[:, None]
    c.q_h[:] = 0.0
    c.q_h[:, :, 0] = 2.0 ** (exponent - exponent // 2)
    c.k.copy_(c.k_h.to(dev)), c.q.copy_(c.q_h.to(dev))
    got = c.run(ctx, scale=1.0)
    assert torch.isfinite(got["out"]).all() and torch.isfinite(got["lse"]).all()
    if exponent >= 20:
        last = N - new + torch.arange(new)
        v = c.v_h[ids[last], at[last]].repeat_interleave(2, 1).double()
        assert ((got["out"].cpu().double() - v).abs() <= 2 * 2.0 ** -11 * v.abs()).all()
