"""Arguments of the paged-cache binding at and beyond the ends of what they can be."""
import pytest

from kv_cases import Case

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx(dev):
    import paper_2607_16892_amd as dro
    c = dro.Context(dev.index or 0)
    yield c
    c.close()


@pytest.mark.parametrize("new", [1, 40])
def test_numbers_beyond_32_bits(ctx, dev, new):
    """A window or a bound of more than 32 bits means what it says, not its low 32 bits."""
    import torch
    import paper_2607_16892_amd as dro
    c = Case(dev, [new + 90, new], [new, new], 4, 2, 128, seed=new)
    ref = c.run(ctx)
    assert not torch.equal(c.run(ctx, window=16)["out"], ref["out"])
    for kw in (dict(window=2 ** 31 - 1), dict(window=2 ** 31), dict(window=2 ** 32 + 16), dict(window=2 ** 80 + 16),
               dict(max_new=2 ** 31), dict(max_new=2 ** 32 + new), dict(max_new=2 ** 32)):
        got = c.run(ctx, **kw)
        c.check(got)
        if "window" in kw:
            assert torch.equal(got["out"], ref["out"]) and torch.equal(got["lse"], ref["lse"]), kw
    for kw in (dict(window=-2 ** 32), dict(max_new=-2 ** 32)):
        with pytest.raises(dro.DroError) as e:
            c.run(ctx, **kw)
        assert e.value.code == -1
    pool = dro.BlockPool.empty(2, 8, 20, 16, dev)
    pool.block = 2 ** 32 + 16
    one = torch.ones(2, dtype=torch.int32, device=dev)
    with pytest.raises(dro.DroError):
        dro.kv_block_tables(ctx, pool, one, one, 2)


def test_inputs_that_require_grad_are_refused(ctx, dev):
    """There is no backward pass, so no gradient is dropped in silence; without gradients recorded
    the same tensors are taken."""
    import torch
    import paper_2607_16892_amd as dro
    c = Case(dev, [50, 60], [1, 20], 4, 2, 128, seed=3)
    slopes = torch.zeros(4, device=dev, requires_grad=True)
    ref = c.run(ctx, slopes=slopes.detach())
    slot = torch.arange(3, device=dev)
    x = torch.ones((3, 2, 128), dtype=torch.bfloat16, device=dev)
    grad = x.clone().requires_grad_()
    out = torch.full_like(ref["out"], 7.0)
    before = c.k.clone(), c.v.clone()
    for k, v in ((grad, x), (x, grad)):
        with pytest.raises(RuntimeError, match="no backward"):
            dro.kv_store(ctx, c.cache, k, v, slot)
    with pytest.raises(RuntimeError, match="no backward"):
        c.run(ctx, slopes=slopes, out=out)
    q = c.q
    c.q = q.clone().requires_grad_()
    with pytest.raises(RuntimeError, match="no backward"):
        c.run(ctx, out=out)
    torch.cuda.synchronize()
    assert (out == 7).all() and torch.equal(c.k, before[0]) and torch.equal(c.v, before[1])
    for off in (torch.no_grad(), torch.inference_mode()):
        with off:
            got = c.run(ctx, slopes=slopes)
            assert torch.equal(got["out"], ref["out"]) and torch.equal(got["lse"], ref["lse"])
    with torch.no_grad():
        dro.kv_store(ctx, c.cache, grad, grad, torch.full((3,), -1, device=dev))
    c.q = c.q.detach()
    got = c.run(ctx, slopes=slopes.detach())
    assert torch.equal(got["out"], ref["out"])


@pytest.mark.parametrize("T", [0, 1, 700, 5000])
def test_a_step_without_requests(ctx, dev, T):
    """R = 0: the pool stays as it is, every token is without a slot, every row zero."""
    import torch
    import paper_2607_16892_amd as dro
    none = torch.empty(0, dtype=torch.int32, device=dev)
    pool = dro.BlockPool.empty(0, 8, 20, 16, dev)
    pool.free.fill_(7)
    stack = pool.free_list.clone()
    plan = dro.kv_block_tables(ctx, pool, none, none, T, reserve=none)
    assert plan["free"].tolist() == [7] and plan["start"].tolist() == [0]
    assert (plan["slot"] == -1).all() and (plan["pos"] == -1).all() and len(plan["slot"]) == T
    assert torch.equal(pool.free_list, stack) and len(pool.take(plan)["held"]) == 0
    cache = dro.KvCache.empty(20, 16, 2, 64, device=dev)
    cache.k.fill_(float("nan")), cache.v.fill_(float("nan"))
    for most in (0, 1, 500):
        out = torch.full((T, 4, 64), 7.0, dtype=torch.bfloat16, device=dev)
        got = dro.kv_attention(ctx, cache, torch.ones_like(out), pool.table, plan["start"], plan["context"],
                               most, out=out)
        assert (out == 0).all() and (got["lse"] == -torch.inf).all()
    torch.cuda.synchronize()


def test_a_context_of_another_device_is_refused(dev):
    import torch
    import paper_2607_16892_amd as dro
    c = Case(dev, [50, 60], [1, 20], 4, 2, 128, seed=3)
    pool = dro.BlockPool.empty(2, 8, 20, 16, dev)
    one = torch.ones(2, dtype=torch.int32, device=dev)
    x = torch.ones((3, 2, 128), dtype=torch.bfloat16, device=dev)
    with dro.Context(dev.index or 0) as ctx:
        ctx.device = torch.device("cuda", 7)         # as if it had been made there
        with pytest.raises(ValueError, match="context"):
            c.run(ctx)
        with pytest.raises(ValueError, match="context"):
            dro.kv_store(ctx, c.cache, x, x, torch.arange(3, device=dev))
        with pytest.raises(ValueError, match="context"):
            dro.kv_block_tables(ctx, pool, one, one, 2)
        ctx.device = torch.device("cuda")            # the first one
        c.check(c.run(ctx))
