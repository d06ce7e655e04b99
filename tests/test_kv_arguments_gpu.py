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
