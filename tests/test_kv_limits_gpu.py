"""The paged cache at the limits of its sizes."""
import pytest

pytestmark = pytest.mark.gpu


def test_rows_that_claim_more_blocks_than_31_bits_count(dev):
    """All of 2^20 requests end and claim 2047 blocks each beside an almost full stack: its free
    places and the rows' claims pass 2^31 together, and only the three places left are written."""
    import torch
    import paper_2607_16892_amd as dro
    R, W, B = 1 << 20, 2047, 16
    nb = (2 ** 31 - 1) // B
    i32 = dict(dtype=torch.int32, device=dev)
    print(f"[gpu] kv tables R={R} W={W} blocks={nb}", flush=True)
    table = torch.full((R, W), 5, **i32)
    table[0, :3] = torch.tensor([11, 12, 13], **i32)
    stack = torch.arange(nb, **i32)
    pool = dro.BlockPool(B, table, torch.full((R,), W, **i32), stack, torch.tensor([nb - 3], **i32))
    want = stack.clone()
    want[-3:] = torch.tensor([11, 12, 13], **i32)
    with dro.Context(dev.index or 0) as ctx:
        got = dro.kv_block_tables(ctx, pool, torch.zeros(R, **i32), torch.full((R,), -1, **i32), 0)
        torch.cuda.synchronize()
    assert torch.equal(stack, want)
    assert got["free"].item() == nb and (got["held"] == 0).all() and (got["granted"] == 0).all()
    assert (table[1:] == 5).all()
