"""Captured paged-cache calls beside calls that need a larger workspace."""
import pytest

from kv_cases import Case

pytestmark = pytest.mark.gpu


def test_replays_after_the_workspace_has_grown(dev):
    """A decode step and its block tables are captured; then prompts that need more workspace run
    on the same context, and other memory is allocated and written.  The replays are right."""
    import torch
    import paper_2607_16892_amd as dro
    with dro.Context(dev.index or 0) as ctx:
        c = Case(dev, [5000, 33, 900], [1, 1, 1], 8, 2, 128, seed=1)
        ref = c.run(ctx)
        i32 = dict(dtype=torch.int32, device=dev)
        pool = dro.BlockPool.empty(3, 400, 1000, 16, dev)
        length, add = torch.tensor([0, 40, 7], **i32), torch.tensor([5000, 33, 900], **i32)
        table, stack = pool.table.clone(), pool.free_list.clone()
        plan = dro.kv_block_tables(ctx, pool, length, add, 5933)
        ref_table, ref_plan = pool.table.clone(), {k: v.clone() for k, v in plan.items()}
        out, lse = torch.zeros_like(ref["out"]), torch.zeros_like(ref["lse"])
        torch.cuda.synchronize()
        s = torch.cuda.Stream(dev)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            c.run(ctx, out=out, lse=lse)
            dro.kv_block_tables(ctx, pool, length, add, 5933, out=plan)
        for T in (300, 3000, 20_000):                    # 67 MB of parts where the step has 34
            p = Case(dev, [T], [T], 8, 8, 128, seed=T)
            big = p.run(ctx)
            torch.cuda.synchronize()
            other = [torch.full((1 << 24,), 0x7fc0dead, **i32) for _ in range(8)]      # 512 MB, NaN as floats
            pool.table.copy_(table), pool.free_list.copy_(stack)
            for t in (out, lse, *plan.values()):
                t.fill_(9)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, ref["out"]) and torch.equal(lse, ref["lse"])
            assert torch.equal(pool.table, ref_table)
            for k, v in ref_plan.items():
                assert torch.equal(plan[k], v), k
            assert all((o == 0x7fc0dead).all() for o in other)
            again = p.run(ctx)
            assert torch.equal(again["out"], big["out"]) and torch.equal(again["lse"], big["lse"])
            del other, p, big, again


def test_a_capture_that_has_to_grow_the_workspace_is_refused(dev):
    """The error leaves the capture as it was: what else it records replays, and the call itself
    can be captured after one call of its size."""
    import torch
    import paper_2607_16892_amd as dro
    c = Case(dev, [700, 90], [300, 1], 8, 2, 128, seed=4)
    with dro.Context(dev.index or 0) as other:
        ref = c.run(other)
    with dro.Context(dev.index or 0) as ctx:
        out, lse = torch.full_like(ref["out"], 7.0), torch.full_like(ref["lse"], 7.0)
        x = torch.zeros(5, device=dev)
        torch.cuda.synchronize()
        s = torch.cuda.Stream(dev)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            x += 1
            with pytest.raises(dro.DroError) as e:
                c.run(ctx, out=out, lse=lse)
        assert e.value.code == -4
        for n in (1, 2):
            graph.replay()
            torch.cuda.synchronize()
            assert (x == n).all() and (out == 7).all() and (lse == 7).all()
        c.run(ctx, out=out, lse=lse)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            c.run(ctx, out=out, lse=lse)
        for _ in range(3):
            out.fill_(7), lse.fill_(7)
            torch.cuda.synchronize()
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, ref["out"]) and torch.equal(lse, ref["lse"])
