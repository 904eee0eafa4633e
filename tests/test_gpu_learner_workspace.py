"""What the learner's operators allocate, and when."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("count", [8448, 8449, 30_000])
def test_no_list_outgrows_the_first_workspace(count):
    """After one norm of any list, a norm and a clip of thousands of tensors can be captured: nothing is
    allocated or synchronised.  The sums stay right where the launches' grids shrink (8,449 tensors)."""
    from paper_2604_21428_b200 import ddmerge as dd
    ctx = dd.Context(0)
    gen = torch.Generator(device="cuda").manual_seed(count)
    sizes = torch.randint(0, 40, (count,), generator=torch.Generator().manual_seed(1)).tolist()
    flat = torch.randn(sum(sizes) + 3_000_000, generator=gen, device="cuda")
    sizes[-1] += 3_000_000                                       # more tiles than any grid in one launch
    grads = list(flat[: sum(sizes)].split(sizes))
    out = [torch.zeros_like(g) for g in grads[:1]]
    record = dd.new_grad_record()
    ctx.grad_norm(out, 1.0, record)                              # the workspace
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.grad_norm(grads, 1.0, record)
    graph.replay()
    r = dd.read_grad_record(record)
    want = float(torch.cat(grads).double().square().sum())
    assert r.status == dd.STATUS_OK and abs(r.norm_sq - want) <= 34 * 2.0 ** -24 * want
    first = record.clone()
    ctx.grad_norm(grads, 1.0, record)
    assert torch.equal(first.view(torch.int32), record.view(torch.int32))
    before = torch.cat(grads)
    ctx.clip_gradients(grads, 1.0, record)
    scaled = before.double() * float(dd.read_grad_record(record).scale)
    assert bool(((torch.cat(grads).double() - scaled).abs() <= 2.0 ** -24 * scaled.abs()).all())
    del graph
    ctx.close()
