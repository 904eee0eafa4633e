"""The decoder's operators past 2^31 elements, and calls that run beside one another."""
import pytest
import torch

from decoder_util import B, UB, loss64, loss_back64, within
from test_gpu_rotary import turned64
from test_gpu_vocab_loss import Case as Loss

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def dd():
    from paper_2604_21428_b200 import ddmerge
    return ddmerge


@pytest.fixture(scope="module")
def ctx(dd):
    c = dd.Context(0)
    yield c
    c.close()


@pytest.fixture(autouse=True)
def room():
    yield
    torch.cuda.empty_cache()


def test_rotary_of_many_elements(dd, ctx):
    """More than 2^31 elements, in place: rows of both ends and of where offsets pass 2^31 and 2^32 bytes."""
    T, heads, dim = (1 << 22) + 3, 4, 128
    x = torch.ones(T, heads, dim, dtype=B, device="cuda")
    rows = torch.tensor([0, 1, (1 << 21) - 1, 1 << 21, (1 << 22) - 1, 1 << 22, T - 1], device="cuda")
    x[rows] = torch.randn(len(rows), heads, dim, device="cuda").to(B)
    positions, (f, _) = torch.arange(T, device="cuda", dtype=torch.int32), dd.rotary_frequencies(dim)
    before = x[rows]
    ctx.rotary(x, None, positions, f)
    want, e = turned64(before, positions[rows], f, 1.0, False, False)
    within(x[rows], want, e * (1 + UB) + UB * want.abs(), "rows")


@pytest.mark.parametrize("order", ["tokens apart", "heads apart"])
def test_attention_in_wide_strides(ctx, order):
    """Rows 2^23 elements apart, or heads 2^26: the bits that compact tensors give."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    T, heads, kv, dim = (300, 2, 1, 64) if order == "tokens apart" else (200, 36, 36, 64)
    shapes = [heads, kv, kv, heads, heads, heads, kv, kv]                     # q, k, v, d_o, o, dq, dk, dv
    if order == "tokens apart":
        buf = torch.empty(T, 1 << 23, dtype=B, device="cuda")
        wide, at = [], 0
        for n in shapes:
            wide.append(buf[:, at: at + n * dim].unflatten(1, (n, dim)))
            at += n * dim
    else:
        buf = torch.empty(heads, 1 << 26, dtype=B, device="cuda")
        wide = [buf[:, i * T * dim: (i + 1) * T * dim].unflatten(1, (T, dim)).transpose(0, 1) for i in range(8)]
    assert max((t.shape[0] - 1) * t.stride(0) + (t.shape[1] - 1) * t.stride(1) for t in wide) > 1 << 31
    compact = [torch.randn(T, n, dim, generator=gen, device="cuda").to(B) for n in shapes]
    for a, b in zip(wide, compact):
        a.copy_(b)
    offsets = torch.tensor([0, 70, 70, T - 1], dtype=torch.int32, device="cuda")
    for x in (wide, compact):
        lse = torch.zeros(heads, T, device="cuda")
        q, k, v, d_o, o, dq, dk, dv = x
        ctx.attention_forward(q, k, v, o, lse, offsets=offsets)
        ctx.attention_backward(q, k, v, o, lse, d_o, dq, dk, dv, offsets=offsets)
    for a, b in zip(wide, compact):
        assert torch.equal(a, b)


def test_loss_in_wide_strides(ctx):
    """Rows of hidden 2^23 elements apart, of the weight 2^22: the bits that compact matrices give."""
    T, d, vocab = 300, 64, 1000
    c = Loss(T, d, vocab, seed=1)
    want = c.gradient(torch.float32)
    c.forward(ctx)
    c.backward(ctx, want)
    loss, lse, dhidden = c.loss.clone(), c.lse.clone(), c.dhidden.clone()
    rows, table = torch.empty(T, 1 << 23, dtype=B, device="cuda"), torch.empty(vocab, 1 << 22, dtype=B, device="cuda")
    hidden, weight = rows[:, :d].copy_(c.hidden), table[:, :d].copy_(c.weight)
    c.hidden, c.weight, c.dhidden = hidden, weight, rows[:, d: 2 * d]
    c.forward(ctx)
    dweight = torch.empty(vocab, 1 << 22, dtype=torch.float32, device="cuda")[:, :d]
    c.backward(ctx, dweight)
    assert torch.equal(c.loss, loss) and torch.equal(c.lse, lse) and torch.equal(c.dhidden, dhidden) and torch.equal(dweight, want)


def test_loss_of_many_tokens(ctx):
    """2^21 tokens and more: the logits' gradient of a piece has more than 2^31 elements.  Checked are some tokens' losses and
    rows of dhidden."""
    T, d, vocab = (1 << 21) + 777, 16, 2500
    c = Loss(T, d, vocab, seed=2)
    c.dloss.mul_(T)
    c.forward(ctx)
    dweight = c.gradient(torch.float32)
    c.backward(ctx, dweight)
    rows = torch.cat([torch.arange(n, n + 300, device="cuda") for n in (0, 1 << 20, (1 << 21) - 150, T - 300)])
    (loss, e_loss), (lse, e_lse), (z, ez) = loss64(c.hidden[rows], c.weight, c.targets[rows])
    within(c.loss[rows], loss, e_loss, "loss")
    within(c.lse[rows], lse, e_lse, "lse")
    (dh, e_dh), _ = loss_back64(c.hidden[rows], c.weight, c.targets[rows], c.dloss[rows])
    within(c.dhidden[rows], dh, e_dh * (1 + UB) + UB * dh.abs(), "dhidden")
    assert bool(dweight.isfinite().all())


def test_two_contexts_on_two_streams(dd):
    """Calls of two contexts beside one another, each of whose kernels takes tensor memory: what each gives alone."""
    from test_gpu_attention import Case as Attention
    contexts, streams = [dd.Context(0) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    attention = [Attention([900, 128, 30, 513], 8, 2, dim, seed=dim) for dim in (64, 128)]
    loss = [Loss(*size, seed=4) for size in ((64, 136, 20000), (520, 136, 4000))]
    grads = [c.gradient(torch.float32) for c in loss]
    status = [torch.zeros(1, dtype=torch.int32, device="cuda") for _ in range(2)]

    def work(i, stream):
        kw = dict(status=status[i], stream=stream)
        for a, c in ((attention[i], loss[i]), (attention[i], loss[i])):
            a.forward(contexts[i], **kw)
            c.forward(contexts[i], **kw)
            a.backward(contexts[i], **kw)
            c.backward(contexts[i], grads[i], **kw)

    def results(i):
        a, c = attention[i], loss[i]
        return [t.clone() for t in (a.o, a.dq, a.dk, a.dv, c.loss, c.lse, c.dhidden, grads[i])]

    torch.cuda.synchronize()
    alone = []
    for i in range(2):
        work(i, streams[i])
        torch.cuda.synchronize()
        alone.append(results(i))
    for _ in range(20):
        for i in range(2):
            work(i, streams[i])
    torch.cuda.synchronize()
    assert [int(s) for s in status] == [0, 0]
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(alone[i], results(i)))
    for c in contexts:
        c.close()
