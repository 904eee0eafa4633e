"""Gradients of attention and of the loss against differences, and the loss's routes that add to what is there."""
import pytest
import torch

from decoder_util import B, U, UB, attention64, loss_back64, within
from test_gpu_attention import Case as Attention
from test_gpu_vocab_loss import Case as Loss

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def ctx():
    from paper_2604_21428_b200 import ddmerge
    c = ddmerge.Context(0)
    yield c
    c.close()


COUNT = 48                     # directions


def slopes(objective, x, directions, eps=1e-3):
    """Central differences of ``objective`` at x along unit vectors."""
    return torch.tensor([(objective(x + eps * u) - objective(x - eps * u)) / (2 * eps) for u in directions], dtype=torch.float64, device=x.device)


def check(objective, x, g):
    """g is the gradient of ``objective`` at x: its 2-norm is the slope along itself, and slopes along random directions
    say how far it is off.  For a unit vector u drawn evenly from n dimensions n E[((G - g) u)^2] = |G - g|^2, with COUNT of
    them within 1 / sqrt(2 COUNT) = 10 % (rms).  A gradient's operands, its own rounding and o's are off by 2^-8 of its
    2-norm each at most, in the mean less than half of it.  What is negated, of another size or short of a row fails."""
    g, gen = g.double(), torch.Generator(device="cuda").manual_seed(3)
    size = float(g.norm())
    assert abs(float(slopes(objective, x, [g / size])[0]) - size) <= 3 * UB * size
    directions = torch.randn(COUNT, *g.shape, generator=gen, dtype=torch.float64, device="cuda")
    directions /= directions.flatten(1).norm(dim=1).reshape(-1, *[1] * g.dim())
    want = slopes(objective, x, directions)

    def distance(y):
        return float(((want - directions.flatten(1) @ y.flatten()).square().mean() * y.numel()).sqrt())

    assert distance(g) <= 3 * UB * size
    row = g.clone()
    row[g.flatten(1).norm(dim=1).argmax()] = 0
    for wrong in (-g, 0.95 * g, 1.05 * g, row):
        assert distance(wrong) > 3 * UB * size


@pytest.mark.parametrize("lengths,heads,kv,dim,causal", [([70, 30], 2, 1, 32, True), ([150], 4, 2, 64, False), ([260, 3], 2, 2, 128, True)], ids=str)
def test_attention(ctx, lengths, heads, kv, dim, causal):
    c = Attention(lengths, heads, kv, dim, seed=6)
    c.forward(ctx, causal=causal)
    c.backward(ctx, causal=causal)
    x = [t.double() for t in (c.q, c.k, c.v)]
    for i, g in enumerate((c.dq, c.dk, c.dv)):
        def objective(y):
            parts = [y if j == i else t for j, t in enumerate(x)]
            return float(sum((attention64(*(t[d] for t in parts), c.scale, causal)[0][0] * c.d_o[d].double()).sum() for d in c.docs))
        check(objective, x[i], g)


@pytest.mark.parametrize("size", [(60, 40, 150), (200, 72, 1000), (3, 64, 300)], ids=str)
def test_loss(ctx, size):
    c = Loss(*size, seed=8)
    c.forward(ctx)
    dweight = c.gradient(torch.float32)
    c.backward(ctx, dweight)
    valid = c.targets >= 0
    x = [c.hidden.double(), c.weight.double()]
    for i, g in enumerate((c.dhidden, dweight)):
        def objective(y):
            h, w = (y if j == i else t for j, t in enumerate(x))
            z = h @ w.t()
            loss = torch.logsumexp(z, -1) - z.gather(1, c.targets.clamp(min=0)[:, None])[:, 0]
            return float((loss * c.dloss.double() * valid).sum())
        check(objective, x[i], g)


@pytest.mark.parametrize("dtype", [B, torch.float32])
@pytest.mark.parametrize("size", [(16, 200, 4700), (100, 136, 5000), (400, 96, 1500), (4100, 64, 130), (12000, 72, 12345)], ids=str)
def test_loss_adds_twice(ctx, size, dtype):
    """Two calls that add to dweight behind one another: few tokens, one piece, tokens split, several pieces.  Each adds
    the sum that a call without rounds, and rounds once."""
    c = Loss(*size, seed=5)
    c.forward(ctx)
    first = torch.randn(c.weight.shape, device="cuda").to(dtype) * 1e-3
    added = c.gradient(dtype)
    added.copy_(first)
    (dh, e_dh), (dw, e_dw) = loss_back64(c.hidden, c.weight, c.targets, c.dloss)
    for _ in range(2):
        c.backward(ctx, added, accumulate=True)
    unit = UB if dtype == B else U
    once, twice = first.double() + dw, first.double() + 2 * dw
    e_once = e_dw + 2 * U * (first.double().abs() + dw.abs())
    e_once = e_once * (1 + unit) + unit * once.abs()
    e_twice = e_once + e_dw + 2 * U * (once.abs() + e_once + dw.abs())
    within(added, twice, e_twice * (1 + unit) + unit * twice.abs(), "dweight")
    within(c.dhidden, dh, e_dh * (1 + UB) + UB * dh.abs(), "dhidden")
    fresh = c.gradient(dtype)
    c.backward(ctx, fresh)
    zero = c.gradient(dtype, 0.0)
    c.backward(ctx, zero, accumulate=True)
    assert torch.equal(fresh, zero)                       # added to zeros: the same sums, rounded once
