"""The learner's inner step as a whole, and learners that train between merges."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mods():
    from paper_2604_21428_b200 import ddmerge, learner
    ctx = ddmerge.Context(0)
    yield ddmerge, learner, ctx
    ctx.close()


@pytest.mark.parametrize("tokens", [7, 300])
def test_inner_step_against_autograd(mods, tokens):
    """Gradients, their norm and the update of a two-block stack against float64 autograd on the same
    bf16 weights.  Per block, a handful of bf16 roundings (2^-9 rms each, independent) enter a
    gradient: 8 of them are under 1.6 % of its 2-norm; the norm is within the same; AdamW's first step
    moves every parameter by lr (1 - eps / |g|) whatever the gradient's size, so only signs count."""
    dd, lm, ctx = mods
    d, f, blocks = 64, 136, 2
    m = lm.Learner(ctx, d, f, blocks, tokens, lr=1e-2, max_norm=0.1)
    gen = torch.Generator(device="cuda").manual_seed(3)
    for p in range(blocks):
        m.receive(p, torch.randn(3 * d * f, generator=gen, device="cuda") * 0.1)
    before = [t.clone() for t in m.params]
    ws = [[w.double().clone().requires_grad_() for w in m.weights[i]] for i in range(blocks)]
    x = torch.randn(tokens, d, generator=gen, device="cuda").to(torch.bfloat16)
    target = torch.randn(tokens, d, generator=gen, device="cuda").to(torch.bfloat16)
    h = x.double()
    for wg, wu, wd in ws:
        g = h @ wg.t()
        h = h + (g * torch.sigmoid(g) * (h @ wu.t())) @ wd.t()
    loss = (h - target.double()).square().mean()
    loss.backward()
    got = m.step(x, target)
    loss = float(loss.detach())
    assert abs(float(got) - loss) <= 0.016 * loss
    want = [torch.cat([w.grad.reshape(-1) for w in ws[i]]) for i in range(blocks)]
    for a, b in zip(m.grads, want):
        assert float((a.double() - b).norm()) <= 0.016 * float(b.norm())
    r = dd.read_grad_record(m.record)
    norm = math.sqrt(sum(float(b.square().sum()) for b in want))
    assert r.status == dd.STATUS_OK and abs(r.norm - norm) <= 0.016 * norm
    for a, b, g, c in zip(m.params, before, m.grads, m.copies):
        step = (b - a).double()
        clear = g.abs() * r.scale > 1e-6                       # eps is 1e-8
        assert bool(((step - 1e-2 * torch.sign(g.double())).abs()[clear] <= 1e-2 * 0.011).all())
        assert torch.equal(c, a.to(torch.bfloat16))


def test_learners_and_merges_fit_a_teacher(mods):
    """Four learners, a merge with push after every thirty steps: the loss falls, and what the learners
    hold after a push is the global fragment."""
    _, lm, ctx = mods
    history = lm.train(ctx, rounds=5, tokens=256, d=128, f=264)
    assert all(math.isfinite(v) for v in history)
    assert history[-1] < 0.5 * history[0], history
