"""A decoder's training step as a whole, and learners that train decoders between merges."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
SIZES = dict(vocab=200, d=64, f=136, layers=2, heads=4, kv_heads=2, dim=16)


@pytest.fixture(scope="module")
def mods():
    from paper_2604_21428_b200 import ddmerge, learner
    ctx = ddmerge.Context(0)
    yield ddmerge, learner, ctx
    ctx.close()


def decoder64(m, weights, ids, targets, positions, offsets):
    """The mean loss in float64 from the weights, by the model's definition."""
    def norm(x):
        return x / (x.square().mean(-1, keepdim=True) + 1e-6).sqrt()

    def turn(x):
        half = m.dim // 2
        w = positions.double()[:, None, None] * m.frequencies
        a, b = x[..., :half], x[..., half:]
        return torch.cat([a * w.cos() - b * w.sin(), b * w.cos() + a * w.sin()], -1)

    embedding, head = weights[-1]
    ends = offsets.tolist()
    x = embedding[ids[: ends[-1]]]
    positions = positions[: ends[-1]]
    for w_qkv, w_o, wg, wu, wd in weights[:-1]:
        qkv = (norm(x) @ w_qkv.t()).unflatten(1, (-1, m.dim))
        q, k, v = qkv[:, :m.heads], qkv[:, m.heads: m.heads + m.kv_heads], qkv[:, m.heads + m.kv_heads:]
        group = m.heads // m.kv_heads
        q, k, v = turn(q).transpose(0, 1), turn(k).transpose(0, 1).repeat_interleave(group, 0), v.transpose(0, 1).repeat_interleave(group, 0)
        outs = []
        for a, b in zip(ends, ends[1:]):
            s = q[:, a:b] @ k[:, a:b].transpose(1, 2) / math.sqrt(m.dim)
            s = s.masked_fill(torch.ones(b - a, b - a, dtype=torch.bool, device=s.device).triu(1), float("-inf"))
            outs.append(torch.softmax(s, -1) @ v[:, a:b])
        x = x + torch.cat(outs, 1).transpose(0, 1).flatten(1) @ w_o.t()
        h = norm(x)
        g = h @ wg.t()
        x = x + (g * torch.sigmoid(g) * (h @ wu.t())) @ wd.t()
    z = norm(x) @ head.t()
    t = targets[: ends[-1]]
    keep = t >= 0
    return (torch.logsumexp(z, -1) - z.gather(1, t.clamp(min=0)[:, None])[:, 0])[keep].mean()


@pytest.mark.parametrize("tokens,sequences", [(40, 3), (500, 4)])
def test_step_against_autograd(mods, tokens, sequences):
    """Gradients and loss against float64 autograd on the same bf16 weights, twice: the second micro-batch has another
    number of rows behind its documents.  About 30 bf16 roundings of activations and as many of gradients
    lie between a weight and the loss, each 2^-9 rms and independent of the others: sqrt(60) 2^-9 = 1.5 % of a
    gradient's 2-norm, held to twice that."""
    dd, lm, ctx = mods
    m = lm.DecoderLearner(ctx, **SIZES, tokens=tokens, sequences=sequences, lr=0.0)
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    for p, fragment in enumerate(m.initial(gen)):
        m.receive(p, fragment)
    for _ in range(2):
        batch = lm.packed_documents(gen, tokens, sequences, SIZES["vocab"])
        weights = [[w.double().clone().requires_grad_() for w in layer] for layer in m.weights]
        loss = decoder64(m, weights, *batch)
        loss.backward()
        got = m.step(*batch)
        assert abs(float(got) - float(loss.detach())) <= 0.03 * float(loss.detach())
        for layer, grads in zip(weights, m.weight_grads):
            for w, g in zip(layer, grads):
                assert float((g.double() - w.grad).norm()) <= 0.03 * float(w.grad.norm())


def test_learners_and_merges_run(mods):
    """Two learners and a merge with push after every few steps; what they hold after a push is the global fragment."""
    _, lm, ctx = mods
    history = lm.train_decoder(ctx, rounds=2, inner_steps=2, tokens=130, sequences=3, **{**SIZES, "layers": 1})
    assert len(history) == 2 and all(math.isfinite(v) for v in history)


def test_command(mods, monkeypatch):
    import runpy
    import sys
    monkeypatch.setattr(sys, "argv", ["learner", "nothing"])
    with pytest.raises(SystemExit):
        runpy.run_module("paper_2604_21428_b200.learner", run_name="__main__")
