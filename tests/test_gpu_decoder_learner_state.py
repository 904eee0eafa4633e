"""What a decoder's learner keeps, skips and reports."""
import pytest
import torch

from decoder_util import U, within

pytestmark = pytest.mark.gpu
SIZES = dict(vocab=200, d=64, f=136, layers=1, heads=4, kv_heads=2, dim=16, tokens=200, sequences=3)


@pytest.fixture(scope="module")
def mods():
    from paper_2604_21428_b200 import ddmerge, learner
    ctx = ddmerge.Context(0)
    yield ddmerge, learner, ctx
    ctx.close()


def start(mods, seed=0, **kw):
    _, lm, ctx = mods
    m = lm.DecoderLearner(ctx, **SIZES, **kw)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    for p, fragment in enumerate(m.initial(gen)):
        m.receive(p, fragment)
    return m, gen


def test_gradients_of_the_projections_are_float32(mods):
    """Sums of products of bf16 operands in float32, not rounded on the way to the float32 buffers."""
    _, lm, _ = mods
    m, gen = start(mods, lr=0.0)
    m.step(*lm.packed_documents(gen, SIZES["tokens"], SIZES["sequences"], SIZES["vocab"]))
    dw_qkv, dw_o = m.weight_grads[0][:2]
    for g in (dw_qkv, dw_o):
        assert not torch.equal(g, g.to(torch.bfloat16).float())
    a, b = m.dqkv.flatten(1).double(), m.kept[0]["h1"].double()
    within(dw_qkv, a.t() @ b, (SIZES["tokens"] + 16) * 2 * U * (a.abs().t() @ b.abs()) + 1e-38, "dw_qkv")
