"""Rotary positions at the ends of what the call takes."""
import pytest
import torch

from decoder_util import B, U, UB, within
from test_gpu_rotary import turned64

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


def test_heads(dd, ctx):
    """2^16 - 1 heads are taken, 2^16 are too many."""
    f = torch.ones(1, dtype=torch.float64, device="cuda")
    positions = torch.tensor([1, -1, 3], device="cuda")
    q, k = (torch.randn(3, 65535, 2, device="cuda").to(B) for _ in range(2))
    before = [x.clone() for x in (q, k)]
    ctx.rotary(q, k, positions, f)
    for x, y in zip((q, k), before):
        want, e = turned64(y, positions.clamp(min=0), f, 1.0, False, False)
        live = positions >= 0
        within(x[live], want[live], (e * (1 + UB) + UB * want.abs())[live], "heads")
        assert torch.equal(x[~live], y[~live])
    many, few = torch.zeros(1, 65536, 2, dtype=B, device="cuda"), torch.zeros(1, 1, 2, dtype=B, device="cuda")
    for q, k in ((many, None), (few, many)):
        with pytest.raises(dd.DDMergeError) as e:
            ctx.rotary(q, k, positions[:1], f)
        assert e.value.rc == dd.ERR_TOO_LARGE


@pytest.mark.parametrize("reach", [28, 31, 40, 50])
def test_far_positions(ctx, reach):
    """Angles of up to 2^reach radians.  Three float64 roundings of a turn count are 2^-51 of the angle at most, beside
    the bound of near ones; frequencies whose products with the positions are exact in float64."""
    f = torch.tensor([1.0, 0.75, 0.5, 0.125], dtype=torch.float64, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(reach)
    positions = (1 << reach) - torch.randint(0, 1 << 20, (200,), generator=gen, device="cuda")
    x = torch.randn(200, 2, 8, generator=gen, device="cuda")
    y = torch.empty_like(x)
    ctx.rotary(x, None, positions, f, q_out=y)
    want, e = turned64(x, positions, f, 1.0, False, False)
    a, b = x.double().abs()[..., :4], x.double().abs()[..., 4:]
    off = (positions.double()[:, None, None] * f) * 2.0 ** -51 * (a + b)
    within(y, want, e + torch.cat([off, off], -1) + U * want.abs(), "far")
