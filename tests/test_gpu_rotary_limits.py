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
