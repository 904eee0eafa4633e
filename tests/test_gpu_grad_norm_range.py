"""The range of elements over which the gradient norm keeps its bound, and what it says beyond."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24


@pytest.fixture(scope="module")
def dd():
    from paper_2604_21428_b200 import ddmerge
    return ddmerge


@pytest.fixture(scope="module")
def ctx(dd):
    c = dd.Context(0)
    yield c
    c.close()


def norm_of(dd, ctx, tensors, max_norm=1.0):
    record = dd.new_grad_record()
    ctx.grad_norm(tensors, max_norm, record)
    return dd.read_grad_record(record), sum(float(t.double().square().sum()) for t in tensors)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("size", [2.9e18, 1e12, 1.0, 1e-12, 2e-19, 1e-19, 1e-20, 1e-22, 1e-25, 1e-38])
def test_range(dd, ctx, size, shift, dtype):
    """Elements of one size throughout: relative 34 u and 2^-149 for each element (the spacing of float32
    below its normal range, once for the square and halved by rounding, once for the sum)."""
    n = 40_000
    base = (torch.ones(n + shift + 9, device="cuda") * size).to(dtype)
    base[::2].neg_()
    ts = [base[shift:shift + n], base[shift:shift + 11]]
    r, want = norm_of(dd, ctx, ts)
    assert r.status == dd.STATUS_OK
    tol = 34 * U * want + 2.0 ** -149 * (n + 11)
    assert abs(r.norm_sq - want) <= tol
    assert abs(r.norm - math.sqrt(r.norm_sq)) <= 2 * U * r.norm + 2.0 ** -149


def test_mixed_sizes(dd, ctx):
    """Tiny elements beside ordinary ones: the ordinary ones decide."""
    g = torch.full((100_000,), 1e-30, device="cuda")
    g[::1000] = 3.0
    r, want = norm_of(dd, ctx, [g])
    assert r.status == dd.STATUS_OK and abs(r.norm_sq - want) <= 34 * U * want


def test_past_the_range(dd, ctx):
    for value in (2e19, 3e38, -3e38):
        g = torch.zeros(50_000, device="cuda")
        g[777] = value
        r, _ = norm_of(dd, ctx, [g])
        assert r.status == dd.STATUS_NONFINITE and r.scale == 1.0 and math.isinf(r.norm)
