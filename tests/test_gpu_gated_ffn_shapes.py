"""The gated block where its kernels take other shapes than small sizes do, against float64 with the bounds
of test_gpu_gated_ffn."""
import pytest
import torch

from test_gpu_gated_ffn import B, UB, U, backward64, forward64, mat, pads_untouched, within

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


def check_forward(ctx, size, act, with_residual, pad=0):
    T, d, f = size
    x, residual = mat(T, d, 1, pad=pad), mat(T, d, 2, pad=pad) if with_residual else None
    w = [mat(f, d, 3, d ** -0.5, pad), mat(f, d, 4, d ** -0.5, pad), mat(d, f, 5, f ** -0.5, pad)]
    y, gate, up = mat(T, d, 6, pad=pad), mat(T, f, 7, pad=pad), mat(T, f, 8, pad=pad)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx.gated_ffn_forward(x, *w, y, activation=act, residual=residual, gate=gate, up=up, status=status)
    assert int(status) == 0
    for got, (ref, tol), what in zip((y, gate, up), forward64(x, *w, residual, act), ("y", "gate", "up")):
        within(got, ref, tol, what)
        assert pads_untouched(got)
    if with_residual:                              # in place on the residual, the same bits
        ctx.gated_ffn_forward(x, *w, residual, activation=act, residual=residual)
        assert torch.equal(residual, y)


def check_backward(ctx, size, act, kind, pad=0):
    T, d, f = size
    x, dy = mat(T, d, 11, pad=pad), mat(T, d, 12, 1e-2, pad=pad)
    w = [mat(f, d, 13, d ** -0.5, pad), mat(f, d, 14, d ** -0.5, pad), mat(d, f, 15, f ** -0.5, pad)]
    gate, up = mat(T, f, 16, 2.0, pad=pad), mat(T, f, 17, pad=pad)
    gk, acc = B if kind.startswith("bf16") else torch.float32, kind.endswith("acc")
    dx = mat(T, d, 18, pad=pad)
    dws = [mat(f, d, 19, 1e-2, pad, gk), mat(f, d, 20, 1e-2, pad, gk), mat(d, f, 21, 1e-2, pad, gk)]
    old = [t.double() for t in dws]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx.gated_ffn_backward(x, *w, gate, up, dy, dx, *dws, activation=act, accumulate=acc, status=status)
    assert int(status) == 0
    want = backward64(x, *w, gate, up, dy, act)
    for got, (ref, tol), before, what in zip((dx, *dws), want, (None, *old), ("dx", "dw_gate", "dw_up", "dw_down")):
        if acc and before is not None:
            ref = ref + before
        within(got, ref, tol * (1 + UB) + (UB if got.dtype == B else 2 * U) * ref.abs(), what)
        assert pads_untouched(got)


# Few tokens in tiles of more than 64: two rounds of the reduction, with features that end inside a warp's four
TWO_ROUNDS = [(97, 2407, 2731), (113, 1001, 2733), (255, 2401, 5003)]


@pytest.mark.parametrize("size", TWO_ROUNDS, ids=str)
def test_two_rounds_ragged(ctx, size):
    for act in (0, 1):
        check_forward(ctx, size, act, True, pad=act)
    check_backward(ctx, size, 0, "bf16")
    check_backward(ctx, size, 1, "f32_acc", pad=1)
