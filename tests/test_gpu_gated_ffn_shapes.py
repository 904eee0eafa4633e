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


# Sizes whose way down, or whose gradients, are cut into 256 x 512 tiles, with d and f ending in either half
# of a tile's columns, tokens inside a tile's rows and K inside a block.  (T, d, f)
WIDE_FORWARD = [(3647, 1060, 1603), (4725, 829, 1561), (2313, 2049, 2731)]
WIDE_BACKWARD = [(3614, 790, 1742), (2445, 1333, 1306), (3992, 2569, 1810), (4758, 2561, 2715)]


def kernels_of(call):
    """Names of the kernels that a call launches; None where the profiler does not see any."""
    from torch.profiler import ProfilerActivity, profile
    call()
    torch.cuda.synchronize()
    with profile(activities=[ProfilerActivity.CUDA]) as prof:
        call()
        torch.cuda.synchronize()
    names = [e.key for e in prof.key_averages()]
    return names if any("ffn_" in n for n in names) else None


def test_sizes_take_wide_tiles(ctx):
    seen = []
    for sizes, backward in ((WIDE_FORWARD, False), (WIDE_BACKWARD, True)):
        for T, d, f in sizes:
            x, y, w = mat(T, d, 1), mat(T, d, 2), [mat(f, d, 3), mat(f, d, 4), mat(d, f, 5)]
            gate, up, dws = mat(T, f, 6), mat(T, f, 7), [mat(f, d, 8), mat(f, d, 9), mat(d, f, 10)]
            if backward:
                names = kernels_of(lambda: ctx.gated_ffn_backward(x, *w, gate, up, x, y, *dws))
            else:
                names = kernels_of(lambda: ctx.gated_ffn_forward(x, *w, y))
            if names is None:
                pytest.skip("no kernel names from the profiler")
            seen.append(any("ffn_gemm_kernel<0, 512" in n for n in names))
    assert all(seen), seen


@pytest.mark.parametrize("with_residual", [False, True])
@pytest.mark.parametrize("size", WIDE_FORWARD, ids=str)
def test_wide_forward(ctx, size, with_residual):
    check_forward(ctx, size, WIDE_FORWARD.index(size) % 2, with_residual, pad=int(with_residual))


@pytest.mark.parametrize("kind", ["bf16", "f32", "bf16_acc", "f32_acc"])
@pytest.mark.parametrize("size", WIDE_BACKWARD, ids=str)
def test_wide_backward(ctx, size, kind):
    check_backward(ctx, size, WIDE_BACKWARD.index(size) % 2, kind, pad=int(kind.endswith("acc")))


LARGE = [(700, 136, 264), (3647, 1060, 1603)]


@pytest.mark.parametrize("size", LARGE, ids=str)
def test_rows_do_not_mix_in_large_products(ctx, size):
    """NaN and infinities in a token's row stay in that row of the results, in tiles of many rows too."""
    T, d, f = size
    x, w = mat(T, d, 1), [mat(f, d, 2, 0.1), mat(f, d, 3, 0.1), mat(d, f, 4, 0.1)]
    clean, dirty = mat(T, d, 5), mat(T, d, 6)
    ctx.gated_ffn_forward(x, *w, clean)
    x2 = mat(T, d, 1)
    x2[1, 5], x2[T - 1, d - 1] = float("nan"), float("inf")
    ctx.gated_ffn_forward(x2, *w, dirty)
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[1] = keep[T - 1] = False
    assert torch.equal(clean[keep], dirty[keep])
    assert bool(torch.isnan(dirty[1].float()).all()) and not bool(torch.isfinite(dirty[T - 1].float()).any())


@pytest.mark.parametrize("scale", [30.0, 3e4])
def test_large_arguments_in_large_products(ctx, scale):
    """Gates far out on both sides: the activation saturates without overflow or NaN."""
    T, d, f = 700, 64, 128
    for act in (0, 1):
        x, w = mat(T, d, 1, scale), [mat(f, d, 2), mat(f, d, 3, 0.1), mat(d, f, 4, 0.1)]
        y, gate, up = mat(T, d, 5), mat(T, f, 6), mat(T, f, 7)
        ctx.gated_ffn_forward(x, *w, y, activation=act, gate=gate, up=up)
        assert bool(torch.isfinite(y.float()).all())
        dx, dws = mat(T, d, 8), [mat(f, d, 9), mat(f, d, 10), mat(d, f, 11)]
        ctx.gated_ffn_backward(x, *w, gate, up, mat(T, d, 12), dx, *dws, activation=act)
        assert all(bool(torch.isfinite(t.float()).all()) for t in (dx, *dws))


def test_bounded_waits_of_wide_tiles_expire(dd, ctx):
    """The test hook holds back the first copies of every launch: the waits run out, the status word says so,
    and the next call on the same context is right."""
    for (T, d, f), backward in ((WIDE_FORWARD[0], False), (WIDE_BACKWARD[0], True)):
        x, w = mat(T, d, 1), [mat(f, d, 2, 0.1), mat(f, d, 3, 0.1), mat(d, f, 4, 0.1)]
        y, gate, up = mat(T, d, 5), mat(T, f, 6), mat(T, f, 7)
        dws = [mat(f, d, 9), mat(f, d, 10), mat(d, f, 11)]
        status = torch.zeros(1, dtype=torch.int32, device="cuda")

        def call(flags):
            if backward:
                ctx.gated_ffn_backward(x, *w, gate, up, x, y, *dws, status=status, flags=flags)
            else:
                ctx.gated_ffn_forward(x, *w, y, status=status, flags=flags)

        call(dd.DEBUG_EXPIRE_WAIT)
        torch.cuda.synchronize()
        assert status.tolist() == [dd.STATUS_WAIT_LIMIT]
        status.zero_()
        call(0)
        assert status.tolist() == [0]
        if not backward:
            within(y, *forward64(x, *w, None, 0)[0], "after the expiry")
            continue
        for got, (ref, tol) in zip((y, *dws), backward64(x, *w, gate, up, x, 0)):
            within(got, ref, tol * (1 + UB) + UB * ref.abs(), "after the expiry")


def halves(rows, cols, seeds, std=1.0, dtype=B):
    """Two matrices side by side in the rows of one buffer, NaN between and behind them."""
    wide = (cols + 7) // 8 * 8
    buf = torch.full((rows, 2 * wide + 8), float("nan"), dtype=dtype, device="cuda")
    pair = buf[:, :cols], buf[:, wide:wide + cols]
    for t, seed in zip(pair, seeds):
        t.copy_(mat(rows, cols, seed, std, dtype=dtype))
    return buf, pair


@pytest.mark.parametrize("size", [(1, 64, 64), (2, 40, 24), (37, 65, 131), (300, 136, 257), (900, 257, 333)], ids=str)
def test_matrices_side_by_side(dd, ctx, size):
    """gate and up, the two weights and their gradients as halves of one buffer's rows: the same bits as in
    buffers of their own, and nothing between them is touched."""
    T, d, f = size
    x, dy = mat(T, d, 1), mat(T, d, 2)
    own = [mat(f, d, 3, d ** -0.5), mat(f, d, 4, d ** -0.5), mat(d, f, 5, f ** -0.5)]
    _, (wg, wu) = halves(f, d, (3, 4), d ** -0.5)
    kept, (gate, up) = halves(T, f, (6, 7))
    grads, (dwg, dwu) = halves(f, d, (8, 9))
    y, y2, dx, dx2 = (mat(T, d, 10 + i) for i in range(4))
    g2, u2, dwd, dwd2 = mat(T, f, 14), mat(T, f, 15), mat(d, f, 16), mat(d, f, 17)
    dw2 = [mat(f, d, 18), mat(f, d, 19)]
    ctx.gated_ffn_forward(x, wg, wu, own[2], y, gate=gate, up=up)
    ctx.gated_ffn_forward(x, *own, y2, gate=g2, up=u2)
    ctx.gated_ffn_backward(x, wg, wu, own[2], gate, up, dy, dx, dwg, dwu, dwd)
    ctx.gated_ffn_backward(x, *own, g2, u2, dy, dx2, *dw2, dwd2)
    for a, b in zip((y, gate, up, dx, dwg, dwu, dwd), (y2, g2, u2, dx2, *dw2, dwd2)):
        assert torch.equal(a, b)
    for buf, n in ((kept, f), (grads, d)):
        wide = (n + 7) // 8 * 8
        assert bool(torch.isnan(buf[:, n:wide].float()).all()) and bool(torch.isnan(buf[:, wide + n:].float()).all())
    # one element into the neighbour: refused
    if T > 1:
        wide = (f + 7) // 8 * 8
        flat = torch.zeros(T * 4 * wide, dtype=B, device="cuda")
        a = flat.as_strided((T, f), (2 * wide, 1), 0)
        for start in (wide - 8, 2 * wide - 8):
            b = flat.as_strided((T, f), (2 * wide, 1), start)
            if start >= f and start + f <= 2 * wide:
                continue
            with pytest.raises(dd.DDMergeError) as e:
                ctx.gated_ffn_forward(x, *own, y, gate=a, up=b)
            assert e.value.rc == dd.ERR_ALIAS
