"""The gated feed-forward block, forward and backward, against float64.

Every output is held to an element-wise bound that follows from the arithmetic: bf16 rounding of
the result (2^-8), bf16 rounding of each operand that the block itself produces (2^-8 of the sum
of the products' sizes), float32 accumulation of K products (K 2^-24 of the same sum), and the fast
exponential and division in the activation (2^-18, scaled by the argument's size).
"""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
U, UB, UA = 2.0 ** -24, 2.0 ** -8, 2.0 ** -18
B = torch.bfloat16


@pytest.fixture(scope="module")
def dd():
    from paper_2604_21428_b200 import ddmerge
    return ddmerge


@pytest.fixture(scope="module")
def ctx(dd):
    c = dd.Context(0)
    yield c
    c.close()


def rows8(n):
    return (n + 7) // 8 * 8


def mat(rows, cols, seed, std=1.0, pad=0, dtype=B):
    """A matrix whose rows are ``pad`` x 8 elements longer than they need to be, NaN in between."""
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((rows, rows8(cols) + 8 * pad), float("nan"), dtype=dtype)
    buf[:, :cols] = (torch.randn(rows, cols, generator=g) * std).to(dtype)
    return buf.cuda()[:, :cols]


def pads_untouched(t):
    """Nothing was written between the rows of a matrix from ``mat``."""
    ld = t.stride(0)
    full = t.as_strided((t.shape[0], ld), (ld, 1))
    return bool(torch.isnan(full[:, t.shape[1]:].float()).all())


def act_parts(g, act):
    """a(g), a'(g) and bounds on the errors of their float32 evaluation, in float64."""
    k, q = 2 * math.sqrt(2 / math.pi), 0.044715
    s, ds = (g, torch.ones_like(g)) if act == 0 else (k * (g + q * g ** 3), k * (1 + 3 * q * g ** 2))
    sg = torch.sigmoid(s)
    a = g * sg
    slope = sg * (1 + g * ds * (1 - sg))
    size = 1 + s.abs() * (1 - sg)
    return a, slope, UA * a.abs() * size + 1e-38, UA * sg * (1 + (g * ds).abs()) * size + 1e-38


def forward64(x, wg, wu, wd, residual, act):
    """Float64 results with bounds: (y, ey), (gate, eg), (up, eu)."""
    x, wg, wu, wd = (t.double() for t in (x, wg, wu, wd))
    d, f = x.shape[1], wg.shape[0]
    G, Up = x @ wg.t(), x @ wu.t()
    sumg, sumu = (d + 2) * U * (x.abs() @ wg.abs().t()), (d + 2) * U * (x.abs() @ wu.abs().t())
    a, slope, ea, _ = act_parts(G, act)
    H = a * Up
    eh = UB * H.abs() + (1 + UB) * (Up.abs() * (ea + (slope.abs() + 0.5) * sumg) + a.abs() * sumu)
    Y = H @ wd.t()
    ey = eh @ wd.abs().t() + (f + 2) * U * (H.abs() @ wd.abs().t())
    if residual is not None:
        Y = Y + residual.double()
    ey = ey * (1 + UB) + UB * Y.abs() + 1e-38
    return (Y, ey), (G, UB * G.abs() + 2 * sumg + 1e-38), (Up, UB * Up.abs() + 2 * sumu + 1e-38)


def backward64(x, wg, wu, wd, gate, up, dy, act):
    """Float64 gradients with bounds: dx, dw_gate, dw_up, dw_down (before rounding of the result)."""
    x, wg, wu, wd, gate, up, dy = (t.double() for t in (x, wg, wu, wd, gate, up, dy))
    T, d, f = x.shape[0], x.shape[1], wg.shape[0]
    a, slope, ea, es = act_parts(gate, act)
    dh = dy @ wd
    edh = (d + 2) * U * (dy.abs() @ wd.abs())
    du, dg, h = dh * a, dh * up * slope, a * up
    edu = UB * du.abs() + (1 + UB) * (edh * a.abs() + dh.abs() * ea)
    edg = UB * dg.abs() + (1 + UB) * up.abs() * (edh * slope.abs() + dh.abs() * es)
    eh = UB * h.abs() + (1 + UB) * up.abs() * ea
    out = []
    for terms, n in (((( dg, edg, wg), (du, edu, wu)), 2 * f), (((dg.t(), edg.t(), x),), T),
                     (((du.t(), edu.t(), x),), T), (((dy.t(), None, h),), T)):
        r = sum(p @ q for p, _, q in terms)
        if terms[0][1] is None:
            e = dy.abs().t() @ eh
        else:
            e = sum(ep @ q.abs() for _, ep, q in terms)
        e = e + (n + 4) * U * sum(p.abs() @ q.abs() for p, _, q in terms)
        out.append((r, e + 1e-38))
    return out


def within(got, ref, tol, what):
    err = (got.double() - ref).abs()
    bad = ~(err <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / tol).max()):.2f} of the bound"


SIZES = [
    (1, 8, 8), (1, 64, 64), (1, 2048, 512), (2, 40, 24), (3, 1, 1), (5, 72, 136), (8, 256, 1000), (9, 264, 520),
    (16, 512, 512), (17, 96, 200), (31, 1000, 120), (33, 136, 264), (64, 128, 384), (65, 257, 131), (100, 520, 1032),
    (127, 64, 128), (128, 128, 256), (129, 136, 264), (200, 333, 777), (256, 1024, 512), (300, 64, 2048),
    (515, 200, 312), (1030, 264, 72), (2100, 136, 520), (300, 257, 131), (290, 333, 777), (700, 1001, 258),
    (600, 100, 8200), (1025, 2056, 640),
]


@pytest.mark.parametrize("act", [0, 1])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_forward(dd, ctx, size, act):
    T, d, f = size
    i = SIZES.index(size) + act
    x, residual = mat(T, d, 1, pad=i % 2), mat(T, d, 2, pad=i % 3) if i % 4 else None
    wg, wu, wd = mat(f, d, 3, d ** -0.5, i % 2), mat(f, d, 4, d ** -0.5, i % 2), mat(d, f, 5, f ** -0.5, (i // 2) % 2)
    want = forward64(x, wg, wu, wd, residual, act)
    for keep in (True, False):
        y = mat(T, d, 6, pad=i % 3)
        gate, up = (mat(T, f, 7, pad=i % 2), mat(T, f, 8, pad=i % 2)) if keep else (None, None)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        ctx.gated_ffn_forward(x, wg, wu, wd, y, activation=act, residual=residual, gate=gate, up=up, status=status)
        assert int(status) == 0
        for got, (ref, tol), what in zip((y, gate, up), want, ("y", "gate", "up")):
            if got is not None:
                within(got, ref, tol, what)
                assert pads_untouched(got)
    y2 = residual                                  # in place on the residual, and the same bits again
    if residual is not None:
        ctx.gated_ffn_forward(x, wg, wu, wd, y2, activation=act, residual=residual)
        assert torch.equal(y2, y)


@pytest.mark.parametrize("kind", ["bf16", "f32", "bf16_acc", "f32_acc"])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_backward(dd, ctx, size, kind):
    T, d, f = size
    i = SIZES.index(size)
    act = i % 2
    x, dy = mat(T, d, 11, pad=i % 2), mat(T, d, 12, 1e-2, pad=i % 3)
    wg, wu, wd = mat(f, d, 13, d ** -0.5, i % 2), mat(f, d, 14, d ** -0.5, i % 2), mat(d, f, 15, f ** -0.5, (i // 2) % 2)
    gate, up = mat(T, f, 16, 2.0, pad=i % 2), mat(T, f, 17, pad=i % 2)
    gk = B if kind.startswith("bf16") else torch.float32
    dx = mat(T, d, 18, pad=i % 2)
    dws = [mat(f, d, 19, 1e-2, i % 2, gk), mat(f, d, 20, 1e-2, i % 2, gk), mat(d, f, 21, 1e-2, (i // 2) % 2, gk)]
    old = [w.double() for w in dws]
    acc = kind.endswith("acc")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    ctx.gated_ffn_backward(x, wg, wu, wd, gate, up, dy, dx, *dws, activation=act, accumulate=acc, status=status)
    assert int(status) == 0
    want = backward64(x, wg, wu, wd, gate, up, dy, act)
    for got, (ref, tol), before, what in zip((dx, *dws), want, (None, *old), ("dx", "dw_gate", "dw_up", "dw_down")):
        if acc and before is not None:
            ref = ref + before
        tol = tol * (1 + UB) + (UB if got.dtype == B else 2 * U) * ref.abs()
        within(got, ref, tol, what)
        assert pads_untouched(got)


def test_gradient_against_differences(dd, ctx):
    """The kernels' gradients of L = <dy, y> along random directions against central differences
    of the float64 block.  Bound: the gradients' own bounds along the direction, plus the
    differences' error (h^2 of the third derivative, under 1e-6 of the terms here)."""
    T, d, f = 70, 96, 136
    for act in (0, 1):
        x, dy = mat(T, d, 1), mat(T, d, 2)
        w = [mat(f, d, 3, d ** -0.5), mat(f, d, 4, d ** -0.5), mat(d, f, 5, f ** -0.5)]
        y, gate, up = mat(T, d, 6), mat(T, f, 7), mat(T, f, 8)
        ctx.gated_ffn_forward(x, *w, y, activation=act, gate=gate, up=up)
        grads = [mat(T, d, 9), mat(f, d, 10), mat(f, d, 11), mat(d, f, 12)]
        ctx.gated_ffn_backward(x, *w, gate, up, dy, *grads, activation=act)
        # gate and up were rounded when they were kept: their error enters the gradient as well
        bounds = backward64(x, *w, gate, up, dy, act)
        exact = backward64(x, *w, x.double() @ w[0].double().t(), x.double() @ w[1].double().t(), dy, act)
        ins = [t.double() for t in (x, *w)]
        for k in range(4):
            g = torch.Generator(device="cuda").manual_seed(50 + k)
            v = torch.randn(ins[k].shape, generator=g, device="cuda", dtype=torch.float64)
            h = 1e-4

            def loss(s):
                a = [t + s * h * v if j == k else t for j, t in enumerate(ins)]
                return float((dy.double() * forward64(*a, None, act)[0][0]).sum())

            slope = (loss(1) - loss(-1)) / (2 * h)
            got = float((grads[k].double() * v).sum())
            (ref, tol), (ref2, _) = bounds[k], exact[k]
            bound = float(((tol + UB * ref.abs() + (ref - ref2).abs()) * v.abs()).sum())
            assert abs(got - slope) <= bound + 1e-6 * float((ref.abs() * v.abs()).sum())


def test_rows_do_not_mix(dd, ctx):
    """NaN and infinities in one token's row stay in that row of the results."""
    for T in (4, 40, 200):
        d, f = 136, 264
        x, w = mat(T, d, 1), [mat(f, d, 2, 0.1), mat(f, d, 3, 0.1), mat(d, f, 4, 0.1)]
        clean, dirty = mat(T, d, 5), mat(T, d, 6)
        ctx.gated_ffn_forward(x, *w, clean)
        x2 = x.clone()
        x2[1, 5], x2[3, 7] = float("nan"), float("inf")
        ctx.gated_ffn_forward(x2, *w, dirty)
        keep = [t for t in range(T) if t not in (1, 3)]
        assert torch.equal(clean[keep], dirty[keep])
        assert bool(torch.isnan(dirty[1].float()).all()) and not bool(torch.isfinite(dirty[3].float()).any())


@pytest.mark.parametrize("scale", [30.0, 3e4])
def test_large_arguments(dd, ctx, scale):
    """Gates far out on both sides: the activation saturates without overflow or NaN."""
    T, d, f = 33, 64, 128
    for act in (0, 1):
        x, w = mat(T, d, 1, scale), [mat(f, d, 2), mat(f, d, 3, 0.1), mat(d, f, 4, 0.1)]
        y, gate, up = mat(T, d, 5), mat(T, f, 6), mat(T, f, 7)
        ctx.gated_ffn_forward(x, *w, y, activation=act, gate=gate, up=up)
        assert bool(torch.isfinite(y.float()).all())
        dx, dws = mat(T, d, 8), [mat(f, d, 9), mat(f, d, 10), mat(d, f, 11)]
        ctx.gated_ffn_backward(x, *w, gate, up, mat(T, d, 12), dx, *dws, activation=act)
        assert all(bool(torch.isfinite(t.float()).all()) for t in (dx, *dws))


def test_no_tokens(dd, ctx):
    d, f = 24, 40
    w = [mat(f, d, 1), mat(f, d, 2), mat(d, f, 3)]
    x, g = torch.empty(0, d, dtype=B, device="cuda"), torch.empty(0, f, dtype=B, device="cuda")
    ctx.gated_ffn_forward(x, *w, torch.empty_like(x), gate=g, up=torch.empty_like(g))
    for acc in (True, False):
        dws = [mat(f, d, 4), mat(f, d, 5), mat(d, f, 6)]
        before = [t.clone() for t in dws]
        ctx.gated_ffn_backward(x, *w, g, g, x, torch.empty_like(x), *dws, accumulate=acc)
        assert all(torch.equal(t, b) if acc else not bool(t.any()) for t, b in zip(dws, before))


def test_other_stream_caller_scratch_and_graph(dd, ctx):
    T, d, f = 50, 72, 100
    x, w = mat(T, d, 1), [mat(f, d, 2, 0.1), mat(f, d, 3, 0.1), mat(d, f, 4, 0.1)]
    y = mat(T, d, 5)
    ctx.gated_ffn_forward(x, *w, y)
    hidden = torch.empty(T * rows8(f), dtype=B, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y2 = mat(T, d, 6)
    torch.cuda.synchronize()
    ctx.gated_ffn_forward(x, *w, y2, hidden=hidden, stream=side)
    side.synchronize()
    assert torch.equal(y, y2)
    gate, up, dy = mat(T, f, 7), mat(T, f, 8), mat(T, d, 9)
    outs = [mat(T, d, 10), mat(f, d, 11), mat(f, d, 12), mat(d, f, 13)]
    scratch = torch.empty(3 * T * rows8(f), dtype=B, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.gated_ffn_forward(x, *w, y2, hidden=hidden, gate=gate, up=up)
        ctx.gated_ffn_backward(x, *w, gate, up, dy, *outs, scratch=scratch)
    x.mul_(0.5)
    graph.replay()
    ctx.gated_ffn_forward(x, *w, y)
    assert torch.equal(y, y2)
    again = [mat(T, d, 14), mat(f, d, 15), mat(f, d, 16), mat(d, f, 17)]
    ctx.gated_ffn_backward(x, *w, gate, up, dy, *again)
    assert all(torch.equal(a, b) for a, b in zip(outs, again))
    del graph


def test_refusals(dd, ctx):
    T, d, f = 16, 32, 48
    x, w, y = mat(T, d, 1), [mat(f, d, 2), mat(f, d, 3), mat(d, f, 4)], mat(T, d, 5)
    gate, up = mat(T, f, 6), mat(T, f, 7)

    def refused(rc, call):
        with pytest.raises(dd.DDMergeError) as e:
            call()
        assert e.value.rc == rc

    refused(dd.ERR_INVALID_ARG, lambda: ctx.gated_ffn_forward(x, *w, y, activation=7))
    refused(dd.ERR_INVALID_ARG, lambda: ctx.gated_ffn_forward(x, *w, y, gate=gate))
    refused(dd.ERR_ALIAS, lambda: ctx.gated_ffn_forward(x, *w, x))
    refused(dd.ERR_ALIAS, lambda: ctx.gated_ffn_forward(x, *w, y, gate=gate, up=gate))
    odd = torch.zeros(T, 33, dtype=B, device="cuda")
    refused(dd.ERR_ALIGNMENT, lambda: ctx.gated_ffn_forward(odd[:, :d], *w, y))
    off = torch.zeros(T * 40 + 8, dtype=B, device="cuda")[1:1 + T * 40].view(T, 40)[:, :d]
    refused(dd.ERR_ALIGNMENT, lambda: ctx.gated_ffn_forward(off, *w, y))
    grads = [mat(f, d, 8), mat(f, d, 9), mat(d, f, 10)]
    refused(dd.ERR_ALIAS, lambda: ctx.gated_ffn_backward(x, *w, gate, up, y, x, *grads))
    refused(dd.ERR_ALIAS, lambda: ctx.gated_ffn_backward(x, *w, gate, up, y, mat(T, d, 11), grads[0], grads[0], grads[2]))
    for call in (lambda: ctx.gated_ffn_forward(x.float(), *w, y), lambda: ctx.gated_ffn_forward(x, w[0], w[1], w[0], y),
                 lambda: ctx.gated_ffn_forward(x, w[0], w[1][:40], w[2], y), lambda: ctx.gated_ffn_forward(x.t(), *w, y),
                 lambda: ctx.gated_ffn_forward(x, *w, y, residual=mat(T, d, 1, pad=1)),
                 lambda: ctx.gated_ffn_backward(x, *w, gate, up, y, mat(T, d, 11, pad=1), *grads),
                 lambda: ctx.gated_ffn_backward(x, *w, gate, up, y, mat(T, d, 11), grads[0].float(), *grads[1:])):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("tokens", [5, 400])
def test_bounded_waits_expire(dd, ctx, tokens):
    """The test hook holds back the first copies: the waits run out, the status word says so, and
    the next call on the same context is right."""
    d, f = 136, 264
    x, w = mat(tokens, d, 1), [mat(f, d, 2, 0.1), mat(f, d, 3, 0.1), mat(d, f, 4, 0.1)]
    y, gate, up = mat(tokens, d, 5), mat(tokens, f, 6), mat(tokens, f, 7)
    outs = [mat(tokens, d, 8), mat(f, d, 9), mat(f, d, 10), mat(d, f, 11)]
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    ctx.gated_ffn_forward(x, *w, y, gate=gate, up=up, status=status[:1], flags=dd.DEBUG_EXPIRE_WAIT)
    ctx.gated_ffn_backward(x, *w, mat(tokens, f, 6), mat(tokens, f, 7), mat(tokens, d, 12), *outs, status=status[1:],
                           flags=dd.DEBUG_EXPIRE_WAIT)
    torch.cuda.synchronize()
    assert status.tolist() == [dd.STATUS_WAIT_LIMIT] * 2
    status.zero_()
    ctx.gated_ffn_forward(x, *w, y, gate=gate, up=up, status=status[:1])
    for got, (ref, tol) in zip((y, gate, up), forward64(x, *w, None, 0)):
        within(got, ref, tol, "after the expiry")
    ctx.gated_ffn_backward(x, *w, gate, up, mat(tokens, d, 12), *outs, status=status[1:])
    for got, (ref, tol) in zip(outs, backward64(x, *w, gate, up, mat(tokens, d, 12), 0)):
        within(got, ref, tol * (1 + UB) + UB * ref.abs(), "after the expiry")
    assert status.tolist() == [0, 0]


def test_beyond_32_bit_offsets(dd, ctx):
    """gate, up and the intermediates of 270,000 tokens x 8192 lie past 2^32 bytes: the last rows
    against float64, and against the first rows, which hold the same tokens."""
    T, d, f = 270_000, 64, 8192
    rows = mat(300, d, 1)
    w = [mat(f, d, 2, 0.1), mat(f, d, 3, 0.1), mat(d, f, 4, 0.02)]
    x = rows.repeat(T // 300, 1)
    y, gate, up = torch.empty_like(x), torch.empty(T, f, dtype=B, device="cuda"), torch.empty(T, f, dtype=B, device="cuda")
    ctx.gated_ffn_forward(x, *w, y, gate=gate, up=up)
    for got, (ref, tol) in zip((y, gate, up), forward64(rows, *w, None, 0)):
        within(got[-300:], ref, tol, "last rows")
        within(got[:300], ref, tol, "first rows")
    dy = torch.zeros_like(x)
    dy[-1] = 1.0
    dx, dws = torch.empty_like(x), [torch.empty_like(t) for t in w]
    ctx.gated_ffn_backward(x, *w, gate, up, dy, dx, *dws)
    want = backward64(rows[-1:], *w, gate[-1:], up[-1:], dy[-1:], 0)
    for got, (ref, tol), what in zip((dx[-1:], *dws), want, ("dx", "dw_gate", "dw_up", "dw_down")):
        within(got, ref, tol * (1 + UB) + UB * ref.abs(), what)
    assert not bool(dx[:-1].any())
