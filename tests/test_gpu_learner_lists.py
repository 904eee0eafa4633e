"""Global gradient norm, clipping and the AdamW step over lists of tensors, against float64.

Tolerances follow from the arithmetic (u = 2^-24): the norm takes at most 32 squares in float32
before float64, so norm^2 is within 34 u relative; a scaled gradient carries the scale's error and
one product; AdamW's bound is written out in ``adamw_reference``.
"""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
UB = 2.0 ** -8            # unit roundoff of bf16


@pytest.fixture(scope="module")
def dd():
    from paper_2604_21428_b200 import ddmerge
    return ddmerge


@pytest.fixture(scope="module")
def ctx(dd):
    c = dd.Context(0)
    yield c
    c.close()


def make(sizes, dtypes, seed, std=1e-2, shift=0):
    """Device tensors, each ``shift`` elements off its allocation's alignment."""
    g = torch.Generator().manual_seed(seed)
    out = []
    for n, dt in zip(sizes, dtypes):
        buf = torch.full((n + shift + 3,), float("nan"), dtype=dt, device="cuda")
        buf[shift:shift + n] = (torch.randn(n, generator=g) * std).to(dt)
        out.append(buf[shift:shift + n])
    return out


def exact_norm(ts):
    return math.sqrt(sum(float(t.double().square().sum()) for t in ts))


def check_record(dd, rec, ts, max_norm):
    r = dd.read_grad_record(rec)
    norm = exact_norm(ts)
    assert r.status == dd.STATUS_OK
    assert abs(r.norm_sq - norm * norm) <= 34 * U * norm * norm
    assert abs(r.norm - norm) <= 20 * U * norm
    want = min(1.0, max_norm / (norm + 1e-6))
    assert abs(r.scale - want) <= 24 * U * want
    return r


F, B = torch.float32, torch.bfloat16
LISTS = [
    ([], []),
    ([0], [F]),
    ([1], [B]),
    ([1, 0, 2, 3], [F, B, B, F]),
    ([8191, 8192, 8193], [F, B, F]),
    ([5, 100_003, 16_384, 7, 70_000], [B, B, F, F, B]),
    ([1000 + 37 * k for k in range(33)], [F, B, B] * 11),             # past the short list's capacity
    ([17 + (k * 7919) % 9001 for k in range(300)], [B, F] * 150),     # two launches
    ([3 * 8192 * 1184 + 5], [B]),                                     # every CTA takes several tiles
]


@pytest.mark.parametrize("shift", [0, 1])
@pytest.mark.parametrize("case", range(len(LISTS)))
def test_norm(dd, ctx, case, shift):
    sizes, dtypes = LISTS[case]
    ts = make(sizes, dtypes, 10 + case, shift=shift)
    rec = dd.new_grad_record()
    for max_norm in (1.0, 0.0, math.inf, 1e-3):
        ctx.grad_norm(ts, max_norm, rec)
        check_record(dd, rec, ts, max_norm)
    first = rec.clone()
    ctx.grad_norm(ts, 1e-3, rec)
    assert torch.equal(first.view(torch.int32), rec.view(torch.int32))       # same bits again


@pytest.mark.parametrize("in_place", [True, False])
@pytest.mark.parametrize("max_norm", [1e-4, 1e6, 0.0])
@pytest.mark.parametrize("case", range(len(LISTS)))
def test_clip(dd, ctx, case, max_norm, in_place):
    sizes, dtypes = LISTS[case]
    shift = case % 2
    ts = make(sizes, dtypes, 40 + case, shift=shift)
    ref = [t.clone() for t in ts]
    out = None if in_place else make(sizes, dtypes, 99, shift=(case // 2) % 2)
    rec = dd.new_grad_record()
    ctx.clip_gradients(ts, max_norm, rec, out=out)
    r = check_record(dd, rec, ref, max_norm)
    for got, src in zip(ts if in_place else out, ref):
        want = src.double() * float(r.scale)
        tol = (UB if src.dtype == B else U) * want.abs() + 1e-45
        assert bool(((got.double() - want).abs() <= tol).all())
    if not in_place:
        assert all(torch.equal(a, b) for a, b in zip(ts, ref))
    if max_norm == 1e6:                      # scale 1: the very same values
        assert all(torch.equal(a, b) for a, b in zip(ts if in_place else out, ref))


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf, 1e30])
def test_non_finite_norm_writes_nothing(dd, ctx, bad):
    """1e30 squares past float32: reported like an infinite gradient."""
    ts = make([5000, 9, 20_000], [F, B, B], 7)
    ts[1][3] = bad
    ref = [t.clone() for t in ts]
    params, m, v = make([5000, 9, 20_000], [F] * 3, 8), make([5000, 9, 20_000], [F] * 3, 9), make([5000, 9, 20_000], [F] * 3, 10)
    copies = make([5000, 9, 20_000], [B] * 3, 11)
    before = [t.clone() for t in params + m + v + copies]
    rec = dd.new_grad_record()
    ctx.clip_gradients(ts, 1.0, rec)
    r = dd.read_grad_record(rec)
    assert r.status == dd.STATUS_NONFINITE and r.scale == 1.0 and not math.isfinite(r.norm)
    assert all(torch.equal(a.nan_to_num(1.0), b.nan_to_num(1.0)) for a, b in zip(ts, ref))
    ctx.adamw_step(params, ts, m, v, 1, 1e-3, copies=copies, clip=rec)
    assert all(torch.equal(a, b) for a, b in zip(params + m + v + copies, before))
    ctx.grad_norm(ref[:1], 1.0, rec)                       # the record recovers
    check_record(dd, rec, ref[:1], 1.0)


def adamw_reference(p, g, m, v, step, lr, b1, b2, eps, wd, scale):
    """Float64 results and error bounds.  m: two products, one sum, the constants' roundings (4 u of
    the terms' sizes); v: five factors (6 u of v); p: the quotient within 10 u plus what m brings,
    the product with the decay and the final sum within 2 u."""
    p, g, m, v = (t.double().cpu() for t in (p, g, m, v))
    g = g * scale
    m1 = b1 * m + (1 - b1) * g
    em = 4 * U * ((b1 * m).abs() + ((1 - b1) * g).abs()) + 1e-45
    v1 = b2 * v + (1 - b2) * g * g
    ev = 6 * U * v1 + 1e-45
    den = (v1 / (1 - b2 ** step)).sqrt() + eps
    st = lr / (1 - b1 ** step)
    upd = st * m1 / den
    p1 = p * (1 - lr * wd) - upd
    ep = 2 * U * (p.abs() + upd.abs()) + 10 * U * upd.abs() + st * em / den + 1e-45
    return (p1, ep), (m1, em), (v1, ev)


@pytest.mark.parametrize("with_clip", [False, True])
@pytest.mark.parametrize("case", range(1, len(LISTS) - 1))
def test_adamw(dd, ctx, case, with_clip):
    sizes, dtypes = LISTS[case]
    P = len(sizes)
    shifts = [0, case % 2, 0, 0]
    params, m = make(sizes, [F] * P, 1, 0.02, shifts[0]), make(sizes, [F] * P, 2, 1e-3, shifts[1])
    v = [t.square() for t in make(sizes, [F] * P, 3, 1e-2)]
    grads = make(sizes, dtypes, 4, 1e-2, case % 3)
    copies = make(sizes, [B] * P, 5)
    copies = [None if i % 5 == 3 else c for i, c in enumerate(copies)]
    kw = dict(beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1)
    for step in (1, 2, 1000):
        rec, scale = None, 1.0
        if with_clip:
            rec = dd.new_grad_record()
            ctx.grad_norm(grads, 0.05, rec)
            scale = float(dd.read_grad_record(rec).scale)
        want = [adamw_reference(p, g, a, b, step, 3e-3, 0.9, 0.95, 1e-8, 0.1, scale)
                for p, g, a, b in zip(params, grads, m, v)]
        ctx.adamw_step(params, grads, m, v, step, 3e-3, copies=copies, clip=rec, **kw)
        for i in range(P):
            for got, (ref, tol) in zip((params[i], m[i], v[i]), want[i]):
                assert bool(((got.double().cpu() - ref).abs() <= tol).all())
            if copies[i] is not None:
                assert torch.equal(copies[i], params[i].to(B))


def test_adamw_extremes(dd, ctx):
    """No decay, zero gradients and moments (0 / eps), betas of zero, a million steps."""
    n = 12_345
    p, g = make([n], [F], 1)[0], torch.zeros(n, device="cuda")
    m, v = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    before = p.clone()
    ctx.adamw_step([p], [g], [m], [v], 1, 1e-3)
    assert torch.equal(p, before) and not m.any() and not v.any()
    g = make([n], [F], 2)[0]
    for b1, b2, step in ((0.0, 0.0, 1), (0.9, 0.999, 1_000_000)):
        want = adamw_reference(p, g, m, v, step, 1e-3, b1, b2, 1e-8, 0.0, 1.0)
        ctx.adamw_step([p], [g], [m], [v], step, 1e-3, beta1=b1, beta2=b2)
        for got, (ref, tol) in zip((p, m, v), want):
            assert bool(((got.double().cpu() - ref).abs() <= tol).all())


def test_on_another_stream_and_under_a_graph(dd, ctx):
    sizes, dtypes = LISTS[5]
    ts = make(sizes, dtypes, 3)
    rec = dd.new_grad_record()
    ctx.grad_norm(ts, 1.0, rec)                            # workspace
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = [torch.zeros_like(t) for t in ts]
    ctx.clip_gradients(ts, 0.5, rec, out=out, stream=side)
    side.synchronize()
    check_record(dd, rec, ts, 0.5)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ctx.clip_gradients(ts, 0.25, rec, out=out)
    for _ in range(2):
        ts[0].mul_(2)
        graph.replay()
        r = check_record(dd, rec, ts, 0.25)
        want = ts[1].double() * float(r.scale)
        assert bool(((out[1].double() - want).abs() <= UB * want.abs()).all())
    del graph


def test_refusals(dd, ctx):
    a, b, m, v = (torch.zeros(64, device="cuda") for _ in range(4))
    rec = dd.new_grad_record()

    def refused(rc, call):
        with pytest.raises(dd.DDMergeError) as e:
            call()
        assert e.value.rc == rc

    refused(dd.ERR_INVALID_ARG, lambda: ctx.grad_norm([a], -1.0, rec))
    refused(dd.ERR_INVALID_ARG, lambda: ctx.grad_norm([a], math.nan, rec))
    refused(dd.ERR_INVALID_ARG, lambda: ctx.grad_norm([a], 1.0, None))
    refused(dd.ERR_ALIGNMENT, lambda: ctx.grad_norm([a], 1.0, rec[1:]))
    refused(dd.ERR_ALIAS, lambda: ctx.clip_gradients([a[:32]], 1.0, rec, out=[a[16:48]]))
    for kw in (dict(step=0), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0), dict(lr=math.inf), dict(weight_decay=math.nan)):
        args = dict(step=1, lr=1e-3) | kw
        step, lr = args.pop("step"), args.pop("lr")
        refused(dd.ERR_INVALID_ARG, lambda: ctx.adamw_step([a], [b], [m], [v], step, lr, **args))
    refused(dd.ERR_ALIAS, lambda: ctx.adamw_step([a], [b], [m], [m], 1, 1e-3))
    refused(dd.ERR_ALIAS, lambda: ctx.adamw_step([a], [a], [m], [v], 1, 1e-3))
    for call in (lambda: ctx.grad_norm([a.half()], 1.0, rec), lambda: ctx.grad_norm([a.view(8, 8).t()], 1.0, rec),
                 lambda: ctx.clip_gradients([a], 1.0, rec, out=[b[:5]]),
                 lambda: ctx.adamw_step([a], [b], [m.to(B)], [v], 1, 1e-3),
                 lambda: ctx.adamw_step([a], [b], [m], [v], 1, 1e-3, copies=[a])):
        with pytest.raises(ValueError):
            call()
    assert not a.any() and not m.any()


def test_beyond_32_bit_byte_offsets(dd, ctx):
    """One tensor of 2^31 + 8195 bf16 elements: byte offsets past 2^32, element offsets past 2^31."""
    n = 2 ** 31 + 8195
    g = torch.zeros(n, dtype=B, device="cuda")
    g[-3:] = 3.0
    g[2 ** 31 - 1] = 4.0
    rec = dd.new_grad_record()
    ctx.clip_gradients([g], 1.0, rec)
    r = dd.read_grad_record(rec)
    norm = math.sqrt(27 + 16)
    assert abs(r.norm - norm) <= 20 * U * norm
    assert torch.equal(g[-4:].float().cpu(), torch.tensor([0, 3 * r.scale, 3 * r.scale, 3 * r.scale]).to(B).float())
    assert float(g[2 ** 31 - 1]) == float(torch.tensor(4 * r.scale).to(B))
