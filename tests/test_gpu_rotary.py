"""Rotary positions against float64.

Bound: the reduced turn is at most 1/2 and rounded to float32 (2^-26 turns, 2^-23 radians), sine and cosine to 2 ulp,
the magnitude, its product and the three operations of a result a rounding each: together below
2^-21 of |a| + |b| times the magnitude; then the result's own rounding.
"""
import pytest
import torch

from decoder_util import B, U, UB, within

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


def turned64(x, positions, f, magnitude, interleaved, inverse):
    """Results with bounds, before their rounding."""
    x, half = x.double(), f.numel()
    w = positions.double()[:, None, None] * f.double() * (-1 if inverse else 1)
    a, b = (x[..., 0:2 * half:2], x[..., 1:2 * half:2]) if interleaved else (x[..., :half], x[..., half:2 * half])
    ra, rb = magnitude * (a * w.cos() - b * w.sin()), magnitude * (b * w.cos() + a * w.sin())
    e = abs(magnitude) * (a.abs() + b.abs()) * 2.0 ** -21
    join = (lambda u, v: torch.stack([u, v], -1).flatten(-2)) if interleaved else (lambda u, v: torch.cat([u, v], -1))
    rest = x[..., 2 * half:]
    return torch.cat([join(ra, rb), rest], -1), torch.cat([join(e, e), torch.zeros_like(rest)], -1)


SIZES = [(1, 1, 0, 2, 2), (1, 3, 1, 64, 64), (7, 2, 2, 9, 6), (33, 5, 2, 40, 20), (64, 12, 12, 64, 64), (129, 4, 1, 96, 48),
         (1000, 16, 4, 128, 128), (5, 70, 3, 1024, 1024), (3, 2000, 1, 16, 8), (9000, 1, 1, 24, 24)]


@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dtype", [B, torch.float32])
@pytest.mark.parametrize("size", SIZES, ids=str)
def test_against_float64(dd, ctx, size, dtype, interleaved, inverse):
    T, h, kv, dim, part = size
    gen = torch.Generator(device="cuda").manual_seed(T + dim)
    q, k = (torch.randn(T, n, dim, generator=gen, device="cuda").to(dtype) for n in (h, max(kv, 1)))
    positions = torch.randint(0, 1 << 20, (T,), generator=gen, device="cuda", dtype=torch.int64 if T % 2 else torch.int32)
    f, magnitude = dd.rotary_frequencies(part, factor=4.0, trained=4096)
    qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
    ctx.rotary(q, k if kv else None, positions, f, q_out=qo, k_out=ko if kv else None, magnitude=magnitude, interleaved=interleaved, inverse=inverse)
    unit = UB if dtype == B else U
    for name, x, y in (("q", q, qo), ("k", k, ko))[: 2 if kv else 1]:
        want, e = turned64(x, positions, f, magnitude, interleaved, inverse)
        within(y, want, e * (1 + unit) + unit * want.abs(), name)
        assert torch.equal(y[..., part:], x[..., part:])
    ctx.rotary(q, k if kv else None, positions, f, magnitude=magnitude, interleaved=interleaved, inverse=inverse)   # in place
    assert torch.equal(q, qo) and (not kv or torch.equal(k, ko))


@pytest.mark.parametrize("interleaved", [False, True])
def test_rows_of_one_buffer_and_tokens_that_are_none(dd, ctx, interleaved):
    """Queries and keys as parts of a projection's rows, at an odd offset for once, and heads before tokens;
    what lies between and rows of negative positions stay as they are."""
    f, _ = dd.rotary_frequencies(32)
    for start in (0, 1):
        buf = torch.randn(50, 8 * 32 + 40, device="cuda").to(B)
        q, k = (buf[:, start + a: start + b].unflatten(1, (-1, 32)) for a, b in ((0, 4 * 32), (4 * 32, 6 * 32)))
        positions = torch.arange(50, device="cuda") - 3
        before, want = buf.clone(), [turned64(x.clone(), positions, f, 1.0, interleaved, False) for x in (q, k)]
        ctx.rotary(q, k, positions, f, interleaved=interleaved)
        for x, (w, e) in zip((q, k), want):
            within(x[3:], w[3:], (e + UB * w.abs())[3:], "rows")
        assert torch.equal(buf[:3], before[:3])
        assert torch.equal(buf[:, start + 6 * 32:], before[:, start + 6 * 32:]) and torch.equal(buf[:, :start], before[:, :start])
    heads_first = torch.randn(4, 50, 32, device="cuda").to(B).transpose(0, 1)
    positions = torch.arange(50, device="cuda")
    want, e = turned64(heads_first.clone(), positions, f, 1.0, interleaved, False)
    ctx.rotary(heads_first, None, positions, f, interleaved=interleaved)
    within(heads_first, want, e + UB * want.abs(), "heads first")


def test_gradient_is_the_inverse_rotation(dd, ctx):
    """<g, R x> = <R^T g, x> for the linear map R: in float32 both sides are sums of the same products."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, g = (torch.randn(40, 3, 48, generator=gen, device="cuda") for _ in range(2))
    positions = torch.randint(0, 100_000, (40,), generator=gen, device="cuda")
    f, _ = dd.rotary_frequencies(32)
    y, dx = torch.empty_like(x), torch.empty_like(x)
    ctx.rotary(x, None, positions, f, q_out=y, magnitude=1.3)
    ctx.rotary(g, None, positions, f, q_out=dx, magnitude=1.3, inverse=True)
    a, b = (y.double() * g.double()).sum(), (dx.double() * x.double()).sum()
    size = 4 * 1.3 * (x.double().abs().amax() * g.double().abs()).sum()
    assert abs(float(a - b)) <= 2.0 ** -20 * float(size)


def test_refusals(dd, ctx):
    f, _ = dd.rotary_frequencies(8)
    q = torch.zeros(4, 2, 16, device="cuda", dtype=B)
    p = torch.zeros(4, device="cuda", dtype=torch.int32)
    for bad in (dict(q=q.half()), dict(q=q[..., ::2]), dict(q=q[0]), dict(q=q[:, :1].expand(4, 2, 16)), dict(positions=p[:3]),
                dict(positions=p.float()), dict(f=f.float()), dict(q=q.cpu())):
        args = dict(q=q, positions=p, f=f) | bad
        with pytest.raises(ValueError):
            ctx.rotary(args["q"], None, args["positions"], args["f"])
    with pytest.raises(ValueError):
        ctx.rotary(q, None, p, f, k_out=q)
    wide = torch.zeros(9, device="cuda", dtype=torch.float64)                        # 18 of 16 elements
    with pytest.raises(dd.DDMergeError):
        ctx.rotary(q, None, p, wide)
    flat = torch.zeros(5 * 32, device="cuda", dtype=B)
    with pytest.raises(dd.DDMergeError) as e:                                        # shifted by one token
        ctx.rotary(flat[:128].view(4, 2, 16), None, p, f, q_out=flat[32:160].view(4, 2, 16))
    assert e.value.rc == dd.ERR_ALIAS
    with pytest.raises(dd.DDMergeError):
        ctx.rotary(q, q, p, f)
    ctx.rotary(q[:0], None, p[:0], f)
