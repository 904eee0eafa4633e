"""Attention over packed sequences, forward and backward, against float64 (bounds in decoder_util)."""
import math

import pytest
import torch

from decoder_util import B, U, UB, attention64, attention_back64, within

pytestmark = pytest.mark.gpu
NAN = float("nan")


@pytest.fixture(scope="module")
def dd():
    from paper_2604_21428_b200 import ddmerge
    return ddmerge


@pytest.fixture(scope="module")
def ctx(dd):
    c = dd.Context(0)
    yield c
    c.close()


class Case:
    """Queries, keys and values in the rows of one buffer; NaN in rows outside the documents and between the heads."""

    def __init__(self, lengths, heads, kv, dim, seed=0, before=0, after=0, std=1.0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.T = before + sum(lengths) + after
        ends = [before]
        for n in lengths:
            ends.append(ends[-1] + n)
        self.docs = [slice(a, b) for a, b in zip(ends, ends[1:]) if b > a]
        self.offsets = torch.tensor(ends, dtype=torch.int32, device="cuda")
        self.inside = torch.zeros(self.T, dtype=torch.bool, device="cuda")
        self.inside[before: before + sum(lengths)] = True

        def rows(n, std=std):
            buf = torch.full((self.T, n, dim + 8), NAN, device="cuda")
            buf[..., :dim] = torch.randn(self.T, n, dim, generator=gen, device="cuda") * std
            buf[~self.inside] = NAN
            return buf.to(B)[..., :dim]

        qkv = rows(heads + 2 * kv)
        self.q, self.k, self.v = qkv[:, :heads], qkv[:, heads: heads + kv], qkv[:, heads + kv:]
        self.d_o = rows(heads, 1e-2)
        self.o = torch.full((self.T, heads, dim), NAN, dtype=B, device="cuda")
        self.lse = torch.full((heads, self.T), NAN, device="cuda")
        grads = torch.full((self.T, heads + 2 * kv, dim), NAN, dtype=B, device="cuda")
        self.dq, self.dk, self.dv = grads[:, :heads], grads[:, heads: heads + kv], grads[:, heads + kv:]
        self.scale = 1 / math.sqrt(dim)

    def forward(self, ctx, **kw):
        ctx.attention_forward(self.q, self.k, self.v, self.o, self.lse, **{"offsets": self.offsets, **kw})

    def backward(self, ctx, **kw):
        ctx.attention_backward(self.q, self.k, self.v, self.o, self.lse, self.d_o, self.dq, self.dk, self.dv, **{"offsets": self.offsets, **kw})

    def check(self, causal, scale=None):
        scale = scale or self.scale
        for d in self.docs:
            (o, eo), (lse, el) = attention64(self.q[d], self.k[d], self.v[d], scale, causal)
            within(self.o[d], o, eo, f"o {d}")
            within(self.lse[:, d], lse, el, f"lse {d}")
        assert bool(self.o[~self.inside].isnan().all()) and bool(self.lse[:, ~self.inside].isnan().all())

    def check_back(self, causal, scale=None):
        for d in self.docs:
            n = d.stop - d.start
            tiled = 128 if causal else n if n <= 128 else 0
            want = attention_back64(self.q[d], self.k[d], self.v[d], self.o[d], self.d_o[d], scale or self.scale, causal, tiled)
            for name, x, (r, e) in zip(("dq", "dk", "dv"), (self.dq, self.dk, self.dv), want):
                within(x[d], r, e, f"{name} {d}")
        for x in (self.dq, self.dk, self.dv):
            assert bool(x[~self.inside].isnan().all())


SHAPES = [([1], 1, 1, 64), ([1], 2, 1, 128), ([2], 1, 1, 8), ([3, 1, 2], 2, 2, 16), ([127], 2, 1, 64), ([128], 1, 1, 128), ([129], 3, 1, 128),
          ([255], 2, 2, 40), ([256], 1, 1, 64), ([257], 2, 1, 128), ([0, 5, 0, 0, 130, 257, 0], 4, 2, 128), ([64] * 9, 3, 3, 72), ([700, 33], 6, 2, 80),
          ([1000], 2, 1, 64), ([513, 1, 384], 8, 1, 128), ([1], 64, 8, 64), (list(range(40)), 2, 2, 24), ([1500], 1, 1, 96)]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_against_float64(ctx, shape, causal):
    c = Case(*shape, before=3, after=5)
    c.forward(ctx, causal=causal)
    c.check(causal)
    c.backward(ctx, causal=causal)
    c.check_back(causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128])
def test_many_more_tiles_than_the_gpu_takes_at_once(ctx, dim, causal):
    """Documents of whole and cut tiles, of one tile of queries and of more, in turn; every third one is NaN throughout, its
    neighbours are not; the same bits twice."""
    lengths = [(37 * i) % 300 for i in range(45)] + [640, 128, 256, 1, 700, 384, 128, 128, 255]
    c = Case(lengths, 16, 4, dim, seed=dim, before=2, after=3)
    for d in c.docs[1::3]:
        c.q[d], c.k[d], c.v[d], c.d_o[d] = NAN, NAN, NAN, NAN
    bad = torch.zeros_like(c.inside)
    for d in c.docs[1::3]:
        bad[d] = True
    c.forward(ctx, causal=causal)
    c.backward(ctx, causal=causal)
    first = [t.clone().view(torch.int16) for t in (c.o, c.dq, c.dk, c.dv)]
    for t in (c.o, c.dq, c.dk, c.dv):
        t[c.inside] = 7.0
    c.forward(ctx, causal=causal)
    c.backward(ctx, causal=causal)
    good = c.inside & ~bad
    assert all(torch.equal(a[good], b.view(torch.int16)[good]) for a, b in zip(first, (c.o, c.dq, c.dk, c.dv)))
    assert bool(c.o[bad].isnan().all())
    c.docs = [d for i, d in enumerate(c.docs) if i % 3 != 1]
    c.check(causal)
    c.check_back(causal)


@pytest.mark.parametrize("std", [4.0, 12.0])
def test_sharp_rows(ctx, std):
    """Scores of hundreds: most weights vanish, and the maximum grows from tile to tile."""
    c = Case([600, 90], 2, 1, 64, std=std)
    order = torch.arange(600, device="cuda")
    c.k[:600] = (c.k[:600].float() * (0.2 + order / 600.0)[:, None, None]).to(B)
    c.forward(ctx)
    c.check(True)
    c.backward(ctx)
    c.check_back(True)


def test_scores_far_below_zero(ctx):
    """All scores of a row near -1e4: their maximum is what the exponents are taken against."""
    c = Case([300], 1, 1, 64)
    c.q[:] = (c.q.float().abs() * 20).to(B)
    c.k[:] = (-c.k.float().abs() * 20).to(B)
    c.forward(ctx)
    c.check(True)


@pytest.mark.parametrize("causal", [True, False])
def test_one_sequence_without_offsets(ctx, causal):
    c = Case([390], 4, 2, 64)
    c.forward(ctx, causal=causal, offsets=None, scale=0.2)
    c.check(causal, scale=0.2)
    c.backward(ctx, causal=causal, offsets=None, scale=0.2)
    c.check_back(causal, scale=0.2)


def test_heads_before_tokens_and_no_lse(ctx):
    """[heads, tokens, dim] in memory, each tensor with strides of its own; without lse."""
    c = Case([200, 100], 4, 2, 64)
    want, lse = c.o.clone(), c.lse
    c.forward(ctx)
    want, c.lse = c.o.clone(), None
    q, k, v = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (c.q, c.k, c.v))
    o = torch.zeros(4, 300, 64, dtype=B, device="cuda").transpose(0, 1)
    ctx.attention_forward(q, k, v, o, None, offsets=c.offsets)
    assert torch.equal(o, want)
    c.lse = lse
    c.backward(ctx)
    grads = [torch.zeros(x.shape[1], 300, 64, dtype=B, device="cuda").transpose(0, 1) for x in (q, k, v)]
    ctx.attention_backward(q, k, v, o, lse, c.d_o, *grads, offsets=c.offsets)
    for a, b in zip(grads, (c.dq, c.dk, c.dv)):
        assert torch.equal(a, b)


def test_nan_stays_in_its_document(ctx):
    """A document of NaN and one of infinities between others change nothing in those."""
    lengths = [150, 60, 200, 70, 129]
    clean, dirty = Case(lengths, 2, 1, 128, seed=4), Case(lengths, 2, 1, 128, seed=4)
    for d, x in ((clean.docs[1], NAN), (clean.docs[3], math.inf)):
        for t in (dirty.q, dirty.k, dirty.v, dirty.d_o):
            t[d] = x
    for c in (clean, dirty):
        c.forward(ctx)
        c.backward(ctx)
    for d in (clean.docs[i] for i in (0, 2, 4)):
        for name in ("o", "dq", "dk", "dv"):
            assert torch.equal(getattr(clean, name)[d], getattr(dirty, name)[d]), name
        assert torch.equal(clean.lse[:, d], dirty.lse[:, d])
    assert bool(dirty.o[clean.docs[1]].isnan().all()) and bool(dirty.lse[:, clean.docs[1]].isnan().all())


@pytest.mark.parametrize("heads,kv", [(16, 1), (2, 2)])
def test_long_sequences_over_clusters(ctx, heads, kv):
    """Few heads of keys: the CTAs of a cluster share each tile of them."""
    c = Case([2100, 17, 900], heads, kv, 64 if kv == 2 else 128, seed=9)
    c.forward(ctx)
    c.check(True)
    c.backward(ctx)
    c.check_back(True)


def test_same_bits_every_time(ctx):
    c = Case([900, 333, 1], 8, 2, 128)
    results = []
    for _ in range(4):
        c.forward(ctx)
        c.backward(ctx)
        results.append([t.clone() for t in (c.o, c.lse, c.dq, c.dk, c.dv)])
    for r in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], r))


@pytest.mark.parametrize("lengths", [[1024] * 16, [4096] * 4, [2900, 17, 1, 1333, 0, 640, 2048, 999, 129, 65]], ids=str)
def test_no_wait_runs_out_in_many_calls(ctx, lengths):
    """A warp that is late may not miss a barrier's turn: many tiles, many times, without a status and with the same bits."""
    c = Case(lengths, 16, 4, 128)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    first = None
    for _ in range(40):
        for t in (c.o, c.dq, c.dk, c.dv):
            t.fill_(7.0)
        c.forward(ctx, status=status)
        c.backward(ctx, status=status)
        got = torch.cat([t.reshape(-1).view(torch.int16) for t in (c.o.clone(), c.dq.clone(), c.dk.clone(), c.dv.clone())])
        first = got if first is None else first
        assert torch.equal(first, got) and int(status) == 0


def test_captured_calls_take_new_lengths(dd, ctx):
    """Forward and backward in a graph with scratch of their own, on a stream of its own: replayed with other
    offsets, they give what eager calls give."""
    c, other = (Case(n, 4, 2, 64, seed=2, after=a) for n, a in (([100, 300, 50], 0), ([1, 440], 9)))
    scratch = torch.zeros(dd.attention_scratch_bytes(450, 4, 2, 64, 3, backward=True), dtype=torch.uint8, device="cuda")
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    c.forward(ctx, scratch=scratch)
    c.backward(ctx, scratch=scratch)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        c.forward(ctx, scratch=scratch)
        c.backward(ctx, scratch=scratch)
    for ends in ([0, 100, 400, 450], [0, 7, 7, 441], [3, 130, 131, 450]):
        c.offsets.copy_(torch.tensor(ends, dtype=torch.int32))
        for t in (c.o, c.dq, c.dk, c.dv):
            t.zero_()
        graph.replay()
        got = [t.clone() for t in (c.o, c.lse, c.dq, c.dk, c.dv)]
        for t in (c.o, c.dq, c.dk, c.dv):
            t.zero_()
        c.forward(ctx)
        c.backward(ctx)
        assert all(torch.equal(a, b) for a, b in zip(got, (c.o, c.lse, c.dq, c.dk, c.dv)))
    del graph, other


def test_bad_offsets_write_nothing(dd, ctx):
    c = Case([50, 50], 2, 1, 64)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for ends in ([0, 60, 50], [-1, 50, 100], [0, 50, 101], [0, 2 ** 31 - 1, 100]):
        c.offsets.copy_(torch.tensor(ends, dtype=torch.int32))
        status.zero_()
        c.forward(ctx, status=status)
        assert int(status) == dd.STATUS_BAD_OFFSETS and bool(c.o.isnan().all()) and bool(c.lse.isnan().all())
        status.zero_()
        c.backward(ctx, status=status)
        assert int(status) == dd.STATUS_BAD_OFFSETS and bool(c.dq.isnan().all()) and bool(c.dk.isnan().all())
    c.offsets.copy_(torch.tensor([0, 50, 100], dtype=torch.int32))
    status.zero_()
    c.forward(ctx, status=status)
    assert int(status) == 0
    c.check(True)


def test_a_wait_that_runs_out_is_reported(dd, ctx):
    c = Case([300, 40], 2, 1, 128)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    c.forward(ctx, status=status, flags=dd.DEBUG_EXPIRE_WAIT)
    assert int(status) == dd.STATUS_WAIT_LIMIT
    status.zero_()
    c.forward(ctx, status=status)
    c.backward(ctx, status=status)
    assert int(status) == 0
    c.check(True)
    c.check_back(True)
    c.backward(ctx, status=status, flags=dd.DEBUG_EXPIRE_WAIT)
    assert int(status) == dd.STATUS_WAIT_LIMIT
    status.zero_()
    c.forward(ctx, status=status)
    c.backward(ctx, status=status)
    assert int(status) == 0
    c.check_back(True)


def test_differences(ctx):
    """The gradients along a random direction against central differences of the float64 form."""
    c = Case([70, 30], 2, 1, 32, seed=6)
    c.forward(ctx)
    c.backward(ctx)
    gen = torch.Generator(device="cuda").manual_seed(1)

    def objective(q, k, v):
        total = 0.0
        for d in c.docs:
            (o, _), _ = attention64(q[d], k[d], v[d], c.scale, True)
            total = total + (o * c.d_o[d].double()).sum()
        return float(total)

    x = [t.double() for t in (c.q, c.k, c.v)]
    for i, g in enumerate((c.dq, c.dk, c.dv)):
        step = torch.randn(x[i].shape, generator=gen, device="cuda", dtype=torch.float64) * 1e-4
        plus, minus = ([t + (s * step if j == i else 0) for j, t in enumerate(x)] for s in (1, -1))
        want = (objective(*plus) - objective(*minus)) / 2
        size = float((g.double().square().sum() * step.square().sum()).sqrt())
        # a gradient's roundings (its operands and its own) are 2^-8 of its 2-norm at most each, o's beside
        assert abs(float((g.double() * step).sum()) - want) <= 3 * UB * size


def test_refusals(dd, ctx):
    c = Case([20], 4, 2, 64)
    with pytest.raises(ValueError):
        ctx.attention_forward(c.q.float(), c.k, c.v, c.o)
    with pytest.raises(ValueError):
        ctx.attention_forward(c.q, c.k, c.v[:10], c.o)
    with pytest.raises(ValueError):
        ctx.attention_forward(c.q, c.k[:, :1].expand(20, 2, 64), c.v, c.o)
    with pytest.raises(ValueError):
        c.forward(ctx, offsets=c.offsets.long())
    with pytest.raises(ValueError):
        c.forward(ctx, scratch=torch.zeros(1, dtype=torch.uint8, device="cuda"))
    for kw, rc in ((dict(scale=0.0), dd.ERR_INVALID_ARG), (dict(scale=-1.0), dd.ERR_INVALID_ARG), (dict(scale=NAN), dd.ERR_INVALID_ARG),
                   (dict(flags=1), dd.ERR_INVALID_ARG)):
        with pytest.raises(dd.DDMergeError) as e:
            c.forward(ctx, **kw)
        assert e.value.rc == rc
    z = [torch.zeros(20, n, d, dtype=B, device="cuda") for n, d in ((3, 64), (2, 64), (2, 136), (2, 12))]
    for t, rc in (((z[0], z[1], z[1], z[0]), dd.ERR_INVALID_ARG), ((z[2],) * 3 + (z[2].clone(),), dd.ERR_TOO_LARGE),
                  ((z[3],) * 3 + (z[3].clone(),), dd.ERR_INVALID_ARG), ((z[1],) * 4, dd.ERR_ALIAS)):
        with pytest.raises(dd.DDMergeError) as e:
            ctx.attention_forward(*t)
        assert e.value.rc == rc
    odd = torch.zeros(20 * 2 * 64 + 1, dtype=B, device="cuda")[1:].view(20, 2, 64)
    with pytest.raises(dd.DDMergeError) as e:
        ctx.attention_forward(odd, z[1], z[1], z[1].clone())
    assert e.value.rc == dd.ERR_ALIGNMENT
    with pytest.raises(dd.DDMergeError) as e:
        ctx.attention_backward(c.q, c.k, c.v, c.o, c.lse, c.d_o, c.dq, c.dk, c.dk)
    assert e.value.rc == dd.ERR_ALIAS
    for empty in (Case([], 2, 1, 64), Case([0, 0], 2, 1, 64, before=3, after=2), Case([], 2, 1, 64, after=4)):
        empty.forward(ctx)
        empty.backward(ctx)
        empty.check(True)
        empty.check_back(True)
