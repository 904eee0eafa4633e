"""The loss over the vocabulary and its gradients against float64 (bounds in decoder_util)."""
import pytest
import torch

from decoder_util import B, U, UB, loss64, loss_back64, within

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


def mat(gen, rows, cols, std=1.0, pad=8, dtype=B):
    """A matrix whose rows are longer than they need to be, NaN in between."""
    buf = torch.full((rows, (cols + 7) // 8 * 8 + pad), NAN, dtype=dtype, device="cuda")
    buf[:, :cols] = (torch.randn(rows, cols, generator=gen, device="cuda") * std).to(dtype)
    return buf[:, :cols]


def pads_untouched(t):
    full = t.as_strided((t.shape[0], t.stride(0)), (t.stride(0), 1))
    return bool(torch.isnan(full[:, t.shape[1]:].float()).all())


class Case:
    def __init__(self, T, d, V, seed=0, std=None, ignored=0.1):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.hidden, self.weight = mat(gen, T, d), mat(gen, V, d, std or 2.0 / d ** 0.5)
        self.targets = torch.randint(0, V, (T,), generator=gen, device="cuda")
        self.targets[torch.rand(T, generator=gen, device="cuda") < ignored] = -100
        self.loss, self.lse = (torch.full((T,), NAN, device="cuda") for _ in range(2))
        self.dloss = torch.rand(T, generator=gen, device="cuda") / T
        self.dhidden = torch.full_like(self.hidden.as_strided((T, self.hidden.stride(0)), (self.hidden.stride(0), 1)), NAN)[:, :d]

    def forward(self, ctx, **kw):
        ctx.vocab_loss_forward(self.hidden, self.weight, self.targets, self.loss, self.lse, **kw)

    def gradient(self, dtype, fill=NAN):
        V, d = self.weight.shape
        return torch.full((V, self.weight.stride(0)), fill, dtype=dtype, device="cuda")[:, :d]

    def backward(self, ctx, dweight, **kw):
        ctx.vocab_loss_backward(self.hidden, self.weight, self.targets, self.lse, self.dloss, self.dhidden, dweight, **kw)


SIZES = [(1, 8, 1), (1, 64, 100), (2, 40, 24), (3, 1, 1), (5, 128, 1000), (96, 768, 5000), (127, 72, 257), (128, 64, 128), (129, 136, 264),
         (300, 40, 255), (255, 333, 777), (257, 64, 70000), (777, 1001, 5003), (2000, 200, 3001), (4100, 64, 130), (1, 2048, 32000)]


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_against_float64(ctx, size):
    c = Case(*size)
    c.forward(ctx)
    (loss, e_loss), (lse, e_lse), _ = loss64(c.hidden, c.weight, c.targets)
    within(c.loss, loss, e_loss, "loss")
    within(c.lse, lse, e_lse, "lse")
    (dh, e_dh), (dw, e_dw) = loss_back64(c.hidden, c.weight, c.targets, c.dloss)
    for dtype, unit in ((B, UB), (torch.float32, U)):
        dweight = c.gradient(dtype)
        c.dhidden.fill_(NAN)
        c.backward(ctx, dweight)
        within(c.dhidden, dh, e_dh * (1 + UB) + UB * dh.abs(), "dhidden")
        within(dweight, dw, e_dw * (1 + unit) + unit * dw.abs(), "dweight")
        assert pads_untouched(dweight) and pads_untouched(c.dhidden)


@pytest.mark.parametrize("size", [(48, 200, 4700), (49, 200, 4700), (128, 136, 5000), (129, 136, 5000), (160, 905, 1187), (256, 520, 1301),
                                  (257, 520, 1301), (200, 2344, 643), (81, 72, 19001)], ids=str)
def test_where_another_kernel_takes_over(ctx, size):
    test_against_float64(ctx, size)


@pytest.mark.parametrize("T", [2, 17, 32, 95, 96, 128, 129])
@pytest.mark.parametrize("large", [False, True])
def test_few_tokens_and_many_columns(ctx, T, large):
    """Enough columns for a tile of them on every SM: targets in the first, a middle and the last, cut tile and of
    no column, logits up to a few hundred as well, a NaN token beside the others; the same bits twice."""
    c = Case(T, 200, 19001, seed=T, std=1.0 if large else None)
    c.targets[0], c.targets[-1], c.targets[T // 2] = 0, 19000, 18944
    c.targets[T // 3] = -2 ** 63 if T > 16 else c.targets[T // 3]
    nan = T // 4 if T > 16 else -1
    if nan >= 0:
        c.hidden[nan, 7] = NAN
    c.forward(ctx)
    (loss, e_loss), (lse, e_lse), _ = loss64(c.hidden, c.weight, c.targets)
    rows = [t for t in range(T) if t != nan]
    within(c.loss[rows], loss[rows], e_loss[rows], "loss")
    within(c.lse[rows], lse[rows], e_lse[rows], "lse")
    assert nan < 0 or bool(c.lse[nan].isnan())
    first = torch.stack([c.loss, c.lse]).clone()
    c.loss.fill_(5.0), c.lse.fill_(5.0)
    c.forward(ctx)
    assert torch.equal(first.view(torch.int32), torch.stack([c.loss, c.lse]).view(torch.int32))


def test_pieces_of_the_vocabulary(ctx):
    """More columns than are held at one time: dhidden is summed over the pieces, the last one of odd width."""
    c = Case(12000, 72, 12345, seed=3)
    c.forward(ctx)
    (loss, e_loss), _, _ = loss64(c.hidden, c.weight, c.targets)
    within(c.loss, loss, e_loss, "loss")
    (dh, e_dh), (dw, e_dw) = loss_back64(c.hidden, c.weight, c.targets, c.dloss)
    dweight = c.gradient(torch.float32)
    c.backward(ctx, dweight)
    within(c.dhidden, dh, e_dh * (1 + UB) + UB * dh.abs(), "dhidden")
    within(dweight, dw, e_dw * (1 + U) + U * dw.abs(), "dweight")


@pytest.mark.parametrize("dtype", [B, torch.float32])
def test_accumulates(ctx, dtype):
    c = Case(400, 96, 1500, seed=5)
    c.forward(ctx)
    fresh, added = c.gradient(dtype), c.gradient(dtype)
    c.backward(ctx, fresh)
    first = torch.randn(fresh.shape, device="cuda", dtype=torch.float32).to(dtype) * 1e-3
    added.copy_(first)
    c.backward(ctx, added, accumulate=True)
    _, (dw, e_dw) = loss_back64(c.hidden, c.weight, c.targets, c.dloss)
    unit = UB if dtype == B else U
    within(added, dw + first.double(), e_dw * (1 + unit) + unit * (dw + first.double()).abs() + 2 * U * first.double().abs(), "dweight")


def test_targets_that_are_none(ctx):
    """Negative targets: no loss, no gradient; targets past the vocabulary: NaN, no gradient; all of them at once too."""
    c = Case(70, 64, 300, seed=1, ignored=0.0)
    c.targets[:5] = torch.tensor([-1, -100, 300, 301, 2 ** 40])
    c.targets[5], c.targets[6], c.targets[7], c.targets[8] = 0, 299, 127, 128
    c.forward(ctx)
    (loss, e_loss), _, _ = loss64(c.hidden, c.weight, c.targets)
    within(c.loss[5:], loss[5:], e_loss[5:], "loss")
    assert c.loss[:2].tolist() == [0.0, 0.0] and bool(c.loss[2:5].isnan().all())
    dweight = c.gradient(torch.float32)
    c.backward(ctx, dweight)
    (dh, e_dh), (dw, e_dw) = loss_back64(c.hidden, c.weight, c.targets, c.dloss)
    within(c.dhidden, dh, e_dh * (1 + UB) + UB * dh.abs(), "dhidden")
    within(dweight, dw, e_dw * (1 + U) + U * dw.abs(), "dweight")
    assert not bool(c.dhidden[:5].any())
    c.targets.fill_(-100)
    c.forward(ctx)
    c.backward(ctx, dweight)
    assert not bool(c.loss.any()) and not bool(c.dhidden.any()) and not bool(dweight.any())


def test_large_logits(ctx):
    """Logits of hundreds: one of them has all the weight."""
    c = Case(130, 64, 1000, seed=2, std=8.0)
    c.forward(ctx)
    (loss, e_loss), (lse, e_lse), _ = loss64(c.hidden, c.weight, c.targets)
    within(c.loss, loss, e_loss, "loss")
    within(c.lse, lse, e_lse, "lse")


def test_no_tokens(ctx):
    c = Case(0, 64, 100)
    c.forward(ctx)
    dweight = c.gradient(B)
    c.backward(ctx, dweight, accumulate=True)
    assert bool(dweight.isnan().all())
    c.backward(ctx, dweight)
    assert not bool(dweight.any()) and pads_untouched(dweight)


def test_same_bits_and_a_graph(dd, ctx):
    """Repeated, and replayed from a graph with scratch of its own on other values."""
    c = Case(520, 136, 4000, seed=7)
    scratch = torch.zeros(max(ctx.vocab_loss_scratch_bytes(520, 136, 4000, backward=b) for b in (False, True)), dtype=torch.uint8, device="cuda")
    dweight = c.gradient(B)

    def both(**kw):
        c.forward(ctx, **kw)
        c.backward(ctx, dweight, **kw)
        return [t.clone() for t in (c.loss, c.lse, c.dhidden, dweight)]

    first = both()
    assert all(torch.equal(a, b) for a, b in zip(first, both(scratch=scratch)))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward(ctx, scratch=scratch)
        c.backward(ctx, dweight, scratch=scratch)
    c.hidden.mul_(0.5)
    c.targets.copy_(c.targets.roll(1))
    graph.replay()
    got = [t.clone() for t in (c.loss, c.lse, c.dhidden, dweight)]
    assert all(torch.equal(a, b) for a, b in zip(got, both())) and not torch.equal(got[0], first[0])
    del graph


def test_differences(ctx):
    """The gradients along a random direction against central differences of the float64 form."""
    c = Case(60, 40, 150, seed=8)
    c.forward(ctx)
    dweight = c.gradient(torch.float32)
    c.backward(ctx, dweight)
    gen = torch.Generator(device="cuda").manual_seed(1)
    valid = c.targets >= 0

    def objective(h, w):
        z = h @ w.t()
        loss = torch.logsumexp(z, -1) - z.gather(1, c.targets.clamp(min=0)[:, None])[:, 0]
        return float((loss * c.dloss.double() * valid).sum())

    h, w = c.hidden.double(), c.weight.double()
    for i, g in enumerate((c.dhidden, dweight)):
        step = torch.randn(g.shape, generator=gen, device="cuda", dtype=torch.float64) * 1e-4
        want = (objective(*(x + (step if j == i else 0) for j, x in enumerate((h, w)))) -
                objective(*(x - (step if j == i else 0) for j, x in enumerate((h, w))))) / 2
        size = float((g.double().square().sum() * step.square().sum()).sqrt())
        assert abs(float((g.double() * step).sum()) - want) <= 3 * UB * size      # its operand's rounding and its own


def test_a_wait_that_runs_out_is_reported(dd, ctx):
    c = Case(300, 64, 500)
    status, dweight = torch.zeros(1, dtype=torch.int32, device="cuda"), c.gradient(B)
    c.forward(ctx, status=status, flags=dd.DEBUG_EXPIRE_WAIT)
    assert int(status) == dd.STATUS_WAIT_LIMIT
    status.zero_()
    c.forward(ctx, status=status)
    assert int(status) == 0
    c.backward(ctx, dweight, status=status, flags=dd.DEBUG_EXPIRE_WAIT)
    assert int(status) == dd.STATUS_WAIT_LIMIT
    status.zero_()
    c.backward(ctx, dweight, status=status)
    (dh, e_dh), _ = loss_back64(c.hidden, c.weight, c.targets, c.dloss)
    within(c.dhidden, dh, e_dh * (1 + UB) + UB * dh.abs(), "dhidden")
    assert int(status) == 0


def test_refusals(dd, ctx):
    c = Case(16, 64, 100)
    dweight = c.gradient(B)
    with pytest.raises(ValueError):
        ctx.vocab_loss_forward(c.hidden.float(), c.weight, c.targets, c.loss, c.lse)
    with pytest.raises(ValueError):
        ctx.vocab_loss_forward(c.hidden, c.weight[:, :32], c.targets, c.loss, c.lse)
    with pytest.raises(ValueError):
        ctx.vocab_loss_forward(c.hidden, c.weight, c.targets.int(), c.loss, c.lse)
    with pytest.raises(ValueError):
        ctx.vocab_loss_forward(c.hidden, c.weight, c.targets, c.loss[:8], c.lse)
    with pytest.raises(ValueError):
        c.backward(ctx, dweight.half())
    with pytest.raises(ValueError):
        c.forward(ctx, scratch=torch.zeros(8, dtype=torch.uint8, device="cuda"))
    for call, rc in ((lambda: ctx.vocab_loss_forward(c.hidden, c.weight, c.targets, c.loss, c.loss), dd.ERR_ALIAS),
                     (lambda: c.forward(ctx, flags=2), dd.ERR_INVALID_ARG),
                     (lambda: ctx.vocab_loss_backward(c.hidden, c.weight, c.targets, c.lse, c.dloss, c.hidden, dweight), dd.ERR_ALIAS),
                     (lambda: ctx.vocab_loss_backward(c.hidden, c.weight, c.targets, c.lse, c.dloss, c.dhidden, c.weight), dd.ERR_ALIAS)):
        with pytest.raises(dd.DDMergeError) as e:
            call()
        assert e.value.rc == rc
