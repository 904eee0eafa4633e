"""What the binding of the learner's operators turns away, and that it does so before anything runs."""
import pytest
import torch

pytestmark = pytest.mark.gpu
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


def zeros(*shape, dtype=B):
    return torch.zeros(*shape, dtype=dtype, device="cuda")


@pytest.mark.parametrize("tokens", [2, 40, 400])
@pytest.mark.parametrize("cols", [1, 64])
def test_expanded_rows_are_refused(ctx, tokens, cols):
    """Matrices of stride 0 along the rows (``expand``, the gradient of a sum over tokens) hold one row
    only; in every place of both calls they are refused and nothing is written."""
    d, f = cols, 128
    full = dict(x=zeros(tokens, d), w_gate=zeros(f, d), w_up=zeros(f, d), w_down=zeros(d, f), y=zeros(tokens, d),
                residual=zeros(tokens, d), gate=zeros(tokens, f), up=zeros(tokens, f), dy=zeros(tokens, d),
                dx=zeros(tokens, d), dw_gate=zeros(f, d), dw_up=zeros(f, d), dw_down=zeros(d, f))
    if cols == 1:                                              # rows of one element still need 16 bytes each
        full = {k: zeros(t.shape[0], 8)[:, :1] if t.shape[1] == 1 else t for k, t in full.items()}
    forward = ("x", "w_gate", "w_up", "w_down", "y", "residual", "gate", "up")
    backward = ("x", "w_gate", "w_up", "w_down", "gate", "up", "dy", "dx", "dw_gate", "dw_up", "dw_down")

    def run(names, m):
        if names is forward:
            ctx.gated_ffn_forward(m["x"], m["w_gate"], m["w_up"], m["w_down"], m["y"], residual=m["residual"],
                                  gate=m["gate"], up=m["up"])
        else:
            ctx.gated_ffn_backward(*(m[k] for k in backward))

    for names in (forward, backward):
        run(names, full)                                       # as they are, they are taken
        for groups in [(k,) for k in names] + [("x", "dx"), ("y", "residual"), ("dy", "y"), ("gate", "up"),
                                               ("w_gate", "w_up", "dw_gate", "dw_up"), ("w_down", "dw_down")]:
            m = dict(full)
            for k in groups:
                if m[k].shape[0] > 1:
                    m[k] = torch.full((m[k].shape[1],), 3.0, dtype=B, device="cuda").expand(m[k].shape)
            if not any(m[k] is not full[k] for k in names):
                continue
            with pytest.raises(ValueError):
                run(names, m)
    overlapping = zeros(tokens * 128).as_strided((tokens, max(cols, 16)), (8, 1))[:, :cols]
    if cols > 8:
        with pytest.raises(ValueError):
            run(forward, dict(full, x=overlapping))
    torch.cuda.synchronize()
    assert not any(bool(t.any()) for t in full.values())


class NoTruth:
    def __bool__(self):
        raise TypeError("neither true nor false")


def test_numbers_that_do_not_convert_run_nothing(dd, ctx):
    """Python's error comes before anything is launched: parameters, moments, copies, gradients and outputs
    keep every bit."""
    gen = torch.Generator(device="cuda").manual_seed(1)

    def randn(*shape, dtype=torch.float32):
        return torch.randn(*shape, generator=gen, device="cuda").to(dtype)

    params, grads, m, copies = ([randn(5000), randn(33)] for _ in range(4))
    v, copies = [t.square() for t in m], [c.to(B) for c in copies]
    record, rec2 = dd.new_grad_record(), dd.new_grad_record()
    tokens, d, f = 24, 64, 128
    x, y, w = randn(tokens, d, dtype=B), randn(tokens, d, dtype=B), [randn(f, d, dtype=B), randn(f, d, dtype=B), randn(d, f, dtype=B)]
    gate, up, dy, dx = randn(tokens, f, dtype=B), randn(tokens, f, dtype=B), randn(tokens, d, dtype=B), randn(tokens, d, dtype=B)
    dws = [randn(*t.shape, dtype=B) for t in w]
    everything = [*params, *grads, *m, *v, *copies, record, x, y, *w, gate, up, dy, dx, *dws]
    before = [t.clone() for t in everything]

    def adamw(step=1, lr=1e-3, **kw):
        ctx.adamw_step(params, grads, m, v, step, lr, copies=copies, **kw)

    def forward(**kw):
        ctx.gated_ffn_forward(x, *w, y, gate=gate, up=up, **kw)

    def backward(**kw):
        ctx.gated_ffn_backward(x, *w, gate, up, dy, dx, *dws, **kw)

    far = 2 ** 70                                              # past every integer type
    for call in [lambda bad=bad, k=k: adamw(**{k: bad}) for k in ("lr", "beta1", "beta2", "eps", "weight_decay") for bad in (None, "x", [1.0])] + [
            lambda: adamw(step=None), lambda: adamw(step=1.5), lambda: adamw(step=far), lambda: adamw(stream=far),
            lambda: adamw(clip=far), lambda: ctx.grad_norm(grads, None, record), lambda: ctx.grad_norm(grads, 1.0, record, stream=far),
            lambda: ctx.clip_gradients(grads, "1", record), lambda: ctx.clip_gradients(grads, 1e-3, record, stream=far),
            lambda: forward(activation=None), lambda: forward(flags=None), lambda: forward(flags=far), lambda: forward(stream=far),
            lambda: forward(hidden=far), lambda: forward(status=far), lambda: backward(accumulate=NoTruth()),
            lambda: backward(activation="silu"), lambda: backward(flags=1.0), lambda: backward(stream=far), lambda: backward(scratch=far)]:
        with pytest.raises((TypeError, OverflowError)):
            call()
    for call in (lambda: forward(activation=2 ** 32), lambda: forward(flags=2 ** 32), lambda: backward(flags=-1)):
        with pytest.raises(dd.DDMergeError) as e:              # in range of Python's numbers, not of the argument's
            call()
        assert e.value.rc == dd.ERR_INVALID_ARG
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(everything, before))
    ctx.grad_norm(grads, 1.0, rec2)                            # the context goes on working
    want = sum(float(g.double().square().sum()) for g in grads) ** 0.5
    assert abs(dd.read_grad_record(rec2).norm - want) <= 20 * 2.0 ** -24 * want
