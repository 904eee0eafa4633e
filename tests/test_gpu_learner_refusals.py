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
