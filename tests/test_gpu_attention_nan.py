"""One NaN in a document reaches every gradient that depends on it."""
import pytest
import torch

from test_gpu_attention import NAN, Case, ctx, dd  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("length,at", [(2, 1), (40, 2), (40, 7), (40, 12), (128, 64), (300, 6), (300, 130), (300, 299)])
def test_gradients_that_depend_on_it(ctx, length, at, dim, causal):  # noqa: F811
    """Query, key, value and output gradient in turn, at places whose exponentials are taken either way."""
    rows = torch.arange(length, device="cuda")
    seen, later = (rows <= at, rows >= at) if causal else (rows >= 0, rows >= 0)
    for name in ("q", "k", "v", "d_o"):
        c = Case([length], 1, 1, dim, seed=at)
        getattr(c, name)[at, 0, 3] = NAN
        c.forward(ctx, causal=causal)
        c.backward(ctx, causal=causal)
        # rows of the scores that hold it, and the keys that those rows see
        if name == "q":
            query, key, value = rows == at, seen, seen
        elif name == "k":
            query, key, value = later, rows <= length - 1, rows <= length - 1
        elif name == "v":
            query, key, value = later, rows <= length - 1, rows < 0
        else:
            query, key, value = rows == at, seen, seen
        # (the value's own gradient does not read it; with d_o only its column's)
        assert not bool(c.dq[query].isfinite().any()), name
        assert not bool(c.dk[key].isfinite().any()), name
        got = c.dv[value] if name != "d_o" else c.dv[value][..., 3]
        assert not bool(got.isfinite().any()), name
