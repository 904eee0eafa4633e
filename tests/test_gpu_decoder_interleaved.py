"""Projections whose rows go head by head: queries, keys and values of a head side by side, no element shared."""
import pytest
import torch

from decoder_util import B

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


def parts(order, T, heads, dim, fill=None):
    """Three [T, heads, dim] tensors of one buffer: [T, heads, 3, dim], [heads, T, 3, dim], or the first with longer rows, by
    whole heads or by eight elements."""
    if order == "heads first":
        buf = torch.zeros(heads, T, 3, dim, dtype=B, device="cuda").transpose(0, 1)
    elif order == "longer rows":
        buf = torch.zeros(T, heads + 2, 3, dim, dtype=B, device="cuda")[:, 1: heads + 1]
    elif order == "padded rows":
        buf = torch.zeros(T, heads * 3 * dim + 8, dtype=B, device="cuda")[:, :-8].unflatten(1, (heads, 3, dim))
    else:
        buf = torch.zeros(T, heads, 3, dim, dtype=B, device="cuda")
    for i in range(3):
        if fill is not None:
            buf[:, :, i] = fill[i]
    return [buf[:, :, i] for i in range(3)]


ORDERS = ["tokens first", "heads first", "longer rows", "padded rows"]
SIZES = [(1, 4, 64), (1, 1, 64), (2, 1, 128), (300, 4, 64), (131, 3, 80)]


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("order", ORDERS)
def test_rotary_in_place(dd, ctx, order, size):
    T, heads, dim = size
    gen = torch.Generator(device="cuda").manual_seed(T)
    x = [torch.randn(T, heads, dim, generator=gen, device="cuda").to(B) for _ in range(3)]
    positions, (f, _) = torch.arange(T, device="cuda"), dd.rotary_frequencies(dim)
    q, k, v = parts(order, T, heads, dim, x)
    ctx.rotary(q, k, positions, f)
    ctx.rotary(x[0], x[1], positions, f)
    assert torch.equal(q, x[0]) and torch.equal(k, x[1]) and torch.equal(v, x[2])


@pytest.mark.parametrize("size", SIZES, ids=str)
@pytest.mark.parametrize("order", ORDERS)
def test_attention_and_its_gradients(ctx, order, size):
    """Inputs, and gradients, in such a buffer: the bits that separate tensors give."""
    T, heads, dim = size
    gen = torch.Generator(device="cuda").manual_seed(T)
    x = [torch.randn(T, heads, dim, generator=gen, device="cuda").to(B) for _ in range(3)]
    d_o = torch.randn(T, heads, dim, generator=gen, device="cuda").to(B)
    o, want = (torch.zeros(T, heads, dim, dtype=B, device="cuda") for _ in range(2))
    lse = torch.zeros(heads, T, device="cuda")
    ctx.attention_forward(*x, want, lse)
    separate = [torch.zeros_like(t) for t in x]
    ctx.attention_backward(*x, want, lse, d_o, *separate)
    mixed, grads = parts(order, T, heads, dim, x), parts(order, T, heads, dim)
    ctx.attention_forward(*mixed, o, lse)
    ctx.attention_backward(*mixed, o, lse, d_o, *grads)
    assert torch.equal(o, want)
    for a, b in zip(grads, separate):
        assert torch.equal(a, b)


def test_keys_and_values_beside_a_group_of_queries(ctx):
    """[tokens, kv_heads, group + 2, dim]: gradients of keys and values in such rows, those of queries elsewhere."""
    T, kv, group, dim = 200, 2, 3, 64
    gen = torch.Generator(device="cuda").manual_seed(1)
    buf = torch.randn(T, kv, group + 2, dim, generator=gen, device="cuda").to(B)
    q, k, v = buf[:, :, :group].flatten(1, 2), buf[:, :, group], buf[:, :, group + 1]
    d_o = torch.randn(T, kv * group, dim, generator=gen, device="cuda").to(B)
    o, lse = torch.zeros_like(d_o), torch.zeros(kv * group, T, device="cuda")
    ctx.attention_forward(q, k, v, o, lse)
    room = torch.zeros_like(buf)
    dq, dk, dv = torch.zeros_like(q), room[:, :, group], room[:, :, group + 1]
    ctx.attention_backward(q, k, v, o, lse, d_o, dq, dk, dv)
    separate = [torch.zeros(t.shape, dtype=B, device="cuda") for t in (q, k, v)]
    ctx.attention_backward(q, k.contiguous(), v.contiguous(), o, lse, d_o, *separate)
    assert all(torch.equal(a, b) for a, b in zip((dq, dk, dv), separate)) and not bool(room[:, :, :group].any())


def test_what_shares_elements_is_still_refused(dd, ctx):
    T, heads, dim = 6, 4, 16
    flat = torch.zeros((T + 2) * heads * 3 * dim, dtype=B, device="cuda")
    positions, (f, _) = torch.arange(T, device="cuda"), dd.rotary_frequencies(dim)

    def at(start, step=3 * dim):
        return flat.as_strided((T, heads, dim), (heads * 3 * dim, step, 1), start)

    for q, k in ((at(0), at(8)), (at(0), at(0)), (at(0), at(3 * dim - 8)), (at(0), at(3 * dim)), (at(dim), at(3 * dim + 8)), (at(0), at(dim, 2 * dim))):
        with pytest.raises(dd.DDMergeError) as e:
            ctx.rotary(q, k, positions, f)
        assert e.value.rc == dd.ERR_ALIAS
    def padded(start):
        return flat.as_strided((T, heads, dim), ((heads * 3 + 1) * dim - 8, 3 * dim, 1), start)

    for q, k in ((padded(0), padded(dim - 8)), (padded(0), padded(3 * dim - 8)), (padded(dim), padded((heads * 3 + 2) * dim - 8))):
        with pytest.raises(dd.DDMergeError) as e:
            ctx.rotary(q, k, positions, f)
        assert e.value.rc == dd.ERR_ALIAS
    o, lse = torch.zeros(T, heads, dim, dtype=B, device="cuda"), torch.zeros(heads, T, device="cuda")
    x = [torch.zeros(T, heads, dim, dtype=B, device="cuda") for _ in range(3)]
    for grads in ((at(0), at(dim), at(dim)), (at(0), at(dim + 8), at(2 * dim + 8)), (at(0), at(dim), at(2 * dim + 8))):
        with pytest.raises(dd.DDMergeError) as e:
            ctx.attention_backward(*x, o, lse, o.clone(), *grads)
        assert e.value.rc == dd.ERR_ALIAS
