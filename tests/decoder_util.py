"""Float64 forms of the decoder's operators with bounds on what float32 sums and bf16 operands may be off by.

A rounding to bf16 is off by at most UB, one to float32 by U, relative to the value.  A float32 sum of n products
on the tensor cores is held to n + 16 roundings of twice U (its additions truncate).  Exponentials below float32's normal
range count as 0, or by the polynomial as anything below 2^-125: TINY each.  Forward, weights are relative to a maximum
that is up to 2^8 above the one in use, so that one of them is 2^8 TINY of the row's sum at most.
"""
import torch

U, UB, TINY = 2.0 ** -24, 2.0 ** -8, 2.0 ** -125
B = torch.bfloat16


def within(got, ref, tol, what):
    err = (got.double() - ref).abs()
    bad = ~(err <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((err / tol).max()):.2f} of the bound"


def scores64(q, k, scale, causal):
    """Scores of one document, [heads, n, n], and a bound on the error of the kernel's exponents: the product's
    sum, its scaling (a rounding each of the score, the base and their difference) and the exponential (2^-21)."""
    group = q.shape[1] // k.shape[1]
    q, k = q.double().transpose(0, 1), k.double().transpose(0, 1).repeat_interleave(group, 0)
    s = q @ k.transpose(1, 2) * scale
    size = q.abs() @ k.abs().transpose(1, 2) * scale
    n, d = s.shape[1], q.shape[2]
    off = ((d + 16) * 2 * U + 4 * U) * size.amax(-1, keepdim=True) + 2.0 ** -21
    if causal:
        s = s.masked_fill(torch.ones(n, n, dtype=torch.bool, device=s.device).triu(1), float("-inf"))
    return s, off


def attention64(q, k, v, scale, causal):
    """o and lse of one document with bounds: (o, eo), (lse, el); o [n, heads, dim], lse [heads, n]."""
    s, off = scores64(q, k, scale, causal)
    group, n = q.shape[1] // k.shape[1], s.shape[1]
    v = v.double().transpose(0, 1).repeat_interleave(group, 0)
    lse = torch.logsumexp(s, -1)
    p = (s - lse[..., None]).exp()
    o = p @ v
    eo = (UB + 2 * off + (n + 16) * 2 * U) * (p @ v.abs()) + UB * o.abs() + 2 ** 8 * TINY * v.abs().sum(1, keepdim=True) + 1e-38
    el = off[..., 0] + (n + 16) * 2 * U + 4 * U * lse.abs()
    return (o.transpose(0, 1), eo.transpose(0, 1)), (lse, el)


def attention_back64(q, k, v, o, d_o, scale, causal, exact_delta):
    """dq, dk, dv of one document with bounds, given the rounded o.  ``exact_delta``: rows whose delta does not come
    from it (all of them if a number of rows is not given)."""
    s, off = scores64(q, k, scale, causal)
    heads, kv = q.shape[1], k.shape[1]
    group, n = heads // kv, s.shape[1]
    lse = torch.logsumexp(s, -1, keepdim=True)
    p = (s - lse).exp()
    ep = off + (n + 16) * 2 * U + 8 * U * lse.abs() + 2.0 ** -18          # of the weights, relative (2^-18: the polynomial)
    Q, D, O = (x.double().transpose(0, 1) for x in (q, d_o, o))
    K, V = (x.double().transpose(0, 1).repeat_interleave(group, 0) for x in (k, v))
    dp = D @ V.transpose(1, 2)
    edp = (q.shape[2] + 16) * 2 * U * (D.abs() @ V.abs().transpose(1, 2))
    delta = (p * dp).sum(-1, keepdim=True)
    edelta = (ep + (n + 16) * 2 * U) * (p * dp.abs()).sum(-1, keepdim=True) + (p * edp).sum(-1, keepdim=True)
    rounded = (UB + 32 * U) * (D.abs() * O.abs()).sum(-1, keepdim=True)   # o's rounding, where o is used
    rows = torch.arange(n, device=s.device)[None, :, None]
    edelta = torch.where(rows < exact_delta, edelta, edelta + rounded)
    ds = p * (dp - delta)
    eds = UB * ds.abs() + (1 + UB) * (ep * ds.abs() + (1 + ep) * p * (edp + edelta) + (4 * U * p + 2 * TINY) * (dp.abs() + delta.abs()))
    if causal:
        eds[:, 0, 0] = 0                                                   # exact: a token that sees itself alone
    if n == 1:
        eds.zero_()

    def out(weights, error, x, by):
        r = weights @ x * by
        e = (error @ x.abs() + (n * group + 16) * 2 * U * (weights.abs() @ x.abs())) * by
        return r, e

    dq, edq = out(ds, eds, K, scale)
    dk, edk = out(ds.transpose(1, 2), eds.transpose(1, 2), Q, scale)
    dv, edv = out(p.transpose(1, 2), ((UB + ep) * p + 2 * TINY).transpose(1, 2), D, 1.0)
    shared = [x.reshape(kv, group, n, -1).sum(1) for x in (dk, edk, dv, edv)]
    results = [(dq, edq), (shared[0], shared[1]), (shared[2], shared[3])]
    return [(r.transpose(0, 1), (e * (1 + UB) + UB * r.abs() + 1e-38).transpose(0, 1)) for r, e in results]


def loss64(hidden, weight, targets):
    """(loss, bound), (lse, bound) and the logits with theirs."""
    h, w = hidden.double(), weight.double()
    z = h @ w.t()
    ez = (h.shape[1] + 16) * 2 * U * (h.abs() @ w.abs().t())
    lse = torch.logsumexp(z, -1)
    el = ez.amax(-1) + 2.0 ** -20 + 4 * U * lse.abs()
    valid = (targets >= 0) & (targets < w.shape[0])
    t = targets.clamp(0, w.shape[0] - 1)[:, None]
    loss = lse - z.gather(1, t)[:, 0]
    loss = torch.where(targets < 0, 0.0, torch.where(valid, loss, float("nan")))
    el_loss = el + ez.gather(1, t)[:, 0] + 2 * U * (lse.abs() + z.gather(1, t)[:, 0].abs())
    return (loss, el_loss), (lse, el), (z, ez)


def loss_back64(hidden, weight, targets, dloss):
    """(dhidden, bound), (dweight, bound), before the rounding of the results."""
    (_, _), (lse, el), (z, ez) = loss64(hidden, weight, targets)
    h, w = hidden.double(), weight.double()
    valid = ((targets >= 0) & (targets < w.shape[0]))[:, None]
    p = (z - lse[:, None]).exp()
    one = torch.zeros_like(p).scatter_(1, targets.clamp(0, w.shape[0] - 1)[:, None], 1.0)
    d = torch.where(valid[:, 0], dloss.double(), 0.0)[:, None]
    g = (p - one) * d
    eg = (p * (ez + el[:, None] + 2.0 ** -20 + 8 * U * z.abs()) + 2 * U) * d.abs() + UB * g.abs()
    out = []
    for a, ea, x, n in ((g, eg, w, w.shape[0]), (g.t(), eg.t(), h, h.shape[0])):
        out.append((a @ x, ea @ x.abs() + (n + 16) * 2 * U * (a.abs() @ x.abs()) + 1e-38))
    return out
