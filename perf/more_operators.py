"""The cases by which the operators of a learner's decoder are measured: rotary positions, attention over packed
sequences (forward and backward), and the loss over the vocabulary (forward and backward).

``run`` computes them in their plain form, in 32 bits with elementary torch operations (angles in 64); with
``own`` set it makes the library's calls.
"""
import math

import torch

own = False

STD_GRAD = 2e-3            # gradients that come from the layers behind
IGNORED = 0.05             # share of the tokens without a target
LOGIT_STD = 2.0            # of the logits of a model in training
LARGEST = {"attention": 16384 ** 2 * 8 * 128, "loss": 8192 * 2048 * 32000, "rotary": 16384 * 20 * 128}   # listed cases


# ---- the cases -------------------------------------------------------------------------------------

def rotary(name, tokens, heads, kv_heads, dim, part, layout, dtype="bf16", inverse=False, scale=1.0):
    return dict(name=name, op="rotary", tokens=tokens, heads=heads, kv_heads=kv_heads, dim=dim, part=part,
                layout=layout, dtype=dtype, inverse=inverse, scale=scale)


def attention(name, op, lengths, heads, kv_heads, dim, causal=True, tail=0, packed=True):
    return dict(name=name, op=op, lengths=" ".join(map(str, lengths)), heads=heads, kv_heads=kv_heads, dim=dim,
                causal=causal, tail=tail, packed=packed)


def loss(name, op, tokens, d, vocab):
    return dict(name=name, op=op, tokens=tokens, d=d, vocab=vocab)


def listed():
    return [
        # queries and keys of one short sequence of a small decoder: latency
        rotary("rotary_short", 64, 12, 12, 64, 64, "half"),
        # a training micro-batch with grouped heads, context stretched to four times its length
        rotary("rotary_train", 16384, 16, 4, 128, 128, "half", scale=4.0),
        # the gradient's way back, a part of each head rotated, neighbours paired, float32, odd token count
        rotary("rotary_back_part", 3001, 8, 8, 96, 48, "interleaved", dtype="f32", inverse=True),
        # one short sequence of a small decoder
        attention("attention_short", "attention_forward", [100], 12, 12, 64, packed=False),
        # a micro-batch of documents packed end to end, grouped heads, some rows of padding behind the last
        attention("attention_packed", "attention_forward", [2900, 17, 1, 1333, 0, 640, 2048, 999, 129, 65], 16, 4, 128, tail=60),
        # one long context
        attention("attention_long", "attention_forward", [16384], 8, 2, 128, packed=False),
        # backward of ragged documents, heads of an odd width, every token attends to its whole document
        attention("attention_back_odd", "attention_backward", [301, 77, 1, 530], 6, 3, 80, causal=False, tail=3),
        # backward of the learner's training micro-batch
        attention("attention_back_train", "attention_backward", [4096, 1500, 2596], 16, 4, 128),
        # loss of a small decoder's short sequence
        loss("loss_short", "loss_forward", 96, 768, 32000),
        # loss of a training micro-batch of a 1.3B-parameter decoder
        loss("loss_train", "loss_forward", 8192, 2048, 32000),
        # gradients at odd sizes
        loss("loss_back_odd", "loss_backward", 777, 1001, 5003),
        # gradients of the training micro-batch above
        loss("loss_back_train", "loss_backward", 8192, 2048, 32000),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["rotary", "attention_forward", "attention_backward", "loss_forward", "loss_backward"])
    if op == "rotary":
        while True:
            kv, dim = rng.randint(1, 16), 8 * rng.randint(4, 16)
            c = rotary("", spread(1, 16384), kv * rng.choice([1, 2, 4, 8]), kv, dim, dim if rng.random() < 0.5 else 16 * rng.randint(1, dim // 16),
                       rng.choice(["half", "interleaved"]), rng.choice(["bf16", "f32"]), rng.random() < 0.5,
                       rng.choice([1.0, 2.0, 8.0]))
            if c["tokens"] * (c["heads"] + c["kv_heads"]) * dim * (2 if c["dtype"] == "f32" else 1) <= LARGEST["rotary"]:
                break
    elif op.startswith("attention"):
        while True:
            tokens, count = spread(1, 16384), spread(1, 64)
            cuts = sorted(rng.randint(0, tokens) for _ in range(count - 1))
            lengths = [b - a for a, b in zip([0] + cuts, cuts + [tokens])]
            kv = rng.randint(1, 8)
            heads, dim = kv * rng.choice([1, 2, 3, 4, 8]), rng.choice([64, 128, 8 * rng.randint(4, 16)])
            work_ = sum(n * n for n in lengths) * heads * dim * (2 if op == "attention_backward" else 1)
            causal = rng.random() < 0.75
            if work_ * (1 if causal else 2) <= LARGEST["attention"] and tokens * heads * dim <= 16384 * 16 * 128:
                break
        c = attention("", op, lengths, heads, kv, dim, causal, rng.choice([0, 0, rng.randint(1, 200)]), packed=True)
    else:
        while True:
            tokens, d, vocab = spread(1, 8192), spread(128, 4096), spread(1000, 64000)
            if rng.random() < 0.5:
                d -= d % 8
            if tokens * d * vocab <= LARGEST["loss"] and d * vocab <= 2048 * 32000:
                break
        c = loss("", op, tokens, d, vocab)
    del c["name"]
    return c


def lengths_of(case):
    return [int(n) for n in case["lengths"].split()]


def rows(n):
    """Row length in memory of a row of n bf16 elements: whole 16 bytes."""
    return (n + 7) // 8 * 8


def work(case):
    op = case["op"]
    if op == "rotary":
        n = case["tokens"] * (case["heads"] + case["kv_heads"])
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": 2 * size * n * case["dim"] + 8 * case["tokens"], "flops": 3 * n * case["part"]}
    if op.startswith("attention"):
        ls, h, kv, d = lengths_of(case), case["heads"], case["kv_heads"], case["dim"]
        pairs, t = sum(n * (n + 1) // 2 if case["causal"] else n * n for n in ls), sum(ls)
        if op == "attention_forward":
            return {"bytes": 2 * t * d * 2 * (h + kv) + 4 * t * h, "flops": 4 * pairs * h * d}
        return {"bytes": 2 * t * d * 4 * (h + kv) + 4 * t * h, "flops": 10 * pairs * h * d}
    t, d, v = case["tokens"], case["d"], case["vocab"]
    if op == "loss_forward":
        return {"bytes": 2 * (t * d + v * d) + 16 * t, "flops": 2 * t * d * v}
    return {"bytes": 4 * (t * d + v * d) + 16 * t, "flops": 6 * t * d * v}


# ---- what a program has in hand --------------------------------------------------------------------

def randn(gen, *shape, std=1.0, dtype=torch.bfloat16):
    """Normal values in a buffer whose rows start on 16-byte boundaries."""
    x = torch.randn(*shape[:-1], rows(shape[-1]), generator=gen, device="cuda", dtype=torch.float32)
    return x.mul_(std).to(dtype)[..., : shape[-1]]


def empty(*shape):
    return torch.zeros(*shape[:-1], rows(shape[-1]), device="cuda", dtype=torch.bfloat16)[..., : shape[-1]]


BASE, TRAINED = 10000.0, 4096      # angles' base, and the context that the frequencies were trained at


def frequencies(case):
    """Radians a position of each pair, stretched by parts for contexts beyond the trained one: pairs that
    turn more than 32 times in it keep their frequency, those that turn less than once are divided by the
    factor, a ramp lies between.  Returns them with the magnitude that goes along."""
    half, s = case["part"] // 2, case["scale"]
    f = torch.tensor([BASE ** (-i / half) for i in range(half)], dtype=torch.float64, device="cuda")
    if s == 1.0:
        return f, 1.0
    turns = TRAINED * f / (2 * math.pi)
    keep = ((turns - 1.0) / (32.0 - 1.0)).clamp(0.0, 1.0)
    return f * (keep + (1 - keep) / s), 0.1 * math.log(s) + 1.0


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s, op = {"case": case}, case["op"]
    if op == "rotary":
        dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        t, d = case["tokens"], case["dim"]
        for name, h in (("q", case["heads"]), ("k", case["kv_heads"])):
            s[name] = torch.randn(t, h, d, generator=gen, device="cuda").to(dtype)
            s[name + "_out"] = torch.zeros(t, h, d, device="cuda", dtype=dtype)
        # documents end to end, each counted from 0; the last positions of a long context
        starts = torch.randint(0, t, (t // 1000 + 1,), generator=gen, device="cuda").sort().values
        i = torch.arange(t, device="cuda")
        s["positions"] = i - torch.cat([i[:1], starts])[torch.searchsorted(starts, i, right=True)]
        s["positions"] = s["positions"] + int(TRAINED * case["scale"]) - min(t, TRAINED)
        s["frequencies"], s["magnitude"] = frequencies(case)
        return s
    if op.startswith("attention"):
        ls, h, kv, d = lengths_of(case), case["heads"], case["kv_heads"], case["dim"]
        t = sum(ls) + case["tail"]
        qkv = torch.randn(t, h + 2 * kv, d, generator=gen, device="cuda").to(torch.bfloat16)   # one projection's rows
        s["q"], s["k"], s["v"] = qkv[:, :h], qkv[:, h: h + kv], qkv[:, h + kv:]
        s["lengths"], s["scale"] = ls, 1 / math.sqrt(d)
        ends = [0]
        for n in ls:
            ends.append(ends[-1] + n)
        s["offsets"] = torch.tensor(ends, dtype=torch.int32, device="cuda") if case["packed"] else None
        s["o"] = torch.zeros(t, h, d, device="cuda", dtype=torch.bfloat16)
        s["lse"] = torch.zeros(h, t, device="cuda")
        if op == "attention_backward":
            attention_plain(s)                                                                 # what the forward pass kept
            s["do"] = torch.randn(t, h, d, generator=gen, device="cuda").mul_(STD_GRAD).to(torch.bfloat16)
            dqkv = torch.zeros(t, h + 2 * kv, d, device="cuda", dtype=torch.bfloat16)
            s["dq"], s["dk"], s["dv"] = dqkv[:, :h], dqkv[:, h: h + kv], dqkv[:, h + kv:]
        return s
    t, d, v = case["tokens"], case["d"], case["vocab"]
    s["hidden"] = randn(gen, t, d)
    s["weight"] = randn(gen, v, d, std=LOGIT_STD / math.sqrt(d))
    s["targets"] = torch.randint(0, v, (t,), generator=gen, device="cuda")
    s["targets"][torch.rand(t, generator=gen, device="cuda") < IGNORED] = -100
    s["loss"], s["lse"] = torch.zeros(t, device="cuda"), torch.zeros(t, device="cuda")
    if op == "loss_backward":
        loss_plain(s)                                                                          # what the forward pass kept
        s["dloss"] = torch.rand(t, generator=gen, device="cuda").add_(0.5).div_(t)             # weights of a mean
        s["dhidden"], s["dweight"] = empty(t, d), empty(v, d)
    return s


# ---- one pass --------------------------------------------------------------------------------------

def rotate(x, cos, sin, part, layout):
    """The pairs of the first `part` elements turned, in x's type; cos, sin: [tokens, 1, part / 2]."""
    a, b = (x[..., : part // 2], x[..., part // 2: part]) if layout == "half" else (x[..., 0:part:2], x[..., 1:part:2])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat([ra, rb], -1) if layout == "half" else torch.stack([ra, rb], -1).flatten(-2)
    return torch.cat([turned, x[..., part:]], -1)


def rotary_plain(s):
    c = s["case"]
    angle = s["positions"].double()[:, None] * s["frequencies"]
    cos, sin = torch.cos(angle), torch.sin(angle)
    if c["inverse"]:
        sin = -sin
    cos, sin = ((s["magnitude"] * x).float()[:, None, :] for x in (cos, sin))
    for name in ("q", "k"):
        s[name + "_out"].copy_(rotate(s[name].float(), cos, sin, c["part"], c["layout"]))
    return s["q_out"], s["k_out"]


def documents(s):
    """The rows of each document."""
    a = 0
    for n in s["lengths"]:
        if n:
            yield slice(a, a + n)
        a += n


def heads_of(s, name, doc):
    """Rows of one document in 32 bits, [heads of keys, query heads that read one (or 1), rows, dim]."""
    x = s[name][doc].float().transpose(0, 1)
    return x.reshape(s["case"]["kv_heads"], -1, *x.shape[1:])


def scores(s, doc):
    x = heads_of(s, "q", doc) @ heads_of(s, "k", doc).transpose(2, 3) * s["scale"]
    if s["case"]["causal"]:
        i = torch.arange(x.shape[-1], device=x.device)
        x = x.masked_fill_(i[None, :] > i[:, None], -math.inf)
    return x


def put(out, doc, x):
    """Results of a document, laid out as heads_of() gives them, rounded into `out`."""
    out[doc] = x.flatten(0, 1).transpose(0, 1).to(out.dtype)


def attention_plain(s):
    for doc in documents(s):
        x = scores(s, doc)
        top = x.amax(-1, keepdim=True)
        p = x.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        put(s["o"], doc, p @ heads_of(s, "v", doc) / total)
        s["lse"][:, doc] = (top + total.log()).reshape(-1, x.shape[-1])
    return s["o"], s["lse"]


def attention_back_plain(s):
    for doc in documents(s):
        p = scores(s, doc)
        p = p.sub_(s["lse"][:, doc].reshape(*p.shape[:3], 1)).exp_()
        q, k, v, do = (heads_of(s, name, doc) for name in ("q", "k", "v", "do"))
        put(s["dv"], doc, (p.transpose(2, 3) @ do).sum(1, keepdim=True))
        dp = do @ v.transpose(2, 3)
        ds = p * (dp - (p * dp).sum(-1, keepdim=True)) * s["scale"]
        put(s["dq"], doc, ds @ k)
        put(s["dk"], doc, (ds.transpose(2, 3) @ q).sum(1, keepdim=True))
    return s["dq"], s["dk"], s["dv"]


def loss_plain(s):
    logits = s["hidden"].float() @ s["weight"].float().t()
    top = logits.amax(-1, keepdim=True)
    lse = (top + (logits - top).exp().sum(-1, keepdim=True).log()).squeeze(-1)
    valid = s["targets"] >= 0
    chosen = logits.gather(1, s["targets"].clamp(min=0)[:, None]).squeeze(1)
    return s["loss"].copy_(torch.where(valid, lse - chosen, torch.zeros_like(lse))), s["lse"].copy_(lse)


def loss_back_plain(s):
    h, w = s["hidden"].float(), s["weight"].float()
    g = (h @ w.t()).sub_(s["lse"][:, None]).exp_()
    valid = s["targets"] >= 0
    g.scatter_add_(1, s["targets"].clamp(min=0)[:, None], torch.full_like(g[:, :1], -1.0))
    g *= torch.where(valid, s["dloss"], torch.zeros_like(s["dloss"]))[:, None]
    s["dhidden"].copy_(g @ w)
    s["dweight"].copy_(g.t() @ h)
    return s["dhidden"], s["dweight"]


PLAIN = {"rotary": rotary_plain, "attention_forward": attention_plain, "attention_backward": attention_back_plain,
         "loss_forward": loss_plain, "loss_backward": loss_back_plain}


def run(s):
    return run_own(s) if own else PLAIN[s["case"]["op"]](s)


_library = {}


def library():
    """The library's binding and this program's context on the current GPU."""
    if not _library:
        from paper_2604_21428_b200 import ddmerge as dd
        _library.update(dd=dd, ctx=dd.Context(torch.cuda.current_device()))
    return _library["dd"], _library["ctx"]


def run_own(s):
    c = s["case"]
    _, ctx = library()
    if c["op"] == "rotary":
        ctx.rotary(s["q"], s["k"], s["positions"], s["frequencies"], q_out=s["q_out"], k_out=s["k_out"],
                   magnitude=s["magnitude"], interleaved=c["layout"] == "interleaved", inverse=c["inverse"])
        return s["q_out"], s["k_out"]
    if c["op"].startswith("attention"):
        if c["op"] == "attention_forward":
            ctx.attention_forward(s["q"], s["k"], s["v"], s["o"], s["lse"], offsets=s["offsets"], scale=s["scale"], causal=c["causal"])
            return s["o"], s["lse"]
        ctx.attention_backward(s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"], s["dq"], s["dk"], s["dv"], offsets=s["offsets"],
                               scale=s["scale"], causal=c["causal"])
        return s["dq"], s["dk"], s["dv"]
    if c["op"] == "loss_forward":
        ctx.vocab_loss_forward(s["hidden"], s["weight"], s["targets"], s["loss"], s["lse"])
        return s["loss"], s["lse"]
    ctx.vocab_loss_backward(s["hidden"], s["weight"], s["targets"], s["lse"], s["dloss"], s["dhidden"], s["dweight"])
    return s["dhidden"], s["dweight"]


# ---- the same in 64 bits, from the definitions -----------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    D = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    if case["op"] == "rotary":
        half, out = case["part"] // 2, []
        turn = torch.polar(torch.full((), s["magnitude"], dtype=torch.float64, device="cuda"),
                           D["positions"][:, None] * D["frequencies"] * (-1 if case["inverse"] else 1))[:, None, :]
        for name in ("q", "k"):
            x = D[name].clone()
            first, second = (slice(0, half), slice(half, 2 * half)) if case["layout"] == "half" else (slice(0, 2 * half, 2), slice(1, 2 * half, 2))
            z = torch.complex(x[..., first], x[..., second]) * turn
            x[..., first], x[..., second] = z.real, z.imag
            out.append(x)
        return tuple(out)
    if case["op"].startswith("attention"):
        h, group = case["heads"], case["heads"] // case["kv_heads"]
        forward = case["op"] == "attention_forward"
        names = ("o", "lse") if forward else ("dq", "dk", "dv")
        R = {n: torch.zeros_like(D[n]) for n in names}
        a = 0
        for n in s["lengths"]:
            b = a + n
            later = torch.ones(n, n, dtype=torch.bool, device="cuda").triu(1) if case["causal"] else None
            for i in range(h if n else 0):
                q, k, v = D["q"][a:b, i], D["k"][a:b, i // group], D["v"][a:b, i // group]
                x = torch.einsum("td,sd->ts", q, k) / math.sqrt(case["dim"])
                if later is not None:
                    x[later] = -math.inf
                z = torch.logsumexp(x, 1)
                p = torch.softmax(x, 1)
                if forward:
                    R["o"][a:b, i], R["lse"][i, a:b] = torch.einsum("ts,sd->td", p, v), z
                    continue
                g = D["do"][a:b, i]
                R["dv"][a:b, i // group] += torch.einsum("ts,td->sd", p, g)
                dp = torch.einsum("td,sd->ts", g, v)
                dx = p * (dp - torch.einsum("ts,ts->t", p, dp)[:, None]) / math.sqrt(case["dim"])
                R["dq"][a:b, i] = torch.einsum("ts,sd->td", dx, k)
                R["dk"][a:b, i // group] += torch.einsum("ts,td->sd", dx, q)
            a = b
        return tuple(R[n] for n in names)
    t = D["targets"].long()
    valid = t >= 0
    out = ([], []) if case["op"] == "loss_forward" else ([], torch.zeros_like(D["dweight"]))
    for a in range(0, case["tokens"], 1024):                       # 64-bit logits of all tokens would be 2 GB and more
        cut, ok = slice(a, a + 1024), valid[a: a + 1024]
        x = torch.einsum("td,vd->tv", D["hidden"][cut], D["weight"])
        z = torch.logsumexp(x, 1)
        if case["op"] == "loss_forward":
            out[0].append(torch.where(ok, z - x[torch.arange(x.shape[0]), t[cut].clamp(min=0)], 0.0))
            out[1].append(z)
            continue
        p = torch.softmax(x, 1)
        p[torch.arange(x.shape[0])[ok.cpu()], t[cut][ok]] -= 1.0
        p *= (D["dloss"][cut] * ok)[:, None]
        out[0].append(torch.einsum("tv,vd->td", p, D["weight"]))
        out[1].add_(torch.einsum("tv,td->vd", p, D["hidden"][cut]))
    return torch.cat(out[0]), out[1] if case["op"] == "loss_backward" else torch.cat(out[1])
