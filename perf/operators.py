"""The cases by which the learner's operators are measured: the gated feed-forward block (forward and
backward), the global gradient norm with clipping, and the AdamW step.

``run`` computes them in their plain form, in 32 bits with elementary torch operations; with ``own`` set it
makes the library's calls.  The tensors of a gradient or parameter list lie in one flat buffer, each on a
boundary of 128 elements with zeros in between, so that the plain form is one expression over the buffer.
"""
import math

import torch

own = False

STD_WEIGHT = 0.02          # parameters, as everywhere in this repository's synthetic inputs
STD_GRAD = 2e-3            # gradients: norms of a few units at 10^6 parameters and more, so that clipping acts
MAX_NORM = 1.0
LR, BETA1, BETA2, EPS, DECAY = 3e-4, 0.9, 0.95, 1e-8, 0.1
STEP = 100
PAD = 128                  # elements between the starts of neighbouring tensors are a multiple of this
COST = {"ffn": 8192 * 2048 * 8192, "list": 3 * (4 * 2048 * 2048 + 2 * 2048 * 8192)}   # largest listed


# ---- the cases -------------------------------------------------------------------------------------

def ffn(name, op, tokens, d, f, act, save=False, residual=True):
    return dict(name=name, op=op, tokens=tokens, d=d, f=f, act=act, save=save, residual=residual)


def tensors(name, op, layers, d, f, dtype, clip=False):
    return dict(name=name, op=op, layers=layers, d=d, f=f, dtype=dtype, clip=clip)


def listed():
    return [
        # one decoded token through the block of a 1.3B-parameter decoder: latency and the matrices' bytes
        ffn("block_one_token", "ffn_forward", 1, 2048, 8192, "silu"),
        # a ragged batch of prompts through a block with odd widths (rows padded to 16 bytes)
        ffn("block_odd", "ffn_forward", 203, 2047, 5461, "gelu", save=True),
        # a learner's training micro-batch: the forward pass that keeps what backward needs
        ffn("block_train", "ffn_forward", 8192, 2048, 8192, "silu", save=True),
        # the backward pass of a small learner with few tokens
        ffn("block_back_small", "ffn_backward", 96, 768, 2048, "silu"),
        # backward at odd sizes throughout
        ffn("block_back_odd", "ffn_backward", 1777, 1001, 2731, "gelu"),
        # the backward pass of the training micro-batch above
        ffn("block_back_train", "ffn_backward", 8192, 2048, 8192, "silu"),
        # the gradient norm of a tiny model: launch latency
        tensors("norm_small", "grad_norm", 1, 256, 1024, "f32"),
        # the gradient norm of a 1.2B-parameter decoder in bf16, 192 tensors
        tensors("norm_model", "grad_norm", 24, 2048, 8192, "bf16"),
        # clipping a small model with odd widths, gradients in fp32
        tensors("clip_odd", "clip", 2, 577, 2311, "f32"),
        # clipping one fragment (three layers, 151M parameters) in bf16
        tensors("clip_fragment", "clip", 3, 2048, 8192, "bf16"),
        # the optimizer step of a small model, gradients in bf16, no clipping
        tensors("adamw_small", "adamw", 1, 512, 2048, "bf16"),
        # the inner step of one fragment: norm, then AdamW with the clip scale, gradients in fp32
        tensors("adamw_fragment", "adamw", 3, 2048, 8192, "f32", clip=True),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["ffn_forward", "ffn_backward", "grad_norm", "clip", "adamw"])
    if op.startswith("ffn"):
        while True:
            t, d, f = spread(1, 8192), spread(256, 4096), spread(512, 12288)
            if rng.random() < 0.5:
                d, f = d - d % 8, f - f % 8
            if t * d * f <= COST["ffn"] and d * f <= 2048 * 8192:
                break
        c = ffn("", op, t, d, f, rng.choice(["silu", "gelu"]), save=rng.random() < 0.5, residual=rng.random() < 0.5)
        if op == "ffn_backward":
            c["save"], c["residual"] = False, True
    else:
        while True:
            layers, d = rng.randint(1, 24), spread(64, 2048)
            f = int(d * rng.uniform(2, 4.5))
            if layers * (4 * d * d + 2 * d * f) <= COST["list"]:
                break
        c = tensors("", op, layers, d, f, rng.choice(["bf16", "f32"]), clip=op == "adamw" and rng.random() < 0.5)
    del c["name"]
    return c


def sizes_of(case):
    """Element counts of the tensors of `layers` decoder layers: four d x d, two d x f, two gains."""
    d, f = case["d"], case["f"]
    return ([d * d] * 4 + [d * f] * 2 + [d] * 2) * case["layers"]


def rows(n):
    """Row length in memory of a row of n bf16 elements: whole 16 bytes."""
    return (n + 7) // 8 * 8


def work(case):
    if case["op"].startswith("ffn"):
        t, d, f = case["tokens"], case["d"], case["f"]
        if case["op"] == "ffn_forward":
            values = 3 * d * f + t * d * (3 if case["residual"] else 2) + (2 * t * f if case["save"] else 0)
            return {"bytes": 2 * values, "flops": 6 * t * d * f}
        return {"bytes": 2 * (6 * d * f + 3 * t * d + 2 * t * f), "flops": 12 * t * d * f}
    n, g = sum(sizes_of(case)), 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "grad_norm":
        return {"bytes": g * n, "flops": 2 * n}
    if case["op"] == "clip":
        return {"bytes": 2 * g * n, "flops": 3 * n}
    return {"bytes": (26 + g) * n, "flops": 16 * n}


# ---- what a program has in hand --------------------------------------------------------------------

def randn(gen, *shape, std=1.0, dtype=torch.bfloat16):
    """Normal values in a buffer whose rows start on 16-byte boundaries."""
    ld = rows(shape[-1])
    x = torch.randn(*shape[:-1], ld, generator=gen, device="cuda", dtype=torch.float32)
    return x.mul_(std).to(dtype)[..., : shape[-1]]


def empty(*shape):
    return torch.zeros(*shape[:-1], rows(shape[-1]), device="cuda", dtype=torch.bfloat16)[..., : shape[-1]]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": case}
    if case["op"].startswith("ffn"):
        t, d, f = case["tokens"], case["d"], case["f"]
        s["x"] = randn(gen, t, d)
        s["w_gate"], s["w_up"] = (randn(gen, f, d, std=STD_WEIGHT) for _ in range(2))
        s["w_down"] = randn(gen, d, f, std=STD_WEIGHT)
        if case["op"] == "ffn_forward":
            s["residual"] = randn(gen, t, d) if case["residual"] else None
            s["y"] = empty(t, d)
            s["gate"], s["up"] = (empty(t, f), empty(t, f)) if case["save"] else (None, None)
        else:
            s["gate"], s["up"] = empty(t, f), empty(t, f)      # what the forward pass kept
            s["gate"].copy_(s["x"] @ s["w_gate"].t())
            s["up"].copy_(s["x"] @ s["w_up"].t())
            s["dy"] = randn(gen, t, d, std=STD_GRAD)
            s["dx"], s["dw_gate"], s["dw_up"], s["dw_down"] = empty(t, d), empty(f, d), empty(f, d), empty(d, f)
        return s
    dtype = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
    sizes, starts, total = sizes_of(case), [], 0
    for n in sizes:
        starts.append(total)
        total += (n + PAD - 1) // PAD * PAD

    def flat(std, kind=torch.float32, square=False):
        x = torch.randn(total, generator=gen, device="cuda", dtype=torch.float32).mul_(std)
        for a, n in zip(starts, sizes):                        # nothing between the tensors
            x[a + n: a + (n + PAD - 1) // PAD * PAD] = 0
        return (x.square_() if square else x).to(kind)

    def views(x):
        return [x[a: a + n] for a, n in zip(starts, sizes)]

    s["flat_grads"] = flat(STD_GRAD, dtype)
    s["grads"] = views(s["flat_grads"])
    if case["op"] == "clip":
        s["flat_out"] = torch.zeros_like(s["flat_grads"])
        s["out"] = views(s["flat_out"])
    if case["op"] == "adamw":
        s["step"] = STEP
        s["flat_params"], s["flat_m"] = flat(STD_WEIGHT), flat(0.2 * STD_GRAD)
        s["flat_v"] = flat(STD_GRAD, square=True)
        s["flat_copy"] = torch.zeros(total, device="cuda", dtype=torch.bfloat16)
        for k in ("params", "m", "v", "copy"):
            s[k] = views(s["flat_" + k])
    return s


# ---- one pass --------------------------------------------------------------------------------------

def activation(g, kind):
    """The activation and its derivative."""
    if kind == "silu":
        p = torch.sigmoid(g)
        return g * p, p * (1 + g * (1 - p))
    c = math.sqrt(2 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * c * (1 + 3 * 0.044715 * g * g)


def block_forward(x, w_gate, w_up, w_down, residual, kind):
    gate, up = x @ w_gate.t(), x @ w_up.t()
    y = (activation(gate, kind)[0] * up) @ w_down.t()
    return y if residual is None else residual + y, gate, up


def block_backward(x, w_gate, w_up, w_down, gate, up, dy, kind):
    a, slope = activation(gate, kind)
    dh = dy @ w_down
    dgate, dup = dh * up * slope, dh * a
    return dgate @ w_gate + dup @ w_up, dgate.t() @ x, dup.t() @ x, dy.t() @ (a * up)


def norm_and_scale(g, max_norm):
    norm = g.square().sum().sqrt()
    return norm, torch.clamp(max_norm / (norm + 1e-6), max=1.0)


def adamw(p, g, m, v, step, scale):
    """The updated parameters and moments."""
    g = g * scale
    m = BETA1 * m + (1 - BETA1) * g
    v = BETA2 * v + (1 - BETA2) * g * g
    hat = m / (1 - BETA1 ** step) / ((v / (1 - BETA2 ** step)).sqrt() + EPS)
    return p * (1 - LR * DECAY) - LR * hat, m, v


def run(s):
    return run_own(s) if own else run_plain(s)


def run_plain(s):
    c, b = s["case"], torch.bfloat16
    if c["op"] == "ffn_forward":
        ins = [None if s[k] is None else s[k].float() for k in ("x", "w_gate", "w_up", "w_down", "residual")]
        y, gate, up = block_forward(*ins, c["act"])
        return (y.to(b), gate.to(b), up.to(b)) if c["save"] else (y.to(b),)
    if c["op"] == "ffn_backward":
        ins = [s[k].float() for k in ("x", "w_gate", "w_up", "w_down", "gate", "up", "dy")]
        return tuple(r.to(b) for r in block_backward(*ins, c["act"]))
    g = s["flat_grads"].float()
    if c["op"] == "grad_norm":
        return torch.stack(norm_and_scale(g, MAX_NORM))
    if c["op"] == "clip":
        norm, scale = norm_and_scale(g, MAX_NORM)
        return s["flat_out"].copy_(g * scale), torch.stack((norm, scale))
    scale = norm_and_scale(g, MAX_NORM)[1] if c["clip"] else 1.0
    p, m, v = adamw(s["flat_params"], g, s["flat_m"], s["flat_v"], s["step"], scale)
    s["step"] += 1
    return s["flat_params"].copy_(p), s["flat_m"].copy_(m), s["flat_v"].copy_(v), s["flat_copy"].copy_(p)


_library = {}


def library():
    """The library's binding and this program's context on the current GPU."""
    if not _library:
        from paper_2604_21428_b200 import ddmerge as dd
        _library.update(dd=dd, ctx=dd.Context(torch.cuda.current_device()), record=dd.new_grad_record())
    return _library["dd"], _library["ctx"], _library["record"]


def run_own(s):
    c = s["case"]
    dd, ctx, record = library()
    act = dd.ACT_SILU if c.get("act") == "silu" else dd.ACT_GELU_TANH
    if c["op"] == "ffn_forward":
        ctx.gated_ffn_forward(s["x"], s["w_gate"], s["w_up"], s["w_down"], s["y"], activation=act,
                              residual=s["residual"], gate=s["gate"], up=s["up"])
        return (s["y"], s["gate"], s["up"]) if c["save"] else (s["y"],)
    if c["op"] == "ffn_backward":
        ctx.gated_ffn_backward(s["x"], s["w_gate"], s["w_up"], s["w_down"], s["gate"], s["up"], s["dy"],
                               s["dx"], s["dw_gate"], s["dw_up"], s["dw_down"], activation=act)
        return s["dx"], s["dw_gate"], s["dw_up"], s["dw_down"]
    if c["op"] == "grad_norm":
        ctx.grad_norm(s["grads"], MAX_NORM, record)
        return record[:2]
    if c["op"] == "clip":
        ctx.clip_gradients(s["grads"], MAX_NORM, record, out=s["out"])
        return s["flat_out"], record[:2]
    if c["clip"]:
        ctx.grad_norm(s["grads"], MAX_NORM, record)
    ctx.adamw_step(s["params"], s["grads"], s["m"], s["v"], s["step"], LR, beta1=BETA1, beta2=BETA2, eps=EPS,
                   weight_decay=DECAY, copies=s["copy"], clip=record if c["clip"] else None)
    s["step"] += 1
    return s["flat_params"], s["flat_m"], s["flat_v"], s["flat_copy"]


# ---- the same in 64 bits, from the definitions -----------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    D = {k: v.double() for k, v in s.items() if isinstance(v, torch.Tensor)}
    if case["op"].startswith("ffn"):
        def sigmoid(z):
            return 1 / (1 + torch.exp(-z))

        k, q = 2 * math.sqrt(2 / math.pi), 0.044715
        fwd = case["op"] == "ffn_forward"
        G = torch.einsum("td,fd->tf", D["x"], D["w_gate"]) if fwd else D["gate"]
        U = torch.einsum("td,fd->tf", D["x"], D["w_up"]) if fwd else D["up"]
        inner = G if case["act"] == "silu" else k * (G + q * G ** 3)       # both are G sigmoid(inner)
        A = G * sigmoid(inner)
        if fwd:
            Y = torch.einsum("tf,df->td", A * U, D["w_down"])
            Y = Y + D["residual"] if case["residual"] else Y
            return (Y, G, U) if case["save"] else (Y,)
        slope = sigmoid(inner) + A * sigmoid(-inner) * (1.0 if case["act"] == "silu" else k * (1 + 3 * q * G ** 2))
        dH = torch.einsum("td,df->tf", D["dy"], D["w_down"])
        dG, dU = dH * U * slope, dH * A
        return (torch.einsum("tf,fd->td", dG, D["w_gate"]) + torch.einsum("tf,fd->td", dU, D["w_up"]),
                torch.einsum("tf,td->fd", dG, D["x"]), torch.einsum("tf,td->fd", dU, D["x"]),
                torch.einsum("td,tf->df", D["dy"], A * U))
    g = D["flat_grads"]
    norm = torch.linalg.vector_norm(g)
    scale = min(1.0, MAX_NORM / (float(norm) + 1e-6))
    both = torch.tensor([float(norm), scale], dtype=torch.float64, device="cuda")
    if case["op"] == "grad_norm":
        return both
    if case["op"] == "clip":
        return g * scale, both
    g = g * scale if case["clip"] else g
    m = torch.lerp(g, D["flat_m"], BETA1)
    v = torch.lerp(g * g, D["flat_v"], BETA2)
    t = s["step"]
    p = D["flat_params"] - LR * DECAY * D["flat_params"]
    p = p - LR * (m / -math.expm1(t * math.log(BETA1))) / (torch.sqrt(v / -math.expm1(t * math.log(BETA2))) + EPS)
    return p, m, v, p
