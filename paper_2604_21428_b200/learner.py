"""A learner's inner steps (Algorithm 1) between the syncer's merges, on the library's operators.

``Learner``'s model is a stack of residual gated feed-forward blocks, one block per fragment.  Every fragment
is a flat concatenation of w_gate, w_up and w_down, held as float32 parameters with AdamW's moments,
float32 gradients, and the bf16 copy that the block computes with and ``dd_merge_fragment`` reads.
An inner step is forward, backward, the gradients' global norm, and AdamW with the clip scale; the
syncer's merge then pushes the new global fragment into the copies.  What the operators report in a learner's status word
(a wait that ran out, offsets that make no sense) holds its steps back until ``check`` has raised it, before a merge.

``DecoderLearner``'s model is a decoder: embedding, layers of attention and gated feed-forward block, and the
loss over the vocabulary, trained on documents packed end to end.  Its fragments are the layers and, last, the
embedding with the head.

    python -m paper_2604_21428_b200.learner              # a few learners fit a random teacher
    python -m paper_2604_21428_b200.learner decoder      # a few learners train a small decoder
"""
from __future__ import annotations

import math
import sys

import torch

from . import ddmerge as dd


def hold_back(record, status) -> None:
    """A step whose operators reported something is not applied, like one whose gradients are not finite."""
    record.view(torch.int32)[2:3].bitwise_or_(status)          # the record's own status


def raise_status(status) -> None:
    """Raises what operators reported since the last time, if anything; waits for them."""
    code = int(status)
    if code:
        status.zero_()
        raise RuntimeError(f"inner steps were not applied: an operator reported status {code}")


class Learner:
    """One learner's model, optimizer state and gradients.  ``d`` and ``f`` are multiples of 8: the rows of a
    fragment's matrices follow one another, and each starts on 16 bytes."""

    def __init__(self, ctx: "dd.Context", d: int, f: int, blocks: int, tokens: int, *, lr: float = 1e-3,
                 weight_decay: float = 0.0, max_norm: float = 1.0, activation: int = dd.ACT_SILU, device="cuda"):
        self.ctx, self.d, self.f, self.tokens = ctx, d, f, tokens
        self.lr, self.weight_decay, self.max_norm, self.activation = lr, weight_decay, max_norm, activation
        self.steps = 0

        def fragments(dtype):
            return [torch.zeros(3 * d * f, dtype=dtype, device=device) for _ in range(blocks)]

        self.params, self.grads = fragments(torch.float32), fragments(torch.float32)
        self.exp_avg, self.exp_avg_sq = fragments(torch.float32), fragments(torch.float32)
        self.copies = fragments(torch.bfloat16)
        self.weights = [self._views(c) for c in self.copies]
        self.weight_grads = [self._views(g) for g in self.grads]

        def rows(n):
            return torch.empty(tokens, n, dtype=torch.bfloat16, device=device)

        self.x = [rows(d) for _ in range(blocks + 1)]          # block inputs, and the output
        self.gate, self.up = [rows(f) for _ in range(blocks)], [rows(f) for _ in range(blocks)]
        self.dx = rows(d)
        self.scratch = torch.empty(3 * tokens * ((f + 7) // 8 * 8), dtype=torch.bfloat16, device=device)
        self.record = dd.new_grad_record(device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)

    def _views(self, flat):
        d, f = self.d, self.f
        return flat[: d * f].view(f, d), flat[d * f: 2 * d * f].view(f, d), flat[2 * d * f:].view(d, f)

    def receive(self, p: int, fragment) -> None:
        """Takes global fragment ``p`` (float32), as after a push."""
        self.params[p].copy_(fragment)
        self.copies[p].copy_(fragment)

    def forward(self, x):
        self.x[0].copy_(x)
        for i, w in enumerate(self.weights):
            self.ctx.gated_ffn_forward(self.x[i], *w, self.x[i + 1], activation=self.activation, residual=self.x[i],
                                       gate=self.gate[i], up=self.up[i], hidden=self.scratch, status=self.status)
        return self.x[-1]

    def backward(self, dy) -> None:
        """Gradients of every block for the output's gradient ``dy`` (bfloat16), into ``grads``."""
        for i in reversed(range(len(self.weights))):
            self.ctx.gated_ffn_backward(self.x[i], *self.weights[i], self.gate[i], self.up[i], dy, self.dx,
                                        *self.weight_grads[i], activation=self.activation, scratch=self.scratch, status=self.status)
            dy = dy + self.dx                                  # the residual branch

    def step(self, x, target) -> torch.Tensor:
        """One inner step on the mean squared error; returns the loss (a device scalar)."""
        diff = self.forward(x).float() - target.float()
        self.backward((diff * (2.0 / diff.numel())).to(torch.bfloat16))
        self.ctx.grad_norm(self.grads, self.max_norm, self.record)
        hold_back(self.record, self.status)
        self.steps += 1
        self.ctx.adamw_step(self.params, self.grads, self.exp_avg, self.exp_avg_sq, self.steps, self.lr,
                            weight_decay=self.weight_decay, copies=self.copies, clip=self.record)
        return diff.square().mean()

    def check(self) -> None:
        """Raises if steps since the last check were held back by what an operator reported."""
        raise_status(self.status)


def train(ctx: "dd.Context", *, learners: int = 4, d: int = 256, f: int = 512, blocks: int = 2, tokens: int = 512,
          rounds: int = 6, inner_steps: int = 30,
          lr: float = 1e-2, outer_lr: float = 0.7, outer_mu: float = 0.9, seed: int = 0):
    """``learners`` learners fit a random teacher; after every ``inner_steps`` steps each fragment is
    merged over all of them and pushed back.  Returns the mean loss of each round."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def randn(*shape, std=1.0):
        return torch.randn(*shape, generator=gen, device="cuda") * std

    teacher = Learner(ctx, d, f, blocks, tokens)
    group = [Learner(ctx, d, f, blocks, tokens, lr=lr) for _ in range(learners)]
    theta = [randn(3 * d * f, std=0.02) for _ in range(blocks)]
    momentum = [torch.zeros_like(t) for t in theta]
    for p in range(blocks):
        teacher.receive(p, theta[p] + randn(3 * d * f, std=0.05))
        for m in group:
            m.receive(p, theta[p])
    everyone = (1 << learners) - 1
    records = dd.new_records(blocks)
    history = []
    for _ in range(rounds):
        total = torch.zeros((), device="cuda")
        for _ in range(inner_steps):
            for m in group:
                x = randn(tokens, d).to(torch.bfloat16)
                total += m.step(x, teacher.forward(x))
        history.append(float(total) / (inner_steps * learners))
        for m in (teacher, *group):
            m.check()
        frags = [dict(global_=theta[p], momentum=momentum[p], learners=[m.copies[p] for m in group],
                      tokens=[inner_steps * tokens] * learners, quorum_mask=everyone, K=learners, n=3 * d * f)
                 for p in range(blocks)]
        ctx.merge_fragments_batched_push(frags, [everyone] * blocks, learners, dd.BF16, outer_lr, outer_mu, records=records)
        for p in range(blocks):
            for m in group:
                m.params[p].copy_(theta[p])                    # the copies were pushed
    return history


def normed(x):
    """Rows of ``x`` over their root mean square, in float32, and what they were divided by."""
    r = (x.float().square().mean(-1, keepdim=True) + 1e-6).sqrt()
    return (x.float() / r), r


def normed_backward(dy, y, r):
    """Gradient of ``normed``'s argument for its result's gradient."""
    return (dy - y * (dy * y).mean(-1, keepdim=True)) / r


class DecoderLearner:
    """One learner's decoder, optimizer state and gradients.

    A layer is ``x += attention(norm(x)); x += gated_ffn(norm(x))`` with rotary positions and grouped heads; norms have
    no gains.  ``tokens`` is the micro-batch's room: documents may leave some of it at the end.  ``d``, ``f``
    and ``dim`` are multiples of 8.  The projections to and from the heads are plain matrix products."""

    def __init__(self, ctx: "dd.Context", *, vocab: int, d: int, f: int, layers: int, heads: int, kv_heads: int, dim: int,
                 tokens: int, sequences: int, lr: float = 1e-3, weight_decay: float = 0.0, max_norm: float = 1.0, device="cuda"):
        self.ctx, self.vocab, self.d, self.f, self.tokens = ctx, vocab, d, f, tokens
        self.heads, self.kv_heads, self.dim = heads, kv_heads, dim
        self.lr, self.weight_decay, self.max_norm, self.steps = lr, weight_decay, max_norm, 0
        rows = (heads + 2 * kv_heads) * dim
        layer = [(rows, d), (d, heads * dim), (f, d), (f, d), (d, f)]
        self.shapes = [layer] * layers + [[(vocab, d), (vocab, d)]]                 # embedding, head
        self.sizes = [sum(m * n for m, n in shapes) for shapes in self.shapes]

        def fragments(dtype):
            return [torch.zeros(n, dtype=dtype, device=device) for n in self.sizes]

        self.params, self.grads = fragments(torch.float32), fragments(torch.float32)
        self.exp_avg, self.exp_avg_sq = fragments(torch.float32), fragments(torch.float32)
        self.copies = fragments(torch.bfloat16)
        self.weights = [self._views(p, c) for p, c in enumerate(self.copies)]
        self.weight_grads = [self._views(p, g) for p, g in enumerate(self.grads)]

        def room(*shape, dtype=torch.bfloat16):
            return torch.zeros(*shape, dtype=dtype, device=device)

        self.frequencies, _ = dd.rotary_frequencies(dim, device=device)
        self.kept = [dict(qkv=room(tokens, heads + 2 * kv_heads, dim), o=room(tokens, heads, dim),
                          lse=room(heads, tokens, dtype=torch.float32), gate=room(tokens, f), up=room(tokens, f)) for _ in range(layers)]
        self.loss, self.lse = room(tokens, dtype=torch.float32), room(tokens, dtype=torch.float32)
        self.dqkv, self.d_o = room(tokens, heads + 2 * kv_heads, dim), room(tokens, heads, dim)
        self.dx = room(tokens, d)
        self.scratch = room(3 * tokens * ((f + 7) // 8 * 8))
        self.attention_scratch = room(dd.attention_scratch_bytes(tokens, heads, kv_heads, dim, sequences, backward=True), dtype=torch.uint8)
        self.loss_scratch = room(max(ctx.vocab_loss_scratch_bytes(tokens, d, vocab, backward=b) for b in (False, True)), dtype=torch.uint8)
        self.record = dd.new_grad_record(device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.trained = torch.zeros((), dtype=torch.int64, device=device)            # tokens with a target, of applied steps

    def _views(self, p, flat):
        views, at = [], 0
        for m, n in self.shapes[p]:
            views.append(flat[at: at + m * n].view(m, n))
            at += m * n
        return views

    def initial(self, gen) -> list:
        """A random global fragment for each of this decoder's fragments."""
        out = []
        for shapes in self.shapes:
            out.append(torch.cat([torch.randn(m * n, generator=gen, device=self.dx.device) / math.sqrt(n) for m, n in shapes]))
        return out

    def receive(self, p: int, fragment) -> None:
        """Takes global fragment ``p`` (float32), as after a push."""
        self.params[p].copy_(fragment)
        self.copies[p].copy_(fragment)

    def _split(self, qkv):
        h, kv = self.heads, self.kv_heads
        return qkv[:, :h], qkv[:, h: h + kv], qkv[:, h + kv:]

    def forward(self, ids, targets, positions, offsets):
        """The loss of every token.  ``ids`` and ``targets`` int64 [tokens], ``targets`` negative where there is none
        (between documents and behind the last); ``positions`` from each document's start, -1 behind the last;
        ``offsets`` int32, where each document starts and the last one ends."""
        bf, b = torch.bfloat16, self.kept
        embedding, head = self.weights[-1]
        x = embedding[ids]
        self.batch = (ids, targets, positions, offsets)
        for i, keep in enumerate(b):
            w_qkv, w_o, *block = self.weights[i]
            keep["y1"], keep["r1"] = normed(x)
            keep["h1"] = keep["y1"].to(bf)
            keep["qkv"].copy_((keep["h1"] @ w_qkv.t()).view_as(keep["qkv"]))
            q, k, v = self._split(keep["qkv"])
            self.ctx.rotary(q, k, positions, self.frequencies)
            keep["o"].zero_()                                  # rows behind the last document stay as they are
            self.ctx.attention_forward(q, k, v, keep["o"], keep["lse"], offsets=offsets, scratch=self.attention_scratch, status=self.status)
            x = x + keep["o"].flatten(1) @ w_o.t()
            keep["y2"], keep["r2"] = normed(x)
            keep["h2"] = keep["y2"].to(bf)
            y = torch.empty_like(x)
            self.ctx.gated_ffn_forward(keep["h2"], *block, y, residual=x, gate=keep["gate"], up=keep["up"], hidden=self.scratch,
                                       status=self.status)
            x = y
        self.y, self.r = normed(x)
        self.hidden = self.y.to(bf)
        self.ctx.vocab_loss_forward(self.hidden, head, targets, self.loss, self.lse, scratch=self.loss_scratch, status=self.status)
        return self.loss

    def backward(self, dloss) -> None:
        """Gradients for ``dloss``, the derivative by each token's loss (float32), into ``grads``."""
        bf, (ids, targets, positions, offsets) = torch.bfloat16, self.batch
        d_embedding, d_head = self.weight_grads[-1]
        self.ctx.vocab_loss_backward(self.hidden, self.weights[-1][1], targets, self.lse, dloss, self.dx, d_head, scratch=self.loss_scratch,
                                     status=self.status)
        dx = normed_backward(self.dx.float(), self.y, self.r)
        for i in reversed(range(len(self.kept))):
            keep, (w_qkv, w_o, *block), (dw_qkv, dw_o, *dblock) = self.kept[i], self.weights[i], self.weight_grads[i]
            self.ctx.gated_ffn_backward(keep["h2"], *block, keep["gate"], keep["up"], dx.to(bf), self.dx, *dblock, scratch=self.scratch,
                                        status=self.status)
            dx = dx + normed_backward(self.dx.float(), keep["y2"], keep["r2"])
            dy = dx.to(bf)
            self.d_o.copy_((dy @ w_o).view_as(self.d_o))
            torch.mm(dy.t(), keep["o"].flatten(1), out_dtype=torch.float32, out=dw_o)      # sums are not rounded to bf16
            q, k, v = self._split(keep["qkv"])
            dq, dk, dv = self._split(self.dqkv)
            self.dqkv.zero_()                                  # as above
            self.ctx.attention_backward(q, k, v, keep["o"], keep["lse"], self.d_o, dq, dk, dv, offsets=offsets, scratch=self.attention_scratch,
                                        status=self.status)
            self.ctx.rotary(dq, dk, positions, self.frequencies, inverse=True)
            dqkv = self.dqkv.flatten(1)
            torch.mm(dqkv.t(), keep["h1"], out_dtype=torch.float32, out=dw_qkv)
            dx = dx + normed_backward((dqkv @ w_qkv).float(), keep["y1"], keep["r1"])
        d_embedding.zero_().index_put_((ids,), dx, accumulate=True)

    def step(self, ids, targets, positions, offsets) -> torch.Tensor:
        """One inner step on the mean loss of the tokens that have a target; returns it (a device scalar).  Without any
        the loss and its gradients are 0."""
        loss = self.forward(ids, targets, positions, offsets)
        some = (targets >= 0).sum()
        count = some.clamp(min=1)
        self.backward((1.0 / count).float().expand(self.tokens).contiguous())
        self.ctx.grad_norm(self.grads, self.max_norm, self.record)
        hold_back(self.record, self.status)
        self.steps += 1
        self.ctx.adamw_step(self.params, self.grads, self.exp_avg, self.exp_avg_sq, self.steps, self.lr,
                            weight_decay=self.weight_decay, copies=self.copies, clip=self.record)
        self.trained += some * (self.record.view(torch.int32)[2] == dd.STATUS_OK)
        return loss.sum() / count

    def check(self) -> None:
        """Raises if steps since the last check were held back by what an operator reported."""
        raise_status(self.status)


def packed_documents(gen, tokens: int, sequences: int, vocab: int, device="cuda"):
    """A micro-batch of up to ``sequences`` documents of random lengths, each counting up in steps of its own
    modulo ``vocab``: ids, targets, positions and offsets for ``DecoderLearner.step``."""
    cuts = torch.randint(1, tokens + 1, (sequences,), generator=gen, device=device).sort().values
    offsets = torch.cat([cuts.new_zeros(1), cuts]).to(torch.int32)
    t = torch.arange(tokens, device=device)
    doc = torch.searchsorted(cuts, t, right=True)
    inside = t < cuts[-1]
    positions = torch.where(inside, t - offsets.long()[doc.clamp(max=sequences - 1)], -1)
    first = torch.randint(0, vocab, (sequences + 1,), generator=gen, device=device)
    stride = torch.randint(1, 4, (sequences + 1,), generator=gen, device=device)
    ids = (first[doc] + stride[doc] * positions.clamp(min=0)) % vocab
    last = torch.cat([doc[1:] != doc[:-1], doc.new_ones(1, dtype=torch.bool)])
    targets = torch.where(inside & ~last, (ids + stride[doc]) % vocab, -100)
    return ids, targets, positions, offsets


def train_decoder(ctx: "dd.Context", *, learners: int = 2, vocab: int = 512, d: int = 128, f: int = 256, layers: int = 2, heads: int = 4,
                  kv_heads: int = 2, dim: int = 32, tokens: int = 512, sequences: int = 6, rounds: int = 5, inner_steps: int = 20,
                  lr: float = 3e-3, outer_lr: float = 0.7, outer_mu: float = 0.9, seed: int = 0):
    """``learners`` learners train one decoder; after every ``inner_steps`` steps each fragment is merged over all
    of them and pushed back, each learner weighed by the tokens with a target that it trained on.  Returns the mean loss of
    each round."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    sizes = dict(vocab=vocab, d=d, f=f, layers=layers, heads=heads, kv_heads=kv_heads, dim=dim, tokens=tokens, sequences=sequences)
    group = [DecoderLearner(ctx, **sizes, lr=lr) for _ in range(learners)]
    theta = group[0].initial(gen)
    momentum = [torch.zeros_like(t) for t in theta]
    for p, fragment in enumerate(theta):
        for m in group:
            m.receive(p, fragment)
    everyone = (1 << learners) - 1
    records = dd.new_records(len(theta))
    history = []
    for _ in range(rounds):
        total = torch.zeros((), device="cuda")
        for _ in range(inner_steps):
            for m in group:
                total += m.step(*packed_documents(gen, tokens, sequences, vocab))
        history.append(float(total) / (inner_steps * learners))
        for m in group:
            m.check()
        trained = [int(m.trained) for m in group]
        for m in group:
            m.trained.zero_()
        frags = [dict(global_=theta[p], momentum=momentum[p], learners=[m.copies[p] for m in group],
                      tokens=trained, quorum_mask=everyone, K=learners, n=theta[p].numel())
                 for p in range(len(theta))]
        ctx.merge_fragments_batched_push(frags, [everyone] * len(theta), learners, dd.BF16, outer_lr, outer_mu, records=records)
        for p in range(len(theta)):
            for m in group:
                m.params[p].copy_(theta[p])                    # the copies were pushed
    return history


if __name__ == "__main__":
    what = sys.argv[1] if len(sys.argv) > 1 else "teacher"
    if what not in ("teacher", "decoder"):
        sys.exit(f"unknown model {what!r}: teacher or decoder")
    context = dd.Context(torch.cuda.current_device())
    if what == "teacher":
        for r, loss in enumerate(train(context)):
            print(f"round {r}: mean squared error {loss:.5f}")
    else:
        for r, loss in enumerate(train_decoder(context)):
            print(f"round {r}: mean loss {loss:.5f}")
