"""A learner's inner steps (Algorithm 1) between the syncer's merges, on the library's operators.

The model is a stack of residual gated feed-forward blocks, one block per fragment.  Every fragment
is a flat concatenation of w_gate, w_up and w_down, held as float32 parameters with AdamW's moments,
float32 gradients, and the bf16 copy that the block computes with and ``dd_merge_fragment`` reads.
An inner step is forward, backward, the gradients' global norm, and AdamW with the clip scale; the
syncer's merge then pushes the new global fragment into the copies.

    python -m paper_2604_21428_b200.learner        # a few learners fit a random teacher
"""
from __future__ import annotations

import torch

from . import ddmerge as dd


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
                                       gate=self.gate[i], up=self.up[i], hidden=self.scratch)
        return self.x[-1]

    def backward(self, dy) -> None:
        """Gradients of every block for the output's gradient ``dy`` (bfloat16), into ``grads``."""
        for i in reversed(range(len(self.weights))):
            self.ctx.gated_ffn_backward(self.x[i], *self.weights[i], self.gate[i], self.up[i], dy, self.dx,
                                        *self.weight_grads[i], activation=self.activation, scratch=self.scratch)
            dy = dy + self.dx                                  # the residual branch

    def step(self, x, target) -> torch.Tensor:
        """One inner step on the mean squared error; returns the loss (a device scalar)."""
        diff = self.forward(x).float() - target.float()
        self.backward((diff * (2.0 / diff.numel())).to(torch.bfloat16))
        self.ctx.grad_norm(self.grads, self.max_norm, self.record)
        self.steps += 1
        self.ctx.adamw_step(self.params, self.grads, self.exp_avg, self.exp_avg_sq, self.steps, self.lr,
                            weight_decay=self.weight_decay, copies=self.copies, clip=self.record)
        return diff.square().mean()


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
        frags = [dict(global_=theta[p], momentum=momentum[p], learners=[m.copies[p] for m in group],
                      tokens=[inner_steps * tokens] * learners, quorum_mask=everyone, K=learners, n=3 * d * f)
                 for p in range(blocks)]
        ctx.merge_fragments_batched_push(frags, [everyone] * blocks, learners, dd.BF16, outer_lr, outer_mu, records=records)
        for p in range(blocks):
            for m in group:
                m.params[p].copy_(theta[p])                    # the copies were pushed
    return history


if __name__ == "__main__":
    for r, loss in enumerate(train(dd.Context(torch.cuda.current_device()))):
        print(f"round {r}: mean squared error {loss:.5f}")
