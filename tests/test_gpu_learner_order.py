"""Calls that follow one another on a stream with nothing in between: each sees all that the one before
wrote, although their launches overlap (programmatic launches)."""
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


class Steps:
    """AdamW, forward, AdamW, backward on one set of weights: each block call multiplies by the copies
    that the AdamW step right before it wrote."""

    def __init__(self, ctx, tokens, d, f, seed=3):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def randn(*shape, std=1.0):
            return torch.randn(*shape, generator=gen, device="cuda") * std

        self.ctx = ctx
        shapes = [(f, d), (f, d), (d, f)]
        self.params = [randn(*s, std=0.05) for s in shapes]
        self.grads = [randn(*s, std=1e-2) for s in shapes]
        self.m, self.v = [torch.zeros_like(p) for p in self.params], [torch.zeros_like(p) for p in self.params]
        self.w = [p.to(B) for p in self.params]
        self.x, self.dy = randn(tokens, d).to(B), randn(tokens, d).to(B)
        self.y, self.dx = torch.zeros_like(self.x), torch.zeros_like(self.x)
        self.gate, self.up = (torch.zeros(tokens, f, dtype=B, device="cuda") for _ in range(2))
        self.dws = [torch.zeros_like(w) for w in self.w]
        self.scratch = torch.zeros(3 * tokens * f, dtype=B, device="cuda")

    def run(self, between=lambda: None):
        def update():
            self.ctx.adamw_step(self.params, self.grads, self.m, self.v, 10, 3e-2, copies=self.w)
            between()

        update()
        self.ctx.gated_ffn_forward(self.x, *self.w, self.y, gate=self.gate, up=self.up, hidden=self.scratch)
        between()
        update()
        self.ctx.gated_ffn_backward(self.x, *self.w, self.gate, self.up, self.dy, self.dx, *self.dws,
                                    scratch=self.scratch)
        between()

    def results(self):
        return [t.clone() for t in (self.y, self.gate, self.up, self.dx, *self.dws, *self.w)]


@pytest.mark.parametrize("graph", [False, True])
@pytest.mark.parametrize("size", [(1, 256, 512), (1, 2048, 512), (40, 256, 512), (300, 128, 384), (320, 1024, 2048),
                                  (500, 256, 512)], ids=str)
def test_block_reads_the_weights_of_the_step_before_it(dd, ctx, size, graph):
    """Lists short enough to leave most of the GPU idle, so that every launch that may start early does;
    the same bits as with a synchronise after every call."""
    rounds = 40
    a, b = Steps(ctx, *size), Steps(ctx, *size)
    want = []
    for _ in range(rounds):
        b.run(torch.cuda.synchronize)
        want.append(b.results())
    got = []
    if graph:
        ctx.gated_ffn_forward(a.x, *a.w, a.y)                # workspaces, before the capture
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            a.run()
        for _ in range(rounds):
            captured.replay()
            got.append(a.results())
    else:
        for _ in range(rounds):
            a.run()
            got.append(a.results())
    torch.cuda.synchronize()
    for i, (g, w) in enumerate(zip(got, want)):
        for k, (p, q) in enumerate(zip(g, w)):
            assert torch.equal(p, q), (i, k)
    if graph:
        del captured


@pytest.mark.parametrize("kind", [B, torch.float32])
@pytest.mark.parametrize("size", [(1, 264, 520), (5, 72, 136), (130, 257, 131), (320, 1000, 312), (500, 264, 520)], ids=str)
def test_gradients_accumulate_over_calls(dd, ctx, size, kind):
    """Micro-batches one after the other into the same gradients, rows that end inside lines: the same bits as
    with a synchronise after every call."""
    tokens, d, f = size
    rows = lambda n: (n + 7) // 8 * 8
    gen = torch.Generator(device="cuda").manual_seed(9)

    def mat(r, c, dtype=B, std=1.0):
        return (torch.randn(r, rows(c), generator=gen, device="cuda") * std).to(dtype)[:, :c]

    w = [mat(f, d), mat(f, d), mat(d, f)]
    x, dy, gate, up, dx = mat(tokens, d), mat(tokens, d), mat(tokens, f), mat(tokens, f), mat(tokens, d)
    start = [mat(f, d, kind), mat(f, d, kind), mat(d, f, kind)]
    scratch = torch.zeros(3 * tokens * rows(f), dtype=B, device="cuda")
    results = []
    for between in (lambda: None, torch.cuda.synchronize):
        dws = [mat(f, d, kind), mat(f, d, kind), mat(d, f, kind)]
        for a, b in zip(dws, start):
            a.copy_(b)
        for _ in range(50):
            ctx.gated_ffn_backward(x, *w, gate, up, dy, dx, *dws, accumulate=True, scratch=scratch)
            between()
        results.append([t.clone() for t in (dx, *dws)])
    for a, b in zip(*results):
        assert torch.equal(a, b)
