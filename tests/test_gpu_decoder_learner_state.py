"""What a decoder's learner keeps, skips and reports."""
import pytest
import torch

from decoder_util import U, within

pytestmark = pytest.mark.gpu
SIZES = dict(vocab=200, d=64, f=136, layers=1, heads=4, kv_heads=2, dim=16, tokens=200, sequences=3)


@pytest.fixture(scope="module")
def mods():
    from paper_2604_21428_b200 import ddmerge, learner
    ctx = ddmerge.Context(0)
    yield ddmerge, learner, ctx
    ctx.close()


def start(mods, seed=0, **kw):
    _, lm, ctx = mods
    m = lm.DecoderLearner(ctx, **SIZES, **kw)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    for p, fragment in enumerate(m.initial(gen)):
        m.receive(p, fragment)
    return m, gen


def test_gradients_of_the_projections_are_float32(mods):
    """Sums of products of bf16 operands in float32, not rounded on the way to the float32 buffers."""
    _, lm, _ = mods
    m, gen = start(mods, lr=0.0)
    m.step(*lm.packed_documents(gen, SIZES["tokens"], SIZES["sequences"], SIZES["vocab"]))
    dw_qkv, dw_o = m.weight_grads[0][:2]
    for g in (dw_qkv, dw_o):
        assert not torch.equal(g, g.to(torch.bfloat16).float())
    a, b = m.dqkv.flatten(1).double(), m.kept[0]["h1"].double()
    within(dw_qkv, a.t() @ b, (SIZES["tokens"] + 16) * 2 * U * (a.abs().t() @ b.abs()) + 1e-38, "dw_qkv")


def test_a_batch_without_targets(mods):
    """Documents of one token have no target: the loss is 0 and nothing moves."""
    m, _ = start(mods, lr=1e-2)
    before = [p.clone() for p in m.params]
    T = SIZES["tokens"]
    ids, targets = torch.zeros(T, dtype=torch.int64, device="cuda"), torch.full((T,), -100, dtype=torch.int64, device="cuda")
    positions = torch.full((T,), -1, dtype=torch.int64, device="cuda")
    positions[:3] = 0
    assert float(m.step(ids, targets, positions, torch.arange(4, dtype=torch.int32, device="cuda"))) == 0.0
    assert not any(bool(g.any()) for g in m.grads)
    assert all(torch.equal(a, b) for a, b in zip(before, m.params))


def test_bad_offsets_change_nothing_and_are_reported(mods):
    """Attention writes nothing for offsets that decrease: the step leaves parameters, moments and copies alone, and the
    learner says so before a merge; after that it goes on."""
    dd, lm, _ = mods
    m, gen = start(mods, lr=1e-2)
    batch = lm.packed_documents(gen, SIZES["tokens"], SIZES["sequences"], SIZES["vocab"])
    m.step(*batch)
    m.check()
    held = [*m.params, *m.exp_avg, *m.exp_avg_sq, *m.copies]
    before = [t.clone() for t in held]
    ids, targets, positions, _ = batch
    bad = torch.tensor([0, 90, 50, 200], dtype=torch.int32, device="cuda")
    m.step(ids, targets, positions, bad)
    m.step(*batch)                                        # until it is looked at
    assert all(torch.equal(a, b) for a, b in zip(before, held))
    with pytest.raises(RuntimeError, match=str(dd.STATUS_BAD_OFFSETS)):
        m.check()
    m.step(*batch)
    m.check()
    assert not any(torch.equal(a, b) for a, b in zip(before, held))


def test_learners_of_blocks_report_too(mods):
    _, lm, ctx = mods
    m = lm.Learner(ctx, 64, 128, 2, 32, lr=1e-2)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for p in range(2):
        m.receive(p, torch.randn(3 * 64 * 128, generator=gen, device="cuda") * 0.1)
    x = torch.randn(32, 64, generator=gen, device="cuda").to(torch.bfloat16)
    before = [t.clone() for t in m.params]
    m.status.fill_(mods[0].STATUS_WAIT_LIMIT)             # as an expired wait leaves it
    m.step(x, x)
    assert all(torch.equal(a, b) for a, b in zip(before, m.params))
    with pytest.raises(RuntimeError):
        m.check()
    m.step(x, x)
    m.check()
    assert not any(torch.equal(a, b) for a, b in zip(before, m.params))


def test_merges_count_trained_tokens_and_learners_hold_the_result(mods, monkeypatch):
    """The merge weighs each learner by the tokens with a target that it trained on since the last one; after the push every
    learner holds the global fragments."""
    _, lm, ctx = mods
    learners, counts, merges = [], [], []
    documents = lm.packed_documents

    class Kept(lm.DecoderLearner):
        def __init__(self, *a, **kw):
            super().__init__(*a, **kw)
            learners.append(self)

    class Seen:
        def __getattr__(self, name):
            return getattr(ctx, name)

        def merge_fragments_batched_push(self, frags, *a, **kw):
            merges.append(frags)
            return ctx.merge_fragments_batched_push(frags, *a, **kw)

    def counted(*a, **kw):
        batch = documents(*a, **kw)
        counts.append(int((batch[1] >= 0).sum()))
        return batch

    monkeypatch.setattr(lm, "DecoderLearner", Kept)
    monkeypatch.setattr(lm, "packed_documents", counted)
    rounds, steps = 2, 3
    lm.train_decoder(Seen(), learners=2, rounds=rounds, inner_steps=steps, **SIZES)
    assert len(merges) == rounds and len(counts) == rounds * steps * 2
    for r, frags in enumerate(merges):
        mine = counts[r * steps * 2: (r + 1) * steps * 2]
        assert all(f["tokens"] == [sum(mine[0::2]), sum(mine[1::2])] for f in frags)
    assert sum(counts[0::2]) != sum(counts[1::2])         # or the test would say little
    for p, f in enumerate(merges[-1]):
        for m in learners:
            assert torch.equal(m.params[p], f["global_"]) and torch.equal(m.copies[p], f["global_"].to(torch.bfloat16))


def test_room_for_the_loss_of_a_wide_vocabulary(mods):
    """Many columns, small d and many tokens: forward, the loss needs more scratch than backward."""
    _, lm, ctx = mods
    sizes = dict(vocab=80000, d=16, f=16, layers=1, heads=1, kv_heads=1, dim=16, tokens=32768, sequences=40)
    assert ctx.vocab_loss_scratch_bytes(32768, 16, 80000) > ctx.vocab_loss_scratch_bytes(32768, 16, 80000, backward=True)
    m = lm.DecoderLearner(ctx, **sizes, lr=1e-3)
    gen = torch.Generator(device="cuda").manual_seed(3)
    for p, fragment in enumerate(m.initial(gen)):
        m.receive(p, fragment)
    assert 0.0 < float(m.step(*lm.packed_documents(gen, 32768, 40, 80000))) < 20.0        # log(80000) = 11.3
    m.check()


def test_rows_behind_the_documents_forget_earlier_batches(mods):
    """Attention leaves rows behind the last document as they are: what an earlier batch left there, NaN included, reaches
    neither loss nor gradients."""
    _, lm, _ = mods
    T = SIZES["tokens"]
    results = []
    for left in (0.0, float("nan")):
        m, gen = start(mods, lr=0.0)
        ids, targets, positions, offsets = lm.packed_documents(gen, T, SIZES["sequences"], SIZES["vocab"])
        offsets = offsets.clamp(max=150)                   # 50 rows of room
        behind = torch.arange(T, device="cuda") >= 150
        targets, positions = targets.masked_fill(behind, -100), positions.masked_fill(behind, -1)
        for keep in m.kept:
            keep["o"].fill_(left)
        m.dqkv.fill_(left)
        loss = m.step(ids, targets, positions, offsets)
        m.check()
        results.append([loss.clone(), *(g.clone() for g in m.grads)])
    for a, b in zip(*results):
        assert bool(b.isfinite().all()) and torch.equal(a, b)
