"""What the decoder's operators do without a GPU: sizes of scratch, frequencies, refusals before anything runs."""
import ctypes
import math

import pytest
import torch


@pytest.fixture(scope="module")
def dd():
    from paper_2604_21428_b200 import build
    build.build()
    from paper_2604_21428_b200 import ddmerge
    return ddmerge


def test_null_contexts_are_rejected(dd):
    a, l = dd.CAttention(tokens=4, heads=1, kv_heads=1, dim=64, scale=1.0), dd.CVocabLoss(tokens=1, d=8, vocab=8)
    n = None
    assert dd.lib.dd_rotary_apply(n, n, n, n, n, n, n, n, n) == dd.ERR_INVALID_ARG
    assert dd.lib.dd_attention_forward(n, ctypes.byref(a), n, n, n, n, n, n, n, n) == dd.ERR_INVALID_ARG
    assert dd.lib.dd_attention_backward(n, ctypes.byref(a), n, n, n, n, n, n, n, n, n, n, n, n) == dd.ERR_INVALID_ARG
    assert dd.lib.dd_vocab_loss_forward(n, ctypes.byref(l), n, n, n, n, n, n) == dd.ERR_INVALID_ARG
    assert dd.lib.dd_vocab_loss_forward(n, n, n, n, n, n, n, n) == dd.ERR_INVALID_ARG
    assert dd.lib.dd_vocab_loss_backward(n, ctypes.byref(l), n, n, n, n, n, 0, 0, n, n, n) == dd.ERR_INVALID_ARG


def test_attention_scratch(dd):
    """A plan item of 16 bytes for each tile there may be, and a float for each row of each head backward."""
    assert dd.attention_scratch_bytes(1000, 8, 2, 64) == 0
    assert dd.attention_scratch_bytes(1000, 8, 2, 64, 5) == 16 + 16 * (1000 // 256 + 5)
    assert dd.attention_scratch_bytes(1000, 8, 2, 64, 5, backward=True) == 4 * 8000 + 16 + 16 * (1000 // 128 + 5)
    assert dd.attention_scratch_bytes(1, 1, 1, 64, backward=True) == 16
    for bad in ((10, 3, 2, 64), (10, 2, 2, 12), (10, 2, 2, 136), (10, 0, 1, 64), (2 ** 31, 1, 1, 64)):
        assert dd.attention_scratch_bytes(*bad, 3) == 0


def test_frequencies(dd):
    f, m = dd.rotary_frequencies(64, device="cpu")
    assert m == 1.0 and f.dtype == torch.float64
    assert torch.allclose(f, 10000.0 ** (-torch.arange(32, dtype=torch.float64) / 32), rtol=1e-15, atol=0)
    g, m = dd.rotary_frequencies(64, factor=4.0, device="cpu")
    assert m == 1.0 and torch.equal(g, f / 4)
    g, m = dd.rotary_frequencies(64, factor=4.0, trained=4096, device="cpu")
    turns = 4096 * f / (2 * math.pi)
    assert m == 0.1 * math.log(4.0) + 1.0
    assert torch.equal(g[turns >= 32], f[turns >= 32]) and torch.equal(g[turns <= 1], f[turns <= 1] / 4)
    between = (turns > 1) & (turns < 32)
    assert bool((g[between] < f[between]).all()) and bool((g[between] > f[between] / 4).all())
    for bad in (dict(rotary_dim=7), dict(rotary_dim=0), dict(rotary_dim=8, base=0.0), dict(rotary_dim=8, factor=0.5),
                dict(rotary_dim=8, low=2.0, high=2.0)):
        with pytest.raises(ValueError):
            dd.rotary_frequencies(**{"device": "cpu", **bad})


def test_packed_documents():
    from paper_2604_21428_b200.learner import packed_documents
    gen = torch.Generator().manual_seed(0)
    for _ in range(20):
        ids, targets, positions, offsets = packed_documents(gen, 50, 4, 30, device="cpu")
        ends = offsets.tolist()
        assert ends[0] == 0 and ends == sorted(ends) and ends[-1] <= 50 and len(ends) == 5
        for a, b in zip(ends, ends[1:]):
            assert positions[a:b].tolist() == list(range(b - a))
            if b > a:
                assert torch.equal(targets[a: b - 1], ids[a + 1: b]) and int(targets[b - 1]) < 0
        assert bool((targets[ends[-1]:] < 0).all()) and bool((positions[ends[-1]:] < 0).all())


def test_refusals_name_no_buffer_of_another_call(dd):
    """Codes that merges and the learner's operators share say what holds for both."""
    for rc in (dd.ERR_INVALID_ARG, dd.ERR_ALIGNMENT, dd.ERR_ALIAS, dd.ERR_TOO_LARGE):
        text = dd.lib.dd_status_string(rc).decode()
        assert not any(word in text for word in ("fragment", "momentum", "learner", "16-byte")), text
