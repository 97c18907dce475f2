"""Arguments of the policy-network wrappers, on the CPU: what reaches the C call is what the caller passes now."""
import contextlib

import pytest
import torch

from paper_2510_03515_b200 import binding as rb

BF = torch.bfloat16


@pytest.fixture
def calls(monkeypatch):
    """Descriptors that the wrappers hand to the C calls, which are not made."""
    seen = []
    monkeypatch.setattr(rb, "_one_device", lambda *tensors: 0)
    monkeypatch.setattr(rb, "_on", lambda index: contextlib.nullcontext())
    for name in ("rapid_embedding_fwd", "rapid_embedding_bwd", "rapid_qk_norm_rope_fwd", "rapid_qk_norm_rope_bwd", "rapid_attention_fwd",
                 "rapid_attention_bwd"):
        monkeypatch.setattr(rb, name, lambda desc, *rest: seen.append(desc))
    return seen


def _embedding(scale):
    rb.embedding(torch.zeros(5, 8), torch.zeros(4, dtype=torch.int32), scale=scale)


def _embedding_grad(scale):
    rb.embedding_grad(torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32), None, 5, scale)


def _heads(h=2, rows=6):
    return torch.zeros(rows, h, 16, dtype=BF)


def _qk(eps):
    w = torch.zeros(16)
    rb.qk_norm_rope(_heads(), _heads(), w, w, w[:8], 2, 3, eps=eps)


def _qk_grad(eps):
    w = torch.zeros(16)
    rb.qk_norm_rope_grad(_heads(), _heads(), w, w, w[:8], _heads(), _heads(), 2, 3, eps=eps)


def _attention(scale):
    rb.attention(_heads(), _heads(), _heads(), 2, 3, scale=scale)


def _attention_grad(scale):
    x = _heads()
    rb.attention_grad(x, x, x, x, torch.zeros(12), x, 2, 3, scale=scale)


@pytest.mark.parametrize("call,field", [(_embedding, "scale"), (_embedding_grad, "scale"), (_qk, "eps"), (_qk_grad, "eps"), (_attention, "scale"),
                                        (_attention_grad, "scale")])
def test_a_changed_number_reaches_the_call(calls, call, field):
    """A number held in a tensor that is changed in place between two calls."""
    x = torch.tensor(0.5)
    call(x)
    x.mul_(4)
    call(x)
    assert [getattr(d, field) for d in calls] == [0.5, 2.0]


def test_a_changed_window_and_length_reach_the_call(calls):
    window, length, n = torch.tensor(2), torch.tensor(3), torch.tensor(2)
    x = _heads()
    for _ in range(2):
        rb.attention(x, x, x, n, length, window=window)
        rb.qk_norm_rope(x, x, torch.zeros(16), torch.zeros(16), torch.zeros(8), n, length)
        window += 1
        n, length = n.mul_(3).floor_divide_(2), length.mul_(2).floor_divide_(3)  # 2 x 3, then 3 x 2
    assert [(d.n_seq, d.seq_len) for d in calls] == [(2, 3), (2, 3), (3, 2), (3, 2)]
    assert [calls[0].window, calls[2].window] == [2, 3]


def test_a_changed_vocabulary_reaches_the_call(calls):
    vocab = torch.tensor(5)
    for want in (5, 9):
        vocab.fill_(want)
        assert rb.embedding_grad(torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32), None, vocab).shape == (want, 8)
        assert calls[-1].vocab == want


def test_numbers_beyond_32_bits_are_refused(calls):
    """A field of the descriptor would keep their low bits: a window of 2^32 + 1 would become 1."""
    x = _heads()
    for window in (2 ** 32, 2 ** 32 + 1, 2 ** 31):
        with pytest.raises(ValueError, match="window"):
            rb.attention(x, x, x, 2, 3, window=window)
        with pytest.raises(ValueError, match="window"):
            rb.attention_grad(x, x, x, x, torch.zeros(12), x, 2, 3, window=window)
    rb.attention(x, x, x, 2, 3, window=2 ** 31 - 1)
    assert calls[-1].window == 2 ** 31 - 1
    big = 2 ** 32 + 2
    for make in (lambda: rb.make_embed_desc(4, big, 8, BF), lambda: rb.make_embed_desc(4, 5, big, BF), lambda: rb.make_qk_desc(big, 3, 2, 1, 16, BF),
                 lambda: rb.make_qk_desc(2, 3, 2, 1, 16, BF, big), lambda: rb.make_attn_desc(2, big, 2, 1, 16), lambda: rb.make_attn_desc(2, 3, 2, 1, big),
                 lambda: rb.make_attn_desc(2, 3, 2, 1, 16, flags=2 ** 32), lambda: rb.make_qk_desc(2, 3, 2, 1, 16, BF, flags=-1)):
        with pytest.raises(ValueError, match="32 bits"):
            make()


@pytest.mark.parametrize("stats", [torch.zeros(rb.STATS_BYTES - 1, dtype=torch.uint8), torch.zeros(0, dtype=torch.uint8),
                                   torch.zeros(2 * rb.STATS_BYTES, dtype=torch.uint8)[::2], torch.zeros(rb.STATS_BYTES + 8, dtype=torch.uint8)[4:],
                                   torch.zeros(rb.STATS_BYTES // 8 - 1, dtype=torch.int64)])
def test_stats_that_are_no_stats_are_refused(calls, stats):
    """Too short, with gaps, or off an 8-byte boundary: the kernels write STATS_BYTES bytes with 8-byte accesses."""
    x = _heads()
    for call in (lambda s: rb.embedding(torch.zeros(5, 8), torch.zeros(4, dtype=torch.int32), stats=s), lambda s: rb.attention(x, x, x, 2, 3, stats=s),
                 lambda s: rb.attention_grad(x, x, x, x, torch.zeros(12), x, 2, 3, stats=s)):
        with pytest.raises(ValueError, match="stats"):
            call(stats)
        call(rb.alloc_stats("cpu"))
    assert len(calls) == 3
