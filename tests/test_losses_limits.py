"""Losses over the logits, host side: the largest sizes that are accepted and the first that are not (no GPU needed: a call that passes
every check stops at the missing device)."""
import pytest

from paper_2510_03515_b200 import binding as rb
from test_losses_host import KINDS, _call, _desc, no_gpu

MOST = 2 ** 31 - 1024  # rows


@no_gpu
@pytest.mark.parametrize("kind", KINDS)
def test_the_most_rows(kind):
    for n, length in ((1, MOST), (1 << 10, MOST >> 10)):
        d = _desc(kind, n=n, length=length, v=1, ld=8)
        assert _call(kind, d, dlogits=None, logits=1 << 48) == rb.RAPID_ERR_CUDA


@pytest.mark.parametrize("kind", KINDS)
def test_rows_whose_numbers_would_pass_31_bits_within_a_block(kind):
    for n, length in ((1, MOST + 1), (1, 2 ** 31 - 1), ((2 ** 31 - 1) // 7, 7)):
        d = _desc(kind, n=n, length=length, v=1, ld=8)
        assert _call(kind, d, dlogits=None, logits=1 << 48) == rb.RAPID_ERR_UNSUPPORTED
        with pytest.raises(rb.RapidError):
            getattr(rb, f"rapid_{kind}_loss_workspace_bytes")(d)


@pytest.mark.parametrize("kind", ["clip", "preference"])
def test_more_pieces_of_rows_than_31_bits_number(kind):
    """Refused before anything is enqueued, not by the second of a call's launches."""
    d = _desc(kind, n=1 << 10, length=1 << 20, v=1 << 20)
    assert _call(kind, d, dlogits=None, logits=1 << 58) == rb.RAPID_ERR_UNSUPPORTED


@no_gpu
@pytest.mark.parametrize("kind", ["clip", "preference"])
def test_as_many_pieces_as_31_bits_number(kind):
    v = {"clip": 1 << 20, "preference": 4096 * 512}[kind]  # four pieces of a row's reading, 512 of its gradient
    n = {"clip": (1 << 29) - 1, "preference": (1 << 22) - 1}[kind]
    d = _desc(kind, n=n, length=1, v=v)
    assert _call(kind, d, dlogits=None, logits=1 << 58, ws_bytes=1 << 60) == rb.RAPID_ERR_CUDA
