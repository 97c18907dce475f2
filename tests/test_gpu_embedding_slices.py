"""Embedding matrices that are column slices of one matrix: the same bits as on matrices of their own, the other columns untouched."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2510_03515_b200 import binding as rb  # noqa: E402

BF = torch.bfloat16


def _apart(x):
    """The same matrix in rows of its own, on 16-byte boundaries."""
    y = x.new_empty(x.shape[0], -(-x.shape[1] // 8) * 8)[:, :x.shape[1]]
    return y.copy_(x)


@pytest.mark.parametrize("T,V,D", [(60, 41, 24), (41, 60, 9), (700, 700, 520)])
def test_slices_of_one_matrix(T, V, D):
    g = torch.Generator().manual_seed(T)
    width = -(-D // 8) * 8 + 8
    wide = torch.randn(max(T, V), 3 * width, generator=g).to(BF).cuda()
    tokens = torch.randint(0, V, (T,), generator=g, dtype=torch.int32).cuda()
    row = 3 * width
    left, right = wide[:V, :D], wide[:T, width:width + D]

    before = wide.clone()
    want = rb.embedding(_apart(left), tokens, scale=2.0)
    rb.rapid_embedding_fwd(rb.make_embed_desc(T, V, D, BF, row, row, 2.0), tokens, None, left, right, None)
    assert torch.equal(right, want)
    before[:T, width:width + D] = want
    assert torch.equal(wide, before)

    desc = rb.make_embed_desc(T, V, D, BF, row, row, 0.5, rb.EMBED_DTABLE_BF16)
    ws = torch.empty(rb.rapid_embedding_bwd_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    want = rb.embedding_grad(_apart(right), tokens, None, V, 0.5, BF)
    rb.rapid_embedding_bwd(desc, tokens, None, right, left, ws)
    assert torch.equal(left, want)
    before[:V, :D] = want
    assert torch.equal(wide, before)
