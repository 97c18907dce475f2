"""Distillation with a bucket on rows of which chunks are loaded again, several for each block: the warp that takes the list's columns
out of the sum goes through every stage with the others, with lists short and long and beside rows that do not count."""
import pytest
import torch

import losses_util as lu
from paper_2510_03515_b200 import binding as rb

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("rows,v,dtype", [(450, 151936, F32), (310, 200001, F32), (450, 250007, BF)])
@pytest.mark.parametrize("k", [1, 8, 256])
def test_lists_beside_chunks_that_are_loaded_again(rows, v, dtype, k):
    z, _, _, g = lu.grid(rows, 1, v, dtype, seed=k + rows, boost=0.0)
    mask = (torch.rand(rows, generator=g) < 0.9).cuda()
    part = v // k
    index = (torch.arange(k) * part + torch.randint(0, part, (rows, k), generator=g)).to(torch.int32).cuda()
    logit = z.float().gather(1, index.long()) + torch.randn(rows, k, generator=g).cuda()
    top_lse = (torch.logsumexp(logit.double(), 1) + 0.3).float()
    stats = rb.alloc_stats()
    first = rb.distill_loss(z, index, logit, mask, top_lse, stats=stats)
    st = rb.read_loss_stats(stats)
    for _ in range(4):
        again = rb.distill_loss(z, index, logit, mask, top_lse, stats=stats)
        assert rb.read_loss_stats(stats) == st
        assert torch.equal(again.dlogits, first.dlogits) and torch.equal(again.token_loss, first.token_loss)
    del again
    for a in range(0, rows, 64):  # rows in pieces: the reference takes several matrices in double
        p = slice(a, a + 64)
        want = lu.distill(z[p], index[p], logit[p], mask[p], top_lse[p], norm=int(mask.sum()))
        got = rb.distill_loss(z[p], index[p], logit[p], mask[p], top_lse[p], flags=rb.LOSS_NORM_GIVEN, norm_z=int(mask.sum()), stats=stats)
        lu.check(want, got, rb.read_loss_stats(stats), dtype)
        assert torch.equal(got.dlogits, first.dlogits[p]) and torch.equal(got.token_loss, first.token_loss[p])
    torch.cuda.empty_cache()
