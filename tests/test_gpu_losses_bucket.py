"""Distillation with a bucket where the student has far less mass outside the list than the teacher: there the gradient is
w / tau (q_v - p_0 q_v / q_0), at most p_0 in sum, although p_0 / q_0 is beyond any type."""
import math

import pytest
import torch

import losses_util as lu
from paper_2510_03515_b200 import binding as rb

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
# two rows by a warp, groups of 8, 4 and 2 warps, a block with two on an SM, a block with one, chunks that are loaded again
SHAPES = [(1300, 1000), (6, 1000), (20, 4097), (700, 20001), (1300, 9000), (5, 70001), (3, 151936), (2, 200001)]


def _gradient(z, index, t, top_lse, tau):
    """The definition, with the softmax over the columns outside the list in its own numbers, and its bound: a probability's error
    (P) on either term and the result's rounding."""
    x = z.double() / tau
    lse = torch.logsumexp(x, 1, keepdim=True)
    rest = x.scatter(1, index.long(), -math.inf)
    s = torch.exp(rest - torch.logsumexp(rest, 1, keepdim=True))
    p = torch.exp(t.double() / tau - top_lse.double()[:, None])
    p0 = 1 - p.sum(1, keepdim=True)
    q = torch.exp(x - lse)
    w = 1.0 / (z.shape[0] * tau)
    want = w * (q - p0 * s)
    want.scatter_(1, index.long(), w * (q.gather(1, index.long()) - p))
    room = (lu.P + 4 * lu.LSE) * w * (q + p0 * s)
    loss = (p * (t.double() / tau - top_lse.double()[:, None] - (x - lse).gather(1, index.long()))).sum(1)
    loss += (p0 * (p0.log() - (torch.logsumexp(rest, 1, keepdim=True) - lse))).squeeze(1)
    return want, room + (lu.HALF[z.dtype] + lu.P) * want.abs() + 2.0 ** -126, loss, w * tau * loss.sum()


@pytest.mark.parametrize("rows,v", SHAPES)
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("gap,tau", [(0.0, 1.0), (30.0, 1.0), (85.0, 1.0), (95.0, 1.0), (10.0, 0.1), (1.0, 0.01), (2.0, 0.001), (1e4, 1.0), (400.0, 1.0), (2e4, 300.0)])
def test_a_student_that_is_sure_of_the_list(rows, v, dtype, gap, tau):
    g = torch.Generator().manual_seed(v + rows)
    z = torch.zeros(rows, -(-v // 8) * 8)
    z[:, :v] = 2.0 * min(tau, 1.0) * torch.randn(rows, v, generator=g)
    index = torch.stack([torch.randperm(v, generator=g)[:8] for _ in range(rows)])
    z.scatter_(1, index, z[:, :v].amax(1, keepdim=True) + gap + tau * torch.rand(rows, 8, generator=g))
    z, index = z.to(dtype).cuda()[:, :v], index.to(torch.int32).cuda()
    t = tau * torch.randn(rows, 8, generator=g).cuda()
    top_lse = (torch.logsumexp(t.double() / tau, 1) + 0.2).float()  # p_0 = 0.18
    stats = rb.alloc_stats()
    got = rb.distill_loss(z, index, t, None, top_lse, tau, stats=stats)
    for a in range(0, rows, 100):
        p = slice(a, a + 100)
        want, room, loss, _ = _gradient(z[p], index[p], t[p], top_lse[p], tau)
        part = z[p].shape[0] / rows
        d = got.dlogits[p].double()
        assert bool(((d - part * want).abs() <= part * room + 2.0 ** -126).all()), f"{float(((d - part * want).abs() / (part * room)).max()):.3g} of its bound"
        assert bool(((got.token_loss[p].double() - loss).abs() <= 2 * lu.LSE + 2.0 ** -24 * loss.abs()).all())
    st = rb.read_loss_stats(stats)
    assert st["status"] == 0 and st["n_bad"] == 0 and math.isfinite(st["loss"])


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("v", [1000, 70001, 200001])
def test_columns_masked_by_a_large_negative_number(dtype, v):
    """An additive mask of -1e4 on what the student may not say, over a part of the columns and over all outside the list."""
    g = torch.Generator().manual_seed(v)
    z = torch.zeros(6, -(-v // 8) * 8)
    z[:, :v] = 3 * torch.randn(6, v, generator=g)
    z[:3] -= 1e4
    z[3:, v // 2:] -= 1e4
    index = torch.stack([torch.randperm(v, generator=g)[:8] for _ in range(6)])
    z.scatter_(1, index, 3 * torch.randn(6, 8, generator=g))
    z, index = z.to(dtype).cuda()[:, :v], index.to(torch.int32).cuda()
    t = torch.randn(6, 8, generator=g).cuda()
    top_lse = (torch.logsumexp(t.double(), 1) + 0.2).float()
    got = rb.distill_loss(z, index, t, None, top_lse)
    want, room, loss, total = _gradient(z, index, t, top_lse, 1.0)
    assert bool(((got.dlogits.double() - want).abs() <= room).all())
    assert bool(((got.token_loss.double() - loss).abs() <= 2 * lu.LSE + 2.0 ** -24 * loss.abs()).all())
    assert abs(float(got.loss) - float(total)) <= 2 * lu.LSE + 2.0 ** -23 * abs(float(total))
    # all of the gradient outside the list goes to what the student says there least unlikely
    outside = got.dlogits.double().scatter(1, index.long(), 0.0).sum(1)
    p0 = 1 - torch.exp(t.double() - top_lse.double()[:, None]).sum(1)
    assert bool(((outside[:3] * 6 + p0[:3]).abs() <= 0.02).all())
