"""Distillation with a bucket where the student has nothing outside the list: a list of the whole vocabulary, or a vocabulary whose other
columns are masked.  p_0 is then the rounding of top_lse, of either sign, and counts as 0."""
import math

import pytest
import torch

import losses_util as lu
from paper_2510_03515_b200 import binding as rb
from test_gpu_losses import _lists

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _rounded(t, tau, how):
    """The list's log-sum-exp as a float: the nearest, the next one above it, below it, or summed in float."""
    x = torch.logsumexp(t.double() / tau, 1)
    if how == "float":
        return torch.logsumexp(t / tau, 1)
    y = x.float()
    if how == "up":
        return torch.where(y.double() < x, torch.nextafter(y, torch.full_like(y, math.inf)), y)
    if how == "down":
        return torch.where(y.double() > x, torch.nextafter(y, torch.full_like(y, -math.inf)), y)
    return y


def _check(z, index, t, top_lse, tau, dtype):
    """Against the list alone, whose teacher differs by the rounding: of the log-sum-exp, 4 steps of 2^-23."""
    stats = rb.alloc_stats()
    want = lu.distill(z, index, t, None, None, tau)
    slack = 4 * 2.0 ** -23 * float(top_lse.abs().max().clamp_min(1.0))  # of every p_j, so of the row's terms and gradient too
    spread = 1 + float(want["token"].abs().max()) + 2 * float((t / tau).abs().max() + (z.float().nan_to_num(neginf=0.0) / tau).abs().max())
    want["token_tol"] += slack * spread
    want["loss_tol"] += slack * spread
    want["grad_tol"] = want["grad_tol"] + slack / (tau * z.shape[0]) * torch.ones_like(want["grad"]).masked_fill(want["grad"] == 0, 0.0)
    for grad in (True, False):
        got = rb.distill_loss(z, index, t, None, top_lse, tau, want_grad=grad, stats=stats)
        lu.check(want, got, rb.read_loss_stats(stats), dtype, grad)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("how", ["nearest", "up", "down", "float"])
@pytest.mark.parametrize("v,tau,shift", [(200, 1.0, 0.0), (256, 0.5, 40.0), (7, 1.0, 0.0), (256, 3.0, -900.0)])
def test_the_whole_vocabulary_listed(dtype, how, v, tau, shift):
    z, _, _, g = lu.grid(1, 64, v, dtype, seed=v)
    index, t = _lists(z, v, g)
    t += shift
    _check(z, index, t, _rounded(t, tau, how), tau, dtype)
    _check(z[:3], index[:3], t[:3], _rounded(t[:3], tau, how), tau, dtype)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("low", ["-inf", "lowest"])
@pytest.mark.parametrize("how", ["nearest", "up", "down", "float"])
@pytest.mark.parametrize("rows,v", [(1300, 500), (5, 500), (700, 20001), (4, 61000), (3, 151936), (2, 200001)])
def test_the_rest_masked(dtype, low, how, rows, v):
    z, _, _, g = lu.grid(1, rows, v, dtype, seed=v + rows)
    index = torch.stack([torch.randperm(v, generator=g)[:9] for _ in range(rows)]).to(torch.int32).cuda()
    t = torch.randn(rows, 9, generator=g).cuda() * 2 + 5
    kept = z.gather(1, index.long())
    only = z.fill_(-math.inf if low == "-inf" else torch.finfo(dtype).min).scatter_(1, index.long(), kept)
    _check(only, index, t, _rounded(t, 1.0, how), 1.0, dtype)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_a_teacher_with_mass_where_the_student_has_none(dtype):
    """That is an infinite loss, of the rows that it is so in."""
    z, _, _, g = lu.grid(1, 40, 900, dtype, seed=3)
    index, t = _lists(z, 6, g)
    kept = z.gather(1, index.long())
    only = z.fill_(-math.inf).scatter_(1, index.long(), kept)
    lse = torch.logsumexp(t.double(), 1).float()
    lse[5] += 1e-4
    lse[17] += 3.0
    got = rb.distill_loss(only, index, t, None, lse)
    bad = torch.zeros(40, dtype=torch.bool, device="cuda")
    bad[5], bad[17] = True, True
    assert torch.equal(got.token_loss.isinf(), bad) and math.isinf(float(got.loss)) and not bool(got.token_loss.isnan().any())
    assert bool(got.dlogits.isfinite().all())
    # a list with places without an entry is not all of the vocabulary
    z, _, _, g = lu.grid(1, 4, 20, dtype, seed=4)
    index, t = _lists(z, 20, g)
    index[:, 3] = -1
    lse = torch.logsumexp(t.masked_fill(index < 0, -math.inf).double(), 1).float() + 0.3
    want = lu.distill(z, index, t, None, lse)
    stats = rb.alloc_stats()
    lu.check(want, rb.distill_loss(z, index, t, None, lse, stats=stats), rb.read_loss_stats(stats), dtype)
