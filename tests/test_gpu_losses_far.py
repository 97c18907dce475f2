"""Logits that are large beside the temperature: probabilities and gradients depend on differences of logits only, and are as exact as
those of small ones."""
import math

import pytest
import torch

import losses_util as lu
from paper_2510_03515_b200 import binding as rb

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
# two rows by a warp, groups of 8, 4 and 2 warps, a block with two on an SM, a block with one, chunks that are loaded again
SHAPES = [(1300, 500), (20, 4097), (700, 20001), (1300, 9000), (5, 70001), (3, 151936), (2, 200001)]


def _near(rows, v, dtype, offset, step, seed):
    """offset + step * (0, -1, -2, -3), with the highest ones seldom; `step` is one that the type has at `offset`."""
    g = torch.Generator().manual_seed(seed)
    u = torch.rand(rows, v, generator=g)
    z = offset + step * ((u < 0.01).float() - (u > 0.3).float() - (u > 0.6).float())
    z[:, 0] = offset + step
    targets = torch.randint(0, v, (rows,), generator=g, dtype=torch.int32)
    pad = torch.full((rows, -(-v // 8) * 8), math.nan)
    pad[:, :v] = z
    assert torch.equal(pad[:, :v].to(dtype).float(), z)
    return pad.to(dtype).cuda()[:, :v], targets.cuda(), g


@pytest.mark.parametrize("rows,v", SHAPES)
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("offset,step,tau", [(11.0, 0.0625, 0.1), (100.0, 0.5, 0.001), (-100.0, 0.5, 0.01), (19968.0, 128.0, 100.0), (-3008.0, 16.0, 2.0)])
def test_distill(rows, v, dtype, offset, step, tau):
    z, _, g = _near(rows, v, dtype, offset, step, seed=v + rows)
    index = torch.stack([torch.randperm(min(v, 400), generator=g)[:4] for _ in range(rows)]).to(torch.int32).cuda()
    logit = tau * torch.randn(rows, 4, generator=g).cuda()
    lse = (torch.logsumexp(logit.double() / tau, 1) + 0.2).float()
    stats = rb.alloc_stats()
    for top_lse in (None, lse):
        want = lu.distill(z, index, logit, None, top_lse, tau)
        got = rb.distill_loss(z, index, logit, None, top_lse, tau, stats=stats)
        lu.check(want, got, rb.read_loss_stats(stats), dtype)


@pytest.mark.parametrize("rows,v", SHAPES)
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("offset", [200.0, -19968.0])
def test_clip_and_preference(rows, v, dtype, offset):
    """Logits of steps of one (200) and 128 (-19968): of the second, one of some hundred equal ones has all but nothing."""
    step = 1.0 if offset == 200.0 else 128.0
    z, targets, g = _near(rows, v, dtype, offset, step, seed=v + rows + 1)
    targets[: rows // 2] = 0
    lp, _, _ = lu._token_logp(z, targets, torch.ones(rows, dtype=torch.bool, device="cuda"))
    old = (lp + 0.05).float()
    adv = torch.randn(rows, generator=g).cuda()
    stats = rb.alloc_stats()
    want = lu.clip(z, targets, None, old, adv, rows)
    lu.check(want, rb.clip_loss(z, targets, None, old, adv, rows, 1, stats=stats), rb.read_loss_stats(stats), dtype)
    pairs = torch.arange(rows // 2 * 2, dtype=torch.int32, device="cuda").view(-1, 2)
    want = lu.preference(z, targets, None, pairs, rows, lp.float(), beta=0.3)
    lu.check(want, rb.preference_loss(z, targets, None, pairs, rows, 1, lp.float(), beta=0.3, stats=stats), rb.read_loss_stats(stats), dtype)


@pytest.mark.parametrize("rows,v", SHAPES)
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("offset,tau", [(2.0 ** 27, 1.0), (-(2.0 ** 27), 1.0), (2.0 ** 17, 0.001), (-130048.0, 0.001)])
def test_at_the_end_of_the_range(rows, v, dtype, offset, tau):
    """Logits over the temperature of 2^27: rows of equal largest ones, the others a step of the type below, which is far."""
    step = 2.0 ** (math.floor(math.log2(abs(offset))) - 6)
    z, _, g = _near(rows, v, dtype, offset - step if offset > 0 else offset + 2 * step, step, seed=v)
    index = torch.stack([torch.randperm(min(v, 400), generator=g)[:4] for _ in range(rows)]).to(torch.int32).cuda()
    logit = tau * torch.randn(rows, 4, generator=g).cuda()
    lse = (torch.logsumexp(logit.double() / tau, 1) + 0.2).float()
    for top_lse in (None, lse):
        want = lu.distill(z, index, logit, None, top_lse, tau)
        got = rb.distill_loss(z, index, logit, None, top_lse, tau)
        room = want["grad_tol"] + (lu.HALF[dtype] + lu.P) * want["grad"].abs() + 2.0 ** -126
        ok = want["grad"].isfinite().all(1)  # (where q_0 is 0 in double too, the utility's 0 x infinity)
        assert bool(((got.dlogits.double() - want["grad"]).abs() <= room)[ok].all()) and bool(got.dlogits.isfinite().all())
        exact = want["token"]
        assert bool(((got.token_loss.double() - exact).abs() <= 2 * lu.LSE + 2.0 ** -23 * exact.abs())[exact.isfinite()].all())
        assert not bool(got.token_loss.isnan().any())


@pytest.mark.parametrize("rows,v", SHAPES)
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("offset,tau", [(12345.6789, 0.001), (123456.789, 0.001), (-98765.4321, 0.001), (7654321.0, 0.07), (1.1e8, 0.9)])
def test_the_log_sum_exp_of_far_rows(rows, v, dtype, offset, tau):
    """Numbers without many zeros: neighbours of the offset in the type, of which the largest hold the row's sum."""
    g = torch.Generator().manual_seed(v)
    top = torch.tensor(offset).to(dtype)
    down = top
    for _ in range(1 if dtype == BF else 2):
        down = torch.nextafter(down, torch.tensor(-math.inf, dtype=dtype))
    z = torch.full((rows, -(-v // 8) * 8), math.nan, dtype=dtype)
    z[:, :v] = torch.where(torch.rand(rows, v, generator=g) < 0.3, top, down)
    z[:, 0] = top
    z = z.cuda()[:, :v]
    index = torch.stack([torch.randperm(v, generator=g)[:3] for _ in range(rows)]).to(torch.int32).cuda()
    logit = tau * torch.randn(rows, 3, generator=g).cuda()
    stats = rb.alloc_stats()
    want = lu.distill(z, index, logit, None, None, tau)
    got = rb.distill_loss(z, index, logit, None, None, tau, stats=stats)
    lu.check(want, got, rb.read_loss_stats(stats), dtype)
    targets = index[:, 0].contiguous()
    lp = lu._token_logp(z, targets, torch.ones(rows, dtype=torch.bool, device="cuda"))[0]
    if tau == 0.9:  # and without a temperature
        got = rb.clip_loss(z, targets, None, lp.float() + 0.1, torch.ones(rows, device="cuda"), rows, 1, stats=stats)
        lu.check(lu.clip(z, targets, None, lp.float() + 0.1, torch.ones(rows, device="cuda"), rows), got, rb.read_loss_stats(stats), dtype)
