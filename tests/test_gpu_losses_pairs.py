"""Preference loss with pairs of very different slopes: what a generation's gradient is does not depend on how far other pairs are
apart, nor on how many there are."""
import math

import pytest
import torch

import losses_util as lu
from paper_2510_03515_b200 import binding as rb

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
FEW, MANY = 40, 5000  # on either side of the number of pairs above which slopes are added up as whole numbers


def _far(n_pairs, far, n=60, v=300, seed=9):
    """Generations of one row each: pairs among the first half, and one pair whose margin is `far` times that of the others."""
    z, targets, _, g = lu.grid(n, 1, v, F32, seed=seed)
    ref = (lu._token_logp(z, targets, torch.ones(n, dtype=torch.bool, device="cuda"))[0] + 0.3 * torch.randn(n, generator=g).cuda()).float()
    ref[n - 1] = far
    pairs = torch.randint(0, n // 2, (n_pairs, 2), generator=g, dtype=torch.int32)
    pairs[:, 0] = torch.arange(n_pairs) % (n // 2)
    pairs[:, 1] = (pairs[:, 0] + 1 + pairs[:, 1] % (n // 2 - 1)) % (n // 2)  # never one with itself
    pairs[n_pairs // 2] = torch.tensor([n - 1, n - 2])
    return z, targets, ref, pairs.cuda()


def _coefficients(z, targets, d):
    """g of every generation from its gradient, least squares over softmax - 1[y], in double."""
    p = torch.softmax(z.double(), 1)
    p[torch.arange(z.shape[0], device="cuda"), targets.long()] -= 1
    return (d.double() * p).sum(1) / (p * p).sum(1)


@pytest.mark.parametrize("n_pairs", [FEW, MANY])
@pytest.mark.parametrize("far", [1e3, 1e8, 1e15, 1e25, 1e37])
def test_one_pair_far_apart(n_pairs, far):
    z, targets, ref, pairs = _far(n_pairs, far)
    n = z.shape[0]
    stats = rb.alloc_stats()
    want = lu.preference(z, targets, None, pairs, n, ref, beta=0.5, kind="squared")
    got = rb.preference_loss(z, targets, None, pairs, n, 1, ref, beta=0.5, flags=rb.PREF_SQUARED, stats=stats)
    st = rb.read_loss_stats(stats)
    assert abs(st["loss"] - want["loss"]) <= (want["loss_tol"] + 1e-12 * want["loss"]) and st["n_pairs"] == n_pairs
    near = slice(0, n // 2)
    room = want["grad_tol"] + (lu.HALF[F32] + lu.P) * want["grad"].abs() + 2.0 ** -126
    assert bool(((got.dlogits.double() - want["grad"]).abs() <= room)[near].all())
    assert bool(want["grad"][near].abs().amax(1).gt(1e-6).all())
    c, w = _coefficients(z[n - 2:], targets[n - 2:], got.dlogits[n - 2:]), 2 * 0.5 * 0.5 * far / n_pairs
    assert bool(((c.abs() - w).abs() <= 1e-4 * w + 2).all()) and float(c[0]) * float(c[1]) < 0


@pytest.mark.parametrize("n_pairs", [FEW, MANY])
def test_logistic_slopes_from_one_to_little(n_pairs):
    """Slopes from 1 to 2.06e-9 (margins of -50 to 20), each of generations of their own."""
    margins = [-50.0, 0.0, 1.0, 8.0, 14.0, 20.0]
    n, v = 2 * len(margins), 200
    z, targets, _, g = lu.grid(n, 1, v, F32, seed=10)
    lp = lu._token_logp(z, targets, torch.ones(n, dtype=torch.bool, device="cuda"))[0]
    ref = lp.float()
    ref[1::2] += torch.tensor(margins, device="cuda")
    pairs = torch.arange(n, dtype=torch.int32).view(-1, 2).repeat(-(-n_pairs // (n // 2)), 1).contiguous().cuda()
    got = rb.preference_loss(z, targets, None, pairs, n, 1, ref, beta=1.0)
    s = lp - ref.double()
    h = s[0::2] - s[1::2]
    want = (1 / (1 + torch.exp(h)) / len(margins)).repeat_interleave(2) * torch.tensor([1.0, -1.0], device="cuda").double().repeat(n // 2)
    c = _coefficients(z, targets, got.dlogits)
    # the log-probabilities' errors (twice LSE in the margin), a probability's error P on three terms
    assert bool(((c - want).abs() <= (2 * lu.LSE + 3 * lu.P) * want.abs()).all())


@pytest.mark.parametrize("kind", ["infinite", "both", "nan"])
def test_slopes_that_are_not_finite_are_alike(kind):
    """With few pairs and with many: the generations of such a pair get what the sum of their slopes is, others keep theirs."""
    results = []
    for n_pairs in (FEW, MANY):
        z, targets, ref, pairs = _far(n_pairs, 0.0)
        n = z.shape[0]
        ref[n - 1] = math.nan if kind == "nan" else math.inf
        if kind == "both":  # one generation beside one infinitely far below and one infinitely far above
            ref[n - 3] = -math.inf
            pairs[1] = torch.tensor([n - 3, n - 2], dtype=torch.int32)
        got = rb.preference_loss(z, targets, None, pairs, n, 1, ref, flags=rb.PREF_SQUARED)
        assert bool(got.dlogits[: n // 2].isfinite().all()) and bool((got.dlogits[: n // 2] != 0).any(1).all())
        at = got.dlogits[torch.arange(n - 3, n), targets[n - 3:].long()]
        results.append(at)
        assert not bool(at[1:].isfinite().any())
    assert torch.equal(results[0].isnan(), results[1].isnan()) and torch.equal(results[0].nan_to_num(), results[1].nan_to_num())
    assert bool(results[0][1].isnan()) == (kind != "infinite")


def test_many_pairs_that_all_hold_one_generation():
    """2^20 pairs of generation 0 with others: its sum of slopes is as good as one in double, and the same every time."""
    n, v, P = 2000, 100, 1 << 20
    z, targets, _, g = lu.grid(n, 1, v, F32, seed=12)
    lp = lu._token_logp(z, targets, torch.ones(n, dtype=torch.bool, device="cuda"))[0]
    ref = (lp + 3 * torch.randn(n, generator=g).cuda()).float()
    pairs = torch.stack([torch.zeros(P, dtype=torch.int32), torch.randint(1, n, (P,), generator=g, dtype=torch.int32)], 1)
    pairs[::2] = pairs[::2].flip(1)
    pairs = pairs.cuda()
    want = lu.preference(z, targets, None, pairs, n, ref, beta=1.0)
    stats = rb.alloc_stats()
    got = rb.preference_loss(z, targets, None, pairs, n, 1, ref, beta=1.0, stats=stats)
    lu.check(want, got, rb.read_loss_stats(stats), F32)
    again = rb.preference_loss(z, targets, None, pairs, n, 1, ref, beta=1.0)
    assert torch.equal(again.dlogits, got.dlogits)
