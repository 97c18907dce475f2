"""Preference loss with margins that are not finite: a generation whose token has no probability."""
import math

import pytest
import torch

import losses_util as lu
from paper_2510_03515_b200 import binding as rb

pytestmark = pytest.mark.gpu
F32 = torch.float32
FLAGS = {"sigmoid": 0, "hinge": rb.PREF_HINGE}


def _grid(dead):
    """Six generations of two rows; a token of those in `dead` is masked out of the vocabulary."""
    z, targets, mask, _ = lu.grid(6, 2, 300, F32, seed=4)
    for n in dead:
        z[2 * n, int(targets[2 * n])] = -math.inf
    return z, targets, mask


def _pairs(first, n_pairs):
    """`first`, and pairs of generations 2 to 5, in all n_pairs of them."""
    p = torch.tensor([[2, 3], [4, 5], [5, 2]], dtype=torch.int32).repeat(-(-n_pairs // 3), 1)[:n_pairs]
    p[0] = torch.tensor(first, dtype=torch.int32)
    return p.cuda()


@pytest.mark.parametrize("n_pairs", [7, 5000])
@pytest.mark.parametrize("kind", ["sigmoid", "hinge"])
def test_one_that_cannot_be_on_the_worse_side(kind, n_pairs):
    """h = inf: the pair's loss is 0, and so is its pull."""
    z, targets, mask = _grid([1])
    pairs = _pairs([0, 1], n_pairs)
    stats = rb.alloc_stats()
    got = rb.preference_loss(z, targets, mask, pairs, 6, 2, beta=0.1, margin=0.2, flags=FLAGS[kind], stats=stats)
    want = rb.preference_loss(z, targets, mask, pairs[1:].contiguous(), 6, 2, beta=0.1, margin=0.2, flags=FLAGS[kind] | rb.LOSS_NORM_GIVEN, norm_z=n_pairs)
    assert float(got.margins[0]) == math.inf and rb.read_loss_stats(stats)["n_pairs"] == n_pairs
    assert abs(float(got.loss) - float(want.loss)) <= 2.0 ** -22 * abs(float(want.loss))
    assert bool(((got.dlogits - want.dlogits).abs() <= 2.0 ** -22 * want.dlogits.abs()).all()) and not bool(got.dlogits[:4].any())


@pytest.mark.parametrize("n_pairs", [7, 5000])
@pytest.mark.parametrize("kind", ["sigmoid", "hinge"])
def test_one_that_cannot_be_on_the_better_side(kind, n_pairs):
    """h = -inf: the loss is infinite, the pull that of any far pair."""
    z, targets, mask = _grid([0])
    got = rb.preference_loss(z, targets, mask, _pairs([0, 1], n_pairs), 6, 2, beta=0.1, flags=FLAGS[kind])
    assert float(got.margins[0]) == -math.inf and float(got.loss) == math.inf
    p = torch.softmax(z[:4].double(), 1)
    hot = torch.zeros_like(p).scatter_(1, targets[:4].long()[:, None], 1.0)
    pull = 0.1 / n_pairs * torch.tensor([1.0, 1.0, -1.0, -1.0], device="cuda", dtype=torch.float64)[:, None]
    want = -pull * (hot - p)
    assert bool(((got.dlogits[:4].double() - want).abs() <= (lu.P + lu.LSE) * pull.abs() * (p + hot) + 2.0 ** -24 * want.abs()).all())
    assert bool(got.dlogits.isfinite().all())


@pytest.mark.parametrize("n_pairs", [7, 5000])
@pytest.mark.parametrize("kind", ["sigmoid", "hinge"])
def test_two_that_cannot_be(kind, n_pairs):
    """-inf - -inf: such a margin is NaN, and says so in the loss and in the gradients of its two generations alone."""
    z, targets, mask = _grid([0, 1])
    got = rb.preference_loss(z, targets, mask, _pairs([0, 1], n_pairs), 6, 2, beta=0.1, flags=FLAGS[kind])
    assert math.isnan(float(got.margins[0])) and math.isnan(float(got.loss)) and bool(got.margins[1:].isfinite().all())
    assert bool(got.dlogits[:4].isnan().any(1).all()) and bool(got.dlogits[4:].isfinite().all())
