"""Rows of 2 GiB and more, whose sizes in bytes do not fit in 31 bits, against 64 bits, a piece of the row at a time."""
import math

import pytest
import torch

import losses_util as lu
from paper_2510_03515_b200 import binding as rb

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
PIECE = 1 << 26


def _row(v, dtype, seed):
    torch.cuda.empty_cache()
    step = 16 // dtype.itemsize
    g = torch.Generator(device="cuda").manual_seed(seed)
    z = torch.empty(1, -(-v // step) * step, dtype=dtype, device="cuda")
    for a in range(0, z.shape[1], PIECE):
        part = z[:, a:a + PIECE]
        part.copy_(torch.randn(part.shape, device="cuda", generator=g) * 2)
    return z[:, :v]


def _lse(z):
    """Of one row in double; the largest logit is below 20, so nothing is taken off."""
    return math.log(sum(float(z[0, a:a + PIECE].double().exp().sum()) for a in range(0, z.shape[1], PIECE)))


def _worst(z, d, lse, factor, columns, values):
    """Largest part of its bound that the gradient takes; factor * softmax but for the columns' values.  The bound: a probability's
    error P, a log-sum-exp's and the result's rounding."""
    worst = 0.0
    for a in range(0, z.shape[1], PIECE):
        want = factor * torch.exp(z[0, a:a + PIECE].double() - lse)
        here = (columns >= a) & (columns < a + PIECE)
        want[columns[here] - a] = values[here]
        room = (lu.P + lu.LSE + lu.HALF[z.dtype]) * want.abs() + 2.0 ** -126
        room[columns[here] - a] += lu.LSE  # a difference of probabilities
        worst = max(worst, float(((d[0, a:a + PIECE].double() - want).abs() / room).max()))
    return worst


@pytest.mark.parametrize("v,dtype", [((1 << 29) + 5, F32), (1 << 30, BF)], ids=["f32", "bf16"])
def test_rows_of_more_than_two_gib(v, dtype):
    z = _row(v, dtype, 3)
    y = v - 2
    z[0, y] = 19.0
    lse = _lse(z)
    lp = float(z[0, y]) - lse
    one = lambda x: torch.full((1,), x, device="cuda")  # noqa: E731
    targets = torch.full((1,), y, dtype=torch.int32, device="cuda")
    columns = torch.tensor([y], device="cuda")
    got = rb.clip_loss(z, targets, None, one(lp - 0.1), one(1.25), 1, 1)
    rho = math.exp(lp - float(one(lp - 0.1)))
    assert abs(float(got.token_logp) - lp) <= lu.LSE + 2.0 ** -24 * abs(lp) and abs(float(got.loss) + 1.25 * rho) <= 4 * lu.LSE
    value = torch.tensor([1.25 * rho * math.expm1(lp)], dtype=torch.float64, device="cuda")
    assert _worst(z, got.dlogits, lse, 1.25 * rho, columns, value) <= 1.0
    for grad in (False, True):
        other = rb.preference_loss(z, targets, None, torch.zeros(1, 2, dtype=torch.int32, device="cuda"), 1, 1, want_grad=grad)
        assert abs(float(other.token_logp) - lp) <= lu.LSE + 2.0 ** -24 * abs(lp) and abs(float(other.loss) - math.log(2.0)) <= 1e-6
    assert not bool(other.dlogits.any())  # a pair of a generation with itself
    del got, other
    # a list with entries at both ends of the row, and the rest in one bucket
    columns = torch.tensor([0, 7, v // 2, y, v - 1], device="cuda")
    for a in columns.tolist():
        z[0, a] = 18.0 + a % 3
    lse = _lse(z)
    t = torch.tensor([[1.0, 0.5, 2.0, 0.0, 1.5]], device="cuda")
    top_lse = one(3.0)
    lt, lq = t[0].double() - 3.0, z[0, columns].double() - lse
    p, p0 = lt.exp(), 1 - float(lt.exp().sum())
    q0 = 1 - float(lq.exp().sum())  # 0.99 and more: nothing is lost in the difference
    assert q0 > 0.5
    want = float((p * (lt - lq)).sum()) + p0 * (math.log(p0) - math.log(q0))
    for grad in (False, True):
        got = rb.distill_loss(z, columns.to(torch.int32)[None], t, None, top_lse, want_grad=grad)
        assert abs(float(got.loss) - want) <= 2 * lu.LSE + 2.0 ** -23 * want
    assert _worst(z, got.dlogits, lse, 1 - p0 / q0, columns, lq.exp() - p) <= 1.0
    del got, z
    torch.cuda.empty_cache()
