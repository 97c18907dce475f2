"""The logistic preference loss's slope where a pair is far on the right side: a small number, exact to its own size."""
import pytest
import torch

import losses_util as lu
from paper_2510_03515_b200 import binding as rb

pytestmark = pytest.mark.gpu
F32 = torch.float32
MARGINS = [-80.0, -20.0, -1.0, 0.0, 1.0, 8.0, 20.0, 25.0, 30.0, 34.0, 36.0, 37.5, 40.0, 50.0, 60.0, 80.0]


@pytest.mark.parametrize("n_pairs", [16, 5008])
@pytest.mark.parametrize("smoothing", [0.0, 0.1, 0.5])
@pytest.mark.parametrize("mean", [False, True])
def test_slopes(n_pairs, smoothing, mean):
    n, v = 2 * len(MARGINS), 200
    z, targets, _, _ = lu.grid(n, 1, v, F32, seed=10)
    lp = lu._token_logp(z, targets, torch.ones(n, dtype=torch.bool, device="cuda"))[0]
    ref = lp.float()
    ref[1::2] += torch.tensor(MARGINS, device="cuda")
    pairs = torch.arange(n, dtype=torch.int32).view(-1, 2).repeat(n_pairs // len(MARGINS), 1).cuda()
    got = rb.preference_loss(z, targets, None, pairs, n, 1, ref, beta=1.0, label_smoothing=smoothing, flags=rb.PREF_TOKEN_MEAN if mean else 0)
    s = lp - ref.double()
    h = s[0::2] - s[1::2]
    right, wrong = 1 / (1 + torch.exp(h)), 1 / (1 + torch.exp(-h))
    g = ((1 - smoothing) * right - smoothing * wrong) / len(MARGINS)
    # the margin's error, 2 LSE, times the slopes of either part; a rounding of the sum of the two
    dg = 2 * lu.LSE * ((1 - smoothing) * right + smoothing * wrong).minimum((right * wrong)) / len(MARGINS) + 2.0 ** -50 * smoothing
    p = torch.softmax(z.double(), 1)
    hot = torch.zeros_like(p).scatter_(1, targets.long()[:, None], 1.0)
    coef, dcoef = torch.stack([g, -g], 1).view(-1, 1), torch.stack([dg, dg], 1).view(-1, 1)
    want = coef * (p - hot)
    room = (dcoef + (lu.P + lu.LSE) * coef.abs()) * (p + hot) + 2.0 ** -24 * want.abs() + 2.0 ** -126
    assert bool(((got.dlogits.double() - want).abs() <= room).all()), f"{float(((got.dlogits.double() - want).abs() / room).max()):.3g} of its bound"
    if smoothing == 0.0:
        assert bool((got.dlogits != 0).any(1).all())
