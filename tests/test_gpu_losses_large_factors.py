"""Factors of a row's gradient that are near the end of the floats' range or beyond it: a ratio or a KL term of e^90 and more.  Columns whose
product with the factor is a float get it, columns without probability get exactly 0, and what is larger becomes infinite."""
import math

import pytest
import torch

import losses_util as lu
from paper_2510_03515_b200 import binding as rb

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("rows,v", [(1300, 700), (10, 700), (700, 20001), (5, 61000), (3, 151936), (2, 200001)])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_clip(rows, v, dtype):
    z, targets, mask, g = lu.grid(rows, 1, v, dtype, seed=v)
    dead = torch.rand(rows, v, generator=g).cuda() < 0.3
    dead.scatter_(1, targets.long()[:, None], False)
    z[dead] = -math.inf
    live = torch.ones(rows, dtype=torch.bool, device="cuda")
    lp, p, _ = lu._token_logp(z, targets, live)
    kind = torch.arange(rows).cuda() % 5  # ratios and KL terms of e^60 to e^300, signs, and one of none
    far = torch.tensor([60.0, 95.0, 130.0, 300.0, 0.5], device="cuda")[kind]
    adv = -1.0 - torch.rand(rows, generator=g).cuda()  # below 0 nothing is cut off
    old, ref = (lp - far).float(), (lp + far.flip(0)).float()
    for beta in (0.0, 0.1):
        want = lu.clip(z, targets, None, old, adv, rows, ref if beta else None, beta=beta)
        got = rb.clip_loss(z, targets, None, old, adv, rows, 1, ref if beta else None, kl_beta=beta)
        d = got.dlogits.double()
        assert bool((d[dead] == 0).all())
        # what is not within a rounding of the type's end; the ratios' own roundings (old in float, times its slope) as in the utility
        room = want["grad_tol"] + (lu.HALF[dtype] + lu.P) * want["grad"].abs() + 2.0 ** -126
        top = torch.finfo(dtype).max
        inside = want["grad"].abs() + room < top
        assert bool(((d - want["grad"]).abs() <= room)[inside].all())
        beyond = want["grad"].abs() - room > top
        assert torch.equal(d[beyond], torch.sign(want["grad"][beyond]) * math.inf)
        assert bool(inside.any()) and bool(beyond.any())
    # a ratio that is infinite
    old[0] = -3e38
    got = rb.clip_loss(z, targets, None, old, adv, rows, 1)
    assert bool((got.dlogits[0][dead[0]] == 0).all()) and math.isinf(float(got.dlogits[0][targets[0].long()]))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_preference(dtype):
    """The squared form's slope grows with the margin: 2e37 and more for sums that are as far apart."""
    z, targets, mask, g = lu.grid(4, 2, 900, dtype, seed=5)
    z[:, 5::7] = -math.inf
    z.scatter_(1, targets.long()[:, None], 2.0)
    ref = torch.zeros(8, device="cuda")
    ref[0] = 1e36
    pairs = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda")
    kw = dict(beta=300.0)
    want = lu.preference(z, targets, mask, pairs, 4, ref, kind="squared", **kw)
    got = rb.preference_loss(z, targets, mask, pairs, 4, 2, ref, flags=rb.PREF_SQUARED, **kw)
    d, top = got.dlogits.double(), torch.finfo(dtype).max
    # the slope's error follows the margin's, 2^-53 of it
    room = (lu.HALF[dtype] + 2 * lu.P) * want["grad"].abs() + 2.0 ** -126
    inside = want["grad"].abs() + room < top
    assert bool(((d - want["grad"]).abs() <= room)[:4][inside[:4]].all())
    assert bool((d[:, 5::7][z[:, 5::7] == -math.inf] == 0).all())
