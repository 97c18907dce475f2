"""Offsets of elements and bytes beyond 2^32, for rows of every kernel: some rows count, all others hold NaN and have to become zeros."""
import math
from types import SimpleNamespace

import pytest
import torch

import losses_util as lu
from paper_2510_03515_b200 import binding as rb

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.mark.parametrize("length,v", [(10000, 160000), (17000, 70000), (75000, 16000), (300000, 4000)])
def test_all_three_past_32_bits(length, v):
    """Four generations with one row that counts in each, two of them beyond 2^32 elements; against these four in 64 bits."""
    torch.cuda.empty_cache()
    T = 4 * length
    assert T * v > 2 ** 32
    z = torch.empty(T, v, dtype=BF, device="cuda")
    rows = torch.tensor([0, length + length // 3, 2 ** 32 // v + 1, T - 1], device="cuda")
    assert rows[2] // length in (2, 3)
    if rows[2] // length == 3:
        rows[2] = 3 * length - 1  # a byte offset beyond 2^32 then
    mask = torch.zeros(T, dtype=torch.bool, device="cuda")
    mask[rows] = True
    small, t4, _, g = lu.grid(1, 4, v, BF, seed=17)
    r = lambda *s: torch.randn(*s, generator=g).cuda()  # noqa: E731
    pairs = torch.tensor([[0, 1], [3, 2], [1, 3]], dtype=torch.int32, device="cuda")
    old4, ref4, adv = r(4) - 8.0, r(4) - 8.0, r(4)
    k = 5
    index4 = torch.stack([torch.randperm(v, generator=g)[:k] for _ in range(4)]).to(torch.int32).cuda()
    logit4, lse4 = r(4, k), torch.full((4,), 3.5, device="cuda")

    def far(x, fill):
        out = torch.full((T,) + tuple(x.shape[1:]), fill, dtype=x.dtype, device="cuda")
        out[rows] = x
        return out

    targets, old, ref = far(t4, 0), far(old4, math.nan), far(ref4, math.nan)
    index, logit, lse = far(index4, 1), far(logit4, math.nan), far(lse4, math.nan)
    stats = rb.alloc_stats()
    calls = {
        "clip": (lambda: rb.clip_loss(z, targets, mask, old, adv, 4, length, ref, kl_beta=0.1, flags=rb.LOSS_NORM_SEQ, in_place=True, stats=stats),
                 lu.clip(small, t4, None, old4, adv, 4, ref4, beta=0.1, by_seq=True)),
        "preference": (lambda: rb.preference_loss(z, targets, mask, pairs, 4, length, ref, in_place=True, stats=stats),
                       lu.preference(small, t4, None, pairs, 4, ref4)),
        "distill": (lambda: rb.distill_loss(z, index, logit, mask, lse, in_place=True, stats=stats), lu.distill(small, index4, logit4, None, lse4)),
    }
    for name, (call, want) in calls.items():
        z.fill_(math.nan)
        z[rows] = small
        got = call()
        token = got.token_loss if name == "distill" else got.token_logp
        assert int((token != 0).sum()) == 4, name
        lu.check(want, SimpleNamespace(loss=got.loss, token_logp=token[rows], dlogits=z[rows]), rb.read_loss_stats(stats), BF)
        z[rows] = 0
        for a in range(0, T, 1 << 14):
            assert not bool((z[a:a + (1 << 14)] != 0).any()), (name, a)
    del z
    torch.cuda.empty_cache()
