"""The losses over the logits at the sizes where another kernel, another way of summing or another number of blocks takes over."""
import math

import pytest
import torch

import losses_util as lu
import test_gpu_losses as base
from paper_2510_03515_b200 import binding as rb

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _ragged(n, length, seed):
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(0, length + 1, (n,), generator=g).tolist()
    return [length] + lens[1:]


# on both sides of every length at which rows go to another kernel (bytes of a row: 8, 32, 72, 110 and 172 KB)
EDGES = [(b, d) for b in (8192, 32768, 73728, 112640, 176128) for d in (-16, 0, 16)]
# more rows than one block sums, more generations than one block counts, rows enough for every warp to take several
MANY = [(9, 300, 500, F32), (33, 70, 4096, BF), (700, 5, 1030, BF), (1100, 3, 500, F32), (5, 501, 16390, BF), (4, 600, 30001, BF), (3, 701, 50257, BF),
        (5, 430, 61000, BF), (3, 700, 33001, F32), (2, 1051, 90001, BF)]


@pytest.mark.parametrize("size,more", EDGES)
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_lengths_where_kernels_change(size, more, dtype):
    v = (size + more) // dtype.itemsize
    for v in (v, v - 1):  # a whole vector at the end, and a part of one
        shape = (3, 5, v, dtype, None, [5, 0, 3])
        base.test_clip(shape)
        base.test_preference(shape, "squared")
        base.test_distill(shape, v % 2 == 0)


@pytest.mark.parametrize("shape", MANY, ids=lambda s: f"{s[0]}x{s[1]}x{s[2]}")
def test_many_rows(shape):
    n, length, v, dtype = shape
    full = (n, length, v, dtype, None, _ragged(n, length, v))
    base.test_clip(full)
    base.test_distill(full, True)
    torch.cuda.empty_cache()


@pytest.mark.parametrize("n,length,v,dtype,k", [(2, 9, 61000, BF, 256), (2, 9, 151936, BF, 256), (2, 5, 300007, BF, 256), (2, 5, 120001, F32, 200),
                                                (150, 3, 61000, BF, 130), (150, 3, 100003, F32, 70), (40, 15, 4096, BF, 256), (5, 300, 30000, BF, 256)])
def test_long_lists_with_a_bucket(n, length, v, dtype, k):
    """Lists of up to 256 columns: drawn from all, side by side (one vector holds several), at the row's end and at its start."""
    z, _, mask, g = lu.grid(n, length, v, dtype, seed=v + k, lens=_ragged(n, length, v))
    T = n * length
    index, _ = base._lists(z, k, g)
    side = torch.arange(k, dtype=torch.int32)
    for r, first in ((0, 0), (1, v - k), (2, v // 2), (3, v // 3 + 1)):
        if r < T:
            index[r] = (side + first)[torch.randperm(k, generator=g)].cuda()
    index[torch.rand(T, k, generator=g).cuda() < 0.1] = -1
    near = torch.nan_to_num(z.float(), nan=0.0).gather(1, index.long().clamp_min(0))
    logit = near + torch.randn(T, k, generator=g).cuda()
    part = torch.logsumexp(torch.where(index >= 0, logit.double(), -math.inf), 1)
    lse = (part + torch.log1p(torch.rand(T, generator=g).cuda().double() * 0.8 + 0.001)).float()
    stats = rb.alloc_stats()
    for top_lse in (lse, None):
        want = lu.distill(z, index, logit, mask, top_lse)
        got = rb.distill_loss(z, index, logit, mask, top_lse, stats=stats)
        lu.check(want, got, rb.read_loss_stats(stats), dtype)
        got = rb.distill_loss(z, index, logit, mask, top_lse, want_grad=False, stats=stats)
        lu.check(want, got, rb.read_loss_stats(stats), dtype, grad=False)


@pytest.mark.parametrize("kind", ["sigmoid", "hinge", "squared"])
@pytest.mark.parametrize("n,length,n_pairs", [(100, 3, 5000), (700, 4, 100), (2, 3, 4097), (300, 5, 4096), (5000, 2, 1 << 20)])
def test_many_pairs(kind, n, length, n_pairs):
    """More pairs, or pairs times generations, than one block goes through."""
    v, dtype = 600, F32
    z, targets, mask, g = lu.grid(n, length, v, dtype, seed=n, lens=_ragged(n, length, n))
    live = lu.rows_that_count(targets, mask, v)
    ref = (lu._token_logp(z, targets, live)[0] + 0.3 * torch.randn(n * length, generator=g).cuda()).float()
    pairs = torch.randint(-1, n + 1, (n_pairs, 2), generator=g, dtype=torch.int32).cuda()
    kw = dict(beta=0.3, margin=0.25)
    m = lu.preference(z, targets, mask, pairs, n, ref, kind=kind, mean=True, **kw)["margins"]
    corner = ((m - (1 if kind == "hinge" else 0)).abs() < 1e-3) | ((m.abs() < 1e-3) & ~m.isnan())
    pairs[corner] = -1  # at a corner the sign of a rounding decides: such pairs are not valid ones here
    want = lu.preference(z, targets, mask, pairs, n, ref, kind=kind, mean=True, **kw)
    flags = {"sigmoid": 0, "hinge": rb.PREF_HINGE, "squared": rb.PREF_SQUARED}[kind] | rb.PREF_TOKEN_MEAN
    stats = rb.alloc_stats()
    for grad in (True, False):
        got = rb.preference_loss(z, targets, mask, pairs, n, length, ref, flags=flags, want_grad=grad, stats=stats, **kw)
        st = rb.read_loss_stats(stats)
        lu.check(want, got, st, dtype, grad)
        assert st["n_pairs"] == want["valid"] and abs(st["mean_kl"] * max(1, want["valid"]) - want["won"]) < 1e-6
        assert torch.equal(got.margins.isnan(), want["margins"].isnan())


def test_many_pairs_one_of_them_without_a_finite_slope():
    """The token of one generation has no probability: its margins are not finite, and other generations keep their gradients."""
    n, v = 400, 64
    z, targets, _, g = lu.grid(n, 1, v, F32, seed=31)
    pairs = torch.randint(0, n // 2, (5000, 2), generator=g, dtype=torch.int32).cuda()
    z[n - 1, targets[n - 1].long()] = -math.inf
    pairs[7] = torch.tensor([n - 1, n - 2], dtype=torch.int32)
    keep = torch.ones(5000, dtype=torch.bool, device="cuda")
    keep[7] = False
    want = rb.preference_loss(z, targets, None, pairs[keep].contiguous(), n, 1, flags=rb.PREF_SQUARED | rb.LOSS_NORM_GIVEN, norm_z=5000)
    got = rb.preference_loss(z, targets, None, pairs, n, 1, flags=rb.PREF_SQUARED)
    assert math.isinf(float(got.margins[7])) and math.isinf(float(got.loss))
    assert torch.equal(got.margins[keep], want.margins)
    a, b = got.dlogits[: n // 2], want.dlogits[: n // 2]
    assert bool(((a - b).abs() <= 2.0 ** -22 * b.abs() + 1e-12).all())  # the same slopes; a rounding of the coefficient and one of the result each


@pytest.mark.parametrize("n,length,v,dtype", [(500, 5, 2048, BF), (6, 400, 61000, BF), (4, 600, 30001, BF)])
def test_same_bits_of_many_rows(n, length, v, dtype):
    """Rows are dealt out as the SMs come to them; what is computed of them does not depend on it, nor on the rows beside them."""
    z, targets, mask, g = lu.grid(n, length, v, dtype, seed=20, lens=_ragged(n, length, v))
    calls = base._calls(z, targets, mask, g, n, length)
    for name, call in calls.items():
        first = call(z)
        for _ in range(3):
            base._same(first, call(z))
