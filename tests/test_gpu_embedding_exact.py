"""The embedding's gradient where every sum is exact: rows of small whole numbers, whose float sums below 2^24 do not depend on
the order of the additions, so a row that is lost, taken twice or added to another token shows."""
import pytest
import torch

import test_gpu_embedding as base

pytestmark = pytest.mark.gpu

from paper_2510_03515_b200 import binding as rb  # noqa: E402


@pytest.mark.parametrize("dtype", [base.BF, base.F32])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("T,V,D,tok,mk", [c for c in base.CASES if c[0] > 1] + [
    (20000, 40, 600, "few", "none"), (9000, 3000, 1544, "zipf", "random"), (66001, 151936, 32, "zipf", "random")])
def test_exact_sums(T, V, D, tok, mk, accumulate, dtype):
    g = torch.Generator().manual_seed(T + V + D)
    tokens, mask = base._tokens(T, V, tok, g), base._mask(T, mk, g)
    bad = torch.rand(T, generator=g) < 0.03
    tokens[bad] = V + tokens[bad]
    live = ~bad if mask is None else (mask != 0) & ~bad
    dout = torch.randint(-3, 4, (T, D), generator=g).to(dtype)
    dout[~live] = float("nan")
    start = torch.randint(-9, 10, (V, D), generator=g).float() if accumulate else torch.zeros(V, D)
    want = start.double().index_add_(0, tokens[live].long(), dout[live].double() * 2)
    assert want.abs().max() < 2 ** 24
    got = rb.embedding_grad(base._pitched(dout.cuda(), 1)[:, :D], tokens.cuda(), None if mask is None else mask.cuda(), V, 2.0,
                            dtable=base._pitched(start.cuda(), 0)[:, :D] if accumulate else None)
    assert torch.equal(got.cpu().double(), want)
