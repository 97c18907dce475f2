"""Distillation with a top_lse that is below the list's own log-sum-exp: the list's probabilities come to more than one, there is nothing
outside it, and the gradient is that of the loss all the same."""
import pytest
import torch

import losses_util as lu
from paper_2510_03515_b200 import binding as rb

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def _inputs(rows, v, k, dtype, tau, over, seed):
    z, _, _, g = lu.grid(1, rows, v, dtype, seed=seed, std=2.0)
    index = torch.stack([torch.randperm(v, generator=g)[:k] for _ in range(rows)]).to(torch.int32).cuda()
    t = torch.randn(rows, k, generator=g).cuda()
    return z, index, t, (torch.logsumexp(t.double() / tau, 1) - over).float()


@pytest.mark.parametrize("rows,v,k", [(1300, 500, 7), (4, 500, 40), (20, 4097, 5), (700, 20001, 8), (4, 61000, 16), (3, 151936, 200), (2, 200001, 3), (9, 32, 32)])
@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("over,tau", [(0.01, 1.0), (0.7, 1.0), (1.5, 2.0)])
def test_gradient(rows, v, k, dtype, over, tau):
    z, index, t, top_lse = _inputs(rows, v, k, dtype, tau, over, v + k)
    x = z.double().requires_grad_()
    lq = torch.log_softmax(x / tau, 1).gather(1, index.long())
    lt = t.double() / tau - top_lse.double()[:, None]
    p = lt.exp()
    assert bool((p.sum(1) > 1).all())
    each = (p * (lt - lq)).sum(1)
    loss = each.mean()
    want = torch.autograd.grad(loss, x)[0]
    q, hot = torch.softmax(x.detach() / tau, 1), torch.zeros_like(want).scatter_(1, index.long(), 1.0)
    got = rb.distill_loss(z, index, t, None, top_lse, tau)
    # a probability's error P on the student's term, times the list's mass; the result's rounding
    room = p.sum(1, keepdim=True) / (rows * tau) * ((lu.P + lu.LSE) * q + 1e-12 * hot) + (lu.HALF[dtype] + lu.P) * want.abs() + 2.0 ** -126
    assert bool(((got.dlogits.double() - want).abs() <= room).all())
    assert bool(((got.token_loss.double() - each).abs() <= 2 * lu.LSE * p.sum(1) + 2.0 ** -24 * each.abs()).all())
    assert abs(float(got.loss) - loss.item()) <= 2 * lu.LSE * p.sum(1).max().item() + 2.0 ** -23 * abs(loss.item())
    assert torch.equal(rb.distill_loss(z, index, t, None, top_lse, tau, want_grad=False).token_loss, got.token_loss)


def test_gradient_against_differences():
    """Central differences of the library's loss: third derivatives below 10, and the loss in double is good to LSE a row."""
    h = 0.03125
    z, index, t, top_lse = _inputs(3, 30, 4, F32, 1.0, 0.9, 5)
    stats = rb.alloc_stats()
    d = rb.distill_loss(z, index, t, None, top_lse).dlogits
    for r in range(3):
        for c in (int(index[r, 0]), int(index[r, 3]), (int(index[r].max()) + 1) % 30):
            value = []
            for sign in (1, -1):
                x = z.clone()
                x = torch.nn.functional.pad(x, (0, 2))[:, :30]
                x[r, c] += sign * h
                rb.distill_loss(x, index, t, None, top_lse, want_grad=False, stats=stats)
                value.append(rb.read_loss_stats(stats)["loss"])
            assert abs((value[0] - value[1]) / (2 * h) - float(d[r, c])) <= 10 * h * h / 6 + 10 * lu.LSE / h
