"""Attention and its gradient against the definition in 64 bits where the scores are not those of the default scale: other scales,
and scores that grow or fall along a generation, so that a row's maximum moves by far more than its rescaling threshold."""
import math

import pytest
import torch

import test_gpu_attention as base

pytestmark = pytest.mark.gpu

from paper_2510_03515_b200 import binding as rb  # noqa: E402

B, U = base.B, base.U


def _check(cpu, dev, bounds, live, dout, n, length, window, scale):
    """Forward and gradient within what their roundings allow.

    Beside the terms of the plain tests: an exponent in base 2 is a fused multiply-add of a score and a rounded shift, both up to z
    = the largest score of the row (1 + 2 roundings of at most 2 z), each rescaling rounds a difference and a product (together
    at most 4 z, as the differences add up to the range of the scores), and the factor scale * log2(e) is rounded to float (z).
    Numerator and denominator: below 20 z U in all.
    """
    q, k, v = cpu
    heads, hd = q.shape[1], q.shape[2]
    b = None if bounds is None else bounds.cuda()
    stats = rb.alloc_stats()
    out, lse = rb.attention(*dev, n, length, b, window, scale, stats)
    assert rb.read_stats(stats)["status"] == 0
    r = rb.attention_grad(*dev, out, lse, dout.cuda(), n, length, b, window, scale, stats)
    assert rb.read_stats(stats)["status"] == 0
    out, lse = out.cpu(), lse.cpu()
    dead = ~live
    assert (out.reshape(n, length, heads, hd)[dead] == 0).all() and (lse.transpose(1, 2)[dead] == -math.inf).all()
    for i, h, at, rows, see, qh, kh, vh, z in base._definition(q, k, v, n, length, window, live, scale):
        want = torch.logsumexp(z, 1)
        p = torch.exp(z - want[:, None])
        top = z.masked_fill(~see, 0).abs().amax(1)
        ds = ((hd + 4) * U * scale * (qh.abs() @ kh.abs().T)).masked_fill(~see, 0).amax(1) + 20 * U * top
        tol_lse = ds + 2.0 ** -21 + 200 * U + 4 * U * (want.abs() + ds + 12)
        assert ((lse[i, h, at].double() - want).abs() <= tol_lse).all()
        o = p @ vh
        tol = (p @ vh.abs()) * (B + 2 * ds[:, None] + 2.0 ** -19 + length * U) + o.abs() * B + 1e-30
        assert ((out[rows, h].double() - o).abs() <= tol).all()
    want = base._reference_grads(q, k, v, out, lse, dout, n, length, window, live, scale)
    rows = dead.reshape(-1)
    for name, got, (ref, tol) in zip(("dq", "dk", "dv"), (r.dq, r.dk, r.dv), want):
        got = got.cpu().double()
        assert (got[rows] == 0).all(), name
        assert ((got - ref).abs() <= tol).all(), name


@pytest.mark.parametrize("scale", [0.3, 1.0 / 64, 1.0])
@pytest.mark.parametrize("n,length,heads,kv,hd,window,kind", [
    (2, 300, 4, 2, 64, 0, "right"), (2, 260, 2, 1, 128, 0, "left"), (1, 400, 2, 2, 80, 70, "full"), (9, 30, 2, 1, 64, 0, "mixed")])
def test_scales(n, length, heads, kv, hd, window, kind, scale):
    cpu, dev, bounds, live, g = base._make(n, length, heads, kv, hd, kind, 11)
    dout = torch.randn(n * length, heads, hd, generator=g).to(base.BF)
    _check(cpu, dev, bounds, live, dout, n, length, window, scale)


@pytest.mark.parametrize("slope", [0.25, 2.0, -0.25])
@pytest.mark.parametrize("n,length,heads,kv,hd,window,kind", [
    (1, 700, 4, 2, 64, 0, "full"), (2, 600, 2, 1, 128, 0, "left"), (2, 640, 2, 1, 128, 200, "right"), (1, 515, 2, 2, 64, 131, "mixed"),
    (5, 60, 2, 1, 128, 0, "mixed"), (9, 40, 2, 1, 64, 11, "right")])
def test_scores_that_grow(n, length, heads, kv, hd, window, kind, slope):
    """Scores rise (or fall) by about `slope` a position: 0.25 moves the maximum by 46 powers of two a tile."""
    (q, k, v), _, bounds, live, g = base._make(n, length, heads, kv, hd, kind, 12)
    q, k = q.clone(), k.clone()
    ramp = slope * (torch.arange(length) - length / 2).repeat(n)
    q[..., 0] = hd ** 0.5
    k[..., 0] = ramp[:, None].to(base.BF)
    dead = ~live.reshape(-1)
    q[dead] = k[dead] = float("nan")
    dev = [x.cuda() for x in (q, k, v)]
    dout = torch.randn(n * length, heads, hd, generator=g).to(base.BF)
    _check((q, k, v), dev, bounds, live, dout, n, length, window, hd ** -0.5)
