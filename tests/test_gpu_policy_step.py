"""One training step of a one-layer policy made of the library's operators: embedding, projection (a plain product),
query/key norm and rotation, causal attention, output projection, loss on the hidden states; then the gradients all the way
back to every weight.  Compared with the same step in 64 bits.

Tolerance.  The step rounds to bf16 at some fifteen places, and no bound per element survives that many products.  The
reference is therefore run twice in 64 bits: exactly, and with a rounding to bf16 wherever the step rounds a matrix.  The
distance of the two, in the norm over a whole tensor, is what such roundings cost; the step's own roundings fall at the same
places with the same sizes, but on other values, so its distance from the exact result is another draw of the same size: four
times it is allowed.  The behaviour log-probabilities are so low that every importance weight is clipped, which makes the
coefficients of the generations the same in all three.
"""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

import oracle  # noqa: E402
from paper_2510_03515_b200 import binding as rb  # noqa: E402

BF, F64 = torch.bfloat16, torch.float64


class _Round(torch.autograd.Function):
    """bf16 on the way forward and on the way back."""

    @staticmethod
    def forward(ctx, x):
        return x.to(BF).to(F64)

    @staticmethod
    def backward(ctx, g):
        return g.to(BF).to(F64)


def _batch(N, L, V, D, H, Hk, hd, side):
    g = torch.Generator().manual_seed(3)
    w = lambda r, c: (torch.randn(r, c, generator=g) / r ** 0.5).to(BF)  # noqa: E731
    T = N * L
    lens = torch.randint(L // 2, L + 1, (N,), generator=g)
    lo = L - lens if side == "left" else torch.zeros(N, dtype=torch.long)
    t = torch.arange(L)
    live = (t >= lo[:, None]) & (t < (lo + lens)[:, None])
    prompt = L // 5
    return dict(
        E=(torch.randn(V, D, generator=g) / D ** 0.5).to(BF), Wqkv=w(D, (H + 2 * Hk) * hd), Wo=w(H * hd, D), W=w(D, V),
        qw=1 + 0.2 * torch.randn(hd, generator=g), kw=1 + 0.2 * torch.randn(hd, generator=g),
        inv=(10000.0 ** (-torch.arange(0, hd, 2, dtype=F64) / hd)).float(),
        tokens=torch.randint(0, V, (T,), generator=g, dtype=torch.int32),
        targets=torch.randint(0, V, (T,), generator=g, dtype=torch.int32),
        live=live.reshape(-1).to(torch.uint8),
        loss_mask=(live & (t >= (lo + prompt)[:, None])).reshape(-1).to(torch.uint8),
        bounds=torch.stack([lo, lo + lens], 1).to(torch.int32),
        positions=(t[None, :] - lo[:, None]).clamp_min(0).reshape(-1).to(torch.int32),
        behav=torch.full((T,), -20.0), rewards=torch.rand(N, generator=g).round(),
        offsets=torch.tensor([0, N // 2, N], dtype=torch.int32))


def _library(b, N, L, V, D, H, Hk, hd, window):
    """The step on the GPU; returns what a user would hand to an optimiser."""
    T, scale = N * L, D ** 0.5
    x = rb.embedding(b["E"], b["tokens"], b["live"], scale)
    qkv = (x @ b["Wqkv"]).view(T, H + 2 * Hk, hd)
    q, k, v = qkv[:, :H], qkv[:, H:H + Hk], qkv[:, H + Hk:]
    norm = (b["qw"], b["kw"], b["inv"])
    qn, kn = rb.qk_norm_rope(q, k, *norm, N, L, b["positions"], b["live"])
    out, lse = rb.attention(qn, kn, v, N, L, b["bounds"], window)
    o = out.view(T, H * hd)
    h = x + o @ b["Wo"]
    desc = rb.make_desc(N, L, V, 2, BF, V)
    loss, dh, dW = b["E"].new_empty(1, dtype=torch.float32), torch.empty_like(h), torch.empty(D, V, device=h.device)
    logp = torch.empty(T, device=h.device)
    rb.rapid_pg_loss_fused_head(desc, h, b["W"], b["targets"], b["loss_mask"], b["behav"], b["rewards"], b["offsets"], loss, dh,
                                dW, logp, None, None, rb.alloc_fused_head_workspace(desc, D, h.device))
    do = (dh @ b["Wo"].T).view(T, H, hd)
    dqkv = torch.empty_like(qkv)
    a = rb.attention_grad(qn, kn, v, out, lse, do, N, L, b["bounds"], window, dv=dqkv[:, H + Hk:])
    r = rb.qk_norm_rope_grad(q, k, *norm, a.dq, a.dk, N, L, b["positions"], b["live"], dq=dqkv[:, :H], dk=dqkv[:, H:H + Hk])
    dqkv = dqkv.view(T, -1)
    dx = dh + dqkv @ b["Wqkv"].T
    return dict(logp=logp, W=dW, Wo=o.float().T @ dh.float(), Wqkv=x.float().T @ dqkv.float(), qw=r.dq_weight, kw=r.dk_weight,
                E=rb.embedding_grad(dx, b["tokens"], b["live"], V, scale))


def _reference(b, N, L, V, D, H, Hk, hd, window, rounded):
    R = _Round.apply if rounded else (lambda x: x)
    T = N * L
    p = {n: b[n].to(F64).requires_grad_() for n in ("E", "Wqkv", "Wo", "qw", "kw")}
    live = b["live"].bool()
    x = R(R(p["E"][b["tokens"].long()] * D ** 0.5 * live[:, None]))
    qkv = R(x @ p["Wqkv"]).view(N, L, H + 2 * Hk, hd)
    angle = (b["positions"].to(F64)[:, None] * b["inv"].to(F64)).view(N, L, 1, hd // 2)

    def turn(m, w):
        n = m * (m.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * w
        lo, hi = n[..., :hd // 2], n[..., hd // 2:]
        return R(torch.cat([lo * angle.cos() - hi * angle.sin(), lo * angle.sin() + hi * angle.cos()], -1))
    q, k, v = turn(qkv[:, :, :H], p["qw"]), turn(qkv[:, :, H:H + Hk], p["kw"]), qkv[:, :, H + Hk:]
    k, v = (m.repeat_interleave(H // Hk, 2) for m in (k, v))
    t = torch.arange(L)
    off = t[:, None] - t[None, :]
    alive = live.view(N, 1, L)
    see = (off >= 0) & (off < (window or L)) & alive[:, :, None, :] & alive[:, :, :, None]
    z = (torch.einsum("nihd,njhd->nhij", q, k) * hd ** -0.5).masked_fill(~see, -1e30)
    o = R(torch.einsum("nhij,njhd->nihd", R(torch.softmax(z, -1) * see), v)).reshape(T, H * hd)
    h = R(x + R(o @ p["Wo"]))
    zl = h @ b["W"].to(F64)
    ok = b["loss_mask"].bool()
    tg = b["targets"].long()
    logp = torch.log_softmax(zl, -1).gather(1, tg[:, None]).squeeze(1) * ok
    s, S, cnt = oracle.seq_reduce(N, L, logp.detach().numpy(), b["behav"].numpy(), b["loss_mask"].numpy())
    ga = oracle.group_advantage(b["rewards"].numpy(), s, b["offsets"].numpy(), 2.0, 0)
    assert (ga["weight"] > 2).all() and (ga["clipped_w"] == 2).all()
    _, coef, _ = oracle.coef_loss(s, S, cnt, ga["weight"], ga["clipped_w"], ga["adv64"], 2.0, 0)
    row = torch.from_numpy(np.repeat(coef, L)) * ok
    dz = row[:, None] * (torch.softmax(zl, -1) - torch.nn.functional.one_hot(tg, V))
    dz = R(dz.detach())
    h.backward(dz @ b["W"].to(F64).T)
    return dict(logp=logp.detach(), W=(h.T @ dz).detach(), **{n: m.grad for n, m in p.items()})


@pytest.mark.parametrize("N,L,V,D,H,Hk,hd,window,side", [(8, 150, 1000, 256, 4, 2, 64, 0, "left"), (6, 131, 520, 128, 3, 1, 128, 40, "right")])
def test_step_against_64_bits(N, L, V, D, H, Hk, hd, window, side):
    size = (N, L, V, D, H, Hk, hd)
    b = _batch(*size, side)
    dev = {n: t.cuda() for n, t in b.items()}
    got = _library(dev, *size, window)
    exact, rounded = (_reference(b, *size, window, r) for r in (False, True))
    for name, want in exact.items():
        cost = float((rounded[name] - want).norm())
        off = float((got[name].cpu().to(F64) - want).norm())
        assert 0 < cost < 0.05 * float(want.norm()), name  # the comparison means something
        assert off <= 4 * cost, (name, off / cost)


def test_step_captured_and_replayed():
    size, window = (4, 100, 520, 128, 4, 2, 64), 0
    dev = {n: t.cuda() for n, t in _batch(*size, "left").items()}
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        _library(dev, *size, window)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        got = _library(dev, *size, window)
    g = torch.Generator(device="cuda").manual_seed(1)
    for _ in range(2):
        dev["tokens"].copy_(torch.randint(0, 520, dev["tokens"].shape, generator=g, device="cuda"))
        dev["E"].mul_(1.25)
        dev["targets"].copy_(dev["tokens"].roll(-1))
        graph.replay()
        want = _library(dev, *size, window)
        for name in want:
            assert torch.equal(got[name], want[name]), name
