"""The losses over the logits in 64 bits, and how far a kernel may be from them.

Tolerances, from the roundings (eps/2 relative each):
 * a row's log-sum-exp: every exponential is off by at most 1.5e-7 (hardware) and by the rounding of its argument (|x| 2^-24 ln 2 times
   its weight 2^-|x|: below 4e-8); a float partial sum has at most 16 additions of 2^-24 each: 1e-6 in all (LSE)
 * a probability: that, and the argument's rounding: |z| k and the constant both stay below 128 here, so 3 * 2^-18 ln 2 < 8e-6 (P)
   where an argument is formed from two large numbers (bf16); float logits have the row's largest taken off: |x| 2^-23 ln 2 < 6e-6
 * the result's own rounding, 2^-8 (bf16) or 2^-24 (float)
 * the factor of a row depends on its log-probability: |d factor / d lp| times LSE
"""
import math

import torch

LSE, P = 1e-6, 1e-5
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def grid(n_seq, seq_len, vocab, dtype, seed, pitch=None, std=3.0, boost=6.0, lens=None, device="cuda"):
    """Logits in rows of `pitch` columns (NaN behind the vocabulary and in masked rows), targets and mask."""
    g = torch.Generator().manual_seed(seed)
    T = n_seq * seq_len
    step = 16 // dtype.itemsize
    pitch = -(-vocab // step) * step if pitch is None else pitch
    z = torch.full((T, pitch), math.nan)
    z[:, :vocab] = torch.randn(T, vocab, generator=g) * std
    targets = torch.randint(0, vocab, (T,), generator=g, dtype=torch.int32)
    z[torch.arange(T), targets.long()] += boost
    mask = None
    if lens is not None:
        mask = (torch.arange(seq_len) < torch.tensor(lens)[:, None]).reshape(-1)
        z[~mask] = math.nan
        mask = mask.to(torch.uint8).to(device)
    return z.to(dtype).to(device)[:, :vocab], targets.to(device), mask, g


def rows_that_count(targets, mask, vocab):
    ok = (targets >= 0) & (targets < vocab)
    return ok if mask is None else ok & (mask != 0)


def _token_logp(z, targets, live):
    z = torch.where(live[:, None], z.double(), 0.0)
    lse = torch.logsumexp(z, 1)
    y = targets.long().clamp(0, z.shape[1] - 1)
    lp = torch.where(live, z.gather(1, y[:, None]).squeeze(1) - lse, 0.0)
    p = torch.exp(z - lse[:, None])
    return lp, p, torch.zeros_like(p).scatter_(1, y[:, None], 1.0)


def clip(z, targets, mask, old, adv, n_seq, ref=None, low=0.2, high=0.2, beta=0.0, scale=1.0, by_seq=False, norm=None):
    live = rows_that_count(targets, mask, z.shape[1])
    lp, p, hot = _token_logp(z, targets, live)
    T = z.shape[0]
    A = adv.double() if adv.numel() == T else adv.double().repeat_interleave(T // n_seq)
    rho = torch.exp(lp - old.double())
    u, v = rho * A, rho.clamp(1 - low, 1 + high) * A
    loss, slope = -torch.minimum(u, v), torch.where(v < u, 0.0, u)
    kl = torch.zeros_like(lp)
    if ref is not None:
        d = ref.double() - lp
        kl = torch.exp(d) - d - 1
        loss, slope = loss + beta * kl, slope + beta * (torch.exp(d) - 1)
    count = live.view(n_seq, -1).sum(1).clamp_min(1).double()
    if by_seq:
        w = (scale / ((norm or n_seq) * count)).repeat_interleave(T // n_seq)
    else:
        w = torch.full_like(lp, scale / (norm or max(1, int(live.sum()))))
    w = torch.where(live, w, 0.0)
    zero = torch.zeros_like(lp)
    g = torch.where(live, w * slope, zero)
    bend = w.abs() * (u.abs() + (beta * torch.exp(ref.double() - lp) if ref is not None else 0.0))  # slope of the factor by lp
    tol = (LSE * torch.where(live, bend, zero) + P * g.abs())[:, None] * (p + hot)
    n = max(1, int(live.sum()))
    mean = lambda x: float(torch.where(live, x, zero).sum()) / n  # noqa: E731
    return {"loss": float(torch.where(live, w * loss, zero).sum()), "loss_tol": float(torch.where(live, LSE * (w.abs() * slope.abs() + bend) + 1e-15, zero).sum()),
            "grad": g[:, None] * (p - hot), "grad_tol": tol, "token": lp, "token_tol": LSE, "live": live,
            "cut": int((live & (v < u)).sum()), "near": bool((live & ((rho - (1 - low)).abs() < 1e-4) | live & ((rho - (1 + high)).abs() < 1e-4)).any()),
            "mean_log_ratio": mean(lp - old.double()), "mean_kl": mean(kl)}


def preference(z, targets, mask, pairs, n_seq, ref=None, beta=0.1, margin=0.0, smoothing=0.0, kind="sigmoid", mean=False, scale=1.0, norm=None):
    live = rows_that_count(targets, mask, z.shape[1])
    lp, p, hot = _token_logp(z, targets, live)
    ratio = torch.where(live, lp - (0.0 if ref is None else ref.double()), 0.0).view(n_seq, -1)
    rows = live.view(n_seq, -1).sum(1).double()
    count = rows.clamp_min(1) if mean else torch.ones_like(rows)
    s = (ratio.sum(1) / count).detach().requires_grad_()
    ok = ((pairs >= 0) & (pairs < n_seq)).all(1)
    i, j = pairs.long().clamp(0, n_seq - 1).unbind(1)
    h = beta * (s[i] - s[j]) - margin
    ls = torch.nn.functional.logsigmoid
    f = {"sigmoid": lambda: -(1 - smoothing) * ls(h) - smoothing * ls(-h), "hinge": lambda: torch.relu(1 - h), "squared": lambda: (h - 0.5) ** 2}[kind]()
    Z = norm or max(1, int(ok.sum()))
    loss = scale * torch.where(ok, f, 0.0).sum() / Z
    ds = torch.autograd.grad(loss, s)[0]
    h, f = h.detach(), f.detach()
    coef = (-ds / count).repeat_interleave(z.shape[0] // n_seq) * live
    # h is off by beta times the rows' errors; the slope by at most that times the second derivative (1/4; 2; hinge: 0 off the corner)
    dh = 2 * beta * LSE * (1.0 if mean else float(rows.max()))
    steep = {"sigmoid": 1.0, "hinge": 1.0, "squared": 2 * float(torch.where(ok, (h - 0.5).abs(), 0.0).max())}[kind]
    bend = {"sigmoid": 0.25, "hinge": 0.0, "squared": 2.0}[kind]
    in_pairs = torch.zeros(n_seq, dtype=torch.float64, device=z.device).index_add_(0, i, ok.double()).index_add_(0, j, ok.double())
    dcoef = (in_pairs * abs(scale) * beta / Z * bend * dh / count).repeat_interleave(z.shape[0] // n_seq) * live
    return {"loss": float(loss.detach()), "loss_tol": abs(scale) * int(ok.sum()) / Z * steep * dh + 1e-15, "grad": coef[:, None] * (p - hot),
            "grad_tol": (dcoef + (P + LSE) * coef.abs())[:, None] * (p + hot), "token": lp, "token_tol": LSE, "live": live,
            "margins": torch.where(ok, h, math.nan), "margins_tol": dh, "valid": int(ok.sum()), "won": int((ok & (h > 0)).sum()),
            "near": bool((ok & ((h - 1).abs() < 10 * dh)).any()) if kind == "hinge" else bool((ok & (h.abs() < 10 * dh) & (i != j)).any())}


def distill(z, index, logit, mask=None, top_lse=None, tau=1.0, scale=1.0, norm=None):
    T, V = z.shape
    there = index >= 0
    t = torch.where(there, logit.double() / tau, -math.inf)
    some = there.any(1) if top_lse is not None else (t > -math.inf).any(1)
    key = torch.where(there, index, -1 - torch.arange(index.shape[1], device=z.device))  # no two places without an entry alike
    twice = (key.sort(1).values.diff(dim=1) == 0).any(1)
    wrong = twice | (there & ((index >= V) | ~(logit < math.inf))).any(1)
    if top_lse is not None:
        wrong |= ~torch.isfinite(top_lse)
    on = torch.ones(T, dtype=torch.bool, device=z.device) if mask is None else mask != 0
    live = on & some & ~wrong
    z = torch.where(live[:, None], z.double(), 0.0) / tau
    lse = torch.logsumexp(z, 1, keepdim=True)
    norm_t = top_lse.double()[:, None] if top_lse is not None else torch.logsumexp(torch.where(live[:, None], t, 0.0), 1, keepdim=True)
    lt = torch.where(there & live[:, None], t - norm_t, -math.inf)
    p = torch.exp(lt)
    # a column behind the last one takes the places without an entry
    at = torch.where(there & live[:, None], index.long().clamp(0, V - 1), V)
    wide = torch.cat([z, torch.zeros(T, 1, dtype=z.dtype, device=z.device)], 1)
    lq = wide.gather(1, at) - lse
    loss = torch.where(p > 0, p * (lt - lq), 0.0).sum(1)
    q = torch.exp(z - lse)
    hit = torch.zeros(T, V + 1, dtype=torch.bool, device=z.device).scatter_(1, at, True)[:, :V]
    full = torch.zeros(T, V + 1, dtype=z.dtype, device=z.device).scatter_(1, at, p)[:, :V]
    grown = torch.ones(T, dtype=z.dtype, device=z.device)
    spread = torch.zeros_like(grown)
    if top_lse is not None:
        p0 = 1 - p.sum(1)
        lq0 = torch.logsumexp(z.masked_fill(hit, -math.inf), 1) - lse.squeeze(1)
        loss = loss + torch.where(p0 > 0, p0 * (p0.clamp_min(1e-300).log() - lq0), 0.0)
        ratio = torch.where((p0 > 0) & (lq0 > -math.inf), torch.exp(p0.clamp_min(1e-300).log() - lq0), 0.0)
        grown, spread = 1 - ratio, ratio
    n = max(1, int(live.sum()))
    w = scale / (norm or n)
    grad = torch.where(hit, q - full, q * grown[:, None]) * (w / tau) * live[:, None]
    # a listed column: its probability's error; another: that, and the error of p0 / q0 (two log-sum-exps)
    tol = abs(w) / tau * torch.where(hit, (P + LSE) * q + 1e-12, q * (P * grown.abs() + 4 * LSE * spread)[:, None]) * live[:, None]
    loss = torch.where(live, loss, 0.0)
    return {"loss": float(w * loss.sum()), "loss_tol": abs(w) * LSE * 2 * n + 1e-15, "grad": grad, "grad_tol": tol, "token": loss,
            "token_tol": 2 * LSE, "live": live, "bad": int((on & wrong).sum())}


def check(want, got, stats, dtype, grad=True):
    """Compare a wrapper's result with a reference's; everything finite unless the reference is not."""
    token = got.token_logp if hasattr(got, "token_logp") else got.token_loss
    off = torch.where(token.double() == want["token"], 0.0, (token.double() - want["token"]).abs())  # equal infinities too
    assert torch.equal(token[~want["live"]], torch.zeros_like(token[~want["live"]]))
    assert bool((off <= want["token_tol"] + 2.0 ** -24 * want["token"].abs().clamp_max(1e30)).all()), f"rows: {float(off.max()):.3g}"
    assert float(got.loss) == want["loss"] or abs(float(got.loss) - want["loss"]) <= want["loss_tol"] + 2.0 ** -23 * abs(want["loss"]), (float(got.loss), want["loss"], want["loss_tol"])
    assert stats["status"] == 0 and stats["n_tokens"] == int(want["live"].sum())
    assert stats["loss"] == want["loss"] or abs(stats["loss"] - want["loss"]) <= want["loss_tol"] + 1e-12 * abs(want["loss"])
    if not grad:
        assert got.dlogits is None
        return
    d, ref = got.dlogits.double(), want["grad"]
    assert torch.equal(d[~want["live"]], torch.zeros_like(d[~want["live"]]))
    room = want["grad_tol"] + (HALF[dtype] + P) * ref.abs() + 2.0 ** -126
    assert bool(((d - ref).abs() <= room).all()), f"gradient: {float(((d - ref).abs() / room).max()):.3g} of its bound"
