"""Timed cases of the losses over logits beside the policy-gradient loss: the clipped policy loss with a KL term, the preference
loss over pairs of generations, and distillation from a teacher's top logits, each with its gradient by the logits.

`own = False` computes them in plain torch operations in 32 bits (sums over the vocabulary and everything of one value a row in 64);
`own = True` calls the library.

All of them work on the token grid of a mini-batch: `n_seq` generations of `seq_len` padded positions, row r = n * seq_len + t, of
which the first `len_n` are live, `len_n` uniform in [len_lo, seq_len].
"""
import math

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- the cases --------------------------------------------------------------------------------------------

def listed():
    return [
        # a debugging-size step of a float model: 32 generations of 8 tokens (latency counts)
        _clip("clip_step", 32, 8, 4096, "f32", len_lo=1, beta=0.04),
        # an inner step of group-relative training on 8 ragged generations, full vocabulary
        _clip("clip_batch", 8, 1024, 151936, len_lo=256, beta=0.04),
        # a float model with an odd vocabulary, an advantage for each token, every generation of equal weight
        _clip("clip_odd", 5, 333, 32001, "f32", len_lo=100, beta=0.0, per_token=True, by_seq=True),
        # the same loss watched on held-out rollouts: no gradient
        _clip("clip_eval", 16, 512, 32000, len_lo=128, beta=0.04, grad=False),
        # one pair of short answers (latency counts)
        _pref("pref_step", 2, 40, 32000, len_lo=20),
        # four pairs of long ragged answers, full vocabulary
        _pref("pref_batch", 8, 1024, 151936, len_lo=256),
        # every pair within groups of four answers to a prompt, squared form on token means
        _pref("pref_groups", 16, 200, 32000, len_lo=50, kind="squared", mean=True, all_pairs=True, beta=0.5),
        # a float model, no reference policy, hinge form
        _pref("pref_odd", 6, 129, 50001, "f32", len_lo=64, kind="hinge", mean=True, ref=False, beta=1.0),
        # the last 64 tokens of one answer with a teacher's 32 best logits for each
        _distill("distill_step", 1, 64, 151936, 32, len_lo=64),
        # a mini-batch with 64 entries a row and the rest of the teacher's mass in one bucket
        _distill("distill_batch", 8, 1024, 151936, 64, len_lo=256, tail=True),
        # a float model, soft targets, lists of different lengths
        _distill("distill_odd", 7, 211, 4099, 20, "f32", len_lo=100, tau=2.0, ragged=True),
        # a small vocabulary (bytes and merges of a specialised model), many rows
        _distill("distill_rows", 64, 1024, 4096, 8, len_lo=512, tail=True, tau=1.5),
    ]


_MOST = 8 * 1024 * 151936  # elements of the largest matrix of logits, bf16


def draw(rng):
    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))

    op = rng.choice(["clip", "pref", "distill"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    vocab = log_int(1000, 151936)
    seq_len = log_int(1, 2048)
    n_lo = 2 if op == "pref" else 1
    room = _MOST // (2 if dtype == "bf16" else 4) * 2 // (vocab * seq_len)
    n_seq = log_int(n_lo, max(n_lo, min(128, room)))
    len_lo = rng.randint(max(1, seq_len // 4), seq_len)
    grad = rng.random() < 0.8
    if op == "clip":
        return _clip(None, n_seq, seq_len, vocab, dtype, len_lo, rng.choice([0.0, 0.04, 0.2]), rng.random() < 0.3, rng.random() < 0.5, grad)
    if op == "pref":
        kind, mean = rng.choice(["sigmoid", "hinge", "squared"]), rng.random() < 0.5
        return _pref(None, n_seq, seq_len, vocab, dtype, len_lo, kind, mean, rng.random() < 0.7, rng.random() < 0.5,
                     1.0 if mean else 0.1, grad)
    return _distill(None, n_seq, seq_len, vocab, log_int(1, 128), dtype, len_lo, rng.choice([1.0, 1.0, 2.0, 0.7]), rng.random() < 0.5,
                    rng.random() < 0.3, grad)


def _named(name, case):
    return case if name is None else {"name": name, **case}


def _clip(name, n_seq, seq_len, vocab, dtype="bf16", len_lo=1, beta=0.0, per_token=False, by_seq=False, grad=True):
    return _named(name, {"op": "clip", "n_seq": n_seq, "seq_len": seq_len, "vocab": vocab, "dtype": dtype, "len_lo": len_lo, "beta": beta,
                         "per_token": per_token, "by_seq": by_seq, "grad": grad, "lo": 0.2, "hi": 0.28})


def _pref(name, n_seq, seq_len, vocab, dtype="bf16", len_lo=1, kind="sigmoid", mean=False, ref=True, all_pairs=False, beta=0.1, grad=True):
    return _named(name, {"op": "pref", "n_seq": n_seq, "seq_len": seq_len, "vocab": vocab, "dtype": dtype, "len_lo": len_lo, "kind": kind,
                         "mean": mean, "ref": ref, "all_pairs": all_pairs, "beta": beta, "grad": grad,
                         "smoothing": 0.1 if kind == "sigmoid" else 0.0, "margin": 0.0 if ref else 0.5})


def _distill(name, n_seq, seq_len, vocab, k, dtype="bf16", len_lo=1, tau=1.0, tail=False, ragged=False, grad=True):
    return _named(name, {"op": "distill", "n_seq": n_seq, "seq_len": seq_len, "vocab": vocab, "k": k, "dtype": dtype, "len_lo": len_lo,
                         "tau": tau, "tail": tail, "ragged": ragged, "grad": grad})


# ---- what a pass cannot do without ------------------------------------------------------------------------

def work(case):
    rows = case["n_seq"] * case["seq_len"]
    live = case["n_seq"] * (case["len_lo"] + case["seq_len"]) / 2  # each length equally likely
    size = 4 if case["dtype"] == "f32" else 2
    row = case["vocab"] * size
    few = {"clip": 16, "pref": 12, "distill": 4 + 8 * case.get("k", 0)}[case["op"]]
    # an element: the exponential's argument, the exponential, the sum; for the gradient argument, exponential, product
    return {"bytes": live * (row + few) + rows * (1 + 4) + (rows * row if case["grad"] else 0),
            "flops": live * case["vocab"] * (6 if case["grad"] else 3)}


# ---- inputs -----------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n_seq, seq_len, vocab = case["n_seq"], case["seq_len"], case["vocab"]
    rows = n_seq * seq_len

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, device="cuda", generator=g).mul_(scale)

    lens = torch.randint(case["len_lo"], seq_len + 1, (n_seq,), device="cuda", generator=g)
    live = (torch.arange(seq_len, device="cuda") < lens[:, None]).reshape(-1)
    s = {"case": case, "mask": live.to(torch.uint8), "logits": _matrix(rows, vocab, _DT[case["dtype"]])}
    if case["op"] == "distill":
        # one entry from each of k equal parts of the vocabulary, in the teacher's order
        k = min(case["k"], vocab)
        part = vocab // k
        index = torch.arange(k, device="cuda") * part + torch.randint(0, part, (rows, k), device="cuda", generator=g)
        index = index.gather(1, torch.rand(rows, k, device="cuda", generator=g).argsort(1))
        rank = torch.arange(1, k + 1, device="cuda", dtype=torch.float32)
        top = 14.0 - 1.5 * torch.log(rank) * (0.5 + torch.rand(rows, 1, device="cuda", generator=g)) + normal(rows, 1, scale=2.0)
        if case["tail"]:
            rest = torch.exp(torch.rand(rows, device="cuda", generator=g) * 6.0 - 6.5)  # mass beside the list's, 0.0015 to 0.6 of it
            s["top_lse"] = (torch.logsumexp(top.double() / case["tau"], 1) + torch.log1p(rest.double())).float()
        s["top_index"], s["top_logit"] = index.to(torch.int32), top
    else:
        s["targets"] = torch.randint(0, vocab, (rows,), device="cuda", generator=g, dtype=torch.int32)
    logp = torch.empty(rows, device="cuda")
    step = max(1, (1 << 28) // vocab)
    for a in range(0, rows, step):  # blocks of rows of the model's output
        b = min(rows, a + step)
        z = normal(b - a, vocab, scale=3.0)
        if case["op"] == "distill":
            at = s["top_index"][a:b].long()
            z.scatter_(1, at, s["top_logit"][a:b] - 2.0 + normal(b - a, at.shape[1]))
        else:
            z.scatter_add_(1, s["targets"][a:b, None].long(), torch.full((b - a, 1), 8.0, device="cuda"))
        s["logits"][a:b] = z
        if case["op"] != "distill":
            z = s["logits"][a:b].float()
            logp[a:b] = z.gather(1, s["targets"][a:b, None].long()).squeeze(1) - torch.logsumexp(z, 1)
    if case["op"] == "distill" and case["ragged"]:  # places behind a list's end hold -1
        count = torch.randint(0, k + 1, (rows, 1), device="cuda", generator=g)
        s["top_index"].masked_fill_(torch.arange(k, device="cuda") >= count, -1)
    if case["op"] == "clip":
        s["old_logp"] = logp + normal(rows, scale=0.25)
        s["ref_logp"] = logp + normal(rows, scale=0.4) if case["beta"] else None
        s["adv"] = normal(rows if case["per_token"] else n_seq)
    if case["op"] == "pref":
        s["ref_logp"] = logp + normal(rows, scale=0.3) if case["ref"] else None
        if case["all_pairs"]:  # within groups of four, the last one smaller
            pairs = [(i, j) for a in range(0, n_seq, 4) for i in range(a, min(a + 4, n_seq)) for j in range(i + 1, min(a + 4, n_seq))]
            s["pairs"] = torch.tensor(pairs or [(0, 1)], device="cuda", dtype=torch.int32)
        else:
            s["pairs"] = torch.randperm(n_seq, device="cuda", generator=g)[: n_seq // 2 * 2].view(-1, 2).to(torch.int32)
    return s


def _matrix(rows, cols, dtype):
    """[rows, cols] with rows on 16-byte boundaries, as a projection with a padded vocabulary leaves them."""
    step = 16 // dtype.itemsize
    return torch.zeros(rows, -(-cols // step) * step, dtype=dtype, device="cuda")[:, :cols]


# ---- one pass ---------------------------------------------------------------------------------------------

def run(state):
    c = state["case"]
    if own:
        return _own(state, c)
    return {"clip": _clip_plain, "pref": _pref_plain, "distill": _distill_plain}[c["op"]](state, c)


def _own(s, c):
    from paper_2510_03515_b200 import binding as rb
    if c["op"] == "clip":
        r = rb.clip_loss(s["logits"], s["targets"], s["mask"], s["old_logp"], s["adv"], c["n_seq"], c["seq_len"], ref_logp=s["ref_logp"],
                         eps_low=c["lo"], eps_high=c["hi"], kl_beta=c["beta"], flags=rb.LOSS_NORM_SEQ if c["by_seq"] else 0, want_grad=c["grad"])
        return _outputs(r.loss, r.dlogits, r.token_logp)
    if c["op"] == "pref":
        flags = {"sigmoid": 0, "hinge": rb.PREF_HINGE, "squared": rb.PREF_SQUARED}[c["kind"]] | (rb.PREF_TOKEN_MEAN if c["mean"] else 0)
        r = rb.preference_loss(s["logits"], s["targets"], s["mask"], s["pairs"], c["n_seq"], c["seq_len"], ref_logp=s["ref_logp"],
                               beta=c["beta"], margin=c["margin"], label_smoothing=c["smoothing"], flags=flags, want_grad=c["grad"])
        return _outputs(r.loss, r.dlogits, r.token_logp, r.margins)
    r = rb.distill_loss(s["logits"], s["top_index"], s["top_logit"], s["mask"], top_lse=s.get("top_lse"), temperature=c["tau"],
                        want_grad=c["grad"])
    return _outputs(r.loss, r.dlogits, r.token_loss)


def _outputs(loss, dlogits, by_token, margins=None):
    r = {"loss": loss, "by_token": by_token}
    if dlogits is not None:
        r["dlogits"] = dlogits
    if margins is not None:
        r["margins"] = margins
    return r


# The plain forms.

def _softmax(s, tau=1.0):
    """exp(z - max) in 32 bits, its sum and the log-sum-exp in 64."""
    z = s["logits"].float()
    m = z.amax(1, keepdim=True)
    e = (z - m).mul_(1.0 / tau).exp_()
    total = e.sum(1, keepdim=True, dtype=torch.float64)
    return z, e, total, m.double() / tau + total.log()


def _token_logp(s, z, lse):
    y = s["targets"].long()[:, None]
    return torch.where(s["mask"].bool(), (z.gather(1, y).double() - lse).squeeze(1), 0.0)


def _dlogits(s, e, total, coef):
    """coef * (softmax - one at the token), in the logits' type."""
    live = s["mask"].bool()
    coef = torch.where(live, coef, 0.0).float()[:, None]
    p = e.div_(total.float())
    p.scatter_add_(1, s["targets"].long()[:, None], torch.full_like(coef, -1.0))
    return p.mul_(coef).to(s["logits"].dtype)


def _clip_plain(s, c):
    z, e, total, lse = _softmax(s)
    live = s["mask"].bool()
    lp = _token_logp(s, z, lse)
    del z
    adv = s["adv"].double() if c["per_token"] else s["adv"].double().repeat_interleave(c["seq_len"])
    rho = (lp - s["old_logp"].double()).exp()
    cut = rho.clamp(1.0 - c["lo"], 1.0 + c["hi"])
    loss = -torch.minimum(rho * adv, cut * adv)
    slope = torch.where(rho * adv <= cut * adv, rho * adv, 0.0)
    if c["beta"]:
        d = s["ref_logp"].double() - lp
        loss = loss + c["beta"] * (torch.expm1(d) - d)
        slope = slope + c["beta"] * torch.expm1(d)
    if c["by_seq"]:
        count = live.view(c["n_seq"], -1).sum(1, keepdim=True).clamp_min(1).double()
        w = (1.0 / (count * c["n_seq"])).expand(-1, c["seq_len"]).reshape(-1)
    else:
        w = 1.0 / live.sum().double()
    total_loss = torch.where(live, w * loss, 0.0).sum().float().reshape(1)
    return _outputs(total_loss, _dlogits(s, e, total, w * slope) if c["grad"] else None, lp.float())


def _pref_plain(s, c):
    z, e, total, lse = _softmax(s)
    live = s["mask"].bool()
    lp = _token_logp(s, z, lse)
    del z
    ratio = lp if s["ref_logp"] is None else torch.where(live, lp - s["ref_logp"].double(), 0.0)
    each = ratio.view(c["n_seq"], -1).sum(1)
    count = live.view(c["n_seq"], -1).sum(1).clamp_min(1).double() if c["mean"] else torch.ones_like(each)
    each = each / count
    i, j = s["pairs"].long().unbind(1)
    h = c["beta"] * (each[i] - each[j]) - c["margin"]
    if c["kind"] == "sigmoid":
        eps = c["smoothing"]
        loss = (1 - eps) * torch.log1p(torch.exp(-h.abs())) + (1 - eps) * (-h).clamp_min(0) + eps * torch.log1p(torch.exp(-h.abs())) + eps * h.clamp_min(0)
        slope = 1.0 / (1.0 + torch.exp(-h)) - (1 - eps)
    elif c["kind"] == "hinge":
        loss = (1.0 - h).clamp_min(0)
        slope = torch.where(h < 1.0, -1.0, 0.0).double()
    else:
        loss = (h - 0.5).square()
        slope = 2.0 * (h - 0.5)
    slope = slope * c["beta"] / h.numel()
    ds = torch.zeros_like(each).index_add_(0, i, slope).index_add_(0, j, -slope) / count
    coef = (-ds)[:, None].expand(-1, c["seq_len"]).reshape(-1)
    return _outputs(loss.mean().float().reshape(1), _dlogits(s, e, total, coef) if c["grad"] else None, lp.float(), h.float())


def _distill_plain(s, c):
    tau = c["tau"]
    z, e, total, lse = _softmax(s, tau)
    on = s["top_index"] >= 0
    live = s["mask"].bool() & on.any(1)
    # places without an entry repeat the first one, with no mass of their own
    at = torch.where(on, s["top_index"].long(), s["top_index"][:, :1].long().clamp_min(0))
    t = torch.where(on, s["top_logit"].double() / tau, -math.inf)
    teacher = s["top_lse"].double()[:, None] if c["tail"] else torch.logsumexp(t, 1, keepdim=True)
    p = torch.where(on, (t - teacher).exp(), 0.0)
    logq = z.gather(1, at).double() / tau - lse
    del z
    loss = torch.where(on, p * (t - teacher - logq), 0.0).sum(1)
    grown = None
    if c["tail"]:
        e.scatter_(1, at, 0.0)
        q0 = e.sum(1, dtype=torch.float64) / total.squeeze(1)
        p0 = (1.0 - p.sum(1)).clamp_min(0.0)
        loss = loss + torch.where(p0 > 0, p0 * (p0.log() - q0.log()), 0.0)
        grown = torch.where(p0 > 0, 1.0 - p0 / q0, 1.0)[:, None]
    w = 1.0 / live.sum().clamp_min(1).double()
    loss = torch.where(live, loss, 0.0)
    grad = None
    if c["grad"]:
        q = e.div_(total.float())
        if grown is not None:
            q.mul_(grown.float())
        first = (logq.exp() - p)
        q.scatter_(1, at, torch.where(on, first, first[:, :1]).float())
        grad = q.mul_(torch.where(live, w / tau, 0.0).float()[:, None]).to(s["logits"].dtype)
    return _outputs((w * loss.sum()).float().reshape(1), grad, loss.float())


# ---- the definitions in 64 bits ---------------------------------------------------------------------------

def exact(case, seed):
    """Losses written out for one generation at a time and differentiated by autograd."""
    s = prepare(case, seed)
    live = (s["mask"] != 0).reshape(case["n_seq"], case["seq_len"])
    grads = torch.zeros(case["n_seq"], case["seq_len"], case["vocab"], dtype=torch.float64, device="cuda") if case["grad"] else None
    by_token = torch.zeros(case["n_seq"], case["seq_len"], dtype=torch.float64, device="cuda")
    total = torch.zeros((), dtype=torch.float64, device="cuda")
    rows = lambda x, n: x.reshape(case["n_seq"], case["seq_len"], *x.shape[1:])[n][live[n]]  # noqa: E731

    def logits(n):
        a = n * case["seq_len"]
        return s["logits"][a:a + case["seq_len"]][live[n]].double().requires_grad_(case["grad"])

    def chosen(z, n):
        return torch.log_softmax(z, 1).gather(1, rows(s["targets"], n).long().unsqueeze(1)).squeeze(1)

    def back(value, z, n):
        if case["grad"] and value.requires_grad:
            grads[n, live[n]] = torch.autograd.grad(value, z)[0]

    if case["op"] == "pref":
        weight, sums = torch.zeros(case["n_seq"], dtype=torch.float64, device="cuda"), []
        for n in range(case["n_seq"]):
            with torch.no_grad():
                lp = chosen(logits(n), n)
            by_token[n, live[n]] = lp
            weight[n] = 1.0 / lp.numel() if case["mean"] else 1.0
            sums.append((lp - (rows(s["ref_logp"], n).double() if case["ref"] else 0.0)).sum() * weight[n])
        sums = torch.stack(sums).requires_grad_()
        a, b = s["pairs"][:, 0].long(), s["pairs"][:, 1].long()
        h = case["beta"] * (sums[a] - sums[b]) - case["margin"]
        ls = torch.nn.functional.logsigmoid
        losses = {"sigmoid": lambda: -(1 - case["smoothing"]) * ls(h) - case["smoothing"] * ls(-h), "hinge": lambda: torch.relu(1 - h),
                  "squared": lambda: (h - 0.5) ** 2}[case["kind"]]()
        pull = torch.autograd.grad(losses.mean(), sums)[0]
        for n in range(case["n_seq"] if case["grad"] else 0):
            z = logits(n)
            back(chosen(z, n).sum() * (pull[n] * weight[n]), z, n)
        return _exact_outputs(losses.mean().detach(), by_token, grads, h.detach())

    if case["op"] == "clip":
        for n in range(case["n_seq"]):
            z = logits(n)
            lp = chosen(z, n)
            adv = rows(s["adv"], n).double() if case["per_token"] else s["adv"][n].double()
            rho = torch.exp(lp - rows(s["old_logp"], n).double())
            each = -torch.minimum(rho * adv, torch.clamp(rho, 1 - case["lo"], 1 + case["hi"]) * adv)
            if case["beta"]:
                off = rows(s["ref_logp"], n).double() - lp
                each = each + case["beta"] * (torch.exp(off) - off - 1)
            value = each.mean() / case["n_seq"] if case["by_seq"] else each.sum() / live.sum()
            by_token[n, live[n]] = lp.detach()
            total += value.detach()
            back(value, z, n)
        return _exact_outputs(total, by_token, grads)

    listed_rows = (live & (s["top_index"] >= 0).any(1).reshape(live.shape)).sum()
    for n in range(case["n_seq"]):
        z = logits(n)
        index, top = rows(s["top_index"], n).long(), rows(s["top_logit"], n).double() / case["tau"]
        there = index >= 0
        some = there.any(1)
        if not bool(some.any()):
            continue
        top = top.masked_fill(~there, -math.inf)
        norm = rows(s["top_lse"], n).double().unsqueeze(1) if case["tail"] else torch.logsumexp(top.masked_fill(~some.unsqueeze(1), 0.0), 1, keepdim=True)
        logp = (top - norm).masked_fill(~there, 0.0)
        p = logp.exp() * there
        # a column behind the last one takes the places without an entry
        full = torch.zeros(z.shape[0], case["vocab"] + 1, dtype=torch.bool, device="cuda")
        full.scatter_(1, index.masked_fill(~there, case["vocab"]), True)
        logq = torch.log_softmax(z / case["tau"], 1)
        each = (p * (logp - logq.gather(1, index.clamp_min(0)))).sum(1)
        if case["tail"]:
            p0 = 1.0 - p.sum(1)
            q0 = torch.logsumexp(logq.masked_fill(full[:, :-1], -math.inf), 1)
            each = each + torch.where(p0 > 0, p0 * (p0.clamp_min(1e-300).log() - q0), 0.0)
        each = torch.where(some, each, 0.0)
        by_token[n, live[n]] = each.detach()
        value = each.sum() / listed_rows
        total += value.detach()
        back(value, z, n)
    return _exact_outputs(total, by_token, grads)


def _exact_outputs(loss, by_token, grads, margins=None):
    r = {"loss": loss.reshape(1), "by_token": by_token.reshape(-1)}
    if grads is not None:
        r["dlogits"] = grads.reshape(-1, grads.shape[-1])
    if margins is not None:
        r["margins"] = margins
    return r
