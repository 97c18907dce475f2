"""Timed cases of the policy-network operators around the loss: the token embedding and its gradient, the norms and
rotation of queries and keys and their gradient, and causal attention and its gradient.

`own = False` computes them in plain torch operations in 32 bits (angles in 64); `own = True` calls the library.

All of them work on the token grid of a mini-batch: `n_seq` generations of `seq_len` padded positions, row
r = n * seq_len + t, of which the first (or, padded on the left, the last) `len_n` are live, `len_n` uniform in
[len_lo, seq_len].
"""
import math

import numpy as np
import torch

own = False

_DT = {"f32": torch.float32, "bf16": torch.bfloat16}


# ---- the cases --------------------------------------------------------------------------------------------

def listed():
    return [
        # one decoding step: the last sampled token of each of 64 generations (latency counts)
        _embed("embed_fwd_step", "embed_fwd", 64, 1, 151936, 1536, len_lo=1, scale=math.sqrt(1536.0)),
        # the input of a training forward pass over one 64 x 1024 mini-batch
        _embed("embed_fwd_batch", "embed_fwd", 64, 1024, 151936, 1536, len_lo=256, scale=math.sqrt(1536.0)),
        # the embedding's gradient at the end of that mini-batch's backward pass
        _embed("embed_bwd_batch", "embed_bwd", 64, 1024, 151936, 1536, len_lo=256, scale=math.sqrt(1536.0)),
        # a float model with the smaller vocabulary, an odd width and an odd number of rows, every row live
        _embed("embed_bwd_odd", "embed_bwd", 15, 333, 32000, 1001, dtype="f32", len_lo=333, scale=1.0),
        # one decoding step far into the generations: one query and key row for each of 64 generations
        _qk("qk_fwd_step", "qk_fwd", 64, 1, 12, 2, 128, 128, len_lo=1, far=30000),
        # every layer of the training forward pass
        _qk("qk_fwd_batch", "qk_fwd", 64, 1024, 12, 2, 128, 128, len_lo=256, unit_offset=True),
        # every layer of the training backward pass
        _qk("qk_bwd_batch", "qk_bwd", 64, 1024, 12, 2, 128, 128, len_lo=256, unit_offset=True),
        # a float model with neighbouring pairs, a partial rotation and odd head counts
        _qk("qk_bwd_odd", "qk_bwd", 7, 211, 5, 1, 80, 32, dtype="f32", len_lo=100, far=1000, interleaved=True),
        # a layer's forward pass over the 64 x 256 mini-batch
        _attn("attn_fwd_short", "attn_fwd", 64, 256, 12, 2, 128, len_lo=256),
        # a layer's forward pass over long generations
        _attn("attn_fwd_long", "attn_fwd", 8, 4096, 16, 4, 64, len_lo=2867),
        # a layer's backward pass over the 64 x 1024 mini-batch with ragged lengths
        _attn("attn_bwd_batch", "attn_bwd", 64, 1024, 12, 2, 128, len_lo=256),
        # a local layer's backward pass over long, left-padded generations of an odd length
        _attn("attn_bwd_window", "attn_bwd", 3, 4095, 16, 8, 64, len_lo=2000, window=1024, left=True),
    ]


def draw(rng):
    kind = rng.choice(["embed_fwd", "embed_bwd", "qk_fwd", "qk_bwd", "attn_fwd", "attn_bwd"])

    def log_int(lo, hi):
        return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))

    seq_len = log_int(1, 4096)
    if kind.startswith("embed"):
        n_seq = log_int(1, max(1, 65536 // seq_len))
        return _embed(None, kind, n_seq, seq_len, log_int(1000, 151936), log_int(64, 1536), rng.choice(["bf16", "bf16", "f32"])
                      if n_seq * seq_len <= 16384 else "bf16", rng.randint(max(1, seq_len // 4), seq_len),
                      rng.choice([1.0, 0.5, 30.0]), rng.choice(["f32", "bf16"]))
    if kind.startswith("qk"):
        n_seq = log_int(1, max(1, 65536 // seq_len))
        hk = rng.choice([1, 2, 3, 4])
        hq = hk * rng.choice([1, 2, 3])
        hd = rng.choice([64, 80, 96, 128])
        return _qk(None, kind, n_seq, seq_len, hq, hk, hd, rng.choice([hd, hd, 32]),
                   rng.choice(["bf16", "bf16", "f32"]) if n_seq * seq_len <= 16384 else "bf16",
                   rng.randint(max(1, seq_len // 4), seq_len), rng.choice([0, 0, 1000, 100000]), rng.random() < 0.3, rng.random() < 0.3)
    hk = rng.choice([1, 2, 3, 4])
    hq = hk * rng.choice([1, 2, 3])
    most = 12 * 64 * 1024 * 1024 // (hq * seq_len * seq_len)
    n_seq = log_int(1, max(1, min(most, 65536 // seq_len)))
    return _attn(None, kind, n_seq, seq_len, hq, hk, rng.choice([64, 80, 128]), rng.randint(max(1, seq_len // 4), seq_len),
                 rng.choice([0, 0, log_int(1, seq_len)]), rng.random() < 0.4)


def _named(name, case):
    return case if name is None else {"name": name, **case}


def _embed(name, op, n_seq, seq_len, vocab, dim, dtype="bf16", len_lo=1, scale=1.0, grad="f32"):
    return _named(name, {"op": op, "n_seq": n_seq, "seq_len": seq_len, "vocab": vocab, "dim": dim, "dtype": dtype,
                         "len_lo": len_lo, "scale": scale, "grad": grad if dtype == "bf16" else "f32"})


def _qk(name, op, n_seq, seq_len, hq, hk, hd, rot, dtype="bf16", len_lo=1, far=0, interleaved=False, unit_offset=False):
    return _named(name, {"op": op, "n_seq": n_seq, "seq_len": seq_len, "hq": hq, "hk": hk, "hd": hd, "rot": rot, "dtype": dtype,
                         "len_lo": len_lo, "far": far, "interleaved": interleaved, "unit_offset": unit_offset})


def _attn(name, op, n_seq, seq_len, hq, hk, hd, len_lo=1, window=0, left=False):
    return _named(name, {"op": op, "n_seq": n_seq, "seq_len": seq_len, "hq": hq, "hk": hk, "hd": hd, "len_lo": len_lo,
                         "window": window, "left": left})


# ---- what a pass cannot do without ------------------------------------------------------------------------

def work(case):
    op, n_rows = case["op"], case["n_seq"] * case["seq_len"]
    lens = np.arange(case["len_lo"], case["seq_len"] + 1, dtype=np.float64)  # equally likely
    live = case["n_seq"] * float(lens.mean())
    size = 4 if case.get("dtype", "bf16") == "f32" else 2
    if op.startswith("embed"):
        # token = floor(exp(u ln(V + 1))) - 1: the expected number of different tokens among the live rows
        v = np.arange(1, case["vocab"] + 1, dtype=np.float64)
        p = np.log1p(1.0 / v) / math.log(case["vocab"] + 1.0)
        used = float(np.sum(-np.expm1(live * np.log1p(-np.minimum(p, 0.999999)))))
        index = 4 * live + n_rows
        if op == "embed_fwd":
            return {"bytes": index + case["dim"] * size * (used + n_rows), "flops": live * case["dim"]}
        grad = 4 if case["grad"] == "f32" else 2
        return {"bytes": index + case["dim"] * (size * live + grad * case["vocab"]), "flops": 2 * live * case["dim"]}
    if op.startswith("qk"):
        elems = (case["hq"] + case["hk"]) * case["hd"]
        if op == "qk_fwd":
            return {"bytes": n_rows + 4 * live + elems * size * (live + n_rows), "flops": 7 * live * elems}
        return {"bytes": n_rows + 4 * live + elems * size * (2 * live + n_rows), "flops": 16 * live * elems}
    # visible pairs of one generation of length len: each position sees itself and up to window - 1 before it
    w = np.minimum(lens, case["window"] or case["seq_len"])
    pairs = case["n_seq"] * case["hq"] * float(np.mean(w * (w + 1) / 2 + (lens - w) * w))
    rows_q, rows_k = case["hq"] * case["hd"] * 2, case["hk"] * case["hd"] * 2
    if op == "attn_fwd":
        return {"bytes": live * (rows_q + 2 * rows_k) + n_rows * (rows_q + 4 * case["hq"]), "flops": 4 * case["hd"] * pairs}
    return {"bytes": live * (3 * rows_q + 2 * rows_k + 4 * case["hq"]) + n_rows * (rows_q + 2 * rows_k), "flops": 10 * case["hd"] * pairs}


# ---- inputs -----------------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, n_seq, seq_len = case["op"], case["n_seq"], case["seq_len"]
    n_rows = n_seq * seq_len

    def normal(*shape, dtype=torch.float32, scale=1.0):
        return torch.randn(*shape, device="cuda", generator=g).mul_(scale).to(dtype)

    lens = torch.randint(case["len_lo"], seq_len + 1, (n_seq,), device="cuda", generator=g)
    t = torch.arange(seq_len, device="cuda")
    left = case.get("left", False)
    lo = seq_len - lens if left else torch.zeros_like(lens)
    hi = lo + lens
    live = ((t >= lo[:, None]) & (t < hi[:, None])).reshape(-1)
    s = {"case": case, "mask": live.to(torch.uint8)}
    if op.startswith("embed"):
        dt, vocab, dim = _DT[case["dtype"]], case["vocab"], case["dim"]
        u = torch.rand(n_rows, device="cuda", generator=g, dtype=torch.float64)
        s["tokens"] = (torch.exp(u * math.log(vocab + 1.0)).long() - 1).clamp_(0, vocab - 1).to(torch.int32)
        if op == "embed_fwd":
            s["table"] = _pitched(normal(vocab, dim, dtype=dt, scale=0.02))
        else:
            s["dout"] = _pitched(normal(n_rows, dim, dtype=dt, scale=1e-3))
        return s
    hq, hk, hd = case["hq"], case["hk"], case["hd"]
    dt = _DT[case.get("dtype", "bf16")]
    # one projection gives queries, keys and values side by side in a row
    qkv = normal(n_rows, hq + 2 * hk, hd, dtype=dt, scale=2.0 if op.startswith("qk") else 1.0)
    if op.startswith("qk"):
        s["q"], s["k"] = qkv[:, :hq], qkv[:, hq:hq + hk]
        near = 0.0 if case["unit_offset"] else 1.0
        s["q_weight"] = near + normal(hd, scale=0.1)
        s["k_weight"] = near + normal(hd, scale=0.1)
        s["inv_freq"] = (10000.0 ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64) / case["rot"])).float().cuda()
        start = torch.randint(0, case["far"] + 1, (n_seq,), device="cuda", generator=g)
        s["positions"] = (start[:, None] + t).reshape(-1).to(torch.int32)
        if op == "qk_bwd":
            s["dq_out"], s["dk_out"] = normal(n_rows, hq, hd, dtype=dt, scale=1e-2), normal(n_rows, hk, hd, dtype=dt, scale=1e-2)
        return s
    # queries and keys come out of the rotation in buffers of their own, values lie in the projection's rows
    s["q"], s["k"], s["v"] = qkv[:, :hq].contiguous(), qkv[:, hq:hq + hk].contiguous(), qkv[:, hq + hk:]
    s["bounds"] = torch.stack([lo, hi], 1).to(torch.int32).contiguous()
    if op == "attn_bwd":
        s["dout"] = normal(n_rows, hq, hd, dtype=dt, scale=1e-2)
        s["out"], s["lse"] = _attn_fwd(s)
    return s


def _pitched(x):
    """The same matrix with rows on 16-byte boundaries, as an allocator of parameters lays them out."""
    step = 16 // x.element_size()
    pitch = -(-x.shape[1] // step) * step
    if pitch == x.shape[1]:
        return x
    wide = torch.zeros(x.shape[0], pitch, dtype=x.dtype, device=x.device)
    wide[:, :x.shape[1]] = x
    return wide[:, :x.shape[1]]


# ---- one pass ---------------------------------------------------------------------------------------------

def run(state):
    c = state["case"]
    if own:
        return _own(state, c)
    return {"embed_fwd": _embed_fwd, "embed_bwd": _embed_bwd, "qk_fwd": _qk_fwd, "qk_bwd": _qk_bwd, "attn_fwd": _attn_fwd,
            "attn_bwd": _attn_bwd}[c["op"]](state)


def _own(s, c):
    from paper_2510_03515_b200 import binding as rb
    op = c["op"]
    if op == "embed_fwd":
        return rb.embedding(s["table"], s["tokens"], s["mask"], scale=c["scale"])
    if op == "embed_bwd":
        return rb.embedding_grad(s["dout"], s["tokens"], s["mask"], c["vocab"], scale=c["scale"], dtable_dtype=_DT[c["grad"]])
    if op.startswith("qk"):
        flags = (rb.QK_INTERLEAVED if c["interleaved"] else 0) | (rb.QK_UNIT_OFFSET if c["unit_offset"] else 0)
        if op == "qk_fwd":
            return rb.qk_norm_rope(s["q"], s["k"], s["q_weight"], s["k_weight"], s["inv_freq"], c["n_seq"], c["seq_len"],
                                   positions=s["positions"], mask=s["mask"], eps=1e-6, flags=flags)
        r = rb.qk_norm_rope_grad(s["q"], s["k"], s["q_weight"], s["k_weight"], s["inv_freq"], s["dq_out"], s["dk_out"], c["n_seq"],
                                 c["seq_len"], positions=s["positions"], mask=s["mask"], eps=1e-6, flags=flags)
        return r.dq, r.dk, r.dq_weight, r.dk_weight
    if op == "attn_fwd":
        return rb.attention(s["q"], s["k"], s["v"], c["n_seq"], c["seq_len"], bounds=s["bounds"], window=c["window"])
    # with one generation the plain forward pass leaves out head by head; a row's heads have to lie side by side
    r = rb.attention_grad(s["q"], s["k"], s["v"], s["out"].contiguous(), s["lse"], s["dout"], c["n_seq"], c["seq_len"], bounds=s["bounds"],
                          window=c["window"])
    return r.dq, r.dk, r.dv


# The plain forms.

def _embed_fwd(s):
    x = s["table"][s["tokens"].long()].float() * s["case"]["scale"]
    return torch.where(s["mask"].bool()[:, None], x, 0.0).to(s["table"].dtype)


def _embed_bwd(s):
    c = s["case"]
    x = torch.where(s["mask"].bool()[:, None], s["dout"].float(), 0.0)
    d = torch.zeros(c["vocab"], c["dim"], device=x.device).index_add_(0, s["tokens"].long(), x)
    return (d * c["scale"]).to(_DT[c["grad"]])


def _turn(s):
    """cos and sin of every row's angles, [T, 1, rot / 2]."""
    a = s["positions"].double()[:, None, None] * s["inv_freq"].double()
    return torch.cos(a).float(), torch.sin(a).float()


def _rotated(x, cos, sin, rot, interleaved):
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    pair = (a * cos - b * sin, a * sin + b * cos)
    y = torch.stack(pair, -1).flatten(-2) if interleaved else torch.cat(pair, -1)
    return torch.cat([y, x[..., rot:]], -1)


def _qk_fwd(s):
    c = s["case"]
    cos, sin = _turn(s)
    live = s["mask"].bool()[:, None, None]

    def one(x, w):
        x = x.float()
        w = w + 1.0 if c["unit_offset"] else w
        y = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * w
        return torch.where(live, _rotated(y, cos, sin, c["rot"], c["interleaved"]), 0.0).to(_DT[c["dtype"]])

    return one(s["q"], s["q_weight"]), one(s["k"], s["k_weight"])


def _qk_bwd(s):
    c = s["case"]
    cos, sin = _turn(s)
    live = s["mask"].bool()[:, None, None]

    def one(x, w, dy):
        x, dy = x.float(), torch.where(live, dy.float(), 0.0)
        w = w + 1.0 if c["unit_offset"] else w
        dn = _rotated(dy, cos, -sin, c["rot"], c["interleaved"])
        r = torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)
        xh = x * r
        dw = (dn * xh).double().sum((0, 1)).float()
        dh = dn * w
        dx = (dh - xh * (dh * xh).mean(-1, keepdim=True)) * r
        return dx.to(_DT[c["dtype"]]), dw

    dq, dqw = one(s["q"], s["q_weight"], s["dq_out"])
    dk, dkw = one(s["k"], s["k_weight"], s["dk_out"])
    return dq, dk, dqw, dkw


def _grid(x, c, heads):
    """[T, heads, hd] -> [N, hk, heads / hk, L, hd] in 32 bits."""
    hk = c["hk"]
    return x.float().reshape(c["n_seq"], c["seq_len"], hk, heads // hk, c["hd"]).permute(0, 2, 3, 1, 4)


def _rows(x):
    """The inverse: [N, hk, group, L, hd] -> [T, heads, hd]."""
    n, hk, group, length, hd = x.shape
    return x.permute(0, 3, 1, 2, 4).reshape(n * length, hk * group, hd)


def _visible(s):
    c = s["case"]
    t = torch.arange(c["seq_len"], device="cuda")
    see = t[:, None] >= t
    if c["window"]:
        see = see & (t[:, None] - t < c["window"])
    lo, hi = s["bounds"][:, 0, None], s["bounds"][:, 1, None]
    live = (t >= lo) & (t < hi)
    return (see & live[:, :, None] & live[:, None, :])[:, None, None], live


def _attn_fwd(s):
    c = s["case"]
    see, live = _visible(s)
    q, k, v = _grid(s["q"], c, c["hq"]), _grid(s["k"], c, c["hk"]), _grid(s["v"], c, c["hk"])
    z = (q @ k.transpose(-1, -2)).mul_(1.0 / math.sqrt(c["hd"])).masked_fill_(~see, -math.inf)
    m = z.amax(-1, keepdim=True).clamp_min_(-1e30)
    p = z.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.where(live[:, None, None, :, None], (p @ v) / total, 0.0)
    lse = (m + torch.log(total)).squeeze(-1).reshape(c["n_seq"], c["hq"], c["seq_len"])
    lse = torch.where(live[:, None], lse, -math.inf)
    return _rows(out).to(torch.bfloat16), lse


def _attn_bwd(s):
    c = s["case"]
    see, live = _visible(s)
    scale = 1.0 / math.sqrt(c["hd"])
    q, k, v = _grid(s["q"], c, c["hq"]), _grid(s["k"], c, c["hk"]), _grid(s["v"], c, c["hk"])
    rows = live[:, None, None, :, None]
    do, out = torch.where(rows, _grid(s["dout"], c, c["hq"]), 0.0), _grid(s["out"], c, c["hq"])
    lse = s["lse"].reshape(c["n_seq"], c["hk"], -1, c["seq_len"], 1).clamp_min(-1e30)
    p = (q @ k.transpose(-1, -2)).mul_(scale).sub_(lse).masked_fill_(~see, -math.inf).exp_()
    dv = (p.transpose(-1, -2) @ do).sum(2, keepdim=True)
    ds = (do @ v.transpose(-1, -2)).sub_((do * out).sum(-1, keepdim=True)).mul_(p).mul_(scale)
    dq, dk = ds @ k, (ds.transpose(-1, -2) @ q).sum(2, keepdim=True)
    return tuple(_rows(x).to(torch.bfloat16) for x in (dq, dk, dv))


# ---- the definitions in 64 bits ---------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    live = s["mask"] != 0
    if op == "embed_fwd":
        return s["table"].double().index_select(0, s["tokens"].long()) * case["scale"] * live.double().unsqueeze(1)
    if op == "embed_bwd":
        at = live.nonzero().squeeze(1)
        d = torch.zeros(case["vocab"], case["dim"], device="cuda", dtype=torch.float64)
        for part in at.split(8192):
            d.index_add_(0, s["tokens"][part].long(), s["dout"][part].double())
        return d.mul_(case["scale"])
    if op.startswith("qk"):
        return _exact_qk(case, s, live)
    return _exact_attn(case, s)


def _exact_qk(case, s, live):
    rot, hd = case["rot"], case["hd"]
    half = torch.arange(rot // 2, device="cuda")
    first, second = (2 * half, 2 * half + 1) if case["interleaved"] else (half, half + rot // 2)
    angle = s["positions"].double().unsqueeze(1) * s["inv_freq"].double().unsqueeze(0)
    z = torch.polar(torch.ones_like(angle), angle).unsqueeze(1)  # one complex factor for each pair
    add = 1.0 if case["unit_offset"] else 0.0

    def turned(x, by):
        y, w = x.clone(), torch.complex(x[..., first], x[..., second]) * by
        y[..., first], y[..., second] = w.real, w.imag
        return y

    results = []
    if case["op"] == "qk_fwd":
        for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
            x = x.double()
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / hd + 1e-6) * (w.double() + add)
            results.append(turned(x, z) * live.double()[:, None, None])
        return tuple(results)
    gains = []
    for x, w, dy in ((s["q"], s["q_weight"], s["dq_out"]), (s["k"], s["k_weight"], s["dk_out"])):
        x, dn = x.double(), turned(dy.double() * live.double()[:, None, None], z.conj())
        root = torch.sqrt((x * x).sum(-1, keepdim=True) / hd + 1e-6)
        gains.append((dn * x / root).sum((0, 1)))
        dn = dn * (w.double() + add)
        # d/dx of x / root: (I - x x^T / (hd root^2)) / root
        results.append(dn / root - x * (dn * x).sum(-1, keepdim=True) / (hd * root ** 3))
    return tuple(results + gains)


def _exact_attn(case, s):
    n_seq, length, hq, hk, hd = case["n_seq"], case["seq_len"], case["hq"], case["hk"], case["hd"]
    group, scale = hq // hk, hd ** -0.5
    q, k, v = (s[x].reshape(n_seq, length, -1, hd) for x in "qkv")
    fwd = case["op"] == "attn_fwd"
    out = torch.zeros(n_seq, length, hq, hd, device="cuda", dtype=torch.float64)
    lse = torch.full((n_seq, hq, length), -math.inf, device="cuda", dtype=torch.float64)
    dk, dv = (torch.zeros(n_seq, length, hk, hd, device="cuda", dtype=torch.float64) for _ in range(2))
    for n, (a, b) in enumerate(s["bounds"].tolist()):
        i = torch.arange(a, b, device="cuda")
        off = i.unsqueeze(1) - i.unsqueeze(0)
        see = (off >= 0) & (off < (case["window"] or length))
        for h in range(hq):
            qh, kh, vh = (x[n, a:b, j].double() for x, j in ((q, h), (k, h // group), (v, h // group)))
            z = (qh @ kh.T) * scale
            z[~see] = -math.inf
            if fwd:
                lse[n, h, a:b] = torch.logsumexp(z, 1)
                out[n, a:b, h] = torch.exp(z - lse[n, h, a:b].unsqueeze(1)) @ vh
                continue
            p = torch.exp(z - s["lse"][n, h, a:b].double().unsqueeze(1))
            do, o = (s[x].reshape(n_seq, length, hq, hd)[n, a:b, h].double() for x in ("dout", "out"))
            dz = p * (do @ vh.T - (do * o).sum(1, keepdim=True)) * scale
            out[n, a:b, h] = dz @ kh
            dk[n, a:b, h // group] += dz.T @ qh
            dv[n, a:b, h // group] += p.T @ do
    flat = lambda x: x.reshape(n_seq * length, -1, hd)  # noqa: E731
    return (flat(out), lse) if fwd else (flat(out), flat(dk), flat(dv))
