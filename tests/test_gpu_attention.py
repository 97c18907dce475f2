"""Causal attention and its gradient on the GPU against the definition in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2510_03515_b200 import binding as rb  # noqa: E402

BF = torch.bfloat16
B = 2.0 ** -8   # half an ulp of bf16, relative
U = 2.0 ** -24  # of float

# n_seq, seq_len, heads, kv_heads, head_dim, window, bounds ("full", "right", "left", "mixed" with empty generations)
CASES = [
    (1, 1, 1, 1, 64, 0, "full"), (3, 2, 2, 1, 128, 0, "full"), (2, 127, 3, 1, 64, 0, "right"), (2, 128, 4, 2, 128, 0, "left"),
    (2, 129, 4, 4, 64, 0, "mixed"), (1, 300, 6, 2, 128, 0, "full"), (5, 257, 2, 2, 80, 0, "mixed"), (2, 640, 5, 1, 40, 0, "right"),
    (1, 1000, 2, 1, 8, 0, "left"), (3, 515, 4, 2, 64, 1, "mixed"), (2, 500, 2, 1, 128, 100, "left"), (2, 700, 6, 2, 64, 128, "right"),
    (1, 900, 3, 3, 128, 257, "full"), (1, 2049, 2, 1, 128, 0, "right"), (7, 60, 12, 2, 120, 17, "mixed"), (1, 4100, 1, 1, 64, 1000, "left"),
]


def _bounds(n, length, kind, g):
    if kind == "full":
        return None
    lens = torch.randint(1, length + 1, (n,), generator=g)
    lo = torch.zeros(n, dtype=torch.long)
    if kind == "left":
        lo = length - lens
    elif kind == "mixed":
        lo = (torch.rand(n, generator=g) * (length - lens + 1)).long()
        lens[0] = 0
        if n > 2:
            lo[1], lens[1] = -5, length + 20  # clipped to the grid
    return torch.stack([lo, lo + lens], 1).to(torch.int32)


def _make(n, length, heads, kv, hd, kind, seed, peak=1.0, pitch=0):
    g = torch.Generator().manual_seed(seed)
    T = n * length
    row = (heads + 2 * kv) * hd
    wide = torch.randn(T, row + pitch, generator=g).to(BF)
    if pitch:
        wide[:, row:] = float("nan")
    x = wide[:, :row].reshape(T, heads + 2 * kv, hd) if not pitch else None
    bounds = _bounds(n, length, kind, g)
    live = torch.ones(n, length, dtype=torch.bool)
    if bounds is not None:
        t = torch.arange(length)
        live = (t >= bounds[:, :1].clamp(0, length)) & (t < bounds[:, 1:].clamp(0, length))
    wide[:, :heads * hd] *= peak
    wide[~live.reshape(-1)] = float("nan")  # what lies outside the bounds influences nothing
    wide[~live.reshape(-1), 0] = float("inf")
    dev = wide.cuda()

    def split(m):
        part = lambda a, b: m[:, a * hd:b * hd].unflatten(1, (b - a, hd))  # noqa: E731
        return part(0, heads), part(heads, heads + kv), part(heads + kv, heads + 2 * kv)
    return split(wide), split(dev), bounds, live, g


def _definition(q, k, v, n, length, window, live, scale):
    """Per (generation, head): positions, visible mask, q, k, v and scores in 64 bits."""
    heads, kv, hd = q.shape[1], k.shape[1], q.shape[2]
    for i in range(n):
        at = live[i].nonzero().squeeze(1)
        if not len(at):
            continue
        off = at[:, None] - at[None, :]
        see = (off >= 0) & (off < (window or length))
        r = i * length + at
        for h in range(heads):
            qh, kh, vh = q[r, h].double(), k[r, h * kv // heads].double(), v[r, h * kv // heads].double()
            z = (qh @ kh.T) * scale
            z[~see] = -math.inf
            yield i, h, at, r, see, qh, kh, vh, z


@pytest.mark.parametrize("n,length,heads,kv,hd,window,kind", CASES)
def test_forward(n, length, heads, kv, hd, window, kind):
    peak = 3.0 if length % 2 else 1.0
    (q, k, v), dev, bounds, live, _ = _make(n, length, heads, kv, hd, kind, 1, peak)
    scale = hd ** -0.5
    stats = rb.alloc_stats()
    out, lse = rb.attention(*dev, n, length, None if bounds is None else bounds.cuda(), window, stats=stats)
    assert rb.read_stats(stats)["status"] == 0
    out, lse = out.cpu(), lse.cpu()
    dead = ~live
    assert (out.reshape(n, length, heads, hd)[dead] == 0).all()
    assert (lse.transpose(1, 2)[dead] == -math.inf).all()
    for i, h, at, r, see, qh, kh, vh, z in _definition(q, k, v, n, length, window, live, scale):
        want = torch.logsumexp(z, 1)
        p = torch.exp(z - want[:, None])
        # scores: hd products summed in float, then scaled: relative to sum |q||k| scale
        ds = ((hd + 4) * U * scale * (qh.abs() @ kh.abs().T)).masked_fill(~see, 0).amax(1)
        # exponentials 2^-22, sums of up to `length` terms (in 64 + 64 steps a tile), logarithm, rounding of lse itself
        tol_lse = ds + 2.0 ** -21 + 200 * U + 4 * U * (want.abs() + ds + 12)
        assert ((lse[i, h, at].double() - want).abs() <= tol_lse).all()
        o = p @ vh
        # each probability is off by the score's error, 2^-21 and its rounding to bf16; then the output's own rounding
        tol = (p @ vh.abs()) * (B + 2 * ds[:, None] + 2.0 ** -19 + length * U) + o.abs() * B + 1e-30
        assert ((out[r, h].double() - o).abs() <= tol).all()


@pytest.mark.parametrize("n,length,heads,kv,hd", [(2, 200, 3, 1, 40), (2, 131, 2, 2, 128)])
def test_forward_pitches_and_scale(n, length, heads, kv, hd):
    """A pitch that is no multiple of a head, another scale, no lse."""
    (q, k, v), dev, bounds, live, _ = _make(n, length, heads, kv, hd, "right", 5, pitch=8)
    want, _ = rb.attention(*[x.contiguous() for x in dev], n, length, bounds.cuda(), scale=0.3)
    T = n * length
    out = torch.full((T, heads * hd + 24), 5.0, dtype=BF, device="cuda")
    row = dev[0].stride(0)
    d = rb.make_attn_desc(n, length, heads, kv, hd, 0, 0.3, row, row, row, heads * hd + 24)
    rb.rapid_attention_fwd(d, *dev, bounds.cuda(), out, None, None)
    assert torch.equal(out[:, :heads * hd].reshape(T, heads, hd), want) and (out[:, heads * hd:] == 5).all()


def _reference_grads(q, k, v, out, lse, dout, n, length, window, live, scale):
    """Gradients in 64 bits and, beside each, the bound on the kernel's error."""
    T, heads, hd = q.shape
    kv = k.shape[1]
    dq, tq = torch.zeros(2, T, heads, hd, dtype=torch.float64)
    dk, tk = torch.zeros(2, T, kv, hd, dtype=torch.float64)
    dv, tv = torch.zeros(2, T, kv, hd, dtype=torch.float64)
    for i, h, at, r, see, qh, kh, vh, z in _definition(q, k, v, n, length, window, live, scale):
        g = h * kv // heads
        do, o = dout[r, h].double(), out[r, h].double()
        p = torch.exp(z - lse[i, h, at].double()[:, None])
        dp, delta = do @ vh.T, (do * o).sum(1, keepdim=True)
        ds = p * (dp - delta)
        # relative error of p: the score's sum of hd products, lse and shift rounded in base 2, the exponential (2^-22)
        ep = (hd + 4) * U * scale * (qh.abs() @ kh.abs().T) + 4 * U * (z.abs().masked_fill(~see, 0) + lse[i, h, at].double().abs()[:, None]) + 2.0 ** -20
        # of dp - delta: sums of hd products each
        ed = (hd + 4) * U * (do.abs() @ vh.abs().T + (do * o).abs().sum(1, keepdim=True))
        es = (ds.abs() * (B + ep) + p * ed * (1 + ep)).masked_fill(~see, 0)  # and the rounding of ds to bf16
        pv = (p * (B + ep + length * U)).masked_fill(~see, 0)
        more = length * heads // kv * U  # the float sum of the product itself
        dq[r, h] = ds @ kh * scale
        tq[r, h] = (es + ds.abs() * more) @ kh.abs() * scale
        dk[r, g] += ds.T @ qh * scale
        tk[r, g] += (es + ds.abs() * more).T @ qh.abs() * scale
        dv[r, g] += p.T @ do
        tv[r, g] += (pv + p * more).T @ do.abs()
    return [(d, t + d.abs() * (B + 2 * U) + 1e-30) for d, t in ((dq, tq), (dk, tk), (dv, tv))]


def _backward_inputs(n, length, heads, kv, hd, window, kind, seed, peak=1.0, pitch=0):
    cpu, dev, bounds, live, g = _make(n, length, heads, kv, hd, kind, seed, peak, pitch)
    b = None if bounds is None else bounds.cuda()
    out, lse = rb.attention(*dev, n, length, b, window)
    dout = torch.randn(n * length, heads, hd, generator=g).to(BF)
    dead = ~live.reshape(-1)
    dout[dead] = float("nan")
    dev_out = out.clone()
    dev_out[dead.cuda()] = float("nan")  # not read either
    return cpu, dev, b, live, out, dev_out, lse, dout


@pytest.mark.parametrize("n,length,heads,kv,hd,window,kind", CASES)
def test_backward(n, length, heads, kv, hd, window, kind):
    peak = 3.0 if length % 2 else 1.0
    (q, k, v), dev, b, live, out, dev_out, lse, dout = _backward_inputs(n, length, heads, kv, hd, window, kind, 2, peak)
    stats = rb.alloc_stats()
    r = rb.attention_grad(*dev, dev_out, lse, dout.cuda(), n, length, b, window, stats=stats)
    assert rb.read_stats(stats)["status"] == 0
    want = _reference_grads(q, k, v, out.cpu(), lse.cpu(), dout, n, length, window, live, hd ** -0.5)
    dead = ~live.reshape(-1)
    for name, got, (ref, tol) in zip(("dv", "dk", "dq"), (r.dv, r.dk, r.dq), want[::-1]):
        got = got.cpu().double()
        assert (got[dead] == 0).all(), name
        assert ((got - ref).abs() <= tol).all(), (name, float(((got - ref).abs() / tol).max()))
    again = rb.attention_grad(*dev, dev_out, lse, dout.cuda(), n, length, b, window)
    assert torch.equal(r.dq, again.dq) and torch.equal(r.dk, again.dk) and torch.equal(r.dv, again.dv)


def test_backward_into_slices_of_one_projection():
    n, length, heads, kv, hd = 2, 150, 4, 2, 64
    (q, k, v), dev, b, live, out, dev_out, lse, dout = _backward_inputs(n, length, heads, kv, hd, 0, "right", 7, pitch=8)
    plain = rb.attention_grad(*[x.contiguous() for x in dev], out, lse, dout.cuda(), n, length, b)
    row = torch.full((n * length, heads + 2 * kv, hd), 3.0, dtype=BF, device="cuda")
    r = rb.attention_grad(*dev, out, lse, dout.cuda(), n, length, b, dq=row[:, :heads], dk=row[:, heads:heads + kv], dv=row[:, heads + kv:])
    assert r.dv.data_ptr() == row[:, heads + kv:].data_ptr()
    assert torch.equal(row, torch.cat([plain.dq, plain.dk, plain.dv], 1))


def test_gradient_against_differences():
    """The slope of sum(dout * out) along random directions, from 64-bit differences of the definition."""
    n, length, heads, kv, hd, window = 2, 90, 4, 2, 32, 30
    (q, k, v), dev, b, live, out, dev_out, lse, dout = _backward_inputs(n, length, heads, kv, hd, window, "left", 9)
    r = rb.attention_grad(*dev, dev_out, lse, dout.cuda(), n, length, b, window)
    g = torch.Generator().manual_seed(1)
    rows = live.reshape(-1)
    for which, got in enumerate((r.dq, r.dk, r.dv)):
        direction = torch.randn(got.shape, generator=g).double() * rows[:, None, None]

        def value(step):
            x = [t.double() for t in (q, k, v)]
            x[which] = x[which] + step * direction
            total = 0.0
            for i, h, at, rr, see, qh, kh, vh, z in _definition(*x, n, length, window, live, hd ** -0.5):
                total += float(((torch.softmax(z, 1) @ vh) * dout[rr, h].double()).sum())
            return total
        slope = (value(1e-4) - value(-1e-4)) / 2e-4
        mine = got.cpu().double() * direction
        # each element of the gradient is off by a few 2^-8 of its terms, independently: far inside 5 sigma of that
        size = float(mine.square().sum().sqrt())
        assert abs(slope - float(mine.sum())) <= 5 * 4 * B * size + 1e-5 * abs(slope)


def test_captured_and_replayed():
    n, length, heads, kv, hd = 2, 200, 4, 2, 64
    mk = lambda s: [x.contiguous() for x in _make(n, length, heads, kv, hd, "full", s)[1]]  # noqa: E731
    q, k, v = mk(1)
    dout = torch.randn_like(q)
    out, lse = torch.empty_like(q), torch.empty(n, heads, length, device="cuda")
    grads = [torch.empty_like(x) for x in (q, k, v)]
    desc = rb.make_attn_desc(n, length, heads, kv, hd)
    ws = torch.empty(rb.rapid_attention_bwd_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    stats = rb.alloc_stats()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rb.rapid_attention_fwd(desc, q, k, v, None, out, lse, stats)
        rb.rapid_attention_bwd(desc, q, k, v, None, out, lse, dout, *grads, stats, ws)
    for seed in (2, 3):
        for x, y in zip((q, k, v), mk(seed)):
            x.copy_(y)
        dout.normal_()
        graph.replay()
        o, l = rb.attention(q, k, v, n, length)
        r = rb.attention_grad(q, k, v, o, l, dout, n, length)
        assert torch.equal(o, out) and torch.equal(l, lse)
        assert all(torch.equal(a, b) for a, b in zip(grads, (r.dq, r.dk, r.dv)))
        assert rb.read_stats(stats)["status"] == 0


def test_two_streams_at_once():
    """Two calls in flight together, each with its own workspace."""
    n, length, heads, kv, hd = 3, 700, 6, 2, 128
    sets = []
    for seed in (1, 2):
        _, dev, b, _, out, dev_out, lse, dout = _backward_inputs(n, length, heads, kv, hd, 0, "right", seed)
        sets.append((dev, b, dev_out, lse, dout.cuda()))
    call = lambda s: rb.attention_grad(*s[0], s[2], s[3], s[4], n, length, s[1])  # noqa: E731
    want = [call(s) for s in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    got = [None, None]
    for _ in range(4):
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[i] = call(sets[i])
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a.dq, b.dq) and torch.equal(a.dk, b.dk) and torch.equal(a.dv, b.dv)


@pytest.mark.parametrize("hd", [64, 128])
def test_most_generations_empty(hd):
    """Long runs of tiles without a live row, between tiles that have some: every block works through many of both."""
    n, length, heads, kv, window = 300, 300, 2, 1, 70
    g = torch.Generator().manual_seed(4)
    qkv = torch.randn(n * length, heads + 2 * kv, hd, generator=g).to(BF)
    lo = torch.randint(0, length, (n,), generator=g)
    lens = torch.where(torch.rand(n, generator=g) < 0.1, torch.randint(1, length, (n,), generator=g), 0)
    bounds = torch.stack([lo, (lo + lens).clamp_max(length)], 1).to(torch.int32)
    t = torch.arange(length)
    live = (t >= bounds[:, :1]) & (t < bounds[:, 1:])
    split = lambda m: (m[:, :heads], m[:, heads:heads + kv], m[:, heads + kv:])  # noqa: E731
    (q, k, v), dev = split(qkv), split(qkv.cuda())
    stats = rb.alloc_stats()
    out, lse = rb.attention(*dev, n, length, bounds.cuda(), window, stats=stats)
    assert rb.read_stats(stats)["status"] == 0
    dout = torch.randn(n * length, heads, hd, generator=g).to(BF)
    r = rb.attention_grad(*dev, out, lse, dout.cuda(), n, length, bounds.cuda(), window, stats=stats)
    assert rb.read_stats(stats)["status"] == 0
    want = _reference_grads(q, k, v, out.cpu(), lse.cpu(), dout, n, length, window, live, hd ** -0.5)
    dead = ~live.reshape(-1)
    assert (out.cpu()[dead] == 0).all()
    for name, got, (ref, tol) in zip(("dq", "dk", "dv"), (r.dq, r.dk, r.dv), want):
        got = got.cpu().double()
        assert (got[dead] == 0).all(), name
        assert ((got - ref).abs() <= tol).all(), name


@pytest.mark.parametrize("window", [0, 2 ** 31 - 1])
def test_window_beyond_the_generation(window):
    q, k, v = _make(2, 300, 2, 1, 64, "full", 6)[1]
    want, lse = rb.attention(q, k, v, 2, 300, None, 300)
    out, l = rb.attention(q, k, v, 2, 300, None, window)
    assert torch.equal(out, want) and torch.equal(l, lse)
    dout = torch.randn_like(out)
    a, b = (rb.attention_grad(q, k, v, out, lse, dout, 2, 300, None, w) for w in (300, window))
    assert torch.equal(a.dq, b.dq) and torch.equal(a.dk, b.dk) and torch.equal(a.dv, b.dv)


# generations of at most 64 positions share tiles; the last tile may hold fewer of them
SHORT = [(17, 8, 4, 2, 128, 3, "mixed"), (40, 33, 3, 1, 64, 0, "mixed"), (9, 64, 2, 2, 80, 0, "left"), (300, 1, 3, 1, 128, 0, "full"),
         (129, 1, 2, 1, 64, 0, "mixed"), (3, 42, 6, 2, 128, 7, "right"), (256, 64, 2, 1, 64, 20, "mixed"), (5, 25, 1, 1, 8, 0, "full"),
         (2, 64, 4, 4, 128, 1, "right"), (63, 5, 9, 3, 128, 0, "left")]


@pytest.mark.parametrize("n,length,heads,kv,hd,window,kind", SHORT)
def test_short_generations(n, length, heads, kv, hd, window, kind):
    test_forward(n, length, heads, kv, hd, window, kind)
    test_backward(n, length, heads, kv, hd, window, kind)


def test_short_generations_do_not_influence_one_another():
    """Generations that share a tile give the same bits whatever their neighbours hold.  (Not the bits of the generation in a tile
    of its own: a key's place in the tile decides which partial sum its exponential goes to, and which form it takes.)"""
    n, length, heads, kv, hd = 11, 21, 4, 2, 64
    _, dev, b, _, out, _, lse, dout = _backward_inputs(n, length, heads, kv, hd, 0, "mixed", 8, pitch=8)
    dout = dout.cuda()
    r = rb.attention_grad(*dev, out, lse, dout, n, length, b)
    kept = [x.contiguous().view(n, length, -1, hd) for x in (*dev, dout)]
    other = [x.clone() for x in kept]
    b2 = b.clone()
    for x in other:
        x[1::2] = torch.randn_like(x[1::2]) * 30
        x[5] = float("nan")
    b2[1::2] = torch.tensor([2, length - 1], dtype=torch.int32, device="cuda")
    b2[5] = 0
    q, k, v, do = [x.view(n * length, -1, hd) for x in other]
    out2, lse2 = rb.attention(q, k, v, n, length, b2)
    r2 = rb.attention_grad(q, k, v, out2, lse2, do, n, length, b2)
    assert torch.equal(lse2[::2], lse[::2])
    for x, y in ((out, out2), (r.dq, r2.dq), (r.dk, r2.dk), (r.dv, r2.dv)):
        x, y = x.view(n, length, -1, hd), y.view(n, length, -1, hd)
        assert torch.equal(x[::2], y[::2]) and (y[5] == 0).all() and y.isfinite().all()
