"""Norms of query and key heads with rotation, and the gradient, on the GPU against the definition in 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu

from paper_2510_03515_b200 import binding as rb  # noqa: E402

BF, F32 = torch.bfloat16, torch.float32
U = 2.0 ** -24  # half an ulp of float


def _pairs(rot, flags):
    i = torch.arange(rot // 2)
    return (2 * i, 2 * i + 1) if flags & rb.QK_INTERLEAVED else (i, i + rot // 2)


def _turn(x, angle, rot, flags, sign=1.0):
    a, b = _pairs(rot, flags)
    y = x.clone()
    c, s = torch.cos(angle)[:, None], sign * torch.sin(angle)[:, None]
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., a] * s + x[..., b] * c
    return y


def _factor(w, flags):
    return None if flags & rb.QK_NO_NORM else w.double() + (1.0 if flags & rb.QK_UNIT_OFFSET else 0.0)


def forward64(x, w, angle, rot, flags, eps):
    x, w = x.double(), _factor(w, flags)
    if w is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + eps) * w
    return _turn(x, angle, rot, flags)


def backward64(x, w, dy, angle, rot, flags, eps):
    """dx, dw, and for each the sum of magnitudes that its rounding errors are relative to."""
    x, w, dn = x.double(), _factor(w, flags), _turn(dy.double(), angle, rot, flags, -1.0)
    size = _size(dn, rot, flags)
    if w is None:
        return dn, None, size, None
    rstd = torch.rsqrt(x.square().mean(-1, keepdim=True) + eps)
    xh = x * rstd
    wd = dn * w
    dx = rstd * (wd - xh * (wd * xh).mean(-1, keepdim=True))
    mag = rstd * (size * w.abs() + xh.abs() * (size * w.abs() * xh.abs()).mean(-1, keepdim=True))
    return dx, (dn * xh).sum((0, 1)), mag, (size * xh.abs()).sum((0, 1))


def _size(x, rot, flags):
    """For each element the length of its rotation pair (its own size where nothing rotates)."""
    a, b = _pairs(rot, flags)
    y = x.abs()
    y[..., a] = y[..., b] = torch.hypot(x[..., a], x[..., b])
    return y


CASES = [  # n_seq, seq_len, hq, hk, hd, rot, flags
    (1, 1, 1, 1, 16, 16, 0), (3, 7, 2, 1, 64, 64, 0), (2, 33, 12, 2, 128, 128, rb.QK_UNIT_OFFSET), (4, 5, 5, 3, 80, 32, rb.QK_INTERLEAVED),
    (2, 9, 3, 3, 256, 256, 0), (2, 50, 4, 2, 96, 48, rb.QK_UNIT_OFFSET | rb.QK_INTERLEAVED), (1, 300, 7, 1, 112, 112, rb.QK_NO_NORM),
    (5, 40, 4, 4, 64, 16, rb.QK_NO_NORM | rb.QK_INTERLEAVED), (40, 257, 3, 2, 48, 48, 0), (64, 1, 12, 2, 128, 128, 0),
]


def _make(n, length, hq, hk, hd, rot, dtype, seed, packed, positions, masked):
    g = torch.Generator().manual_seed(seed)
    T = n * length
    qkv = torch.randn(T, hq + 2 * hk, hd, generator=g).mul_(3).to(dtype)
    mask = (torch.rand(T, generator=g) < 0.8).to(torch.uint8) if masked else None
    if masked:
        qkv[mask == 0] = float("nan")
    qw, kw = 1 + 0.3 * torch.randn(hd, generator=g), 1 + 0.3 * torch.randn(hd, generator=g)
    inv = (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float()
    pos = torch.randint(0, 1 << 20, (T,), generator=g, dtype=torch.int32) if positions else None
    at = (pos if positions else torch.arange(length).repeat(n)).double()
    angle = at[:, None] * inv.double()
    q, k = qkv[:, :hq], qkv[:, hq:hq + hk]
    dev = qkv.cuda()
    dq_, dk_ = (dev[:, :hq], dev[:, hq:hq + hk]) if packed else (q.contiguous().cuda(), k.contiguous().cuda())
    return dict(q=q, k=k, mask=mask, qw=qw, kw=kw, inv=inv, pos=pos, angle=angle, g=g, live=torch.ones(T, dtype=torch.bool) if mask is None else mask != 0,
                gpu=[dq_, dk_, qw.cuda(), kw.cuda(), inv.cuda()], kw_gpu=dict(positions=None if pos is None else pos.cuda(), mask=None if mask is None else mask.cuda()))


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("packed,positions,masked", [(False, False, False), (True, True, True)])
@pytest.mark.parametrize("n,length,hq,hk,hd,rot,flags", CASES)
def test_forward(n, length, hq, hk, hd, rot, flags, packed, positions, masked, dtype):
    s = _make(n, length, hq, hk, hd, rot, dtype, 1, packed, positions, masked)
    got = rb.qk_norm_rope(*s["gpu"], n, length, eps=1e-5, flags=flags, **s["kw_gpu"])
    for y, x, w in zip(got, (s["q"], s["k"]), (s["qw"], s["kw"])):
        ref = torch.zeros(x.shape, dtype=torch.float64)
        m = s["live"]
        ref[m] = forward64(x[m], w, s["angle"][m], rot, flags, 1e-5)
        # float steps: a lane's 16 squares and up to 4 exchanges (half of 20 U through the root), mean, eps, root, quotient, two
        # products: 15 U; the angle's fraction rounded to float (1.6 U), sine and cosine 2 ulp (4 U), three operations of
        # the rotation: relative to the pair's length, below 32 U in all; then one rounding
        tol = 32 * U * _size(ref, rot, flags) + torch.finfo(dtype).eps / 2 * ref.abs()
        assert ((y.cpu().double() - ref).abs() <= tol).all()
        assert (y.cpu()[~m] == 0).all()


@pytest.mark.parametrize("dtype", [BF, F32])
@pytest.mark.parametrize("packed,positions,masked", [(False, False, False), (True, True, True)])
@pytest.mark.parametrize("n,length,hq,hk,hd,rot,flags", CASES)
def test_backward(n, length, hq, hk, hd, rot, flags, packed, positions, masked, dtype):
    s = _make(n, length, hq, hk, hd, rot, dtype, 2, packed, positions, masked)
    T = n * length
    dy = [torch.randn(T, h, hd, generator=s["g"]).to(dtype) for h in (hq, hk)]
    if masked:
        for d in dy:
            d[~s["live"]] = float("nan")
    grads = [d.cuda() for d in dy]
    extra = {}
    if packed:  # gradients of the slices of one projection
        row = torch.full((T, hq + 2 * hk, hd), 7.0, dtype=dtype, device="cuda")
        extra = dict(dq=row[:, :hq], dk=row[:, hq:hq + hk])
    r = rb.qk_norm_rope_grad(*s["gpu"], *grads, n, length, eps=1e-5, flags=flags, **s["kw_gpu"], **extra)
    if packed:
        assert (row[:, hq + hk:] == 7).all() and r.dq.data_ptr() == row.data_ptr()
    m = s["live"]
    for dx, dw, x, w, d, heads in ((r.dq, r.dq_weight, s["q"], s["qw"], dy[0], hq), (r.dk, r.dk_weight, s["k"], s["kw"], dy[1], hk)):
        rx, rw, mag, mass = backward64(x[m], w, d[m], s["angle"][m], rot, flags, 1e-5)
        # as in the forward pass, and the dot product's 20 additions: below 64 U of the magnitudes
        tol = 64 * U * mag + torch.finfo(dtype).eps / 2 * rx.abs()
        assert ((dx.cpu()[m].double() - rx).abs() <= tol).all()
        assert (dx.cpu()[~m] == 0).all()
        if rw is None:
            assert dw is None
        else:
            # each term 32 U; a sum of `terms` floats off by at most terms U of the sum of magnitudes
            assert ((dw.cpu().double() - rw).abs() <= (32 + min(T * heads, 4096)) * U * mass).all()
    again = rb.qk_norm_rope_grad(*s["gpu"], *grads, n, length, eps=1e-5, flags=flags, **s["kw_gpu"])
    for a, b in ((r.dq, again.dq), (r.dk, again.dk), (r.dq_weight, again.dq_weight), (r.dk_weight, again.dk_weight)):
        assert a is None or torch.equal(a, b)


@pytest.mark.parametrize("flags", [0, rb.QK_UNIT_OFFSET | rb.QK_INTERLEAVED, rb.QK_NO_NORM])
def test_gradient_against_differences(flags):
    n, length, hq, hk, hd, rot = 3, 11, 3, 2, 32, 16
    s = _make(n, length, hq, hk, hd, rot, F32, 3, False, True, False)
    dy = [torch.randn(n * length, h, hd, generator=s["g"]) for h in (hq, hk)]
    r = rb.qk_norm_rope_grad(*s["gpu"], *[d.cuda() for d in dy], n, length, eps=1e-5, flags=flags, **s["kw_gpu"])
    for x, w, d, dx, dw in ((s["q"], s["qw"], dy[0], r.dq, r.dq_weight), (s["k"], s["kw"], dy[1], r.dk, r.dk_weight)):
        vx, vw = torch.randn(x.shape, generator=s["g"]).double(), torch.randn(w.shape, generator=s["g"]).double()
        if flags & rb.QK_NO_NORM:
            vw = vw * 0

        def value(t):
            return (forward64(x.double() + t * vx, w.double() + t * vw, s["angle"], rot, flags, 1e-5) * d.double()).sum()
        h = 1e-5
        slope = (value(h) - value(-h)) / (2 * h)
        mine = (dx.cpu().double() * vx).sum() + (0 if dw is None else (dw.cpu().double() * vw).sum())
        # differences: h^2 of the third derivative, below 1e-6 here; floats: 1e-6 of the terms' magnitudes
        assert abs(slope - mine) <= 1e-5 * (dx.cpu().double() * vx).abs().sum()


def test_in_place():
    s = _make(2, 19, 4, 2, 64, 64, BF, 4, True, False, False)
    q, k, qw, kw, inv = s["gpu"]
    want = rb.qk_norm_rope(q, k, qw, kw, inv, 2, 19)
    row = q.stride(0)
    desc = rb.make_qk_desc(2, 19, 4, 2, 64, BF, ld_q=row, ld_k=row, ld_q_out=row, ld_k_out=row)
    rb.rapid_qk_norm_rope_fwd(desc, q, k, qw, kw, inv, None, None, q, k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    g = [torch.randn_like(x) for x in want]
    ref = rb.qk_norm_rope_grad(*[x.contiguous() for x in want], qw, kw, inv, *g, 2, 19)
    got = rb.qk_norm_rope_grad(*[x.contiguous() for x in want], qw, kw, inv, *g, 2, 19, dq=g[0], dk=g[1])
    assert got.dq.data_ptr() == g[0].data_ptr() and torch.equal(got.dq, ref.dq) and torch.equal(got.dk, ref.dk)


def test_far_position_equals_the_same_angle_nearby():
    """A frequency of exactly 2^-10 turns' worth cannot be had in float; but position p and frequency f give the angle of
    position 1 and frequency p f when that product is exact."""
    q = torch.randn(1, 1, 16, device="cuda")
    f = torch.tensor([2.0 ** -k for k in range(8)], device="cuda")
    a = rb.qk_norm_rope(q, q, None, None, f, 1, 1, positions=torch.tensor([3 << 20], dtype=torch.int32, device="cuda"), flags=rb.QK_NO_NORM)
    b = rb.qk_norm_rope(q, q, None, None, f * (3 << 20), 1, 1, positions=torch.tensor([1], dtype=torch.int32, device="cuda"), flags=rb.QK_NO_NORM)
    assert torch.equal(a[0], b[0])
