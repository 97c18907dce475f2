"""Policy-network operators, host side: bad descriptors, pointers, pitches and workspaces are refused before anything is
enqueued (no GPU needed: a call that passes every check stops at the missing device)."""
import ctypes as C
import math

import pytest
import torch

from paper_2510_03515_b200 import binding as rb

FAKE = 0x10000  # an aligned non-NULL address that nothing dereferences
FAR = 1 << 40   # distance between the fake arrays
BF, F32 = torch.bfloat16, torch.float32
INVALID, ALIGN, UNSUP, WORK = (rb.RAPID_ERR_INVALID_ARG, rb.RAPID_ERR_ALIGNMENT, rb.RAPID_ERR_UNSUPPORTED, rb.RAPID_ERR_WORKSPACE)
# what a call that passes every check returns here: no device, or (on a GPU machine) not run at all
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="fake pointers must not reach a device")


def _args(names, **over):
    base = {n: FAKE + i * FAR for i, n in enumerate(names)}
    base.update(over)
    return [base[n] for n in names]


def test_struct_sizes():
    assert C.sizeof(rb.EmbedDesc) == 48 and rb.EmbedDesc.scale.offset == 40
    assert C.sizeof(rb.AttnDesc) == 104 and rb.AttnDesc.ld_q.offset == 24 and rb.AttnDesc.scale.offset == 96
    assert C.sizeof(rb.QkDesc) == 88 and rb.QkDesc.ld_q.offset == 24 and rb.QkDesc.eps.offset == 80


# ---- embedding ------------------------------------------------------------------------------------------------

def _embed_fwd(d, **over):
    a = _args(["tokens", "mask", "table", "out"], **over)
    return rb.lib().rapid_embedding_fwd(C.byref(d), *a, None, None)


def _embed_bwd(d, ws=FAKE, ws_bytes=1 << 50, **over):
    a = _args(["tokens", "mask", "dout", "dtable"], **over)
    return rb.lib().rapid_embedding_bwd(C.byref(d), *a, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [_embed_fwd, _embed_bwd])
def test_embedding_refusals(call):
    def d(n=8, v=100, dim=16, dtype=BF, **kw):
        return rb.make_embed_desc(n, v, dim, dtype, **kw)
    assert call(d(n=0)) == INVALID and call(d(v=0)) == INVALID and call(d(dim=0)) == INVALID
    assert call(d(ld_table=8)) == INVALID and call(d(ld_rows=15)) == INVALID
    assert call(d(scale=math.inf)) == INVALID and call(d(scale=math.nan)) == INVALID
    assert call(d(flags=8)) == INVALID
    assert call(d(dtype=F32, flags=rb.EMBED_DTABLE_BF16)) == INVALID
    assert call(d(ld_rows=20)) == ALIGN and call(d(dim=15, ld_rows=16)) == ALIGN
    assert call(d(n=1 << 31)) == UNSUP and call(d(v=(1 << 27) - 1)) == UNSUP
    assert call(d(), tokens=None) == INVALID and call(d(), tokens=FAKE + 2) == ALIGN
    bad = d()
    bad.dtype = 7
    assert call(bad) == INVALID
    bad = d()
    bad.reserved = 1
    assert call(bad) == INVALID
    rows, table = ("out", "table") if call is _embed_fwd else ("dout", "dtable")
    for name in (rows, table):
        assert call(d(), **{name: None}) == INVALID
        assert call(d(), **{name: FAKE + 8}) == ALIGN
    assert call(d(), **{rows: FAKE + 64, table: FAKE}) == INVALID  # the two overlap
    assert rb.lib().rapid_embedding_fwd(None, FAKE, None, FAKE, FAKE, None, None) == INVALID


def test_embedding_workspace():
    d = rb.make_embed_desc(1000, 50, 24, BF)
    n = rb.rapid_embedding_bwd_workspace_bytes(d)
    assert 16 * 1000 + 1000 // 32 * 24 * 4 <= n <= 32 * 1000 + 4 * 51 + 1000 // 32 * 24 * 4 + (1 << 18)
    assert _embed_bwd(d, ws=None) == WORK and _embed_bwd(d, ws=FAKE + 16) == WORK and _embed_bwd(d, ws_bytes=n - 1) == WORK
    assert rb.lib().rapid_embedding_bwd_workspace_bytes(C.byref(d), None) == INVALID


@no_gpu
def test_embedding_without_a_device():
    d = rb.make_embed_desc(1000, 50, 24, BF)
    assert _embed_fwd(d) == rb.RAPID_ERR_CUDA and _embed_bwd(d) == rb.RAPID_ERR_CUDA


# ---- query/key norm and rotation --------------------------------------------------------------------------------

def _qk_fwd(d, **over):
    a = _args(["q", "k", "qw", "kw", "freq", "pos", "mask", "q_out", "k_out"], **over)
    return rb.lib().rapid_qk_norm_rope_fwd(C.byref(d), *a, None)


def _qk_bwd(d, ws=FAKE, ws_bytes=1 << 50, **over):
    a = _args(["q", "k", "qw", "kw", "freq", "pos", "mask", "dq_out", "dk_out", "dq", "dk", "dqw", "dkw"], **over)
    return rb.lib().rapid_qk_norm_rope_bwd(C.byref(d), *a, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [_qk_fwd, _qk_bwd])
def test_qk_refusals(call):
    def d(n=4, length=8, hq=4, hk=2, hd=64, dtype=BF, **kw):
        return rb.make_qk_desc(n, length, hq, hk, hd, dtype, **kw)
    for kw in (dict(n=0), dict(length=0), dict(hq=0), dict(hk=0), dict(hd=0), dict(rot_dim=0), dict(rot_dim=80), dict(eps=-1.0),
               dict(eps=math.nan), dict(flags=8), dict(ld_q=255), dict(ld_k=64), dict(ld_q_out=248), dict(ld_k_out=120)):
        assert call(d(**kw)) == INVALID, kw
    for kw in (dict(hd=24, rot_dim=16), dict(hd=272), dict(rot_dim=24), dict(n=1 << 20, length=1 << 12)):
        assert call(d(**kw)) == UNSUP, kw
    for kw in (dict(ld_q=260), dict(ld_k_out=132), dict(ld_q=258, dtype=F32)):
        assert call(d(**kw)) == ALIGN, kw
    ins = ["q", "k", "freq"] + (["q_out", "k_out"] if call is _qk_fwd else ["dq_out", "dk_out", "dq", "dk"])
    for name in ins + ["qw", "kw"] + ([] if call is _qk_fwd else ["dqw", "dkw"]):
        assert call(d(), **{name: None}) == INVALID, name
    for name in ins:
        if name != "freq":
            assert call(d(), **{name: FAKE + FAR // 2 + 8}) == ALIGN, name
    if call is _qk_bwd:
        assert call(d(ld_dq=250)) == INVALID and call(d(ld_dk=132)) == ALIGN
        assert call(d(), ws=None) == WORK and call(d(), ws=FAKE + 8) == WORK and call(d(), ws_bytes=1000) == WORK
    # outputs on one another or on another input
    first, second = ("q_out", "k_out") if call is _qk_fwd else ("dq", "dk")
    assert call(d(), **{first: FAKE + 100 * FAR, second: FAKE + 100 * FAR + 512}) == INVALID
    assert call(d(), **{second: FAKE}) == INVALID
    # half a head further on in the same rows
    assert call(d(), **{first: FAKE + 64}) == INVALID


@no_gpu
def test_qk_slices_of_one_projection_are_accepted():
    """Queries, keys and values side by side in a row; outputs in place, or in rows of a packed gradient."""
    row = (4 + 2 + 2) * 64
    d = rb.make_qk_desc(4, 8, 4, 2, 64, BF, ld_q=row, ld_k=row, ld_q_out=row, ld_k_out=row, ld_dq=row, ld_dk=row)
    keys = FAKE + 4 * 64 * 2
    assert _qk_fwd(d, k=keys, q_out=FAKE, k_out=keys) == rb.RAPID_ERR_CUDA
    grads = FAKE + 50 * FAR
    assert _qk_bwd(d, k=keys, dq_out=grads, dk_out=grads + 512, dq=grads, dk=grads + 512) == rb.RAPID_ERR_CUDA
    d2 = rb.make_qk_desc(4, 8, 4, 2, 64, BF, flags=rb.QK_NO_NORM)
    assert _qk_bwd(d2, ws=None, ws_bytes=0, qw=None, kw=None, dqw=None, dkw=None) == rb.RAPID_ERR_CUDA


# ---- attention ----------------------------------------------------------------------------------------------------

def _attn_fwd(d, **over):
    a = _args(["q", "k", "v", "bounds", "out", "lse"], **over)
    return rb.lib().rapid_attention_fwd(C.byref(d), *a, None, None)


def _attn_bwd(d, ws=FAKE, ws_bytes=1 << 50, **over):
    a = _args(["q", "k", "v", "bounds", "out", "lse", "dout", "dq", "dk", "dv"], **over)
    return rb.lib().rapid_attention_bwd(C.byref(d), *a, None, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [_attn_fwd, _attn_bwd])
def test_attention_refusals(call):
    def d(n=4, length=8, h=4, hk=2, hd=64, **kw):
        return rb.make_attn_desc(n, length, h, hk, hd, **kw)
    for kw in (dict(n=0), dict(length=0), dict(h=0), dict(hk=0), dict(hd=0), dict(h=5), dict(window=-1), dict(scale=0.0), dict(scale=-1.0),
               dict(scale=math.inf), dict(scale=math.nan), dict(flags=1), dict(dtype=F32), dict(ld_q=248), dict(ld_k=120),
               dict(ld_v=64), dict(ld_out=0)):
        assert call(d(**kw)) == INVALID, kw
    for kw in (dict(hd=20), dict(hd=136), dict(n=1 << 20, length=1 << 12), dict(length=(1 << 24) + 1, n=1), dict(ld_q=1 << 36),
               dict(h=8192, hk=8192)):
        assert call(d(**kw)) == UNSUP, kw
    for kw in (dict(ld_q=260), dict(ld_k=132), dict(ld_v=129), dict(ld_out=257)):
        assert call(d(**kw)) == ALIGN, kw
    bwd = call is _attn_bwd
    names = ["q", "k", "v", "out"] + (["dout", "dq", "dk", "dv"] if bwd else [])
    for name in names + (["lse"] if bwd else []):
        assert call(d(), **{name: None}) == INVALID, name
    for name in names:
        assert call(d(), **{name: FAKE + FAR // 2 + 8}) == ALIGN, name
    for name in ("dq", "dk", "dv") if bwd else ("out",):
        assert call(d(), **{name: FAKE + 256}) == INVALID, name  # on q
        assert call(d(), **{name: FAKE + 2 * FAR}) == INVALID, name  # on v
    if bwd:
        assert call(d(), dk=FAKE + 7 * FAR) == INVALID  # on dq
        for kw in (dict(ld_dout=248), dict(ld_dq=8), dict(ld_dk=64), dict(ld_dv=120)):
            assert call(d(**kw)) == INVALID, kw
        assert call(d(ld_dq=258)) == ALIGN and call(d(ld_dk=1 << 36)) == UNSUP
        n = rb.rapid_attention_bwd_workspace_bytes(d())
        assert n == 2 * 4 * 4 * 4 * 128
        assert call(d(), ws=None) == WORK and call(d(), ws=FAKE + 8) == WORK and call(d(), ws_bytes=n - 1) == WORK


@no_gpu
def test_attention_without_a_device():
    d = rb.make_attn_desc(4, 8, 4, 2, 64)
    assert _attn_fwd(d, bounds=None, lse=None) == rb.RAPID_ERR_CUDA and _attn_bwd(d) == rb.RAPID_ERR_CUDA


def test_wrappers_check_shapes_and_types_before_the_call():
    x = torch.zeros(4, 2, 16)
    w = torch.zeros(16)
    with pytest.raises(ValueError):
        rb.qk_norm_rope(x, x, None, None, w[:8], 2, 2)
    with pytest.raises(ValueError):
        rb.qk_norm_rope(x, x[:3], w, w, w[:8], 2, 2)
    with pytest.raises(TypeError):
        rb.qk_norm_rope(x, x, w, w.double(), w[:8], 2, 2)
    with pytest.raises(ValueError, match="CUDA"):
        rb.qk_norm_rope(x, x, w, w, w[:8], 2, 2)
    tok = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(TypeError):
        rb.embedding(torch.zeros(5, 8), tok.long())
    with pytest.raises(ValueError):
        rb.embedding(torch.zeros(5, 8), tok, torch.zeros(3, dtype=torch.uint8))
    with pytest.raises(TypeError):
        rb.embedding_grad(torch.zeros(4, 8), tok, None, 5, dtable_dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        rb.embedding_grad(torch.zeros(4, 8), tok, None, 5, dtable=torch.zeros(5, 9))
    b = x.to(BF)
    with pytest.raises(TypeError):
        rb.attention(x, x, x, 2, 2)
    with pytest.raises(ValueError):
        rb.attention(b, b, b, 2, 3)
    with pytest.raises(TypeError):
        rb.attention(b, b, b, 2, 2, torch.zeros(2, 2))
    with pytest.raises(ValueError):
        rb.attention_grad(b, b, b, b, torch.zeros(3), b, 2, 2)


@no_gpu
def test_embedding_matrices_may_end_where_the_next_begins():
    """The last row of a slice ends with its columns, not with its pitch."""
    d = rb.make_embed_desc(2, 2, 16, BF, 64, 64)
    end = FAKE + (64 + 16) * 2
    assert _embed_fwd(d, table=FAKE, out=end) == rb.RAPID_ERR_CUDA
    assert _embed_fwd(d, table=FAKE, out=end - 16) == INVALID
    d = rb.make_embed_desc(2, 2, 16, BF, 64, 64, flags=rb.EMBED_DTABLE_BF16)
    assert _embed_bwd(d, dout=end, dtable=FAKE) == rb.RAPID_ERR_CUDA
    assert _embed_bwd(d, dout=FAKE, dtable=end) == rb.RAPID_ERR_CUDA
    assert _embed_bwd(d, dout=FAKE, dtable=end - 16) == INVALID
