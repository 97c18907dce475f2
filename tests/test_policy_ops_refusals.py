"""Policy-network operators, host side: calls whose numbers or addresses the kernels could not work with are refused before anything is
enqueued (no GPU needed; what is accepted stops at the missing device)."""

import ctypes as C

import pytest
import torch

import test_policy_ops_host as base
from paper_2510_03515_b200 import binding as rb

ATTENTION = [base._attn_fwd, base._attn_bwd]


def _attn(**kw):
    return rb.make_attn_desc(4, 8, 4, 2, 64, **kw)


# ---- the factor of the scores ----------------------------------------------------------------------------------

FLT_MIN, FLT_MAX = torch.finfo(torch.float32).tiny, torch.finfo(torch.float32).max


@pytest.mark.parametrize("call", ATTENTION)
@pytest.mark.parametrize("scale", [1e39, 1e300, FLT_MAX, FLT_MAX / 1.44, 1e-39, 1e-50, 5e-324, FLT_MIN * 0.999])
def test_a_scale_that_is_no_float_is_refused(call, scale):
    """The kernels work with scale and scale * log2(e) in float: neither may be infinite, zero or subnormal."""
    assert call(_attn(scale=scale)) == base.INVALID


@base.no_gpu
@pytest.mark.parametrize("call", ATTENTION)
@pytest.mark.parametrize("scale", [FLT_MAX / 1.45, FLT_MIN, 1.0, 64 ** -0.5])
def test_any_other_scale_is_accepted(call, scale):
    assert call(_attn(scale=scale)) == rb.RAPID_ERR_CUDA


# ---- arrays of numbers and stats off their boundaries ------------------------------------------------------------

ODD = base.FAKE + base.FAR // 2 + 2


@pytest.mark.parametrize("call,names", [(base._qk_fwd, ["qw", "kw", "freq", "pos"]), (base._qk_bwd, ["qw", "kw", "freq", "pos", "dqw", "dkw"])])
def test_qk_arrays_off_a_boundary_are_refused(call, names):
    d = rb.make_qk_desc(4, 8, 4, 2, 64, base.BF)
    for name in names:
        assert call(d, **{name: ODD}) == base.ALIGN, name


@pytest.mark.parametrize("call", ATTENTION)
def test_attention_arrays_off_a_boundary_are_refused(call):
    for name in ("bounds", "lse"):
        assert call(_attn(), **{name: ODD}) == base.ALIGN, name


def test_stats_off_a_boundary_are_refused():
    stats = base.FAKE + 90 * base.FAR + 4
    a = base._args(["tokens", "mask", "table", "out"])
    assert rb.lib().rapid_embedding_fwd(C.byref(rb.make_embed_desc(8, 100, 16, base.BF)), *a, stats, None) == base.ALIGN
    a = base._args(["q", "k", "v", "bounds", "out", "lse"])
    assert rb.lib().rapid_attention_fwd(C.byref(_attn()), *a, stats, None) == base.ALIGN
    a = base._args(["q", "k", "v", "bounds", "out", "lse", "dout", "dq", "dk", "dv"])
    assert rb.lib().rapid_attention_bwd(C.byref(_attn()), *a, stats, base.FAKE + 80 * base.FAR, 1 << 50, None) == base.ALIGN


# ---- scratch of the attention gradient -----------------------------------------------------------------------------

@pytest.mark.parametrize("n,length,heads", [(65536, 1, 12), (4877, 8, 9), (1335, 40, 2), (1000, 64, 3), (300, 43, 4), (129, 1, 2), (7, 60, 12)])
def test_scratch_follows_the_rows_of_short_generations(n, length, heads):
    """Generations that share a tile share its scratch: at most half of a tile's places are empty, the last tile's aside."""
    got = rb.rapid_attention_bwd_workspace_bytes(rb.make_attn_desc(n, length, heads, 1, 64))
    assert got <= 2 * 4 * heads * (2 * n * length + 128) + 2 * 8192
    # the generations that fill whole tiles at the least; those of the last tile come after them, in the same place
    parts = min(128 // length, n)
    assert got >= 2 * 4 * heads * (n // parts * parts) * length


@pytest.mark.parametrize("n,length,heads", [(64, 1024, 12), (3, 4095, 16), (5, 65, 3), (1, 64, 1), (2, 127, 8)])
def test_scratch_of_longer_generations(n, length, heads):
    got = rb.rapid_attention_bwd_workspace_bytes(rb.make_attn_desc(n, length, heads, 1, 64))
    need = 2 * 4 * heads * n * (-(-length // 128) * 128)
    assert need <= got <= need + 2 * 8192
    d = rb.make_attn_desc(n, length, heads, 1, 64)
    assert base._attn_bwd(d, ws_bytes=got - 1) == base.WORK


# ---- work behind one wait --------------------------------------------------------------------------------------------

def _long(length, h, hk, window=0):
    return rb.make_attn_desc(1, length, h, hk, 8, window)


def test_gradients_whose_waits_would_run_out_are_refused():
    """One key tile's walk over all query tiles and heads of its group takes 1.5 us a step; a warp that has nothing to do in it waits
    for the next one, at most 4 s."""
    for d in (_long(1 << 24, 16, 1), _long(1 << 24, 64, 4), _long((1 << 23) + 1, 16, 1), _long(1 << 20, 256, 1), _long(1 << 24, 16, 1, 1 << 23)):
        assert base._attn_bwd(d) == base.UNSUP
    with pytest.raises(rb.RapidError):
        rb.rapid_attention_bwd_workspace_bytes(_long(1 << 24, 16, 1))


@base.no_gpu
def test_long_gradients_with_short_walks_are_accepted():
    for d in (_long(1 << 23, 16, 1), _long(1 << 24, 16, 2), _long(1 << 24, 16, 1, 4096), _long(1 << 20, 256, 2)):
        assert base._attn_bwd(d) == rb.RAPID_ERR_CUDA
    assert base._attn_fwd(_long(1 << 24, 16, 1)) == rb.RAPID_ERR_CUDA


# ---- embedding matrices side by side in the same rows ------------------------------------------------------------------

@base.no_gpu
@pytest.mark.parametrize("n,v", [(8, 100), (100, 8), (1, 100), (100, 1)])
def test_embedding_matrices_may_share_rows(n, v):
    """Column slices of one matrix: table and out, or dout and a bf16 dtable."""
    d = rb.make_embed_desc(n, v, 16, base.BF, 48, 48)
    assert base._embed_fwd(d, table=base.FAKE, out=base.FAKE + 32) == rb.RAPID_ERR_CUDA
    assert base._embed_fwd(d, table=base.FAKE + 64, out=base.FAKE) == rb.RAPID_ERR_CUDA
    d = rb.make_embed_desc(n, v, 16, base.BF, 48, 48, flags=rb.EMBED_DTABLE_BF16)
    assert base._embed_bwd(d, dout=base.FAKE + 32, dtable=base.FAKE) == rb.RAPID_ERR_CUDA
    # float columns beside bf16 ones, 160 bytes a row both ways
    d = rb.make_embed_desc(n, v, 16, base.BF, 40, 80)
    assert base._embed_bwd(d, dout=base.FAKE + 64, dtable=base.FAKE) == rb.RAPID_ERR_CUDA


@pytest.mark.parametrize("n,v", [(8, 100), (100, 8)])
def test_embedding_matrices_that_share_elements_are_refused(n, v):
    d = rb.make_embed_desc(n, v, 16, base.BF, 48, 48)
    for off in (0, 16, 80):  # the last: into the next row's first columns
        assert base._embed_fwd(d, table=base.FAKE, out=base.FAKE + off) == base.INVALID, off
        assert base._embed_fwd(d, table=base.FAKE + off, out=base.FAKE) == base.INVALID, off
    d = rb.make_embed_desc(n, v, 16, base.BF, 48, 56, flags=rb.EMBED_DTABLE_BF16)  # other pitches: apart altogether
    assert base._embed_bwd(d, dout=base.FAKE + 32, dtable=base.FAKE) == base.INVALID
    d = rb.make_embed_desc(n, v, 16, base.BF, 48, 96)
    assert base._embed_bwd(d, dout=base.FAKE + 48, dtable=base.FAKE) == base.INVALID


# ---- sizes beyond 64 bits ------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("call", [base._embed_fwd, base._embed_bwd])
def test_embedding_matrices_beyond_any_memory_are_refused(call):
    """2^31 rows of 2^32 floats are 2^65 bytes; the overlap checks count bytes in 64 bits."""
    for d in (rb.make_embed_desc(2 ** 31 - 1, 5, 8, torch.float32, 8, 2 ** 32), rb.make_embed_desc(2 ** 31 - 1, 5, 8, base.BF, 8, 2 ** 32),
              rb.make_embed_desc(1, 2 ** 27 - 2, 8, torch.float32, 2 ** 32, 8)):
        assert call(d) == base.UNSUP


@pytest.mark.parametrize("call", [base._qk_fwd, base._qk_bwd])
def test_qk_matrices_beyond_any_memory_are_refused(call):
    for name in ("ld_q", "ld_k", "ld_q_out", "ld_k_out") + (("ld_dq", "ld_dk") if call is base._qk_bwd else ()):
        assert call(rb.make_qk_desc(2 ** 31 - 1, 1, 1, 1, 16, torch.float32, **{name: 2 ** 31})) == base.UNSUP, name
