"""Losses over the logits, host side: bad descriptors, pointers, pitches and workspaces are refused before anything is enqueued, and
the wrappers refuse tensors that the calls could not work with (no GPU needed: a call that passes every check stops at the missing
device)."""
import contextlib
import ctypes as C
import math

import pytest
import torch

from paper_2510_03515_b200 import binding as rb

FAKE = 0x10000  # an aligned non-NULL address that nothing dereferences
FAR = 1 << 40   # distance between the fake arrays
BF, F32 = torch.bfloat16, torch.float32
INVALID, ALIGN, UNSUP, WORK = (rb.RAPID_ERR_INVALID_ARG, rb.RAPID_ERR_ALIGNMENT, rb.RAPID_ERR_UNSUPPORTED, rb.RAPID_ERR_WORKSPACE)
no_gpu = pytest.mark.skipif(torch.cuda.is_available(), reason="fake pointers must not reach a device")

ARRAYS = {
    "clip": ["logits", "targets", "mask", "old_logp", "ref_logp", "adv", "dlogits", "loss", "token_logp", "stats"],
    "preference": ["logits", "targets", "mask", "pairs", "ref_logp", "dlogits", "loss", "margins", "token_logp", "stats"],
    "distill": ["logits", "top_index", "top_logit", "top_lse", "mask", "dlogits", "loss", "token_loss", "stats"],
}
NEEDED = {"clip": ["logits", "targets", "old_logp", "adv", "loss"], "preference": ["logits", "targets", "pairs", "loss"],
          "distill": ["logits", "top_index", "top_logit", "loss"]}
KINDS = list(ARRAYS)


def _call(kind, d, ws=FAKE, ws_bytes=1 << 50, **over):
    base = {n: FAKE + (i + 1) * FAR for i, n in enumerate(ARRAYS[kind])}
    base.update(over)
    return getattr(rb.lib(), f"rapid_{kind}_loss")(C.byref(d), *[base[n] for n in ARRAYS[kind]], ws, ws_bytes, None)


def _desc(kind, n=4, length=8, v=104, dtype=BF, k=5, n_pairs=3, **kw):
    if kind == "clip":
        return rb.make_clip_desc(n, length, v, dtype, **kw)
    if kind == "preference":
        return rb.make_pref_desc(n, length, v, dtype, n_pairs, **kw)
    return rb.make_distill_desc(n * length, v, k, dtype, **kw)


def test_struct_sizes():
    assert C.sizeof(rb.ClipDesc) == 80 and rb.ClipDesc.eps_low.offset == 40
    assert C.sizeof(rb.PrefDesc) == 80 and rb.PrefDesc.beta.offset == 40
    assert C.sizeof(rb.DistillDesc) == 72 and rb.DistillDesc.temperature.offset == 48
    assert C.sizeof(rb.LossStats) == rb.STATS_BYTES == 48 and rb.LossStats.mean_log_ratio.offset == 24


@no_gpu
@pytest.mark.parametrize("kind", KINDS)
def test_what_is_accepted_stops_at_the_device(kind):
    for d in (_desc(kind), _desc(kind, dtype=F32), _desc(kind, v=1, ld=8), _desc(kind, ld=112, ld_grad=120), _desc(kind, scale=-2.0),
              _desc(kind, flags=rb.LOSS_NORM_GIVEN, norm_z=0.5)):
        assert _call(kind, d) == rb.RAPID_ERR_CUDA
        assert _call(kind, d, dlogits=None, stats=None) == rb.RAPID_ERR_CUDA
    same = FAKE + FAR
    assert _call(kind, _desc(kind), dlogits=same, logits=same) == rb.RAPID_ERR_CUDA
    # side by side in the same rows
    assert _call(kind, _desc(kind, ld=208, ld_grad=208), logits=same, dlogits=same + 208) == rb.RAPID_ERR_CUDA
    if kind == "clip":
        assert _call(kind, _desc(kind), ref_logp=None) == rb.RAPID_ERR_CUDA
        assert _call(kind, _desc(kind, eps_low=math.inf, eps_high=math.inf)) == rb.RAPID_ERR_CUDA


@pytest.mark.parametrize("kind", KINDS)
def test_refusals(kind):
    for kw in (dict(n=0), dict(length=0), dict(v=0), dict(ld=96), dict(ld_grad=96), dict(scale=math.inf), dict(scale=math.nan),
               dict(flags=1 << 20), dict(flags=8), dict(flags=rb.LOSS_NORM_GIVEN), dict(flags=rb.LOSS_NORM_GIVEN, norm_z=math.inf),
               dict(flags=rb.LOSS_NORM_GIVEN, norm_z=-1.0)):
        assert _call(kind, _desc(kind, **kw)) == INVALID, kw
    for kw in (dict(v=100), dict(ld=108), dict(ld_grad=108), dict(v=102, dtype=F32)):
        assert _call(kind, _desc(kind, **kw)) == ALIGN, kw
    for kw in (dict(n=1 << 16, length=1 << 16), dict(n=1 << 20, ld=1 << 40), dict(n=1 << 20, ld_grad=1 << 40)):
        assert _call(kind, _desc(kind, **kw)) == UNSUP, kw
    bad = _desc(kind)
    bad.dtype = 7
    assert _call(kind, bad) == INVALID
    for name in NEEDED[kind]:
        assert _call(kind, _desc(kind), **{name: None}) == INVALID, name
    for name in ARRAYS[kind]:
        if name != "mask":
            assert _call(kind, _desc(kind), **{name: FAKE + 50 * FAR + 2}) == ALIGN, name
    assert _call(kind, _desc(kind), stats=FAKE + 50 * FAR + 4) == ALIGN
    assert _call(kind, _desc(kind), logits=FAKE + 50 * FAR + 8) == ALIGN
    base = FAKE + 50 * FAR
    for off in (16, 104 * 2 * 31, -64):  # overlapping, not in place
        assert _call(kind, _desc(kind), logits=base, dlogits=base + off) == INVALID
    assert _call(kind, _desc(kind, ld_grad=112), logits=base, dlogits=base) == INVALID
    assert _call(kind, _desc(kind, ld=208, ld_grad=208), logits=base, dlogits=base + 192) == INVALID
    fn = getattr(rb.lib(), f"rapid_{kind}_loss")
    assert fn(None, *[FAKE] * len(ARRAYS[kind]), FAKE, 1 << 50, None) == INVALID


@pytest.mark.parametrize("kind,kw,want", [
    ("clip", dict(eps_low=-0.1), INVALID), ("clip", dict(eps_high=math.nan), INVALID), ("clip", dict(kl_beta=-1.0), INVALID),
    ("clip", dict(kl_beta=math.inf), INVALID), ("clip", dict(flags=rb.PREF_HINGE), INVALID),
    ("preference", dict(beta=0.0), INVALID), ("preference", dict(beta=math.nan), INVALID), ("preference", dict(margin=math.inf), INVALID),
    ("preference", dict(label_smoothing=0.6), INVALID), ("preference", dict(label_smoothing=0.1, flags=rb.PREF_HINGE), INVALID),
    ("preference", dict(flags=rb.PREF_HINGE | rb.PREF_SQUARED), INVALID), ("preference", dict(flags=rb.LOSS_NORM_SEQ), INVALID),
    ("preference", dict(n_pairs=0), INVALID), ("preference", dict(n_pairs=(1 << 20) + 1), UNSUP),
    ("distill", dict(k=0), INVALID), ("distill", dict(ld_top=4), INVALID), ("distill", dict(temperature=0.0), INVALID),
    ("distill", dict(temperature=math.nan), INVALID), ("distill", dict(temperature=math.inf), INVALID), ("distill", dict(flags=rb.CLIP_ADV_TOKEN), INVALID),
    ("distill", dict(k=257, ld_top=300), UNSUP), ("distill", dict(temperature=1e-4), UNSUP), ("distill", dict(temperature=2e3), UNSUP),
    ("distill", dict(ld_top=1 << 60), UNSUP)])
def test_refusals_of_one(kind, kw, want):
    assert _call(kind, _desc(kind, **kw)) == want


def test_a_kl_term_needs_its_reference():
    assert _call("clip", _desc("clip", kl_beta=0.1), ref_logp=None) == INVALID


@pytest.mark.parametrize("kind", KINDS)
def test_workspaces(kind):
    for d, rows in ((_desc(kind), 32), (_desc(kind, n=100, length=1000, v=8), 100000)):
        n = getattr(rb, f"rapid_{kind}_loss_workspace_bytes")(d)
        assert 21 * rows <= n <= 42 * rows + 48 * 100 + 16 * 3 + (128 << 10)
        assert _call(kind, d, ws_bytes=n - 1) == WORK and _call(kind, d, ws=None) == WORK and _call(kind, d, ws=FAKE + 64) == WORK
    fn = getattr(rb.lib(), f"rapid_{kind}_loss_workspace_bytes")
    assert fn(C.byref(_desc(kind)), None) == INVALID and fn(None, C.byref(C.c_size_t())) == INVALID


# ---- the wrappers ------------------------------------------------------------------------------------------------

@pytest.fixture
def calls(monkeypatch):
    """Descriptors and arrays that the wrappers hand to the C calls, which are not made."""
    seen = []
    monkeypatch.setattr(rb, "_one_device", lambda *tensors: 0)
    monkeypatch.setattr(rb, "_on", lambda index: contextlib.nullcontext())
    for name in ("rapid_clip_loss", "rapid_preference_loss", "rapid_distill_loss"):
        monkeypatch.setattr(rb, name, lambda desc, *rest: seen.append((desc, rest)))
    return seen


N, L, V, K = 2, 3, 16, 4
T = N * L


def _z(dtype=F32, cols=V, rows=T):
    return torch.zeros(rows, cols, dtype=dtype)


def _clip(z=None, **kw):
    a = dict(targets=torch.zeros(T, dtype=torch.int32), mask=None, old_logp=torch.zeros(T), adv=torch.zeros(N))
    a.update({k: kw.pop(k) for k in list(kw) if k in a})
    return rb.clip_loss(_z() if z is None else z, a["targets"], a["mask"], a["old_logp"], a["adv"], N, L, **kw)


def _pref(z=None, **kw):
    a = dict(targets=torch.zeros(T, dtype=torch.int32), mask=None, pairs=torch.tensor([[0, 1]], dtype=torch.int32))
    a.update({k: kw.pop(k) for k in list(kw) if k in a})
    return rb.preference_loss(_z() if z is None else z, a["targets"], a["mask"], a["pairs"], N, L, **kw)


def _distill(z=None, **kw):
    a = dict(top_index=torch.zeros(T, K, dtype=torch.int32), top_logit=torch.zeros(T, K))
    a.update({k: kw.pop(k) for k in list(kw) if k in a})
    return rb.distill_loss(_z() if z is None else z, a["top_index"], a["top_logit"], **kw)


WRAPPERS = [_clip, _pref, _distill]


@pytest.mark.parametrize("call", WRAPPERS)
def test_wrappers_allocate_what_they_return(calls, call):
    r = call()
    assert r.dlogits.shape == (T, V) and r.dlogits.dtype == F32 and r.loss.shape == (1,)
    z = torch.zeros(T, 24, dtype=BF)[:, :13]  # 13 columns of rows of 48 bytes
    r = call(z)
    desc = calls[-1][0]
    assert (desc.vocab, desc.ld, desc.ld_grad, desc.dtype) == (13, 24, 16, rb.RAPID_BF16) and r.dlogits.stride() == (16, 1)
    assert call(z, in_place=True).dlogits is z and calls[-1][0].ld_grad == 24
    assert call(want_grad=False).dlogits is None
    assert call(mask=torch.ones(T, dtype=torch.bool)).loss.dtype == F32


@pytest.mark.parametrize("call", WRAPPERS)
def test_wrappers_refuse(calls, call):
    for kw in (dict(z=_z(rows=T + 1)), dict(z=torch.zeros(V, T).t()), dict(z=torch.zeros(T, 0)), dict(mask=torch.ones(T + 1, dtype=torch.uint8)),
               dict(in_place=True, want_grad=False), dict(stats=torch.zeros(8, dtype=torch.uint8)), dict(flags=-1), dict(flags=2 ** 32)):
        with pytest.raises(ValueError):
            call(**kw)
    for kw in (dict(z=_z(torch.float16)), dict(mask=torch.ones(T))):
        with pytest.raises(TypeError):
            call(**kw)
    assert calls == []


def test_each_wrapper_refuses_its_own(calls):
    i32 = torch.int32
    for kw in (dict(adv=torch.zeros(N + 1)), dict(old_logp=torch.zeros(T + 1)), dict(ref_logp=torch.zeros(T - 1)), dict(targets=torch.zeros(1, dtype=i32))):
        with pytest.raises(ValueError):
            _clip(**kw)
    for kw in (dict(adv=torch.zeros(N, dtype=torch.float64)), dict(targets=torch.zeros(T, dtype=torch.int64))):
        with pytest.raises(TypeError):
            _clip(**kw)
    for kw in (dict(pairs=torch.zeros(0, 2, dtype=i32)), dict(pairs=torch.zeros(4, dtype=i32)), dict(pairs=torch.zeros(2, 3, dtype=i32)),
               dict(pairs=torch.zeros(2, 4, dtype=i32).t()[:2].t())):
        with pytest.raises(ValueError):
            _pref(**kw)
    with pytest.raises(TypeError):
        _pref(pairs=torch.zeros(1, 2, dtype=torch.int64))
    for kw in (dict(top_index=torch.zeros(T, K + 1, dtype=i32)), dict(top_index=torch.zeros(K, T, dtype=i32).t()), dict(top_lse=torch.zeros(T + 1)),
               dict(top_logit=torch.zeros(T, 2 * K)[:, :K])):
        with pytest.raises(ValueError):
            _distill(**kw)
    with pytest.raises(TypeError):
        _distill(top_logit=torch.zeros(T, K, dtype=BF))
    assert calls == []


def test_an_advantage_for_each_row_is_told_by_its_size(calls):
    _clip()
    _clip(adv=torch.zeros(T))
    _clip(flags=rb.LOSS_NORM_SEQ)
    assert [c[0].flags for c in calls] == [0, rb.CLIP_ADV_TOKEN, rb.LOSS_NORM_SEQ]


@pytest.mark.parametrize("call,field", [(_clip, "kl_beta"), (_clip, "scale"), (_pref, "beta"), (_pref, "margin"), (_distill, "temperature"), (_distill, "scale")])
def test_a_changed_number_reaches_the_call(calls, call, field):
    """A number held in a tensor that is changed in place between two calls."""
    x = torch.tensor(0.5)
    call(**{field: x})
    x.mul_(4)
    call(**{field: x})
    assert [getattr(c[0], field) for c in calls] == [0.5, 2.0]
