"""ctypes binding over librapid_pg.so: same names as the C ABI (include/rapid_pg.h, include/rapid_policy_ops.h and
include/rapid_losses.h), argument marshalling only.  Tensors are PyTorch CUDA tensors used purely as device memory; every step of
the computation runs in the library's kernels on torch's current stream.

There is no fallback: if the shared library is missing the first call raises.
"""
from __future__ import annotations

import ctypes as C
import functools
import math
import operator
import os
from dataclasses import dataclass
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librapid_pg.so")

RAPID_OK = 0
RAPID_ERR_INVALID_ARG = 1
RAPID_ERR_ALIGNMENT = 2
RAPID_ERR_UNSUPPORTED = 3
RAPID_ERR_WORKSPACE = 4
RAPID_ERR_CUDA = 5
RAPID_ERR_TIMEOUT = 6

RAPID_F32 = 0
RAPID_BF16 = 1

FLAG_OUTER_UNCLIPPED = 1
FLAG_NORM_TOKENS = 2
FLAG_ADV_INPUT_IS_WEIGHT = 4
FLAG_LEAVE_ONE_OUT = 8
FLAG_LOO_LITERAL_DIVISOR = 16
FLAG_NORM_GIVEN = 32
FLAG_HEAD_STORE_LOGITS = 64
FLAG_HEAD_CTA_PAIRS = 128
FLAG_HEAD_SINGLE_CTA = 256
FLAG_HEAD_DW_BF16 = 512

EMBED_DTABLE_BF16 = 1
EMBED_ACCUMULATE = 2

QK_NO_NORM = 1
QK_UNIT_OFFSET = 2
QK_INTERLEAVED = 4

LOSS_NORM_SEQ = 1
LOSS_NORM_GIVEN = 2
CLIP_ADV_TOKEN = 4
PREF_HINGE = 16
PREF_SQUARED = 32
PREF_TOKEN_MEAN = 64

# every symbol declared in include/
EXPORTS = (
    "rapid_status_string", "rapid_version", "rapid_workspace_bytes", "rapid_group_advantage",
    "rapid_pg_loss_fwd_bwd", "rapid_pg_stats_chunk", "rapid_pg_finalize", "rapid_pg_dlogits_chunk",
    "rapid_pg_loss_fwd_bwd_noalloc", "rapid_fused_head_workspace_bytes", "rapid_pg_loss_fused_head",
    "rapid_pg_loss_onpolicy_fwd_bwd", "rapid_pg_loss_fwd_bwd_hostlogits", "rapid_selftest_bounded_wait",
    "rapid_embedding_fwd", "rapid_embedding_bwd_workspace_bytes", "rapid_embedding_bwd",
    "rapid_qk_norm_rope_fwd", "rapid_qk_norm_rope_bwd_workspace_bytes", "rapid_qk_norm_rope_bwd",
    "rapid_attention_fwd", "rapid_attention_bwd_workspace_bytes", "rapid_attention_bwd",
    "rapid_clip_loss_workspace_bytes", "rapid_clip_loss", "rapid_preference_loss_workspace_bytes", "rapid_preference_loss",
    "rapid_distill_loss_workspace_bytes", "rapid_distill_loss",
)


class RapidDesc(C.Structure):
    _fields_ = [("n_seq", C.c_int32), ("seq_len", C.c_int32), ("vocab", C.c_int32),
                ("n_groups", C.c_int32), ("ld", C.c_int64), ("dtype", C.c_int32),
                ("flags", C.c_uint32), ("eta", C.c_double), ("norm_z", C.c_double)]


class RapidStats(C.Structure):
    _fields_ = [("n_tokens", C.c_int64), ("n_clipped", C.c_int32), ("n_bad_token", C.c_int32),
                ("n_empty_group", C.c_int32), ("status", C.c_int32), ("mean_log_cw", C.c_double),
                ("mean_abs_log_cw", C.c_double), ("loss", C.c_double)]


STATS_BYTES = C.sizeof(RapidStats)


class EmbedDesc(C.Structure):
    _fields_ = [("n_rows", C.c_int64), ("vocab", C.c_int32), ("dim", C.c_int32), ("ld_table", C.c_int64),
                ("ld_rows", C.c_int64), ("dtype", C.c_int32), ("flags", C.c_uint32), ("scale", C.c_float),
                ("reserved", C.c_int32)]


class QkDesc(C.Structure):
    _fields_ = [("n_seq", C.c_int32), ("seq_len", C.c_int32), ("n_q_heads", C.c_int32), ("n_k_heads", C.c_int32),
                ("head_dim", C.c_int32), ("rot_dim", C.c_int32), ("ld_q", C.c_int64), ("ld_k", C.c_int64),
                ("ld_q_out", C.c_int64), ("ld_k_out", C.c_int64), ("ld_dq", C.c_int64), ("ld_dk", C.c_int64), ("dtype", C.c_int32), ("flags", C.c_uint32),
                ("eps", C.c_float), ("reserved", C.c_int32)]


class AttnDesc(C.Structure):
    _fields_ = [("n_seq", C.c_int32), ("seq_len", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("window", C.c_int32), ("ld_q", C.c_int64), ("ld_k", C.c_int64), ("ld_v", C.c_int64),
                ("ld_out", C.c_int64), ("ld_dout", C.c_int64), ("ld_dq", C.c_int64), ("ld_dk", C.c_int64),
                ("ld_dv", C.c_int64), ("dtype", C.c_int32), ("flags", C.c_uint32), ("scale", C.c_double)]


class LossStats(C.Structure):
    _fields_ = [("n_tokens", C.c_int64), ("n_clipped", C.c_int32), ("n_bad", C.c_int32), ("n_pairs", C.c_int32), ("status", C.c_int32),
                ("mean_log_ratio", C.c_double), ("mean_kl", C.c_double), ("loss", C.c_double)]


class ClipDesc(C.Structure):
    _fields_ = [("n_seq", C.c_int32), ("seq_len", C.c_int32), ("vocab", C.c_int32), ("dtype", C.c_int32), ("ld", C.c_int64),
                ("ld_grad", C.c_int64), ("flags", C.c_uint32), ("reserved", C.c_int32), ("eps_low", C.c_double), ("eps_high", C.c_double),
                ("kl_beta", C.c_double), ("scale", C.c_double), ("norm_z", C.c_double)]


class PrefDesc(C.Structure):
    _fields_ = [("n_seq", C.c_int32), ("seq_len", C.c_int32), ("vocab", C.c_int32), ("dtype", C.c_int32), ("ld", C.c_int64),
                ("ld_grad", C.c_int64), ("flags", C.c_uint32), ("n_pairs", C.c_int32), ("beta", C.c_double), ("margin", C.c_double),
                ("label_smoothing", C.c_double), ("scale", C.c_double), ("norm_z", C.c_double)]


class DistillDesc(C.Structure):
    _fields_ = [("n_rows", C.c_int64), ("vocab", C.c_int32), ("k", C.c_int32), ("ld", C.c_int64), ("ld_grad", C.c_int64),
                ("ld_top", C.c_int64), ("dtype", C.c_int32), ("flags", C.c_uint32), ("temperature", C.c_double), ("scale", C.c_double),
                ("norm_z", C.c_double)]


class RapidError(RuntimeError):
    def __init__(self, code: int, where: str):
        self.code = code
        super().__init__(f"{where}: {status_string(code)} ({code})")


_lib = None


def lib():
    """Load librapid_pg.so (once).  Raises if it has not been built: there is no other path."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2510_03515_b200.build` "
                "(there is no CPU or PyTorch fallback)")
        L = C.CDLL(LIB_PATH)
        vp, i64, sz = C.c_void_p, C.c_int64, C.c_size_t
        dp = C.POINTER(RapidDesc)
        L.rapid_status_string.restype = C.c_char_p
        L.rapid_status_string.argtypes = [C.c_int]
        L.rapid_version.restype = C.c_int32
        L.rapid_workspace_bytes.restype = C.c_int
        L.rapid_workspace_bytes.argtypes = [dp, C.POINTER(C.c_size_t)]
        L.rapid_group_advantage.restype = C.c_int
        L.rapid_group_advantage.argtypes = [dp, vp, vp, vp, vp, vp, vp, vp]
        L.rapid_pg_loss_fwd_bwd.restype = C.c_int
        L.rapid_pg_loss_fwd_bwd.argtypes = [dp] + [vp] * 12 + [sz, vp]
        L.rapid_pg_loss_fwd_bwd_noalloc.restype = C.c_int
        L.rapid_pg_loss_fwd_bwd_noalloc.argtypes = [dp] + [vp] * 12
        L.rapid_pg_loss_fwd_bwd_hostlogits.restype = C.c_int
        L.rapid_pg_loss_fwd_bwd_hostlogits.argtypes = [dp] + [vp] * 13 + [sz, vp]
        L.rapid_pg_loss_onpolicy_fwd_bwd.restype = C.c_int
        L.rapid_pg_loss_onpolicy_fwd_bwd.argtypes = [dp] + [vp] * 11 + [sz, vp]
        L.rapid_fused_head_workspace_bytes.restype = C.c_int
        L.rapid_fused_head_workspace_bytes.argtypes = [dp, C.c_int32, C.POINTER(C.c_size_t)]
        L.rapid_pg_loss_fused_head.restype = C.c_int
        L.rapid_pg_loss_fused_head.argtypes = [dp, C.c_int32] + [vp] * 14 + [sz, vp]
        L.rapid_selftest_bounded_wait.restype = C.c_int
        L.rapid_selftest_bounded_wait.argtypes = [C.c_uint64, vp, vp]
        L.rapid_pg_stats_chunk.restype = C.c_int
        L.rapid_pg_stats_chunk.argtypes = [dp, vp, i64, i64, vp, vp, vp, sz, vp]
        L.rapid_pg_finalize.restype = C.c_int
        L.rapid_pg_finalize.argtypes = [dp] + [vp] * 8 + [sz, vp]
        L.rapid_pg_dlogits_chunk.restype = C.c_int
        L.rapid_pg_dlogits_chunk.argtypes = [dp, vp, vp, i64, i64, vp, vp, vp, sz, vp]
        ep, qp, ap = C.POINTER(EmbedDesc), C.POINTER(QkDesc), C.POINTER(AttnDesc)
        for name, argtypes in {
            "rapid_embedding_fwd": [ep] + [vp] * 6,
            "rapid_embedding_bwd_workspace_bytes": [ep, C.POINTER(sz)],
            "rapid_embedding_bwd": [ep] + [vp] * 5 + [sz, vp],
            "rapid_qk_norm_rope_fwd": [qp] + [vp] * 10,
            "rapid_qk_norm_rope_bwd_workspace_bytes": [qp, C.POINTER(sz)],
            "rapid_qk_norm_rope_bwd": [qp] + [vp] * 14 + [sz, vp],
            "rapid_attention_fwd": [ap] + [vp] * 8,
            "rapid_attention_bwd_workspace_bytes": [ap, C.POINTER(sz)],
            "rapid_attention_bwd": [ap] + [vp] * 12 + [sz, vp],
            "rapid_clip_loss_workspace_bytes": [C.POINTER(ClipDesc), C.POINTER(sz)],
            "rapid_clip_loss": [C.POINTER(ClipDesc)] + [vp] * 11 + [sz, vp],
            "rapid_preference_loss_workspace_bytes": [C.POINTER(PrefDesc), C.POINTER(sz)],
            "rapid_preference_loss": [C.POINTER(PrefDesc)] + [vp] * 11 + [sz, vp],
            "rapid_distill_loss_workspace_bytes": [C.POINTER(DistillDesc), C.POINTER(sz)],
            "rapid_distill_loss": [C.POINTER(DistillDesc)] + [vp] * 10 + [sz, vp],
        }.items():
            getattr(L, name).restype = C.c_int
            getattr(L, name).argtypes = argtypes
        _lib = L
    return _lib


def status_string(code: int) -> str:
    return lib().rapid_status_string(int(code)).decode()


def rapid_version() -> int:
    return int(lib().rapid_version())


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream() -> C.c_void_p:
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(code: int, where: str) -> None:
    if code != RAPID_OK:
        raise RapidError(code, where)


def make_desc(n_seq: int, seq_len: int, vocab: int, n_groups: int, dtype: torch.dtype,
              ld: Optional[int] = None, eta: float = 2.0, flags: int = 0,
              norm_z: float = 0.0) -> RapidDesc:
    if dtype == torch.float32:
        dt = RAPID_F32
    elif dtype == torch.bfloat16:
        dt = RAPID_BF16
    else:
        raise TypeError("logits must be float32 or bfloat16")
    return RapidDesc(n_seq, seq_len, vocab, n_groups, vocab if ld is None else ld, dt, flags,
                     float(eta), float(norm_z))


def rapid_workspace_bytes(desc: RapidDesc) -> int:
    n = C.c_size_t(0)
    _check(lib().rapid_workspace_bytes(C.byref(desc), C.byref(n)), "rapid_workspace_bytes")
    return int(n.value)


def alloc_workspace(desc: RapidDesc, device="cuda") -> torch.Tensor:
    """Device memory for the scratch workspace (torch's allocator returns >= 256-byte alignment)."""
    return torch.empty(rapid_workspace_bytes(desc), dtype=torch.uint8, device=device)


def alloc_stats(device="cuda") -> torch.Tensor:
    return torch.zeros(STATS_BYTES, dtype=torch.uint8, device=device)


def read_stats(stats: torch.Tensor) -> dict:
    """Copy a device rapid_stats_t to the host (synchronises) and return it as a dict."""
    raw = bytes(stats.cpu().numpy().tobytes())
    s = RapidStats.from_buffer_copy(raw)
    return {k: getattr(s, k) for k, _ in RapidStats._fields_}


def rapid_group_advantage(desc: RapidDesc, rewards: torch.Tensor,
                          seq_log_ratio: Optional[torch.Tensor], group_offsets: torch.Tensor,
                          adv: torch.Tensor, clipped_w: Optional[torch.Tensor] = None,
                          stats: Optional[torch.Tensor] = None) -> None:
    _check(lib().rapid_group_advantage(C.byref(desc), _ptr(rewards), _ptr(seq_log_ratio),
                                       _ptr(group_offsets), _ptr(adv), _ptr(clipped_w),
                                       _ptr(stats), _stream()), "rapid_group_advantage")


def rapid_pg_loss_fwd_bwd(desc: RapidDesc, logits: torch.Tensor, targets: torch.Tensor,
                          mask: Optional[torch.Tensor], behav_logp: torch.Tensor,
                          rewards: torch.Tensor, group_offsets: torch.Tensor,
                          dlogits: torch.Tensor, loss: torch.Tensor,
                          token_logp: Optional[torch.Tensor], adv: Optional[torch.Tensor],
                          stats: Optional[torch.Tensor], workspace: torch.Tensor) -> None:
    _check(lib().rapid_pg_loss_fwd_bwd(
        C.byref(desc), _ptr(logits), _ptr(targets), _ptr(mask), _ptr(behav_logp), _ptr(rewards),
        _ptr(group_offsets), _ptr(dlogits), _ptr(loss), _ptr(token_logp), _ptr(adv), _ptr(stats),
        _ptr(workspace), workspace.numel(), _stream()), "rapid_pg_loss_fwd_bwd")


NOALLOC_SCRATCH_BYTES = 4 << 20


def rapid_pg_loss_fwd_bwd_noalloc(desc: RapidDesc, logits: torch.Tensor, targets: torch.Tensor,
                                  mask: Optional[torch.Tensor], behav_logp: torch.Tensor,
                                  rewards: torch.Tensor, group_offsets: torch.Tensor,
                                  dlogits: torch.Tensor, loss: torch.Tensor,
                                  token_logp: Optional[torch.Tensor], adv: Optional[torch.Tensor],
                                  stats: Optional[torch.Tensor]) -> None:
    """rapid_pg_loss_fwd_bwd for callers that cannot allocate a workspace: the scratch is a fixed
    array inside the library (at most NOALLOC_SCRATCH_BYTES; larger problems raise
    RAPID_ERR_UNSUPPORTED).  Calls on one device share that array, so do not let two overlap."""
    _check(lib().rapid_pg_loss_fwd_bwd_noalloc(
        C.byref(desc), _ptr(logits), _ptr(targets), _ptr(mask), _ptr(behav_logp), _ptr(rewards),
        _ptr(group_offsets), _ptr(dlogits), _ptr(loss), _ptr(token_logp), _ptr(adv), _ptr(stats),
        _stream()), "rapid_pg_loss_fwd_bwd_noalloc")


def rapid_pg_stats_chunk(desc: RapidDesc, logits_chunk: torch.Tensor, row0: int, n_rows: int,
                         targets: torch.Tensor, mask: Optional[torch.Tensor],
                         workspace: torch.Tensor) -> None:
    _check(lib().rapid_pg_stats_chunk(C.byref(desc), _ptr(logits_chunk), row0, n_rows,
                                      _ptr(targets), _ptr(mask), _ptr(workspace),
                                      workspace.numel(), _stream()), "rapid_pg_stats_chunk")


def rapid_pg_finalize(desc: RapidDesc, behav_logp: torch.Tensor, rewards: torch.Tensor,
                      group_offsets: torch.Tensor, loss: torch.Tensor,
                      token_logp: Optional[torch.Tensor], adv: Optional[torch.Tensor],
                      stats: Optional[torch.Tensor], workspace: torch.Tensor) -> None:
    _check(lib().rapid_pg_finalize(C.byref(desc), _ptr(behav_logp), _ptr(rewards),
                                   _ptr(group_offsets), _ptr(loss), _ptr(token_logp), _ptr(adv),
                                   _ptr(stats), _ptr(workspace), workspace.numel(), _stream()),
           "rapid_pg_finalize")


def rapid_pg_dlogits_chunk(desc: RapidDesc, logits_chunk: torch.Tensor,
                           dlogits_chunk: torch.Tensor, row0: int, n_rows: int,
                           targets: torch.Tensor, stats: Optional[torch.Tensor],
                           workspace: torch.Tensor) -> None:
    _check(lib().rapid_pg_dlogits_chunk(C.byref(desc), _ptr(logits_chunk), _ptr(dlogits_chunk),
                                        row0, n_rows, _ptr(targets), _ptr(stats), _ptr(workspace),
                                        workspace.numel(), _stream()), "rapid_pg_dlogits_chunk")


def rapid_pg_loss_fwd_bwd_hostlogits(desc: RapidDesc, logits_host: torch.Tensor, logits_staging: torch.Tensor,
                                     targets: torch.Tensor, mask: Optional[torch.Tensor],
                                     behav_logp: torch.Tensor, rewards: torch.Tensor,
                                     group_offsets: torch.Tensor, dlogits: torch.Tensor, loss: torch.Tensor,
                                     token_logp: Optional[torch.Tensor], adv: Optional[torch.Tensor],
                                     stats: Optional[torch.Tensor], workspace: torch.Tensor) -> None:
    """`logits_host` is a PINNED CPU tensor; everything else lives on the device."""
    _check(lib().rapid_pg_loss_fwd_bwd_hostlogits(
        C.byref(desc), _ptr(logits_host), _ptr(logits_staging), _ptr(targets), _ptr(mask), _ptr(behav_logp),
        _ptr(rewards), _ptr(group_offsets), _ptr(dlogits), _ptr(loss), _ptr(token_logp), _ptr(adv),
        _ptr(stats), _ptr(workspace), workspace.numel(), _stream()), "rapid_pg_loss_fwd_bwd_hostlogits")


def rapid_pg_loss_onpolicy_fwd_bwd(desc: RapidDesc, logits: torch.Tensor, targets: torch.Tensor,
                                   mask: Optional[torch.Tensor], rewards: torch.Tensor,
                                   group_offsets: torch.Tensor, dlogits: torch.Tensor, loss: torch.Tensor,
                                   token_logp: Optional[torch.Tensor], adv: Optional[torch.Tensor],
                                   stats: Optional[torch.Tensor], workspace: torch.Tensor) -> None:
    _check(lib().rapid_pg_loss_onpolicy_fwd_bwd(
        C.byref(desc), _ptr(logits), _ptr(targets), _ptr(mask), _ptr(rewards), _ptr(group_offsets),
        _ptr(dlogits), _ptr(loss), _ptr(token_logp), _ptr(adv), _ptr(stats), _ptr(workspace),
        workspace.numel(), _stream()), "rapid_pg_loss_onpolicy_fwd_bwd")


def rapid_selftest_bounded_wait(limit_ns: int, stats: torch.Tensor) -> None:
    _check(lib().rapid_selftest_bounded_wait(int(limit_ns), _ptr(stats), _stream()), "rapid_selftest_bounded_wait")


def rapid_fused_head_workspace_bytes(desc: RapidDesc, hidden_dim: int) -> int:
    n = C.c_size_t(0)
    _check(lib().rapid_fused_head_workspace_bytes(C.byref(desc), int(hidden_dim), C.byref(n)),
           "rapid_fused_head_workspace_bytes")
    return int(n.value)


def alloc_fused_head_workspace(desc: RapidDesc, hidden_dim: int, device="cuda") -> torch.Tensor:
    """Device scratch for rapid_pg_loss_fused_head, on a 1024-byte boundary."""
    n = rapid_fused_head_workspace_bytes(desc, hidden_dim)
    buf = torch.empty(n + 1024, dtype=torch.uint8, device=device)
    off = (-buf.data_ptr()) % 1024
    return buf[off:off + n]


def rapid_pg_loss_fused_head(desc: RapidDesc, hidden: torch.Tensor, w_vocab: torch.Tensor,
                             targets: torch.Tensor, mask: Optional[torch.Tensor],
                             behav_logp: torch.Tensor, rewards: torch.Tensor,
                             group_offsets: torch.Tensor, loss: torch.Tensor, dhidden: torch.Tensor,
                             dW: torch.Tensor, token_logp: Optional[torch.Tensor],
                             adv: Optional[torch.Tensor], stats: Optional[torch.Tensor],
                             workspace: torch.Tensor) -> None:
    _check(lib().rapid_pg_loss_fused_head(
        C.byref(desc), int(hidden.shape[1]), _ptr(hidden), _ptr(w_vocab), _ptr(targets), _ptr(mask),
        _ptr(behav_logp), _ptr(rewards), _ptr(group_offsets), _ptr(loss), _ptr(dhidden), _ptr(dW),
        _ptr(token_logp), _ptr(adv), _ptr(stats), _ptr(workspace), workspace.numel(), _stream()),
        "rapid_pg_loss_fused_head")


@dataclass
class PgResult:
    loss: torch.Tensor        # [1] float32, device
    dlogits: torch.Tensor     # [T, ld]
    token_logp: torch.Tensor  # [T] float32
    adv: torch.Tensor         # [N] float32
    stats: torch.Tensor       # raw rapid_stats_t bytes, device


def pg_loss(logits: torch.Tensor, targets, mask, behav_logp, rewards, group_offsets, n_seq: int,
            seq_len: int, eta: float = 2.0, flags: int = 0, in_place: bool = False,
            workspace: Optional[torch.Tensor] = None, norm_z: float = 0.0) -> PgResult:
    """Convenience wrapper: allocate the outputs and make ONE rapid_pg_loss_fwd_bwd call."""
    T, ld = logits.shape[0], logits.stride(0)
    vocab = logits.shape[1]
    assert T == n_seq * seq_len
    desc = make_desc(n_seq, seq_len, vocab, group_offsets.numel() - 1, logits.dtype, ld, eta, flags, norm_z)
    dev = logits.device
    ws = workspace if workspace is not None else alloc_workspace(desc, dev)
    dlogits = logits if in_place else torch.empty_like(logits)
    loss = torch.empty(1, dtype=torch.float32, device=dev)
    token_logp = torch.empty(T, dtype=torch.float32, device=dev)
    adv = torch.empty(n_seq, dtype=torch.float32, device=dev)
    stats = alloc_stats(dev)
    rapid_pg_loss_fwd_bwd(desc, logits, targets, mask, behav_logp, rewards, group_offsets, dlogits,
                          loss, token_logp, adv, stats, ws)
    return PgResult(loss, dlogits, token_logp, adv, stats)


# ---- policy-network operators (include/rapid_policy_ops.h) ---------------------------------------------------
#
# The rapid_* functions marshal the arguments of the C calls; embedding(), embedding_grad(), qk_norm_rope(),
# qk_norm_rope_grad(), attention() and attention_grad() check shapes and types, allocate the outputs and make one call.


def _dtype_code(dtype: torch.dtype) -> int:
    if dtype == torch.float32:
        return RAPID_F32
    if dtype == torch.bfloat16:
        return RAPID_BF16
    raise TypeError(f"float32 or bfloat16 expected, got {dtype}")


def _one_device(first: torch.Tensor, *others: Optional[torch.Tensor]) -> int:
    """Number of the CUDA device that all the tensors lie on."""
    index = first.get_device()
    if index < 0:
        raise ValueError("tensors must be CUDA tensors")
    for t in others:
        if t is not None and t.get_device() != index:
            raise ValueError("tensors must be CUDA tensors of one device")
    return index


def _vector(t: Optional[torch.Tensor], n: int, dtype, name: str) -> None:
    if t is None:
        return
    if t.numel() != n or not t.is_contiguous():
        raise ValueError(f"{name}: {n} contiguous elements expected")
    if t.dtype != dtype:
        raise TypeError(f"{name}: {dtype} expected, got {t.dtype}")


def _mask8(mask: Optional[torch.Tensor], n: int) -> Optional[torch.Tensor]:
    if mask is None:
        return None
    if mask.dtype == torch.bool:
        mask = mask.view(torch.uint8)
    _vector(mask, n, torch.uint8, "mask")
    return mask


def _stats_room(stats: Optional[torch.Tensor]) -> None:
    if stats is not None and (stats.numel() * stats.element_size() < STATS_BYTES or not stats.is_contiguous() or stats.data_ptr() % 8):
        raise ValueError(f"stats: {STATS_BYTES} bytes side by side on an 8-byte boundary expected (alloc_stats)")


def _pitch(t: torch.Tensor, name: str) -> int:
    """Row pitch of a matrix [rows, cols] or of rows of heads [rows, heads, head_dim]."""
    shape, stride = t.shape, t.stride()
    if len(shape) == 3:
        rows, heads, dim = shape
        inner = (stride[2] == 1 or dim == 1) and (stride[1] == dim or heads == 1)
        width = heads * dim
    else:
        rows, width = shape
        inner = stride[1] == 1 or width == 1
    if not inner:
        raise ValueError(f"{name}: the elements of a row must lie side by side")
    if rows == 1:  # one row has no pitch: the narrowest that 16-byte rows allow
        step = 16 // t.element_size()
        return -(-width // step) * step
    return stride[0]


def _matrix(rows: int, cols: int, dtype, like: torch.Tensor) -> torch.Tensor:
    """An uninitialised [rows, cols] on like's device whose rows begin on 16-byte boundaries."""
    step = 16 // dtype.itemsize
    pitch = -(-cols // step) * step
    buf = like.new_empty((rows, pitch), dtype=dtype)
    return buf if pitch == cols else buf[:, :cols]


def _new(x: torch.Tensor) -> torch.Tensor:
    """A contiguous tensor of x's shape and type (half the time of torch.empty with a shape, a type and a device)."""
    return torch.empty_like(x, memory_format=torch.contiguous_format)


def _like(out: Optional[torch.Tensor], x: torch.Tensor, name: str) -> torch.Tensor:
    """`out`, or a contiguous tensor of x's shape and type where there is none."""
    if out is None:
        return _new(x)
    if out.shape != x.shape:
        raise ValueError(f"{name}: shape {tuple(x.shape)} expected")
    if out.dtype != x.dtype:
        raise TypeError(f"{name}: {x.dtype} expected, got {out.dtype}")
    return out


class _on:
    """Make device number `index` current for the calls inside (nothing to do when it is already)."""

    def __init__(self, index: int):
        self.guard = None if index == torch.cuda.current_device() else torch.cuda.device(index)

    def __enter__(self):
        if self.guard is not None:
            self.guard.__enter__()

    def __exit__(self, *exc):
        if self.guard is not None:
            self.guard.__exit__(*exc)


# torch.cuda.current_stream() builds an object for each call, 3 us; torch's own generated code asks for the bare handle.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream_here() -> int:
    """Handle of the current device's current stream."""
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _addr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _workspace(query, desc, where: str) -> int:
    n = C.c_size_t(0)
    _check(query(C.byref(desc), C.byref(n)), where)
    return int(n.value)


# Descriptors by their values, with the workspace size where one is needed: shapes repeat from call to call, and building a
# descriptor of 17 fields takes longer than a small kernel.  Only the convenience functions use these, and never change them.
# Every number among the keys is a Python int or float by then: a tensor is found again by its identity, whatever it holds.

def _int(x) -> int:
    return x if type(x) is int else operator.index(x)


def _float(x) -> float:
    return x if type(x) is float else float(x)


@functools.lru_cache(maxsize=512)
def _embed_plan(n_rows, vocab, dim, dtype, ld_table, ld_rows, scale, flags, bwd):
    desc = make_embed_desc(n_rows, vocab, dim, dtype, ld_table, ld_rows, scale, flags)
    return desc, rapid_embedding_bwd_workspace_bytes(desc) if bwd else 0


@functools.lru_cache(maxsize=512)
def _qk_plan(n_seq, seq_len, hq, hk, hd, dtype, rot, pitches, eps, flags, bwd):
    desc = make_qk_desc(n_seq, seq_len, hq, hk, hd, dtype, rot, *pitches, eps=eps, flags=flags)
    return desc, rapid_qk_norm_rope_bwd_workspace_bytes(desc) if bwd and not flags & QK_NO_NORM else 0


@functools.lru_cache(maxsize=512)
def _attn_plan(n_seq, seq_len, h, hk, hd, window, scale, pitches, bwd):
    desc = make_attn_desc(n_seq, seq_len, h, hk, hd, window, scale, *pitches)
    return desc, rapid_attention_bwd_workspace_bytes(desc) if bwd else 0


def _fits(flags: int, **numbers: int) -> None:
    """A field of 32 bits would keep a larger number's low bits."""
    for name, x in numbers.items():
        if not -2 ** 31 <= x < 2 ** 31:
            raise ValueError(f"{name}: {x} is not a number of 32 bits")
    if not 0 <= flags < 2 ** 32:
        raise ValueError(f"flags: {flags} is not a set of 32 bits")


def make_embed_desc(n_rows: int, vocab: int, dim: int, dtype: torch.dtype, ld_table: Optional[int] = None,
                    ld_rows: Optional[int] = None, scale: float = 1.0, flags: int = 0) -> EmbedDesc:
    _fits(flags, vocab=vocab, dim=dim)
    return EmbedDesc(n_rows, vocab, dim, dim if ld_table is None else ld_table, dim if ld_rows is None else ld_rows,
                     _dtype_code(dtype), flags, float(scale), 0)


def rapid_embedding_fwd(desc: EmbedDesc, tokens: torch.Tensor, mask: Optional[torch.Tensor], table: torch.Tensor,
                        out: torch.Tensor, stats: Optional[torch.Tensor]) -> None:
    _check(lib().rapid_embedding_fwd(C.byref(desc), _addr(tokens), _addr(mask), _addr(table), _addr(out), _addr(stats),
                                     _stream_here()), "rapid_embedding_fwd")


def rapid_embedding_bwd_workspace_bytes(desc: EmbedDesc) -> int:
    return _workspace(lib().rapid_embedding_bwd_workspace_bytes, desc, "rapid_embedding_bwd_workspace_bytes")


def rapid_embedding_bwd(desc: EmbedDesc, tokens: torch.Tensor, mask: Optional[torch.Tensor], dout: torch.Tensor,
                        dtable: torch.Tensor, workspace: torch.Tensor) -> None:
    _check(lib().rapid_embedding_bwd(C.byref(desc), _addr(tokens), _addr(mask), _addr(dout), _addr(dtable), _addr(workspace),
                                     workspace.numel(), _stream_here()), "rapid_embedding_bwd")


def embedding(table: torch.Tensor, tokens: torch.Tensor, mask: Optional[torch.Tensor] = None, scale: float = 1.0,
              stats: Optional[torch.Tensor] = None) -> torch.Tensor:
    """scale * table[tokens], [T, D] in the table's type; rows that are masked or whose token is no row of the table are
    zeros.  tokens [T] int32, table [V, D] (rows on 16-byte boundaries)."""
    if table.dim() != 2:
        raise ValueError("table: a matrix [V, D] expected")
    scale = _float(scale)
    T, (V, D) = tokens.numel(), table.shape
    mask = _mask8(mask, T)
    _vector(tokens, T, torch.int32, "tokens")
    _stats_room(stats)
    dev = _one_device(table, tokens, mask, stats)
    with _on(dev):
        out = _matrix(T, D, table.dtype, table)
        if T:
            desc, _ = _embed_plan(T, V, D, table.dtype, _pitch(table, "table"), _pitch(out, "out"), scale, 0, False)
            rapid_embedding_fwd(desc, tokens, mask, table, out, stats)
        elif stats is not None:
            stats.zero_()
    return out


def embedding_grad(dout: torch.Tensor, tokens: torch.Tensor, mask: Optional[torch.Tensor], vocab: int, scale: float = 1.0,
                   dtable_dtype: torch.dtype = torch.float32, dtable: Optional[torch.Tensor] = None) -> torch.Tensor:
    """The gradient of embedding() with respect to its table: [vocab, D] in `dtable_dtype`, or added to `dtable`, which
    is then returned (its type counts, not `dtable_dtype`)."""
    if dout.dim() != 2:
        raise ValueError("dout: a matrix [T, D] expected")
    vocab, scale = _int(vocab), _float(scale)
    T, D = dout.shape
    mask = _mask8(mask, T)
    _vector(tokens, T, torch.int32, "tokens")
    flags = 0
    if dtable is not None:
        if tuple(dtable.shape) != (vocab, D):
            raise ValueError("dtable: [vocab, D] expected")
        dtable_dtype, flags = dtable.dtype, EMBED_ACCUMULATE
    if _dtype_code(dtable_dtype) == RAPID_BF16:
        if dout.dtype != torch.bfloat16:
            raise TypeError("a bfloat16 dtable needs a bfloat16 dout")
        flags |= EMBED_DTABLE_BF16
    dev = _one_device(dout, tokens, mask, dtable)
    with _on(dev):
        if T == 0:
            return torch.zeros(vocab, D, dtype=dtable_dtype, device=dout.device) if dtable is None else dtable
        out = _matrix(vocab, D, dtable_dtype, dout) if dtable is None else dtable
        desc, ws_bytes = _embed_plan(T, vocab, D, dout.dtype, _pitch(out, "dtable"), _pitch(dout, "dout"), scale, flags, True)
        ws = dout.new_empty(ws_bytes, dtype=torch.uint8)
        rapid_embedding_bwd(desc, tokens, mask, dout, out, ws)
    return out


def make_qk_desc(n_seq: int, seq_len: int, n_q_heads: int, n_k_heads: int, head_dim: int, dtype: torch.dtype,
                 rot_dim: Optional[int] = None, ld_q: Optional[int] = None, ld_k: Optional[int] = None,
                 ld_q_out: Optional[int] = None, ld_k_out: Optional[int] = None, ld_dq: Optional[int] = None,
                 ld_dk: Optional[int] = None, eps: float = 1e-6, flags: int = 0) -> QkDesc:
    _fits(flags, n_seq=n_seq, seq_len=seq_len, n_q_heads=n_q_heads, n_k_heads=n_k_heads, head_dim=head_dim,
          rot_dim=head_dim if rot_dim is None else rot_dim)
    wq, wk = n_q_heads * head_dim, n_k_heads * head_dim
    pitches = [w if ld is None else ld for w, ld in ((wq, ld_q), (wk, ld_k), (wq, ld_q_out), (wk, ld_k_out), (wq, ld_dq), (wk, ld_dk))]
    return QkDesc(n_seq, seq_len, n_q_heads, n_k_heads, head_dim, head_dim if rot_dim is None else rot_dim, *pitches,
                  _dtype_code(dtype), flags, float(eps), 0)


def rapid_qk_norm_rope_fwd(desc: QkDesc, q: torch.Tensor, k: torch.Tensor, q_weight: Optional[torch.Tensor],
                           k_weight: Optional[torch.Tensor], inv_freq: torch.Tensor, positions: Optional[torch.Tensor],
                           mask: Optional[torch.Tensor], q_out: torch.Tensor, k_out: torch.Tensor) -> None:
    _check(lib().rapid_qk_norm_rope_fwd(C.byref(desc), _addr(q), _addr(k), _addr(q_weight), _addr(k_weight), _addr(inv_freq),
                                        _addr(positions), _addr(mask), _addr(q_out), _addr(k_out), _stream_here()),
           "rapid_qk_norm_rope_fwd")


def rapid_qk_norm_rope_bwd_workspace_bytes(desc: QkDesc) -> int:
    return _workspace(lib().rapid_qk_norm_rope_bwd_workspace_bytes, desc, "rapid_qk_norm_rope_bwd_workspace_bytes")


def rapid_qk_norm_rope_bwd(desc: QkDesc, q: torch.Tensor, k: torch.Tensor, q_weight: Optional[torch.Tensor],
                           k_weight: Optional[torch.Tensor], inv_freq: torch.Tensor, positions: Optional[torch.Tensor],
                           mask: Optional[torch.Tensor], dq_out: torch.Tensor, dk_out: torch.Tensor, dq: torch.Tensor,
                           dk: torch.Tensor, dq_weight: Optional[torch.Tensor], dk_weight: Optional[torch.Tensor],
                           workspace: Optional[torch.Tensor]) -> None:
    _check(lib().rapid_qk_norm_rope_bwd(
        C.byref(desc), _addr(q), _addr(k), _addr(q_weight), _addr(k_weight), _addr(inv_freq), _addr(positions), _addr(mask),
        _addr(dq_out), _addr(dk_out), _addr(dq), _addr(dk), _addr(dq_weight), _addr(dk_weight), _addr(workspace),
        0 if workspace is None else workspace.numel(), _stream_here()), "rapid_qk_norm_rope_bwd")


def _qk_args(q, k, q_weight, k_weight, inv_freq, n_seq, seq_len, positions, mask, flags):
    T = n_seq * seq_len
    if q.dim() != 3 or k.dim() != 3 or q.shape[0] != T or k.shape[0] != T or q.shape[2] != k.shape[2]:
        raise ValueError("q, k: [n_seq * seq_len, heads, head_dim] expected")
    if q.dtype != k.dtype:
        raise TypeError("q and k must have one type")
    hd = q.shape[2]
    if flags & QK_NO_NORM:
        q_weight = k_weight = None
    elif q_weight is None or k_weight is None:
        raise ValueError("weights are needed unless QK_NO_NORM is set")
    _vector(q_weight, hd, torch.float32, "q_weight")
    _vector(k_weight, hd, torch.float32, "k_weight")
    _vector(inv_freq, inv_freq.numel(), torch.float32, "inv_freq")
    _vector(positions, T, torch.int32, "positions")
    return q_weight, k_weight, _mask8(mask, T)


def qk_norm_rope(q: torch.Tensor, k: torch.Tensor, q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor],
                 inv_freq: torch.Tensor, n_seq: int, seq_len: int, positions: Optional[torch.Tensor] = None,
                 mask: Optional[torch.Tensor] = None, eps: float = 1e-6, flags: int = 0):
    """Norm of every head of q [T, Hq, D] and k [T, Hk, D], then rotation by position (2 * inv_freq.numel() elements of a
    head); returns contiguous (q_out, k_out).  q and k may be slices of one projection's rows."""
    n_seq, seq_len, eps, flags = _int(n_seq), _int(seq_len), _float(eps), _int(flags)
    q_weight, k_weight, mask = _qk_args(q, k, q_weight, k_weight, inv_freq, n_seq, seq_len, positions, mask, flags)
    dev = _one_device(q, k, q_weight, k_weight, inv_freq, positions, mask)
    with _on(dev):
        q_out, k_out = _new(q), _new(k)
        if q.shape[0]:
            desc, _ = _qk_plan(n_seq, seq_len, q.shape[1], k.shape[1], q.shape[2], q.dtype, 2 * inv_freq.numel(),
                               (_pitch(q, "q"), _pitch(k, "k")), eps, flags, False)
            rapid_qk_norm_rope_fwd(desc, q, k, q_weight, k_weight, inv_freq, positions, mask, q_out, k_out)
    return q_out, k_out


@dataclass
class QkGrads:
    dq: torch.Tensor                    # [T, Hq, D]
    dk: torch.Tensor                    # [T, Hk, D]
    dq_weight: Optional[torch.Tensor]   # like q_weight; None with QK_NO_NORM
    dk_weight: Optional[torch.Tensor]


def qk_norm_rope_grad(q: torch.Tensor, k: torch.Tensor, q_weight: Optional[torch.Tensor], k_weight: Optional[torch.Tensor],
                      inv_freq: torch.Tensor, dq_out: torch.Tensor, dk_out: torch.Tensor, n_seq: int, seq_len: int,
                      positions: Optional[torch.Tensor] = None, mask: Optional[torch.Tensor] = None, eps: float = 1e-6,
                      flags: int = 0, dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None) -> QkGrads:
    """The gradient of qk_norm_rope() from its inputs and the gradients of its outputs.  dq and dk may be given (slices of the
    gradient of one projection, say, or dq_out and dk_out themselves)."""
    n_seq, seq_len, eps, flags = _int(n_seq), _int(seq_len), _float(eps), _int(flags)
    q_weight, k_weight, mask = _qk_args(q, k, q_weight, k_weight, inv_freq, n_seq, seq_len, positions, mask, flags)
    if dq_out.shape != q.shape or dk_out.shape != k.shape:
        raise ValueError("dq_out, dk_out: the shapes of q and k expected")
    if dq_out.dtype != q.dtype or dk_out.dtype != k.dtype:
        raise TypeError("dq_out and dk_out must have the type of q and k")
    dev = _one_device(q, k, q_weight, k_weight, inv_freq, positions, mask, dq_out, dk_out, dq, dk)
    with _on(dev):
        T, hq, hd = q.shape
        hk = k.shape[1]
        dq, dk = _like(dq, q, "dq"), _like(dk, k, "dk")
        dw = (None, None) if flags & QK_NO_NORM else (_new(q_weight), _new(k_weight))
        if T == 0:
            for x in dw:
                if x is not None:
                    x.zero_()
            return QkGrads(dq, dk, *dw)
        pitches = (_pitch(q, "q"), _pitch(k, "k"), _pitch(dq_out, "dq_out"), _pitch(dk_out, "dk_out"), _pitch(dq, "dq"), _pitch(dk, "dk"))
        desc, ws_bytes = _qk_plan(n_seq, seq_len, hq, hk, hd, q.dtype, 2 * inv_freq.numel(), pitches, eps, flags, True)
        ws = q.new_empty(ws_bytes, dtype=torch.uint8) if ws_bytes else None
        rapid_qk_norm_rope_bwd(desc, q, k, q_weight, k_weight, inv_freq, positions, mask, dq_out, dk_out, dq, dk, dw[0], dw[1], ws)
    return QkGrads(dq, dk, *dw)


def make_attn_desc(n_seq: int, seq_len: int, n_heads: int, n_kv_heads: int, head_dim: int, window: int = 0,
                   scale: Optional[float] = None, ld_q: Optional[int] = None, ld_k: Optional[int] = None,
                   ld_v: Optional[int] = None, ld_out: Optional[int] = None, ld_dout: Optional[int] = None,
                   ld_dq: Optional[int] = None, ld_dk: Optional[int] = None, ld_dv: Optional[int] = None,
                   dtype: torch.dtype = torch.bfloat16, flags: int = 0) -> AttnDesc:
    _fits(flags, n_seq=n_seq, seq_len=seq_len, n_heads=n_heads, n_kv_heads=n_kv_heads, head_dim=head_dim, window=window)
    wq, wk = n_heads * head_dim, n_kv_heads * head_dim
    pitches = [w if ld is None else ld for w, ld in ((wq, ld_q), (wk, ld_k), (wk, ld_v), (wq, ld_out), (wq, ld_dout), (wq, ld_dq),
                                                     (wk, ld_dk), (wk, ld_dv))]
    return AttnDesc(n_seq, seq_len, n_heads, n_kv_heads, head_dim, window, *pitches, _dtype_code(dtype), flags,
                    max(head_dim, 1) ** -0.5 if scale is None else float(scale))


def rapid_attention_fwd(desc: AttnDesc, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, bounds: Optional[torch.Tensor],
                        out: torch.Tensor, lse: Optional[torch.Tensor], stats: Optional[torch.Tensor]) -> None:
    _check(lib().rapid_attention_fwd(C.byref(desc), _addr(q), _addr(k), _addr(v), _addr(bounds), _addr(out), _addr(lse), _addr(stats),
                                     _stream_here()), "rapid_attention_fwd")


def rapid_attention_bwd_workspace_bytes(desc: AttnDesc) -> int:
    return _workspace(lib().rapid_attention_bwd_workspace_bytes, desc, "rapid_attention_bwd_workspace_bytes")


def rapid_attention_bwd(desc: AttnDesc, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, bounds: Optional[torch.Tensor],
                        out: torch.Tensor, lse: torch.Tensor, dout: torch.Tensor, dq: torch.Tensor, dk: torch.Tensor,
                        dv: torch.Tensor, stats: Optional[torch.Tensor], workspace: torch.Tensor) -> None:
    _check(lib().rapid_attention_bwd(
        C.byref(desc), _addr(q), _addr(k), _addr(v), _addr(bounds), _addr(out), _addr(lse), _addr(dout), _addr(dq), _addr(dk), _addr(dv),
        _addr(stats), _addr(workspace), workspace.numel(), _stream_here()), "rapid_attention_bwd")


def _attn_args(q, k, v, n_seq, seq_len, bounds, stats):
    T = n_seq * seq_len
    if q.dim() != 3 or k.dim() != 3 or k.shape != v.shape or q.shape[0] != T or k.shape[0] != T or q.shape[2] != k.shape[2]:
        raise ValueError("q: [n_seq * seq_len, heads, head_dim], k, v: [n_seq * seq_len, kv_heads, head_dim] expected")
    if not q.dtype == k.dtype == v.dtype == torch.bfloat16:
        raise TypeError("q, k and v must be bfloat16")
    _vector(bounds, 2 * n_seq, torch.int32, "bounds")
    _stats_room(stats)


def attention(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, n_seq: int, seq_len: int, bounds: Optional[torch.Tensor] = None,
              window: int = 0, scale: Optional[float] = None, stats: Optional[torch.Tensor] = None):
    """Causal attention over the padded token grid, q [T, H, D], k and v [T, Hk, D] bfloat16 (rows may be slices of one
    projection); bounds [n_seq, 2] int32 gives each generation's live positions.  Returns out [T, H, D] and lse
    [n_seq, H, seq_len] float32.  The default scale is D ** -0.5.  A wait that gives up is reported in stats (alloc_stats, read_stats)
    and nowhere else."""
    n_seq, seq_len, window, scale = _int(n_seq), _int(seq_len), _int(window), None if scale is None else _float(scale)
    _attn_args(q, k, v, n_seq, seq_len, bounds, stats)
    dev = _one_device(q, k, v, bounds, stats)
    with _on(dev):
        out = _new(q)
        lse = q.new_empty((n_seq, q.shape[1], seq_len), dtype=torch.float32)
        if q.shape[0]:
            desc, _ = _attn_plan(n_seq, seq_len, q.shape[1], k.shape[1], q.shape[2], window, scale,
                                 (_pitch(q, "q"), _pitch(k, "k"), _pitch(v, "v")), False)
            rapid_attention_fwd(desc, q, k, v, bounds, out, lse, stats)
        elif stats is not None:
            stats.zero_()
    return out, lse


@dataclass
class AttnGrads:
    dq: torch.Tensor  # [T, H, D]
    dk: torch.Tensor  # [T, Hk, D]
    dv: torch.Tensor  # [T, Hk, D]


def attention_grad(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, out: torch.Tensor, lse: torch.Tensor, dout: torch.Tensor,
                   n_seq: int, seq_len: int, bounds: Optional[torch.Tensor] = None, window: int = 0, scale: Optional[float] = None,
                   stats: Optional[torch.Tensor] = None, dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None,
                   dv: Optional[torch.Tensor] = None) -> AttnGrads:
    """The gradient of attention() from its inputs, its outputs out and lse, and the gradient of out.  dq, dk and dv may be
    given (slices of the gradient of one projection, say).  stats as in attention()."""
    n_seq, seq_len, window, scale = _int(n_seq), _int(seq_len), _int(window), None if scale is None else _float(scale)
    _attn_args(q, k, v, n_seq, seq_len, bounds, stats)
    if out.shape != q.shape or dout.shape != q.shape:
        raise ValueError("out, dout: the shape of q expected")
    if not out.dtype == dout.dtype == torch.bfloat16:
        raise TypeError("out and dout must be bfloat16")
    _vector(lse, q.shape[0] * q.shape[1], torch.float32, "lse")
    dev = _one_device(q, k, v, out, lse, dout, bounds, stats, dq, dk, dv)
    with _on(dev):
        dq, dk, dv = _like(dq, q, "dq"), _like(dk, k, "dk"), _like(dv, v, "dv")
        if q.shape[0]:
            pitches = (_pitch(q, "q"), _pitch(k, "k"), _pitch(v, "v"), _pitch(out, "out"), _pitch(dout, "dout"), _pitch(dq, "dq"),
                       _pitch(dk, "dk"), _pitch(dv, "dv"))
            desc, ws_bytes = _attn_plan(n_seq, seq_len, q.shape[1], k.shape[1], q.shape[2], window, scale, pitches, True)
            ws = q.new_empty(ws_bytes, dtype=torch.uint8)
            rapid_attention_bwd(desc, q, k, v, bounds, out, lse, dout, dq, dk, dv, stats, ws)
        elif stats is not None:
            stats.zero_()
    return AttnGrads(dq, dk, dv)


# ---- further losses over the logits (include/rapid_losses.h) ------------------------------------------------------
#
# rapid_clip_loss(), rapid_preference_loss() and rapid_distill_loss() marshal the arguments of the C calls; clip_loss(),
# preference_loss() and distill_loss() check shapes and types, allocate the outputs and the workspace and make one call.


def read_loss_stats(stats: torch.Tensor) -> dict:
    """Copy a device rapid_loss_stats_t (alloc_stats) to the host (synchronises) and return it as a dict."""
    s = LossStats.from_buffer_copy(bytes(stats.cpu().numpy().tobytes())[:STATS_BYTES])
    return {k: getattr(s, k) for k, _ in LossStats._fields_}


def make_clip_desc(n_seq: int, seq_len: int, vocab: int, dtype: torch.dtype, ld: Optional[int] = None, ld_grad: Optional[int] = None,
                   eps_low: float = 0.2, eps_high: float = 0.2, kl_beta: float = 0.0, scale: float = 1.0, flags: int = 0,
                   norm_z: float = 0.0) -> ClipDesc:
    _fits(flags, n_seq=n_seq, seq_len=seq_len, vocab=vocab)
    ld = vocab if ld is None else ld
    return ClipDesc(n_seq, seq_len, vocab, _dtype_code(dtype), ld, ld if ld_grad is None else ld_grad, flags, 0, float(eps_low), float(eps_high),
                    float(kl_beta), float(scale), float(norm_z))


def make_pref_desc(n_seq: int, seq_len: int, vocab: int, dtype: torch.dtype, n_pairs: int, ld: Optional[int] = None,
                   ld_grad: Optional[int] = None, beta: float = 0.1, margin: float = 0.0, label_smoothing: float = 0.0, scale: float = 1.0,
                   flags: int = 0, norm_z: float = 0.0) -> PrefDesc:
    _fits(flags, n_seq=n_seq, seq_len=seq_len, vocab=vocab, n_pairs=n_pairs)
    ld = vocab if ld is None else ld
    return PrefDesc(n_seq, seq_len, vocab, _dtype_code(dtype), ld, ld if ld_grad is None else ld_grad, flags, n_pairs, float(beta), float(margin),
                    float(label_smoothing), float(scale), float(norm_z))


def make_distill_desc(n_rows: int, vocab: int, k: int, dtype: torch.dtype, ld: Optional[int] = None, ld_grad: Optional[int] = None,
                      ld_top: Optional[int] = None, temperature: float = 1.0, scale: float = 1.0, flags: int = 0,
                      norm_z: float = 0.0) -> DistillDesc:
    _fits(flags, vocab=vocab, k=k)
    ld = vocab if ld is None else ld
    return DistillDesc(n_rows, vocab, k, ld, ld if ld_grad is None else ld_grad, k if ld_top is None else ld_top, _dtype_code(dtype), flags,
                       float(temperature), float(scale), float(norm_z))


def rapid_clip_loss_workspace_bytes(desc: ClipDesc) -> int:
    return _workspace(lib().rapid_clip_loss_workspace_bytes, desc, "rapid_clip_loss_workspace_bytes")


def rapid_clip_loss(desc: ClipDesc, logits: torch.Tensor, targets: torch.Tensor, mask: Optional[torch.Tensor], old_logp: torch.Tensor,
                    ref_logp: Optional[torch.Tensor], adv: torch.Tensor, dlogits: Optional[torch.Tensor], loss: torch.Tensor,
                    token_logp: Optional[torch.Tensor], stats: Optional[torch.Tensor], workspace: torch.Tensor) -> None:
    _check(lib().rapid_clip_loss(C.byref(desc), _addr(logits), _addr(targets), _addr(mask), _addr(old_logp), _addr(ref_logp), _addr(adv),
                                 _addr(dlogits), _addr(loss), _addr(token_logp), _addr(stats), _addr(workspace), workspace.numel(),
                                 _stream_here()), "rapid_clip_loss")


def rapid_preference_loss_workspace_bytes(desc: PrefDesc) -> int:
    return _workspace(lib().rapid_preference_loss_workspace_bytes, desc, "rapid_preference_loss_workspace_bytes")


def rapid_preference_loss(desc: PrefDesc, logits: torch.Tensor, targets: torch.Tensor, mask: Optional[torch.Tensor], pairs: torch.Tensor,
                          ref_logp: Optional[torch.Tensor], dlogits: Optional[torch.Tensor], loss: torch.Tensor,
                          margins: Optional[torch.Tensor], token_logp: Optional[torch.Tensor], stats: Optional[torch.Tensor],
                          workspace: torch.Tensor) -> None:
    _check(lib().rapid_preference_loss(C.byref(desc), _addr(logits), _addr(targets), _addr(mask), _addr(pairs), _addr(ref_logp),
                                       _addr(dlogits), _addr(loss), _addr(margins), _addr(token_logp), _addr(stats), _addr(workspace),
                                       workspace.numel(), _stream_here()), "rapid_preference_loss")


def rapid_distill_loss_workspace_bytes(desc: DistillDesc) -> int:
    return _workspace(lib().rapid_distill_loss_workspace_bytes, desc, "rapid_distill_loss_workspace_bytes")


def rapid_distill_loss(desc: DistillDesc, logits: torch.Tensor, top_index: torch.Tensor, top_logit: torch.Tensor,
                       top_lse: Optional[torch.Tensor], mask: Optional[torch.Tensor], dlogits: Optional[torch.Tensor], loss: torch.Tensor,
                       token_loss: Optional[torch.Tensor], stats: Optional[torch.Tensor], workspace: torch.Tensor) -> None:
    _check(lib().rapid_distill_loss(C.byref(desc), _addr(logits), _addr(top_index), _addr(top_logit), _addr(top_lse), _addr(mask),
                                    _addr(dlogits), _addr(loss), _addr(token_loss), _addr(stats), _addr(workspace), workspace.numel(),
                                    _stream_here()), "rapid_distill_loss")


@functools.lru_cache(maxsize=512)
def _clip_plan(n_seq, seq_len, vocab, dtype, ld, ld_grad, eps_low, eps_high, kl_beta, scale, flags, norm_z):
    desc = make_clip_desc(n_seq, seq_len, vocab, dtype, ld, ld_grad, eps_low, eps_high, kl_beta, scale, flags, norm_z)
    return desc, rapid_clip_loss_workspace_bytes(desc)


@functools.lru_cache(maxsize=512)
def _pref_plan(n_seq, seq_len, vocab, dtype, n_pairs, ld, ld_grad, beta, margin, label_smoothing, scale, flags, norm_z):
    desc = make_pref_desc(n_seq, seq_len, vocab, dtype, n_pairs, ld, ld_grad, beta, margin, label_smoothing, scale, flags, norm_z)
    return desc, rapid_preference_loss_workspace_bytes(desc)


@functools.lru_cache(maxsize=512)
def _distill_plan(n_rows, vocab, k, dtype, ld, ld_grad, ld_top, temperature, scale, flags, norm_z):
    desc = make_distill_desc(n_rows, vocab, k, dtype, ld, ld_grad, ld_top, temperature, scale, flags, norm_z)
    return desc, rapid_distill_loss_workspace_bytes(desc)


def _loss_args(logits, n_rows, mask, stats, want_grad, in_place):
    if logits.dim() != 2 or logits.shape[0] != n_rows:
        raise ValueError("logits: a matrix of one row for each position expected")
    if n_rows <= 0 or logits.shape[1] <= 0:
        raise ValueError("logits: at least one row and one column expected")
    if in_place and not want_grad:
        raise ValueError("in_place: there is no gradient to put in the place of the logits")
    _stats_room(stats)
    return _mask8(mask, n_rows)


def _loss_grad(logits, want_grad, in_place):
    return None if not want_grad else logits if in_place else _matrix(logits.shape[0], logits.shape[1], logits.dtype, logits)


@dataclass
class ClipResult:
    loss: torch.Tensor               # [1] float32
    dlogits: Optional[torch.Tensor]  # [T, V], None without want_grad
    token_logp: torch.Tensor         # [T] float32


def clip_loss(logits: torch.Tensor, targets: torch.Tensor, mask: Optional[torch.Tensor], old_logp: torch.Tensor, adv: torch.Tensor,
              n_seq: int, seq_len: int, ref_logp: Optional[torch.Tensor] = None, eps_low: float = 0.2, eps_high: float = 0.2,
              kl_beta: float = 0.0, scale: float = 1.0, flags: int = 0, norm_z: float = 0.0, want_grad: bool = True, in_place: bool = False,
              stats: Optional[torch.Tensor] = None) -> ClipResult:
    """Clipped policy loss over the token grid, logits [T, V], with a KL term to ref_logp where kl_beta > 0, and its gradient by the
    logits.  adv holds an advantage for each generation, or (T of them) for each row.  Weights of the rows: one over their number,
    or by LOSS_NORM_SEQ / LOSS_NORM_GIVEN in flags.  stats (alloc_stats, read_loss_stats) gets the side statistics."""
    n_seq, seq_len, flags = _int(n_seq), _int(seq_len), _int(flags)
    T = n_seq * seq_len
    mask = _loss_args(logits, T, mask, stats, want_grad, in_place)
    _vector(targets, T, torch.int32, "targets")
    _vector(old_logp, T, torch.float32, "old_logp")
    _vector(ref_logp, T, torch.float32, "ref_logp")
    if adv.numel() not in (n_seq, T):
        raise ValueError("adv: one element for each generation or for each row expected")
    by_token = adv.numel() != n_seq or bool(flags & CLIP_ADV_TOKEN)
    _vector(adv, T if by_token else n_seq, torch.float32, "adv")
    flags |= CLIP_ADV_TOKEN if by_token else 0
    dev = _one_device(logits, targets, mask, old_logp, ref_logp, adv, stats)
    with _on(dev):
        ld = _pitch(logits, "logits")
        dlogits = _loss_grad(logits, want_grad, in_place)
        desc, ws_bytes = _clip_plan(n_seq, seq_len, logits.shape[1], logits.dtype, ld, ld if dlogits is None else _pitch(dlogits, "dlogits"),
                                    _float(eps_low), _float(eps_high), _float(kl_beta), _float(scale), flags, _float(norm_z))
        loss, token_logp = old_logp.new_empty(1), _new(old_logp)
        rapid_clip_loss(desc, logits, targets, mask, old_logp, ref_logp, adv, dlogits, loss, token_logp, stats,
                        logits.new_empty(ws_bytes, dtype=torch.uint8))
    return ClipResult(loss, dlogits, token_logp)


@dataclass
class PrefResult:
    loss: torch.Tensor               # [1] float32
    dlogits: Optional[torch.Tensor]  # [T, V], None without want_grad
    margins: torch.Tensor            # [P] float32, h of every pair
    token_logp: torch.Tensor         # [T] float32


def preference_loss(logits: torch.Tensor, targets: torch.Tensor, mask: Optional[torch.Tensor], pairs: torch.Tensor, n_seq: int,
                    seq_len: int, ref_logp: Optional[torch.Tensor] = None, beta: float = 0.1, margin: float = 0.0,
                    label_smoothing: float = 0.0, scale: float = 1.0, flags: int = 0, norm_z: float = 0.0, want_grad: bool = True,
                    in_place: bool = False, stats: Optional[torch.Tensor] = None) -> PrefResult:
    """Preference loss over pairs [P, 2] int32 of generations (preferred, other) of the token grid, logits [T, V], and its gradient
    by the logits.  flags: PREF_HINGE or PREF_SQUARED instead of the logistic form, PREF_TOKEN_MEAN, LOSS_NORM_GIVEN."""
    n_seq, seq_len, flags = _int(n_seq), _int(seq_len), _int(flags)
    T = n_seq * seq_len
    mask = _loss_args(logits, T, mask, stats, want_grad, in_place)
    _vector(targets, T, torch.int32, "targets")
    _vector(ref_logp, T, torch.float32, "ref_logp")
    if pairs.dim() != 2 or pairs.shape[1] != 2 or pairs.shape[0] == 0:
        raise ValueError("pairs: [P, 2] expected")
    P = pairs.shape[0]
    _vector(pairs, 2 * P, torch.int32, "pairs")
    dev = _one_device(logits, targets, mask, pairs, ref_logp, stats)
    with _on(dev):
        ld = _pitch(logits, "logits")
        dlogits = _loss_grad(logits, want_grad, in_place)
        desc, ws_bytes = _pref_plan(n_seq, seq_len, logits.shape[1], logits.dtype, P, ld, ld if dlogits is None else _pitch(dlogits, "dlogits"),
                                    _float(beta), _float(margin), _float(label_smoothing), _float(scale), flags, _float(norm_z))
        loss, margins, token_logp = (logits.new_empty(n, dtype=torch.float32) for n in (1, P, T))
        rapid_preference_loss(desc, logits, targets, mask, pairs, ref_logp, dlogits, loss, margins, token_logp, stats,
                              logits.new_empty(ws_bytes, dtype=torch.uint8))
    return PrefResult(loss, dlogits, margins, token_logp)


@dataclass
class DistillResult:
    loss: torch.Tensor               # [1] float32
    dlogits: Optional[torch.Tensor]  # [T, V], None without want_grad
    token_loss: torch.Tensor         # [T] float32


def distill_loss(logits: torch.Tensor, top_index: torch.Tensor, top_logit: torch.Tensor, mask: Optional[torch.Tensor] = None,
                 top_lse: Optional[torch.Tensor] = None, temperature: float = 1.0, scale: float = 1.0, flags: int = 0, norm_z: float = 0.0,
                 want_grad: bool = True, in_place: bool = False, stats: Optional[torch.Tensor] = None) -> DistillResult:
    """Divergence of the student's logits [T, V] from a teacher's top ones, top_index [T, K] int32 (negative: no entry) and top_logit
    [T, K] float32, and its gradient by the logits.  With top_lse [T], the teacher's log-sum-exp of logits / temperature over its whole
    vocabulary, the tokens outside the list are one outcome more; without it the list is all of the teacher's probability."""
    flags = _int(flags)
    T = logits.shape[0]
    mask = _loss_args(logits, T, mask, stats, want_grad, in_place)
    if top_index.dim() != 2 or top_index.shape != top_logit.shape or top_index.shape[0] != T or top_index.shape[1] == 0:
        raise ValueError("top_index, top_logit: [T, K] expected")
    if top_index.dtype != torch.int32 or top_logit.dtype != torch.float32:
        raise TypeError("top_index must be int32 and top_logit float32")
    K = top_index.shape[1]
    for x, name in ((top_index, "top_index"), (top_logit, "top_logit")):
        if K > 1 and x.stride(1) != 1:
            raise ValueError(f"{name}: the elements of a row must lie side by side")
    pitch = K if T == 1 else top_index.stride(0)
    if T > 1 and top_logit.stride(0) != pitch:
        raise ValueError("top_index and top_logit must have one row pitch")
    _vector(top_lse, T, torch.float32, "top_lse")
    dev = _one_device(logits, top_index, top_logit, top_lse, mask, stats)
    with _on(dev):
        ld = _pitch(logits, "logits")
        dlogits = _loss_grad(logits, want_grad, in_place)
        desc, ws_bytes = _distill_plan(T, logits.shape[1], K, logits.dtype, ld, ld if dlogits is None else _pitch(dlogits, "dlogits"), pitch,
                                       _float(temperature), _float(scale), flags, _float(norm_z))
        loss, token_loss = (logits.new_empty(n, dtype=torch.float32) for n in (1, T))
        rapid_distill_loss(desc, logits, top_index, top_logit, top_lse, mask, dlogits, loss, token_loss, stats,
                           logits.new_empty(ws_bytes, dtype=torch.uint8))
    return DistillResult(loss, dlogits, token_loss)
