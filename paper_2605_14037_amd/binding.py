"""Thin ctypes binding of include/spkv.h: argument marshalling only.

Every step of the path runs in the library's HIP kernels; PyTorch supplies device
memory (the arena and the tensors) and the current stream.
"""

from __future__ import annotations

import ctypes as C
import itertools
import os
import struct
import threading

import torch

HERE = os.path.dirname(os.path.abspath(__file__))
_LIB = None

OK, E_INVAL, E_STATE, E_CAPACITY, E_HIP, E_NOMEM, E_DEVICE = 0, -1, -2, -3, -4, -5, -6
OPT_ITEM_TARGET, OPT_KERNEL_TIMING, OPT_SPLIT_ONLY, OPT_SINK_TOKENS, OPT_MERGE_WAVES = 1, 2, 3, 4, 5
OPT_STEP_LAUNCHES = 6
MAX_BATCH, PAGE_TOKENS, MAX_TREE_NODES = 512, 64, 64
FORK_KEEP, FORK_EMPTY = -1, -2

EXPORTED_SYMBOLS = [
    "spkv_cache_required_bytes", "spkv_cache_create", "spkv_cache_destroy", "spkv_cache_grow",
    "spkv_cache_reset",
    "spkv_append", "spkv_decode_attention", "spkv_decode_attention_static", "spkv_decode_step",
    "spkv_decode_chunk",
    "spkv_decode_step_predict_workspace_bytes", "spkv_decode_step_predict", "spkv_score_chunk",
    "spkv_prefill_workspace_bytes", "spkv_prefill_attention",
    "spkv_soft_gated_workspace_bytes", "spkv_soft_gated_attention", "spkv_cache_release_sequence", "spkv_utility_logits", "spkv_cache_safe_steps", "spkv_cache_advance", "spkv_cache_stats", "spkv_cache_kept_positions",
    "spkv_cache_threshold_logit", "spkv_cache_set_tau", "spkv_cache_prune", "spkv_cache_set_option", "spkv_cache_read_kernel_timing",
    "spkv_debug_layout_offset", "spkv_debug_copy", "spkv_debug_read", "spkv_strerror",
    "spkv_qk_norm_rope", "spkv_qk_norm_rope_backward", "spkv_qk_norm_rope_backward_workspace_bytes",
    "spkv_prefix_workspace_bytes", "spkv_prefix_attention", "spkv_decode_attention_shared",
    "spkv_score_tree", "spkv_append_rows", "spkv_cache_fork", "spkv_cache_gather",
]

BF16, FP32 = 0, 1
_HEAD_TYPES = {torch.bfloat16: BF16, torch.float32: FP32}


class SPKVConfig(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("window", C.c_int32), ("page_tokens", C.c_int32),
                ("tau", C.c_float), ("max_context", C.c_int32),
                ("max_total_kept_tokens", C.c_int64)]


class SPKVStats(C.Structure):
    _fields_ = [("total_tokens", C.c_int64), ("evicted_tokens", C.c_int64),
                ("window_tokens", C.c_int64), ("kept_tokens", C.c_int64),
                ("gate_on_tokens", C.c_int64), ("density_evicted", C.c_double),
                ("density_all", C.c_double), ("kept_kv_bytes", C.c_int64),
                ("dense_kv_bytes", C.c_int64), ("pool_pages_used", C.c_int64),
                ("pool_pages_total", C.c_int64), ("arena_bytes", C.c_int64),
                ("device_error", C.c_int32), ("n_work_items", C.c_int32),
                ("n_work_items_last_call", C.c_int32), ("reserved_", C.c_int32)]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class SPKVRope(C.Structure):
    _fields_ = [("head_dim", C.c_int32), ("rot_dim", C.c_int32), ("adjacent", C.c_int32),
                ("n_axes", C.c_int32), ("inv_freq", C.c_void_p), ("axis", C.c_void_p)]


class SPKVError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} ({code})")


def library_path():
    return os.path.join(HERE, "libspkv.so")


def load_library():
    """Load libspkv.so once and declare the prototypes of include/spkv.h."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = library_path()
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it first "
                           "(python -m paper_2605_14037_amd.build); there is no fallback path")
    lib = C.CDLL(path)
    vp, i32, i64, f32 = C.c_void_p, C.c_int32, C.c_int64, C.c_float
    P = C.POINTER
    lib.spkv_cache_required_bytes.restype = C.c_size_t
    lib.spkv_cache_required_bytes.argtypes = [P(SPKVConfig)]
    lib.spkv_cache_create.restype = C.c_int
    lib.spkv_cache_create.argtypes = [P(SPKVConfig), vp, C.c_size_t, vp, P(vp)]
    lib.spkv_cache_destroy.restype = C.c_int
    lib.spkv_cache_destroy.argtypes = [vp]
    lib.spkv_cache_grow.restype = C.c_int
    lib.spkv_cache_grow.argtypes = [vp, P(SPKVConfig), vp, C.c_size_t, vp]
    lib.spkv_cache_reset.restype = C.c_int
    lib.spkv_cache_reset.argtypes = [vp, vp]
    lib.spkv_append.restype = C.c_int
    lib.spkv_append.argtypes = [vp, vp, vp, vp, P(i32), vp]
    lib.spkv_decode_attention.restype = C.c_int
    lib.spkv_decode_attention.argtypes = [vp, vp, vp, vp, f32, vp]
    lib.spkv_decode_attention_static.restype = C.c_int
    lib.spkv_decode_attention_static.argtypes = [vp, vp, vp, vp, f32, vp]
    lib.spkv_decode_step.restype = C.c_int
    lib.spkv_decode_step.argtypes = [vp, vp, vp, vp, vp, vp, vp, f32, vp]
    lib.spkv_decode_step_predict_workspace_bytes.restype = C.c_size_t
    lib.spkv_decode_step_predict_workspace_bytes.argtypes = [i32, i32]
    lib.spkv_decode_step_predict.restype = C.c_int
    lib.spkv_decode_step_predict.argtypes = [vp, vp, vp, vp, vp, vp, i32, i32, vp, vp, vp, vp, vp,
                                             vp, vp, C.c_size_t, f32, vp]
    lib.spkv_decode_chunk.restype = C.c_int
    lib.spkv_decode_chunk.argtypes = [vp, vp, vp, vp, vp, P(i32), vp, vp, f32, vp]
    lib.spkv_score_chunk.restype = C.c_int
    lib.spkv_score_chunk.argtypes = [vp, vp, vp, vp, P(i32), vp, vp, f32, vp]
    lib.spkv_prefill_workspace_bytes.restype = C.c_size_t
    lib.spkv_prefill_workspace_bytes.argtypes = [vp, i32, i64]
    lib.spkv_prefill_attention.restype = C.c_int
    lib.spkv_prefill_attention.argtypes = [vp, vp, vp, vp, vp, P(i32), vp, vp, f32, vp, C.c_size_t, vp]
    lib.spkv_soft_gated_workspace_bytes.restype = C.c_size_t
    lib.spkv_soft_gated_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
    lib.spkv_soft_gated_attention.restype = C.c_int
    lib.spkv_soft_gated_attention.argtypes = [vp, vp, vp, vp, P(i32), i32, i32, i32, i32, i32, vp, vp,
                                              f32, vp, C.c_size_t, vp]
    lib.spkv_cache_release_sequence.restype = C.c_int
    lib.spkv_cache_release_sequence.argtypes = [vp, i32, vp]
    lib.spkv_utility_logits.restype = C.c_int
    lib.spkv_utility_logits.argtypes = [vp, vp, vp, vp, vp, vp, vp, i32, i32, i32, i32, vp]
    lib.spkv_prefix_workspace_bytes.restype = C.c_size_t
    lib.spkv_prefix_workspace_bytes.argtypes = [vp, i64]
    lib.spkv_prefix_attention.restype = C.c_int
    lib.spkv_prefix_attention.argtypes = [vp, vp, P(i32), vp, P(i32), i32, vp, vp, vp, vp, f32, vp, C.c_size_t, vp]
    lib.spkv_decode_attention_shared.restype = C.c_int
    lib.spkv_decode_attention_shared.argtypes = [vp, vp, P(i32), vp, vp, vp, f32, vp, C.c_size_t, vp]
    ph, pr = vp, P(SPKVRope)                 # (heads: addresses into one block of memory, see _block)
    lib.spkv_qk_norm_rope.restype = C.c_int
    lib.spkv_qk_norm_rope.argtypes = [ph, ph, ph, vp, vp, f32, vp, pr, i32, i64, i32, i32, ph, ph, ph, vp]
    lib.spkv_qk_norm_rope_backward_workspace_bytes.restype = C.c_size_t
    lib.spkv_qk_norm_rope_backward_workspace_bytes.argtypes = [i64, i32, i32, i32]
    lib.spkv_qk_norm_rope_backward.restype = C.c_int
    lib.spkv_qk_norm_rope_backward.argtypes = [ph, ph, ph, ph, ph, vp, vp, f32, vp, pr, i32, i64, i32, i32,
                                               ph, ph, ph, vp, vp, vp, C.c_size_t, vp]
    lib.spkv_score_tree.restype = C.c_int
    lib.spkv_score_tree.argtypes = [vp, vp, vp, vp, vp, vp, P(i32), vp, vp, f32, vp]
    lib.spkv_append_rows.restype = C.c_int
    lib.spkv_append_rows.argtypes = [vp, vp, vp, vp, vp, i32, P(i32), vp]
    lib.spkv_cache_fork.restype = C.c_int
    lib.spkv_cache_fork.argtypes = [vp, vp, P(i32), vp]
    lib.spkv_cache_gather.restype = C.c_int
    lib.spkv_cache_gather.argtypes = [vp, P(i32), i32, i64, vp, vp, vp, vp, vp, vp]
    lib.spkv_cache_prune.restype = C.c_int
    lib.spkv_cache_prune.argtypes = [vp, vp]
    lib.spkv_cache_safe_steps.restype = C.c_int
    lib.spkv_cache_safe_steps.argtypes = [vp, vp, P(i64)]
    lib.spkv_cache_advance.restype = C.c_int
    lib.spkv_cache_advance.argtypes = [vp, i64]
    lib.spkv_cache_stats.restype = C.c_int
    lib.spkv_cache_stats.argtypes = [vp, P(SPKVStats), P(i32), vp]
    lib.spkv_cache_kept_positions.restype = C.c_int
    lib.spkv_cache_kept_positions.argtypes = [vp, i32, i32, P(i32), i32, P(i32), vp]
    lib.spkv_cache_threshold_logit.restype = C.c_int
    lib.spkv_cache_threshold_logit.argtypes = [vp, P(f32)]
    lib.spkv_cache_set_tau.restype = C.c_int
    lib.spkv_cache_set_tau.argtypes = [vp, f32]
    lib.spkv_cache_set_option.restype = C.c_int
    lib.spkv_cache_set_option.argtypes = [vp, i32, i64]
    lib.spkv_cache_read_kernel_timing.restype = C.c_int
    lib.spkv_cache_read_kernel_timing.argtypes = [vp, P(f32), i32, P(i32)]
    lib.spkv_debug_layout_offset.restype = i64
    lib.spkv_debug_layout_offset.argtypes = [i32, i32, i32, i32]
    lib.spkv_debug_copy.restype = C.c_int
    lib.spkv_debug_copy.argtypes = [vp, vp, C.c_size_t, vp]
    lib.spkv_debug_read.restype = C.c_int
    lib.spkv_debug_read.argtypes = [vp, C.c_size_t, i32, i64, i64, i64, i32, vp, vp]
    lib.spkv_strerror.restype = C.c_char_p
    lib.spkv_strerror.argtypes = [C.c_int]
    _LIB = lib
    return lib


def strerror(code):
    return load_library().spkv_strerror(int(code)).decode()


def required_bytes(cfg: SPKVConfig) -> int:
    return int(load_library().spkv_cache_required_bytes(C.byref(cfg)))


def layout_offset(head_dim, is_v, kidx, d) -> int:
    return int(load_library().spkv_debug_layout_offset(head_dim, int(is_v), kidx, d))


def debug_copy(dst: torch.Tensor, src: torch.Tensor):
    """Plain copy kernel of known traffic (src.nbytes read + written); see spkv_debug_copy."""
    nbytes = src.numel() * src.element_size()
    if not (dst.is_cuda and src.is_cuda and dst.is_contiguous() and src.is_contiguous()
            and dst.numel() * dst.element_size() == nbytes):
        raise ValueError("debug_copy: need contiguous cuda tensors of equal byte size")
    _check(load_library().spkv_debug_copy(C.c_void_p(dst.data_ptr()), C.c_void_p(src.data_ptr()),
                                          nbytes, _stream()), "spkv_debug_copy")


def debug_read(src: torch.Tensor, run_bytes, first_run, n_runs, stride, n_workgroups, sink):
    """Plain streaming read with the decode kernel's launch shape (spkv_debug_read)."""
    if not (src.is_cuda and src.is_contiguous() and sink.is_cuda and sink.is_contiguous()
            and sink.numel() * sink.element_size() >= n_workgroups * 1024):
        raise ValueError("debug_read: need contiguous cuda tensors, sink of n_workgroups KB")
    _check(load_library().spkv_debug_read(C.c_void_p(src.data_ptr()), src.numel() * src.element_size(),
                                          int(run_bytes), int(first_run), int(n_runs), int(stride),
                                          int(n_workgroups), C.c_void_p(sink.data_ptr()), _stream()),
           "spkv_debug_read")


def soft_gated_attention(q, k, v, util_logits, cu_seqlens, window=128, sm_scale=0.0, out=None,
                         want_lse=False, workspace=None):
    """Soft-gated attention forward over packed sequences (spkv_soft_gated_attention).
    q: bf16 [total, H_q, D]; k, v: bf16 [total, H_kv, D]; util_logits: fp32 [total, H_kv]."""
    lib = load_library()
    total, Hq, D = q.shape
    Hkv = k.shape[1]
    batch = len(cu_seqlens) - 1
    cu = (C.c_int32 * (batch + 1))(*[int(x) for x in cu_seqlens])
    if cu[batch] != total:
        raise ValueError("cu_seqlens does not cover the rows")
    qp = _dev_ptr(q, torch.bfloat16, (total, Hq, D), "q")
    kp = _dev_ptr(k, torch.bfloat16, (total, Hkv, D), "k")
    vp = _dev_ptr(v, torch.bfloat16, (total, Hkv, D), "v")
    fp = _dev_ptr(util_logits, torch.float32, (total, Hkv), "util_logits")
    n_max = max(cu[b + 1] - cu[b] for b in range(batch))
    if workspace is None:
        need = int(lib.spkv_soft_gated_workspace_bytes(batch, Hkv, D, int(window), max(n_max, 1)))
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=q.device)
    if out is None:
        out = torch.empty_like(q)
    op = _dev_ptr(out, torch.bfloat16, (total, Hq, D), "out")
    lse = torch.empty((total, Hq), dtype=torch.float32, device=q.device) if want_lse else None
    lp = _dev_ptr(lse, torch.float32, (total, Hq), "lse") if lse is not None else None
    _check(lib.spkv_soft_gated_attention(qp, kp, vp, fp, cu, batch, Hq, Hkv, D, int(window), op, lp,
                                         float(sm_scale), workspace.data_ptr(), workspace.numel(),
                                         _stream()), "spkv_soft_gated_attention")
    return (out, lse) if want_lse else out


def utility_logits(hidden, w1, b1, w2, b2, out=None, workspace=None):
    """Pre-sigmoid utility logits of the two-layer predictor (spkv_utility_logits)."""
    n, d_model = hidden.shape
    d_hidden, n_heads = w1.shape[0], w2.shape[0]
    hp = _dev_ptr(hidden, torch.bfloat16, (n, d_model), "hidden")
    w1p = _dev_ptr(w1, torch.bfloat16, (d_hidden, d_model), "w1")
    w2p = _dev_ptr(w2, torch.bfloat16, (n_heads, d_hidden), "w2")
    b1p = _dev_ptr(b1, torch.float32, (d_hidden,), "b1") if b1 is not None else None
    b2p = _dev_ptr(b2, torch.float32, (n_heads,), "b2") if b2 is not None else None
    if out is None:
        out = torch.empty(n, n_heads, dtype=torch.float32, device=hidden.device)
    if workspace is None:
        workspace = torch.empty(max(1, n * d_hidden), dtype=torch.float32, device=hidden.device)
    op = _dev_ptr(out, torch.float32, (n, n_heads), "logits")
    _check(load_library().spkv_utility_logits(hp, w1p, b1p, w2p, b2p, op,
                                              C.c_void_p(workspace.data_ptr()), n, d_model,
                                              d_hidden, n_heads, _stream()), "spkv_utility_logits")
    return out


class Rope:
    """Rotation of heads by positions (spkv_rope_t): which elements form pairs, how fast each pair turns
    and with which axis of the positions.  Made once per model, host memory only.

    rot_dim elements of a head are rotated (all by default).  Pair i turns by theta ** (-2 i / rot_dim), or
    inv_freq[i], radians per position.  sections = pairs of every axis in order (time, height, width), or
    axis[i] = the axis of each pair.  adjacent: pair i is elements (2 i, 2 i + 1) instead of
    (i, i + rot_dim / 2)."""

    def __init__(self, head_dim, rot_dim=None, theta=10000.0, sections=None, axis=None, adjacent=False,
                 inv_freq=None):
        self.head_dim = int(head_dim)
        self.rot_dim = self.head_dim if rot_dim is None else int(rot_dim)
        pairs = self.rot_dim // 2
        if inv_freq is None:
            inv_freq = [float(theta) ** (-2.0 * i / self.rot_dim) for i in range(pairs)]
        inv_freq = [float(f) for f in inv_freq]
        if sections is not None:
            if axis is not None:
                raise ValueError("rope: sections or axis, not both")
            axis = [a for a, n in enumerate(sections) for _ in range(int(n))]
            self.n_axes = len(sections)
        else:
            axis = [0] * pairs if axis is None else [int(a) for a in axis]
            self.n_axes = max(axis, default=0) + 1
        if len(inv_freq) != pairs or len(axis) != pairs or any(not 0 <= a < 256 for a in axis):
            raise ValueError(f"rope: need a frequency and an axis for each of {pairs} pairs")
        self.adjacent = bool(adjacent)
        self._freq = (C.c_double * max(pairs, 1))(*inv_freq)
        self._axis = (C.c_uint8 * max(pairs, 1))(*axis)
        self.struct = SPKVRope(self.head_dim, self.rot_dim, int(self.adjacent), self.n_axes,
                               C.addressof(self._freq), C.addressof(self._axis))


def _heads(t, dtype, shape, name):
    """Address and strides of one set of heads (the fields of spkv_heads_t)."""
    st = t.stride()
    if not t.is_cuda or t.dtype != dtype or t.shape != shape or (st[2] != 1 and shape[2] != 1):
        raise ValueError(f"{name}: need a cuda {dtype} tensor of shape {tuple(shape)} with dense heads, "
                         f"got {t.dtype} {tuple(t.shape)} strides {st} on {t.device}")
    return t.data_ptr(), st[0], st[1]


_NO_HEADS = (0, 0, 0)


class _Block(threading.local):
    """Memory for the sets of heads of a call (the calls read them before they return): each thread's own."""

    def __init__(self):
        self.block = (C.c_int64 * 24)()
        at = C.addressof(self.block)
        self.at = [at + 24 * i for i in range(8)]


_block = _Block()
_PACK = {n: struct.Struct(f"{3 * n}q").pack_into for n in (6, 8)}


def _packed(sets):
    """Address of each set of heads (None where there is none)."""
    block = _block
    _PACK[len(sets)](block.block, 0, *itertools.chain.from_iterable(sets))
    return [None if h is _NO_HEADS else at for h, at in zip(sets, block.at)]


def _rope_call(q, k, v, positions, rope, q_weight, k_weight, eps, names):
    """What both directions check and pass: shapes, type, weights, norm, positions."""
    dtype = q.dtype
    if q.dim() != 3 or k.dim() != 3 or dtype not in _HEAD_TYPES:
        raise ValueError(f"{names[0]}, {names[1]}: need bf16 or fp32 [tokens, heads, head_dim]")
    n, hq, d = q.shape
    if d != rope.head_dim:
        raise ValueError(f"{names[0]}: heads of {d} elements, rope made for {rope.head_dim}")
    hk = k.shape[1]
    ins = [_heads(q, dtype, (n, hq, d), names[0]), _heads(k, dtype, (n, hk, d), names[1]),
           _NO_HEADS if v is None else _heads(v, dtype, (n, hk, d), names[2])]
    shape = (n,) if rope.n_axes == 1 and positions.dim() == 1 else (rope.n_axes, n)
    pp = _dev_ptr(positions, torch.int32, shape, "positions")
    if eps is None:
        if q_weight is not None or k_weight is not None:
            raise ValueError("weights of the norm without eps")
        return n, hq, hk, d, ins, pp, None, None, -1.0
    if not eps >= 0.0:
        raise ValueError("eps: need a value >= 0, or None for no norm")
    qw = _dev_ptr(q_weight, torch.float32, (d,), "q_weight") if q_weight is not None else None
    kw = _dev_ptr(k_weight, torch.float32, (d,), "k_weight") if k_weight is not None else None
    return n, hq, hk, d, ins, pp, qw, kw, float(eps)


def _rope_out(out, q, v, n, hq, hk, d):
    """Tensors to write -- those given, or new dense ones -- and the sets of heads that they are."""
    dtype, many, few = q.dtype, (n, hq, d), (n, hk, d)
    if out is not None:
        out = (out[0], out[1], None) if v is None else out
        return out, [_heads(out[0], dtype, many, "out[0]"), _heads(out[1], dtype, few, "out[1]"),
                     _NO_HEADS if v is None else _heads(out[2], dtype, few, "out[2]")]
    device, of_many, of_few = q.device, (hq * d, d, 1), (hk * d, d, 1)       # (empty_strided takes less host time than empty)
    a = torch.empty_strided(many, of_many, dtype=dtype, device=device)
    b = torch.empty_strided(few, of_few, dtype=dtype, device=device)
    if v is None:
        return (a, b, None), [(a.data_ptr(), hq * d, d), (b.data_ptr(), hk * d, d), _NO_HEADS]
    c = torch.empty_strided(few, of_few, dtype=dtype, device=device)
    return (a, b, c), [(a.data_ptr(), hq * d, d), (b.data_ptr(), hk * d, d), (c.data_ptr(), hk * d, d)]


def qk_norm_rope(q, k, positions, rope, q_weight=None, k_weight=None, eps=None, v=None, out=None):
    """RMS norm of every head (eps None: no norm), rotation by positions, dense layout, in one launch
    (spkv_qk_norm_rope).  q: bf16 or fp32 [tokens, H_q, D]; k, v: [tokens, H_kv, D], slices of a
    projection's rows as they are; positions: int32 [tokens] or [axes, tokens].  out: tensors to write
    (the inputs themselves may be passed).  Returns (q, k) or, with v, (q, k, v); where an input or a weight
    requires a gradient (and none is given to write), outputs whose backward pass is qk_norm_rope_backward."""
    if torch.is_grad_enabled() and (q.requires_grad or k.requires_grad or (v is not None and v.requires_grad) or
                                    (q_weight is not None and q_weight.requires_grad) or
                                    (k_weight is not None and k_weight.requires_grad)):
        if out is not None:
            raise ValueError("out: no gradient passes through tensors to write; leave it out, or call under torch.no_grad()")
        return _NormRope.apply(q, k, v, q_weight, k_weight, positions, rope, eps)
    n, hq, hk, d, ins, pp, qw, kw, eps = _rope_call(q, k, v, positions, rope, q_weight, k_weight, eps, "qkv")
    out, outs = _rope_out(out, q, v, n, hq, hk, d)
    at = _packed(ins + outs)
    _check((_LIB or load_library()).spkv_qk_norm_rope(at[0], at[1], at[2], qw, kw, eps, pp, rope.struct, _HEAD_TYPES[q.dtype],
                                                      n, hq, hk, at[3], at[4], at[5], _stream()), "spkv_qk_norm_rope")
    return tuple(out[:2]) if v is None else tuple(out)


def qk_norm_rope_backward(dq, dk, positions, rope, q=None, k=None, q_weight=None, k_weight=None, eps=None,
                          dv=None, out=None, want_weights=None, workspace=None):
    """Gradients of qk_norm_rope (spkv_qk_norm_rope_backward) from those of its outputs: dq, dk, dv.
    q, k: the forward's inputs (only with a norm).  out: tensors for the inputs' gradients, for example
    slices of one buffer for the projection's rows.  Returns (dq, dk), with dv (dq, dk, dv) -- or nothing
    of these if `out` was given -- and then, with a norm and unless want_weights is False, the
    fp32 gradients of both weights.  What it returns carries no gradient of its own."""
    n, hq, hk, d, ins, pp, qw, kw, eps = _rope_call(dq, dk, dv, positions, rope, q_weight, k_weight, eps,
                                                    ("dq", "dk", "dv"))
    given, dtype = out is not None, dq.dtype
    out, outs = _rope_out(out, dq, dv, n, hq, hk, d)
    xs, weights = [_NO_HEADS, _NO_HEADS], ()
    if eps >= 0.0:
        if q is None or k is None:
            raise ValueError("q, k: the forward's inputs are needed with a norm")
        xs = [_heads(q, dtype, (n, hq, d), "q"), _heads(k, dtype, (n, hk, d), "k")]
        if want_weights is None or want_weights:
            weights = torch.empty_strided((2, d), (d, 1), dtype=torch.float32, device=dq.device).unbind(0)
    elif want_weights:
        raise ValueError("want_weights: there are no weights without a norm")
    lib = load_library()
    if weights and workspace is None:
        workspace = torch.empty(int(lib.spkv_qk_norm_rope_backward_workspace_bytes(n, hq, hk, d)),
                                dtype=torch.uint8, device=dq.device)
    if workspace is not None and (workspace.dtype != torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous()):
        raise ValueError("workspace must be a contiguous uint8 device tensor")
    at = _packed(ins + xs + outs)
    dqw, dkw = (weights[0].data_ptr(), weights[1].data_ptr()) if weights else (None, None)
    ws, ws_bytes = (workspace.data_ptr(), workspace.numel()) if workspace is not None else (None, 0)
    _check(lib.spkv_qk_norm_rope_backward(*at[:5], qw, kw, eps, pp, rope.struct, _HEAD_TYPES[dtype], n, hq, hk, *at[5:],
                                          dqw, dkw, ws, ws_bytes, _stream()), "spkv_qk_norm_rope_backward")
    first = () if given else tuple(out[:2]) if dv is None else tuple(out)
    return first + tuple(weights)


def _as_heads(t):
    """t, or a dense copy where its strides or address are not those of a set of heads."""
    unit, st = 16 // t.element_size(), t.stride()
    if st[2] == 1 and st[1] % unit == 0 and st[0] % unit == 0 and t.data_ptr() % 16 == 0:
        return t
    return t.clone(memory_format=torch.contiguous_format)


class _NormRope(torch.autograd.Function):
    """qk_norm_rope with qk_norm_rope_backward as its gradient; the values' is theirs as it comes."""

    @staticmethod
    def forward(ctx, q, k, v, q_weight, k_weight, positions, rope, eps):
        ctx.rope, ctx.eps = rope, eps
        ctx.save_for_backward(positions, *((q, k, q_weight, k_weight) if eps is not None else ()))
        return qk_norm_rope(q, k, positions, rope, q_weight, k_weight, eps, v)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dq, dk, dv=None):
        need = ctx.needs_input_grad
        if not (need[0] or need[1] or need[3] or need[4]):
            return None, None, dv, None, None, None, None, None
        positions, *x = ctx.saved_tensors
        norm = dict(zip(("q", "k", "q_weight", "k_weight"), x), eps=ctx.eps, want_weights=need[3] or need[4]) if x else {}
        got = qk_norm_rope_backward(_as_heads(dq), _as_heads(dk), positions, ctx.rope, **norm) + (None, None)
        wanted = [g if n else None for g, n in zip((got[0], got[1], dv, got[2], got[3]), need)]
        return (*wanted, None, None, None)


def _check(code, where):
    if code != OK:
        raise SPKVError(code, where)


# The raw handle of a device's current stream.  Building a torch.cuda.Stream object to read it from
# took 2.9 us of the 10 us that a short decode step cost the host; asked for directly 0.3 (a step of
# one sequence of 2048 tokens 10.4 -> 6.9 us, append and attention as two calls 20.8 -> 15.5).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream():
    if _raw_stream is None:
        return torch.cuda.current_stream().cuda_stream
    return _raw_stream(torch.cuda.current_device())


def _dev_ptr(t: torch.Tensor, dtype, shape: tuple, name):
    if not t.is_cuda or t.dtype != dtype or t.shape != shape or not t.is_contiguous():
        raise ValueError(f"{name}: need a contiguous cuda {dtype} tensor of shape {tuple(shape)}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")
    return t.data_ptr()                    # (every entry point declares its argument types)


class SPKVCache:
    """One attention layer's SP-KV cache on the current CUDA (HIP) device."""

    def __init__(self, batch, n_q_heads, n_kv_heads, head_dim, max_context,
                 max_total_kept_tokens, window=128, tau=0.5, device="cuda"):
        self.lib = load_library()
        self.cfg = SPKVConfig(batch, n_q_heads, n_kv_heads, head_dim, window, 0, tau,
                              max_context, max_total_kept_tokens)
        nbytes = required_bytes(self.cfg)
        if nbytes == 0:
            raise SPKVError(E_INVAL, "spkv_cache_required_bytes")
        self.device = torch.device(device)
        self.arena = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        self.index = self.arena.get_device()
        self.handle = C.c_void_p()
        _check(self.lib.spkv_cache_create(C.byref(self.cfg), C.c_void_p(self.arena.data_ptr()),
                                          nbytes, _stream(), C.byref(self.handle)),
               "spkv_cache_create")

    def grow(self, max_context=None, max_total_kept_tokens=None):
        """Move the cache into a new, larger arena (spkv_cache_grow).  The old arena is
        released once the copy has completed."""
        old = self.cfg
        cfg = SPKVConfig(old.batch, old.n_q_heads, old.n_kv_heads, old.head_dim, old.window, 0,
                         old.tau,
                         old.max_context if max_context is None else int(max_context),
                         old.max_total_kept_tokens if max_total_kept_tokens is None
                         else int(max_total_kept_tokens))
        nbytes = required_bytes(cfg)
        if nbytes == 0:
            raise SPKVError(E_INVAL, "spkv_cache_required_bytes")
        arena = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        _check(self.lib.spkv_cache_grow(self.handle, C.byref(cfg), C.c_void_p(arena.data_ptr()),
                                        nbytes, _stream()), "spkv_cache_grow")
        torch.cuda.current_stream(self.device).synchronize()    # the old arena is read until here
        self.arena, self.cfg = arena, cfg

    def close(self):
        if getattr(self, "handle", None) is not None and self.handle.value:
            torch.cuda.synchronize(self.device)
            self.lib.spkv_cache_destroy(self.handle)
            self.handle = C.c_void_p()
        self.arena = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- write path
    def make_cu(self, cu_seqlens):
        """cu_seqlens as the C array spkv_append takes (build once, reuse every step)."""
        return (C.c_int32 * (self.cfg.batch + 1))(*[int(x) for x in cu_seqlens])

    def append(self, k, v, util_logits, cu_seqlens):
        cfg = self.cfg
        cu = cu_seqlens if isinstance(cu_seqlens, C.Array) else self.make_cu(cu_seqlens)
        total = cu[cfg.batch]
        if total == 0:
            _check(self.lib.spkv_append(self.handle, None, None, None, cu, _stream()), "spkv_append")
            return
        kp = _dev_ptr(k, torch.bfloat16, (total, cfg.n_kv_heads, cfg.head_dim), "k")
        vp = _dev_ptr(v, torch.bfloat16, (total, cfg.n_kv_heads, cfg.head_dim), "v")
        fp = _dev_ptr(util_logits, torch.float32, (total, cfg.n_kv_heads), "util_logits")
        _check(self.lib.spkv_append(self.handle, kp, vp, fp, cu, _stream()), "spkv_append")

    # ---- read path
    def decode_attention(self, q, out=None, lse=None, sm_scale=0.0, want_lse=False):
        cfg = self.cfg
        shape = (cfg.batch, cfg.n_q_heads, cfg.head_dim)
        qp = _dev_ptr(q, torch.bfloat16, shape, "q")
        if out is None:
            out = torch.empty(shape, dtype=torch.bfloat16, device=q.device)
        op = _dev_ptr(out, torch.bfloat16, shape, "out")
        if lse is None and want_lse:
            lse = torch.empty(shape[:2], dtype=torch.float32, device=q.device)
        lp = _dev_ptr(lse, torch.float32, shape[:2], "lse") if lse is not None else None
        _check(self.lib.spkv_decode_attention(self.handle, qp, op, lp, float(sm_scale), _stream()),
               "spkv_decode_attention")
        return (out, lse) if lse is not None else out

    def decode_attention_static(self, q, out, lse=None, sm_scale=0.0):
        """spkv_decode_attention_static: partials in the library's static device array; the
        caller passes every buffer (nothing is allocated here either)."""
        cfg = self.cfg
        shape = (cfg.batch, cfg.n_q_heads, cfg.head_dim)
        qp = _dev_ptr(q, torch.bfloat16, shape, "q")
        op = _dev_ptr(out, torch.bfloat16, shape, "out")
        lp = _dev_ptr(lse, torch.float32, shape[:2], "lse") if lse is not None else None
        _check(self.lib.spkv_decode_attention_static(self.handle, qp, op, lp, float(sm_scale),
                                                     _stream()), "spkv_decode_attention_static")
        return out

    def decode_step(self, k, v, util_logits, q, out=None, lse=None, sm_scale=0.0, want_lse=False):
        """Append one token per sequence and decode, fused (spkv_decode_step)."""
        cfg = self.cfg
        kv_shape = (cfg.batch, cfg.n_kv_heads, cfg.head_dim)
        shape = (cfg.batch, cfg.n_q_heads, cfg.head_dim)
        kp = _dev_ptr(k, torch.bfloat16, kv_shape, "k")
        vp = _dev_ptr(v, torch.bfloat16, kv_shape, "v")
        fp = _dev_ptr(util_logits, torch.float32, kv_shape[:2], "util_logits")
        qp = _dev_ptr(q, torch.bfloat16, shape, "q")
        if out is None:
            out = torch.empty(shape, dtype=torch.bfloat16, device=q.device)
        op = _dev_ptr(out, torch.bfloat16, shape, "out")
        if lse is None and want_lse:
            lse = torch.empty(shape[:2], dtype=torch.float32, device=q.device)
        lp = _dev_ptr(lse, torch.float32, shape[:2], "lse") if lse is not None else None
        _check(self.lib.spkv_decode_step(self.handle, kp, vp, fp, qp, op, lp, float(sm_scale),
                                         _stream()), "spkv_decode_step")
        return (out, lse) if lse is not None else out

    def decode_step_predict(self, hidden, w1, b1, w2, b2, k, v, q, out=None, lse=None,
                            util_logits=None, workspace=None, sm_scale=0.0, want_lse=False):
        """Fused step whose gate logits come from the utility predictor, computed inside the
        step's two launches (spkv_decode_step_predict).  Returns (out, util_logits) or
        (out, lse, util_logits)."""
        cfg = self.cfg
        kv_shape = (cfg.batch, cfg.n_kv_heads, cfg.head_dim)
        shape = (cfg.batch, cfg.n_q_heads, cfg.head_dim)
        d_model, d_hidden = hidden.shape[1], w1.shape[0]
        hp = _dev_ptr(hidden, torch.bfloat16, (cfg.batch, d_model), "hidden")
        w1p = _dev_ptr(w1, torch.bfloat16, (d_hidden, d_model), "w1")
        w2p = _dev_ptr(w2, torch.bfloat16, (cfg.n_kv_heads, d_hidden), "w2")
        b1p = _dev_ptr(b1, torch.float32, (d_hidden,), "b1") if b1 is not None else None
        b2p = _dev_ptr(b2, torch.float32, (cfg.n_kv_heads,), "b2") if b2 is not None else None
        kp = _dev_ptr(k, torch.bfloat16, kv_shape, "k")
        vp = _dev_ptr(v, torch.bfloat16, kv_shape, "v")
        qp = _dev_ptr(q, torch.bfloat16, shape, "q")
        if out is None:
            out = torch.empty(shape, dtype=torch.bfloat16, device=q.device)
        op = _dev_ptr(out, torch.bfloat16, shape, "out")
        if lse is None and want_lse:
            lse = torch.empty(shape[:2], dtype=torch.float32, device=q.device)
        lp = _dev_ptr(lse, torch.float32, shape[:2], "lse") if lse is not None else None
        if util_logits is None:
            util_logits = torch.empty(kv_shape[:2], dtype=torch.float32, device=q.device)
        fp = _dev_ptr(util_logits, torch.float32, kv_shape[:2], "util_logits")
        if workspace is None:
            need = self.lib.spkv_decode_step_predict_workspace_bytes(cfg.batch, d_hidden)
            workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
        if workspace.dtype != torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous uint8 device tensor")
        _check(self.lib.spkv_decode_step_predict(self.handle, hp, w1p, b1p, w2p, b2p, d_model,
                                                 d_hidden, kp, vp, qp, op, lp, fp,
                                                 workspace.data_ptr(), workspace.numel(),
                                                 float(sm_scale), _stream()),
               "spkv_decode_step_predict")
        return (out, lse, util_logits) if lse is not None else (out, util_logits)

    def decode_chunk(self, k, v, util_logits, q, cu_seqlens, out=None, lse=None, sm_scale=0.0,
                     want_lse=False):
        """Append up to 16 tokens per sequence and return each one's attention output
        (spkv_decode_chunk)."""
        cfg = self.cfg
        cu = cu_seqlens if isinstance(cu_seqlens, C.Array) else self.make_cu(cu_seqlens)
        total = cu[cfg.batch]
        if total == 0:
            _check(self.lib.spkv_decode_chunk(self.handle, None, None, None, None, cu, None, None,
                                              float(sm_scale), _stream()), "spkv_decode_chunk")
            return None
        kv_shape = (total, cfg.n_kv_heads, cfg.head_dim)
        shape = (total, cfg.n_q_heads, cfg.head_dim)
        kp = _dev_ptr(k, torch.bfloat16, kv_shape, "k")
        vp = _dev_ptr(v, torch.bfloat16, kv_shape, "v")
        fp = _dev_ptr(util_logits, torch.float32, kv_shape[:2], "util_logits")
        qp = _dev_ptr(q, torch.bfloat16, shape, "q")
        if out is None:
            out = torch.empty(shape, dtype=torch.bfloat16, device=q.device)
        op = _dev_ptr(out, torch.bfloat16, shape, "out")
        if lse is None and want_lse:
            lse = torch.empty(shape[:2], dtype=torch.float32, device=q.device)
        lp = _dev_ptr(lse, torch.float32, shape[:2], "lse") if lse is not None else None
        _check(self.lib.spkv_decode_chunk(self.handle, kp, vp, fp, qp, cu, op, lp, float(sm_scale),
                                          _stream()), "spkv_decode_chunk")
        return (out, lse) if lse is not None else out

    def score_chunk(self, k, v, q, cu_seqlens, out=None, lse=None, sm_scale=0.0, want_lse=False):
        """Attention outputs of up to 16 draft tokens per sequence, the cache left unchanged
        (spkv_score_chunk)."""
        cfg = self.cfg
        cu = cu_seqlens if isinstance(cu_seqlens, C.Array) else self.make_cu(cu_seqlens)
        total = cu[cfg.batch]
        if total == 0:
            _check(self.lib.spkv_score_chunk(self.handle, None, None, None, cu, None, None,
                                             float(sm_scale), _stream()), "spkv_score_chunk")
            return None
        kv_shape = (total, cfg.n_kv_heads, cfg.head_dim)
        shape = (total, cfg.n_q_heads, cfg.head_dim)
        kp = _dev_ptr(k, torch.bfloat16, kv_shape, "k")
        vp = _dev_ptr(v, torch.bfloat16, kv_shape, "v")
        qp = _dev_ptr(q, torch.bfloat16, shape, "q")
        if out is None:
            out = torch.empty(shape, dtype=torch.bfloat16, device=q.device)
        op = _dev_ptr(out, torch.bfloat16, shape, "out")
        if lse is None and want_lse:
            lse = torch.empty(shape[:2], dtype=torch.float32, device=q.device)
        lp = _dev_ptr(lse, torch.float32, shape[:2], "lse") if lse is not None else None
        _check(self.lib.spkv_score_chunk(self.handle, kp, vp, qp, cu, op, lp, float(sm_scale),
                                         _stream()), "spkv_score_chunk")
        return (out, lse) if lse is not None else out

    def prefill_workspace_bytes(self, max_tokens_per_sequence, max_total_tokens):
        return int(self.lib.spkv_prefill_workspace_bytes(self.handle, int(max_tokens_per_sequence),
                                                         int(max_total_tokens)))

    def prefill_attention(self, k, v, util_logits, q, cu_seqlens, workspace=None, out=None,
                          lse=None, sm_scale=0.0, want_lse=False):
        """Append any number of tokens per sequence and return each one's attention output
        (spkv_prefill_attention).  workspace: uint8 device tensor of at least
        prefill_workspace_bytes(max n_b, sum n_b) bytes; allocated here if None."""
        cfg = self.cfg
        cu = cu_seqlens if isinstance(cu_seqlens, C.Array) else self.make_cu(cu_seqlens)
        total = cu[cfg.batch]
        if total == 0:
            _check(self.lib.spkv_prefill_attention(self.handle, None, None, None, None, cu, None,
                                                   None, float(sm_scale), None, 0, _stream()),
                   "spkv_prefill_attention")
            return None
        kv_shape = (total, cfg.n_kv_heads, cfg.head_dim)
        shape = (total, cfg.n_q_heads, cfg.head_dim)
        kp = _dev_ptr(k, torch.bfloat16, kv_shape, "k")
        vp = _dev_ptr(v, torch.bfloat16, kv_shape, "v")
        fp = _dev_ptr(util_logits, torch.float32, kv_shape[:2], "util_logits")
        qp = _dev_ptr(q, torch.bfloat16, shape, "q")
        if workspace is None:
            n_max = max(cu[b + 1] - cu[b] for b in range(cfg.batch))
            workspace = torch.empty(self.prefill_workspace_bytes(n_max, total), dtype=torch.uint8,
                                    device=q.device)
        if workspace.dtype != torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous uint8 device tensor")
        if out is None:
            out = torch.empty(shape, dtype=torch.bfloat16, device=q.device)
        op = _dev_ptr(out, torch.bfloat16, shape, "out")
        if lse is None and want_lse:
            lse = torch.empty(shape[:2], dtype=torch.float32, device=q.device)
        lp = _dev_ptr(lse, torch.float32, shape[:2], "lse") if lse is not None else None
        _check(self.lib.spkv_prefill_attention(self.handle, kp, vp, fp, qp, cu, op, lp,
                                               float(sm_scale), workspace.data_ptr(),
                                               workspace.numel(), _stream()),
               "spkv_prefill_attention")
        return (out, lse) if lse is not None else out

    # ---- shared prompts
    def _share_workspace(self, sharing, rows, workspace, device):
        if sharing.batch != self.cfg.batch:
            raise ValueError(f"sharing: made for {sharing.batch} sequences, the cache has {self.cfg.batch}")
        if workspace is None:
            return torch.empty_strided((sharing.workspace_bytes(rows),), (1,), dtype=torch.uint8, device=device)
        if workspace.dtype != torch.uint8 or not workspace.is_cuda or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous uint8 device tensor")
        return workspace

    def decode_attention_shared(self, sharing, q, out=None, lse=None, sm_scale=0.0, want_lse=False,
                                workspace=None):
        """decode_attention over the sequences and the prompts that they continue
        (spkv_decode_attention_shared).  sharing: a PrefixSharing."""
        cfg = self.cfg
        shape = (cfg.batch, cfg.n_q_heads, cfg.head_dim)
        qp = _dev_ptr(q, torch.bfloat16, shape, "q")
        workspace = self._share_workspace(sharing, cfg.batch, workspace, q.device)
        if out is None:
            out = torch.empty_strided(shape, (shape[1] * shape[2], shape[2], 1), dtype=torch.bfloat16, device=q.device)
            op = out.data_ptr()
        else:
            op = _dev_ptr(out, torch.bfloat16, shape, "out")
        if lse is not None:
            lp = _dev_ptr(lse, torch.float32, shape[:2], "lse")
        elif want_lse:
            lse = torch.empty_strided(shape[:2], (shape[1], 1), dtype=torch.float32, device=q.device)
            lp = lse.data_ptr()
        else:
            lp = None
        _check(self.lib.spkv_decode_attention_shared(self.handle, sharing.prefix.handle, sharing.prefix_of, qp, op, lp,
                                                     float(sm_scale), workspace.data_ptr(), workspace.numel(),
                                                     _stream()), "spkv_decode_attention_shared")
        return (out, lse) if lse is not None else out

    def prefix_attention(self, sharing, q, cu_seqlens, own_out, own_lse, appended=True, out=None, lse=None,
                         sm_scale=0.0, workspace=None):
        """Join own_out, own_lse -- the attention of a call's tokens over their own sequences -- with that over
        the prompts that these continue (spkv_prefix_attention).  cu_seqlens as in that call, None: one token
        per sequence.  out, lse may be own_out, own_lse.  Returns (out, lse)."""
        cfg = self.cfg
        cu = cu_seqlens if cu_seqlens is None or isinstance(cu_seqlens, C.Array) else self.make_cu(cu_seqlens)
        total = cfg.batch if cu is None else cu[cfg.batch]
        shape = (total, cfg.n_q_heads, cfg.head_dim)
        qp = _dev_ptr(q, torch.bfloat16, shape, "q")
        ip = _dev_ptr(own_out, torch.bfloat16, shape, "own_out")
        zp = _dev_ptr(own_lse, torch.float32, shape[:2], "own_lse")
        workspace = self._share_workspace(sharing, max(total, 1), workspace, q.device)
        if out is None:
            out = torch.empty_strided(shape, (shape[1] * shape[2], shape[2], 1), dtype=torch.bfloat16, device=q.device)
        if lse is None:
            lse = torch.empty_strided(shape[:2], (shape[1], 1), dtype=torch.float32, device=q.device)
        op = _dev_ptr(out, torch.bfloat16, shape, "out")
        lp = _dev_ptr(lse, torch.float32, shape[:2], "lse")
        _check(self.lib.spkv_prefix_attention(sharing.prefix.handle, self.handle, sharing.prefix_of, qp, cu, int(appended), ip, zp,
                                              op, lp, float(sm_scale), workspace.data_ptr(), workspace.numel(),
                                              _stream()), "spkv_prefix_attention")
        return out, lse

    # ---- sequences that branch
    def _ptr(self, t, dtype, shape, name):
        """_dev_ptr, of a tensor on the cache's own device."""
        if t.get_device() != self.index or t.dtype != dtype or t.shape != shape or not t.is_contiguous():
            raise ValueError(f"{name}: need a contiguous {dtype} tensor of shape {tuple(shape)} on cuda:{self.index}, "
                             f"got {t.dtype} {tuple(t.shape)} on {t.device}")
        return t.data_ptr()

    def _stream(self):
        current = torch.cuda.current_device()
        if current != self.index:
            raise ValueError(f"the cache is on cuda:{self.index}, the current device is cuda:{current}")
        return _stream() if _raw_stream is None else _raw_stream(current)

    def score_tree(self, k, v, q, parents, cu_seqlens, util_logits=None, out=None, lse=None, sm_scale=0.0, want_lse=False):
        """Attention outputs of a tree of up to 64 drafts per sequence, the cache left unchanged (spkv_score_tree).
        parents: int32 [total] on the device, the index of an earlier draft of the same sequence or -1.  util_logits: the
        drafts', needed where a sequence has more drafts than the window has tokens."""
        cfg = self.cfg
        cu = cu_seqlens if isinstance(cu_seqlens, C.Array) else self.make_cu(cu_seqlens)
        total = cu[cfg.batch]
        if total == 0:
            _check(self.lib.spkv_score_tree(self.handle, None, None, None, None, None, cu, None, None, float(sm_scale),
                                            self._stream()), "spkv_score_tree")
            return None
        kv_shape = (total, cfg.n_kv_heads, cfg.head_dim)
        shape = (total, cfg.n_q_heads, cfg.head_dim)
        kp = self._ptr(k, torch.bfloat16, kv_shape, "k")
        vp = self._ptr(v, torch.bfloat16, kv_shape, "v")
        qp = self._ptr(q, torch.bfloat16, shape, "q")
        fp = self._ptr(util_logits, torch.float32, kv_shape[:2], "util_logits") if util_logits is not None else None
        pp = self._ptr(parents, torch.int32, (total,), "parents")
        if out is None:                       # (with strides: half a microsecond less than torch.empty)
            out = torch.empty_strided(shape, (shape[1] * shape[2], shape[2], 1), dtype=torch.bfloat16, device=q.device)
            op = out.data_ptr()
        else:
            op = self._ptr(out, torch.bfloat16, shape, "out")
        if lse is not None:
            lp = self._ptr(lse, torch.float32, shape[:2], "lse")
        elif want_lse:
            lse = torch.empty_strided(shape[:2], (shape[1], 1), dtype=torch.float32, device=q.device)
            lp = lse.data_ptr()
        else:
            lp = None
        _check(self.lib.spkv_score_tree(self.handle, kp, vp, fp, qp, pp, cu, op, lp, float(sm_scale), self._stream()),
               "spkv_score_tree")
        return (out, lse) if lse is not None else out

    def append_rows(self, k, v, util_logits, rows, cu_seqlens):
        """Append the rows `rows` (int32 [total], on the device) of k, v, util_logits: sequence b's tokens are
        rows[cu[b]:cu[b + 1]] (spkv_append_rows).  For the drafts of a tree that were accepted."""
        cfg = self.cfg
        cu = cu_seqlens if isinstance(cu_seqlens, C.Array) else self.make_cu(cu_seqlens)
        total, n = cu[cfg.batch], k.shape[0]
        kv_shape = (n, cfg.n_kv_heads, cfg.head_dim)
        kp = self._ptr(k, torch.bfloat16, kv_shape, "k")
        vp = self._ptr(v, torch.bfloat16, kv_shape, "v")
        fp = self._ptr(util_logits, torch.float32, kv_shape[:2], "util_logits")
        rp = self._ptr(rows, torch.int32, (total,), "rows")
        _check(self.lib.spkv_append_rows(self.handle, kp, vp, fp, rp, n, cu, self._stream()), "spkv_append_rows")

    def fork(self, source, other=None):
        """Sequence b becomes what sequence source[b] -- of `other`, or of this cache -- was before the call; FORK_KEEP
        leaves it, FORK_EMPTY empties it and gives its pages back (spkv_cache_fork)."""
        if not isinstance(source, C.Array):
            source = (C.c_int32 * len(source))(*[int(x) for x in source])
        if len(source) != self.cfg.batch:
            raise ValueError(f"source: need one entry for each of {self.cfg.batch} sequences, got {len(source)}")
        if other is not None and other.index != self.index:
            raise ValueError(f"other: on cuda:{other.index}, this cache is on cuda:{self.index}")
        _check(self.lib.spkv_cache_fork(self.handle, other.handle if other is not None else None, source,
                                        self._stream()), "spkv_cache_fork")

    def gather(self, sequences=None, rows=None, out=None):
        """The pairs that sequences hold (all of them by default; up to 512, also repeated), kept ones and then the window's, positions ascending, as
        (k, v, util_logits, positions, counts): bf16 [n, H_kv, rows, D] twice, fp32 and int32 [n, H_kv, rows], int32
        [n, H_kv] (spkv_cache_gather).  rows None: as many as the longest head holds (synchronises).  out: those five
        tensors, to write; rows behind a head's last pair are left as they were (undefined in new tensors)."""
        cfg = self.cfg
        if sequences is None:
            n, which = cfg.batch, None
        else:
            n, which = len(sequences), (C.c_int32 * max(len(sequences), 1))(*[int(b) for b in sequences])
        if out is None:
            if rows is None:
                counts = torch.zeros(n, cfg.n_kv_heads, dtype=torch.int32, device=self.device)
                _check(self.lib.spkv_cache_gather(self.handle, which, n, 0, None, None, None, None, counts.data_ptr(),
                                                  self._stream()), "spkv_cache_gather")
                rows = int(counts.max()) if n > 0 else 0
            shape = (n, cfg.n_kv_heads, int(rows))
            k, v = (torch.empty(*shape, cfg.head_dim, dtype=torch.bfloat16, device=self.device) for _ in range(2))
            out = (k, v, torch.empty(shape, dtype=torch.float32, device=self.device),
                   torch.empty(shape, dtype=torch.int32, device=self.device),
                   torch.empty(shape[:2], dtype=torch.int32, device=self.device))
        k, v, f, positions, counts = out
        shape = (n, cfg.n_kv_heads, k.shape[2] if k.dim() == 4 else -1)
        kp = self._ptr(k, torch.bfloat16, (*shape, cfg.head_dim), "out[0]")
        vp = self._ptr(v, torch.bfloat16, (*shape, cfg.head_dim), "out[1]")
        fp = self._ptr(f, torch.float32, shape, "out[2]")
        pp = self._ptr(positions, torch.int32, shape, "out[3]")
        cp = self._ptr(counts, torch.int32, shape[:2], "out[4]")
        _check(self.lib.spkv_cache_gather(self.handle, which, n, shape[2], kp, vp, fp, pp, cp, self._stream()),
               "spkv_cache_gather")
        return k, v, f, positions, counts

    # ---- bookkeeping
    def reset(self):
        _check(self.lib.spkv_cache_reset(self.handle, _stream()), "spkv_cache_reset")

    def release_sequence(self, b):
        _check(self.lib.spkv_cache_release_sequence(self.handle, int(b), _stream()),
               "spkv_cache_release_sequence")

    def stats(self, with_kept_len=False):
        st = SPKVStats()
        n = self.cfg.batch * self.cfg.n_kv_heads
        buf = (C.c_int32 * n)()
        _check(self.lib.spkv_cache_stats(self.handle, C.byref(st), buf, _stream()),
               "spkv_cache_stats")
        if with_kept_len:
            return st, [list(buf[b * self.cfg.n_kv_heads:(b + 1) * self.cfg.n_kv_heads])
                        for b in range(self.cfg.batch)]
        return st

    def kept_positions(self, b, h):
        cap = max(1, self.cfg.max_context)
        buf = (C.c_int32 * cap)()
        n = C.c_int32()
        _check(self.lib.spkv_cache_kept_positions(self.handle, b, h, buf, cap, C.byref(n),
                                                  _stream()), "spkv_cache_kept_positions")
        return list(buf[:n.value])

    def threshold_logit(self):
        th = C.c_float()
        _check(self.lib.spkv_cache_threshold_logit(self.handle, C.byref(th)),
               "spkv_cache_threshold_logit")
        return th.value

    def safe_steps(self):
        """Single-token steps guaranteed to fit (spkv_cache_safe_steps; synchronises)."""
        n = C.c_int64()
        _check(self.lib.spkv_cache_safe_steps(self.handle, _stream(), C.byref(n)),
               "spkv_cache_safe_steps")
        return n.value

    def advance(self, n_steps):
        """Account for n_steps steps executed by graph replays (spkv_cache_advance)."""
        _check(self.lib.spkv_cache_advance(self.handle, int(n_steps)), "spkv_cache_advance")

    def prune(self):
        """Drop every kept pair whose logit fails the current threshold (spkv_cache_prune)."""
        _check(self.lib.spkv_cache_prune(self.handle, _stream()), "spkv_cache_prune")

    def set_tau(self, tau):
        _check(self.lib.spkv_cache_set_tau(self.handle, float(tau)), "spkv_cache_set_tau")

    def set_option(self, option, value):
        _check(self.lib.spkv_cache_set_option(self.handle, option, int(value)),
               "spkv_cache_set_option")

    def read_kernel_timing(self, cap=8192):
        buf = (C.c_float * cap)()
        n = C.c_int32()
        _check(self.lib.spkv_cache_read_kernel_timing(self.handle, buf, cap, C.byref(n)),
               "spkv_cache_read_kernel_timing")
        return list(buf[:n.value])


class PrefixSharing:
    """Which sequence of `prefix`, a cache that holds prompts, every sequence of another cache continues
    (-1: none).  Host memory only; prefix_of may be changed in place (sharing[b] = p) as sequences come and go: calls
    from then on see it, launches captured before keep what they were captured with."""

    def __init__(self, prefix, prefix_of):
        self.prefix, self.batch = prefix, len(prefix_of)
        self.prefix_of = (C.c_int32 * self.batch)(*[int(p) for p in prefix_of])

    def __setitem__(self, b, p):
        self.prefix_of[b] = int(p)

    def workspace_bytes(self, rows):
        """Bytes that serve any call of at most `rows` rows (spkv_prefix_workspace_bytes)."""
        return int(self.prefix.lib.spkv_prefix_workspace_bytes(self.prefix.handle, int(rows)))
