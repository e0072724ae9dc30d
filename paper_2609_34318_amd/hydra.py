"""ctypes binding of libhydra_attn.so: argument marshalling only.

Every compute step runs in the library's HIP kernels; torch supplies device memory and
the current stream.  If the library is missing this module raises on first use: there
is no fallback path.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Optional, Sequence, Tuple

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libhydra_attn.so")

HYDRA_OK = 0
MAX_SEGS = 4
STATUS = {0: "ok", -1: "invalid", -2: "unsupported", -3: "align", -4: "workspace", -5: "hip", -6: "too large"}


class Chunk(ctypes.Structure):
    _fields_ = [("n_segs", ctypes.c_int32),
                ("start", ctypes.c_int32 * MAX_SEGS),
                ("len", ctypes.c_int32 * MAX_SEGS)]


class ProblemC(ctypes.Structure):
    _fields_ = [("n_heads", ctypes.c_int32),
                ("d_qk", ctypes.c_int32),
                ("d_v", ctypes.c_int32),
                ("softmax_scale", ctypes.c_float),
                ("cu_seqlens", ctypes.POINTER(ctypes.c_int32)),
                ("n_docs", ctypes.c_int32),
                ("q", Chunk),
                ("kv", Chunk),
                ("n_kv_heads", ctypes.c_int32),
                ("q_tok_stride", ctypes.c_int32),
                ("k_tok_stride", ctypes.c_int32),
                ("v_tok_stride", ctypes.c_int32)]


class ScoresC(ctypes.Structure):
    _fields_ = [("softcap", ctypes.c_float),
                ("slopes", ctypes.c_void_p),
                ("prefix_len", ctypes.POINTER(ctypes.c_int32)),
                ("window", ctypes.c_int32),
                ("sinks", ctypes.c_int32)]


ROPE_MAX_AXES = 4


class RopeC(ctypes.Structure):
    _fields_ = [("n_axes", ctypes.c_int32),
                ("pairs", ctypes.c_int32 * ROPE_MAX_AXES),
                ("pairing", ctypes.c_int32),
                ("per_axis", ctypes.c_int32),
                ("base", ctypes.c_double),
                ("inv_freq", ctypes.POINTER(ctypes.c_double))]


class LinearC(ctypes.Structure):
    _fields_ = [("n_heads", ctypes.c_int32),
                ("n_kv_heads", ctypes.c_int32),
                ("d_k", ctypes.c_int32),
                ("d_v", ctypes.c_int32),
                ("scale", ctypes.c_float),
                ("cu_seqlens", ctypes.POINTER(ctypes.c_int32)),
                ("n_seqs", ctypes.c_int32),
                ("q_tok_stride", ctypes.c_int32),
                ("k_tok_stride", ctypes.c_int32),
                ("v_tok_stride", ctypes.c_int32)]


class NormC(ctypes.Structure):
    _fields_ = [("n_tokens", ctypes.c_int64),
                ("n_heads", ctypes.c_int32),
                ("d", ctypes.c_int32),
                ("cp_u", ctypes.c_int32),
                ("center", ctypes.c_int32),
                ("activation", ctypes.c_int32),
                ("eps", ctypes.c_float)]


class SchedConfig(ctypes.Structure):
    _fields_ = [("n_ranks", ctypes.c_int32),
                ("token_budget", ctypes.c_int64),
                ("pp", ctypes.c_int32),
                ("theta_over_c", ctypes.c_double),
                ("cap", ctypes.c_int32),
                ("balance_ratio", ctypes.c_double)]


class SchedSummary(ctypes.Structure):
    _fields_ = [("w_hi", ctypes.c_int64),
                ("w_lo", ctypes.c_int64),
                ("s_max", ctypes.c_int64),
                ("c_mem", ctypes.c_int32),
                ("c_hat", ctypes.c_double),
                ("cap", ctypes.c_int32),
                ("m_target", ctypes.c_int64),
                ("n_mbs", ctypes.c_int32),
                ("max_load_x_cap", ctypes.c_int64)]


class KernelStat(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 32),
                ("launches", ctypes.c_int64),
                ("total_ms", ctypes.c_double),
                ("min_ms", ctypes.c_double),
                ("max_ms", ctypes.c_double)]


class HydraError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what} failed: status {status} ({lib().hydra_strerror(status).decode()})")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded library (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2609_34318_amd.build_lib`")
        L = ctypes.CDLL(LIB_PATH)
        P = ctypes.POINTER(ProblemC)
        vp, f = ctypes.c_void_p, ctypes.POINTER(ctypes.c_float)
        L.hydra_workspace_size.argtypes = [P]
        L.hydra_workspace_size.restype = ctypes.c_size_t
        L.hydra_attn_fwd.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.hydra_attn_fwd.restype = ctypes.c_int
        L.hydra_attn_fwd_merge.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, ctypes.c_int32, vp]
        L.hydra_attn_fwd_merge.restype = ctypes.c_int
        L.hydra_attn_fwd_split.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp, ctypes.c_size_t,
                                           ctypes.c_int32, ctypes.c_int32, vp]
        L.hydra_attn_fwd_split.restype = ctypes.c_int
        L.hydra_split_scratch_size.argtypes = [P]
        L.hydra_split_scratch_size.restype = ctypes.c_size_t
        L.hydra_attn_bwd.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
        L.hydra_attn_bwd.restype = ctypes.c_int
        L.hydra_attn_bwd_ds.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp,
                                        ctypes.c_size_t, vp]
        L.hydra_attn_bwd_ds.restype = ctypes.c_int
        L.hydra_attn_bwd_split.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp,
                                           ctypes.c_size_t, vp, ctypes.c_size_t, ctypes.c_int32, vp]
        L.hydra_attn_bwd_split.restype = ctypes.c_int
        L.hydra_bwd_ds_bytes.argtypes = [P, ctypes.c_int32]
        L.hydra_bwd_ds_bytes.restype = ctypes.c_size_t
        L.hydra_attn_bwd_noalloc.argtypes = [P, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
        L.hydra_attn_bwd_noalloc.restype = ctypes.c_int
        L.hydra_noalloc_scratch_bytes.argtypes = []
        L.hydra_noalloc_scratch_bytes.restype = ctypes.c_size_t
        L.hydra_noalloc_size.argtypes = [P]
        L.hydra_noalloc_size.restype = ctypes.c_size_t
        L.hydra_attn_plan.argtypes = [P, vp, ctypes.c_size_t, vp]
        L.hydra_attn_plan.restype = ctypes.c_int
        L.hydra_attn_fwd_planned.argtypes = L.hydra_attn_fwd.argtypes
        L.hydra_attn_fwd_planned.restype = ctypes.c_int
        L.hydra_attn_bwd_planned.argtypes = L.hydra_attn_bwd.argtypes
        L.hydra_attn_bwd_planned.restype = ctypes.c_int
        L.hydra_lse_merge.argtypes = [ctypes.c_int64, ctypes.c_int32, ctypes.c_int32, vp, vp, vp, vp, vp, vp]
        L.hydra_lse_merge.restype = ctypes.c_int
        L.hydra_strerror.argtypes = [ctypes.c_int]
        L.hydra_strerror.restype = ctypes.c_char_p
        L.hydra_visible_pairs.argtypes = [P]
        L.hydra_visible_pairs.restype = ctypes.c_int64
        L.hydra_plan_items.argtypes = [P, ctypes.c_int32, ctypes.POINTER(ctypes.c_int32), ctypes.c_int64]
        L.hydra_plan_items.restype = ctypes.c_int64
        L.hydra_tile_rows.argtypes = [ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32)]
        L.hydra_tile_rows.restype = None
        L.hydra_profile_start.argtypes = []
        L.hydra_profile_start.restype = ctypes.c_int
        L.hydra_profile_stop.argtypes = [ctypes.POINTER(KernelStat), ctypes.c_int32]
        L.hydra_profile_stop.restype = ctypes.c_int
        i32, i64 = ctypes.c_int32, ctypes.c_int64
        for name in ("hydra_pack_heads", "hydra_unpack_heads"):
            getattr(L, name).argtypes = [i64, i32, i32, i32, vp, vp, vp]
            getattr(L, name).restype = ctypes.c_int
        L.hydra_schedule.argtypes = [ctypes.POINTER(ctypes.c_int64), i64, ctypes.POINTER(SchedConfig),
                                     ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(ctypes.c_int32),
                                     ctypes.POINTER(ctypes.c_int32), ctypes.POINTER(SchedSummary)]
        L.hydra_schedule.restype = ctypes.c_int
        for name in ("hydra_zigzag_gather", "hydra_zigzag_scatter"):
            getattr(L, name).argtypes = [i64, i64, i32, i32, vp, vp, vp]
            getattr(L, name).restype = ctypes.c_int
        L.hydra_unpack_heads_gated.argtypes = [i64, i32, i32, i32, i32, vp, vp, vp, vp]
        L.hydra_unpack_heads_gated.restype = ctypes.c_int
        L.hydra_pack_heads_gated_bwd.argtypes = [i64, i32, i32, i32, i32, vp, vp, vp, vp, vp, vp]
        L.hydra_pack_heads_gated_bwd.restype = ctypes.c_int
        S, sz = ctypes.POINTER(ScoresC), ctypes.c_size_t
        for name, more, res in (("workspace_size", [], sz), ("scratch_size", [], sz), ("ds_bytes", [i32], sz),
                                ("visible_pairs", [], i64),
                                ("plan_items", [i32, ctypes.POINTER(ctypes.c_int32), i64], i64),
                                ("plan", [vp, sz, vp], ctypes.c_int),
                                ("fwd", [vp, vp, vp, vp, vp, vp, vp, sz, vp, sz, i32, i32, vp], ctypes.c_int),
                                ("bwd", [vp] * 4 + [i32] + [vp] * 5 + [vp, sz, vp, sz, vp, sz, i32, vp], ctypes.c_int)):
            getattr(L, "hydra_scores_" + name).argtypes = [P, S] + more
            getattr(L, "hydra_scores_" + name).restype = res
        R = ctypes.POINTER(RopeC)
        L.hydra_rope_q.argtypes = [R, i64, i32, i32, i32, vp, i64, vp, vp, vp]
        L.hydra_rope_kv.argtypes = [R, i64, i32, i32, i32, i32, vp, i64, vp, i64, vp, vp, vp, vp]
        L.hydra_rope_q_bwd.argtypes = [R, i64, i32, i32, i32, i32, vp, vp, vp, i64, vp]
        L.hydra_rope_kv_bwd.argtypes = [R, i64, i32, i32, i32, i32, i32, vp, vp, vp, vp, i64, vp, i64, vp]
        for name in ("hydra_rope_q", "hydra_rope_kv", "hydra_rope_q_bwd", "hydra_rope_kv_bwd"):
            getattr(L, name).restype = ctypes.c_int
        N = ctypes.POINTER(LinearC)
        L.hydra_linear_workspace_size.argtypes = [N]
        L.hydra_linear_workspace_size.restype = sz
        L.hydra_linear_plan.argtypes = [N, vp, sz, vp]
        L.hydra_linear_fwd.argtypes = [N] + [vp] * 8 + [sz, i32, vp]
        L.hydra_linear_bwd.argtypes = [N] + [vp] * 12 + [sz, i32, vp]
        L.hydra_linear_step.argtypes = [i32] * 6 + [ctypes.c_float] + [vp] * 9
        for name in ("hydra_linear_plan", "hydra_linear_fwd", "hydra_linear_bwd", "hydra_linear_step"):
            getattr(L, name).restype = ctypes.c_int
        M = ctypes.POINTER(NormC)
        L.hydra_norm_workspace_size.argtypes = [i64, i32, i32]
        L.hydra_norm_workspace_size.restype = sz
        L.hydra_unpack_heads_normed.argtypes = [M] + [vp] * 6
        L.hydra_unpack_heads_normed.restype = ctypes.c_int
        L.hydra_pack_heads_normed_bwd.argtypes = [M] + [vp] * 10 + [sz, vp]
        L.hydra_pack_heads_normed_bwd.restype = ctypes.c_int
        _lib = L
    return _lib


def _chunk(segs: Sequence[Tuple[int, int]]) -> Chunk:
    segs = list(segs)
    if len(segs) > MAX_SEGS:
        raise ValueError(f"at most {MAX_SEGS} segments per chunk")
    c = Chunk()
    c.n_segs = len(segs)
    for i, (s, n) in enumerate(segs):
        c.start[i] = int(s)
        c.len[i] = int(n)
    return c


class Scores:
    """How a problem's scores are modified: capped by a tanh (softcap), biased by minus slope times the
    distance of query and key (slopes: float32 device tensor, one per query head), and a prefix of each
    document that all of its tokens see (prefix: a length per document) or a sliding window (a token sees the
    last `window` keys up to its own and its document's first `sinks`).  The cap and the slopes are
    constants: they get no gradient."""

    def __init__(self, softcap: float = 0.0, slopes=None, prefix: Optional[Sequence[int]] = None, window: int = 0,
                 sinks: int = 0):
        self.softcap, self.slopes = float(softcap), slopes
        self.window, self.sinks = int(window), int(sinks)
        if not (0 <= self.window < 1 << 31 and 0 <= self.sinks < 1 << 31) or self.window != window or self.sinks != sinks:
            raise ValueError(f"window {window}, sinks {sinks}: integers of 32 bits, not negative, are required")
        self.prefix = None
        if prefix is not None:
            given = np.asarray(prefix)
            self.prefix = np.ascontiguousarray(given.astype(np.int32))
            if not np.array_equal(self.prefix, given):
                raise ValueError("prefix: lengths must be integers of 32 bits")
        self.c = ScoresC()
        self.c.softcap, self.c.window, self.c.sinks = self.softcap, self.window, self.sinks
        if self.softcap and not self.c.softcap:  # no cap to the library
            raise ValueError(f"softcap: {self.softcap} is 0 in 32 bits")
        if slopes is not None:
            self.c.slopes = _ptr(slopes, "slopes", _F32)
        if self.prefix is not None:
            self.c.prefix_len = self.prefix.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))

    @property
    def any(self) -> bool:
        return self.softcap != 0 or self.slopes is not None or self.prefix is not None or self.window != 0 or self.sinks != 0


class Problem:
    """One ring step of one rank: head shard, documents, Q chunk and KV chunk; with `scores`, modified
    scores in every call that takes the problem."""

    def __init__(self, cu_seqlens, n_heads: int, q_segs, kv_segs, softmax_scale: float = 0.0,
                 d_qk: int = 192, d_v: int = 128, n_kv_heads: int = 0, scores: Optional[Scores] = None):
        if scores is not None and scores.slopes is not None and scores.slopes.numel() != n_heads:
            raise ValueError(f"slopes: {scores.slopes.numel()} elements, expected {n_heads}")
        if scores is not None and scores.prefix is not None and scores.prefix.shape != (len(cu_seqlens) - 1,):
            raise ValueError(f"prefix: shape {scores.prefix.shape}, expected {(len(cu_seqlens) - 1,)}")
        self.scores = scores
        self.cu = np.ascontiguousarray(np.asarray(cu_seqlens, dtype=np.int32))
        self.q_segs = [tuple(map(int, s)) for s in q_segs]
        self.kv_segs = [tuple(map(int, s)) for s in kv_segs]
        self.c = ProblemC()
        self.c.n_heads = n_heads
        self.c.d_qk = d_qk
        self.c.d_v = d_v
        self.c.softmax_scale = softmax_scale
        self.c.cu_seqlens = self.cu.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
        self.c.n_docs = len(self.cu) - 1
        self.c.q = _chunk(self.q_segs)
        self.c.kv = _chunk(self.kv_segs)
        self.c.n_kv_heads = n_kv_heads
        self.n_heads = n_heads
        self.n_kv_heads = n_kv_heads or n_heads
        self.nq = sum(n for _, n in self.q_segs)
        self.nk = sum(n for _, n in self.kv_segs)

    @property
    def ref(self):
        return ctypes.byref(self.c)

    @property
    def scores_ref(self):
        return None if self.scores is None else ctypes.byref(self.scores.c)


def workspace_size(p: Problem) -> int:
    return int(lib().hydra_scores_workspace_size(p.ref, p.scores_ref))


def split_scratch_size(p: Problem) -> int:
    """Bytes of scratch for the calls' `scratch` (0: nothing of p is split)."""
    return int(lib().hydra_scores_scratch_size(p.ref, p.scores_ref))


def noalloc_size(p: Problem) -> int:
    """What counts of p against the limit of attn_bwd_noalloc."""
    return int(lib().hydra_noalloc_size(p.ref))


def visible_pairs(p: Problem) -> int:
    n = int(lib().hydra_scores_visible_pairs(p.ref, p.scores_ref))
    if n < 0:
        raise HydraError(-1, "hydra_visible_pairs")
    return n


def plan_items(p: Problem, which: int) -> np.ndarray:
    n = int(lib().hydra_scores_plan_items(p.ref, p.scores_ref, which, None, 0))
    if n < 0:
        raise HydraError(n, "hydra_plan_items")
    out = np.zeros((max(n, 1), 16), dtype=np.int32)
    lib().hydra_scores_plan_items(p.ref, p.scores_ref, which, out.ctypes.data_as(ctypes.POINTER(ctypes.c_int32)), n)
    return out[:n]


def tile_rows() -> Tuple[int, int]:
    a, b = ctypes.c_int32(), ctypes.c_int32()
    lib().hydra_tile_rows(ctypes.byref(a), ctypes.byref(b))
    return a.value, b.value


# ------------------------------------------------------------------ device calls (torch tensors)

def _ptr(t, what: str = "tensor", dtypes=None, numel: Optional[int] = None) -> Optional[int]:
    """Device address of a dense device tensor (None passes through).  The library only sees
    plain pointers, so a host, strided, wrongly typed or wrongly sized tensor is refused here
    instead of reaching a kernel."""
    if t is None:
        return None
    # one condition in the common case: a small call's time is its checks
    if not (t.is_cuda and t.is_contiguous() and (dtypes is None or _DTYPE_NAMES.get(t.dtype) in dtypes)
            and (numel is None or t.numel() == numel)):
        _refuse(t, what, dtypes, numel)
    return t.data_ptr()


def _refuse(t, what: str, dtypes, numel: Optional[int]):
    """Raises what _ptr found wrong (nothing where it only had not met the dtype yet)."""
    if not t.is_cuda:
        raise ValueError(f"{what}: a device tensor is required")
    if not t.is_contiguous():
        raise ValueError(f"{what}: a contiguous tensor is required")
    if dtypes is not None and _dt(t) not in dtypes:
        raise ValueError(f"{what}: dtype {t.dtype} is not one of {dtypes}")
    if numel is not None and t.numel() != numel:
        raise ValueError(f"{what}: {t.numel()} elements, expected {numel}")


def _shaped(t, what: str, dtypes, shape: Tuple[int, ...]) -> Optional[int]:
    """_ptr of a tensor of one shape: as many elements in another order would be read as if they lay in this one."""
    if t is None:
        return None
    if not (t.shape == shape and t.is_cuda and t.is_contiguous() and _DTYPE_NAMES.get(t.dtype) in dtypes):
        if t.shape != shape:
            raise ValueError(f"{what}: shape {tuple(t.shape)}, expected {tuple(shape)}")
        _refuse(t, what, dtypes, None)
    return t.data_ptr()


_DTYPE_NAMES = {}  # torch dtype -> its name


def _dt(t) -> str:
    name = _DTYPE_NAMES.get(t.dtype)
    if name is None:
        name = _DTYPE_NAMES[t.dtype] = str(t.dtype).replace("torch.", "")
    return name


_BF16 = ("bfloat16", "int16")  # bf16 values, or their raw 16-bit patterns


def _rows(t, what: str, rows: int, heads: int, d: int) -> Tuple[Optional[int], int]:
    """Address and token-row stride (elements) of a token-major [rows, heads, d] bf16 device
    tensor whose heads are contiguous within a row; its rows may be further apart (a view
    into a fused buffer).  None passes through with stride 0 (dense)."""
    if t is None:
        return None, 0
    if not t.is_cuda:
        raise ValueError(f"{what}: a device tensor is required")
    if _dt(t) not in _BF16:
        raise ValueError(f"{what}: dtype {t.dtype} is not one of {_BF16}")
    if t.shape != (rows, heads, d):
        raise ValueError(f"{what}: shape {tuple(t.shape)}, expected {(rows, heads, d)}")
    s0, s1, s2 = t.stride()
    if rows and (s2 != 1 or (heads > 1 and s1 != d)):
        raise ValueError(f"{what}: heads and channels must be contiguous within a token row")
    if rows > 1 and s0 < heads * d:
        # an expanded (broadcast) or overlapping view: the library would read rows that the
        # allocation does not hold (a stride of 0 even means "dense" to it)
        raise ValueError(f"{what}: token rows {s0} elements apart overlap; at least {heads * d} needed")
    return t.data_ptr(), (s0 if rows > 1 else heads * d)
_F32 = ("float32",)


def _stream(stream) -> int:
    if stream is not None:
        return stream.cuda_stream
    import torch
    # the handle of torch.cuda.current_stream() without building the object (a quarter of a small call's time)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _check(rc: int, what: str):
    if rc != HYDRA_OK:
        raise HydraError(rc, what)


def _set_rows(p: Problem, q, k, v):
    """Checks q, k, v against the problem and records their token-row strides in it."""
    qp, p.c.q_tok_stride = _rows(q, "q", p.nq, p.n_heads, 192)
    kp, p.c.k_tok_stride = _rows(k, "k", p.nk, p.n_kv_heads, 192)
    vp, p.c.v_tok_stride = _rows(v, "v", p.nk, p.n_kv_heads, 128)
    return qp, kp, vp


def attn_plan(p: Problem, workspace, stream=None):
    """Uploads the complete work plan of p into workspace (outside any graph capture), for
    the planned calls below."""
    _check(lib().hydra_scores_plan(p.ref, p.scores_ref, _ptr(workspace, "workspace"),
                                   workspace.numel() * workspace.element_size(), _stream(stream)), "hydra_attn_plan")


def _scratch(t) -> Tuple[Optional[int], int]:
    return _ptr(t, "scratch"), 0 if t is None else t.numel() * t.element_size()


def _fwd(what: str, merge: bool, p: Problem, q, k, v, o, lse, workspace, o_bf16, stream, planned, scratch):
    nqh = p.nq * p.n_heads
    if p.scores is not None:
        _here(p.scores.slopes, q, k, v, o, lse, o_bf16, workspace, scratch)
    qp, kp, vp = _set_rows(p, q, k, v)
    _check(lib().hydra_scores_fwd(p.ref, p.scores_ref, qp, kp, vp, _ptr(o, "o", _F32, nqh * 128),
                                  _ptr(lse, "lse", _F32, nqh), _ptr(o_bf16, "o_bf16", _BF16, nqh * 128),
                                  _ptr(workspace, "workspace"), workspace.numel() * workspace.element_size(),
                                  *_scratch(scratch), int(merge), int(planned), _stream(stream)), what)


def attn_fwd(p: Problem, q, k, v, o_part, lse_part, workspace, o_bf16=None, stream=None, planned=False, scratch=None):
    """Partial O (fp32) and LSE of one ring step; optional bf16 copy of O.  q, k, v may be
    views whose token rows are further apart than dense (e.g. slices of a fused buffer).
    planned: the workspace already holds p's plan (attn_plan); only kernels are launched,
    so the call can be recorded into a graph.  scratch: a uint8 device tensor of
    split_scratch_size(p), used by this call alone, in which a step of few work items is split
    over more workgroups (results then differ by rounding)."""
    _fwd("hydra_attn_fwd", False, p, q, k, v, o_part, lse_part, workspace, o_bf16, stream, planned, scratch)


def attn_fwd_merge(p: Problem, q, k, v, o_acc, lse_acc, workspace, o_bf16=None, stream=None, planned=False,
                   scratch=None):
    """(o_acc, lse_acc) <- exact merge with the partial that attn_fwd computes, in place and in the
    same kernel; optional bf16 copy of the merged O.  q, k, v, planned and scratch as in attn_fwd."""
    _fwd("hydra_attn_fwd_merge", True, p, q, k, v, o_acc, lse_acc, workspace, o_bf16, stream, planned, scratch)


def _bwd(what: str, p: Problem, q, k, v, o_final, lse_final, d_o, dq_acc, dk_acc, dv_acc, ds_buf, workspace,
         stream, planned, scratch):
    nqh, nkh = p.nq * p.n_heads, p.nk * p.n_kv_heads
    if p.scores is not None:
        _here(p.scores.slopes, q, k, v, o_final, lse_final, d_o, dq_acc, dk_acc, dv_acc, ds_buf, workspace, scratch)
    qp, kp, vp = _set_rows(p, q, k, v)
    _check(lib().hydra_scores_bwd(p.ref, p.scores_ref, qp, kp, vp,
                                  _ptr(o_final, "o_final", _BF16 + _F32 if p.scores else _BF16, nqh * 128),
                                  2 if o_final is None else o_final.element_size(),
                                  _ptr(lse_final, "lse_final", _F32, nqh), _ptr(d_o, "d_o", _BF16, nqh * 128),
                                  _ptr(dq_acc, "dq_acc", _F32, nqh * 192), _ptr(dk_acc, "dk_acc", _F32, nkh * 192),
                                  _ptr(dv_acc, "dv_acc", _F32, nkh * 128), _ptr(ds_buf, "ds_buf"),
                                  0 if ds_buf is None else ds_buf.numel() * ds_buf.element_size(),
                                  _ptr(workspace, "workspace"), workspace.numel() * workspace.element_size(),
                                  *_scratch(scratch), int(planned), _stream(stream)), what)


def attn_bwd(p: Problem, q, k, v, o_final_bf16, lse_final, d_o, dq_acc, dk_acc, dv_acc, workspace,
             stream=None, planned=False, scratch=None):
    """dQ/dK/dV of one ring step, accumulated (+=) into fp32 buffers (q, k, v, planned and scratch
    as in attn_fwd).  With modified scores o_final may also be the merged fp32 O: dQ and dK then do not
    carry its rounding to bf16."""
    _bwd("hydra_attn_bwd", p, q, k, v, o_final_bf16, lse_final, d_o, dq_acc, dk_acc, dv_acc, None, workspace, stream,
         planned, scratch)


def attn_bwd_noalloc(p: Problem, q, k, v, o_final_bf16, lse_final, d_o, dq_acc, dk_acc, dv_acc, stream=None):
    """attn_bwd with the library's own per-GPU scratch as the workspace (allocates nothing;
    calls on one GPU must not overlap).  For problems whose noalloc_size is within its 32 MiB, without
    modified scores."""
    if p.scores is not None and p.scores.any:
        raise ValueError("attn_bwd_noalloc has no form for modified scores")
    nqh, nkh = p.nq * p.n_heads, p.nk * p.n_kv_heads
    qp, kp, vp = _set_rows(p, q, k, v)
    _check(lib().hydra_attn_bwd_noalloc(p.ref, qp, kp, vp, _ptr(o_final_bf16, "o_final", _BF16, nqh * 128),
                                        _ptr(lse_final, "lse_final", _F32, nqh), _ptr(d_o, "d_o", _BF16, nqh * 128),
                                        _ptr(dq_acc, "dq_acc", _F32, nqh * 192),
                                        _ptr(dk_acc, "dk_acc", _F32, nkh * 192),
                                        _ptr(dv_acc, "dv_acc", _F32, nkh * 128), _stream(stream)),
           "hydra_attn_bwd_noalloc")


def bwd_ds_bytes(p: Problem, kv_heads_per_pass: int) -> int:
    """Bytes of dS scratch attn_bwd_ds needs per pass of that many K/V heads (0: the
    stored-dS path does not apply to p)."""
    return int(lib().hydra_scores_ds_bytes(p.ref, p.scores_ref, kv_heads_per_pass))


def attn_bwd_ds(p: Problem, q, k, v, o_final_bf16, lse_final, d_o, dq_acc, dk_acc, dv_acc, ds_buf, workspace,
                stream=None, scratch=None):
    """attn_bwd with dQ from the dS the dK/dV kernel stores into ds_buf (a uint8 device
    tensor; None or too small: the recompute path)."""
    _bwd("hydra_attn_bwd_ds", p, q, k, v, o_final_bf16, lse_final, d_o, dq_acc, dk_acc, dv_acc, ds_buf, workspace,
         stream, False, scratch)


def lse_merge(o_acc, lse_acc, o_part, lse_part, o_bf16=None, stream=None):
    """(o_acc, lse_acc) <- exact merge with (o_part, lse_part), in place."""
    n_rows, n_heads, d_v = o_acc.shape
    n = n_rows * n_heads
    _check(lib().hydra_lse_merge(n_rows, n_heads, d_v, _ptr(o_acc, "o_acc", _F32), _ptr(lse_acc, "lse_acc", _F32, n),
                                 _ptr(o_part, "o_part", _F32, n * d_v), _ptr(lse_part, "lse_part", _F32, n),
                                 _ptr(o_bf16, "o_bf16", _BF16, n * d_v), _stream(stream)), "hydra_lse_merge")


# ------------------------------------------------------------------ Ulysses x ring layout

def pack_heads(src, dst, cp_u: int, stream=None):
    """src [T, H, ...] -> dst [cp_u, T, H/cp_u, ...]: the send buffers of the forward exchange."""
    T, H = src.shape[0], src.shape[1]
    hb = src[0, 0].numel() * src.element_size()
    _check(lib().hydra_pack_heads(T, H, hb, cp_u, _ptr(src, "src"), _ptr(dst, "dst", (_dt(src),), src.numel()),
                                  _stream(stream)), "hydra_pack_heads")


def unpack_heads(src, dst, cp_u: int, stream=None):
    """src [cp_u, T, H/cp_u, ...] -> dst [T, H, ...]: the inverse of pack_heads."""
    T, H = dst.shape[0], dst.shape[1]
    hb = dst[0, 0].numel() * dst.element_size()
    _check(lib().hydra_unpack_heads(T, H, hb, cp_u, _ptr(src, "src", (_dt(dst),), dst.numel()), _ptr(dst, "dst"),
                                    _stream(stream)), "hydra_unpack_heads")


def zigzag_gather(src, dst, cp_r: int, r: int, stream=None):
    """Natural-order rows src [S, ...] -> ring rank r's rows dst [S/cp_r, ...]."""
    S = src.shape[0]
    rb = src[0].numel() * src.element_size()
    n = src.numel() // cp_r if cp_r > 0 else None
    _check(lib().hydra_zigzag_gather(S, rb, cp_r, r, _ptr(src, "src"), _ptr(dst, "dst", (_dt(src),), n),
                                     _stream(stream)), "hydra_zigzag_gather")


def zigzag_scatter(src, dst, cp_r: int, r: int, stream=None):
    """Ring rank r's rows src [S/cp_r, ...] -> their natural positions in dst [S, ...]."""
    S = dst.shape[0]
    rb = dst[0].numel() * dst.element_size()
    n = dst.numel() // cp_r if cp_r > 0 else None
    _check(lib().hydra_zigzag_scatter(S, rb, cp_r, r, _ptr(src, "src", (_dt(dst),), n), _ptr(dst, "dst"),
                                      _stream(stream)), "hydra_zigzag_scatter")


# ------------------------------------------------------------------ gated output

def unpack_heads_gated(recv, gate, y, stream=None):
    """recv [cp_u, T, H/cp_u, d_v] bf16, gate logits [T, H, 1 or d_v] bf16 -> y [T, H, d_v] bf16,
    y = unpacked output * sigmoid(gate)."""
    cp_u = recv.shape[0]
    T, H, d_v = y.shape
    e = gate.shape[-1]
    _check(lib().hydra_unpack_heads_gated(T, H, d_v, e, cp_u, _ptr(recv, "recv", _BF16, T * H * d_v),
                                          _ptr(gate, "gate", _BF16, T * H * e), _ptr(y, "y", _BF16),
                                          _stream(stream)), "hydra_unpack_heads_gated")


def pack_heads_gated_bwd(y, gate, d_y, d_send, d_gate, stream=None):
    """Backward of unpack_heads_gated from the gated output y: d_send [cp_u, T, H/cp_u, d_v] and
    d_gate [T, H, 1 or d_v], all bf16."""
    cp_u = d_send.shape[0]
    T, H, d_v = y.shape
    e, n = gate.shape[-1], T * H * d_v
    _check(lib().hydra_pack_heads_gated_bwd(T, H, d_v, e, cp_u, _ptr(y, "y", _BF16), _ptr(gate, "gate", _BF16, T * H * e),
                                            _ptr(d_y, "d_y", _BF16, n), _ptr(d_send, "d_send", _BF16, n),
                                            _ptr(d_gate, "d_gate", _BF16, T * H * e), _stream(stream)),
           "hydra_pack_heads_gated_bwd")


# ------------------------------------------------------------------ head norm

ACTIVATIONS = ("sigmoid", "silu")


def norm_workspace_size(n_tokens: int, n_heads: int, d: int) -> int:
    return int(lib().hydra_norm_workspace_size(n_tokens, n_heads, d))


def _norm(x, weight, bias, gate, center: bool, activation: str, eps: float):
    """The problem and the addresses of what both calls take, x [cp_u, T, H / cp_u, d]."""
    if activation not in ACTIVATIONS:
        raise ValueError(f"activation {activation!r}: one of {ACTIVATIONS} is required")
    cp_u, T, Hg, d = x.shape
    H = cp_u * Hg
    p = NormC(n_tokens=T, n_heads=H, d=d, cp_u=cp_u, center=int(bool(center)), activation=ACTIVATIONS.index(activation), eps=eps)
    return ctypes.byref(p), (T, H, d), (_ptr(x, "x", _BF16), _channels(weight, "weight", H, d), _channels(bias, "bias", H, d),
                                        _shaped(gate, "gate", _BF16, (T, H, d)))


def _channels(t, what: str, H: int, d: int) -> Optional[int]:
    """Address of float32 values per head and channel, [H, d] or one row of them."""
    return _shaped(t, what, _F32, (H * d,) if t is not None and t.dim() == 1 else (H, d))


def unpack_heads_normed(x, y, weight=None, bias=None, gate=None, center=True, activation="silu", eps: float = 1e-5,
                        stream=None):
    """x [cp_u, T, H/cp_u, d] bf16 -> y [T, H, d] bf16: every head normalised (center: its mean taken off), times weight
    plus bias [H, d] (or [H * d]) float32, times activation(gate), gate logits [T, H, d] bf16; without a gate, activation of
    that."""
    p, rows, ins = _norm(x, weight, bias, gate, center, activation, eps)
    _here(x, y, weight, bias, gate)
    _check(lib().hydra_unpack_heads_normed(p, *ins, _shaped(y, "y", _BF16, rows), _stream(stream)), "hydra_unpack_heads_normed")


def pack_heads_normed_bwd(x, d_y, d_x, weight=None, bias=None, gate=None, d_gate=None, d_weight=None, d_bias=None,
                          workspace=None, center=True, activation="silu", eps: float = 1e-5, stream=None):
    """Backward of unpack_heads_normed from its inputs and d_y [T, H, d] bf16: writes d_x (as x), with a gate d_gate, and
    where given d_weight and d_bias [H, d] (or [H * d]) float32, for which workspace is a uint8 device tensor of
    norm_workspace_size(T, H, d)."""
    p, rows, ins = _norm(x, weight, bias, gate, center, activation, eps)
    _here(x, d_y, d_x, weight, bias, gate, d_gate, d_weight, d_bias, workspace)
    _check(lib().hydra_pack_heads_normed_bwd(p, *ins, _shaped(d_y, "d_y", _BF16, rows), _shaped(d_x, "d_x", _BF16, x.shape),
                                             _shaped(d_gate, "d_gate", _BF16, rows), _channels(d_weight, "d_weight", *rows[1:]),
                                             _channels(d_bias, "d_bias", *rows[1:]), *_scratch(workspace), _stream(stream)),
           "hydra_pack_heads_normed_bwd")


# ------------------------------------------------------------------ rotary positions

class Rope:
    """Which columns are rotated, in which pairs, by which position and frequency (hydra_rope.h).

    pairs     pairs of each axis (text: one axis; their sum is half the rotated columns)
    pairing   "interleaved": columns (2j, 2j + 1); "halves": (j, j + half); "axis_halves": halves of each
              axis' own columns
    ladder    "whole": frequencies base^(-j / pairs) over all pairs; "axis": anew for each axis
    inv_freq  instead: every pair's frequency in radians per position
    """
    PAIRINGS = ("interleaved", "halves", "axis_halves")

    def __init__(self, pairs: Sequence[int] = (32,), pairing: str = "interleaved", base: float = 10000.0,
                 ladder: str = "whole", inv_freq: Optional[Sequence[float]] = None):
        pairs = [int(n) for n in pairs]
        if not 1 <= len(pairs) <= ROPE_MAX_AXES:
            raise ValueError(f"1 to {ROPE_MAX_AXES} axes")
        if pairing not in self.PAIRINGS or ladder not in ("whole", "axis"):
            raise ValueError(f"unknown pairing {pairing!r} or ladder {ladder!r}")
        self.n_axes, self.cols = len(pairs), 2 * sum(pairs)
        self.c = RopeC()
        self.c.n_axes = len(pairs)
        for i, n in enumerate(pairs):
            self.c.pairs[i] = n
        self.c.pairing = self.PAIRINGS.index(pairing)
        self.c.per_axis = int(ladder == "axis")
        self.c.base = base
        if inv_freq is None and 1 <= base < math.inf:  # made once here, not in every call (the library refuses other bases)
            n = sum(pairs)
            inv_freq = [base ** -(j / m if ladder == "axis" else (j + j0) / n)
                        for m, j0 in zip(pairs, [sum(pairs[:a]) for a in range(len(pairs))]) for j in range(m)]
        if inv_freq is not None:
            self.inv_freq = np.array(inv_freq, dtype=np.float64, order="C")  # a copy: the library reads it in every call
            if self.inv_freq.shape != (sum(pairs),):
                raise ValueError(f"inv_freq: shape {self.inv_freq.shape}, expected {(sum(pairs),)}")
            self.c.inv_freq = self.inv_freq.ctypes.data_as(ctypes.POINTER(ctypes.c_double))

    @property
    def ref(self):
        return ctypes.byref(self.c)


def _here(*tensors):
    """The launch goes to the current device: every tensor must be there."""
    import torch
    dev = torch.cuda.current_device()
    for t in tensors:
        if t is not None and t.get_device() not in (dev, -1):  # -1: on the host, which the addresses' check refuses
            raise ValueError(f"tensor on device {t.get_device()}, the current device is {dev}")


def _tok_rows(t, what: str, width: int) -> Tuple[int, int]:
    """Address and token-row stride of bf16 rows of `width` contiguous elements, [T, heads, d] or [T, d]."""
    if not t.is_cuda:
        raise ValueError(f"{what}: a device tensor is required")
    if _dt(t) not in _BF16:
        raise ValueError(f"{what}: dtype {t.dtype} is not one of {_BF16}")
    rows, *inner = t.shape
    s0, *strides = t.stride()
    if math.prod(inner) != width:
        raise ValueError(f"{what}: rows of {math.prod(inner)} elements, expected {width}")
    if not rows or not width:
        return t.data_ptr(), 0
    step = 1
    for n, s in zip(reversed(inner), reversed(strides)):
        if n > 1 and s != step:
            raise ValueError(f"{what}: heads and channels must be contiguous within a token row")
        step *= n
    if rows > 1 and s0 < width:
        raise ValueError(f"{what}: token rows {s0} elements apart overlap; at least {width} needed")
    return t.data_ptr(), (s0 if rows > 1 else 0)


def _positions(r: Rope, positions, n_tokens: int) -> int:
    if positions.shape != (r.n_axes, n_tokens) and (r.n_axes > 1 or positions.shape != (n_tokens,)):
        raise ValueError(f"positions: shape {tuple(positions.shape)}, expected {(r.n_axes, n_tokens)}")
    return _ptr(positions, "positions", ("int32",), r.n_axes * n_tokens)


def _grad(t, what: str, n: int) -> Tuple[int, int]:
    if _dt(t) not in _F32 + ("bfloat16",):
        raise ValueError(f"{what}: dtype {t.dtype} is neither float32 nor bfloat16")
    return _ptr(t, what, None, n), t.element_size()


def rope_q(r: Rope, src, positions, dst, cp_u: int = 1, stream=None):
    """src [T, H, d] bf16 -> dst [cp_u, T, H/cp_u, d] (cp_u = 1: also [T, H, d]) with the last r.cols columns
    of every head rotated by positions [n_axes, T] (one axis: also [T]) int32.  dst may be src (cp_u = 1): in place."""
    _here(src, positions, dst)
    T, H, d = src.shape
    sp, stride = _tok_rows(src, "src", H * d)
    if dst.data_ptr() == sp and T:
        if dst.shape != src.shape or dst.stride() != src.stride():
            raise ValueError("dst: in place, a tensor of src's shape and strides is required")
        dp = sp
    else:
        dp = _ptr(dst, "dst", _BF16, T * H * d)
    _check(lib().hydra_rope_q(r.ref, T, H, d, cp_u, sp, stride, _positions(r, positions, T), dp, _stream(stream)),
           "hydra_rope_q")


def rope_q_bwd(r: Rope, dq, positions, d_src, cp_u: int = 1, stream=None):
    """dq [cp_u, T, H/cp_u, d] float32 (the attention's accumulator) or bf16 -> d_src [T, H, d] bf16, the gradient
    of rope_q's src."""
    _here(dq, positions, d_src)
    T, H, d = d_src.shape
    gp, gb = _grad(dq, "dq", T * H * d)
    dp, stride = _tok_rows(d_src, "d_src", H * d)
    _check(lib().hydra_rope_q_bwd(r.ref, T, H, d, cp_u, gb, gp, _positions(r, positions, T), dp, stride,
                                  _stream(stream)), "hydra_rope_q_bwd")


def _kv_dims(r: Rope, kv, k, v) -> Tuple[int, int, int, int]:
    T, H, d = kv.shape
    d_v = 0 if v is None else v.shape[-1]
    if k.shape[-1] != d - d_v + r.cols:
        raise ValueError(f"k: heads of {k.shape[-1]} columns, expected {d - d_v + r.cols}")
    return T, H, d - d_v, d_v


def rope_kv(r: Rope, kv, k_pe, positions, k, v=None, cp_u: int = 1, stream=None):
    """kv [T, H, d_nope + d_v] and the heads' shared k_pe [T, r.cols], bf16 -> k [cp_u, T, H/cp_u, d_nope + r.cols]
    (a head's keys, then k_pe rotated) and v [cp_u, T, H/cp_u, d_v] (None: kv holds keys only)."""
    _here(kv, k_pe, positions, k, v)
    T, H, d_nope, d_v = _kv_dims(r, kv, k, v)
    sp, stride = _tok_rows(kv, "kv", H * (d_nope + d_v))
    if k_pe.shape[0] != T:
        raise ValueError(f"k_pe: {k_pe.shape[0]} rows, expected {T}")
    pp, pe_stride = _tok_rows(k_pe, "k_pe", r.cols)
    _check(lib().hydra_rope_kv(r.ref, T, H, d_nope, d_v, cp_u, sp, stride, pp, pe_stride, _positions(r, positions, T),
                               _ptr(k, "k", _BF16, T * H * (d_nope + r.cols)), _ptr(v, "v", _BF16, T * H * d_v),
                               _stream(stream)), "hydra_rope_kv")


def rope_kv_bwd(r: Rope, dk, dv, positions, d_kv, d_k_pe, cp_u: int = 1, stream=None):
    """Backward of rope_kv: dk and dv (None: no values), float32 or bf16, as rope_kv's k and v -> d_kv
    [T, H, d_nope + d_v] and d_k_pe [T, r.cols] (summed over the heads), bf16."""
    _here(dk, dv, positions, d_kv, d_k_pe)
    T, H, d_nope, d_v = _kv_dims(r, d_kv, dk, dv)
    gp, gb = _grad(dk, "dk", T * H * (d_nope + r.cols))
    vp = None
    if dv is not None:
        vp, vb = _grad(dv, "dv", T * H * d_v)
        if vb != gb:
            raise ValueError("dk and dv must have one dtype")
    dp, stride = _tok_rows(d_kv, "d_kv", H * (d_nope + d_v))
    if d_k_pe.shape[0] != T:
        raise ValueError(f"d_k_pe: {d_k_pe.shape[0]} rows, expected {T}")
    pp, pe_stride = _tok_rows(d_k_pe, "d_k_pe", r.cols)
    _check(lib().hydra_rope_kv_bwd(r.ref, T, H, d_nope, d_v, cp_u, gb, gp, vp, _positions(r, positions, T), dp,
                                   stride, pp, pe_stride, _stream(stream)), "hydra_rope_kv_bwd")


# ------------------------------------------------------------------ linear attention

class Linear:
    """Linear attention with a decay for each head over packed sequences (hydra_linear.h): rows
    cu_seqlens[s] .. cu_seqlens[s + 1] - 1 are sequence s."""

    def __init__(self, cu_seqlens, n_heads: int, d_k: int = 128, d_v: int = 128, n_kv_heads: int = 0, scale: float = 0.0):
        given = np.asarray(cu_seqlens)
        self.cu = np.ascontiguousarray(given.astype(np.int32))
        if self.cu.ndim != 1 or len(self.cu) < 2 or not np.array_equal(self.cu, given):
            raise ValueError("cu_seqlens: a list of at least two integers of 32 bits is required")
        self.n_seqs, self.n_tokens = len(self.cu) - 1, int(self.cu[-1])
        self.n_heads, self.n_kv_heads, self.d_k, self.d_v = n_heads, n_kv_heads or n_heads, d_k, d_v
        self.c = LinearC(n_heads=n_heads, n_kv_heads=n_kv_heads, d_k=d_k, d_v=d_v, scale=scale, n_seqs=self.n_seqs)
        self.c.cu_seqlens = self.cu.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))

    @property
    def ref(self):
        return ctypes.byref(self.c)

    @property
    def state_shape(self) -> Tuple[int, int, int, int]:
        return self.n_seqs, self.n_heads, self.d_k, self.d_v

    @property
    def state_numel(self) -> int:
        return math.prod(self.state_shape)


def linear_workspace_size(p: Linear) -> int:
    return int(lib().hydra_linear_workspace_size(p.ref))


def linear_plan(p: Linear, workspace, stream=None):
    """Uploads the work plan of p into workspace (outside any graph capture), for calls with planned=True."""
    _here(workspace)
    _check(lib().hydra_linear_plan(p.ref, _ptr(workspace, "workspace"), workspace.numel() * workspace.element_size(),
                                   _stream(stream)), "hydra_linear_plan")


def _linear_rows(p: Linear, q, k, v) -> Tuple[int, int, int]:
    """Checks q, k, v (tensors may have more rows than p) and records their token-row strides in it."""
    out = []
    for t, what, heads, d in ((q, "q", p.n_heads, p.d_k), (k, "k", p.n_kv_heads, p.d_k), (v, "v", p.n_kv_heads, p.d_v)):
        ptr, stride = _rows(t, what, _more_rows(t, what, p.n_tokens), heads, d)
        setattr(p.c, what + "_tok_stride", stride)
        out.append(ptr)
    return tuple(out)


def _more_rows(t, what: str, rows: int) -> int:
    if t.shape[0] < rows:
        raise ValueError(f"{what}: {t.shape[0]} rows, at least {rows} needed")
    return t.shape[0]


def _dense_rows(t, what: str, rows: int, heads: int, d: int) -> Optional[int]:
    """Address of a dense [rows or more, heads, d] bf16 tensor."""
    if t is None:
        return None
    if tuple(t.shape[1:]) != (heads, d):
        raise ValueError(f"{what}: shape {tuple(t.shape)}, expected {(rows, heads, d)}")
    return _ptr(t, what, _BF16, _more_rows(t, what, rows) * heads * d)


def linear_fwd(p: Linear, q, k, v, decay, o, workspace, state_in=None, state_out=None, planned=False, stream=None):
    """o [T, H, d_v] bf16 (None: the last states alone) and, where given, state_out [n_seqs, H, d_k, d_v] float32 from
    q [T, H, d_k], k [T, Hkv, d_k], v [T, Hkv, d_v] bf16 (token rows may be further apart than dense), the log decays
    [H] float32 and the states that the sequences start from (None: zero; may be state_out).  Rows from
    cu_seqlens[-1] on are left as they are.  workspace: a uint8 device tensor of linear_workspace_size(p), written by
    the call; planned: it already holds p's plan, and only kernels are launched."""
    _here(q, k, v, decay, o, workspace, state_in, state_out)
    qp, kp, vp = _linear_rows(p, q, k, v)
    _check(lib().hydra_linear_fwd(p.ref, qp, kp, vp, _ptr(decay, "decay", _F32, p.n_heads),
                                  _shaped(state_in, "state_in", _F32, p.state_shape),
                                  _dense_rows(o, "o", p.n_tokens, p.n_heads, p.d_v),
                                  _shaped(state_out, "state_out", _F32, p.state_shape), _ptr(workspace, "workspace"),
                                  workspace.numel() * workspace.element_size(), int(planned), _stream(stream)),
           "hydra_linear_fwd")


def linear_bwd(p: Linear, q, k, v, decay, d_o, dq, dk, dv, workspace, state_in=None, d_state_out=None, d_state_in=None,
               planned=False, stream=None):
    """Backward of linear_fwd: writes dq, dk, dv (bf16, as q, k, v, dense) and, where given, d_state_in, from d_o and the
    gradients of the last states (None: zero)."""
    _here(q, k, v, decay, d_o, dq, dk, dv, workspace, state_in, d_state_out, d_state_in)
    qp, kp, vp = _linear_rows(p, q, k, v)
    T, H, Hk = p.n_tokens, p.n_heads, p.n_kv_heads
    _check(lib().hydra_linear_bwd(p.ref, qp, kp, vp, _ptr(decay, "decay", _F32, H),
                                  _shaped(state_in, "state_in", _F32, p.state_shape), _dense_rows(d_o, "d_o", T, H, p.d_v),
                                  _shaped(d_state_out, "d_state_out", _F32, p.state_shape),
                                  _dense_rows(dq, "dq", T, H, p.d_k), _dense_rows(dk, "dk", T, Hk, p.d_k),
                                  _dense_rows(dv, "dv", T, Hk, p.d_v),
                                  _shaped(d_state_in, "d_state_in", _F32, p.state_shape), _ptr(workspace, "workspace"),
                                  workspace.numel() * workspace.element_size(), int(planned), _stream(stream)),
           "hydra_linear_bwd")


def linear_step(q, k, v, decay, state, o, slots=None, state_out=None, scale: float = 0.0, stream=None):
    """One token of every row's sequence: q [n, H, d_k], k [n, Hkv, d_k], v [n, Hkv, d_v] -> o [n, H, d_v], bf16.
    state [n_slots, H, d_k, d_v] float32 is replaced (or state_out, of its shape, receives the new states).  slots:
    int32 [n], the state of each row (None: row i has state i); rows whose slot is not in the pool are padding and are
    left as they are; rows of one slot are taken in their order."""
    _here(q, k, v, decay, state, o, slots, state_out)
    n, H, d_k = q.shape
    Hk, d_v = v.shape[1], v.shape[2]
    out = state if state_out is None else state_out
    if state.shape[1:] != (H, d_k, d_v) or (out is not state and out.shape != state.shape):
        raise ValueError(f"state: shape {tuple(state.shape)}, expected {('n_slots', H, d_k, d_v)}, and state_out the same")
    _check(lib().hydra_linear_step(n, state.shape[0], H, Hk, d_k, d_v, scale, _ptr(q, "q", _BF16),
                                   _shaped(k, "k", _BF16, (n, Hk, d_k)), _shaped(v, "v", _BF16, (n, Hk, d_v)),
                                   _ptr(decay, "decay", _F32, H), _ptr(state, "state", _F32), _ptr(out, "state_out", _F32),
                                   _ptr(slots, "slots", ("int32",), n), _shaped(o, "o", _BF16, (n, H, d_v)),
                                   _stream(stream)), "hydra_linear_step")


# ------------------------------------------------------------------ scheduler (host only)

def schedule(lengths, n_ranks: int, token_budget: int, pp: int = 1, theta_over_c: float = 0.0, cap: int = 0,
             balance_ratio: float = 0.0):
    """Load-driven DCP placement of a batch: per sequence (micro-batch, group start, group
    size) as three int32 arrays, plus the targets and counts as a dict."""
    ln = np.ascontiguousarray(np.asarray(lengths, dtype=np.int64))
    n = ln.size
    mb, st, sz = (np.empty(n, np.int32) for _ in range(3))
    cfg = SchedConfig(n_ranks, token_budget, pp, theta_over_c, cap, balance_ratio)
    summ = SchedSummary()
    p32 = lambda a: a.ctypes.data_as(ctypes.POINTER(ctypes.c_int32))
    _check(lib().hydra_schedule(ln.ctypes.data_as(ctypes.POINTER(ctypes.c_int64)), n, ctypes.byref(cfg), p32(mb),
                                p32(st), p32(sz), ctypes.byref(summ)), "hydra_schedule")
    info = {f: getattr(summ, f) for f, _ in SchedSummary._fields_}
    info["W"] = (info.pop("w_hi") << 62) + info.pop("w_lo")
    return mb, st, sz, info


def profile_start():
    """Start timing every kernel the library launches (HIP events on the launch stream)."""
    _check(lib().hydra_profile_start(), "hydra_profile_start")


def profile_stop() -> dict:
    """Stop timing; returns {kernel: {launches, total_ms, min_ms, max_ms, avg_ms}}."""
    buf = (KernelStat * 64)()
    n = lib().hydra_profile_stop(buf, 64)
    if n < 0:
        raise HydraError(n, "hydra_profile_stop")
    out = {}
    for i in range(min(n, 64)):
        k = buf[i]
        out[k.name.decode()] = dict(launches=k.launches, total_ms=k.total_ms, min_ms=k.min_ms,
                                    max_ms=k.max_ms, avg_ms=k.total_ms / max(k.launches, 1))
    return out
