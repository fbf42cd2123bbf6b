"""MI355X (gfx950) Fast Multipole Attention forward pass.

Thin ctypes binding of the C ABI in include/fma.h (libfma_mi355x.so, built by
``paper_2310_11960_amd.build``).  The functions ``fma_*`` below carry the C
names and only marshal arguments: every step of the computation runs in the
library's HIP kernels.  PyTorch supplies device memory and the current
stream.  There is no CPU fallback: without the built library every call
raises.

High-level use::

    op = FMA(ndim=1, batch=B, heads=H, seq_len=n, block=128, causal=True,
             dtype=torch.bfloat16)
    out = op.forward(q, k, v, wk, wv)        # q, k, v: [B, H, n, d] on cuda
"""
from __future__ import annotations

import contextlib
import ctypes
import os
import re
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libfma_mi355x.so")
HEADER_PATH = os.path.join(os.path.dirname(_HERE), "include", "fma.h")

FMA_OK = 0
FMA_ERR_NULL = 1
FMA_ERR_SHAPE = 2
FMA_ERR_UNSUPPORTED = 3
FMA_ERR_WORKSPACE = 4
FMA_ERR_HIP = 5
FMA_ERR_HOST_ALLOC = 6
FMA_ERR_ALIGN = 7
FMA_ERR_ARG = 8
FMA_F32 = 0
FMA_BF16 = 1
FMA_NORM_JOINT = 0
FMA_NORM_PER_LEVEL = 1

HEAD_DIM = 64


class FmaError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__("FMA status %d: %s" % (status, message))
        self.status = status


class fma_desc_t(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_int32),
        ("ndim", ctypes.c_int32),
        ("batch", ctypes.c_int32),
        ("heads", ctypes.c_int32),
        ("seq_len", ctypes.c_int64),
        ("side", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("block", ctypes.c_int32),
        ("num_levels", ctypes.c_int32),
        ("causal", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("weights_per_head", ctypes.c_int32),
        ("softmax_scale", ctypes.c_float),
        ("rank", ctypes.c_int32),
        ("norm", ctypes.c_int32),
        ("query_downsample", ctypes.c_int32),
    ]


class fma_view_t(ctypes.Structure):
    _fields_ = [
        ("data", ctypes.c_void_p),
        ("batch_stride", ctypes.c_int64),
        ("head_stride", ctypes.c_int64),
        ("token_stride", ctypes.c_int64),
    ]


class fma_qk_desc_t(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("heads", ctypes.c_int32),
        ("kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("rotary_dim", ctypes.c_int32),
        ("axes", ctypes.c_int32),
        ("side", ctypes.c_int32),
        ("interleaved", ctypes.c_int32),
        ("repeat_kv", ctypes.c_int32),
        ("eps", ctypes.c_float),
        ("base", ctypes.c_double),
    ]


class fma_cache_desc_t(ctypes.Structure):
    _fields_ = [
        ("struct_size", ctypes.c_int32),
        ("dtype", ctypes.c_int32),
        ("heads", ctypes.c_int32),
        ("kv_heads", ctypes.c_int32),
        ("head_dim", ctypes.c_int32),
        ("block", ctypes.c_int32),
        ("max_seq_len", ctypes.c_int64),
        ("rank", ctypes.c_int32),
        ("weights_per_head", ctypes.c_int32),
        ("norm", ctypes.c_int32),
        ("softmax_scale", ctypes.c_float),
    ]


class fma_cache_batch_t(ctypes.Structure):
    _fields_ = [
        ("k_pages", ctypes.c_void_p),
        ("v_pages", ctypes.c_void_p),
        ("summaries", ctypes.c_void_p),
        ("num_pages", ctypes.c_int64),
        ("num_summaries", ctypes.c_int64),
        ("page_table", ctypes.c_void_p),
        ("summary_table", ctypes.c_void_p),
        ("table_stride", ctypes.c_int64),
        ("cu_tokens", ctypes.c_void_p),
        ("start", ctypes.c_void_p),
        ("sequences", ctypes.c_int32),
        ("max_chunk", ctypes.c_int32),
        ("rows", ctypes.c_int64),
    ]


_lib = None


def library() -> ctypes.CDLL:
    """Load the built HIP library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("libfma_mi355x.so is not built; run `python -m paper_2310_11960_amd.build`")
    lib = ctypes.CDLL(LIB_PATH)
    vp, st, i32, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int32, ctypes.c_int64
    lib.fma_plan.argtypes = [ctypes.POINTER(fma_desc_t), ctypes.POINTER(vp)]
    lib.fma_destroy.argtypes = [vp]
    lib.fma_workspace_size.argtypes = [vp, ctypes.POINTER(ctypes.c_size_t)]
    lib.fma_weights_len.argtypes = [vp, ctypes.POINTER(i64)]
    lib.fma_coarse_rows.argtypes = [vp, ctypes.POINTER(i64)]
    lib.fma_num_levels.argtypes = [vp, ctypes.POINTER(i32)]
    for name in ("fma_forward_1d", "fma_forward_2d"):
        getattr(lib, name).argtypes = [vp, vp, vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.fma_coarsen.argtypes = [vp, vp, vp, vp, vp, vp, ctypes.c_size_t, vp]
    lib.fma_attend.argtypes = [vp, vp, vp, vp, vp, ctypes.c_size_t, vp, vp]
    lib.fma_interaction_lists.argtypes = [vp, vp, vp]
    lib.fma_dense_reference.argtypes = [vp, vp, vp, vp, vp, vp]
    lib.fma_backward_workspace_size.argtypes = [vp, ctypes.POINTER(ctypes.c_size_t)]
    lib.fma_forward_linear.argtypes = [vp] * 9 + [ctypes.c_size_t, vp]
    lib.fma_backward.argtypes = [vp] + [vp] * 12 + [vp, ctypes.c_size_t, vp]
    lib.fma_backward_linear.argtypes = [vp] + [vp] * 14 + [vp, ctypes.c_size_t, vp]
    lib.fma_forward_static.argtypes = [vp] * 8
    lib.fma_stream_reference.argtypes = [vp, ctypes.c_size_t, vp, ctypes.c_size_t, i32, vp]
    lib.fma_plan_params.argtypes = [vp, ctypes.POINTER(i64), i32, ctypes.POINTER(i32)]
    view = vp   # (structs by reference, or the addresses of some that lie together)
    lib.fma_qk_plan.argtypes = [ctypes.POINTER(fma_qk_desc_t), ctypes.POINTER(ctypes.c_double), ctypes.POINTER(vp)]
    lib.fma_qk_destroy.argtypes = [vp]
    lib.fma_qk_norm_rope.argtypes = [vp, i32, i64, view, view, view, vp, vp, vp, view, view, view, vp]
    lib.fma_qk_backward_workspace_size.argtypes = [vp, i32, i64, ctypes.POINTER(ctypes.c_size_t)]
    lib.fma_qk_norm_rope_backward.argtypes = [vp, i32, i64, view, view, vp, vp, vp] + [view] * 6 + [
        vp, vp, vp, ctypes.c_size_t, vp]
    batch = vp
    lib.fma_cache_plan.argtypes = [ctypes.POINTER(fma_cache_desc_t), ctypes.POINTER(vp)]
    lib.fma_cache_destroy.argtypes = [vp]
    lib.fma_cache_sizes.argtypes = [vp, ctypes.POINTER(i32), ctypes.POINTER(i64), ctypes.POINTER(i64)]
    lib.fma_cache_append.argtypes = [vp, batch, view, view, vp, vp, vp]
    lib.fma_cache_attend.argtypes = [vp, batch, view, view, vp]
    lib.fma_cache_step.argtypes = [vp, batch, view, view, view, vp, vp, view, vp]
    for name in ("fma_cache_plan", "fma_cache_destroy", "fma_cache_sizes", "fma_cache_append", "fma_cache_attend",
                 "fma_cache_step", "fma_qk_plan", "fma_qk_destroy", "fma_qk_norm_rope", "fma_qk_backward_workspace_size",
                 "fma_qk_norm_rope_backward", "fma_plan", "fma_destroy", "fma_workspace_size", "fma_weights_len", "fma_coarse_rows",
                 "fma_num_levels", "fma_forward_1d", "fma_forward_2d", "fma_coarsen", "fma_attend",
                 "fma_interaction_lists", "fma_dense_reference", "fma_backward_workspace_size",
                 "fma_backward", "fma_backward_linear", "fma_forward_linear", "fma_forward_static",
                 "fma_stream_reference", "fma_plan_params"):
        getattr(lib, name).restype = st
    lib.fma_last_error.argtypes = []
    lib.fma_last_error.restype = ctypes.c_char_p
    _lib = lib
    return lib


def header_functions() -> list[str]:
    """Names of the functions include/fma.h declares."""
    text = open(HEADER_PATH).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    return sorted(set(re.findall(r"\b(fma_[a-z0-9_]+)\s*\(", text)))


def _check(status: int) -> None:
    if status != FMA_OK:
        raise FmaError(status, library().fma_last_error().decode())


def _ptr(t) -> int | None:
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


# the current stream's handle without the objects around it, where torch has such a call
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream) -> int | None:
    if stream is None:
        if _raw_stream is not None and torch.cuda.is_initialized():
            return _raw_stream(torch.cuda.current_device())
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


# ---------------------------------------------------------------- C names
def fma_plan(desc: fma_desc_t) -> int:
    h = ctypes.c_void_p()
    _check(library().fma_plan(ctypes.byref(desc), ctypes.byref(h)))
    return h.value


def fma_destroy(plan: int) -> None:
    _check(library().fma_destroy(plan))


def fma_workspace_size(plan: int) -> int:
    x = ctypes.c_size_t()
    _check(library().fma_workspace_size(plan, ctypes.byref(x)))
    return x.value


def fma_weights_len(plan: int) -> int:
    x = ctypes.c_int64()
    _check(library().fma_weights_len(plan, ctypes.byref(x)))
    return x.value


def fma_coarse_rows(plan: int) -> int:
    x = ctypes.c_int64()
    _check(library().fma_coarse_rows(plan, ctypes.byref(x)))
    return x.value


def fma_num_levels(plan: int) -> int:
    x = ctypes.c_int32()
    _check(library().fma_num_levels(plan, ctypes.byref(x)))
    return x.value


def fma_forward_1d(plan, q, k, v, wk, wv, out, workspace, workspace_bytes, stream=None):
    _check(library().fma_forward_1d(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(wk), _ptr(wv), _ptr(out),
                                    _ptr(workspace), workspace_bytes, _stream(stream)))


def fma_forward_2d(plan, q, k, v, wk, wv, out, workspace, workspace_bytes, stream=None):
    _check(library().fma_forward_2d(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(wk), _ptr(wv), _ptr(out),
                                    _ptr(workspace), workspace_bytes, _stream(stream)))


def fma_coarsen(plan, k, v, wk, wv, workspace, workspace_bytes, stream=None):
    _check(library().fma_coarsen(plan, _ptr(k), _ptr(v), _ptr(wk), _ptr(wv), _ptr(workspace),
                                 workspace_bytes, _stream(stream)))


def fma_attend(plan, q, k, v, workspace, workspace_bytes, out, stream=None):
    _check(library().fma_attend(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(workspace), workspace_bytes,
                                _ptr(out), _stream(stream)))


def fma_interaction_lists(plan, dev_out, stream=None):
    _check(library().fma_interaction_lists(plan, _ptr(dev_out), _stream(stream)))


def fma_dense_reference(plan, q, k, v, out, stream=None):
    _check(library().fma_dense_reference(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(out), _stream(stream)))


def fma_forward_linear(plan, q, k, v, wq, wk, wv, out, workspace, workspace_bytes, stream=None):
    _check(library().fma_forward_linear(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(wq), _ptr(wk), _ptr(wv), _ptr(out),
                                        _ptr(workspace), workspace_bytes, _stream(stream)))


def fma_forward_static(plan, q, k, v, wk, wv, out, stream=None):
    _check(library().fma_forward_static(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(wk), _ptr(wv), _ptr(out),
                                        _stream(stream)))


def fma_stream_reference(src, src_bytes, dst, dst_bytes, write_every, stream=None):
    _check(library().fma_stream_reference(_ptr(src), src_bytes, _ptr(dst), dst_bytes, write_every, _stream(stream)))


PLAN_PARAM_NAMES = [
    "n", "side", "block", "nbx", "qtile", "tiles_per_slice", "nslice", "R", "causal", "nslot", "slot_group",
    "rank", "norm_level", "ndim", "esize", "heads", "w_stride", "wlen", "nsets", "chunk", "run", "nchunk",
    "tiles_y", "first_partial", "npartial", "part_span", "part_count", "depth", "wave_lds",
    "coarsen_smem", "part_offset", "coarse_bytes", "ws_bytes", "linear", "heads_w", "dtype", "pair2d",
    "height", "nby", "tiles_x", "head_dim"]
SET_PARAM_NAMES = ("off", "M", "My", "size", "woff", "lvl")


def fma_plan_params(plan: int) -> dict:
    """The plan's launch parameters (fma_plan_params) as a dict; per-set
    tables under "sets" (dicts of off, M, My, size, woff, lvl)."""
    nb, ns = len(PLAN_PARAM_NAMES), len(SET_PARAM_NAMES)
    cap = nb + ns * 64
    buf = (ctypes.c_int64 * cap)()
    cnt = ctypes.c_int32()
    _check(library().fma_plan_params(plan, buf, cap, ctypes.byref(cnt)))
    vals = list(buf[:cnt.value])
    d = dict(zip(PLAN_PARAM_NAMES, vals[:nb]))
    d["sets"] = [dict(zip(SET_PARAM_NAMES, vals[nb + ns * e:nb + ns * (e + 1)])) for e in range(d["nsets"])]
    return d


def fma_backward_workspace_size(plan: int) -> int:
    x = ctypes.c_size_t()
    _check(library().fma_backward_workspace_size(plan, ctypes.byref(x)))
    return x.value


def fma_backward(plan, q, k, v, wk, wv, out, dout, dq, dk, dv, dwk, dwv, workspace, workspace_bytes,
                 stream=None):
    _check(library().fma_backward(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(wk), _ptr(wv), _ptr(out), _ptr(dout),
                                  _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dwk), _ptr(dwv), _ptr(workspace),
                                  workspace_bytes, _stream(stream)))


def fma_backward_linear(plan, q, k, v, wk, wv, wq, out, dout, dq, dk, dv, dwk, dwv, dwq, workspace,
                        workspace_bytes, stream=None):
    _check(library().fma_backward_linear(plan, _ptr(q), _ptr(k), _ptr(v), _ptr(wk), _ptr(wv), _ptr(wq),
                                         _ptr(out), _ptr(dout), _ptr(dq), _ptr(dk), _ptr(dv), _ptr(dwk),
                                         _ptr(dwv), _ptr(dwq), _ptr(workspace), workspace_bytes, _stream(stream)))


def _ref(x):
    """A struct argument: the struct, its address or None."""
    return x if x is None or isinstance(x, int) else ctypes.byref(x)


def fma_qk_plan(desc: fma_qk_desc_t, inv_freq=None) -> int:
    h = ctypes.c_void_p()
    rates = None if inv_freq is None else (ctypes.c_double * len(inv_freq))(*inv_freq)
    _check(library().fma_qk_plan(ctypes.byref(desc), rates, ctypes.byref(h)))
    return h.value


def fma_qk_destroy(plan: int) -> None:
    _check(library().fma_qk_destroy(plan))


def fma_qk_norm_rope(plan, batch, tokens, q, k, v, gamma_q, gamma_k, positions, q_out, k_out, v_out, stream=None):
    """q, k, v, q_out, k_out, v_out: fma_view_t (v, v_out may be None)."""
    _check(library().fma_qk_norm_rope(plan, batch, tokens, _ref(q), _ref(k), _ref(v), _ptr(gamma_q), _ptr(gamma_k),
                                      _ptr(positions), _ref(q_out), _ref(k_out), _ref(v_out), _stream(stream)))


def fma_qk_backward_workspace_size(plan: int, batch: int, tokens: int) -> int:
    x = ctypes.c_size_t()
    _check(library().fma_qk_backward_workspace_size(plan, batch, tokens, ctypes.byref(x)))
    return x.value


def fma_qk_norm_rope_backward(plan, batch, tokens, q, k, gamma_q, gamma_k, positions, g_q, g_k, g_v, dq, dk, dv,
                              dgamma_q, dgamma_k, workspace, workspace_bytes, stream=None):
    """q, k, g_q, g_k, g_v, dq, dk, dv: fma_view_t (g_v, dv may be None)."""
    _check(library().fma_qk_norm_rope_backward(plan, batch, tokens, _ref(q), _ref(k), _ptr(gamma_q), _ptr(gamma_k),
                                               _ptr(positions), _ref(g_q), _ref(g_k), _ref(g_v), _ref(dq), _ref(dk),
                                               _ref(dv), _ptr(dgamma_q), _ptr(dgamma_k), _ptr(workspace),
                                               workspace_bytes, _stream(stream)))


def fma_cache_plan(desc: fma_cache_desc_t) -> int:
    h = ctypes.c_void_p()
    _check(library().fma_cache_plan(ctypes.byref(desc), ctypes.byref(h)))
    return h.value


def fma_cache_destroy(plan: int) -> None:
    _check(library().fma_cache_destroy(plan))


def fma_cache_sizes(plan: int) -> tuple[int, int, int]:
    """(coarse sets, weights per head, blocks of the longest sequence)."""
    sets, wlen, blocks = ctypes.c_int32(), ctypes.c_int64(), ctypes.c_int64()
    _check(library().fma_cache_sizes(plan, ctypes.byref(sets), ctypes.byref(wlen), ctypes.byref(blocks)))
    return sets.value, wlen.value, blocks.value


def fma_cache_append(plan, batch, k, v, wk, wv, stream=None):
    """batch: fma_cache_batch_t; k, v: fma_view_t."""
    _check(library().fma_cache_append(plan, _ref(batch), _ref(k), _ref(v), _ptr(wk), _ptr(wv), _stream(stream)))


def fma_cache_attend(plan, batch, q, out, stream=None):
    _check(library().fma_cache_attend(plan, _ref(batch), _ref(q), _ref(out), _stream(stream)))


def fma_cache_step(plan, batch, q, k, v, wk, wv, out, stream=None):
    _check(library().fma_cache_step(plan, _ref(batch), _ref(q), _ref(k), _ref(v), _ptr(wk), _ptr(wv), _ref(out),
                                    _stream(stream)))


def fma_last_error() -> str:
    return library().fma_last_error().decode()


# ---------------------------------------------------------------- object API
_DTYPES = {torch.float32: FMA_F32, torch.bfloat16: FMA_BF16}


def make_desc(ndim=1, batch=1, heads=1, seq_len=0, block=64, causal=False, dtype=torch.bfloat16,
              side=0, head_dim=HEAD_DIM, num_levels=-1, weights_per_head=True, softmax_scale=0.0,
              rank=1, norm=FMA_NORM_JOINT, linear=False):
    d = fma_desc_t()
    d.struct_size = ctypes.sizeof(fma_desc_t)
    d.ndim = ndim
    d.batch = batch
    d.heads = heads
    d.seq_len = seq_len
    d.side = side
    d.head_dim = head_dim
    d.block = block
    d.num_levels = num_levels
    d.causal = int(bool(causal))
    d.dtype = _DTYPES[dtype] if isinstance(dtype, torch.dtype) else int(dtype)
    d.weights_per_head = int(bool(weights_per_head))
    d.softmax_scale = softmax_scale
    d.rank = rank
    d.norm = norm
    d.query_downsample = int(bool(linear))
    return d


class FMA:
    """One plan (shape + options) and the calls that use it."""

    def __init__(self, ndim=1, batch=1, heads=1, seq_len=0, block=64, causal=False,
                 dtype=torch.bfloat16, side=0, weights_per_head=True, softmax_scale=0.0,
                 num_levels=-1, head_dim=HEAD_DIM, rank=1, norm=FMA_NORM_JOINT, linear=False):
        if ndim == 2 and side == 0:
            side = int(round(seq_len ** 0.5))
        self.desc = make_desc(ndim, batch, heads, seq_len, block, causal, dtype, side, head_dim,
                              num_levels, weights_per_head, softmax_scale, rank, norm, linear)
        self.rank, self.norm, self.linear = rank, norm, linear
        self.ndim, self.batch, self.heads, self.n = ndim, batch, heads, seq_len
        self.side, self.block, self.causal, self.dtype = side, block, causal, dtype
        self.head_dim = head_dim
        self.handle = fma_plan(self.desc)
        self.workspace_bytes = fma_workspace_size(self.handle)
        self.weights_len = fma_weights_len(self.handle)
        self.coarse_rows = fma_coarse_rows(self.handle)
        self.levels = fma_num_levels(self.handle)
        self.backward_workspace_bytes = fma_backward_workspace_size(self.handle)

    def __del__(self):
        h = getattr(self, "handle", None)
        if h:
            try:
                library().fma_destroy(h)
            except Exception:
                pass
            self.handle = None

    # ---------------------------------------------------------- helpers
    def new_workspace(self, device) -> torch.Tensor:
        return torch.empty(max(self.workspace_bytes, 16), dtype=torch.uint8, device=device)

    def coarse_views(self, workspace: torch.Tensor):
        """(K_bar, V_bar) views [B, H, R, d] of a workspace filled by coarsen()."""
        R = self.coarse_rows
        numel = self.batch * self.heads * R * self.head_dim
        flat = workspace[: 2 * numel * (2 if self.dtype == torch.bfloat16 else 4)].view(self.dtype)
        kb = flat[:numel].view(self.batch, self.heads, R, self.head_dim)
        vb = flat[numel:2 * numel].view(self.batch, self.heads, R, self.head_dim)
        return kb, vb

    # ---------------------------------------------------------- calls
    def forward(self, q, k, v, wk=None, wv=None, out=None, workspace=None, stream=None):
        if out is None:
            out = torch.empty_like(q)
        if workspace is None:
            workspace = self.new_workspace(q.device)
        fn = fma_forward_1d if self.ndim == 1 else fma_forward_2d
        fn(self.handle, q, k, v, wk, wv, out, workspace, workspace.numel(), stream)
        return out

    def forward_static(self, q, k, v, wk=None, wv=None, out=None, stream=None):
        """The forward pass with the library's static per-GPU workspace
        (fma_forward_static): no workspace argument, nothing allocated."""
        if out is None:
            out = torch.empty_like(q)
        fma_forward_static(self.handle, q, k, v, wk, wv, out, stream)
        return out

    def forward_linear(self, q, k, v, wq, wk, wv, out=None, workspace=None, stream=None):
        """FMA-linear (plan made with linear=True): wq aggregates the queries."""
        if out is None:
            out = torch.empty_like(q)
        if workspace is None:
            workspace = self.new_workspace(q.device)
        fma_forward_linear(self.handle, q, k, v, wq, wk, wv, out, workspace, workspace.numel(), stream)
        return out

    def coarsen(self, k, v, wk, wv, workspace=None, stream=None):
        if workspace is None:
            workspace = self.new_workspace(k.device)
        fma_coarsen(self.handle, k, v, wk, wv, workspace, workspace.numel(), stream)
        return workspace

    def attend(self, q, k, v, workspace, out=None, stream=None):
        if out is None:
            out = torch.empty_like(q)
        fma_attend(self.handle, q, k, v, workspace, workspace.numel(), out, stream)
        return out

    def backward(self, q, k, v, wk, wv, out, dout, workspace=None, stream=None):
        """Gradients (dq, dk, dv, dwk, dwv) of sum(dout * out) for out =
        forward(q, k, v, wk, wv); dwk, dwv shaped like wk, wv (None when the
        plan has no coarse level)."""
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        dwk = torch.empty_like(wk) if wk is not None and wk.numel() else None
        dwv = torch.empty_like(wv) if wv is not None and wv.numel() else None
        if workspace is None:
            workspace = torch.empty(max(self.backward_workspace_bytes, 16), dtype=torch.uint8, device=q.device)
        fma_backward(self.handle, q, k, v, wk if dwk is not None else None, wv if dwv is not None else None,
                     out, dout, dq, dk, dv, dwk, dwv, workspace, workspace.numel(), stream)
        return dq, dk, dv, dwk, dwv

    def backward_linear(self, q, k, v, wk, wv, wq, out, dout, workspace=None, stream=None):
        """FMA-linear plans: gradients (dq, dk, dv, dwk, dwv, dwq) of
        sum(dout * out) for out = forward_linear(q, k, v, wk, wv, wq)."""
        dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
        has_w = wk is not None and wk.numel() > 0
        dwk = torch.empty_like(wk) if has_w else None
        dwv = torch.empty_like(wv) if has_w else None
        dwq = torch.empty_like(wq) if has_w else None
        if workspace is None:
            workspace = torch.empty(max(self.backward_workspace_bytes, 16), dtype=torch.uint8, device=q.device)
        fma_backward_linear(self.handle, q, k, v, wk if has_w else None, wv if has_w else None,
                            wq if has_w else None, out, dout, dq, dk, dv, dwk, dwv, dwq, workspace,
                            workspace.numel(), stream)
        return dq, dk, dv, dwk, dwv, dwq

    def interaction_lists(self, device, stream=None) -> torch.Tensor:
        K = 3 if self.ndim == 1 else 27
        nb = self.n // self.block if self.ndim == 1 else (self.side // self.block) * (self.n // self.side // self.block)
        out = torch.empty((nb, max(self.levels - 1, 0), K), dtype=torch.int32, device=device)
        if out.numel():
            fma_interaction_lists(self.handle, out, stream)
        return out

    def dense_reference(self, q, k, v, out=None, stream=None):
        if out is None:
            out = torch.empty_like(q)
        fma_dense_reference(self.handle, q, k, v, out, stream)
        return out


# ---------------------------------------------------------------- strided calls
def _dtype_code(dtype):
    if dtype not in _DTYPES:
        _refuse(FMA_ERR_ARG, "dtype %s is neither float32 nor bfloat16", dtype)
    return _DTYPES[dtype]


def _refuse(status, message, *args):
    raise FmaError(status, message % args)


def _explain(t, name, shape, dtype, gpu):
    """Raises what is wrong with a tensor."""
    if t.shape != shape:
        _refuse(FMA_ERR_SHAPE, "%s has shape %s, expected %s", name, tuple(t.shape), tuple(shape))
    if t.dtype is not dtype or t.get_device() != gpu:
        _refuse(FMA_ERR_ARG, "%s is %s on %s, expected %s on GPU %d", name, t.dtype, t.device, dtype, gpu)


def _view(t, name, shape, axes, dtype, gpu):
    """The fields of the fma_view_t of a tensor whose axes (batch, heads,
    tokens) are `axes`."""
    if t.shape != shape or t.dtype is not dtype or t.get_device() != gpu:
        _explain(t, name, shape, dtype, gpu)
    s = t.stride()
    if s[3] != 1:
        _refuse(FMA_ERR_SHAPE, "the channels of %s are not adjacent", name)
    return t.data_ptr(), s[axes[0]], s[axes[1]], s[axes[2]]


_TOKEN_MAJOR, _HEAD_MAJOR = (0, 2, 1), (0, 1, 2)   # [batch, tokens, heads, d], [batch, heads, tokens, d]
_VIEW = ctypes.sizeof(fma_view_t)
_VIEWS = {n: ctypes.c_int64 * (4 * n) for n in range(1, 9)}   # n views that lie together


def _plain(t, name, shape, dtype, gpu):
    """A dense side input (None passes)."""
    if t is None:
        return
    if t.shape != shape or t.dtype is not dtype or t.get_device() != gpu:
        _explain(t, name, shape, dtype, gpu)
    if not t.is_contiguous():
        _refuse(FMA_ERR_SHAPE, "%s is not contiguous", name)


class _Launch:
    """Makes `device` current for a call, and `stream`, if the caller names
    one, the stream that the call's allocations belong to."""

    def __init__(self, device, stream):
        self.entered = []
        if device.index != torch.cuda.current_device():
            self.entered.append(torch.cuda.device(device))
        if stream is not None:
            if isinstance(stream, int):
                stream = torch.cuda.ExternalStream(stream, device=device)
            if stream.device != device:
                _refuse(FMA_ERR_ARG, "the stream belongs to %s, the tensors are on %s", stream.device, device)
            self.entered.append(torch.cuda.stream(stream))

    def __enter__(self):
        for c in self.entered:
            c.__enter__()

    def __exit__(self, *exc):
        for c in reversed(self.entered):
            c.__exit__(*exc)


_HERE = contextlib.nullcontext()


def _launch(t, stream):
    """Context of a call on t's device, which must be a GPU."""
    gpu = t.get_device()
    if gpu < 0:
        _refuse(FMA_ERR_ARG, "tensors are on %s, expected a GPU", t.device)
    if stream is None and gpu == torch.cuda.current_device():
        return _HERE
    return _Launch(t.device, stream)


class QKNormRope:
    """Per-head RMS norm and rotation of queries and keys, and the layout that
    ``FMA.forward`` reads, in one pass over a projection's output; its
    backward pass goes from ``FMA.backward``'s gradients to the projection's::

        op = QKNormRope(heads=16, kv_heads=4, repeat_kv=True, dtype=torch.bfloat16)
        q, k, v = op.forward(q, k, v, gamma_q, gamma_k)      # [B, n, heads, d] -> [B, heads, n, d]
        dq, dk, dv, dgamma_q, dgamma_k = op.backward(q_in, k_in, gamma_q, gamma_k, gq, gk, gv)

    axes = 2 rotates a map's tokens by row and column; inv_freq (a sequence of
    rates per position) replaces base ** (-i / half).  repeat_kv gives keys and
    values out once per query head.
    """

    def __init__(self, heads, kv_heads=None, head_dim=HEAD_DIM, dtype=torch.bfloat16, rotary_dim=None,
                 base=10000.0, eps=1e-6, axes=1, side=0, interleaved=False, repeat_kv=False, inv_freq=None):
        kv_heads = heads if kv_heads is None else kv_heads
        rotary_dim = head_dim if rotary_dim is None else rotary_dim
        if inv_freq is not None and len(inv_freq) != rotary_dim // (2 * max(axes, 1)):
            _refuse(FMA_ERR_SHAPE, "inv_freq has %d rates, expected %d", len(inv_freq), rotary_dim // (2 * max(axes, 1)))
        self.desc = fma_qk_desc_t(ctypes.sizeof(fma_qk_desc_t), _dtype_code(dtype), heads, kv_heads, head_dim, rotary_dim,
                                  axes, side, int(bool(interleaved)), int(bool(repeat_kv)), eps, base)
        self.handle = fma_qk_plan(self.desc, inv_freq)
        self.heads, self.kv_heads, self.head_dim, self.dtype, self.axes = heads, kv_heads, head_dim, dtype, axes
        self.kv_out = heads if repeat_kv else kv_heads

    def __del__(self):
        h = getattr(self, "handle", None)
        if h:
            try:
                library().fma_qk_destroy(h)
            except Exception:
                pass
            self.handle = None

    def _side(self, gpu, gamma_q, gamma_k, positions, B, n):
        f32, d = torch.float32, (self.head_dim,)
        _plain(gamma_q, "gamma_q", d, f32, gpu)
        _plain(gamma_k, "gamma_k", d, f32, gpu)
        if positions is not None and positions.dim() == 2 and self.axes == 1:
            positions = positions[..., None]
        _plain(positions, "positions", (B, n, self.axes), torch.int32, gpu)
        return positions

    def forward(self, q, k, v=None, gamma_q=None, gamma_k=None, positions=None, q_out=None, k_out=None, v_out=None,
                stream=None):
        """q [B, n, heads, d], k and v [B, n, kv_heads, d], any strides with
        adjacent channels -> q_out, k_out, v_out [B, heads, n, d] (new dense
        tensors, or the ones given, of any strides; token-major ones as
        ``t.transpose(1, 2)``).  positions: int32 [B, n] or [B, n, axes]."""
        if q.dim() != 4:
            _refuse(FMA_ERR_SHAPE, "q has %d axes, expected [B, n, heads, d]", q.dim())
        (B, n), gpu, d, dt = q.shape[:2], q.get_device(), self.head_dim, self.dtype
        ins, kvs, outs, kvo = (B, n, self.heads, d), (B, n, self.kv_heads, d), (B, self.heads, n, d), (B, self.kv_out, n, d)
        with _launch(q, stream):
            positions = self._side(gpu, gamma_q, gamma_k, positions, B, n)
            if q_out is None:
                q_out = q.new_empty(outs)
            if k_out is None:
                k_out = q.new_empty(kvo)
            views = [*_view(q, "q", ins, _TOKEN_MAJOR, dt, gpu), *_view(k, "k", kvs, _TOKEN_MAJOR, dt, gpu),
                     *_view(q_out, "q_out", outs, _HEAD_MAJOR, dt, gpu), *_view(k_out, "k_out", kvo, _HEAD_MAJOR, dt, gpu)]
            if v is not None:
                if v_out is None:
                    v_out = q.new_empty(kvo)
                views += _view(v, "v", kvs, _TOKEN_MAJOR, dt, gpu)
            if v_out is not None:
                views += _view(v_out, "v_out", kvo, _HEAD_MAJOR, dt, gpu)
            buf = _VIEWS[len(views) // 4](*views)
            at = ctypes.addressof(buf)
            vi, vo = (at + 4 * _VIEW if v is not None else None), (at + (len(views) // 4 - 1) * _VIEW if v_out is not None else None)
            fma_qk_norm_rope(self.handle, B, n, at, at + _VIEW, vi, gamma_q, gamma_k, positions, at + 2 * _VIEW,
                             at + 3 * _VIEW, vo)
        return q_out, k_out, v_out

    def backward(self, q, k, gamma_q, gamma_k, g_q, g_k, g_v=None, positions=None, dq=None, dk=None, dv=None,
                 workspace=None, stream=None):
        """(dq, dk, dv, dgamma_q, dgamma_k) from the forward's q, k and the
        gradients of its outputs; dq, dk, dv [B, n, heads, d] (new, or the
        tensors given, of any strides: the heads of one packed gradient).  A
        gamma of None has no gradient."""
        if q.dim() != 4:
            _refuse(FMA_ERR_SHAPE, "q has %d axes, expected [B, n, heads, d]", q.dim())
        (B, n), gpu, d, dt = q.shape[:2], q.get_device(), self.head_dim, self.dtype
        ins, kvs, outs, kvo = (B, n, self.heads, d), (B, n, self.kv_heads, d), (B, self.heads, n, d), (B, self.kv_out, n, d)
        with _launch(q, stream):
            positions = self._side(gpu, gamma_q, gamma_k, positions, B, n)
            dq = q.new_empty(ins) if dq is None else dq
            dk = q.new_empty(kvs) if dk is None else dk
            if g_v is not None and dv is None:
                dv = q.new_empty(kvs)
            dgq = None if gamma_q is None else torch.empty_like(gamma_q)
            dgk = None if gamma_k is None else torch.empty_like(gamma_k)
            need = fma_qk_backward_workspace_size(self.handle, B, n)
            if workspace is None:
                workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=q.device)
            views = [*_view(q, "q", ins, _TOKEN_MAJOR, dt, gpu), *_view(k, "k", kvs, _TOKEN_MAJOR, dt, gpu),
                     *_view(g_q, "g_q", outs, _HEAD_MAJOR, dt, gpu), *_view(g_k, "g_k", kvo, _HEAD_MAJOR, dt, gpu),
                     *_view(dq, "dq", ins, _TOKEN_MAJOR, dt, gpu), *_view(dk, "dk", kvs, _TOKEN_MAJOR, dt, gpu)]
            if g_v is not None:
                views += _view(g_v, "g_v", kvo, _HEAD_MAJOR, dt, gpu)
            if dv is not None:
                views += _view(dv, "dv", kvs, _TOKEN_MAJOR, dt, gpu)
            buf = _VIEWS[len(views) // 4](*views)
            at = ctypes.addressof(buf)
            gv, dvv = (at + 6 * _VIEW if g_v is not None else None), (at + (len(views) // 4 - 1) * _VIEW if dv is not None else None)
            fma_qk_norm_rope_backward(self.handle, B, n, at, at + _VIEW, gamma_q, gamma_k, positions, at + 2 * _VIEW,
                                      at + 3 * _VIEW, gv, at + 4 * _VIEW, at + 5 * _VIEW, dvv, dgq, dgk, workspace,
                                      workspace.numel() * workspace.element_size())
        return dq, dk, dv, dgq, dgk


class CachePages(NamedTuple):
    """Storage of a paged cache: k, v [pages, kv_heads, block, d]; summaries
    fp32 [pages, kv_heads, 2, sets, d] (None without coarse sets)."""
    k: torch.Tensor
    v: torch.Tensor
    summaries: torch.Tensor | None = None


class CacheBatch(NamedTuple):
    """One call's sequences, int32 on the GPU: sequence i has start[i] tokens
    and rows cu_tokens[i] .. cu_tokens[i + 1] - 1 of the call's tensors are its
    next ones, at most max_chunk; page_table, summary_table [sequences,
    blocks]: the pages of its blocks."""
    cu_tokens: torch.Tensor
    start: torch.Tensor
    page_table: torch.Tensor
    summary_table: torch.Tensor | None
    max_chunk: int


class FMACache:
    """Paged cache of a causal FMA layer: prompts in pieces, single tokens, or
    both in one ragged batch, with what ``FMA.forward`` gives for the whole
    sequences (causal, joint normalisation)::

        op = FMACache(heads=16, kv_heads=4, block=128, max_seq_len=65536, dtype=torch.bfloat16)
        pages = op.new_pages(num_pages, num_summaries, "cuda")
        op.append(k, v, wk, wv, pages, batch)             # k, v: [tokens, kv_heads, d]
        out = op.step(q, k, v, wk, wv, pages, batch)      # appends and attends, q, out: [tokens, heads, d]
    """

    def __init__(self, heads, max_seq_len, kv_heads=None, head_dim=HEAD_DIM, block=64, dtype=torch.bfloat16, rank=1,
                 weights_per_head=True, softmax_scale=0.0, norm=FMA_NORM_JOINT):
        kv_heads = heads if kv_heads is None else kv_heads
        self.desc = fma_cache_desc_t(ctypes.sizeof(fma_cache_desc_t), _dtype_code(dtype), heads, kv_heads, head_dim, block,
                                     max_seq_len, rank, int(bool(weights_per_head)), norm, softmax_scale)
        self.handle = fma_cache_plan(self.desc)
        self.heads, self.kv_heads, self.head_dim, self.block, self.dtype = heads, kv_heads, head_dim, block, dtype
        self.weights_per_head = bool(weights_per_head)
        self.sets, self.weights_len, self.blocks = fma_cache_sizes(self.handle)

    def __del__(self):
        h = getattr(self, "handle", None)
        if h:
            try:
                library().fma_cache_destroy(h)
            except Exception:
                pass
            self.handle = None

    def new_pages(self, num_pages, num_summaries, device) -> CachePages:
        page = (num_pages, self.kv_heads, self.block, self.head_dim)
        sums = (num_summaries, self.kv_heads, 2, self.sets, self.head_dim)
        return CachePages(torch.empty(page, dtype=self.dtype, device=device),
                          torch.empty(page, dtype=self.dtype, device=device),
                          torch.empty(sums, dtype=torch.float32, device=device) if self.sets else None)

    # ---------------------------------------------------------- helpers
    def _batch(self, pages, batch, rows, gpu):
        kp, vp, sums = pages
        cu, start, table, stable, chunk = batch
        i32 = torch.int32
        if kp.dim() != 4 or table.dim() != 2 or start.dim() != 1:
            _refuse(FMA_ERR_SHAPE, "expected pages [n, kv_heads, block, d], tables [sequences, blocks], start [sequences]")
        S, width, npage, nsum = start.shape[0], table.shape[1], kp.shape[0], 0
        page = (npage, self.kv_heads, self.block, self.head_dim)
        _plain(kp, "k_pages", page, self.dtype, gpu)
        _plain(vp, "v_pages", page, self.dtype, gpu)
        _plain(cu, "cu_tokens", (S + 1,), i32, gpu)
        _plain(start, "start", (S,), i32, gpu)
        _plain(table, "page_table", (S, width), i32, gpu)
        at_sum = at_stable = None
        if self.sets:
            if sums is None or stable is None:
                _refuse(FMA_ERR_NULL, "the plan's coarse sets need summaries and a summary_table")
            nsum = sums.shape[0]
            _plain(sums, "summaries", (nsum, self.kv_heads, 2, self.sets, self.head_dim), torch.float32, gpu)
            _plain(stable, "summary_table", (S, width), i32, gpu)
            at_sum, at_stable = sums.data_ptr(), stable.data_ptr()
        return fma_cache_batch_t(kp.data_ptr(), vp.data_ptr(), at_sum, npage, nsum, table.data_ptr(), at_stable, width,
                                 cu.data_ptr(), start.data_ptr(), S, chunk, rows)

    def _rows(self, t, name, heads, rows, gpu):
        """The fields of the fma_view_t of [tokens, heads, d]."""
        shape = (rows, heads, self.head_dim)
        if t.shape != shape or t.dtype is not self.dtype or t.get_device() != gpu:
            _explain(t, name, shape, self.dtype, gpu)
        s = t.stride()
        if s[2] != 1:
            _refuse(FMA_ERR_SHAPE, "the channels of %s are not adjacent", name)
        return t.data_ptr(), 0, s[1], s[0]

    def _weights(self, wk, wv, gpu):
        if not self.sets:
            return None, None
        if wk is None or wv is None:
            _refuse(FMA_ERR_NULL, "the plan's coarse sets need wk and wv")
        shape = (self.kv_heads, self.weights_len) if self.weights_per_head else (self.weights_len,)
        _plain(wk, "wk", shape, torch.float32, gpu)
        _plain(wv, "wv", shape, torch.float32, gpu)
        return wk, wv

    # ---------------------------------------------------------- calls
    def append(self, k, v, wk, wv, pages, batch, stream=None):
        """New keys and values [tokens, kv_heads, d] (any strides, adjacent
        channels) into the pages, and the summaries that they complete."""
        rows, gpu, kv = k.shape[0], k.get_device(), self.kv_heads
        with _launch(k, stream):
            wk, wv = self._weights(wk, wv, gpu)
            buf = _VIEWS[2](*self._rows(k, "k", kv, rows, gpu), *self._rows(v, "v", kv, rows, gpu))
            at = ctypes.addressof(buf)
            fma_cache_append(self.handle, self._batch(pages, batch, rows, gpu), at, at + _VIEW, wk, wv)

    def attend(self, q, pages, batch, out=None, stream=None):
        """Attention of q [tokens, heads, d], whose keys and values are in the
        cache, -> out (a new one is zero in rows of no sequence)."""
        rows, gpu, h = q.shape[0], q.get_device(), self.heads
        with _launch(q, stream):
            if out is None:
                out = torch.zeros((rows, h, self.head_dim), dtype=self.dtype, device=q.device)
            buf = _VIEWS[2](*self._rows(q, "q", h, rows, gpu), *self._rows(out, "out", h, rows, gpu))
            at = ctypes.addressof(buf)
            fma_cache_attend(self.handle, self._batch(pages, batch, rows, gpu), at, at + _VIEW)
        return out

    def step(self, q, k, v, wk, wv, pages, batch, out=None, stream=None):
        """append, then attend."""
        rows, gpu, h, kv = q.shape[0], q.get_device(), self.heads, self.kv_heads
        with _launch(q, stream):
            wk, wv = self._weights(wk, wv, gpu)
            if out is None:
                out = torch.zeros((rows, h, self.head_dim), dtype=self.dtype, device=q.device)
            buf = _VIEWS[4](*self._rows(q, "q", h, rows, gpu), *self._rows(k, "k", kv, rows, gpu),
                            *self._rows(v, "v", kv, rows, gpu), *self._rows(out, "out", h, rows, gpu))
            at = ctypes.addressof(buf)
            fma_cache_step(self.handle, self._batch(pages, batch, rows, gpu), at, at + _VIEW, at + 2 * _VIEW, wk, wv,
                           at + 3 * _VIEW)
        return out
