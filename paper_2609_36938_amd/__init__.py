"""Python binding of libjanus (gfx950): the sparse-selection hot path of append
prefill for top-k sparse-attention LLMs.

Every function here only marshals arguments to the C ABI declared in
``include/janus.h``; all arithmetic runs in the library's HIP kernels.  Torch
provides device memory and the current stream.  There is no fallback: if the
library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Sequence

import numpy as np
import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libjanus.so")

JANUS_F32, JANUS_BF16, JANUS_FP8_E4M3 = 0, 1, 2
_DT_NAMES = {"f32": JANUS_F32, "bf16": JANUS_BF16, "fp8": JANUS_FP8_E4M3}


class JanusError(RuntimeError):
    pass


class _Batch(ctypes.Structure):
    _fields_ = [
        ("num_seqs", ctypes.c_int32),
        ("total_q", ctypes.c_int32),
        ("max_q", ctypes.c_int32),
        ("max_ctx", ctypes.c_int32),
        ("total_ctx", ctypes.c_int64),
        ("q_start", ctypes.c_void_p),
        ("ctx_start", ctypes.c_void_p),
        ("hist_len", ctypes.c_void_p),
        ("score_start", ctypes.c_void_p),
        ("entry_shift", ctypes.c_int32),
    ]


class _Rotary(ctypes.Structure):
    _fields_ = [
        ("dim", ctypes.c_int32),
        ("offset", ctypes.c_int32),
        ("layout", ctypes.c_int32),
        ("inverse", ctypes.c_int32),
        ("magnitude", ctypes.c_float),
        ("inv_freq", ctypes.c_void_p),
        ("positions", ctypes.c_void_p),
    ]


_lib = None


def lib():
    """The loaded libjanus; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise JanusError(f"{LIB_PATH} is missing: build it with python -m paper_2609_36938_amd.build")
        L = ctypes.CDLL(LIB_PATH)
        P, i32, i64, f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float
        BP = ctypes.POINTER(_Batch)
        SZ = ctypes.POINTER(ctypes.c_size_t)
        L.janus_index_scores.argtypes = [BP, P, i32, P, P, i32, P, P, i32, i32, P, P]
        L.janus_topk.argtypes = [BP, P, i32, P, P, SZ, P]
        L.janus_topk_sharded.argtypes = [BP, P, i32, i32, i32, P, P, SZ, P]
        L.janus_page_demand.argtypes = [BP, P, i32, P, i32, i32, P, i32, i32, P, P, P, P, P, SZ, P]
        L.janus_predict_diff.argtypes = [P, P, i32, i32, P, P, P, P]
        L.janus_sparse_attn.argtypes = [BP, P, i32, i32, i32, P, P, i64, i64, P, i32, i32, P, i32, f32, P, i32,
                                        P, P]
        L.janus_index_scores_mxfp4.argtypes = [BP, P, P, P, P, P, P, i32, i32, P, P]
        L.janus_sparse_attn_split.argtypes = [BP, P, i32, i32, i32, P, P, i64, i64, P, i32, i32, P, i32, f32, P,
                                              i32, P, i32, P, SZ, P]
        L.janus_sparse_attn_fp8kv.argtypes = [BP, P, i32, P, i64, P, i32, i32, P, i32, f32, P, i32, P, i32, P, SZ, P]
        L.janus_sparse_attn_split_noalloc.argtypes = [BP, P, i32, i32, i32, P, P, i64, i64, P, i32, i32, P, i32, f32,
                                                      P, i32, P, i32, P]
        RP, f64 = ctypes.POINTER(_Rotary), ctypes.c_double
        L.janus_page_grow.argtypes = [BP, i32, P, i32, P, P, i32, P, P, P]
        L.janus_rotary_frequencies.argtypes = [i32, f64, f64, i32, i32, f64, f64, P, ctypes.POINTER(f32)]
        L.janus_rope.argtypes = [BP, RP, P, i32, i64, i64, i32, i32, P, i32, i64, i64, P, P]
        L.janus_kv_append.argtypes = [BP, RP, P, i32, i64, P, i64, i32, P, i64, P, i32, i64, P, P]
        L.janus_prefix_attn.argtypes = [BP, P, i32, i32, i32, P, P, i64, i64, P, i32, i32, i32, f32, P, i32, P, P, SZ, P]
        for f in ("janus_page_grow", "janus_rotary_frequencies", "janus_rope", "janus_kv_append", "janus_prefix_attn",
                  "janus_index_scores", "janus_topk", "janus_topk_sharded", "janus_page_demand",
                  "janus_predict_diff", "janus_sparse_attn", "janus_sparse_attn_split", "janus_index_scores_mxfp4",
                  "janus_sparse_attn_fp8kv", "janus_sparse_attn_split_noalloc"):
            getattr(L, f).restype = ctypes.c_int
        L.janus_status_string.argtypes = [ctypes.c_int]
        L.janus_status_string.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _check(rc: int, what: str):
    if rc != 0:
        msg = lib().janus_status_string(rc).decode()
        raise JanusError(f"{what}: {msg} (status {rc})")


def _ptr(t: Optional[torch.Tensor]):
    if t is None:
        return None
    if not t.is_cuda:
        raise JanusError("device tensor expected")
    return ctypes.c_void_p(t.data_ptr())


def _workspace(t: torch.Tensor, out: torch.Tensor):
    """Address and bytes of a caller's workspace.  An empty tensor has no address, and NULL would be the size
    query, which does nothing: it goes in as 0 bytes at out, which the library does not touch as a workspace."""
    if not t.is_cuda:
        raise JanusError("device tensor expected")
    if not t.is_contiguous():
        raise JanusError("the workspace is to be contiguous: its bytes are counted by its elements")
    return t.data_ptr() or out.data_ptr(), ctypes.c_size_t(t.numel() * t.element_size())


def _stream(stream=None):
    s = torch.cuda.current_stream() if stream is None else stream
    return ctypes.c_void_p(s.cuda_stream)


def _dtype_code(t: torch.Tensor, dt: Optional[str]) -> int:
    if dt is not None:
        return _DT_NAMES[dt]
    if t.dtype in (torch.float8_e4m3fn, torch.uint8):
        return JANUS_FP8_E4M3
    if t.dtype in (torch.bfloat16, torch.int16):
        return JANUS_BF16
    if t.dtype == torch.float32:
        return JANUS_F32
    raise JanusError(f"unsupported dtype {t.dtype}")


def _table(batch: "Batch", page_table, page_size: int) -> int:
    """pt_ld of a [B, pt_ld] page table, which must cover the longest session."""
    pt_ld = int(page_table.shape[1])
    if pt_ld * int(page_size) < batch.max_ctx:
        raise JanusError(f"page table covers {pt_ld} x {page_size} ids, the longest session has {batch.max_ctx}")
    return pt_ld


class Batch:
    """A ragged batch of sessions: history lengths M_b and appended lengths N_b
    (tokens).  entry_shift = e > 0 selects entry granularity: candidates are
    entries of 2^e tokens, and session b holds (M_b + N_b) >> e of them."""

    def __init__(self, hist_len: Sequence[int], new_len: Sequence[int], device="cuda", entry_shift: int = 0):
        hl = np.asarray(hist_len, dtype=np.int64).reshape(-1)
        nl = np.asarray(new_len, dtype=np.int64).reshape(-1)
        if hl.shape != nl.shape or hl.size < 1:
            raise JanusError("hist_len and new_len must be equal-length, non-empty")
        self.entry_shift = int(entry_shift)
        ctx = (hl + nl) >> self.entry_shift
        self.hist_len_host = hl.astype(np.int32)
        self.new_len_host = nl.astype(np.int32)
        self.q_start_host = np.concatenate([[0], np.cumsum(nl)]).astype(np.int32)
        self.ctx_start_host = np.concatenate([[0], np.cumsum(ctx)]).astype(np.int32)
        self.score_start_host = np.concatenate([[0], np.cumsum(nl * ctx)]).astype(np.int64)
        self.q_start = torch.from_numpy(self.q_start_host).to(device)
        self.ctx_start = torch.from_numpy(self.ctx_start_host).to(device)
        self.hist_len = torch.from_numpy(self.hist_len_host).to(device)
        self.score_start = torch.from_numpy(self.score_start_host).to(device)
        self.total_q = int(nl.sum())
        self.total_ctx = int(ctx.sum())
        self.max_ctx = int(ctx.max())
        self.total_scores = int(self.score_start_host[-1])
        self.c = _Batch(len(hl), self.total_q, int(nl.max()), self.max_ctx, self.total_ctx,
                        self.q_start.data_ptr(), self.ctx_start.data_ptr(), self.hist_len.data_ptr(),
                        self.score_start.data_ptr(), self.entry_shift)

    @property
    def ref(self):
        return ctypes.byref(self.c)


def index_scores(batch: Batch, q, kI, w, q_scale=None, k_scale=None, scores=None, dtype=None, stream=None):
    """janus_index_scores: returns the flat fp32 score buffer (batch.total_scores)."""
    H, d = int(q.shape[-2]), int(q.shape[-1])
    if scores is None:
        scores = torch.empty(batch.total_scores, dtype=torch.float32, device=q.device)
    qd, kd = _dtype_code(q, dtype), _dtype_code(kI, dtype)
    rc = lib().janus_index_scores(batch.ref, _ptr(q), qd, _ptr(q_scale), _ptr(kI), kd, _ptr(k_scale), _ptr(w), H, d,
                                  _ptr(scores), _stream(stream))
    _check(rc, "janus_index_scores")
    return scores


def index_scores_mxfp4(batch: Batch, q, kI, k_block_scale, w, q_scale=None, k_scale=None, scores=None, stream=None):
    """janus_index_scores_mxfp4: q fp8 bytes [total_q, H, d]; kI MXFP4 bytes
    [total_ctx, d/2] with E8M0 block scales [total_ctx, d/32]; returns the flat
    fp32 score buffer laid out as for index_scores."""
    H, d = int(q.shape[1]), int(q.shape[2])
    if scores is None:
        scores = torch.empty(batch.total_scores, dtype=torch.float32, device=q.device)
    rc = lib().janus_index_scores_mxfp4(batch.ref, _ptr(q), _ptr(q_scale), _ptr(kI), _ptr(k_block_scale),
                                        _ptr(k_scale), _ptr(w), H, d, _ptr(scores), _stream(stream))
    _check(rc, "janus_index_scores_mxfp4")
    return scores


def topk(batch: Batch, scores, k: int, out=None, stream=None):
    """janus_topk: [total_q, k] int32 ids, ascending, -1 padded."""
    if out is None:
        out = torch.empty((batch.total_q, k), dtype=torch.int32, device=scores.device)
    ws = ctypes.c_size_t(0)
    rc = lib().janus_topk(batch.ref, _ptr(scores), int(k), _ptr(out), None, ctypes.byref(ws), _stream(stream))
    _check(rc, "janus_topk")
    return out


def topk_sharded(batch: Batch, scores, k: int, num_shards: int, align: int, out=None, stream=None):
    """janus_topk_sharded: [total_q, k] int32; slots n*(k/num_shards) .. hold
    shard n's history ids, ascending, -1 padded."""
    if out is None:
        out = torch.empty((batch.total_q, k), dtype=torch.int32, device=scores.device)
    ws = ctypes.c_size_t(0)
    rc = lib().janus_topk_sharded(batch.ref, _ptr(scores), int(k), int(num_shards), int(align), _ptr(out), None,
                                  ctypes.byref(ws), _stream(stream))
    _check(rc, "janus_topk_sharded")
    return out


def page_demand(batch: Batch, topk_idx, page_table, page_size: int, num_phys_pages: int, max_run: int,
                limit=None, out=None, stream=None):
    """janus_page_demand: (bitmap, page_list, runs, counts) device tensors.

    page_list and runs are sized to the pool; counts = [num_pages, num_runs]."""
    dev = topk_idx.device
    nw = max(1, (num_phys_pages + 31) // 32)
    if out is None:
        out = (torch.empty(nw, dtype=torch.int32, device=dev),
               torch.empty(max(1, num_phys_pages), dtype=torch.int32, device=dev),
               torch.empty(max(1, 2 * num_phys_pages), dtype=torch.int32, device=dev),
               torch.empty(2, dtype=torch.int32, device=dev))
    bm, lst, runs, counts = out
    ws = ctypes.c_size_t(0)
    rc = lib().janus_page_demand(batch.ref, _ptr(topk_idx), int(topk_idx.shape[1]), _ptr(page_table),
                                 _table(batch, page_table, page_size), int(page_size), _ptr(limit), int(num_phys_pages),
                                 int(max_run), _ptr(bm), _ptr(lst), _ptr(runs), _ptr(counts), None,
                                 ctypes.byref(ws), _stream(stream))
    _check(rc, "janus_page_demand")
    return out


def predict_diff(actual, predicted, num_phys_pages: int, max_run: int, out=None, stream=None):
    """janus_predict_diff: (miss bitmap, miss runs, counts[5])."""
    dev = actual.device
    nw = max(1, (num_phys_pages + 31) // 32)
    if out is None:
        out = (torch.empty(nw, dtype=torch.int32, device=dev),
               torch.empty(max(1, 2 * num_phys_pages), dtype=torch.int32, device=dev),
               torch.empty(5, dtype=torch.int32, device=dev))
    miss, runs, counts = out
    rc = lib().janus_predict_diff(_ptr(actual), _ptr(predicted), int(num_phys_pages), int(max_run), _ptr(miss),
                                  _ptr(runs), _ptr(counts), _stream(stream))
    _check(rc, "janus_predict_diff")
    return out


def sparse_attn(batch: Batch, q, k_pool, v_pool, page_table, page_size: int, topk_idx, scale: float,
                k_row_stride: Optional[int] = None, v_row_stride: Optional[int] = None, dv: Optional[int] = None,
                out_dtype: str = "bf16", want_lse: bool = False, out=None, lse=None, stream=None):
    """janus_sparse_attn: returns (out [total_q, Hq, dv], lse or None).

    q is [total_q, Hq, dqk] bf16; pools are bf16 rows (k_row_stride / v_row_stride
    elements each; default: the pool's last dimension).  Pass v_pool = k_pool for
    the latent-KV layout, where V is the first dv elements of each row."""
    Hq, dqk = int(q.shape[-2]), int(q.shape[-1])
    krs = int(k_row_stride if k_row_stride is not None else k_pool.shape[-1])
    vrs = int(v_row_stride if v_row_stride is not None else v_pool.shape[-1])
    dv = int(dv if dv is not None else (v_pool.shape[-1] if v_pool is not k_pool else dqk))
    odt = {"bf16": (JANUS_BF16, torch.bfloat16), "f32": (JANUS_F32, torch.float32)}[out_dtype]
    if out is None:
        out = torch.empty((batch.total_q, Hq, dv), dtype=odt[1], device=q.device)
    if want_lse and lse is None:
        lse = torch.empty((batch.total_q, Hq), dtype=torch.float32, device=q.device)
    rc = lib().janus_sparse_attn(batch.ref, _ptr(q), Hq, dqk, dv, _ptr(k_pool), _ptr(v_pool), krs, vrs,
                                 _ptr(page_table), _table(batch, page_table, page_size), int(page_size), _ptr(topk_idx),
                                 int(topk_idx.shape[1]), float(scale), _ptr(out), odt[0], _ptr(lse),
                                 _stream(stream))
    _check(rc, "janus_sparse_attn")
    return out, lse


def sparse_attn_split(batch: Batch, q, k_pool, v_pool, page_table, page_size: int, topk_idx, scale: float,
                      num_splits: int = 0, k_row_stride: Optional[int] = None, v_row_stride: Optional[int] = None,
                      dv: Optional[int] = None, out_dtype: str = "bf16", want_lse: bool = False, out=None,
                      lse=None, workspace=None, stream=None):
    """janus_sparse_attn_split: as sparse_attn, each row's selection split
    over num_splits blocks (0: the library picks); returns (out, lse or None).
    workspace: a device uint8 tensor of at least the byte count the library
    reports for these arguments (its NULL-workspace size query, made here
    first), or None to allocate one here."""
    Hq, dqk = int(q.shape[-2]), int(q.shape[-1])
    krs = int(k_row_stride if k_row_stride is not None else k_pool.shape[-1])
    vrs = int(v_row_stride if v_row_stride is not None else v_pool.shape[-1])
    dv = int(dv if dv is not None else (v_pool.shape[-1] if v_pool is not k_pool else dqk))
    odt = {"bf16": (JANUS_BF16, torch.bfloat16), "f32": (JANUS_F32, torch.float32)}[out_dtype]
    if out is None:
        out = torch.empty((batch.total_q, Hq, dv), dtype=odt[1], device=q.device)
    if want_lse and lse is None:
        lse = torch.empty((batch.total_q, Hq), dtype=torch.float32, device=q.device)
    args = (batch.ref, _ptr(q), Hq, dqk, dv, _ptr(k_pool), _ptr(v_pool), krs, vrs, _ptr(page_table),
            _table(batch, page_table, page_size), int(page_size), _ptr(topk_idx), int(topk_idx.shape[1]),
            float(scale), _ptr(out), odt[0], _ptr(lse), int(num_splits))
    need = ctypes.c_size_t(0)
    _check(lib().janus_sparse_attn_split(*args, None, ctypes.byref(need), _stream(stream)), "janus_sparse_attn_split")
    if workspace is None:
        workspace = torch.empty(max(int(need.value), 1), dtype=torch.uint8, device=q.device)
    at, have = _workspace(workspace, out)
    rc = lib().janus_sparse_attn_split(*args, at, ctypes.byref(have), _stream(stream))
    _check(rc, "janus_sparse_attn_split")
    return out, lse


def sparse_attn_split_noalloc(batch: Batch, q, k_pool, v_pool, page_table, page_size: int, topk_idx, scale: float,
                              num_splits: int = 0, k_row_stride: Optional[int] = None,
                              v_row_stride: Optional[int] = None, dv: Optional[int] = None, out_dtype: str = "bf16",
                              want_lse: bool = False, out=None, lse=None, stream=None):
    """janus_sparse_attn_split_noalloc: as sparse_attn_split, with the slices'
    partial results in the library's own per-GPU scratch array instead of a
    workspace (pass out, and lse if wanted, to allocate nothing here either);
    returns (out, lse or None)."""
    Hq, dqk = int(q.shape[-2]), int(q.shape[-1])
    krs = int(k_row_stride if k_row_stride is not None else k_pool.shape[-1])
    vrs = int(v_row_stride if v_row_stride is not None else v_pool.shape[-1])
    dv = int(dv if dv is not None else (v_pool.shape[-1] if v_pool is not k_pool else dqk))
    odt = {"bf16": (JANUS_BF16, torch.bfloat16), "f32": (JANUS_F32, torch.float32)}[out_dtype]
    if out is None:
        out = torch.empty((batch.total_q, Hq, dv), dtype=odt[1], device=q.device)
    if want_lse and lse is None:
        lse = torch.empty((batch.total_q, Hq), dtype=torch.float32, device=q.device)
    rc = lib().janus_sparse_attn_split_noalloc(batch.ref, _ptr(q), Hq, dqk, dv, _ptr(k_pool), _ptr(v_pool), krs, vrs,
                                               _ptr(page_table), _table(batch, page_table, page_size),
                                               int(page_size), _ptr(topk_idx), int(topk_idx.shape[1]), float(scale),
                                               _ptr(out), odt[0], _ptr(lse), int(num_splits), _stream(stream))
    _check(rc, "janus_sparse_attn_split_noalloc")
    return out, lse


def sparse_attn_fp8kv(batch: Batch, q, kv_pool, page_table, page_size: int, topk_idx, scale: float,
                      num_splits: int = 1, out_dtype: str = "bf16", want_lse: bool = False, out=None, lse=None,
                      workspace=None, stream=None):
    """janus_sparse_attn_fp8kv: MLA attention (576/512) over fp8 KV rows
    (uint8 [..., row_bytes]: 576 e4m3 bytes, the fp32 scale at byte 576);
    num_splits as for sparse_attn_split (1: unsplit).  Returns (out, lse or None)."""
    Hq = int(q.shape[-2])
    row_bytes = int(kv_pool.shape[-1])
    odt = {"bf16": (JANUS_BF16, torch.bfloat16), "f32": (JANUS_F32, torch.float32)}[out_dtype]
    if out is None:
        out = torch.empty((batch.total_q, Hq, 512), dtype=odt[1], device=q.device)
    if want_lse and lse is None:
        lse = torch.empty((batch.total_q, Hq), dtype=torch.float32, device=q.device)
    args = (batch.ref, _ptr(q), Hq, _ptr(kv_pool), row_bytes, _ptr(page_table),
            _table(batch, page_table, page_size), int(page_size), _ptr(topk_idx), int(topk_idx.shape[1]),
            float(scale), _ptr(out), odt[0], _ptr(lse), int(num_splits))
    need = ctypes.c_size_t(0)
    _check(lib().janus_sparse_attn_fp8kv(*args, None, ctypes.byref(need), _stream(stream)), "janus_sparse_attn_fp8kv")
    if workspace is None:
        workspace = torch.empty(max(int(need.value), 1), dtype=torch.uint8, device=q.device)
    at, have = _workspace(workspace, out)
    rc = lib().janus_sparse_attn_fp8kv(*args, at, ctypes.byref(have), _stream(stream))
    _check(rc, "janus_sparse_attn_fp8kv")
    return out, lse


_LAYOUTS = {"half": 0, "interleaved": 1}
_SCALINGS = {None: 0, "linear": 1, "yarn": 2}


def _device(what: str, *tensors) -> int:
    """Index of the one GPU that all the tensors (None: absent) are on."""
    dev = tensors[0].get_device()  # -1 on the host
    for t in tensors:
        if t is not None and t.get_device() != dev:
            dev = -1
    if dev < 0:
        raise JanusError(f"{what}: tensors of one GPU expected")
    return dev


def _want(what: str, name: str, t, dtype, *shape):
    """t has this dtype, these sizes (None: any) and adjacent elements."""
    have = t.shape
    if t.dtype is not dtype or not t.is_contiguous() or (have != shape and (
            len(have) != len(shape) or any(n is not None and n != m for n, m in zip(shape, have)))):
        raise JanusError(f"{what}: {name} is to be a contiguous {dtype} tensor of shape "
                         f"{tuple('any' if n is None else n for n in shape)}, not {t.dtype} {tuple(have)}")


def _at(t: Optional[torch.Tensor]):
    """Address of a tensor that _device has seen."""
    return None if t is None else t.data_ptr()


def _followed(what: str):
    """A tensor of the call requires a gradient.  The calls record nothing for autograd: they refuse a tensor that it
    follows rather than cut it off."""
    if torch.is_grad_enabled():
        raise JanusError(f"{what}: a gradient would be lost here; call under torch.no_grad(), or in the forward "
                         "and backward functions of a torch.autograd.Function")


# A tensor of the caller's has been written: a graph that keeps it for its backward pass will notice.
_written = torch.autograd.graph.increment_version


def _empty(dtype, device, stream, *shape):
    """A new tensor that belongs to the stream of the launch: its memory is not given to other
    streams' work before, or after it is dropped, while that launch may use it.  (torch takes sizes
    one by one faster than as a tuple.)"""
    if stream is None:
        return torch.empty(*shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        return torch.empty(*shape, dtype=dtype, device=device)


def _launch(what: str, dev: int, stream, fn, *args):
    """fn(*args, stream) on GPU dev, whatever device is current.  (The raw stream: the object around it
    takes as long as the launch.)"""
    if stream is None:
        s = torch._C._cuda_getCurrentRawStream(dev)
    else:
        s = stream.cuda_stream
        if stream.device_index != dev:
            raise JanusError(f"{what}: tensors of GPU {dev}, a stream of GPU {stream.device_index}")
    if torch._C._cuda_getDevice() == dev:
        rc = fn(*args, s)
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, s)
    if rc != 0:
        _check(rc, what)


def rotary_frequencies(dim: int, base: float = 10000.0, scaling: Optional[str] = None, factor: float = 1.0,
                       original_ctx: int = 0, beta_fast: float = 32.0, beta_slow: float = 1.0):
    """janus_rotary_frequencies: (float64 array [dim/2], magnitude); scaling is
    None, "linear" or "yarn"."""
    if scaling not in _SCALINGS:
        raise JanusError(f"unknown scaling {scaling!r}")
    freq = np.zeros(max(int(dim) // 2, 1), dtype=np.float64)
    mag = ctypes.c_float(1.0)
    _check(lib().janus_rotary_frequencies(int(dim), float(base), float(factor), _SCALINGS[scaling], int(original_ctx),
                                          float(beta_fast), float(beta_slow), freq.ctypes.data, ctypes.byref(mag)),
           "janus_rotary_frequencies")
    return freq, float(mag.value)


class Rotary:
    """Rotary positions: dim elements of every head, from offset on, in pairs
    (j, j + dim/2) (layout "half") or (2j, 2j + 1) ("interleaved").

    Frequencies come from inv_freq (float64 [dim/2] on the GPU, with mscale as the
    factor of the rotated elements) or from rotary_frequencies(dim, base,
    scaling, factor, ...).  positions: int32 [total_q] on the GPU, or None for each
    appended token's own.  inverse: the transpose (the gradient)."""

    def __init__(self, dim: int, offset: int = 0, layout: str = "half", base: float = 10000.0,
                 scaling: Optional[str] = None, factor: float = 1.0, original_ctx: int = 0, beta_fast: float = 32.0,
                 beta_slow: float = 1.0, inv_freq=None, mscale: Optional[float] = None, inverse: bool = False,
                 positions=None, device="cuda"):
        if layout not in _LAYOUTS:
            raise JanusError(f"unknown layout {layout!r}")
        mag = 1.0
        if inv_freq is None:
            freq, mag = rotary_frequencies(dim, base, scaling, factor, original_ctx, beta_fast, beta_slow)
            inv_freq = torch.from_numpy(freq).to(device)
        _want("Rotary", "inv_freq", inv_freq, torch.float64, int(dim) // 2)
        if positions is not None:
            _want("Rotary", "positions", positions, torch.int32, None)
        _device("Rotary", inv_freq, positions)
        self.inv_freq, self.positions = inv_freq, positions
        self.mscale = float(mag if mscale is None else mscale)
        self.dim, self.offset, self.layout = int(dim), int(offset), layout
        self.c = _Rotary(self.dim, self.offset, _LAYOUTS[layout], int(bool(inverse)), self.mscale, inv_freq.data_ptr(),
                         None if positions is None else positions.data_ptr())

    def inverted(self) -> "Rotary":
        """The transpose of this rotation."""
        return Rotary(self.dim, self.offset, self.layout, inv_freq=self.inv_freq, mscale=self.mscale,
                      inverse=not self.c.inverse, positions=self.positions)

    def _check(self, what: str, batch: "Batch"):
        if self.positions is not None and self.positions.numel() < batch.total_q:
            raise JanusError(f"{what}: {self.positions.numel()} positions for {batch.total_q} tokens")

    @property
    def ref(self):
        return ctypes.byref(self.c)


def page_grow(batch: Batch, page_size: int, free_list, page_table, free_head=None, out=None, stream=None):
    """janus_page_grow: extends page_table [B, pt_ld] (int32, in place) by the
    pages the appended tokens need, off free_list (int32) from free_head (int32 [1],
    None: 0) on.  Returns (page_table, slots [total_q] int64, counts [3] int32 =
    pages taken, the next free_head, pages short); out = (slots, counts) to
    write those tensors."""
    what = "janus_page_grow"
    i32, total, shape = torch.int32, batch.total_q, page_table.shape
    if page_table.dtype is not i32 or len(shape) != 2 or shape[0] != batch.c.num_seqs or not page_table.is_contiguous():
        _want(what, "page_table", page_table, i32, batch.c.num_seqs, None)
    if free_list.dtype is not i32 or free_list.dim() != 1 or not free_list.is_contiguous():
        _want(what, "free_list", free_list, i32, None)
    if free_head is not None and (free_head.dtype is not i32 or free_head.numel() != 1):
        raise JanusError(f"{what}: free_head is to be one int32")
    if out is None:
        slots = _empty(torch.int64, page_table.device, stream, total)
        counts = _empty(i32, page_table.device, stream, 3)
    else:
        slots, counts = out
        _want(what, "slots", slots, torch.int64, total)
        _want(what, "counts", counts, i32, 3)
    dev = _device(what, page_table, free_list, free_head, slots, counts, batch.q_start)
    at = counts.data_ptr()
    # (an empty tensor has no address)
    _launch(what, dev, stream, lib().janus_page_grow, batch.ref, page_size, free_list.data_ptr(), free_list.numel(),
            _at(free_head), page_table.data_ptr(), _table(batch, page_table, page_size),
            slots.data_ptr() if total else at, at)
    _written(page_table if out is None else [page_table, slots, counts])
    return page_table, slots, counts


_ROPE_OUT = {"f32": (JANUS_F32, torch.float32), "bf16": (JANUS_BF16, torch.bfloat16),
             "fp8": (JANUS_FP8_E4M3, torch.uint8)}


def _float_code(what: str, name: str, t) -> int:
    dt = t.dtype
    if dt is torch.bfloat16:
        return JANUS_BF16
    if dt is torch.float32:
        return JANUS_F32
    raise JanusError(f"{what}: {name} is to be float32 or bfloat16, not {dt}")


def rope(batch: Batch, rotary: Rotary, x, out=None, out_dtype: Optional[str] = None, out_scale=None, stream=None):
    """janus_rope: x [total_q, heads, size] (float32 or bfloat16, adjacent elements
    in a head, any other strides) with its rotated elements turned.  Returns (out,
    out_scale or None).

    out: a tensor of x's shape, x itself to turn it in place, or None for a new
    one; out_dtype "f32", "bf16" or "fp8" (None: out's, or x's).  fp8 outputs are e4m3
    bytes (uint8, or float8_e4m3fn if given) with one scale per token.  Nothing is recorded
    for autograd: the gradient of x is rope of out's gradient with rotary.inverted()."""
    what = "janus_rope"
    total, shape = batch.total_q, x.shape
    if len(shape) != 3 or shape[0] != total:
        raise JanusError(f"{what}: x is to be [{total}, heads, size], not {tuple(shape)}")
    xdt = _float_code(what, "x", x)
    if out_dtype is None:
        given = (x if out is None else out).dtype
        out_dtype = "bf16" if given is torch.bfloat16 else "f32" if given is torch.float32 else "fp8"
    if out_dtype not in _ROPE_OUT:
        raise JanusError(f"{what}: unknown out_dtype {out_dtype!r}")
    odt, torch_dt = _ROPE_OUT[out_dtype]
    given, given_scale = out, out_scale
    if x.requires_grad or (out is not None and out.requires_grad):
        _followed(what)
    if out is None:
        out = _empty(torch_dt, x.device, stream, *shape)
    elif out.dtype is not torch_dt and not (out_dtype == "fp8" and out.dtype is torch.float8_e4m3fn):
        raise JanusError(f"{what}: out is {out.dtype}, not {out_dtype}")
    xs, os_ = x.stride(), out.stride()
    if out.shape != shape or (shape[2] > 1 and (xs[2] != 1 or os_[2] != 1)):
        raise JanusError(f"{what}: x and out are to have one shape and adjacent elements in a head")
    if out_dtype == "fp8":
        if out_scale is None:
            out_scale = _empty(torch.float32, x.device, stream, total)
        else:
            _want(what, "out_scale", out_scale, torch.float32, total)
            if out_scale.requires_grad:
                _followed(what)
    elif out_scale is not None:
        raise JanusError(f"{what}: out_scale goes with fp8 outputs")
    if rotary.positions is not None:
        rotary._check(what, batch)
    dev = _device(what, x, out, out_scale, batch.q_start, rotary.inv_freq)
    if total:
        _launch(what, dev, stream, lib().janus_rope, batch.ref, rotary.ref, x.data_ptr(), xdt, xs[0], xs[1], shape[1],
                shape[2], out.data_ptr(), odt, os_[0], os_[1], _at(out_scale))
        if given is not None:
            _written(given)
        if given_scale is not None:
            _written(given_scale)
    return out, out_scale


def kv_append(batch: Batch, x, out, rotary: Optional[Rotary] = None, x_rot=None, rows=None, out_scale=None,
              stream=None):
    """janus_kv_append: the appended tokens' rows into a cache; returns out.

    x [total_q, size] (float32 or bfloat16), or [total_q, size - rotary.dim] beside
    x_rot [total_q, rotary.dim] (x None if that is empty).  rows: int64 [total_q]
    output rows (page_grow's slots; outside the cache: skipped), or None for the
    ragged key arrays of index_scores.  out [..., row]: float32, bfloat16, or e4m3
    bytes (uint8 or float8_e4m3fn) with their scales in out_scale (float32, one
    per row), or in the row behind its elements if that is None."""
    what = "janus_kv_append"
    total, n, given = batch.total_q, 0, x if x is not None else x_rot
    for t in (x, x_rot):
        if t is not None:
            shape = t.shape
            if len(shape) != 2 or shape[0] != total or t.dtype is not given.dtype or (shape[1] > 1 and t.stride(1) != 1):
                raise JanusError(f"{what}: x and x_rot are to be [{total}, elements] of one type, elements adjacent")
            n += shape[1]
            if t.requires_grad:
                _followed(what)
    if given is None or (x_rot is not None and (rotary is None or x_rot.shape[1] != rotary.dim)):
        raise JanusError(f"{what}: x, or x_rot with the elements that rotary turns, or both")
    xdt, odt = _float_code(what, "x", given), _dtype_code(out, None)
    width = out.shape[-1] if out.dim() else 0
    if width < max(n, 1) or not out.is_contiguous() or out.dtype is torch.int16:
        raise JanusError(f"{what}: out is to be contiguous rows of at least {n} elements, float32, bfloat16 or fp8")
    num_rows = out.numel() // width
    if rows is not None:
        _want(what, "rows", rows, torch.int64, total)
    elif num_rows < batch.total_ctx:
        raise JanusError(f"{what}: {num_rows} rows for {batch.total_ctx} keys")
    if out_scale is not None:
        if odt != JANUS_FP8_E4M3:
            raise JanusError(f"{what}: out_scale goes with fp8 rows")
        if out_scale.dtype is not torch.float32 or not out_scale.is_contiguous() or out_scale.numel() != num_rows:
            raise JanusError(f"{what}: out_scale is to hold one float32 for each of {num_rows} rows")
    if out.requires_grad or (out_scale is not None and out_scale.requires_grad):
        _followed(what)
    if rotary is not None and rotary.positions is not None:
        rotary._check(what, batch)
    dev = _device(what, out, x, x_rot, rows, out_scale, batch.q_start, None if rotary is None else rotary.inv_freq)
    if total:
        _launch(what, dev, stream, lib().janus_kv_append, batch.ref, None if rotary is None else rotary.ref, _at(x),
                xdt, 0 if x is None else x.stride(0), _at(x_rot), 0 if x_rot is None else x_rot.stride(0), n,
                _at(rows), num_rows, out.data_ptr(), odt, width * out.element_size(), _at(out_scale))
        _written(out if out_scale is None else [out, out_scale])
    return out


def _row_stride(what: str, name: str, t, given: Optional[int]) -> int:
    """Elements between the rows of a pool: as given, or those of the tensor, whose last dimension is a row and
    whose other dimensions are the rows in order."""
    if given is not None:
        return int(given)
    shape = t.shape
    if len(shape) > 1:
        if t.is_contiguous():
            return shape[-1]
        step = t.stride()
        outer = [i for i in range(len(shape) - 1) if shape[i] > 1] or [len(shape) - 2]
        if (step[-1] == 1 or shape[-1] == 1) and all(step[i] == step[j] * shape[j] for i, j in zip(outer, outer[1:])):
            return step[outer[-1]]
    raise JanusError(f"{what}: {name} is to be rows of adjacent elements at one distance from each other, not a "
                     f"tensor of shape {tuple(shape)} and strides {t.stride()}")


def prefix_attn(batch: Batch, q, k_pool, v_pool, page_table, page_size: int, prefix_len: int, scale: float,
                k_row_stride: Optional[int] = None, v_row_stride: Optional[int] = None, dv: Optional[int] = None,
                out_dtype: str = "bf16", want_lse: bool = False, out=None, lse=None, workspace=None, stream=None):
    """janus_prefix_attn: dense causal attention of the appended tokens over all
    cached ids, the first prefix_len of them common to the batch's sessions;
    returns (out, lse or None).  q, out and lse as for sparse_attn, workspace as for
    sparse_attn_split.  Pools are bf16 rows [..., elements], also views of wider ones, at
    the tensors' own distances (or k_row_stride and v_row_stride elements apart)."""
    what = "janus_prefix_attn"
    total, shape, bf16, dev = batch.total_q, q.shape, torch.bfloat16, q.device
    if len(shape) != 3 or shape[0] != total or q.dtype is not bf16 or not q.is_contiguous():
        raise JanusError(f"{what}: q is to be a contiguous bfloat16 [{total}, heads, dims], not {tuple(shape)}")
    Hq, dqk = shape[1], shape[2]
    krs = _row_stride(what, "k_pool", k_pool, k_row_stride)
    vrs = krs if v_pool is k_pool and v_row_stride is k_row_stride else _row_stride(what, "v_pool", v_pool, v_row_stride)
    if dv is None:
        dv = v_pool.shape[-1] if v_pool is not k_pool else dqk
    if k_pool.dtype is not bf16 or v_pool.dtype is not bf16 or out_dtype not in ("bf16", "f32"):
        raise JanusError(f"{what}: bfloat16 pools and out_dtype bf16 or f32 expected")
    if not 0 <= prefix_len <= batch.max_ctx:  # (past 32 bits it would wrap round on its way)
        raise JanusError(f"{what}: prefix_len is to be 0 to {batch.max_ctx}, not {prefix_len}")
    _want(what, "page_table", page_table, torch.int32, batch.c.num_seqs, None)
    odt, torch_dt = (JANUS_BF16, bf16) if out_dtype == "bf16" else (JANUS_F32, torch.float32)
    given, given_lse = out, lse
    if out is None:
        out = _empty(torch_dt, dev, stream, total, Hq, dv)
    else:
        _want(what, "out", out, torch_dt, total, Hq, dv)
    if lse is not None:
        _want(what, "lse", lse, torch.float32, total, Hq)
    elif want_lse:
        lse = _empty(torch.float32, dev, stream, total, Hq)
    if q.requires_grad or k_pool.requires_grad or v_pool.requires_grad or out.requires_grad or (
            lse is not None and lse.requires_grad):
        _followed(what)
    index = _device(what, q, k_pool, v_pool, page_table, out, lse, workspace, batch.q_start)
    if total == 0:
        return out, lse
    fn = lib().janus_prefix_attn
    args = (batch.ref, q.data_ptr(), Hq, dqk, dv, k_pool.data_ptr(), v_pool.data_ptr(), krs, vrs, page_table.data_ptr(),
            _table(batch, page_table, page_size), page_size, prefix_len, scale, out.data_ptr(), odt, _at(lse))
    if workspace is None:
        size = ctypes.c_size_t(0)
        _check(fn(*args, None, ctypes.byref(size), None), what)
        workspace = _empty(torch.uint8, dev, stream, max(size.value, 1))
        at = workspace.data_ptr()
    else:
        at, size = _workspace(workspace, out)
    _launch(what, index, stream, fn, *args, at, ctypes.byref(size))
    if given is not None:
        _written(given)
    if given_lse is not None:
        _written(given_lse)
    return out, lse
