"""ctypes binding of libpec_attn.so: argument marshalling only.

Function names and argument order follow include/pec_attn.h.  torch supplies
device memory and the current HIP stream; every step of the computation runs in
the library's kernels.  There is no fallback: a missing library or a non-zero
status raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
import struct

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpec_attn.so")

PEC_BF16, PEC_F32 = 0, 1
PEC_FLAG_SIMPLE_KERNEL, PEC_FLAG_SP_SEPARATE_MERGE, PEC_FLAG_SP_STEP_LAUNCHES = 1, 2, 4
# by flags: the kernel of calls that fill the chip (smaller ones run on pec::fwd_split_kernel), and the plain one
KERNEL_NAMES = {0: "pec::fwd_il_kernel", PEC_FLAG_SIMPLE_KERNEL: "pec::fwd_simple_kernel"}

EXPORTS = (
    "pec_attn_chunk", "pec_attn_chunk_merge", "pec_attn_merge", "pec_finalize", "pec_sp_prefill",
    "pec_sp_workspace_bytes", "pec_sp_prefill_resumable", "pec_sp_resumable_workspace_bytes", "pec_sp_resumable_best_workspace_bytes", "pec_sp_prefill_num_steps", "pec_sp_prefill_step", "pec_decode_splitkv", "pec_ulysses_layout", "pec_sp_select_strategy", "pec_decode_default_splits",
    "pec_decode_workspace_bytes", "pec_decode_splitkv_static", "pec_mfma_probe", "pec_hbm_read_probe", "pec_attn_colocated", "pec_colocated_workspace_bytes", "pec_attn_varlen", "pec_varlen_workspace_bytes", "pec_status_string",
    "pec_qk_norm_rope", "pec_paged_append", "pec_attn_paged", "pec_paged_workspace_bytes",
    "pec_paged_append_mx", "pec_paged_read_mx", "pec_attn_paged_mx", "pec_paged_mx_workspace_bytes",
)


class PecShape(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("out_dtype", ctypes.c_int32), ("scale", ctypes.c_float), ("flags", ctypes.c_uint32)]


class PecSpModel(ctypes.Structure):
    _fields_ = [("d_model", ctypes.c_int64), ("n_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("seg_len", ctypes.c_int64), ("tp", ctypes.c_int32),
                ("gpus_per_node", ctypes.c_int32), ("bytes_per_element", ctypes.c_double),
                ("node_bandwidth", ctypes.c_double), ("gpu_flops", ctypes.c_double)]


class PecSpChoice(ctypes.Structure):
    _fields_ = [("attn_comm", ctypes.c_double * 2), ("attn_compute", ctypes.c_double * 2),
                ("mlp_comm", ctypes.c_double * 2), ("mlp_compute", ctypes.c_double * 2),
                ("seconds", (ctypes.c_double * 2) * 2), ("best_attn", ctypes.c_int32), ("best_mlp", ctypes.c_int32)]


class PecPagedCache(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("n_pages", ctypes.c_int64), ("page_size", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("page_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


class PecPagedCacheMx(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("n_pages", ctypes.c_int64), ("page_size", ctypes.c_int32), ("reserved", ctypes.c_int32),
                ("page_stride", ctypes.c_int64), ("row_stride", ctypes.c_int64), ("head_stride", ctypes.c_int64),
                ("scale_page_stride", ctypes.c_int64), ("scale_head_stride", ctypes.c_int64)]


class PecPagedBatch(ctypes.Structure):
    _fields_ = [("cu_seqlens_q", ctypes.c_void_p), ("seqlens_k", ctypes.c_void_p), ("block_table", ctypes.c_void_p),
                ("batch", ctypes.c_int32), ("table_len", ctypes.c_int32), ("total_q", ctypes.c_int64),
                ("max_len_q", ctypes.c_int64), ("max_len_k", ctypes.c_int64)]


class PecNormRope(ctypes.Structure):
    _fields_ = [("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("cos_sin", ctypes.c_void_p),
                ("n_positions", ctypes.c_int64), ("rotary_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("eps", ctypes.c_float), ("reserved", ctypes.c_int32)]


class PecError(RuntimeError):
    def __init__(self, fn: str, status: int):
        self.status = status
        super().__init__("%s failed: %s (%d)" % (fn, status_string(status), status))


_lib = None


def lib() -> ctypes.CDLL:
    """Load the HIP library; raises if it has not been built (no CPU fallback exists)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                "libpec_attn.so is missing: run `python -m paper_2409_15104_amd.build` (hipcc, gfx950) first")
        L = ctypes.CDLL(LIB_PATH)
        vp, i64, i32, ci, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_int, ctypes.c_size_t
        sp = ctypes.POINTER(PecShape)
        L.pec_attn_chunk.argtypes = [sp, vp, vp, vp, i64, i64, i64, i64, ci, vp, vp, vp]
        L.pec_attn_chunk_merge.argtypes = [sp, vp, vp, vp, i64, i64, i64, i64, ci, vp, vp, vp, vp]
        L.pec_attn_merge.argtypes = [sp, vp, vp, vp, vp, i64, vp]
        L.pec_finalize.argtypes = [sp, vp, vp, i64, vp]
        L.pec_sp_prefill.argtypes = [sp, vp, vp, vp, i64, i64, i64, i64, ci, vp, vp, vp, sz, vp]
        L.pec_sp_workspace_bytes.argtypes = [sp, i64]
        L.pec_sp_workspace_bytes.restype = sz
        L.pec_sp_prefill_resumable.argtypes = [sp, vp, vp, vp, i64, i64, i64, i64, ci, vp, vp, vp, sz, vp, vp, ci, vp]
        L.pec_sp_resumable_workspace_bytes.argtypes = [sp, i64]
        L.pec_sp_resumable_workspace_bytes.restype = sz
        L.pec_sp_resumable_best_workspace_bytes.argtypes = [sp, i64]
        L.pec_sp_resumable_best_workspace_bytes.restype = sz
        L.pec_sp_prefill_num_steps.argtypes = [sp, i64, i64, i64, i64, ci]
        L.pec_sp_prefill_num_steps.restype = i64
        L.pec_sp_prefill_step.argtypes = [sp, vp, vp, vp, i64, i64, i64, i64, ci, i64, vp, vp, vp, vp]
        L.pec_decode_splitkv.argtypes = [sp, vp, vp, vp, i64, i32, vp, vp, vp, sz, vp]
        L.pec_decode_splitkv_static.argtypes = [sp, vp, vp, vp, i64, i32, vp, vp, vp]
        L.pec_decode_splitkv_static.restype = ci
        L.pec_decode_default_splits.argtypes = [sp, i64]
        L.pec_decode_default_splits.restype = i32
        L.pec_decode_workspace_bytes.argtypes = [sp, i32]
        L.pec_decode_workspace_bytes.restype = sz
        L.pec_ulysses_layout.argtypes = [vp, vp, i64, i32, i32, i32, ci, vp]
        L.pec_sp_select_strategy.argtypes = [ctypes.POINTER(PecSpModel), ctypes.POINTER(PecSpChoice)]
        L.pec_attn_varlen.argtypes = [sp, vp, vp, vp, vp, i32, i64, i32, ci, vp, vp, vp, sz, vp]
        L.pec_varlen_workspace_bytes.argtypes = [i32, i64]
        L.pec_varlen_workspace_bytes.restype = sz
        L.pec_attn_colocated.argtypes = [sp, vp, vp, vp, vp, vp, i32, i64, i64, ci, vp, vp, vp, sz, vp]
        L.pec_attn_colocated.restype = ci
        L.pec_colocated_workspace_bytes.argtypes = [sp, i32, i64, i64]
        L.pec_colocated_workspace_bytes.restype = sz
        nr, pc, pb = ctypes.POINTER(PecNormRope), ctypes.POINTER(PecPagedCache), vp      # (a batch is packed per call, see _paged_batch)
        L.pec_qk_norm_rope.argtypes = [sp, nr, vp, i64, vp, i64, vp, i64, i64, vp, vp, vp]
        L.pec_qk_norm_rope.restype = ci
        L.pec_paged_append.argtypes = [sp, nr, pc, pb, vp, i64, vp, i64, vp, i64, vp, vp]
        L.pec_paged_append.restype = ci
        L.pec_attn_paged.argtypes = [sp, pc, pb, vp, i64, ci, vp, vp, vp, sz, vp]
        L.pec_attn_paged.restype = ci
        L.pec_paged_workspace_bytes.argtypes = [sp, i32, i64]
        L.pec_paged_workspace_bytes.restype = sz
        pm = ctypes.POINTER(PecPagedCacheMx)
        L.pec_paged_append_mx.argtypes = [sp, nr, pm, pb, vp, i64, vp, i64, vp, i64, vp, vp]
        L.pec_paged_append_mx.restype = ci
        L.pec_paged_read_mx.argtypes = [sp, pm, pb, vp, vp, vp]
        L.pec_paged_read_mx.restype = ci
        L.pec_attn_paged_mx.argtypes = [sp, pm, pb, vp, i64, ci, vp, vp, vp, sz, vp]
        L.pec_attn_paged_mx.restype = ci
        L.pec_paged_mx_workspace_bytes.argtypes = [sp, i32, i64, i64]
        L.pec_paged_mx_workspace_bytes.restype = sz
        L.pec_hbm_read_probe.argtypes = [vp, sz, vp, vp]
        L.pec_hbm_read_probe.restype = ci
        L.pec_mfma_probe.argtypes = [vp, sz, i32, vp, sz, vp]
        L.pec_mfma_probe.restype = i64
        L.pec_status_string.argtypes = [ci]
        L.pec_status_string.restype = ctypes.c_char_p
        for name in ("pec_attn_chunk", "pec_attn_chunk_merge", "pec_attn_merge", "pec_finalize", "pec_sp_prefill",
                     "pec_sp_prefill_step", "pec_decode_splitkv", "pec_ulysses_layout", "pec_sp_select_strategy",
                     "pec_attn_varlen"):
            getattr(L, name).restype = ci
        _lib = L
    return _lib


def status_string(status: int) -> str:
    return lib().pec_status_string(int(status)).decode()


def _check(fn: str, status: int) -> None:
    if status != 0:
        raise PecError(fn, status)


# Marshalling is on the path of every call, and the smallest ones (a decode step over a short cache: 10 us of GPU time, 9 of the
# host's) are as long as it takes: addresses go over as plain integers, one shape struct is kept per set of values, and the
# current stream is asked for its handle (0.2 us; building torch's Stream object takes 3.1 us).  Decode step over 4,096 keys,
# when it still was two launches: 15.8 -> 11.6 us per call.
@functools.lru_cache(maxsize=256)
def _shape_of(n_q_heads, n_kv_heads, head_dim, out_dtype, scale, flags) -> PecShape:
    return PecShape(n_q_heads, n_kv_heads, head_dim, PEC_F32 if out_dtype == torch.float32 else PEC_BF16, scale, flags)


def _shape(q: torch.Tensor, k: torch.Tensor, out_dtype, scale: float, flags: int = 0) -> PecShape:
    sizes = q.shape
    return _shape_of(sizes[1], k.shape[1], sizes[2], out_dtype, float(scale), int(flags))


def _ptr(t):
    return t.data_ptr() if t is not None else None


def _stream(stream):
    return stream.cuda_stream if stream is not None else _current_stream()


try:
    from torch._C import _cuda_getCurrentRawStream, _cuda_getDevice

    def _current_stream() -> int:
        return _cuda_getCurrentRawStream(_cuda_getDevice())
except ImportError:      # a torch without GPU support, or one that calls these something else
    _cuda_getDevice = None

    def _current_stream() -> int:
        return torch.cuda.current_stream().cuda_stream


def _empty(shape, dtype, device, stream, result: bool = True):
    """Memory for a call on `stream` (None: the current one).  The allocator hands out again at once what the host has freed on the
    stream that it is asked on, however much of that stream's work with it is still queued: memory for a call on another
    stream comes from that stream's own, or both work on it at the same time.  A result is held for the current stream too."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    if result:
        t.record_stream(torch.cuda.current_stream(device))
    return t


def _require(t: torch.Tensor, dtype, name: str):
    if not (t.is_cuda and t.is_contiguous() and t.dtype == dtype):
        raise ValueError("%s must be a contiguous %s tensor on the GPU" % (name, dtype))


def pec_attn_chunk(q, k, v, q_off: int, kv_off: int, causal: bool = True, out_dtype=torch.bfloat16,
                   scale: float = 0.0, flags: int = 0, out=None, lse=None, stream=None):
    """q [sq,Hq,128], k/v [sk,Hkv,128] bf16 -> (out [sq,Hq,128] out_dtype, lse [Hq,sq] fp32)."""
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _require(t, torch.bfloat16, n)
    sq, hq, d = q.shape
    sk = k.shape[0]
    if out is None:
        out = _empty((sq, hq, d), out_dtype, q.device, stream)
    if lse is None:
        lse = _empty((hq, sq), torch.float32, q.device, stream)
    _require(out, out_dtype, "out")
    _require(lse, torch.float32, "lse")
    shp = _shape(q, k, out_dtype, scale, flags)
    _check("pec_attn_chunk", lib().pec_attn_chunk(ctypes.byref(shp), _ptr(q), _ptr(k), _ptr(v), sq, sk, int(q_off),
                                                  int(kv_off), int(bool(causal)), _ptr(out), _ptr(lse),
                                                  _stream(stream)))
    return out, lse


def pec_attn_chunk_merge(q, k, v, q_off: int, kv_off: int, o_acc, lse_acc, causal: bool = True, out_final=None,
                         scale: float = 0.0, flags: int = 0, stream=None):
    """Fold one KV segment into the running fp32 (o_acc, lse_acc) in place; optionally also emit out_final."""
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _require(t, torch.bfloat16, n)
    _require(o_acc, torch.float32, "o_acc")
    _require(lse_acc, torch.float32, "lse_acc")
    out_dtype = out_final.dtype if out_final is not None else torch.bfloat16
    shp = _shape(q, k, out_dtype, scale, flags)
    _check("pec_attn_chunk_merge",
           lib().pec_attn_chunk_merge(ctypes.byref(shp), _ptr(q), _ptr(k), _ptr(v), q.shape[0], k.shape[0], int(q_off),
                                      int(kv_off), int(bool(causal)), _ptr(o_acc), _ptr(lse_acc), _ptr(out_final),
                                      _stream(stream)))
    return o_acc, lse_acc


def pec_attn_merge(o_acc, lse_acc, o_part, lse_part, stream=None):
    """In-place exact merge of (o_part, lse_part) into (o_acc, lse_acc); o_* share a dtype (bf16 or fp32)."""
    if o_acc.dtype != o_part.dtype:
        raise ValueError("o_acc and o_part must share a dtype")
    _require(o_acc, o_acc.dtype, "o_acc")
    _require(o_part, o_acc.dtype, "o_part")
    _require(lse_acc, torch.float32, "lse_acc")
    _require(lse_part, torch.float32, "lse_part")
    sq, hq, d = o_acc.shape
    shp = PecShape(hq, hq, d, PEC_F32 if o_acc.dtype == torch.float32 else PEC_BF16, 0.0, 0)
    _check("pec_attn_merge", lib().pec_attn_merge(ctypes.byref(shp), _ptr(o_acc), _ptr(lse_acc), _ptr(o_part),
                                                  _ptr(lse_part), sq, _stream(stream)))
    return o_acc, lse_acc


def pec_finalize(o_f32, o_bf16=None, stream=None):
    _require(o_f32, torch.float32, "o_f32")
    sq, hq, d = o_f32.shape
    if o_bf16 is None:
        o_bf16 = _empty((sq, hq, d), torch.bfloat16, o_f32.device, stream)
    shp = PecShape(hq, hq, d, PEC_BF16, 0.0, 0)
    _check("pec_finalize", lib().pec_finalize(ctypes.byref(shp), _ptr(o_f32), _ptr(o_bf16), sq, _stream(stream)))
    return o_bf16


def pec_sp_workspace_bytes(n_q_heads: int, n_kv_heads: int, s_q: int) -> int:
    shp = PecShape(n_q_heads, n_kv_heads, 128, PEC_BF16, 0.0, 0)
    return int(lib().pec_sp_workspace_bytes(ctypes.byref(shp), int(s_q)))


def pec_sp_prefill(q, k, v, q_off: int, chunk: int, causal: bool = True, out_dtype=torch.bfloat16,
                   scale: float = 0.0, flags: int = 0, out=None, lse=None, workspace=None, stream=None):
    """One ring member's prefill: q [s_q,Hq,128] at q_off vs k/v [s_kv,Hkv,128] in segments of `chunk`."""
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _require(t, torch.bfloat16, n)
    s_q, hq, d = q.shape
    s_kv = k.shape[0]
    if out is None:
        out = _empty((s_q, hq, d), out_dtype, q.device, stream)
    if lse is None:
        lse = _empty((hq, s_q), torch.float32, q.device, stream)
    shp = _shape(q, k, out_dtype, scale, flags)
    if workspace is None:   # only the modes that launch once per ring step keep state between launches
        per_step = flags & (PEC_FLAG_SP_STEP_LAUNCHES | PEC_FLAG_SP_SEPARATE_MERGE)
        nbytes = int(lib().pec_sp_workspace_bytes(ctypes.byref(shp), s_q)) if per_step else 0
        workspace = _empty(max(16, nbytes), torch.uint8, q.device, stream, result=False)
    _check("pec_sp_prefill",
           lib().pec_sp_prefill(ctypes.byref(shp), _ptr(q), _ptr(k), _ptr(v), s_q, int(q_off), s_kv, int(chunk),
                                int(bool(causal)), _ptr(out), _ptr(lse), _ptr(workspace), workspace.numel(),
                                _stream(stream)))
    return out, lse


def pec_sp_resumable_workspace_bytes(q, k, least: bool = False) -> int:
    """The size with which the sweep is fastest, or the least one that it takes (for a scheduler that copies it away and back)."""
    shp = _shape(q, k, torch.bfloat16, 0.0)
    size = lib().pec_sp_resumable_workspace_bytes if least else lib().pec_sp_resumable_best_workspace_bytes
    return int(size(ctypes.byref(shp), q.shape[0]))


def pec_sp_prefill_resumable(q, k, v, q_off: int, chunk: int, out, lse, workspace, pending, stop=None, resume: bool = False,
                             causal: bool = True, scale: float = 0.0, flags: int = 0, stream=None):
    """One launch of the stoppable sweep; `stop` (int32 tensor the GPU can read, or None) and `pending` (device int32
    tensor of one element) as in the C header.  Returns nothing: read `pending` to learn whether out / lse are complete."""
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _require(t, torch.bfloat16, n)
    _require(lse, torch.float32, "lse")
    _require(pending, torch.int32, "pending")
    shp = _shape(q, k, out.dtype, scale, flags)
    stop_ptr = None
    if stop is not None:
        if stop.dtype != torch.int32:
            raise ValueError("stop must be an int32 tensor")
        stop_ptr = stop.data_ptr()      # device memory or pinned host memory
    _check("pec_sp_prefill_resumable",
           lib().pec_sp_prefill_resumable(ctypes.byref(shp), _ptr(q), _ptr(k), _ptr(v), q.shape[0], int(q_off), k.shape[0],
                                          int(chunk), int(bool(causal)), _ptr(out), _ptr(lse), _ptr(workspace),
                                          workspace.numel(), stop_ptr, _ptr(pending), int(bool(resume)), _stream(stream)))


def pec_sp_prefill_num_steps(q, k, q_off: int, chunk: int, causal: bool = True) -> int:
    shp = _shape(q, k, torch.bfloat16, 0.0)
    n = int(lib().pec_sp_prefill_num_steps(ctypes.byref(shp), q.shape[0], int(q_off), k.shape[0], int(chunk),
                                           int(bool(causal))))
    if n < 0:
        raise PecError("pec_sp_prefill_num_steps", n)
    return n


def pec_sp_prefill_step(q, k, v, q_off: int, chunk: int, step: int, o_acc, lse_acc, causal: bool = True,
                        out_final=None, scale: float = 0.0, flags: int = 0, stream=None):
    """Ring step number `step` of the member's prefill, folded into the caller-kept state (o_acc, lse_acc)."""
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _require(t, torch.bfloat16, n)
    _require(o_acc, torch.float32, "o_acc")
    _require(lse_acc, torch.float32, "lse_acc")
    out_dtype = out_final.dtype if out_final is not None else torch.bfloat16
    shp = _shape(q, k, out_dtype, scale, flags)
    _check("pec_sp_prefill_step",
           lib().pec_sp_prefill_step(ctypes.byref(shp), _ptr(q), _ptr(k), _ptr(v), q.shape[0], int(q_off), k.shape[0],
                                     int(chunk), int(bool(causal)), int(step), _ptr(o_acc), _ptr(lse_acc),
                                     _ptr(out_final), _stream(stream)))
    return o_acc, lse_acc


def pec_decode_splitkv(q, k, v, n_splits: int = 0, out_dtype=torch.float32, scale: float = 0.0, flags: int = 0, out=None, lse=None,
                       workspace=None, stream=None):
    """One new token q [1,Hq,128] against a KV-cache shard k/v [sk,Hkv,128] -> (out [1,Hq,128], lse [Hq])."""
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _require(t, torch.bfloat16, n)
    if q.shape[0] != 1:
        raise ValueError("pec_decode_splitkv takes exactly one query token")
    hq = q.shape[1]
    sk = k.shape[0]
    shp = _shape(q, k, out_dtype, scale, flags)
    if n_splits == 0:
        n_splits = int(lib().pec_decode_default_splits(ctypes.byref(shp), sk))
    if out is None:
        out = _empty((1, hq, 128), out_dtype, q.device, stream)
    if lse is None:
        lse = _empty((hq,), torch.float32, q.device, stream)
    if workspace is None:
        nbytes = int(lib().pec_decode_workspace_bytes(ctypes.byref(shp), n_splits))
        workspace = _empty(max(16, nbytes), torch.uint8, q.device, stream, result=False)
    _check("pec_decode_splitkv",
           lib().pec_decode_splitkv(ctypes.byref(shp), _ptr(q), _ptr(k), _ptr(v), sk, int(n_splits), _ptr(out),
                                    _ptr(lse), _ptr(workspace), workspace.numel(), _stream(stream)))
    return out, lse


def pec_decode_splitkv_static(q, k, v, out, lse, n_splits: int = 0, scale: float = 0.0, stream=None):
    """pec_decode_splitkv without a workspace: partials live in the library's static device buffer.
    `out` [1,Hq,128] (bf16 or fp32) and `lse` [Hq] are supplied by the caller; nothing is allocated."""
    shp = _shape(q, k, out.dtype, scale)
    _check("pec_decode_splitkv_static",
           lib().pec_decode_splitkv_static(ctypes.byref(shp), _ptr(q), _ptr(k), _ptr(v), k.shape[0], int(n_splits),
                                           _ptr(out), _ptr(lse), _stream(stream)))
    return out, lse


def pec_ulysses_layout(x, n_gpus: int, to_messages: bool, out=None, stream=None):
    """to_messages: x [s,H,128] -> [G,s,H/G,128]; otherwise x [G,s,H/G,128] -> [s,H,128] (bf16)."""
    _require(x, torch.bfloat16, "x")
    if to_messages:
        s, h, d = x.shape
        shape = (n_gpus, s, h // n_gpus, d)
    else:
        g, s, hg, d = x.shape
        h = g * hg
        shape = (s, h, d)
    if out is None:
        out = _empty(shape, torch.bfloat16, x.device, stream)
    _check("pec_ulysses_layout", lib().pec_ulysses_layout(_ptr(x), _ptr(out), s, h, d, int(n_gpus),
                                                          int(bool(to_messages)), _stream(stream)))
    return out


def pec_sp_select_strategy(d_model, n_heads, n_kv_heads, head_dim, seg_len, tp, gpus_per_node, bytes_per_element,
                           node_bandwidth, gpu_flops) -> dict:
    """Host-only: volumes and time estimates of the four Megatron/Ulysses combinations and the best one."""
    m = PecSpModel(int(d_model), int(n_heads), int(n_kv_heads), int(head_dim), int(seg_len), int(tp),
                   int(gpus_per_node), float(bytes_per_element), float(node_bandwidth), float(gpu_flops))
    c = PecSpChoice()
    _check("pec_sp_select_strategy", lib().pec_sp_select_strategy(ctypes.byref(m), ctypes.byref(c)))
    return {"attn_comm": list(c.attn_comm), "attn_compute": list(c.attn_compute), "mlp_comm": list(c.mlp_comm),
            "mlp_compute": list(c.mlp_compute), "seconds": [list(c.seconds[0]), list(c.seconds[1])],
            "best": (int(c.best_attn), int(c.best_mlp))}


def pec_attn_colocated(q, k, v, cu_seqlens_q, cu_seqlens_k, causal: bool = True, out_dtype=torch.bfloat16,
                       scale: float = 0.0, flags: int = 0, out=None, lse=None, workspace=None, stream=None):
    """Colocated batch: q [Tq,Hq,128], k/v [Tk,Hkv,128], separate int32 offsets [B+1] for queries and keys."""
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _require(t, torch.bfloat16, n)
    _require(cu_seqlens_q, torch.int32, "cu_seqlens_q")
    _require(cu_seqlens_k, torch.int32, "cu_seqlens_k")
    total_q, hq, d = q.shape
    total_k = k.shape[0]
    batch = cu_seqlens_q.numel() - 1
    if out is None:
        out = _empty((total_q, hq, d), out_dtype, q.device, stream)
    if lse is None:
        lse = _empty((hq, total_q), torch.float32, q.device, stream)
    shp = _shape(q, k, out_dtype, scale, flags)
    if workspace is None:
        nbytes = int(lib().pec_colocated_workspace_bytes(ctypes.byref(shp), batch, total_q, total_k))
        workspace = _empty(max(16, nbytes), torch.uint8, q.device, stream, result=False)
    _check("pec_attn_colocated",
           lib().pec_attn_colocated(ctypes.byref(shp), _ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens_q), _ptr(cu_seqlens_k),
                                    batch, total_q, total_k, int(bool(causal)), _ptr(out), _ptr(lse), _ptr(workspace),
                                    workspace.numel(), _stream(stream)))
    return out, lse


def pec_hbm_read_probe(src, sink, stream=None) -> None:
    """One streaming read of the whole tensor `src` (any dtype, contiguous, on the GPU)."""
    _check("pec_hbm_read_probe", lib().pec_hbm_read_probe(_ptr(src), (src.numel() * src.element_size()) // 16 * 16,
                                                          _ptr(sink), _stream(stream)))


def pec_mfma_probe(operands, iters: int, sink, stream=None) -> int:
    """Launches the bare-MFMA loop on `operands` (bf16, >= 8192 elements); returns the flop count of the launch."""
    _require(operands, torch.bfloat16, "operands")
    _require(sink, torch.float32, "sink")
    n = int(lib().pec_mfma_probe(_ptr(operands), operands.numel() * 2, int(iters), _ptr(sink), sink.numel(),
                                 _stream(stream)))
    if n < 0:
        raise PecError("pec_mfma_probe", n)
    return n


def pec_varlen_workspace_bytes(batch: int, total_tokens: int) -> int:
    return int(lib().pec_varlen_workspace_bytes(int(batch), int(total_tokens)))


def pec_attn_varlen(q, k, v, cu_seqlens, max_seqlen: int, causal: bool = True, out_dtype=torch.bfloat16,
                    scale: float = 0.0, flags: int = 0, out=None, lse=None, workspace=None, stream=None):
    """Packed batch: q [T,Hq,128], k/v [T,Hkv,128], cu_seqlens int32 [B+1] on the GPU."""
    for t, n in ((q, "q"), (k, "k"), (v, "v")):
        _require(t, torch.bfloat16, n)
    _require(cu_seqlens, torch.int32, "cu_seqlens")
    total, hq, d = q.shape
    batch = cu_seqlens.numel() - 1
    if out is None:
        out = _empty((total, hq, d), out_dtype, q.device, stream)
    if lse is None:
        lse = _empty((hq, total), torch.float32, q.device, stream)
    if workspace is None:
        workspace = _empty(max(16, pec_varlen_workspace_bytes(batch, total)), torch.uint8, q.device, stream, result=False)
    shp = _shape(q, k, out_dtype, scale, flags)
    _check("pec_attn_varlen",
           lib().pec_attn_varlen(ctypes.byref(shp), _ptr(q), _ptr(k), _ptr(v), _ptr(cu_seqlens), batch, total,
                                 int(max_seqlen), int(bool(causal)), _ptr(out), _ptr(lse), _ptr(workspace),
                                 workspace.numel(), _stream(stream)))
    return out, lse


# ---- keys and values in pages

class PagedCache:
    """A server's key / value pages, laid out once: k, v [n_pages, page_size, Hkv, 128] bf16 on the GPU with a contiguous last
    dim and any other strides (multiples of 8), the same for both; a cache laid out by heads is passed as its transpose(1, 2)."""

    def __init__(self, k, v):
        for t, n in ((k, "k"), (v, "v")):
            if not (t.is_cuda and t.dtype == torch.bfloat16 and t.dim() == 4 and t.shape[3] == 128 and t.stride(3) == 1):
                raise ValueError("%s must be a bfloat16 tensor [n_pages, page_size, heads, 128] on the GPU, its last dim contiguous" % n)
        if k.shape != v.shape or k.stride() != v.stride() or k.device != v.device:
            raise ValueError("k and v must have the same shape and strides, on the same GPU")
        self.k, self.v, self.index, self.n_kv_heads = k, v, k.get_device(), k.shape[2]
        self.struct = PecPagedCache(k.data_ptr(), v.data_ptr(), k.shape[0], k.shape[1], 0, k.stride(0), k.stride(1), k.stride(2))
        self.ref = ctypes.byref(self.struct)


class PagedCacheMx:
    """A server's key / value pages held in 4 bits, laid out once: k, v uint8 [n_pages, page_size, Hkv, 64], two codes a byte, with a
    contiguous last dim and any other strides (multiples of 16; a cache laid out by heads is passed as its transpose(1, 2)); k_scale,
    v_scale uint8 [n_pages, Hkv, 4, page_size], a byte for 32 dims, their last two dims contiguous.  All on one GPU, k and v with the same strides."""

    def __init__(self, k, v, k_scale, v_scale):
        for t, n in ((k, "k"), (v, "v")):
            if not (t.is_cuda and t.dtype == torch.uint8 and t.dim() == 4 and t.shape[3] == 64 and t.stride(3) == 1):
                raise ValueError("%s must be a uint8 tensor [n_pages, page_size, heads, 64] on the GPU, its last dim contiguous" % n)
        if k.shape != v.shape or k.stride() != v.stride() or k.device != v.device:
            raise ValueError("k and v must have the same shape and strides, on the same GPU")
        n_pages, page, heads, _ = k.shape
        for t, n in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            if t.dtype != torch.uint8 or t.shape != (n_pages, heads, 4, page) or t.stride()[2:] != (page, 1) or t.device != k.device:
                raise ValueError("%s must be a uint8 tensor [n_pages, heads, 4, page_size], its last two dims contiguous, on the GPU of k" % n)
        if k_scale.stride() != v_scale.stride():
            raise ValueError("k_scale and v_scale must have the same strides")
        self.k, self.v, self.k_scale, self.v_scale, self.index, self.n_kv_heads = k, v, k_scale, v_scale, k.get_device(), heads
        self.struct = PecPagedCacheMx(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), n_pages, page, 0,
                                      k.stride(0), k.stride(1), k.stride(2), k_scale.stride(0), k_scale.stride(1))
        self.ref = ctypes.byref(self.struct)


class NormRope:
    """What a model does to its query and key rows: norm weights (fp32 [128] or None) and the rotation's angles (cos_sin fp32
    [n_positions, R], the R / 2 cosines of a position, then its sines; None: no rotation)."""

    def __init__(self, cos_sin=None, q_weight=None, k_weight=None, eps: float = 1e-6, interleaved: bool = False):
        for t, n in ((cos_sin, "cos_sin"), (q_weight, "q_weight"), (k_weight, "k_weight")):
            if t is not None:
                _require(t, torch.float32, n)
        for t, n in ((q_weight, "q_weight"), (k_weight, "k_weight")):
            if t is not None and t.shape != (128,):
                raise ValueError("%s must have 128 elements" % n)
        if cos_sin is not None and cos_sin.dim() != 2:
            raise ValueError("cos_sin must be [n_positions, rotary_dim]")
        given = [t for t in (cos_sin, q_weight, k_weight) if t is not None]
        if any(t.device != given[0].device for t in given):
            raise ValueError("cos_sin and the weights must be on the same GPU")
        self.tensors, self.index = (cos_sin, q_weight, k_weight), given[0].get_device() if given else None
        n_pos, rot = cos_sin.shape if cos_sin is not None else (0, 0)
        self.struct = PecNormRope(_ptr(q_weight), _ptr(k_weight), _ptr(cos_sin), n_pos, rot, int(bool(interleaved)), float(eps), 0)
        self.ref = ctypes.byref(self.struct)


# Checks are on the path of every call, and of small ones (a step's new tokens: 4 us of kernel, 4 of the C call with its launch)
# they were the longer half: attributes are asked for once, a device is its index, a struct is packed instead of built field by
# field.  pec_paged_append 10.9 -> 8.3 us of the host's, pec_qk_norm_rope 9.6 -> 7.8, pec_attn_paged 13.5 -> 10.9.
_BF16, _F32, _I32, _U8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
_BATCH_FORMAT = struct.Struct("@PPPiiqqq").pack      # pec_paged_batch_t


def _rows(t, name: str, index: int) -> int:
    """Checks head rows [tokens, heads, 128] whose tokens may be apart; returns the stride between them (0: packed)."""
    sizes, strides = t.shape, t.stride()
    if t.dtype is not _BF16 or t.get_device() != index or len(sizes) != 3 or sizes[2] != 128:
        raise ValueError("%s must be a bfloat16 tensor [tokens, heads, 128] on the GPU of the call" % name)
    if sizes[0] <= 1 and strides[2] == 1 and (strides[1] == 128 or sizes[1] == 1):
        return 0
    if strides[2] != 1 or (strides[1] != 128 and sizes[1] != 1):
        if sizes[0] == 0:
            return 0
        raise ValueError("the heads of a token must be contiguous in %s" % name)
    if strides[0] < 128 * sizes[1] and sizes[0] > 0:
        raise ValueError("the tokens of %s overlap" % name)
    return strides[0]


def _on(t, dtype, name: str, index: int, shape=None) -> int:
    """Checks a contiguous tensor; returns its address."""
    if t.dtype is not dtype or t.get_device() != index or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor on the GPU of the call" % (name, dtype))
    if shape is not None and t.shape != shape:
        raise ValueError("%s must have shape %s" % (name, tuple(shape)))
    return t.data_ptr()


def _paged_batch(block_table, cu_seqlens_q, seqlens_k, total_q, max_len_q, max_len_k, index: int) -> bytes:
    sizes, batch = block_table.shape, seqlens_k.numel()
    if len(sizes) != 2 or sizes[0] != batch or cu_seqlens_q.numel() != batch + 1:
        raise ValueError("block_table must be [batch, pages], cu_seqlens_q [batch + 1] and seqlens_k [batch]")
    return _BATCH_FORMAT(_on(cu_seqlens_q, _I32, "cu_seqlens_q", index), _on(seqlens_k, _I32, "seqlens_k", index),
                         _on(block_table, _I32, "block_table", index), batch, sizes[1], total_q, int(max_len_q), int(max_len_k))


@functools.lru_cache(maxsize=256)
def _shape_ref(n_q_heads, n_kv_heads, out_dtype, scale, flags):
    return ctypes.byref(_shape_of(n_q_heads, n_kv_heads, 128, out_dtype, scale, flags))


def _call(fn, name: str, index: int, stream, *args) -> None:
    """The C call, with the device of its tensors as the current one."""
    current = torch.cuda.current_device() if _cuda_getDevice is None else _cuda_getDevice()
    if current == index:
        status = fn(*args, stream.cuda_stream if stream is not None else _current_stream())
    else:
        with torch.cuda.device(index):
            status = fn(*args, stream.cuda_stream if stream is not None else _current_stream())
    if status != 0:
        raise PecError(name, status)


def pec_qk_norm_rope(q, k, norm_rope: NormRope, positions=None, pos0: int = 0, q_out=None, k_out=None, stream=None):
    """q [T,Hq,128], k [T,Hkv,128] bf16 (parts of one projection's output will do) -> normed and rotated, packed.  `positions`
    int32 [T], or None: token i is at pos0 + i.  q or k may be None; q_out may be a packed q, k_out a packed k."""
    given = q if q is not None else k
    if given is None:
        raise ValueError("neither q nor k")
    index, tokens = given.get_device(), given.shape[0]
    if index < 0 or norm_rope.index not in (None, index):
        raise ValueError("q, k and norm_rope must be on the same GPU")
    q_stride = k_stride = 0
    q_at = k_at = qo_at = ko_at = None
    if q is not None:
        q_stride, q_at = _rows(q, "q", index), q.data_ptr()
        if q_out is None:
            q_out = _empty(q.shape, _BF16, q.device, stream)
        qo_at = _on(q_out, _BF16, "q_out", index, q.shape)
    if k is not None:
        k_stride, k_at = _rows(k, "k", index), k.data_ptr()
        if k.shape[0] != tokens:
            raise ValueError("q and k must have the same number of tokens")
        if k_out is None:
            k_out = _empty(k.shape, _BF16, k.device, stream)
        ko_at = _on(k_out, _BF16, "k_out", index, k.shape)
    at = _on(positions, _I32, "positions", index, (tokens,)) if positions is not None else None
    hkv = given.shape[1] if k is None else k.shape[1]      # (of queries or keys alone: as many of the other)
    shp = _shape_ref(given.shape[1], hkv, _BF16, 0.0, 0)
    _call(lib().pec_qk_norm_rope, "pec_qk_norm_rope", index, stream, shp, norm_rope.ref, q_at, q_stride, k_at, k_stride, at, int(pos0),
          tokens, qo_at, ko_at)
    return q_out, k_out


def _append(fn, name, k, v, cache, block_table, cu_seqlens_q, seqlens_k, norm_rope, q, q_out, stream):
    index, sizes = cache.index, k.shape
    k_stride, v_stride = _rows(k, "k", index), _rows(v, "v", index)
    tokens, hkv = sizes[0], sizes[1]
    if v.shape != sizes or hkv != cache.n_kv_heads:
        raise ValueError("k and v must have the same shape, with the heads of the cache")
    q_stride, hq, q_at, qo_at, turn = 0, hkv, None, None, None
    if q is not None:
        q_stride, hq, q_at = _rows(q, "q", index), q.shape[1], q.data_ptr()
        if q.shape[0] != tokens:
            raise ValueError("q and k must have the same number of tokens")
        if q_out is None:
            q_out = _empty(q.shape, _BF16, q.device, stream)
        qo_at = _on(q_out, _BF16, "q_out", index, q.shape)
    elif q_out is not None:
        raise ValueError("q_out without q")
    if norm_rope is not None:
        turn = norm_rope.ref
        if norm_rope.index not in (None, index):
            raise ValueError("norm_rope is on another GPU")
    batch = _paged_batch(block_table, cu_seqlens_q, seqlens_k, tokens, 0, 0, index)
    _call(fn, name, index, stream, _shape_ref(hq, hkv, _BF16, 0.0, 0), turn, cache.ref, batch, q_at, q_stride,
          k.data_ptr(), k_stride, v.data_ptr(), v_stride, qo_at)
    return q_out


def pec_paged_append(k, v, cache: PagedCache, block_table, cu_seqlens_q, seqlens_k, norm_rope: NormRope = None, q=None, q_out=None,
                     stream=None):
    """The new tokens' k (normed and rotated), v [T,Hkv,128] into their sequences' pages; q [T,Hq,128], if given, normed and
    rotated into q_out, which is returned.  cu_seqlens_q [B+1], seqlens_k [B] (the new tokens among them) and block_table
    [B, pages], all int32 on the GPU."""
    return _append(lib().pec_paged_append, "pec_paged_append", k, v, cache, block_table, cu_seqlens_q, seqlens_k, norm_rope, q, q_out, stream)


def pec_paged_workspace_bytes(n_q_heads: int, n_kv_heads: int, batch: int, total_q: int) -> int:
    return int(lib().pec_paged_workspace_bytes(_shape_ref(n_q_heads, n_kv_heads, _BF16, 0.0, 0), int(batch), int(total_q)))


def pec_attn_paged(q, cache: PagedCache, block_table, cu_seqlens_q, seqlens_k, max_len_q: int = 0, max_len_k: int = 0,
                   causal: bool = True, out_dtype=torch.bfloat16, scale: float = 0.0, flags: int = 0, out=None, lse=None,
                   workspace=None, stream=None):
    """Attention of every sequence's new tokens q [T,Hq,128] over its pages -> (out [T,Hq,128], lse [Hq,T]).  Arguments as for
    pec_paged_append; max_len_q, max_len_k: the longest of the batch where the caller knows it, 0 otherwise (hints)."""
    index, sizes = cache.index, q.shape
    q_stride = _rows(q, "q", index)
    total, hq = sizes[0], sizes[1]
    if out is None:
        out = _empty(sizes, out_dtype, q.device, stream)
    if lse is None:
        lse = _empty((hq, total), _F32, q.device, stream)
    out_at, lse_at = _on(out, out_dtype, "out", index, sizes), _on(lse, _F32, "lse", index, (hq, total))
    batch = _paged_batch(block_table, cu_seqlens_q, seqlens_k, total, max_len_q, max_len_k, index)
    shp = _shape_ref(hq, cache.n_kv_heads, out_dtype, float(scale), int(flags))
    if workspace is None:
        n = int(lib().pec_paged_workspace_bytes(shp, seqlens_k.numel(), total))
        workspace = _empty(max(16, n), _U8, q.device, stream, result=False)
    _call(lib().pec_attn_paged, "pec_attn_paged", index, stream, shp, cache.ref, batch, q.data_ptr(), q_stride, 1 if causal else 0, out_at,
          lse_at, _on(workspace, _U8, "workspace", index), workspace.numel())
    return out, lse


# ---- keys and values in pages, held in 4 bits

def pec_paged_append_mx(k, v, cache: PagedCacheMx, block_table, cu_seqlens_q, seqlens_k, norm_rope: NormRope = None, q=None, q_out=None,
                        stream=None):
    """pec_paged_append into a cache in 4 bits: k (normed, rotated and rounded to bf16) and v are rounded to codes on their way."""
    return _append(lib().pec_paged_append_mx, "pec_paged_append_mx", k, v, cache, block_table, cu_seqlens_q, seqlens_k, norm_rope, q, q_out,
                   stream)


def pec_paged_read_mx(cache: PagedCacheMx, block_table, cu_seqlens_q, seqlens_k, total_q: int = None, k=None, v=None, stream=None):
    """The batch's tokens (as pec_paged_append_mx takes them) back from the cache -> (k, v) [T,Hkv,128] bf16.  T is total_q, or the rows of
    the tensors given for the results."""
    index, given = cache.index, k if k is not None else v
    if given is None and total_q is None:
        raise ValueError("total_q, or a tensor for the results")
    shape = (given.shape[0] if total_q is None else int(total_q), cache.n_kv_heads, 128)
    if k is None:
        k = _empty(shape, _BF16, cache.k.device, stream)
    if v is None:
        v = _empty(shape, _BF16, cache.k.device, stream)
    k_at, v_at = _on(k, _BF16, "k", index, shape), _on(v, _BF16, "v", index, shape)
    batch = _paged_batch(block_table, cu_seqlens_q, seqlens_k, shape[0], 0, 0, index)
    _call(lib().pec_paged_read_mx, "pec_paged_read_mx", index, stream, _shape_ref(shape[1], shape[1], _BF16, 0.0, 0), cache.ref, batch,
          k_at, v_at)
    return k, v


def pec_paged_mx_workspace_bytes(n_q_heads: int, n_kv_heads: int, batch: int, total_q: int, total_k: int = 0) -> int:
    """total_k: keys of sequences with many new tokens that room is made for (see pec_attn.h)."""
    return int(lib().pec_paged_mx_workspace_bytes(_shape_ref(n_q_heads, n_kv_heads, _BF16, 0.0, 0), int(batch), int(total_q), int(total_k)))


def pec_attn_paged_mx(q, cache: PagedCacheMx, block_table, cu_seqlens_q, seqlens_k, max_len_q: int = 0, max_len_k: int = 0,
                      causal: bool = True, out_dtype=torch.bfloat16, scale: float = 0.0, flags: int = 0, out=None, lse=None,
                      workspace=None, total_k: int = 0, stream=None):
    """pec_attn_paged over a cache in 4 bits.  total_k: keys of sequences with many new tokens, the sum of their seqlens_k, that a
    workspace made here has room for (see pec_attn.h): without it chunks behind long prefixes take half as long again."""
    index, sizes = cache.index, q.shape
    q_stride = _rows(q, "q", index)
    total, hq = sizes[0], sizes[1]
    if out is None:
        out = _empty(sizes, out_dtype, q.device, stream)
    if lse is None:
        lse = _empty((hq, total), _F32, q.device, stream)
    out_at, lse_at = _on(out, out_dtype, "out", index, sizes), _on(lse, _F32, "lse", index, (hq, total))
    batch = _paged_batch(block_table, cu_seqlens_q, seqlens_k, total, max_len_q, max_len_k, index)
    shp = _shape_ref(hq, cache.n_kv_heads, out_dtype, float(scale), int(flags))
    if workspace is None:
        n = int(lib().pec_paged_mx_workspace_bytes(shp, seqlens_k.numel(), total, int(total_k)))
        workspace = _empty(max(16, n), _U8, q.device, stream, result=False)
    _call(lib().pec_attn_paged_mx, "pec_attn_paged_mx", index, stream, shp, cache.ref, batch, q.data_ptr(), q_stride, 1 if causal else 0,
          out_at, lse_at, _on(workspace, _U8, "workspace", index), workspace.numel())
    return out, lse
