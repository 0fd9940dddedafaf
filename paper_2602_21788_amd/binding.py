"""Thin ctypes binding of libfcp.so: the same entry points as include/fcp.h, argument
marshalling only.  Device buffers are torch tensors (PyTorch is used for device memory and
streams, nothing else); every step of the path runs in the library's own kernels.

There is no fallback: if libfcp.so is missing or does not load, importing a function from
here raises.
"""
from __future__ import annotations

import ctypes
import os
import struct

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libfcp.so")

FCP_OK, FCP_ERR_INVALID_ARG, FCP_ERR_CAPACITY, FCP_ERR_UNSUPPORTED, FCP_ERR_HIP, FCP_ERR_STALLED = 0, -1, -2, -3, -4, -5
FCP_SCRATCH_FWD, FCP_SCRATCH_BWD = 0, 1
FCP_SCRATCH_CACHE_ATTN, FCP_SCRATCH_CACHE_WEIGH, FCP_SCRATCH_CACHE_EVICT = 2, 3, 4
FCP_SCRATCH_CACHE_SHARED, FCP_SCRATCH_CACHE_FORK, FCP_SCRATCH_CACHE_COMPACT = 5, 6, 7
FCP_BEAM_MAX_BEAMS, FCP_BEAM_MAX_KEEP = 256, 64
FCP_BF16, FCP_F32 = 0, 1
FCP_ROTARY_HALF, FCP_ROTARY_PAIRS = 0, 1
FCP_ROTARY_PLAIN, FCP_ROTARY_LINEAR, FCP_ROTARY_BASE, FCP_ROTARY_PARTS = 0, 1, 2, 3
FCP_ROTARY_MAX_PARTS = 4
FCP_CACHE_E4M3, FCP_CACHE_INT8 = 0, 1

CHUNK_DTYPE = np.dtype([("seq", "<i4"), ("rank", "<i4"), ("chunk", "<i4"),
                        ("seq_start", "<i4"), ("len", "<i4"), ("local_off", "<i4")])
WORK_DTYPE = np.dtype([("seq", "<i4"), ("rank", "<i4"), ("step", "<i4"),
                       ("q_local_off", "<i4"), ("q_seq_start", "<i4"), ("q_len", "<i4"),
                       ("n_seg", "<i4"), ("k_seq_start", "<i4", (2,)), ("k_len", "<i4", (2,))])
SPAN_DTYPE = np.dtype([("seq", "<i4"), ("start", "<i4"), ("len", "<i4")])

EXPORTS = ["fcp_last_error", "fcp_shard_plan", "fcp_plan_groups", "fcp_scratch_bytes", "fcp_attn_fwd_step", "fcp_lse_merge",
           "fcp_attn_bwd_delta", "fcp_attn_bwd_step", "fcp_grad_finalize", "fcp_scratch_status",
           "fcp_group_shard_args", "fcp_attn_fwd_step_running", "fcp_shard_plan_mixed", "fcp_mask_tables", "fcp_attn_fwd_step_mixed", "fcp_attn_bwd_step_mixed",
           "fcp_attn_bwd_step_direct", "fcp_grad_finalize_direct", "fcp_attn_fwd_step_direct", "fcp_lse_merge_direct", "fcp_attn_fwd_step_static",
           "fcp_rotary_frequencies", "fcp_rotary", "fcp_cache_scratch_bytes", "fcp_cache_append", "fcp_cache_attn", "fcp_cache_weigh", "fcp_cache_evict",
           "fcp_cache_fork", "fcp_cache_compact", "fcp_cache_attn_shared", "fcp_beam_scratch_bytes", "fcp_beam_select"]


class FcpError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"libfcp error {code}: {msg}")
        self.code = code


_lib = None


def lib() -> ctypes.CDLL:
    """Loads libfcp.so (built in-tree by paper_2602_21788_amd.build); builds it if absent."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            from . import build as _build
            _build.build()
        # torch first: it ships its own HIP runtime, and a process must not end up with two (libfcp.so loaded before
        # torch would bind to the system's copy, and the second runtime to start finds no device)
        import torch  # noqa: F401
        L = ctypes.CDLL(LIB_PATH)
        P, I32, I64, F, SZ = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_float, ctypes.c_size_t
        L.fcp_last_error.restype = ctypes.c_char_p
        L.fcp_last_error.argtypes = []
        L.fcp_shard_plan.restype = ctypes.c_int
        L.fcp_shard_plan.argtypes = [P, P, P, I32, P, I64, P, P, I64, P]
        L.fcp_plan_groups.restype = ctypes.c_int
        L.fcp_plan_groups.argtypes = [P, P, I32, I32, I64, P, P, P, P, P, P, P]
        L.fcp_scratch_bytes.restype = SZ
        L.fcp_scratch_bytes.argtypes = [ctypes.c_int, I32, I32, I32, I32, I32, I64, I32]
        L.fcp_attn_fwd_step.restype = ctypes.c_int
        L.fcp_attn_fwd_step.argtypes = [P, P, P, P, I32, P, I64, I32, I32, I32, I32, I32, I32, F, P, P, P, SZ, P]
        L.fcp_attn_fwd_step_static.restype = ctypes.c_int
        L.fcp_attn_fwd_step_static.argtypes = [P, P, P, P, I32, P, I64, I32, I32, I32, I32, I32, I32, F, P, P, P]
        L.fcp_lse_merge.restype = ctypes.c_int
        L.fcp_lse_merge.argtypes = [P, P, I32, I32, I32, I32, P, P, P]
        L.fcp_attn_bwd_delta.restype = ctypes.c_int
        L.fcp_attn_bwd_delta.argtypes = [P, P, I32, I32, I32, P, P]
        L.fcp_attn_bwd_step.restype = ctypes.c_int
        L.fcp_attn_bwd_step.argtypes = [P, P, P, P, P, P, P, I32, P, I64, I32, I32, I32, I32, I32, F, P, P, P, P, SZ, P]
        L.fcp_grad_finalize.restype = ctypes.c_int
        L.fcp_grad_finalize.argtypes = [P, P, I64, P]
        L.fcp_scratch_status.restype = ctypes.c_int
        L.fcp_scratch_status.argtypes = [P, P, P, P]
        L.fcp_group_shard_args.restype = ctypes.c_int
        L.fcp_group_shard_args.argtypes = [P, I32, P, P, I32, P, P]
        L.fcp_shard_plan_mixed.restype = ctypes.c_int
        L.fcp_shard_plan_mixed.argtypes = [P, P, P, I32, P, I32, P, I64, P, P, I64, P]
        L.fcp_mask_tables.restype = ctypes.c_int
        L.fcp_mask_tables.argtypes = [P, I32, P, I32, P, I64, I32, P, I64, P, P, P]
        L.fcp_attn_fwd_step_mixed.restype = ctypes.c_int
        L.fcp_attn_fwd_step_mixed.argtypes = [P, P, P, P, I32, P, I64, I32, I32, I32, I32, I32, I32, F, P, P, P, P, SZ, P]
        L.fcp_attn_fwd_step_running.restype = ctypes.c_int
        L.fcp_attn_fwd_step_running.argtypes = [P, P, P, P, I32, P, I64, I32, I32, I32, I32, I32, F, P, P, P, P, P, SZ, P]
        L.fcp_attn_bwd_step_mixed.restype = ctypes.c_int
        L.fcp_attn_bwd_step_mixed.argtypes = [P, P, P, P, P, P, P, I32, P, I64, I32, I32, I32, I32, I32, F, P, P, P, P, P, P,
                                              SZ, P]
        L.fcp_attn_bwd_step_direct.restype = ctypes.c_int
        L.fcp_attn_bwd_step_direct.argtypes = [P, P, P, P, P, P, P, I32, P, I64, I32, I32, I32, I32, I32, F, P, P, P, P, P, P,
                                               P, P, P, SZ, P]
        L.fcp_grad_finalize_direct.restype = ctypes.c_int
        L.fcp_grad_finalize_direct.argtypes = [P, P, P, P, P, P, P, I64, I32, I32, I32, I32, I32, P]
        L.fcp_attn_fwd_step_direct.restype = ctypes.c_int
        L.fcp_attn_fwd_step_direct.argtypes = [P, P, P, P, I32, P, I64, I32, I32, I32, I32, I32, I32, F, P, P, P, P, P, P, SZ, P]
        L.fcp_lse_merge_direct.restype = ctypes.c_int
        L.fcp_lse_merge_direct.argtypes = [P, P, I32, I32, I32, I32, I32, P, P, P, I64, P]
        D = ctypes.c_double
        L.fcp_rotary_frequencies.restype = ctypes.c_int
        L.fcp_rotary_frequencies.argtypes = [I32, D, I32, D, D, D, D, P, P]
        L.fcp_rotary.restype = ctypes.c_int
        L.fcp_rotary.argtypes = [P, I32, P, I32, I32, I32, F, I32, P]
        L.fcp_cache_scratch_bytes.restype = SZ
        L.fcp_cache_scratch_bytes.argtypes = [ctypes.c_int, P, I32, I32, I32, I32]
        L.fcp_cache_append.restype = ctypes.c_int
        L.fcp_cache_append.argtypes = [P, P, I64, P, I64, I32, P, P, P, I32, I32, P]
        L.fcp_cache_attn.restype = ctypes.c_int
        L.fcp_cache_attn.argtypes = [P, P, I64, I32, I32, P, P, P, I32, I32, F, I32, P, P, P, SZ, P]
        L.fcp_cache_weigh.restype = ctypes.c_int
        L.fcp_cache_weigh.argtypes = [P, P, I64, I32, I32, P, P, P, P, I32, I32, F, P]
        L.fcp_cache_evict.restype = ctypes.c_int
        L.fcp_cache_evict.argtypes = [P, P, P, I32, I32, P, I32, I32, I32, I32, P, P, P, SZ, P]
        L.fcp_cache_fork.restype = ctypes.c_int
        L.fcp_cache_fork.argtypes = [P, P, P, I32, I32, P, P, I32, P, P, P, P, P, SZ, P]
        L.fcp_cache_compact.restype = ctypes.c_int
        L.fcp_cache_compact.argtypes = [P, P, P, I32, I32, P, P, P, P, SZ, P]
        L.fcp_cache_attn_shared.restype = ctypes.c_int
        L.fcp_cache_attn_shared.argtypes = [P, P, I64, I32, I32, P, P, P, I32, I32, P, P, I32, F, P, P, P, SZ, P]
        L.fcp_beam_scratch_bytes.restype = SZ
        L.fcp_beam_scratch_bytes.argtypes = [I32, I32, I32, I32]
        L.fcp_beam_select.restype = ctypes.c_int
        L.fcp_beam_select.argtypes = [P, I32, I64, I32, I32, I32, P, P, I32, I32, P, P, P, P, P, SZ, P]
        _lib = L
    return _lib


def _check(rc: int):
    if rc != FCP_OK:
        raise FcpError(rc, lib().fcp_last_error().decode())


_char_at, _addressof = ctypes.c_char.from_buffer, ctypes.addressof


def _np_ptr(a):
    """Address of a contiguous numpy array (by the buffer protocol: a third of the cost of a.ctypes.data)."""
    if a is None:
        return None
    try:
        return _addressof(_char_at(a))
    except (TypeError, ValueError):               # read-only or empty
        return a.ctypes.data


def _dev_ptr(t):
    """Device pointer of a torch tensor (must be contiguous and on a GPU)."""
    if t is None:
        return None
    if t.is_cuda and t.is_contiguous():
        return t.data_ptr()                       # (an int: ctypes makes the pointer of it)
    raise ValueError("expected a contiguous device tensor")


# A forward of one short prompt takes the GPU 10 us, so what a call costs on the host shows: pointers and streams are passed as plain integers, and
# the current stream is asked for by its handle, without a stream object (0.3 instead of 3 us; the two calls of the direct forward 9.5 instead of 16.5).
def _stream(stream):
    """Handle of a stream (torch's, or a handle); None: torch's current one on the current device."""
    if stream is not None:
        return int(getattr(stream, "cuda_stream", stream))
    import torch
    try:
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    except AttributeError:                        # (a torch that has no such call)
        return torch.cuda.current_stream().cuda_stream


# ---------------------------------------------------------------------------------------
def fcp_shard_plan(seq_lens, cp_degree, base_rank=None):
    """Host only.  Returns (chunks, work) numpy structured arrays (CHUNK_DTYPE, WORK_DTYPE)."""
    sl = np.ascontiguousarray(seq_lens, dtype=np.int32)
    cd = np.ascontiguousarray(cp_degree, dtype=np.int32)
    if sl.shape != cd.shape or sl.ndim != 1:
        raise ValueError("seq_lens and cp_degree must be 1-D and the same length")
    br = None if base_rank is None else np.ascontiguousarray(base_rank, dtype=np.int32)
    if br is not None and br.shape != sl.shape:
        raise ValueError("base_rank must match seq_lens")
    nc, nw = ctypes.c_int64(0), ctypes.c_int64(0)
    plan, lists, pc, pw = lib().fcp_shard_plan, (_np_ptr(sl), _np_ptr(cd), _np_ptr(br), len(sl)), ctypes.byref(nc), ctypes.byref(nw)
    _check(plan(*lists, None, 0, pc, None, 0, pw))
    chunks = np.empty(nc.value, CHUNK_DTYPE)      # (every field of every entry is written)
    work = np.empty(nw.value, WORK_DTYPE)
    _check(plan(*lists, _np_ptr(chunks), nc.value, pc, _np_ptr(work), nw.value, pw))
    return chunks, work


def _spans(spans):
    """list of (seq, start, len) or a SPAN_DTYPE array -> contiguous SPAN_DTYPE array (order kept: the library
    checks it)"""
    if isinstance(spans, np.ndarray) and spans.dtype == SPAN_DTYPE:
        return np.ascontiguousarray(spans)
    a = np.zeros(len(spans), SPAN_DTYPE)
    for i, (k, st, ln) in enumerate(spans):
        a[i] = (k, st, ln)
    return a


def fcp_shard_plan_mixed(seq_lens, cp_degree, spans, base_rank=None):
    """Host only.  fcp_shard_plan for sequences with full-attention spans [(seq, start, len), ...]."""
    sl = np.ascontiguousarray(seq_lens, dtype=np.int32)
    cd = np.ascontiguousarray(cp_degree, dtype=np.int32)
    if sl.shape != cd.shape or sl.ndim != 1:
        raise ValueError("seq_lens and cp_degree must be 1-D and the same length")
    br = None if base_rank is None else np.ascontiguousarray(base_rank, dtype=np.int32)
    if br is not None and br.shape != sl.shape:
        raise ValueError("base_rank must match seq_lens")
    sp = _spans(spans)
    nc, nw = ctypes.c_int64(0), ctypes.c_int64(0)
    _check(lib().fcp_shard_plan_mixed(_np_ptr(sl), _np_ptr(cd), _np_ptr(br), len(sl), _np_ptr(sp), len(sp), None, 0,
                                      ctypes.byref(nc), None, 0, ctypes.byref(nw)))
    chunks = np.empty(nc.value, CHUNK_DTYPE)
    work = np.empty(nw.value, WORK_DTYPE)
    _check(lib().fcp_shard_plan_mixed(_np_ptr(sl), _np_ptr(cd), _np_ptr(br), len(sl), _np_ptr(sp), len(sp),
                                      _np_ptr(chunks), nc.value, ctypes.byref(nc), _np_ptr(work), nw.value,
                                      ctypes.byref(nw)))
    return chunks, work


def fcp_mask_tables(seq_lens, spans, chunks, rank):
    """Host only.  Returns (q_limit [tq of rank] int32, k_from [sum of seq_lens] int32, eta [n_seqs] float32)."""
    sl = np.ascontiguousarray(seq_lens, dtype=np.int32)
    sp = _spans(spans)
    ch = np.ascontiguousarray(chunks)
    if ch.dtype != CHUNK_DTYPE:
        raise ValueError("chunks must be a CHUNK_DTYPE array")
    nq = ctypes.c_int64(0)
    _check(lib().fcp_mask_tables(_np_ptr(sl), len(sl), _np_ptr(sp), len(sp), _np_ptr(ch), len(ch), int(rank), None, 0,
                                 ctypes.byref(nq), None, None))
    q_limit = np.zeros(nq.value, np.int32)
    k_from = np.zeros(int(sl.sum()), np.int32)
    eta = np.zeros(len(sl), np.float32)
    _check(lib().fcp_mask_tables(_np_ptr(sl), len(sl), _np_ptr(sp), len(sp), _np_ptr(ch), len(ch), int(rank),
                                 _np_ptr(q_limit), len(q_limit), ctypes.byref(nq), _np_ptr(k_from), _np_ptr(eta)))
    return q_limit, k_from, eta


class CostModel(ctypes.Structure):
    """fcp_cost_model: coefficients of the scheduler's time model (Eq. 8-9)."""
    _fields_ = [("alpha1", ctypes.c_double), ("alpha2", ctypes.c_double), ("beta1", ctypes.c_double),
                ("alpha3_over_v", ctypes.c_double), ("beta2", ctypes.c_double)]


def fcp_plan_groups(seq_lens, n_ranks, tokens_per_rank, cost_model, eta=None):
    """Host only.  Returns dict(group_of_seq, d_min, degree, base_rank, makespan); raises FcpError (capacity) if
    the groups' minimum degrees do not fit n_ranks.  cost_model: CostModel or a 5-tuple in its field order."""
    sl = np.ascontiguousarray(seq_lens, dtype=np.int32)
    if sl.ndim != 1:
        raise ValueError("seq_lens must be 1-D")
    et = None if eta is None else np.ascontiguousarray(eta, dtype=np.float32)
    if et is not None and et.shape != sl.shape:
        raise ValueError("eta must match seq_lens")
    cm = cost_model if isinstance(cost_model, CostModel) else CostModel(*[float(x) for x in cost_model])
    k = len(sl)
    group_of, d_min, degree, base = (np.empty(max(k, 1), np.int32) for _ in range(4))
    ng, mk = ctypes.c_int32(0), ctypes.c_double(0.0)
    _check(lib().fcp_plan_groups(_np_ptr(sl), _np_ptr(et), k, int(n_ranks), int(tokens_per_rank), ctypes.byref(cm),
                                 _np_ptr(group_of), ctypes.byref(ng), _np_ptr(d_min), _np_ptr(degree), _np_ptr(base),
                                 ctypes.byref(mk)))
    n = ng.value
    return {"group_of_seq": group_of[:k], "d_min": d_min[:n].copy(), "degree": degree[:n].copy(),
            "base_rank": base[:n].copy(), "makespan": mk.value}


def fcp_group_shard_args(group_of_seq, group_degree, group_base_rank):
    """Host only.  (cp_degree, base_rank) per sequence for fcp_shard_plan: every sequence at its group's degree."""
    go = np.ascontiguousarray(group_of_seq, dtype=np.int32)
    gd = np.ascontiguousarray(group_degree, dtype=np.int32)
    gb = np.ascontiguousarray(group_base_rank, dtype=np.int32)
    if gd.shape != gb.shape or go.ndim != 1 or gd.ndim != 1:
        raise ValueError("group_degree and group_base_rank must be 1-D and the same length")
    cd, br = np.empty(len(go), np.int32), np.empty(len(go), np.int32)
    _check(lib().fcp_group_shard_args(_np_ptr(go), len(go), _np_ptr(gd), _np_ptr(gb), len(gd), _np_ptr(cd), _np_ptr(br)))
    return cd, br


def fcp_scratch_bytes(which, tq, tkv, hq, hkv, head_dim, n_work, n_parts) -> int:
    return int(lib().fcp_scratch_bytes(which, tq, tkv, hq, hkv, head_dim, n_work, n_parts))


def fcp_attn_fwd_step(q, k, v, cu_seqlens_kv, work, n_parts, softmax_scale, o_part, lse_part, scratch, stream=None):
    """q [tq,hq,D], k/v [tkv,hkv,D] bf16; cu_seqlens_kv int32 [n_seqs+1]; work: uint8 device tensor
    holding fcp_work_desc records; o_part [n_parts,tq,hq,D] fp32; lse_part [n_parts,hq,tq] fp32."""
    tq, hq, D = q.shape
    tkv, hkv, _ = k.shape
    n_work = work.numel() // WORK_DTYPE.itemsize
    _check(lib().fcp_attn_fwd_step(_dev_ptr(q), _dev_ptr(k), _dev_ptr(v), _dev_ptr(cu_seqlens_kv),
                                   cu_seqlens_kv.numel() - 1, _dev_ptr(work), n_work, n_parts, tq, tkv, hq, hkv, D,
                                   float(softmax_scale), _dev_ptr(o_part), _dev_ptr(lse_part), _dev_ptr(scratch),
                                   scratch.numel() * scratch.element_size(), _stream(stream)))


def fcp_attn_fwd_step_static(q, k, v, cu_seqlens_kv, work, n_parts, softmax_scale, o_part, lse_part, stream=None):
    """fcp_attn_fwd_step with the library's static work area (no scratch argument, no allocation)."""
    tq, hq, D = q.shape
    tkv, hkv, _ = k.shape
    n_work = work.numel() // WORK_DTYPE.itemsize
    _check(lib().fcp_attn_fwd_step_static(_dev_ptr(q), _dev_ptr(k), _dev_ptr(v), _dev_ptr(cu_seqlens_kv),
                                          cu_seqlens_kv.numel() - 1, _dev_ptr(work), n_work, n_parts, tq, tkv, hq, hkv, D,
                                          float(softmax_scale), _dev_ptr(o_part), _dev_ptr(lse_part), _stream(stream)))


def fcp_attn_fwd_step_mixed(q, k, v, cu_seqlens_kv, work, n_parts, softmax_scale, q_limit, o_part, lse_part, scratch,
                            stream=None):
    """fcp_attn_fwd_step under a mixed mask; q_limit: int32 device tensor [tq]."""
    tq, hq, D = q.shape
    tkv, hkv, _ = k.shape
    if q_limit.numel() != tq:
        raise ValueError("q_limit must have one entry per local query row")
    n_work = work.numel() // WORK_DTYPE.itemsize
    _check(lib().fcp_attn_fwd_step_mixed(_dev_ptr(q), _dev_ptr(k), _dev_ptr(v), _dev_ptr(cu_seqlens_kv),
                                         cu_seqlens_kv.numel() - 1, _dev_ptr(work), n_work, n_parts, tq, tkv, hq, hkv, D,
                                         float(softmax_scale), _dev_ptr(q_limit), _dev_ptr(o_part), _dev_ptr(lse_part),
                                         _dev_ptr(scratch), scratch.numel() * scratch.element_size(), _stream(stream)))


def fcp_attn_fwd_step_running(q, k, v, cu_seqlens_kv, work, softmax_scale, o_run, lse_run, scratch, o_out=None,
                              q_limit=None, stream=None):
    """One ring step merged into the running result (o_run [tq,hq,D] fp32, lse_run [hq,tq] fp32, in/out);
    o_out: optional bf16 [tq,hq,D]; q_limit: optional int32 [tq] (mixed mask)."""
    tq, hq, D = q.shape
    tkv, hkv, _ = k.shape
    n_work = work.numel() // WORK_DTYPE.itemsize
    _check(lib().fcp_attn_fwd_step_running(_dev_ptr(q), _dev_ptr(k), _dev_ptr(v), _dev_ptr(cu_seqlens_kv),
                                           cu_seqlens_kv.numel() - 1, _dev_ptr(work), n_work, tq, tkv, hq, hkv, D,
                                           float(softmax_scale), _dev_ptr(q_limit), _dev_ptr(o_run), _dev_ptr(lse_run),
                                           _dev_ptr(o_out), _dev_ptr(scratch), scratch.numel() * scratch.element_size(),
                                           _stream(stream)))


def fcp_lse_merge(o_part, lse_part, o, lse, stream=None):
    n_parts, tq, hq, D = o_part.shape
    _check(lib().fcp_lse_merge(_dev_ptr(o_part), _dev_ptr(lse_part), n_parts, tq, hq, D, _dev_ptr(o), _dev_ptr(lse),
                               _stream(stream)))


def fcp_attn_bwd_delta(o, d_o, delta, stream=None):
    tq, hq, D = o.shape
    _check(lib().fcp_attn_bwd_delta(_dev_ptr(o), _dev_ptr(d_o), tq, hq, D, _dev_ptr(delta), _stream(stream)))


def fcp_attn_bwd_step(q, k, v, d_o, lse, delta, cu_seqlens_kv, work, softmax_scale, dq_acc, dk_acc, dv_acc, scratch,
                      stream=None):
    tq, hq, D = q.shape
    tkv, hkv, _ = k.shape
    n_work = work.numel() // WORK_DTYPE.itemsize
    _check(lib().fcp_attn_bwd_step(_dev_ptr(q), _dev_ptr(k), _dev_ptr(v), _dev_ptr(d_o), _dev_ptr(lse), _dev_ptr(delta),
                                   _dev_ptr(cu_seqlens_kv), cu_seqlens_kv.numel() - 1, _dev_ptr(work), n_work, tq, tkv,
                                   hq, hkv, D, float(softmax_scale), _dev_ptr(dq_acc), _dev_ptr(dk_acc), _dev_ptr(dv_acc),
                                   _dev_ptr(scratch), scratch.numel() * scratch.element_size(), _stream(stream)))


def fcp_attn_bwd_step_mixed(q, k, v, d_o, lse, delta, cu_seqlens_kv, work, softmax_scale, q_limit, k_from, dq_acc, dk_acc,
                            dv_acc, scratch, stream=None):
    """fcp_attn_bwd_step under a mixed mask; q_limit [tq], k_from [tkv]: int32 device tensors."""
    tq, hq, D = q.shape
    tkv, hkv, _ = k.shape
    if q_limit.numel() != tq or k_from.numel() != tkv:
        raise ValueError("q_limit / k_from must have one entry per local query row / pool row")
    n_work = work.numel() // WORK_DTYPE.itemsize
    _check(lib().fcp_attn_bwd_step_mixed(_dev_ptr(q), _dev_ptr(k), _dev_ptr(v), _dev_ptr(d_o), _dev_ptr(lse),
                                         _dev_ptr(delta), _dev_ptr(cu_seqlens_kv), cu_seqlens_kv.numel() - 1,
                                         _dev_ptr(work), n_work, tq, tkv, hq, hkv, D, float(softmax_scale),
                                         _dev_ptr(q_limit), _dev_ptr(k_from), _dev_ptr(dq_acc), _dev_ptr(dk_acc),
                                         _dev_ptr(dv_acc), _dev_ptr(scratch), scratch.numel() * scratch.element_size(),
                                         _stream(stream)))


def fcp_attn_fwd_step_direct(q, k, v, cu_seqlens_kv, work, n_parts, softmax_scale, o_part, lse_part, o, lse, scratch,
                             q_limit=None, stream=None):
    """Whole forward of a rank: rows fed by one work item get their final O / LSE at once (see include/fcp.h)."""
    tq, hq, D = q.shape
    tkv, hkv, _ = k.shape
    n_work = work.numel() // WORK_DTYPE.itemsize
    _check(lib().fcp_attn_fwd_step_direct(_dev_ptr(q), _dev_ptr(k), _dev_ptr(v), _dev_ptr(cu_seqlens_kv),
                                          cu_seqlens_kv.numel() - 1, _dev_ptr(work), n_work, int(n_parts), tq, tkv, hq, hkv,
                                          D, float(softmax_scale), _dev_ptr(q_limit), _dev_ptr(o_part), _dev_ptr(lse_part),
                                          _dev_ptr(o), _dev_ptr(lse), _dev_ptr(scratch),
                                          scratch.numel() * scratch.element_size(), _stream(stream)))


def fcp_lse_merge_direct(o_part, lse_part, o, lse, tkv, scratch, n_work, stream=None):
    """Second half of the direct forward: merges the rows that have partial results."""
    n_parts, tq, hq, D = o_part.shape
    _check(lib().fcp_lse_merge_direct(_dev_ptr(o_part), _dev_ptr(lse_part), n_parts, tq, int(tkv), hq, D, _dev_ptr(o),
                                      _dev_ptr(lse), _dev_ptr(scratch), int(n_work), _stream(stream)))


def fcp_attn_bwd_step_direct(q, k, v, d_o, lse, delta, cu_seqlens_kv, work, softmax_scale, dq_acc, dk_acc, dv_acc,
                             dq_out, dk_out, dv_out, scratch, q_limit=None, k_from=None, stream=None):
    """Whole backward of a rank: rows owned by one unit are written to the bf16 outputs at once (see include/fcp.h)."""
    tq, hq, D = q.shape
    tkv, hkv, _ = k.shape
    n_work = work.numel() // WORK_DTYPE.itemsize
    _check(lib().fcp_attn_bwd_step_direct(_dev_ptr(q), _dev_ptr(k), _dev_ptr(v), _dev_ptr(d_o), _dev_ptr(lse),
                                          _dev_ptr(delta), _dev_ptr(cu_seqlens_kv), cu_seqlens_kv.numel() - 1,
                                          _dev_ptr(work), n_work, tq, tkv, hq, hkv, D, float(softmax_scale),
                                          _dev_ptr(q_limit), _dev_ptr(k_from), _dev_ptr(dq_acc), _dev_ptr(dk_acc),
                                          _dev_ptr(dv_acc), _dev_ptr(dq_out), _dev_ptr(dk_out), _dev_ptr(dv_out),
                                          _dev_ptr(scratch), scratch.numel() * scratch.element_size(), _stream(stream)))


def fcp_grad_finalize_direct(dq_acc, dk_acc, dv_acc, dq_out, dk_out, dv_out, scratch, n_work, stream=None):
    """Second half of the direct backward: converts the accumulated rows, zeroes the untouched ones."""
    tq, hq, D = dq_acc.shape
    tkv, hkv, _ = dk_acc.shape
    _check(lib().fcp_grad_finalize_direct(_dev_ptr(dq_acc), _dev_ptr(dk_acc), _dev_ptr(dv_acc), _dev_ptr(dq_out),
                                          _dev_ptr(dk_out), _dev_ptr(dv_out), _dev_ptr(scratch), int(n_work), tq, tkv, hq,
                                          hkv, D, _stream(stream)))


def fcp_grad_finalize(acc, out_bf16, stream=None):
    _check(lib().fcp_grad_finalize(_dev_ptr(acc), _dev_ptr(out_bf16), acc.numel(), _stream(stream)))


def fcp_scratch_status(scratch, stream=None):
    """(n_tiles, n_rejected) recorded by the last step that used `scratch`; synchronises.  Raises FcpError
    (FCP_ERR_STALLED) if units of a backward waited for each other in vain."""
    a, b = ctypes.c_int32(0), ctypes.c_int32(0)
    _check(lib().fcp_scratch_status(_dev_ptr(scratch), _stream(stream), ctypes.byref(a), ctypes.byref(b)))
    return a.value, b.value


# ---------------------------------------------------------------------------------------
# Rotary positions and the paged 8-bit cache.  Tensors that the library reads by plain size are checked here for type and size, since
# the C ABI sees addresses only.  The smallest calls take the GPU 4 to 7 us, so what the checks cost on the host shows: torch and its types are looked up once,
# descriptors are packed as bytes (rotary positions of 16 rows of queries and keys 8.6 -> 6.7 us a call, one token of 64 sequences appended 7.0 -> 6.6).
_bf16 = _f32 = _f64 = _i32 = _u8 = None


def _types():
    global _bf16, _f32, _f64, _i32, _u8
    if _bf16 is None:
        import torch
        lib()
        _f32, _f64, _i32, _u8, _bf16 = torch.float32, torch.float64, torch.int32, torch.uint8, torch.bfloat16
    return _bf16


def _int_ptr(t, name, n=0):
    if t.dtype is not _i32 or t.numel() < n:
        raise ValueError(f"{name} must be an int32 tensor of at least {n} entries")
    return _dev_ptr(t)


def _rows(t, heads, dim, name):
    """(address, elements between rows) of a [rows, heads, dim] bf16 device tensor whose rows are whole (heads and channels next to each other)."""
    shape, stride = t.shape, t.stride()
    if t.dtype is not _bf16 or len(shape) != 3 or shape[1] != heads or shape[2] != dim or not t.is_cuda:
        raise ValueError(f"{name} must be a bf16 device tensor [rows, {heads}, {dim}]")
    if shape[0] and (stride[2] != 1 or (heads > 1 and stride[1] != dim)):
        raise ValueError(f"{name}: the heads of a row must lie next to each other")
    return t.data_ptr(), stride[0] if shape[0] > 1 else heads * dim


class RotaryPart(ctypes.Structure):
    """fcp_rotary_part"""
    _fields_ = [("x", ctypes.c_void_p), ("y", ctypes.c_void_p), ("pos", ctypes.c_void_p),
                ("x_row", ctypes.c_int64), ("x_head", ctypes.c_int64), ("y_row", ctypes.c_int64), ("y_head", ctypes.c_int64),
                ("rows", ctypes.c_int32), ("heads", ctypes.c_int32), ("x_type", ctypes.c_int32), ("y_type", ctypes.c_int32)]


_pack_part = struct.Struct("=QQQqqqqiiii").pack
assert struct.calcsize("=QQQqqqqiiii") == ctypes.sizeof(RotaryPart)


def fcp_rotary_frequencies(rot_dim, base=10000.0, scaling=FCP_ROTARY_PLAIN, factor=1.0, original_len=0.0, low=1.0, high=32.0):
    """Host only.  (turns [rot_dim / 2] float64 in turns per position, magnitude); scaling: FCP_ROTARY_PLAIN, _LINEAR, _BASE or _PARTS."""
    turns, magnitude = np.empty(max(int(rot_dim) // 2, 1), np.float64), ctypes.c_float(1.0)
    _check(lib().fcp_rotary_frequencies(int(rot_dim), float(base), int(scaling), float(factor), float(original_len), float(low),
                                        float(high), _np_ptr(turns), ctypes.byref(magnitude)))
    return turns, magnitude.value


def fcp_rotary(parts, turns, rot_dim, layout=FCP_ROTARY_HALF, magnitude=1.0, backward=False, stream=None):
    """parts: up to four (x, y, pos), x and y [rows, heads, D] bf16 or fp32 device tensors with any row and head strides (y may be x), pos int32 [rows].
    turns: fp64 device tensor [rot_dim / 2]."""
    _bf16 or _types()
    if turns.dtype is not _f64 or turns.numel() * 2 < rot_dim:
        raise ValueError("turns must be a float64 tensor of rot_dim / 2 entries")
    packed, dim = [], 0
    for x, y, pos in parts:
        shape, xs, ys, xt, yt = x.shape, x.stride(), y.stride(), x.dtype, y.dtype
        if len(shape) != 3 or shape != y.shape or (xt is not _bf16 and xt is not _f32) or (yt is not _bf16 and yt is not _f32) or not (x.is_cuda and y.is_cuda):
            raise ValueError("x and y must be bf16 or fp32 device tensors [rows, heads, head_dim] of one shape")
        n, h, d = shape
        if (dim and dim != d) or (d > 1 and (xs[2] != 1 or ys[2] != 1)):
            raise ValueError("all parts have one head_dim, channels next to each other")
        dim = d
        packed.append(_pack_part(x.data_ptr(), y.data_ptr(), _int_ptr(pos, "pos", n) or 0, xs[0], xs[1], ys[0], ys[1], n, h, xt is _f32, yt is _f32))
    _check(lib().fcp_rotary(b"".join(packed), len(packed), _dev_ptr(turns), dim or max(int(rot_dim), 2), int(rot_dim), layout, magnitude, 1 if backward else 0,
                            _stream(stream)))


class Cache(ctypes.Structure):
    """fcp_cache: a view of the caller's tensors, which it keeps.  k [n_pages, hkv, page_tokens, D] and v [n_pages, hkv, page_tokens / 16, D, 16]
    float8_e4m3fn or int8, k_scale and v_scale [n_pages, hkv] fp32, weight [n_pages, hkv, page_tokens] fp32 or None."""
    _fields_ = [("_k", ctypes.c_void_p), ("_v", ctypes.c_void_p), ("_k_scale", ctypes.c_void_p), ("_v_scale", ctypes.c_void_p),
                ("_weight", ctypes.c_void_p), ("n_pages", ctypes.c_int32), ("hkv", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_tokens", ctypes.c_int32), ("format", ctypes.c_int32)]

    def __init__(self, k, v, k_scale, v_scale, weight=None):
        import torch
        _types()
        formats = {torch.float8_e4m3fn: FCP_CACHE_E4M3, torch.int8: FCP_CACHE_INT8}
        if k.dtype not in formats or v.dtype != k.dtype or k.dim() != 4:
            raise ValueError("k and v must be float8_e4m3fn or int8 tensors, k [n_pages, hkv, page_tokens, head_dim]")
        n, h, p, d = k.shape
        if tuple(v.shape) != (n, h, p // 16, d, 16):
            raise ValueError("v must be [n_pages, hkv, page_tokens / 16, head_dim, 16]")
        for t, shape in ((k_scale, (n, h)), (v_scale, (n, h)), (weight, (n, h, p))):
            if t is not None and (t.dtype != torch.float32 or tuple(t.shape) != shape):
                raise ValueError(f"scales and weights must be float32 tensors; expected the shape {shape}")
        super().__init__(_dev_ptr(k), _dev_ptr(v), _dev_ptr(k_scale), _dev_ptr(v_scale), _dev_ptr(weight), n, h, d, p, formats[k.dtype])
        self.k, self.v, self.k_scale, self.v_scale, self.weight = k, v, k_scale, v_scale, weight


def fcp_cache_scratch_bytes(which, cache, n_seqs, max_pages, tq=0, hq=0) -> int:
    n = int(lib().fcp_cache_scratch_bytes(int(which), ctypes.byref(cache), int(n_seqs), int(max_pages), int(tq), int(hq)))
    if n == 0:
        raise FcpError(FCP_ERR_INVALID_ARG, lib().fcp_last_error().decode())
    return n


def _seqs(cu_seqlens, kv_len, pages):
    """(cu_seqlens, kv_len, pages) addresses, sequences, entries of a row of the table"""
    if len(pages.shape) != 2:
        raise ValueError("pages must be [n_seqs, max_pages]")
    n, m = pages.shape
    return None if cu_seqlens is None else _int_ptr(cu_seqlens, "cu_seqlens", n + 1), _int_ptr(kv_len, "kv_len", n), _int_ptr(pages, "pages"), n, m


def fcp_cache_append(cache, k, v, cu_seqlens, kv_len, pages, stream=None):
    """Quantises new rows k, v [n_rows, hkv, D] bf16, the last tokens of their sequences, into the cache (see include/fcp.h)."""
    h, d, n_rows = cache.hkv, cache.head_dim, k.shape[0]
    (kp, kr), (vp, vr) = _rows(k, h, d, "k"), _rows(v, h, d, "v")
    if v.shape[0] != n_rows:
        raise ValueError("k and v must have the same rows")
    cu, kl, pg, n, m = _seqs(cu_seqlens, kv_len, pages)
    _check(lib().fcp_cache_append(ctypes.byref(cache), kp, kr, vp, vr, n_rows, cu, kl, pg, n, m, _stream(stream)))


def _queries(cache, q, lse):
    """(address, row stride, rows, heads) of the queries; checks the LSE's type and shape"""
    if len(q.shape) != 3 or lse.dtype is not _f32 or len(lse.shape) != 2 or lse.shape[0] != q.shape[1] or lse.shape[1] != q.shape[0]:
        raise ValueError("q must be [tq, hq, head_dim] and lse a float32 tensor [hq, tq]")
    tq, hq, _ = q.shape
    return *_rows(q, hq, cache.head_dim, "q"), tq, hq


def fcp_cache_attn(cache, q, cu_seqlens, kv_len, pages, softmax_scale, o, lse, scratch, weigh=False, stream=None):
    """Attention of the rows q [tq, hq, D], the last tokens of their sequences, over the cache: o [tq, hq, D] bf16, lse [hq, tq] fp32."""
    qp, qr, tq, hq = _queries(cache, q, lse)
    if o.dtype is not _bf16 or o.shape != q.shape:
        raise ValueError("o must be a bf16 tensor of q's shape")
    cu, kl, pg, n, m = _seqs(cu_seqlens, kv_len, pages)
    _check(lib().fcp_cache_attn(ctypes.byref(cache), qp, qr, tq, hq, cu, kl, pg, n, m, softmax_scale, 1 if weigh else 0, _dev_ptr(o), _dev_ptr(lse),
                                _dev_ptr(scratch), scratch.numel() * scratch.element_size(), _stream(stream)))


def fcp_cache_weigh(cache, q, lse, cu_seqlens, kv_len, pages, softmax_scale, stream=None):
    """Adds the attention weights of the rows q, whose log-sum-exp lse [hq, tq] is known, to the cache's weights."""
    qp, qr, tq, hq = _queries(cache, q, lse)
    cu, kl, pg, n, m = _seqs(cu_seqlens, kv_len, pages)
    _check(lib().fcp_cache_weigh(ctypes.byref(cache), qp, qr, tq, hq, _dev_ptr(lse), cu, kl, pg, n, m, softmax_scale, _stream(stream)))


def fcp_cache_evict(cache, pages, kv_len, new_pages, budget, n_first, n_recent, kept, new_len, scratch, stream=None):
    """Cuts every sequence to at most `budget` tokens per KV head and moves them to new_pages; kept [n_seqs, hkv, budget], new_len [n_seqs] int32 out."""
    _, kl, pg, n, m = _seqs(None, kv_len, pages)
    if len(new_pages.shape) != 2 or new_pages.shape[0] != n:
        raise ValueError("new_pages must be [n_seqs, max_new_pages]")
    _check(lib().fcp_cache_evict(ctypes.byref(cache), pg, kl, n, m, _int_ptr(new_pages, "new_pages"), new_pages.shape[1], budget, n_first,
                                 n_recent, _int_ptr(kept, "kept", n * cache.hkv * budget), _int_ptr(new_len, "new_len", n), _dev_ptr(scratch),
                                 scratch.numel() * scratch.element_size(), _stream(stream)))


# ---------------------------------------------------------------------------------------
# Several continuations of a prompt: who holds which page, and which beams go on.
def _bytes_ptr(t, name, n):
    if t is not None and (t.dtype is not _u8 or t.numel() < n):
        raise ValueError(f"{name} must be a uint8 tensor of at least {n} entries")
    return _dev_ptr(t)


def fcp_cache_fork(cache, pages, kv_len, parent, news, new_pages, new_len, counts, scratch, busy=None, stream=None):
    """Tables of the sequences that continue those of pages [n_seqs, max_pages], kv_len: sequence i has the tokens of sequence parent[i] and room for news[i] more.  new_pages [n_new,
    max_pages], new_len [n_new], counts [3] (pages handed out, lacking, free) int32 out; busy: uint8 [n_pages] or None (see include/fcp.h)."""
    _, kl, pg, n, m = _seqs(None, kv_len, pages)
    if len(new_pages.shape) != 2 or new_pages.shape[1] != m:
        raise ValueError("new_pages must be [n_new, max_pages], its rows as long as those of pages")
    n_new = new_pages.shape[0]
    _check(lib().fcp_cache_fork(ctypes.byref(cache), pg, kl, n, m, _int_ptr(parent, "parent", n_new), _int_ptr(news, "news", n_new), n_new,
                                _bytes_ptr(busy, "busy", cache.n_pages), _int_ptr(new_pages, "new_pages"), _int_ptr(new_len, "new_len", n_new), _int_ptr(counts, "counts", 3),
                                _dev_ptr(scratch), scratch.numel() * scratch.element_size(), _stream(stream)))


def fcp_cache_compact(cache, pages, kv_len, new_pages, counts, scratch, busy=None, stream=None):
    """Moves the pages in use to the lowest numbers: new_pages [n_seqs, max_pages] (may be pages), counts [3] (pages moved, in use, first number past all) int32 out."""
    _, kl, pg, n, m = _seqs(None, kv_len, pages)
    if tuple(new_pages.shape) != (n, m):
        raise ValueError("new_pages must have the shape of pages")
    _check(lib().fcp_cache_compact(ctypes.byref(cache), pg, kl, n, m, _bytes_ptr(busy, "busy", cache.n_pages), _int_ptr(new_pages, "new_pages"),
                                   _int_ptr(counts, "counts", 3), _dev_ptr(scratch), scratch.numel() * scratch.element_size(), _stream(stream)))


def fcp_cache_attn_shared(cache, q, cu_seqlens, kv_len, pages, groups, shared_len, softmax_scale, o, lse, scratch, stream=None):
    """fcp_cache_attn where the sequences groups[g] .. groups[g + 1] - 1 have their first shared_len[g] tokens in common; groups [n_groups + 1], shared_len [n_groups] int32."""
    qp, qr, tq, hq = _queries(cache, q, lse)
    if o.dtype is not _bf16 or o.shape != q.shape:
        raise ValueError("o must be a bf16 tensor of q's shape")
    cu, kl, pg, n, m = _seqs(cu_seqlens, kv_len, pages)
    n_groups = shared_len.numel()
    _check(lib().fcp_cache_attn_shared(ctypes.byref(cache), qp, qr, tq, hq, cu, kl, pg, n, m, _int_ptr(groups, "groups", n_groups + 1), _int_ptr(shared_len, "shared_len"), n_groups,
                                       softmax_scale, _dev_ptr(o), _dev_ptr(lse), _dev_ptr(scratch), scratch.numel() * scratch.element_size(), _stream(stream)))


def fcp_beam_scratch_bytes(n_prompts, beams, vocab, keep) -> int:
    n = int(lib().fcp_beam_scratch_bytes(int(n_prompts), int(beams), int(vocab), int(keep)))
    if n == 0:
        raise FcpError(FCP_ERR_INVALID_ARG, lib().fcp_last_error().decode())
    return n


def fcp_beam_select(logits, score, beams, parent, token, new_score, scratch, done=None, end_token=-1, new_done=None, stream=None):
    """The best continuations of every prompt: logits [n_prompts * beams, vocab] bf16 or fp32 (rows with any stride), score [n_prompts * beams] fp32, done uint8 or None.  parent, token int32,
    new_score fp32, new_done uint8 or None, all [n_prompts, keep]: out, best first (see include/fcp.h)."""
    _bf16 or _types()
    if len(logits.shape) != 2 or (logits.dtype is not _bf16 and logits.dtype is not _f32) or not logits.is_cuda or (logits.shape[1] > 1 and logits.stride(1) != 1):
        raise ValueError("logits must be a bf16 or fp32 device tensor [rows, vocab], the logits of a row next to each other")
    rows, vocab = logits.shape
    n = parent.shape[0] if len(parent.shape) == 2 else -1
    if n < 0 or n * beams != rows:
        raise ValueError("parent must be [n_prompts, keep], with n_prompts * beams rows of logits")
    keep = parent.shape[1]
    for t, name in ((token, "token"), (new_score, "new_score"), (new_done, "new_done")):
        if t is not None and t.shape != parent.shape:
            raise ValueError(f"{name} must have the shape of parent")
    if score.dtype is not _f32 or score.numel() != rows or new_score.dtype is not _f32:
        raise ValueError("score and new_score must be float32 tensors, score with an entry for every row")
    _check(lib().fcp_beam_select(logits.data_ptr(), 1 if logits.dtype is _f32 else 0, logits.stride(0) if rows > 1 else vocab, n, int(beams), vocab, _dev_ptr(score),
                                 _bytes_ptr(done, "done", rows), int(end_token), keep, _int_ptr(parent, "parent"), _int_ptr(token, "token"), _dev_ptr(new_score),
                                 _bytes_ptr(new_done, "new_done", n * keep), _dev_ptr(scratch), scratch.numel() * scratch.element_size(), _stream(stream)))
