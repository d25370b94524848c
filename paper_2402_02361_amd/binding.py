"""ctypes binding of the C boundary declared in include/pruner.h.

Argument marshalling only.  Device buffers are torch tensors on the GPU (PyTorch supplies memory and
streams, nothing else); descriptors are the dataclasses of the `workloads` package or anything with the
same attribute names.
"""
import contextlib
import ctypes as C
import math
import os
import struct
from typing import NamedTuple

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
_LIB_PATH = os.path.join(_HERE, "libpruner_hip.so")

NO_COMPUTE_PENALTY = 1
NO_MEMORY_PENALTY = 2
REFERENCE_ROUNDING = 4
FUSED_ARITHMETIC = 8
NSYM = 12
SYMBOL_NAMES = ("S1", "S2", "S3", "S4", "S6", "S8", "S5_in0", "S7_in0", "S5_in1", "S7_in1", "S5_out", "S7_out")
WS_DRAFT, WS_TOPK, WS_VERIFY, WS_PRIOR_FILTER, WS_LSE, WS_PACM = 0, 1, 2, 3, 4, 5


class PrunerError(RuntimeError):
    def __init__(self, code, what):
        super().__init__(f"{what}: {strerror(code)} ({code})")
        self.code = code


class CDevice(C.Structure):
    _fields_ = [("T_p", C.c_float), ("T_m", C.c_float), ("m_l0", C.c_int32), ("m_l1", C.c_int32),
                ("pu_l1", C.c_int32), ("n_l1", C.c_int32), ("pu_l2", C.c_int32), ("n_l2", C.c_int32)]


class CDim(C.Structure):
    _fields_ = [("axis", C.c_int32 * 2), ("coef", C.c_int32 * 2)]


class CBuffer(C.Structure):
    _fields_ = [("ndim", C.c_int32), ("dim", CDim * 4)]


class CSubgraph(C.Structure):
    _fields_ = [("n_sp", C.c_int32), ("n_rd", C.c_int32), ("extent", C.c_int32 * 7),
                ("sp_levels", C.c_int32), ("rd_levels", C.c_int32), ("dtype_bytes", C.c_int32),
                ("frag", C.c_int32 * 3), ("n_in", C.c_int32), ("inp", CBuffer * 2), ("out", CBuffer), ("hw", CDevice)]


class CPacm(C.Structure):
    _fields_ = [("W1", C.c_void_p), ("b1", C.c_void_p), ("W2", C.c_void_p), ("b2", C.c_void_p), ("We", C.c_void_p), ("be", C.c_void_p),
                ("Wq", C.c_void_p), ("Wk", C.c_void_p), ("Wv", C.c_void_p), ("Wo", C.c_void_p), ("Wh", C.c_void_p), ("bh", C.c_void_p),
                ("wo", C.c_void_p), ("bo", C.c_float)]


class CMlp(C.Structure):
    _fields_ = [("W1", C.c_void_p), ("b1", C.c_void_p), ("W2", C.c_void_p), ("b2", C.c_void_p), ("w3", C.c_void_p),
                ("b3", C.c_float)]


class CCheckpoint(C.Structure):
    _fields_ = [("codes", C.c_void_p), ("exps", C.c_void_p)]


class CNorm(C.Structure):
    _fields_ = [("rows", C.c_int64), ("dim", C.c_int32), ("dtype", C.c_int32), ("center", C.c_int32), ("alpha", C.c_float), ("eps", C.c_float),
                ("w_post", C.c_void_p), ("w_pre", C.c_void_p), ("gate", C.c_void_p), ("gate_pitch", C.c_int64)]


class CHeads(C.Structure):
    _fields_ = [("p", C.c_void_p), ("batch", C.c_int64), ("token", C.c_int64), ("head", C.c_int64)]


class CAttention(C.Structure):
    _fields_ = [("dtype", C.c_int32), ("batch", C.c_int32), ("q_tokens", C.c_int32), ("k_tokens", C.c_int32), ("q_heads", C.c_int32), ("kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("flags", C.c_int32), ("scale", C.c_float), ("q_len", C.c_void_p), ("k_len", C.c_void_p), ("table", C.c_void_p),
                ("edges", C.c_void_p), ("n_edges", C.c_int32)]


class Checkpoint(NamedTuple):
    """A matrix of activations in 8 bits: codes int8 [rows, dim], exps uint8 [rows, ceil(dim / 32)]."""
    codes: object
    exps: object


_lib = None


def library_path():
    return _LIB_PATH


def load_library():
    """Load libpruner_hip.so; raises if it has not been built (there is no fallback path)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise ImportError(f"{_LIB_PATH} is missing: build it with `python -m paper_2402_02361_amd.build` "
                              "(or __graft_entry__.build()); there is no CPU fallback")
        lib = C.CDLL(_LIB_PATH)
        P = C.POINTER
        lib.pruner_draft_score.restype = C.c_int
        lib.pruner_draft_score.argtypes = [P(CSubgraph), C.c_int32, P(C.c_int64), C.c_void_p, C.c_int64, C.c_int32,
                                           C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        lib.pruner_topk.restype = C.c_int
        lib.pruner_topk.argtypes = [C.c_void_p, P(C.c_int64), C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                    C.c_void_p, C.c_size_t, C.c_void_p]
        lib.pruner_topk_static.restype = C.c_int
        lib.pruner_topk_static.argtypes = [C.c_void_p, P(C.c_int64), C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
        lib.pruner_prior_filter.restype = C.c_int
        lib.pruner_prior_filter.argtypes = [P(CSubgraph), C.c_int32, P(C.c_int64), C.c_void_p, C.c_int64, C.c_int32, C.c_int32,
                                            C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        lib.pruner_random_init_workspace_bytes.restype = C.c_size_t
        lib.pruner_random_init_workspace_bytes.argtypes = [P(CSubgraph), C.c_int32]
        lib.pruner_random_init.restype = C.c_int
        lib.pruner_random_init.argtypes = [P(CSubgraph), C.c_int32, P(C.c_int64), C.c_void_p, C.c_int64, C.c_int32, C.c_uint64,
                                           C.c_void_p, C.c_size_t, C.c_void_p]
        lib.pruner_moa_update.restype = C.c_int
        lib.pruner_moa_update.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_float, C.c_void_p, C.c_void_p]
        lib.pruner_time_dominant_draft_launch.restype = C.c_int
        lib.pruner_time_dominant_draft_launch.argtypes = [C.c_void_p, C.c_void_p, P(C.c_int64)]
        lib.pruner_pacm_score.restype = C.c_int
        lib.pruner_pacm_score.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, P(CPacm), C.c_void_p, C.c_void_p, C.c_size_t,
                                          C.c_void_p]
        lib.pruner_lse.restype = C.c_int
        lib.pruner_lse.argtypes = [P(CSubgraph), C.c_int32, P(C.c_int64), C.c_void_p, C.c_int64, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                   C.c_uint64, C.c_uint32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        lib.pruner_verify_score.restype = C.c_int
        lib.pruner_verify_score.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, P(CMlp), C.c_void_p,
                                            C.c_void_p, C.c_size_t, C.c_void_p]
        lib.pruner_checkpoint_pack.restype = C.c_int
        lib.pruner_checkpoint_pack.argtypes = [C.c_void_p, C.c_int32, C.c_int64, C.c_int32, C.c_int64, C.c_void_p, C.c_void_p]
        lib.pruner_checkpoint_restore.restype = C.c_int
        lib.pruner_checkpoint_restore.argtypes = [C.c_void_p, C.c_int32, C.c_int64, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p]
        lib.pruner_checkpoint_wgrad_workspace_bytes.restype = C.c_size_t
        lib.pruner_checkpoint_wgrad_workspace_bytes.argtypes = [C.c_int64, C.c_int32, C.c_int32]
        lib.pruner_checkpoint_wgrad.restype = C.c_int
        lib.pruner_checkpoint_wgrad.argtypes = [C.c_void_p, C.c_int32, C.c_int64, C.c_void_p, C.c_int64, C.c_int32, C.c_int32, C.c_void_p, C.c_int32,
                                                C.c_void_p, C.c_size_t, C.c_void_p]
        lib.pruner_gated_norm.restype = C.c_int
        lib.pruner_gated_norm.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        lib.pruner_gated_norm_grad_workspace_bytes.restype = C.c_size_t
        lib.pruner_gated_norm_grad_workspace_bytes.argtypes = [C.c_int64, C.c_int32]
        lib.pruner_gated_norm_grad.restype = C.c_int
        lib.pruner_gated_norm_grad.argtypes = [C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_void_p,
                                               C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        lib.pruner_rel_attention_workspace_bytes.restype = C.c_size_t
        lib.pruner_rel_attention_workspace_bytes.argtypes = [C.c_void_p]
        lib.pruner_rel_attention.restype = C.c_int
        lib.pruner_rel_attention.argtypes = [C.c_void_p] * 5 + [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        lib.pruner_rel_attention_grad_workspace_bytes.restype = C.c_size_t
        lib.pruner_rel_attention_grad_workspace_bytes.argtypes = [C.c_void_p]
        lib.pruner_rel_attention_grad.restype = C.c_int
        lib.pruner_rel_attention_grad.argtypes = [C.c_void_p] * 10 + [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        lib.pruner_workspace_bytes.restype = C.c_size_t
        lib.pruner_workspace_bytes.argtypes = [C.c_int32, C.c_int64, C.c_int32, C.c_int32]
        lib.pruner_strerror.restype = C.c_char_p
        lib.pruner_strerror.argtypes = [C.c_int]
        _lib = lib
    return _lib


def strerror(code):
    return load_library().pruner_strerror(int(code)).decode()


def workspace_bytes(which, n, n_sg, k):
    return int(load_library().pruner_workspace_bytes(which, n, n_sg, k))


def _c_buffer(b):
    out = CBuffer()
    out.ndim = len(b.dims)
    for d in range(4):
        out.dim[d].axis[:] = [-1, -1]
        out.dim[d].coef[:] = [0, 0]
    for d, terms in enumerate(b.dims):
        for t, (axis, coef) in enumerate(terms):
            out.dim[d].axis[t] = axis
            out.dim[d].coef[t] = coef
    return out


def to_c_subgraphs(subgraphs):
    """Marshal descriptors (workloads.Subgraph or look-alikes) into a C array of pruner_subgraph."""
    arr = (CSubgraph * len(subgraphs))()
    for i, sg in enumerate(subgraphs):
        s = arr[i]
        s.n_sp, s.n_rd = sg.n_sp, sg.n_rd
        for a, e in enumerate(sg.extent):
            s.extent[a] = e
        s.sp_levels, s.rd_levels, s.dtype_bytes = sg.sp_levels, sg.rd_levels, sg.dtype_bytes
        s.frag[:] = list(sg.frag)
        s.n_in = len(sg.inputs)
        for j, b in enumerate(sg.inputs):
            s.inp[j] = _c_buffer(b)
        if len(sg.inputs) < 2:
            s.inp[1] = CBuffer()
        s.out = _c_buffer(sg.out)
        h = sg.hw
        s.hw = CDevice(h.T_p, h.T_m, h.m_l0, h.m_l1, h.pu_l1, h.n_l1, h.pu_l2, h.n_l2)
    return arr


def _seg(seg_off):
    seg = np.ascontiguousarray(seg_off, dtype=np.int64)
    return seg, seg.ctypes.data_as(C.POINTER(C.c_int64))


def _stream(stream):
    import torch
    s = torch.cuda.current_stream() if stream is None else stream
    return s.cuda_stream   # (a number: the prototypes make the pointer)


# A call on a given stream takes what it makes from that stream's memory, and what it returns may be used on the current stream once that has
# waited.  That its inputs are there when the given stream reads them, and stay until it has, is the caller's to see to, as it is with torch's own calls.
_HERE = contextlib.nullcontext()


def _made_on(stream):
    """Where a call on a given stream makes tensors: from that stream's own memory.  Of another stream's, what has just been dropped there may
    still be read or written by work that is under way."""
    if stream is None:
        return _HERE
    import torch
    return torch.cuda.stream(stream)


def _returned(stream, *tensors):
    """Results of a call on a given stream will be used on the current one: once dropped, their memory is kept until what is enqueued there is done."""
    if stream is not None:
        import torch
        for t in tensors:
            if t is not None:
                t.record_stream(torch.cuda.current_stream(t.device))


def _new(stream, shape, dtype, device):
    """A tensor that a call makes and returns."""
    import torch
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    with _made_on(stream):
        t = torch.empty(shape, dtype=dtype, device=device)
    _returned(stream, t)
    return t


def _workspace(workspace, need, device, stream):
    import torch
    if workspace is None:
        with _made_on(stream):
            workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=device)
    return workspace


def _ptr(t):
    return t.data_ptr() if t is not None else None   # (a number: a ctypes object per argument costs 0.2 us more)


def draft_score(subgraphs, seg_off, tiles, flags=0, score=None, symbols=False, workspace=None, stream=None):
    """pruner_draft_score.  tiles: uint16 CUDA tensor [slots, pitch].  Returns score (and symbols int64 [12, n])."""
    import torch
    lib = load_library()
    assert tiles.is_cuda and tiles.dtype == torch.uint16 and tiles.dim() == 2 and tiles.is_contiguous()
    seg, seg_p = _seg(seg_off)
    n_sg, n = len(seg) - 1, int(seg[-1])
    arr = subgraphs if isinstance(subgraphs, C.Array) else to_c_subgraphs(subgraphs)
    if score is None:
        score = _new(stream, n, torch.float32, tiles.device)
    sym = _new(stream, (NSYM, n), torch.int64, tiles.device) if symbols is True else (symbols or None)
    need = workspace_bytes(WS_DRAFT, n, n_sg, 0)
    ws = _workspace(workspace, need, tiles.device, stream)
    rc = lib.pruner_draft_score(arr, n_sg, seg_p, _ptr(tiles), tiles.shape[1], flags, _ptr(score), _ptr(sym),
                                _ptr(ws), ws.numel(), _stream(stream))
    if rc:
        raise PrunerError(rc, "pruner_draft_score")
    return (score, sym) if sym is not None else score


def topk(score, seg_off, k, idx_out=None, val_out=None, want_values=True, workspace=None, stream=None):
    """pruner_topk.  score: float32 CUDA tensor [n].  Returns (idx int32 [n_sg, k], val float32 [n_sg, k] or None)."""
    import torch
    lib = load_library()
    assert score.is_cuda and score.dtype == torch.float32 and score.is_contiguous()
    seg, seg_p = _seg(seg_off)
    n_sg, n = len(seg) - 1, int(seg[-1])
    if idx_out is None:
        idx_out = _new(stream, (max(n_sg, 0), max(k, 0)), torch.int32, score.device)
    if val_out is None and want_values:
        val_out = _new(stream, (max(n_sg, 0), max(k, 0)), torch.float32, score.device)
    need = workspace_bytes(WS_TOPK, n, n_sg, k)
    ws = _workspace(workspace, need, score.device, stream)
    rc = lib.pruner_topk(_ptr(score), seg_p, n_sg, k, _ptr(idx_out), _ptr(val_out), _ptr(ws), ws.numel(), _stream(stream))
    if rc:
        raise PrunerError(rc, "pruner_topk")
    return idx_out, val_out


def topk_static(score, seg_off, k, idx_out, val_out=None, stream=None):
    """pruner_topk_static: pruner_topk with the scratch inside the library; the caller passes every buffer (nothing is allocated
    here either).  Returns (idx_out, val_out)."""
    import torch
    lib = load_library()
    assert score.is_cuda and score.dtype == torch.float32 and score.is_contiguous()
    seg, seg_p = _seg(seg_off)
    rc = lib.pruner_topk_static(_ptr(score), seg_p, len(seg) - 1, k, _ptr(idx_out), _ptr(val_out), _stream(stream))
    if rc:
        raise PrunerError(rc, "pruner_topk_static")
    return idx_out, val_out


def prior_filter(subgraphs, seg_off, tiles, k, flags=0, score=None, idx_out=None, val_out=None, want_values=True, workspace=None,
                 stream=None, scored_event=None):
    """pruner_prior_filter.  Returns (score float32 [n], idx int32 [n_sg, k], val float32 [n_sg, k] or None).
    scored_event: a torch.cuda.Event that has been recorded once already (its handle must exist), or None."""
    import torch
    lib = load_library()
    assert tiles.is_cuda and tiles.dtype == torch.uint16 and tiles.dim() == 2 and tiles.is_contiguous()
    seg, seg_p = _seg(seg_off)
    n_sg, n = len(seg) - 1, int(seg[-1])
    arr = subgraphs if isinstance(subgraphs, C.Array) else to_c_subgraphs(subgraphs)
    if score is None:
        score = _new(stream, n, torch.float32, tiles.device)
    if idx_out is None:
        idx_out = _new(stream, (max(n_sg, 0), max(k, 0)), torch.int32, tiles.device)
    if val_out is None and want_values:
        val_out = _new(stream, (max(n_sg, 0), max(k, 0)), torch.float32, tiles.device)
    need = workspace_bytes(WS_PRIOR_FILTER, n, n_sg, k)
    ws = _workspace(workspace, need, tiles.device, stream)
    ev = C.c_void_p(scored_event.cuda_event) if scored_event is not None else None
    rc = lib.pruner_prior_filter(arr, n_sg, seg_p, _ptr(tiles), tiles.shape[1], flags, k, _ptr(score), _ptr(idx_out), _ptr(val_out),
                                 _ptr(ws), ws.numel(), _stream(stream), ev)
    if rc:
        raise PrunerError(rc, "pruner_prior_filter")
    return score, idx_out, val_out


def lse(subgraphs, seg_off, tiles, k, n_steps, seed, mutate_q16, flags=0, score=None, workspace=None, stream=None):
    """pruner_lse.  tiles (uint16 CUDA [rows, pitch]) is updated in place.  Returns (score float32 [n],
    spec_tiles uint16 [rows, n_sg * k], spec_score float32 [n_sg, k], spec_count int32 [n_sg])."""
    import torch
    lib = load_library()
    assert tiles.is_cuda and tiles.dtype == torch.uint16 and tiles.dim() == 2 and tiles.is_contiguous()
    seg, seg_p = _seg(seg_off)
    n_sg, n = len(seg) - 1, int(seg[-1])
    arr = subgraphs if isinstance(subgraphs, C.Array) else to_c_subgraphs(subgraphs)
    if score is None:
        score = _new(stream, n, torch.float32, tiles.device)
    rows = tiles.shape[0]
    spec_tiles = _new(stream, (rows, max(n_sg * k, 0)), torch.uint16, tiles.device)
    spec_score = _new(stream, (max(n_sg, 0), max(k, 0)), torch.float32, tiles.device)
    spec_count = _new(stream, max(n_sg, 0), torch.int32, tiles.device)
    need = workspace_bytes(WS_LSE, n, n_sg, k)
    ws = _workspace(workspace, need, tiles.device, stream)
    rc = lib.pruner_lse(arr, n_sg, seg_p, _ptr(tiles), tiles.shape[1], rows, flags, k, n_steps, seed & 0xFFFFFFFFFFFFFFFF, mutate_q16,
                        _ptr(score), _ptr(spec_tiles), _ptr(spec_score), _ptr(spec_count), _ptr(ws), ws.numel(), _stream(stream))
    if rc:
        raise PrunerError(rc, "pruner_lse")
    return score, spec_tiles, spec_score, spec_count


def random_init(subgraphs, seg_off, rows, seed, tiles=None, workspace=None, stream=None, device="cuda"):
    """pruner_random_init.  Returns tiles (uint16 CUDA [rows, pitch]; a given tensor is filled in place)."""
    import torch
    lib = load_library()
    seg, seg_p = _seg(seg_off)
    n_sg, n = len(seg) - 1, int(seg[-1])
    arr = subgraphs if isinstance(subgraphs, C.Array) else to_c_subgraphs(subgraphs)
    if tiles is None:
        tiles = _new(stream, (rows, n), torch.uint16, device)
    assert tiles.is_cuda and tiles.dtype == torch.uint16 and tiles.dim() == 2 and tiles.is_contiguous() and tiles.shape[0] == rows
    need = int(lib.pruner_random_init_workspace_bytes(arr, n_sg))
    ws = _workspace(workspace, max(need, 256), tiles.device, stream)
    rc = lib.pruner_random_init(arr, n_sg, seg_p, _ptr(tiles), tiles.shape[1], rows, seed & 0xFFFFFFFFFFFFFFFF, _ptr(ws), ws.numel(),
                                _stream(stream))
    if rc:
        raise PrunerError(rc, "pruner_random_init")
    return tiles


def pacm_score(feat, n_stmt, flow, n_blk, weights, y=None, workspace=None, stream=None):
    """pruner_pacm_score.  feat float32 CUDA [n_d, 8, 164], n_stmt int32 CUDA [n_d]; flow float32 CUDA [n_d, 8, 23], n_blk
    int32 CUDA [n_d]; weights: dict of CUDA tensors W1 b1 W2 b2 We be Wq Wk Wv Wo Wh bh wo (matrices uint16 bf16 bits or
    torch.bfloat16, biases float32) and float bo."""
    import torch
    lib = load_library()
    n_d = feat.shape[0]
    assert feat.is_cuda and feat.dtype == torch.float32 and feat.is_contiguous() and feat.shape[1:] == (8, 164)
    assert flow.is_cuda and flow.dtype == torch.float32 and flow.is_contiguous() and flow.shape == (n_d, 8, 23)
    assert n_stmt.is_cuda and n_stmt.dtype == torch.int32 and n_stmt.is_contiguous() and n_stmt.numel() == n_d
    assert n_blk.is_cuda and n_blk.dtype == torch.int32 and n_blk.is_contiguous() and n_blk.numel() == n_d
    if y is None:
        y = _new(stream, n_d, torch.float32, feat.device)
    names = ("W1", "b1", "W2", "b2", "We", "be", "Wq", "Wk", "Wv", "Wo", "Wh", "bh", "wo")
    m = CPacm(*[weights[k].data_ptr() for k in names], float(weights["bo"]))
    need = workspace_bytes(WS_PACM, n_d, 0, 0)
    ws = _workspace(workspace, need, feat.device, stream)
    rc = lib.pruner_pacm_score(_ptr(feat), _ptr(n_stmt), _ptr(flow), _ptr(n_blk), n_d, C.byref(m), _ptr(y), _ptr(ws), ws.numel(), _stream(stream))
    if rc:
        raise PrunerError(rc, "pruner_pacm_score")
    return y


def moa_update(phi_s, phi_t, m, bf16=None, stream=None):
    """pruner_moa_update.  phi_s (float32 CUDA, updated in place), phi_t (float32 CUDA, same size); bf16: a uint16 CUDA
    tensor of the same size that receives the new phi_s as bfloat16 bits, or None."""
    import torch
    lib = load_library()
    assert phi_s.is_cuda and phi_s.dtype == torch.float32 and phi_s.is_contiguous()
    assert phi_t.is_cuda and phi_t.dtype == torch.float32 and phi_t.is_contiguous() and phi_t.numel() == phi_s.numel()
    if bf16 is not None:
        assert bf16.is_cuda and bf16.dtype == torch.uint16 and bf16.is_contiguous() and bf16.numel() == phi_s.numel()
    rc = lib.pruner_moa_update(_ptr(phi_s), _ptr(phi_t), phi_s.numel(), float(m), _ptr(bf16) if bf16 is not None else None, _stream(stream))
    if rc:
        raise PrunerError(rc, "pruner_moa_update")
    return phi_s


def time_dominant_draft_launch(start_event=None, stop_event=None, bytes_out=None):
    """pruner_time_dominant_draft_launch.  Events: torch.cuda.Event objects that have been recorded once (so that their
    handles exist), or None for both to switch the hook off; bytes_out: a ctypes.c_int64 that receives the launch's
    algorithmic bytes at every scoring call, or None."""
    lib = load_library()
    a = C.c_void_p(start_event.cuda_event) if start_event is not None else None
    b = C.c_void_p(stop_event.cuda_event) if stop_event is not None else None
    rc = lib.pruner_time_dominant_draft_launch(a, b, C.byref(bytes_out) if bytes_out is not None else None)
    if rc:
        raise PrunerError(rc, "pruner_time_dominant_draft_launch")


def verify_score(feat, n_stmt, weights, vscore=None, workspace=None, stream=None):
    """pruner_verify_score.  feat float32 CUDA [n_d, 8, 164]; n_stmt int32 CUDA [n_d];
    weights: dict of CUDA tensors W1/W2/w3 (uint16 bf16 bits or torch.bfloat16), b1/b2 (float32), and float b3."""
    import torch
    lib = load_library()
    assert feat.is_cuda and feat.dtype == torch.float32 and feat.is_contiguous() and feat.shape[1:] == (8, 164)
    assert n_stmt.is_cuda and n_stmt.dtype == torch.int32 and n_stmt.is_contiguous()
    n_d = feat.shape[0]
    if vscore is None:
        vscore = _new(stream, n_d, torch.float32, feat.device)
    m = CMlp(weights["W1"].data_ptr(), weights["b1"].data_ptr(), weights["W2"].data_ptr(), weights["b2"].data_ptr(),
             weights["w3"].data_ptr(), float(weights["b3"]))
    need = workspace_bytes(WS_VERIFY, n_d, 0, 0)
    ws = _workspace(workspace, need, feat.device, stream)
    rc = lib.pruner_verify_score(_ptr(feat), _ptr(n_stmt), n_d, C.byref(m), _ptr(vscore), _ptr(ws), ws.numel(), _stream(stream))
    if rc:
        raise PrunerError(rc, "pruner_verify_score")
    return vscore


# ---- operators of a trainable Transformer block

MAX_BIAS_EDGES, MAX_BIAS_DISTANCE, MAX_NORM_DIM, CHECKPOINT_GROUP = 64, 1024, 8192, 32
_BF16, _F16, _F32 = 0, 1, 2
_ATTENTION_CAUSAL, _ATTENTION_TWO_SIDED = 1, 2


_dtypes, _raw_stream = {}, None
# The structs of include/pruner.h as bytes, which a call takes like a pointer to them (a ctypes structure takes a call of a few microseconds half of one more).
_PACK_CHECKPOINT, _PACK_HEADS = struct.Struct("@2P"), struct.Struct("@P3q")
_PACK_NORM, _PACK_ATTENTION = struct.Struct("@q3i2f4x3Pq"), struct.Struct("@8if4x4Pi4x")


def _dtype(t):
    if not _dtypes:
        import torch
        _dtypes.update({torch.bfloat16: _BF16, torch.float16: _F16, torch.float32: _F32})
    return _dtypes.get(t, -1)


def _stream_on(stream, t):
    """The given stream, or the current one of t's device (a call of a few microseconds notices the 2.7 that torch.cuda.current_stream takes)."""
    global _raw_stream
    if stream is not None:
        return stream.cuda_stream
    if _raw_stream is None:
        import torch
        _raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
    return _raw_stream(t.get_device())


def _scratch(workspace, need, device, stream):
    """(tensor, pointer, bytes) of the given workspace, or of a new one that is held until the call has been made; nothing where none is needed."""
    if workspace is None:
        if need == 0:
            return None, None, 0
        import torch
        with _made_on(stream):
            workspace = torch.empty(need, dtype=torch.uint8, device=device)
    return workspace, workspace.data_ptr(), workspace.numel()


def _rows_of(t, what):
    """A matrix [rows, dim] whose rows may lie further apart than dim: (pointer, pitch)."""
    assert t.is_cuda and t.dim() == 2 and (t.stride(1) == 1 or t.shape[1] == 1) and (t.shape[0] <= 1 or t.stride(0) >= t.shape[1]), what
    return t.data_ptr(), (t.stride(0) if t.shape[0] > 1 else max(t.shape[1], 1))


def _c_checkpoint(kept, rows, dim):
    import torch
    codes, exps = kept
    assert codes.is_cuda and codes.dtype == torch.int8 and codes.is_contiguous() and codes.shape == (rows, dim), "codes"
    assert exps.is_cuda and exps.dtype == torch.uint8 and exps.is_contiguous() and exps.shape == (rows, -(-dim // CHECKPOINT_GROUP)), "exps"
    return _PACK_CHECKPOINT.pack(codes.data_ptr(), exps.data_ptr())


def _new_checkpoint(rows, dim, device):
    import torch
    return Checkpoint(torch.empty((rows, dim), dtype=torch.int8, device=device), torch.empty((rows, -(-dim // CHECKPOINT_GROUP)), dtype=torch.uint8, device=device))


def checkpoint_pack(x, kept=None, stream=None):
    """pruner_checkpoint_pack.  x: bfloat16, float16 or float32 CUDA [rows, dim] (rows may be further apart).  Returns a Checkpoint."""
    lib = load_library()
    p, pitch = _rows_of(x, "x")
    rows, dim = x.shape
    if kept is None:
        with _made_on(stream):
            kept = _new_checkpoint(rows, dim, x.device)
        _returned(stream, *kept)
    rc = lib.pruner_checkpoint_pack(p, _dtype(x.dtype), rows, dim, pitch, _c_checkpoint(kept, rows, dim), _stream_on(stream, x))
    if rc:
        raise PrunerError(rc, "pruner_checkpoint_pack")
    return kept


def checkpoint_restore(kept, dtype=None, x=None, stream=None):
    """pruner_checkpoint_restore.  Returns x (of `dtype`, or a given tensor's)."""
    import torch
    lib = load_library()
    rows, dim = kept[0].shape
    if x is None:
        with _made_on(stream):
            x = torch.empty((rows, dim), dtype=dtype, device=kept[0].device)
        _returned(stream, x)
    assert x.shape == (rows, dim), "x"
    p, pitch = _rows_of(x, "x")
    rc = lib.pruner_checkpoint_restore(_c_checkpoint(kept, rows, dim), _dtype(x.dtype), rows, dim, p, pitch, _stream_on(stream, x))
    if rc:
        raise PrunerError(rc, "pruner_checkpoint_restore")
    return x


def checkpoint_wgrad(dy, kept, dw=None, accumulate=False, workspace=None, stream=None):
    """pruner_checkpoint_wgrad: the weight gradient [n_out, dim] (float32) of a linear layer whose output's gradient is dy (bfloat16 or float16
    CUDA [rows, n_out]) and whose input is kept as a Checkpoint.  accumulate: dw is added to."""
    import torch
    lib = load_library()
    p, pitch = _rows_of(dy, "dy")
    rows, n_out = dy.shape
    dim = kept[0].shape[1]
    if dw is None:
        assert not accumulate, "accumulate needs dw"
        with _made_on(stream):
            dw = torch.empty((n_out, dim), dtype=torch.float32, device=dy.device)
        _returned(stream, dw)
    assert dw.is_cuda and dw.dtype == torch.float32 and dw.is_contiguous() and dw.shape == (n_out, dim), "dw"
    held, ws, size = _scratch(workspace, lib.pruner_checkpoint_wgrad_workspace_bytes(rows, n_out, dim), dy.device, stream)
    rc = lib.pruner_checkpoint_wgrad(p, _dtype(dy.dtype), pitch, _c_checkpoint(kept, rows, dim), rows, n_out, dim, dw.data_ptr(), int(accumulate), ws, size,
                                     _stream_on(stream, dy))
    if rc:
        raise PrunerError(rc, "pruner_checkpoint_wgrad")
    return dw


def _vector(t, dim, what):
    import torch
    assert t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() and t.shape == (dim,), what
    return t.data_ptr()


def _c_norm(x, has_f, w_post, w_pre, gate, alpha, eps, center):
    rows, dim = x.shape
    pitch = 0
    if gate is not None and gate.dim() == 1:
        _vector(gate, dim, "gate")
    elif gate is not None:
        assert gate.dtype == x.dtype and gate.shape == x.shape, "gate"
        pitch = _rows_of(gate, "gate")[1]
    return _PACK_NORM.pack(rows, dim, _dtype(x.dtype), 1 if center else 0, alpha, eps, _vector(w_post, dim, "w_post") if has_f else 0,
                           _vector(w_pre, dim, "w_pre") if w_pre is not None else 0, gate.data_ptr() if gate is not None else 0, pitch)


def gated_norm(x, f, w_post, w_pre, gate=None, alpha=1.0, eps=1e-6, center=False, checkpoint=False, stream=None):
    """pruner_gated_norm: h = alpha x + sigmoid(gate) norm(f) w_post, y = norm(h) w_pre.  x, f: CUDA [rows, dim] of one type (f None: the first norm
    of a model; w_post may then be None); w_post, w_pre float32 [dim]; gate None, [rows, dim] of x's type, or float32 [dim]; w_pre None: y is not formed.
    Returns (h, y, kept): kept is y's Checkpoint with checkpoint=True, else None."""
    import torch
    lib = load_library()
    rows, dim = x.shape
    px, x_pitch = _rows_of(x, "x")
    pf, f_pitch = None, 0
    if f is not None:
        assert f.dtype == x.dtype and f.shape == x.shape, "f"
        pf, f_pitch = _rows_of(f, "f")
    with _made_on(stream):
        h = torch.empty_like(x, memory_format=torch.contiguous_format)
        y = torch.empty_like(h) if w_pre is not None else None
        kept = _new_checkpoint(rows, dim, x.device) if checkpoint else None
    _returned(stream, h, y, *(kept or ()))
    p = _c_norm(x, f is not None, w_post, w_pre, gate, alpha, eps, center)
    rc = lib.pruner_gated_norm(p, px, x_pitch, pf, f_pitch, _ptr(h), _ptr(y), _c_checkpoint(kept, rows, dim) if checkpoint else None, _stream_on(stream, x))
    if rc:
        raise PrunerError(rc, "pruner_gated_norm")
    return h, y, kept


def gated_norm_grad(dh, dy, x, f, w_post, w_pre, gate=None, alpha=1.0, eps=1e-6, center=False, workspace=None, stream=None):
    """pruner_gated_norm_grad.  dh (or None: zero), dy: the gradients of gated_norm's h and y (dy and w_pre None where y was not formed; dh is then
    needed); f: the block's output, its Checkpoint, or None as in the forward pass.  Returns (dx, df, dgate, dw_post, dw_pre); those of what was None are None."""
    import torch
    lib = load_library()
    rows, dim = x.shape
    kept = f if isinstance(f, tuple) else None
    px, x_pitch = _rows_of(x, "x")
    for t, what in ((dh, "dh"), (dy, "dy"), (f if kept is None else None, "f")):
        assert t is None or (t.dtype == x.dtype and t.shape == x.shape), what
    assert (dy is None) == (w_pre is None) and (dy is not None or dh is not None), "dy and w_pre go together, without them dh is needed"
    pdy, dy_pitch = _rows_of(dy, "dy") if dy is not None else (None, 0)
    pdh, dh_pitch = _rows_of(dh, "dh") if dh is not None else (None, 0)
    pf, f_pitch = _rows_of(f, "f") if f is not None and kept is None else (None, 0)
    p = _c_norm(x, f is not None, w_post, w_pre, gate, alpha, eps, center)
    df = dgate = dw_post = None
    with _made_on(stream):
        dx = torch.empty_like(x, memory_format=torch.contiguous_format)
        if f is not None:
            df = torch.empty_like(dx)
            dw_post = torch.empty_like(w_post)
            if gate is not None:
                dgate = torch.empty_like(gate, memory_format=torch.contiguous_format)
        dw_pre = torch.empty_like(w_pre) if w_pre is not None else None
    _returned(stream, dx, df, dgate, dw_post, dw_pre)
    held, ws, size = _scratch(workspace, lib.pruner_gated_norm_grad_workspace_bytes(rows, dim), x.device, stream)
    rc = lib.pruner_gated_norm_grad(p, pdh, dh_pitch, pdy, dy_pitch, px, x_pitch, pf, f_pitch, _c_checkpoint(kept, rows, dim) if kept is not None else None,
                                    _ptr(dx), _ptr(df), _ptr(dgate), _ptr(dw_post), _ptr(dw_pre), ws, size, _stream_on(stream, x))
    if rc:
        raise PrunerError(rc, "pruner_gated_norm_grad")
    return dx, df, dgate, dw_post, dw_pre


def relative_edges(n, max_distance):
    """Distances at which a new bucket begins, for a table with n of them on a side: 1, 2, .. up to about half of them, the others spread evenly over the
    logarithm up to max_distance (int32 numpy array, ascending strictly)."""
    exact = max(1, (n + 1) // 2)
    assert 1 <= n <= MAX_BIAS_EDGES and n <= max_distance <= MAX_BIAS_DISTANCE, "edges"
    found = list(range(1, exact + 1))
    for i in range(1, n - exact + 1):
        at = int(round(exact * (max_distance / exact) ** (i / (n - exact))))
        found.append(min(max(at, found[-1] + 1), max_distance - (n - exact - i)))
    return np.array(found, dtype=np.int32)


def _heads(t, what):
    """A tensor [batch, tokens, heads, head_dim], the last dimension contiguous, as a pruner_heads (dimensions of one element have no stride of their own)."""
    (b, n, h, d), (sb, sn, sh, sd) = t.shape, t.stride()
    assert t.is_cuda and (sd == 1 or d == 1), what
    return _PACK_HEADS.pack(t.data_ptr(), sb if b > 1 else 0, sn if n > 1 else 0, sh if h > 1 else 0)


def _lengths(t, batch, what):
    import torch
    if t is None:
        return 0
    assert t.is_cuda and t.dtype == torch.int32 and t.is_contiguous() and t.numel() == batch, what
    return t.data_ptr()


def _c_attention(q, k, v, table, edges, q_len, k_len, causal, scale):
    batch, q_tokens, q_heads, head_dim = q.shape
    k_tokens, kv_heads = k.shape[1], k.shape[2]
    assert k.shape == (batch, k_tokens, kv_heads, head_dim) and v.shape == k.shape and k.dtype == q.dtype and v.dtype == q.dtype, "q, k, v"
    flags = _ATTENTION_CAUSAL if causal else 0
    n_edges = 0
    if table is not None:
        if not (isinstance(edges, np.ndarray) and edges.dtype == np.int32 and edges.flags.c_contiguous):
            edges = np.ascontiguousarray(edges if edges is not None else (), dtype=np.int32)
        n_edges = len(edges)
        assert table.is_cuda and table.dtype == q.dtype and table.is_contiguous() and table.dim() == 2 and table.shape[1] == q_heads, "table"
        assert table.shape[0] in (n_edges + 1, 2 * (n_edges + 1)), "table: n_edges + 1 buckets, or twice as many"
        flags |= _ATTENTION_TWO_SIDED if table.shape[0] == 2 * (n_edges + 1) else 0
    if scale is None:
        scale = 1.0 / math.sqrt(head_dim)
    # (the edges are held until the call has been made)
    return _PACK_ATTENTION.pack(_dtype(q.dtype), batch, q_tokens, k_tokens, q_heads, kv_heads, head_dim, flags, scale, _lengths(q_len, batch, "q_len"),
                                _lengths(k_len, batch, "k_len"), table.data_ptr() if table is not None else 0, edges.__array_interface__["data"][0] if n_edges else 0,
                                n_edges), edges


def rel_attention(q, k, v, table=None, edges=None, q_len=None, k_len=None, causal=False, scale=None, o=None, want_lse=False, workspace=None, stream=None):
    """pruner_rel_attention: softmax(scale q k^T + bias by relative position) v.  q: bfloat16 or float16 CUDA [batch, q_tokens, q_heads, head_dim], k, v
    [batch, k_tokens, kv_heads, head_dim], any strides with contiguous heads of at most 128; q_heads a multiple of kv_heads.  table: of the same type,
    [len(edges) + 1, q_heads] (one-sided) or [2 (len(edges) + 1), q_heads] (two-sided), or None; edges: ascending distances on the host, e.g. from
    relative_edges.  q_len, k_len: int32 CUDA [batch] or None; query i of a sequence stands at position k_len - q_len + i.  scale None: 1 / sqrt(head_dim).
    Returns o [batch, q_tokens, q_heads, head_dim], with want_lse=True (o, lse float32 [batch, q_heads, q_tokens])."""
    import torch
    lib = load_library()
    a, held_edges = _c_attention(q, k, v, table, edges, q_len, k_len, causal, scale)
    batch, q_tokens, q_heads, _ = q.shape
    made_o = o is None
    with _made_on(stream):
        if made_o:
            o = torch.empty_like(q, memory_format=torch.contiguous_format)
        lse = torch.empty((batch, q_heads, q_tokens), dtype=torch.float32, device=q.device) if want_lse else None
    _returned(stream, o if made_o else None, lse)
    assert o.shape == q.shape and o.dtype == q.dtype, "o"
    held, ws, size = _scratch(workspace, lib.pruner_rel_attention_workspace_bytes(a), q.device, stream)
    rc = lib.pruner_rel_attention(a, _heads(q, "q"), _heads(k, "k"), _heads(v, "v"), _heads(o, "o"), _ptr(lse), ws, size, _stream_on(stream, q))
    if rc:
        raise PrunerError(rc, "pruner_rel_attention")
    return (o, lse) if want_lse else o


def rel_attention_grad(do, q, k, v, o, lse, table=None, edges=None, q_len=None, k_len=None, causal=False, scale=None, workspace=None, stream=None):
    """pruner_rel_attention_grad.  do: the gradient of rel_attention's o; o, lse: what it returned; the rest as it was called.
    Returns (dq, dk, dv, dtable), dtable None without table."""
    import torch
    lib = load_library()
    a, held_edges = _c_attention(q, k, v, table, edges, q_len, k_len, causal, scale)
    batch, q_tokens, q_heads, _ = q.shape
    assert do.shape == q.shape and do.dtype == q.dtype and o.shape == q.shape and o.dtype == q.dtype, "do, o"
    assert lse.is_cuda and lse.dtype == torch.float32 and lse.is_contiguous() and lse.shape == (batch, q_heads, q_tokens), "lse"
    dense = torch.contiguous_format
    with _made_on(stream):
        dq, dk, dv = torch.empty_like(q, memory_format=dense), torch.empty_like(k, memory_format=dense), torch.empty_like(v, memory_format=dense)
        dtable = torch.empty_like(table) if table is not None else None
    _returned(stream, dq, dk, dv, dtable)
    held, ws, size = _scratch(workspace, lib.pruner_rel_attention_grad_workspace_bytes(a), q.device, stream)
    rc = lib.pruner_rel_attention_grad(a, _heads(do, "do"), _heads(q, "q"), _heads(k, "k"), _heads(v, "v"), _heads(o, "o"), _ptr(lse), _heads(dq, "dq"),
                                       _heads(dk, "dk"), _heads(dv, "dv"), _ptr(dtable), ws, size, _stream_on(stream, q))
    if rc:
        raise PrunerError(rc, "pruner_rel_attention_grad")
    return dq, dk, dv, dtable
