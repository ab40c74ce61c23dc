"""Thin ctypes binding of libsvg2_hip.so (include/svg2.h).

Argument marshalling only: tensors are torch CUDA(=HIP) tensors used as device
buffers, outputs and the workspace are allocated with torch, the current torch
stream is passed through, and every step of the path runs in the library's
kernels.  There is no fallback: if the library is missing or a call fails, an
exception is raised.
"""
from __future__ import annotations

import contextlib
import ctypes
import functools
import os
import struct
from types import SimpleNamespace
from typing import Optional

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsvg2_hip.so")

SVG2_F32, SVG2_BF16 = 0, 1
SVG2_OK = 0
MAX_CLUSTERS = 4096

EXPORTS = (
    "svg2_last_error", "svg2_version",
    "svg2_kmeans_workspace_size", "svg2_kmeans",
    "svg2_permute_workspace_size", "svg2_permute", "svg2_permute_noalloc",
    "svg2_select_topp_workspace_size", "svg2_select_topp",
    "svg2_sparse_attn_workspace_size", "svg2_sparse_attn", "svg2_sparse_attn_gather_free",
    "svg2_forward_workspace_size", "svg2_forward",
    "svg2_forward_gather_free_workspace_size", "svg2_forward_gather_free",
    "svg2_quantize_fp8_workspace_size", "svg2_quantize_fp8", "svg2_sparse_attn_fp8",
    "svg2_forward_fp8_workspace_size", "svg2_forward_fp8",
    "svg2_attention_recall_workspace_size", "svg2_attention_recall",
    "svg2_kmeans_pp_init_workspace_size", "svg2_kmeans_pp_init",
    "svg2_rope", "svg2_rope_backward_workspace_size", "svg2_rope_backward",
    "svg2_quantize_mxfp4", "svg2_dequantize_mxfp4", "svg2_matmul_mxfp4_workspace_size", "svg2_matmul_mxfp4",
    "svg2_layer_norm", "svg2_layer_norm_fp8", "svg2_layer_norm_backward_workspace_size", "svg2_layer_norm_backward",
    "svg2_quantize_fp8_blocks", "svg2_dequantize_fp8_blocks", "svg2_matmul_fp8_blocks_workspace_size", "svg2_matmul_fp8_blocks",
    "svg2_profile_enable", "svg2_profile_read", "svg2_profile_read_kernels",
)
STAGES = ("kmeans", "permute", "select", "attn_plan", "attn")
KERNEL_CLASSES = ("kmeans_assign", "kmeans_settle", "kmeans_sort", "kmeans_segsum_full", "kmeans_segsum_delta",
                  "kmeans_finalize", "permute_sort", "permute_gather")


class Svg2Error(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__("svg2 error %d: %s" % (code, msg))
        self.code = code


class _ForwardAux(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in (
        "labels_q", "labels_k", "counts_q", "counts_k", "offsets_q", "offsets_k",
        "perm_q", "perm_k", "row_ptr", "col_idx", "density", "lse")]


ROPE_PAIRINGS = ("adjacent", "halves")
NORM_SCOPES = ("head", "token")


# svg2_rope_args, packed as the C compiler lays it out (a ctypes structure takes twice as long to fill)
_ROPE_ARGS = struct.Struct("@6i3P3P3i3P3q3qPqPi4iiif0q")


# svg2_layer_norm_args, likewise
_NORM_ARGS = struct.Struct("@5iPqqPPqqifPqq")


_P3, _I3, _I2 = ctypes.c_void_p * 3, ctypes.c_int64 * 3, ctypes.c_int64 * 2

_lib = None


def load_library() -> ctypes.CDLL:
    """Load the C-ABI library; raises if it has not been built (python -m paper_2505_18875_amd.build)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                "%s not found: build it with `python paper_2505_18875_amd/build.py` "
                "(there is no CPU fallback)" % LIB_PATH)
        lib = ctypes.CDLL(LIB_PATH)
        lib.svg2_last_error.restype = ctypes.c_char_p
        lib.svg2_version.restype = ctypes.c_int
        for n in EXPORTS:
            if n.endswith("_workspace_size"):
                getattr(lib, n).restype = ctypes.c_size_t
        vp, i, f, sz = ctypes.c_void_p, ctypes.c_int, ctypes.c_float, ctypes.c_size_t
        lib.svg2_kmeans_workspace_size.argtypes = [i, i, i, i, i]
        lib.svg2_kmeans.argtypes = [vp, i, i, i, i, i, i, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.svg2_permute_workspace_size.argtypes = [i, i, i]
        lib.svg2_permute.argtypes = [vp, i, i, i, vp, vp, vp, i, vp, vp, i, i, vp, sz, vp]
        lib.svg2_permute_noalloc.argtypes = [vp, i, i, i, vp, vp, vp, i, vp, vp, i, i, vp]
        lib.svg2_select_topp_workspace_size.argtypes = [i, i, i]
        lib.svg2_select_topp.argtypes = [vp, vp, vp, vp, i, i, i, i, f, vp, vp, vp, vp, vp, sz, vp]
        lib.svg2_sparse_attn_workspace_size.argtypes = [i, i, i, i, i, i]
        lib.svg2_sparse_attn.argtypes = [vp, vp, vp, i, i, i, i, i, i, vp, vp, vp, vp, vp, f, vp, vp, vp, sz, vp]
        lib.svg2_sparse_attn_gather_free.argtypes = [vp, vp, vp, i, i, i, i, i, i, vp, vp, vp, vp, vp, vp, f, vp, vp, vp,
                                                     sz, vp]
        lib.svg2_forward_workspace_size.argtypes = [i, i, i, i, i, i]
        lib.svg2_forward.argtypes = [vp, vp, vp, i, i, i, i, i, i, f, i, vp, vp, vp, vp, vp, sz, vp]
        lib.svg2_forward_gather_free_workspace_size.argtypes = [i, i, i, i, i, i]
        lib.svg2_forward_gather_free.argtypes = lib.svg2_forward.argtypes
        lib.svg2_quantize_fp8_workspace_size.argtypes = [i]
        lib.svg2_quantize_fp8.argtypes = [vp, i, i, i, i, vp, vp, vp, sz, vp]
        lib.svg2_sparse_attn_fp8.argtypes = [vp, vp, vp, vp, vp, vp, i, i, i, i, i, vp, vp, vp, vp, vp, vp, f, vp, vp,
                                             vp, sz, vp]
        lib.svg2_forward_fp8_workspace_size.argtypes = [i, i, i, i, i, i]
        lib.svg2_forward_fp8.argtypes = lib.svg2_forward.argtypes
        lib.svg2_attention_recall_workspace_size.argtypes = [i, i]
        lib.svg2_attention_recall.argtypes = [vp, vp, i, i, vp, vp, vp, sz, vp]
        lib.svg2_kmeans_pp_init_workspace_size.argtypes = [i, i, i]
        lib.svg2_kmeans_pp_init.argtypes = [vp, i, i, i, i, i, vp, vp, vp, vp, sz, vp]
        lib.svg2_rope.argtypes = [vp, vp]
        lib.svg2_rope_backward_workspace_size.argtypes = [vp]
        lib.svg2_rope_backward.argtypes = [vp, vp, vp, vp, vp, vp, sz, vp]
        i64 = ctypes.c_int64
        lib.svg2_quantize_mxfp4.argtypes = [vp, i, i, i, i, i64, i64, i, vp, vp, vp]
        lib.svg2_dequantize_mxfp4.argtypes = [vp, vp, i, i, i, vp, i64, vp]
        lib.svg2_matmul_mxfp4_workspace_size.argtypes = [i, i, i]
        lib.svg2_matmul_mxfp4.argtypes = [vp, vp, vp, vp, i, i, i, vp, i, vp, i64, vp, sz, vp]
        lib.svg2_layer_norm.argtypes = [vp, vp]
        lib.svg2_layer_norm_fp8.argtypes = [vp, vp, vp, vp]
        lib.svg2_layer_norm_backward_workspace_size.argtypes = [vp]
        lib.svg2_layer_norm_backward.argtypes = [vp, vp, vp, vp, vp, vp, vp, sz, vp]
        lib.svg2_quantize_fp8_blocks.argtypes = [vp, i, i, i, i, i64, i64, i, vp, vp, vp, vp, vp]
        lib.svg2_dequantize_fp8_blocks.argtypes = lib.svg2_dequantize_mxfp4.argtypes
        lib.svg2_matmul_fp8_blocks_workspace_size.argtypes = [i, i, i]
        lib.svg2_matmul_fp8_blocks.argtypes = lib.svg2_matmul_mxfp4.argtypes
        lib.svg2_profile_enable.argtypes = [i]
        lib.svg2_profile_read.argtypes = [vp, vp]
        lib.svg2_profile_read_kernels.argtypes = [vp, vp]
        _lib = lib
    return _lib


def _check(rc: int):
    if rc != SVG2_OK:
        raise Svg2Error(rc, load_library().svg2_last_error().decode())


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return SVG2_F32
    if t.dtype == torch.bfloat16:
        return SVG2_BF16
    raise TypeError("svg2 supports float32 and bfloat16 tensors, got %s" % t.dtype)


def _dev(t: Optional[torch.Tensor], dtype=None, name="tensor"):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("%s must live on the GPU" % name)
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    if dtype is not None and t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    return ctypes.c_void_p(t.data_ptr())


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _workspace(nbytes: int, device) -> torch.Tensor:
    return torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=device)


def svg2_kmeans(X, init_centroids, iters, *, centroids=None, want_objective=False, ws=None):
    """Section 4.1.  X [H,N,d]; init_centroids [H,C,d] fp32 -> centroids, labels, counts (, objective)."""
    lib = load_library()
    H, N, d = X.shape
    C = init_centroids.shape[1]
    dt = _dtype_code(X)
    dev = X.device
    centroids = torch.empty_like(init_centroids) if centroids is None else centroids
    labels = torch.empty((H, N), dtype=torch.int32, device=dev)
    counts = torch.empty((H, C), dtype=torch.int32, device=dev)
    objective = torch.empty((H, iters), dtype=torch.float32, device=dev) if want_objective else None
    need = lib.svg2_kmeans_workspace_size(dt, H, N, d, C)
    ws = _workspace(need, dev) if ws is None else ws
    _check(lib.svg2_kmeans(_dev(X, name="X"), dt, H, N, d, C, int(iters),
                           _dev(init_centroids, torch.float32, "init_centroids"),
                           _dev(centroids, torch.float32, "centroids"), _dev(labels), _dev(counts),
                           _dev(objective), _dev(ws), ws.numel(), _stream()))
    return SimpleNamespace(centroids=centroids, labels=labels, counts=counts, objective=objective)


def svg2_permute(labels, C, tensors=(), *, want_inverse=True, ws=None):
    """Section 4.1.  labels [H,N] int32 -> offsets, perm, inv_perm and the permuted copies of `tensors`."""
    lib = load_library()
    H, N = labels.shape
    dev = labels.device
    offsets = torch.empty((H, C + 1), dtype=torch.int32, device=dev)
    perm = torch.empty((H, N), dtype=torch.int32, device=dev)
    inv = torch.empty((H, N), dtype=torch.int32, device=dev) if want_inverse else None
    n = len(tensors)
    outs = [torch.empty_like(t) for t in tensors]
    dt, d = (SVG2_F32, 0)
    src = dst = None
    if n:
        dt, d = _dtype_code(tensors[0]), tensors[0].shape[-1]
        for t in tensors:
            if t.shape != (H, N, d) or _dtype_code(t) != dt:
                raise ValueError("tensors must all be [H,N,d] of one dtype")
            _dev(t, name="tensor")
        src = (ctypes.c_void_p * n)(*[t.data_ptr() for t in tensors])
        dst = (ctypes.c_void_p * n)(*[t.data_ptr() for t in outs])
    need = lib.svg2_permute_workspace_size(H, N, C)
    ws = _workspace(need, dev) if ws is None else ws
    _check(lib.svg2_permute(_dev(labels, torch.int32, "labels"), H, N, C, _dev(offsets), _dev(perm), _dev(inv),
                            n, src, dst, dt, d, _dev(ws), ws.numel(), _stream()))
    return SimpleNamespace(offsets=offsets, perm=perm, inv_perm=inv, tensors=outs)


def svg2_permute_noalloc(labels, C, offsets, perm, inv_perm=None, tensors=(), outs=()):
    """svg2_permute on the library's built-in scratch: every buffer is the caller's, nothing is allocated here
    or in the library.  labels [H,N] int32; offsets [H,C+1], perm [H,N], inv_perm [H,N] or None int32 outputs;
    outs[t] receives the permuted copy of tensors[t]."""
    lib = load_library()
    H, N = labels.shape
    n = len(tensors)
    if len(outs) != n:
        raise ValueError("one output per tensor")
    dt, d = (SVG2_F32, 0)
    src = dst = None
    if n:
        dt, d = _dtype_code(tensors[0]), tensors[0].shape[-1]
        for t, o in zip(tensors, outs):
            if t.shape != (H, N, d) or _dtype_code(t) != dt or o.shape != t.shape or o.dtype != t.dtype:
                raise ValueError("tensors and outs must all be [H,N,d] of one dtype")
            _dev(t, name="tensor")
            _dev(o, name="out")
        src = (ctypes.c_void_p * n)(*[t.data_ptr() for t in tensors])
        dst = (ctypes.c_void_p * n)(*[t.data_ptr() for t in outs])
    _check(lib.svg2_permute_noalloc(_dev(labels, torch.int32, "labels"), H, N, C, _dev(offsets, torch.int32, "offsets"),
                                    _dev(perm, torch.int32, "perm"), _dev(inv_perm, torch.int32, "inv_perm"),
                                    n, src, dst, dt, d, _stream()))


def svg2_select_topp(cq, ck, counts_q, counts_k, top_p, *, want_p_est=False, ws=None):
    """Section 4.2, Eq. 1-2 and the top-p rule -> CSR (row_ptr, col_idx), density (, p_est)."""
    lib = load_library()
    H, Cq, d = cq.shape
    Ck = ck.shape[1]
    dev = cq.device
    row_ptr = torch.empty((H, Cq + 1), dtype=torch.int32, device=dev)
    col_idx = torch.empty((H, Cq * Ck), dtype=torch.int32, device=dev)
    p_est = torch.empty((H, Cq, Ck), dtype=torch.float32, device=dev) if want_p_est else None
    density = torch.empty((H,), dtype=torch.float32, device=dev) if counts_q is not None else None
    need = lib.svg2_select_topp_workspace_size(H, Cq, Ck)
    ws = _workspace(need, dev) if ws is None else ws
    _check(lib.svg2_select_topp(_dev(cq, torch.float32, "cq"), _dev(ck, torch.float32, "ck"),
                                _dev(counts_q, torch.int32, "counts_q"), _dev(counts_k, torch.int32, "counts_k"),
                                H, Cq, Ck, d, float(top_p), _dev(row_ptr), _dev(col_idx), _dev(p_est),
                                _dev(density), _dev(ws), ws.numel(), _stream()))
    return SimpleNamespace(row_ptr=row_ptr, col_idx=col_idx, p_est=p_est, density=density)


def svg2_sparse_attn(Qp, Kp, Vp, offsets_q, offsets_k, row_ptr, col_idx, perm_q=None, *, scale=0.0,
                     want_lse=False, out=None, ws=None):
    """Section 4.3.  Permuted Q, K, V [H,N,d] + block list -> O [H,N,d] (original order if perm_q is given)."""
    lib = load_library()
    H, N, d = Qp.shape
    Cq, Ck = offsets_q.shape[1] - 1, offsets_k.shape[1] - 1
    dt = _dtype_code(Qp)
    dev = Qp.device
    if col_idx.numel() < H * Cq * Ck:
        raise ValueError("col_idx must have capacity H*Cq*Ck")
    O = torch.empty_like(Qp) if out is None else out
    lse = torch.empty((H, N), dtype=torch.float32, device=dev) if want_lse else None
    need = lib.svg2_sparse_attn_workspace_size(dt, H, N, d, Cq, Ck)
    ws = _workspace(need, dev) if ws is None else ws
    _check(lib.svg2_sparse_attn(_dev(Qp, name="Qp"), _dev(Kp, Qp.dtype, "Kp"), _dev(Vp, Qp.dtype, "Vp"), dt, H, N, d,
                                Cq, Ck, _dev(offsets_q, torch.int32, "offsets_q"),
                                _dev(offsets_k, torch.int32, "offsets_k"), _dev(row_ptr, torch.int32, "row_ptr"),
                                _dev(col_idx, torch.int32, "col_idx"), _dev(perm_q, torch.int32, "perm_q"),
                                float(scale), _dev(O, Qp.dtype, "O"), _dev(lse), _dev(ws), ws.numel(), _stream()))
    return SimpleNamespace(O=O, lse=lse)


def svg2_sparse_attn_gather_free(Q, K, V, offsets_q, offsets_k, row_ptr, col_idx, perm_q, perm_k, *, scale=0.0,
                                 want_lse=False, out=None, ws=None):
    """Section 4.3 with sparse loading: Q, K, V [H,N,d] in token order + both permutations + block list -> O."""
    lib = load_library()
    H, N, d = Q.shape
    Cq, Ck = offsets_q.shape[1] - 1, offsets_k.shape[1] - 1
    dt = _dtype_code(Q)
    dev = Q.device
    if col_idx.numel() < H * Cq * Ck:
        raise ValueError("col_idx must have capacity H*Cq*Ck")
    O = torch.empty_like(Q) if out is None else out
    lse = torch.empty((H, N), dtype=torch.float32, device=dev) if want_lse else None
    need = lib.svg2_sparse_attn_workspace_size(dt, H, N, d, Cq, Ck)
    ws = _workspace(need, dev) if ws is None else ws
    _check(lib.svg2_sparse_attn_gather_free(
        _dev(Q, name="Q"), _dev(K, Q.dtype, "K"), _dev(V, Q.dtype, "V"), dt, H, N, d, Cq, Ck,
        _dev(offsets_q, torch.int32, "offsets_q"), _dev(offsets_k, torch.int32, "offsets_k"),
        _dev(row_ptr, torch.int32, "row_ptr"), _dev(col_idx, torch.int32, "col_idx"),
        _dev(perm_q, torch.int32, "perm_q"), _dev(perm_k, torch.int32, "perm_k"), float(scale),
        _dev(O, Q.dtype, "O"), _dev(lse), _dev(ws), ws.numel(), _stream()))
    return SimpleNamespace(O=O, lse=lse)


def svg2_quantize_fp8(X, *, ws=None):
    """Table 1 (+ FP8): X [H,N,d] -> (X8 [H,N,d] uint8 E4M3 codes, scale [H] fp32), X ~ decode(X8) * scale[h]."""
    lib = load_library()
    H, N, d = X.shape
    dev = X.device
    X8 = torch.empty((H, N, d), dtype=torch.uint8, device=dev)
    scale = torch.empty((H,), dtype=torch.float32, device=dev)
    ws = _workspace(lib.svg2_quantize_fp8_workspace_size(H), dev) if ws is None else ws
    _check(lib.svg2_quantize_fp8(_dev(X, name="X"), _dtype_code(X), H, N, d, _dev(X8), _dev(scale), _dev(ws),
                                 ws.numel(), _stream()))
    return X8, scale


def svg2_sparse_attn_fp8(Q8, K8, V8, scale_q, scale_k, scale_v, offsets_q, offsets_k, row_ptr, col_idx,
                         perm_q=None, perm_k=None, *, scale=0.0, want_lse=False, out=None, ws=None):
    """Section 4.3 on E4M3 operands.  perm_k None: permuted copies; perm_k given: token order (gather-free)."""
    lib = load_library()
    H, N, d = Q8.shape
    Cq, Ck = offsets_q.shape[1] - 1, offsets_k.shape[1] - 1
    dev = Q8.device
    if col_idx.numel() < H * Cq * Ck:
        raise ValueError("col_idx must have capacity H*Cq*Ck")
    O = torch.empty((H, N, d), dtype=torch.bfloat16, device=dev) if out is None else out
    lse = torch.empty((H, N), dtype=torch.float32, device=dev) if want_lse else None
    need = lib.svg2_sparse_attn_workspace_size(SVG2_BF16, H, N, d, Cq, Ck)
    ws = _workspace(need, dev) if ws is None else ws
    _check(lib.svg2_sparse_attn_fp8(
        _dev(Q8, torch.uint8, "Q8"), _dev(K8, torch.uint8, "K8"), _dev(V8, torch.uint8, "V8"),
        _dev(scale_q, torch.float32, "scale_q"), _dev(scale_k, torch.float32, "scale_k"),
        _dev(scale_v, torch.float32, "scale_v"), H, N, d, Cq, Ck,
        _dev(offsets_q, torch.int32, "offsets_q"), _dev(offsets_k, torch.int32, "offsets_k"),
        _dev(row_ptr, torch.int32, "row_ptr"), _dev(col_idx, torch.int32, "col_idx"),
        _dev(perm_q, torch.int32, "perm_q"), _dev(perm_k, torch.int32, "perm_k"), float(scale),
        _dev(O, torch.bfloat16, "O"), _dev(lse), _dev(ws), ws.numel(), _stream()))
    return SimpleNamespace(O=O, lse=lse)


def svg2_forward_workspace_size(dtype_code, H, N, d, Cq, Ck, gather_free=False, fp8=False) -> int:
    lib = load_library()
    fn = (lib.svg2_forward_fp8_workspace_size if fp8 else
          lib.svg2_forward_gather_free_workspace_size if gather_free else lib.svg2_forward_workspace_size)
    return fn(dtype_code, H, N, d, Cq, Ck)


def svg2_forward_fp8(Q, K, V, cq_inout, ck_inout, top_p, iters, **kw):
    """svg2_forward with the attention step on E4M3 copies of Q, K, V (Table 1, + FP8)."""
    return svg2_forward(Q, K, V, cq_inout, ck_inout, top_p, iters, fp8=True, **kw)


def svg2_forward_gather_free(Q, K, V, cq_inout, ck_inout, top_p, iters, **kw):
    """svg2_forward without permuted copies of Q, K, V (Section 4.3, sparse loading)."""
    return svg2_forward(Q, K, V, cq_inout, ck_inout, top_p, iters, gather_free=True, **kw)


def svg2_forward(Q, K, V, cq_inout, ck_inout, top_p, iters, *, want_aux=False, out=None, ws=None,
                 gather_free=False, fp8=False):
    """Section 4, the whole layer.  cq_inout / ck_inout [H,C,d] fp32 are updated in place (centroid cache)."""
    lib = load_library()
    H, N, d = Q.shape
    Cq, Ck = cq_inout.shape[1], ck_inout.shape[1]
    dt = _dtype_code(Q)
    dev = Q.device
    O = torch.empty_like(Q) if out is None else out
    aux_t = None
    aux_p = None
    if want_aux:
        i32 = dict(dtype=torch.int32, device=dev)
        aux_t = SimpleNamespace(
            labels_q=torch.empty((H, N), **i32), labels_k=torch.empty((H, N), **i32),
            counts_q=torch.empty((H, Cq), **i32), counts_k=torch.empty((H, Ck), **i32),
            offsets_q=torch.empty((H, Cq + 1), **i32), offsets_k=torch.empty((H, Ck + 1), **i32),
            perm_q=torch.empty((H, N), **i32), perm_k=torch.empty((H, N), **i32),
            row_ptr=torch.empty((H, Cq + 1), **i32), col_idx=torch.empty((H, Cq * Ck), **i32),
            density=torch.empty((H,), dtype=torch.float32, device=dev),
            lse=torch.empty((H, N), dtype=torch.float32, device=dev))
        aux_s = _ForwardAux(**{n: getattr(aux_t, n).data_ptr() for n, _ in _ForwardAux._fields_})
        aux_p = ctypes.cast(ctypes.pointer(aux_s), ctypes.c_void_p)
    need = svg2_forward_workspace_size(dt, H, N, d, Cq, Ck, gather_free, fp8)
    ws = _workspace(need, dev) if ws is None else ws
    entry = lib.svg2_forward_fp8 if fp8 else lib.svg2_forward_gather_free if gather_free else lib.svg2_forward
    _check(entry(_dev(Q, name="Q"), _dev(K, Q.dtype, "K"), _dev(V, Q.dtype, "V"), dt, H, N, d, Cq, Ck,
                            float(top_p), int(iters), _dev(cq_inout, torch.float32, "cq_inout"),
                            _dev(ck_inout, torch.float32, "ck_inout"), _dev(O, Q.dtype, "O"), aux_p,
                            _dev(ws), ws.numel(), _stream()))
    return SimpleNamespace(O=O, aux=aux_t)


def svg2_attention_recall(lse_selected, lse_all, *, want_rows=True, ws=None):
    """Section 3.1.  lse of the selected keys and of all keys [H,N] fp32 -> recall per query (, mean per head)."""
    lib = load_library()
    H, N = lse_selected.shape
    dev = lse_selected.device
    rows = torch.empty((H, N), dtype=torch.float32, device=dev) if want_rows else None
    mean = torch.empty((H,), dtype=torch.float32, device=dev)
    need = lib.svg2_attention_recall_workspace_size(H, N)
    ws = _workspace(need, dev) if ws is None else ws
    _check(lib.svg2_attention_recall(_dev(lse_selected, torch.float32, "lse_selected"),
                                     _dev(lse_all, torch.float32, "lse_all"), H, N, _dev(rows), _dev(mean),
                                     _dev(ws), ws.numel(), _stream()))
    return SimpleNamespace(recall=rows, mean=mean)


def svg2_kmeans_pp_init(X, C, u, *, ws=None):
    """Sections 4.3 / 5.3: k-means++ seeding with the caller's uniform numbers u [H,C] fp64 -> centroids, picked."""
    lib = load_library()
    H, N, d = X.shape
    dev = X.device
    if u.shape != (H, C):
        raise ValueError("u must be [H,C]")
    centroids = torch.empty((H, C, d), dtype=torch.float32, device=dev)
    picked = torch.empty((H, C), dtype=torch.int32, device=dev)
    need = lib.svg2_kmeans_pp_init_workspace_size(H, N, C)
    ws = _workspace(need, dev) if ws is None else ws
    _check(lib.svg2_kmeans_pp_init(_dev(X, name="X"), _dtype_code(X), H, N, d, C, _dev(u, torch.float64, "u"),
                                   _dev(centroids), _dev(picked), _dev(ws), ws.numel(), _stream()))
    return SimpleNamespace(centroids=centroids, picked=picked)


# The calls below are short on the GPU where there are few tokens, so their checks are written to cost little: one condition per
# tensor, and what exactly is wrong is found out only then.

def _raw_stream(device: torch.device) -> int:
    return torch._C._cuda_getCurrentRawStream(device.index)


def _on(device: torch.device):
    """Context in which `device` is the current one."""
    return _HERE_ALREADY if torch._C._cuda_getDevice() == device.index else torch.cuda.device(device)


_HERE_ALREADY = contextlib.nullcontext()


def _gpu(t: torch.Tensor, name: str) -> torch.device:
    if not t.is_cuda:
        raise ValueError("%s must live on the GPU" % name)
    return t.device


def _refuse(t: torch.Tensor, name: str, device, dtype, shape):
    if t.device != device:
        raise ValueError("%s is on %s, not on %s" % (name, t.device, device))
    if t.dtype is not dtype:
        raise TypeError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if t.shape != shape:
        raise ValueError("%s must be %s, got %s" % (name, list(shape), list(t.shape)))
    raise ValueError("%s must be contiguous" % name)


def _dense(t: Optional[torch.Tensor], name: str, device, dtype, shape) -> int:
    """Address of a dense tensor; 0 for None."""
    if t is None:
        return 0
    if t.shape != shape or t.dtype is not dtype or t.device != device or not t.is_contiguous():
        _refuse(t, name, device, dtype, shape)
    return t.data_ptr()


def _outer_strides(shape, stride):
    """Strides of all but the last dimension, which has to be contiguous; 0 where a dimension has one entry (torch leaves anything
    there)."""
    if stride[-1] != 1 and shape[-1] > 1:
        raise ValueError("a tensor's last dimension must be contiguous")
    return [s if n > 1 else 0 for n, s in zip(shape[:-1], stride[:-1])]


def _three(xs):
    return xs if len(xs) == 3 else (*xs, 0, 0, 0)[:3]


def _views(tensors, name, device, dtype, own):
    """One to three tensors of shape `own` and one set of strides -> outer strides, addresses."""
    stride = tensors[0].stride()
    outer = _outer_strides(own, stride)
    ptrs = []
    for t in tensors:
        if t.shape != own or t.dtype is not dtype or t.device != device or (
                t.stride() != stride and _outer_strides(own, t.stride()) != outer):
            if t.shape == own and t.dtype is dtype and t.device == device:
                raise ValueError("%s must share one set of strides" % name)
            _refuse(t, name, device, dtype, own)
        ptrs.append(t.data_ptr())
    return outer, ptrs


def _token_views(tensors, name, device, dtype, shape=None):
    """One to three [N,H,d] or [B,N,H,d] tensors of one shape and one set of strides -> (B,N,H,d), the three outer strides,
    addresses."""
    own = tensors[0].shape
    full = tuple(own) if len(own) == 4 else (1, *own)
    if len(full) != 4:
        raise ValueError("%s must be [N,H,d] or [B,N,H,d]" % name)
    if shape is not None and full != shape:
        raise ValueError("%s must be %s, got %s" % (name, list(shape), list(own)))
    outer, ptrs = _views(tensors, name, device, dtype, own)
    return full, outer if len(own) == 4 else [0] + outer, ptrs


def _head_order(tensors, name, device, dtype, shape):
    """As _token_views for [B*H,N,d] tensors that stand for [B,N,H,d]; [B,N,H,d] tensors themselves are taken too."""
    B, N, H, d = shape
    if tensors[0].dim() != 3:
        return _token_views(tensors, name, device, dtype, shape)[1:]
    s, ptrs = _views(tensors, name, device, dtype, (B * H, N, d))
    return [H * s[0] if B > 1 else 0, s[1], s[0] if H > 1 else 0], ptrs


def svg2_grid_positions(grid, *, first=None, extra=0, device="cuda"):
    """Positions (time, height, width) of a video's tokens in raster order, int32 [T*Y*X + extra, 3], the grid starting at
    `first` (0 on every axis); `extra` tokens behind the video's (text) get position 0, which rotates nothing.  A grid of
    other axes (one to the rotary call's four) gives as many columns."""
    first = (0,) * len(grid) if first is None else first
    if len(first) < len(grid):
        raise ValueError("first has %d axes, the grid has %d" % (len(first), len(grid)))
    axes = [torch.arange(n, dtype=torch.int32, device=device) + f for n, f in zip(grid, first)]
    video = torch.stack([a.reshape(-1) for a in torch.meshgrid(*axes, indexing="ij")], 1)
    return torch.cat([video, video.new_zeros((extra, len(axes)))]).contiguous()


def svg2_rope_frequencies(axis_pairs, *, theta=10000.0, device="cuda"):
    """Frequencies of the usual rotary positions, fp64 [sum(axis_pairs)]: pair i of an axis of n pairs has theta^(-i/n)."""
    return torch.cat([torch.as_tensor(float(theta), dtype=torch.float64) ** (-torch.arange(n, dtype=torch.float64) / n)
                      for n in axis_pairs if n > 0]).to(device)


def _rope_args(n, dtype, device, shape, src, src_stride, dst, dst_stride, pos, freq, axis_pairs, rotate, norm_weights, norm_scope,
               eps, pairing):
    """svg2_rope_args, with every check that needs the tensors themselves; the norms' weights."""
    B, N, H, d = shape
    if pairing not in ROPE_PAIRINGS:
        raise ValueError("pairing must be one of %s" % (ROPE_PAIRINGS,))
    if norm_scope not in NORM_SCOPES:
        raise ValueError("norm_scope must be one of %s" % (NORM_SCOPES,))
    rotate = (True,) * n if rotate is None else rotate
    weights = (None,) * n if norm_weights is None else norm_weights
    if len(rotate) != n or len(weights) != n:
        raise ValueError("rotate and norm_weights need one entry per tensor")
    wshape = (d,) if norm_scope == "head" else (H, d)
    w = [0 if x is None else _dense(x, "norm_weights", device, torch.float32, wshape) for x in weights]
    pos_ptr = freq_ptr = pos_stride = 0
    axes = ()
    if any(rotate):
        if pos is None or freq is None:
            raise ValueError("pos and freq are needed where a tensor is rotated")
        axes = axis_pairs
        k = len(axes)
        if not 1 <= k <= 4:
            raise ValueError("axis_pairs must have 1 to 4 entries")
        have = pos.shape
        if have == (N, k):
            pos_ptr = _dense(pos, "pos", device, torch.int32, have)
        elif have == (B, N, k) or have == (1, N, k):
            pos_ptr = pos.data_ptr()
            _dense(pos[0], "pos", device, torch.int32, (N, k))
            pos_stride = pos.stride(0) if have[0] > 1 else 0
        else:
            raise ValueError("pos must be [N,%d] or [B,N,%d], got %s" % (k, k, list(have)))
        freq_ptr = _dense(freq, "freq", device, torch.float64, (d // 2,))
    r = [1 if x else 0 for x in rotate]
    return _ROPE_ARGS.pack(n, dtype, B, N, H, d, *_three(src), *_three(dst), *_three(r), *_three(w), *src_stride, *dst_stride, pos_ptr,
                           pos_stride, freq_ptr, len(axes), *(*axes, 0, 0, 0, 0)[:4], ROPE_PAIRINGS.index(pairing),
                           NORM_SCOPES.index(norm_scope), eps), weights


def svg2_rope(tensors, pos=None, freq=None, *, axis_pairs=(), rotate=None, norm_weights=None, norm_scope="head", eps=1e-6,
              pairing="adjacent", outs=None):
    """RMS norm, rotary positions over several axes and the move to head order of up to three tensors (Q, K, V).

    tensors: [N,H,d] or [B,N,H,d] views of one shape and set of strides (slices of a packed projection); pos int32
    [N,axes] or [B,N,axes]; freq fp64 [d/2]; axis_pairs: pairs of each axis; rotate: per tensor, default all;
    norm_weights: per tensor fp32 [d] (norm_scope "head") or [H,d] ("token"), or None.  Returns [B*H,N,d] tensors, or
    `outs` ([N,H,d] or [B,N,H,d] views of any strides; `tensors` themselves for a call in place)."""
    lib = load_library()
    n = len(tensors)
    if not 1 <= n <= 3:
        raise ValueError("one to three tensors")
    first = tensors[0]
    dtype, dev = first.dtype, _gpu(first, "tensors")
    shape, src_stride, src = _token_views(tensors, "tensors", dev, dtype)
    B, N, H, d = shape
    if outs is None:
        outs = [first.new_empty((B * H, N, d)) for _ in range(n)]
        dst_stride, dst = (H * N * d, d, N * d), [t.data_ptr() for t in outs]
    else:
        if len(outs) != n:
            raise ValueError("one output per tensor")
        _, dst_stride, dst = _token_views(outs, "outs", dev, dtype, shape)
    a, _ = _rope_args(n, _dtype_code(first), dev, shape, src, src_stride, dst, dst_stride, pos, freq, axis_pairs, rotate, norm_weights,
                      norm_scope, eps, pairing)
    with _on(dev):
        _check(lib.svg2_rope(a, _raw_stream(dev)))
    return outs


def svg2_rope_backward(grads, tensors, pos=None, freq=None, *, axis_pairs=(), rotate=None, norm_weights=None,
                       norm_scope="head", eps=1e-6, pairing="adjacent", outs=None, ws=None):
    """Gradients of svg2_rope: grads ([B*H,N,d], or [B,N,H,d] views of one set of strides) and the forward call's arguments
    -> grads of `tensors` (dense [B,N,H,d], or `outs`, views of any strides) and of norm_weights (None where None)."""
    lib = load_library()
    n = len(tensors)
    if not 1 <= n <= 3:
        raise ValueError("one to three tensors")
    first = tensors[0]
    dtype, dev = first.dtype, _gpu(first, "tensors")
    shape, src_stride, src = _token_views(tensors, "tensors", dev, dtype)
    if outs is None:
        outs = [first.new_empty(shape) for _ in range(n)]
    if len(grads) != n or len(outs) != n:
        raise ValueError("one gradient and one output per tensor")
    g_stride, g = _head_order(grads, "grads", dev, dtype, shape)
    _, dx_stride, dx = _token_views(outs, "outs", dev, dtype, shape)
    # the C entry takes the gradients' layout as that of the forward's results; they are only read
    a, weights = _rope_args(n, _dtype_code(first), dev, shape, src, src_stride, (), g_stride, pos, freq, axis_pairs, rotate,
                            norm_weights, norm_scope, eps, pairing)
    dw = [None if w is None else torch.empty_like(w) for w in weights]
    with _on(dev):
        ws = _workspace(lib.svg2_rope_backward_workspace_size(a), dev) if ws is None else ws
        _check(lib.svg2_rope_backward(a, _P3(*g), _P3(*dx), _I3(*dx_stride),
                                      _P3(*[None if t is None else t.data_ptr() for t in dw]), _dev(ws), ws.numel(), _raw_stream(dev)))
    return SimpleNamespace(grads=outs, dweights=dw)


def _mxfp4_operand(codes, scales, name, device):
    """Checks an operand's two tensors; rows and padded columns."""
    shape = codes.shape
    if len(shape) != 2 or shape[1] % 64:
        raise ValueError("%s: codes must be [R, Kp/2] with Kp a multiple of 128, got %s" % (name, list(shape)))
    R, half = shape
    return R, 2 * half, _dense(codes, name, device, torch.uint8, shape), _dense(scales, name, device, torch.uint8, (half // 64, R, 4))


def _rows(t, name, device, shape):
    """Address and row stride of a matrix whose rows are contiguous."""
    if t.shape != shape or t.device != device:
        _refuse(t, name, device, t.dtype, shape)
    stride = t.stride()
    if stride[1] != 1 and shape[1] > 1:
        raise ValueError("%s must be contiguous in its last dimension" % name)
    return t.data_ptr(), stride[0] if shape[0] > 1 else shape[1]


def svg2_quantize_mxfp4(X, *, transposed=False):
    """X [M,K], or [M,G,Kg] for K = G*Kg columns in groups of any stride (the layer's O as O.transpose(0, 1)) -> MXFP4
    operand (codes [M,Kp/2], scales [Kp/128,M,4] uint8); transposed: of X^T, [K rows, M columns]."""
    lib = load_library()
    dev, shape = _gpu(X, "X"), X.shape
    strides = _outer_strides(shape, X.stride())
    if len(shape) == 2:
        (M, K), G, (sm,), sg = shape, 1, strides, 0
        Kg = K
    elif len(shape) == 3:
        (M, G, Kg), (sm, sg) = shape, strides
        K = G * Kg
    else:
        raise ValueError("X must be [M,K] or [M,G,Kg]")
    R, nk = (K, -(-M // 128)) if transposed else (M, -(-K // 128))
    codes = torch.empty((R, nk * 64), dtype=torch.uint8, device=dev)
    scales = codes.new_empty((nk, R, 4))
    with _on(dev):
        _check(lib.svg2_quantize_mxfp4(X.data_ptr(), _dtype_code(X), M, G, Kg, sm, sg, 1 if transposed else 0, codes.data_ptr(),
                                       scales.data_ptr(), _raw_stream(dev)))
    return codes, scales


def svg2_dequantize_mxfp4(codes, scales, K=None, *, dtype=torch.bfloat16, out=None):
    """The values of an MXFP4 operand, [R,K] (K: all padded columns where None)."""
    lib = load_library()
    dev = _gpu(codes, "codes")
    R, Kp, c, s = _mxfp4_operand(codes, scales, "operand", dev)
    K = Kp if K is None else K
    if not Kp - 128 < K <= Kp:
        raise ValueError("K = %d does not belong to %d padded columns" % (K, Kp))
    out = torch.empty((R, K), dtype=dtype, device=dev) if out is None else out
    ptr, ld = _rows(out, "out", dev, (R, K))
    with _on(dev):
        _check(lib.svg2_dequantize_mxfp4(c, s, R, K, _dtype_code(out), ptr, ld, _raw_stream(dev)))
    return out


@functools.lru_cache(maxsize=4096)
def _matmul_workspace_size(M, N, K):
    return load_library().svg2_matmul_mxfp4_workspace_size(M, N, K)


def svg2_matmul_mxfp4(A, A_scales, B, B_scales, *, bias=None, out_dtype=torch.bfloat16, out=None, ws=None):
    """C [M,N] = A B^T + bias of two MXFP4 operands (M and N rows of the same columns); bias fp32 [N]."""
    lib = load_library()
    dev = _gpu(A, "A")
    M, Kp, a, sa = _mxfp4_operand(A, A_scales, "A", dev)
    N, Kb, b, sb = _mxfp4_operand(B, B_scales, "B", dev)
    if Kb != Kp:
        raise ValueError("A has %d padded columns, B has %d" % (Kp, Kb))
    C = torch.empty((M, N), dtype=out_dtype, device=dev) if out is None else out
    ptr, ld = _rows(C, "out", dev, (M, N))
    if ws is None:
        need = _matmul_workspace_size(M, N, Kp)
        if need > 256:                  # at 256 the product uses none
            ws = _workspace(need, dev)
    with _on(dev):
        _check(lib.svg2_matmul_mxfp4(a, sa, b, sb, M, N, Kp, _dense(bias, "bias", dev, torch.float32, (N,)), _dtype_code(C), ptr, ld,
                                     _dev(ws), 0 if ws is None else ws.numel(), _raw_stream(dev)))
    return C


def _norm_args(x, weight, bias, eps, one_plus, y_dtype, y, y_stride, dev):
    """svg2_layer_norm_args of x [N,D] or [B,N,D], with every check that needs the tensors; groups, rows and columns."""
    shape = x.shape
    if len(shape) == 3:
        B, N, D = shape
        xs = _outer_strides(shape, x.stride())
    elif len(shape) == 2:
        (N, D), B = shape, 1
        xs = [0, *_outer_strides(shape, x.stride())]
    else:
        raise ValueError("x must be [N,D] or [B,N,D], got %s" % list(shape))
    w, ws = _per_group(weight, "weight", dev, B, D)
    b, bs = _per_group(bias, "bias", dev, B, D)
    return _NORM_ARGS.pack(_dtype_code(x), y_dtype, B, N, D, x.data_ptr(), *xs, w, b, ws, bs, 1 if one_plus else 0, eps, y,
                           *y_stride), B, N, D


def _per_group(t, name, dev, B, D):
    """Address and group stride of fp32 [D], or [B,D] of any row stride; 0, 0 for None."""
    if t is None:
        return 0, 0
    shape = t.shape
    if (shape != (D,) and shape != (B, D)) or t.dtype is not torch.float32 or t.device != dev:
        _refuse(t, name, dev, torch.float32, (B, D) if len(shape) == 2 else (D,))
    stride = t.stride()
    if stride[-1] != 1 and D > 1:
        raise ValueError("%s must be contiguous in its last dimension" % name)
    return t.data_ptr(), stride[0] if len(shape) == 2 and B > 1 else 0


def _norm_out(t, name, dev, dtype, shape):
    """Address and (group, row) strides of a [N,D] or [B,N,D] result or gradient."""
    if t.shape != shape or t.device != dev or (dtype is not None and t.dtype is not dtype):
        _refuse(t, name, dev, t.dtype if dtype is None else dtype, shape)
    outer = _outer_strides(shape, t.stride())
    return t.data_ptr(), outer if len(shape) == 3 else [0, *outer]


def _dense_like(x, dtype):
    """A dense tensor of x's shape, its address and (group, row) strides; one of fewer than two dimensions is refused with x."""
    t = torch.empty_like(x) if dtype is x.dtype and x.is_contiguous() else torch.empty(x.shape, dtype=dtype, device=x.device)
    stride = t.stride()
    return t, t.data_ptr(), stride[:2] if len(stride) == 3 else (0, *stride[:1])


def svg2_layer_norm(x, weight=None, bias=None, *, eps=1e-6, one_plus=False, out_dtype=None, out=None):
    """(x - mean) / sqrt(variance + eps) * s + bias over the last dimension, s = weight, or 1 + weight with one_plus.

    x: [N,D] or [B,N,D], any strides; weight, bias: fp32 [D] for all rows, [B,D] for each group (rows of a wider table of
    modulations), or None.  The result has x's type, or out_dtype, or goes to `out` (any strides; x itself)."""
    lib = load_library()
    dev, shape = _gpu(x, "x"), x.shape
    if out is None:
        out, y, ys = _dense_like(x, x.dtype if out_dtype is None else out_dtype)
    else:
        y, ys = _norm_out(out, "out", dev, out_dtype, shape)
    a = _norm_args(x, weight, bias, eps, one_plus, _dtype_code(out), y, ys, dev)[0]
    with _on(dev):
        _check(lib.svg2_layer_norm(a, _raw_stream(dev)))
    return out


def svg2_layer_norm_fp8(x, weight=None, bias=None, *, eps=1e-6, one_plus=False):
    """svg2_layer_norm's result as an operand of svg2_matmul_fp8_blocks (codes, scales), row b*N + n of x [B,N,D]."""
    lib = load_library()
    dev = _gpu(x, "x")
    a, B, N, D = _norm_args(x, weight, bias, eps, one_plus, 0, 0, (0, 0), dev)
    codes, scales = _fp8_blocks_empty(B * N, D, dev)
    with _on(dev):
        _check(lib.svg2_layer_norm_fp8(a, codes.data_ptr(), scales.data_ptr(), _raw_stream(dev)))
    return codes, scales


def svg2_layer_norm_backward(grad, x, weight=None, bias=None, *, eps=1e-6, one_plus=False, out=None, ws=None):
    """Gradients of svg2_layer_norm: grad (x's shape, any strides) and the forward call's arguments -> grad of x (dense, or
    `out`), dweight and dbias (fp32 [D] or [B,D], None where the argument is None)."""
    lib = load_library()
    dev, shape = _gpu(x, "x"), x.shape
    g, gs = _norm_out(grad, "grad", dev, None, shape)
    if out is None:
        out, dx, ds = _dense_like(x, x.dtype)
    else:
        dx, ds = _norm_out(out, "out", dev, x.dtype, shape)
    a, B, N, D = _norm_args(x, weight, bias, eps, one_plus, _dtype_code(grad), 0, gs, dev)
    for t in (weight, bias):
        if t is not None and B > 1 and t.dim() == 2 and t.stride(0) == 0:
            raise ValueError("weight and bias of a group each must be rows of their own: expanded rows are shared ones, [D]")
    dw, db = [None if t is None else torch.empty_like(t) if t.is_contiguous() else torch.empty(t.shape, dtype=torch.float32, device=dev)
              for t in (weight, bias)]
    with _on(dev):
        if ws is None:
            need = lib.svg2_layer_norm_backward_workspace_size(a)
            if need > 256:              # at 256 the call uses none
                ws = _workspace(need, dev)
        _check(lib.svg2_layer_norm_backward(a, g, dx, _I2(*ds), None if dw is None else dw.data_ptr(), None if db is None else db.data_ptr(),
                                            _dev(ws), 0 if ws is None else ws.numel(), _raw_stream(dev)))
    return SimpleNamespace(grad=out, dweight=dw, dbias=db)


def _fp8_blocks_empty(R, K, device):
    nk = -(-K // 128)
    codes = torch.empty((R, nk * 128), dtype=torch.uint8, device=device)
    return codes, codes.new_empty((-(-nk // 4), R, 4))


def _fp8_blocks_operand(codes, scales, name, device):
    """Checks an operand's two tensors; rows and padded columns."""
    shape = codes.shape
    if len(shape) != 2 or shape[1] % 128:
        raise ValueError("%s: codes must be [R, Kp] with Kp a multiple of 128, got %s" % (name, list(shape)))
    R, Kp = shape
    return R, Kp, _dense(codes, name, device, torch.uint8, shape), _dense(scales, name, device, torch.uint8, (-(-Kp // 512), R, 4))


def svg2_quantize_fp8_blocks(X, *, transposed=False, square=False):
    """X [M,K], or [M,G,Kg] for K = G*Kg columns in groups of any stride (the layer's O as O.transpose(0, 1)) -> E4M3 operand
    with a power of two for each block of 128 columns: codes [M,Kp], scales [ceil(Kp/512),M,4] uint8.  transposed: of X^T, [K
    rows, M columns]; transposed="both": ((codes, scales), (codes, scales)) of X and of X^T from one read.  square: one scale for
    128 x 128 values."""
    lib = load_library()
    dev, shape = _gpu(X, "X"), X.shape
    strides = _outer_strides(shape, X.stride())
    if len(shape) == 2:
        (M, K), G, (sm,), sg = shape, 1, strides, 0
        Kg = K
    elif len(shape) == 3:
        (M, G, Kg), (sm, sg) = shape, strides
        K = G * Kg
    else:
        raise ValueError("X must be [M,K] or [M,G,Kg]")
    if transposed not in (False, True, "both"):
        raise ValueError("transposed must be False, True or \"both\"")
    codes, scales = (None, None) if transposed is True else _fp8_blocks_empty(M, K, dev)
    codes_t, scales_t = _fp8_blocks_empty(K, M, dev) if transposed else (None, None)
    with _on(dev):
        _check(lib.svg2_quantize_fp8_blocks(X.data_ptr(), _dtype_code(X), M, G, Kg, sm, sg, 1 if square else 0,
                                            *[None if t is None else t.data_ptr() for t in (codes, scales, codes_t, scales_t)],
                                            _raw_stream(dev)))
    return (codes, scales) if not transposed else (codes_t, scales_t) if transposed is True else ((codes, scales), (codes_t, scales_t))


def svg2_dequantize_fp8_blocks(codes, scales, K=None, *, dtype=torch.bfloat16, out=None):
    """The values of such an operand, [R,K] (K: all padded columns where None)."""
    lib = load_library()
    dev = _gpu(codes, "codes")
    R, Kp, c, s = _fp8_blocks_operand(codes, scales, "operand", dev)
    K = Kp if K is None else K
    if not Kp - 128 < K <= Kp:
        raise ValueError("K = %d does not belong to %d padded columns" % (K, Kp))
    out = torch.empty((R, K), dtype=dtype, device=dev) if out is None else out
    ptr, ld = _rows(out, "out", dev, (R, K))
    with _on(dev):
        _check(lib.svg2_dequantize_fp8_blocks(c, s, R, K, _dtype_code(out), ptr, ld, _raw_stream(dev)))
    return out


@functools.lru_cache(maxsize=4096)
def _fp8_blocks_workspace_size(M, N, K):
    return load_library().svg2_matmul_fp8_blocks_workspace_size(M, N, K)


def svg2_matmul_fp8_blocks(A, A_scales, B, B_scales, *, bias=None, out_dtype=torch.bfloat16, out=None, ws=None):
    """C [M,N] = A B^T + bias of two such operands (M and N rows of the same columns); bias fp32 [N]."""
    lib = load_library()
    dev = _gpu(A, "A")
    M, Kp, a, sa = _fp8_blocks_operand(A, A_scales, "A", dev)
    N, Kb, b, sb = _fp8_blocks_operand(B, B_scales, "B", dev)
    if Kb != Kp:
        raise ValueError("A has %d padded columns, B has %d" % (Kp, Kb))
    C = torch.empty((M, N), dtype=out_dtype, device=dev) if out is None else out
    ptr, ld = _rows(C, "out", dev, (M, N))
    if ws is None:
        need = _fp8_blocks_workspace_size(M, N, Kp)
        if need > 256:                  # at 256 the product uses none
            ws = _workspace(need, dev)
    with _on(dev):
        _check(lib.svg2_matmul_fp8_blocks(a, sa, b, sb, M, N, Kp, _dense(bias, "bias", dev, torch.float32, (N,)), _dtype_code(C), ptr,
                                          ld, _dev(ws), 0 if ws is None else ws.numel(), _raw_stream(dev)))
    return C


def svg2_profile_enable(level) -> None:
    """0 / False: stop; 1 / True: record HIP events around the stages of svg2_forward; 2: also around every
    kernel launch of k-means and the permutation."""
    _check(load_library().svg2_profile_enable(int(level)))


def svg2_profile_read():
    """(dict stage -> summed milliseconds, number of recorded svg2_forward calls); clears the record."""
    ms = (ctypes.c_float * len(STAGES))()
    n = ctypes.c_int(0)
    _check(load_library().svg2_profile_read(ctypes.cast(ms, ctypes.c_void_p), ctypes.cast(ctypes.pointer(n), ctypes.c_void_p)))
    return {k: float(v) for k, v in zip(STAGES, ms)}, n.value


def svg2_profile_read_kernels():
    """dict kernel class -> (summed milliseconds, launches) of the spans recorded at profile level 2; clears them."""
    n = len(KERNEL_CLASSES)
    ms = (ctypes.c_float * n)()
    cnt = (ctypes.c_int * n)()
    _check(load_library().svg2_profile_read_kernels(ctypes.cast(ms, ctypes.c_void_p), ctypes.cast(cnt, ctypes.c_void_p)))
    return {k: (float(m), int(c)) for k, m, c in zip(KERNEL_CLASSES, ms, cnt)}
