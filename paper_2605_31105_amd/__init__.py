"""MI355X (gfx950) GRKV prefill-compression path: Python binding.

Argument marshalling only.  Every step of the computation runs in the HIP
kernels of ``libgrkv.so`` behind the C ABI declared in ``include/grkv.h``;
PyTorch supplies device memory and the stream.  Importing works without a GPU;
calling ``compress`` requires the built library and a ROCm device, and raises
if either is missing (there is no CPU fallback).
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

__all__ = [
    "GRKV_OK", "GRKV_ERR_INVALID", "GRKV_ERR_WORKSPACE", "GRKV_ERR_UNSUPPORTED",
    "GRKV_ERR_HIP", "GrkvError", "lib", "lib_path", "Problem", "Options", "Outputs",
    "Layout", "workspace_bytes", "workspace_layout", "compress", "Result",
    "intermediates", "EXPORTED_SYMBOLS", "KeyOptions", "workspace_bytes_kv", "compress_kv",
    "KEY_CONVERGED", "KEY_MAX_ITER", "KEY_SKIPPED", "KEY_BREAKDOWN", "carrier_stats",
    "CARRIER_METRICS", "compress_ragged", "pyramid_budgets", "adaptive_budgets",
    "workspace_bytes_ragged", "compress_noalloc", "NOALLOC_SCRATCH_BYTES", "h2o_scores",
    "compress_scored", "h2o_workspace_bytes", "Pages", "new_pages", "pages_init", "pages_append",
    "pages_fork", "pages_compact", "pages_free", "pages_workspace_bytes", "PAGES_OK", "PAGES_FULL",
    "PAGES_LENGTH", "PAGES_UNIT", "PAGES_RANGE", "tree_attention", "sink_attention",
    "tree_attention_workspace_bytes", "sink_attention_workspace_bytes", "Step", "pages_extend",
    "pages_extend_workspace_bytes", "rotary", "rotary_freqs", "NO_POSITION", "pages_store",
    "chunk_attention", "chunk_attention_workspace_bytes",
]

GRKV_OK, GRKV_ERR_INVALID, GRKV_ERR_WORKSPACE, GRKV_ERR_UNSUPPORTED, GRKV_ERR_HIP = 0, -1, -2, -3, -4
GRKV_BF16, GRKV_F32 = 0, 1
STAGES = ("full_lse", "full_lse_combine", "full_prob", "full_y", "select", "gather",
          "ret_lse", "ret_lse_combine", "ret_prob", "resid", "gram", "solve", "update", "key")
NUM_STAGES = len(STAGES)
EXPORTED_SYMBOLS = ("grkv_compress", "grkv_workspace_bytes", "grkv_workspace_layout",
                    "grkv_default_options", "grkv_status_string", "grkv_compress_kv",
                    "grkv_workspace_bytes_kv", "grkv_default_key_options", "grkv_carrier_stats",
                    "grkv_compress_ragged", "grkv_workspace_bytes_ragged", "grkv_pyramid_budgets",
                    "grkv_adaptive_budgets", "grkv_compress_noalloc", "grkv_h2o_scores",
                    "grkv_h2o_workspace_bytes", "grkv_compress_scored", "grkv_pages_init",
                    "grkv_pages_append", "grkv_pages_fork", "grkv_pages_compact",
                    "grkv_pages_free", "grkv_pages_workspace_bytes", "grkv_tree_attention",
                    "grkv_tree_attention_workspace_bytes", "grkv_sink_attention",
                    "grkv_sink_attention_workspace_bytes", "grkv_pages_extend",
                    "grkv_pages_extend_workspace_bytes", "grkv_rotary", "grkv_rotary_freqs",
                    "grkv_pages_store", "grkv_chunk_attention",
                    "grkv_chunk_attention_workspace_bytes")
NOALLOC_SCRATCH_BYTES = 64 << 20
KEY_CONVERGED, KEY_MAX_ITER, KEY_SKIPPED, KEY_BREAKDOWN = 1, 2, 3, 4
PAGES_OK, PAGES_FULL, PAGES_LENGTH, PAGES_UNIT, PAGES_RANGE = 0, 1, 2, 3, 4
NO_POSITION = -(1 << 31)
ROTARY_METHODS = ("plain", "linear", "base", "parts")
CARRIER_METRICS = ("b", "b_eff", "a_max", "gini", "boundary_fraction", "boundary_share",
                   "enrichment", "boundary_interior_load")

_PKG = os.path.dirname(os.path.abspath(__file__))


def lib_path() -> str:
    return os.path.join(_PKG, "libgrkv.so")


class GrkvError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__("grkv status %d: %s" % (status, msg))
        self.status = status


class Problem(ctypes.Structure):
    _fields_ = [("units", ctypes.c_int32), ("group", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class Options(ctypes.Structure):
    _fields_ = [("n_sink", ctypes.c_int32), ("beta", ctypes.c_float),
                ("fix_window", ctypes.c_int32), ("causal_window", ctypes.c_int32)]


class Outputs(ctypes.Structure):
    _fields_ = [("idx", ctypes.c_void_p), ("k_out", ctypes.c_void_p),
                ("v_out", ctypes.c_void_p), ("stats", ctypes.c_void_p),
                ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t),
                ("stage_events", ctypes.POINTER(ctypes.c_void_p))]


class KeyOptions(ctypes.Structure):
    _fields_ = [("lambda_k", ctypes.c_float), ("max_iter", ctypes.c_int32), ("tol", ctypes.c_float),
                ("steps", ctypes.c_int32)]


class Layout(ctypes.Structure):
    _fields_ = [(f, ctypes.c_size_t) for f in
                ("lse", "y", "score", "pooled", "fixed", "resid", "gram", "z", "total")]


class _PagesC(ctypes.Structure):
    _fields_ = [(f, ctypes.c_void_p) for f in ("k", "v", "table", "lens", "refs", "free_bits")] + [
        (f, ctypes.c_int32) for f in ("pages", "page_size", "units", "max_pages", "head_dim", "dtype")]


class _PageEntries(ctypes.Structure):
    _fields_ = [("entries", ctypes.c_int32), ("units", ctypes.c_void_p), ("rows", ctypes.c_int32),
                ("counts", ctypes.c_void_p), ("starts", ctypes.c_void_p),
                ("source_rows", ctypes.c_int64), ("status", ctypes.c_void_p)]


class _Tree(ctypes.Structure):
    _fields_ = [("entries", ctypes.c_int32), ("group", ctypes.c_int32), ("tokens", ctypes.c_int32),
                ("units", ctypes.c_void_p), ("counts", ctypes.c_void_p), ("parents", ctypes.c_void_p),
                ("trees", ctypes.c_int32), ("window", ctypes.c_int32), ("n_sink", ctypes.c_int32)]


class _StepC(ctypes.Structure):
    _fields_ = [("sequences", ctypes.c_int32), ("heads", ctypes.c_int32), ("units", ctypes.c_void_p),
                ("unit_stride", ctypes.c_int64), ("tokens", ctypes.c_int32)]


class _Rotation(ctypes.Structure):
    _fields_ = [("freqs", ctypes.c_void_p), ("dims", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("inverse", ctypes.c_int32), ("scale", ctypes.c_float)]


class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("token_stride", ctypes.c_int64),
                ("head_stride", ctypes.c_int64)]


class _Chunk(ctypes.Structure):
    _fields_ = [("group", ctypes.c_int32), ("longest", ctypes.c_int32), ("window", ctypes.c_int32),
                ("n_sink", ctypes.c_int32)]


_LIB = None


def lib() -> ctypes.CDLL:
    """Load libgrkv.so (once).  Raises if it has not been built."""
    global _LIB
    if _LIB is None:
        path = lib_path()
        if not os.path.exists(path):
            raise RuntimeError("libgrkv.so is not built: run `python -m paper_2605_31105_amd.build`")
        L = ctypes.CDLL(path)
        P = ctypes.POINTER
        L.grkv_compress.restype = ctypes.c_int
        L.grkv_compress.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                    ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                                    ctypes.c_int32, ctypes.c_float, ctypes.c_void_p,
                                    P(Problem), P(Options), P(Outputs)]
        L.grkv_compress_noalloc.restype = ctypes.c_int
        L.grkv_compress_noalloc.argtypes = L.grkv_compress.argtypes
        L.grkv_compress_scored.restype = ctypes.c_int
        L.grkv_compress_scored.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                           ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                                           ctypes.c_int32, ctypes.c_float, ctypes.c_void_p,
                                           P(Problem), P(Options), ctypes.c_void_p, P(Outputs)]
        L.grkv_h2o_scores.restype = ctypes.c_int
        L.grkv_h2o_scores.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int64,
                                      ctypes.c_int32, ctypes.c_void_p, P(Problem), ctypes.c_void_p,
                                      ctypes.c_void_p, ctypes.c_size_t]
        L.grkv_h2o_workspace_bytes.restype = ctypes.c_size_t
        L.grkv_h2o_workspace_bytes.argtypes = [P(Problem), ctypes.c_int64]
        L.grkv_workspace_bytes.restype = ctypes.c_size_t
        L.grkv_workspace_bytes.argtypes = [P(Problem), ctypes.c_int64, ctypes.c_int32, ctypes.c_int32]
        L.grkv_workspace_layout.restype = ctypes.c_int
        L.grkv_workspace_layout.argtypes = [P(Problem), ctypes.c_int64, ctypes.c_int32,
                                            ctypes.c_int32, P(Layout)]
        L.grkv_default_options.restype = None
        L.grkv_default_options.argtypes = [P(Options)]
        L.grkv_compress_kv.restype = ctypes.c_int
        L.grkv_compress_kv.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                       ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                                       ctypes.c_int32, ctypes.c_float, ctypes.c_void_p,
                                       P(Problem), P(Options), P(Outputs), P(KeyOptions),
                                       ctypes.c_void_p, ctypes.c_void_p]
        L.grkv_workspace_bytes_kv.restype = ctypes.c_size_t
        L.grkv_workspace_bytes_kv.argtypes = [P(Problem), ctypes.c_int64, ctypes.c_int32,
                                              ctypes.c_int32, ctypes.c_int32]
        L.grkv_default_key_options.restype = None
        L.grkv_default_key_options.argtypes = [P(KeyOptions), ctypes.c_float]
        L.grkv_carrier_stats.restype = ctypes.c_int
        L.grkv_carrier_stats.argtypes = [ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32,
                                         P(Problem), ctypes.c_void_p, ctypes.c_void_p,
                                         ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                         ctypes.c_void_p, ctypes.c_void_p]
        L.grkv_compress_ragged.restype = ctypes.c_int
        L.grkv_compress_ragged.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
                                           ctypes.c_int64, ctypes.c_int32, ctypes.c_void_p,
                                           ctypes.c_int32, ctypes.c_float, ctypes.c_void_p,
                                           P(Problem), P(Options), P(Outputs)]
        L.grkv_workspace_bytes_ragged.restype = ctypes.c_size_t
        L.grkv_workspace_bytes_ragged.argtypes = [P(Problem), ctypes.c_int64, ctypes.c_int32,
                                                  ctypes.c_void_p]
        L.grkv_pyramid_budgets.restype = ctypes.c_int
        L.grkv_pyramid_budgets.argtypes = [ctypes.c_int32, ctypes.c_int32, ctypes.c_int32,
                                           ctypes.c_int32, ctypes.c_int64, ctypes.c_float,
                                           ctypes.c_void_p]
        L.grkv_adaptive_budgets.restype = ctypes.c_int
        L.grkv_adaptive_budgets.argtypes = [ctypes.c_void_p, ctypes.c_int32, ctypes.c_int32,
                                            ctypes.c_int64, ctypes.c_int32, ctypes.c_int32,
                                            ctypes.c_void_p, ctypes.c_void_p]
        vp, i32, sz = ctypes.c_void_p, ctypes.c_int32, ctypes.c_size_t
        pg, en = P(_PagesC), P(_PageEntries)
        for name, args in (("init", [pg, vp]),
                           ("append", [pg, en, vp, i32, vp, i32, vp, vp, sz]),
                           ("fork", [pg, en, vp, vp, vp, sz]),
                           ("compact", [pg, en, vp, vp, vp, vp, vp, sz]),
                           ("free", [pg, en, vp])):
            fn = getattr(L, "grkv_pages_" + name)
            fn.restype = ctypes.c_int
            fn.argtypes = args
        L.grkv_pages_workspace_bytes.restype = sz
        L.grkv_pages_workspace_bytes.argtypes = [pg, i32]
        L.grkv_tree_attention.restype = ctypes.c_int
        L.grkv_tree_attention.argtypes = [vp, pg, P(_Tree), vp, vp, vp, vp, sz]
        L.grkv_tree_attention_workspace_bytes.restype = sz
        L.grkv_tree_attention_workspace_bytes.argtypes = [pg, P(_Tree)]
        L.grkv_sink_attention.restype = ctypes.c_int
        L.grkv_sink_attention.argtypes = [vp, vp, vp, ctypes.c_int64, i32, i32, i32, vp,
                                          P(Problem), vp, vp, vp, sz]
        L.grkv_sink_attention_workspace_bytes.restype = sz
        L.grkv_sink_attention_workspace_bytes.argtypes = [P(Problem), ctypes.c_int64, i32, i32, i32]
        st, rw, i64, f64 = P(_StepC), P(_Rows), ctypes.c_int64, ctypes.c_double
        for name, res, args in (
                ("pages_extend", ctypes.c_int, [pg, st, vp, vp, vp, vp, vp, vp, vp, vp, sz]),
                ("pages_extend_workspace_bytes", sz, [pg, st]),
                ("rotary", ctypes.c_int, [rw, rw, i32, i32, i32, i32, vp, P(_Rotation), vp]),
                ("rotary_freqs", ctypes.c_int, [i32, f64, i32, f64, f64, f64, f64, vp]),
                ("pages_store", ctypes.c_int, [pg, i32, i32, vp, i64, rw, rw, i32, rw, rw, i32, vp,
                                               P(_Rotation), vp]),
                ("chunk_attention", ctypes.c_int, [vp, pg, st, vp, P(_Chunk), vp, vp, vp, vp, sz]),
                ("chunk_attention_workspace_bytes", sz, [pg, st, P(_Chunk)])):
            fn = getattr(L, "grkv_" + name)
            fn.restype = res
            fn.argtypes = args
        L.grkv_status_string.restype = ctypes.c_char_p
        L.grkv_status_string.argtypes = [ctypes.c_int]
        _LIB = L
    return _LIB


def status_string(status: int) -> str:
    return lib().grkv_status_string(status).decode()


def _check(status: int):
    if status != GRKV_OK:
        raise GrkvError(status, status_string(status))


def workspace_bytes(units, group, head_dim, dtype, n, window, budget) -> int:
    prob = Problem(units, group, head_dim, dtype)
    return int(lib().grkv_workspace_bytes(ctypes.byref(prob), n, window, budget))


def workspace_layout(units, group, head_dim, dtype, n, window, budget) -> Layout:
    prob = Problem(units, group, head_dim, dtype)
    lay = Layout()
    _check(lib().grkv_workspace_layout(ctypes.byref(prob), n, window, budget, ctypes.byref(lay)))
    return lay


def workspace_bytes_kv(units, group, head_dim, dtype, n, window, budget, steps=1) -> int:
    prob = Problem(units, group, head_dim, dtype)
    return int(lib().grkv_workspace_bytes_kv(ctypes.byref(prob), n, window, budget, steps))


def workspace_bytes_ragged(units, group, head_dim, dtype, n, window, budgets) -> int:
    import numpy as np
    prob = Problem(units, group, head_dim, dtype)
    b = np.ascontiguousarray(np.asarray(budgets, dtype=np.int32))
    return int(lib().grkv_workspace_bytes_ragged(ctypes.byref(prob), n, window,
                                                 b.ctypes.data_as(ctypes.c_void_p)))


@dataclass
class Result:
    idx: "object"        # int32 [U, c]
    k_out: "object"      # input dtype [U, c, d]
    v_out: "object"      # float32 [U, c, d]
    stats: "object"      # float32 [U, 4]
    workspace: "object"  # uint8 workspace, see intermediates()
    shape: tuple         # (U, G, d, dtype, n, window, budget)


def _prepare(q_obs, K, V, window, budget, need_fn, n_sink, beta, fix_window, causal_window,
             stream, workspace, out, stage_events):
    import torch

    if not (q_obs.is_cuda and K.is_cuda and V.is_cuda):
        raise ValueError("q_obs, K and V must be device tensors")
    if not (q_obs.dtype == K.dtype == V.dtype) or K.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("q_obs, K, V must share dtype bfloat16 or float32")
    if not (q_obs.is_contiguous() and K.is_contiguous() and V.is_contiguous()):
        raise ValueError("inputs must be contiguous")
    U, G, w, d = q_obs.shape
    if w != window or K.shape[0] != U or K.shape[2] != d or V.shape != K.shape:
        raise ValueError("shape mismatch: q_obs %s K %s V %s window %d"
                         % (tuple(q_obs.shape), tuple(K.shape), tuple(V.shape), window))
    n = K.shape[1]
    dt = GRKV_BF16 if K.dtype == torch.bfloat16 else GRKV_F32
    dev = K.device
    need = need_fn(U, G, d, dt, n, window, budget)
    if need == 0:
        # let the library report the precise error
        need = 256
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(need, dtype=torch.uint8, device=dev)
    if out is None:
        out = Result(idx=torch.empty((U, budget), dtype=torch.int32, device=dev),
                     k_out=torch.empty((U, budget, d), dtype=K.dtype, device=dev),
                     v_out=torch.empty((U, budget, d), dtype=torch.float32, device=dev),
                     stats=torch.empty((U, 4), dtype=torch.float32, device=dev),
                     workspace=workspace, shape=())
    out.workspace = workspace
    out.shape = (U, G, d, dt, n, window, budget)
    prob = Problem(U, G, d, dt)
    opt = Options(n_sink, beta, 1 if fix_window else 0, 1 if causal_window else 0)
    outs = Outputs(out.idx.data_ptr(), out.k_out.data_ptr(), out.v_out.data_ptr(),
                   out.stats.data_ptr(), workspace.data_ptr(), workspace.numel(),
                   stage_events)
    if stream is None:
        stream = torch.cuda.current_stream(dev)
    handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    return out, prob, opt, outs, handle, n


def compress(q_obs, K, V, window: int, budget: int, pool_kernel: int, lam: float, *,
             n_sink: int = 4, beta: float = 0.10, fix_window: bool = True,
             causal_window: bool = True, stream=None, workspace=None, out=None,
             stage_events=None) -> Result:
    """GRKV compression of U units on the GPU.

    q_obs [U, G, w, d], K and V [U, n, d]: contiguous CUDA tensors of one dtype
    (bfloat16 or float32).  Returns the retained indices, K0, the merged V*,
    per-unit stats {||Y||^2, D_before, D_after, status} and the workspace.
    ``workspace`` (uint8, >= workspace_bytes) and ``out`` (a Result whose
    tensors are reused) avoid allocations in timed loops.  ``stage_events`` is
    an optional ctypes array of 2 * NUM_STAGES event handles (see grkv.h).
    """
    out, prob, opt, outs, handle, n = _prepare(
        q_obs, K, V, window, budget, workspace_bytes, n_sink, beta, fix_window, causal_window,
        stream, workspace, out, stage_events)
    st = lib().grkv_compress(q_obs.data_ptr(), K.data_ptr(), V.data_ptr(), n, window, budget,
                             pool_kernel, float(lam), ctypes.c_void_p(handle),
                             ctypes.byref(prob), ctypes.byref(opt), ctypes.byref(outs))
    _check(st)
    return out


def compress_noalloc(q_obs, K, V, window: int, budget: int, pool_kernel: int, lam: float, *,
                     out: Result, n_sink: int = 4, beta: float = 0.10, fix_window: bool = True,
                     causal_window: bool = True, stream=None) -> Result:
    """``compress`` through the entry point that allocates nothing: the
    library's own per-device scratch array (NOALLOC_SCRATCH_BYTES) serves as the
    workspace.  ``out`` (a Result with idx, k_out, v_out and stats of the
    right shapes) is required, so this call allocates no device memory either.
    Calls that overlap on one device race on the shared scratch array."""
    import torch

    if not (q_obs.is_cuda and K.is_cuda and V.is_cuda):
        raise ValueError("q_obs, K and V must be device tensors")
    if not (q_obs.dtype == K.dtype == V.dtype) or K.dtype not in (torch.bfloat16, torch.float32):
        raise ValueError("q_obs, K, V must share dtype bfloat16 or float32")
    if not (q_obs.is_contiguous() and K.is_contiguous() and V.is_contiguous()):
        raise ValueError("inputs must be contiguous")
    U, G, w, d = q_obs.shape
    if w != window or K.shape[0] != U or K.shape[2] != d or V.shape != K.shape:
        raise ValueError("shape mismatch: q_obs %s K %s V %s window %d"
                         % (tuple(q_obs.shape), tuple(K.shape), tuple(V.shape), window))
    n = K.shape[1]
    if (tuple(out.idx.shape) != (U, budget) or tuple(out.k_out.shape) != (U, budget, d)
            or tuple(out.v_out.shape) != (U, budget, d) or tuple(out.stats.shape) != (U, 4)
            or out.k_out.dtype != K.dtype or out.v_out.dtype != torch.float32
            or out.idx.dtype != torch.int32 or out.stats.dtype != torch.float32):
        raise ValueError("out tensors do not match the call's shapes")
    dt = GRKV_BF16 if K.dtype == torch.bfloat16 else GRKV_F32
    prob = Problem(U, G, d, dt)
    opt = Options(n_sink, beta, 1 if fix_window else 0, 1 if causal_window else 0)
    outs = Outputs(out.idx.data_ptr(), out.k_out.data_ptr(), out.v_out.data_ptr(),
                   out.stats.data_ptr(), None, 0, None)
    if stream is None:
        stream = torch.cuda.current_stream(K.device)
    handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    with torch.cuda.device(K.device):
        st = lib().grkv_compress_noalloc(q_obs.data_ptr(), K.data_ptr(), V.data_ptr(), n, window,
                                         budget, pool_kernel, float(lam), ctypes.c_void_p(handle),
                                         ctypes.byref(prob), ctypes.byref(opt), ctypes.byref(outs))
    _check(st)
    out.workspace = None
    out.shape = (U, G, d, dt, n, window, budget)
    return out


def h2o_workspace_bytes(units, group, head_dim, dtype, n) -> int:
    prob = Problem(units, group, head_dim, dtype)
    return int(lib().grkv_h2o_workspace_bytes(ctypes.byref(prob), n))


def h2o_scores(q_all, K, window: int, *, stream=None, workspace=None, out=None):
    """H2O accumulated-attention scores of every prefix token (grkv_h2o_scores).

    q_all [U, G, n, d] (the queries of every prompt position) and K [U, n, d]:
    contiguous bfloat16 device tensors.  Returns float32 scores [U, n - window]."""
    import torch

    if not (q_all.is_cuda and K.is_cuda) or not (q_all.is_contiguous() and K.is_contiguous()):
        raise ValueError("q_all and K must be contiguous device tensors")
    if q_all.dtype != torch.bfloat16 or K.dtype != torch.bfloat16:
        raise ValueError("q_all and K must be bfloat16")
    U, Gq, n, d = q_all.shape
    if tuple(K.shape) != (U, n, d):
        raise ValueError("shape mismatch: q_all %s K %s" % (tuple(q_all.shape), tuple(K.shape)))
    need = max(256, h2o_workspace_bytes(U, Gq, d, GRKV_BF16, n))
    if workspace is None or workspace.numel() < need:
        workspace = torch.empty(need, dtype=torch.uint8, device=K.device)
    if out is None:
        out = torch.empty((U, max(n - window, 0)), dtype=torch.float32, device=K.device)
    prob = Problem(U, Gq, d, GRKV_BF16)
    if stream is None:
        stream = torch.cuda.current_stream(K.device)
    handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    _check(lib().grkv_h2o_scores(q_all.data_ptr(), K.data_ptr(), n, window,
                                 ctypes.c_void_p(handle), ctypes.byref(prob),
                                 out.data_ptr() if out.numel() else None, workspace.data_ptr(),
                                 workspace.numel()))
    return out


def compress_scored(q_obs, K, V, window: int, budget: int, pool_kernel: int, lam: float,
                    scores, *, n_sink: int = 4, beta: float = 0.10, fix_window: bool = True,
                    causal_window: bool = True, stream=None, workspace=None, out=None,
                    stage_events=None) -> Result:
    """``compress`` with the selection ranking caller-supplied per-token scores
    (float32 [U, n - window], finite and non-negative) pooled with pool_kernel,
    instead of the window attention's column sums (grkv_compress_scored)."""
    import torch

    out, prob, opt, outs, handle, n = _prepare(
        q_obs, K, V, window, budget, workspace_bytes, n_sink, beta, fix_window, causal_window,
        stream, workspace, out, stage_events)
    if not (scores.is_cuda and scores.dtype == torch.float32 and scores.is_contiguous()):
        raise ValueError("scores must be a contiguous float32 device tensor")
    if tuple(scores.shape) != (K.shape[0], n - window):
        raise ValueError("scores must be [U, n - window]")
    st = lib().grkv_compress_scored(q_obs.data_ptr(), K.data_ptr(), V.data_ptr(), n, window,
                                    budget, pool_kernel, float(lam), ctypes.c_void_p(handle),
                                    ctypes.byref(prob), ctypes.byref(opt),
                                    scores.data_ptr() if scores.numel() else None,
                                    ctypes.byref(outs))
    _check(st)
    return out


def compress_kv(q_obs, K, V, window: int, budget: int, pool_kernel: int, lam: float, *,
                lambda_k=None, max_iter: int = 64, tol: float = 1e-5, steps: int = 1,
                n_sink: int = 4,
                beta: float = 0.10, fix_window: bool = True, causal_window: bool = True,
                stream=None, workspace=None, out=None, k_star=None, cg_info=None,
                stage_events=None):
    """``compress`` followed by the key step (bfloat16 inputs, G*w <= 128), and
    for ``steps`` > 1 further alternating value and key steps.

    Returns ``(result, k_star, cg_info)``: k_star float32 [U, c, d] holds the
    merged keys K*, cg_info float32 [U, 4] holds {CG iterations, final
    relative residual, KEY_* outcome, ||rhs||} of the last key step.
    ``lambda_k`` defaults to ``lam``."""
    import torch

    out, prob, opt, outs, handle, n = _prepare(
        q_obs, K, V, window, budget,
        lambda *a: workspace_bytes_kv(*a, steps=steps), n_sink, beta, fix_window,
        causal_window, stream, workspace, out, stage_events)
    U, d = q_obs.shape[0], q_obs.shape[3]
    if k_star is None:
        k_star = torch.empty((U, budget, d), dtype=torch.float32, device=K.device)
    if cg_info is None:
        cg_info = torch.empty((U, 4), dtype=torch.float32, device=K.device)
    kopt = KeyOptions(float(lam if lambda_k is None else lambda_k), int(max_iter), float(tol),
                      int(steps))
    st = lib().grkv_compress_kv(q_obs.data_ptr(), K.data_ptr(), V.data_ptr(), n, window, budget,
                                pool_kernel, float(lam), ctypes.c_void_p(handle),
                                ctypes.byref(prob), ctypes.byref(opt), ctypes.byref(outs),
                                ctypes.byref(kopt), ctypes.c_void_p(k_star.data_ptr()),
                                ctypes.c_void_p(cg_info.data_ptr()))
    _check(st)
    return out, k_star, cg_info


def carrier_stats(K, idx, group: int, stats=None, *, stream=None, assign=None, counts=None,
                  metrics=None, l_common=None):
    """Key-cosine carrier assignment and its load metrics (see grkv.h).

    K [U, n, d] bfloat16 device tensor, idx [U, c] int32 (from ``compress``),
    stats [U, 4] optional (gives L_common).  Returns ``(assign [U, n] int32,
    counts [U, c] int32, metrics [U, 8] float32, l_common [1] float32 or None)``;
    the metric columns are named in CARRIER_METRICS."""
    import torch

    if not (K.is_cuda and idx.is_cuda) or not K.is_contiguous() or not idx.is_contiguous():
        raise ValueError("K and idx must be contiguous device tensors")
    U, n, d = K.shape
    c = idx.shape[1]
    dt = GRKV_BF16 if K.dtype == torch.bfloat16 else GRKV_F32
    dev = K.device
    if assign is None:
        assign = torch.empty((U, n), dtype=torch.int32, device=dev)
    if counts is None:
        counts = torch.empty((U, c), dtype=torch.int32, device=dev)
    if metrics is None:
        metrics = torch.empty((U, 8), dtype=torch.float32, device=dev)
    if stats is not None and l_common is None:
        l_common = torch.empty(1, dtype=torch.float32, device=dev)
    if stream is None:
        stream = torch.cuda.current_stream(dev)
    handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    prob = Problem(U, group, d, dt)
    ptr = lambda t: None if t is None else ctypes.c_void_p(t.data_ptr())
    st = lib().grkv_carrier_stats(K.data_ptr(), n, c, ctypes.byref(prob), idx.data_ptr(),
                                  ptr(stats), ctypes.c_void_p(handle), assign.data_ptr(),
                                  ptr(counts), metrics.data_ptr(),
                                  ptr(l_common) if stats is not None else None)
    _check(st)
    return assign, counts, metrics, (l_common if stats is not None else None)


def pyramid_budgets(layers: int, kv_heads: int, mean_budget: int, window: int, n: int,
                    ratio: float = 0.5):
    """Per-unit budgets (numpy int32 [layers * kv_heads]) of the pyramid schedule."""
    import numpy as np
    out = np.empty(layers * kv_heads, dtype=np.int32)
    _check(lib().grkv_pyramid_budgets(layers, kv_heads, mean_budget, window, n, float(ratio),
                                      out.ctypes.data_as(ctypes.c_void_p)))
    return out


def adaptive_budgets(pooled, layers: int, kv_heads: int, budget: int, window: int, *,
                     stream=None, out=None):
    """Per-unit budgets (int32 device tensor [U]) from the pooled scores [U, n - w]
    of a ``compress`` call (see ``intermediates``)."""
    import torch

    if not pooled.is_cuda or pooled.dtype != torch.float32 or not pooled.is_contiguous():
        raise ValueError("pooled must be a contiguous float32 device tensor")
    U, P = pooled.shape
    n = P + window
    if out is None:
        out = torch.empty(U, dtype=torch.int32, device=pooled.device)
    if stream is None:
        stream = torch.cuda.current_stream(pooled.device)
    handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    _check(lib().grkv_adaptive_budgets(ctypes.c_void_p(pooled.data_ptr()), layers, kv_heads, n,
                                       window, budget, ctypes.c_void_p(handle),
                                       ctypes.c_void_p(out.data_ptr())))
    return out


def compress_ragged(q_obs, K, V, window: int, budgets, pool_kernel: int, lam: float, *,
                    n_sink: int = 4, beta: float = 0.10, fix_window: bool = True,
                    causal_window: bool = True, stream=None, workspace=None, out=None,
                    stage_events=None):
    """Every unit compressed with its own budget (``budgets``: host sequence of U
    ints).  Returns ``(idx, k_out, v_out, stats, offsets)`` with the packed
    layout of grkv.h (unit u at slots offsets[u] .. offsets[u] + budgets[u]).
    ``out``: the first four of a previous call's results with the same budgets,
    reused as the outputs.  ``stage_events``: as for ``compress`` (recorded on
    the bf16 path, where one launch per stage serves every unit)."""
    import numpy as np
    import torch

    if not (q_obs.is_cuda and K.is_cuda and V.is_cuda):
        raise ValueError("q_obs, K and V must be device tensors")
    U, G, w, d = q_obs.shape
    n = K.shape[1]
    b = np.ascontiguousarray(np.asarray(budgets, dtype=np.int32))
    if b.shape != (U,) or w != window:
        raise ValueError("budgets must hold one budget per unit")
    dt = GRKV_BF16 if K.dtype == torch.bfloat16 else GRKV_F32
    prob = Problem(U, G, d, dt)
    need = int(lib().grkv_workspace_bytes_ragged(ctypes.byref(prob), n, window,
                                                 b.ctypes.data_as(ctypes.c_void_p)))
    dev = K.device
    if workspace is None or workspace.numel() < max(need, 256):
        workspace = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)
    tot = int(b.sum())
    if out is not None:
        idx, k_out, v_out, stats = out[:4]
        if idx.numel() != tot or k_out.shape != (tot, d) or stats.shape != (U, 4):
            raise ValueError("out does not match the budgets")
    else:
        idx = torch.empty(tot, dtype=torch.int32, device=dev)
        k_out = torch.empty((tot, d), dtype=K.dtype, device=dev)
        v_out = torch.empty((tot, d), dtype=torch.float32, device=dev)
        stats = torch.empty((U, 4), dtype=torch.float32, device=dev)
    opt = Options(n_sink, beta, 1 if fix_window else 0, 1 if causal_window else 0)
    outs = Outputs(idx.data_ptr(), k_out.data_ptr(), v_out.data_ptr(), stats.data_ptr(),
                   workspace.data_ptr(), workspace.numel(), stage_events)
    if stream is None:
        stream = torch.cuda.current_stream(dev)
    handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    _check(lib().grkv_compress_ragged(q_obs.data_ptr(), K.data_ptr(), V.data_ptr(), n, window,
                                      b.ctypes.data_as(ctypes.c_void_p), pool_kernel, float(lam),
                                      ctypes.c_void_p(handle), ctypes.byref(prob),
                                      ctypes.byref(opt), ctypes.byref(outs)))
    offsets = np.concatenate([[0], np.cumsum(b)[:-1]]).astype(np.int64)
    return idx, k_out, v_out, stats, offsets


def intermediates(res: Result) -> dict:
    """Views of the workspace intermediates of the last call (see grkv.h)."""
    import torch

    U, G, d, dt, n, w, c = res.shape
    lay = workspace_layout(U, G, d, dt, n, w, c)
    m = G * w
    mp = 32
    while mp < m:
        mp *= 2
    P = n - w
    ws = res.workspace

    def view(off, dtype, shape):
        count = 1
        for s in shape:
            count *= s
        nbytes = count * torch.empty((), dtype=dtype).element_size()
        return ws[off:off + nbytes].view(dtype).view(*shape)

    return {
        "lse": view(lay.lse, torch.float64, (U, mp))[:, :m],
        "y": view(lay.y, torch.float32, (U, mp, d))[:, :m],
        "score": view(lay.score, torch.float32, (U, P)),
        "pooled": view(lay.pooled, torch.float32, (U, P)),
        "fixed": view(lay.fixed, torch.uint8, (U, c)),
        "resid": view(lay.resid, torch.float32, (U, mp, d))[:, :m],
        "gram": view(lay.gram, torch.float32, (U, mp, mp))[:, :m, :m],
        "z": view(lay.z, torch.float32, (U, d, mp))[:, :, :m],
    }


# ------------------------------------------------------- pages of a cache ----

@dataclass(frozen=True, eq=False, init=False)
class Pages:
    """The pool of pages of grkv.h (``grkv_pages``): contiguous tensors of one
    device.  ``new_pages`` makes an empty one."""
    k: "object"       # bfloat16 or float32 [pages, page_size, head_dim]
    v: "object"       # the same
    table: "object"   # int32 [units, max_pages]
    lens: "object"    # int32 [units]
    refs: "object"    # int32 [pages]
    free: "object"    # int32 [ceil(pages / 32)], bit p % 32 of word p // 32: page p is free

    def __init__(self, k, v, table, lens, refs, free):
        import torch

        i32, dev = torch.int32, k.get_device()
        if dev < 0:
            raise ValueError("a pool's tensors must be device tensors")
        code = _dtype_code(k)
        if code is None or v.dtype != k.dtype:
            raise ValueError("k and v must share dtype bfloat16 or float32")
        if k.dim() != 3 or k.shape != v.shape or table.dim() != 2:
            raise ValueError("k and v must be [pages, page_size, head_dim] and table [units, max_pages]")
        (n, ps, d), (units, width) = k.shape, table.shape
        _int32(n | units | width)
        if lens.shape != (units,) or refs.shape != (n,) or free.shape != ((n + 31) // 32,):
            raise ValueError("lens, refs and free must be [units], [pages] and [ceil(pages / 32)]")
        for t in (k, v, table, lens, refs, free):
            if not t.is_contiguous() or t.get_device() != dev:
                raise ValueError("a pool's tensors must be contiguous and on one device")
        if not (table.dtype == lens.dtype == refs.dtype == free.dtype == i32):
            raise ValueError("table, lens, refs and free must be int32")
        # (a pool is often wrapped anew for a call: one update instead of a guarded assignment
        # per field)
        self.__dict__.update(k=k, v=v, table=table, lens=lens, refs=refs, free=free, _c=_PagesC(
            k.data_ptr(), v.data_ptr(), table.data_ptr(), lens.data_ptr(), refs.data_ptr(),
            free.data_ptr(), n, ps, units, width, d, code))

    @property
    def device(self):
        return self.k.device


_CODES = {}


def _dtype_code(t):
    """grkv_dtype of a tensor, or None."""
    if not _CODES:
        import torch

        _CODES.update({torch.bfloat16: GRKV_BF16, torch.float32: GRKV_F32})
    return _CODES.get(t.dtype)


def _on(dev: int, stream):
    """(handle, context) of a call on device ``dev``.  The context, None where nothing has to
    change, makes that device and stream current, so that a workspace dropped after the call is
    not handed to another stream while it is in use."""
    import torch

    if stream is None:
        if torch._C._cuda_getDevice() == dev:   # (a tensor of the call is there, so it is set up)
            return torch._C._cuda_getCurrentRawStream(dev), None
        stream = torch.cuda.current_stream(dev)
    elif not hasattr(stream, "cuda_stream"):
        stream = torch.cuda.ExternalStream(int(stream), device=dev)
    elif stream.device.index != dev:
        raise ValueError("stream is one of %s, the call's tensors are on cuda:%d" % (stream.device, dev))
    return None, torch.cuda.stream(stream)


def _vector(t, name, dtype, size, dev):
    """A device vector of a call, as its address; None stays."""
    if t is None:
        return None
    if t.dtype != dtype or t.get_device() != dev or t.shape != (size,) or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s vector of %d on cuda:%d" % (name, dtype, size, dev))
    return t.data_ptr()


def _workspace(workspace, need, dev):
    import torch

    if workspace is not None:
        if workspace.get_device() != dev or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor on cuda:%d" % dev)
        if workspace.numel() >= need:
            return workspace
    return torch.empty(max(need, 256), dtype=torch.uint8, device=dev)


def _int32(bits):
    """The bits of a call's sizes, which ctypes would cut to 32 without a word."""
    if bits >> 31 not in (0, -1):
        raise ValueError("sizes must fit 32 bits")


def new_pages(units: int, max_pages: int, pages: int, page_size: int, head_dim: int, dtype=None,
              device=None, *, stream=None) -> Pages:
    """An empty pool of ``pages`` pages of ``page_size`` rows for ``units`` units of at most
    ``max_pages`` pages each.  With ``stream`` its memory is that stream's, which writes it."""
    import torch

    dtype = torch.bfloat16 if dtype is None else dtype
    if min(units, max_pages, pages, page_size, head_dim) < 1:
        raise ValueError("a pool needs units, pages and rows")
    device = torch.device("cuda" if device is None else device)
    if stream is not None and device.type == "cuda":
        dev = torch.cuda.current_device() if device.index is None else device.index
        with _on(dev, stream)[1]:
            return new_pages(units, max_pages, pages, page_size, head_dim, dtype, torch.device("cuda", dev))
    i32 = dict(dtype=torch.int32, device=device)
    pg = Pages(k=torch.empty((pages, page_size, head_dim), dtype=dtype, device=device),
               v=torch.empty((pages, page_size, head_dim), dtype=dtype, device=device),
               table=torch.empty((units, max_pages), **i32), lens=torch.empty(units, **i32),
               refs=torch.empty(pages, **i32), free=torch.empty((pages + 31) // 32, **i32))
    return pages_init(pg)


def pages_init(pages: Pages, *, stream=None) -> Pages:
    """Empties a pool: no unit holds a row, every page is free."""
    handle, on = _on(pages.k.get_device(), stream)
    if on is not None:
        with on:
            return pages_init(pages)
    _check(lib().grkv_pages_init(pages._c, handle))
    return pages


def pages_workspace_bytes(pages: Pages, entries: int) -> int:
    _int32(entries)
    return int(lib().grkv_pages_workspace_bytes(pages._c, entries))


def _page_call(name, pages, entries, args, units, rows, counts, starts, source_rows, status,
               workspace, stream):
    """One call on pages; ``args`` are those between the entries and the stream."""
    import torch

    dev, i32 = pages.k.get_device(), torch.int32
    handle, on = _on(dev, stream)
    if on is not None:
        with on:
            return _page_call(name, pages, entries, args, units, rows, counts, starts, source_rows,
                              status, workspace, None)
    _int32(entries | rows)
    L = lib()
    if status is None:
        status = torch.empty(entries, dtype=i32, device=dev)
        at = status.data_ptr()
    else:
        at = _vector(status, "status", i32, entries, dev)
    en = _PageEntries(entries, _vector(units, "units", i32, entries, dev), rows,
                      _vector(counts, "counts", i32, entries, dev),
                      _vector(starts, "starts", torch.int64, entries, dev), source_rows, at)
    if name == "grkv_pages_free":
        _check(L.grkv_pages_free(pages._c, en, handle))
        return status
    workspace = _workspace(workspace, L.grkv_pages_workspace_bytes(pages._c, entries), dev)
    _check(getattr(L, name)(pages._c, en, *args, handle, workspace.data_ptr(), workspace.numel()))
    return status


def _packed(t, dims, rows, starts, name):
    """(entries, rows, source rows) of [E, rows, ..] or of packed [N, ..] with starts."""
    if t.dim() == dims and starts is None:
        if rows is not None and rows != t.shape[1]:
            raise ValueError("rows is %s's second size" % name)
        return t.shape[0], t.shape[1], t.shape[0] * t.shape[1]
    if t.dim() == dims - 1 and starts is not None and rows is not None:
        return starts.shape[0], int(rows), t.shape[0]
    raise ValueError("%s must have %d dimensions, or %d with starts and rows" % (name, dims, dims - 1))


def pages_append(pages: Pages, k, v, *, units=None, counts=None, starts=None, rows=None,
                 status=None, workspace=None, stream=None):
    """Appends rows to units (grkv_pages_append).

    k, v: contiguous device tensors, bfloat16 or float32 each (rounded to the pool's type):
    [E, rows, head_dim], ``rows`` for each of E entries, or packed [N, head_dim] with
    ``starts`` int64 [E] (the first row of each entry) and ``rows``, a bound on the
    counts.  ``counts`` int32 [E]: the rows of each entry (default: all ``rows``).
    ``units`` int32 [E]: their units (default 0 .. E - 1).  Returns the status of every
    entry, int32 [E] (PAGES_OK or why its unit is as it was)."""
    E, rows, n = _packed(k, 3, rows, starts, "k")
    dev = pages.k.get_device()
    kc, vc = _dtype_code(k), _dtype_code(v)
    for t, code in ((k, kc), (v, vc)):
        if t.get_device() != dev or code is None or not t.is_contiguous():
            raise ValueError("k and v must be contiguous bfloat16 or float32 tensors on the pool's device")
    if k.shape != v.shape or k.shape[-1] != pages.k.shape[2]:
        raise ValueError("shape mismatch: k %s v %s head_dim %d"
                         % (tuple(k.shape), tuple(v.shape), pages.k.shape[2]))
    return _page_call("grkv_pages_append", pages, E,
                      (k.data_ptr(), kc, v.data_ptr(), vc),
                      units, rows, counts, starts, n, status, workspace, stream)


def pages_fork(pages: Pages, src, dst, *, status=None, workspace=None, stream=None):
    """Units ``dst`` (int32 [E], empty) become copies of units ``src``, full pages shared; a
    unit that is its own destination stays as it is (grkv_pages_fork).  Returns the status of
    every entry."""
    import torch

    E = src.shape[0]
    return _page_call("grkv_pages_fork", pages, E,
                      (_vector(dst, "dst", torch.int32, E, pages.k.get_device()),),
                      src, 0, None, None, 0, status, workspace, stream)


def pages_compact(pages: Pages, idx=None, *, units=None, dst=None, keep=None, counts=None,
                  starts=None, rows=None, status=None, workspace=None, stream=None):
    """Units keep their first ``keep`` slots and the slots ``idx`` behind them
    (grkv_pages_compact), in place or, with ``dst`` (int32 [E]), in empty units.

    idx: int32 [E, rows] (the ``idx`` of ``compress``), or packed [N] with ``starts`` int64
    [E] and ``rows`` (``compress_ragged``, with its budgets as ``counts``); None takes the
    units back to ``keep``.  ``units`` int32 [E] (default 0 .. E - 1); ``keep`` int32 [E]
    (default 0).  Returns the status of every entry."""
    import torch

    dev, i32 = pages.k.get_device(), torch.int32
    if idx is None:
        if counts is not None or starts is not None or rows:
            raise ValueError("counts, starts and rows belong to idx")
        known = next((t for t in (units, keep, dst) if t is not None), pages.lens)
        E, rows, n, at = known.shape[0], 0, 0, None
    else:
        if idx.dtype != i32 or idx.get_device() != dev or not idx.is_contiguous():
            raise ValueError("idx must be a contiguous int32 tensor on the pool's device")
        E, rows, n = _packed(idx, 2, rows, starts, "idx")
        at = idx.data_ptr()
    args = (_vector(dst, "dst", i32, E, dev), _vector(keep, "keep", i32, E, dev), at)
    return _page_call("grkv_pages_compact", pages, E, args, units, rows, counts, starts, n,
                      status, workspace, stream)


def pages_free(pages: Pages, units=None, *, status=None, stream=None):
    """Units (int32 [E]; default all) give up their rows and pages (grkv_pages_free)."""
    E = (pages.lens if units is None else units).shape[0]
    return _page_call("grkv_pages_free", pages, E, (), units, 0, None, None, 0, status, None, stream)


# ---------------------------------------------------- attention over a cache ----

def tree_attention_workspace_bytes(pages: Pages, entries, group, tokens, window=0, n_sink=0) -> int:
    _int32(entries | group | tokens | window | n_sink)
    tr = _Tree(entries, group, tokens, None, None, None, 0, window, n_sink)
    return int(lib().grkv_tree_attention_workspace_bytes(pages._c, tr))


def _given(t, name, dtype, shape, dev):
    if t.dtype != dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        raise ValueError("%s must be a contiguous %s tensor %s on cuda:%d"
                         % (name, dtype, tuple(shape), dev))


def _outputs(q, shape, dev, out, lse, return_lse):
    """o, lse and lse's address."""
    import torch

    if out is None:
        out = torch.empty_like(q)
    else:
        _given(out, "out", q.dtype, q.shape, dev)
    if lse is not None:
        _given(lse, "lse", torch.float32, shape, dev)
    elif return_lse:
        lse = torch.empty(*shape, dtype=torch.float32, device=dev)
    return out, lse, None if lse is None else lse.data_ptr()


def tree_attention(q, pages: Pages, parents=None, *, units=None, counts=None, window: int = 0,
                   n_sink: int = 0, return_lse: bool = False, out=None, lse=None, workspace=None,
                   stream=None):
    """Attention of drafted tokens over the pages of a cache (grkv_tree_attention).

    q: [E, G, t, d] of the pool's type; its tokens' keys and values are the last t
    slots of the units (``pages_append``), so decoding one token is t = 1.
    ``parents``: int32 [trees, t], trees dividing E (consecutive entries share one), or
    None for a chain.  ``units``: int32 [E] (default 0 .. E - 1).  ``counts``: int32 [E],
    the drafted tokens of each entry in a padded batch (the rows behind them stay as they
    were).  ``window`` > 0: only the last ``window`` positions and the first ``n_sink``.
    Returns o [E, G, t, d], with ``return_lse`` (o, lse float32 [E, G, t])."""
    import torch

    dev, i32 = pages.k.get_device(), torch.int32
    handle, on = _on(dev, stream)
    if on is not None:
        with on:
            return tree_attention(q, pages, parents, units=units, counts=counts, window=window,
                                  n_sink=n_sink, return_lse=return_lse, out=out, lse=lse,
                                  workspace=workspace)
    if q.get_device() != dev or q.dtype != pages.k.dtype or q.dim() != 4 or not q.is_contiguous():
        raise ValueError("q must be a contiguous [E, G, t, d] tensor of the pool's type and device")
    E, G, t, d = q.shape
    c = pages._c
    _int32(window | n_sink)
    if d != c.head_dim:
        raise ValueError("head_dim %d, the pool's is %d" % (d, c.head_dim))
    trees, up = 0, None
    if parents is not None:
        trees, up = parents.shape[0], parents.data_ptr()
        if (parents.dtype != i32 or parents.get_device() != dev or parents.shape != (trees, t)
                or trees < 1 or not parents.is_contiguous()):
            raise ValueError("parents must be a contiguous int32 [trees, %d] tensor on cuda:%d, "
                             "trees >= 1" % (t, dev))
    tr = _Tree(E, G, t, _vector(units, "units", i32, E, dev), _vector(counts, "counts", i32, E, dev),
               up, trees, window, n_sink)
    out, lse, lp = _outputs(q, (E, G, t), dev, out, lse, return_lse)
    L = lib()
    workspace = _workspace(workspace, L.grkv_tree_attention_workspace_bytes(c, tr), dev)
    _check(L.grkv_tree_attention(q.data_ptr(), c, tr, out.data_ptr(), lp, handle,
                                 workspace.data_ptr(), workspace.numel()))
    return (out, lse) if return_lse else out


def sink_attention_workspace_bytes(units, group, head_dim, dtype, n, nq, window, n_sink) -> int:
    _int32(units | group | head_dim | nq | window | n_sink)
    prob = Problem(units, group, head_dim, dtype)
    return int(lib().grkv_sink_attention_workspace_bytes(prob, n, nq, window, n_sink))


def sink_attention(q, K, V, window: int, n_sink: int = 4, *, return_lse: bool = False, out=None,
                   lse=None, workspace=None, stream=None):
    """Causal attention with a sliding window and sink tokens (grkv_sink_attention).

    q [U, G, nq, d] (the last nq positions), K and V [U, n, d]: contiguous device tensors of
    one dtype, bfloat16 or float32.  ``window`` 0: none.  Returns o [U, G, nq, d], with
    ``return_lse`` (o, lse float32 [U, G, nq])."""
    dev = q.get_device()
    if dev < 0 or K.get_device() != dev or V.get_device() != dev:
        raise ValueError("q, K and V must be tensors of one device")
    handle, on = _on(dev, stream)
    if on is not None:
        with on:
            return sink_attention(q, K, V, window, n_sink, return_lse=return_lse, out=out, lse=lse,
                                  workspace=workspace)
    code = _dtype_code(q)
    if code is None or not (q.dtype == K.dtype == V.dtype):
        raise ValueError("q, K, V must share dtype bfloat16 or float32")
    if not (q.is_contiguous() and K.is_contiguous() and V.is_contiguous()):
        raise ValueError("inputs must be contiguous")
    kv = K.shape
    if q.dim() != 4 or len(kv) != 3 or kv != V.shape or q.shape[::3] != kv[::2]:
        raise ValueError("shape mismatch: q %s K %s V %s"
                         % (tuple(q.shape), tuple(K.shape), tuple(V.shape)))
    U, G, nq, d = q.shape
    n = kv[1]
    _int32(window | n_sink)
    prob = Problem(U, G, d, code)
    out, lse, lp = _outputs(q, (U, G, nq), dev, out, lse, return_lse)
    L = lib()
    workspace = _workspace(workspace, L.grkv_sink_attention_workspace_bytes(prob, n, nq, window, n_sink),
                           dev)
    _check(L.grkv_sink_attention(q.data_ptr(), K.data_ptr(), V.data_ptr(), n, nq, window, n_sink,
                                 handle, prob, out.data_ptr(), lp, workspace.data_ptr(),
                                 workspace.numel()))
    return (out, lse) if return_lse else out


# ------------------------------------------------- a served model's step ----

def rotary_freqs(dims: int, base: float = 1e4, *, method: str = "plain", factor: float = 1.0,
                 length: float = 0.0, low: float = 1.0, high: float = 32.0, device=None):
    """Radians per position of the ``dims`` / 2 pairs, float64 [dims / 2] on ``device``
    (grkv_rotary_freqs): "plain", or for contexts ``factor`` times as long as ``length`` "linear",
    "base" or "parts" (pairs of ``high`` turns over the length stay, those of ``low`` are
    divided)."""
    import torch

    if method not in ROTARY_METHODS:
        raise ValueError("method must be one of %s" % (ROTARY_METHODS,))
    _int32(dims)
    out = torch.empty(max(dims // 2, 1), dtype=torch.float64)
    _check(lib().grkv_rotary_freqs(dims, float(base), ROTARY_METHODS.index(method), float(factor),
                                   float(length), float(low), float(high), out.data_ptr()))
    return out if device is None else out.to(device)


def _rotation(freqs, scale, interleaved, inverse, dev):
    import torch

    if freqs.dtype != torch.float64 or freqs.dim() != 1 or freqs.get_device() != dev or not freqs.is_contiguous():
        raise ValueError("freqs must be a contiguous float64 vector on cuda:%d" % dev)
    return _Rotation(freqs.data_ptr(), 2 * freqs.shape[0], bool(interleaved), bool(inverse), scale)


def _rows(t, name, dev):
    """A [tokens, heads, columns] tensor of whole rows."""
    step = t.stride()
    if t.get_device() != dev or len(step) != 3 or (step[2] != 1 and t.shape[2] > 1) or _dtype_code(t) is None:
        raise ValueError("%s must be a bfloat16 or float32 [tokens, heads, columns] tensor on cuda:%d whose "
                         "last dimension is contiguous" % (name, dev))
    return _Rows(t.data_ptr(), step[0], step[1])


def _rows_meet(x, y):
    """Whether rows of x [T, H, d] and of y, of the same shape and type, share an element without
    being the same rows."""
    import torch

    T, H, d = x.shape
    at = (y.data_ptr() - x.data_ptr()) // x.element_size()   # where y begins, in x's elements
    (xt, xh, _), (yt, yh, _) = x.stride(), y.stride()
    if not -((T - 1) * yt + (H - 1) * yh + d) < at < (T - 1) * xt + (H - 1) * xh + d or x.numel() == 0:
        return False
    if T == 1 or H == 1:   # (the other's stride alone counts)
        xt, xh = (0, 0 if H == 1 else xh) if T == 1 else (xt, 0)
        yt, yh = (0, 0 if H == 1 else yh) if T == 1 else (yt, 0)
    if at == 0 and (xt, xh) == (yt, yh):   # the same rows
        return False
    if (xt, xh) != (yt, yh):   # any two sets of rows, which hardly ever lie among one another
        t, h = torch.arange(T)[:, None], torch.arange(H)
        a, b = (t * xt + h * xh).flatten().sort().values, (t * yt + h * yh).flatten() + at
        i = torch.searchsorted(a, b)
        return bool(((a[(i - 1).clamp(min=0)] - b).abs() < d).any() or ((a[i.clamp(max=a.numel() - 1)] - b).abs() < d).any())
    if xh == d:            # heads side by side are one row
        H, d, xh = 1, H * d, 0
    (n, step), (m, far) = sorted([(T, xt), (H, xh)])
    for i in range(1 - n, n):   # rows that lie i and j steps apart
        r = at + i * step
        j = -r // far if far else 0
        for k in (j, j + 1):
            if abs(r + max(1 - m, min(m - 1, k)) * far) < d:
                return True
    return False


def _out_rows(x, out, name, dev):
    """The output of rotated rows: ``out``, or a tensor like x."""
    import torch

    if out is None:
        out = torch.empty_like(x)
        return out, _rows(out, name, dev)
    if out is x:
        apart = x.is_contiguous()
    else:
        if out.shape != x.shape or out.dtype != x.dtype:
            raise ValueError("%s must have %s and dtype %s" % (name, tuple(x.shape), x.dtype))
        apart = out.is_contiguous()
    rows = _rows(out, name, dev)
    if out is not x and _rows_meet(x, out):
        raise ValueError("%s overlaps its input" % name)
    if not apart:   # rows that are written do not overlap
        ends = out.shape[2]
        for step, n in sorted((out.stride(i), out.shape[i]) for i in (0, 1) if out.shape[i] > 1):
            if step < ends:
                raise ValueError("%s has rows that overlap" % name)
            ends = step * (n - 1) + ends
    return out, rows


def rotary(x, positions, freqs, *, scale: float = 1.0, interleaved: bool = False,
           inverse: bool = False, out=None, stream=None):
    """Rows rotated by their positions (grkv_rotary): x [tokens, heads, columns], bfloat16 or
    float32, of any strides with whole rows (queries as ``compress`` takes them, [G, w, d], as
    ``x.transpose(0, 1)``); positions int32 [tokens]; freqs float64 [dims / 2] (``rotary_freqs``).
    Pairs are columns (i, i + dims / 2), or (2 i, 2 i + 1) with ``interleaved``; columns from
    dims on stay.  ``inverse`` rotates back, which is the gradient of the call.  ``out`` may be x, and else
    shares no element with it.
    Rows at NO_POSITION are left as they were.  Returns out, which carries x's gradient (zero in those
    rows; positions and freqs are to stay until then, freqs have none); a call whose x needs one takes no
    ``out``."""
    import torch

    dev = x.get_device()
    if dev < 0:
        raise ValueError("x must be a device tensor")
    handle, on = _on(dev, stream)
    if on is not None:
        with on:
            return rotary(x, positions, freqs, scale=scale, interleaved=interleaved, inverse=inverse,
                          out=out)
    if x.requires_grad and torch.is_grad_enabled():
        if out is not None:
            raise ValueError("rotary into out records no gradient, which x needs (torch.no_grad for none)")
        return _rotated()(x, positions, freqs, scale, interleaved, inverse, False)
    xr = _rows(x, "x", dev)
    out, yr = _out_rows(x, out, "out", dev)
    T, H, d = x.shape
    _int32(T | H | d)
    _check(lib().grkv_rotary(xr, yr, T, H, d, _dtype_code(x), _vector(positions, "positions", torch.int32, T, dev),
                             _rotation(freqs, scale, interleaved, inverse, dev), handle))
    return out


_ROTATED = None


def _rotated():
    """``rotary`` for autograd: the gradient is the call with ``inverse`` the other way round, and zero
    in rows that the call did not write."""
    global _ROTATED
    if _ROTATED is None:
        import torch

        class Rotated(torch.autograd.Function):
            @staticmethod
            def forward(ctx, x, positions, freqs, scale, interleaved, inverse, clear):
                ctx.save_for_backward(positions, freqs)
                ctx.how = scale, interleaved, inverse
                out = torch.zeros(x.shape, dtype=x.dtype, device=x.device) if clear else None
                return rotary(x, positions, freqs, scale=scale, interleaved=interleaved, inverse=inverse, out=out)

            @staticmethod
            def backward(ctx, g):
                positions, freqs = ctx.saved_tensors
                scale, interleaved, inverse = ctx.how
                if g.shape[2] > 1 and g.stride(2) != 1:   # (of a sum: one element as all)
                    g = g.contiguous()
                return (Rotated.apply(g, positions, freqs, scale, interleaved, not inverse, True),) + (None,) * 6

        _ROTATED = Rotated.apply
    return _ROTATED


def _step(pages, B, T, heads, units):
    """The sequences of a step and their units."""
    import torch

    at, stride = None, 0
    if units is not None:
        if (units.dtype != torch.int32 or units.get_device() != pages.k.get_device() or units.dim() != 2
                or units.shape[0] != B or (units.shape[1] > 1 and units.stride(1) != 1)):
            raise ValueError("units must be an int32 [%d, heads] tensor on the pool's device whose last "
                             "dimension is contiguous" % B)
        if heads is not None and heads != units.shape[1]:
            raise ValueError("units has %d heads, not %d" % (units.shape[1], heads))
        heads, at = units.shape[1], units.data_ptr()
        stride = units.stride(0) if B > 1 else max(units.stride(0), heads)
    elif heads is None:
        raise ValueError("a step needs units or heads")
    _int32(B | T | heads)
    return _StepC(B, heads, at, stride, T)


@dataclass
class Step:
    """What ``pages_extend`` gives for the new tokens of a step."""
    starts: "object"      # int32 [sequences + 1]: a sequence's rows are starts[b] .. starts[b + 1] - 1
    positions: "object"   # int32 [tokens], NO_POSITION where there is none
    slots: "object"       # int64 [tokens, heads]: rows of the pool, -1 where there is none
    status: "object"      # int32 [sequences]: PAGES_OK, or why a sequence is as it was


def pages_extend_workspace_bytes(pages: Pages, sequences: int, heads: int, tokens: int) -> int:
    _int32(sequences | heads | tokens)
    return int(lib().grkv_pages_extend_workspace_bytes(pages._c, _StepC(sequences, heads, None, 0, tokens)))


def pages_extend(pages: Pages, counts, tokens: int, *, heads=None, units=None, seen=None, out=None,
                 workspace=None, stream=None) -> Step:
    """Grows the units of sequences by their new tokens, and gives every token's position and
    slots (grkv_pages_extend).

    counts: int32 [B], the new tokens of each sequence, packed into ``tokens`` rows.  ``units``:
    int32 [B, heads] (default: unit b * heads + h).  ``seen``: int32 [B], the tokens that a
    sequence had (default: the length of its first unit).  ``out``: the Step of a previous call
    of these sizes, written again."""
    import torch

    dev, i32 = pages.k.get_device(), torch.int32
    handle, on = _on(dev, stream)
    if on is not None:
        with on:
            return pages_extend(pages, counts, tokens, heads=heads, units=units, seen=seen, out=out,
                                workspace=workspace)
    B = counts.shape[0] if counts.dim() else 0
    st = _step(pages, B, tokens, heads, units)
    if out is None:
        if min(tokens, st.heads) < 0:
            raise ValueError("a step needs heads, and tokens of 0 or more")
        out = Step(torch.empty(B + 1, dtype=i32, device=dev), torch.empty(tokens, dtype=i32, device=dev),
                   torch.empty((tokens, st.heads), dtype=torch.int64, device=dev),
                   torch.empty(B, dtype=i32, device=dev))
    else:
        _given(out.slots, "out.slots", torch.int64, (tokens, st.heads), dev)
        _vector(out.starts, "out.starts", i32, B + 1, dev)
        _vector(out.positions, "out.positions", i32, tokens, dev)
        _vector(out.status, "out.status", i32, B, dev)
    L = lib()
    args = (_vector(counts, "counts", i32, B, dev), _vector(seen, "seen", i32, B, dev), out.starts.data_ptr(),
            out.positions.data_ptr(), out.slots.data_ptr(), out.status.data_ptr())
    workspace = _workspace(workspace, L.grkv_pages_extend_workspace_bytes(pages._c, st), dev)
    _check(L.grkv_pages_extend(pages._c, st, *args, handle, workspace.data_ptr(), workspace.numel()))
    if B == 0:   # (the call does nothing)
        out.starts.zero_()
        out.positions.fill_(NO_POSITION)
        out.slots.fill_(-1)
    return out


def pages_store(pages: Pages, slots, k, v, *, q=None, positions=None, freqs=None, scale: float = 1.0,
                interleaved: bool = False, out=None, stream=None):
    """Stores a step's keys and values at their slots, keys rotated (grkv_pages_store).

    slots: int64 [tokens, heads] (``pages_extend``; a layer's columns of a model's); k, v:
    [tokens, heads, d], bfloat16 or float32, of any strides with whole rows, rounded to the
    pool's type.  With ``freqs`` (float64 [dims / 2]) and ``positions`` (int32 [tokens]) keys are
    rotated as by ``rotary``, and so are queries q [tokens, query heads, d] of k's type into ``out``
    (which may be q, and else overlaps none of the call's rows).  No gradient is recorded.  Returns out,
    None without q."""
    import torch

    dev = pages.k.get_device()
    handle, on = _on(dev, stream)
    if on is not None:
        with on:
            return pages_store(pages, slots, k, v, q=q, positions=positions, freqs=freqs, scale=scale,
                               interleaved=interleaved, out=out)
    kr, vr = _rows(k, "k", dev), _rows(v, "v", dev)
    T, H, d = k.shape
    _int32(T | H)
    if v.shape != k.shape or v.dtype != k.dtype or d != pages._c.head_dim:
        raise ValueError("shape mismatch: k %s %s v %s %s head_dim %d"
                         % (tuple(k.shape), k.dtype, tuple(v.shape), v.dtype, pages._c.head_dim))
    if (slots.dtype != torch.int64 or slots.get_device() != dev or slots.shape != (T, H)
            or (H > 1 and slots.stride(1) != 1)):
        raise ValueError("slots must be an int64 [%d, %d] tensor on cuda:%d whose last dimension is "
                         "contiguous" % (T, H, dev))
    if (freqs is None) != (positions is None) or (q is not None and freqs is None):
        raise ValueError("positions and freqs belong together, and q needs them")
    if out is not None and q is None:
        raise ValueError("out belongs to q")
    rot = qr = yr = at = None
    Q = 0
    if freqs is not None:
        rot, at = _rotation(freqs, scale, interleaved, False, dev), _vector(positions, "positions", torch.int32, T, dev)
    if q is not None:
        qr = _rows(q, "q", dev)
        out, yr = _out_rows(q, out, "out", dev)
        Q = q.shape[1]
        _int32(Q)
        if q.shape[::2] != (T, d) or q.dtype != k.dtype:
            raise ValueError("q must have k's tokens, columns and dtype")
    step = slots.stride(0) if T > 1 else H
    _check(lib().grkv_pages_store(pages._c, T, H, slots.data_ptr(), step, kr, vr, _dtype_code(k), qr, yr, Q, at, rot, handle))
    return out


def chunk_attention_workspace_bytes(pages: Pages, sequences, heads, tokens, group, longest=None, window=0,
                                    n_sink=0) -> int:
    longest = max(tokens, 1) if longest is None else longest
    _int32(sequences | heads | tokens | group | longest | window | n_sink)
    return int(lib().grkv_chunk_attention_workspace_bytes(
        pages._c, _StepC(sequences, heads, None, 0, tokens), _Chunk(group, longest, window, n_sink)))


def chunk_attention(q, pages: Pages, starts, *, heads=None, units=None, longest=None, window: int = 0,
                    n_sink: int = 0, return_lse: bool = False, out=None, lse=None, workspace=None,
                    stream=None):
    """Attention of a step's new tokens over their units (grkv_chunk_attention).

    q: [tokens, heads * G, d] of the pool's type, the tokens of all sequences one behind the other;
    starts: int32 [B + 1] (``pages_extend``), sequence b's rows; its keys and values are the
    last slots of the sequence's units.  ``units``: int32 [B, heads] (default: unit b * heads +
    h).  ``longest``: the most new tokens of a sequence (default: all rows), which bounds the
    workspace.  ``window`` > 0: only the last ``window`` slots and the first ``n_sink``.  Rows of no
    sequence stay as they were.  No gradient is recorded.  Returns o, with ``return_lse`` (o, lse float32 [tokens, heads *
    G])."""
    import torch

    dev = pages.k.get_device()
    handle, on = _on(dev, stream)
    if on is not None:
        with on:
            return chunk_attention(q, pages, starts, heads=heads, units=units, longest=longest, window=window,
                                   n_sink=n_sink, return_lse=return_lse, out=out, lse=lse, workspace=workspace)
    if q.get_device() != dev or q.dtype != pages.k.dtype or q.dim() != 3 or not q.is_contiguous():
        raise ValueError("q must be a contiguous [tokens, query heads, d] tensor of the pool's type and device")
    T, Q, d = q.shape
    B = starts.shape[0] - 1 if starts.dim() else -1
    if B < 0:
        raise ValueError("starts must hold a number for each sequence and one more")
    st = _step(pages, B, T, heads, units)
    if d != pages._c.head_dim or st.heads < 1 or Q < 1 or Q % st.heads:
        raise ValueError("q %s does not fit %d heads of %d columns" % (tuple(q.shape), st.heads, pages._c.head_dim))
    longest = max(T, 1) if longest is None else int(longest)
    _int32(longest | window | n_sink)
    ch = _Chunk(Q // st.heads, longest, window, n_sink)
    out, lse, lp = _outputs(q, (T, Q), dev, out, lse, return_lse)
    L = lib()
    workspace = _workspace(workspace, L.grkv_chunk_attention_workspace_bytes(pages._c, st, ch), dev)
    _check(L.grkv_chunk_attention(q.data_ptr(), pages._c, st, _vector(starts, "starts", torch.int32, B + 1, dev), ch,
                                  out.data_ptr(), lp, handle, workspace.data_ptr(), workspace.numel()))
    return (out, lse) if return_lse else out
