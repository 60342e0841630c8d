"""Python binding of libpark (ctypes).  Argument marshalling only.

Every function here has the name of the C entry point it calls, takes torch
tensors that live on the GPU, allocates its outputs with torch (PyTorch is
used for device memory and streams only) and launches on torch's current
stream.  All computation happens in the HIP kernels of libpark.so; when the
library is missing every call raises instead of falling back to anything.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import json
import os

import torch

PARK_OK, PARK_ERR_INVALID_ARG, PARK_ERR_UNSUPPORTED, PARK_ERR_WORKSPACE = 0, 1, 2, 3
PARK_ERR_HIP, PARK_ERR_NUMERIC = 4, 5
PARK_F32, PARK_BF16 = 0, 1
PARK_METRIC_EUCLID, PARK_METRIC_QRKC = 0, 1
PARK_SELECT_TOPK, PARK_SELECT_TOPP = 0, 1
PARK_RECOMPUTE, PARK_REUSE_CLUSTERS, PARK_REUSE_CLUSTERS_AND_MASK = 0, 1, 2
PARK_EST_PAMA, PARK_EST_QCENTROID = 0, 1
PARK_BLOCKS_CLUSTER, PARK_BLOCKS_FIXED = 0, 1
PARK_INIT_SEEDED, PARK_INIT_WARM = 0, 1

LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libpark.so")

# names of every entry point declared in include/park.h
EXPORTS = (
    "park_workspace_size", "park_cluster_keys", "park_gather_rows", "park_block_centroids",
    "park_retrieve_blocks", "park_block_sparse_attn", "park_forward", "park_check",
    "park_status_string", "park_last_error", "park_profile_enable", "park_profile_reset",
    "park_profile_read", "park_schedule_step", "park_state_sizes", "park_probe_exp2",
    "park_probe_mfma_bf16", "park_probe_mfma_f16", "park_block_sparse_attn_static",
    "park_attention_workspace_size", "park_attention", "park_attention_backward",
    "park_cache_append", "park_cache_workspace_size", "park_cache_attention",
)


class ParkError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"park status {status}: {msg}")
        self.status = status


class Dims(C.Structure):
    _fields_ = [("H", C.c_int32), ("N", C.c_int32), ("d", C.c_int32), ("dtype", C.c_int32)]


class Params(C.Structure):
    _fields_ = [("CQ", C.c_int32), ("CK", C.c_int32), ("T", C.c_int32), ("select", C.c_int32),
                ("topk_ratio", C.c_double), ("topp", C.c_double), ("alpha", C.c_double),
                ("eps", C.c_double), ("s_min", C.c_double), ("seed", C.c_uint64),
                ("key_metric", C.c_int32), ("out_dtype", C.c_int32),
                ("estimator", C.c_int32), ("block_mode", C.c_int32), ("init", C.c_int32)]


class State(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("q_perm", "k_perm", "q_offsets", "k_offsets",
                                          "k_centroids", "k_sizes", "kv_count", "kv_index",
                                          "Qp", "Kp", "Vp", "W", "q_mu", "k_mu")]


class Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("batch", C.c_int64), ("head", C.c_int64), ("row", C.c_int64)]


class AttnDims(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("B", "Hq", "Hkv", "Nq", "Nk", "d", "dtype", "out_dtype")]


class AttnOpts(C.Structure):
    _fields_ = [("scale", C.c_double), ("softcap", C.c_double), ("slopes", C.c_void_p),
                ("causal", C.c_int32), ("q_pos", C.c_int32), ("prefix", C.c_void_p),
                ("q_doc", C.c_void_p), ("k_doc", C.c_void_p)]


class KvCache(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_exp", C.c_void_p), ("v_exp", C.c_void_p),
                ("n_pages", C.c_int32), ("page", C.c_int32), ("Hkv", C.c_int32), ("d", C.c_int32),
                ("status", C.c_void_p)]


_lib = None


def lib():
    """The loaded libpark.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: build it with __graft_entry__.build()")
    L = C.CDLL(LIB_PATH)
    vp, i32, u64, f64, sz = C.c_void_p, C.c_int32, C.c_uint64, C.c_double, C.c_size_t
    pd = C.POINTER(Dims)
    sig = {
        "park_workspace_size": [pd, i32, i32, C.POINTER(C.c_size_t)],
        "park_cluster_keys": [vp, vp, pd, i32, i32, u64, i32, i32, f64, f64, f64, vp, vp, vp, vp,
                              vp, vp, sz, vp],
        "park_gather_rows": [vp, vp, pd, vp, vp],
        "park_block_centroids": [vp, vp, vp, pd, i32, vp, vp, vp],
        "park_retrieve_blocks": [vp, vp, vp, vp, pd, i32, i32, i32, f64, vp, vp, vp, vp, sz, vp],
        "park_block_sparse_attn": [vp, vp, vp, vp, vp, vp, vp, vp, pd, i32, i32, vp, i32, vp, vp,
                                   sz, vp],
        "park_block_sparse_attn_static": [vp, vp, vp, vp, vp, vp, vp, vp, pd, i32, i32, vp, i32,
                                          vp, vp],
        "park_state_sizes": [pd, i32, i32, C.POINTER(C.c_size_t), i32],
        "park_forward": [vp, vp, vp, pd, C.POINTER(Params), i32, C.POINTER(State), vp, vp, sz,
                         vp],
        "park_attention_workspace_size": [vp, vp, i32, C.POINTER(C.c_size_t)],
        "park_attention": [vp, vp, vp, vp, vp, vp, vp, vp, sz, vp],
        "park_attention_backward": [vp] * 13 + [sz, vp],
        "park_cache_append": [vp, vp, vp, i32, i32, i32, vp, i32, vp, vp, vp],
        "park_cache_workspace_size": [vp, vp, i32, C.POINTER(C.c_size_t)],
        "park_cache_attention": [vp, vp, vp, i32, vp, vp, vp, vp, vp, vp, vp, sz, vp],
        "park_check": [vp, vp],
        "park_probe_exp2": [vp, vp, C.c_int64, vp],
        "park_probe_mfma_bf16": [vp, vp, vp, vp, i32, i32, vp],
        "park_probe_mfma_f16": [vp, vp, vp, vp, i32, i32, vp],
        "park_schedule_step": [i32, C.POINTER(C.c_int32), i32, C.POINTER(C.c_int32)],
        "park_status_string": [i32],
        "park_last_error": [],
        "park_profile_enable": [i32],
        "park_profile_reset": [],
        "park_profile_read": [C.c_char_p, sz],
    }
    for name, args in sig.items():
        f = getattr(L, name)
        f.argtypes = args
        f.restype = C.c_char_p if name in ("park_status_string", "park_last_error") else C.c_int
    _lib = L
    return L


def _check(status: int):
    if status != PARK_OK:
        raise ParkError(status, lib().park_last_error().decode())


def _ptr(t):
    return None if t is None else C.c_void_p(t.data_ptr())


def _stream():
    return C.c_void_p(torch.cuda.current_stream().cuda_stream)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.float32:
        return PARK_F32
    if t.dtype == torch.bfloat16:
        return PARK_BF16
    raise TypeError(f"unsupported dtype {t.dtype}")


def _dims(X: torch.Tensor) -> Dims:
    if X.dim() != 3 or not X.is_cuda or not X.is_contiguous():
        raise ValueError("expected a contiguous [H, N, d] CUDA tensor")
    H, N, d = X.shape
    return Dims(H, N, d, _dtype_code(X))


def _dev(X):
    return dict(device=X.device)


def park_workspace_size(H: int, N: int, d: int, dtype: int, CQ: int, CK: int) -> int:
    out = C.c_size_t(0)
    dims = Dims(H, N, d, dtype)
    _check(lib().park_workspace_size(C.byref(dims), CQ, CK, C.byref(out)))
    return out.value


def workspace(X: torch.Tensor, CQ: int, CK: int) -> torch.Tensor:
    H, N, d = X.shape
    n = park_workspace_size(H, N, d, _dtype_code(X), CQ, CK)
    return torch.empty(n, dtype=torch.uint8, device=X.device)


def park_cluster_keys(X, C_: int, T: int, seed: int = 0, side: int = 1,
                      metric: int = PARK_METRIC_QRKC, Qmetric=None, alpha: float = 0.05,
                      eps: float = 1e-6, s_min: float = 1e-12, want_R: bool = False,
                      want_Xt: bool = False, ws=None):
    """k-means of one side; returns dict(labels, perm, offsets[, R, Xt])."""
    dims = _dims(X)
    H, N, d = X.shape
    ws = workspace(X, C_, C_) if ws is None else ws
    out = {"labels": torch.empty(H, N, dtype=torch.int32, **_dev(X)),
           "perm": torch.empty(H, N, dtype=torch.int32, **_dev(X)),
           "offsets": torch.empty(H, C_ + 1, dtype=torch.int32, **_dev(X))}
    if want_R:
        out["R"] = torch.empty(H, d, d, dtype=torch.float64, **_dev(X))
    if want_Xt:
        out["Xt"] = torch.empty(H, N, d, dtype=torch.float32, **_dev(X))
    _check(lib().park_cluster_keys(
        _ptr(X), _ptr(Qmetric), C.byref(dims), C_, T, seed, side, metric, alpha, eps, s_min,
        _ptr(out["labels"]), _ptr(out["perm"]), _ptr(out["offsets"]), _ptr(out.get("R")),
        _ptr(out.get("Xt")), _ptr(ws), ws.numel(), _stream()))
    out["ws"] = ws
    return out


def park_gather_rows(X, perm):
    dims = _dims(X)
    Xp = torch.empty_like(X)
    _check(lib().park_gather_rows(_ptr(X), _ptr(perm), C.byref(dims), _ptr(Xp), _stream()))
    return Xp


def park_block_centroids(X, perm, offsets, C_: int):
    dims = _dims(X)
    H, N, d = X.shape
    cen = torch.empty(H, C_, d, dtype=torch.float32, **_dev(X))
    sizes = torch.empty(H, C_, dtype=torch.int32, **_dev(X))
    _check(lib().park_block_centroids(_ptr(X), _ptr(perm), _ptr(offsets), C.byref(dims), C_,
                                      _ptr(cen), _ptr(sizes), _stream()))
    return cen, sizes


def park_retrieve_blocks(Qp, q_offsets, centroids, k_sizes, CQ: int, CK: int, select: int,
                         param: float, want_W: bool = False, ws=None):
    """Returns (kv_count [H,CQ], kv_index [H,CQ,CK], W [H,CQ,CK] or None)."""
    dims = _dims(Qp)
    H = Qp.shape[0]
    ws = workspace(Qp, CQ, CK) if ws is None else ws
    kv_count = torch.empty(H, CQ, dtype=torch.int32, **_dev(Qp))
    kv_index = torch.empty(H, CQ, CK, dtype=torch.int32, **_dev(Qp))
    W = torch.empty(H, CQ, CK, dtype=torch.float32, **_dev(Qp)) if want_W else None
    _check(lib().park_retrieve_blocks(_ptr(Qp), _ptr(q_offsets), _ptr(centroids), _ptr(k_sizes),
                                      C.byref(dims), CQ, CK, select, param, _ptr(W),
                                      _ptr(kv_count), _ptr(kv_index), _ptr(ws), ws.numel(),
                                      _stream()))
    return kv_count, kv_index, W


def park_block_sparse_attn(Qp, Kp, Vp, q_offsets, k_offsets, kv_count, kv_index, q_perm,
                           CQ: int, CK: int, out_dtype: int = PARK_F32, ws=None,
                           want_lse: bool = False):
    """Returns O, or (O, lse [H, N] float32) when want_lse."""
    dims = _dims(Qp)
    O = torch.empty(Qp.shape, dtype=torch.float32 if out_dtype == PARK_F32 else torch.bfloat16,
                    **_dev(Qp))
    lse = torch.empty(Qp.shape[:2], dtype=torch.float32, **_dev(Qp)) if want_lse else None
    ws = workspace(Qp, CQ, CK) if ws is None else ws
    _check(lib().park_block_sparse_attn(_ptr(Qp), _ptr(Kp), _ptr(Vp), _ptr(q_offsets),
                                        _ptr(k_offsets), _ptr(kv_count), _ptr(kv_index),
                                        _ptr(q_perm), C.byref(dims), CQ, CK, _ptr(O), out_dtype,
                                        _ptr(lse), _ptr(ws), ws.numel(), _stream()))
    return (O, lse) if want_lse else O


def park_block_sparse_attn_static(Qp, Kp, Vp, q_offsets, k_offsets, kv_count, kv_index, q_perm,
                                  CQ: int, CK: int, out_dtype: int = PARK_F32, O=None, lse=None):
    """The workspace-free entry point: writes into the given O (and lse) tensors,
    allocating nothing when both are given; returns (O, lse)."""
    dims = _dims(Qp)
    if O is None:
        O = torch.empty(Qp.shape, dtype=torch.float32 if out_dtype == PARK_F32
                        else torch.bfloat16, **_dev(Qp))
    _check(lib().park_block_sparse_attn_static(_ptr(Qp), _ptr(Kp), _ptr(Vp), _ptr(q_offsets),
                                               _ptr(k_offsets), _ptr(kv_count), _ptr(kv_index),
                                               _ptr(q_perm), C.byref(dims), CQ, CK, _ptr(O),
                                               out_dtype, _ptr(lse), _stream()))
    return O, lse


STATE_FIELDS = ("q_perm", "k_perm", "q_offsets", "k_offsets", "k_centroids", "k_sizes",
                "kv_count", "kv_index", "Qp", "Kp", "Vp", "W", "q_mu", "k_mu")


def park_state_sizes(H: int, N: int, d: int, dtype: int, CQ: int, CK: int) -> dict:
    """Bytes of each park_state buffer, keyed by member name."""
    n = len(STATE_FIELDS)
    out = (C.c_size_t * n)()
    dims = Dims(H, N, d, dtype)
    _check(lib().park_state_sizes(C.byref(dims), CQ, CK, out, n))
    return dict(zip(STATE_FIELDS, out))


def make_params(CQ, CK, T=10, select="topk", ratio=0.25, topp=0.9, alpha=0.05, eps=1e-6,
                s_min=1e-12, seed=0, key_metric=PARK_METRIC_QRKC, out_dtype=PARK_F32,
                estimator=PARK_EST_PAMA, block_mode=PARK_BLOCKS_CLUSTER,
                init=PARK_INIT_SEEDED) -> Params:
    sel = PARK_SELECT_TOPK if select in ("topk", PARK_SELECT_TOPK) else PARK_SELECT_TOPP
    return Params(CQ, CK, T, sel, ratio, topp, alpha, eps, s_min, seed, key_metric, out_dtype,
                  estimator, block_mode, init)


def make_state(Q, CQ: int, CK: int, want_W: bool = False, want_mu: bool = False) -> dict:
    """Caller-owned device buffers for park_forward (a dict of tensors); want_mu
    adds the float64 centroids a warm-started recomputation reads and every
    recomputation writes."""
    H, N, d = Q.shape
    i32 = dict(dtype=torch.int32, **_dev(Q))
    st = {"q_perm": torch.empty(H, N, **i32), "k_perm": torch.empty(H, N, **i32),
          "q_offsets": torch.empty(H, CQ + 1, **i32), "k_offsets": torch.empty(H, CK + 1, **i32),
          "k_centroids": torch.empty(H, CK, d, dtype=torch.float32, **_dev(Q)),
          "k_sizes": torch.empty(H, CK, **i32), "kv_count": torch.empty(H, CQ, **i32),
          "kv_index": torch.empty(H, CQ, CK, **i32), "Qp": torch.empty_like(Q),
          "Kp": torch.empty_like(Q), "Vp": torch.empty_like(Q),
          "W": torch.empty(H, CQ, CK, dtype=torch.float32, **_dev(Q)) if want_W else None,
          "q_mu": torch.empty(H, CQ, d, dtype=torch.float64, **_dev(Q)) if want_mu else None,
          "k_mu": torch.empty(H, CK, d, dtype=torch.float64, **_dev(Q)) if want_mu else None}
    return st


def _state_struct(st: dict) -> State:
    return State(*[(None if st.get(n) is None else st[n].data_ptr()) for n, _ in State._fields_])


def park_forward(Q, K, V, params: Params, reuse: int = PARK_RECOMPUTE, state: dict | None = None,
                 out=None, ws=None):
    """Whole layer; returns (O, state).  `state` is a dict from make_state."""
    dims = _dims(Q)
    state = make_state(Q, params.CQ, params.CK) if state is None else state
    ws = workspace(Q, params.CQ, params.CK) if ws is None else ws
    if out is None:
        out = torch.empty(Q.shape, dtype=torch.float32 if params.out_dtype == PARK_F32
                          else torch.bfloat16, **_dev(Q))
    s = _state_struct(state)
    _check(lib().park_forward(_ptr(Q), _ptr(K), _ptr(V), C.byref(dims), C.byref(params), reuse,
                              C.byref(s), _ptr(out), _ptr(ws), ws.numel(), _stream()))
    return out, state


PARK_STEP_DENSE = -1


def park_schedule_step(step: int, steps) -> int:
    """Mode of denoising step `step` under the recomputation set `steps`:
    PARK_RECOMPUTE, PARK_REUSE_CLUSTERS_AND_MASK or PARK_STEP_DENSE."""
    arr = (C.c_int32 * len(steps))(*steps)
    out = C.c_int32(0)
    _check(lib().park_schedule_step(int(step), arr, len(steps), C.byref(out)))
    return out.value


def park_probe_exp2(x):
    """2^x by the device's v_exp_f32 (x: float32 CUDA tensor)."""
    x = x.contiguous()
    y = torch.empty_like(x)
    _check(lib().park_probe_exp2(_ptr(x), _ptr(y), x.numel(), _stream()))
    return y


def _probe_mfma(fn, A, Bt, C0):
    A, Bt, C0 = A.contiguous(), Bt.contiguous(), C0.contiguous()
    out = torch.empty_like(C0)
    _check(fn(_ptr(A), _ptr(Bt), _ptr(C0), _ptr(out), A.shape[0], A.shape[2], _stream()))
    return out


def park_probe_mfma_bf16(A, Bt, C0):
    """C0 + A Bt^T by a chain of 32x32x16 bf16 MFMAs (A, Bt: [P, 32, K] bf16, C0: [P, 32, 32])."""
    return _probe_mfma(lib().park_probe_mfma_bf16, A, Bt, C0)


def park_probe_mfma_f16(A, Bt, C0):
    """The same by 32x32x16 f16 MFMAs (A, Bt: [P, 32, K] f16)."""
    return _probe_mfma(lib().park_probe_mfma_f16, A, Bt, C0)


# ---------------------------------------------------------------------------
# dense attention and the 8-bit key/value cache
# ---------------------------------------------------------------------------


def _view(t: torch.Tensor, name: str, like: torch.Tensor | None = None, dtype=None, shape=None):
    """A [B, H, N, d] (or [H, N, d]) tensor as a Rows struct; its elements of a
    row are contiguous, the other strides are its own."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dim() not in (3, 4):
        raise ValueError(f"{name}: expected a [B, H, N, d] or [H, N, d] CUDA tensor")
    if like is not None and (t.device != like.device or t.dim() != like.dim()):
        raise ValueError(f"{name}: not on the same device, or not of as many dimensions, as Q")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name}: expected {dtype}, got {t.dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    s = t.stride()
    if t.shape[-1] > 1 and s[-1] != 1:
        raise ValueError(f"{name}: the last dimension must be contiguous")
    return Rows(t.data_ptr(), s[0] if t.dim() == 4 else 0, s[-3], s[-2])


def _array(t, name: str, dtype, shape, device):
    """Device pointer of a contiguous tensor (None: NULL)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.device != device or t.dtype != dtype \
            or tuple(t.shape) != tuple(shape) or not t.is_contiguous():
        raise ValueError(f"{name}: expected a contiguous {dtype} tensor of shape {tuple(shape)} "
                         f"on {device}")
    return t.data_ptr()


def _attn_dims(Q, Hkv, Nk, out_dtype) -> AttnDims:
    B = Q.shape[0] if Q.dim() == 4 else 1
    H, N, d = Q.shape[-3:]
    return AttnDims(B, H, Hkv, N, Nk, d, _dtype_code(Q), out_dtype)


def _attn_opts(m: AttnDims, dev, scale, softcap, slopes, causal, q_pos, prefix, q_doc,
               k_doc) -> AttnOpts:
    if (q_doc is None) != (k_doc is None):
        raise ValueError("q_doc and k_doc come together")
    return AttnOpts(m.d ** -0.5 if scale is None else scale, softcap,
                    _array(slopes, "slopes", torch.float32, (m.Hq,), dev), int(causal),
                    m.Nk - m.Nq if q_pos is None else q_pos,
                    _array(prefix, "prefix", torch.int32, (m.B,), dev),
                    _array(q_doc, "q_doc", torch.int32, (m.B, m.Nq), dev),
                    _array(k_doc, "k_doc", torch.int32, (m.B, m.Nk), dev))


def _code_of(dtype) -> int:
    if dtype not in (torch.float32, torch.bfloat16):
        raise TypeError(f"unsupported output dtype {dtype}")
    return PARK_F32 if dtype == torch.float32 else PARK_BF16


def _scratch(ws, need: int, dev):
    """(workspace tensor to keep until the call, pointer, bytes)"""
    if ws is None:
        ws = torch.empty(need, dtype=torch.uint8, device=dev) if need else None
    elif not ws.is_cuda or ws.device != dev or ws.dtype != torch.uint8 or not ws.is_contiguous():
        raise ValueError(f"ws: expected a contiguous uint8 tensor on {dev}")
    return ws, (None if ws is None else ws.data_ptr()), (0 if ws is None else ws.numel())


def _stream_of(dev):
    return torch.cuda.current_stream(dev).cuda_stream


def _on(dev):
    """Makes dev the current device for a call (nothing to do if it is)."""
    return contextlib.nullcontext() if torch.cuda.current_device() == dev.index else torch.cuda.device(dev)


def park_attention_workspace_size(dims: AttnDims, opts: AttnOpts, backward: bool) -> int:
    out = C.c_size_t(0)
    _check(lib().park_attention_workspace_size(C.byref(dims), C.byref(opts), int(backward),
                                               C.byref(out)))
    return out.value


def park_attention(Q, K, V, *, scale=None, softcap: float = 0.0, slopes=None,
                   causal: bool = False, q_pos=None, prefix=None, q_doc=None, k_doc=None,
                   out_dtype=None, out=None, lse=None, want_lse: bool = False, ws=None):
    """Dense attention of Q [B, Hq, Nq, d] over K, V [B, Hkv, Nk, d] (or all
    without B); any strides with contiguous rows.  Returns O, or (O, lse) with
    want_lse or a given lse [B, Hq, Nq] float32.

    scale (1/sqrt(d)), softcap (0: none), slopes [Hq] float32, causal, q_pos (the
    position of query 0 among the keys, Nk - Nq), prefix [B] int32 (causal only)
    and the documents q_doc [B, Nq], k_doc [B, Nk] int32 are park_attn_opts of
    include/park.h.  O has Q's dtype unless out or out_dtype says otherwise.

    As everywhere here autograd sees nothing of the call: O carries no history,
    whatever Q, K and V require.  The gradient is park_attention_backward, which a
    torch.autograd.Function's backward can call with what its forward kept.
    """
    q = _view(Q, "Q")
    Hkv, Nk = (K.shape[-3], K.shape[-2]) if K.dim() == Q.dim() else (0, 0)
    shape = (*Q.shape[:-3], Hkv, Nk, Q.shape[-1])
    k, v = _view(K, "K", Q, Q.dtype, shape), _view(V, "V", Q, Q.dtype, shape)
    dev = Q.device
    if out is None:
        out = torch.empty(Q.shape, dtype=out_dtype or Q.dtype, device=dev)
    o = _view(out, "out", Q, out_dtype, Q.shape)
    m = _attn_dims(Q, Hkv, Nk, _code_of(out.dtype))
    opts = _attn_opts(m, dev, scale, softcap, slopes, causal, q_pos, prefix, q_doc, k_doc)
    if lse is None and want_lse:
        lse = torch.empty(Q.shape[:-1], dtype=torch.float32, device=dev)
    lp = _array(lse, "lse", torch.float32, Q.shape[:-1], dev)
    with _on(dev):
        need = park_attention_workspace_size(m, opts, False) if ws is None else 0
        ws, wp, wn = _scratch(ws, need, dev)
        _check(lib().park_attention(C.byref(q), C.byref(k), C.byref(v), C.byref(m), C.byref(opts),
                                    C.byref(o), lp, wp, wn, _stream_of(dev)))
    return out if lse is None else (out, lse)


def park_attention_backward(dO, Q, K, V, O, lse, *, dlse=None, scale=None, softcap: float = 0.0,
                            slopes=None, causal: bool = False, q_pos=None, prefix=None, q_doc=None,
                            k_doc=None, dQ=None, dK=None, dV=None, ws=None):
    """Gradients (dQ, dK, dV) of park_attention for the same arguments, from its
    O and lse, the output gradient dO (Q's dtype) and, if given, that of lse."""
    q = _view(Q, "Q")
    Hkv, Nk = (K.shape[-3], K.shape[-2]) if K.dim() == Q.dim() else (0, 0)
    shape = (*Q.shape[:-3], Hkv, Nk, Q.shape[-1])
    k, v = _view(K, "K", Q, Q.dtype, shape), _view(V, "V", Q, Q.dtype, shape)
    g, o = _view(dO, "dO", Q, Q.dtype, Q.shape), _view(O, "O", Q, None, Q.shape)
    dev = Q.device
    dQ = torch.empty(Q.shape, dtype=Q.dtype, device=dev) if dQ is None else dQ
    dK = torch.empty(shape, dtype=Q.dtype, device=dev) if dK is None else dK
    dV = torch.empty(shape, dtype=Q.dtype, device=dev) if dV is None else dV
    gq, gk, gv = (_view(t, n, Q, Q.dtype, s) for t, n, s in
                  ((dQ, "dQ", Q.shape), (dK, "dK", shape), (dV, "dV", shape)))
    m = _attn_dims(Q, Hkv, Nk, _code_of(O.dtype))
    opts = _attn_opts(m, dev, scale, softcap, slopes, causal, q_pos, prefix, q_doc, k_doc)
    lp = _array(lse, "lse", torch.float32, Q.shape[:-1], dev)
    dlp = _array(dlse, "dlse", torch.float32, Q.shape[:-1], dev)
    with _on(dev):
        need = park_attention_workspace_size(m, opts, True) if ws is None else 0
        ws, wp, wn = _scratch(ws, need, dev)
        _check(lib().park_attention_backward(
            C.byref(g), C.byref(q), C.byref(k), C.byref(v), C.byref(o), lp, dlp, C.byref(m),
            C.byref(opts), C.byref(gq), C.byref(gk), C.byref(gv), wp, wn, _stream_of(dev)))
    return dQ, dK, dV


CACHE_FIELDS = ("k", "v", "k_exp", "v_exp")


def make_kv_cache(n_pages: int, Hkv: int, page: int, d: int, device="cuda") -> dict:
    """Empty 8-bit cache: a dict of its device buffers (park_kv_cache), with a
    status word that park_check reads."""
    pool = dict(dtype=torch.uint8, device=device)
    exps = dict(dtype=torch.int8, device=device)
    return {"k": torch.zeros(n_pages, Hkv, page, d, **pool),
            "v": torch.zeros(n_pages, Hkv, page, d, **pool),
            "k_exp": torch.zeros(n_pages, Hkv, **exps), "v_exp": torch.zeros(n_pages, Hkv, **exps),
            "status": torch.zeros(1, dtype=torch.int32, device=device)}


def _cache_struct(cache: dict, dev) -> KvCache:
    shape = cache["k"].shape
    if len(shape) != 4:
        raise ValueError("cache k: expected [n_pages, Hkv, page, d]")
    status = cache.get("status")
    return KvCache(_array(cache["k"], "cache k", torch.uint8, shape, dev),
                   _array(cache["v"], "cache v", torch.uint8, shape, dev),
                   _array(cache["k_exp"], "cache k_exp", torch.int8, shape[:2], dev),
                   _array(cache["v_exp"], "cache v_exp", torch.int8, shape[:2], dev),
                   shape[0], shape[2], shape[1], shape[3],
                   _array(status, "cache status", torch.int32, (1,), dev))


def _table(block_table, B: int, dev):
    if not isinstance(block_table, torch.Tensor) or block_table.dim() != 2:
        raise ValueError("block_table: expected a [B, max_pages] tensor")
    n = block_table.shape[1]
    return _array(block_table, "block_table", torch.int32, (B, n), dev), n


def park_cache_append(cache: dict, K, V, block_table, lens, n_new=None):
    """Writes rows 0 .. n_new[b] - 1 (None: all) of K, V [B, Hkv, N, d] as tokens
    lens[b] .. of sequence b into the pages block_table [B, max_pages] names
    (int32, as lens and n_new [B]; lens is not changed)."""
    k = _view(K, "K")
    v = _view(V, "V", K, K.dtype, K.shape)
    if K.dim() != 4:
        raise ValueError("K: expected [B, Hkv, N, d]")
    B, Hkv, N, d = K.shape
    dev = K.device
    c = _cache_struct(cache, dev)
    if (Hkv, d) != (c.Hkv, c.d):
        raise ValueError(f"K has Hkv = {Hkv}, d = {d}, the cache {c.Hkv}, {c.d}")
    table, n = _table(block_table, B, dev)
    lp = _array(lens, "lens", torch.int32, (B,), dev)
    np_ = _array(n_new, "n_new", torch.int32, (B,), dev)
    with _on(dev):
        _check(lib().park_cache_append(C.byref(c), C.byref(k), C.byref(v), B, N, _dtype_code(K),
                                       table, n, lp, np_, _stream_of(dev)))


def park_cache_workspace_size(cache: KvCache, dims: AttnDims, max_pages: int) -> int:
    out = C.c_size_t(0)
    _check(lib().park_cache_workspace_size(C.byref(cache), C.byref(dims), max_pages, C.byref(out)))
    return out.value


def park_cache_attention(Q, cache: dict, block_table, lens, *, q_lens=None, scale=None,
                         softcap: float = 0.0, slopes=None, causal: bool = True, prefix=None,
                         out_dtype=None, out=None, lse=None, want_lse: bool = False, ws=None):
    """park_attention of Q [B, Hq, Nq, d] (bf16), the last q_lens[b] (None: Nq)
    tokens of sequences of lens[b] tokens, over the cache.  Rows past q_lens[b]
    of O and lse are not written."""
    q = _view(Q, "Q")
    if Q.dim() != 4:
        raise ValueError("Q: expected [B, Hq, Nq, d]")
    dev = Q.device
    c = _cache_struct(cache, dev)
    if out is None:
        out = torch.empty(Q.shape, dtype=out_dtype or Q.dtype, device=dev)
    o = _view(out, "out", Q, out_dtype, Q.shape)
    m = _attn_dims(Q, c.Hkv, 0, _code_of(out.dtype))
    opts = _attn_opts(m, dev, scale, softcap, slopes, causal, 0, prefix, None, None)
    if lse is None and want_lse:
        lse = torch.empty(Q.shape[:-1], dtype=torch.float32, device=dev)
    lse_p = _array(lse, "lse", torch.float32, Q.shape[:-1], dev)
    table, n = _table(block_table, m.B, dev)
    lp = _array(lens, "lens", torch.int32, (m.B,), dev)
    qp = _array(q_lens, "q_lens", torch.int32, (m.B,), dev)
    with _on(dev):
        need = park_cache_workspace_size(c, m, n) if ws is None else 0
        ws, wp, wn = _scratch(ws, need, dev)
        _check(lib().park_cache_attention(C.byref(q), C.byref(c), table, n, lp, qp, C.byref(m),
                                          C.byref(opts), C.byref(o), lse_p, wp, wn,
                                          _stream_of(dev)))
    return out if lse is None else (out, lse)


def park_check(ws):
    """Synchronises and raises ParkError if the last call on `ws` failed on the device."""
    _check(lib().park_check(_ptr(ws), _stream()))


def park_profile_enable(on: bool = True):
    _check(lib().park_profile_enable(1 if on else 0))


def park_profile_reset():
    _check(lib().park_profile_reset())


def park_profile_read() -> dict:
    buf = C.create_string_buffer(1 << 16)
    _check(lib().park_profile_read(buf, len(buf)))
    return json.loads(buf.value.decode())
