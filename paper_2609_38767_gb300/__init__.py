"""GB300 (sm_103a) training-data-attribution hot path of the dattri-LLM paper.

Python binding of the C ABI in ``include/tda.h``: every function here has the
name and argument order of its C entry point and only marshals arguments
(torch tensors become device pointers, ``stream=None`` becomes torch's current
CUDA stream). All computation happens in ``libtda.so``. Importing this package
loads nothing; the first call loads the library and raises if it is missing,
so there is no silent CPU path.
"""
from __future__ import annotations

import ctypes
import importlib
import os
import threading

__all__ = [
    "LayerDesc", "TdaError", "load", "tda_proj_entries", "tda_workspace_size", "tda_project",
    "tda_project_engine", "tda_project_host_ws_min", "tda_project_host", "tda_noalloc_scratch_bytes",
    "tda_project_materialized_noalloc",
    "tda_similarity_projected", "tda_similarity_exact", "tda_norms", "tda_cosine", "tda_kfac_state_bytes", "tda_kfac_workspace_size",
    "tda_kfac_reset", "tda_kfac_accumulate_factors", "tda_project_kfac", "tda_kfac_eigen",
    "tda_kfac_accumulate_eigenvalues", "tda_kfac_apply",
    "tda_token_scores_workspace_size", "tda_token_scores", "tda_mask_gather", "tda_precondition_state_bytes", "tda_precondition",
    "tda_precondition_info", "tda_score", "tda_score_engine", "tda_similarity_gram_engine", "tda_topk", "tda_route", "tda_route_calibrate",
    "tda_route_set_model", "tda_device_status", "tda_selftest_bounded_wait", "tda_last_error", "tda_version", "tda_launch_count",
    "tda_set_sm_budget", "tda_get_sm_budget",
    "TensorRef", "tensor_list", "tda_embedding_forward", "tda_embedding_workspace_size", "tda_embedding_backward",
    "tda_grad_clip_workspace_size", "tda_grad_clip",
    "LinearDesc", "tda_linear_workspace_size", "tda_linear_forward", "tda_linear_backward",
    "AttentionDesc", "tda_attention_workspace_size", "tda_attention_ranges", "tda_position_buckets", "tda_attention_forward",
    "tda_attention_backward", "tda_rmsnorm_forward", "tda_rmsnorm_workspace_size", "tda_rmsnorm_backward",
]

_HERE = os.path.dirname(os.path.abspath(__file__))
_lock = threading.Lock()
_lib = None

# enums of include/tda.h
TDA_OK, TDA_ERR_INVALID_ARG, TDA_ERR_UNSUPPORTED, TDA_ERR_WORKSPACE = 0, 1, 2, 3
TDA_ERR_CUDA, TDA_ERR_NOT_SPD, TDA_ERR_TIMEOUT = 4, 5, 6
TDA_F32, TDA_BF16, TDA_F64 = 0, 1, 2
TDA_PROJ_RADEMACHER, TDA_PROJ_IDENTITY = 0, 1
TDA_ROUTE_AUTO, TDA_ROUTE_FACTORED, TDA_ROUTE_MATERIALIZE, TDA_ROUTE_GRAM = -1, 0, 1, 2
TDA_OP_PROJECT, TDA_OP_SIMILARITY_PROJECTED, TDA_OP_SIMILARITY_EXACT = 0, 1, 2
TDA_OP_NORM_PROJECTED, TDA_OP_NORM_EXACT = 3, 4
TDA_PC_RESET, TDA_PC_FIT_ACCUM, TDA_PC_FACTOR, TDA_PC_APPLY, TDA_PC_FACTOR_APPLY = 0, 1, 2, 3, 4
TDA_KFAC, TDA_EKFAC = 0, 1
TDA_I32, TDA_I64 = 0, 1
TDA_ACT_NONE, TDA_ACT_RELU, TDA_ACT_GELU, TDA_ACT_GELU_TANH, TDA_ACT_SILU = 0, 1, 2, 3, 4
TDA_LINEAR_FORWARD, TDA_LINEAR_BACKWARD, TDA_LINEAR_ANY_STRIDE = 0, 1, 256
TDA_ATTENTION_FORWARD, TDA_ATTENTION_BACKWARD = 0, 1
TDA_CALIBRATE_WS_BYTES = 768 << 20
_STATUS = {0: "TDA_OK", 1: "TDA_ERR_INVALID_ARG", 2: "TDA_ERR_UNSUPPORTED", 3: "TDA_ERR_WORKSPACE",
           4: "TDA_ERR_CUDA", 5: "TDA_ERR_NOT_SPD", 6: "TDA_ERR_TIMEOUT"}


class LayerDesc(ctypes.Structure):
    """tda_layer_desc."""
    _fields_ = [("d_in", ctypes.c_int64), ("d_out", ctypes.c_int64), ("T", ctypes.c_int64),
                ("k_in", ctypes.c_int32), ("k_out", ctypes.c_int32), ("seed", ctypes.c_uint64),
                ("layer", ctypes.c_uint32), ("kind", ctypes.c_int32)]

    def __init__(self, d_in, d_out, T, k_in, k_out, seed=0, layer=0, kind=TDA_PROJ_RADEMACHER):
        super().__init__(d_in, d_out, T, k_in, k_out, seed, layer, kind)


class LinearDesc(ctypes.Structure):
    """tda_linear_desc."""
    _fields_ = [("d_in", ctypes.c_int64), ("d_out", ctypes.c_int64), ("act", ctypes.c_int32), ("dtype", ctypes.c_int32)]

    def __init__(self, d_in, d_out, act=TDA_ACT_NONE, dtype=TDA_BF16):
        super().__init__(d_in, d_out, act, dtype)


class AttentionDesc(ctypes.Structure):
    """tda_attention_desc."""
    _fields_ = [("N", ctypes.c_int64), ("T", ctypes.c_int64), ("heads", ctypes.c_int32), ("kv_heads", ctypes.c_int32),
                ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32), ("scale", ctypes.c_float), ("cap", ctypes.c_float),
                ("causal", ctypes.c_int32), ("n_buckets", ctypes.c_int32), ("max_distance", ctypes.c_int64)]

    def __init__(self, N, T, heads, kv_heads, head_dim, dtype=TDA_BF16, scale=None, cap=0.0, causal=True, n_buckets=0,
                 max_distance=0):
        super().__init__(N, T, heads, kv_heads, head_dim, dtype, scale if scale is not None else max(head_dim, 1) ** -0.5, cap,
                         int(causal), n_buckets, max_distance)


class TensorRef(ctypes.Structure):
    """tda_tensor_ref."""
    _fields_ = [("in_", ctypes.c_void_p), ("out", ctypes.c_void_p), ("n", ctypes.c_int64), ("dtype", ctypes.c_int32),
                ("pad", ctypes.c_int32)]


class TdaError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{_STATUS.get(status, status)}: {message}")
        self.status = status


def lib_path(name: str = "libtda.so") -> str:
    return os.path.join(_HERE, name)


def load() -> ctypes.CDLL:
    """Load libtda.so (built by ``build.build()``); raises if it is absent."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is not None:
            return _lib
        path = lib_path()
        if not os.path.exists(path):
            raise ImportError(f"{path} is missing: run paper_2609_38767_gb300.build.build() first")
        lib = ctypes.CDLL(path)
        P, I32, I64, U32, U64 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_int64, ctypes.c_uint32, ctypes.c_uint64
        D, F, SZ = ctypes.c_double, ctypes.c_float, ctypes.c_size_t
        LP = ctypes.POINTER(LayerDesc)
        sig = {
            "tda_proj_entries": (I32, [U64, U32, I32, I32, I64, I32, P, P]),
            "tda_workspace_size": (I32, [I32, LP, I32, I64, I64, I32, ctypes.POINTER(SZ)]),
            "tda_project": (I32, [LP, I32, P, P, I64, P, I64, I32, P, SZ, P]),
            "tda_project_engine": (I32, [LP, I32, P, P]),
            "tda_project_host_ws_min": (SZ, [LP, I32]),
            "tda_project_host": (I32, [LP, I32, P, P, I64, P, I64, P, SZ, P]),
            "tda_noalloc_scratch_bytes": (SZ, []),
            "tda_project_materialized_noalloc": (I32, [LP, I32, P, P, I64, P, I64, P]),
            "tda_similarity_projected": (I32, [LP, I32, P, P, I64, P, P, I64, P, I64, F, I32, P, SZ, P]),
            "tda_norms": (I32, [I32, LP, I32, P, P, I64, P, I32, P, SZ, P]),
            "tda_cosine": (I32, [P, I64, I64, I64, P, P, P]),
            "tda_similarity_exact": (I32, [LP, I32, P, P, I64, P, P, I64, P, I64, F, I32, P, SZ, P]),
            "tda_precondition_state_bytes": (SZ, [I64, I32]),
            "tda_kfac_state_bytes": (SZ, [I32, I32]),
            "tda_token_scores_workspace_size": (SZ, [LP]),
            "tda_token_scores": (I32, [LP, I32, P, P, I64, P, I64, I64, P, I64, F, P, SZ, P]),
            "tda_mask_gather": (I32, [LP, I32, P, P, I64, P, P, I64, P, I64, P]),
            "tda_kfac_workspace_size": (SZ, [LP, I32]),
            "tda_kfac_reset": (I32, [I32, I32, I32, P, P]),
            "tda_kfac_accumulate_factors": (I32, [LP, I32, P, P, I64, P, P, SZ, P]),
            "tda_project_kfac": (I32, [LP, I32, P, P, I64, P, I64, P, P, SZ, P]),
            "tda_kfac_eigen": (I32, [I32, I32, I32, P, P]),
            "tda_kfac_accumulate_eigenvalues": (I32, [I32, I32, I32, P, P, I64, I64, P, SZ, P]),
            "tda_kfac_apply": (I32, [I32, I32, I32, I32, P, D, D, P, I64, I64, P, I64, P]),
            "tda_precondition": (I32, [I32, I32, I64, I32, P, P, I64, I64, I64, D, D, P, I64, I64, P, I64, P]),
            "tda_precondition_info": (I32, [I32, I64, I32, P, ctypes.POINTER(D), P]),
            "tda_score": (I32, [P, I32, I64, I64, P, I64, I64, I64, P, I64, F, P]),
            "tda_topk": (I32, [P, I64, I64, I64, I32, P, P, P]),
            "tda_score_engine": (I32, [P, I32, I64, I64, P, I64, I64, I64]),
            "tda_similarity_gram_engine": (I32, [LP, I32, P, P, P, P]),
            "tda_route": (I32, [LP, I32, I64, I64, I32, ctypes.POINTER(I32), ctypes.POINTER(D)]),
            "tda_route_calibrate": (I32, [P, SZ, P, ctypes.POINTER(D)]),
            "tda_route_set_model": (I32, [I32]),
            "tda_device_status": (I32, [P]),
            "tda_selftest_bounded_wait": (I32, [U64, P]),
            "tda_last_error": (ctypes.c_char_p, []),
            "tda_version": (I32, []),
            "tda_launch_count": (U64, []),
            "tda_set_sm_budget": (I32, [I32]),
            "tda_get_sm_budget": (I32, []),
            "tda_linear_workspace_size": (I32, [I32, ctypes.POINTER(LinearDesc), I64, ctypes.POINTER(SZ)]),
            "tda_linear_forward": (I32, [ctypes.POINTER(LinearDesc), P, I64, I64, P, I64, P, P, I64, P, I64, P, I64, P,
                                         SZ, P]),
            "tda_linear_backward": (I32, [ctypes.POINTER(LinearDesc), P, I64, P, I64, I64, P, I64, P, I64, P, I64, P,
                                          I64, P, I64, P, I32, F, P, SZ, P]),
            "tda_attention_workspace_size": (I32, [I32, ctypes.POINTER(AttentionDesc), ctypes.POINTER(SZ)]),
            "tda_position_buckets": (I32, [I32, I64, I32, P]),
            "tda_attention_ranges": (I32, [I64, I64, P, P, I32, I64, P, P]),
            "tda_attention_forward": (I32, [ctypes.POINTER(AttentionDesc), P, I64, P, I64, P, I64, P, P, P, P, P, I64, P, P,
                                            SZ, P]),
            "tda_attention_backward": (I32, [ctypes.POINTER(AttentionDesc), P, I64, P, I64, P, I64, P, P, P, P, P, I64, P, P,
                                             I64, P, I64, P, I64, P, I64, P, I32, F, P, SZ, P]),
            "tda_rmsnorm_forward": (I32, [I32, P, I64, P, I64, I64, I64, P, F, P, I64, P, I64, P, P]),
            "tda_rmsnorm_workspace_size": (SZ, [I64, I64]),
            "tda_rmsnorm_backward": (I32, [I32, P, I64, P, P, P, I64, P, I64, I64, I64, P, I64, P, I32, F, P, SZ, P]),
            "tda_embedding_forward": (I32, [I32, P, I64, I64, I64, I32, P, I64, F, P, I64, P]),
            "tda_embedding_workspace_size": (SZ, [I64, I64, I64]),
            "tda_embedding_backward": (I32, [I32, P, I64, I64, I64, I32, P, I64, F, I32, P, I64, F, P, SZ, P]),
            "tda_grad_clip_workspace_size": (SZ, [ctypes.POINTER(TensorRef), I64]),
            "tda_grad_clip": (I32, [ctypes.POINTER(TensorRef), I64, F, P, P, SZ, P]),
        }
        for name, (res, args) in sig.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
        return lib


def _ptr(x):
    """Device (or host) address of a tensor, an int, or None."""
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


_raw_stream = None


def _current_stream():
    """torch's current stream on the current device, without making a Stream object where torch offers that."""
    global _raw_stream
    if _raw_stream is None:
        import torch
        c = torch._C
        if hasattr(c, "_cuda_getCurrentRawStream") and hasattr(c, "_cuda_getDevice"):
            torch.cuda.current_stream()  # initialises CUDA
            _raw_stream = lambda: c._cuda_getCurrentRawStream(c._cuda_getDevice())  # noqa: E731
        else:
            _raw_stream = lambda: torch.cuda.current_stream().cuda_stream  # noqa: E731
    return _raw_stream()


def _stream(stream):
    if stream is None:
        return _current_stream()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _check(status: int) -> None:
    if status != TDA_OK:
        raise TdaError(status, load().tda_last_error().decode())


def tda_last_error() -> str:
    return load().tda_last_error().decode()


def tda_version() -> int:
    return int(load().tda_version())


def tda_launch_count() -> int:
    return int(load().tda_launch_count())


def tda_set_sm_budget(n_sms: int) -> None:
    _check(load().tda_set_sm_budget(n_sms))


def tda_get_sm_budget() -> int:
    return int(load().tda_get_sm_budget())


def tda_proj_entries(seed, layer, side, kind, rows, cols, out, stream=None):
    _check(load().tda_proj_entries(seed, layer, side, kind, rows, cols, _ptr(out), _stream(stream)))


def tda_workspace_size(op, L, dtype, n1, n2, route=TDA_ROUTE_AUTO) -> int:
    b = ctypes.c_size_t(0)
    _check(load().tda_workspace_size(op, ctypes.byref(L), dtype, n1, n2, route, ctypes.byref(b)))
    return int(b.value)


def tda_project(L, dtype, A, B, N, phi, ld_phi, route=TDA_ROUTE_AUTO, ws=None, ws_bytes=0, stream=None):
    _check(load().tda_project(ctypes.byref(L), dtype, _ptr(A), _ptr(B), N, _ptr(phi), ld_phi, route,
                              _ptr(ws), ws_bytes, _stream(stream)))


def tda_project_engine(L, dtype, A, B) -> int:
    return int(load().tda_project_engine(ctypes.byref(L), dtype, _ptr(A), _ptr(B)))


def tda_project_host_ws_min(L, dtype) -> int:
    return int(load().tda_project_host_ws_min(ctypes.byref(L), dtype))


def tda_project_host(L, dtype, A_h, B_h, N, phi, ld_phi, ws, ws_bytes, stream=None):
    _check(load().tda_project_host(ctypes.byref(L), dtype, _ptr(A_h), _ptr(B_h), N, _ptr(phi), ld_phi,
                                   _ptr(ws), ws_bytes, _stream(stream)))


def tda_noalloc_scratch_bytes() -> int:
    return int(load().tda_noalloc_scratch_bytes())


def tda_project_materialized_noalloc(L, dtype, A, B, N, phi, ld_phi, stream=None):
    _check(load().tda_project_materialized_noalloc(ctypes.byref(L), dtype, _ptr(A), _ptr(B), N, _ptr(phi),
                                                   ld_phi, _stream(stream)))


def tda_similarity_projected(L, dtype, Aq, Bq, n_q, At, Bt, n_t, S, ld_S, beta=0.0, route=TDA_ROUTE_AUTO,
                             ws=None, ws_bytes=0, stream=None):
    _check(load().tda_similarity_projected(ctypes.byref(L), dtype, _ptr(Aq), _ptr(Bq), n_q, _ptr(At), _ptr(Bt),
                                           n_t, _ptr(S), ld_S, beta, route, _ptr(ws), ws_bytes, _stream(stream)))


def tda_norms(op, L, dtype, A, B, N, out, route=TDA_ROUTE_AUTO, ws=None, ws_bytes=0, stream=None):
    _check(load().tda_norms(op, ctypes.byref(L), dtype, _ptr(A), _ptr(B), N, _ptr(out), route, _ptr(ws), ws_bytes,
                            _stream(stream)))


def tda_cosine(S, n_q, n_t, ld_S, nq, nt, stream=None):
    _check(load().tda_cosine(_ptr(S), n_q, n_t, ld_S, _ptr(nq), _ptr(nt), _stream(stream)))


def tda_similarity_exact(L, dtype, Aq, Bq, n_q, At, Bt, n_t, S, ld_S, beta=0.0, route=TDA_ROUTE_AUTO,
                         ws=None, ws_bytes=0, stream=None):
    _check(load().tda_similarity_exact(ctypes.byref(L), dtype, _ptr(Aq), _ptr(Bq), n_q, _ptr(At), _ptr(Bt),
                                       n_t, _ptr(S), ld_S, beta, route, _ptr(ws), ws_bytes, _stream(stream)))


def tda_token_scores_workspace_size(L) -> int:
    return int(load().tda_token_scores_workspace_size(ctypes.byref(L)))


def tda_token_scores(L, dtype, A, B, N, R, n_q, ld_R, out, ld_q_out, beta=0.0, ws=None, ws_bytes=0, stream=None):
    _check(load().tda_token_scores(ctypes.byref(L), dtype, _ptr(A), _ptr(B), N, _ptr(R), n_q, ld_R, _ptr(out),
                                   ld_q_out, beta, _ptr(ws), ws_bytes, _stream(stream)))


def tda_mask_gather(L, dtype, A, B, N, rows, cols, n_coords, out, ld_out, stream=None):
    _check(load().tda_mask_gather(ctypes.byref(L), dtype, _ptr(A), _ptr(B), N, _ptr(rows), _ptr(cols), n_coords,
                                  _ptr(out), ld_out, _stream(stream)))


def tda_kfac_state_bytes(k_in, k_out) -> int:
    return int(load().tda_kfac_state_bytes(k_in, k_out))


def tda_kfac_workspace_size(L, dtype) -> int:
    return int(load().tda_kfac_workspace_size(ctypes.byref(L), dtype))


def tda_kfac_reset(k_in, k_out, state, stream=None, n_layers=1):
    _check(load().tda_kfac_reset(n_layers, k_in, k_out, _ptr(state), _stream(stream)))


def tda_kfac_accumulate_factors(L, dtype, A, B, N, state, ws, ws_bytes, stream=None):
    _check(load().tda_kfac_accumulate_factors(ctypes.byref(L), dtype, _ptr(A), _ptr(B), N, _ptr(state), _ptr(ws),
                                              ws_bytes, _stream(stream)))


def tda_project_kfac(L, dtype, A, B, N, phi, ld_phi, state, ws, ws_bytes, stream=None):
    _check(load().tda_project_kfac(ctypes.byref(L), dtype, _ptr(A), _ptr(B), N, _ptr(phi), ld_phi, _ptr(state),
                                   _ptr(ws), ws_bytes, _stream(stream)))


def tda_kfac_eigen(k_in, k_out, state, stream=None, n_layers=1):
    _check(load().tda_kfac_eigen(n_layers, k_in, k_out, _ptr(state), _stream(stream)))


def tda_kfac_accumulate_eigenvalues(k_in, k_out, state, phi, n, ld_phi, ws, ws_bytes, stream=None, n_layers=1):
    _check(load().tda_kfac_accumulate_eigenvalues(n_layers, k_in, k_out, _ptr(state), _ptr(phi), n, ld_phi, _ptr(ws),
                                                  ws_bytes, _stream(stream)))


def tda_kfac_apply(kind, k_in, k_out, state, lambda_abs, lambda_rel, q, n_q, ld_q, qhat, ld_qhat, stream=None,
                   n_layers=1):
    _check(load().tda_kfac_apply(kind, n_layers, k_in, k_out, _ptr(state), float(lambda_abs), float(lambda_rel),
                                 _ptr(q), n_q, ld_q, _ptr(qhat), ld_qhat, _stream(stream)))


def tda_precondition_state_bytes(D, state_dtype) -> int:
    return int(load().tda_precondition_state_bytes(D, state_dtype))


def tda_precondition(op, n_layers, D, state_dtype, state, phi=None, n=0, ld_phi=0, n_total=0, lambda_abs=0.0,
                     lambda_rel_mean_eig=0.0, q=None, n_q=0, ld_q=0, qhat=None, ld_qhat=0, stream=None):
    _check(load().tda_precondition(op, n_layers, D, state_dtype, _ptr(state), _ptr(phi), n, ld_phi, n_total,
                                   lambda_abs, lambda_rel_mean_eig, _ptr(q), n_q, ld_q, _ptr(qhat),
                                   ld_qhat, _stream(stream)))


def tda_precondition_info(n_layers, D, state_dtype, state, stream=None) -> list[float]:
    info = (ctypes.c_double * (4 * n_layers))()
    _check(load().tda_precondition_info(n_layers, D, state_dtype, _ptr(state), info, _stream(stream)))
    return list(info)


def tda_score(Qhat, q_dtype, n_q, ld_q, Phi, n_t, ld_phi, D, S, ld_S, beta=0.0, stream=None):
    _check(load().tda_score(_ptr(Qhat), q_dtype, n_q, ld_q, _ptr(Phi), n_t, ld_phi, D, _ptr(S), ld_S,
                            beta, _stream(stream)))


def tda_similarity_gram_engine(L, dtype, Aq, Bq, At, Bt) -> int:
    return int(load().tda_similarity_gram_engine(ctypes.byref(L), dtype, _ptr(Aq), _ptr(Bq), _ptr(At), _ptr(Bt)))


def tda_score_engine(Qhat, q_dtype, n_q, ld_q, Phi, n_t, ld_phi, D) -> int:
    return int(load().tda_score_engine(_ptr(Qhat), q_dtype, n_q, ld_q, _ptr(Phi), n_t, ld_phi, D))


def tda_topk(S, n_q, n_t, ld_S, k, idx, val=None, stream=None):
    _check(load().tda_topk(_ptr(S), n_q, n_t, ld_S, k, _ptr(idx), _ptr(val), _stream(stream)))


def tda_route(L, op, n1, n2, dtype) -> tuple[int, list[float]]:
    chosen = ctypes.c_int32(0)
    cost = (ctypes.c_double * 3)()
    _check(load().tda_route(ctypes.byref(L), op, n1, n2, dtype, ctypes.byref(chosen), cost))
    return int(chosen.value), list(cost)


def tda_route_calibrate(ws, ws_bytes, stream=None) -> list[float]:
    rates = (ctypes.c_double * 7)()
    _check(load().tda_route_calibrate(_ptr(ws), ws_bytes, _stream(stream), rates))
    return list(rates)


def tda_route_set_model(model: int) -> None:
    _check(load().tda_route_set_model(model))


def tda_selftest_bounded_wait(timeout_ns, stream=None) -> None:
    _check(load().tda_selftest_bounded_wait(timeout_ns, _stream(stream)))


def tda_device_status(stream=None) -> None:
    _check(load().tda_device_status(_stream(stream)))


def tda_linear_workspace_size(op, L, M) -> int:
    b = ctypes.c_size_t(0)
    _check(load().tda_linear_workspace_size(op, ctypes.byref(L), M, ctypes.byref(b)))
    return int(b.value)


_calls = None


def _train():
    """The extension module that calls the training step's entry points (csrc/fastcall.c), bound to libtda.so."""
    global _calls
    if _calls is None:
        lib = load()
        try:
            mod = importlib.import_module("paper_2609_38767_gb300._fast")
        except ImportError as e:
            raise ImportError(f"_fast.so is missing: run paper_2609_38767_gb300.build.build() first ({e})") from e
        addr = lambda f: ctypes.cast(f, ctypes.c_void_p).value  # noqa: E731
        mod.bind(_current_stream, LinearDesc, addr(lib.tda_linear_forward), addr(lib.tda_linear_backward),
                 addr(lib.tda_embedding_forward), addr(lib.tda_embedding_backward), addr(lib.tda_grad_clip))
        mod.bind_block(AttentionDesc, addr(lib.tda_attention_ranges), addr(lib.tda_attention_forward),
                       addr(lib.tda_attention_backward), addr(lib.tda_rmsnorm_forward), addr(lib.tda_rmsnorm_backward))
        _calls = mod
    return _calls


def tda_linear_forward(L, X, ld_x, M, W, ld_w, bias, R, ld_r, Y, ld_y, Z=None, ld_z=0, ws=None, ws_bytes=0,
                       stream=None):
    st = (_calls or _train()).linear_forward(L, X, ld_x, M, W, ld_w, bias, R, ld_r, Y, ld_y, Z, ld_z, ws, ws_bytes,
                                            stream)
    if st:
        _check(st)


def tda_linear_backward(L, dY, ld_dy, Z, ld_z, M, X, ld_x, W, ld_w, B, ld_b, dX, ld_dx, dW, ld_dw, db,
                        grad_dtype=TDA_F32, beta=0.0, ws=None, ws_bytes=0, stream=None):
    st = (_calls or _train()).linear_backward(L, dY, ld_dy, Z, ld_z, M, X, ld_x, W, ld_w, B, ld_b, dX, ld_dx, dW, ld_dw,
                                             db, grad_dtype, beta, ws, ws_bytes, stream)
    if st:
        _check(st)


def tda_embedding_forward(dtype, E, ld_e, V, d, it, tokens, n, scale, out, ld_out, stream=None):
    st = (_calls or _train()).embedding_forward(dtype, E, ld_e, V, d, it, tokens, n, scale, out, ld_out, stream)
    if st:
        _check(st)


def tda_embedding_workspace_size(V, d, n) -> int:
    return int(load().tda_embedding_workspace_size(V, d, n))


def tda_embedding_backward(dtype, dout, ld_d, V, d, it, tokens, n, scale, grad_dtype, dE, ld_e, beta=0.0, ws=None,
                           ws_bytes=0, stream=None):
    st = (_calls or _train()).embedding_backward(dtype, dout, ld_d, V, d, it, tokens, n, scale, grad_dtype, dE, ld_e,
                                                beta, ws, ws_bytes, stream)
    if st:
        _check(st)


def tensor_list(tensors, outs=None):
    """The host array of tda_tensor_ref that tda_grad_clip takes: contiguous bf16 or fp32 tensors,
    clipped into `outs` (same sizes and types; None entries are left unclipped), or in place
    (outs None). The array holds addresses only: keep the tensors alive."""
    import torch
    kinds = {torch.float32: TDA_F32, torch.bfloat16: TDA_BF16}
    outs = list(tensors) if outs is None else list(outs)
    if len(outs) != len(tensors):
        raise ValueError("tensor_list: one output per tensor")
    refs = (TensorRef * max(len(outs), 1))()
    for r, t, o in zip(refs, tensors, outs):
        if not t.is_contiguous() or t.dtype not in kinds:
            raise ValueError("tensor_list: tensors must be contiguous bf16 or fp32")
        if o is not None and (not o.is_contiguous() or o.dtype != t.dtype or o.numel() != t.numel()):
            raise ValueError("tensor_list: an output must have its tensor's size and type and be contiguous")
        r.in_, r.out, r.n, r.dtype = t.data_ptr(), o.data_ptr() if o is not None else None, t.numel(), kinds[t.dtype]
    return refs


def tda_grad_clip_workspace_size(refs, n_tensors) -> int:
    return int(load().tda_grad_clip_workspace_size(refs, n_tensors))


def tda_grad_clip(refs, n_tensors, max_norm, norm, ws, ws_bytes, stream=None):
    st = (_calls or _train()).grad_clip(refs, n_tensors, max_norm, norm, ws, ws_bytes, stream)
    if st:
        _check(st)


def tda_attention_workspace_size(op, L) -> int:
    b = ctypes.c_size_t(0)
    _check(load().tda_attention_workspace_size(op, ctypes.byref(L), ctypes.byref(b)))
    return int(b.value)


def tda_position_buckets(n_buckets, max_distance, bidirectional, bucket):
    """bucket: a contiguous int32 CPU tensor of 2 * max_distance + 1 values (or the address of such memory)."""
    if not isinstance(bucket, int) and bucket is not None:
        import torch
        if bucket.dtype != torch.int32 or bucket.is_cuda or not bucket.is_contiguous() or bucket.numel() < 2 * max_distance + 1:
            raise ValueError("tda_position_buckets: bucket is a contiguous int32 CPU tensor of 2 * max_distance + 1 values")
    _check(load().tda_position_buckets(n_buckets, max_distance, int(bidirectional), _ptr(bucket)))


def tda_attention_ranges(N, T, doc, prefix, causal, window, range, stream=None):
    st = (_calls or _train()).attention_ranges(N, T, doc, prefix, causal, window, range, stream)
    if st:
        _check(st)


def tda_attention_forward(L, Q, ld_q, K, ld_k, V, ld_v, range, bucket, table, slope, O, ld_o, lse=None, ws=None, ws_bytes=0,
                          stream=None):
    st = (_calls or _train()).attention_forward(L, Q, ld_q, K, ld_k, V, ld_v, range, bucket, table, slope, O, ld_o, lse, ws,
                                               ws_bytes, stream)
    if st:
        _check(st)


def tda_attention_backward(L, Q, ld_q, K, ld_k, V, ld_v, range, bucket, table, slope, O, ld_o, lse, dO, ld_do, dQ, ld_dq, dK,
                           ld_dk, dV, ld_dv, dtable=None, grad_dtype=TDA_F32, beta=0.0, ws=None, ws_bytes=0, stream=None):
    st = (_calls or _train()).attention_backward(L, Q, ld_q, K, ld_k, V, ld_v, range, bucket, table, slope, O, ld_o, lse, dO,
                                                ld_do, dQ, ld_dq, dK, ld_dk, dV, ld_dv, dtable, grad_dtype, beta, ws, ws_bytes,
                                                stream)
    if st:
        _check(st)


def tda_rmsnorm_forward(dtype, x, ld_x, r, ld_r, M, d, w, eps, h, ld_h, y, ld_y, rstd=None, stream=None):
    st = (_calls or _train()).rmsnorm_forward(dtype, x, ld_x, r, ld_r, M, d, w, eps, h, ld_h, y, ld_y, rstd, stream)
    if st:
        _check(st)


def tda_rmsnorm_workspace_size(M, d) -> int:
    return int(load().tda_rmsnorm_workspace_size(M, d))


def tda_rmsnorm_backward(dtype, h, ld_h, rstd, w, dy, ld_dy, dres, ld_r, M, d, dx, ld_dx, dw=None, grad_dtype=TDA_F32, beta=0.0,
                         ws=None, ws_bytes=0, stream=None):
    st = (_calls or _train()).rmsnorm_backward(dtype, h, ld_h, rstd, w, dy, ld_dy, dres, ld_r, M, d, dx, ld_dx, dw, grad_dtype,
                                              beta, ws, ws_bytes, stream)
    if st:
        _check(st)
