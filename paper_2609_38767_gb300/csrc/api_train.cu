// api_train.cu -- the extern "C" entry points of the training step's operators
// (include/tda.h): host-side argument validation and kernel dispatch.
#include <cmath>

#include "tda_internal.cuh"

using namespace tda;

namespace {

size_t el_size(int32_t dt) { return dt == TDA_BF16 ? 2 : 4; }
bool float_type(int32_t dt) { return dt == TDA_BF16 || dt == TDA_F32; }
bool aligned_to(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
constexpr int64_t kMaxCount = ((int64_t)1 << 31) - 2;

tda_status check_table(tda_dtype dtype, int64_t V, int64_t d, int32_t it, const void* tokens, int64_t n, float scale,
                       const char* who) {
    if (!float_type(dtype)) return fail(TDA_ERR_INVALID_ARG, "%s: dtype must be TDA_F32 or TDA_BF16", who);
    if (it != TDA_I32 && it != TDA_I64) return fail(TDA_ERR_INVALID_ARG, "%s: index type must be TDA_I32 or TDA_I64", who);
    if (V < 1 || V > kMaxCount || d < 1 || n < 0 || n > kMaxCount)
        return fail(TDA_ERR_INVALID_ARG, "%s: bad sizes V=%lld d=%lld n=%lld", who, (long long)V, (long long)d,
                    (long long)n);
    if (!std::isfinite(scale)) return fail(TDA_ERR_INVALID_ARG, "%s: scale must be finite", who);
    if (n > 0 && (!tokens || !aligned_to(tokens, it == TDA_I64 ? 8 : 4)))
        return fail(TDA_ERR_INVALID_ARG, "%s: tokens is NULL or misaligned", who);
    return TDA_OK;
}

}  // namespace

extern "C" {

tda_status tda_embedding_forward(tda_dtype dtype, const void* E, int64_t ld_e, int64_t V, int64_t d,
                                 tda_index_type it, const void* tokens, int64_t n, float scale, void* out,
                                 int64_t ld_out, void* stream) {
    clear_message();
    tda_status st = check_table(dtype, V, d, it, tokens, n, scale, "tda_embedding_forward");
    if (st) return st;
    if (ld_e < d || ld_out < d) return fail(TDA_ERR_INVALID_ARG, "tda_embedding_forward: ld_e or ld_out < d");
    if (n == 0) return TDA_OK;
    if (!E || !out || !aligned_to(E, el_size(dtype)) || !aligned_to(out, el_size(dtype)))
        return fail(TDA_ERR_INVALID_ARG, "tda_embedding_forward: E or out is NULL or misaligned");
    return cuda_check(launch_embedding_forward(dtype, E, ld_e, V, d, it, tokens, n, scale, out, ld_out,
                                               (cudaStream_t)stream),
                      "embedding forward");
}

size_t tda_embedding_workspace_size(int64_t V, int64_t d, int64_t n) {
    if (V < 1 || d < 1 || n < 0 || n > kMaxCount) return 0;
    return embedding_workspace_bytes(d, n);
}

tda_status tda_embedding_backward(tda_dtype dtype, const void* dout, int64_t ld_d, int64_t V, int64_t d,
                                  tda_index_type it, const void* tokens, int64_t n, float scale,
                                  tda_dtype grad_dtype, void* dE, int64_t ld_e, float beta, void* ws,
                                  size_t ws_bytes, void* stream) {
    clear_message();
    tda_status st = check_table(dtype, V, d, it, tokens, n, scale, "tda_embedding_backward");
    if (st) return st;
    if (!float_type(grad_dtype))
        return fail(TDA_ERR_INVALID_ARG, "tda_embedding_backward: grad_dtype must be TDA_F32 or TDA_BF16");
    if (dtype == TDA_F32 && grad_dtype == TDA_BF16)
        return fail(TDA_ERR_UNSUPPORTED, "tda_embedding_backward: bf16 gradients need bf16 dout");
    if (ld_d < d || ld_e < d) return fail(TDA_ERR_INVALID_ARG, "tda_embedding_backward: ld_d or ld_e < d");
    if (!std::isfinite(beta)) return fail(TDA_ERR_INVALID_ARG, "tda_embedding_backward: beta must be finite");
    if (!dE || !aligned_to(dE, el_size(grad_dtype)))
        return fail(TDA_ERR_INVALID_ARG, "tda_embedding_backward: dE is NULL or misaligned");
    if (n > 0) {
        if (!dout || !aligned_to(dout, el_size(dtype)))
            return fail(TDA_ERR_INVALID_ARG, "tda_embedding_backward: dout is NULL or misaligned");
        const size_t need = embedding_workspace_bytes(d, n);
        if (!ws || ws_bytes < need)
            return fail(TDA_ERR_WORKSPACE, "tda_embedding_backward needs >= %zu bytes of ws, got %zu", need, ws_bytes);
        if (!aligned_to(ws, 256)) return fail(TDA_ERR_INVALID_ARG, "ws must be 256-byte aligned");
    }
    return cuda_check(launch_embedding_backward(dtype, dout, ld_d, V, d, it, tokens, n, scale, grad_dtype, dE, ld_e,
                                                beta, ws, (cudaStream_t)stream),
                      "embedding backward");
}

size_t tda_grad_clip_workspace_size(const tda_tensor_ref* list, int64_t n_tensors) {
    (void)list;
    if (n_tensors < 0) return 0;
    return clip_workspace_bytes(n_tensors);
}

tda_status tda_grad_clip(const tda_tensor_ref* list, int64_t n_tensors, float max_norm, float* norm, void* ws,
                         size_t ws_bytes, void* stream) {
    clear_message();
    if (n_tensors < 0 || n_tensors > (1LL << 20) || (n_tensors > 0 && !list))
        return fail(TDA_ERR_INVALID_ARG, "tda_grad_clip: list is NULL or n_tensors not in [0, 2^20]");
    if (!(max_norm > 0)) return fail(TDA_ERR_INVALID_ARG, "tda_grad_clip: max_norm must be > 0");
    if (!norm || !aligned_to(norm, 4)) return fail(TDA_ERR_INVALID_ARG, "tda_grad_clip: norm is NULL or misaligned");
    for (int64_t i = 0; i < n_tensors; ++i) {
        const tda_tensor_ref& r = list[i];
        if (!float_type(r.dtype))
            return fail(TDA_ERR_INVALID_ARG, "tda_grad_clip: tensor %lld is neither TDA_F32 nor TDA_BF16", (long long)i);
        if (r.n < 0 || r.n > (1LL << 48)) return fail(TDA_ERR_INVALID_ARG, "tda_grad_clip: bad size of tensor %lld", (long long)i);
        if (r.n > 0 && (!r.in || !aligned_to(r.in, el_size(r.dtype)) || !aligned_to(r.out, el_size(r.dtype))))
            return fail(TDA_ERR_INVALID_ARG, "tda_grad_clip: tensor %lld is NULL or misaligned", (long long)i);
    }
    const size_t need = clip_workspace_bytes(n_tensors);
    if (!ws || ws_bytes < need)
        return fail(TDA_ERR_WORKSPACE, "tda_grad_clip needs >= %zu bytes of ws, got %zu", need, ws_bytes);
    if (!aligned_to(ws, 16)) return fail(TDA_ERR_INVALID_ARG, "ws must be 16-byte aligned");
    return cuda_check(launch_grad_clip(list, n_tensors, max_norm, norm, (double*)ws, (cudaStream_t)stream),
                      "gradient clip");
}

}  // extern "C"
