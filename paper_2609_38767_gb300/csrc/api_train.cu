// api_train.cu -- the extern "C" entry points of the training step's operators
// (include/tda.h): host-side argument validation and kernel dispatch.
#include <cmath>

#include "linear.cuh"

using namespace tda;

namespace {

size_t el_size(int32_t dt) { return dt == TDA_BF16 ? 2 : 4; }
bool float_type(int32_t dt) { return dt == TDA_BF16 || dt == TDA_F32; }
bool aligned_to(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
constexpr int64_t kMaxCount = ((int64_t)1 << 31) - 2, kMaxRow = 1 << 22, kMaxMatrix = (int64_t)1 << 47;
constexpr int64_t kMaxTensors = 1 << 20;

tda_status check_table(tda_dtype dtype, int64_t V, int64_t d, int32_t it, const void* tokens, int64_t n, float scale,
                       const char* who) {
    if (!float_type(dtype)) return fail(TDA_ERR_INVALID_ARG, "%s: dtype must be TDA_F32 or TDA_BF16", who);
    if (it != TDA_I32 && it != TDA_I64) return fail(TDA_ERR_INVALID_ARG, "%s: index type must be TDA_I32 or TDA_I64", who);
    if (V < 1 || V > kMaxCount || d < 1 || d > kMaxRow || n < 0 || n > kMaxCount)
        return fail(TDA_ERR_INVALID_ARG, "%s: bad sizes V=%lld d=%lld n=%lld", who, (long long)V, (long long)d,
                    (long long)n);
    if (!std::isfinite(scale)) return fail(TDA_ERR_INVALID_ARG, "%s: scale must be finite", who);
    if (n > 0 && (!tokens || !aligned_to(tokens, it == TDA_I64 ? 8 : 4)))
        return fail(TDA_ERR_INVALID_ARG, "%s: tokens is NULL or misaligned", who);
    return TDA_OK;
}

tda_status check_linear(const tda_linear_desc* L, int64_t M, const char* who) {
    if (!L) return fail(TDA_ERR_INVALID_ARG, "%s: layer descriptor is NULL", who);
    if (L->d_in < 1 || L->d_out < 1 || L->d_in > kMaxCount || L->d_out > kMaxCount || M < 0 || M > kMaxCount)
        return fail(TDA_ERR_INVALID_ARG, "%s: bad sizes d_in=%lld d_out=%lld M=%lld", who, (long long)L->d_in,
                    (long long)L->d_out, (long long)M);
    // matrices past any memory, whose scratch would wrap a size_t
    for (int64_t n : {M * L->d_in, M * L->d_out, L->d_in * L->d_out})
        if (n > kMaxMatrix)
            return fail(TDA_ERR_INVALID_ARG, "%s: a matrix of more than 2^47 elements (d_in=%lld d_out=%lld M=%lld)", who,
                        (long long)L->d_in, (long long)L->d_out, (long long)M);
    if (L->act < TDA_ACT_NONE || L->act > TDA_ACT_SILU) return fail(TDA_ERR_INVALID_ARG, "%s: bad activation %d", who, L->act);
    if (!float_type(L->dtype)) return fail(TDA_ERR_INVALID_ARG, "%s: dtype must be TDA_F32 or TDA_BF16", who);
    return TDA_OK;
}

// A tensor argument of `cols` values a row: present unless optional, aligned to its type, rows not overlapping.
// Row strides stay below 2^39 bytes, the tensor maps' limit.
tda_status check_rows(const void* p, int64_t ld, int64_t cols, int32_t dt, bool optional, const char* name) {
    if (!p) return optional ? TDA_OK : fail(TDA_ERR_INVALID_ARG, "%s is NULL", name);
    if (!aligned_to(p, el_size(dt))) return fail(TDA_ERR_INVALID_ARG, "%s is misaligned", name);
    if (ld < cols || ld > (1LL << 37)) return fail(TDA_ERR_INVALID_ARG, "%s: row stride %lld for %lld columns", name,
                                                   (long long)ld, (long long)cols);
    return TDA_OK;
}

tda_status linear_device(unsigned int** err) {
    if (!linear_tc_available()) return fail(TDA_ERR_UNSUPPORTED, "the linear layer needs an sm_103 device");
    *err = device_error_word();
    if (!*err) return fail(TDA_ERR_CUDA, "cannot resolve the device error word");
    return TDA_OK;
}

tda_status check_ws(const void* ws, size_t ws_bytes, size_t need, const char* who) {
    if (need && (!ws || ws_bytes < need))
        return fail(TDA_ERR_WORKSPACE, "%s needs >= %zu bytes of ws, got %zu", who, need, ws ? ws_bytes : 0);
    if (need && !aligned_to(ws, 256)) return fail(TDA_ERR_INVALID_ARG, "ws must be 256-byte aligned");
    return TDA_OK;
}

}  // namespace

int tda::train_sms() {
    static std::atomic<int> sms{0};
    int v = sms.load(std::memory_order_relaxed);
    if (!v) {
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess ||
            cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || v <= 0)
            v = 152;
        sms.store(v, std::memory_order_relaxed);
    }
    return v;
}

extern "C" {

tda_status tda_linear_workspace_size(int32_t op, const tda_linear_desc* L, int64_t M, size_t* bytes) {
    clear_message();
    if (!bytes) return fail(TDA_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = 0;
    tda_status st = check_linear(L, M, "tda_linear_workspace_size");
    if (st) return st;
    const int32_t pass = op & ~TDA_LINEAR_ANY_STRIDE;
    if (pass != TDA_LINEAR_FORWARD && pass != TDA_LINEAR_BACKWARD) return fail(TDA_ERR_INVALID_ARG, "bad linear op %d", op);
    *bytes = M == 0 ? 0
                    : linear_ws_bound(pass == TDA_LINEAR_BACKWARD, M, L->d_in, L->d_out, (tda_dtype)L->dtype,
                                      (op & TDA_LINEAR_ANY_STRIDE) != 0);
    return TDA_OK;
}

tda_status tda_linear_forward(const tda_linear_desc* L, const void* X, int64_t ld_x, int64_t M, const void* W,
                              int64_t ld_w, const void* bias, const void* R, int64_t ld_r, void* Y, int64_t ld_y,
                              void* Z, int64_t ld_z, void* ws, size_t ws_bytes, void* stream) {
    clear_message();
    tda_status st = check_linear(L, M, "tda_linear_forward");
    if (st) return st;
    if (M == 0) return TDA_OK;
    if ((st = check_rows(X, ld_x, L->d_in, L->dtype, false, "X")) ||
        (st = check_rows(W, ld_w, L->d_in, L->dtype, false, "W")) ||
        (st = check_rows(bias, L->d_out, L->d_out, L->dtype, true, "bias")) ||
        (st = check_rows(R, ld_r, L->d_out, L->dtype, true, "R")) ||
        (st = check_rows(Y, ld_y, L->d_out, L->dtype, false, "Y")) ||
        (st = check_rows(Z, ld_z, L->d_out, L->dtype, true, "Z")))
        return st;
    LinearForward f;
    f.M = M, f.d_in = L->d_in, f.d_out = L->d_out, f.act = L->act, f.dt = (tda_dtype)L->dtype;
    f.X = X, f.W = W, f.bias = bias, f.R = R, f.Y = Y, f.Z = Z;
    f.ld_x = ld_x, f.ld_w = ld_w, f.ld_r = ld_r, f.ld_y = ld_y, f.ld_z = ld_z;
    if ((st = check_ws(ws, ws_bytes, linear_forward_ws(f), "tda_linear_forward"))) return st;
    unsigned int* err = nullptr;
    if ((st = linear_device(&err))) return st;
    return cuda_check(launch_linear_forward(f, ws, err, (cudaStream_t)stream), "linear forward");
}

tda_status tda_linear_backward(const tda_linear_desc* L, const void* dY, int64_t ld_dy, const void* Z, int64_t ld_z,
                               int64_t M, const void* X, int64_t ld_x, const void* W, int64_t ld_w, void* B,
                               int64_t ld_b, void* dX, int64_t ld_dx, void* dW, int64_t ld_dw, void* db,
                               tda_dtype grad_dtype, float beta, void* ws, size_t ws_bytes, void* stream) {
    clear_message();
    tda_status st = check_linear(L, M, "tda_linear_backward");
    if (st) return st;
    if (!float_type(grad_dtype)) return fail(TDA_ERR_INVALID_ARG, "tda_linear_backward: grad_dtype must be TDA_F32 or TDA_BF16");
    if (!std::isfinite(beta)) return fail(TDA_ERR_INVALID_ARG, "tda_linear_backward: beta must be finite");
    if (L->dtype == TDA_F32 && grad_dtype == TDA_BF16)
        return fail(TDA_ERR_UNSUPPORTED, "tda_linear_backward: bf16 gradients need a bf16 layer");
    const bool act = L->act != TDA_ACT_NONE;
    if ((st = check_rows(dW, ld_dw, L->d_in, grad_dtype, true, "dW")) ||
        (st = check_rows(db, L->d_out, L->d_out, grad_dtype, true, "db")))
        return st;
    cudaStream_t s = (cudaStream_t)stream;
    if (M == 0) {
        if (dW && beta != 1.f &&
            (st = cuda_check(launch_scale_matrix(grad_dtype, dW, L->d_out, L->d_in, ld_dw, beta, s), "scale dW")))
            return st;
        if (db && beta != 1.f)
            return cuda_check(launch_scale_matrix(grad_dtype, db, 1, L->d_out, L->d_out, beta, s), "scale db");
        return TDA_OK;
    }
    if ((st = check_rows(dY, ld_dy, L->d_out, L->dtype, false, "dY")) ||
        (st = check_rows(Z, ld_z, L->d_out, L->dtype, !act, "Z")) ||
        (st = check_rows(B, ld_b, L->d_out, L->dtype, !act, "B")) ||
        (st = check_rows(X, ld_x, L->d_in, L->dtype, !dW, "X")) ||
        (st = check_rows(W, ld_w, L->d_in, L->dtype, !dX, "W")) ||
        (st = check_rows(dX, ld_dx, L->d_in, L->dtype, true, "dX")))
        return st;
    LinearBackward b;
    b.M = M, b.d_in = L->d_in, b.d_out = L->d_out, b.act = L->act, b.dt = (tda_dtype)L->dtype, b.gt = grad_dtype;
    b.beta = beta;
    b.dY = dY, b.Z = Z, b.X = X, b.W = W, b.B = B, b.dX = dX, b.dW = dW, b.db = db;
    b.ld_dy = ld_dy, b.ld_z = ld_z, b.ld_x = ld_x, b.ld_w = ld_w, b.ld_b = ld_b, b.ld_dx = ld_dx, b.ld_dw = ld_dw;
    if ((st = check_ws(ws, ws_bytes, linear_backward_ws(b), "tda_linear_backward"))) return st;
    unsigned int* err = nullptr;
    if ((st = linear_device(&err))) return st;
    return cuda_check(launch_linear_backward(b, ws, err, s), "linear backward");
}

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
    if (V < 1 || V > kMaxCount || d < 1 || d > kMaxRow || n < 0 || n > kMaxCount) return 0;
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
    if (n_tensors < 0 || n_tensors > kMaxTensors) return 0;
    return clip_workspace_bytes(n_tensors);
}

tda_status tda_grad_clip(const tda_tensor_ref* list, int64_t n_tensors, float max_norm, float* norm, void* ws,
                         size_t ws_bytes, void* stream) {
    clear_message();
    if (n_tensors < 0 || n_tensors > kMaxTensors || (n_tensors > 0 && !list))
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
