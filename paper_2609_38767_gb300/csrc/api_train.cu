// api_train.cu -- the extern "C" entry points of the training step's operators
// (include/tda.h): host-side argument validation and kernel dispatch.
#include <cmath>

#include "attention.cuh"
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

constexpr int kMaxHeadDim = 128;
constexpr int64_t kMaxReach = 1 << 20, kMaxBuckets = 1024, kMaxTokens = 1 << 29;  // a window of distances is 2 T + 513 long

tda_status check_attention(const tda_attention_desc* L, const char* who) {
    if (!L) return fail(TDA_ERR_INVALID_ARG, "%s: attention descriptor is NULL", who);
    if (L->N < 0 || L->T < 0 || L->N > kMaxCount || L->T > kMaxTokens || L->heads < 1 || L->heads > 65535 || L->kv_heads < 1 ||
        L->head_dim < 1)
        return fail(TDA_ERR_INVALID_ARG, "%s: bad sizes N=%lld T=%lld heads=%d kv_heads=%d head_dim=%d", who, (long long)L->N,
                    (long long)L->T, L->heads, L->kv_heads, L->head_dim);
    if (L->heads % L->kv_heads)
        return fail(TDA_ERR_INVALID_ARG, "%s: kv_heads=%d does not divide heads=%d", who, L->kv_heads, L->heads);
    if (L->head_dim > kMaxHeadDim) return fail(TDA_ERR_UNSUPPORTED, "%s: head_dim %d > %d", who, L->head_dim, kMaxHeadDim);
    // one CTA per 64 queries of a head, and per 64 keys
    if ((L->T && L->N > (kMaxCount - 65536) / L->heads / L->T) || L->N * ((L->T + 63) / 64) > (kMaxCount - 65536) / 2 / L->heads)
        return fail(TDA_ERR_INVALID_ARG, "%s: too many tokens or heads (N=%lld T=%lld heads=%d)", who, (long long)L->N,
                    (long long)L->T, L->heads);
    if (!float_type(L->dtype)) return fail(TDA_ERR_INVALID_ARG, "%s: dtype must be TDA_F32 or TDA_BF16", who);
    if (!(L->scale > 0) || !std::isfinite(L->scale)) return fail(TDA_ERR_INVALID_ARG, "%s: scale must be finite and > 0", who);
    if (!(L->cap >= 0) || !std::isfinite(L->cap)) return fail(TDA_ERR_INVALID_ARG, "%s: cap must be finite and >= 0", who);
    if (L->causal != 0 && L->causal != 1) return fail(TDA_ERR_INVALID_ARG, "%s: causal must be 0 or 1", who);
    if (L->n_buckets < 0 || L->n_buckets > kMaxBuckets || L->max_distance < 0 || L->max_distance > kMaxReach)
        return fail(TDA_ERR_INVALID_ARG, "%s: n_buckets=%d not in [0, %lld] or max_distance=%lld not in [0, %lld]", who, L->n_buckets,
                    (long long)kMaxBuckets, (long long)L->max_distance, (long long)kMaxReach);
    return TDA_OK;
}

// The arguments that both passes share; the tensors of a batch without tokens are not looked at.
tda_status check_attention_inputs(const tda_attention_desc* L, const void* Q, int64_t ld_q, const void* K, int64_t ld_k,
                                  const void* V, int64_t ld_v, const int32_t* range, const int32_t* bucket, const void* table,
                                  const float* slope) {
    const int64_t q = (int64_t)L->heads * L->head_dim, kv = (int64_t)L->kv_heads * L->head_dim;
    tda_status st;
    if ((st = check_rows(Q, ld_q, q, L->dtype, false, "Q")) || (st = check_rows(K, ld_k, kv, L->dtype, false, "K")) ||
        (st = check_rows(V, ld_v, kv, L->dtype, false, "V")))
        return st;
    if (!aligned_to(range, 8)) return fail(TDA_ERR_INVALID_ARG, "range is misaligned");
    if (L->n_buckets) {
        if (!bucket || !aligned_to(bucket, 4)) return fail(TDA_ERR_INVALID_ARG, "bucket is NULL or misaligned");
        if (!table || !aligned_to(table, el_size(L->dtype))) return fail(TDA_ERR_INVALID_ARG, "table is NULL or misaligned");
    }
    if (!aligned_to(slope, 4)) return fail(TDA_ERR_INVALID_ARG, "slope is misaligned");
    return TDA_OK;
}

Attention attention_of(const tda_attention_desc* L) {
    Attention a = {};
    a.N = L->N, a.T = L->T, a.H = L->heads, a.KV = L->kv_heads, a.hd = L->head_dim, a.dt = (tda_dtype)L->dtype;
    // cap tanh(x / cap) is x in fp32 for any |x| < 2^88 then; x / cap would lose its digits below fp32's smallest normal number
    a.scale = L->scale, a.cap = L->cap < 0x1p100f ? L->cap : 0.f, a.causal = L->causal, a.n_buckets = L->n_buckets, a.reach = L->max_distance;
    return a;
}

tda_status check_norm(tda_dtype dtype, int64_t M, int64_t d, const char* who) {
    if (!float_type(dtype)) return fail(TDA_ERR_INVALID_ARG, "%s: dtype must be TDA_F32 or TDA_BF16", who);
    if (M < 0 || M > kMaxCount || d < 1 || d > kMaxCount)
        return fail(TDA_ERR_INVALID_ARG, "%s: bad sizes M=%lld d=%lld", who, (long long)M, (long long)d);
    if (d > kNormMaxRow) return fail(TDA_ERR_UNSUPPORTED, "%s: rows of %lld > %lld values", who, (long long)d, (long long)kNormMaxRow);
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

tda_status tda_attention_workspace_size(int32_t op, const tda_attention_desc* L, size_t* bytes) {
    clear_message();
    if (!bytes) return fail(TDA_ERR_INVALID_ARG, "bytes is NULL");
    *bytes = 0;
    tda_status st = check_attention(L, "tda_attention_workspace_size");
    if (st) return st;
    if (op != TDA_ATTENTION_FORWARD && op != TDA_ATTENTION_BACKWARD) return fail(TDA_ERR_INVALID_ARG, "bad attention op %d", op);
    if (L->N && L->T) *bytes = attention_ws_bytes(attention_of(L), op == TDA_ATTENTION_BACKWARD, true);
    return TDA_OK;
}

tda_status tda_attention_ranges(int64_t N, int64_t T, const int32_t* doc, const int32_t* prefix, int32_t causal, int64_t window,
                                int32_t* range, void* stream) {
    clear_message();
    if (N < 0 || T < 0 || N > kMaxCount || T > kMaxCount || (N && T > kMaxCount / N))
        return fail(TDA_ERR_INVALID_ARG, "tda_attention_ranges: bad sizes N=%lld T=%lld", (long long)N, (long long)T);
    if (causal != 0 && causal != 1) return fail(TDA_ERR_INVALID_ARG, "tda_attention_ranges: causal must be 0 or 1");
    if (window < 0 || window > kMaxCount) return fail(TDA_ERR_INVALID_ARG, "tda_attention_ranges: bad window %lld", (long long)window);
    if (N == 0 || T == 0) return TDA_OK;
    if (!aligned_to(doc, 4) || !aligned_to(prefix, 4)) return fail(TDA_ERR_INVALID_ARG, "doc or prefix is misaligned");
    if (!range || !aligned_to(range, 8)) return fail(TDA_ERR_INVALID_ARG, "range is NULL or misaligned");
    return cuda_check(launch_attention_ranges(N, T, doc, prefix, causal, window, (int2*)range, (cudaStream_t)stream),
                      "attention ranges");
}

tda_status tda_position_buckets(int32_t n_buckets, int64_t max_distance, int32_t bidirectional, int32_t* bucket) {
    clear_message();
    if (!bucket) return fail(TDA_ERR_INVALID_ARG, "bucket is NULL");
    if (bidirectional != 0 && bidirectional != 1) return fail(TDA_ERR_INVALID_ARG, "bidirectional must be 0 or 1");
    if (n_buckets < (bidirectional ? 4 : 2) || n_buckets > kMaxBuckets || (bidirectional && n_buckets % 2))
        return fail(TDA_ERR_INVALID_ARG, "tda_position_buckets: bad n_buckets %d", n_buckets);
    const int32_t side = bidirectional ? n_buckets / 2 : n_buckets, single = side / 2;
    if (max_distance <= single || max_distance > kMaxReach)
        return fail(TDA_ERR_INVALID_ARG, "tda_position_buckets: max_distance %lld not in (%d, %lld]", (long long)max_distance, single,
                    (long long)kMaxReach);
    const double per = (side - single) / std::log((double)max_distance / single);
    for (int64_t d = -max_distance; d <= max_distance; ++d) {
        const int64_t a = d < 0 ? (bidirectional ? -d : 0) : d;
        // the margin keeps distances on a border, whose logarithms are exact in the reals, in the bucket they begin
        const int64_t far = a < single ? a : single + (int64_t)std::floor(std::log((double)a / single) * per + 1e-9);
        bucket[d + max_distance] = (int32_t)(far < side ? far : side - 1) + (bidirectional && d < 0 ? side : 0);
    }
    return TDA_OK;
}

tda_status tda_attention_forward(const tda_attention_desc* L, const void* Q, int64_t ld_q, const void* K, int64_t ld_k, const void* V,
                                 int64_t ld_v, const int32_t* range, const int32_t* bucket, const void* table, const float* slope,
                                 void* O, int64_t ld_o, float* lse, void* ws, size_t ws_bytes, void* stream) {
    clear_message();
    tda_status st = check_attention(L, "tda_attention_forward");
    if (st) return st;
    if (L->N == 0 || L->T == 0) return TDA_OK;
    if ((st = check_attention_inputs(L, Q, ld_q, K, ld_k, V, ld_v, range, bucket, table, slope)) ||
        (st = check_rows(O, ld_o, (int64_t)L->heads * L->head_dim, L->dtype, false, "O")))
        return st;
    if (!aligned_to(lse, 4)) return fail(TDA_ERR_INVALID_ARG, "lse is misaligned");
    Attention a = attention_of(L);
    a.Q = Q, a.K = K, a.V = V, a.ld_q = ld_q, a.ld_k = ld_k, a.ld_v = ld_v;
    a.range = (const int2*)range, a.bucket = bucket, a.table = table, a.slope = slope, a.O = O, a.ld_o = ld_o, a.lse = lse;
    if ((st = check_ws(ws, ws_bytes, attention_ws_bytes(a, false, false), "tda_attention_forward"))) return st;
    unsigned int* err = device_error_word();
    if (!err) return fail(TDA_ERR_CUDA, "cannot resolve the device error word");
    return cuda_check(launch_attention_forward(a, ws, err, (cudaStream_t)stream), "attention forward");
}

tda_status tda_attention_backward(const tda_attention_desc* L, const void* Q, int64_t ld_q, const void* K, int64_t ld_k, const void* V,
                                  int64_t ld_v, const int32_t* range, const int32_t* bucket, const void* table, const float* slope,
                                  const void* O, int64_t ld_o, const float* lse, const void* dO, int64_t ld_do, void* dQ, int64_t ld_dq,
                                  void* dK, int64_t ld_dk, void* dV, int64_t ld_dv, void* dtable, tda_dtype grad_dtype, float beta,
                                  void* ws, size_t ws_bytes, void* stream) {
    clear_message();
    tda_status st = check_attention(L, "tda_attention_backward");
    if (st) return st;
    if (!float_type(grad_dtype)) return fail(TDA_ERR_INVALID_ARG, "tda_attention_backward: grad_dtype must be TDA_F32 or TDA_BF16");
    if (!std::isfinite(beta)) return fail(TDA_ERR_INVALID_ARG, "tda_attention_backward: beta must be finite");
    if (L->dtype == TDA_F32 && grad_dtype == TDA_BF16)
        return fail(TDA_ERR_UNSUPPORTED, "tda_attention_backward: a bf16 dtable needs bf16 inputs");
    if (dtable && !L->n_buckets) return fail(TDA_ERR_INVALID_ARG, "tda_attention_backward: dtable without n_buckets");
    if (!aligned_to(dtable, el_size(grad_dtype))) return fail(TDA_ERR_INVALID_ARG, "dtable is misaligned");
    if (L->N == 0 || L->T == 0) {
        if (!dtable || beta == 1.f) return TDA_OK;
        return cuda_check(launch_scale_matrix(grad_dtype, dtable, L->n_buckets, L->heads, L->heads, beta, (cudaStream_t)stream),
                          "scale dtable");
    }
    const int64_t q = (int64_t)L->heads * L->head_dim, kv = (int64_t)L->kv_heads * L->head_dim;
    if ((st = check_attention_inputs(L, Q, ld_q, K, ld_k, V, ld_v, range, bucket, table, slope)) ||
        (st = check_rows(O, ld_o, q, L->dtype, false, "O")) || (st = check_rows(dO, ld_do, q, L->dtype, false, "dO")) ||
        (st = check_rows(dQ, ld_dq, q, L->dtype, false, "dQ")) || (st = check_rows(dK, ld_dk, kv, L->dtype, false, "dK")) ||
        (st = check_rows(dV, ld_dv, kv, L->dtype, false, "dV")))
        return st;
    if (!lse || !aligned_to(lse, 4)) return fail(TDA_ERR_INVALID_ARG, "lse is NULL or misaligned");
    Attention a = attention_of(L);
    a.Q = Q, a.K = K, a.V = V, a.ld_q = ld_q, a.ld_k = ld_k, a.ld_v = ld_v;
    a.range = (const int2*)range, a.bucket = bucket, a.table = table, a.slope = slope;
    a.O = const_cast<void*>(O), a.ld_o = ld_o, a.lse = const_cast<float*>(lse), a.dO = dO, a.ld_do = ld_do;
    a.dQ = dQ, a.dK = dK, a.dV = dV, a.ld_dq = ld_dq, a.ld_dk = ld_dk, a.ld_dv = ld_dv;
    a.dtable = dtable, a.gt = grad_dtype, a.beta = beta;
    if ((st = check_ws(ws, ws_bytes, attention_ws_bytes(a, true, false), "tda_attention_backward"))) return st;
    unsigned int* err = device_error_word();
    if (!err) return fail(TDA_ERR_CUDA, "cannot resolve the device error word");
    return cuda_check(launch_attention_backward(a, ws, err, (cudaStream_t)stream), "attention backward");
}

tda_status tda_rmsnorm_forward(tda_dtype dtype, const void* x, int64_t ld_x, const void* r, int64_t ld_r, int64_t M, int64_t d,
                               const void* w, float eps, void* h, int64_t ld_h, void* y, int64_t ld_y, float* rstd, void* stream) {
    clear_message();
    tda_status st = check_norm(dtype, M, d, "tda_rmsnorm_forward");
    if (st) return st;
    if (!(eps > 0) || !std::isfinite(eps)) return fail(TDA_ERR_INVALID_ARG, "tda_rmsnorm_forward: eps must be finite and > 0");
    if (M == 0) return TDA_OK;
    if ((st = check_rows(x, ld_x, d, dtype, false, "x")) || (st = check_rows(r, ld_r, d, dtype, true, "r")) ||
        (st = check_rows(w, d, d, dtype, false, "w")) || (st = check_rows(h, ld_h, d, dtype, true, "h")) ||
        (st = check_rows(y, ld_y, d, dtype, false, "y")))
        return st;
    if (!aligned_to(rstd, 4)) return fail(TDA_ERR_INVALID_ARG, "rstd is misaligned");
    return cuda_check(launch_norm_forward(dtype, x, ld_x, r, ld_r, M, d, w, eps, h, ld_h, y, ld_y, rstd, (cudaStream_t)stream),
                      "norm forward");
}

size_t tda_rmsnorm_workspace_size(int64_t M, int64_t d) {
    if (M < 0 || M > kMaxCount || d < 1 || d > kNormMaxRow) return 0;
    return norm_ws_bytes(M, d);
}

tda_status tda_rmsnorm_backward(tda_dtype dtype, const void* h, int64_t ld_h, const float* rstd, const void* w, const void* dy,
                                int64_t ld_dy, const void* dres, int64_t ld_r, int64_t M, int64_t d, void* dx, int64_t ld_dx,
                                void* dw, tda_dtype grad_dtype, float beta, void* ws, size_t ws_bytes, void* stream) {
    clear_message();
    tda_status st = check_norm(dtype, M, d, "tda_rmsnorm_backward");
    if (st) return st;
    if (!float_type(grad_dtype)) return fail(TDA_ERR_INVALID_ARG, "tda_rmsnorm_backward: grad_dtype must be TDA_F32 or TDA_BF16");
    if (!std::isfinite(beta)) return fail(TDA_ERR_INVALID_ARG, "tda_rmsnorm_backward: beta must be finite");
    if (dtype == TDA_F32 && grad_dtype == TDA_BF16)
        return fail(TDA_ERR_UNSUPPORTED, "tda_rmsnorm_backward: bf16 gradients of w need bf16 rows");
    if ((st = check_rows(dw, d, d, grad_dtype, true, "dw"))) return st;
    if (M == 0) {
        if (!dw || beta == 1.f) return TDA_OK;
        return cuda_check(launch_scale_matrix(grad_dtype, dw, 1, d, d, beta, (cudaStream_t)stream), "scale dw");
    }
    if ((st = check_rows(h, ld_h, d, dtype, false, "h")) || (st = check_rows(w, d, d, dtype, false, "w")) ||
        (st = check_rows(dy, ld_dy, d, dtype, false, "dy")) || (st = check_rows(dres, ld_r, d, dtype, true, "dres")) ||
        (st = check_rows(dx, ld_dx, d, dtype, true, "dx")))
        return st;
    if (!rstd || !aligned_to(rstd, 4)) return fail(TDA_ERR_INVALID_ARG, "rstd is NULL or misaligned");
    if (!dx && !dw) return TDA_OK;
    if (dw && (st = check_ws(ws, ws_bytes, norm_ws_bytes(M, d), "tda_rmsnorm_backward"))) return st;
    return cuda_check(launch_norm_backward(dtype, h, ld_h, rstd, w, dy, ld_dy, dres, ld_r, M, d, dx, ld_dx, dw, grad_dtype, beta,
                                           (float*)ws, (cudaStream_t)stream),
                      "norm backward");
}

}  // extern "C"
