// attention.cuh -- what the translation units of the attention share: the arguments of a
// pass, a row's visible keys, the scores' cap and biases. Internal.
#pragma once

#include <cfloat>

#include <cuda_bf16.h>

#include "tda_internal.cuh"

namespace tda {

// One call. Row i of example n is token n T + i; head h's values start at column h hd of its row.
struct Attention {
    int64_t N, T;
    int H, KV, hd;
    tda_dtype dt;
    float scale, cap;
    int causal, n_buckets;
    int64_t reach;          // distances are held within +-reach for the table
    const void *Q, *K, *V;
    int64_t ld_q, ld_k, ld_v;
    const int2* range;      // [N][T] keys [lo, hi), or NULL
    const int32_t* bucket;  // [2 reach + 1]
    const void* table;      // [n_buckets][H]
    const float* slope;     // [H] or NULL
    void* O;
    int64_t ld_o;
    float* lse;             // [N][H][T]
    // backward pass
    const void* dO;
    void *dQ, *dK, *dV, *dtable;
    int64_t ld_do, ld_dq, ld_dk, ld_dv;
    tda_dtype gt;
    float beta;
    // tensor-core kernels with a cap: tanh(x / cap) of a dot product d up to near_limit is d P(d^2), times what the kernel wants
    float near_limit;
    float2 near[5];  // P's coefficients, the highest first, in pairs as the instructions take them
};

// Division of numbers below 2^31 by a number that a launch knows.
struct FastDiv {
    uint32_t d = 1, mul = 0, shift = 0;
    FastDiv() = default;
    explicit FastDiv(uint32_t n) : d(n) {
        uint32_t bits = 0;
        while ((1ull << bits) < n) ++bits;
        if (n > 1) mul = (uint32_t)(((1ull << (31 + bits)) + n - 1) / n), shift = bits - 1;
    }
    __host__ __device__ __forceinline__ int div(int x) const {
#ifdef __CUDA_ARCH__
        return d == 1 ? x : (int)(__umulhi((uint32_t)x, mul) >> shift);
#else
        return d == 1 ? x : (int)((((uint64_t)(uint32_t)x * mul) >> 32) >> shift);
#endif
    }
    __host__ __device__ __forceinline__ int mod(int x) const { return x - div(x) * (int)d; }
};

// Keys [x, y) that row i of an example sees; rows past T see none.
__device__ __forceinline__ int2 visible(const int2* range, int causal, int T, int64_t row0, int i) {
    if (i >= T) return make_int2(0, 0);
    if (range) {
        const int2 r = range[row0 + i];
        return make_int2(min(max(r.x, 0), T), min(max(r.y, 0), T));  // both ways: differences of the ends fit an int then
    }
    return make_int2(0, causal ? i + 1 : T);
}

// What distance d = i - j adds to a score of head h.
template <typename T>
__device__ __forceinline__ float distance_bias(const int32_t* bucket, const T* table, const float* slope, int n_buckets,
                                               int64_t reach, int H, int h, int64_t d) {
    float v = 0.f;
    if (n_buckets) {
        const int64_t c = d < -reach ? -reach : d > reach ? reach : d;
        const int b = bucket[c + reach];
        if (b >= 0 && b < n_buckets) v = (float)table[(int64_t)b * H + h];
    }
    if (slope) v -= slope[h] * (float)(d < 0 ? -d : d);
    return v;
}

// What a call's first kernel finds for the tensor-core kernels, in the workspace.
struct AttentionTile {  // of 128 tokens
    int lo, hi;         // keys that its queries see: all within [lo, hi)
    int most, least;    // largest start and smallest end of a query's keys: what lies between is seen by all
    uint32_t unseen[4]; // keys of this tile that no query of the example sees
    uint32_t idle[4];   // queries that see nothing
};
struct AttentionPlan {
    AttentionTile* tiles;  // [N][tiles], where a range is given
    int* taken;            // the same: items of the forward pass that CTAs have taken
    float* lut;            // [H][lut_len] bias of a distance times log2 e, where there is any; distance 0 at lut_mid
    int lut_len, lut_mid;
    int reach;             // distances beyond it have the bias of +-reach
};

// The tensor-core kernels sum dS by distance where the distances within the table's reach fit 1024 values (distance 0 at the
// returned place), else by bucket (-1).
__host__ __device__ inline int attention_dense_mid(const Attention& a) {
    const int64_t reach = a.reach < a.T - 1 ? a.reach : a.T - 1;
    return 2 * reach + 1 <= 1024 ? (int)reach : -1;
}
inline int attention_part_width(const Attention& a) {
    const int mid = attention_dense_mid(a);
    return a.n_buckets == 0 ? 0 : mid >= 0 ? 2 * mid + 1 : a.n_buckets;
}

// Workspace of a call, and its launches; bound: enough for any range, slope and alignment. The CUDA-core kernels
// (k_attention.cu) take every shape; the tensor-core ones (k_attention_tc.cu, k_attention_grad_tc.cu) bf16 with aligned rows.
size_t attention_ws_bytes(const Attention& a, bool backward, bool bound);
cudaError_t launch_attention_forward(const Attention& a, void* ws, unsigned int* err, cudaStream_t s);
cudaError_t launch_attention_backward(const Attention& a, void* ws, unsigned int* err, cudaStream_t s);
cudaError_t launch_attention_ranges(int64_t N, int64_t T, const int32_t* doc, const int32_t* prefix, int causal,
                                    int64_t window, int2* range, cudaStream_t s);

bool attention_tc_supported(const Attention& a, bool backward);
// a.near_limit and a.near for d P(d^2) = by * tanh(d scale / cap).
void attention_near(Attention& a, float by);
size_t attention_plan_bytes(const Attention& a, bool bound);
// Fills the plan; *chained: a kernel was launched, the next may be chained to it.
cudaError_t launch_attention_plan(const Attention& a, void* ws, AttentionPlan* plan, bool* chained, cudaStream_t s);
bool attention_head_map(void* map, const void* p, int64_t ld, int heads, int hd, int64_t T, int64_t N, int rows);
cudaError_t launch_attention_forward_tc(const Attention& a, void* ws, unsigned int* err, cudaStream_t s);
// *part: [H][N * tiles][attention_part_width] sums of dS, where a.dtable is wanted.
size_t attention_grad_tc_bytes(const Attention& a, bool bound);
cudaError_t launch_attention_backward_tc(const Attention& a, void* ws, unsigned int* err, float** part, cudaStream_t s);

}  // namespace tda
