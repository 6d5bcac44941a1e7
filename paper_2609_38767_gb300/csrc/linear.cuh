// linear.cuh -- what the translation units of the linear layer share: the
// activations with their derivatives, the operands and the epilogue of the
// tensor-core product. Internal.
#pragma once

#include <cuda_bf16.h>

#include "tda_internal.cuh"

namespace tda {

// ------------------------------------------------------------------ activations
// Values in forms without cancellation or overflow: gelu through the normal tail, the tanh form as
// z sigmoid(2u) (tanh(u) = 2 sigmoid(2u) - 1). exp of a large argument gives 0 or inf,
// and 1 / (1 + inf) = 0, so finite z of any size give finite results. Slopes of an infinite z are their limits,
// the value of +inf is +inf; the value of -inf is NaN (-inf times 0) but for relu.
// FAST (bf16 results): the exponential and the reciprocal by the approximate instructions, good to
// 2^-21 |x| and 2^-22 of their value, far below bf16's 2^-8 (4096 x 2048 -> 8192 with tanh-gelu and Z 94 -> 93 us).
template <bool FAST>
__device__ __forceinline__ float exp_of(float x) {
    if (!FAST) return expf(x);
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(1.4426950408889634f * x));
    return y;
}
template <bool FAST>
__device__ __forceinline__ float reciprocal(float x) {
    if (!FAST) return 1.f / x;
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
template <bool FAST>
__device__ __forceinline__ float sigmoid(float x) {
    return reciprocal<FAST>(1.f + exp_of<FAST>(-x));
}

// q = Phi(-|z|) and e = exp(-z^2/2). FAST: q = e t P(t), t = 1 / (1 + 0.2895 |z|), whose form has the tail's 1 / |z|; P of
// degree 5 fitted for |z| <= 13.3, past which e is 0, to a relative error of 1.1e-4 (2^-13, below bf16's rounding) in
// the far tail and an absolute one of 2e-7, fp32's roundings included.
template <bool FAST>
__device__ __forceinline__ float normal_tail(float z, float* e) {
    const float a = fabsf(z);
    *e = exp_of<FAST>(-0.5f * z * z);
    if (!FAST) return 0.5f * erfcf(0.70710678118654752f * a);
    const float t = reciprocal<FAST>(fmaf(0.28948054575753167f, a, 1.f));
    float s = fmaf(t, -0.0903595890286826f, 0.2922750212769822f);
    s = fmaf(t, s, -0.10288718530166549f);
    s = fmaf(t, s, 0.1853646140376046f);
    s = fmaf(t, s, 0.09875243697672076f);
    s = fmaf(t, s, 0.11685465736958278f);
    return t * s * *e;
}

template <int ACT, bool FAST>
__device__ __forceinline__ float act_value(float z) {
    if (ACT == TDA_ACT_RELU) return z > 0.f ? z : z != z ? z : 0.f;
    if (ACT == TDA_ACT_GELU) {
        float e;
        const float q = normal_tail<FAST>(z, &e);
        return z * (z > 0.f ? 1.f - q : q);  // +inf stays +inf
    }
    if (ACT == TDA_ACT_GELU_TANH) return z * sigmoid<FAST>(1.5957691216057308f * fmaf(0.044715f * z * z, z, z));
    if (ACT == TDA_ACT_SILU) return z * sigmoid<FAST>(z);
    return z;
}

template <int ACT, bool FAST>
__device__ __forceinline__ float act_slope(float z) {
    if (ACT == TDA_ACT_RELU) return z > 0.f ? 1.f : z != z ? z : 0.f;
    if (ACT == TDA_ACT_GELU) {
        float e;
        const float q = normal_tail<FAST>(z, &e);
        // past |z| = 20 e is 0: an infinite z has the slope's limit, 0 or 1 (a NaN is one in q)
        return fmaf(0.39894228040143268f * fminf(fmaxf(z, -20.f), 20.f), e, z > 0.f ? 1.f - q : q);
    }
    if (ACT == TDA_ACT_GELU_TANH) {
        // past |z| = 9.9 the slope is 0 or 1 to fp32, while z^2 or the exponential could overflow;
        // 1 - s = e s without the cancellation
        const float c = fminf(fmaxf(z, -9.9f), 9.9f);
        const float x = -1.5957691216057308f * fmaf(0.044715f * c * c, c, c), e = exp_of<FAST>(x);
        const float s = reciprocal<FAST>(1.f + e);
        const float r = fmaf(c * s * (e * s), 1.5957691216057308f * fmaf(0.134145f * c, c, 1.f), s);
        return z != z ? z : r;
    }
    if (ACT == TDA_ACT_SILU) {
        // 1 - s = e s; e stays below 2^126, and past z = 86 it is 0 beside 1
        const float c = fminf(fmaxf(z, -86.f), 86.f), e = exp_of<FAST>(-c);
        const float s = reciprocal<FAST>(1.f + e);
        const float r = s * fmaf(c, e * s, 1.f);
        return z != z ? z : r;
    }
    return 1.f;
}

// ------------------------------------------------------------------ the tensor-core product
// D[i][j] = sum_k P[i][k] Q[j][k]. An operand is a matrix in memory of `rows` rows of `cols`
// contiguous bf16 values, K-major (rows are i or j, columns k) or MN-major (mn: rows are k),
// with 16-byte aligned rows. planes = 3: three such matrices whose sum is an fp32 operand.
struct LinearOperand {
    const void* p;
    int64_t rows, cols, ld;
    int64_t plane_stride;  // elements
    int planes;
    bool mn;
    int64_t extent() const { return mn ? cols : rows; }
    int64_t depth() const { return mn ? rows : cols; }
};

// The epilogue: z = D + bias[n]; Z = z; Y = act(z) + r_scale R. All of the output's type.
struct LinearEpilogue {
    int64_t M, N;  // output rows and columns
    const void* bias;
    const void* R;
    int64_t ld_r;
    float r_scale;
    void* Y;
    int64_t ld_y;
    void* Z;
    int64_t ld_z;
    int act;
    int vec;  // all of bias, R, Y, Z may be moved four values at a time
    int wide; // rows of all of them start on 16 bytes
    int f32;  // type of bias, R, Y, Z (set by the launch)
};

// ------------------------------------------------------------------ the two passes (k_linear.cu)
struct LinearForward {
    int64_t M, d_in, d_out;
    int act;
    tda_dtype dt;
    const void *X, *W, *bias, *R;
    void *Y, *Z;
    int64_t ld_x, ld_w, ld_r, ld_y, ld_z;
};
struct LinearBackward {
    int64_t M, d_in, d_out;
    int act;
    tda_dtype dt, gt;
    float beta;
    const void *dY, *Z, *X, *W;
    void *B, *dX, *dW, *db;
    int64_t ld_dy, ld_z, ld_x, ld_w, ld_b, ld_dx, ld_dw;
};
size_t linear_forward_ws(const LinearForward& f);
size_t linear_backward_ws(const LinearBackward& b);
// The same from the sizes alone: packed = every operand needs planes of its own.
size_t linear_ws_bound(bool backward, int64_t M, int64_t d_in, int64_t d_out, tda_dtype dt, bool packed);
cudaError_t launch_linear_forward(const LinearForward& f, void* ws, unsigned int* err, cudaStream_t s);
cudaError_t launch_linear_backward(const LinearBackward& b, void* ws, unsigned int* err, cudaStream_t s);
cudaError_t launch_scale_matrix(tda_dtype dt, void* x, int64_t rows, int64_t cols, int64_t ld, float beta,
                                cudaStream_t s);

bool linear_tc_available();
// One product, or two that do not read each other's output, each with its epilogue; out: type of bias, R, Y, Z.
struct LinearProduct {
    LinearOperand P, Q;
    LinearEpilogue ep;
    tda_dtype out;
};
// A few rows on the CUDA cores (k_linear_rows.cu): the forward product with its epilogue, and dX of fp32 layers.
bool linear_rows_preferred(int64_t M, tda_dtype dt);
cudaError_t launch_linear_rows(const void* X, int64_t ld_x, const void* W, int64_t ld_w, int64_t K,
                               const LinearEpilogue& ep, tda_dtype dt, cudaStream_t s);
cudaError_t launch_linear_cols(const float* B, int64_t ld_b, const float* W, int64_t ld_w, float* dX, int64_t ld_dx,
                               int64_t M, int64_t N, int64_t K, bool chained, cudaStream_t s);
// chained: after another kernel of the same call.
// dW of a few rows: rank-M updates on the CUDA cores.
cudaError_t launch_linear_outer(const void* B, int64_t ld_b, const void* X, int64_t ld_x, int64_t M, int64_t N, int64_t K,
                                tda_dtype dt, void* dW, int64_t ld_dw, tda_dtype gt, float beta, bool chained,
                                cudaStream_t s);
cudaError_t launch_linear_products(const LinearProduct* x, int count, bool chained, unsigned int* err,
                                   cudaStream_t s);

}  // namespace tda
