// k_norm.cu -- root-mean-square norm with the residual's addition, and its gradient.
//   h = x + r (stored),  rstd = 1 / sqrt(mean h^2 + eps),  y = h rstd w
//   n = h rstd,  g = dy w,  dx = dres + rstd (g - n mean(g n)),  dw = beta dw + sum over rows of dy n
// Bound by HBM: a row is read once, held in registers between its sum and its use, and written once. A warp (short rows)
// or a CTA has a row, 16 or 32 values a thread in 16-byte vectors where every tensor allows it.
#include <cuda_bf16.h>

#include <algorithm>

#include "linear.cuh"
#include "tda_internal.cuh"

namespace tda {
namespace {

constexpr int kWarpCta = 128;  // threads of a CTA whose warps have a row each

template <typename T>
struct Vec;
template <>
struct Vec<float> {
    static constexpr int n = 4;
};
template <>
struct Vec<__nv_bfloat16> {
    static constexpr int n = 8;
};

__device__ __forceinline__ float wide(float x) { return x; }
__device__ __forceinline__ float wide(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void narrow(float x, float* p) { *p = x; }
__device__ __forceinline__ void narrow(float x, __nv_bfloat16* p) { *p = __float2bfloat16(x); }

// The columns of thread t of G: vectors t, t + G, ... of a row, or its single values.
template <typename T, int VALS, bool ALIGNED>
struct Row {
    static constexpr int kVec = ALIGNED ? Vec<T>::n : 1, kParts = VALS / kVec;
    __device__ static __forceinline__ void load(const T* p, int d, int t, int G, T (&v)[VALS]) {
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            const int c = (t + i * G) * kVec;
            if constexpr (ALIGNED) {
                *(uint4*)&v[i * kVec] = c < d ? *(const uint4*)(p + c) : make_uint4(0, 0, 0, 0);
            } else {
                if (c < d) v[i] = p[c];
                else narrow(0.f, &v[i]);
            }
        }
    }
    __device__ static __forceinline__ void store(T* p, int d, int t, int G, const T (&v)[VALS]) {
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            const int c = (t + i * G) * kVec;
            if (c >= d) continue;
            if constexpr (ALIGNED) *(uint4*)(p + c) = *(const uint4*)&v[i * kVec];
            else p[c] = v[i];
        }
    }
};

// Sum over the threads of a row's group, the same in all of them.
template <bool WARP>
__device__ __forceinline__ float group_sum(float v, float* parts) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (!WARP) {
        if (threadIdx.x % 32 == 0) parts[threadIdx.x / 32] = v;
        __syncthreads();
        v = 0.f;
        for (int i = 0; i < (int)blockDim.x / 32; ++i) v += parts[i];
        __syncthreads();
    }
    return v;
}

template <typename T, int VALS, bool ALIGNED, bool WARP>
__global__ __launch_bounds__(WARP ? kWarpCta : 1024) void norm_kernel(const T* x, int64_t ld_x, const T* r, int64_t ld_r, int64_t M,
                                                                     int d, const T* w, float eps, T* h, int64_t ld_h, T* y,
                                                                     int64_t ld_y, float* rstd) {
    using R = Row<T, VALS, ALIGNED>;
    __shared__ float parts[32];
    const int G = WARP ? 32 : blockDim.x, t = WARP ? threadIdx.x % 32 : threadIdx.x;
    const int64_t row = WARP ? (int64_t)blockIdx.x * (kWarpCta / 32) + threadIdx.x / 32 : blockIdx.x;
    if (row >= M) return;
    alignas(16) T v[VALS], u[VALS], weight[VALS];
    R::load(x + row * ld_x, d, t, G, v);
    if (r) {
        R::load(r + row * ld_r, d, t, G, u);
#pragma unroll
        for (int i = 0; i < VALS; ++i) narrow(wide(v[i]) + wide(u[i]), &v[i]);
    }
    R::load(w, d, t, G, weight);
    if (h) R::store(h + row * ld_h, d, t, G, v);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < VALS; ++i) sum = fmaf(wide(v[i]), wide(v[i]), sum);
    sum = group_sum<WARP>(sum, parts);
    const float by = 1.f / sqrtf(sum / (float)d + eps);
    if (rstd && t == 0) rstd[row] = by;
#pragma unroll
    for (int i = 0; i < VALS; ++i) narrow(wide(v[i]) * by * wide(weight[i]), &u[i]);
    R::store(y + row * ld_y, d, t, G, u);
}

// Group g of `groups` takes rows g, g + groups, ... and keeps its share of dw in registers; a CTA's share goes to
// part[CTA][d], the warps of a CTA joined in order.
template <typename T, int VALS, bool ALIGNED, bool WARP>
__global__ __launch_bounds__(WARP ? kWarpCta : 1024) void norm_grad_kernel(const T* h, int64_t ld_h, const float* rstd, const T* w,
                                                                          const T* dy, int64_t ld_dy, const T* dres, int64_t ld_r,
                                                                          int64_t M, int d, T* dx, int64_t ld_dx, float* part) {
    using R = Row<T, VALS, ALIGNED>;
    extern __shared__ float joined[];  // WARP: 4 rows of VALS * 32 values
    __shared__ float parts[32];
    constexpr int kRows = WARP ? kWarpCta / 32 : 1;
    const int G = WARP ? 32 : blockDim.x, t = WARP ? threadIdx.x % 32 : threadIdx.x;
    const int64_t groups = (int64_t)gridDim.x * kRows;
    alignas(16) T weight[VALS];
    float dw[VALS];
    R::load(w, d, t, G, weight);
#pragma unroll
    for (int i = 0; i < VALS; ++i) dw[i] = 0.f;
    for (int64_t row = (int64_t)blockIdx.x * kRows + (WARP ? threadIdx.x / 32 : 0); row < M; row += groups) {
        alignas(16) T v[VALS], u[VALS], q[VALS];
        R::load(h + row * ld_h, d, t, G, v);
        R::load(dy + row * ld_dy, d, t, G, u);
        if (dres) R::load(dres + row * ld_r, d, t, G, q);
        const float by = rstd[row];
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < VALS; ++i) {
            const float n = wide(v[i]) * by, g = wide(u[i]);
            dw[i] = fmaf(g, n, dw[i]);
            sum = fmaf(g * wide(weight[i]), n, sum);
        }
        if (!dx) continue;
        sum = group_sum<WARP>(sum, parts) / (float)d;
#pragma unroll
        for (int i = 0; i < VALS; ++i) {
            const float n = wide(v[i]) * by, g = wide(u[i]) * wide(weight[i]);
            float o = by * fmaf(-n, sum, g);
            if (dres) o += wide(q[i]);
            narrow(o, &v[i]);
        }
        R::store(dx + row * ld_dx, d, t, G, v);
    }
    if (!part) return;
    float* out = part + (int64_t)blockIdx.x * d;
    if constexpr (WARP) {
#pragma unroll
        for (int i = 0; i < VALS; ++i) {
            const int c = (t + i / R::kVec * 32) * R::kVec + i % R::kVec;
            joined[threadIdx.x / 32 * VALS * 32 + c] = dw[i];
        }
        __syncthreads();
        for (int c = threadIdx.x; c < d; c += kWarpCta) {
            float s = 0.f;
            for (int k = 0; k < kRows; ++k) s += joined[k * VALS * 32 + c];
            out[c] = s;
        }
    } else {
#pragma unroll
        for (int i = 0; i < VALS; ++i) {
            const int c = (t + i / R::kVec * G) * R::kVec + i % R::kVec;
            if (c < d) out[c] = dw[i];
        }
    }
}

// dw[c] = beta dw[c] + sum of the CTAs' shares: 8 threads a column at different shares, joined in order.
template <typename G>
__global__ __launch_bounds__(256) void norm_dw_kernel(const float* part, int rows, int d, float beta, G* dw) {
    chain_wait();
    __shared__ float sums[8][33];
    const int c = blockIdx.x * 32 + threadIdx.x % 32, k = threadIdx.x / 32;
    float s = 0.f;
    if (c < d)
        for (int i = k; i < rows; i += 8) s += part[(int64_t)i * d + c];
    sums[k][threadIdx.x % 32] = s;
    __syncthreads();
    if (k == 0 && c < d) {
        s = 0.f;
        for (int i = 0; i < 8; ++i) s += sums[i][threadIdx.x];
        if (beta != 0.f) s = fmaf(beta, wide(dw[c]), s);
        narrow(s, &dw[c]);
    }
}

struct Plan {
    int vals, threads;
    bool warp;
};
Plan plan_of(int d) {
    if (d <= 512) return {16, kWarpCta, true};
    if (d <= 1024) return {32, kWarpCta, true};
    const int vals = d <= 16384 ? 16 : 32;
    return {vals, std::max(64, (d + vals - 1) / vals + 31) / 32 * 32, false};
}
int64_t grad_ctas(int64_t M, int d) {
    const Plan p = plan_of(d);
    const int64_t rows = p.warp ? kWarpCta / 32 : 1, each = p.warp ? 8 : std::max(1, 1024 / p.threads);
    return std::min<int64_t>((M + rows - 1) / rows, (int64_t)train_sms() * each);
}

bool vectors(const void* p, int64_t ld, size_t el) { return !p || (((uintptr_t)p | (uintptr_t)(ld * (int64_t)el)) & 15) == 0; }

// f.template operator()<VALS, ALIGNED, WARP>() for a plan.
template <typename F>
cudaError_t with_plan(const Plan& p, bool aligned, F&& f) {
    auto go = [&](auto vals, auto warp) {
        return aligned ? f(vals, std::true_type(), warp) : f(vals, std::false_type(), warp);
    };
    using V16 = std::integral_constant<int, 16>;
    using V32 = std::integral_constant<int, 32>;
    if (p.warp) return p.vals == 16 ? go(V16(), std::true_type()) : go(V32(), std::true_type());
    return p.vals == 16 ? go(V16(), std::false_type()) : go(V32(), std::false_type());
}

template <typename T>
cudaError_t forward(const void* x, int64_t ld_x, const void* r, int64_t ld_r, int64_t M, int d, const void* w, float eps, void* h,
                    int64_t ld_h, void* y, int64_t ld_y, float* rstd, cudaStream_t s) {
    constexpr size_t el = sizeof(T);
    const bool aligned = d % Vec<T>::n == 0 && vectors(x, ld_x, el) && vectors(r, ld_r, el) && vectors(w, 0, el) &&
                         vectors(h, ld_h, el) && vectors(y, ld_y, el);
    const Plan p = plan_of(d);
    const unsigned grid = (unsigned)(p.warp ? (M + kWarpCta / 32 - 1) / (kWarpCta / 32) : M);
    note_launches(1);
    return with_plan(p, aligned, [&](auto vals, auto al, auto warp) {
        norm_kernel<T, vals.value, al.value, warp.value><<<grid, p.threads, 0, s>>>(
            (const T*)x, ld_x, (const T*)r, ld_r, M, d, (const T*)w, eps, (T*)h, ld_h, (T*)y, ld_y, rstd);
        return cudaGetLastError();
    });
}

template <typename T>
cudaError_t backward(const void* h, int64_t ld_h, const float* rstd, const void* w, const void* dy, int64_t ld_dy, const void* dres,
                     int64_t ld_r, int64_t M, int d, void* dx, int64_t ld_dx, void* dw, tda_dtype gt, float beta, float* part,
                     cudaStream_t s) {
    constexpr size_t el = sizeof(T);
    const bool aligned = d % Vec<T>::n == 0 && vectors(h, ld_h, el) && vectors(w, 0, el) && vectors(dy, ld_dy, el) &&
                         vectors(dres, ld_r, el) && vectors(dx, ld_dx, el);
    const Plan p = plan_of(d);
    const int64_t ctas = grad_ctas(M, d);
    note_launches(1);
    cudaError_t e = with_plan(p, aligned, [&](auto vals, auto al, auto warp) {
        const size_t smem = warp.value ? (size_t)kWarpCta * vals.value * 4 : 0;
        norm_grad_kernel<T, vals.value, al.value, warp.value><<<(unsigned)ctas, p.threads, smem, s>>>(
            (const T*)h, ld_h, rstd, (const T*)w, (const T*)dy, ld_dy, (const T*)dres, ld_r, M, d, (T*)dx, ld_dx,
            dw ? part : nullptr);
        return cudaGetLastError();
    });
    if (e || !dw) return e;
    const dim3 grid((unsigned)((d + 31) / 32));
    return gt == TDA_BF16 ? launch_chained(true, norm_dw_kernel<__nv_bfloat16>, grid, dim3(256), 0, s, (const float*)part, (int)ctas, d,
                                           beta, (__nv_bfloat16*)dw)
                          : launch_chained(true, norm_dw_kernel<float>, grid, dim3(256), 0, s, (const float*)part, (int)ctas, d, beta,
                                           (float*)dw);
}

}  // namespace

size_t norm_ws_bytes(int64_t M, int64_t d) { return M == 0 ? 0 : (size_t)grad_ctas(M, (int)d) * d * 4; }

cudaError_t launch_norm_forward(tda_dtype dt, const void* x, int64_t ld_x, const void* r, int64_t ld_r, int64_t M, int64_t d,
                                const void* w, float eps, void* h, int64_t ld_h, void* y, int64_t ld_y, float* rstd, cudaStream_t s) {
    return dt == TDA_BF16 ? forward<__nv_bfloat16>(x, ld_x, r, ld_r, M, (int)d, w, eps, h, ld_h, y, ld_y, rstd, s)
                          : forward<float>(x, ld_x, r, ld_r, M, (int)d, w, eps, h, ld_h, y, ld_y, rstd, s);
}

cudaError_t launch_norm_backward(tda_dtype dt, const void* h, int64_t ld_h, const float* rstd, const void* w, const void* dy,
                                 int64_t ld_dy, const void* dres, int64_t ld_r, int64_t M, int64_t d, void* dx, int64_t ld_dx, void* dw,
                                 tda_dtype gt, float beta, float* part, cudaStream_t s) {
    return dt == TDA_BF16
               ? backward<__nv_bfloat16>(h, ld_h, rstd, w, dy, ld_dy, dres, ld_r, M, (int)d, dx, ld_dx, dw, gt, beta, part, s)
               : backward<float>(h, ld_h, rstd, w, dy, ld_dy, dres, ld_r, M, (int)d, dx, ld_dx, dw, gt, beta, part, s);
}

}  // namespace tda
