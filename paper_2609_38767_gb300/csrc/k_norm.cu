// k_norm.cu -- root-mean-square norm with the residual's addition, and its gradient.
//   h = x + r (stored),  rstd = 1 / sqrt(mean h^2 + eps),  y = h rstd w
//   n = h rstd,  g = dy w,  dx = dres + rstd (g - n mean(g n)),  dw = beta dw + sum over rows of dy n
// Bound by HBM: a row is read once, held in registers between its sum and its use, and written once. A warp (short rows)
// or a CTA has a row, 32 to 128 bytes a thread in 16-byte vectors where every tensor allows it.
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

// The columns of thread t of G: vectors t, t + G, ... of a row, or its single values, as they lie in 32-bit words (two bf16 each:
// arrays of single bf16 took 38 instructions a value in the gradient's kernel).
template <typename T, int VALS, bool ALIGNED>
struct Row {
    static constexpr int kVec = ALIGNED ? Vec<T>::n : 1, kParts = VALS / kVec, kWords = VALS * (int)sizeof(T) / 4;
    static constexpr bool kPairs = sizeof(T) == 2;
    uint32_t r[kWords];
    __device__ __forceinline__ float at(int i) const {
        if constexpr (!kPairs) return __uint_as_float(r[i]);
        else return __uint_as_float(i % 2 ? r[i / 2] & 0xffff0000u : r[i / 2] << 16);
    }
    // values i and i + 1, i even
    __device__ __forceinline__ void put(int i, float x, float y) {
        if constexpr (!kPairs) r[i] = __float_as_uint(x), r[i + 1] = __float_as_uint(y);
        else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r[i / 2]) : "f"(y), "f"(x));
    }
    __device__ __forceinline__ void put_bits(int i, uint32_t bits) {  // in the order of i
        if constexpr (!kPairs) r[i] = bits;
        else r[i / 2] = i % 2 ? r[i / 2] | bits << 16 : bits;
    }
    __device__ __forceinline__ uint32_t bits(int i) const {
        if constexpr (!kPairs) return r[i];
        else return i % 2 ? r[i / 2] >> 16 : r[i / 2] & 0xffffu;
    }
    __device__ __forceinline__ void put_vector(int part, uint4 x) {
        r[4 * part] = x.x, r[4 * part + 1] = x.y, r[4 * part + 2] = x.z, r[4 * part + 3] = x.w;
    }
    __device__ __forceinline__ void load(const T* p, int d, int t, int G) {
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            const int c = (t + i * G) * kVec;
            if constexpr (ALIGNED) put_vector(i, c < d ? *(const uint4*)(p + c) : make_uint4(0, 0, 0, 0));
            else if constexpr (kPairs) put_bits(i, c < d ? ((const uint16_t*)p)[c] : 0);
            else put_bits(i, c < d ? ((const uint32_t*)p)[c] : 0);
        }
    }
    __device__ __forceinline__ void store(T* p, int d, int t, int G) const {
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            const int c = (t + i * G) * kVec;
            if (c >= d) continue;
            if constexpr (ALIGNED) *(uint4*)(p + c) = make_uint4(r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]);
            else if constexpr (kPairs) ((uint16_t*)p)[c] = (uint16_t)bits(i);
            else ((uint32_t*)p)[c] = bits(i);
        }
    }
};

// Sum over the threads of a row's group, the same in all of them.
// parts: 32 values that the next sum does not use.
template <bool WARP>
__device__ __forceinline__ float group_sum(float v, float* parts) {
#pragma unroll
    for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if constexpr (!WARP) {
        if (threadIdx.x % 32 == 0) parts[threadIdx.x / 32] = v;
        __syncthreads();
        v = threadIdx.x % 32 < blockDim.x / 32 ? parts[threadIdx.x % 32] : 0.f;
#pragma unroll
        for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
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
    R v, u, weight;
    v.load(x + row * ld_x, d, t, G);
    if (r) {
        u.load(r + row * ld_r, d, t, G);
#pragma unroll
        for (int i = 0; i < VALS; i += 2) v.put(i, v.at(i) + u.at(i), v.at(i + 1) + u.at(i + 1));
    }
    weight.load(w, d, t, G);
    if (h) v.store(h + row * ld_h, d, t, G);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < VALS; ++i) sum = fmaf(v.at(i), v.at(i), sum);
    sum = group_sum<WARP>(sum, parts);
    const float by = 1.f / sqrtf(sum / (float)d + eps);
    if (rstd && t == 0) rstd[row] = by;
#pragma unroll
    for (int i = 0; i < VALS; i += 2) u.put(i, v.at(i) * by * weight.at(i), v.at(i + 1) * by * weight.at(i + 1));
    u.store(y + row * ld_y, d, t, G);
}

// A thread's own columns of up to three rows on their way to its own places in shared memory (nobody else's, so no barrier).
template <typename T, int VALS, bool ALIGNED>
struct Ahead {
    static constexpr bool kOn = VALS * sizeof(T) <= 32 && (ALIGNED || sizeof(T) == 4);  // copies of 16 or 4 bytes
    static constexpr int kVec = ALIGNED ? Vec<T>::n : 1, kParts = VALS / kVec, kBytes = kVec * (int)sizeof(T);
    static constexpr int kThreadBytes = kOn ? 2 * 3 * kParts * kBytes : 0;
    char* at;  // the thread's first place
    int stride;
    __device__ __forceinline__ char* place(int stage, int row, int i) const { return at + ((stage * 3 + row) * kParts + i) * stride; }
    __device__ __forceinline__ void fetch(int stage, int row, const T* p, int d, int t, int G) const {
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            const int c = (t + i * G) * kVec;
            const uint32_t to = (uint32_t)__cvta_generic_to_shared(place(stage, row, i));
            if (c < d) {
                if constexpr (ALIGNED) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(p + c) : "memory");
                else asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(to), "l"(p + c) : "memory");
            }
        }
    }
    __device__ __forceinline__ void read(int stage, int row, int d, int t, int G, Row<T, VALS, ALIGNED>& v) const {
#pragma unroll
        for (int i = 0; i < kParts; ++i) {
            const int c = (t + i * G) * kVec;
            if constexpr (ALIGNED) v.put_vector(i, c < d ? *(const uint4*)place(stage, row, i) : make_uint4(0, 0, 0, 0));
            else v.put_bits(i, c < d ? *(const uint32_t*)place(stage, row, i) : 0);
        }
    }
};

// Group g of `groups` takes rows g, g + groups, ... and keeps its share of dw in registers; a CTA's share goes to
// part[CTA][d], the warps of a CTA joined in order. The next row is on its way to shared memory while a row is summed (in
// registers it left room for two thirds of the warps: 8192 x 4096 bf16 78 us, without 66, 56 this way).
template <typename T, int VALS, bool ALIGNED, bool WARP>
__global__ __launch_bounds__(WARP ? kWarpCta : 1024) void norm_grad_kernel(
    const T* h, int64_t ld_h, const float* rstd, const T* w, const T* dy, int64_t ld_dy, const T* dres, int64_t ld_r, int64_t M, int d,
    T* dx, int64_t ld_dx, float* part) {
    using R = Row<T, VALS, ALIGNED>;
    using A = Ahead<T, VALS, ALIGNED>;
    extern __shared__ __align__(16) char shared[];  // the rows on their way; at the end, WARP: 4 rows of VALS * 32 sums
    __shared__ float parts[2][32];
    constexpr int kRows = WARP ? kWarpCta / 32 : 1;
    const int G = WARP ? 32 : blockDim.x, t = WARP ? threadIdx.x % 32 : threadIdx.x;
    const int64_t groups = (int64_t)gridDim.x * kRows;
    const A ahead = {shared + threadIdx.x * A::kBytes, (int)blockDim.x * A::kBytes};
    float dw[VALS];
#pragma unroll
    for (int i = 0; i < VALS; ++i) dw[i] = 0.f;
    int64_t row = (int64_t)blockIdx.x * kRows + (WARP ? threadIdx.x / 32 : 0);
    auto fetch = [&](int stage, int64_t r) {
        if constexpr (A::kOn) {
            if (r < M) {
                ahead.fetch(stage, 0, h + r * ld_h, d, t, G);
                ahead.fetch(stage, 1, dy + r * ld_dy, d, t, G);
                if (dres) ahead.fetch(stage, 2, dres + r * ld_r, d, t, G);
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
        }
    };
    fetch(0, row);
    float by = row < M ? rstd[row] : 0.f;
    for (int turn = 0; row < M; row += groups, turn ^= 1) {
        R v, u, q, weight;
        weight.load(w, d, t, G);  // from the cache again: no registers for it between rows
        fetch(turn ^ 1, row + groups);
        const float by_then = row + groups < M ? rstd[row + groups] : 0.f;
        if constexpr (A::kOn) {
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            ahead.read(turn, 0, d, t, G, v);
            ahead.read(turn, 1, d, t, G, u);
            if (dres) ahead.read(turn, 2, d, t, G, q);
        } else {
            v.load(h + row * ld_h, d, t, G);
            u.load(dy + row * ld_dy, d, t, G);
            if (dres) q.load(dres + row * ld_r, d, t, G);
        }
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < VALS; ++i) {
            const float n = v.at(i) * by, g = u.at(i);
            dw[i] = fmaf(g, n, dw[i]);
            sum = fmaf(g * weight.at(i), n, sum);
        }
        if (dx) {
            sum = group_sum<WARP>(sum, parts[turn]) / (float)d;
#pragma unroll
            for (int i = 0; i < VALS; i += 2) {
                float o[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    o[e] = by * fmaf(-v.at(i + e) * by, sum, u.at(i + e) * weight.at(i + e));
                    if (dres) o[e] += q.at(i + e);
                }
                v.put(i, o[0], o[1]);
            }
            v.store(dx + row * ld_dx, d, t, G);
        }
        by = by_then;
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();
    if (!part) return;
    float* out = part + (int64_t)blockIdx.x * d;
    if constexpr (WARP) {
        float* joined = (float*)shared;
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

// dw[c] = beta dw[c] + sum of the CTAs' shares: 32 threads a column at different shares, eight on their way at a time, joined in
// order.
template <typename G>
__global__ __launch_bounds__(1024) void norm_dw_kernel(const float* part, int rows, int d, float beta, G* dw) {
    chain_wait();
    __shared__ float sums[32][33];
    const int lane = threadIdx.x % 32, c = blockIdx.x * 32 + lane, k = threadIdx.x / 32;
    float s = 0.f;
    if (c < d) {
        int i = k;
        for (; i + 7 * 32 < rows; i += 8 * 32) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = part[(int64_t)(i + 32 * e) * d + c];
            s += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
        }
        for (; i < rows; i += 32) s += part[(int64_t)i * d + c];
    }
    sums[k][lane] = s;
    __syncthreads();
    s = sums[lane][k];  // column k of the CTA's 32, the lane's share
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    const int mine = blockIdx.x * 32 + k;
    if (lane == 0 && mine < d) {
        if (beta != 0.f) s = fmaf(beta, wide(dw[mine]), s);
        narrow(s, &dw[mine]);
    }
}

struct Plan {
    int vals, threads;
    bool warp;
};
// 32 bytes of a row a thread (the gradient's kernel then fits 64 registers, four CTAs of 256 threads an SM), up to 128 where a
// warp or a CTA of 1024 threads would not reach.
Plan plan_of(int d, int el) {
    const int vals = 32 / el;
    if (d <= 1024) return {d <= 32 * vals ? vals : d <= 512 ? 16 : 32, kWarpCta, true};
    if (d <= 1024 * vals) return {vals, ((d + vals - 1) / vals + 31) / 32 * 32, false};
    return {32, ((d + 31) / 32 + 31) / 32 * 32, false};
}
// CTAs of the gradient's kernel: what fits the SMs, four rows a group at least (their shares of dw are written and read again: 1999 x
// 1363 fp32 in 1520 CTAs 17 + 18 us; in 500, with rows fetched ahead, 16 for both kernels), but one CTA per SM.
int64_t grad_ctas(int64_t M, int d, int el) {
    const Plan p = plan_of(d, el);
    const int64_t rows = p.warp ? kWarpCta / 32 : 1, each = p.warp ? 6 : std::max(1, 1024 / p.threads);
    const int64_t most = (M + rows - 1) / rows, least = std::min<int64_t>(most, train_sms());
    return std::min(std::max(least, most / 4), (int64_t)train_sms() * each);
}

bool vectors(const void* p, int64_t ld, size_t el) { return !p || (((uintptr_t)p | (uintptr_t)(ld * (int64_t)el)) & 15) == 0; }

// f.template operator()<VALS, ALIGNED, WARP>() for a plan.
template <typename F>
cudaError_t with_plan(const Plan& p, bool aligned, F&& f) {
    auto go = [&](auto vals, auto warp) {
        return aligned ? f(vals, std::true_type(), warp) : f(vals, std::false_type(), warp);
    };
    using V8 = std::integral_constant<int, 8>;
    using V16 = std::integral_constant<int, 16>;
    using V32 = std::integral_constant<int, 32>;
    if (p.warp) return p.vals == 8 ? go(V8(), std::true_type()) : p.vals == 16 ? go(V16(), std::true_type()) : go(V32(), std::true_type());
    return p.vals == 8 ? go(V8(), std::false_type()) : p.vals == 16 ? go(V16(), std::false_type()) : go(V32(), std::false_type());
}

template <typename T>
cudaError_t forward(const void* x, int64_t ld_x, const void* r, int64_t ld_r, int64_t M, int d, const void* w, float eps, void* h,
                    int64_t ld_h, void* y, int64_t ld_y, float* rstd, cudaStream_t s) {
    constexpr size_t el = sizeof(T);
    const bool aligned = d % Vec<T>::n == 0 && vectors(x, ld_x, el) && vectors(r, ld_r, el) && vectors(w, 0, el) &&
                         vectors(h, ld_h, el) && vectors(y, ld_y, el);
    const Plan p = plan_of(d, el);
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
    const Plan p = plan_of(d, el);
    const int64_t ctas = grad_ctas(M, d, el);
    note_launches(1);
    cudaError_t e = with_plan(p, aligned, [&](auto vals, auto al, auto warp) {
        constexpr size_t ahead = (size_t)Ahead<T, vals.value, al.value>::kThreadBytes;
        const size_t smem = std::max((size_t)p.threads * ahead, warp.value ? (size_t)kWarpCta * vals.value * 4 : 0);
        constexpr size_t most = std::max<size_t>((warp.value ? kWarpCta : 1024) * ahead, 48 << 10);
        if (cudaError_t e = smem_attr_once<norm_grad_kernel<T, vals.value, al.value, warp.value>>((int)most))
            return e;
        norm_grad_kernel<T, vals.value, al.value, warp.value><<<(unsigned)ctas, p.threads, smem, s>>>(
            (const T*)h, ld_h, rstd, (const T*)w, (const T*)dy, ld_dy, (const T*)dres, ld_r, M, d, (T*)dx, ld_dx,
            dw ? part : nullptr);
        return cudaGetLastError();
    });
    if (e || !dw) return e;
    const dim3 grid((unsigned)((d + 31) / 32));
    return gt == TDA_BF16 ? launch_chained(true, norm_dw_kernel<__nv_bfloat16>, grid, dim3(1024), 0, s, (const float*)part, (int)ctas, d,
                                           beta, (__nv_bfloat16*)dw)
                          : launch_chained(true, norm_dw_kernel<float>, grid, dim3(1024), 0, s, (const float*)part, (int)ctas, d, beta,
                                           (float*)dw);
}

}  // namespace

// Enough for either type.
size_t norm_ws_bytes(int64_t M, int64_t d) {
    return M == 0 ? 0 : (size_t)std::max(grad_ctas(M, (int)d, 2), grad_ctas(M, (int)d, 4)) * d * 4;
}

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
