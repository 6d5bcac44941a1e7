// k_linear_rows.cu -- the linear layer for a few rows (a decoded token, a handful of
// them), where the time is that of reading W once: plain dot products on the CUDA
// cores with wide loads, no tile to fill.
//
// rows_kernel: Z[m][n] = sum_k X[m][k] W[n][k]. A warp takes kRows rows of W, its lanes
// run along k in 16-byte vectors; where d_out is short the warps of a CTA share the rows
// and split k, and their sums are added in order. X is read through L1, kRows times less
// often than W. One token through 4096 -> 14336 (117 MB): see the figures at the rule below.
//
// cols_kernel: dX[m][k] = sum_n B[m][n] W[n][k], fp32. A lane holds four columns k, the
// warps of a cluster of CTAs split the rows n, and the sums are added in warp and CTA order
// through (distributed) shared memory.
//
// outer_kernel: dW[n][k] = sum_m B[m][n] X[m][k] for at most 16 rows m, bound by writing dW.
//
// Sums are fp32 (a lane adds a 32nd of the products or fewer, then the lanes' sums pairwise).
#include <type_traits>

#include "linear.cuh"

namespace tda {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
// rows_kernel: CTAs of four warps, four rows of W a warp. Of eight warps: one token through 4096 -> 14336 21.2 us
// against 20.4, 2048 -> 2048 3.6 against 3.2, eight fp32 tokens through 4096 -> 4096 19.4 against 18.6; of sixteen 27 us.
constexpr int kRowThreads = 128, kRowWarps = kRowThreads / 32, kRows = 4;

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void set_f(float* p, float x) { *p = x; }
__device__ __forceinline__ void set_f(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// N consecutive values as fp32: one 16-byte access, or one value.
template <typename T, int N>
struct Piece {
    uint4 q;
    __device__ __forceinline__ void load(const T* p) { q = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void load_once(const T* p) {  // past L1, which keeps X
        asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(q.x), "=r"(q.y), "=r"(q.z), "=r"(q.w)
                     : "l"(p));
    }
    __device__ __forceinline__ float get(int i) const {
        const int w = sizeof(T) == 4 ? i : i >> 1;
        const uint32_t b = w == 0 ? q.x : w == 1 ? q.y : w == 2 ? q.z : q.w;
        return __uint_as_float(sizeof(T) == 4 ? b : i & 1 ? b & 0xFFFF0000u : b << 16);
    }
};
template <typename T>
struct Piece<T, 1> {
    T q;
    __device__ __forceinline__ void load(const T* p) { q = *p; }
    __device__ __forceinline__ void load_once(const T* p) { q = *p; }
    __device__ __forceinline__ float get(int) const { return to_f(q); }
};

struct RowsParams {
    const void *X, *W;
    int64_t ld_x, ld_w, K;
    LinearEpilogue ep;  // M, N and everything after the sum
    int wk;             // warps that share rows of W and split k: 1, 2 or 4
};

template <typename T>
__device__ __forceinline__ void finish1(const LinearEpilogue& e, int64_t m, int64_t n, float z) {
    constexpr bool FAST = sizeof(T) == 2;
    if (e.bias) z += to_f(((const T*)e.bias)[n]);
    if (e.Z) set_f((T*)e.Z + m * e.ld_z + n, z);
    switch (e.act) {
        case TDA_ACT_RELU: z = act_value<TDA_ACT_RELU, FAST>(z); break;
        case TDA_ACT_GELU: z = act_value<TDA_ACT_GELU, FAST>(z); break;
        case TDA_ACT_GELU_TANH: z = act_value<TDA_ACT_GELU_TANH, FAST>(z); break;
        case TDA_ACT_SILU: z = act_value<TDA_ACT_SILU, FAST>(z); break;
        default: break;
    }
    if (e.R) z = fmaf(e.r_scale, to_f(((const T*)e.R)[m * e.ld_r + n]), z);
    set_f((T*)e.Y + m * e.ld_y + n, z);
}

// MT rows of X; N: values per access.
template <typename T, int MT, int N>
__global__ void __launch_bounds__(kRowThreads) rows_kernel(const __grid_constant__ RowsParams p) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, wk = p.wk, part = warp % wk;
    const int64_t n0 = ((int64_t)blockIdx.x * (kRowWarps / wk) + warp / wk) * kRows;
    const int64_t m0 = (int64_t)blockIdx.y * MT;
    float acc[kRows][MT] = {};
    const T *W[kRows], *X[MT];
#pragma unroll
    for (int r = 0; r < kRows; ++r) W[r] = (const T*)p.W + (n0 + r < p.ep.N ? n0 + r : p.ep.N - 1) * p.ld_w;
#pragma unroll
    for (int m = 0; m < MT; ++m) X[m] = (const T*)p.X + (m0 + m < p.ep.M ? m0 + m : p.ep.M - 1) * p.ld_x;
    const int64_t step = (int64_t)wk * 32 * N;
    int64_t k = ((int64_t)part * 32 + lane) * N;
    auto run = [&](auto ahead) {  // U accesses ahead per row of W
        constexpr int U = decltype(ahead)::value;
        for (; k + (U - 1) * step + N <= p.K; k += U * step) {
            Piece<T, N> w[U][kRows], x[U][MT];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int r = 0; r < kRows; ++r) w[u][r].load_once(W[r] + k + u * step);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int m = 0; m < MT; ++m) x[u][m].load(X[m] + k + u * step);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int i = 0; i < N; ++i)
#pragma unroll
                    for (int m = 0; m < MT; ++m) {
                        const float a = x[u][m].get(i);
#pragma unroll
                        for (int r = 0; r < kRows; ++r) acc[r][m] = fmaf(w[u][r].get(i), a, acc[r][m]);
                    }
        }
    };
    if (MT <= 2) run(std::integral_constant<int, 2>());
    run(std::integral_constant<int, 1>());
    for (; k < p.K; k += step)  // what is left of the row, a value at a time
        for (int i = 0; i < N && k + i < p.K; ++i)
#pragma unroll
            for (int m = 0; m < MT; ++m) {
                const float a = to_f(X[m][k + i]);
#pragma unroll
                for (int r = 0; r < kRows; ++r) acc[r][m] = fmaf(to_f(W[r][k + i]), a, acc[r][m]);
            }
    // lanes' sums; lane r * MT + m keeps sum (r, m)
    float mine = 0.f;
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            float v = acc[r][m];
#pragma unroll
            for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
            if (lane == r * MT + m) mine = v;
        }
    if (wk > 1) {
        __shared__ float sh[kRowWarps][32];
        sh[warp][lane] = mine;
        __syncthreads();
        if (part) return;
        for (int w = 1; w < wk; ++w) mine += sh[warp + w][lane];
    }
    const int64_t n = n0 + lane / MT, m = m0 + lane % MT;
    if (lane < kRows * MT && n < p.ep.N && m < p.ep.M) finish1<T>(p.ep, m, n, mine);
}

template <typename T, int MT>
void run_rows(const RowsParams& p, bool vec, cudaStream_t s) {
    const int64_t per = (int64_t)(kRowWarps / p.wk) * kRows;
    const dim3 grid((unsigned)((p.ep.N + per - 1) / per), (unsigned)((p.ep.M + MT - 1) / MT));
    if (vec)
        rows_kernel<T, MT, 16 / (int)sizeof(T)><<<grid, kRowThreads, 0, s>>>(p);
    else
        rows_kernel<T, MT, 1><<<grid, kRowThreads, 0, s>>>(p);
}

template <typename T>
cudaError_t rows(RowsParams p, cudaStream_t s) {
    const bool vec = (((uintptr_t)p.X | (uintptr_t)p.W | (uintptr_t)(p.ld_x * (int64_t)sizeof(T)) |
                       (uintptr_t)(p.ld_w * (int64_t)sizeof(T))) & 15) == 0;
    // about 16 warps per SM
    p.wk = 1;
    while (p.wk < kRowWarps && (p.ep.N + kRows - 1) / kRows * p.wk < train_sms() * 16) p.wk *= 2;
    note_launches(1);
    if (p.ep.M == 1)
        run_rows<T, 1>(p, vec, s);
    else if (p.ep.M == 2)
        run_rows<T, 2>(p, vec, s);
    else if (p.ep.M <= 4)
        run_rows<T, 4>(p, vec, s);
    else if constexpr (sizeof(T) == 4)
        run_rows<T, 8>(p, vec, s);
    return cudaGetLastError();
}

// ------------------------------------------------------------------ dX of a few fp32 rows
constexpr int kColsCluster = 8;

struct ColsParams {
    const float *B, *W;
    float* dX;
    int64_t ld_b, ld_w, ld_dx, M, N, K;
};

__device__ __forceinline__ uint32_t cluster_rank_of() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float remote_f(const float* p, uint32_t rank) {
    uint32_t a, b = (uint32_t)__cvta_generic_to_shared(p);
    float v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(b), "r"(rank));
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}

// Cluster (x): columns [128 x, 128 x + 128), CTA rank and warp: an even share of W's rows. C: columns a lane.
template <int MT, bool VEC>
__global__ void __launch_bounds__(kThreads) cols_kernel(const __grid_constant__ ColsParams p) {
    chain_wait();
    chain_next();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t rank = cluster_rank_of();
    const int64_t col = (int64_t)(blockIdx.x / kColsCluster) * 128 + (VEC ? lane * 4 : lane);
    const int64_t m0 = (int64_t)blockIdx.y * MT;
    constexpr int kShares = kColsCluster * kWarps;
    const int share = (int)rank * kWarps + warp;
    const int64_t n0 = p.N * share / kShares, n1 = p.N * (share + 1) / kShares;
    float acc[MT][4] = {};
    const float* B[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) B[m] = p.B + (m0 + m < p.M ? m0 + m : p.M - 1) * p.ld_b;
    constexpr int U = MT == 1 ? 8 : 4;
    for (int64_t n = n0; n < n1; n += U) {
        float w[U][4], b[U][MT];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool in = n + u < n1;
            const float* src = p.W + (n + u) * p.ld_w + col;
            if (VEC) {
                float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
                if (in && col < p.K) x = __ldg(reinterpret_cast<const float4*>(src));
                w[u][0] = x.x, w[u][1] = x.y, w[u][2] = x.z, w[u][3] = x.w;
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i) w[u][i] = in && col + 32 * i < p.K ? src[32 * i] : 0.f;
            }
#pragma unroll
            for (int m = 0; m < MT; ++m) b[u][m] = in ? B[m][n + u] : 0.f;
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) acc[m][i] = fmaf(w[u][i], b[u][m], acc[m][i]);
    }
    __shared__ float sh[kWarps][MT][128], sum[MT][128];
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) sh[warp][m][VEC ? lane * 4 + i : lane + 32 * i] = acc[m][i];
    __syncthreads();
    for (int i = threadIdx.x; i < MT * 128; i += kThreads) {
        float v = (&sh[0][0][0])[i];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) v += (&sh[w][0][0])[i];
        (&sum[0][0])[i] = v;
    }
    __syncwarp();  // the barrier's aligned form is one instruction of the whole warp
    cluster_barrier();
    // each CTA adds a share of the columns over the cluster, in rank order
    constexpr int kOut = MT * 128 / kColsCluster;
    for (int j = threadIdx.x; j < kOut; j += kThreads) {
        const int i = (int)rank * kOut + j;
        float v = 0.f;
#pragma unroll
        for (int r = 0; r < kColsCluster; ++r) v += remote_f(&sum[0][0] + i, r);
        const int64_t m = m0 + i / 128, k = (int64_t)(blockIdx.x / kColsCluster) * 128 + i % 128;
        if (m < p.M && k < p.K) p.dX[m * p.ld_dx + k] = v;
    }
    __syncwarp();
    cluster_barrier();  // no CTA leaves while its sums are still read
}

// ------------------------------------------------------------------ dW of a few rows
// dW[n][k] = beta dW[n][k] + sum_m B[m][n] X[m][k], M <= 16: bound by writing dW. A thread holds X's values of
// four columns k for all rows m and walks down kOuterRows rows n, whose B values every lane reads alike.
constexpr int kOuterRows = 32;

struct OuterParams {
    const void *B, *X;
    void* dW;
    int64_t ld_b, ld_x, ld_dw, M, N, K;
    float beta;
    int vec;  // X and dW may be moved four values at a time
};

template <typename T>
__device__ __forceinline__ void read4(const T* p, bool vec, int have, float* v) {
    if (vec) {
        if constexpr (sizeof(T) == 4) {
            const float4 x = *reinterpret_cast<const float4*>(p);
            v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
        } else {
            const uint2 x = *reinterpret_cast<const uint2*>(p);
            v[0] = __uint_as_float(x.x << 16), v[1] = __uint_as_float(x.x & 0xFFFF0000u);
            v[2] = __uint_as_float(x.y << 16), v[3] = __uint_as_float(x.y & 0xFFFF0000u);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = i < have ? to_f(p[i]) : 0.f;
    }
}
template <typename T>
__device__ __forceinline__ void write4(T* p, bool vec, int have, const float* v) {
    if (vec) {
        if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
            const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
            *reinterpret_cast<uint2*>(p) =
                make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < have) set_f(p + i, v[i]);
    }
}

template <typename T, typename TG, int MT>
__global__ void __launch_bounds__(kThreads) outer_kernel(const __grid_constant__ OuterParams p) {
    chain_wait();
    chain_next();
    const int64_t n0 = (int64_t)blockIdx.y * kOuterRows, k = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 4;
    __shared__ alignas(16) float b[kOuterRows][MT];
    for (int i = threadIdx.x; i < kOuterRows * MT; i += kThreads) {
        const int64_t n = n0 + i % kOuterRows, m = i / kOuterRows;
        b[i % kOuterRows][m] = n < p.N && m < p.M ? to_f(((const T*)p.B)[m * p.ld_b + n]) : 0.f;
    }
    __syncthreads();
    if (k >= p.K) return;
    const int have = p.K - k < 4 ? (int)(p.K - k) : 4;
    const bool vec = p.vec && have == 4;
    float x[MT][4];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        x[m][0] = x[m][1] = x[m][2] = x[m][3] = 0.f;
        if (m < p.M) read4((const T*)p.X + m * p.ld_x + k, vec, have, x[m]);
    }
    const int rows = p.N - n0 < kOuterRows ? (int)(p.N - n0) : kOuterRows;
#pragma unroll 4
    for (int r = 0; r < rows; ++r) {
        TG* out = (TG*)p.dW + (n0 + r) * p.ld_dw + k;
        float a[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = fmaf(b[r][m], x[m][i], a[i]);
        if (p.beta != 0.f) {
            float old[4];
            read4(out, vec, have, old);
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = fmaf(p.beta, old[i], a[i]);
        }
        write4(out, vec, have, a);
    }
}

}  // namespace

// Few rows, by type. Measured against the tensor-core path (us, device): bf16 4096 -> 14336, 1 row 21 / 25, 4 rows
// 23 / 27, 8 rows 25 there; fp32 4096 -> 4096 (which there needs W's planes written and read again), 1 row 13 / 49,
// 16 rows 33 / 49; with dW in the backward pass 1 row 59 / 87, 16 rows 77 / 87.
bool linear_rows_preferred(int64_t M, tda_dtype dt) { return M <= (dt == TDA_BF16 ? 4 : 16); }

cudaError_t launch_linear_rows(const void* X, int64_t ld_x, const void* W, int64_t ld_w, int64_t K,
                               const LinearEpilogue& ep, tda_dtype dt, cudaStream_t s) {
    RowsParams p;
    p.X = X, p.W = W, p.ld_x = ld_x, p.ld_w = ld_w, p.K = K, p.ep = ep, p.wk = 1;
    return dt == TDA_BF16 ? rows<__nv_bfloat16>(p, s) : rows<float>(p, s);
}

cudaError_t launch_linear_cols(const float* B, int64_t ld_b, const float* W, int64_t ld_w, float* dX, int64_t ld_dx,
                               int64_t M, int64_t N, int64_t K, bool chained, cudaStream_t s) {
    ColsParams p = {B, W, dX, ld_b, ld_w, ld_dx, M, N, K};
    const bool vec = (((uintptr_t)W | (uintptr_t)(ld_w * 4)) & 15) == 0 && K % 4 == 0;
    const int mt = M == 1 ? 1 : M <= 4 ? 4 : 8;
    const int64_t blocks = (K + 127) / 128;
    if (blocks > ((int64_t)1 << 31) / kColsCluster - 1) return cudaErrorInvalidConfiguration;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(blocks * kColsCluster), (unsigned)((M + mt - 1) / mt));
    cfg.blockDim = dim3(kThreads);
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = kColsCluster;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = chained ? 2 : 1;
    note_launches(1);
    const auto kernel = mt == 1   ? (vec ? cols_kernel<1, true> : cols_kernel<1, false>)
                        : mt == 4 ? (vec ? cols_kernel<4, true> : cols_kernel<4, false>)
                                  : (vec ? cols_kernel<8, true> : cols_kernel<8, false>);
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

cudaError_t launch_linear_outer(const void* B, int64_t ld_b, const void* X, int64_t ld_x, int64_t M, int64_t N, int64_t K,
                                tda_dtype dt, void* dW, int64_t ld_dw, tda_dtype gt, float beta, bool chained,
                                cudaStream_t s) {
    OuterParams p = {B, X, dW, ld_b, ld_x, ld_dw, M, N, K, beta, 0};
    const int64_t ex = dt == TDA_BF16 ? 2 : 4, eg = gt == TDA_BF16 ? 2 : 4;
    p.vec = (((uintptr_t)X | (uintptr_t)(ld_x * ex)) & (4 * ex - 1)) == 0 &&
            (((uintptr_t)dW | (uintptr_t)(ld_dw * eg)) & (4 * eg - 1)) == 0;
    const dim3 block(kThreads);
    const int64_t strips = (N + kOuterRows - 1) / kOuterRows;
    for (int64_t y0 = 0; y0 < strips; y0 += 65535, chained = true) {  // a launch has at most 65535 strips
        const int64_t y = strips - y0 < 65535 ? strips - y0 : 65535;
        const dim3 grid((unsigned)((K + 4 * kThreads - 1) / (4 * kThreads)), (unsigned)y);
        p.N = N - y0 * kOuterRows;
        p.B = (const char*)B + y0 * kOuterRows * ex;
        p.dW = (char*)dW + y0 * kOuterRows * ld_dw * eg;
#define TDA_OUTER(T, TG)                                                                                    \
    (M <= 4 ? launch_chained(chained, outer_kernel<T, TG, 4>, grid, block, 0, s, p)                         \
            : launch_chained(chained, outer_kernel<T, TG, 16>, grid, block, 0, s, p))
        const cudaError_t e = dt == TDA_F32    ? TDA_OUTER(float, float)
                              : gt == TDA_BF16 ? TDA_OUTER(__nv_bfloat16, __nv_bfloat16)
                                               : TDA_OUTER(__nv_bfloat16, float);
#undef TDA_OUTER
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace tda
