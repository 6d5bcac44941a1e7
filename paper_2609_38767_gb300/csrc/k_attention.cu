// k_attention.cu -- masked attention on the CUDA cores (fp32, and bf16 rows that TMA cannot take), the visible ranges of
// packed documents, and the small kernels around the attention's backward pass.
//
//   x = scale q.k,  c = cap tanh(x / cap),  s = c + bias(i - j),  P = exp(s - lse),  O = P V
//   dP = dO V^T,  dS = P (dP - dO.O),  dX = scale dS (1 - (c / cap)^2),  dQ = dX K,  dK = dX^T Q,  dV = P^T dO
//
// One CTA has a tile of 64 queries (forward, dQ) or 64 keys (dK, dV) in shared memory as fp32 and goes over the tiles
// of the other side that its rows reach; scores never leave the SM. dQ and dK, dV are two kernels that each compute the
// scores again, so that no sum depends on the order of atomics.
#include <math_constants.h>

#include <algorithm>
#include <type_traits>

#include "attention.cuh"

namespace tda {
namespace {

constexpr int kTile = 64, kThreads = 256;

__device__ __forceinline__ float wide(float x) { return x; }
__device__ __forceinline__ float wide(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T narrow(float x);
template <>
__device__ __forceinline__ float narrow<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 narrow<__nv_bfloat16>(float x) { return __float2bfloat16(x); }

// Sum and maximum over the 16 threads that share a row of scores.
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = 8; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}
__device__ __forceinline__ float row_max(float v) {
#pragma unroll
    for (int o = 8; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

// Rows [first, first + 64) of one head into shared memory as fp32, zeros past the example, past hd, and for rows
// that `live` leaves out (a token that nothing sees may hold anything, and zero times NaN is NaN). vec: fp32 rows on 16 bytes.
template <typename T, int HD>
__device__ __forceinline__ void load_tile(float* dst, const void* src, int64_t ld, int64_t row0, int first, int rows, int col,
                                          int hd, const uint8_t* live, bool vec) {
    const T* p = (const T*)src + (row0 + first) * ld + col;
    if (sizeof(T) == 4 && vec) {
        constexpr int kQuads = HD / 4, kTimes = kTile * kQuads / kThreads;
        float4 v[kTimes];
#pragma unroll
        for (int k = 0; k < kTimes; ++k) {
            const int i = threadIdx.x + k * kThreads, r = i / kQuads, c = i % kQuads * 4;
            v[k] = first + r < rows && c < hd && (!live || live[r]) ? *(const float4*)((const float*)p + r * ld + c)
                                                                    : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int k = 0; k < kTimes; ++k) {
            const int i = threadIdx.x + k * kThreads, r = i / kQuads, c = i % kQuads * 4;
            *(float4*)&dst[r * (HD + 4) + c] = v[k];
        }
        return;
    }
#pragma unroll 4
    for (int i = threadIdx.x; i < kTile * HD; i += kThreads) {
        const int r = i / HD, c = i % HD;
        dst[r * (HD + 4) + c] = first + r < rows && c < hd && (!live || live[r]) ? wide(p[r * ld + c]) : 0.f;
    }
}
// Whether an fp32 tensor's rows and heads start on 16 bytes.
template <typename T>
__device__ __forceinline__ bool vectors(const void* p, int64_t ld, int hd) {
    return sizeof(T) == 4 && (((uint64_t)p | (uint64_t)(ld * 4)) & 15) == 0 && hd % 4 == 0;
}

// a b + c of two fp32 pairs in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(*(uint64_t*)&d)
        : "l"(*(uint64_t*)&a), "l"(*(uint64_t*)&b), "l"(*(uint64_t*)&c));
    return d;
}

// s[r][c] = a_row . b_row for rows ty + 16 r of A, r < R, and tx + 16 c of B: even and odd terms beside one another.
template <int HD, int R>
__device__ __forceinline__ void dots(const float* A, const float* B, float (&s)[4][4]) {
    const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
    float2 sum[R][4];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) sum[r][c] = make_float2(0.f, 0.f);
#pragma unroll 4
    for (int d = 0; d < HD; d += 4) {
        float4 a[R], b[4];
#pragma unroll
        for (int r = 0; r < R; ++r) a[r] = *(const float4*)&A[(ty + 16 * r) * (HD + 4) + d];
#pragma unroll
        for (int c = 0; c < 4; ++c) b[c] = *(const float4*)&B[(tx + 16 * c) * (HD + 4) + d];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                sum[r][c] = fma2(make_float2(a[r].x, a[r].y), make_float2(b[c].x, b[c].y), sum[r][c]);
                sum[r][c] = fma2(make_float2(a[r].z, a[r].w), make_float2(b[c].z, b[c].w), sum[r][c]);
            }
    }
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int c = 0; c < 4; ++c) s[r][c] = sum[r][c].x + sum[r][c].y;
}

// acc[r][c] += sum over k < n of W[ty + 16 r][k] V[k][c'], c' = 4 tx + 64 (c / 4) + c % 4, r < R: 64 rows of W with stride 68.
template <int HD, int R>
__device__ __forceinline__ void weigh(const float* W, const float* V, float (&acc)[4][HD / 16], int n) {
    const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
#pragma unroll 2
    for (int k = 0; k < n; k += 4) {
        float4 w[R];
#pragma unroll
        for (int r = 0; r < R; ++r) w[r] = *(const float4*)&W[(ty + 16 * r) * (kTile + 4) + k];
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int b = 0; b < HD / 64; ++b) {
                const float4 v = *(const float4*)&V[(k + j) * (HD + 4) + 4 * tx + 64 * b];
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float x = j == 0 ? w[r].x : j == 1 ? w[r].y : j == 2 ? w[r].z : w[r].w;
                    acc[r][4 * b + 0] = fmaf(x, v.x, acc[r][4 * b + 0]);
                    acc[r][4 * b + 1] = fmaf(x, v.y, acc[r][4 * b + 1]);
                    acc[r][4 * b + 2] = fmaf(x, v.z, acc[r][4 * b + 2]);
                    acc[r][4 * b + 3] = fmaf(x, v.w, acc[r][4 * b + 3]);
                }
            }
    }
}
// f with the number of 16-row groups that a tile with `rows` rows left has, 1, 2 or 4: the last tile of an example is not paid for in
// full (with fma2 in dots, 4 x 515 tokens of 8 heads 69 -> 59 us, the backward pass of 2 x 515 140 -> 133).
template <typename F>
__device__ __forceinline__ void by_rows(int rows, F&& f) {
    if (rows <= 16) f(std::integral_constant<int, 1>());
    else if (rows <= 32) f(std::integral_constant<int, 2>());
    else f(std::integral_constant<int, 4>());
}

template <typename T, int HD>
__device__ __forceinline__ void store_tile(void* dst, int64_t ld, int64_t row0, int first, int rows, int col, int hd,
                                           const float (&acc)[4][HD / 16], const float (&by)[4]) {
    const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int row = first + ty + 16 * r;
        if (row >= rows) continue;
        T* p = (T*)dst + (row0 + row) * ld + col;
#pragma unroll
        for (int c = 0; c < HD / 16; ++c) {
            const int d = 4 * tx + 64 * (c / 4) + c % 4;
            if (d < hd) p[d] = narrow<T>(acc[r][c] * by[r]);
        }
    }
}

// The score of a pair from its dot product; *bend: its slope by x.
__device__ __forceinline__ float score(float dot, float scale, float cap, float bias, float* bend) {
    float x = dot * scale;
    *bend = 1.f;
    if (cap > 0.f) {
        const float t = tanhf(x / cap);
        x = cap * t;
        *bend = fmaf(-t, t, 1.f);
    }
    return x + bias;
}

// biases[64 + d]: what the distances q0 - k0 + d, -64 < d < 64, of a pair of tiles add to the scores.
template <typename T>
__device__ __forceinline__ void load_biases(const Attention& a, float* biases, int h, int64_t apart) {
    const int t = threadIdx.x;
    if (t < 2 * kTile)
        biases[t] = a.n_buckets || a.slope ? distance_bias(a.bucket, (const T*)a.table, a.slope, a.n_buckets, a.reach, a.H, h,
                                                           apart + t - kTile)
                                           : 0.f;
}

template <int HD>
constexpr size_t smem_of(int tiles, int squares) {
    return (size_t)(tiles * kTile * (HD + 4) + squares * kTile * (kTile + 4)) * 4 + 4096;
}

struct Small {  // the last 4 KiB of a CTA's shared memory
    float biases[2 * kTile];
    int2 see[kTile];
    float lse[kTile], delta[kTile];
    float diag[2 * kTile];
    int ids[2 * kTile];
    uint8_t live[kTile];
    int lo, hi;
};
static_assert(sizeof(Small) <= 4096, "");

// The queries of a tile: what they see, and the hull of it in lo, hi.
__device__ __forceinline__ void load_rows(const Attention& a, Small& m, int64_t row0, int q0) {
    const int t = threadIdx.x;
    if (t == 0) m.lo = INT32_MAX, m.hi = 0;
    __syncthreads();
    if (t < kTile) {
        const int2 v = visible(a.range, a.causal, (int)a.T, row0, q0 + t);
        m.see[t] = v;
        if (v.x < v.y) atomicMin(&m.lo, v.x), atomicMax(&m.hi, v.y);
    }
    __syncthreads();
}

// live[j]: some query of the tile sees key k0 + j.
__device__ __forceinline__ void mark_keys(Small& m, int k0) {
    const int t = threadIdx.x;
    if (t < kTile) {
        bool any = false;
        for (int i = 0; i < kTile; ++i) any |= m.see[i].x <= k0 + t && k0 + t < m.see[i].y;
        m.live[t] = any;
    }
    __syncthreads();
}

template <typename T, int HD>
__global__ __launch_bounds__(kThreads, 2) void attention_kernel(const Attention a) {
    extern __shared__ __align__(16) float sm[];
    float *Q = sm, *K = Q + kTile * (HD + 4), *V = K + kTile * (HD + 4), *P = V + kTile * (HD + 4);
    Small& m = *(Small*)(P + kTile * (kTile + 4));
    const int tiles = (int)((a.T + kTile - 1) / kTile), heads = (int)(a.N * a.H);
    const int q0 = (tiles - 1 - (int)(blockIdx.x / heads)) * kTile;  // long rows first
    const int n = (int)(blockIdx.x % heads) / a.H, h = (int)(blockIdx.x % heads) % a.H, kv = h / (a.H / a.KV);
    const int64_t row0 = n * a.T;
    const int ty = threadIdx.x / 16, tx = threadIdx.x % 16, rows = (int)a.T;
    load_tile<T, HD>(Q, a.Q, a.ld_q, row0, q0, rows, h * a.hd, a.hd, nullptr, vectors<T>(a.Q, a.ld_q, a.hd));
    load_rows(a, m, row0, q0);
    float acc[4][HD / 16], top[4], sum[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        top[r] = -CUDART_INF_F, sum[r] = 0.f;
#pragma unroll
        for (int c = 0; c < HD / 16; ++c) acc[r][c] = 0.f;
    }
    const uint8_t* live = a.range ? m.live : nullptr;
    by_rows(rows - q0, [&](auto groups) {
        constexpr int R = decltype(groups)::value;
        for (int k0 = m.lo / kTile * kTile; k0 < m.hi; k0 += kTile) {
            if (live) mark_keys(m, k0);
            load_tile<T, HD>(K, a.K, a.ld_k, row0, k0, rows, kv * a.hd, a.hd, live, vectors<T>(a.K, a.ld_k, a.hd));
            load_tile<T, HD>(V, a.V, a.ld_v, row0, k0, rows, kv * a.hd, a.hd, live, vectors<T>(a.V, a.ld_v, a.hd));
            load_biases<T>(a, m.biases, h, (int64_t)q0 - k0);
            __syncthreads();
            float s[4][4];
            dots<HD, R>(Q, K, s);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int i = ty + 16 * r;
                const int2 see = m.see[i];
                float most = -CUDART_INF_F;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const int j = tx + 16 * c;
                    float bend;
                    const float x = score(s[r][c], a.scale, a.cap, m.biases[kTile + i - j], &bend);
                    s[r][c] = k0 + j >= see.x && k0 + j < see.y ? x : -CUDART_INF_F;
                    most = fmaxf(most, s[r][c]);
                }
                const float now = fmaxf(top[r], row_max(most));
                const float base = now == -CUDART_INF_F ? 0.f : now;
                const float by = expf(top[r] - base);
                float part = 0.f;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const float p = expf(s[r][c] - base);
                    part += p;
                    P[i * (kTile + 4) + tx + 16 * c] = p;
                }
                sum[r] = sum[r] * by + row_sum(part);
                top[r] = now;
#pragma unroll
                for (int c = 0; c < HD / 16; ++c) acc[r][c] *= by;
            }
            __syncthreads();
            weigh<HD, R>(P, V, acc, min(rows - k0, kTile));
            __syncthreads();
        }
    });
    float by[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        by[r] = sum[r] != 0.f ? 1.f / sum[r] : 0.f;  // NaN sums stay NaN
        const int i = q0 + ty + 16 * r;
        if (a.lse && tx == 0 && i < rows) a.lse[((int64_t)n * a.H + h) * a.T + i] = sum[r] != 0.f ? top[r] + logf(sum[r]) : -CUDART_INF_F;
    }
    store_tile<T, HD>(a.O, a.ld_o, row0, q0, rows, h * a.hd, a.hd, acc, by);
}

// delta[n][h][t] = dO . O, a warp per token and head.
template <typename T>
__global__ __launch_bounds__(256) void attention_delta_kernel(const Attention a, float* delta) {
    const int64_t at = (int64_t)blockIdx.x * 8 + threadIdx.x / 32;
    if (at >= a.N * a.T * a.H) return;
    const int lane = threadIdx.x % 32, h = (int)(at % a.H);
    const int64_t row = at / a.H;
    const T *o = (const T*)a.O + row * a.ld_o + h * a.hd, *g = (const T*)a.dO + row * a.ld_do + h * a.hd;
    float v = 0.f;
    for (int c = lane; c < a.hd; c += 32) v = fmaf(wide(o[c]), wide(g[c]), v);
#pragma unroll
    for (int s = 16; s; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
    if (lane == 0) delta[((row / a.T) * a.H + h) * a.T + row % a.T] = v;
}

__device__ __forceinline__ void load_stats(const Attention& a, Small& m, const float* delta, int n, int h, int q0) {
    const int t = threadIdx.x;
    if (t < kTile && q0 + t < a.T) {
        const int64_t at = ((int64_t)n * a.H + h) * a.T + q0 + t;
        const float l = a.lse[at];
        m.lse[t] = l == -CUDART_INF_F ? CUDART_INF_F : l;  // a row without keys: P = 0
        m.delta[t] = delta[at];
    }
}

// From dot products to P and to the gradient of the scores. A row that sees one key has P = 1 whatever the score, so its
// gradient is zero, not the rounding of dP - delta.
__device__ __forceinline__ void gradient(const Attention& a, const Small& m, int i, int j, int k0, float dot, float dp, float* p,
                                         float* ds, float* dx) {
    const int2 see = m.see[i];
    float bend;
    const float x = score(dot, a.scale, a.cap, m.biases[kTile + i - j], &bend);
    const bool in = k0 + j >= see.x && k0 + j < see.y;
    *p = in ? expf(x - m.lse[i]) : 0.f;
    const bool more = in && see.y - see.x > 1;
    *ds = more ? *p * (dp - m.delta[i]) : 0.f;
    *dx = more ? *ds * bend : 0.f;
}

template <typename T, int HD>
__device__ __forceinline__ void dq_tile(const Attention& a, const float* delta, float* part, int block, float* sm) {
    float *Q = sm, *K = Q + kTile * (HD + 4), *V = K + kTile * (HD + 4), *G = V + kTile * (HD + 4);
    float* S = G + kTile * (HD + 4);
    Small& m = *(Small*)(S + kTile * (kTile + 4));
    const int tiles = (int)((a.T + kTile - 1) / kTile), heads = (int)(a.N * a.H);
    const int q0 = (tiles - 1 - (int)(block / heads)) * kTile;
    const int n = (int)(block % heads) / a.H, h = (int)(block % heads) % a.H, kv = h / (a.H / a.KV);
    const int64_t row0 = n * a.T;
    const int ty = threadIdx.x / 16, tx = threadIdx.x % 16, rows = (int)a.T;
    load_tile<T, HD>(Q, a.Q, a.ld_q, row0, q0, rows, h * a.hd, a.hd, nullptr, vectors<T>(a.Q, a.ld_q, a.hd));
    load_tile<T, HD>(G, a.dO, a.ld_do, row0, q0, rows, h * a.hd, a.hd, nullptr, vectors<T>(a.dO, a.ld_do, a.hd));
    load_rows(a, m, row0, q0);
    load_stats(a, m, delta, n, h, q0);
    const bool learned = a.dtable != nullptr;
    float acc[4][HD / 16];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < HD / 16; ++c) acc[r][c] = 0.f;
    // buckets t and t + 256 ... of this tile's sum, in the order of the key tiles
    float* mine = part + ((int64_t)h * a.N * tiles + (int64_t)n * tiles + q0 / kTile) * a.n_buckets;
    if (learned)
        for (int b = threadIdx.x; b < a.n_buckets; b += kThreads) mine[b] = 0.f;
    const uint8_t* live = a.range ? m.live : nullptr;
    by_rows(learned ? kTile : rows - q0, [&](auto groups) {  // the diagonals' sums read every row
        constexpr int R = decltype(groups)::value;
        for (int k0 = m.lo / kTile * kTile; k0 < m.hi; k0 += kTile) {
            if (live) mark_keys(m, k0);
            load_tile<T, HD>(K, a.K, a.ld_k, row0, k0, rows, kv * a.hd, a.hd, live, vectors<T>(a.K, a.ld_k, a.hd));
            load_tile<T, HD>(V, a.V, a.ld_v, row0, k0, rows, kv * a.hd, a.hd, live, vectors<T>(a.V, a.ld_v, a.hd));
            load_biases<T>(a, m.biases, h, (int64_t)q0 - k0);
            __syncthreads();
            float s[4][4], dp[4][4], ds[4][4], p;
            dots<HD, R>(Q, K, s);
            dots<HD, R>(G, V, dp);
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    float dx;
                    gradient(a, m, ty + 16 * r, tx + 16 * c, k0, s[r][c], dp[r][c], &p, &ds[r][c], &dx);
                    s[r][c] = dx;
                    if (learned) S[(ty + 16 * r) * (kTile + 4) + tx + 16 * c] = ds[r][c];
                }
            if (learned) {
                __syncthreads();
                const int t = threadIdx.x;
                if (t > 0 && t < 2 * kTile) {  // diagonal i - j = t - 64, top to bottom
                    const int d = t - kTile;
                    float v = 0.f;
                    for (int i = max(d, 0); i < min(kTile, kTile + d); ++i) v += S[i * (kTile + 4) + i - d];
                    m.diag[t] = v;
                    const int64_t far = min(max((int64_t)q0 - k0 + d, -a.reach), a.reach);
                    m.ids[t] = a.bucket[far + a.reach];
                }
                __syncthreads();
                for (int b = t; b < a.n_buckets; b += kThreads) {
                    float v = mine[b];
                    for (int i = 1; i < 2 * kTile; ++i)
                        if (m.ids[i] == b) v += m.diag[i];
                    mine[b] = v;
                }
                __syncthreads();
            }
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int c = 0; c < 4; ++c) S[(ty + 16 * r) * (kTile + 4) + tx + 16 * c] = s[r][c];
            __syncthreads();
            weigh<HD, R>(S, K, acc, min(rows - k0, kTile));
            __syncthreads();
        }
    });
    const float by[4] = {a.scale, a.scale, a.scale, a.scale};
    store_tile<T, HD>(a.dQ, a.ld_dq, row0, q0, rows, h * a.hd, a.hd, acc, by);
}

template <typename T, int HD>
__device__ __forceinline__ void dkv_tile(const Attention& a, const float* delta, int block, float* sm) {
    float *Q = sm, *K = Q + kTile * (HD + 4), *V = K + kTile * (HD + 4), *G = V + kTile * (HD + 4);
    float *P = G + kTile * (HD + 4), *S = P + kTile * (kTile + 4);
    Small& m = *(Small*)(S + kTile * (kTile + 4));
    const int heads = (int)(a.N * a.KV), group = a.H / a.KV;
    const int k0 = (int)(block / heads) * kTile, n = (int)(block % heads) / a.KV, kv = (int)(block % heads) % a.KV;
    const int64_t row0 = n * a.T;
    const int ty = threadIdx.x / 16, tx = threadIdx.x % 16, rows = (int)a.T;
    load_tile<T, HD>(K, a.K, a.ld_k, row0, k0, rows, kv * a.hd, a.hd, nullptr, vectors<T>(a.K, a.ld_k, a.hd));
    load_tile<T, HD>(V, a.V, a.ld_v, row0, k0, rows, kv * a.hd, a.hd, nullptr, vectors<T>(a.V, a.ld_v, a.hd));
    float dk[4][HD / 16], dv[4][HD / 16];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int c = 0; c < HD / 16; ++c) dk[r][c] = dv[r][c] = 0.f;
    by_rows(rows - k0, [&](auto groups) {
        constexpr int R = decltype(groups)::value;
        for (int q0 = !a.range && a.causal ? k0 : 0; q0 < rows; q0 += kTile) {
            bool any = false;
            if (threadIdx.x < kTile) {
                const int2 v = visible(a.range, a.causal, rows, row0, q0 + threadIdx.x);
                m.see[threadIdx.x] = v;
                any = max(v.x, k0) < min(v.y, k0 + kTile);
                m.live[threadIdx.x] = any;
            }
            if (!__syncthreads_or(any)) continue;
            for (int h = kv * group; h < (kv + 1) * group; ++h) {
                load_tile<T, HD>(Q, a.Q, a.ld_q, row0, q0, rows, h * a.hd, a.hd, a.range ? m.live : nullptr, vectors<T>(a.Q, a.ld_q, a.hd));
                load_tile<T, HD>(G, a.dO, a.ld_do, row0, q0, rows, h * a.hd, a.hd, a.range ? m.live : nullptr, vectors<T>(a.dO, a.ld_do, a.hd));
                load_stats(a, m, delta, n, h, q0);
                load_biases<T>(a, m.biases, h, (int64_t)q0 - k0);
                __syncthreads();
                float s[4][4], dp[4][4];
                dots<HD, R>(K, Q, s);  // rows are keys
                dots<HD, R>(V, G, dp);
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        float p, ds, dx;
                        gradient(a, m, tx + 16 * c, ty + 16 * r, k0, s[r][c], dp[r][c], &p, &ds, &dx);
                        P[(ty + 16 * r) * (kTile + 4) + tx + 16 * c] = p;
                        S[(ty + 16 * r) * (kTile + 4) + tx + 16 * c] = dx;
                    }
                __syncthreads();
                weigh<HD, R>(P, G, dv, min(rows - q0, kTile));
                weigh<HD, R>(S, Q, dk, min(rows - q0, kTile));
                __syncthreads();
            }
        }
    });
    const float by[4] = {a.scale, a.scale, a.scale, a.scale}, one[4] = {1.f, 1.f, 1.f, 1.f};
    store_tile<T, HD>(a.dK, a.ld_dk, row0, k0, rows, kv * a.hd, a.hd, dk, by);
    store_tile<T, HD>(a.dV, a.ld_dv, row0, k0, rows, kv * a.hd, a.hd, dv, one);
}

// dK, dV of a tile of keys, or dQ of a tile of queries: the two kinds of CTAs in one launch, so that an SM has one of either (2 x 515
// tokens of 8 heads fp32 one after the other 202 + 175 us).
template <typename T, int HD>
__global__ __launch_bounds__(kThreads, HD == 64 ? 2 : 1) void attention_grad_kernel(const Attention a, const float* delta, float* part,
                                                                                   int kv_tiles) {
    extern __shared__ __align__(16) float sm[];
    if ((int)blockIdx.x < kv_tiles) dkv_tile<T, HD>(a, delta, blockIdx.x, sm);
    else dq_tile<T, HD>(a, delta, part, blockIdx.x - kv_tiles, sm);
}

// dtable[b][h] = beta dtable[b][h] + the sum of head h's partial sums, in order: a warp per entry, 32 running sums joined
// at the end, the long sum in 64 bits.
template <typename T>
__global__ __launch_bounds__(256) void attention_dtable_kernel(const float* part, int64_t rows, int n_buckets, int H, float beta,
                                                               T* out) {
    const int at = blockIdx.x * 8 + threadIdx.x / 32, lane = threadIdx.x % 32;
    if (at >= n_buckets * H) return;
    const int b = at / H, h = at % H;
    double v = 0;
    for (int64_t i = lane; i < rows; i += 32) v += part[(h * rows + i) * n_buckets + b];
#pragma unroll
    for (int s = 16; s; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
    if (lane == 0) out[at] = narrow<T>((float)(beta != 0.f ? beta * (double)wide(out[at]) + v : v));
}

// The same from sums by distance, width = 2 mid + 1 of them: a CTA per head adds up each distance over its rows, then each bucket over
// its distances, both in order.
template <typename T>
__global__ __launch_bounds__(1024) void attention_distances_kernel(const float* part, int64_t rows, int mid, const int32_t* bucket,
                                                                  int64_t reach, int n_buckets, int H, float beta, T* out) {
    chain_wait();
    __shared__ float sums[1024];
    __shared__ int ids[1024];
    const int h = blockIdx.x, t = threadIdx.x, width = 2 * mid + 1;
    // threads in groups of `width` rounded up to warps, each group every `groups`-th row
    const int span = (width + 31) / 32 * 32, groups = max(1, 1024 / span), g = t / span, d = t % span;
    float v = 0.f, low = 0.f;  // the sum and what its roundings lost: the SM has 64-bit adders for two lanes
    auto add = [&](float x) {
        const float y = x - low, s = v + y;
        low = (s - v) - y, v = s;
    };
    if (g < groups && d < width) {
        const float* p = part + h * rows * width + d;
        int64_t i = g;
        for (; i + 7 * groups < rows; i += 8 * groups) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = p[(i + e * groups) * width];
#pragma unroll
            for (int e = 0; e < 8; ++e) add(x[e]);
        }
        for (; i < rows; i += groups) add(p[i * width]);
    }
    sums[t] = v;
    if (t < width) ids[t] = bucket[t - mid + reach];
    __syncthreads();
    if (t < width) {
        for (int k = 1; k < groups; ++k) v += sums[k * span + t];
        sums[t] = v;  // other groups' places are past the first
    }
    __syncthreads();
    for (int b = t / 32; b < n_buckets; b += 32) {
        float s = 0.f;
        for (int i = t % 32; i < width; i += 32)
            if (ids[i] == b) s += sums[i];
#pragma unroll
        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        if (t % 32 == 0) {
            T& x = out[(int64_t)b * H + h];
            x = narrow<T>(beta != 0.f ? fmaf(beta, wide(x), s) : s);
        }
    }
}

// ------------------------------------------------------------------ ranges
constexpr int kScan = 1024, kEach = 8;

// Inclusive scan over the CTA's threads, the last thread's first where REVERSE; `identity` leaves the other operand.
template <bool MAX, bool REVERSE>
__device__ __forceinline__ int scan(int v, int identity, int* parts) {
    const int t = REVERSE ? kScan - 1 - threadIdx.x : threadIdx.x, lane = threadIdx.x % 32;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int u = REVERSE ? __shfl_down_sync(0xffffffffu, v, o) : __shfl_up_sync(0xffffffffu, v, o);
        if (REVERSE ? lane + o < 32 : lane >= o) v = MAX ? max(v, u) : min(v, u);
    }
    const int w = t / 32;
    if ((t & 31) == 31) parts[w] = v;
    __syncthreads();
    int before = identity;
    for (int i = 0; i < w; ++i) before = MAX ? max(before, parts[i]) : min(before, parts[i]);
    __syncthreads();
    return MAX ? max(v, before) : min(v, before);
}

// Up to 8192 tokens: one CTA per example, EACH tokens a thread in registers, and the three steps of the kernel below at once:
// scans over the warps' tokens, over the warps by each warp, and the ends of the prefixes through shared memory.
// 4 x 2047 tokens 5 us (the kernel below 12).
template <int EACH>
__global__ __launch_bounds__(kScan) void attention_ranges_short_kernel(const int32_t* doc, const int32_t* prefix, int causal, int T,
                                                                       int64_t window, int2* range) {
    __shared__ int stops[kScan * EACH], firsts[kScan / 32], ends[kScan / 32];
    const int64_t row0 = (int64_t)blockIdx.x * T;
    const int32_t* pre = causal ? prefix : nullptr;
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, at = threadIdx.x * EACH;
    int ids[EACH + 2], flags[EACH];  // from token at - 1 to at + EACH
#pragma unroll
    for (int e = 0; e < EACH + 2; ++e) {
        const int i = at + e - 1;
        ids[e] = doc && i >= 0 && i < T ? doc[row0 + i] : 0;
    }
#pragma unroll
    for (int e = 0; e < EACH; ++e) flags[e] = pre && at + e < T ? pre[row0 + at + e] : 0;
    int first[EACH], stop[EACH], f = 0, s = T;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        if (at + e > 0 && ids[e + 1] != ids[e]) f = at + e;
        first[e] = f;
    }
#pragma unroll
    for (int e = EACH - 1; e >= 0; --e) {
        const int i = at + e;
        if (i < T) {
            const bool last = i == T - 1 || ids[e + 2] != ids[e + 1];
            if (pre) {
                if (last || !flags[e]) s = i + (flags[e] != 0);
            } else if (last) {
                s = i + 1;
            }
        }
        stop[e] = s;
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, f, o), y = __shfl_down_sync(0xffffffffu, s, o);
        if (lane >= o) f = max(f, x);
        if (lane + o < 32) s = min(s, y);
    }
    if (lane == 31) firsts[warp] = f;
    if (lane == 0) ends[warp] = s;
    f = __shfl_up_sync(0xffffffffu, f, 1), s = __shfl_down_sync(0xffffffffu, s, 1);
    if (lane == 0) f = 0;
    if (lane == 31) s = T;
    __syncthreads();
    f = max(f, __reduce_max_sync(0xffffffffu, lane < warp ? firsts[lane] : 0));
    s = min(s, __reduce_min_sync(0xffffffffu, lane > warp ? ends[lane] : T));
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        first[e] = max(first[e], f), stop[e] = min(stop[e], s);
        stops[at + e] = stop[e];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const int i = at + e;
        if (i >= T) continue;
        int64_t lo = first[e], hi = !causal ? stop[e] : pre ? max(i + 1, stops[first[e]]) : i + 1;
        if (window) lo = max(lo, i - window + 1), hi = min(hi, i + window);
        range[row0 + i] = ids[e + 1] < 0 ? make_int2(0, 0) : make_int2((int)lo, (int)hi);
    }
}

// Longer ones: one CTA per example, 8 tokens a thread at a time: forwards for the first token of each document, backwards for its end
// (or, with a prefix, for the first token from here on that is not prefix), and once more for the ranges.
__global__ __launch_bounds__(kScan) void attention_ranges_kernel(const int32_t* doc, const int32_t* prefix, int causal, int T,
                                                                 int64_t window, int2* range) {
    __shared__ int parts[kScan / 32];
    __shared__ int carry;
    const int64_t row0 = (int64_t)blockIdx.x * T;
    const int32_t* ids = doc ? doc + row0 : nullptr;
    const int32_t* pre = prefix && causal ? prefix + row0 : nullptr;
    int2* out = range + row0;
    constexpr int64_t kChunk = kScan * kEach;
    const int64_t chunks = (T + kChunk - 1) / kChunk;
    if (threadIdx.x == 0) carry = 0;
    __syncthreads();
    for (int64_t c = 0; c < chunks; ++c) {
        const int64_t at = c * kChunk + (int64_t)threadIdx.x * kEach;
        int first[kEach], run = 0;
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int64_t i = at + e;
            if (ids && i > 0 && i < T && ids[i] != ids[i - 1]) run = (int)i;
            first[e] = run;
        }
        int before = scan<true, false>(run, 0, parts);
        const int last = before;  // inclusive: this thread's own comes below
        before = __shfl_up_sync(0xffffffffu, before, 1);
        __shared__ int edge[kScan / 32];
        if (threadIdx.x % 32 == 31) edge[threadIdx.x / 32] = last;
        __syncthreads();
        if (threadIdx.x % 32 == 0) before = threadIdx.x ? edge[threadIdx.x / 32 - 1] : 0;
        before = max(before, carry);
        __syncthreads();
        if (threadIdx.x == kScan - 1) carry = max(last, carry);
#pragma unroll
        for (int e = 0; e < kEach; ++e)
            if (at + e < T) out[at + e].x = max(first[e], before);
        __syncthreads();
    }
    if (threadIdx.x == 0) carry = T;
    __syncthreads();
    for (int64_t c = chunks - 1; c >= 0; --c) {
        const int64_t at = c * kChunk + (int64_t)threadIdx.x * kEach;
        int stop[kEach], run = T;
#pragma unroll
        for (int e = kEach - 1; e >= 0; --e) {
            const int64_t i = at + e;
            if (i < T) {
                const bool last = i == T - 1 || (ids && ids[i + 1] != ids[i]);
                if (pre) {
                    const bool p = pre[i] != 0;
                    if (last || !p) run = (int)i + p;
                } else if (last) {
                    run = (int)i + 1;
                }
            }
            stop[e] = run;
        }
        int after = scan<false, true>(run, T, parts);
        const int own = after;
        after = __shfl_down_sync(0xffffffffu, after, 1);
        __shared__ int edge[kScan / 32];
        if (threadIdx.x % 32 == 0) edge[threadIdx.x / 32] = own;
        __syncthreads();
        if (threadIdx.x % 32 == 31) after = threadIdx.x < kScan - 1 ? edge[threadIdx.x / 32 + 1] : T;
        after = min(after, carry);
        __syncthreads();
        if (threadIdx.x == 0) carry = min(own, carry);
#pragma unroll
        for (int e = 0; e < kEach; ++e)
            if (at + e < T) out[at + e].y = min(stop[e], after);
        __syncthreads();
    }
    // last chunk first: a document's first token still has its own value when later ones read it
    for (int64_t c = chunks - 1; c >= 0; --c) {
        const int64_t at = c * kChunk + (int64_t)threadIdx.x * kEach;
        int2 r[kEach];
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int64_t i = at + e;
            if (i >= T) continue;
            const int2 v = out[i];
            int64_t lo = v.x, hi = !causal ? v.y : pre ? max((int)i + 1, out[v.x].y) : (int)i + 1;
            if (window) lo = max(lo, i - window + 1), hi = min(hi, i + window);
            r[e] = ids && ids[i] < 0 ? make_int2(0, 0) : make_int2((int)lo, (int)hi);
        }
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kEach; ++e)
            if (at + e < T) out[at + e] = r[e];
        __syncthreads();
    }
}

template <typename T, int HD>
cudaError_t forward_simt(const Attention& a, cudaStream_t s) {
    constexpr size_t smem = smem_of<HD>(3, 1);
    if (cudaError_t e = smem_attr_once<attention_kernel<T, HD>>(smem)) return e;
    const int64_t tiles = (a.T + kTile - 1) / kTile;
    note_launches(1);
    attention_kernel<T, HD><<<(unsigned)(tiles * a.N * a.H), kThreads, smem, s>>>(a);
    return cudaGetLastError();
}

cudaError_t join_table(const Attention& a, const float* part, int64_t rows, cudaStream_t s) {
    if (!a.dtable) return cudaSuccess;
    note_launches(1);
    const unsigned grid = (unsigned)((a.n_buckets * a.H + 7) / 8);
    if (a.gt == TDA_BF16)
        attention_dtable_kernel<<<grid, 256, 0, s>>>(part, rows, a.n_buckets, a.H, a.beta, (__nv_bfloat16*)a.dtable);
    else
        attention_dtable_kernel<<<grid, 256, 0, s>>>(part, rows, a.n_buckets, a.H, a.beta, (float*)a.dtable);
    return cudaGetLastError();
}

template <typename T, int HD>
cudaError_t backward_simt(const Attention& a, float* delta, float* part, cudaStream_t s) {
    constexpr size_t smem = smem_of<HD>(4, 2);
    if (cudaError_t e = smem_attr_once<attention_grad_kernel<T, HD>>(smem)) return e;
    const int64_t tiles = (a.T + kTile - 1) / kTile;
    note_launches(2);
    attention_delta_kernel<T><<<(unsigned)((a.N * a.T * a.H + 7) / 8), 256, 0, s>>>(a, delta);
    attention_grad_kernel<T, HD><<<(unsigned)(tiles * a.N * (a.KV + a.H)), kThreads, smem, s>>>(a, delta, part, (int)(tiles * a.N * a.KV));
    if (cudaError_t e = cudaGetLastError()) return e;
    return join_table(a, part, a.N * tiles, s);
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }

}  // namespace

size_t attention_ws_bytes(const Attention& a, bool backward, bool bound) {
    const bool aligned = bound ? a.dt == TDA_BF16 && a.hd % 8 == 0 : attention_tc_supported(a, backward);
    if (!backward) return aligned ? attention_plan_bytes(a, bound) : 0;
    const size_t tc = aligned ? attention_grad_tc_bytes(a, bound) : 0;
    if (aligned && !bound) return tc;
    const size_t tiles = (size_t)((a.T + kTile - 1) / kTile);
    return std::max(tc, up((size_t)a.N * a.T * a.H * 4) + up((size_t)a.N * a.H * tiles * a.n_buckets * 4));
}

cudaError_t launch_attention_forward(const Attention& a, void* ws, unsigned int* err, cudaStream_t s) {
    if (attention_tc_supported(a, false)) return launch_attention_forward_tc(a, ws, err, s);
    if (a.dt == TDA_BF16) return a.hd <= 64 ? forward_simt<__nv_bfloat16, 64>(a, s) : forward_simt<__nv_bfloat16, 128>(a, s);
    return a.hd <= 64 ? forward_simt<float, 64>(a, s) : forward_simt<float, 128>(a, s);
}

cudaError_t launch_attention_backward(const Attention& a, void* ws, unsigned int* err, cudaStream_t s) {
    if (attention_tc_supported(a, true)) {
        float* part;
        if (cudaError_t e = launch_attention_backward_tc(a, ws, err, &part, s)) return e;
        const int64_t rows = a.N * ((a.T + 127) / 128);
        const int mid = attention_dense_mid(a);
        if (!a.dtable || mid < 0) return join_table(a, part, rows, s);
        return a.gt == TDA_BF16 ? launch_chained(true, attention_distances_kernel<__nv_bfloat16>, dim3(a.H), dim3(1024), 0, s, (const float*)part,
                                                 rows, mid, a.bucket, a.reach, a.n_buckets, a.H, a.beta, (__nv_bfloat16*)a.dtable)
                                : launch_chained(true, attention_distances_kernel<float>, dim3(a.H), dim3(1024), 0, s, (const float*)part, rows,
                                                 mid, a.bucket, a.reach, a.n_buckets, a.H, a.beta, (float*)a.dtable);
    }
    float* delta = (float*)ws;
    float* part = (float*)((char*)ws + up((size_t)a.N * a.T * a.H * 4));
    if (a.dt == TDA_BF16)
        return a.hd <= 64 ? backward_simt<__nv_bfloat16, 64>(a, delta, part, s)
                          : backward_simt<__nv_bfloat16, 128>(a, delta, part, s);
    return a.hd <= 64 ? backward_simt<float, 64>(a, delta, part, s) : backward_simt<float, 128>(a, delta, part, s);
}

cudaError_t launch_attention_ranges(int64_t N, int64_t T, const int32_t* doc, const int32_t* prefix, int causal, int64_t window,
                                    int2* range, cudaStream_t s) {
    note_launches(1);
    if (T <= 2 * kScan) attention_ranges_short_kernel<2><<<(unsigned)N, kScan, 0, s>>>(doc, prefix, causal, (int)T, window, range);
    else if (T <= 8 * kScan) attention_ranges_short_kernel<8><<<(unsigned)N, kScan, 0, s>>>(doc, prefix, causal, (int)T, window, range);
    else attention_ranges_kernel<<<(unsigned)N, kScan, 0, s>>>(doc, prefix, causal, (int)T, window, range);
    return cudaGetLastError();
}

}  // namespace tda
