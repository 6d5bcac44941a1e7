// k_embedding.cu -- embedding lookup with scaling, and its gradient.
//
// Lookup: out[i] = scale E[t_i]; a padded token (t_i < 0) gives a zero row, an
// id outside the table (t_i >= V) a NaN row, so that it is seen. Bound by HBM:
// the rows read plus the rows written. A group of lanes copies up to four
// vectors per lane of one row, all loads before the first store.
//
// Gradient: dE[v] = beta dE[v] + scale sum_{i : t_i = v} dOut[i]. The positions
// are sorted by (token, position), the sorted list is cut into chunks of equal
// length, and each chunk adds its rows up in that order, so hot tokens are
// spread over the GPU and the sums do not depend on timing. A token whose run
// lies inside one chunk is finished there; a run that crosses a chunk's edge
// leaves one fp32 partial row per chunk, and a last launch adds a run's partials
// in order. Rows of E that no token names are cleared (or scaled by beta) by
// further CTAs of the same launch. Bound by HBM: n rows read, V rows written.
// Sums are fp32, rounded once to dE's type.
#include <cuda_bf16.h>

#include "tda_internal.cuh"

namespace tda {
namespace {

// ------------------------------------------------------------------ element helpers
// N consecutive values, moved as one access or as several of 16 bytes.
template <typename T, int N>
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Vec {
    T v[N];
};
__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void set_f(float* p, float x) { *p = x; }
__device__ __forceinline__ void set_f(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// A token id as the sort sees it: valid ids as they are, padding and ids outside the table as V (last).
template <typename I>
__device__ __forceinline__ uint32_t sort_key(const I* tok, int64_t i, uint32_t V) {
    const I t = tok[i];
    return t >= 0 && (uint64_t)t < V ? (uint32_t)t : V;
}

// ------------------------------------------------------------------ lookup
constexpr int kLookThreads = 256, kLookVecs = 4;

// lanes (a power of two <= 32) copy one segment of lanes * kLookVecs vectors of a row.
template <typename T, typename I, int N>
__global__ void __launch_bounds__(kLookThreads)
lookup_kernel(const T* __restrict__ E, int64_t ld_e, int64_t V, int64_t d, const I* __restrict__ tok, int64_t n,
              float scale, T* __restrict__ out, int64_t ld_out, int lanes, int64_t segs) {
    const int64_t g = ((int64_t)blockIdx.x * kLookThreads + threadIdx.x) / lanes;
    const int64_t row = g / segs;
    if (row >= n) return;
    const int64_t v0 = (g % segs) * lanes * kLookVecs + threadIdx.x % lanes, nv = d / N;
    const I t = tok[row];
    const bool in = t >= 0 && (uint64_t)t < (uint64_t)V;
    Vec<T, N> x[kLookVecs];
    if (in) {
        const Vec<T, N>* src = reinterpret_cast<const Vec<T, N>*>(E + (int64_t)t * ld_e);
#pragma unroll
        for (int j = 0; j < kLookVecs; ++j)
            if (v0 + j * lanes < nv) x[j] = src[v0 + j * lanes];
    }
    Vec<T, N>* dst = reinterpret_cast<Vec<T, N>*>(out + row * ld_out);
    const float fill = t < 0 ? 0.f : __int_as_float(0x7fc00000);
#pragma unroll
    for (int j = 0; j < kLookVecs; ++j) {
        if (v0 + j * lanes >= nv) break;
        Vec<T, N> y;
#pragma unroll
        for (int e = 0; e < N; ++e) set_f(&y.v[e], in ? to_f(x[j].v[e]) * scale : fill);
        dst[v0 + j * lanes] = y;
    }
}

// ------------------------------------------------------------------ sort by (token, position)
// Up to kRankMax tokens: the place of token i in the sorted list is the number of tokens before it,
// #{j < i : k_j <= k_i} + #{j > i : k_j < k_i}, counted directly: one launch, n^2 comparisons over all SMs.
constexpr int kRankMax = 8192, kRankThreads = 256;

template <typename I>
__global__ void __launch_bounds__(kRankThreads)
rank_kernel(const I* __restrict__ tok, int n, uint32_t V, uint32_t* __restrict__ skey, int32_t* __restrict__ order) {
    __shared__ alignas(16) uint32_t key[kRankMax];
    __shared__ int cnt[kRankThreads / 32][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int np = (n + 31) & ~31;
    for (int j = threadIdx.x; j < np; j += kRankThreads) key[j] = j < n ? sort_key(tok, j, V) : 0xFFFFFFFFu;
    __syncthreads();
    const int i0 = blockIdx.x * 32, i = i0 + lane;
    const uint32_t k = key[i];  // np covers i; a lane past n counts in vain
    const int groups = np / 32, g0 = groups * warp / (kRankThreads / 32), g1 = groups * (warp + 1) / (kRankThreads / 32);
    int c = 0;
    for (int g = g0; g < g1; ++g) {
        const uint4* q = reinterpret_cast<const uint4*>(key + g * 32);
        if (g * 32 < i0) {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const uint4 w = q[u];
                c += (w.x <= k) + (w.y <= k) + (w.z <= k) + (w.w <= k);
            }
        } else if (g * 32 > i0) {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const uint4 w = q[u];
                c += (w.x < k) + (w.y < k) + (w.z < k) + (w.w < k);
            }
        } else {
#pragma unroll 4
            for (int u = 0; u < 32; ++u) c += key[i0 + u] < k || (key[i0 + u] == k && u < lane);
        }
    }
    cnt[warp][lane] = c;
    __syncthreads();
    if (warp == 0 && i < n) {
#pragma unroll
        for (int w = 1; w < kRankThreads / 32; ++w) c += cnt[w][lane];
        skey[c] = k;
        order[c] = i;
    }
}

// More tokens: a stable radix sort from the low digit up, digits of at most 9 bits (2 passes up to 2^18 ids),
// three launches a pass: digit counts per tile, their scan per digit, the scatter.
constexpr int kTile = 4096, kSortThreads = 256, kBins = 512, kRounds = kTile / kSortThreads;

template <typename I>
__global__ void __launch_bounds__(kSortThreads)
digit_count_kernel(const I* __restrict__ tok, const uint32_t* __restrict__ key, int n, uint32_t V, int shift,
                   uint32_t mask, uint32_t* __restrict__ hist) {
    __shared__ uint32_t h[kBins];
    for (int b = threadIdx.x; b < kBins; b += kSortThreads) h[b] = 0;
    __syncthreads();
    const int64_t base = (int64_t)blockIdx.x * kTile;
#pragma unroll 4
    for (int r = 0; r < kRounds; ++r) {
        const int64_t i = base + r * kSortThreads + threadIdx.x;
        if (i < n) atomicAdd(&h[((key ? key[i] : sort_key(tok, i, V)) >> shift) & mask], 1u);
    }
    __syncthreads();
    for (uint32_t b = threadIdx.x; b <= mask; b += kSortThreads) hist[(int64_t)b * gridDim.x + blockIdx.x] = h[b];
}

// CTA b: exclusive scan of digit b's counts over the tiles, and their total.
__global__ void __launch_bounds__(kSortThreads) digit_scan_kernel(uint32_t* __restrict__ hist, int tiles,
                                                                  uint32_t* __restrict__ total) {
    __shared__ uint32_t w[kSortThreads / 32];
    uint32_t* h = hist + (int64_t)blockIdx.x * tiles;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t before = 0;
    for (int t0 = 0; t0 < tiles; t0 += kSortThreads) {
        const int t = t0 + threadIdx.x;
        const uint32_t x = t < tiles ? h[t] : 0;
        uint32_t s = x;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, s, o);
            if (lane >= o) s += y;
        }
        if (lane == 31) w[warp] = s;
        __syncthreads();
        uint32_t add = before, all = 0;
#pragma unroll
        for (int i = 0; i < kSortThreads / 32; ++i) {
            if (i < warp) add += w[i];
            all += w[i];
        }
        if (t < tiles) h[t] = add + s - x;
        before += all;
        __syncthreads();
    }
    if (threadIdx.x == 0) total[blockIdx.x] = before;
}

template <typename I>
__global__ void __launch_bounds__(kSortThreads)
digit_scatter_kernel(const I* __restrict__ tok, const uint32_t* __restrict__ key, const int32_t* __restrict__ val,
                     int n, uint32_t V, int shift, uint32_t mask, const uint32_t* __restrict__ hist,
                     const uint32_t* __restrict__ total, uint32_t* __restrict__ key_out,
                     int32_t* __restrict__ val_out) {
    constexpr int W = kSortThreads / 32, kPer = kTile / W / 32;
    __shared__ uint32_t pos[W][kBins];  // counts of each warp's run, then the next place of each digit
    __shared__ uint32_t start[kBins];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int b = threadIdx.x; b < W * kBins; b += kSortThreads) (&pos[0][0])[b] = 0;
    // first place of each digit: scan of the totals (warp 0, 16 digits a lane)
    if (warp == 0) {
        uint32_t x[kBins / 32], s = 0;
#pragma unroll
        for (int u = 0; u < kBins / 32; ++u) {
            const uint32_t b = lane * (kBins / 32) + u;
            x[u] = s;
            s += b <= mask ? total[b] : 0;
        }
        uint32_t inc = s;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t y = __shfl_up_sync(0xffffffffu, inc, o);
            if (lane >= o) inc += y;
        }
#pragma unroll
        for (int u = 0; u < kBins / 32; ++u) start[lane * (kBins / 32) + u] = inc - s + x[u];
    }
    __syncthreads();
    const int64_t base = (int64_t)blockIdx.x * kTile + (int64_t)warp * (kTile / W);
    uint32_t k[kPer];
#pragma unroll
    for (int r = 0; r < kPer; ++r) {
        const int64_t i = base + r * 32 + lane;
        k[r] = i < n ? (key ? key[i] : sort_key(tok, i, V)) : 0;
    }
#pragma unroll
    for (int r = 0; r < kPer; ++r) {
        const bool live = base + r * 32 + lane < n;
        const uint32_t dg = live ? (k[r] >> shift) & mask : 0xFFFFFFFFu;
        const uint32_t same = __match_any_sync(0xffffffffu, dg);
        if (live && (same & ((1u << lane) - 1)) == 0) pos[warp][dg] += __popc(same);
        __syncwarp();
    }
    __syncthreads();
    for (uint32_t b = threadIdx.x; b <= mask; b += kSortThreads) {
        uint32_t at = start[b] + hist[(int64_t)b * gridDim.x + blockIdx.x];
#pragma unroll
        for (int w = 0; w < W; ++w) {
            const uint32_t c = pos[w][b];
            pos[w][b] = at;
            at += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kPer; ++r) {
        const int64_t i = base + r * 32 + lane;
        const bool live = i < n;
        const uint32_t dg = live ? (k[r] >> shift) & mask : 0xFFFFFFFFu;
        const uint32_t same = __match_any_sync(0xffffffffu, dg);
        const uint32_t below = __popc(same & ((1u << lane) - 1));
        if (live) {
            const uint32_t p = pos[warp][dg] + below;
            key_out[p] = k[r];
            val_out[p] = val ? val[i] : (int32_t)i;
        }
        __syncwarp();
        if (live && below == 0) pos[warp][dg] += __popc(same);
        __syncwarp();
    }
}

// ------------------------------------------------------------------ sums over the sorted list
constexpr int kSumThreads = 128, kBatch = 8, kZeroRows = 32;

struct GradParams {
    int64_t n, d, ld_d, V, ld_e, dp;  // dp: row length of the partials
    int64_t chunks, col_blocks;
    int C;
    float scale, beta;
    const uint32_t* skey;
    const int32_t* order;
    float* part;  // [chunk][head, tail][dp]
};

template <typename TO, int N>
__device__ __forceinline__ void store_row(TO* p, const float* acc, float scale, float beta) {
    Vec<TO, N>* q = reinterpret_cast<Vec<TO, N>*>(p);
    Vec<TO, N> y;
    if (beta != 0.f) {
        const Vec<TO, N> old = *q;
#pragma unroll
        for (int e = 0; e < N; ++e) set_f(&y.v[e], fmaf(acc[e], scale, beta * to_f(old.v[e])));
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) set_f(&y.v[e], acc[e] * scale);
    }
    *q = y;
}

template <typename TI, typename TO, int N>
__global__ void __launch_bounds__(kSumThreads)
grad_sum_kernel(const TI* __restrict__ dout, TO* __restrict__ dE, const GradParams p) {
    const int64_t sums = p.chunks * p.col_blocks;
    if ((int64_t)blockIdx.x >= sums) {
        // rows of E that no token names
        __shared__ bool named[kZeroRows];
        const int64_t v0 = ((int64_t)blockIdx.x - sums) * kZeroRows;
        if (threadIdx.x < kZeroRows) {
            const int64_t v = v0 + threadIdx.x;
            int64_t lo = 0, hi = p.n;  // first place whose key is >= v
            while (lo < hi) {
                const int64_t mid = (lo + hi) >> 1;
                if ((int64_t)p.skey[mid] < v)
                    lo = mid + 1;
                else
                    hi = mid;
            }
            named[threadIdx.x] = v >= p.V || (lo < p.n && (int64_t)p.skey[lo] == v);
        }
        __syncthreads();
        for (int r = 0; r < kZeroRows; ++r) {
            if (named[r]) continue;
            TO* row = dE + (v0 + r) * p.ld_e;
            for (int64_t c = (int64_t)threadIdx.x * N; c < p.d; c += kSumThreads * N) {
                const float zero[N] = {};
                store_row<TO, N>(row + c, zero, 0.f, p.beta);
            }
        }
        return;
    }
    extern __shared__ uint32_t sm[];
    uint32_t* key = sm;                     // [C]
    int32_t* pos = (int32_t*)(sm + p.C);    // [C]
    const int64_t ch = (int64_t)blockIdx.x / p.col_blocks, i0 = ch * p.C;
    const int64_t col = ((int64_t)blockIdx.x % p.col_blocks) * kSumThreads * N + (int64_t)threadIdx.x * N;
    const int have = p.n - i0 < p.C ? (int)(p.n - i0) : p.C;
    for (int i = threadIdx.x; i < have; i += kSumThreads) {
        key[i] = p.skey[i0 + i];
        pos[i] = p.order[i0 + i];
    }
    const uint32_t none = (uint32_t)p.V;
    const uint32_t prev = i0 > 0 ? p.skey[i0 - 1] : none, next = i0 + p.C < p.n ? p.skey[i0 + p.C] : none;
    __syncthreads();
    if (col >= p.d) return;
    float acc[N] = {};
    int from = 0;  // where the current run starts in this chunk
    uint32_t cur = key[0];
    auto flush = [&](int to) {
        if (from == 0 && cur == prev)
            store_row<float, N>(p.part + (2 * ch) * p.dp + col, acc, 1.f, 0.f);
        else if (to == p.C && cur == next)
            store_row<float, N>(p.part + (2 * ch + 1) * p.dp + col, acc, 1.f, 0.f);
        else
            store_row<TO, N>(dE + (int64_t)cur * p.ld_e + col, acc, p.scale, p.beta);
    };
    const TI* src = dout + col;
    for (int i = 0; i < have && cur != none; i += kBatch) {
        Vec<TI, N> x[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (i + u < have && key[i + u] != none)
                x[u] = *reinterpret_cast<const Vec<TI, N>*>(src + (int64_t)pos[i + u] * p.ld_d);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (i + u >= have) break;
            if (key[i + u] != cur) {
                flush(i + u);
                cur = key[i + u];
                from = i + u;
#pragma unroll
                for (int e = 0; e < N; ++e) acc[e] = 0.f;
            }
            if (cur == none) break;
#pragma unroll
            for (int e = 0; e < N; ++e) acc[e] += to_f(x[u].v[e]);
        }
    }
    if (cur != none) flush(have);
}

// A run that crosses chunk edges: the CTA of the chunk where it starts adds its partials in order.
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32;

template <typename TO>
__global__ void __launch_bounds__(kJoinThreads) grad_join_kernel(TO* __restrict__ dE, const GradParams p) {
    const int64_t ch = blockIdx.x, i0 = ch * p.C, i1 = i0 + p.C;  // i1 < n: the last chunk starts no such run
    const uint32_t k = p.skey[i1 - 1], none = (uint32_t)p.V;
    if (k == none || p.skey[i1] != k) return;
    if (i0 > 0 && p.skey[i0 - 1] == k) return;  // the run started earlier
    int64_t lo = ch + 1, hi = p.chunks - 1;     // last chunk whose first key is k
    while (lo < hi) {
        const int64_t mid = (lo + hi + 1) >> 1;
        if (p.skey[mid * p.C] == k)
            lo = mid;
        else
            hi = mid - 1;
    }
    const int64_t parts = lo - ch + 1;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // partial 0: the tail of chunk ch; partial j: the head of chunk ch + j. Unrolled loads, ordered additions.
    auto add = [&](int64_t j0, int64_t j1, int64_t col) {
        float a = 0.f;
        for (int64_t j = j0; j < j1; j += 8) {
            float x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                x[u] = j + u < j1 ? p.part[(2 * (ch + j + u) + (j + u == 0)) * p.dp + col] : 0.f;
#pragma unroll
            for (int u = 0; u < 8; ++u) a += x[u];
        }
        return a;
    };
    __shared__ float sh[kJoinWarps][32];
    if (parts < 4 * kJoinWarps) {  // a thread adds all partials of a column
        for (int64_t col = (int64_t)blockIdx.y * kJoinThreads + threadIdx.x; col < p.d;
             col += (int64_t)gridDim.y * kJoinThreads) {
            const float a = add(0, parts, col);
            store_row<TO, 1>(dE + (int64_t)k * p.ld_e + col, &a, p.scale, p.beta);
        }
        return;
    }
    // a long run: each warp adds an eighth of the partials, then the eighths in order
    for (int64_t c0 = (int64_t)blockIdx.y * 32; c0 < p.d; c0 += (int64_t)gridDim.y * 32) {
        const int64_t col = c0 + lane;
        float a = 0.f;
        if (col < p.d) a = add(parts * warp / kJoinWarps, parts * (warp + 1) / kJoinWarps, col);
        sh[warp][lane] = a;
        __syncthreads();
        if (warp == 0 && col < p.d) {
#pragma unroll
            for (int w = 1; w < kJoinWarps; ++w) a += sh[w][lane];
            store_row<TO, 1>(dE + (int64_t)k * p.ld_e + col, &a, p.scale, p.beta);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------ host side
// Bytes of alignment that a pointer and its row stride share (a power of two, at most 16).
int row_align(const void* p, int64_t ld, size_t el) {
    const uintptr_t v = (uintptr_t)p | (uintptr_t)(ld * (int64_t)el) | 16;
    return (int)(v & (~v + 1));
}

struct GradLayout {
    int C;
    int64_t chunks, dp, tiles;
    size_t skey, order, key2, val2, hist, total, part, bytes;
};

// Sorted positions per chunk: small lists are cut finely, to have enough CTAs; long ones coarsely, to
// leave few partials (2 rows of fp32 per chunk against C rows read).
GradLayout grad_layout(int64_t d, int64_t n) {
    GradLayout g;
    g.C = n <= 16384 ? 32 : n <= 131072 ? 64 : 256;
    g.chunks = (n + g.C - 1) / g.C;
    g.dp = (d + 7) & ~(int64_t)7;
    g.tiles = (n + kTile - 1) / kTile;
    size_t at = 0;
    auto take = [&](size_t b) {
        const size_t o = at;
        at += (b + 255) & ~(size_t)255;
        return o;
    };
    g.skey = take(4 * (size_t)n);
    g.order = take(4 * (size_t)n);
    g.key2 = g.val2 = g.hist = g.total = 0;
    if (n > kRankMax) {
        g.key2 = take(4 * (size_t)n);
        g.val2 = take(4 * (size_t)n);
        g.hist = take(4 * (size_t)kBins * (size_t)g.tiles);
        g.total = take(4 * (size_t)kBins);
    }
    g.part = take(sizeof(float) * 2 * (size_t)g.chunks * (size_t)g.dp);
    g.bytes = at;
    return g;
}

template <typename T, typename I>
cudaError_t lookup(const T* E, int64_t ld_e, int64_t V, int64_t d, const I* tok, int64_t n, float scale, T* out,
                   int64_t ld_out, cudaStream_t s) {
    const int al = row_align(E, ld_e, sizeof(T)), bl = row_align(out, ld_out, sizeof(T));
    int N = (int)((al < bl ? al : bl) / sizeof(T));
    while (d % N) N >>= 1;
    const int64_t nv = d / N;
    int lanes = 1;
    while (lanes < 32 && (int64_t)lanes * kLookVecs < nv) lanes <<= 1;
    const int64_t segs = (nv + lanes * kLookVecs - 1) / (lanes * kLookVecs);
    const int64_t per = kLookThreads / lanes;
    // at most 2^31 - 1 CTAs a launch: rows in pieces
    const int64_t most = (((int64_t)1 << 31) - 1) / segs * per;
    for (int64_t r0 = 0; r0 < n; r0 += most) {
        const int64_t m = n - r0 < most ? n - r0 : most, grid = (m * segs + per - 1) / per;
        note_launches(1);
#define TDA_LOOKUP(NN)                                                                                            \
    lookup_kernel<T, I, NN><<<(unsigned)grid, kLookThreads, 0, s>>>(E, ld_e, V, d, tok + r0, m, scale,            \
                                                                     out + r0 * ld_out, ld_out, lanes, segs)
        if (N * sizeof(T) == 16)
            TDA_LOOKUP(16 / sizeof(T));
        else if (N * sizeof(T) == 8)
            TDA_LOOKUP(8 / sizeof(T));
        else if (N * sizeof(T) == 4)
            TDA_LOOKUP(4 / sizeof(T));
        else
            TDA_LOOKUP(1);
#undef TDA_LOOKUP
        cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

template <typename I>
cudaError_t sort_tokens(const I* tok, int64_t n, int64_t V, const GradLayout& g, char* ws, cudaStream_t s) {
    uint32_t* skey = (uint32_t*)(ws + g.skey);
    int32_t* order = (int32_t*)(ws + g.order);
    if (n <= kRankMax) {
        note_launches(1);
        rank_kernel<I><<<(unsigned)((n + 31) / 32), kRankThreads, 0, s>>>(tok, (int)n, (uint32_t)V, skey, order);
        return cudaGetLastError();
    }
    int bits = 1;  // of the keys 0 .. V
    while (V >> bits) ++bits;
    const int passes = (bits + 8) / 9, width = (bits + passes - 1) / passes;
    uint32_t *hist = (uint32_t*)(ws + g.hist), *total = (uint32_t*)(ws + g.total);
    const uint32_t* kin = nullptr;
    const int32_t* vin = nullptr;
    for (int p = 0; p < passes; ++p) {
        // the last pass ends in skey, order
        const bool here = (passes - 1 - p) % 2 == 0;
        uint32_t* ko = here ? skey : (uint32_t*)(ws + g.key2);
        int32_t* vo = here ? order : (int32_t*)(ws + g.val2);
        const uint32_t mask = (1u << width) - 1;
        note_launches(3);
        digit_count_kernel<I><<<(unsigned)g.tiles, kSortThreads, 0, s>>>(tok, kin, (int)n, (uint32_t)V, p * width, mask,
                                                                        hist);
        digit_scan_kernel<<<mask + 1, kSortThreads, 0, s>>>(hist, (int)g.tiles, total);
        digit_scatter_kernel<I><<<(unsigned)g.tiles, kSortThreads, 0, s>>>(tok, kin, vin, (int)n, (uint32_t)V,
                                                                          p * width, mask, hist, total, ko, vo);
        cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
        kin = ko;
        vin = vo;
    }
    return cudaSuccess;
}

template <typename TI, typename TO>
cudaError_t sums(const TI* dout, int64_t ld_d, int64_t V, int64_t d, int64_t n, float scale, TO* dE, int64_t ld_e,
                 float beta, const GradLayout& g, char* ws, cudaStream_t s) {
    GradParams p;
    p.n = n, p.d = d, p.ld_d = ld_d, p.V = V, p.ld_e = ld_e, p.dp = g.dp;
    p.chunks = g.chunks, p.C = g.C, p.scale = scale, p.beta = beta;
    p.skey = (const uint32_t*)(ws + g.skey);
    p.order = (const int32_t*)(ws + g.order);
    p.part = (float*)(ws + g.part);
    const int ai = row_align(dout, ld_d, sizeof(TI)) / (int)sizeof(TI), ao = row_align(dE, ld_e, sizeof(TO));
    constexpr int kFull = 16 / sizeof(TI);
    auto fits = [&](int N) { return d % N == 0 && ai >= N && (size_t)ao >= (N * sizeof(TO) < 16 ? N * sizeof(TO) : 16); };
    const int N = fits(kFull) ? kFull : fits(2) ? 2 : 1;
    p.col_blocks = (d + (int64_t)kSumThreads * N - 1) / ((int64_t)kSumThreads * N);
    const int64_t zero = beta == 1.f ? 0 : (V + kZeroRows - 1) / kZeroRows;
    const int64_t grid = p.chunks * p.col_blocks + zero;
    if (grid > 0) {
        if (grid > 2147483647LL) return cudaErrorInvalidConfiguration;
        const size_t sm = 8 * (size_t)g.C;
        note_launches(1);
        if (N == kFull)
            grad_sum_kernel<TI, TO, kFull><<<(unsigned)grid, kSumThreads, sm, s>>>(dout, dE, p);
        else if (N == 2)
            grad_sum_kernel<TI, TO, 2><<<(unsigned)grid, kSumThreads, sm, s>>>(dout, dE, p);
        else
            grad_sum_kernel<TI, TO, 1><<<(unsigned)grid, kSumThreads, sm, s>>>(dout, dE, p);
        cudaError_t e = cudaGetLastError();
        if (e != cudaSuccess) return e;
    }
    if (p.chunks < 2) return cudaSuccess;
    int64_t cols = (d + kJoinThreads - 1) / kJoinThreads;
    note_launches(1);
    grad_join_kernel<TO><<<dim3((unsigned)(p.chunks - 1), (unsigned)(cols < 8 ? cols : 8)), kJoinThreads, 0, s>>>(dE, p);
    return cudaGetLastError();
}

}  // namespace

size_t embedding_workspace_bytes(int64_t d, int64_t n) { return n > 0 ? grad_layout(d, n).bytes : 0; }

cudaError_t launch_embedding_forward(tda_dtype dt, const void* E, int64_t ld_e, int64_t V, int64_t d,
                                     tda_index_type it, const void* tok, int64_t n, float scale, void* out,
                                     int64_t ld_out, cudaStream_t s) {
#define TDA_CALL(T, I) lookup((const T*)E, ld_e, V, d, (const I*)tok, n, scale, (T*)out, ld_out, s)
    if (dt == TDA_BF16) return it == TDA_I64 ? TDA_CALL(__nv_bfloat16, int64_t) : TDA_CALL(__nv_bfloat16, int32_t);
    return it == TDA_I64 ? TDA_CALL(float, int64_t) : TDA_CALL(float, int32_t);
#undef TDA_CALL
}

cudaError_t launch_embedding_backward(tda_dtype dt, const void* dout, int64_t ld_d, int64_t V, int64_t d,
                                      tda_index_type it, const void* tok, int64_t n, float scale, tda_dtype gt,
                                      void* dE, int64_t ld_e, float beta, void* ws, cudaStream_t s) {
    GradLayout g;
    if (n > 0) {
        g = grad_layout(d, n);
        cudaError_t e = it == TDA_I64 ? sort_tokens((const int64_t*)tok, n, V, g, (char*)ws, s)
                                      : sort_tokens((const int32_t*)tok, n, V, g, (char*)ws, s);
        if (e != cudaSuccess) return e;
    } else {  // no token: every row is cleared or scaled
        g = GradLayout{};
        g.C = 32;
    }
#define TDA_CALL(TI, TO) sums((const TI*)dout, ld_d, V, d, n, scale, (TO*)dE, ld_e, beta, g, (char*)ws, s)
    if (dt == TDA_BF16) return gt == TDA_BF16 ? TDA_CALL(__nv_bfloat16, __nv_bfloat16) : TDA_CALL(__nv_bfloat16, float);
    return TDA_CALL(float, float);
#undef TDA_CALL
}

}  // namespace tda
