// k_embedding.cu -- embedding lookup with scaling, and its gradient.
//
// Lookup: out[i] = scale E[t_i]; a padded token (t_i < 0) gives a zero row, an
// id outside the table (t_i >= V) a NaN row, so that it is seen. Bound by HBM:
// the rows read plus the rows written. A group of lanes copies up to four
// 16-byte vectors per lane of one row (more of the narrower ones that rows of
// other alignments take), all loads before the first store. 32768 rows of
// 4096 bf16 values from a table of 131072 (365 MB in all): 62 us = 5.9 TB/s (in
// CTAs of 256 threads 64, of 512 with half the vectors 73).
//
// Gradient: dE[v] = beta dE[v] + scale sum_{i : t_i = v} dOut[i]. The positions
// are sorted by (token, position), the sorted list is cut into chunks of equal
// length, and each chunk adds its rows up in that order, so hot tokens are
// spread over the GPU and the sums do not depend on timing. A token whose run
// lies inside one chunk is finished there; a run that crosses a chunk's edge
// leaves one fp32 partial row per chunk, and a last launch adds a run's partials
// in order. Rows of E that no token names are cleared (or scaled by beta) by
// further CTAs: of the sums' launch, or, for short lists, of the sort's. Bound by
// HBM: n rows read, V rows written. Sums are fp32, rounded once to dE's type.
// 65536 rows into 131072 x 4096 bf16 (1.6 GB): 273 us = 5.9 TB/s; 4096 rows into
// 32000 x 2048 fp32 (279 MB): 52 us = 5.4 TB/s, the clearing alone 38.
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
constexpr int kLookThreads = 128;
// Vectors of `bytes` each that a lane moves: enough bytes in flight for rows of any alignment (20000 rows of 1001 bf16
// values: 4 vectors 36 us, 8 26, 16 22; of 1001 fp32 values 36, 26, 22; 30000 of 3004 bf16 values 56, 53, 80).
constexpr int look_vecs(int bytes) { return bytes == 16 ? 4 : bytes == 8 ? 8 : 16; }

// lanes (a power of two <= 32) copy one segment of lanes * kVecs vectors of a row.
template <typename T, typename I, int N>
__global__ void __launch_bounds__(kLookThreads)
lookup_kernel(const T* __restrict__ E, int64_t ld_e, int64_t V, int64_t d, const I* __restrict__ tok, int64_t n,
              float scale, T* __restrict__ out, int64_t ld_out, int lanes, int64_t segs) {
    constexpr int kVecs = look_vecs(N * (int)sizeof(T));
    const int64_t g = ((int64_t)blockIdx.x * kLookThreads + threadIdx.x) / lanes;
    const int64_t row = g / segs;
    if (row >= n) return;
    const int64_t v0 = (g % segs) * lanes * kVecs + threadIdx.x % lanes, nv = d / N;
    const I t = tok[row];
    const bool in = t >= 0 && (uint64_t)t < (uint64_t)V;
    Vec<T, N> x[kVecs];
    if (in) {
        const Vec<T, N>* src = reinterpret_cast<const Vec<T, N>*>(E + (int64_t)t * ld_e);
#pragma unroll
        for (int j = 0; j < kVecs; ++j)
            if (v0 + j * lanes < nv) x[j] = src[v0 + j * lanes];
    }
    Vec<T, N>* dst = reinterpret_cast<Vec<T, N>*>(out + row * ld_out);
    const float fill = t < 0 ? 0.f : __int_as_float(0x7fc00000);
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
        if (v0 + j * lanes >= nv) break;
        Vec<T, N> y;
#pragma unroll
        for (int e = 0; e < N; ++e) set_f(&y.v[e], in ? to_f(x[j].v[e]) * scale : fill);
        dst[v0 + j * lanes] = y;
    }
}

// ------------------------------------------------------------------ sort by (token, position)
// Up to kRankMax tokens: the place of token i in the sorted list is the number of tokens before it,
// #{j < i : k_j <= k_i} + #{j > i : k_j < k_i}, counted directly: one launch, n^2 comparisons over all SMs
// (4096 tokens 7 us, where the radix sort below takes six launches and about 25).
constexpr int kRankMax = 8192, kRankThreads = 256;

//
// With `clear` set the launch also zeroes the gradient's rows, all of them, beside the counting: the few
// that tokens name are written twice, but no row waits for the sorted list (85 tokens of 69041 x 256 fp32 19 us; 24
// with a whole CTA at each row).
struct ClearParams {
    uint4* p;          // NULL: nothing to clear; rows 16-byte aligned, whole 16-byte vectors
    int64_t rows, vecs, ld;  // vectors of a row, row stride in vectors
    int log_lanes;           // threads of a row, as a power of two: short rows are cleared several at a time
};
constexpr int kClearRows = 16;

template <typename I>
__global__ void __launch_bounds__(kRankThreads)
rank_kernel(const I* __restrict__ tok, int n, uint32_t V, uint32_t* __restrict__ skey, int32_t* __restrict__ order,
            int ctas, const ClearParams clear) {
    if ((int)blockIdx.x >= ctas) {
        chain_next();
        const int64_t r0 = (int64_t)((int)blockIdx.x - ctas) * kClearRows;
        const int ll = clear.log_lanes, lanes = 1 << ll;
        for (int64_t r = r0 + (threadIdx.x >> ll); r < r0 + kClearRows && r < clear.rows; r += kRankThreads >> ll)
            for (int64_t c = threadIdx.x & (lanes - 1); c < clear.vecs; c += lanes)
                clear.p[r * clear.ld + c] = make_uint4(0, 0, 0, 0);
        return;
    }
    __shared__ alignas(16) uint32_t key[kRankMax];
    __shared__ int cnt[kRankThreads / 32][32];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int np = (n + 31) & ~31;
    chain_next();
#pragma unroll 8
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

// The kernels from here on start while the launch before them still runs (chain_wait): nothing that it writes may be
// __restrict__ in them, which would let the compiler read it ahead of the wait. The call's own inputs may be.
//
// More tokens: a stable radix sort from the low digit up, digits of at most 9 bits (2 passes up to 2^18 ids),
// three launches a pass: digit counts per tile, their scan per digit, the scatter.
// Tiles are small, so that a list of some ten thousand tokens still spreads over the SMs.
constexpr int kTile = 512, kSortThreads = 256, kBins = 512, kRounds = kTile / kSortThreads;

template <typename I>
__global__ void __launch_bounds__(kSortThreads)
digit_count_kernel(const I* __restrict__ tok, const uint32_t* key, int n, uint32_t V, int shift,
                   uint32_t mask, uint32_t* hist) {
    __shared__ uint32_t h[kBins];
    chain_wait();
    chain_next();
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
__global__ void __launch_bounds__(kSortThreads) digit_scan_kernel(uint32_t* hist, int tiles, uint32_t* total) {
    __shared__ uint32_t w[kSortThreads / 32];
    chain_wait();
    chain_next();
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
digit_scatter_kernel(const I* __restrict__ tok, const uint32_t* key, const int32_t* val, int n, uint32_t V, int shift,
                     uint32_t mask, const uint32_t* hist, const uint32_t* total, uint32_t* key_out, int32_t* val_out) {
    constexpr int W = kSortThreads / 32, kPer = kTile / W / 32;
    __shared__ uint32_t pos[W][kBins];  // counts of each warp's run, then the next place of each digit
    __shared__ uint32_t start[kBins];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    chain_wait();
    chain_next();
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
// kZeroRows: rows that a clearing CTA looks up and clears (8, 16, 32: 318, 323, 335 us for the large case above, then).
// kBatch: rows whose loads are in flight per thread, kSumCtas: CTAs meant for an SM, which caps the registers. Eight
// rows in 64 registers spilled (313 us); four rows and nine CTAs run without (274; 8 CTAs 277, 12 331; three rows
// and ten CTAs 275, two rows and twelve 283).
constexpr int kSumThreads = 128, kBatch = 4, kZeroRows = 8, kSumCtas = 9;

struct GradParams {
    int64_t n, d, ld_d, V, ld_e, dp;  // dp: row length of the partials
    int64_t chunks, col_blocks;
    int C;
    int quads;  // rows of dE may be moved four values at a time
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
__global__ void __launch_bounds__(kSumThreads, kSumCtas)
grad_sum_kernel(const TI* __restrict__ dout, TO* dE, const GradParams p) {
    chain_wait();
    chain_next();
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
            constexpr int kZ = N == 1 ? 1 : N == 2 ? 2 : 16 / sizeof(TO);  // 16 bytes, neighbours side by side
            for (int64_t c = (int64_t)threadIdx.x * kZ; c < p.d; c += kSumThreads * kZ) {
                const float zero[kZ] = {};
                store_row<TO, kZ>(row + c, zero, 0.f, p.beta);
            }
        }
        return;
    }
    // For each position of the chunk: where its row is, and, if a run ends there, where the sum goes: a row of
    // dE or a row of partials (byte offsets).
    extern __shared__ int64_t sm[];
    int64_t* dst = sm;                             // [C]
    int32_t* pos = (int32_t*)(sm + p.C);           // [C]
    uint32_t* key = (uint32_t*)(pos + p.C);        // [C]
    uint8_t* end = (uint8_t*)(key + p.C);          // [C]: 0 the run goes on, 1 ends in dE, 2 in partials
    const int64_t ch = (int64_t)blockIdx.x / p.col_blocks, i0 = ch * p.C;
    const int64_t col = ((int64_t)blockIdx.x % p.col_blocks) * kSumThreads * N + (int64_t)threadIdx.x * N;
    const int in = p.n - i0 < p.C ? (int)(p.n - i0) : p.C;
    const uint32_t none = (uint32_t)p.V;
    const uint32_t prev = i0 > 0 ? p.skey[i0 - 1] : none, next = i0 + p.C < p.n ? p.skey[i0 + p.C] : none;
    for (int i = threadIdx.x; i < in; i += kSumThreads) {
        key[i] = p.skey[i0 + i];
        pos[i] = p.order[i0 + i];
    }
    __syncthreads();
    int live = 0;
    for (int i = threadIdx.x; i < in; i += kSumThreads) {
        const uint32_t k = key[i];
        const bool last = i + 1 == in || key[i + 1] != k;
        end[i] = 0;
        if (last) {
            // the first run of the chunk may have begun before it, the last one may go on after it
            const bool head = key[0] == k && k == prev, tail = i + 1 == p.C && k == next;
            end[i] = head || tail ? 2 : 1;
            dst[i] = head ? 2 * ch * p.dp : tail ? (2 * ch + 1) * p.dp : (int64_t)k * p.ld_e;
        }
        live += k != none;
    }
    const int have = [&] {  // ids outside the table come last and are left out
        int c = live;
#pragma unroll
        for (int o = 16; o; o >>= 1) c += __shfl_xor_sync(0xffffffffu, c, o);
        __shared__ int w[kSumThreads / 32];
        if ((threadIdx.x & 31) == 0) w[threadIdx.x >> 5] = c;
        __syncthreads();
        c = 0;
#pragma unroll
        for (int i = 0; i < kSumThreads / 32; ++i) c += w[i];
        return c;
    }();
    if (col >= p.d) return;
    float acc[N] = {};
    const TI* src = dout + col;
    TO* out = dE + col;
    float* part = p.part + col;
    for (int i = 0; i < have; i += kBatch) {
        Vec<TI, N> x[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u)
            if (i + u < have) x[u] = *reinterpret_cast<const Vec<TI, N>*>(src + (int64_t)pos[i + u] * p.ld_d);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            if (i + u >= have) break;
#pragma unroll
            for (int e = 0; e < N; ++e) acc[e] += to_f(x[u].v[e]);
            if (const int f = end[i + u]) {
                if (f == 1)
                    store_row<TO, N>(out + dst[i + u], acc, p.scale, p.beta);
                else
                    store_row<float, N>(part + dst[i + u], acc, 1.f, 0.f);
#pragma unroll
                for (int e = 0; e < N; ++e) acc[e] = 0.f;
            }
        }
    }
}

// A run that crosses chunk edges: the CTA of the chunk where it starts adds its partials in order.
constexpr int kJoinThreads = 256, kJoinWarps = kJoinThreads / 32;

// Four columns of a finished sum to dE.
template <typename TO>
__device__ __forceinline__ void store_join(const GradParams& p, TO* dE, uint32_t k, int64_t col, const float4& a) {
    const float v[4] = {a.x, a.y, a.z, a.w};
    TO* q = dE + (int64_t)k * p.ld_e + col;
    if (p.quads && col + 4 <= p.d) {
        store_row<TO, 4>(q, v, p.scale, p.beta);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (col + i < p.d) store_row<TO, 1>(q + i, v + i, p.scale, p.beta);
    }
}

// CTA (x, y): the runs that start in kJoinChunks chunks, 128 columns of them (4 a lane). A warp looks through
// each chunk; then each warp takes a run of its own, or all of them share a long one.
constexpr int kJoinChunks = kJoinWarps;

template <typename TO>
__global__ void __launch_bounds__(kJoinThreads) grad_join_kernel(TO* dE, const GradParams p) {
    chain_wait();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t none = (uint32_t)p.V;
    __shared__ int parts_of[kJoinChunks];  // 0: no run starts in the chunk and leaves it
    __shared__ uint32_t key_of[kJoinChunks];
    const int64_t ch0 = (int64_t)blockIdx.x * kJoinChunks;
    if (const int64_t ch = ch0 + warp; warp < kJoinChunks) {
        const int64_t i0 = ch * p.C, i1 = i0 + p.C;
        int parts = 0;
        uint32_t k = none;
        if (ch + 1 < p.chunks) {
            k = p.skey[i1 - 1];
            const uint32_t after = p.skey[i1], before = i0 > 0 ? p.skey[i0 - 1] : none;
            if (k != none && after == k && before != k) {
                // the chunks after ch whose first key is k, 32 at a time
                parts = 1;
                for (int64_t c = ch + 1;; c += 32) {
                    const uint32_t other = ~__ballot_sync(0xffffffffu, c + lane < p.chunks && p.skey[(c + lane) * p.C] == k);
                    parts += other ? __ffs(other) - 1 : 32;
                    if (other) break;
                }
            }
        }
        if (lane == 0) {
            parts_of[warp] = parts;
            key_of[warp] = k;
        }
    }
    __syncthreads();
    const int64_t col = (int64_t)blockIdx.y * 128 + lane * 4;
    // partial 0 of a run is the tail of its first chunk, partial j the head of the j-th after it; rows of partials
    // are padded to a multiple of 8 columns. Eight loads ahead, additions in order.
    auto add = [&](int64_t ch, int j0, int j1) {
        const float* base = p.part + 2 * ch * p.dp + col;
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
        if (col >= p.d) return a;
        for (int j = j0; j < j1; j += 8) {
            float4 x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (j + u < j1) x[u] = *reinterpret_cast<const float4*>(base + (2 * (int64_t)(j + u) + (j + u == 0)) * p.dp);
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) a.x += x[u].x, a.y += x[u].y, a.z += x[u].z, a.w += x[u].w;
        }
        return a;
    };
    constexpr int kLong = 2 * kJoinWarps;  // partials from which a run is shared (4 x: 275 us, 2 x: 273)
    int seen = 0;
    for (int c = 0; c < kJoinChunks; ++c) {
        const int parts = parts_of[c];
        if (parts == 0 || parts >= kLong) continue;
        if (seen++ % kJoinWarps != warp) continue;
        const float4 a = add(ch0 + c, 0, parts);
        if (col < p.d) store_join(p, dE, key_of[c], col, a);
    }
    __shared__ float4 sh[kJoinWarps][32];
    for (int c = 0; c < kJoinChunks; ++c) {
        const int parts = parts_of[c];
        if (parts < kLong) continue;
        float4 a = add(ch0 + c, (int)((int64_t)parts * warp / kJoinWarps), (int)((int64_t)parts * (warp + 1) / kJoinWarps));
        sh[warp][lane] = a;
        __syncthreads();
        if (warp == 0 && col < p.d) {
#pragma unroll
            for (int w = 1; w < kJoinWarps; ++w)
                a.x += sh[w][lane].x, a.y += sh[w][lane].y, a.z += sh[w][lane].z, a.w += sh[w][lane].w;
            store_join(p, dE, key_of[c], col, a);
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
    g.C = n <= 8192 ? 16 : n <= 16384 ? 32 : n <= 131072 ? 64 : 256;
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
    const int vecs = look_vecs(N * (int)sizeof(T));
    int lanes = 1;
    while (lanes < 32 && (int64_t)lanes * vecs < nv) lanes <<= 1;
    const int64_t segs = (nv + lanes * vecs - 1) / (lanes * vecs);
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
cudaError_t sort_tokens(const I* tok, int64_t n, int64_t V, const GradLayout& g, const ClearParams& clear, char* ws,
                        cudaStream_t s) {
    uint32_t* skey = (uint32_t*)(ws + g.skey);
    int32_t* order = (int32_t*)(ws + g.order);
    if (n <= kRankMax) {
        const int64_t ctas = (n + 31) / 32, more = clear.p ? (clear.rows + kClearRows - 1) / kClearRows : 0;
        return launch_chained(false, rank_kernel<I>, dim3((unsigned)(ctas + more)), dim3(kRankThreads), 0, s, tok, (int)n,
                              (uint32_t)V, skey, order, (int)ctas, clear);
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
        const dim3 tiles((unsigned)g.tiles), block(kSortThreads);
        cudaError_t e = launch_chained(p > 0, digit_count_kernel<I>, tiles, block, 0, s, tok, kin, (int)n, (uint32_t)V,
                                       p * width, mask, hist);
        if (e != cudaSuccess) return e;
        e = launch_chained(true, digit_scan_kernel, dim3(mask + 1), block, 0, s, hist, (int)g.tiles, total);
        if (e != cudaSuccess) return e;
        e = launch_chained(true, digit_scatter_kernel<I>, tiles, block, 0, s, tok, kin, vin, (int)n, (uint32_t)V, p * width,
                           mask, hist, total, ko, vo);
        if (e != cudaSuccess) return e;
        kin = ko;
        vin = vo;
    }
    return cudaSuccess;
}

template <typename TI, typename TO>
cudaError_t sums(const TI* dout, int64_t ld_d, int64_t V, int64_t d, int64_t n, float scale, TO* dE, int64_t ld_e,
                 float beta, bool cleared, const GradLayout& g, char* ws, cudaStream_t s) {
    GradParams p;
    p.n = n, p.d = d, p.ld_d = ld_d, p.V = V, p.ld_e = ld_e, p.dp = g.dp;
    p.chunks = g.chunks, p.C = g.C, p.scale = scale, p.beta = beta;
    p.skey = (const uint32_t*)(ws + g.skey);
    p.order = (const int32_t*)(ws + g.order);
    p.part = (float*)(ws + g.part);
    const int ai = row_align(dout, ld_d, sizeof(TI)) / (int)sizeof(TI), ao = row_align(dE, ld_e, sizeof(TO));
    constexpr int kFull = 16 / sizeof(TI);
    auto fits = [&](int N) { return d % N == 0 && ai >= N && (size_t)ao >= (N * sizeof(TO) < 16 ? N * sizeof(TO) : 16); };
    p.quads = ao >= (int)(4 * sizeof(TO));
    const int N = fits(kFull) ? kFull : fits(2) ? 2 : 1;
    p.col_blocks = (d + (int64_t)kSumThreads * N - 1) / ((int64_t)kSumThreads * N);
    const int64_t zero = beta == 1.f || cleared ? 0 : (V + kZeroRows - 1) / kZeroRows;
    const int64_t grid = p.chunks * p.col_blocks + zero;
    if (grid > 0) {
        if (grid > 2147483647LL) return cudaErrorInvalidConfiguration;
        const auto kernel = N == kFull ? grad_sum_kernel<TI, TO, kFull>
                            : N == 2   ? grad_sum_kernel<TI, TO, 2>
                                       : grad_sum_kernel<TI, TO, 1>;
        cudaError_t e = launch_chained(n > 0, kernel, dim3((unsigned)grid), dim3(kSumThreads), 17 * (size_t)g.C, s, dout,
                                       dE, p);
        if (e != cudaSuccess) return e;
    }
    if (p.chunks < 2) return cudaSuccess;
    const dim3 grid2((unsigned)((p.chunks - 1 + kJoinChunks - 1) / kJoinChunks), (unsigned)((d + 127) / 128));
    return launch_chained(true, grad_join_kernel<TO>, grid2, dim3(kJoinThreads), 0, s, dE, p);
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
    GradLayout g = {};
    g.C = 32;
    ClearParams clear = {};
    if (n > 0) {
        g = grad_layout(d, n);
        const size_t el = gt == TDA_BF16 ? 2 : 4;
        if (beta == 0.f && n <= kRankMax && d * el % 16 == 0 && row_align(dE, ld_e, el) == 16) {
            clear.p = (uint4*)dE;
            clear.rows = V;
            clear.vecs = d * (int64_t)el / 16;
            clear.ld = ld_e * (int64_t)el / 16;
            clear.log_lanes = 0;
            while ((1 << clear.log_lanes) < kRankThreads && (1 << clear.log_lanes) < clear.vecs) ++clear.log_lanes;
        }
        cudaError_t e = it == TDA_I64 ? sort_tokens((const int64_t*)tok, n, V, g, clear, (char*)ws, s)
                                      : sort_tokens((const int32_t*)tok, n, V, g, clear, (char*)ws, s);
        if (e != cudaSuccess) return e;
    }
#define TDA_CALL(TI, TO) \
    sums((const TI*)dout, ld_d, V, d, n, scale, (TO*)dE, ld_e, beta, clear.p != nullptr, g, (char*)ws, s)
    if (dt == TDA_BF16) return gt == TDA_BF16 ? TDA_CALL(__nv_bfloat16, __nv_bfloat16) : TDA_CALL(__nv_bfloat16, float);
    return TDA_CALL(float, float);
#undef TDA_CALL
}

}  // namespace tda
