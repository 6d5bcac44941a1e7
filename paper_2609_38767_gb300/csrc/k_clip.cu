// k_clip.cu -- the global norm of many gradient tensors and their clipping:
//   norm = sqrt(sum over tensors and elements of g^2),
//   out  = c g,  c = max_norm / norm if norm > max_norm, else 1.
//
// Two launches: the sums of squares (one partial per CTA, in a fixed order),
// then the scaling, whose CTAs each add the partials (at most 1280) up in the same
// fixed order (no counter to clear, no atomics: the result does not depend on
// timing). A launch takes up to 256 tensors; longer lists take several of each kind, and one CTA between them
// that adds all partials up once (else every scaling CTA of every launch would read them all: 65536
// tensors of 100 fp32 values 11.2 ms that way, 2.0 this; 2000 of 10000 119 us and 81). Both are bound by HBM. The bytes that must move are one read and one
// write of every element, plus a second read of what the L2 has dropped since
// the first; the scaling walks the tensors backwards, so it starts with what the
// sums read last, while that is still in the L2. 537M bf16 values (1.07 GB): 500 us,
// the sums 161 (6.7 TB/s), the scaling 325 (6.5 TB/s read and written); 2.6M fp32
// values, which stay in the L2: 10.4 us for both launches.
//
// Sums: a thread adds the squares of one chunk's elements (at most 32) in fp32,
// and the chunks' sums as an fp32 pair (the rounding error of each addition kept
// beside it); the pairs are added across the CTA in fp64. A thread whose
// chunk sum has left the range in which fp32 squares are exact enough (elements
// above about 1e14, or only such below 1e-14) squares that chunk again in fp64.
#include <cuda_bf16.h>

#include "tda_internal.cuh"

namespace tda {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 8192;  // elements per unit of work: 16 or 32 KiB
constexpr int kMaxTensors = 256;  // tensors of one launch: their table travels in the kernel's parameters (10.8 KB)

struct ClipTensor {
    const void* in;
    void* out;
    int64_t n;
    int64_t first;  // index of its first chunk, with bit 62 set for bf16
};
constexpr int64_t kBf16Bit = (int64_t)1 << 62;

constexpr int kMaxGrid = 1280;    // CTAs of one launch: eight per SM of 160
struct ClipTable {
    ClipTensor t[kMaxTensors];
    int32_t count;
    int64_t chunks;
    uint16_t first_of[kMaxGrid + 1];  // tensor that holds CTA b's first chunk; [b + 1]: about its last
};

__device__ __forceinline__ float2 two_sum(float a, float b) {
    const float s = __fadd_rn(a, b), bb = __fsub_rn(s, a);
    return make_float2(s, __fadd_rn(__fsub_rn(a, __fsub_rn(s, bb)), __fsub_rn(b, bb)));
}

struct Sum {
    float hi = 0.f, lo = 0.f;  // sum of squares of the ordinary chunks
    double wide = 0.0;         // of the chunks whose squares leave fp32's range
};

// Adds the squares of v[0..N): one chunk's elements of this thread.
template <int N>
__device__ __forceinline__ void add_squares(Sum& s, const float* v) {
    float q = 0.f, top = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        q = fmaf(v[i], v[i], q);
        top = fmaxf(top, fabsf(v[i]));
    }
    if (q < 1e30f && (q > 1e-28f || top == 0.f)) {
        const float2 r = two_sum(s.hi, q);
        s.hi = r.x;
        s.lo += r.y;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i) s.wide = fma((double)v[i], (double)v[i], s.wide);
    }
}

__device__ __forceinline__ void unpack(const uint4& r, float* v, const float*) {
    v[0] = __uint_as_float(r.x), v[1] = __uint_as_float(r.y), v[2] = __uint_as_float(r.z), v[3] = __uint_as_float(r.w);
}
__device__ __forceinline__ void unpack(const uint4& r, float* v, const __nv_bfloat16*) {
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        v[2 * i] = __uint_as_float(w[i] << 16);
        v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ uint4 pack(const float* v, const float*) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
}
__device__ __forceinline__ uint4 pack(const float* v, const __nv_bfloat16*) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_f(float x, float* p) { *p = x; }
__device__ __forceinline__ void from_f(float x, __nv_bfloat16* p) { *p = __float2bfloat16_rn(x); }

template <typename T>
__device__ __forceinline__ void chunk_squares(Sum& s, const T* g, int n) {
    constexpr int E = 16 / sizeof(T), kVecs = kChunk / E, kPer = kVecs / kThreads, U = kPer;
    if (n == kChunk && ((uintptr_t)g & 15) == 0) {
#pragma unroll
        for (int j = 0; j < kPer; j += U) {
            uint4 r[U];
#pragma unroll
            for (int u = 0; u < U; ++u) r[u] = __ldg((const uint4*)g + (j + u) * kThreads + threadIdx.x);
            float v[U * E];
#pragma unroll
            for (int u = 0; u < U; ++u) unpack(r[u], v + u * E, g);
            add_squares<U * E>(s, v);
        }
        return;
    }
    for (int i = threadIdx.x; i < n; i += 8 * kThreads) {  // a tensor's ragged end, or an unaligned one
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = i + u * kThreads < n ? to_f(g[i + u * kThreads]) : 0.f;
        add_squares<8>(s, v);
    }
}

// CTA b owns chunks [chunks b / grid, chunks (b+1) / grid).
__global__ void __launch_bounds__(kThreads) clip_squares_kernel(const __grid_constant__ ClipTable T, double* part) {
    chain_wait();
    chain_next();
    const int64_t c0 = T.chunks * blockIdx.x / gridDim.x, c1 = T.chunks * (blockIdx.x + 1) / gridDim.x;
    Sum s;
    int t = T.first_of[blockIdx.x];
    for (int64_t c = c0; c < c1; ++c) {
        while (t + 1 < T.count && (T.t[t + 1].first & ~kBf16Bit) <= c) ++t;
        const int64_t off = (c - (T.t[t].first & ~kBf16Bit)) * kChunk, left = T.t[t].n - off;
        const int n = left < kChunk ? (int)left : kChunk;
        if (T.t[t].first & kBf16Bit)
            chunk_squares(s, (const __nv_bfloat16*)T.t[t].in + off, n);
        else
            chunk_squares(s, (const float*)T.t[t].in + off, n);
    }
    double d = (double)s.hi + (double)s.lo + s.wide;
#pragma unroll
    for (int o = 16; o; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
    __shared__ double w[kThreads / 32];
    if ((threadIdx.x & 31) == 0) w[threadIdx.x >> 5] = d;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < kThreads / 32; ++i) d += w[i];
        part[blockIdx.x] = d;
    }
}

// The sum of the partials in a fixed order, complete in thread 0.
__device__ __forceinline__ double sum_partials(const double* part, int n_part) {
    double d = 0.0;
    for (int i = threadIdx.x; i < n_part; i += kThreads) d += part[i];
#pragma unroll
    for (int o = 16; o; o >>= 1) d += __shfl_xor_sync(0xffffffffu, d, o);
    __shared__ double w[kThreads / 32];
    if ((threadIdx.x & 31) == 0) w[threadIdx.x >> 5] = d;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int i = 1; i < kThreads / 32; ++i) d += w[i];
    return d;
}

// Several launches of clip_squares_kernel: all their partials added up into part[0].
__global__ void __launch_bounds__(kThreads) clip_total_kernel(double* part, int n_part) {
    chain_wait();
    chain_next();
    const double d = sum_partials(part, n_part);
    if (threadIdx.x == 0) part[0] = d;
}

// A whole, aligned chunk's share of a thread: 4 (bf16) or 8 accesses of 16 bytes.
template <typename T>
constexpr int kPieces = kChunk * (int)sizeof(T) / 16 / kThreads;

template <typename T>
__device__ __forceinline__ void chunk_load(const T* g, uint4* r) {
#pragma unroll
    for (int u = 0; u < kPieces<T>; ++u) r[u] = __ldcs((const uint4*)g + u * kThreads + threadIdx.x);
}
template <typename T>
__device__ __forceinline__ void chunk_store(T* out, const uint4* r, float c) {
    constexpr int E = 16 / sizeof(T);
#pragma unroll
    for (int u = 0; u < kPieces<T>; ++u) {
        float v[E];
        unpack(r[u], v, out);
#pragma unroll
        for (int e = 0; e < E; ++e) v[e] *= c;
        __stcs((uint4*)out + u * kThreads + threadIdx.x, pack(v, out));
    }
}
// A ragged end, or a tensor that is not aligned.
template <typename T>
__device__ __forceinline__ void chunk_scale(const T* g, T* out, int n, float c) {
    for (int i = threadIdx.x; i < n; i += 8 * kThreads) {
        float v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = i + u * kThreads < n ? to_f(g[i + u * kThreads]) : 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (i + u * kThreads < n) from_f(v[u] * c, out + i + u * kThreads);
    }
}

// n_part partials of one launch of clip_squares_kernel, or the one that clip_total_kernel left. norm_out, where it is
// given (in the first of several launches), is written by the first CTA.
__global__ void __launch_bounds__(kThreads)
clip_scale_kernel(const __grid_constant__ ClipTable T, const double* part, int n_part, float max_norm, float* norm_out) {
    const int64_t c0 = T.chunks * blockIdx.x / gridDim.x, c1 = T.chunks * (blockIdx.x + 1) / gridDim.x;
    int t = T.first_of[blockIdx.x + 1];  // the next CTA's first tensor: this CTA's last one or the one after it
    // chunk k: its tensor, elements, and whether it goes by whole accesses
    auto find = [&](int64_t k, const ClipTensor** x, int64_t* off, int* n) {
        while (t > 0 && (T.t[t].first & ~kBf16Bit) > k) --t;
        *x = &T.t[t];
        *off = (k - (T.t[t].first & ~kBf16Bit)) * kChunk;
        const int64_t left = T.t[t].n - *off;
        *n = left < kChunk ? (int)left : kChunk;
        return *n == kChunk && (((uintptr_t)T.t[t].in | (uintptr_t)T.t[t].out) & 15) == 0;
    };
    const ClipTensor* x = nullptr;
    int64_t off = 0;
    int n = 0;
    uint4 r[kPieces<float>];
    auto load = [&]() {
        if (x->first & kBf16Bit)
            chunk_load((const __nv_bfloat16*)x->in + off, r);
        else
            chunk_load((const float*)x->in + off, r);
    };
    // The first chunk is read while the sums are still being taken, which write none of it (nor does any CTA here
    // write another's chunks).
    bool whole = false;
    if (c1 > c0 && (whole = find(c1 - 1, &x, &off, &n))) load();
    chain_wait();
    chain_next();
    const double d = sum_partials(part, n_part);
    __shared__ float coef;
    if (threadIdx.x == 0) {
        // fp32 where the sum is an fp32 number (an fp64 root and quotient take a microsecond on these SMs);
        // a NaN norm is not <= max_norm and passes into every output
        float norm;
        if (d > 1e-30 && d < 1e30) {
            norm = sqrtf((float)d);
            coef = norm <= max_norm ? 1.f : max_norm / norm;
        } else {
            const double exact = sqrt(d);
            norm = (float)exact;
            coef = exact <= (double)max_norm ? 1.f : (float)((double)max_norm / exact);
        }
        if (norm_out && blockIdx.x == 0) *norm_out = norm;
    }
    __syncthreads();
    const float c = coef;
    for (int64_t k = c1 - 1; k >= c0; --k) {
        if (k < c1 - 1) whole = find(k, &x, &off, &n);
        if (!x->out || (c == 1.f && x->out == x->in)) continue;  // norm only, or nothing changes in place
        if (whole) {
            if (k < c1 - 1) load();
            if (x->first & kBf16Bit)
                chunk_store((__nv_bfloat16*)x->out + off, r, c);
            else
                chunk_store((float*)x->out + off, r, c);
        } else if (x->first & kBf16Bit) {
            chunk_scale((const __nv_bfloat16*)x->in + off, (__nv_bfloat16*)x->out + off, n, c);
        } else {
            chunk_scale((const float*)x->in + off, (float*)x->out + off, n, c);
        }
    }
}

// Fills the table with tensors from *i on (empty ones left out) for at most `most` CTAs; false when none is left.
bool next_table(const tda_tensor_ref* list, int64_t n_tensors, int64_t* i, int64_t most, ClipTable* T, int64_t* grid) {
    T->count = 0;
    T->chunks = 0;
    for (; *i < n_tensors && T->count < kMaxTensors; ++*i) {
        const tda_tensor_ref& r = list[*i];
        if (r.n == 0) continue;
        ClipTensor& t = T->t[T->count++];
        t.in = r.in;
        t.out = r.out;
        t.n = r.n;
        t.first = T->chunks | (r.dtype == TDA_BF16 ? kBf16Bit : 0);
        T->chunks += (r.n + kChunk - 1) / kChunk;
    }
    *grid = T->chunks < 1 ? 1 : T->chunks < most ? T->chunks : most;
    // CTA b starts at chunk floor(chunks b / grid)
    const int64_t step = T->chunks / *grid, rem = T->chunks % *grid;
    int t = 0;
    for (int64_t b = 0, c = 0, over = 0; b <= *grid; ++b, c += step, over += rem) {
        if (over >= *grid) over -= *grid, ++c;
        while (t + 1 < T->count && (T->t[t + 1].first & ~kBf16Bit) <= c) ++t;
        T->first_of[b] = (uint16_t)t;
    }
    return T->count > 0;
}

}  // namespace

constexpr int kClipCtasPerSm = 8;  // enough to fill an SM

size_t clip_workspace_bytes(int64_t n_tensors) {
    const int64_t tables = (n_tensors + kMaxTensors - 1) / kMaxTensors;
    return sizeof(double) * (size_t)(kMaxGrid * (tables > 1 ? tables : 1));
}

cudaError_t launch_grad_clip(const tda_tensor_ref* list, int64_t n_tensors, float max_norm, float* norm, double* part,
                             cudaStream_t s) {
    int64_t most = (int64_t)train_sms() * kClipCtasPerSm, grid;
    if (most > kMaxGrid) most = kMaxGrid;
    ClipTable T;
    int n_part = 0, tables = 0;
    for (int64_t i = 0; next_table(list, n_tensors, &i, most, &T, &grid); ++tables) {
        cudaError_t e = launch_chained(tables > 0, clip_squares_kernel, dim3((unsigned)grid), dim3(kThreads), 0, s, T,
                                       part + n_part);
        if (e != cudaSuccess) return e;
        n_part += (int)grid;
        if (i == n_tensors && tables == 0) {  // one table: it serves the scaling as well
            return launch_chained(true, clip_scale_kernel, dim3((unsigned)grid), dim3(kThreads), 0, s, T, part, n_part,
                                  max_norm, norm);
        }
    }
    if (tables > 1) {
        const cudaError_t e = launch_chained(true, clip_total_kernel, dim3(1), dim3(kThreads), 0, s, part, n_part);
        if (e != cudaSuccess) return e;
        n_part = 1;
    }
    int64_t i = 0;
    for (int k = 0; k < tables || k == 0; ++k) {  // without a tensor: one CTA, for the norm
        next_table(list, n_tensors, &i, most, &T, &grid);
        cudaError_t e = launch_chained(tables > 0, clip_scale_kernel, dim3((unsigned)grid), dim3(kThreads), 0, s, T, part,
                                       n_part, max_norm, k == 0 ? norm : nullptr);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace tda
