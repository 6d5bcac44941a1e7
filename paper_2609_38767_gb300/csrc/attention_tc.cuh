// attention_tc.cuh -- what the tensor-core kernels of the attention share: MMAs with an operand in TMEM, wide TMEM
// loads and stores, exponentials, pairs of fp32, tensor maps of heads. Included inside namespace tda::{anonymous},
// after tc_ptx.cuh.
#pragma once

constexpr int kTileT = 128;                      // tokens of a tile
constexpr uint32_t kPanel = kTileT * 128;        // 128 tokens x 64 values: 16 KiB
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Shared-memory descriptors, 128-byte swizzle, of `panel` bytes per 64 values of a head. K-major: 8-row groups 1 KiB apart;
// MN-major: the panels are the 64-value atoms (LBO), 8-row groups of k 1 KiB apart (SBO).
__device__ __forceinline__ uint64_t k_major(uint32_t saddr) { return sw128_desc(saddr); }
__device__ __forceinline__ uint64_t mn_major(uint32_t saddr, uint32_t panel) {
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(panel >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) |
           ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
constexpr uint32_t kBMn = 1u << 16;  // instruction descriptor: B is MN-major

__device__ __forceinline__ uint32_t elect_one() {
    uint32_t r;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(r));
    return r;
}
// Issued by the elected lane of a converged warp. A and B in shared memory, or A in TMEM (a row per lane, two bf16 a column).
__device__ __forceinline__ void mma_ss(uint32_t lead, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %5, 0;\n"
        " @q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(lead)
        : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t lead, uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    asm volatile(
        "{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %5, 0;\n"
        " @q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"(acc), "r"(lead)
        : "memory");
}
__device__ __forceinline__ void commit(uint32_t lead, uint32_t bar) {
    asm volatile(
        "{\n .reg .pred q;\n setp.ne.b32 q, %1, 0;\n"
        " @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar),
        "r"(lead)
        : "memory");
}
// D = A B^T over the head: A and B tiles of panels, K-major, `steps` of HD / 16 steps. The descriptors are a base and constants: the
// issuing warp must keep ahead of the tensor pipe, which takes 64 cycles a step.
template <int HD>
__device__ __forceinline__ void mma_heads(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, int steps) {
    const uint64_t da = k_major(a), db = k_major(b);
#pragma unroll
    for (int k = 0; k < HD / 16; ++k)
        if (k < steps) mma_ss(lead, d, da + ((k / 4 * kPanel + k % 4 * 32) >> 4), db + ((k / 4 * kPanel + k % 4 * 32) >> 4), idesc, k > 0);
}
// 32 lanes x 32 columns into registers; nothing may use them before tmem_wait_ld and tmem_use.
__device__ __forceinline__ void tmem_ld32(uint32_t t, float* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,"
        "%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=f"(r[0]), "=f"(r[1]), "=f"(r[2]), "=f"(r[3]), "=f"(r[4]), "=f"(r[5]), "=f"(r[6]), "=f"(r[7]), "=f"(r[8]), "=f"(r[9]),
          "=f"(r[10]), "=f"(r[11]), "=f"(r[12]), "=f"(r[13]), "=f"(r[14]), "=f"(r[15]), "=f"(r[16]), "=f"(r[17]), "=f"(r[18]),
          "=f"(r[19]), "=f"(r[20]), "=f"(r[21]), "=f"(r[22]), "=f"(r[23]), "=f"(r[24]), "=f"(r[25]), "=f"(r[26]), "=f"(r[27]),
          "=f"(r[28]), "=f"(r[29]), "=f"(r[30]), "=f"(r[31])
        : "r"(t)
        : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// Ties 32 loaded registers to what precedes: no use of them moves before it.
__device__ __forceinline__ void tmem_use(float* r) {
    asm volatile(""
                 : "+f"(r[0]), "+f"(r[1]), "+f"(r[2]), "+f"(r[3]), "+f"(r[4]), "+f"(r[5]), "+f"(r[6]), "+f"(r[7]), "+f"(r[8]),
                   "+f"(r[9]), "+f"(r[10]), "+f"(r[11]), "+f"(r[12]), "+f"(r[13]), "+f"(r[14]), "+f"(r[15]), "+f"(r[16]),
                   "+f"(r[17]), "+f"(r[18]), "+f"(r[19]), "+f"(r[20]), "+f"(r[21]), "+f"(r[22]), "+f"(r[23]), "+f"(r[24]),
                   "+f"(r[25]), "+f"(r[26]), "+f"(r[27]), "+f"(r[28]), "+f"(r[29]), "+f"(r[30]), "+f"(r[31])::"memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t t, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
        "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(t),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]),
        "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]),
        "r"(r[31])
        : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t t, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(t),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// 2^x to 2^-22 of its value, 1 / x to 2^-23.
__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp_fast(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c);
__device__ __forceinline__ float2 mul2(float2 a, float2 b);
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
// What a dot product is of the cap; held finite, as 0 times it is 0 however small the cap.
__device__ __forceinline__ float over_cap(const Attention& a) { return a.cap > 0.f ? fminf(a.scale / a.cap, FLT_MAX) : 0.f; }
// d P(d^2) for two dot products within a.near_limit, |x| <= 1/2: tanh to a relative error of 2^-23.1 (the fit is in
// attention_near), five instructions a pair and the caller's product with d. Any x: 1 - 2 / (1 + e^2x), right at both
// infinities, 2^-22 absolute, two special functions a value beside its weight's exponential, of which the SM has 32 (exp2) and
// 16 (reciprocal) a cycle.
__device__ __forceinline__ float2 tanh_near(const Attention& a, float2 d) {
    const float2 z = mul2(d, d);
    float2 p = fma2(z, a.near[0], a.near[1]);
    p = fma2(z, p, a.near[2]);
    p = fma2(z, p, a.near[3]);
    return fma2(z, p, a.near[4]);
}
__device__ __forceinline__ float2 tanh_any(float2 x) {
    const float k = 2.f * kLog2e;
    return make_float2(fmaf(-2.f, rcp_fast(1.f + exp2_fast(k * x.x)), 1.f), fmaf(-2.f, rcp_fast(1.f + exp2_fast(k * x.y)), 1.f));
}
// The largest of three, in one instruction; a NaN gives way to a number.
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
template <int N>
__device__ __forceinline__ float largest(const float* x, float m) {
    float u = m, v = m;
#pragma unroll
    for (int j = 0; j < N; j += 4) u = max3(u, x[j], x[j + 1]), v = max3(v, x[j + 2], x[j + 3]);
    return fmaxf(u, v);
}
// Whether all of a warp's 32 x N dot products stay within a limit.
template <int N>
__device__ __forceinline__ bool all_near(const float* x, float limit) {
    float u = 0.f, v = 0.f;
#pragma unroll
    for (int j = 0; j < N; j += 4) u = max3(u, fabsf(x[j]), fabsf(x[j + 1])), v = max3(v, fabsf(x[j + 2]), fabsf(x[j + 3]));
    return __all_sync(0xffffffffu, fmaxf(u, v) <= limit);
}
// Two bf16 of a column of TMEM, the first in the low half.
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// a b + c of two fp32 pairs in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(*(uint64_t*)&d)
        : "l"(*(uint64_t*)&a), "l"(*(uint64_t*)&b), "l"(*(uint64_t*)&c));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(*(uint64_t*)&d) : "l"(*(uint64_t*)&a), "l"(*(uint64_t*)&b));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(*(uint64_t*)&d) : "l"(*(uint64_t*)&a), "l"(*(uint64_t*)&b));
    return d;
}

// rows of 64 values of one head: {64, 1, rows, 1} boxes of {head_dim, heads, T, N}; values past head_dim and tokens past T
// arrive as zeros.
__device__ __forceinline__ void tma_load_head(uint32_t dst, const CUtensorMap* tm, int col, int head, int row, int n, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"((uint64_t)tm), "r"(col), "r"(head), "r"(row), "r"(n), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void tma_store_head(const CUtensorMap* tm, uint32_t src, int col, int head, int row, int n) {
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%1, %2, %3, %4}], [%5];" ::"l"((uint64_t)tm), "r"(col),
                 "r"(head), "r"(row), "r"(n), "r"(src)
                 : "memory");
}
// Zeros the 128-byte rows of a tile's panels whose bit is set (a warp's work): what no query sees may hold anything, and
// zero times NaN is NaN.
__device__ __forceinline__ void clear_rows(uint32_t tile, int panels, const uint32_t* bits) {
    const int lane = threadIdx.x % 32;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (!(bits[w] >> lane & 1)) continue;
        for (int p = 0; p < panels; ++p)
            for (int c = 0; c < 8; ++c)
                asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(tile + p * kPanel + (w * 32 + lane) * 128 + c * 16), "r"(0)
                             : "memory");
    }
    fence_proxy_async();
    __syncwarp();
}

// A window has the biases of a pair of tiles by distance, so that what row r reads for column j is V[128 - r + j]. Four copies, each
// one value behind the other: 4 columns are a 16-byte load for every row, and the copies lie on banks such that 8 rows, which read
// two pieces of a copy each, find 8 pieces beside one another.
constexpr int kWindow = 4 * 288;
__device__ __forceinline__ int copy_of(int c) { return c * 256 + (c == 0 ? 0 : 4 + 8 * c); }
__device__ __forceinline__ int window_row(int row) { return copy_of(-row & 3) + (128 - row & ~3); }
// The window of a pair of tiles q0 - k0 apart (a warp's work); BY_QUERY: rows are queries, else keys.
template <bool BY_QUERY>
__device__ __forceinline__ void load_window(const AttentionPlan& plan, int h, int apart, float* dst) {
    const int lane = threadIdx.x % 32;
    const float* src = plan.lut + (int64_t)h * plan.lut_len + plan.lut_mid + min(max(apart, -plan.reach - 127), plan.reach + 127) - 127;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = src[min(32 * e + lane, 254)];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int at = BY_QUERY ? 255 - 32 * e - lane : 32 * e + lane + 1;
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (at >= c && at < 256) dst[copy_of(c) + at - c] = v[e];
    }
}

// wait_bounded by a whole warp, its outcome the same in all lanes, in few instructions: the many roles of these kernels share the
// SM's instruction cache, and what runs seldom is fetched again each time (with wait_bounded in their place and loops unrolled
// over the two tiles 8 x 1024 tokens took 96 us, 71 this way).
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile int* abort, unsigned int* err) {
    uint32_t tries = 0;
    uint64_t since = 0;
    bool ok = true;
#pragma unroll 1
    while (!mbar_try_wait(bar, parity)) {
        if (++tries & 63) continue;
        const uint64_t now = global_ns();
        if (!since) since = now;
        if (*abort || now - since > kTimeoutNs) {
            atomicOr(err, kErrTimeout);
            *abort = 1;
            ok = false;
            break;
        }
    }
    return __all_sync(0xffffffffu, ok);
}

// A barrier of `threads` threads; whether none of them brings a failure. All come, whatever went wrong before, so that nobody is
// left alone at it.
__device__ __forceinline__ bool all_came_well(int id, int threads, bool ok) {
    uint32_t bad;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 p, %3, 0;\n bar.red.or.pred q, %1, %2, p;\n selp.u32 %0, 1, 0, q;\n}"
                 : "=r"(bad)
                 : "r"(id), "r"(threads), "r"((uint32_t)!ok)
                 : "memory");
    return !bad;
}

// Waits, up to the time limit, for what is in flight before a CTA may leave.
__device__ __forceinline__ void wait_settled(uint32_t bar, uint32_t parity, unsigned int* err) {
    const uint64_t since = global_ns();
    while (!mbar_try_wait(bar, parity))
        if (global_ns() - since > kTimeoutNs) {
            atomicOr(err, kErrTimeout);
            return;
        }
}
