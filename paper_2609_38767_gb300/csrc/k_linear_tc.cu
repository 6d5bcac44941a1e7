// k_linear_tc.cu -- the products of the linear layer on the tcgen05 tensor cores:
// Z = X W^T + b, Y = act(Z) + R; dX = B W; dW = B^T X. All are
// D[i][j] = sum_k P[i][k] Q[j][k] with operands that are K-major (X, W, B) or
// MN-major (W for dX, B and X for dW) in memory; TMA copies either kind into the
// matching 128-byte-swizzled shared-memory layout, 64 values of k per stage, so
// nothing is transposed in memory.
//
// fp32 operands arrive as three bf16 planes x = x0 + x1 + x2 (each the rounding of
// what the ones before leave, exact to 2^-24). The planes of a chunk of k are staged
// once and feed the six plane pairs whose products matter, smallest first. The
// tensor pipe adds into its fp32 accumulators with truncation, so for these every
// chunk's sum is drained and added up in registers with rounding (error against 64
// bits 1e-7 to 2e-7 of the result's norm up to K = 14336, below an fp32 FMA chain's).
// So are the sums of bf16 products whose output is fp32, every 64 chunks.
//
// linear_pair_kernel, for products with a tile for most SM pairs: two CTAs of a
// cluster hold one 256 x BN tile (cta_group::2), each staging 128 rows of P and half
// of Q, so an operand byte that reaches an SM feeds twice the MMAs; persistent, the
// epilogue of a tile beside the next tile's MMAs, bf16 outputs by TMA. Bound by the
// tensor pipe at the clock that the power limit leaves: 8192 x 14336 -> 4096 bf16
// 590-605 us = 1.59-1.63 PFLOP/s as calls on new inputs, 512-580 one launch after another (468 without loads and
// epilogue), 4096 x 2048 -> 8192 with tanh-gelu and Z 99 us as calls, 86 launch after launch (75 without its
// epilogue); fp32 2048 x 4096 -> 4096 300 us = 229 TFLOP/s, six bf16 products each.
//
// linear_tile_kernel: one 128 x BN tile per CTA. Few rows (a short batch) swap the
// operands, so the long side fills the 128 rows of a tile, and split the K loop over
// the CTAs of a cluster, whose fp32 tiles are added in rank order through distributed
// shared memory. Bound by reading W: 16 x 4096 -> 14336 23-25 us = 4.7-5.1 TB/s.
//
// Warp roles: warp 0 TMA producer (lane 0), warp 1 TMEM allocator and MMA issuer,
// warps 2-9 epilogue (TMEM lane quadrant warp % 4, column half by warp). Waits are
// bounded (about 1 s) and set kErrTimeout on expiry.
#include <cuda.h>

#include <mutex>
#include <type_traits>

#include "linear.cuh"

namespace tda {
namespace {

#include "tc_ptx.cuh"

constexpr int kThreads = 320, kEpiWarps = 8;
constexpr int kTM = 128;
constexpr int kTK = 64;                  // values of k per chunk
constexpr uint32_t kBox = 64 * kTK * 2;  // one MN-major box of 64 values: 8 KiB

// Accumulators in TMEM. One is handed to the epilogue and back per tile, for fp32 operands per chunk (24 MMAs,
// 0.8 us), where the way there and back takes about 1.6 us.
template <bool ROUND>
constexpr int kAcc = ROUND ? 4 : 2;

// The truncation is always towards zero, so a long sum of one sign drifts with its length: weight gradients of 8192
// tokens of 2048 -> 2304 were 2.4e-5 short, of 262144 1.5e-3. fp32 outputs are therefore drained every this many chunks
// and are 8e-6 short at any length. In the pair kernel that costs 2 to 8 % from 4097 tokens on (us without / with, dX
// beside dW: 8192 tokens of 2048 -> 8192 338 / 344, of 4096 -> 4096 317 / 323; dW alone 189 / 198; every 16 chunks,
// 8e-7, 13 %), in the tile kernel nothing.
constexpr int kWindow = 64;

struct TileParams {
    LinearEpilogue ep;
    int64_t tiles_p, tiles_q;
    int nk;             // chunks of kTK along K
    bool drain;         // bf16 operands: a fill of the accumulator is kWindow chunks, not all
    int split;          // CTAs of a cluster along K
    bool p_mn, q_mn;
    bool swap;          // tile rows are output columns
    unsigned int* err;
};

// fp32 operands: each plane of a chunk is a stage of its own, loaded in the order 0, 2, 1. The products
// P2 Q0, P0 Q2 free plane 2's stage, then P1 Q1, P1 Q0, P0 Q1 plane 1's, then P0 Q0: smallest first, and the
// next chunk's loads run through all of them. (Stages of all three planes left room for two, which did
// not cover the loads: 1.43 us a chunk of a 256 x 128 tile against 1.17.)
__device__ __forceinline__ constexpr int plane_of(int i) { return i == 0 ? 0 : i == 1 ? 2 : 1; }

// Shared-memory descriptors, 128-byte swizzle. K-major tiles: 8-row groups 1 KiB apart. MN-major tiles: 64-value
// atoms one box apart (LBO), 8-row groups of k 1 KiB apart (SBO).
__device__ __forceinline__ uint64_t desc_of(uint32_t saddr, bool mn) {
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(mn ? kBox >> 4 : 1) << 16) |
           ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// 16 values of k further: 32 bytes along a K-major row, two 8-row groups of an MN-major box.
__device__ __forceinline__ uint64_t desc_step(bool mn) { return mn ? 2048 >> 4 : 32 >> 4; }

__device__ __forceinline__ uint32_t elect_one() {
    uint32_t r;
    asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}" : "=r"(r));
    return r;
}
// Issued by the elected lane of a converged warp, so that the operands stay in uniform registers: a single-lane
// branch issued the 4 MMAs of a bf16 chunk up to a fifth slower than the tensor pipe runs them, depending on
// the code around them (fp32 2048 x 4096 -> 4096 366 us, 306 this way).
template <bool PAIR>
__device__ __forceinline__ void mma_one(uint32_t lead, uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t acc) {
    if constexpr (PAIR)
        asm volatile(
            "{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %5, 0;\n"
            " @q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(lead)
            : "memory");
    else
        asm volatile(
            "{\n .reg .pred p, q;\n setp.ne.b32 p, %4, 0;\n setp.ne.b32 q, %5, 0;\n"
            " @q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(acc), "r"(lead)
            : "memory");
}
// Arrives on `bar` (in both CTAs of a pair) once the MMAs so far are done.
template <bool PAIR>
__device__ __forceinline__ void commit_one(uint32_t lead, uint32_t bar) {
    if constexpr (PAIR)
        asm volatile(
            "{\n .reg .pred q;\n setp.ne.b32 q, %2, 0;\n"
            " @q tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n}" ::"r"(bar),
            "h"((uint16_t)3), "r"(lead)
            : "memory");
    else
        asm volatile(
            "{\n .reg .pred q;\n setp.ne.b32 q, %1, 0;\n"
            " @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(bar),
            "r"(lead)
            : "memory");
}
// The products of a chunk's four steps along k.
template <bool PAIR>
__device__ __forceinline__ void mma_chunk(uint32_t lead, uint32_t d, uint64_t a, uint64_t b, uint64_t sa, uint64_t sb,
                                          uint32_t idesc, bool first) {
#pragma unroll
    for (int k = 0; k < kTK / 16; ++k) mma_one<PAIR>(lead, d, a + k * sa, b + k * sb, idesc, first && k == 0 ? 0u : 1u);
}

// Waits, up to the time limit, for what is still in flight before a CTA may leave. Tries first: reading the clock
// takes longer than most of these waits.
__device__ __forceinline__ void wait_settled(uint32_t bar, uint32_t parity, unsigned int* err) {
#pragma unroll 1
    for (int i = 0; i < 128; ++i)
        if (mbar_try_wait(bar, parity)) return;
    const uint64_t since = global_ns();
    while (!mbar_try_wait(bar, parity))
        if (global_ns() - since > kTimeoutNs) {
            atomicOr(err, kErrTimeout);
            return;
        }
}

// A wait that the whole warp made, its outcome the same in all lanes.
__device__ __forceinline__ bool all_waited(bool ok) { return __all_sync(0xffffffffu, ok); }

// The stage in turn and its phase.
template <int STAGES>
struct Ring {
    uint32_t s = 0, ph = 0;
    __device__ __forceinline__ void next() {
        if (++s == STAGES) s = 0, ph ^= 1u;
    }
};

// 32 lanes x N consecutive fp32 columns of TMEM into registers, one instruction and one wait.
template <int N>
__device__ __forceinline__ void tmem_load(uint32_t taddr, float* v);
template <>
__device__ __forceinline__ void tmem_load<16>(uint32_t taddr, float* v) {
    uint32_t r[16];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 {"
        "%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15"
        "}, [%16];\n tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}
template <>
__device__ __forceinline__ void tmem_load<32>(uint32_t taddr, float* v) {
    uint32_t r[32];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 {"
        "%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%2"
        "6,%27,%28,%29,%30,%31"
        "}, [%32];\n tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}
template <>
__device__ __forceinline__ void tmem_load<64>(uint32_t taddr, float* v) {
    uint32_t r[64];
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x64.b32 {"
        "%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%2"
        "6,%27,%28,%29,%30,%31,%32,%33,%34,%35,%36,%37,%38,%39,%40,%41,%42,%43,%44,%45,%46,%47,%48,%49,%5"
        "0,%51,%52,%53,%54,%55,%56,%57,%58,%59,%60,%61,%62,%63"
        "}, [%64];\n tcgen05.wait::ld.sync.aligned;"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
          "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
          "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
          "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31]),
          "=r"(r[32]), "=r"(r[33]), "=r"(r[34]), "=r"(r[35]), "=r"(r[36]), "=r"(r[37]), "=r"(r[38]), "=r"(r[39]),
          "=r"(r[40]), "=r"(r[41]), "=r"(r[42]), "=r"(r[43]), "=r"(r[44]), "=r"(r[45]), "=r"(r[46]), "=r"(r[47]),
          "=r"(r[48]), "=r"(r[49]), "=r"(r[50]), "=r"(r[51]), "=r"(r[52]), "=r"(r[53]), "=r"(r[54]), "=r"(r[55]),
          "=r"(r[56]), "=r"(r[57]), "=r"(r[58]), "=r"(r[59]), "=r"(r[60]), "=r"(r[61]), "=r"(r[62]), "=r"(r[63])
        : "r"(taddr)
        : "memory");
#pragma unroll
    for (int i = 0; i < 64; ++i) v[i] = __uint_as_float(r[i]);
}

template <typename T>
__device__ __forceinline__ float ld1(const T* p);
template <>
__device__ __forceinline__ float ld1(const float* p) {
    return *p;
}
template <>
__device__ __forceinline__ float ld1(const __nv_bfloat16* p) {
    return __bfloat162float(*p);
}
__device__ __forceinline__ void ld4(const float* p, float* v) {
    const float4 x = *reinterpret_cast<const float4*>(p);
    v[0] = x.x, v[1] = x.y, v[2] = x.z, v[3] = x.w;
}
__device__ __forceinline__ void ld4(const __nv_bfloat16* p, float* v) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    v[0] = __uint_as_float(x.x << 16), v[1] = __uint_as_float(x.x & 0xFFFF0000u);
    v[2] = __uint_as_float(x.y << 16), v[3] = __uint_as_float(x.y & 0xFFFF0000u);
}
__device__ __forceinline__ void st1(float* p, float v) { *p = v; }
__device__ __forceinline__ void st1(__nv_bfloat16* p, float v) { *p = __float2bfloat16_rn(v); }
__device__ __forceinline__ void st4(float* p, const float* v) {
    *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}
__device__ __forceinline__ void st4(__nv_bfloat16* p, const float* v) {
    const __nv_bfloat162 a = __floats2bfloat162_rn(v[0], v[1]), b = __floats2bfloat162_rn(v[2], v[3]);
    *reinterpret_cast<uint2*>(p) =
        make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
}

// act of U x 4 values, the choice made once for all.
template <typename T, int U>
__device__ __forceinline__ void activate(int act, float (*v)[4]) {
    constexpr bool FAST = sizeof(T) == 2;
#define TDA_ACT_CASE(A)                                                          \
    case A:                                                                      \
        _Pragma("unroll") for (int u = 0; u < U; ++u)                            \
            _Pragma("unroll") for (int i = 0; i < 4; ++i) v[u][i] = act_value<A, FAST>(v[u][i]); \
        break
    switch (act) {
        TDA_ACT_CASE(TDA_ACT_RELU);
        TDA_ACT_CASE(TDA_ACT_GELU);
        TDA_ACT_CASE(TDA_ACT_GELU_TANH);
        TDA_ACT_CASE(TDA_ACT_SILU);
        default: break;
    }
#undef TDA_ACT_CASE
}

// Four sums of output row m, columns n .. n + 3, a value at a time: the last columns of aligned rows.
template <typename T>
__device__ __noinline__ void finish_edge(const LinearEpilogue& e, int64_t m, int64_t n, float x0, float x1, float x2,
                                         float x3) {
    float v[1][4] = {{x0, x1, x2, x3}};
    const int have = (int)(e.N - n < 4 ? e.N - n : 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (e.bias && i < have) v[0][i] += ld1((const T*)e.bias + n + i);
        if (e.Z && i < have) st1((T*)e.Z + m * e.ld_z + n + i, v[0][i]);
    }
    activate<T, 1>(e.act, v);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (i >= have) break;
        if (e.R) v[0][i] = fmaf(e.r_scale, ld1((const T*)e.R + m * e.ld_r + n + i), v[0][i]);
        st1((T*)e.Y + m * e.ld_y + n + i, v[0][i]);
    }
}

// U groups of four sums through the epilogue and out: group u is output row m[u], columns n[u] .. + 3, inside the
// output where ok[u]. All loads come before the first store.
template <typename T, int U>
__device__ __forceinline__ void finish(const LinearEpilogue& e, const int64_t* m, const int64_t* n, const bool* ok,
                                       float (*v)[4]) {
    bool whole[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        whole[u] = ok[u] && n[u] + 4 <= e.N;
        if (ok[u] && !whole[u]) finish_edge<T>(e, m[u], n[u], v[u][0], v[u][1], v[u][2], v[u][3]);
    }
    float r[U][4], b[U][4];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        if (e.R && whole[u]) ld4((const T*)e.R + m[u] * e.ld_r + n[u], r[u]);
        if (e.bias && whole[u]) ld4((const T*)e.bias + n[u], b[u]);
    }
    if (e.bias)
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[u][i] += b[u][i];
    if (e.Z)
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (whole[u]) st4((T*)e.Z + m[u] * e.ld_z + n[u], v[u]);
    activate<T, U>(e.act, v);
    if (e.R)
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[u][i] = fmaf(e.r_scale, r[u][i], v[u][i]);
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (whole[u]) st4((T*)e.Y + m[u] * e.ld_y + n[u], v[u]);
}

// U sums through the epilogue and out a value at a time, for rows that do not start on an aligned place: sum u is
// output row m[u], column n[u], inside the output where ok[u]. Neighbouring lanes hold
// neighbouring columns. All loads come before the first store.
template <typename T, int U>
__device__ __forceinline__ void finish_values(const LinearEpilogue& e, const int64_t* m, const int64_t* n, const bool* ok,
                                              float (*v)[4]) {
    float r[U], b[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        r[u] = e.R && ok[u] ? ld1((const T*)e.R + m[u] * e.ld_r + n[u]) : 0.f;
        b[u] = e.bias && n[u] < e.N ? ld1((const T*)e.bias + n[u]) : 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        v[u / 4][u % 4] += b[u];
        if (e.Z && ok[u]) st1((T*)e.Z + m[u] * e.ld_z + n[u], v[u / 4][u % 4]);
    }
    activate<T, U / 4>(e.act, v);
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (ok[u]) {
            const float y = v[u / 4][u % 4];
            st1((T*)e.Y + m[u] * e.ld_y + n[u], e.R ? fmaf(e.r_scale, r[u], y) : y);
        }
}

// ---- units of 32 rows x 64 bytes, the grain of the pair kernel's outputs
__device__ __forceinline__ void tma_store_2d(const CUtensorMap* tm, uint32_t src, int c0, int c1) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"((uint64_t)tm),
                 "r"(c0), "r"(c1), "r"(src)
                 : "memory");
}
__device__ __forceinline__ void bulk_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_read1() { asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_read0() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait_all() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// 16-byte piece j of row r in a unit's shared memory: the 64-byte swizzle, conflict-free by rows and by pieces.
__device__ __forceinline__ uint32_t unit_at(int r, int j) { return (uint32_t)(r * 64 + ((j ^ ((r >> 1) & 3)) << 4)); }

// Piece of 16 bytes of a row, n its first column: whole, or value by value at the matrix's edge.
template <typename T>
__device__ __forceinline__ uint4 load_piece(const T* row, int64_t n, int64_t N) {
    constexpr int E = 16 / sizeof(T);
    uint4 q = make_uint4(0, 0, 0, 0);
    if (n + E <= N) {
        q = *reinterpret_cast<const uint4*>(row + n);
    } else if (n < N) {
        T x[E];
#pragma unroll
        for (int i = 0; i < E; ++i) x[i] = n + i < N ? row[n + i] : T(0.f);
        q = *reinterpret_cast<const uint4*>(x);
    }
    return q;
}
template <typename T>
__device__ __forceinline__ float piece_get(const uint4& x, int i) {  // i known at compile time
    const int w = sizeof(T) == 4 ? i : i >> 1;
    const uint32_t b = w == 0 ? x.x : w == 1 ? x.y : w == 2 ? x.z : x.w;
    return __uint_as_float(sizeof(T) == 4 ? b : i & 1 ? b & 0xFFFF0000u : b << 16);
}
template <typename T>
__device__ __forceinline__ uint4 piece_of(const float* v) {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        if constexpr (sizeof(T) == 4) {
            w[j] = __float_as_uint(v[j]);
        } else {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
            w[j] = *reinterpret_cast<const uint32_t*>(&h);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ float4 ld_cluster_f4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(addr)
                 : "memory");
    return v;
}

// ------------------------------------------------------------------ one tile per CTA
template <int BN, bool ROUND>
struct TileShape {
    static constexpr int kPlanes = ROUND ? 3 : 1;  // stages of a chunk
    static constexpr uint32_t kP = kTM * kTK * 2, kQ = BN * kTK * 2, kStage = kP + kQ;
    // two CTAs share an SM (96 to 100 KiB of stages each); the rounding variant keeps its sums in
    // registers and takes an SM alone
    static constexpr int kStages = ROUND ? (BN == 128 ? 6 : 8) : BN == 128 ? 3 : BN == 64 ? 4 : 5;
    static constexpr size_t kSmem = 1024 + (size_t)kStages * kStage + 8 * (2 * kStages + 2 * kAcc<ROUND> + 1) + 16;
    static constexpr uint32_t kCols = kAcc<ROUND> * BN;
    static_assert((BN + 4) * kTM * 4 <= kStages * kStage, "the fp32 tile reuses the stages");
};

// One product, or two in one launch: CTAs below ctas0 work on the first.
struct TileLaunch {
    TileParams g[2];
    CUtensorMap tmP[2], tmQ[2];
    int ctas0;
};

// A CTA's work on product g; the parameters stay at fixed places of the constant bank.
template <int BN, bool ROUND, int g>
__device__ __forceinline__ void tile_body(const TileLaunch& pp) {
    using S = TileShape<BN, ROUND>;
    const TileParams& p = pp.g[g];
    const CUtensorMap &tmP = pp.tmP[g], &tmQ = pp.tmQ[g];
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint64_t* bars = (uint64_t*)(smem + (size_t)S::kStages * S::kStage);
    uint64_t* full = bars;                    // TMA bytes landed
    uint64_t* empty = bars + S::kStages;      // MMAs done with the stage
    uint64_t* tfull = bars + 2 * S::kStages;  // accumulator ready
    uint64_t* tempty = tfull + kAcc<ROUND>;   // accumulator drained
    uint64_t* mma_done = tempty + kAcc<ROUND>;
    uint32_t* tmem_slot = (uint32_t*)(mma_done + 1);
    volatile int* abort = (volatile int*)(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(smem_u32(&full[s]), 1);
            mbar_init(smem_u32(&empty[s]), 1);
        }
        for (int b = 0; b < kAcc<ROUND>; ++b) {
            mbar_init(smem_u32(&tfull[b]), 1);
            mbar_init(smem_u32(&tempty[b]), kEpiWarps);
        }
        mbar_init(smem_u32(mma_done), 1);
        *abort = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(tmem_slot), S::kCols);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    chain_wait();
    chain_next();

    const int cta = (int)blockIdx.x - (g ? pp.ctas0 : 0);
    const int64_t tile = cta / p.split;
    const int rank = cta % p.split;
    const int64_t i0 = (tile / p.tiles_q) * kTM, j0 = (tile % p.tiles_q) * BN;
    const int t0 = (int)((int64_t)p.nk * rank / p.split), t1 = (int)((int64_t)p.nk * (rank + 1) / p.split);
    const int windows = ROUND ? t1 - t0 : p.drain ? (t1 - t0 + kWindow - 1) / kWindow : 1;  // accumulator fills

    if (warp == 0) {
        if (lane == 0) {
            // ---------------- TMA producer
            uint32_t last_par[S::kStages];
            bool issued[S::kStages];
            for (int s = 0; s < S::kStages; ++s) issued[s] = false;
            bool ok = true;
            Ring<S::kStages> ring;
            for (int i = t0 * S::kPlanes; ok && i < t1 * S::kPlanes; ++i, ring.next()) {
                const int k0 = i / S::kPlanes * kTK, pl = plane_of(i % S::kPlanes);
                const uint32_t s = ring.s, ph = ring.ph;
                if (!(ok = wait_bounded(smem_u32(&empty[s]), ph ^ 1u, abort, p.err))) break;
                const uint32_t dp = smem_u32(smem + (size_t)s * S::kStage), dq = dp + S::kP, bar = smem_u32(&full[s]);
                mbar_arrive_tx(bar, S::kStage);
                if (p.p_mn) {
                    for (int j = 0; j < kTM / 64; ++j) tma_load_3d(dp + j * kBox, &tmP, (int)i0 + 64 * j, k0, pl, bar);
                } else {
                    tma_load_3d(dp, &tmP, k0, (int)i0, pl, bar);
                }
                if (BN >= 64 && p.q_mn) {
                    for (int j = 0; j < BN / 64; ++j) tma_load_3d(dq + j * kBox, &tmQ, (int)j0 + 64 * j, k0, pl, bar);
                } else {
                    tma_load_3d(dq, &tmQ, k0, (int)j0, pl, bar);
                }
                issued[s] = true;
                last_par[s] = ph;
            }
            // copies still in flight when the MMA side stopped early land before the CTA exits
            for (int s = 0; s < S::kStages; ++s)
                if (issued[s]) {
                    wait_settled(smem_u32(&full[s]), last_par[s], p.err);
                }
        }
    } else if (warp == 1) {
        {
            // ---------------- MMA issuer: the whole warp runs the loop, one lane issues
            const uint32_t lead = elect_one();
            const uint32_t idesc = idesc_bf16(kTM, BN) | (p.p_mn ? 1u << 15 : 0u) | (p.q_mn ? 1u << 16 : 0u);
            const uint64_t sp = desc_step(p.p_mn), sq = desc_step(p.q_mn);
            const uint32_t bar_full = smem_u32(full), bar_empty = smem_u32(empty);
            const uint64_t low_p = desc_of(smem_u32(smem), p.p_mn), low_q = desc_of(smem_u32(smem) + S::kP, p.q_mn);
            bool ok = true;
            int t = t0;
            Ring<S::kStages> ring;
            for (int w = 0; ok && w < windows; ++w) {
                const uint32_t b = w % kAcc<ROUND>, use = w / kAcc<ROUND>;
                if (!all_waited(wait_bounded(smem_u32(&tempty[b]), (use & 1u) ^ 1u, abort, p.err))) break;
                tc_fence_after();
                const uint32_t d = tmem + b * BN;
                auto await = [&](const Ring<S::kStages>& r) {
                    if (ok) ok = all_waited(wait_bounded(bar_full + 8 * r.s, r.ph, abort, p.err));
                    tc_fence_after();
                    return r.s * (S::kStage >> 4);
                };
                if (ROUND) {
                    const uint32_t s0 = ring.s, o0 = await(ring);
                    ring.next();
                    const uint32_t s2 = ring.s, o2 = await(ring);
                    ring.next();
                    if (ok) {
                        mma_chunk<false>(lead, d, low_p + o2, low_q + o0, sp, sq, idesc, true);
                        mma_chunk<false>(lead, d, low_p + o0, low_q + o2, sp, sq, idesc, false);
                        commit_one<false>(lead, bar_empty + 8 * s2);
                    }
                    const uint32_t s1 = ring.s, o1 = await(ring);
                    ring.next();
                    if (ok) {
                        mma_chunk<false>(lead, d, low_p + o1, low_q + o1, sp, sq, idesc, false);
                        mma_chunk<false>(lead, d, low_p + o1, low_q + o0, sp, sq, idesc, false);
                        mma_chunk<false>(lead, d, low_p + o0, low_q + o1, sp, sq, idesc, false);
                        commit_one<false>(lead, bar_empty + 8 * s1);
                        mma_chunk<false>(lead, d, low_p + o0, low_q + o0, sp, sq, idesc, false);
                        commit_one<false>(lead, bar_empty + 8 * s0);
                    }
                    ++t;
                } else {
                    const int end = p.drain && t1 - t > kWindow ? t + kWindow : t1;
                    for (bool first = true; ok && t < end; ++t, first = false) {
                        const uint32_t s = ring.s, o = await(ring);
                        ring.next();
                        if (!ok) break;
                        mma_chunk<false>(lead, d, low_p + o, low_q + o, sp, sq, idesc, first);
                        commit_one<false>(lead, bar_empty + 8 * s);
                    }
                }
                if (ok) commit_one<false>(lead, smem_u32(&tfull[b]));
            }
            commit_one<false>(lead, smem_u32(mma_done));
            wait_settled(smem_u32(mma_done), 0, p.err);
        }
    } else {
        // ---------------- accumulators -> shared fp32 tile, the output's columns contiguous
        const int half = (warp - 2) >> 2, q = warp & 3;
        constexpr int kC = BN / 2;  // columns of this warp
        float* ft = reinterpret_cast<float*>(smem);
        const uint32_t tb = tmem + ((uint32_t)(q * 32) << 16) + half * kC;
        const int row = q * 32 + lane;
        auto put = [&](int c, const float* v) {  // 16 columns from c on
            if (p.swap) {
#pragma unroll
                for (int i = 0; i < 16; ++i) ft[(c + i) * kTM + row] = v[i];
            } else {
#pragma unroll
                for (int i = 0; i < 16; i += 4)
                    *reinterpret_cast<float4*>(ft + row * (BN + 4) + c + i) =
                        make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
            }
        };
        auto wait_for = [&](int w) {
            bool got = true;
            if (lane == 0)
                got = wait_bounded(smem_u32(&tfull[w % kAcc<ROUND>]), (uint32_t)(w / kAcc<ROUND>) & 1u, abort, p.err);
            got = __shfl_sync(0xffffffffu, got, 0);
            tc_fence_after();
            return got;
        };
        if (!ROUND && windows == 1) {
            if (wait_for(0)) {
#pragma unroll
                for (int c = 0; c < kC; c += 16) {
                    float v[16];
                    tmem_load<16>(tb + c, v);
                    put(half * kC + c, v);
                }
            }
        } else {
            constexpr int kL = ROUND ? kC : 16;  // columns loaded at once
            float acc[kC];
#pragma unroll
            for (int i = 0; i < kC; ++i) acc[i] = 0.f;
            bool got = true;
            for (int w = 0; got && w < windows; ++w) {
                if (!(got = wait_for(w))) break;
#pragma unroll
                for (int c = 0; c < kC; c += kL) {
                    float v[kL];
                    tmem_load<kL>(tb + (w % kAcc<ROUND>) * BN + c, v);
                    if (c + kL == kC) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&tempty[w % kAcc<ROUND>]));
                    }
#pragma unroll
                    for (int i = 0; i < kL; ++i) acc[c + i] += v[i];
                }
            }
            // the last window's MMAs have read every stage: the tile may take their place
            if (got)
#pragma unroll
                for (int c = 0; c < kC; c += 16) put(half * kC + c, acc + c);
        }
    }
    __syncwarp();
    tc_fence_before();
    if (p.split > 1)
        cluster_sync();
    else
        __syncthreads();
    if (!*abort) {
        // ---------------- the cluster's tiles added in rank order, this CTA's share of the rows out
        const int inner = p.swap ? kTM : BN, stride = p.swap ? kTM : BN + 4;
        const int groups = kTM * BN / 4, g0 = groups * rank / p.split, g1 = groups * (rank + 1) / p.split;
        const int64_t m0 = p.swap ? j0 : i0, n0 = p.swap ? i0 : j0;
        const uint32_t base = smem_u32(smem);
        if (p.ep.vec) {
            constexpr int U = ROUND ? 4 : 2;
            for (int g = g0 + threadIdx.x; g < g1; g += U * kThreads) {
                int64_t m[U], n[U];
                bool ok[U];
                float v[U][4];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int gu = g + u * kThreads, o = gu * 4 / inner, c = gu * 4 % inner;
                    m[u] = m0 + o, n[u] = n0 + c;
                    ok[u] = gu < g1 && m[u] < p.ep.M && n[u] < p.ep.N;
                    v[u][0] = v[u][1] = v[u][2] = v[u][3] = 0.f;
                    if (!ok[u]) continue;
                    const uint32_t at = base + (uint32_t)(o * stride + c) * 4;
                    for (int r = 0; r < p.split; ++r) {
                        const float4 x = ld_cluster_f4(map_rank(at, r));
                        v[u][0] += x.x, v[u][1] += x.y, v[u][2] += x.z, v[u][3] += x.w;
                    }
                }
                if (ROUND || p.ep.f32)
                    finish<float, U>(p.ep, m, n, ok, v);
                else
                    finish<__nv_bfloat16, U>(p.ep, m, n, ok, v);
            }
        } else {
            // the sums to this CTA's own tile, whose share of the rows no other CTA reads, and out a value a lane
            const float* ft = reinterpret_cast<const float*>(smem);
            if (p.split > 1) {
                for (int g = g0 + threadIdx.x; g < g1; g += kThreads) {
                    const uint32_t off = (uint32_t)(g * 4 / inner * stride + g * 4 % inner) * 4;
                    float4 t = make_float4(0.f, 0.f, 0.f, 0.f);
                    for (int r = 0; r < p.split; ++r) {
                        const float4 x = ld_cluster_f4(map_rank(base + off, r));
                        t.x += x.x, t.y += x.y, t.z += x.z, t.w += x.w;
                    }
                    *reinterpret_cast<float4*>(smem + off) = t;
                }
                __syncthreads();
            }
            const int lg = p.swap ? 7 : BN == 128 ? 7 : BN == 64 ? 6 : 5;
            constexpr int U = 8;
            for (int g = g0 * 4 + threadIdx.x; g < g1 * 4; g += U * kThreads) {
                int64_t m[U], n[U];
                bool ok[U];
                float v[U / 4][4];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int gu = g + u * kThreads, o = gu >> lg, c = gu & ((1 << lg) - 1);
                    m[u] = m0 + o, n[u] = n0 + c;
                    ok[u] = gu < g1 * 4 && m[u] < p.ep.M && n[u] < p.ep.N;
                    v[u / 4][u % 4] = ok[u] ? ft[o * stride + c] : 0.f;
                }
                if (ROUND || p.ep.f32)
                    finish_values<float, U>(p.ep, m, n, ok, v);
                else
                    finish_values<__nv_bfloat16, U>(p.ep, m, n, ok, v);
            }
        }
    }
    __syncwarp();
    if (p.split > 1)
        cluster_sync();  // no CTA leaves while its tile is still read
    else
        __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, S::kCols);
    }
}

template <int BN, bool ROUND>
__global__ void __launch_bounds__(kThreads, ROUND ? 1 : 2) linear_tile_kernel(const __grid_constant__ TileLaunch pp) {
    if ((int)blockIdx.x < pp.ctas0)
        tile_body<BN, ROUND, 0>(pp);
    else
        tile_body<BN, ROUND, 1>(pp);
}

// ------------------------------------------------------------------ one tile per CTA pair, persistent
__device__ __forceinline__ void pair_alloc(uint32_t dst, uint32_t cols) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(dst), "r"(cols) : "memory");
}
__device__ __forceinline__ void pair_relinquish() {
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void pair_dealloc(uint32_t taddr, uint32_t cols) {
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(cols) : "memory");
}
// A box into this CTA's shared memory whose bytes count on a barrier of either CTA of the pair.
__device__ __forceinline__ void pair_load_3d(uint32_t dst, const CUtensorMap* tm, int c0, int c1, int c2, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, "
        "%4}], [%5];" ::"r"(dst),
        "l"((uint64_t)tm), "r"(c0), "r"(c1), "r"(c2), "r"(bar)
        : "memory");
}

// Arrive on the leader's barrier: orders what the thread has read from TMEM (before a tcgen05 fence), no memory
// is handed over, so nothing wider than the default scope is waited for.
__device__ __forceinline__ void pair_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(map_rank(bar, 0)) : "memory");
}

template <int BN, bool ROUND>
struct PairShape {
    static constexpr int kPlanes = ROUND ? 3 : 1;  // stages of a chunk
    static constexpr uint32_t kP = kTM * kTK * 2, kQ = BN / 2 * kTK * 2, kStage = kP + kQ;
    static constexpr int kStages = ROUND ? 8 : 6;
    static constexpr uint32_t kUnit = 32 * 64;       // one output unit
    static constexpr uint32_t kBlock = 2 * kUnit;    // two per epilogue warp
    static_assert(32 * 32 * 4 <= kBlock, "a unit in fp32");
    static constexpr size_t kSmem = 1024 + (size_t)kStages * kStage + kEpiWarps * kBlock + 8 * (2 * kStages + 2 * kAcc<ROUND> + 1) + 16;
    static constexpr uint32_t kCols = 512;  // the SM's whole TMEM: both CTAs' columns start at the same place
    static_assert(kSmem <= 232448, "shared memory per CTA");
};

// One or two products (dX and dW of a layer) in one launch, the one with the longer K loop first. Its tiles go
// round the pairs; where the last round is short, the pairs left out take `extra` tiles of the second product
// each (about as long as one of the first) before the rest of those goes round all pairs.
struct PairParams {
    TileParams g[2];
    CUtensorMap tmP[2], tmQ[2];
    CUtensorMap tmY[2], tmZ;  // outputs with 16-byte aligned rows, of bf16 operands; tmZ: of product 0
    int64_t tiles[2];  // tiles[1] = 0: one product
    int extra;
    unsigned int* err;
};

// The j-th tile of product g for pair i of n; >= pp.tiles[g]: there is none.
template <int g>
__device__ __forceinline__ int64_t pair_tile(const PairParams& pp, int64_t i, int64_t n, int64_t j) {
    if (g == 0) return i + j * n;
    const int64_t rem = pp.tiles[0] % n, idle = n - rem;  // pairs rem .. n - 1 have one tile less of product 0
    if (i >= rem) {
        if (j < pp.extra) return i - rem + j * idle;
        j -= pp.extra;
    }
    return pp.extra * idle + (i >= rem ? i - rem : i + idle) + j * n;
}

// DRAIN: a product has fp32 outputs of bf16 operands and more than a window of chunks. A variant of its own: its 128 sums
// a thread do not all fit the registers (1.1 KB of spills outside the loop over chunks), which the others need not pay.
template <int BN, bool ROUND, bool DRAIN>
__global__ void __launch_bounds__(kThreads, 1) linear_pair_kernel(const __grid_constant__ PairParams pp) {
    static_assert(!ROUND || !DRAIN, "fp32 operands are always drained");
    using S = PairShape<BN, ROUND>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint8_t* blocks = smem + (size_t)S::kStages * S::kStage;
    uint64_t* bars = (uint64_t*)(blocks + kEpiWarps * S::kBlock);
    uint64_t* full = bars;                    // leader's: both CTAs' bytes landed
    uint64_t* empty = bars + S::kStages;      // each CTA's own: MMAs done with the stage
    uint64_t* tfull = bars + 2 * S::kStages;  // each CTA's own: accumulator ready
    uint64_t* tempty = tfull + kAcc<ROUND>;   // leader's: accumulator drained by both CTAs' warps
    uint64_t* mma_done = tempty + kAcc<ROUND>;
    uint32_t* tmem_slot = (uint32_t*)(mma_done + 1);
    volatile int* abort = (volatile int*)(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(smem_u32(&full[s]), 1);
            mbar_init(smem_u32(&empty[s]), 1);
        }
        for (int b = 0; b < kAcc<ROUND>; ++b) {
            mbar_init(smem_u32(&tfull[b]), 1);
            mbar_init(smem_u32(&tempty[b]), 2 * kEpiWarps);
        }
        mbar_init(smem_u32(mma_done), 1);
        *abort = 0;
        fence_mbar_init();
    }
    if (warp == 1) {
        pair_alloc(smem_u32(tmem_slot), S::kCols);
        pair_relinquish();
    }
    tc_fence_before();
    __syncwarp();
    cluster_sync();  // both CTAs' barriers exist before either signals the other's
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    chain_wait();
    chain_next();

    const int64_t me = blockIdx.x >> 1, pairs = gridDim.x >> 1;
    // A product's tiles go in bands of 8 tile rows, down each column of a band: the
    // pairs at work share operand rows in L2.
    // Each role runs its loop once per product, with that product's parameters at fixed places of the constant
    // bank: reading them through an index made the loops a fifth slower.
    auto place = [](const TileParams& p, int64_t u, int64_t* i0, int64_t* j0) {
        const int64_t band = u / (8 * p.tiles_q), in = u % (8 * p.tiles_q);
        const int64_t h = p.tiles_p - band * 8 < 8 ? p.tiles_p - band * 8 : 8;
        *i0 = (band * 8 + in % h) * (2 * kTM);
        *j0 = (in / h) * BN;
    };

    if (warp == 0) {
        if (lane == 0) {
            // ---------------- TMA producer of this CTA's halves
            Ring<S::kStages> ring;
            uint32_t last_par[S::kStages];
            bool issued[S::kStages], ok = true;
            for (int s = 0; s < S::kStages; ++s) issued[s] = false;
            auto feed = [&](auto G) {
              constexpr int g = decltype(G)::value;
              const TileParams& p = pp.g[g];
              const CUtensorMap *tmP = &pp.tmP[g], *tmQ = &pp.tmQ[g];
              const int total = p.nk;
              for (int64_t j = 0, u; ok && (u = pair_tile<g>(pp, me, pairs, j)) < pp.tiles[g]; ++j) {
                int64_t i0, j0;
                place(p, u, &i0, &j0);
                const int pr = (int)i0 + (int)rank * kTM, qr = (int)j0 + (int)rank * (BN / 2);
                for (int i = 0; i < total * S::kPlanes; ++i, ring.next()) {
                    const int k0 = i / S::kPlanes * kTK, pl = plane_of(i % S::kPlanes);
                    const uint32_t s = ring.s, ph = ring.ph;
                    if (!wait_bounded(smem_u32(&empty[s]), ph ^ 1u, abort, pp.err)) {
                        ok = false;
                        break;
                    }
                    const uint32_t dp = smem_u32(smem + (size_t)s * S::kStage), dq = dp + S::kP, bar = smem_u32(&full[s]);
                    const uint32_t lead = map_rank(bar, 0);
                    if (rank == 0) mbar_arrive_tx(bar, 2 * S::kStage);
                    if (p.p_mn) {
                        for (int j = 0; j < kTM / 64; ++j) pair_load_3d(dp + j * kBox, tmP, pr + 64 * j, k0, pl, lead);
                    } else {
                        pair_load_3d(dp, tmP, k0, pr, pl, lead);
                    }
                    if (p.q_mn) {
                        for (int j = 0; j < BN / 128; ++j) pair_load_3d(dq + j * kBox, tmQ, qr + 64 * j, k0, pl, lead);
                    } else {
                        pair_load_3d(dq, tmQ, k0, qr, pl, lead);
                    }
                    issued[s] = true;
                    last_par[s] = ph;
                }
              }
            };
            feed(std::integral_constant<int, 0>());
            feed(std::integral_constant<int, 1>());
            // copies still in flight when the MMA side stopped early land before the pair exits
            if (rank == 0)
                for (int s = 0; s < S::kStages; ++s)
                    if (issued[s]) {
                        wait_settled(smem_u32(&full[s]), last_par[s], pp.err);
                    }
            // and so do the last signals that the pair's MMAs send to this CTA's stages; a signal sent means that both
            // CTAs' copies into the stage have landed
            for (int s = 0; s < S::kStages; ++s)
                if (issued[s]) wait_bounded(smem_u32(&empty[s]), last_par[s], abort, pp.err);
        }
    } else if (warp == 1) {
        if (rank == 0) {
            // ---------------- MMA issuer of the pair: the whole warp runs the loop, one lane issues
            const uint32_t lead = elect_one();
            Ring<S::kStages> ring;
            Ring<kAcc<ROUND>> acc;
            bool ok = true;
            auto issue = [&](auto G) {
              constexpr int g = decltype(G)::value;
              const TileParams& p = pp.g[g];
              const bool p_mn = p.p_mn, q_mn = p.q_mn;
              const uint32_t idesc = idesc_bf16(2 * kTM, BN) | (p_mn ? 1u << 15 : 0u) | (q_mn ? 1u << 16 : 0u);
              const uint64_t sp = desc_step(p_mn), sq = desc_step(q_mn);
              const uint32_t bar_full = smem_u32(full), bar_empty = smem_u32(empty);
              const uint64_t low_p = desc_of(smem_u32(smem), p_mn), low_q = desc_of(smem_u32(smem) + S::kP, q_mn);
              const int total = p.nk, windows = ROUND ? total : DRAIN && p.drain ? (total + kWindow - 1) / kWindow : 1;  // fills of a tile
              for (int64_t j = 0; ok && pair_tile<g>(pp, me, pairs, j) < pp.tiles[g]; ++j) {
                int t = 0;
                for (int w = 0; ok && w < windows; ++w, acc.next()) {
                    const uint32_t b = acc.s;
                    if (!all_waited(wait_bounded(smem_u32(&tempty[b]), acc.ph ^ 1u, abort, pp.err))) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t d = tmem + b * BN;
                    auto await = [&](const Ring<S::kStages>& r) {
                        if (ok) ok = all_waited(wait_bounded(bar_full + 8 * r.s, r.ph, abort, pp.err));
                        tc_fence_after();
                        return r.s * (S::kStage >> 4);
                    };
                    if (ROUND) {
                        const uint32_t s0 = ring.s, o0 = await(ring);
                        ring.next();
                        const uint32_t s2 = ring.s, o2 = await(ring);
                        ring.next();
                        if (ok) {
                            mma_chunk<true>(lead, d, low_p + o2, low_q + o0, sp, sq, idesc, true);
                            mma_chunk<true>(lead, d, low_p + o0, low_q + o2, sp, sq, idesc, false);
                            commit_one<true>(lead, bar_empty + 8 * s2);
                        }
                        const uint32_t s1 = ring.s, o1 = await(ring);
                        ring.next();
                        if (ok) {
                            mma_chunk<true>(lead, d, low_p + o1, low_q + o1, sp, sq, idesc, false);
                            mma_chunk<true>(lead, d, low_p + o1, low_q + o0, sp, sq, idesc, false);
                            mma_chunk<true>(lead, d, low_p + o0, low_q + o1, sp, sq, idesc, false);
                            commit_one<true>(lead, bar_empty + 8 * s1);
                            mma_chunk<true>(lead, d, low_p + o0, low_q + o0, sp, sq, idesc, false);
                            commit_one<true>(lead, bar_empty + 8 * s0);
                        }
                        ++t;
                    } else {
                        const int end = DRAIN && p.drain && total - t > kWindow ? t + kWindow : total;
                        for (bool first = true; ok && t < end; ++t, first = false) {
                            const uint32_t s = ring.s, o = await(ring);
                            ring.next();
                            if (!ok) break;
                            mma_chunk<true>(lead, d, low_p + o, low_q + o, sp, sq, idesc, first);
                            commit_one<true>(lead, bar_empty + 8 * s);
                        }
                    }
                    if (ok) commit_one<true>(lead, smem_u32(&tfull[b]));
                }
              }
            };
            issue(std::integral_constant<int, 0>());
            issue(std::integral_constant<int, 1>());
            commit_one<true>(lead, smem_u32(mma_done));
            wait_settled(smem_u32(mma_done), 0, pp.err);
        }
    } else {
        // ---------------- epilogue of this CTA's 128 rows: 32 x 32 blocks through shared memory
        const int half = (warp - 2) >> 2, q = warp & 3;
        constexpr int kC = BN / 2;  // columns of this warp
        float* blk = reinterpret_cast<float*>(blocks + (warp - 2) * S::kBlock);
        const uint32_t tb = tmem + ((uint32_t)(q * 32) << 16) + half * kC;
        uint32_t use = 0;
        auto wait_for = [&]() {
            bool got = true;
            if (lane == 0)
                got = wait_bounded(smem_u32(&tfull[use % kAcc<ROUND>]), (use / kAcc<ROUND>) & 1u, abort, pp.err);
            got = __shfl_sync(0xffffffffu, got, 0);
            tc_fence_after();
            return got;
        };
        auto release = [&]() {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) pair_arrive(smem_u32(&tempty[use % kAcc<ROUND>]));
            ++use;
        };
        bool got = true;
        auto drain = [&](auto G) {
          constexpr int g = decltype(G)::value;
          const TileParams& p = pp.g[g];
          for (int64_t j = 0, u; got && (u = pair_tile<g>(pp, me, pairs, j)) < pp.tiles[g]; ++j) {
            int64_t i0, j0;
            place(p, u, &i0, &j0);
            const int64_t m0 = i0 + rank * kTM + q * 32, n0 = j0 + half * kC;
            // This warp's rows and columns, a unit at a time: the row in registers (from `get`) through the epilogue
            // into shared memory, and out by TMA, which clips it at the matrix's edges. The residual's unit is
            // loaded 8 rows an access, one unit ahead, and handed to the rows' lanes through shared memory.
            // held: the sums are registers already (`get` with places known at compile time), not one accumulator.
            auto column_units = [&](auto zero, auto held, auto get) {
                using T = decltype(zero);
                constexpr bool kHeld = decltype(held)::value;
                constexpr int kU = 64 / sizeof(T), E = 16 / sizeof(T);
                // fp32 outputs of bf16 products are gradients: nothing but beta times themselves is added
                constexpr bool kPlain = g == 1 || (!ROUND && sizeof(T) == 4);
                const bool has_r = !ROUND && p.ep.R != nullptr && p.ep.wide;
                uint4 r[4];
                auto load_r = [&](int64_t n) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int64_t m = m0 + i * 8 + (lane >> 2);
                        if (m < p.ep.M) r[i] = load_piece((const T*)p.ep.R + m * p.ep.ld_r, n + (lane & 3) * E, p.ep.N);
                    }
                };
                uint32_t which = 0;
                // a unit that may be written: all but the last store have read theirs
                auto take = [&]() {
                    if (lane == 0) bulk_wait_read1();
                    __syncwarp();
                    which ^= 1;
                    return blocks + (warp - 2) * S::kBlock + which * S::kUnit;
                };
                auto send = [&](const CUtensorMap* tm, uint8_t* unit, const float* v, int64_t n) {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        *reinterpret_cast<uint4*>(unit + unit_at(lane, j)) = piece_of<T>(v + j * E);
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) {
                        if (m0 < p.ep.M && n < p.ep.N) tma_store_2d(tm, smem_u32(unit), (int)n, (int)m0);
                        bulk_commit();
                    }
                };
                auto unit = [&](int c) {
                    const int64_t n = n0 + c;
                    float v[kU];
                    get(c, v);
                    if (!kPlain && p.ep.bias) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) {  // the same addresses in every lane
                            const uint4 b = load_piece((const T*)p.ep.bias, n + j * E, p.ep.N);
#pragma unroll
                            for (int i = 0; i < E; ++i) v[j * E + i] += piece_get<T>(b, i);
                        }
                    }
                    if (!kPlain && p.ep.Z) send(&pp.tmZ, take(), v, n);
                    uint8_t* y = take();
                    if (!kPlain) activate<T, kU / 4>(p.ep.act, reinterpret_cast<float(*)[4]>(v));
                    if (has_r) {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            *reinterpret_cast<uint4*>(y + unit_at(i * 8 + (lane >> 2), lane & 3)) = r[i];
                        __syncwarp();
#pragma unroll
                        for (int j = 0; j < 4; ++j) {
                            const uint4 x = *reinterpret_cast<const uint4*>(y + unit_at(lane, j));
#pragma unroll
                            for (int i = 0; i < E; ++i)
                                v[j * E + i] = fmaf(p.ep.r_scale, piece_get<T>(x, i), v[j * E + i]);
                        }
                        if (c + kU < kC) load_r(n + kU);
                        __syncwarp();  // every row has been read before its lane's outputs take the place
                    }
                    send(&pp.tmY[g], y, v, n);
                };
                // The same without TMA, for rows that it cannot write and for the sums of fp32 operands, which are registers
                // (4096 x 512 -> 4096 with Z 113 us, by units 136; with a residual 132 / 150): turned by way of shared
                // memory (a row a lane in, columns over lanes out; 16-byte pieces at places that leave no bank conflict
                // either way) and stored a value a lane: 4096 x 2048 -> 8191 bf16 89 us (four values a lane, one after
                // the other: 386).
                auto values = [&](int c) {
                    constexpr int kPer = 32 / kU, kMask = kU / 4 - 1;  // rows in 128 bytes; pieces of a row, less one
                    float v[kU];
                    get(c, v);
                    auto piece = [](int r, int j) { return r * kU + ((j ^ (r / kPer & kMask)) << 2); };
                    __syncwarp();  // the unit before has been read
#pragma unroll
                    for (int j = 0; j <= kMask; ++j)
                        *reinterpret_cast<float4*>(blk + piece(lane, j)) =
                            make_float4(v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                    __syncwarp();
                    constexpr int U = 8;  // accesses in flight, of kPer rows each
                    const int sub = lane / kU, col = lane % kU;
                    const int64_t n = n0 + c + col, left = p.ep.M - m0;
                    const int rows = n < p.ep.N ? (int)(left < 32 ? left : 32) : 0;
                    const float bias = !kPlain && p.ep.bias && rows > 0 ? ld1((const T*)p.ep.bias + n) : 0.f;
                    const T* rp = (const T*)p.ep.R + (m0 + sub) * p.ep.ld_r + n;
                    T *y = (T*)p.ep.Y + (m0 + sub) * p.ep.ld_y + n, *z = (T*)p.ep.Z + (m0 + sub) * p.ep.ld_z + n;
#pragma unroll 1
                    for (int r0 = 0; r0 < rows; r0 += U * kPer) {
                        float x[U / 4][4], r[U];
                        const int have = (rows - r0 - sub + kPer - 1) / kPer;  // accesses inside the output
#pragma unroll
                        for (int u = 0; u < U; ++u)
                            x[u / 4][u % 4] = blk[(r0 + u * kPer + sub) * kU + (col ^ ((u & kMask) << 2))] + bias;
                        if (p.ep.R)
#pragma unroll
                            for (int u = 0; u < U; ++u) r[u] = u < have ? ld1(rp + u * kPer * p.ep.ld_r) : 0.f;
                        if (!kPlain && p.ep.Z)
#pragma unroll
                            for (int u = 0; u < U; ++u)
                                if (u < have) st1(z + u * kPer * p.ep.ld_z, x[u / 4][u % 4]);
                        if (!kPlain) activate<T, U / 4>(p.ep.act, x);
                        if (p.ep.R)
#pragma unroll
                            for (int u = 0; u < U; ++u) x[u / 4][u % 4] = fmaf(p.ep.r_scale, r[u], x[u / 4][u % 4]);
#pragma unroll
                        for (int u = 0; u < U; ++u)
                            if (u < have) st1(y + u * kPer * p.ep.ld_y, x[u / 4][u % 4]);
                        rp += U * kPer * p.ep.ld_r, y += U * kPer * p.ep.ld_y, z += U * kPer * p.ep.ld_z;
                    }
                };
                if (has_r) load_r(n0);
                if constexpr (ROUND) {
                    if (lane == 0) bulk_wait_read0();
#pragma unroll
                    for (int c = 0; c < kC; c += kU) values(c);
                } else if constexpr (kHeld) {
                    if (!p.ep.wide) {
                        if (lane == 0) bulk_wait_read0();
#pragma unroll
                        for (int c = 0; c < kC; c += kU) values(c);
                    } else {
#pragma unroll
                        for (int c = 0; c < kC; c += kU) unit(c);
                    }
                } else {
                    if (!(got = wait_for())) return;
                    if (!p.ep.wide) {
                        if (lane == 0) bulk_wait_read0();
#pragma unroll 1
                        for (int c = 0; c < kC; c += kU) values(c);
                    } else {
#pragma unroll 1
                        for (int c = 0; c < kC; c += kU) unit(c);
                    }
                    release();
                }
            };
            if (!ROUND && !(DRAIN && p.drain)) {
                if constexpr (!ROUND) {
                    const uint32_t at = tb + (use & 1u) * BN;
                    if (p.ep.f32)
                        column_units(float(), std::false_type(), [&](int c, float* v) { tmem_load<16>(at + c, v); });
                    else
                        column_units(__nv_bfloat16(), std::false_type(), [&](int c, float* v) { tmem_load<32>(at + c, v); });
                }
            } else if constexpr (ROUND || DRAIN) {
                float acc[kC];
#pragma unroll
                for (int i = 0; i < kC; ++i) acc[i] = 0.f;
                const int windows = ROUND ? p.nk : (p.nk + kWindow - 1) / kWindow;
                for (int w = 0; w < windows; ++w) {
                    if (!(got = wait_for())) break;
                    const uint32_t at = tb + (use % kAcc<ROUND>) * BN;
#pragma unroll
                    for (int c = 0; c < kC; c += 32) {
                        float v[32];
                        tmem_load<32>(at + c, v);
#pragma unroll
                        for (int i = 0; i < 32; ++i) acc[c + i] += v[i];
                    }
                    release();
                }
                if (!got) break;
                column_units(float(), std::true_type(), [&](int c, float* v) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) v[i] = acc[c + i];
                });
            }
          }
        };
        drain(std::integral_constant<int, 0>());
        drain(std::integral_constant<int, 1>());
        if (lane == 0) bulk_wait_all();  // the outputs are written before the CTA exits
        // The leader's last signal comes to the other CTA too: waited for here, where the last tile is done, as a wait
        // from the kernel's start would run into its limit in a long launch.
        if (rank != 0 && warp == 2) wait_settled(smem_u32(mma_done), 0, pp.err);
    }
    __syncwarp();
    tc_fence_before();
    cluster_sync();  // neither CTA leaves while the pair's MMAs, copies or signals may touch it
    if (warp == 1) {
        tc_fence_after();
        pair_dealloc(tmem, S::kCols);
    }
}

// ------------------------------------------------------------------ host side
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                  const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                  CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) ==
                cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = (EncodeTiledFn)f;
    });
    bind_thread_context();
    return fn;
}

// 3-D map over [plane][row][column], 128-byte swizzle, zero fill: boxes of 64 columns x box_rows rows.
bool make_map(CUtensorMap* tm, const LinearOperand& o, int box_rows) {
    EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    cuuint64_t dims[3] = {(cuuint64_t)o.cols, (cuuint64_t)o.rows, (cuuint64_t)o.planes};
    const int64_t plane = o.planes > 1 ? o.plane_stride : o.ld * o.rows;
    cuuint64_t strides[2] = {(cuuint64_t)(o.ld * 2), (cuuint64_t)(plane * 2)};
    cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1};
    cuuint32_t estr[3] = {1, 1, 1};
    return enc(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(o.p), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// The map of an operand whose tile has `extent` values along MN.
bool operand_map(CUtensorMap* tm, const LinearOperand& o, int extent) { return make_map(tm, o, o.mn ? kTK : extent); }

// 2-D map over an output's rows: boxes of 64 bytes x 32 rows, 64-byte swizzle.
bool make_out_map(CUtensorMap* tm, void* p, int64_t rows, int64_t cols, int64_t ld, bool f32) {
    EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    const int el = f32 ? 4 : 2;
    cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows};
    cuuint64_t strides[1] = {(cuuint64_t)(ld * el)};
    cuuint32_t box[2] = {(cuuint32_t)(64 / el), 32};
    cuuint32_t estr[2] = {1, 1};
    return enc(tm, f32 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT32 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, p, dims, strides, box,
               estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_NONE,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}


// The cluster's size, and (second) a chained launch.
void cluster_attributes(cudaLaunchAttribute* at, int size) {
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)size;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
}

struct Product {
    LinearOperand P, Q;
    TileParams p;
    tda_dtype out;
};

// CTAs along K of a tile launch: as many as fit the GPU at once, a few chunks each.
int tile_split(int64_t tiles, int nk, bool round) {
    const int least = round ? 1 : 4;
    const int64_t slots = (int64_t)train_sms() * (round ? 1 : 2);
    int split = 1;
    while (split < 8 && tiles * split * 2 <= slots && nk >= 2 * least * split) split *= 2;
    // clusters of eight find room on three quarters of the SMs at best (fp32 500 x 512 -> 512: 16 clusters of eight
    // 17.7 us, of four 11.0)
    if (split == 8 && tiles * 8 * 4 > slots * 3) split = 4;
    return split;
}

template <int BN, bool ROUND>
cudaError_t run_tile(const Product* const* pr, int count, bool chained, cudaStream_t s) {
    using S = TileShape<BN, ROUND>;
    TileLaunch pp = {};
    int64_t tiles[2] = {0, 0};
    int nk = 1 << 30;
    for (int i = 0; i < count; ++i) {
        const Product& x = *pr[i];
        if (!operand_map(&pp.tmP[i], x.P, kTM) || !operand_map(&pp.tmQ[i], x.Q, BN)) return cudaErrorInvalidValue;
        pp.g[i] = x.p;
        pp.g[i].tiles_p = (x.P.extent() + kTM - 1) / kTM;
        pp.g[i].tiles_q = (x.Q.extent() + BN - 1) / BN;
        tiles[i] = pp.g[i].tiles_p * pp.g[i].tiles_q;
        if (x.p.nk < nk) nk = x.p.nk;
    }
    const int64_t all = tiles[0] + tiles[1];
    const int split = tile_split(all, nk, ROUND);
    if (all * split > 2147483647LL) return cudaErrorInvalidConfiguration;
    pp.g[0].split = pp.g[1].split = split;
    pp.ctas0 = (int)(tiles[0] * split);
    cudaError_t e = smem_attr_once<linear_tile_kernel<BN, ROUND>>((int)S::kSmem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(all * split));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    cluster_attributes(at, split);
    cfg.attrs = at;
    cfg.numAttrs = chained ? 2 : 1;
    note_launches(1);
    return cudaLaunchKernelEx(&cfg, linear_tile_kernel<BN, ROUND>, pp);
}

template <int BN, bool ROUND, bool DRAIN>
cudaError_t run_pair(const Product* const* pr, int count, bool chained, cudaStream_t s) {
    using S = PairShape<BN, ROUND>;
    PairParams pp = {};
    pp.tiles[0] = pp.tiles[1] = 0;
    for (int i = 0; i < count; ++i) {
        const Product& x = *pr[i];
        if (!operand_map(&pp.tmP[i], x.P, kTM) || !operand_map(&pp.tmQ[i], x.Q, BN / 2))
            return cudaErrorInvalidValue;
        const LinearEpilogue& e = x.p.ep;
        if (!ROUND && e.wide &&
            (!make_out_map(&pp.tmY[i], e.Y, e.M, e.N, e.ld_y, e.f32) ||
             (e.Z && !make_out_map(&pp.tmZ, e.Z, e.M, e.N, e.ld_z, e.f32))))
            return cudaErrorInvalidValue;
        pp.g[i] = x.p;
        pp.g[i].tiles_p = (x.P.extent() + 2 * kTM - 1) / (2 * kTM);
        pp.g[i].tiles_q = (x.Q.extent() + BN - 1) / BN;
        pp.tiles[i] = pp.g[i].tiles_p * pp.g[i].tiles_q;
    }
    if (count == 1) {
        pp.g[1] = pp.g[0];
        pp.tmP[1] = pp.tmP[0], pp.tmQ[1] = pp.tmQ[0];
    }
    pp.err = pr[0]->p.err;
    // a tile costs its K loop and about two chunks of set-up
    pp.extra = count == 2 ? (pp.g[0].nk + 2 + (pp.g[1].nk + 2) / 2) / (pp.g[1].nk + 2) : 0;
    cudaError_t e = smem_attr_once<linear_pair_kernel<BN, ROUND, DRAIN>>((int)S::kSmem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = s;
    cudaLaunchAttribute at[2];
    cluster_attributes(at, 2);
    cfg.attrs = at;
    cfg.numAttrs = 1;
    cfg.gridDim = dim3(2);
    const int64_t most = max_clusters_once<linear_pair_kernel<BN, ROUND, DRAIN>>(cfg, 2, train_sms() / 2);
    const int64_t tiles = pp.tiles[0] + pp.tiles[1];
    cfg.gridDim = dim3((unsigned)(2 * (tiles < most ? tiles : most)));
    cfg.numAttrs = chained ? 2 : 1;
    note_launches(1);
    return cudaLaunchKernelEx(&cfg, linear_pair_kernel<BN, ROUND, DRAIN>, pp);
}

template <bool ROUND>
cudaError_t pick_tile(const Product* const* pr, int count, bool chained, cudaStream_t s) {
    const LinearOperand& Q = pr[0]->Q;
    if (count == 1 && Q.extent() <= 32 && !Q.mn) return run_tile<32, ROUND>(pr, count, chained, s);
    if (count == 1 && Q.extent() <= 64) return run_tile<64, ROUND>(pr, count, chained, s);
    return run_tile<128, ROUND>(pr, count, chained, s);
}

}  // namespace

bool linear_tc_available() {
    static std::atomic<int> sm103{-1};
    int v = sm103.load(std::memory_order_relaxed);
    if (v < 0) {
        int dev = 0, major = 0, minor = 0;
        cudaGetDevice(&dev);
        cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
        cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev);
        v = (major == 10 && minor == 3) ? 1 : 0;
        sm103.store(v, std::memory_order_relaxed);
    }
    return v && encode_fn();
}

static Product make_product(const LinearProduct& x, unsigned int* err) {
    Product r;
    // a short side takes the narrow dimension of the tile
    r.p.swap = x.P.extent() <= 64 && x.Q.extent() > x.P.extent();
    r.P = r.p.swap ? x.Q : x.P;
    r.Q = r.p.swap ? x.P : x.Q;
    r.out = x.out;
    r.p.ep = x.ep;
    r.p.ep.f32 = x.out == TDA_F32;
    r.p.nk = (int)((r.P.depth() + kTK - 1) / kTK);
    r.p.drain = x.out == TDA_F32 && r.P.planes == 1 && r.p.nk > kWindow;
    r.p.split = 1;
    r.p.p_mn = r.P.mn;
    r.p.q_mn = r.Q.mn;
    r.p.err = err;
    return r;
}

static int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Tiles of 256 x 256 (fp32 operands: 128) of a product; 0 where a side is too short for them.
static int64_t pair_tiles(const Product& x) {
    return x.p.swap ? 0 : ceil_div(x.P.extent(), 2 * kTM) * ceil_div(x.Q.extent(), x.P.planes == 3 ? 128 : 256);
}

// Estimated times, in chunks of an SM pair (0.36 us; fp32 1.2 us). The pair kernel: its longest list of tiles
// (pair_tile's order), each its chunks and about two more of set-up. Rows that are not aligned cost little more
// (4096 x 2048 -> 8191 89 us, -> 8192 81; taken for 8 or 16 chunks more, the tile kernel was chosen where it is
// slower: 406 x 768 -> 12485 39 us, 28 this way).
static double pair_time(const Product* const* r, int count) {
    const int64_t n = train_sms() / 2, t0 = pair_tiles(*r[0]), c0 = r[0]->p.nk + 2;
    if (count == 1) return (double)(ceil_div(t0, n) * c0);
    const int64_t t1 = pair_tiles(*r[1]), c1 = r[1]->p.nk + 2, idle = n - t0 % n;
    int64_t extra = (c0 + c1 / 2) / c1;
    if (extra > ceil_div(t1, idle)) extra = ceil_div(t1, idle);
    const int64_t left = t1 > extra * idle ? t1 - extra * idle : 0;
    return (double)(t0 / n * c0 + (c0 > extra * c1 ? c0 : extra * c1) + ceil_div(left, n) * c1);
}

// The tile kernel: bf16 CTAs share an SM by twos, at the pace of its operand loads; fp32 CTAs take an SM each, in
// rounds, a chunk 1.4 times as long as a pair's.
static double tile_time(const Product* const* r, int count, bool round) {
    int64_t tiles = 0;
    int most = 0, least = 1 << 30;
    for (int i = 0; i < count; ++i) {
        tiles += ceil_div(r[i]->P.extent(), kTM) * ceil_div(r[i]->Q.extent(), 128);
        if (r[i]->p.nk > most) most = r[i]->p.nk;
        if (r[i]->p.nk < least) least = r[i]->p.nk;
    }
    const int split = tile_split(tiles, least, round);
    const double chunks = (double)ceil_div(most, split), fill = (double)(tiles * split) / train_sms();
    if (round) return (double)ceil_div(tiles * split, train_sms()) * (1.4 * chunks + 4);
    return (fill > 1 ? fill : 1) * chunks + 4;
}

// Which kernel, by these estimates. Whole passes (us, pair / tile): fp32 forward 2048 x 2048 -> 2048 84 / 109,
// 1024 x 2048 -> 1024 45 / 35, backward of 1021 x 1000 -> 1363 58 / 56; bf16 forward 2048 x 2048 -> 2048 17 / 24,
// 700 x 4096 -> 2000 24 / 22, 1024 x 2048 -> 1024 15 / 13. Two products share a launch unless one has few tiles and a
// long K loop, which alone is split over more SMs (backward of 128 x 512 -> 8192, together / apart: bf16 49 / 18,
// fp32 148 / 51).
cudaError_t launch_linear_products(const LinearProduct* x, int count, bool chained, unsigned int* err, cudaStream_t s) {
    Product r[2];
    const Product* order[2];
    bool wide = true;  // both products have whole tiles
    for (int i = 0; i < count; ++i) {
        r[i] = make_product(x[i], err);
        order[i] = &r[i];
        wide = wide && pair_tiles(r[i]) > 0;
    }
    const bool round = r[0].P.planes == 3;
    if (count == 2 && r[1].P.depth() > r[0].P.depth()) order[0] = &r[1], order[1] = &r[0];
    const double never = 1e30, pair = wide ? pair_time(order, count) : never;
    const double tile = wide || count == 1 ? tile_time(order, count, round) : never;
    if (count == 2) {
        double apart = round ? 3 : 10;  // the second launch
        for (int i = 0; i < 2; ++i) {
            const double a = pair_tiles(*order[i]) > 0 ? pair_time(order + i, 1) : never, b = tile_time(order + i, 1, round);
            apart += a < b ? a : b;
        }
        if (apart < pair && apart < tile) {
            for (int i = 0; i < 2; ++i, chained = true) {
                cudaError_t e = launch_linear_products(x + i, 1, chained, err, s);
                if (e != cudaSuccess) return e;
            }
            return cudaSuccess;
        }
    }
    if (pair <= tile) {
        if (round) return run_pair<128, true, false>(order, count, chained, s);
        const bool drain = order[0]->p.drain || (count == 2 && order[1]->p.drain);
        return drain ? run_pair<256, false, true>(order, count, chained, s)
                     : run_pair<256, false, false>(order, count, chained, s);
    }
    return round ? pick_tile<true>(order, count, chained, s) : pick_tile<false>(order, count, chained, s);
}

}  // namespace tda
