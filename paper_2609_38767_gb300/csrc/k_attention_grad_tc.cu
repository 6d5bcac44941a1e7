// k_attention_grad_tc.cu -- the attention's backward pass on the tcgen05 tensor cores, bf16: two kernels that each compute
// the scores again, so that every sum has a fixed order.
//
// attention_dkv_tc_kernel: a CTA has 128 keys of a key/value head and goes over the query tiles that see them, of every head
// that shares them. S^T = K Q^T and dP^T = V dO^T are in TMEM with a key per lane; eight warps (a lane and half of the queries
// per thread) turn S^T into P^T over its own columns, and dP^T into dX^T, both bf16, which are the MMAs' operands from TMEM:
//   dV += P^T dO,  dK += dX^T Q.
// attention_dq_tc_kernel: a CTA has 128 queries of a head; S = Q K^T and dP = dO V^T with a query per lane, dX over the columns
// that S had, dQ += dX K; with a learned bias also the sums of dS along the diagonals.
// The order of MMAs keeps the tensor pipe busy while the warps work: dV(i) S(i+1) | dK(i) dP(i+1), and S(i+1) dP(i+1) | dQ(i).
//
// Warps 0-7: rows; 8: MMAs; 9: TMA; 10 (dQ with a learned bias): sums by bucket. Waits are bounded (about 1 s) and set
// kErrTimeout on expiry.
#include <cuda.h>
#include <math_constants.h>

#include <algorithm>

#include "attention.cuh"
#include "linear.cuh"

namespace tda {
namespace {

#include "tc_ptx.cuh"

#include "attention_tc.cuh"

constexpr int kThreads = 384;  // three warpgroups: 168 registers each at the launch, then 224, 224 and 56

__device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 56;"); }
__device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 224;"); }

// A tile's statistics: -lse times log2 e and -dO.O of 128 queries, as delta_kernel
// writes them; rows that see nothing have -inf and 0.
constexpr uint32_t kStatBytes = 2 * kTileT * 4;

template <int HD>
struct Tiles {
    static constexpr int kPanels = HD / 64;
    static constexpr uint32_t kBytes = kPanels * kPanel;
};

__device__ __forceinline__ bool wait_all(uint64_t* bar, uint32_t parity, volatile int* abort, unsigned int* err) {
    return __all_sync(0xffffffffu, wait_bounded(smem_u32(bar), parity, abort, err));
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src),
                 "r"(bytes), "r"(bar)
                 : "memory");
}
template <int HD>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap* tm, int head, int row, int n, uint32_t bar) {
#pragma unroll
    for (int p = 0; p < Tiles<HD>::kPanels; ++p) tma_load_head(dst + p * kPanel, tm, 64 * p, head, row, n, bar);
}
// 32 columns of an accumulator from column 32 b on, times `by`, into this thread's row of a bf16 tile in shared memory
// (128-byte swizzle, as TMA stores it).
__device__ __forceinline__ void stage_columns(uint32_t t, uint32_t tile, int row, int b, float by, bool any) {
    float o[32];
    tmem_ld32(t + 32 * b, o);
    tmem_wait_ld();
    tmem_use(o);
    const uint32_t at = tile + (b / 2) * kPanel + row * 128;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
        const float* x = o + 8 * g;
        const uint32_t c = (uint32_t)((b & 1) * 4 + g) ^ (row & 7);
        const uint32_t v[4] = {any ? pack_bf16(x[0] * by, x[1] * by) : 0, any ? pack_bf16(x[2] * by, x[3] * by) : 0,
                               any ? pack_bf16(x[4] * by, x[5] * by) : 0, any ? pack_bf16(x[6] * by, x[7] * by) : 0};
        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at + c * 16), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
    }
}

// From a dot product to x and to its slope by the dot product's scaled value.
__device__ __forceinline__ float capped(float dot, float cap, float inv_cap, float* bend) {
    const float t = tanh_any(both(dot * inv_cap)).x;
    *bend = fmaf(-t, t, 1.f);
    return cap * t;
}

// ------------------------------------------------------------------------------------------------ dK, dV
template <int HD>
struct DkvShape {
    static constexpr int kQ = HD == 64 ? 5 : 3, kG = HD == 64 ? 4 : 2;
    static constexpr uint32_t kStats = (2 + kQ + kG) * Tiles<HD>::kBytes;
    static constexpr uint32_t kBars = kStats + kG * kStatBytes, kSmem = kBars + 512;
};
struct DkvBars {
    uint64_t kv_full, q_full[5], q_empty[5], g_full[4], g_empty[4], s_full, p_ready, dp_full, ds_ready, done;
    uint32_t tmem;
    int abort, first, last;
};
static_assert(sizeof(DkvBars) <= 512, "");

template <int HD, bool RICH>
__global__ __launch_bounds__(kThreads, 1) void attention_dkv_tc_kernel(
    const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
    const __grid_constant__ CUtensorMap tmG, const __grid_constant__ CUtensorMap tmdK, const __grid_constant__ CUtensorMap tmdV,
    const Attention a, const AttentionPlan plan, const float* stats, unsigned int* err) {
    using S = DkvShape<HD>;
    constexpr uint32_t kBytes = Tiles<HD>::kBytes;
    constexpr int kPanels = Tiles<HD>::kPanels;
    extern __shared__ __align__(1024) uint8_t raw[];
    const uint32_t base = smem_u32(raw);
    DkvBars& bars = *(DkvBars*)(raw + S::kBars);
    const uint32_t sk = base, sv = base + kBytes, sq = base + 2 * kBytes, sg = sq + S::kQ * kBytes;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const int T = (int)a.T, tiles = (T + kTileT - 1) / kTileT, heads = (int)(a.N * a.KV), group = a.H / a.KV;
    const int kt = (int)(blockIdx.x / heads), n = (int)(blockIdx.x % heads) / a.KV, kv = (int)(blockIdx.x % heads) % a.KV;
    const int k0 = kt * kTileT;
    volatile int* abort = &bars.abort;
    if (base & 1023u) {
        if (threadIdx.x == 0) atomicOr(err, kErrBadLaunch);
        return;
    }
    if (warp == 8) {
        tmem_alloc(smem_u32(&bars.tmem), 512);
        tmem_relinquish();
        if (lane == 0) {
            for (uint64_t* b : {&bars.kv_full, &bars.s_full, &bars.dp_full, &bars.done}) mbar_init(smem_u32(b), 1);
            for (uint64_t* b : {&bars.p_ready, &bars.ds_ready}) mbar_init(smem_u32(b), 256);
            for (int i = 0; i < S::kQ; ++i) mbar_init(smem_u32(&bars.q_full[i]), 1), mbar_init(smem_u32(&bars.q_empty[i]), 1);
            for (int i = 0; i < S::kG; ++i) mbar_init(smem_u32(&bars.g_full[i]), 1), mbar_init(smem_u32(&bars.g_empty[i]), 1 + 8);
            bars.abort = 0, bars.first = tiles, bars.last = -1;
            fence_mbar_init();
        }
        __syncwarp();
        tc_fence_before();
    }
    chain_wait();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars.tmem;
    // the query tiles that see these keys
    if (a.range) {
        for (int t = threadIdx.x; t < tiles; t += kThreads) {
            const AttentionTile& q = plan.tiles[(int64_t)n * tiles + t];
            if (q.lo < k0 + kTileT && q.hi > k0) atomicMin(&bars.first, t), atomicMax(&bars.last, t);
        }
        __syncthreads();
    }
    const int q_first = a.range ? bars.first : a.causal ? kt : 0, q_last = a.range ? bars.last : tiles - 1;
    const int each = q_last - q_first + 1, total = each > 0 ? each * group : 0;
    const uint32_t tS = tmem, tP = tmem + 128, tdV = tmem + 256, tdK = tmem + 256 + HD;

    if (warp < 8) {
        take_registers();
        const int half = warp / 4, row = threadIdx.x % 128, key = k0 + row;
        const uint32_t lanes = (uint32_t)(warp % 4) << 21;
        const uint32_t ts = tS + lanes + 64 * half, tp = tP + lanes + 64 * half;
        const float c = a.scale * kLog2e, inv_cap = RICH && a.cap > 0.f ? a.scale / a.cap : 0.f;
        bool ok = true;
        for (int it = 0; it < total; ++it) {
            const int qt = q_first + it % each, h = kv * group + it / each, q0 = qt * kTileT;
            const int g = it % S::kG;
            bool masked;
            if (a.range) {
                const AttentionTile& t = plan.tiles[(int64_t)n * tiles + qt];
                masked = t.most > k0 || t.least < k0 + kTileT;
            } else {
                masked = (a.causal && q0 < k0 + kTileT) || k0 + kTileT > T;
            }
            // bit j: query q0 + 64 half + j sees the key; more: and another one
            uint32_t seen[2] = {~0u, ~0u}, more[2] = {~0u, ~0u};
            if (masked) {
                if (a.range) {
                    seen[0] = seen[1] = more[0] = more[1] = 0;
                    for (int j = 0; j < 64; ++j) {
                        const int2 v = visible(a.range, 0, T, (int64_t)n * T, q0 + 64 * half + j);
                        const uint32_t in = key >= v.x && key < v.y;
                        seen[j / 32] |= in << (j % 32);
                        more[j / 32] |= (in & (uint32_t)(v.y - v.x > 1)) << (j % 32);
                    }
                } else if (a.causal) {
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        const int from = key - (q0 + 64 * half + 32 * w);  // the first query that sees the key
                        seen[w] = more[w] = from <= 0 ? ~0u : from > 31 ? 0u : ~0u << from;
                        if (q0 + 64 * half + 32 * w == 0) more[w] &= ~1u;
                    }
                } else if (T == 1) {
                    more[0] = more[1] = 0;
                }
            }
            ok = wait_all(&bars.g_full[g], (it / S::kG) & 1, abort, err) && wait_all(&bars.s_full, it & 1, abort, err);
            if (!ok) break;
            tc_fence_after();
            const float4* nl = (const float4*)(raw + S::kStats + g * kStatBytes + 256 * half);
            const float4* nd = (const float4*)(raw + S::kStats + g * kStatBytes + 512 + 256 * half);
            float p[64];
            tmem_ld32(ts, p);
            tmem_ld32(ts + 32, p + 32);
            tmem_wait_ld();
            tmem_use(p);
            tmem_use(p + 32);
            uint32_t w[32];
            const float* bias = nullptr;
            if (RICH && plan.lut) {
                const int apart = min(max(q0 - k0, -plan.reach - 127), plan.reach + 127);
                bias = plan.lut + (int64_t)h * plan.lut_len + plan.lut_mid + apart + 64 * half - row;
            }
#pragma unroll
            for (int j = 0; j < 64; j += 4) {
                const float4 l = nl[j / 4];
                const float less[4] = {l.x, l.y, l.z, l.w};
                float q[4], bend[4] = {1.f, 1.f, 1.f, 1.f};
                if constexpr (RICH) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float x = kLog2e * (a.cap > 0.f ? capped(p[j + e], a.cap, inv_cap, &bend[e]) : p[j + e] * a.scale);
                        if (bias) x += bias[j + e];
                        q[e] = exp2_fast(x + less[e]);
                    }
                } else {
                    const float2 c2 = make_float2(c, c);
                    const float2 u = fma2(make_float2(p[j], p[j + 1]), c2, make_float2(l.x, l.y));
                    const float2 v = fma2(make_float2(p[j + 2], p[j + 3]), c2, make_float2(l.z, l.w));
                    q[0] = exp2_fast(u.x), q[1] = exp2_fast(u.y), q[2] = exp2_fast(v.x), q[3] = exp2_fast(v.y);
                }
                if (masked) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (!(seen[(j + e) / 32] >> ((j + e) % 32) & 1)) q[e] = 0.f;
                }
                w[j / 2] = pack_bf16(q[0], q[1]);
                w[j / 2 + 1] = pack_bf16(q[2], q[3]);
#pragma unroll
                for (int e = 0; e < 4; ++e) p[j + e] = RICH ? q[e] * bend[e] : q[e];
            }
            tmem_st32(ts, w);
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(smem_u32(&bars.p_ready));
            ok = wait_all(&bars.dp_full, it & 1, abort, err);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                float d[32];
                tmem_ld32(tp + 32 * b, d);
                tmem_wait_ld();
                tmem_use(d);
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                    const float4 l = nd[(32 * b + j) / 4];
                    float2 u = add2(make_float2(d[j], d[j + 1]), make_float2(l.x, l.y));
                    float2 v = add2(make_float2(d[j + 2], d[j + 3]), make_float2(l.z, l.w));
                    u = mul2(u, make_float2(p[32 * b + j], p[32 * b + j + 1]));
                    v = mul2(v, make_float2(p[32 * b + j + 2], p[32 * b + j + 3]));
                    if (masked) {
                        const uint32_t m = more[b] >> j;
                        if (!(m & 1)) u.x = 0.f;
                        if (!(m & 2)) u.y = 0.f;
                        if (!(m & 4)) v.x = 0.f;
                        if (!(m & 8)) v.y = 0.f;
                    }
                    w[(32 * b + j) / 2] = pack_bf16(u.x, u.y);
                    w[(32 * b + j) / 2 + 1] = pack_bf16(v.x, v.y);
                }
            }
            tmem_st32(tp, w);
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(smem_u32(&bars.ds_ready));
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars.g_empty[g]));
        }
        // warps 0-3: dV, 4-7: dK, through the shared memory of the first query tiles, which nothing reads any more
        if (ok) ok = wait_all(&bars.done, 0, abort, err);
        if (ok) {
            tc_fence_after();
            const uint32_t tile = sq + half * kBytes;
            const float by = half ? a.scale : 1.f;
#pragma unroll
            for (int b = 0; b < HD / 32; ++b) stage_columns((half ? tdK : tdV) + lanes, tile, row, b, by, total > 0);
            fence_proxy_async();
            if (half) asm volatile("bar.sync 2, 128;" ::: "memory");
            else asm volatile("bar.sync 1, 128;" ::: "memory");
            if (warp % 4 == 0 && elect_one()) {
#pragma unroll
                for (int p = 0; p < kPanels; ++p)
                    if (64 * p < a.hd) tma_store_head(half ? &tmdK : &tmdV, tile + p * kPanel, 64 * p, kv, k0, n);
                asm volatile("cp.async.bulk.commit_group;\n cp.async.bulk.wait_group 0;" ::: "memory");
            }
            __syncwarp();
        }
        tc_fence_before();
    } else {
        give_registers();
        if (warp == 9) {
            if (elect_one()) {
                bool ok = true;
                int it = 0;
                if (total) {
                    mbar_arrive_tx(smem_u32(&bars.kv_full), 2 * kBytes);
                    load_tile<HD>(sk, &tmK, kv, k0, n, smem_u32(&bars.kv_full));
                    load_tile<HD>(sv, &tmV, kv, k0, n, smem_u32(&bars.kv_full));
                }
                for (; it < total; ++it) {
                    const int qt = q_first + it % each, h = kv * group + it / each;
                    const int q = it % S::kQ, g = it % S::kG;
                    if (it >= S::kQ && !(ok = wait_bounded(smem_u32(&bars.q_empty[q]), (it / S::kQ - 1) & 1, abort, err))) break;
                    mbar_arrive_tx(smem_u32(&bars.q_full[q]), kBytes);
                    load_tile<HD>(sq + q * kBytes, &tmQ, h, qt * kTileT, n, smem_u32(&bars.q_full[q]));
                    if (it >= S::kG && !(ok = wait_bounded(smem_u32(&bars.g_empty[g]), (it / S::kG - 1) & 1, abort, err))) {
                        wait_settled(smem_u32(&bars.q_full[q]), (it / S::kQ) & 1, err);
                        break;
                    }
                    mbar_arrive_tx(smem_u32(&bars.g_full[g]), kBytes + kStatBytes);
                    load_tile<HD>(sg + g * kBytes, &tmG, h, qt * kTileT, n, smem_u32(&bars.g_full[g]));
                    bulk_load(base + S::kStats + g * kStatBytes, stats + (((int64_t)n * a.H + h) * tiles + qt) * 2 * kTileT, kStatBytes,
                              smem_u32(&bars.g_full[g]));
                }
                if (total) wait_settled(smem_u32(&bars.kv_full), 0, err);
                for (int s = 0; s < S::kQ; ++s)
                    if (it > s) wait_settled(smem_u32(&bars.q_full[s]), ((it - 1 - s) / S::kQ) & 1, err);
                for (int s = 0; s < S::kG; ++s)
                    if (it > s) wait_settled(smem_u32(&bars.g_full[s]), ((it - 1 - s) / S::kG) & 1, err);
            }
            __syncwarp();
        } else if (warp == 8) {
            const uint32_t lead = elect_one();
            const int steps = (a.hd + 15) / 16;
            constexpr uint32_t kIdS = idesc_bf16(kTileT, kTileT), kIdO = idesc_bf16(kTileT, HD) | kBMn;
            bool ok = true;
            auto tile_of = [&](int it) -> const AttentionTile& { return plan.tiles[(int64_t)n * tiles + q_first + it % each]; };
            auto clear = [&](uint32_t tile, int it) {
                if (!a.range) return;
                uint32_t bits[4];
                *(uint4*)bits = *(const uint4*)tile_of(it).idle;
                if (bits[0] | bits[1] | bits[2] | bits[3]) clear_rows(tile, kPanels, bits);
            };
            auto scores = [&](int it) {
                ok = wait_all(&bars.q_full[it % S::kQ], (it / S::kQ) & 1, abort, err);
                if (!ok) return;
                clear(sq + it % S::kQ * kBytes, it);
                tc_fence_after();
                mma_heads<HD>(lead, tS, sk, sq + it % S::kQ * kBytes, kIdS, steps);
                commit(lead, smem_u32(&bars.s_full));
            };
            auto gradients = [&](int it) {
                ok = wait_all(&bars.g_full[it % S::kG], (it / S::kG) & 1, abort, err);
                if (!ok) return;
                clear(sg + it % S::kG * kBytes, it);
                tc_fence_after();
                mma_heads<HD>(lead, tP, sv, sg + it % S::kG * kBytes, kIdS, steps);
                commit(lead, smem_u32(&bars.dp_full));
            };
            // D += A B, A's halves 64 columns apart
            auto sums = [&](uint32_t d, uint32_t t, uint32_t b, bool first) {
                mma_tokens<64>(lead, d, t, b, kIdO, first);
                mma_tokens<64>(lead, d, t + 64, b + 64 * 128, kIdO, false);
            };
            if (total) ok = wait_all(&bars.kv_full, 0, abort, err);
            if (ok && total) scores(0);
            if (ok && total) gradients(0);
            for (int it = 0; ok && it < total; ++it) {
                ok = wait_all(&bars.p_ready, it & 1, abort, err);
                if (!ok) break;
                tc_fence_after();
                sums(tdV, tS, sg + it % S::kG * kBytes, it == 0);
                commit(lead, smem_u32(&bars.g_empty[it % S::kG]));
                if (it + 1 < total) scores(it + 1);
                ok = ok && wait_all(&bars.ds_ready, it & 1, abort, err);
                if (!ok) break;
                tc_fence_after();
                sums(tdK, tP, sq + it % S::kQ * kBytes, it == 0);
                commit(lead, smem_u32(&bars.q_empty[it % S::kQ]));
                if (it + 1 < total) gradients(it + 1);
            }
            commit(lead, smem_u32(&bars.done));
            wait_settled(smem_u32(&bars.done), 0, err);
        }
    }
    __syncthreads();
    if (warp == 8) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// ------------------------------------------------------------------------------------------------ dQ
template <int HD, bool RICH>
struct DqShape {
    static constexpr int kK = HD == 64 ? 4 : RICH ? 2 : 3, kV = HD == 64 ? 3 : 2;
    static constexpr uint32_t kDiag = (2 + kK + kV) * Tiles<HD>::kBytes;  // RICH: 2 x [8 warps][96] diagonals, then buckets
    static constexpr uint32_t kHist = kDiag + (RICH ? 2 * 8 * 96 * 4 : 0), kSmem = kHist + (RICH ? 1024 * 4 : 0) + 1024;
};
struct DqBars {
    uint64_t q_full, k_full[4], k_empty[4], v_full[3], v_empty[3], s_full[2], dp_full, dp_free, ds_ready, diag_full[2], diag_empty[2], done;
    uint32_t tmem;
    int abort;
    float flat[8][2];
};

template <int HD, bool RICH>
__global__ __launch_bounds__(kThreads, 1) void attention_dq_tc_kernel(
    const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
    const __grid_constant__ CUtensorMap tmG, const __grid_constant__ CUtensorMap tmdQ, const Attention a, const AttentionPlan plan,
    const float* stats, float* part, unsigned int* err) {
    using S = DqShape<HD, RICH>;
    constexpr uint32_t kBytes = Tiles<HD>::kBytes;
    constexpr int kPanels = Tiles<HD>::kPanels;
    extern __shared__ uint8_t raw[];
    __shared__ DqBars bars;
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    uint8_t* from = raw + (base - smem_u32(raw));
    const uint32_t sq = base, sg = base + kBytes, sk = base + 2 * kBytes, sv = sk + S::kK * kBytes;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const int T = (int)a.T, tiles = (T + kTileT - 1) / kTileT, heads = (int)(a.N * a.H);
    const int tile = tiles - 1 - (int)(blockIdx.x / heads);  // long rows first
    const int n = (int)(blockIdx.x % heads) / a.H, h = (int)(blockIdx.x % heads) % a.H, kv = h / (a.H / a.KV);
    const int q0 = tile * kTileT;
    volatile int* abort = &bars.abort;
    if (warp == 8) {
        tmem_alloc(smem_u32(&bars.tmem), 512);
        tmem_relinquish();
        if (lane == 0) {
            for (uint64_t* b : {&bars.q_full, &bars.s_full[0], &bars.s_full[1], &bars.dp_full, &bars.done, &bars.diag_empty[0],
                                &bars.diag_empty[1]})
                mbar_init(smem_u32(b), 1);
            for (uint64_t* b : {&bars.dp_free, &bars.ds_ready, &bars.diag_full[0], &bars.diag_full[1]}) mbar_init(smem_u32(b), 256);
            for (int i = 0; i < S::kK; ++i) mbar_init(smem_u32(&bars.k_full[i]), 1), mbar_init(smem_u32(&bars.k_empty[i]), 1);
            for (int i = 0; i < S::kV; ++i) mbar_init(smem_u32(&bars.v_full[i]), 1), mbar_init(smem_u32(&bars.v_empty[i]), 1);
            bars.abort = 0;
            fence_mbar_init();
        }
        __syncwarp();
        tc_fence_before();
    }
    chain_wait();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = bars.tmem;
    int k_first = 0, k_last, most = 0, least;
    if (a.range) {
        const AttentionTile& t = plan.tiles[(int64_t)n * tiles + tile];
        k_first = t.lo / kTileT, k_last = t.lo < t.hi ? (t.hi - 1) / kTileT : -1, most = t.most, least = t.least;
    } else {
        k_last = (a.causal ? min(q0 + kTileT, T) - 1 : T - 1) / kTileT, least = a.causal ? q0 + 1 : T;
    }
    const int total = k_last >= k_first ? k_last - k_first + 1 : 0;
    const uint32_t tP = tmem + 256, tdQ = tmem + 384;
    const bool learned = RICH && part != nullptr;
    // every distance of the pair of tiles is beyond the table's reach
    auto flat_at = [&](int kt) {
        const int64_t apart = (int64_t)q0 - (int64_t)kt * kTileT;
        return apart - 127 >= a.reach ? 1 : apart + 127 <= -a.reach ? -1 : 0;
    };

    if (warp < 8) {
        take_registers();
        const int half = warp / 4, row = threadIdx.x % 128, i = q0 + row;
        const uint32_t lanes = (uint32_t)(warp % 4) << 21;
        const float c = a.scale * kLog2e, inv_cap = RICH && a.cap > 0.f ? a.scale / a.cap : 0.f;
        const int2 see = visible(a.range, a.causal, T, (int64_t)n * T, i);
        const float* st = stats + (((int64_t)n * a.H + h) * tiles + tile) * 2 * kTileT;
        const float nl = st[row], nd = st[kTileT + row];
        const bool single = see.y - see.x <= 1;
        float flat[2] = {0.f, 0.f};
        uint32_t diags = 0;
        bool ok = true;
        for (int it = 0; it < total; ++it) {
            const int kt = k_first + it, k0 = kt * kTileT;
            const uint32_t ts = tmem + (it & 1) * 128 + lanes + 64 * half;
            const bool masked = most > k0 || least < k0 + kTileT;
            uint32_t seen[2] = {~0u, ~0u};
            if (masked) {
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const int at = k0 + 64 * half + 32 * w;
                    const int lo = min(max(see.x - at, 0), 32), hi = min(max(see.y - at, 0), 32);
                    seen[w] = lo < hi && !single ? (hi == 32 ? ~0u : (1u << hi) - 1) & (~0u << lo) : 0u;
                }
            }
            ok = wait_all(&bars.s_full[it & 1], (it / 2) & 1, abort, err);
            if (!ok) break;
            tc_fence_after();
            float p[64], bend[RICH ? 64 : 1];
            tmem_ld32(ts, p);
            tmem_ld32(ts + 32, p + 32);
            tmem_wait_ld();
            tmem_use(p);
            tmem_use(p + 32);
            if constexpr (RICH) {
                const int apart = min(max(q0 - k0, -plan.reach - 127), plan.reach + 127);
                const float* bias = plan.lut ? plan.lut + (int64_t)h * plan.lut_len + plan.lut_mid + apart + row - 64 * half : nullptr;
#pragma unroll
                for (int j = 0; j < 64; ++j) {
                    bend[j] = 1.f;
                    float x = kLog2e * (a.cap > 0.f ? capped(p[j], a.cap, inv_cap, &bend[j]) : p[j] * a.scale);
                    if (bias) x += bias[-j];
                    p[j] = exp2_fast(x + nl);
                }
            } else {
                const float2 c2 = make_float2(c, c), l2 = make_float2(nl, nl);
#pragma unroll
                for (int j = 0; j < 64; j += 2) {
                    const float2 x = fma2(make_float2(p[j], p[j + 1]), c2, l2);
                    p[j] = exp2_fast(x.x), p[j + 1] = exp2_fast(x.y);
                }
            }
            ok = wait_all(&bars.dp_full, it & 1, abort, err);
            if (!ok) break;
            tc_fence_after();
            uint32_t w[32];
            float acc = 0.f, sum = 0.f;
            const int flat_side = learned ? flat_at(kt) : 0;
            float* diag = nullptr;
            if (learned && flat_side == 0) {
                diag = (float*)(from + S::kDiag) + ((diags & 1) * 8 + warp) * 96;
                if (diags >= 2) {
                    ok = wait_all(&bars.diag_empty[diags & 1], (diags / 2 - 1) & 1, abort, err);
                    if (!ok) break;
                }
            }
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                float d[32];
                tmem_ld32(tP + lanes + 64 * half + 32 * b, d);
                tmem_wait_ld();
                tmem_use(d);
                if (b == 1) {
                    tc_fence_before();
                    mbar_arrive(smem_u32(&bars.dp_free));
                }
                const float2 d2 = make_float2(nd, nd);
#pragma unroll
                for (int j = 0; j < 32; j += 2) {
                    float2 x = mul2(add2(make_float2(d[j], d[j + 1]), d2), make_float2(p[32 * b + j], p[32 * b + j + 1]));
                    if (masked) {
                        const uint32_t m = seen[b] >> j;
                        if (!(m & 1)) x.x = 0.f;
                        if (!(m & 2)) x.y = 0.f;
                    }
                    if constexpr (RICH) {
                        if (diag) {
                            // a diagonal's sum moves down the lanes with the columns and leaves at lane 31
#pragma unroll
                            for (int e = 0; e < 2; ++e) {
                                acc += e ? x.y : x.x;
                                if (lane == 31) diag[31 - (32 * b + j + e) + 63] = acc;
                                if (32 * b + j + e < 63) {
                                    acc = __shfl_up_sync(0xffffffffu, acc, 1);
                                    if (lane == 0) acc = 0.f;
                                }
                            }
                        } else {
                            sum += x.x + x.y;
                        }
                        // masked pairs stay zero whatever their slope is
                        x.x = masked && x.x == 0.f ? 0.f : x.x * bend[32 * b + j];
                        x.y = masked && x.y == 0.f ? 0.f : x.y * bend[32 * b + j + 1];
                    }
                    w[(32 * b + j) / 2] = pack_bf16(x.x, x.y);
                }
            }
            tmem_st32(ts, w);
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(smem_u32(&bars.ds_ready));
            if constexpr (RICH) {
                if (diag) {
                    diag[lane] = acc;  // diagonals lane - 63
                    mbar_arrive(smem_u32(&bars.diag_full[diags & 1]));
                    ++diags;
                } else if (flat_side) {
                    flat[flat_side > 0] += sum;
                }
            }
        }
        if constexpr (RICH) {
            if (learned) {
#pragma unroll
                for (int e = 0; e < 2; ++e) {
#pragma unroll
                    for (int o = 16; o; o >>= 1) flat[e] += __shfl_xor_sync(0xffffffffu, flat[e], o);
                    if (lane == 0) bars.flat[warp][e] = flat[e];
                }
            }
        }
        if (ok) ok = wait_all(&bars.done, 0, abort, err);
        if (ok) {
            tc_fence_after();
            // half of the columns each
#pragma unroll
            for (int b = 0; b < HD / 64; ++b) stage_columns(tdQ + lanes, sq, row, half * (HD / 64) + b, a.scale, total > 0);
            fence_proxy_async();
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if (warp == 0 && elect_one()) {
#pragma unroll
                for (int p = 0; p < kPanels; ++p)
                    if (64 * p < a.hd) tma_store_head(&tmdQ, sq + p * kPanel, 64 * p, h, q0, n);
                asm volatile("cp.async.bulk.commit_group;\n cp.async.bulk.wait_group 0;" ::: "memory");
            }
            __syncwarp();
        }
        tc_fence_before();
    } else {
        give_registers();
        if (warp == 9) {
            if (elect_one()) {
                int it = 0, loaded_v = 0;
                if (total) {
                    mbar_arrive_tx(smem_u32(&bars.q_full), 2 * kBytes);
                    load_tile<HD>(sq, &tmQ, h, q0, n, smem_u32(&bars.q_full));
                    load_tile<HD>(sg, &tmG, h, q0, n, smem_u32(&bars.q_full));
                }
                for (; it < total; ++it) {
                    const int k = it % S::kK, v = it % S::kV, k0 = (k_first + it) * kTileT;
                    if (it >= S::kK && !wait_bounded(smem_u32(&bars.k_empty[k]), (it / S::kK - 1) & 1, abort, err)) break;
                    mbar_arrive_tx(smem_u32(&bars.k_full[k]), kBytes);
                    load_tile<HD>(sk + k * kBytes, &tmK, kv, k0, n, smem_u32(&bars.k_full[k]));
                    if (it >= S::kV && !wait_bounded(smem_u32(&bars.v_empty[v]), (it / S::kV - 1) & 1, abort, err)) {
                        ++it;
                        break;
                    }
                    mbar_arrive_tx(smem_u32(&bars.v_full[v]), kBytes);
                    load_tile<HD>(sv + v * kBytes, &tmV, kv, k0, n, smem_u32(&bars.v_full[v]));
                    ++loaded_v;
                }
                if (total) wait_settled(smem_u32(&bars.q_full), 0, err);
                for (int s = 0; s < S::kK; ++s)
                    if (it > s) wait_settled(smem_u32(&bars.k_full[s]), ((it - 1 - s) / S::kK) & 1, err);
                for (int s = 0; s < S::kV; ++s)
                    if (loaded_v > s) wait_settled(smem_u32(&bars.v_full[s]), ((loaded_v - 1 - s) / S::kV) & 1, err);
            }
            __syncwarp();
        } else if (warp == 8) {
            const uint32_t lead = elect_one();
            const int steps = (a.hd + 15) / 16;
            constexpr uint32_t kIdS = idesc_bf16(kTileT, kTileT), kIdO = idesc_bf16(kTileT, HD) | kBMn;
            bool ok = true;
            auto scores = [&](int it) {
                const uint32_t tile_k = sk + it % S::kK * kBytes;
                ok = wait_all(&bars.k_full[it % S::kK], (it / S::kK) & 1, abort, err);
                if (!ok) return;
                if (a.range) {
                    uint32_t bits[4];
                    *(uint4*)bits = *(const uint4*)plan.tiles[(int64_t)n * tiles + k_first + it].unseen;
                    if (bits[0] | bits[1] | bits[2] | bits[3]) clear_rows(tile_k, kPanels, bits);
                }
                tc_fence_after();
                mma_heads<HD>(lead, tmem + (it & 1) * 128, sq, tile_k, kIdS, steps);
                commit(lead, smem_u32(&bars.s_full[it & 1]));
            };
            auto gradients = [&](int it) {
                ok = wait_all(&bars.v_full[it % S::kV], (it / S::kV) & 1, abort, err);
                if (!ok) return;
                tc_fence_after();
                mma_heads<HD>(lead, tP, sg, sv + it % S::kV * kBytes, kIdS, steps);
                commit(lead, smem_u32(&bars.dp_full));
                commit(lead, smem_u32(&bars.v_empty[it % S::kV]));
            };
            if (total) ok = wait_all(&bars.q_full, 0, abort, err);
            if (ok && total) scores(0);
            if (ok && total) gradients(0);
            for (int it = 0; ok && it < total; ++it) {
                if (it + 1 < total) {
                    scores(it + 1);
                    ok = ok && wait_all(&bars.dp_free, it & 1, abort, err);
                    if (ok) gradients(it + 1);
                }
                ok = ok && wait_all(&bars.ds_ready, it & 1, abort, err);
                if (!ok) break;
                tc_fence_after();
                const uint32_t t = tmem + (it & 1) * 128, tile_k = sk + it % S::kK * kBytes;
                mma_tokens<64>(lead, tdQ, t, tile_k, kIdO, it == 0);
                mma_tokens<64>(lead, tdQ, t + 64, tile_k + 64 * 128, kIdO, false);
                commit(lead, smem_u32(&bars.k_empty[it % S::kK]));
            }
            commit(lead, smem_u32(&bars.done));
            wait_settled(smem_u32(&bars.done), 0, err);
        } else if (RICH && warp == 10 && learned) {
            // sums of the diagonals of each pair of tiles by bucket, in the order of the tiles
            float* hist = (float*)(from + S::kHist);
            for (int b = lane; b < a.n_buckets; b += 32) hist[b] = 0.f;
            __syncwarp();
            uint32_t diags = 0;
            for (int it = 0; it < total; ++it) {
                const int kt = k_first + it;
                if (flat_at(kt)) continue;
                if (!wait_all(&bars.diag_full[diags & 1], (diags / 2) & 1, abort, err)) break;
                const float* diag = (const float*)(from + S::kDiag) + (diags & 1) * 8 * 96;
                for (int x = 0; x < 8; ++x) {
                    const int d = 32 * x + lane - 127;  // of the pair of tiles
                    float v = 0.f;
                    int id = -1;
                    if (d <= 127) {
#pragma unroll
                        for (int w = 0; w < 8; ++w) {
                            const int own = d - 32 * (w % 4) + 64 * (w / 4);
                            if (own >= -63 && own <= 31) v += diag[w * 96 + own + 63];
                        }
                        const int64_t far = min(max((int64_t)q0 - (int64_t)kt * kTileT + d, -a.reach), a.reach);
                        id = a.bucket[far + a.reach];
                        if (id >= a.n_buckets) id = -1;
                    }
                    uint32_t left = __ballot_sync(0xffffffffu, id >= 0);
                    while (left) {
                        const int who = __shfl_sync(0xffffffffu, id, __ffs(left) - 1);
                        const bool in = id == who;
                        float s = in ? v : 0.f;
#pragma unroll
                        for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                        if (lane == 0) hist[who] += s;
                        left &= ~__ballot_sync(0xffffffffu, in);
                    }
                }
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bars.diag_empty[diags & 1]));
                ++diags;
            }
        }
    }
    __syncthreads();
    if (warp == 8) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    } else if (RICH && warp == 10 && learned) {
        float* hist = (float*)(from + S::kHist);
        if (lane == 0) {
            for (int e = 0; e < 2; ++e) {
                float s = 0.f;
                for (int w = 0; w < 8; ++w) s += bars.flat[w][e];
                const int id = a.bucket[e ? 2 * a.reach : 0];
                if (id >= 0 && id < a.n_buckets) hist[id] += s;
            }
        }
        __syncwarp();
        float* mine = part + ((int64_t)h * a.N * tiles + (int64_t)n * tiles + tile) * a.n_buckets;
        for (int b = lane; b < a.n_buckets; b += 32) mine[b] = hist[b];
    }
}

// stats of a tile of 128 queries of a head, 8 lanes per query: -lse and -dO.O.
__global__ __launch_bounds__(256) void attention_stats_kernel(const Attention a, float* stats) {
    const int T = (int)a.T, tiles = (T + kTileT - 1) / kTileT;
    const int64_t at = (int64_t)blockIdx.x * 32 + threadIdx.x / 8;  // over [N][tiles * 128][H]: a token's heads lie together
    const int64_t total = a.N * tiles * kTileT * a.H;
    if (at >= total) return;
    const int h = (int)(at % a.H), sub = threadIdx.x % 8;
    const int64_t token = at / a.H;
    const int i = (int)(token % (tiles * kTileT)), n = (int)(token / (tiles * kTileT));
    float v = 0.f, l = -CUDART_INF_F;
    if (i < T) {
        const int64_t row = (int64_t)n * T + i;
        const __nv_bfloat16 *o = (const __nv_bfloat16*)a.O + row * a.ld_o + h * a.hd, *g = (const __nv_bfloat16*)a.dO + row * a.ld_do + h * a.hd;
        for (int c = sub * 8; c < a.hd; c += 64) {
            const uint4 x = *(const uint4*)(o + c), y = *(const uint4*)(g + c);
            const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v = fmaf(__uint_as_float(xs[e] << 16), __uint_as_float(ys[e] << 16), v);
                v = fmaf(__uint_as_float(xs[e] & 0xffff0000u), __uint_as_float(ys[e] & 0xffff0000u), v);
            }
        }
        l = a.lse[((int64_t)n * a.H + h) * T + i];
    }
#pragma unroll
    for (int o = 4; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    if (sub == 0) {
        const bool none = l == -CUDART_INF_F;
        float* out = stats + (((int64_t)n * a.H + h) * tiles + i / kTileT) * 2 * kTileT + i % kTileT;
        out[0] = none ? -CUDART_INF_F : -l * kLog2e;
        out[kTileT] = none ? 0.f : -v;
    }
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }

template <int HD, bool RICH>
cudaError_t run(const Attention& a, void* ws, unsigned int* err, cudaStream_t s) {
    using Kv = DkvShape<HD>;
    using Q = DqShape<HD, RICH>;
    if (cudaError_t e = smem_attr_once<attention_dkv_tc_kernel<HD, RICH>>(Kv::kSmem)) return e;
    if (cudaError_t e = smem_attr_once<attention_dq_tc_kernel<HD, RICH>>(Q::kSmem)) return e;
    CUtensorMap q, k, v, g, dq, dk, dv;
    auto map = [&](CUtensorMap* m, const void* p, int64_t ld, int heads) {
        return attention_head_map(m, p, ld, heads, a.hd, a.T, a.N, kTileT);
    };
    if (!map(&q, a.Q, a.ld_q, a.H) || !map(&k, a.K, a.ld_k, a.KV) || !map(&v, a.V, a.ld_v, a.KV) || !map(&g, a.dO, a.ld_do, a.H) ||
        !map(&dq, a.dQ, a.ld_dq, a.H) || !map(&dk, a.dK, a.ld_dk, a.KV) || !map(&dv, a.dV, a.ld_dv, a.KV))
        return cudaErrorInvalidValue;
    const int64_t tiles = (a.T + kTileT - 1) / kTileT;
    AttentionPlan plan;
    bool chained;
    if (cudaError_t e = launch_attention_plan(a, ws, &plan, &chained, s)) return e;
    float* stats = (float*)((char*)ws + attention_plan_bytes(a, false));
    float* part = a.dtable ? (float*)((char*)stats + up((size_t)a.N * a.H * tiles * kStatBytes)) : nullptr;
    note_launches(1);
    attention_stats_kernel<<<(unsigned)((a.N * tiles * kTileT * a.H + 31) / 32), 256, 0, s>>>(a, stats);
    if (cudaError_t e = cudaGetLastError()) return e;
    if (cudaError_t e = launch_chained(true, attention_dq_tc_kernel<HD, RICH>, dim3((unsigned)(tiles * a.N * a.H)), dim3(kThreads),
                                       Q::kSmem, s, q, k, v, g, dq, a, plan, (const float*)stats, part, err))
        return e;
    return launch_chained(true, attention_dkv_tc_kernel<HD, RICH>, dim3((unsigned)(tiles * a.N * a.KV)), dim3(kThreads), Kv::kSmem, s, q,
                          k, v, g, dk, dv, a, plan, (const float*)stats, err);
}

}  // namespace

size_t attention_grad_tc_bytes(const Attention& a, bool bound) {
    const int64_t tiles = (a.T + kTileT - 1) / kTileT;
    return attention_plan_bytes(a, bound) + up((size_t)a.N * a.H * tiles * kStatBytes) +
           (a.dtable || bound ? up((size_t)a.N * a.H * tiles * a.n_buckets * 4) : 0);
}

cudaError_t launch_attention_backward_tc(const Attention& a, void* ws, unsigned int* err, float** part, cudaStream_t s) {
    const bool rich = a.cap > 0.f || a.n_buckets || a.slope;
    const int64_t tiles = (a.T + kTileT - 1) / kTileT;
    *part = (float*)((char*)ws + attention_plan_bytes(a, false) + up((size_t)a.N * a.H * tiles * kStatBytes));
    if (a.hd <= 64) return rich ? run<64, true>(a, ws, err, s) : run<64, false>(a, ws, err, s);
    return rich ? run<128, true>(a, ws, err, s) : run<128, false>(a, ws, err, s);
}

}  // namespace tda
