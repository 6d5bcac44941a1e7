// k_attention_grad_tc.cu -- the attention's backward pass on the tcgen05 tensor cores, bf16: two kernels that each compute
// the scores again, so that every sum has a fixed order.
//
// attention_dkv_tc_kernel: a CTA has 128 keys of a key/value head and goes over the query tiles that see them, of every head
// that shares them. S^T = K Q^T and dP^T = V dO^T are in TMEM with a key per lane; sixteen warps (a lane and a quarter of the
// queries per thread) turn S^T into P^T over its own columns, and dP^T into dX^T, both bf16, which are the MMAs' operands from TMEM:
//   dV += P^T dO,  dK += dX^T Q.
// attention_dq_tc_kernel: an item is 128 queries of a head, a CTA per SM takes them in turn; S = Q K^T and dP = dO V^T with a
// query per lane, dX over the columns that S had, dQ += dX K; with a learned bias also the sums of dS along the diagonals.
// The order of MMAs keeps the tensor pipe busy while the warps work: dV(i) S(i+1) | dK(i) dP(i+1), and S(i+1) dP(i+1) | dQ(i).
// 8 x 1024 tokens, 32/8 heads of 128: dQ 102 us, dK and dV 108, the tensor pipe 51 and 68 % active; statistics 23, bound by HBM.
//
// Warps 0-15: rows; 16: MMAs; 17: TMA; 18: biases by distance, in dQ also items and their queries; 19 (dQ): outputs, or sums by
// distance or bucket of a learned bias. Waits are bounded (about 1 s) and set kErrTimeout on expiry.
#include <cuda.h>
#include <math_constants.h>

#include <algorithm>

#include "attention.cuh"
#include "linear.cuh"

namespace tda {
namespace {

#include "tc_ptx.cuh"

#include "attention_tc.cuh"

// Five warpgroups: 96 registers a thread at the launch, then 104 for the four that hold rows and 64 for the fifth, 61,440 in all
// either way. A thread has a row of a pair of tiles and a quarter of the columns: with half of them in half as many warps each warp
// waited for its own instructions (8 x 1024 tokens 283 us, 258 this way).
constexpr int kThreads = 640, kRowWarps = 16;

__device__ __forceinline__ void give_registers() { asm volatile("setmaxnreg.dec.sync.aligned.u32 64;"); }
__device__ __forceinline__ void take_registers() { asm volatile("setmaxnreg.inc.sync.aligned.u32 104;"); }

// A tile's statistics: -lse times log2 e and -dO.O of 128 queries, as delta_kernel
// writes them; rows that see nothing have -inf and 0.
constexpr uint32_t kStatBytes = 2 * kTileT * 4;

template <int HD>
struct Tiles {
    static constexpr int kPanels = HD / 64;
    static constexpr uint32_t kBytes = kPanels * kPanel;
};

__device__ __forceinline__ bool wait_all(uint64_t* bar, uint32_t parity, volatile int* abort, unsigned int* err) {
    return wait_warp(smem_u32(bar), parity, abort, err);
}
__device__ __forceinline__ void arrive_warp(uint64_t* bar) {
    __syncwarp();
    if (threadIdx.x % 32 == 0) mbar_arrive(smem_u32(bar));
}
// D (+)= A B over 128 tokens: A in TMEM, 16 columns of every 32 (the quarters that the row warps write), B [tokens][head] MN-major in
// panels.
__device__ __forceinline__ void mma_quarters(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, bool first) {
    const uint64_t db = mn_major(b, kPanel);
#pragma unroll
    for (int k = 0; k < 8; ++k) mma_ts(lead, d, a + 32 * (k / 2) + 8 * (k % 2), db + (k * 2048 >> 4), idesc, !first || k > 0);
}
// Bits of a 32 x 32 matrix, a row per lane, to its columns.
__device__ __forceinline__ uint32_t transpose_bits(uint32_t x) {
    const int lane = threadIdx.x % 32;
    uint32_t m = 0x0000ffffu;
#pragma unroll
    for (int s = 16; s; s >>= 1, m ^= m << s) {
        const uint32_t y = __shfl_xor_sync(0xffffffffu, x, s);
        x = lane & s ? (x & ~m) | (y >> s & m) : (x & m) | (y << s & ~m);
    }
    return x;
}
// Bits [lo, hi) of a word, the bounds cut to [0, 32].
__device__ __forceinline__ uint32_t bits_of(int lo, int hi) {
    lo = min(max(lo, 0), 32), hi = min(max(hi, 0), 32);
    return lo < hi ? (hi == 32 ? ~0u : (1u << hi) - 1) & (~0u << lo) : 0u;
}
__device__ __forceinline__ float4 add4(float4 a, float4 b) {
    const float2 x = add2(make_float2(a.x, a.y), make_float2(b.x, b.y)), y = add2(make_float2(a.z, a.w), make_float2(b.z, b.w));
    return make_float4(x.x, x.y, y.x, y.y);
}
// Scores times log2 e of a thread's 32 dot products, and in RICH the cap's slope less its sign, t^2 - 1; bias(j): what columns
// j to j + 3 get beside.
template <bool RICH, typename F>
__device__ __forceinline__ void scores_of(const Attention& a, float inv_cap, float* s, float* bend, F&& bias) {
    const float2 c2 = both(a.scale * kLog2e), cap2 = both(a.cap * kLog2e);
    if (RICH && a.cap > 0.f) {
        auto all = [&](auto tanh_of) {
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
                const float4 more = bias(j);
                const float2 t = tanh_of(make_float2(s[j], s[j + 1])), u = tanh_of(make_float2(s[j + 2], s[j + 3]));
                const float2 x = fma2(t, cap2, make_float2(more.x, more.y)), y = fma2(u, cap2, make_float2(more.z, more.w));
                const float2 b = fma2(t, t, both(-1.f)), c = fma2(u, u, both(-1.f));
                s[j] = x.x, s[j + 1] = x.y, s[j + 2] = y.x, s[j + 3] = y.y;
                bend[j] = b.x, bend[j + 1] = b.y, bend[j + 2] = c.x, bend[j + 3] = c.y;
            }
        };
        if (all_near<32>(s, a.near_limit)) all([&](float2 d) { return mul2(d, tanh_near(a, d)); });
        else all([&](float2 d) { return tanh_any(mul2(d, both(inv_cap))); });
    } else {
#pragma unroll
        for (int j = 0; j < 32; j += 4) {
            const float4 more = bias(j);
            const float2 x = fma2(make_float2(s[j], s[j + 1]), c2, make_float2(more.x, more.y));
            const float2 y = fma2(make_float2(s[j + 2], s[j + 3]), c2, make_float2(more.z, more.w));
            s[j] = x.x, s[j + 1] = x.y, s[j + 2] = y.x, s[j + 3] = y.y;
        }
    }
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

// ------------------------------------------------------------------------------------------------ dK, dV
template <int HD, bool RICH>
struct DkvShape {
    static constexpr int kQ = HD == 64 ? 5 : RICH ? 2 : 3, kG = HD == 64 ? 4 : 2;
    static constexpr uint32_t kStats = (2 + kQ + kG) * Tiles<HD>::kBytes;
    static constexpr uint32_t kBias = kStats + kG * kStatBytes;  // RICH: 2 windows of biases
    static constexpr uint32_t kBars = kBias + (RICH ? 8 * kWindow : 0), kSmem = kBars + 512;
};
struct DkvBars {
    uint64_t kv_full, q_full[5], q_empty[5], g_full[4], g_empty[4], s_full, p_ready, dp_full, ds_ready, bias_full[2], bias_empty[2], done;
    uint32_t tmem;
    int abort, first, last;
};
static_assert(sizeof(DkvBars) <= 512, "");

template <int HD, bool RICH>
__global__ __launch_bounds__(kThreads, 1) void attention_dkv_tc_kernel(
    const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
    const __grid_constant__ CUtensorMap tmG, const __grid_constant__ CUtensorMap tmdK, const __grid_constant__ CUtensorMap tmdV,
    const Attention a, const AttentionPlan plan, const float* stats, unsigned int* err) {
    using S = DkvShape<HD, RICH>;
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
    if (warp == kRowWarps) {
        tmem_alloc(smem_u32(&bars.tmem), 512);
        tmem_relinquish();
        if (lane == 0) {
            for (uint64_t* b : {&bars.kv_full, &bars.s_full, &bars.dp_full, &bars.done}) mbar_init(smem_u32(b), 1);
            for (uint64_t* b : {&bars.p_ready, &bars.ds_ready, &bars.bias_empty[0], &bars.bias_empty[1]}) mbar_init(smem_u32(b), kRowWarps);
            for (uint64_t* b : {&bars.bias_full[0], &bars.bias_full[1]}) mbar_init(smem_u32(b), 32);
            for (int i = 0; i < S::kQ; ++i) mbar_init(smem_u32(&bars.q_full[i]), 1), mbar_init(smem_u32(&bars.q_empty[i]), 1);
            for (int i = 0; i < S::kG; ++i) mbar_init(smem_u32(&bars.g_full[i]), 1), mbar_init(smem_u32(&bars.g_empty[i]), 1 + kRowWarps);
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
    // step it: query tile qt of head h
    struct Step {
        int it = 0, qt, h;
    };
    auto begin = [&]() { return Step{0, q_first, kv * group}; };
    auto next = [&](Step& x) {
        ++x.it;
        if (++x.qt > q_last) x.qt = q_first, ++x.h;
    };

    if (warp < kRowWarps) {
        take_registers();
        const int quarter = warp / 4, row = warp % 4 * 32 + lane, key = k0 + row;
        const uint32_t lanes = (uint32_t)(warp % 4) << 21;
        const uint32_t ts = tS + lanes + 32 * quarter, tp = tP + lanes + 32 * quarter;
        const float inv_cap = RICH ? over_cap(a) : 0.f;
        bool ok = true;
        int2 range = make_int2(0, 0);  // what query 32 quarter + lane of the step's tile sees
        auto look = [&](int qt) {
            if (a.range) range = visible(a.range, 0, T, (int64_t)n * T, qt * kTileT + 32 * quarter + lane);
        };
        if (total) look(q_first);
        for (Step x = begin(); x.it < total; next(x)) {
            const int q0 = x.qt * kTileT + 32 * quarter, g = x.it % S::kG;
            // bit j: query q0 + j sees the key; more: and another one
            uint32_t seen, more;
            if (a.range) {
                const uint32_t many = __ballot_sync(0xffffffffu, range.y - range.x > 1);
                const int from = k0 + warp % 4 * 32;
                seen = transpose_bits(bits_of(range.x - from, range.y - from));
                more = seen & many;
                look(x.qt < q_last ? x.qt + 1 : q_first);
            } else {
                seen = more = a.causal ? bits_of(key - q0, 32) : ~0u;
                if (q0 == 0 && (a.causal || T == 1)) more &= ~1u;
            }
            const bool whole = __all_sync(0xffffffffu, more == ~0u), some = __any_sync(0xffffffffu, seen != 0);
            ok = wait_all(&bars.g_full[g], (x.it / S::kG) & 1, abort, err) && wait_all(&bars.s_full, x.it & 1, abort, err);
            if (!ok) break;
            tc_fence_after();
            const float4* nl = (const float4*)(raw + S::kStats + g * kStatBytes) + 8 * quarter;
            const float4* nd = nl + kTileT / 4;
            float p[32], bend[RICH ? 32 : 1];
            tmem_ld32(ts, p);
            const float* bias = nullptr;
            if (RICH && plan.lut) {
                ok = wait_all(&bars.bias_full[x.it & 1], (x.it / 2) & 1, abort, err);
                if (!ok) break;
                bias = (const float*)(raw + S::kBias) + (x.it & 1) * kWindow + window_row(row) + 32 * quarter;
            }
            tmem_wait_ld();
            tmem_use(p);
            uint32_t w[16];
            if (some) {
                if (bias) scores_of<RICH>(a, inv_cap, p, bend, [&](int j) { return add4(nl[j / 4], *(const float4*)(bias + j)); });
                else scores_of<RICH>(a, inv_cap, p, bend, [&](int j) { return nl[j / 4]; });
#pragma unroll
                for (int j = 0; j < 32; ++j) p[j] = exp2_fast(p[j]);
                if (!whole) {
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (!(seen >> j & 1)) p[j] = 0.f;
                }
#pragma unroll
                for (int j = 0; j < 32; j += 2) w[j / 2] = pack_bf16(p[j], p[j + 1]);
                if (RICH && a.cap > 0.f) {
#pragma unroll
                    for (int j = 0; j < 32; j += 2) {
                        const float2 x = mul2(make_float2(p[j], p[j + 1]), make_float2(bend[j], bend[j + 1]));
                        p[j] = x.x, p[j + 1] = x.y;
                    }
                }
            } else {
#pragma unroll
                for (int j = 0; j < 16; ++j) w[j] = 0;
            }
            tmem_st16(ts, w);
            tmem_wait_st();
            tc_fence_before();
            arrive_warp(&bars.p_ready);
            if (RICH && bias && lane == 0) mbar_arrive(smem_u32(&bars.bias_empty[x.it & 1]));
            ok = wait_all(&bars.dp_full, x.it & 1, abort, err);
            if (!ok) break;
            tc_fence_after();
            if (some) {
                float d[32];
                tmem_ld32(tp, d);
                tmem_wait_ld();
                tmem_use(d);
#pragma unroll
                for (int j = 0; j < 32; j += 4) {
                    const float4 l = nd[j / 4];
                    const float2 u = mul2(add2(make_float2(d[j], d[j + 1]), make_float2(l.x, l.y)), make_float2(p[j], p[j + 1]));
                    const float2 v = mul2(add2(make_float2(d[j + 2], d[j + 3]), make_float2(l.z, l.w)), make_float2(p[j + 2], p[j + 3]));
                    d[j] = u.x, d[j + 1] = u.y, d[j + 2] = v.x, d[j + 3] = v.y;
                }
                if (!whole) {
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (!(more >> j & 1)) d[j] = 0.f;
                }
#pragma unroll
                for (int j = 0; j < 32; j += 2) w[j / 2] = pack_bf16(d[j], d[j + 1]);
            }  // else w is zeros still
            tmem_st16(tp, w);
            tmem_wait_st();
            tc_fence_before();
            arrive_warp(&bars.ds_ready);
            if (lane == 0) mbar_arrive(smem_u32(&bars.g_empty[g]));
        }
        // warps 0-7: dV, 8-15: dK, half of the columns each, through the shared memory of the first query tiles, which nothing reads
        // any more
        if (ok) ok = wait_all(&bars.done, 0, abort, err);
        if (ok) {
            tc_fence_after();
            const int second = warp / 8, half = quarter & 1;
            const uint32_t tile = sq + second * kBytes;
            const float by = second ? RICH && a.cap > 0.f ? -a.scale : a.scale : 1.f;  // the slope's sign
#pragma unroll 1
            for (int b = 0; b < HD / 64; ++b)
                stage_columns((second ? tdK : tdV) + lanes, tile, row, half * (HD / 64) + b, by, total > 0);
            fence_proxy_async();
        }
        const int second = warp / 8;
        if (all_came_well(1 + second, 256, ok) && warp % 8 == 0 && elect_one()) {
#pragma unroll
            for (int p = 0; p < kPanels; ++p)
                if (64 * p < a.hd) tma_store_head(second ? &tmdK : &tmdV, sq + second * kBytes + p * kPanel, 64 * p, kv, k0, n);
            asm volatile("cp.async.bulk.commit_group;\n cp.async.bulk.wait_group.read 0;" ::: "memory");
        }
        __syncwarp();
        tc_fence_before();
    } else {
        give_registers();
        if (warp == kRowWarps + 1) {
            const uint32_t lead = elect_one();
            bool ok = true;
            if (total && lead) {
                mbar_arrive_tx(smem_u32(&bars.kv_full), 2 * kBytes);
                load_tile<HD>(sk, &tmK, kv, k0, n, smem_u32(&bars.kv_full));
                load_tile<HD>(sv, &tmV, kv, k0, n, smem_u32(&bars.kv_full));
            }
            int loaded_q = 0, loaded_g = 0;
            for (Step x = begin(); x.it < total; next(x)) {
                const int q = x.it % S::kQ, g = x.it % S::kG;
                if (x.it >= S::kQ) ok = wait_all(&bars.q_empty[q], (x.it / S::kQ - 1) & 1, abort, err);
                if (!ok) break;
                if (lead) {
                    mbar_arrive_tx(smem_u32(&bars.q_full[q]), kBytes);
                    load_tile<HD>(sq + q * kBytes, &tmQ, x.h, x.qt * kTileT, n, smem_u32(&bars.q_full[q]));
                }
                ++loaded_q;
                __syncwarp();
                if (x.it >= S::kG) ok = wait_all(&bars.g_empty[g], (x.it / S::kG - 1) & 1, abort, err);
                if (!ok) break;
                if (lead) {
                    mbar_arrive_tx(smem_u32(&bars.g_full[g]), kBytes + kStatBytes);
                    load_tile<HD>(sg + g * kBytes, &tmG, x.h, x.qt * kTileT, n, smem_u32(&bars.g_full[g]));
                    bulk_load(base + S::kStats + g * kStatBytes, stats + (((int64_t)n * a.H + x.h) * tiles + x.qt) * 2 * kTileT, kStatBytes,
                              smem_u32(&bars.g_full[g]));
                }
                ++loaded_g;
                __syncwarp();
            }
            if (total) wait_settled(smem_u32(&bars.kv_full), 0, err);
            for (int s = 0; s < S::kQ; ++s)
                if (loaded_q > s) wait_settled(smem_u32(&bars.q_full[s]), ((loaded_q - 1 - s) / S::kQ) & 1, err);
            for (int s = 0; s < S::kG; ++s)
                if (loaded_g > s) wait_settled(smem_u32(&bars.g_full[s]), ((loaded_g - 1 - s) / S::kG) & 1, err);
        } else if (warp == kRowWarps) {
            const uint32_t lead = elect_one();
            const int steps = (a.hd + 15) / 16;
            constexpr uint32_t kIdS = idesc_bf16(kTileT, kTileT), kIdO = idesc_bf16(kTileT, HD) | kBMn;
            bool ok = total == 0 || wait_all(&bars.kv_full, 0, abort, err);
            // what a token holds that sees nothing may be anything
            auto clear = [&](uint32_t tile, int qt) {
                if (!a.range) return;
                uint32_t bits[4];
                *(uint4*)bits = *(const uint4*)plan.tiles[(int64_t)n * tiles + qt].idle;
                if (bits[0] | bits[1] | bits[2] | bits[3]) clear_rows(tile, kPanels, bits);
            };
            // dV(i), S(i + 1), dK(i), dP(i + 1); i = -1 has only the two
            Step x = begin();
            for (int it = -1; ok && it < total && total; ++it) {
                const bool more = it + 1 < total;
                if (it >= 0) {
                    ok = wait_all(&bars.p_ready, it & 1, abort, err);
                    if (!ok) break;
                    tc_fence_after();
                    mma_quarters(lead, tdV, tS, sg + it % S::kG * kBytes, kIdO, it == 0);
                    commit(lead, smem_u32(&bars.g_empty[it % S::kG]));
                }
                if (more) {
                    const int s = x.it % S::kQ;
                    ok = wait_all(&bars.q_full[s], (x.it / S::kQ) & 1, abort, err);
                    if (!ok) break;
                    clear(sq + s * kBytes, x.qt);
                    tc_fence_after();
                    mma_heads<HD>(lead, tS, sk, sq + s * kBytes, kIdS, steps);
                    commit(lead, smem_u32(&bars.s_full));
                }
                if (it >= 0) {
                    ok = wait_all(&bars.ds_ready, it & 1, abort, err);
                    if (!ok) break;
                    tc_fence_after();
                    mma_quarters(lead, tdK, tP, sq + it % S::kQ * kBytes, kIdO, it == 0);
                    commit(lead, smem_u32(&bars.q_empty[it % S::kQ]));
                }
                if (more) {
                    const int s = x.it % S::kG;
                    ok = wait_all(&bars.g_full[s], (x.it / S::kG) & 1, abort, err);
                    if (!ok) break;
                    clear(sg + s * kBytes, x.qt);
                    tc_fence_after();
                    mma_heads<HD>(lead, tP, sv, sg + s * kBytes, kIdS, steps);
                    commit(lead, smem_u32(&bars.dp_full));
                    next(x);
                }
            }
            commit(lead, smem_u32(&bars.done));
            wait_settled(smem_u32(&bars.done), 0, err);
        } else if (RICH && warp == kRowWarps + 2 && plan.lut) {
            for (Step x = begin(); x.it < total; next(x)) {
                if (x.it >= 2 && !wait_all(&bars.bias_empty[x.it & 1], (x.it / 2 - 1) & 1, abort, err)) break;
                load_window<false>(plan, x.h, x.qt * kTileT - k0, (float*)(raw + S::kBias) + (x.it & 1) * kWindow);
                mbar_arrive(smem_u32(&bars.bias_full[x.it & 1]));
            }
        }
    }
    __syncthreads();
    if (warp == kRowWarps) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// ------------------------------------------------------------------------------------------------ dQ
template <int HD, bool RICH>
struct DqShape {
    static constexpr int kK = HD == 64 ? 4 : RICH ? 2 : 3, kV = HD == 64 ? 3 : 2;
    static constexpr uint32_t kBias = (2 + kK + kV) * Tiles<HD>::kBytes;  // RICH: 2 windows of biases, 2 x [16 warps][64]
    static constexpr uint32_t kDiag = kBias + (RICH ? 8 * kWindow : 0);  // diagonals, the sums of an item
    static constexpr uint32_t kHalves = kDiag + (RICH ? 2 * kRowWarps * 64 * 4 : 0);  // a warp's diagonals of 16 columns each
    static constexpr uint32_t kHist = kHalves + (RICH ? kRowWarps * 128 * 4 : 0), kSmem = kHist + (RICH ? 1024 * 4 : 0);
};
struct DqBars {
    uint64_t item_full[4], item_empty[4], q_full, q_empty, k_full[4], k_empty[4], v_full[3], v_empty[3], s_full[2], dp_full, dp_free,
        ds_ready[2], dq_done, bias_full[2], bias_empty[2], diag_full[2], diag_empty[2], flat_full, flat_empty, delta_full[4], out_full, done;
    int4 items[4][2];
    float flat[kRowWarps][2], delta[4][kTileT];
    uint32_t tmem;
    int abort;
};
// The query tiles of all heads, long ones first where the mask is causal, and how CTAs take them (see the forward pass).
struct DqItems {
    int total, tiles;
    FastDiv heads, H, group;
};
// An item as warp 18 leaves it for the others, four at a time.
struct DqItem {
    int n, h, tile;  // h < 0: no more
    int first, last, most, least;
};
struct DqReader {
    uint32_t r = 0;
    __device__ __forceinline__ bool next(DqItem& x, DqBars& bars, bool* ok, volatile int* abort, unsigned int* err) {
        *ok = *ok && wait_all(&bars.item_full[r % 4], (r / 4) & 1, abort, err);
        if (!*ok) return false;
        const int4 a = bars.items[r % 4][0], b = bars.items[r % 4][1];
        x.n = a.x, x.h = a.y, x.tile = a.z;
        x.first = b.x, x.last = b.y, x.most = b.z, x.least = b.w;
        arrive_warp(&bars.item_empty[r % 4]);
        ++r;
        return x.h >= 0;
    }
};
// The key tiles of one item after the other. busy: see the forward pass; here the rows' warps wait for dQ's products before they read on.
struct DqWalk {
    DqItem item;
    int kt = 0, last = 0;
    bool valid = true, ended = false;
    DqReader reader;
    __device__ __forceinline__ void next(bool busy, DqBars& bars, bool* ok, volatile int* abort, unsigned int* err) {
        if (kt < last) {
            ++kt;
            return;
        }
        valid = false;
        while (!ended && !valid) {
            ended = !reader.next(item, bars, ok, abort, err);
            valid = !ended && item.first <= item.last;
            if (busy) break;
        }
        kt = item.first, last = item.last;
    }
};
// Lane l of four gets the l-th 16 bytes of each of the four lanes' 64.
__device__ __forceinline__ void transpose_quads(uint4 (&v)[4]) {
    const int lane = threadIdx.x % 32;
    auto swap = [&](uint4& low, uint4& high, int by) {  // the lane without the bit gives its high, the other its low
        const bool up = lane & by;
        uint4 out = up ? low : high;
        out.x = __shfl_xor_sync(0xffffffffu, out.x, by), out.y = __shfl_xor_sync(0xffffffffu, out.y, by);
        out.z = __shfl_xor_sync(0xffffffffu, out.z, by), out.w = __shfl_xor_sync(0xffffffffu, out.w, by);
        if (up) low = out;
        else high = out;
    };
    swap(v[0], v[1], 1), swap(v[2], v[3], 1);
    swap(v[0], v[2], 2), swap(v[1], v[3], 2);
}

template <int HD, bool RICH>
__global__ __launch_bounds__(kThreads, 1) void attention_dq_tc_kernel(
    const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
    const __grid_constant__ CUtensorMap tmG, const __grid_constant__ CUtensorMap tmdQ, const Attention a, const AttentionPlan plan,
    const DqItems items, float* stats,
    float* part, unsigned int* err) {
    using S = DqShape<HD, RICH>;
    constexpr uint32_t kBytes = Tiles<HD>::kBytes;
    constexpr int kPanels = Tiles<HD>::kPanels;
    extern __shared__ __align__(1024) uint8_t raw[];
    __shared__ DqBars bars;
    const uint32_t base = smem_u32(raw);
    const uint32_t sq = base, sg = base + kBytes, sk = base + 2 * kBytes, sv = sk + S::kK * kBytes;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const int T = (int)a.T, tiles = items.tiles;
    volatile int* abort = &bars.abort;
    const bool learned = RICH && part != nullptr;
    const int dense_mid = attention_dense_mid(a);  // where the sums are by distance, the place of distance 0
    const bool dense = dense_mid >= 0;
    if (base & 1023u) {
        if (threadIdx.x == 0) atomicOr(err, kErrBadLaunch);
        return;
    }
    if (warp == kRowWarps) {
        tmem_alloc(smem_u32(&bars.tmem), 512);
        tmem_relinquish();
        if (lane == 0) {
            for (int i = 0; i < 4; ++i) mbar_init(smem_u32(&bars.item_full[i]), 1), mbar_init(smem_u32(&bars.item_empty[i]), kRowWarps + 2 + (!RICH || learned));
            for (uint64_t* b : {&bars.q_full, &bars.q_empty, &bars.s_full[0], &bars.s_full[1], &bars.dp_full, &bars.dq_done, &bars.done,
                                &bars.diag_empty[0], &bars.diag_empty[1], &bars.flat_empty})
                mbar_init(smem_u32(b), 1);
            for (uint64_t* b : {&bars.dp_free, &bars.ds_ready[0], &bars.ds_ready[1], &bars.diag_full[0], &bars.diag_full[1], &bars.bias_empty[0],
                                &bars.bias_empty[1], &bars.flat_full, &bars.out_full})
                mbar_init(smem_u32(b), kRowWarps);
            for (uint64_t* b : {&bars.bias_full[0], &bars.bias_full[1]}) mbar_init(smem_u32(b), 32);
            for (int i = 0; i < 4; ++i) mbar_init(smem_u32(&bars.delta_full[i]), 4);
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
    const uint32_t tP = tmem + 256, tdQ = tmem + 384;
    // every distance of a pair of tiles is beyond the table's reach
    auto flat_at = [&](int tile, int kt) {
        const int64_t apart = ((int64_t)tile - kt) * kTileT;
        return apart - 127 >= a.reach ? 1 : apart + 127 <= -a.reach ? -1 : 0;
    };

    if (warp < kRowWarps) {
        take_registers();
        const int quarter = warp / 4, row = warp % 4 * 32 + lane;
        const uint32_t lanes = (uint32_t)(warp % 4) << 21;
        const float inv_cap = RICH ? over_cap(a) : 0.f;
        const float by = RICH && a.cap > 0.f ? -a.scale : a.scale;  // the slope's sign
        uint32_t it = 0, diags = 0, done = 0, written = 0, sums = 0;  // key tiles, diagonals, outputs, items' sums, rows' sums so far
        float* halves = (float*)(raw + S::kHalves) + warp * 128;
        if (learned)
            for (int i = lane; i < 128; i += 32) halves[i] = 0.f;  // some are never written
        bool ok = true;
        DqReader reader;
        DqItem item, then;
        int2 see, see_then = make_int2(0, 0);
        float2 stat, stat_then = make_float2(0.f, 0.f);
        // the next item and what this thread's row sees and has in it
        auto look = [&]() {
            if (!reader.next(then, bars, &ok, abort, err)) {
                then.h = -1;
                return;
            }
            see_then = visible(a.range, a.causal, T, (int64_t)then.n * T, then.tile * kTileT + row);
            const float* st = stats + (((int64_t)then.n * a.H + then.h) * tiles + then.tile) * 2 * kTileT;
            stat_then = make_float2(st[row], st[kTileT + row]);
        };
        look();
        while (ok && then.h >= 0) {
            item = then, see = see_then, stat = stat_then;
            const int q0 = item.tile * kTileT;
            const float2 nl = both(stat.x);
            float2 nd = both(stat.y);
            const bool single = see.y - see.x <= 1, idle = __any_sync(0xffffffffu, see.x >= see.y);
            float flat[2] = {0.f, 0.f};
            for (int kt = item.first; kt <= item.last; ++kt, ++it) {
                const int k0 = kt * kTileT;
                const uint32_t ts = tmem + (it & 1) * 128 + lanes + 32 * quarter;
                const bool whole = item.most <= k0 && item.least >= k0 + kTileT;
                const int at = k0 + 32 * quarter;
                const uint32_t seen = whole ? ~0u : single ? 0u : bits_of(see.x - at, see.y - at);
                // blocks of 32 x 32 without a gradient leave zeros (packed documents 363 us, 355 so)
                const bool some = __any_sync(0xffffffffu, seen != 0);
                ok = wait_all(&bars.s_full[it & 1], (it / 2) & 1, abort, err);
                if (!ok) break;
                tc_fence_after();
                float p[32], bend[RICH ? 32 : 1];
                tmem_ld32(ts, p);
                const float* bias = nullptr;
                if (RICH && plan.lut) {
                    ok = wait_all(&bars.bias_full[it & 1], (it / 2) & 1, abort, err);
                    if (!ok) break;
                    bias = (const float*)(raw + S::kBias) + (it & 1) * kWindow + window_row(row) + 32 * quarter;
                }
                tmem_wait_ld();
                tmem_use(p);
                if (some) {
                    if (RICH && idle) {  // the queries of rows that see nothing may be anything, and zero times a slope of NaN is NaN
#pragma unroll
                        for (int j = 0; j < 32; ++j) p[j] = see.x < see.y ? p[j] : 0.f;
                    }
                    if (bias) scores_of<RICH>(a, inv_cap, p, bend, [&](int j) { return add4(make_float4(nl.x, nl.x, nl.x, nl.x), *(const float4*)(bias + j)); });
                    else scores_of<RICH>(a, inv_cap, p, bend, [&](int) { return make_float4(nl.x, nl.x, nl.x, nl.x); });
#pragma unroll
                    for (int j = 0; j < 32; ++j) p[j] = exp2_fast(p[j]);
                }
                if (RICH && bias) arrive_warp(&bars.bias_empty[it & 1]);
                ok = wait_all(&bars.dp_full, it & 1, abort, err);
                if (!ok) break;
                tc_fence_after();
                float d[32];
                tmem_ld32(tP + lanes + 32 * quarter, d);
                tmem_wait_ld();
                tmem_use(d);
                // Where all of a row's keys are here, dO.O is the sum of P dP, without the rounding that O was stored with: few keys
                // leave little of dP - dO.O (6 tokens of 2 heads: gradients 0.0046 of their norm off, 0.0023 so). For dK and dV too.
                const bool within = see.x >= k0 && see.y <= k0 + kTileT && !single;
                if (__any_sync(0xffffffffu, within)) {
                    float sum = 0.f;
                    if (some) {
#pragma unroll
                        for (int j = 0; j < 32; ++j) sum = seen >> j & 1 ? fmaf(p[j], d[j], sum) : sum;
                    }
                    bars.delta[quarter][row] = sum;
                    arrive_warp(&bars.delta_full[warp % 4]);
                    ok = wait_all(&bars.delta_full[warp % 4], sums++ & 1, abort, err);
                    if (!ok) break;
                    sum = bars.delta[0][row] + bars.delta[1][row] + bars.delta[2][row] + bars.delta[3][row];
                    if (within) nd = both(-sum);
                    if (quarter == 0 && within) stats[(((int64_t)item.n * a.H + item.h) * tiles + item.tile) * 2 * kTileT + kTileT + row] = -sum;
                }
                tc_fence_before();
                arrive_warp(&bars.dp_free);  // nobody writes to delta again before all have read it
                uint32_t w[16];
                if (some) {
#pragma unroll
                    for (int j = 0; j < 32; j += 2) {
                        const float2 x = mul2(add2(make_float2(d[j], d[j + 1]), nd), make_float2(p[j], p[j + 1]));
                        d[j] = x.x, d[j + 1] = x.y;
                    }
                    if (!whole) {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (!(seen >> j & 1)) d[j] = 0.f;
                    }
                }
                if constexpr (RICH) {
                    if (learned) {
                        if (const int side = flat_at(item.tile, kt)) {
                            if (some) {
                                float sum = 0.f;
#pragma unroll
                                for (int j = 0; j < 32; ++j) sum += d[j];
                                flat[side > 0] += sum;
                            }
                        } else {
                            float* diag = (float*)(raw + S::kDiag) + ((diags & 1) * kRowWarps + warp) * 64;
                            if (some) {
                                // a diagonal's sum moves down the lanes with the columns and leaves at lane 31; of 16 columns at a
                                // time, side by side, as each step waits for the shuffle before it (packed documents 355 us with
                                // all 32 in a row, 331 so, 341 with 8 at a time, whose sums take more to join)
                                float acc[2] = {0.f, 0.f};
#pragma unroll
                                for (int j = 0; j < 16; ++j) {
                                    acc[0] += d[j], acc[1] += d[16 + j];
                                    if (lane == 31) halves[62 - j] = acc[0], halves[64 + 46 - j] = acc[1];  // row - column + 31
                                    if (j < 15) {
#pragma unroll
                                        for (int e = 0; e < 2; ++e) {
                                            acc[e] = __shfl_up_sync(0xffffffffu, acc[e], 1);
                                            if (lane == 0) acc[e] = 0.f;
                                        }
                                    }
                                }
                                if (lane < 31) halves[16 + lane] = acc[0], halves[64 + lane] = acc[1];
                                __syncwarp();
                            }
                            if (diags >= 2) {
                                ok = wait_all(&bars.diag_empty[diags & 1], (diags / 2 - 1) & 1, abort, err);
                                if (!ok) break;
                            }
                            diag[lane] = some ? halves[lane] + halves[64 + lane] : 0.f;
                            if (lane < 31) diag[32 + lane] = some ? halves[32 + lane] + halves[96 + lane] : 0.f;
                            arrive_warp(&bars.diag_full[diags & 1]);
                            ++diags;
                        }
                    }
                }
                if (some) {
                    if (RICH && a.cap > 0.f) {
#pragma unroll
                        for (int j = 0; j < 32; j += 2) {
                            const float2 x = mul2(make_float2(d[j], d[j + 1]), make_float2(bend[j], bend[j + 1]));
                            d[j] = x.x, d[j + 1] = x.y;
                        }
                    }
#pragma unroll
                    for (int j = 0; j < 32; j += 2) w[j / 2] = pack_bf16(d[j], d[j + 1]);
                } else {
#pragma unroll
                    for (int j = 0; j < 16; ++j) w[j] = 0;
                }
                tmem_st16(ts, w);
                tmem_wait_st();
                tc_fence_before();
                // two barriers in turn: a warp may be done with the next pair of tiles (dP is free as soon as all have read it) before another,
                // which has diagonals to sum, is with this one
                arrive_warp(&bars.ds_ready[it & 1]);
            }
            if (!ok) break;
            if constexpr (RICH) {
                if (learned) {
                    if (written++) ok = wait_all(&bars.flat_empty, written & 1, abort, err);
                    if (!ok) break;
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
#pragma unroll
                        for (int o = 16; o; o >>= 1) flat[e] += __shfl_xor_sync(0xffffffffu, flat[e], o);
                        if (lane == 0) bars.flat[warp][e] = flat[e];
                    }
                    arrive_warp(&bars.flat_full);
                }
            }
            const bool any = item.first <= item.last;
            look();  // while the last MMAs are under way
            if (any) ok = ok && wait_all(&bars.dq_done, done++ & 1, abort, err);
            if (!ok) break;
            tc_fence_after();
            if constexpr (RICH) {
                // 32 columns each (all quarters, or the first two), four lanes to 64 bytes of a row on the way out: warp 19 would be
                // late with them here, busy with diagonals (packed documents 330 us, 334 with it)
                if (quarter < HD / 32 && 32 * quarter < a.hd) {
                    float o[32];
                    uint4 v[4];
                    tmem_ld32(tdQ + lanes + 32 * quarter, o);
                    tmem_wait_ld();
                    tmem_use(o);
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const float* x = o + 8 * g;
                        v[g] = any ? make_uint4(pack_bf16(x[0] * by, x[1] * by), pack_bf16(x[2] * by, x[3] * by), pack_bf16(x[4] * by, x[5] * by),
                                                pack_bf16(x[6] * by, x[7] * by))
                                   : make_uint4(0, 0, 0, 0);
                    }
                    transpose_quads(v);
                    const int col = 32 * quarter + lane % 4 * 8, first_row = q0 + warp % 4 * 32 + lane / 4 * 4;
                    __nv_bfloat16* out = (__nv_bfloat16*)a.dQ + ((int64_t)item.n * T + first_row) * a.ld_dq + item.h * a.hd + col;
                    if (col < a.hd) {
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (first_row + k < T) *(uint4*)(out + k * a.ld_dq) = v[k];
                    }
                }
            } else if (any) {
                // to where the last tile of keys was; warp 19 sends them on (8 x 1024 tokens 232 us with the stores above, 227 so)
                if (quarter < HD / 32) stage_columns(tdQ + lanes, sk + (it - 1) % S::kK * kBytes, row, quarter, by, true);
                fence_proxy_async();
                arrive_warp(&bars.out_full);
            } else if (q0 + row < T) {
                uint4* out = (uint4*)((__nv_bfloat16*)a.dQ + ((int64_t)item.n * T + q0 + row) * a.ld_dq + item.h * a.hd);
                for (int c = quarter; c < a.hd / 8; c += 4) out[c] = make_uint4(0, 0, 0, 0);
            }
            tc_fence_before();
        }
    } else {
        give_registers();
        bool ok = true;
        if (warp == kRowWarps + 1) {
            const uint32_t lead = elect_one();
            uint32_t used = 0;  // key tiles so far
            uint32_t loaded_v = 0;
            DqWalk x;
            while (true) {
                x.next(false, bars, &ok, abort, err);
                if (!ok || !x.valid) break;
                const uint32_t k = used % S::kK, v = used % S::kV;
                const int kv = items.group.div(x.item.h), k0 = x.kt * kTileT;
                if (used >= S::kK) ok = wait_all(&bars.k_empty[k], (used / S::kK - 1) & 1, abort, err);
                if (!ok) break;
                if (lead) {
                    mbar_arrive_tx(smem_u32(&bars.k_full[k]), kBytes);
                    load_tile<HD>(sk + k * kBytes, &tmK, kv, k0, x.item.n, smem_u32(&bars.k_full[k]));
                }
                ++used;
                __syncwarp();
                if (loaded_v >= S::kV) ok = wait_all(&bars.v_empty[v], (loaded_v / S::kV - 1) & 1, abort, err);
                if (!ok) break;
                if (lead) {
                    mbar_arrive_tx(smem_u32(&bars.v_full[v]), kBytes);
                    load_tile<HD>(sv + v * kBytes, &tmV, kv, k0, x.item.n, smem_u32(&bars.v_full[v]));
                }
                ++loaded_v;
                __syncwarp();
            }
            for (uint32_t s = 0; s < (uint32_t)S::kK; ++s)
                if (used > s) wait_settled(smem_u32(&bars.k_full[s]), ((used - 1 - s) / S::kK) & 1, err);
            for (uint32_t s = 0; s < (uint32_t)S::kV; ++s)
                if (loaded_v > s) wait_settled(smem_u32(&bars.v_full[s]), ((loaded_v - 1 - s) / S::kV) & 1, err);
        } else if (warp == kRowWarps) {
            const uint32_t lead = elect_one();
            const int steps = (a.hd + 15) / 16;
            constexpr uint32_t kIdS = idesc_bf16(kTileT, kTileT), kIdO = idesc_bf16(kTileT, HD) | kBMn;
            uint32_t it = 0, queries = 0;  // key tiles (`now`), query tiles so far
            DqWalk now, then;
            now.valid = false;
            // S, dP of the key tile after `now`, then dQ of `now`
            while (true) {
                const uint32_t at = now.valid ? it + 1 : it;
                then.next(now.valid, bars, &ok, abort, err);
                if (!ok || (!now.valid && !then.valid)) break;
                if (then.valid) {
                    const uint32_t tile_k = sk + at % S::kK * kBytes;
                    if (then.kt == then.item.first) ok = wait_all(&bars.q_full, queries++ & 1, abort, err);
                    ok = ok && wait_all(&bars.k_full[at % S::kK], (at / S::kK) & 1, abort, err);
                    if (!ok) break;
                    if (a.range) {
                        uint32_t bits[4];
                        *(uint4*)bits = *(const uint4*)plan.tiles[(int64_t)then.item.n * tiles + then.kt].unseen;
                        if (bits[0] | bits[1] | bits[2] | bits[3]) clear_rows(tile_k, kPanels, bits);
                    }
                    tc_fence_after();
                    mma_heads<HD>(lead, tmem + (at & 1) * 128, sq, tile_k, kIdS, steps);
                    commit(lead, smem_u32(&bars.s_full[at & 1]));
                    if (at) ok = wait_all(&bars.dp_free, (at - 1) & 1, abort, err);
                    ok = ok && wait_all(&bars.v_full[at % S::kV], (at / S::kV) & 1, abort, err);
                    if (!ok) break;
                    tc_fence_after();
                    mma_heads<HD>(lead, tP, sg, sv + at % S::kV * kBytes, kIdS, steps);
                    commit(lead, smem_u32(&bars.dp_full));
                    commit(lead, smem_u32(&bars.v_empty[at % S::kV]));
                    if (then.kt == then.last) commit(lead, smem_u32(&bars.q_empty));
                }
                if (now.valid) {
                    ok = wait_all(&bars.ds_ready[it & 1], (it / 2) & 1, abort, err);
                    if (!ok) break;
                    tc_fence_after();
                    mma_quarters(lead, tdQ, tmem + (it & 1) * 128, sk + it % S::kK * kBytes, kIdO, now.kt == now.item.first);
                    if (RICH || now.kt != now.last) commit(lead, smem_u32(&bars.k_empty[it % S::kK]));
                    if (now.kt == now.last) commit(lead, smem_u32(&bars.dq_done));
                    ++it;
                }
                now = then;
            }
            commit(lead, smem_u32(&bars.done));
            wait_settled(smem_u32(&bars.done), 0, err);
        } else if (warp == kRowWarps + 2) {
            // the items, one ahead; the queries and gradients of an item as soon as there is room; its biases
            const uint32_t lead = elect_one();
            uint32_t queries = 0, windows = 0;
            for (uint32_t r = 0;; ++r) {  // makes item r, loads for item r - 1
                if (r && bars.items[(r - 1) % 4][0].y < 0) break;
                if (r >= 4) ok = wait_all(&bars.item_empty[r % 4], (r / 4 - 1) & 1, abort, err);
                if (!ok) break;
                const int g = gridDim.x;
                int id = (int)r * g + (r & 1 ? g - 1 - (int)blockIdx.x : (int)blockIdx.x);
                if (a.range) {
                    if (lane == 0) id = atomicAdd(plan.taken, 1);
                    id = __shfl_sync(0xffffffffu, id, 0);
                }
                int4 x = make_int4(0, -1, 0, 0), y = make_int4(0, -1, 0, 0);
                if ((uint32_t)id < (uint32_t)items.total) {
                    const int tile = tiles - 1 - items.heads.div(id), of = items.heads.mod(id), q0 = tile * kTileT;
                    x = make_int4(items.H.div(of), items.H.mod(of), tile, 0);
                    if (a.range) {
                        const AttentionTile& t = plan.tiles[(int64_t)x.x * tiles + tile];
                        // in range whatever a workspace in other use by now holds
                        const int lo = max(t.lo, 0), hi = min(t.hi, T);
                        y = make_int4(lo / kTileT, lo < hi ? (hi - 1) / kTileT : -1, t.most, t.least);
                    } else {
                        y = make_int4(0, (a.causal ? min(q0 + kTileT, T) - 1 : T - 1) / kTileT, 0, a.causal ? q0 + 1 : T);
                    }
                }
                if (lead) {
                    bars.items[r % 4][0] = x, bars.items[r % 4][1] = y;
                    mbar_arrive(smem_u32(&bars.item_full[r % 4]));
                }
                __syncwarp();
                if (r == 0) continue;
                // nobody can have replaced what this warp made: the slot is free for item r + 3 once its readers have passed it
                x = bars.items[(r - 1) % 4][0], y = bars.items[(r - 1) % 4][1];
                if (y.x > y.y) continue;
                if (queries) ok = wait_all(&bars.q_empty, (queries - 1) & 1, abort, err);
                if (!ok) break;
                if (lead) {
                    mbar_arrive_tx(smem_u32(&bars.q_full), 2 * kBytes);
                    load_tile<HD>(sq, &tmQ, x.y, x.z * kTileT, x.x, smem_u32(&bars.q_full));
                    load_tile<HD>(sg, &tmG, x.y, x.z * kTileT, x.x, smem_u32(&bars.q_full));
                }
                ++queries;
                __syncwarp();
                if (RICH && plan.lut) {
                    for (int kt = y.x; kt <= y.y; ++kt, ++windows) {
                        if (windows >= 2) ok = wait_all(&bars.bias_empty[windows & 1], (windows / 2 - 1) & 1, abort, err);
                        if (!ok) break;
                        load_window<true>(plan, x.y, (x.z - kt) * kTileT, (float*)(raw + S::kBias) + (windows & 1) * kWindow);
                        mbar_arrive(smem_u32(&bars.bias_full[windows & 1]));
                    }
                    if (!ok) break;
                }
            }
            if (queries) wait_settled(smem_u32(&bars.q_full), (queries - 1) & 1, err);
        } else if (!RICH || learned) {
            // the outputs, or the sums of the diagonals of each pair of tiles, in the order of the tiles: by distance where there is
            // room for all of them, else by bucket
            float* hist = (float*)(raw + S::kHist);
            const int width = dense ? 2 * dense_mid + 1 : a.n_buckets;
            for (int i = lane; RICH && i < 2 * kRowWarps; i += 32) ((float*)(raw + S::kDiag))[i * 64 + 63] = 0.f;  // read below, never written
            const uint32_t lead = elect_one();
            uint32_t diags = 0, read = 0, used = 0, outs = 0;
            DqReader reader;
            DqItem item;
            while (reader.next(item, bars, &ok, abort, err)) {
                if constexpr (RICH) {
                    for (int b = lane; b < width; b += 32) hist[b] = 0.f;
                    __syncwarp();
                    for (int kt = item.first; ok && kt <= item.last; ++kt) {
                        if (flat_at(item.tile, kt)) continue;
                        ok = wait_all(&bars.diag_full[diags & 1], (diags / 2) & 1, abort, err);
                        if (!ok) break;
                        const float* diag = (const float*)(raw + S::kDiag) + (diags & 1) * kRowWarps * 64;
#pragma unroll 1
                        for (int x = 0; x < 8; ++x) {
                            // row - column = 32 x - 127 + lane in the pair of tiles; 32 (row quarter - column quarter) is 32 (x - 3) with
                            // lane - 31 left, or 32 (x - 4) with lane + 1
                            float v = 0.f;
#pragma unroll
                            for (int e = 0; e < 2; ++e)
#pragma unroll
                                for (int c = 0; c < 4; ++c) {
                                    const int r = c + x - 3 - e;
                                    if (r >= 0 && r < 4) v += diag[(c * 4 + r) * 64 + lane + 32 * e];
                                }
                            const int64_t apart = ((int64_t)item.tile - kt) * kTileT + 32 * x + lane - 127;
                            const int64_t far = min(max(apart, -a.reach), a.reach);
                            if (dense) {
                                // the distances beyond the table's reach meet, at either end once: with a reach of 0 all are beyond
                                // it, and distance 0 is both ends'
                                float ends[2] = {apart <= -a.reach && apart < a.reach ? v : 0.f, apart >= a.reach ? v : 0.f};
                                if (apart > -a.reach && apart < a.reach && apart >= -dense_mid && apart <= dense_mid) hist[apart + dense_mid] += v;
                                if (__any_sync(0xffffffffu, ends[0] != 0.f || ends[1] != 0.f)) {
#pragma unroll
                                    for (int e = 0; e < 2; ++e) {
#pragma unroll
                                        for (int o = 16; o; o >>= 1) ends[e] += __shfl_xor_sync(0xffffffffu, ends[e], o);
                                        if (lane == 0) hist[e ? 2 * dense_mid : 0] += ends[e];
                                    }
                                }
                                __syncwarp();
                                continue;
                            }
                            int id = a.bucket[far + a.reach];
                            if (id >= a.n_buckets) id = -1;
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
                        arrive_warp(&bars.diag_empty[diags & 1]);
                        ++diags;
                    }
                    ok = ok && wait_all(&bars.flat_full, read++ & 1, abort, err);
                    if (!ok) break;
                    if (lane == 0) {
                        for (int e = 0; e < 2; ++e) {
                            float s = 0.f;
                            for (int w = 0; w < kRowWarps; ++w) s += bars.flat[w][e];
                            const int id = dense ? (e ? 2 * dense_mid : 0) : a.bucket[e ? 2 * a.reach : 0];
                            if (dense || (id >= 0 && id < a.n_buckets)) hist[id] += s;
                        }
                    }
                    arrive_warp(&bars.flat_empty);
                    float* mine = part + ((int64_t)item.h * a.N * tiles + (int64_t)item.n * tiles + item.tile) * width;
                    for (int b = lane; b < width; b += 32) mine[b] = hist[b];
                    __syncwarp();
                }
                if (RICH || item.first > item.last) continue;
                used += item.last - item.first + 1;
                ok = wait_all(&bars.out_full, outs++ & 1, abort, err);
                if (!ok) break;
                const uint32_t at = (used - 1) % S::kK;
                if (lead) {
#pragma unroll
                    for (int p = 0; p < kPanels; ++p)
                        if (64 * p < a.hd) tma_store_head(&tmdQ, sk + at * kBytes + p * kPanel, 64 * p, item.h, item.tile * kTileT, item.n);
                    asm volatile("cp.async.bulk.commit_group;\n cp.async.bulk.wait_group.read 0;" ::: "memory");
                    mbar_arrive(smem_u32(&bars.k_empty[at]));
                }
                __syncwarp();
            }
        }
    }
    __syncthreads();
    if (warp == kRowWarps) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// stats of a tile of 128 queries of a head, LANES lanes a query: -lse log2 e and -dO.O. Bound by reading O and dO.
template <int LANES>
__global__ __launch_bounds__(256) void attention_stats_kernel(const Attention a, const FastDiv heads, int tokens, float* stats) {
    const int T = (int)a.T, tiles = (T + kTileT - 1) / kTileT;
    const int at = (int)(blockIdx.x * (256 / LANES)) + threadIdx.x / LANES, sub = threadIdx.x % LANES;  // over [tokens][H]
    const int token = heads.div(at), h = at - token * a.H;  // a token's heads lie together
    if (token >= tokens) return;
    const int n = token / T, i = token - n * T;
    const __nv_bfloat16 *o = (const __nv_bfloat16*)a.O + (int64_t)token * a.ld_o + h * a.hd,
                        *g = (const __nv_bfloat16*)a.dO + (int64_t)token * a.ld_do + h * a.hd;
    const int64_t where = (int64_t)n * a.H + h;
    const float l = sub == 0 ? a.lse[where * T + i] : 0.f;
    uint4 x[2], y[2];  // 16 values of 16 bytes each at most
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const int c = (sub + e * LANES) * 8;
        x[e] = y[e] = make_uint4(0, 0, 0, 0);
        if (c < a.hd) x[e] = *(const uint4*)(o + c), y[e] = *(const uint4*)(g + c);
    }
    float v = 0.f;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
        const uint32_t xs[4] = {x[e].x, x[e].y, x[e].z, x[e].w}, ys[4] = {y[e].x, y[e].y, y[e].z, y[e].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            v = fmaf(__uint_as_float(xs[k] << 16), __uint_as_float(ys[k] << 16), v);
            v = fmaf(__uint_as_float(xs[k] & 0xffff0000u), __uint_as_float(ys[k] & 0xffff0000u), v);
        }
    }
#pragma unroll
    for (int s = LANES / 2; s; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
    if (sub) return;
    const bool none = l == -CUDART_INF_F;
    float* out = stats + (where * tiles + i / kTileT) * 2 * kTileT + i % kTileT;
    out[0] = none ? -CUDART_INF_F : -l * kLog2e;
    out[kTileT] = none ? 0.f : -v;
    if (i == T - 1)  // the rest of the last tile: no queries
        for (int k = 1; k < tiles * kTileT - i; ++k) out[k] = -CUDART_INF_F, out[kTileT + k] = 0.f;
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }

template <int HD, bool RICH>
cudaError_t run(const Attention& a, void* ws, unsigned int* err, cudaStream_t s) {
    using Kv = DkvShape<HD, RICH>;
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
    // 16 bytes a lane, or twice; a head's last lanes idle where hd is no power of two
    note_launches(1);
    constexpr int kLanes = HD / 16;
    const unsigned grid = (unsigned)((a.N * a.T * a.H + 256 / kLanes - 1) / (256 / kLanes));
    attention_stats_kernel<kLanes><<<grid, 256, 0, s>>>(a, FastDiv(a.H), (int)(a.N * a.T), stats);
    if (cudaError_t e = cudaGetLastError()) return e;
    Attention with = a;
    attention_near(with, 1.f);
    DqItems items;
    items.tiles = (int)tiles, items.total = (int)(tiles * a.N * a.H);
    items.heads = FastDiv((uint32_t)(a.N * a.H)), items.H = FastDiv(a.H), items.group = FastDiv(a.H / a.KV);
    if (cudaError_t e = launch_chained(true, attention_dq_tc_kernel<HD, RICH>, dim3((unsigned)std::min(items.total, train_sms())),
                                       dim3(kThreads), Q::kSmem, s, q, k, v, g, dq, with, plan, items, stats, part, err))
        return e;
    return launch_chained(true, attention_dkv_tc_kernel<HD, RICH>, dim3((unsigned)(tiles * a.N * a.KV)), dim3(kThreads), Kv::kSmem, s, q,
                          k, v, g, dk, dv, with, plan, (const float*)stats, err);
}

}  // namespace

size_t attention_grad_tc_bytes(const Attention& a, bool bound) {
    const int64_t tiles = (a.T + kTileT - 1) / kTileT;
    return attention_plan_bytes(a, bound) + up((size_t)a.N * a.H * tiles * kStatBytes) +
           (a.dtable || bound ? up((size_t)a.N * a.H * tiles * attention_part_width(a) * 4) : 0);
}

cudaError_t launch_attention_backward_tc(const Attention& a, void* ws, unsigned int* err, float** part, cudaStream_t s) {
    const bool rich = a.cap > 0.f || a.n_buckets || a.slope;
    const int64_t tiles = (a.T + kTileT - 1) / kTileT;
    *part = (float*)((char*)ws + attention_plan_bytes(a, false) + up((size_t)a.N * a.H * tiles * kStatBytes));
    if (a.hd <= 64) return rich ? run<64, true>(a, ws, err, s) : run<64, false>(a, ws, err, s);
    return rich ? run<128, true>(a, ws, err, s) : run<128, false>(a, ws, err, s);
}

}  // namespace tda
