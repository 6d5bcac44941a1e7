// k_attention_tc.cu -- the attention's forward pass on the tcgen05 tensor cores, bf16.
//
// An item is 256 queries of a head as two tiles of 128; a CTA goes once over the keys that they see, 128 at a time, with
// the running maximum and sum of each row. One CTA per SM takes items in turn: loads and MMAs of the next begin while the rows
// of the last are still being written. S = Q K^T lands in TMEM with a query per lane; four warps per tile turn it into
// P = 2^(c s - m) there, as bf16 over the columns that S had, and P is the MMA's operand from TMEM for O += P V. The tensor
// pipe works for one tile while the warps of the other have its scores: S0 | P0 V, S0' | P1 V, S1' | ... TMEM holds two
// S and two O tiles of 128 columns, all of its 512.
// O is rescaled only where a row's maximum has grown by more than 2^8 since the last time; P stays below 2^8 then, which
// costs bf16 nothing, and sums are fp32.
//
// Warps 0-3 and 4-7: rows of the tiles (a row per thread); warp 8 issues the MMAs; warp 9 loads by TMA (10 and 11
// are there because registers are shared out by warpgroups). Waits are bounded
// (about 1 s) and set kErrTimeout on expiry.
#include <cuda.h>
#include <math_constants.h>

#include <algorithm>
#include <mutex>

#include "attention.cuh"
#include "linear.cuh"

namespace tda {
namespace {

#include "tc_ptx.cuh"

#include "attention_tc.cuh"

// Three warpgroups, whose registers are shared out anew: 168 each at the launch, then 224 for the two that hold rows of
// scores and 56 for the third, 64,512 in all either way.
constexpr int kThreads = 384;

template <int HD>
struct Shape {
    static constexpr int kPanels = HD / 64;
    static constexpr uint32_t kTileBytes = kPanels * kPanel;
    static constexpr int kStages = HD == 64 ? 6 : 4;
    static constexpr uint32_t kSmem = (2 + kStages) * kTileBytes + 1024;
};

struct Bars {
    uint64_t q_full[2], q_empty[2], s_full[2], p_ready[2], o_done[2], done;
    uint64_t full[8], empty[8];
    uint32_t tmem;
    int abort;
};

// Keys that a tile's queries see, and between which all of them see all.
struct Hull {
    int lo, hi, most, least;
    __device__ __forceinline__ bool any() const { return lo < hi; }
    __device__ __forceinline__ int first() const { return lo / kTileT; }
    __device__ __forceinline__ int last() const { return (hi - 1) / kTileT; }
};
__device__ __forceinline__ Hull hull_of(const Attention& a, const AttentionPlan& plan, int n, int tiles, int tile) {
    const int q0 = tile * kTileT;
    if (q0 >= a.T) return {0, 0, 0, 0};
    if (a.range) {
        const AttentionTile& t = plan.tiles[(int64_t)n * tiles + tile];
        return {t.lo, t.hi, t.most, t.least};
    }
    const int T = (int)a.T;
    return a.causal ? Hull{0, min(q0 + kTileT, T), 0, q0 + 1} : Hull{0, T, 0, T};
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

// The items (pairs of query tiles of a head) of this CTA, long ones first where the mask is causal; every other round
// backwards, which evens out what the rounds leave.
struct Items {
    int total, pairs, heads, H, tiles;
    __device__ __forceinline__ int at(int round) const {
        const int g = gridDim.x, b = blockIdx.x;
        return round * g + (round & 1 ? g - 1 - b : b);
    }
    __device__ __forceinline__ int pair(int item) const { return pairs - 1 - item / heads; }
    __device__ __forceinline__ int example(int item) const { return item % heads / H; }
    __device__ __forceinline__ int head(int item) const { return item % heads % H; }
};

// A key tile of an item, and which tiles of queries see it; next() goes on to the next item with any.
struct Walk {
    int round, item, kt, last, n, first0, last0, first1, last1;
    bool valid;
    __device__ __forceinline__ void start(const Attention& a, const AttentionPlan& plan, const Items& items) {
        round = -1, kt = last = 0;
        next(a, plan, items);
    }
    __device__ __forceinline__ void next(const Attention& a, const AttentionPlan& plan, const Items& items) {
        if (kt < last) {
            ++kt;
            return;
        }
        while (true) {
            item = items.at(++round);
            valid = item < items.total;
            if (!valid) {
                if ((round + 1) * (int)gridDim.x >= items.total) return;
                continue;
            }
            n = items.example(item);
            const int tile = 2 * items.pair(item);
            const Hull a0 = hull_of(a, plan, n, items.tiles, tile), a1 = hull_of(a, plan, n, items.tiles, tile + 1);
            first0 = a0.any() ? a0.first() : 1 << 30, last0 = a0.any() ? a0.last() : -1;
            first1 = a1.any() ? a1.first() : 1 << 30, last1 = a1.any() ? a1.last() : -1;
            kt = min(first0, first1), last = max(last0, last1);
            if (kt <= last) return;
        }
    }
    __device__ __forceinline__ int first_of(int w) const { return w ? first1 : first0; }
    __device__ __forceinline__ int last_of(int w) const { return w ? last1 : last0; }
    __device__ __forceinline__ bool active(int w) const { return kt >= first_of(w) && kt <= last_of(w); }
};

template <int HD, bool RICH>
__global__ __launch_bounds__(kThreads, 1) void attention_tc_kernel(const __grid_constant__ CUtensorMap tmQ,
                                                                   const __grid_constant__ CUtensorMap tmK,
                                                                   const __grid_constant__ CUtensorMap tmV, const Attention a,
                                                                   const AttentionPlan plan, unsigned int* err) {
    using S = Shape<HD>;
    extern __shared__ uint8_t raw[];
    __shared__ Bars bars;
    const uint32_t base = (smem_u32(raw) + 1023u) & ~1023u;
    const uint32_t sq = base, ring = base + 2 * S::kTileBytes;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const int T = (int)a.T;
    Items items;
    items.tiles = (T + kTileT - 1) / kTileT, items.pairs = (items.tiles + 1) / 2, items.H = a.H, items.heads = (int)(a.N * a.H);
    items.total = items.pairs * items.heads;
    volatile int* abort = &bars.abort;

    if (warp == 8) {
        tmem_alloc(smem_u32(&bars.tmem), 512);
        tmem_relinquish();
        if (lane == 0) {
            for (int w = 0; w < 2; ++w) {
                mbar_init(smem_u32(&bars.q_full[w]), 1);
                mbar_init(smem_u32(&bars.q_empty[w]), 1);
                mbar_init(smem_u32(&bars.s_full[w]), 1);
                mbar_init(smem_u32(&bars.p_ready[w]), 128);
                mbar_init(smem_u32(&bars.o_done[w]), 1);
            }
            mbar_init(smem_u32(&bars.done), 1);
            for (int s = 0; s < S::kStages; ++s) mbar_init(smem_u32(&bars.full[s]), 1), mbar_init(smem_u32(&bars.empty[s]), 1);
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

    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        const int w = warp / 4, row = threadIdx.x % 128;
        const uint32_t lanes = (uint32_t)(warp % 4) << 21;  // TMEM lane of the warp's first row
        const uint32_t ts = tmem + lanes + w * 128, to = tmem + lanes + 256 + w * 128;
        const float c = RICH ? kLog2e : a.scale * kLog2e;  // s is x (RICH) or the dot product
        const float grow = 8.f / c, inv_cap = RICH && a.cap > 0.f ? a.scale / a.cap : 0.f;
        bool ok = true;
        uint32_t turn = 0;  // key tiles so far
        for (int round = 0; ok && round * (int)gridDim.x < items.total; ++round) {
            const int item = items.at(round);
            if (item >= items.total) break;
            const int n = items.example(item), h = items.head(item), tile = 2 * items.pair(item) + w, q0 = tile * kTileT, i = q0 + row;
            if (q0 >= T) continue;
            const Hull my = hull_of(a, plan, n, items.tiles, tile);
            const int2 see = visible(a.range, a.causal, T, (int64_t)n * T, i);
            float top = -CUDART_INF_F, sum = 0.f;
            const int first = my.first(), last = my.any() ? my.last() : -1;
            for (int kt = first; kt <= last; ++kt, ++turn) {
                const int k0 = kt * kTileT;
                ok = __all_sync(0xffffffffu, wait_bounded(smem_u32(&bars.s_full[w]), turn & 1, abort, err));
                if (!ok) break;
                tc_fence_after();
                float s[128];
#pragma unroll
                for (int b = 0; b < 4; ++b) tmem_ld32(ts + 32 * b, s + 32 * b);
                tmem_wait_ld();
#pragma unroll
                for (int b = 0; b < 4; ++b) tmem_use(s + 32 * b);
                if constexpr (RICH) {
                    if (a.cap > 0.f) {
#pragma unroll
                        for (int j = 0; j < 128; ++j) s[j] = a.cap * tanh_fast(s[j] * inv_cap);
                    } else {
#pragma unroll
                        for (int j = 0; j < 128; ++j) s[j] *= a.scale;
                    }
                    if (plan.lut) {
                        const int apart = min(max(q0 - k0, -plan.reach - 127), plan.reach + 127);
                        const float* bias = plan.lut + (int64_t)h * plan.lut_len + plan.lut_mid + apart + row;
#pragma unroll
                        for (int j = 0; j < 128; ++j) s[j] += bias[-j];
                    }
                }
                if (my.most > k0 || my.least < k0 + kTileT) {
                    const int lo = see.x - k0;
                    const uint32_t len = (uint32_t)max(see.y - see.x, 0);
#pragma unroll
                    for (int j = 0; j < 128; ++j)
                        if ((uint32_t)(j - lo) >= len) s[j] = -CUDART_INF_F;
                }
                float m4[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
                for (int j = 4; j < 128; ++j) m4[j & 3] = fmaxf(m4[j & 3], s[j]);
                const float most = fmaxf(fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])), top);
                if (kt == first) {
                    top = most;
                } else if (__any_sync(0xffffffffu, most > top + grow)) {
                    ok = __all_sync(0xffffffffu, wait_bounded(smem_u32(&bars.o_done[w]), (turn - 1) & 1, abort, err));
                    if (!ok) break;
                    tc_fence_after();
                    const float by = most == -CUDART_INF_F ? 1.f : exp2_fast((top - most) * c);
                    top = most;
                    sum *= by;
#pragma unroll
                    for (int b = 0; b < HD / 32; ++b) {
                        float o[32];
                        tmem_ld32(to + 32 * b, o);
                        tmem_wait_ld();
                        tmem_use(o);
#pragma unroll
                        for (int j = 0; j < 32; ++j) o[j] *= by;
                        tmem_st32(to + 32 * b, (const uint32_t*)o);
                    }
                }
                const float from = top == -CUDART_INF_F ? 0.f : top;
                uint32_t p[64];
                float2 part[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                const float2 c2 = make_float2(c, c);
                const float2 less = RICH ? make_float2(-from, -from) : make_float2(-from * c, -from * c);
#pragma unroll
                for (int j = 0; j < 64; ++j) {
                    float2 x = make_float2(s[2 * j], s[2 * j + 1]);
                    // the score less the maximum first where a bias may be as large as fp32 goes
                    x = RICH ? mul2(add2(x, less), c2) : fma2(x, c2, less);
                    x.x = exp2_fast(x.x), x.y = exp2_fast(x.y);
                    part[j & 1] = add2(part[j & 1], x);
                    p[j] = pack_bf16(x.x, x.y);
                }
                tmem_st32(ts, p);
                tmem_st32(ts + 32, p + 32);
                sum += part[0].x + part[0].y + part[1].x + part[1].y;
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(smem_u32(&bars.p_ready[w]));
            }
            if (ok && first <= last)
                ok = __all_sync(0xffffffffu, wait_bounded(smem_u32(&bars.o_done[w]), (turn - 1) & 1, abort, err));
            if (!ok) break;
            tc_fence_after();
            const float by = sum != 0.f ? 1.f / sum : 0.f;  // NaN sums stay NaN
            if (a.lse && i < T)
                a.lse[((int64_t)n * a.H + h) * T + i] = sum != 0.f ? fmaf(top, RICH ? 1.f : a.scale, logf(sum)) : -CUDART_INF_F;
            __nv_bfloat16* out = (__nv_bfloat16*)a.O + ((int64_t)n * T + i) * a.ld_o + h * a.hd;
#pragma unroll
            for (int b = 0; b < HD / 32; ++b) {
                float o[32];
                tmem_ld32(to + 32 * b, o);
                tmem_wait_ld();
                tmem_use(o);
                if (i < T) {
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        if (32 * b + 8 * g >= a.hd) continue;
                        uint4 v = make_uint4(0, 0, 0, 0);
                        if (by != 0.f) {  // rows that see nothing: TMEM may hold anything
                            const float* x = o + 8 * g;
                            v = make_uint4(pack_bf16(x[0] * by, x[1] * by), pack_bf16(x[2] * by, x[3] * by),
                                           pack_bf16(x[4] * by, x[5] * by), pack_bf16(x[6] * by, x[7] * by));
                        }
                        *(uint4*)(out + 32 * b + 8 * g) = v;
                    }
                }
            }
        }
        tc_fence_before();
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == 9) {
            if (elect_one()) {
                uint32_t used = 0, queries[2] = {0, 0};  // loads so far
                Walk at;
                bool ok = true;
                auto load = [&](const CUtensorMap* tm, int kv) {
                    const uint32_t s = used % S::kStages, turn = used / S::kStages;
                    if (turn && !wait_bounded(smem_u32(&bars.empty[s]), (turn - 1) & 1, abort, err)) return false;
                    const uint32_t bar = smem_u32(&bars.full[s]);
                    mbar_arrive_tx(bar, S::kTileBytes);
                    for (int p = 0; p < S::kPanels; ++p)
                        tma_load_head(ring + s * S::kTileBytes + p * kPanel, tm, 64 * p, kv, at.kt * kTileT, at.n, bar);
                    ++used;
                    return true;
                };
                auto load_q = [&](int w, int h, int pair) {
                    if (at.first_of(w) > at.last_of(w)) return true;
                    if (queries[w] && !wait_bounded(smem_u32(&bars.q_empty[w]), (queries[w] - 1) & 1, abort, err)) return false;
                    const uint32_t bar = smem_u32(&bars.q_full[w]);
                    mbar_arrive_tx(bar, S::kTileBytes);
                    for (int p = 0; p < S::kPanels; ++p)
                        tma_load_head(sq + w * S::kTileBytes + p * kPanel, &tmQ, 64 * p, h, (2 * pair + w) * kTileT, at.n, bar);
                    ++queries[w];
                    return true;
                };
                for (at.start(a, plan, items); ok && at.valid; at.next(a, plan, items)) {
                    const int h = items.head(at.item), pair = items.pair(at.item), kv = h / (a.H / a.KV);
                    const bool first = at.kt == min(at.first0, at.first1);
                    if (first) ok = load_q(0, h, pair);
                    ok = ok && load(&tmK, kv);
                    if (first) ok = ok && load_q(1, h, pair);
                    ok = ok && load(&tmV, kv);
                }
#pragma unroll
                for (int w = 0; w < 2; ++w)
                    if (queries[w]) wait_settled(smem_u32(&bars.q_full[w]), (queries[w] - 1) & 1, err);
                for (uint32_t s = 0; s < (uint32_t)S::kStages; ++s)
                    if (used > s) wait_settled(smem_u32(&bars.full[s]), ((used - 1 - s) / S::kStages) & 1, err);
            }
            __syncwarp();
        } else if (warp == 8) {
            const uint32_t lead = elect_one();
            const int steps = (a.hd + 15) / 16;
            constexpr uint32_t kIdS = idesc_bf16(kTileT, kTileT), kIdO = idesc_bf16(kTileT, HD) | kBMn;
            uint32_t queries[2] = {0, 0}, weights[2] = {0, 0};  // query tiles, key tiles so far
            uint32_t used = 0;                                  // stages so far: K, V, K, V ...
            auto full = [&](uint32_t at) {
                return __all_sync(0xffffffffu, wait_bounded(smem_u32(&bars.full[at % S::kStages]), (at / S::kStages) & 1, abort, err));
            };
            auto release = [&](uint32_t at) { commit(lead, smem_u32(&bars.empty[at % S::kStages])); };
            auto stage = [&](uint32_t at) { return ring + (at % S::kStages) * S::kTileBytes; };
            bool ok = true;
            // scores of tile w with the keys of stage `at`
            auto scores = [&](const Walk& k, int w, uint32_t at) {
                if (k.kt == k.first_of(w)) {
                    ok = __all_sync(0xffffffffu, wait_bounded(smem_u32(&bars.q_full[w]), queries[w] & 1, abort, err));
                    if (!ok) return;
                    ++queries[w];
                }
                tc_fence_after();
                mma_heads(lead, tmem + w * 128, sq + w * S::kTileBytes, kPanel, stage(at), kPanel, kIdS, steps);
                commit(lead, smem_u32(&bars.s_full[w]));
                if (k.kt == k.last_of(w)) commit(lead, smem_u32(&bars.q_empty[w]));
            };
            uint32_t bits[4], next[4];
            auto unseen = [&](const Walk& k) {
                if (a.range && k.valid) *(uint4*)next = *(const uint4*)plan.tiles[(int64_t)k.n * items.tiles + k.kt].unseen;
            };
            Walk now;
            now.start(a, plan, items);
            if (now.valid) {
                unseen(now);
                ok = full(0);
#pragma unroll
                for (int w = 0; w < 2; ++w)
                    if (ok && now.active(w)) scores(now, w, 0);
                if (ok) release(0);
                used = 1;
            }
            while (ok && now.valid) {
                const uint32_t at_v = used, at_k = used + 1;
                Walk then = now;
                then.next(a, plan, items);
                *(uint4*)bits = *(const uint4*)next;
                unseen(then);
                ok = full(at_v);
                if (!ok) break;
                if (a.range && (bits[0] | bits[1] | bits[2] | bits[3])) clear_rows(stage(at_v), S::kPanels, bits);
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    if (ok && now.active(w)) {
                        ok = __all_sync(0xffffffffu, wait_bounded(smem_u32(&bars.p_ready[w]), weights[w] & 1, abort, err));
                        if (ok) {
                            tc_fence_after();
                            mma_tokens<kTileT>(lead, tmem + 256 + w * 128, tmem + w * 128, stage(at_v), kPanel, kIdO,
                                               now.kt == now.first_of(w));
                            commit(lead, smem_u32(&bars.o_done[w]));
                            ++weights[w];
                        }
                    }
                    if (w == 0 && ok && then.valid) ok = full(at_k);
                    if (ok && then.valid && then.active(w)) scores(then, w, at_k);
                }
                if (!ok) break;
                release(at_v);
                if (then.valid) release(at_k);
                used += 2;
                now = then;
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

// One CTA per tile of 128 tokens and example: what its queries see, and which of its tokens nothing sees; the CTAs
// behind them fill the biases by distance.
__global__ __launch_bounds__(256) void attention_plan_kernel(const Attention a, const AttentionPlan plan, int ranged) {
    const int t = threadIdx.x;
    if ((int)blockIdx.x >= ranged) {
        const int64_t at = (int64_t)(blockIdx.x - ranged) * 256 + t;
        if (at < (int64_t)a.H * plan.lut_len) {
            const int h = (int)(at / plan.lut_len);
            plan.lut[at] = distance_bias(a.bucket, (const __nv_bfloat16*)a.table, a.slope, a.n_buckets, a.reach, a.H, h,
                                         at % plan.lut_len - plan.lut_mid);
        }
        return;
    }
    __shared__ AttentionTile tile;
    const int T = (int)a.T, tiles = (T + kTileT - 1) / kTileT, n = blockIdx.x / tiles, k0 = (int)(blockIdx.x % tiles) * kTileT;
    const int2* range = a.range + (int64_t)n * T;
    if (t == 0) {
        tile.lo = INT32_MAX, tile.hi = 0, tile.most = 0, tile.least = INT32_MAX;
        for (int w = 0; w < 4; ++w) tile.unseen[w] = tile.idle[w] = 0;
    }
    __syncthreads();
    if (t < kTileT) {
        const int2 r = visible(a.range, 0, T, (int64_t)n * T, k0 + t);
        const bool none = r.x >= r.y;
        if (k0 + t < T) {
            if (none) {
                atomicMin(&tile.least, 0);
            } else {
                atomicMin(&tile.lo, r.x), atomicMax(&tile.hi, r.y), atomicMax(&tile.most, r.x), atomicMin(&tile.least, r.y);
            }
        }
        const uint32_t idle = __ballot_sync(0xffffffffu, none && k0 + t < T);
        if (t % 32 == 0) tile.idle[t / 32] = idle;
    }
    uint32_t seen[4] = {0, 0, 0, 0};
    for (int i = t; i < T; i += 256) {
        const int2 r = range[i];
        const int lo = max(r.x, 0) - k0, hi = min(r.y, T) - k0;
        if (hi <= 0 || lo >= kTileT || lo >= hi) continue;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int x = min(max(lo - 32 * w, 0), 32), y = min(max(hi - 32 * w, 0), 32);
            if (x < y) seen[w] |= (y == 32 ? ~0u : (1u << y) - 1) & (~0u << x);
        }
    }
    __shared__ uint32_t all[4];
    if (t < 4) all[t] = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const uint32_t v = __reduce_or_sync(0xffffffffu, seen[w]);
        if (t % 32 == 0) atomicOr(&all[w], v);
    }
    __syncthreads();
    if (t < 4) {
        const int in = min(max(T - k0 - 32 * t, 0), 32);  // tokens of the example
        tile.unseen[t] = ~all[t] & (in == 32 ? ~0u : (1u << in) - 1);
    }
    __syncthreads();
    static_assert(sizeof(AttentionTile) == 48, "");
    if (t < 12) ((uint32_t*)&plan.tiles[blockIdx.x])[t] = ((const uint32_t*)&tile)[t];
}

typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiledFn encode_fn() {
    static EncodeTiledFn fn = nullptr;
    static std::once_flag once;
    std::call_once(once, [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &q) == cudaSuccess &&
            q == cudaDriverEntryPointSuccess)
            fn = (EncodeTiledFn)f;
    });
    bind_thread_context();
    return fn;
}

bool head_rows(const void* p, int64_t ld, int64_t T) {
    return (((uintptr_t)p | (uintptr_t)(ld * 2)) & 15) == 0 && T < (1LL << 39) / std::max<int64_t>(ld, 1);
}

size_t up(size_t n) { return (n + 255) / 256 * 256; }

int lut_reach(const Attention& a, bool bound) {
    return (int)((a.slope || bound) ? a.T - 1 : std::min(a.reach, a.T - 1));
}
bool has_lut(const Attention& a, bool bound) { return a.n_buckets || a.slope || bound; }

template <int HD, bool RICH>
cudaError_t run(const Attention& a, void* ws, unsigned int* err, cudaStream_t s) {
    using Sh = Shape<HD>;
    if (cudaError_t e = smem_attr_once<attention_tc_kernel<HD, RICH>>(Sh::kSmem)) return e;
    CUtensorMap q, k, v;
    if (!attention_head_map(&q, a.Q, a.ld_q, a.H, a.hd, a.T, a.N, kTileT) ||
        !attention_head_map(&k, a.K, a.ld_k, a.KV, a.hd, a.T, a.N, kTileT) ||
        !attention_head_map(&v, a.V, a.ld_v, a.KV, a.hd, a.T, a.N, kTileT))
        return cudaErrorInvalidValue;
    AttentionPlan plan;
    bool chained;
    if (cudaError_t e = launch_attention_plan(a, ws, &plan, &chained, s)) return e;
    const int64_t tiles = (a.T + kTileT - 1) / kTileT;
    const int64_t items = (tiles + 1) / 2 * a.N * a.H;
    return launch_chained(chained, attention_tc_kernel<HD, RICH>, dim3((unsigned)std::min<int64_t>(items, train_sms())), dim3(kThreads),
                          Sh::kSmem, s, q, k, v, a, plan, err);
}

}  // namespace

bool attention_tc_supported(const Attention& a, bool backward) {
    bool ok = a.dt == TDA_BF16 && a.hd % 8 == 0 && head_rows(a.Q, a.ld_q, a.T) && head_rows(a.K, a.ld_k, a.T) &&
              head_rows(a.V, a.ld_v, a.T) && head_rows(a.O, a.ld_o, a.T);
    if (backward)
        ok = ok && head_rows(a.dO, a.ld_do, a.T) && head_rows(a.dQ, a.ld_dq, a.T) && head_rows(a.dK, a.ld_dk, a.T) &&
             head_rows(a.dV, a.ld_dv, a.T);
    return ok && linear_tc_available();
}

size_t attention_plan_bytes(const Attention& a, bool bound) {
    size_t n = 0;
    if (a.range || bound) n += up((size_t)a.N * ((a.T + kTileT - 1) / kTileT) * sizeof(AttentionTile));
    if (has_lut(a, bound)) n += up((size_t)a.H * (2 * lut_reach(a, bound) + 513) * 4);
    return n;
}

cudaError_t launch_attention_plan(const Attention& a, void* ws, AttentionPlan* plan, bool* chained, cudaStream_t s) {
    *plan = {};
    const int64_t tiles = (a.T + kTileT - 1) / kTileT;
    int64_t ranged = 0, filled = 0;
    char* at = (char*)ws;
    if (a.range) {
        plan->tiles = (AttentionTile*)at;
        at += up((size_t)a.N * tiles * sizeof(AttentionTile));
        ranged = a.N * tiles;
    }
    if (has_lut(a, false)) {
        plan->lut = (float*)at;
        plan->reach = lut_reach(a, false);
        plan->lut_len = 2 * plan->reach + 513;
        plan->lut_mid = plan->reach + 256;
        filled = ((int64_t)a.H * plan->lut_len + 255) / 256;
    }
    *chained = ranged + filled > 0;
    if (!*chained) return cudaSuccess;
    note_launches(1);
    attention_plan_kernel<<<(unsigned)(ranged + filled), 256, 0, s>>>(a, *plan, (int)ranged);
    return cudaGetLastError();
}

bool attention_head_map(void* map, const void* p, int64_t ld, int heads, int hd, int64_t T, int64_t N, int rows) {
    EncodeTiledFn enc = encode_fn();
    if (!enc) return false;
    cuuint64_t dims[4] = {(cuuint64_t)hd, (cuuint64_t)heads, (cuuint64_t)T, (cuuint64_t)N};
    cuuint64_t strides[3] = {(cuuint64_t)(hd * 2), (cuuint64_t)(ld * 2), (cuuint64_t)(T * ld * 2)};
    cuuint32_t box[4] = {64, 1, (cuuint32_t)rows, 1};
    cuuint32_t estr[4] = {1, 1, 1, 1};
    return enc((CUtensorMap*)map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(p), dims, strides, box, estr,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t launch_attention_forward_tc(const Attention& a, void* ws, unsigned int* err, cudaStream_t s) {
    const bool rich = a.cap > 0.f || a.n_buckets || a.slope;
    if (a.hd <= 64) return rich ? run<64, true>(a, ws, err, s) : run<64, false>(a, ws, err, s);
    return rich ? run<128, true>(a, ws, err, s) : run<128, false>(a, ws, err, s);
}

}  // namespace tda
