// k_attention_tc.cu -- the attention's forward pass on the tcgen05 tensor cores, bf16.
//
// An item is 256 queries of a head as two tiles of 128; a CTA goes once over the keys that they see, 128 at a time, with
// the running maximum and sum of each row. One CTA per SM takes items in turn: loads and MMAs of the next begin while the rows
// of the last are still being written. S = Q K^T lands in TMEM with a query per lane; four warps per tile turn it into
// P = 2^(c s - m) there, as bf16 over the columns that S had, and P is the MMA's operand from TMEM for O += P V. The tensor
// pipe works for one tile while the warps of the other have its scores: S0 | P0 V, S0' | P1 V, S1' | ... TMEM holds two
// S and two O tiles of 128 columns, all of its 512.
// O is rescaled only where a row's maximum has grown by more than 2^8 since the last time; P stays below 2^8 then, which
// costs bf16 nothing, and sums are fp32. Capped scores with a small bias become weights without their maximum, in one pass (packed
// documents 134 us with it, 111 so).
//
// Warps 0-3 and 4-7: rows of the tiles (a row per thread; of capped or biased scores half a row, 16 warps); then one each for the
// MMAs (a warp per tile was slower, the two streams share the pipe so that both end late: 8192 tokens 428 us, 344 with one), keys and
// values, items and queries, biases by distance; four for the outputs of finished tiles. Waits are bounded
// (about 1 s) and set kErrTimeout on expiry.
#include <cuda.h>
#include <math_constants.h>

#include <algorithm>
#include <cmath>
#include <mutex>

#include "attention.cuh"
#include "linear.cuh"

namespace tda {
namespace {

#include "tc_ptx.cuh"

#include "attention_tc.cuh"

// Registers are shared out anew after the launch, by warpgroup: of 128 a thread 184 for the two that hold rows of scores and 72 for
// the one that loads and issues and the one that writes outputs, 65,536 in all either way. Scores with cap or bias (RICH) take
// four times the instructions, and one warp a scheduler and tile waits for its own; there a row's keys are halved over two warps:
// of 80 a thread 88 for four warpgroups and 64 for two, 61,440 (packed documents 169 us with two and items in
// rounds, 142 with four and items taken as CTAs come free).
template <bool RICH>
struct Warps {
    static constexpr int kRows = RICH ? 16 : 8, kMma = kRows, kLoad = kRows + 1, kItems = kRows + 2, kBias = kRows + 3,
                         kOut = kRows + 4, kThreads = 32 * (kRows + 8), kCols = RICH ? 64 : 128;
    __device__ static __forceinline__ void row_registers() {
        if constexpr (RICH) asm volatile("setmaxnreg.inc.sync.aligned.u32 88;");
        else asm volatile("setmaxnreg.inc.sync.aligned.u32 184;");
    }
    __device__ static __forceinline__ void other_registers() {
        if constexpr (RICH) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
        else asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    }
};

constexpr float kLowest = -20.f;  // base of bounded scores

template <int HD, bool RICH>
struct Shape {
    static constexpr int kPanels = HD / 64;
    static constexpr uint32_t kTileBytes = kPanels * kPanel;
    static constexpr int kStages = HD == 64 ? 6 : RICH ? 3 : 4;
    static constexpr uint32_t kOut = (2 + kStages) * kTileBytes;  // 32 rows of output for each of 4 warps
    static constexpr uint32_t kBias = kOut + 4 * 32 * HD * 2;                  // RICH: 2 x 2 windows of biases
    static constexpr uint32_t kSwap = kBias + (RICH ? 16 * kWindow : 0);  // RICH: 16 warps' maxima, at two places in turn
    static constexpr uint32_t kSmem = kSwap + (RICH ? 16 * 256 : 0);
};

template <bool RICH>
struct BarsOf {
    uint64_t q_full[2], q_empty[2], s_full[2], p_ready[2][2], o_done[2], o_free[2], sum_full[2], done;
    uint64_t item_full[4], item_empty[4], full[8], empty[8], bias_full[2][2], bias_empty[2][2];
    uint32_t tmem;
    int abort;
    float2 sums[2][RICH ? 2 : 1][kTileT];  // maximum and sum of a finished row
    int4 items[4][2];
    int example[4];
};

// Keys that a tile's queries see.
struct Hull {
    int lo, hi;
    __device__ __forceinline__ bool any() const { return lo < hi; }
    __device__ __forceinline__ int first() const { return lo / kTileT; }
    __device__ __forceinline__ int last() const { return (hi - 1) / kTileT; }
};
__device__ __forceinline__ Hull hull_of(const Attention& a, const AttentionPlan& plan, int n, int tiles, int tile) {
    const int q0 = tile * kTileT, T = (int)a.T;
    if (q0 >= T) return {0, 0};
    if (a.range) {
        const AttentionTile& t = plan.tiles[(int64_t)n * tiles + tile];
        return {max(t.lo, 0), min(t.hi, T)};  // in range whatever a workspace in other use by now holds
    }
    return {0, a.causal ? min(q0 + kTileT, T) : T};
}

// The items of this CTA, long ones first where the mask is causal; every other round backwards, which evens out what the rounds
// leave. With ranges, which rounds do not even out, CTAs take items as they come free. An item's two tiles are the same queries of two
// heads that share their keys, where there are such heads and enough items for the SMs: they are equally long then (neighbours of
// one head are not where the mask is causal, and the longer one's last key tile has the CTA to itself: 8 x 1024 tokens 72 us, 65 so).
struct Items {
    int total, tiles, groups, by_head;  // groups of tiles
    FastDiv heads, H, group;            // N heads, heads (or pairs of heads), query heads per key head
    __device__ __forceinline__ int at(int round) const {
        const int g = gridDim.x, b = blockIdx.x;
        return round * g + (round & 1 ? g - 1 - b : b);
    }
    __device__ __forceinline__ int tile(int item) const { return (groups - 1 - heads.div(item)) << !by_head; }
    __device__ __forceinline__ int example(int item) const { return H.div(heads.mod(item)); }
    __device__ __forceinline__ int head(int item) const { return H.mod(heads.mod(item)) << by_head; }
};

// An item as the warp that makes them leaves it for the others, four at a time: working it out takes longer than a step of the MMAs.
struct Part {  // of an item: a tile of queries
    int n, h, tile, first, last;  // h < 0: no more items; first > last: no keys
    __device__ __forceinline__ int q0() const { return tile * kTileT; }
};
struct Item {
    Part of[2];
    __device__ __forceinline__ bool any() const { return min(of[0].first, of[1].first) <= max(of[0].last, of[1].last); }
};
struct ItemReader {
    uint32_t r = 0;
    // The next item, or one of its parts; false after the last one, or where a wait ran out (*ok). Called by whole warps.
    template <typename Bars>
    __device__ __forceinline__ bool next(Part& x, int w, Bars& bars, bool* ok, volatile int* abort, unsigned int* err) {
        *ok = *ok && wait_warp(smem_u32(&bars.item_full[r % 4]), (r / 4) & 1, abort, err);
        if (!*ok) return false;
        read(x, w, bars);
        done(bars);
        return x.h >= 0;
    }
    template <typename Bars>
    __device__ __forceinline__ bool next(Item& x, Bars& bars, bool* ok, volatile int* abort, unsigned int* err) {
        *ok = *ok && wait_warp(smem_u32(&bars.item_full[r % 4]), (r / 4) & 1, abort, err);
        if (!*ok) return false;
        read(x.of[0], 0, bars), read(x.of[1], 1, bars);
        done(bars);
        return x.of[0].h >= 0;
    }
    template <typename Bars>
    __device__ __forceinline__ void read(Part& x, int w, Bars& bars) const {
        const int4 a = bars.items[r % 4][w];
        x.n = bars.example[r % 4], x.h = a.x, x.tile = a.y, x.first = a.z, x.last = a.w;
    }
    template <typename Bars>
    __device__ __forceinline__ void done(Bars& bars) {
        __syncwarp();
        if (threadIdx.x % 32 == 0) mbar_arrive(smem_u32(&bars.item_empty[r % 4]));
        ++r;
    }
};

// A key tile of an item; next() goes on to the next item that has any, whose first one it gives. busy: products of the tile before
// are still to be issued, so only the item right behind is looked at, and where it has no keys there is no tile for now (!valid): items
// come four at a time, the outputs' warps do not pass theirs before its products, and the one wanted may not be made until they do.
struct Walk {
    Item item;
    int kt, last;
    bool valid = true, ended = false;
    ItemReader reader;
    __device__ __forceinline__ void clear() { kt = last = 0; }  // next() then gives the first
    template <typename Bars>
    __device__ __forceinline__ void next(bool busy, Bars& bars, bool* ok, volatile int* abort, unsigned int* err) {
        if (kt < last) {
            ++kt;
            return;
        }
        valid = false;
        while (!ended && !valid) {
            ended = !reader.next(item, bars, ok, abort, err);
            valid = !ended && item.any();
            if (busy) break;
        }
        kt = min(item.of[0].first, item.of[1].first), last = max(item.of[0].last, item.of[1].last);
    }
    __device__ __forceinline__ bool active(int w) const { return kt >= item.of[w].first && kt <= item.of[w].last; }
};

template <int HD, bool RICH>
__global__ __launch_bounds__(Warps<RICH>::kThreads, 1) void attention_tc_kernel(const __grid_constant__ CUtensorMap tmQ,
                                                                   const __grid_constant__ CUtensorMap tmK,
                                                                   const __grid_constant__ CUtensorMap tmV, const Attention a,
                                                                   const AttentionPlan plan, const Items items, unsigned int* err) {
    using S = Shape<HD, RICH>;
    using W = Warps<RICH>;
    extern __shared__ __align__(1024) uint8_t raw[];
    __shared__ BarsOf<RICH> bars;
    const uint32_t base = smem_u32(raw);
    uint8_t* from = raw;
    if (base & 1023u) {  // the tiles' swizzle needs it
        if (threadIdx.x == 0) atomicOr(err, kErrBadLaunch);
        return;
    }
    const uint32_t sq = base, ring = base + 2 * S::kTileBytes;
    const int warp = __shfl_sync(0xffffffffu, threadIdx.x / 32, 0), lane = threadIdx.x % 32;
    const int T = (int)a.T;
    volatile int* abort = &bars.abort;

    if (warp == W::kMma) {
        tmem_alloc(smem_u32(&bars.tmem), 512);
        tmem_relinquish();
        if (lane == 0) {
            for (int w = 0; w < 2; ++w) {
                mbar_init(smem_u32(&bars.q_full[w]), 1);
                mbar_init(smem_u32(&bars.q_empty[w]), 1);
                mbar_init(smem_u32(&bars.s_full[w]), 1);
                mbar_init(smem_u32(&bars.p_ready[w][0]), 4);
                mbar_init(smem_u32(&bars.p_ready[w][1]), 4);
                mbar_init(smem_u32(&bars.o_free[w]), 4);
                mbar_init(smem_u32(&bars.sum_full[w]), W::kRows / 2);
                mbar_init(smem_u32(&bars.o_done[w]), 1);
            }
            mbar_init(smem_u32(&bars.done), 1);
            for (int s = 0; s < S::kStages; ++s) mbar_init(smem_u32(&bars.full[s]), 1), mbar_init(smem_u32(&bars.empty[s]), 1);
            for (int r = 0; r < 4; ++r)  // read by the warps of rows and outputs, by the MMAs', the loads' and the biases'
                mbar_init(smem_u32(&bars.item_full[r]), 1), mbar_init(smem_u32(&bars.item_empty[r]), W::kRows + 6 + (RICH && plan.lut));
            for (int w = 0; w < 2; ++w)
                for (int b = 0; b < 2; ++b) mbar_init(smem_u32(&bars.bias_full[w][b]), 32), mbar_init(smem_u32(&bars.bias_empty[w][b]), W::kRows / 2);
            bars.abort = 0;
            fence_mbar_init();
        }
        __syncwarp();
        tc_fence_before();
    }
    chain_wait();
    // Capped scores with a small learned bias lie in +-90 (times log2 e): their weights need no maximum first, 2^x of a row's
    // scores less a base that is -20 at least stays in fp32's range. Slopes and large tables take the maximum.
    bool bounded = false;
    if constexpr (RICH) {
        const float limit = 90.f / kLog2e - a.cap;
        const int64_t entries = (int64_t)a.n_buckets * a.H;  // read by every CTA
        bool beyond = !(a.cap > 0.f && limit >= 0.f) || a.slope || entries > 16384;
        const int read = beyond ? 0 : (int)entries;
#pragma unroll 4
        for (int i = threadIdx.x; i < read; i += W::kThreads) {
            const float x = (float)((const __nv_bfloat16*)a.table)[i];
            beyond |= !(fabsf(x) <= limit || x == -CUDART_INF_F);
        }
        if (!plan.lut)
            for (int i = threadIdx.x; i < 4 * kWindow; i += W::kThreads) ((float*)(from + S::kBias))[i] = 0.f;
        bounded = !__syncthreads_or(beyond);
    } else {
        __syncthreads();
    }
    tc_fence_after();
    const uint32_t tmem = bars.tmem;

    if (warp < W::kRows) {
        W::row_registers();
        // tile w; RICH: columns 64 half + [0, 64) of its scores
        const int w = warp / (W::kRows / 2), half = RICH ? warp / 4 % 2 : 0, row = warp % 4 * 32 + lane;
        const uint32_t lanes = (uint32_t)(warp % 4) << 21;  // TMEM lane of the warp's first row
        const uint32_t ts = tmem + lanes + w * 128, to = tmem + lanes + 256 + w * 128 + half * (HD / 2);
        const float* biases = (const float*)(from + S::kBias) + w * 2 * kWindow + window_row(row) + 64 * half;
        const float c = RICH ? 1.f : a.scale * kLog2e;  // s is the score times log2 e (RICH) or the dot product
        const float2 c2 = both(c);
        const float grow = 8.f / c, inv_cap = RICH ? over_cap(a) : 0.f, cap2 = a.cap * kLog2e;
        bool ok = true;
        // RICH: a barrier of the two warps that share rows, and the larger of their maxima. A wait that ran out in one of them ends
        // both here: until then either goes on, so that the other is not left alone.
        auto join = [&](float mine, uint32_t turn) {
            float* at = (float*)(from + S::kSwap) + (turn & 1) * 32 + lane;
            at[warp * 64] = mine;
            ok = all_came_well(1 + w * 4 + warp % 4, 64, ok);
            return fmaxf(mine, at[(warp ^ 4) * 64]);
        };
        // O of the rows (RICH: half of its columns) times a number, once the MMAs before key tile `turn` are done. RICH: the weights of
        // one half of the keys are added to all columns as soon as their warps are ready, so both warps of a row have its O rescaled
        // before either goes on. Whether `by` is asked for is the same in both.
        auto rescale = [&](uint32_t turn, float by) {
            ok = ok && wait_warp(smem_u32(&bars.o_done[w]), (turn - 1) & 1, abort, err);
            if (ok) {
                tc_fence_after();
#pragma unroll 1
                for (int b = 0; b < HD / 16 / (RICH ? 2 : 1); ++b) {
                    float o[16];
                    tmem_ld16(to + 16 * b, o);
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[j] *= by;
                    tmem_st16(to + 16 * b, (const uint32_t*)o);
                }
                if (RICH) tmem_wait_st();
            }
            if (RICH) {
                tc_fence_before();
                ok = all_came_well(1 + w * 4 + warp % 4, 64, ok);
            }
        };
        uint32_t turn = 0, outputs = 0;  // key tiles, outputs so far
        ItemReader reader;
        Part item, then;
        int2 see, see_then = make_int2(0, 0);
        then.h = -2;
        while (ok) {
            // the next item and what this thread's row sees in it, one item ahead
            item = then, see = see_then;
            if (item.h == -1) break;
            bool there = reader.next(then, w, bars, &ok, abort, err);
            if (RICH) there = (ok = all_came_well(1 + w * 4 + warp % 4, 64, ok)) && there;
            if (!there) then.h = -1;
            else see_then = visible(a.range, a.causal, T, (int64_t)then.n * T, then.q0() + row);
            if (item.h < 0) continue;
            const int first = item.first, last = item.last;
            if (first > last) continue;
            const int i = item.q0() + row;
            // what the warp's rows see: nothing outside [lo, hi), everything within [most, least)
            const bool none = see.x >= see.y;
            const int most = __reduce_max_sync(0xffffffffu, none ? 0 : see.x);
            const int least = __reduce_min_sync(0xffffffffu, i >= T ? T : none ? 0 : see.y);
            const int lo = RICH ? __reduce_min_sync(0xffffffffu, none ? T : see.x) : 0;
            const int hi = RICH ? __reduce_max_sync(0xffffffffu, none ? 0 : see.y) : 0;
            float top = -CUDART_INF_F, sum = 0.f;
            for (int kt = first; kt <= last; ++kt, ++turn) {
                const int k0 = kt * kTileT + 64 * half;
                ok = ok && wait_warp(smem_u32(&bars.s_full[w]), turn & 1, abort, err);
                if (!RICH && !ok) break;
                tc_fence_after();
                float most_now = top;
                float s[RICH ? 32 : 128];
                const bool whole = most <= k0 && least >= k0 + W::kCols;
                auto sees = [&](int b) { return lo < k0 + 32 * b + 32 && hi > k0 + 32 * b; };
                auto mask = [&](int b, float* x) {
                    const int at = k0 + 32 * b;
                    if (most <= at && least >= at + 32) return;
                    const int from = min(max(see.x - at, 0), 32), to = min(max(see.y - at, 0), 32);
                    const uint32_t bits = from < to ? (to == 32 ? ~0u : (1u << to) - 1) & (~0u << from) : 0u;
#pragma unroll
                    for (int j = 0; j < 32; ++j)
                        if (!(bits >> j & 1)) x[j] = -CUDART_INF_F;
                };
                if constexpr (RICH) {
                    const float* bias = biases + (turn & 1) * kWindow;
                    if (plan.lut) ok = ok && wait_warp(smem_u32(&bars.bias_full[w][turn & 1]), (turn / 2) & 1, abort, err);
                    // the scores of 32 columns, biases as moved() leaves them
                    auto scored = [&](int b, auto moved) {
                        tmem_ld32(ts + 64 * half + 32 * b, s);
                        tmem_wait_ld();
                        tmem_use(s);
                        auto all = [&](auto score) {
#pragma unroll
                            for (int j = 0; j < 32; j += 4) {
                                const float4 x = *(const float4*)(bias + 32 * b + j);
                                const float2 u = score(make_float2(s[j], s[j + 1]), moved(make_float2(x.x, x.y)));
                                const float2 v = score(make_float2(s[j + 2], s[j + 3]), moved(make_float2(x.z, x.w)));
                                s[j] = u.x, s[j + 1] = u.y, s[j + 2] = v.x, s[j + 3] = v.y;
                            }
                        };
                        if (a.cap <= 0.f) all([&](float2 d, float2 x) { return fma2(d, both(a.scale * kLog2e), x); });
                        else if (all_near<32>(s, a.near_limit)) all([&](float2 d, float2 x) { return fma2(d, tanh_near(a, d), x); });
                        else all([&](float2 d, float2 x) { return fma2(tanh_any(mul2(d, both(inv_cap))), both(cap2), x); });
                        if (!whole) mask(b, s);
                    };
                    auto bias_read = [&]() {
                        if (!plan.lut) return;
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&bars.bias_empty[w][turn & 1]));
                    };
                    if (bounded) {
                        // weights by the row's base so far, in one go; they cannot overflow
                        if (kt == first) top = 0.f;
                        const float2 less = both(-top);
                        float2 part[2] = {both(0.f), both(0.f)};
#pragma unroll 1
                        for (int b = 0; b < 2; ++b) {
                            uint32_t p[16];
                            if (sees(b)) {
                                scored(b, [&](float2 x) { return add2(x, less); });
#pragma unroll
                                for (int j = 0; j < 16; ++j) {
                                    const float2 v = make_float2(exp2_fast(s[2 * j]), exp2_fast(s[2 * j + 1]));
                                    part[j & 1] = add2(part[j & 1], v);
                                    p[j] = pack_bf16(v.x, v.y);
                                }
                            } else {
#pragma unroll
                                for (int j = 0; j < 16; ++j) p[j] = 0;
                            }
                            tmem_st16(ts + 64 * half + 16 * b, p);
                        }
                        bias_read();
                        float now = part[0].x + part[0].y + part[1].x + part[1].y;
                        tmem_wait_st();
                        const bool fits = now <= 0x1p16f && (sum > 0.f || now >= 0x1p-16f || now == 0.f);
                        if (!all_came_well(1 + w * 4 + warp % 4, 64, ok && fits)) {
                            // a base by the sum of both halves of a row, by a power of two: the weights' scaling is exact
                            float* swap = (float*)(from + S::kSwap) + lane;
                            swap[warp * 64] = now, swap[warp * 64 + 32] = sum;
                            ok = all_came_well(1 + w * 4 + warp % 4, 64, ok);
                            if (!ok) break;
                            const float tile = now + swap[(warp ^ 4) * 64], before = sum + swap[(warp ^ 4) * 64 + 32];
                            int by2 = (int)(__float_as_uint(tile) >> 23) - 127;  // sums are positive, or NaN
                            if (tile == 0.f || by2 > 126 || (by2 <= 16 && (before > 0.f || by2 >= -16))) by2 = 0;
                            by2 = max(by2, (int)(kLowest - top));
                            top += (float)by2;
                            const float by = __int_as_float((127 - by2) << 23);
                            now *= by, sum *= by;
                            const __nv_bfloat162 by_pair = __float2bfloat162_rn(by);
#pragma unroll 1
                            for (int b = 0; b < 2; ++b) {
                                uint32_t p[16];
                                tmem_ld16(ts + 64 * half + 16 * b, (float*)p);
#pragma unroll
                                for (int j = 0; j < 16; ++j) {
                                    __nv_bfloat162 v = __hmul2(*(const __nv_bfloat162*)&p[j], by_pair);
                                    p[j] = *(const uint32_t*)&v;
                                }
                                tmem_st16(ts + 64 * half + 16 * b, p);
                            }
                            tmem_wait_st();
                            if (kt != first) rescale(turn, by);
                            if (!ok) break;
                        }
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&bars.p_ready[w][half]));
                        sum += now;
                        continue;
                    }
                    // scores go back to TMEM, 32 columns at a time, until their maximum is known
#pragma unroll 1
                    for (int b = 0; b < 2; ++b) {
                        if (!sees(b)) continue;
                        scored(b, [](float2 x) { return x; });
                        most_now = largest<32>(s, most_now);
                        tmem_st32(ts + 64 * half + 32 * b, (const uint32_t*)s);
                    }
                    tmem_wait_st();
                    bias_read();
                    most_now = join(most_now, turn);
                    if (!ok) break;
                } else {
                    if (!whole) {
                        // masked scores go back to TMEM, 32 columns at a time: fewer instructions than masks for all 128 in place
#pragma unroll 1
                        for (int b = 0; b < 4; ++b) {
                            const int at = k0 + 32 * b;
                            if (most <= at && least >= at + 32) continue;
                            tmem_ld32(ts + 32 * b, s);
                            tmem_wait_ld();
                            tmem_use(s);
                            mask(b, s);
                            tmem_st32(ts + 32 * b, (const uint32_t*)s);
                        }
                        tmem_wait_st();
                    }
#pragma unroll
                    for (int b = 0; b < 4; ++b) tmem_ld32(ts + 32 * b, s + 32 * b);
                    tmem_wait_ld();
#pragma unroll
                    for (int b = 0; b < 4; ++b) tmem_use(s + 32 * b);
                    most_now = largest<128>(s, most_now);
                }
                if (kt == first) {
                    top = most_now;
                } else if (__any_sync(0xffffffffu, most_now > top + grow)) {
                    const float by = most_now == -CUDART_INF_F ? 1.f : exp2_fast((top - most_now) * c);
                    top = most_now;
                    sum *= by;
                    rescale(turn, by);
                    if (!ok) break;
                }
                const float base_of = top == -CUDART_INF_F ? 0.f : top;
                const float2 less = both(RICH ? -base_of : -base_of * c);
                float2 part[2] = {both(0.f), both(0.f)};
                // P of 32 columns of scores
                auto weigh = [&](const float* x, uint32_t* p) {
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float2 v = make_float2(x[2 * j], x[2 * j + 1]);
                        v = RICH ? add2(v, less) : fma2(v, c2, less);
                        v.x = exp2_fast(v.x), v.y = exp2_fast(v.y);
                        part[j & 1] = add2(part[j & 1], v);
                        p[j] = pack_bf16(v.x, v.y);
                    }
                };
                // over columns of S that have been read (RICH: the chunks of one's own half, whose first column their P begins at), in
                // two parts of 64 keys: the MMAs of the first begin while the second is computed, or the other warp's is
                if constexpr (RICH) {
#pragma unroll 1
                    for (int b = 0; b < 2; ++b) {
                        uint32_t p[16];
                        if (sees(b)) {
                            tmem_ld32(ts + 64 * half + 32 * b, s);
                            tmem_wait_ld();
                            tmem_use(s);
                            weigh(s, p);
                        } else {
#pragma unroll
                            for (int j = 0; j < 16; ++j) p[j] = 0;
                        }
                        tmem_st16(ts + 64 * half + 16 * b, p);
                    }
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&bars.p_ready[w][half]));
                } else {
#pragma unroll
                    for (int part_of = 0; part_of < 2; ++part_of) {
                        uint32_t p[32];
                        weigh(s + 64 * part_of, p);
                        weigh(s + 64 * part_of + 32, p + 16);
                        tmem_st32(ts + 32 * part_of, p);
                        tmem_wait_st();
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(smem_u32(&bars.p_ready[w][part_of]));
                    }
                }
                sum += part[0].x + part[0].y + part[1].x + part[1].y;
            }
            // an item of one key tile does not wait for the output before it: here it does, as that one's sums may not have been read
            if (outputs++) ok = ok && wait_warp(smem_u32(&bars.o_free[w]), outputs & 1, abort, err);
            if (RICH) ok = all_came_well(1 + w * 4 + warp % 4, 64, ok);
            if (!ok) break;
            // negative: of one key, whose weight is no power of two
            bars.sums[w][half][row] = make_float2(top, RICH && bounded && see.y - see.x == 1 ? -sum : sum);
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&bars.sum_full[w]));
        }
        tc_fence_before();
    } else if (warp >= W::kOut) {
        W::other_registers();
        // outputs of either tile, beside the rows of the next item
        const int q = warp % 4, row = q * 32 + lane;
        const uint32_t out = base + S::kOut + q * 64 * HD;
        uint32_t turns[2] = {0, 0}, done[2] = {0, 0};  // key tiles, outputs so far
        bool ok = true;
        ItemReader reader;
        Item item;
        while (reader.next(item, bars, &ok, abort, err)) {
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const Part& x = item.of[w];
                const int n = x.n, h = x.h, q0 = x.q0(), i = q0 + row;
                if (!ok || q0 >= T) continue;
                const bool any = x.first <= x.last;
                float top = 0.f, sum = 0.f;
                if (any) {
                    turns[w] += x.last - x.first + 1;
                    ok = wait_warp(smem_u32(&bars.sum_full[w]), done[w]++ & 1, abort, err) &&
                         wait_warp(smem_u32(&bars.o_done[w]), (turns[w] - 1) & 1, abort, err);
                    if (!ok) continue;
                    top = bars.sums[w][0][row].x, sum = bars.sums[w][0][row].y;
                    if (RICH) sum += bars.sums[w][RICH][row].y;
                    tc_fence_after();
                }
                // one key's value is divided by its weight as that was rounded; NaN sums stay NaN
                const float over = RICH && sum < 0.f ? __bfloat162float(__float2bfloat16(sum)) : sum;
                const float by = sum != 0.f ? 1.f / fabsf(over) : 0.f;
                sum = fabsf(sum);
                const uint32_t to = tmem + ((uint32_t)q << 21) + 256 + w * 128;
#pragma unroll 1
                for (int b = 0; b < HD / 32; ++b) {
                    float o[32];
                    tmem_ld32(to + 32 * b, o);
                    tmem_wait_ld();
                    tmem_use(o);
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const float* x = o + 8 * g;
                        uint32_t v[4] = {0, 0, 0, 0};
                        if (by != 0.f)  // rows that see nothing: TMEM may hold anything
                            v[0] = pack_bf16(x[0] * by, x[1] * by), v[1] = pack_bf16(x[2] * by, x[3] * by),
                            v[2] = pack_bf16(x[4] * by, x[5] * by), v[3] = pack_bf16(x[6] * by, x[7] * by);
                        asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(out + lane * 2 * HD + ((4 * b + g) ^ (lane & 7)) * 16),
                                     "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3])
                                     : "memory");
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (any && lane == 0) mbar_arrive(smem_u32(&bars.o_free[w]));
                if (a.lse && i < T)
                    a.lse[((int64_t)n * a.H + h) * T + i] = sum != 0.f ? fmaf(top, RICH ? kLn2 : a.scale, logf(sum)) : -CUDART_INF_F;
                // whole rows on the way out
                constexpr int kLanes = HD / 8;  // of a row
                const int col = lane % kLanes * 8;
                __nv_bfloat16* dst = (__nv_bfloat16*)a.O + ((int64_t)n * T + q0 + q * 32) * a.ld_o + h * a.hd + col;
#pragma unroll
                for (int r = lane / kLanes; r < 32; r += 32 / kLanes) {
                    uint32_t v[4];
                    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3])
                                 : "r"(out + r * 2 * HD + ((lane % kLanes) ^ (r & 7)) * 16)
                                 : "memory");
                    if (col < a.hd && q0 + q * 32 + r < T) *(uint4*)(dst + r * a.ld_o) = make_uint4(v[0], v[1], v[2], v[3]);
                }
                __syncwarp();
            }
        }
        tc_fence_before();
    } else {
        W::other_registers();
        if (warp == W::kLoad) {
            const uint32_t lead = elect_one();
            uint32_t used = 0;  // loads so far
            bool ok = true;
            Walk at;
            at.clear();
            while (true) {
                at.next(false, bars, &ok, abort, err);
                if (!ok || !at.valid) break;
                const int kv = items.group.div(at.item.of[0].h);
#pragma unroll 1
                for (int e = 0; e < 2; ++e) {
                    const uint32_t s = used % S::kStages, turn = used / S::kStages;
                    if (turn) ok = ok && wait_warp(smem_u32(&bars.empty[s]), (turn - 1) & 1, abort, err);
                    if (!ok) break;
                    if (lead) {
                        const uint32_t bar = smem_u32(&bars.full[s]);
                        mbar_arrive_tx(bar, S::kTileBytes);
#pragma unroll
                        for (int p = 0; p < S::kPanels; ++p)
                            tma_load_head(ring + s * S::kTileBytes + p * kPanel, e ? &tmV : &tmK, 64 * p, kv, at.kt * kTileT, at.item.of[0].n, bar);
                    }
                    __syncwarp();
                    ++used;
                }
            }
            for (uint32_t s = 0; s < (uint32_t)S::kStages; ++s)
                if (used > s) wait_settled(smem_u32(&bars.full[s]), ((used - 1 - s) / S::kStages) & 1, err);
        } else if (warp == W::kItems) {
            // the items, one ahead of their queries, which are loaded as soon as there is room
            const uint32_t lead = elect_one();
            uint32_t asked0 = 0, asked1 = 0, made = 0;  // query tiles of either kind, items so far
            bool ok = true;
            auto make = [&]() {
                const uint32_t r = made++;
                if (r >= 4) ok = ok && wait_warp(smem_u32(&bars.item_empty[r % 4]), (r / 4 - 1) & 1, abort, err);
                if (!ok) return;
                int id = items.at((int)r);
                if (a.range) {  // their lengths are known here only: whoever is done takes the next
                    if (lane == 0) id = atomicAdd(plan.taken, 1);
                    id = __shfl_sync(0xffffffffu, id, 0);
                }
                int n = 0, h = -2, tile = 0;
                Hull hull[2] = {{0, 0}, {0, 0}};
                if ((uint32_t)id < (uint32_t)items.total) {
                    n = items.example(id), h = items.head(id), tile = items.tile(id);
                    hull[0] = hull_of(a, plan, n, items.tiles, tile), hull[1] = hull_of(a, plan, n, items.tiles, tile + !items.by_head);
                }
                if (lead) {
                    bars.example[r % 4] = n;
#pragma unroll
                    for (int w = 0; w < 2; ++w)
                        bars.items[r % 4][w] = make_int4(h + (w & items.by_head), tile + (w & ~items.by_head), hull[w].any() ? hull[w].first() : 1 << 30,
                                                         hull[w].any() ? hull[w].last() : -1);
                    mbar_arrive(smem_u32(&bars.item_full[r % 4]));
                }
                __syncwarp();
            };
            for (uint32_t r = 0; ok; ++r) {  // makes item r, loads the queries of item r - 1
                if (r && bars.items[(r - 1) % 4][0].x < 0) break;
                make();
                if (r == 0) continue;
                // nobody can have replaced what this warp made: the slot is free for item r + 3 once its readers have passed it
                const int example = bars.example[(r - 1) % 4];
#pragma unroll 1
                for (int w = 0; w < 2; ++w) {
                    const int4 x = bars.items[(r - 1) % 4][w];
                    if (!ok || x.z > x.w) continue;
                    const uint32_t turn = w ? asked1 : asked0;
                    if (turn) ok = wait_warp(smem_u32(&bars.q_empty[w]), (turn - 1) & 1, abort, err);
                    if (!ok) continue;
                    if (lead) {
                        const uint32_t bar = smem_u32(&bars.q_full[w]);
                        mbar_arrive_tx(bar, S::kTileBytes);
#pragma unroll
                        for (int p = 0; p < S::kPanels; ++p)
                            tma_load_head(sq + w * S::kTileBytes + p * kPanel, &tmQ, 64 * p, x.x, x.y * kTileT, example, bar);
                    }
                    __syncwarp();
                    w ? ++asked1 : ++asked0;
                }
            }
            if (asked0) wait_settled(smem_u32(&bars.q_full[0]), (asked0 - 1) & 1, err);
            if (asked1) wait_settled(smem_u32(&bars.q_full[1]), (asked1 - 1) & 1, err);
        } else if (warp == W::kMma) {
            const uint32_t lead = elect_one();
            const int steps = (a.hd + 15) / 16;
            constexpr uint32_t kIdS = idesc_bf16(kTileT, kTileT), kIdO = idesc_bf16(kTileT, HD) | kBMn;
            // bit w: parity of the query tiles, of the key tiles, of the outputs of tile w so far; some output; stages (K, V, K ...)
            uint32_t par_q = 0, par_p = 0, par_o = 0, some_o = 0, used = 0;
            auto full = [&](uint32_t at) { return wait_warp(smem_u32(&bars.full[at % S::kStages]), (at / S::kStages) & 1, abort, err); };
            auto release = [&](uint32_t at) { commit(lead, smem_u32(&bars.empty[at % S::kStages])); };
            auto stage = [&](uint32_t at) { return ring + (at % S::kStages) * S::kTileBytes; };
            bool ok = true;
            Walk now, then;
            then.clear();
            now.valid = false;
            // a step: O += P V of the key tile `now`, then S of the one after it, for either tile of queries
            while (true) {
                const uint32_t at_v = used, at_k = now.valid ? used + 1 : used;
                then.next(now.valid, bars, &ok, abort, err);
                if (!ok || (!now.valid && !then.valid)) break;
                uint64_t v = 0;
                if (now.valid) {
                    ok = full(at_v);
                    if (!ok) break;
                    if (a.range) {
                        uint32_t bits[4];
                        *(uint4*)bits = *(const uint4*)plan.tiles[(int64_t)now.item.of[0].n * items.tiles + now.kt].unseen;
                        if (bits[0] | bits[1] | bits[2] | bits[3]) clear_rows(stage(at_v), S::kPanels, bits);
                    }
                    v = mn_major(stage(at_v), kPanel);
                }
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const uint32_t ts = tmem + w * 128, to = tmem + 256 + w * 128;
                    const int first = now.item.of[w].first, last = now.item.of[w].last;
                    if (now.valid && now.kt >= first && now.kt <= last) {
                        if (now.kt == first) {  // the tile's last output has been read
                            if (some_o >> w & 1) ok = wait_warp(smem_u32(&bars.o_free[w]), ~par_o >> w & 1, abort, err);
                            some_o |= 1u << w, par_o ^= 1u << w;
                        }
#pragma unroll
                        for (int b = 0; b < 2; ++b) {  // 64 keys each
                            ok = ok && wait_warp(smem_u32(&bars.p_ready[w][b]), par_p >> w & 1, abort, err);
                            if (!ok) break;
                            tc_fence_after();
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                mma_ts(lead, to, ts + (RICH ? 64 : 32) * b + 8 * e, v + ((4 * b + e) * 2048 >> 4), kIdO, now.kt != first || b + e > 0);
                        }
                        if (!ok) break;
                        commit(lead, smem_u32(&bars.o_done[w]));
                        par_p ^= 1u << w;
                    }
                    if (!then.valid) continue;
                    if (w == 0) ok = full(at_k);
                    const int first_k = then.item.of[w].first, last_k = then.item.of[w].last;
                    if (ok && then.kt >= first_k && then.kt <= last_k) {
                        if (then.kt == first_k) {
                            ok = wait_warp(smem_u32(&bars.q_full[w]), par_q >> w & 1, abort, err);
                            par_q ^= 1u << w;
                        }
                        if (!ok) break;
                        tc_fence_after();
                        mma_heads<HD>(lead, ts, sq + w * S::kTileBytes, stage(at_k), kIdS, steps);
                        commit(lead, smem_u32(&bars.s_full[w]));
                        if (then.kt == last_k) commit(lead, smem_u32(&bars.q_empty[w]));
                    }
                    if (!ok) break;
                }
                if (!ok) break;
                if (now.valid) release(at_v);
                if (then.valid) release(at_k);
                used += (now.valid ? 1 : 0) + (then.valid ? 1 : 0);
                now = then;
            }
            commit(lead, smem_u32(&bars.done));
            wait_settled(smem_u32(&bars.done), 0, err);
        } else if (RICH && plan.lut) {
            // the biases of a tile's 255 distances, ahead of its rows
            uint32_t turns[2] = {0, 0};
            bool ok = true;
            Walk at;
            at.clear();
            while (true) {
                at.next(false, bars, &ok, abort, err);
                if (!ok || !at.valid) break;
#pragma unroll
                for (int w = 0; w < 2; ++w) {
                    const uint32_t turn = turns[w];
                    if (!at.active(w)) continue;
                    if (turn >= 2)
                        ok = wait_warp(smem_u32(&bars.bias_empty[w][turn & 1]), (turn / 2 - 1) & 1, abort, err);
                    if (!ok) break;
                    load_window<true>(plan, at.item.of[w].h, at.item.of[w].q0() - at.kt * kTileT, (float*)(from + S::kBias) + (2 * w + (turn & 1)) * kWindow);
                    mbar_arrive(smem_u32(&bars.bias_full[w][turn & 1]));
                    ++turns[w];
                }
            }
        }
    }
    __syncthreads();
    if (warp == W::kMma) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// One CTA per tile of 128 tokens and example: what its queries see, and which of its tokens nothing sees; the CTAs
// behind them fill the biases by distance. Every CTA reads all ranges of its example, T^2 / 128 in all: simple, and 10 us with the
// ranges' own kernel at 4 x 2047 tokens, but where the attention is linear in T (windows of 511) half of the 7.7 ms of 1,048,576 tokens.
__global__ __launch_bounds__(256) void attention_plan_kernel(const Attention a, const AttentionPlan plan, int ranged) {
    const int t = threadIdx.x;
    if ((int)blockIdx.x >= ranged) {
        const int64_t at = (int64_t)(blockIdx.x - ranged) * 256 + t;
        if (at < (int64_t)a.H * plan.lut_len) {
            const int h = (int)(at / plan.lut_len);
            const float v = distance_bias(a.bucket, (const __nv_bfloat16*)a.table, a.slope, a.n_buckets, a.reach, a.H, h,
                                          at % plan.lut_len - plan.lut_mid);
            plan.lut[at] = kLog2e * (v < -0x1p127f && v > -CUDART_INF_F ? -0x1p127f : v);
        }
        return;
    }
    __shared__ AttentionTile tile;
    if (blockIdx.x == 0 && t == 0) *plan.taken = 0;
    const int T = (int)a.T, tiles = (T + kTileT - 1) / kTileT, n = blockIdx.x / tiles, k0 = (int)(blockIdx.x % tiles) * kTileT;
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
    for (int at = t; at < T; at += 8 * 256) {  // eight loads on their way at a time
        int2 r[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) r[e] = visible(a.range, 0, T, (int64_t)n * T, at + 256 * e);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int lo = r[e].x - k0, hi = r[e].y - k0;
            if (hi <= 0 || lo >= kTileT || lo >= hi) continue;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int x = min(max(lo - 32 * w, 0), 32), y = min(max(hi - 32 * w, 0), 32);
                if (x < y) seen[w] |= (y == 32 ? ~0u : (1u << y) - 1) & (~0u << x);
            }
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
    using Sh = Shape<HD, RICH>;
    if (cudaError_t e = smem_attr_once<attention_tc_kernel<HD, RICH>>(Sh::kSmem)) return e;
    CUtensorMap q, k, v;
    if (!attention_head_map(&q, a.Q, a.ld_q, a.H, a.hd, a.T, a.N, kTileT) ||
        !attention_head_map(&k, a.K, a.ld_k, a.KV, a.hd, a.T, a.N, kTileT) ||
        !attention_head_map(&v, a.V, a.ld_v, a.KV, a.hd, a.T, a.N, kTileT))
        return cudaErrorInvalidValue;
    AttentionPlan plan;
    bool chained;
    if (cudaError_t e = launch_attention_plan(a, ws, &plan, &chained, s)) return e;
    Attention with = a;
    attention_near(with, a.cap * kLog2e);
    const int64_t tiles = (a.T + kTileT - 1) / kTileT;
    Items items;
    const int64_t group = a.H / a.KV, by_head = group % 2 == 0 && tiles * a.N * a.H / 2 >= train_sms(), heads = a.H >> by_head;
    items.tiles = (int)tiles, items.by_head = (int)by_head, items.groups = (int)(by_head ? tiles : (tiles + 1) / 2);
    items.total = (int)(items.groups * a.N * heads);
    items.heads = FastDiv((uint32_t)(a.N * heads)), items.H = FastDiv((uint32_t)heads), items.group = FastDiv((uint32_t)group);
    return launch_chained(chained, attention_tc_kernel<HD, RICH>, dim3((unsigned)std::min(items.total, train_sms())), dim3(Warps<RICH>::kThreads),
                          Sh::kSmem, s, q, k, v, with, plan, items, err);
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

void attention_near(Attention& a, float by) {
    // tanh x = x P(x^2) for |x| <= 1/2, a minimax fit. Where the cap is so large that a coefficient leaves fp32's range, it and
    // those above it are left out, and what is near ends where they would be 2^-24 of the value.
    constexpr double fit[5] = {0.017135003581643105, -0.05298607423901558, 0.13324779272079468, -0.3333306908607483, 1.0};
    constexpr double near[5] = {0.21, 0.1, 0.026, 0.0004, 0.0};  // without a term and those above it
    a.near_limit = -1.f;                                         // no dot product is near
    if (!(a.cap > 0.f)) return;
    const double x = (double)a.scale / a.cap;
    double most = 0.5;
    for (int k = 0; k < 5; ++k) {
        float c = (float)(fit[k] * by * std::pow(x, 9 - 2 * k));
        if (!std::isfinite(c)) return;
        if (!std::isnormal(c)) c = 0.f, most = near[k];
        a.near[k] = make_float2(c, c);
    }
    if (most > 0) a.near_limit = (float)std::min(most / x, 0x1p60);  // its square is finite
}

size_t attention_plan_bytes(const Attention& a, bool bound) {
    size_t n = 0;
    if (a.range || bound) n += up((size_t)a.N * ((a.T + kTileT - 1) / kTileT) * sizeof(AttentionTile) + 4);
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
        plan->taken = (int*)(plan->tiles + a.N * tiles);
        at += up((size_t)a.N * tiles * sizeof(AttentionTile) + 4);
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
