// k_linear_tc.cu -- the products of the linear layer on the tcgen05 tensor cores:
// Z = X W^T + b, Y = act(Z) + R; dX = B W; dW = B^T X. All are
// D[i][j] = sum_k P[i][k] Q[j][k] with operands that are K-major (X, W, B) or
// MN-major (W for dX, B and X for dW) in memory; TMA copies either kind into the
// matching 128-byte-swizzled shared-memory layout, 64 values of k per stage, so
// nothing is transposed in memory.
//
// fp32 operands arrive as three bf16 planes x = x0 + x1 + x2 (each the rounding of
// what the ones before leave, exact to 2^-24): the K loop then runs over the six
// plane pairs whose products matter, smallest first. The tensor pipe adds into its
// fp32 accumulators with truncation, so for these a run of kWindow chunks is
// drained and added up in registers with rounding.
//
// linear_tile_kernel: one 128 x BN tile per CTA. Few rows (a decoded token, a
// short batch) swap the operands, so the long side fills the 128 rows of a tile,
// and split the K loop over the CTAs of a cluster, whose fp32 tiles are added in
// rank order through distributed shared memory.
//
// Warp roles: warp 0 TMA producer (lane 0), warp 1 TMEM allocator and MMA issuer
// (lane 0), warps 2-9 epilogue (TMEM lane quadrant warp % 4, column half by warp).
// Waits are bounded (about 1 s) and set kErrTimeout on expiry.
#include <cuda.h>

#include <mutex>

#include "linear.cuh"

namespace tda {
namespace {

#include "tc_ptx.cuh"

constexpr int kThreads = 320, kEpiWarps = 8;
constexpr int kTM = 128, kTK = 64;
constexpr uint32_t kBox = 64 * kTK * 2;  // one 64 x 64 MN-major box: 8 KiB
constexpr int kWindow = 4;               // chunks accumulated in TMEM before rounding, fp32 operands

struct TileParams {
    LinearEpilogue ep;
    int64_t tiles_p, tiles_q;
    int nk, pairs;      // K chunks of one plane pair, plane pairs
    int window;         // chunks per accumulator
    int split;          // CTAs of a cluster along K
    bool p_mn, q_mn;
    bool swap;          // tile rows are output columns
    unsigned int* err;
};

// Planes of P and Q of the t-th pair of fp32 operands.
__device__ __forceinline__ int pair_p(int pairs, int t) { return pairs == 1 ? 0 : (0x001102 >> (4 * t)) & 15; }
__device__ __forceinline__ int pair_q(int pairs, int t) { return pairs == 1 ? 0 : (0x010120 >> (4 * t)) & 15; }

// Descriptor fields beside the address: K-major tiles have 8-row groups 1 KiB apart; MN-major
// tiles 64-element atoms one box apart (LBO) and 8-row K groups 1 KiB apart (SBO).
__device__ __forceinline__ uint64_t desc_of(uint32_t saddr, bool mn) {
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | ((uint64_t)(mn ? kBox >> 4 : 1) << 16) |
           ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// 16 values of k further: 32 bytes along a K-major row, two 8-row groups of an MN-major box.
__device__ __forceinline__ uint64_t desc_step(bool mn) { return mn ? 2048 >> 4 : 32 >> 4; }

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

template <int ACT>
__device__ __forceinline__ void act4(float* v) {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = act_value<ACT>(v[i]);
}

// Four sums of output row m, columns n .. n + 3, through the epilogue and out.
template <typename T>
__device__ __forceinline__ void finish4(const LinearEpilogue& e, int64_t m, int64_t n, float* v) {
    const bool vec = e.vec && n + 4 <= e.N;
    const T* bias = (const T*)e.bias + n;
    const T* R = (const T*)e.R + m * e.ld_r + n;
    T* Y = (T*)e.Y + m * e.ld_y + n;
    T* Z = (T*)e.Z + m * e.ld_z + n;
    const int have = vec ? 4 : (int)(e.N - n < 4 ? e.N - n : 4);
    float r[4];
    if (e.R) {
        if (vec)
            ld4(R, r);
        else
            for (int i = 0; i < have; ++i) r[i] = ld1(R + i);
    }
    if (e.bias) {
        float b[4];
        if (vec) {
            ld4(bias, b);
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += b[i];
        } else {
            for (int i = 0; i < have; ++i) v[i] += ld1(bias + i);
        }
    }
    if (e.Z) {
        if (vec)
            st4(Z, v);
        else
            for (int i = 0; i < have; ++i) st1(Z + i, v[i]);
    }
    switch (e.act) {
        case TDA_ACT_RELU: act4<TDA_ACT_RELU>(v); break;
        case TDA_ACT_GELU: act4<TDA_ACT_GELU>(v); break;
        case TDA_ACT_GELU_TANH: act4<TDA_ACT_GELU_TANH>(v); break;
        case TDA_ACT_SILU: act4<TDA_ACT_SILU>(v); break;
        default: break;
    }
    if (e.R) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i < have) v[i] = fmaf(e.r_scale, r[i], v[i]);
    }
    if (vec)
        st4(Y, v);
    else
        for (int i = 0; i < have; ++i) st1(Y + i, v[i]);
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
    static constexpr uint32_t kP = kTM * kTK * 2, kQ = BN * kTK * 2, kStage = kP + kQ;
    // two CTAs share an SM (96 to 100 KiB of stages each); the rounding variant keeps its sums in
    // registers and takes an SM alone
    static constexpr int kStages = ROUND ? 5 : BN == 128 ? 3 : BN == 64 ? 4 : 5;
    static constexpr size_t kSmem = 1024 + (size_t)kStages * kStage + 8 * (2 * kStages + 5) + 16;
    static constexpr uint32_t kCols = 2 * BN;  // two accumulators
    static_assert((BN + 4) * kTM * 4 <= kStages * kStage, "the fp32 tile reuses the stages");
};

template <typename T, int BN, bool ROUND>
__global__ void __launch_bounds__(kThreads, ROUND ? 1 : 2)
linear_tile_kernel(const __grid_constant__ CUtensorMap tmP, const __grid_constant__ CUtensorMap tmQ,
                   const __grid_constant__ TileParams p) {
    using S = TileShape<BN, ROUND>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = (uint8_t*)(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
    uint64_t* bars = (uint64_t*)(smem + (size_t)S::kStages * S::kStage);
    uint64_t* full = bars;                    // TMA bytes landed
    uint64_t* empty = bars + S::kStages;      // MMAs done with the stage
    uint64_t* tfull = bars + 2 * S::kStages;  // [2] accumulator ready
    uint64_t* tempty = tfull + 2;             // [2] accumulator drained
    uint64_t* mma_done = tempty + 2;
    uint32_t* tmem_slot = (uint32_t*)(mma_done + 1);
    volatile int* abort = (volatile int*)(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            mbar_init(smem_u32(&full[s]), 1);
            mbar_init(smem_u32(&empty[s]), 1);
        }
        for (int b = 0; b < 2; ++b) {
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

    const int64_t tile = blockIdx.x / p.split;
    const int rank = blockIdx.x % p.split;
    const int64_t i0 = (tile / p.tiles_q) * kTM, j0 = (tile % p.tiles_q) * BN;
    const int total = p.nk * p.pairs;
    const int t0 = (int)((int64_t)total * rank / p.split), t1 = (int)((int64_t)total * (rank + 1) / p.split);
    const int windows = (t1 - t0 + p.window - 1) / p.window;

    if (warp == 0) {
        if (lane == 0) {
            // ---------------- TMA producer
            uint32_t last_par[S::kStages];
            bool issued[S::kStages];
            for (int s = 0; s < S::kStages; ++s) issued[s] = false;
            int pair = t0 / p.nk, kc = t0 % p.nk;
            for (int t = t0, ring = 0; t < t1; ++t, ++ring) {
                const int s = ring % S::kStages;
                const uint32_t ph = (ring / S::kStages) & 1u;
                if (!wait_bounded(smem_u32(&empty[s]), ph ^ 1u, abort, p.err)) break;
                const uint32_t st = smem_u32(smem + (size_t)s * S::kStage), bar = smem_u32(&full[s]);
                const int pp = pair_p(p.pairs, pair), pq = pair_q(p.pairs, pair), k0 = kc * kTK;
                mbar_arrive_tx(bar, S::kStage);
                if (p.p_mn) {
                    for (int j = 0; j < kTM / 64; ++j) tma_load_3d(st + j * kBox, &tmP, (int)i0 + 64 * j, k0, pp, bar);
                } else {
                    tma_load_3d(st, &tmP, k0, (int)i0, pp, bar);
                }
                if (BN >= 64 && p.q_mn) {
                    for (int j = 0; j < BN / 64; ++j)
                        tma_load_3d(st + S::kP + j * kBox, &tmQ, (int)j0 + 64 * j, k0, pq, bar);
                } else {
                    tma_load_3d(st + S::kP, &tmQ, k0, (int)j0, pq, bar);
                }
                issued[s] = true;
                last_par[s] = ph;
                if (++kc == p.nk) kc = 0, ++pair;
            }
            // copies still in flight when the MMA side stopped early land before the CTA exits
            for (int s = 0; s < S::kStages; ++s)
                if (issued[s]) {
                    const uint64_t since = global_ns();
                    while (!mbar_try_wait(smem_u32(&full[s]), last_par[s]))
                        if (global_ns() - since > kTimeoutNs) {
                            atomicOr(p.err, kErrTimeout);
                            break;
                        }
                }
        }
    } else if (warp == 1) {
        if (lane == 0) {
            // ---------------- MMA issuer
            const uint32_t idesc = idesc_bf16(kTM, BN) | (p.p_mn ? 1u << 15 : 0u) | (p.q_mn ? 1u << 16 : 0u);
            const uint64_t sp = desc_step(p.p_mn), sq = desc_step(p.q_mn);
            bool ok = true;
            int t = t0, ring = 0;
            for (int w = 0; ok && w < windows; ++w) {
                const uint32_t b = w & 1u, use = w >> 1;
                if (!wait_bounded(smem_u32(&tempty[b]), (use & 1u) ^ 1u, abort, p.err)) break;
                tc_fence_after();
                const int end = t + p.window < t1 ? t + p.window : t1;
                for (bool first = true; t < end; ++t, ++ring) {
                    const int s = ring % S::kStages;
                    const uint32_t ph = (ring / S::kStages) & 1u;
                    if (!wait_bounded(smem_u32(&full[s]), ph, abort, p.err)) {
                        ok = false;
                        break;
                    }
                    tc_fence_after();
                    const uint32_t st = smem_u32(smem + (size_t)s * S::kStage);
                    const uint64_t dp = desc_of(st, p.p_mn), dq = desc_of(st + S::kP, p.q_mn);
#pragma unroll
                    for (int k = 0; k < kTK / 16; ++k) {
                        mma_bf16(tmem + b * BN, dp + k * sp, dq + k * sq, idesc, first ? 0u : 1u);
                        first = false;
                    }
                    mma_commit(smem_u32(&empty[s]));
                }
                if (ok) mma_commit(smem_u32(&tfull[b]));
            }
            mma_commit(smem_u32(mma_done));
            const uint64_t since = global_ns();
            while (!mbar_try_wait(smem_u32(mma_done), 0))
                if (global_ns() - since > kTimeoutNs) {
                    atomicOr(p.err, kErrTimeout);
                    break;
                }
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
            if (lane == 0) got = wait_bounded(smem_u32(&tfull[w & 1]), (uint32_t)(w >> 1) & 1u, abort, p.err);
            got = __shfl_sync(0xffffffffu, got, 0);
            tc_fence_after();
            return got;
        };
        if (!ROUND) {
            if (wait_for(0)) {
#pragma unroll
                for (int c = 0; c < kC; c += 16) {
                    float v[16];
                    tmem_ld16(tb + c, v);
                    put(half * kC + c, v);
                }
            }
        } else {
            float acc[kC];
#pragma unroll
            for (int i = 0; i < kC; ++i) acc[i] = 0.f;
            bool got = true;
            for (int w = 0; got && w < windows; ++w) {
                if (!(got = wait_for(w))) break;
#pragma unroll
                for (int c = 0; c < kC; c += 16) {
                    float v[16];
                    tmem_ld16(tb + (w & 1) * BN + c, v);
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[c + i] += v[i];
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&tempty[w & 1]));
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
        for (int g = g0 + threadIdx.x; g < g1; g += kThreads) {
            const int o = g * 4 / inner, c = g * 4 % inner;
            const int64_t m = m0 + o, n = n0 + c;
            if (m >= p.ep.M || n >= p.ep.N) continue;
            const uint32_t at = base + (uint32_t)(o * stride + c) * 4;
            float v[4] = {0.f, 0.f, 0.f, 0.f};
            for (int r = 0; r < p.split; ++r) {
                const float4 x = ld_cluster_f4(map_rank(at, r));
                v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w;
            }
            finish4<T>(p.ep, m, n, v);
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

int sm_count() {
    static std::atomic<int> sms{0};
    int v = sms.load(std::memory_order_relaxed);
    if (!v) {
        int dev = 0;
        if (cudaGetDevice(&dev) != cudaSuccess ||
            cudaDeviceGetAttribute(&v, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || v <= 0)
            v = 152;
        sms.store(v, std::memory_order_relaxed);
    }
    return v;
}

template <typename T, int BN, bool ROUND>
cudaError_t run_tile(const LinearOperand& P, const LinearOperand& Q, TileParams& p, cudaStream_t s) {
    using S = TileShape<BN, ROUND>;
    CUtensorMap mP, mQ;
    if (!make_map(&mP, P, P.mn ? kTK : kTM) || !make_map(&mQ, Q, Q.mn ? kTK : BN)) return cudaErrorInvalidValue;
    p.tiles_p = (P.extent() + kTM - 1) / kTM;
    p.tiles_q = (Q.extent() + BN - 1) / BN;
    const int64_t tiles = p.tiles_p * p.tiles_q;
    // split the K loop while the CTAs still fit the GPU at once and each keeps four chunks
    const int64_t slots = (int64_t)sm_count() * (ROUND ? 1 : 2);
    p.split = 1;
    while (p.split < 8 && tiles * p.split * 2 <= slots && p.nk * p.pairs >= 8 * p.split) p.split *= 2;
    if (tiles * p.split > 2147483647LL) return cudaErrorInvalidConfiguration;
    cudaError_t e = smem_attr_once<linear_tile_kernel<T, BN, ROUND>>((int)S::kSmem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(tiles * p.split));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = S::kSmem;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = (unsigned)p.split;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    note_launches(1);
    return cudaLaunchKernelEx(&cfg, linear_tile_kernel<T, BN, ROUND>, mP, mQ, p);
}

template <typename T, bool ROUND>
cudaError_t pick_tile(const LinearOperand& P, const LinearOperand& Q, TileParams& p, cudaStream_t s) {
    const int64_t q = Q.extent();
    if (q <= 32 && !Q.mn) return run_tile<T, 32, ROUND>(P, Q, p, s);
    if (q <= 64) return run_tile<T, 64, ROUND>(P, Q, p, s);
    return run_tile<T, 128, ROUND>(P, Q, p, s);
}

}  // namespace

bool linear_tc_available() {
    static int sm103 = -1;
    if (sm103 < 0) {
        int dev = 0, major = 0, minor = 0;
        cudaGetDevice(&dev);
        cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev);
        cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev);
        sm103 = (major == 10 && minor == 3) ? 1 : 0;
    }
    return sm103 && encode_fn();
}

cudaError_t launch_linear_product(const LinearOperand& P0, const LinearOperand& Q0, LinearEpilogue ep, tda_dtype out,
                                  unsigned int* err, cudaStream_t s) {
    TileParams p;
    // a short side takes the narrow dimension of the tile
    p.swap = P0.extent() <= 64 && Q0.extent() > P0.extent();
    const LinearOperand &P = p.swap ? Q0 : P0, &Q = p.swap ? P0 : Q0;
    p.ep = ep;
    p.nk = (int)((P.depth() + kTK - 1) / kTK);
    p.pairs = P.planes == 3 ? 6 : 1;
    p.window = P.planes == 3 ? kWindow : p.nk;
    p.p_mn = P.mn;
    p.q_mn = Q.mn;
    p.err = err;
    const bool round = p.pairs > 1;
    if (out == TDA_BF16) return round ? cudaErrorInvalidValue : pick_tile<__nv_bfloat16, false>(P, Q, p, s);
    return round ? pick_tile<float, true>(P, Q, p, s) : pick_tile<float, false>(P, Q, p, s);
}

}  // namespace tda
