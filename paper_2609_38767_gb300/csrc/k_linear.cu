// k_linear.cu -- the linear layer around its tensor-core products (k_linear_tc.cu):
// the operands' planes, the factor B = dY act'(Z) with the bias gradient, and the
// order of the launches.
//
// All kernels here are bound by memory: a plane copy reads an operand once and
// writes it once (fp32: 4 bytes in, 6 out); the factor reads dY and Z and writes B.
#include "linear.cuh"

namespace tda {
namespace {

// ------------------------------------------------------------------ planes
// Rows of any type, stride and alignment -> bf16 planes with 16-byte aligned rows.
// fp32: x = x0 + x1 + x2, x0 = bf16(x), x1 = bf16(x - x0), x2 = x - x0 - x1: 24 bits in all.
constexpr int kPackThreads = 256;

struct PackJob {
    const void* src;
    int64_t rows, cols, ld;
    __nv_bfloat16* dst;
    int64_t ld_dst, plane;  // dst row length (a multiple of 8) and plane stride, elements
    int vec;                // rows may be read 16 bytes at a time
};
struct PackJobs {
    PackJob j[3];
};

__device__ __forceinline__ uint32_t bf16_bits(float x) { return __bfloat16_as_ushort(__float2bfloat16_rn(x)); }

template <typename T>
__device__ __forceinline__ void load8(const PackJob& j, int64_t r, int64_t c, T* x) {
    const T* s = (const T*)j.src + r * j.ld + c;
    if (j.vec && c + 8 <= j.cols) {
        const uint4* q = reinterpret_cast<const uint4*>(s);
        uint4* o = reinterpret_cast<uint4*>(x);
#pragma unroll
        for (int i = 0; i < (int)sizeof(T) / 2; ++i) o[i] = q[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = c + i < j.cols ? s[i] : T(0.f);
    }
}

template <typename T>
__global__ void __launch_bounds__(kPackThreads) pack_kernel(const __grid_constant__ PackJobs jobs) {
    chain_wait();
    chain_next();
    const PackJob& j = jobs.j[blockIdx.y];
    const int64_t per = j.ld_dst / 8, total = j.rows * per;
    for (int64_t i = (int64_t)blockIdx.x * kPackThreads + threadIdx.x; i < total; i += (int64_t)gridDim.x * kPackThreads) {
        const int64_t r = i / per, c = (i % per) * 8;
        alignas(16) T x[8];
        load8(j, r, c, x);
        __nv_bfloat16* d = j.dst + r * j.ld_dst + c;
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint4*>(d) = *reinterpret_cast<const uint4*>(x);
        } else {
            uint32_t w[3][4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                uint32_t b[3][2];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    float v = x[2 * k + h];
                    b[0][h] = bf16_bits(v);
                    // a finite value that rounds to infinity is cut instead
                    if ((b[0][h] & 0x7FFFu) == 0x7F80u && isfinite(v)) b[0][h] = __float_as_uint(v) >> 16;
                    const bool fin = isfinite(v);
                    v -= __uint_as_float(b[0][h] << 16);
                    b[1][h] = fin ? bf16_bits(v) : 0u;
                    v -= __uint_as_float(b[1][h] << 16);
                    b[2][h] = fin ? bf16_bits(v) : 0u;
                }
#pragma unroll
                for (int q = 0; q < 3; ++q) w[q][k] = b[q][0] | (b[q][1] << 16);
            }
#pragma unroll
            for (int q = 0; q < 3; ++q)
                *reinterpret_cast<uint4*>(d + q * j.plane) = make_uint4(w[q][0], w[q][1], w[q][2], w[q][3]);
        }
    }
}

// ------------------------------------------------------------------ factor and bias gradient
// CTA (x, y): columns of one block x rows of one run. A thread owns N columns (side by side and moved at once, or, where
// rows are not aligned, kColLanes apart and moved one by one: 4096 x 4095 bf16 25 us, with one column a thread 52) and
// every kRowLanes-th row of the run; the column sums of the rows are added over the row lanes in shared memory.
constexpr int kFacThreads = 256, kColLanes = 32, kRowLanes = kFacThreads / kColLanes;

struct FactorParams {
    const void* dY;
    const void* Z;
    void* B;
    int64_t ld_dy, ld_z, ld_b, M, N;
    int64_t run;   // rows per CTA
    float* sums;   // [runs][N] column sums, or NULL
};

template <typename T, int N>
struct alignas(sizeof(T) * N) Vec {
    T v[N];
};
__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void set_f(float* p, float x) { *p = x; }
__device__ __forceinline__ void set_f(__nv_bfloat16* p, float x) { *p = __float2bfloat16_rn(x); }

// have: a thread's columns inside the matrix.
template <typename T, int N, bool VEC>
__device__ __forceinline__ Vec<T, N> load_cols(const T* p, int have) {
    if (VEC) return *reinterpret_cast<const Vec<T, N>*>(p);
    Vec<T, N> x;
#pragma unroll
    for (int i = 0; i < N; ++i) x.v[i] = i < have ? p[i * kColLanes] : T(0.f);
    return x;
}
template <typename T, int N, bool VEC>
__device__ __forceinline__ void store_cols(T* p, const Vec<T, N>& x, int have) {
    if (VEC) {
        *reinterpret_cast<Vec<T, N>*>(p) = x;
    } else {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (i < have) p[i * kColLanes] = x.v[i];
    }
}

template <typename T, int ACT, int N, bool VEC>
__global__ void __launch_bounds__(kFacThreads, 4) factor_kernel(const __grid_constant__ FactorParams p) {
    constexpr int U = 2;  // rows in flight
    chain_next();
    const int lane = threadIdx.x % kColLanes, rl = threadIdx.x / kColLanes;
    const int64_t col = (int64_t)blockIdx.x * kColLanes * N + lane * (VEC ? N : 1);
    const int64_t left = (p.N - col + kColLanes - 1) / kColLanes;
    const int have = VEC ? N : (int)(left < N ? left : N);
    const int64_t r0 = (int64_t)blockIdx.y * p.run, r1 = r0 + p.run < p.M ? r0 + p.run : p.M;
    float sum[N] = {};
    if (col < p.N) {
        for (int64_t r = r0 + rl; r < r1; r += kRowLanes * U) {
            Vec<T, N> g[U], z[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t m = r + u * kRowLanes;
                if (m >= r1) break;
                g[u] = load_cols<T, N, VEC>((const T*)p.dY + m * p.ld_dy + col, have);
                if (ACT != TDA_ACT_NONE) z[u] = load_cols<T, N, VEC>((const T*)p.Z + m * p.ld_z + col, have);
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t m = r + u * kRowLanes;
                if (m >= r1) break;
                Vec<T, N> b;
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    float v = to_f(g[u].v[i]);
                    // a padded token (a zero of dY) has a zero factor whatever its Z holds
                    if (ACT != TDA_ACT_NONE && v != 0.f) v *= act_slope<ACT, sizeof(T) == 2>(to_f(z[u].v[i]));
                    sum[i] += v;
                    set_f(&b.v[i], v);
                }
                if (p.B) store_cols<T, N, VEC>((T*)p.B + m * p.ld_b + col, b, have);
            }
        }
    }
    if (!p.sums) return;
    __shared__ float sh[kRowLanes][kColLanes * N];
#pragma unroll
    for (int i = 0; i < N; ++i) sh[rl][VEC ? lane * N + i : i * kColLanes + lane] = sum[i];
    __syncthreads();
    for (int c = threadIdx.x; c < kColLanes * N; c += kFacThreads) {
        const int64_t n = (int64_t)blockIdx.x * kColLanes * N + c;
        if (n >= p.N) break;
        float s = sh[0][c];
#pragma unroll
        for (int i = 1; i < kRowLanes; ++i) s += sh[i][c];
        p.sums[(int64_t)blockIdx.y * p.N + n] = s;
    }
}

// db[n] = beta db[n] + sum of the runs' sums, in order. The factor's launch still writes the sums when this one starts:
// they are not __restrict__.
template <typename TG>
__global__ void bias_grad_kernel(const float* sums, int64_t runs, int64_t N, float beta, TG* db) {
    chain_wait();
    chain_next();
    const int64_t n = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (n >= N) return;
    float s = 0.f;
    for (int64_t r = 0; r < runs; r += 8) {
        float x[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = r + u < runs ? sums[(r + u) * N + n] : 0.f;
#pragma unroll
        for (int u = 0; u < 8; ++u) s += x[u];
    }
    if (beta != 0.f) s = fmaf(beta, to_f(db[n]), s);
    set_f(db + n, s);
}

// A matrix scaled in place: the gradients of an empty batch.
template <typename TG>
__global__ void scale_kernel(TG* x, int64_t rows, int64_t cols, int64_t ld, float beta) {
    const int64_t total = rows * cols;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (int64_t)gridDim.x * blockDim.x) {
        TG* p = x + (i / cols) * ld + i % cols;
        set_f(p, beta == 0.f ? 0.f : beta * to_f(*p));
    }
}

// ------------------------------------------------------------------ host side
bool rows16(const void* p, int64_t ld, size_t el) { return (((uintptr_t)p | (uintptr_t)(ld * (int64_t)el)) & 15) == 0; }
bool rows_by(const void* p, int64_t ld, size_t bytes, size_t el) {
    return !p || ((((uintptr_t)p | (uintptr_t)(ld * (int64_t)el)) & (bytes - 1)) == 0);
}
int64_t up8(int64_t x) { return (x + 7) & ~(int64_t)7; }
size_t up256(size_t x) { return (x + 255) & ~(size_t)255; }

// Columns of a CTA of the factor kernel.
int64_t factor_width(tda_dtype dt) { return (int64_t)kColLanes * (dt == TDA_BF16 ? 8 : 4); }

// Runs of rows of the factor kernel: as many as make at most one wave of four CTAs per SM (where one run of all rows
// does not make more), at least 32 rows each, at most 256 runs. Rounded up instead, the few CTAs of a second wave cost
// a whole one: 8192 tokens of 14336 bf16 columns (56 column blocks, 10 runs against 11) 227 us with their products,
// against 271. fp32 columns, whose blocks are half as wide, factor and bias sums: 4096 x 2048 silu 19.1 us (two waves
// 24.2), 2048 x 4096 tanh-gelu 19.8 (21.9), 8192 x 8192 silu 129.9 (128.4), 4096 x 8192 gelu 98.6 (92.4).
int64_t factor_run(int64_t M, int64_t N, tda_dtype dt) {
    const int64_t blocks = (N + factor_width(dt) - 1) / factor_width(dt);
    int64_t runs = 4 * train_sms() / blocks;
    if (runs < 1) runs = 1;
    if (runs > 256) runs = 256;
    int64_t run = (M + runs - 1) / runs;
    return run < 32 ? 32 : run;
}

template <typename T, int N, bool VEC>
void factor_act(int act, const FactorParams& p, dim3 grid, cudaStream_t s) {
    switch (act) {
        case TDA_ACT_RELU: factor_kernel<T, TDA_ACT_RELU, N, VEC><<<grid, kFacThreads, 0, s>>>(p); break;
        case TDA_ACT_GELU: factor_kernel<T, TDA_ACT_GELU, N, VEC><<<grid, kFacThreads, 0, s>>>(p); break;
        case TDA_ACT_GELU_TANH: factor_kernel<T, TDA_ACT_GELU_TANH, N, VEC><<<grid, kFacThreads, 0, s>>>(p); break;
        case TDA_ACT_SILU: factor_kernel<T, TDA_ACT_SILU, N, VEC><<<grid, kFacThreads, 0, s>>>(p); break;
        default: factor_kernel<T, TDA_ACT_NONE, N, VEC><<<grid, kFacThreads, 0, s>>>(p); break;
    }
}

template <typename T>
cudaError_t launch_factor(int act, FactorParams p, cudaStream_t s) {
    constexpr int kVec = 16 / sizeof(T);
    const bool vec = p.N % kVec == 0 && rows16(p.dY, p.ld_dy, sizeof(T)) &&
                     (act == TDA_ACT_NONE || rows16(p.Z, p.ld_z, sizeof(T))) &&
                     (!p.B || rows16(p.B, p.ld_b, sizeof(T)));
    const int64_t w = (int64_t)kColLanes * kVec;
    const dim3 grid((unsigned)((p.N + w - 1) / w), (unsigned)((p.M + p.run - 1) / p.run));
    note_launches(1);
    if (vec)
        factor_act<T, kVec, true>(act, p, grid, s);
    else
        factor_act<T, kVec, false>(act, p, grid, s);
    return cudaGetLastError();
}

// Whether an operand needs planes of its own in the workspace, and their bytes.
size_t plane_bytes(int64_t rows, int64_t cols, tda_dtype dt) {
    return up256((size_t)(dt == TDA_F32 ? 3 : 1) * (size_t)rows * (size_t)up8(cols) * 2);
}

struct Planner {
    PackJobs jobs;
    int count = 0;
    tda_dtype dt;
    char* ws;
    size_t at = 0;

    LinearOperand add(const void* p, int64_t rows, int64_t cols, int64_t ld) {
        LinearOperand o;
        o.p = p, o.rows = rows, o.cols = cols, o.ld = ld;
        o.plane_stride = 0, o.planes = 1, o.mn = false;
        if (dt == TDA_BF16 && rows16(p, ld, 2)) return o;
        PackJob& j = jobs.j[count++];
        j.src = p, j.rows = rows, j.cols = cols, j.ld = ld;
        j.dst = (__nv_bfloat16*)(ws + at);
        j.ld_dst = up8(cols);
        j.plane = rows * j.ld_dst;
        j.vec = rows16(p, ld, dt == TDA_F32 ? 4 : 2);
        at += plane_bytes(rows, cols, dt);
        o.p = j.dst, o.ld = j.ld_dst, o.plane_stride = j.plane, o.planes = dt == TDA_F32 ? 3 : 1;
        return o;
    }
    cudaError_t run(bool chained, cudaStream_t s) {
        if (!count) return cudaSuccess;
        int64_t most = 0;
        for (int i = 0; i < count; ++i) {
            const int64_t t = (jobs.j[i].rows * (jobs.j[i].ld_dst / 8) + kPackThreads - 1) / kPackThreads;
            if (t > most) most = t;
        }
        const int64_t cap = train_sms() * 16;
        const dim3 grid((unsigned)(most < cap ? most : cap), (unsigned)count);
        return launch_chained(chained, dt == TDA_F32 ? pack_kernel<float> : pack_kernel<__nv_bfloat16>, grid,
                              dim3(kPackThreads), 0, s, jobs);
    }
};

// How far the epilogue's tensors are aligned.
void align_epilogue(LinearEpilogue* e, tda_dtype out) {
    const size_t el = out == TDA_BF16 ? 2 : 4;
    auto all = [&](size_t bytes) {
        return rows_by(e->Y, e->ld_y, bytes, el) && rows_by(e->Z, e->ld_z, bytes, el) &&
               rows_by(e->R, e->ld_r, bytes, el) && rows_by(e->bias, 0, bytes, el);
    };
    e->vec = all(4 * el);
    e->wide = all(16);
}

LinearEpilogue plain_epilogue(int64_t M, int64_t N, void* Y, int64_t ld_y, tda_dtype out) {
    LinearEpilogue e = {};
    e.M = M, e.N = N, e.Y = Y, e.ld_y = ld_y, e.act = TDA_ACT_NONE;
    align_epilogue(&e, out);
    return e;
}

}  // namespace

// ------------------------------------------------------------------ entry points of this file
// Scratch of a forward: planes of X and W where they need them.
static bool needs_planes(tda_dtype dt, const void* p, int64_t ld) { return dt == TDA_F32 || !rows16(p, ld, 2); }

// Rows up to which dW is written by plain rank-M updates.
constexpr int64_t kOuterMost = 16;
static bool few_cols(const LinearBackward& b) { return b.dt == TDA_F32 && linear_rows_preferred(b.M, b.dt); }

size_t linear_forward_ws(const LinearForward& f) {
    size_t b = 0;
    if (linear_rows_preferred(f.M, f.dt)) return 0;
    if (needs_planes(f.dt, f.X, f.ld_x)) b += plane_bytes(f.M, f.d_in, f.dt);
    if (needs_planes(f.dt, f.W, f.ld_w)) b += plane_bytes(f.d_out, f.d_in, f.dt);
    return b;
}

size_t linear_backward_ws(const LinearBackward& b) {
    size_t n = 0;
    const void* G = b.B ? b.B : b.dY;
    const int64_t ld_g = b.B ? b.ld_b : b.ld_dy;
    const bool dX = b.dX && !few_cols(b), dW = b.dW && b.M > kOuterMost;
    if ((dX || dW) && needs_planes(b.dt, G, ld_g)) n += plane_bytes(b.M, b.d_out, b.dt);
    if (dX && needs_planes(b.dt, b.W, b.ld_w)) n += plane_bytes(b.d_out, b.d_in, b.dt);
    if (dW && needs_planes(b.dt, b.X, b.ld_x)) n += plane_bytes(b.M, b.d_in, b.dt);
    if (b.db) {
        const int64_t run = factor_run(b.M, b.d_out, b.dt);
        n += up256(sizeof(float) * (size_t)((b.M + run - 1) / run) * (size_t)b.d_out);
    }
    return n;
}

size_t linear_ws_bound(bool backward, int64_t M, int64_t d_in, int64_t d_out, tda_dtype dt, bool packed) {
    const bool in = packed || dt == TDA_F32 || d_in % 8, out = packed || dt == TDA_F32 || d_out % 8;
    size_t n = in ? plane_bytes(M, d_in, dt) + plane_bytes(d_out, d_in, dt) : 0;
    if (!backward) return n;
    if (out) n += plane_bytes(M, d_out, dt);
    const int64_t run = factor_run(M, d_out, dt);
    return n + up256(sizeof(float) * (size_t)((M + run - 1) / run) * (size_t)d_out);
}

cudaError_t launch_linear_forward(const LinearForward& f, void* ws, unsigned int* err, cudaStream_t s) {
    LinearEpilogue ep = plain_epilogue(f.M, f.d_out, f.Y, f.ld_y, f.dt);
    ep.bias = f.bias;
    ep.R = f.R, ep.ld_r = f.ld_r, ep.r_scale = 1.f;
    ep.Z = f.Z, ep.ld_z = f.ld_z;
    ep.act = f.act;
    align_epilogue(&ep, f.dt);
    if (linear_rows_preferred(f.M, f.dt)) return launch_linear_rows(f.X, f.ld_x, f.W, f.ld_w, f.d_in, ep, f.dt, s);
    Planner pl;
    pl.dt = f.dt;
    pl.ws = (char*)ws;
    const LinearOperand X = pl.add(f.X, f.M, f.d_in, f.ld_x), W = pl.add(f.W, f.d_out, f.d_in, f.ld_w);
    cudaError_t e = pl.run(false, s);
    if (e != cudaSuccess) return e;
    const LinearProduct pr = {X, W, ep, f.dt};
    return launch_linear_products(&pr, 1, pl.count > 0, err, s);
}

cudaError_t launch_linear_backward(const LinearBackward& b, void* ws, unsigned int* err, cudaStream_t s) {
    cudaError_t e;
    const int64_t run = factor_run(b.M, b.d_out, b.dt), runs = (b.M + run - 1) / run;
    float* sums = nullptr;
    Planner pl;
    pl.dt = b.dt;
    pl.ws = (char*)ws;
    if (b.db) {
        sums = (float*)ws;
        pl.at = up256(sizeof(float) * (size_t)runs * (size_t)b.d_out);
    }
    if (b.B || b.db) {
        FactorParams p;
        p.dY = b.dY, p.Z = b.Z, p.B = b.B, p.ld_dy = b.ld_dy, p.ld_z = b.ld_z, p.ld_b = b.ld_b;
        p.M = b.M, p.N = b.d_out, p.run = run, p.sums = sums;
        e = b.dt == TDA_BF16 ? launch_factor<__nv_bfloat16>(b.act, p, s) : launch_factor<float>(b.act, p, s);
        if (e != cudaSuccess) return e;
    }
    bool chained = b.B || b.db;
    if (b.db) {
        const dim3 grid((unsigned)((b.d_out + 127) / 128));
        e = b.gt == TDA_BF16 ? launch_chained(true, bias_grad_kernel<__nv_bfloat16>, grid, dim3(128), 0, s,
                                              (const float*)sums, runs, b.d_out, b.beta, (__nv_bfloat16*)b.db)
                             : launch_chained(true, bias_grad_kernel<float>, grid, dim3(128), 0, s, (const float*)sums,
                                              runs, b.d_out, b.beta, (float*)b.db);
        if (e != cudaSuccess) return e;
    }
    // few rows: dW (and dX of fp32 layers) read their operands as they are
    const void* F = b.B ? b.B : b.dY;
    const int64_t ld_f = b.B ? b.ld_b : b.ld_dy;
    const bool outer = b.dW && b.M <= kOuterMost, few = b.dX && few_cols(b);
    if (few) {
        e = launch_linear_cols((const float*)F, ld_f, (const float*)b.W, b.ld_w, (float*)b.dX, b.ld_dx, b.M, b.d_out, b.d_in,
                               chained, s);
        if (e != cudaSuccess) return e;
        chained = true;
    }
    if (outer) {
        e = launch_linear_outer(F, ld_f, b.X, b.ld_x, b.M, b.d_out, b.d_in, b.dt, b.dW, b.ld_dw, b.gt, b.beta, chained, s);
        if (e != cudaSuccess) return e;
        chained = true;
    }
    const bool dX = b.dX && !few, dW = b.dW && !outer;
    if (!dX && !dW) return cudaSuccess;
    // the products read the factor as it is stored: B, or dY itself without an activation
    const LinearOperand G = b.B ? pl.add(b.B, b.M, b.d_out, b.ld_b) : pl.add(b.dY, b.M, b.d_out, b.ld_dy);
    LinearOperand W = {}, X = {};
    if (dX) W = pl.add(b.W, b.d_out, b.d_in, b.ld_w);
    if (dW) X = pl.add(b.X, b.M, b.d_in, b.ld_x);
    if ((e = pl.run(chained, s)) != cudaSuccess) return e;
    LinearProduct pr[2];
    int count = 0;
    if (dX) {
        W.mn = true;  // the contraction runs over W's rows
        pr[count++] = {G, W, plain_epilogue(b.M, b.d_in, b.dX, b.ld_dx, b.dt), b.dt};
    }
    if (dW) {
        LinearOperand Gt = G;
        Gt.mn = X.mn = true;  // over the tokens
        LinearEpilogue ep = plain_epilogue(b.d_out, b.d_in, b.dW, b.ld_dw, b.gt);
        if (b.beta != 0.f) ep.R = b.dW, ep.ld_r = b.ld_dw, ep.r_scale = b.beta;
        align_epilogue(&ep, b.gt);
        pr[count++] = {Gt, X, ep, b.gt};
    }
    return launch_linear_products(pr, count, chained || pl.count > 0, err, s);
}

// beta x for an empty batch.
cudaError_t launch_scale_matrix(tda_dtype dt, void* x, int64_t rows, int64_t cols, int64_t ld, float beta,
                                cudaStream_t s) {
    const int64_t blocks = (rows * cols + 255) / 256, cap = train_sms() * 16;
    const unsigned grid = (unsigned)(blocks < cap ? blocks : cap);
    note_launches(1);
    if (dt == TDA_BF16)
        scale_kernel<<<grid, 256, 0, s>>>((__nv_bfloat16*)x, rows, cols, ld, beta);
    else
        scale_kernel<<<grid, 256, 0, s>>>((float*)x, rows, cols, ld, beta);
    return cudaGetLastError();
}

}  // namespace tda
