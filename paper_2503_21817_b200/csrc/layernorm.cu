// Layer normalisation of packed rows (the vision tower's blocks and its projector; the decoder's RMS norm is
// fused into the routing, prenorm.cu):
//   forward : mean, var over the C columns;  rstd = (var + eps)^-1/2;  y = (x - mean) rstd gamma + beta
//   backward: xh = (x - mean) rstd, t = dy gamma;  dx = rstd (t - mean_c(t) - xh mean_c(t xh));
//             dgamma = sum_rows dy xh;  dbeta = sum_rows dy
// HBM-bound: a row is read once into registers (16-byte loads, at most four per thread), the variance is
// the mean of squared deviations (a second look at the registers, not E[x^2] - mean^2), and the backward
// reads x and dy once for both its results.  Statistics and sums are fp32 in a fixed order (no atomics).
// Measured (B200, bf16, replayed from a graph): forward 9376 x 4096 in 25.9 us (5.9 TB/s, 0.90 of the copy rate),
// 577 x 1024 in 2.4 us; backward 4927 x 5120 in 40.4 us (3.7 TB/s; rows 36, partial sums 4; fp32 77 us, 3.9 TB/s, with 92
// bytes spilled), 4096 x 6144, one row per SM, 45 us (3.4 TB/s): an SM has two rows at a time and 20 warps that
// issue in 57 % of its cycles (latency of a row's chain: sums, barrier, results).  From 42.8 us, the next row's sums
// before this row's results (44.5) did not help, nor half the shared-memory reads (42.5); partial sums with 32 lanes per
// column instead of eight did (2 us less).
#include "common.cuh"

namespace skipffn {

namespace {

constexpr int LN_NV = 4;                      // 16-byte vectors per thread

template <typename T> struct Vec { static constexpr int N = 16 / (int)sizeof(T); };   // elements of a vector

template <int N> __device__ __forceinline__ uint4 pack(const float (&v)[N])
{
    uint32_t u[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (N == 8) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(v[2 * k], v[2 * k + 1]);
            u[k] = *reinterpret_cast<const uint32_t *>(&h);
        } else {
            u[k] = __float_as_uint(v[k]);
        }
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
}

__device__ __forceinline__ float warp_add(float v)
{
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
// Barrier of the `threads` threads of row group `id` (every group of a CTA has its own)
__device__ __forceinline__ void group_sync(int id, int threads)
{
    asm volatile("bar.sync %0, %1;" ::"r"(id + 1), "r"(threads) : "memory");
}
// Sum over a row group in a fixed order, valid in every thread.  `red` holds one float per warp of the
// group and alternates between two halves from call to call, so one barrier per call is enough.
__device__ __forceinline__ float group_add(float v, float *red, int id, int threads)
{
    v = warp_add(v);
    if (threads == 32) return v;
    const int w = threadIdx.x >> 5;
    if ((threadIdx.x & 31) == 0) red[w] = v;
    group_sync(id, threads);
    float s = 0.0f;
    for (int k = 0; k < threads / 32; ++k) s += red[k];
    return s;
}

// 16 bytes of a row as fp32 pairs, and back
template <int N> __device__ __forceinline__ void unpack2(const uint4 &q, uint64_t (&v)[N / 2])
{
    const uint32_t u[4] = {q.x, q.y, q.z, q.w};
    if constexpr (N == 8) {
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = pair2(__uint_as_float(u[k] << 16), __uint_as_float(u[k] & 0xffff0000u));
    } else {
        v[0] = pair2(__uint_as_float(u[0]), __uint_as_float(u[1]));
        v[1] = pair2(__uint_as_float(u[2]), __uint_as_float(u[3]));
    }
}
template <int N> __device__ __forceinline__ uint4 pack2(const uint64_t (&v)[N / 2])
{
    float f[N];
#pragma unroll
    for (int k = 0; k < N / 2; ++k) unpair2(v[k], f[2 * k], f[2 * k + 1]);
    return pack(f);
}
// Forward.  ONE_WARP: a row per warp, blockDim.y of them; else a row per CTA.  The CTA walks rows with the grid's
// stride; the next row is on its way while the current one is worked on.  gamma and beta sit in shared memory in
// their own type (as fp32 their reads alone, two-way conflicts included, took 17 of 39 us at 9376 x 4096),
// arithmetic is on pairs (18 instructions per element before), and a CTA has one barrier (a named one per group
// held an SM to four CTAs).  FULL: every thread owns LN_NV vectors.
constexpr int LN_FWD_REGS = 80, LN_FWD_REGS_FP32 = 64;       // fp32: CTAs of up to 1024 threads
template <typename T, bool ONE_WARP, bool FULL>
__global__ void __maxnreg__(sizeof(T) == 2 ? LN_FWD_REGS : LN_FWD_REGS_FP32)
k_layernorm_fwd(const T *x, const T *__restrict__ gamma, const T *__restrict__ beta, int64_t rows, int C, float eps, T *y,
                float *__restrict__ mean_out, float *__restrict__ rstd_out)
{
    constexpr int N = Vec<T>::N, P = N / 2;
    __shared__ float red[2][2][32];
    extern __shared__ uint4 affine[];                      // gamma [C], beta [C]
    const int tx = threadIdx.x, threads = ONE_WARP ? 32 : blockDim.x, vecs = C / N;
    const int64_t step = (int64_t)gridDim.x * (ONE_WARP ? blockDim.y : 1);
    int64_t row = (int64_t)blockIdx.x * (ONE_WARP ? blockDim.y : 1) + threadIdx.y;
    auto owns = [&](int k) { return FULL || tx + k * threads < vecs; };
    auto row_sum = [&](uint64_t v, float *r) {
        float a, b;
        unpair2(v, a, b);
        a = warp_add(a + b);
        if (ONE_WARP) return a;
        if ((tx & 31) == 0) r[tx >> 5] = a;
        __syncthreads();
        a = 0.0f;
        for (int k = 0; k < threads / 32; ++k) a += r[k];
        return a;
    };
    pdl_enter();
    uint4 xq[LN_NV];
    auto fetch = [&](int64_t r) {
        const uint4 *src = reinterpret_cast<const uint4 *>(x + r * C) + tx;
#pragma unroll
        for (int k = 0; k < LN_NV; ++k)
            if (owns(k)) xq[k] = src[k * threads];
    };
#pragma unroll
    for (int k = 0; k < LN_NV; ++k) xq[k] = make_uint4(0, 0, 0, 0);
    if (row < rows) fetch(row);
    for (int i = threadIdx.y * blockDim.x + tx; i < vecs; i += blockDim.x * blockDim.y) {
        affine[i] = reinterpret_cast<const uint4 *>(gamma)[i];
        affine[vecs + i] = beta ? reinterpret_cast<const uint4 *>(beta)[i] : make_uint4(0, 0, 0, 0);
    }
    __syncthreads();
    for (int turn = 0; row < rows; row += step, turn ^= 1) {
        uint64_t v[LN_NV][P], s = 0, ss = 0;
#pragma unroll
        for (int k = 0; k < LN_NV; ++k) {
            unpack2<N>(xq[k], v[k]);
#pragma unroll
            for (int e = 0; e < P; ++e) s = add2(s, v[k][e]);
        }
        if (row + step < rows) fetch(row + step);
        const float mean = row_sum(s, red[turn][0]) / (float)C;
        const uint64_t neg = pair2(-mean, -mean);
#pragma unroll
        for (int k = 0; k < LN_NV; ++k)
            if (owns(k))
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    v[k][e] = add2(v[k][e], neg);
                    ss = fma2(v[k][e], v[k][e], ss);
                }
        const float rstd = 1.0f / sqrtf(row_sum(ss, red[turn][1]) / (float)C + eps);
        const uint64_t r2 = pair2(rstd, rstd);
        uint4 *dst = reinterpret_cast<uint4 *>(y + row * C) + tx;
#pragma unroll
        for (int k = 0; k < LN_NV; ++k) {
            if (!owns(k)) break;
            uint64_t g[P], b[P];
            unpack2<N>(affine[tx + k * threads], g);
            unpack2<N>(affine[vecs + tx + k * threads], b);
#pragma unroll
            for (int e = 0; e < P; ++e) v[k][e] = fma2(mul2(v[k][e], r2), g[e], b[e]);
            dst[k * threads] = pack2<N>(v[k]);
        }
        if (tx == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
    }
}

__device__ __forceinline__ void copy_async16(uint32_t dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copy_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_async_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// Sums of a and b over a warp with six shuffles instead of ten: the lanes' halves take one sum each.  Lanes 0..15
// get the sum of a, lanes 16..31 that of b.
__device__ __forceinline__ float warp_add_two(float a, float b)
{
    const bool high = (threadIdx.x & 16) != 0;
    float v = high ? b : a;
    v += __shfl_xor_sync(0xffffffffu, high ? a : b, 16);
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}

// Backward: group g of CTA b walks rows b groups + g, + grid x groups, ...; dx row by row, dgamma and dbeta of the
// group's rows in registers (16 columns per thread).  A thread copies its own columns of the next rows to its own
// words of shared memory asynchronously, so nothing but the two row sums needs a barrier and no registers wait for
// loads.  At the end the groups add up in order through shared memory and the CTA leaves one partial row of each
// in part[b][2][C].
constexpr int LN_BWD_THREADS = 640, LN_BWD_COLS = 16;
template <typename T> struct LnBwd {
    static constexpr int N = Vec<T>::N, P = N / 2, NV = LN_BWD_COLS / N;
    static constexpr int STAGES = sizeof(T) == 2 ? 3 : 2;                    // rows on their way, the current one included
    static size_t smem(int C, int threads, int groups)
    {
        return (size_t)threads * groups * STAGES * 2 * NV * 16 + C * (sizeof(T) + (groups > 1 ? 2 * sizeof(float) : 0));
    }
};
template <typename T, bool FULL>
__global__ void __launch_bounds__(LN_BWD_THREADS, 1)
k_layernorm_bwd(const T *dy, const T *x, const T *__restrict__ gamma, const float *__restrict__ mean_in,
                const float *__restrict__ rstd_in, int64_t rows, int C, T *dx, float *__restrict__ part)
{
    using L = LnBwd<T>;
    constexpr int N = L::N, P = L::P, NV = L::NV, STAGES = L::STAGES;
    __shared__ float2 red[2][LN_BWD_THREADS / 32];
    extern __shared__ uint4 dyn[];
    const int tx = threadIdx.x, threads = blockDim.x, id = threadIdx.y, groups = blockDim.y, vecs = C / N, all = threads * groups;
    const int64_t step = (int64_t)gridDim.x * groups;
    uint4 *ring = dyn + id * threads + tx;             // [stage][x, dy][k][thread]
    uint4 *gam = dyn + (size_t)all * STAGES * 2 * NV;  // gamma [C]; with several groups also their sums [2][C]
    float *sums = reinterpret_cast<float *>(gam + vecs);
    const float inv_c = 1.0f / (float)C;
    uint64_t dg[NV][P], db[NV][P];
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
        for (int e = 0; e < P; ++e) dg[k][e] = db[k][e] = 0;
    auto owns = [&](int k) { return FULL || tx + k * threads < vecs; };
    auto slot = [&](int stage, int which, int k) { return ring + (size_t)((stage * 2 + which) * NV + k) * all; };
    auto fetch = [&](int64_t row, int stage) {         // always one copy group, so that the waits can count
        if (row < rows) {
            const uint4 *xs = reinterpret_cast<const uint4 *>(x + row * C) + tx, *ys = reinterpret_cast<const uint4 *>(dy + row * C) + tx;
#pragma unroll
            for (int k = 0; k < NV; ++k)
                if (owns(k)) {
                    copy_async16((uint32_t)__cvta_generic_to_shared(slot(stage, 0, k)), xs + k * threads);
                    copy_async16((uint32_t)__cvta_generic_to_shared(slot(stage, 1, k)), ys + k * threads);
                }
        }
        copy_async_commit();
    };
    pdl_enter();
    int64_t row = (int64_t)blockIdx.x * groups + id;
#pragma unroll
    for (int k = 0; k < STAGES - 1; ++k) fetch(row + k * step, k);
    float mean_next = row < rows ? mean_in[row] : 0.0f, rstd_next = row < rows ? rstd_in[row] : 0.0f;
    for (int i = id * threads + tx; i < vecs; i += all) gam[i] = reinterpret_cast<const uint4 *>(gamma)[i];
    __syncthreads();
    int stage = 0;
    for (int turn = 0; row < rows; row += step, turn ^= 1) {
        const float rstd = rstd_next;
        const uint64_t neg_mean = pair2(-mean_next, -mean_next), r2 = pair2(rstd, rstd);
        if (row + step < rows) { mean_next = mean_in[row + step]; rstd_next = rstd_in[row + step]; }
        fetch(row + (STAGES - 1) * step, stage == 0 ? STAGES - 1 : stage - 1);
        copy_async_wait<STAGES - 1>();
        // x - mean, dy and dy gamma of vector k, read twice from shared memory: held in registers as read (24 for
        // bf16) the row cost as much (42.5 for 42.8 us), held unpacked it spills
        auto vectors = [&](int k, uint64_t (&xm)[P], uint64_t (&yv)[P], uint64_t (&t)[P]) {
            uint64_t g[P];
            unpack2<N>(*slot(stage, 0, k), xm);
            unpack2<N>(*slot(stage, 1, k), yv);
            unpack2<N>(gam[tx + k * threads], g);
#pragma unroll
            for (int e = 0; e < P; ++e) {
                xm[e] = add2(xm[e], neg_mean);
                t[e] = mul2(yv[e], g[e]);
            }
        };
        uint64_t p0 = 0, p1 = 0;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (owns(k)) {
                uint64_t xm[P], yv[P], t[P];
                vectors(k, xm, yv, t);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    const uint64_t xh = mul2(xm[e], r2);
                    p0 = add2(p0, t[e]);
                    p1 = fma2(t[e], xh, p1);
                    dg[k][e] = fma2(yv[e], xh, dg[k][e]);
                    db[k][e] = add2(db[k][e], yv[e]);
                }
            }
        float a, b, c, d;
        unpair2(p0, a, b);
        unpair2(p1, c, d);
        float s = warp_add_two(a + b, c + d), s0, s1;
        if (threads > 32) {
            float2 *r = red[turn] + id * (threads / 32);
            if ((tx & 15) == 0) reinterpret_cast<float *>(r + (tx >> 5))[(tx >> 4) & 1] = s;
            group_sync(id, threads);
            uint64_t sum = 0;
#pragma unroll 5
            for (int k = 0; k < threads / 32; ++k) sum = add2(sum, *reinterpret_cast<const uint64_t *>(r + k));
            unpair2(sum, s0, s1);
        } else {
            s0 = __shfl_sync(0xffffffffu, s, 0);
            s1 = __shfl_sync(0xffffffffu, s, 16);
        }
        // dx = rstd t + xh (rstd m1) + rstd m0 with m0, m1 the means of -t and -t xh  (rstd^2 could leave fp32's range)
        s0 *= -inv_c * rstd;
        s1 *= -inv_c * rstd;
        const uint64_t m0 = pair2(s0, s0), m1 = pair2(s1, s1);
        uint4 *dst = reinterpret_cast<uint4 *>(dx + row * C) + tx;
#pragma unroll
        for (int k = 0; k < NV; ++k)
            if (owns(k)) {
                uint64_t xm[P], yv[P], t[P];
                vectors(k, xm, yv, t);
#pragma unroll
                for (int e = 0; e < P; ++e) xm[e] = fma2(mul2(xm[e], r2), m1, fma2(t[e], r2, m0));
                dst[k * threads] = pack2<N>(xm);
            }
        if (++stage == STAGES) stage = 0;
    }
    copy_async_wait<0>();
    if (part == nullptr) return;
    float *out = part + (int64_t)blockIdx.x * 2 * C;
    for (int g = 0; g < groups; ++g) {
        if (groups > 1) __syncthreads();
        if (g != id) continue;
        float *acc = g == groups - 1 ? out : sums;
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            const int i = tx + k * threads;
            if (i >= vecs) break;
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const int c = i * N + 2 * e;
                float2 a, b;
                unpair2(dg[k][e], a.x, a.y);
                unpair2(db[k][e], b.x, b.y);
                if (g) {
                    const float2 pa = *reinterpret_cast<const float2 *>(sums + c), pb = *reinterpret_cast<const float2 *>(sums + C + c);
                    a.x += pa.x; a.y += pa.y; b.x += pb.x; b.y += pb.y;
                }
                *reinterpret_cast<float2 *>(acc + c) = a;
                *reinterpret_cast<float2 *>(acc + C + c) = b;
            }
        }
    }
}

// Rows too long for the registers of the kernel above: dx alone, one CTA per row, sums first.
constexpr int LN_LONG_THREADS = 512;
template <typename T>
__global__ void __launch_bounds__(LN_LONG_THREADS)
k_layernorm_bwd_rows(const T *dy, const T *x, const T *__restrict__ gamma, const float *__restrict__ mean_in,
                     const float *__restrict__ rstd_in, int C, T *dx)
{
    __shared__ float red[2][LN_LONG_THREADS / 32];
    pdl_enter();
    const int64_t row = blockIdx.x;
    const float mean = mean_in[row], rstd = rstd_in[row];
    const T *xs = x + row * C, *ys = dy + row * C;
    float s0 = 0.0f, s1 = 0.0f;
    for (int c = 4 * threadIdx.x; c < C; c += 4 * LN_LONG_THREADS) {
        float xv[4], yv[4], g[4];
        load4(xs + c, xv); load4(ys + c, yv); load4(gamma + c, g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            s0 = fmaf(yv[e], g[e], s0);
            s1 = fmaf(yv[e] * g[e], (xv[e] - mean) * rstd, s1);
        }
    }
    s0 = group_add(s0, red[0], 0, LN_LONG_THREADS) / (float)C;
    s1 = group_add(s1, red[1], 0, LN_LONG_THREADS) / (float)C;
    for (int c = 4 * threadIdx.x; c < C; c += 4 * LN_LONG_THREADS) {
        float xv[4], yv[4], g[4], o[4];
        load4(xs + c, xv); load4(ys + c, yv); load4(gamma + c, g);
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = rstd * (fmaf(yv[e], g[e], -s0) - (xv[e] - mean) * rstd * s1);
        store4(dx + row * C + c, o);
    }
}
// ... and the column sums of its rows, one column per lane, 8 row lanes added in order: part[chunk][2][C]
constexpr int LN_COLS = 32, LN_LANES = 8;
template <typename T>
__global__ void __launch_bounds__(LN_COLS * LN_LANES)
k_layernorm_bwd_cols(const T *dy, const T *x, const float *__restrict__ mean_in, const float *__restrict__ rstd_in,
                     int64_t rows, int C, float *__restrict__ part)
{
    __shared__ float red[2][LN_LANES][LN_COLS];
    pdl_enter();
    const int64_t per = (rows + gridDim.y - 1) / gridDim.y, r0 = blockIdx.y * per, r1 = r0 + per < rows ? r0 + per : rows;
    const int cl = threadIdx.x % LN_COLS, lane = threadIdx.x / LN_COLS, c = blockIdx.x * LN_COLS + cl;
    float g = 0.0f, b = 0.0f;
    if (c < C)
#pragma unroll 4
        for (int64_t r = r0 + lane; r < r1; r += LN_LANES) {
            const float d = to_f32(dy[r * C + c]);
            g = fmaf(d, (to_f32(x[r * C + c]) - mean_in[r]) * rstd_in[r], g);
            b += d;
        }
    red[0][lane][cl] = g;
    red[1][lane][cl] = b;
    __syncthreads();
    if (lane < 2 && c < C) {
        float s = 0.0f;
#pragma unroll
        for (int l = 0; l < LN_LANES; ++l) s += red[lane][l][cl];
        part[((int64_t)blockIdx.y * 2 + lane) * C + c] = s;
    }
}

// Sum of the partial rows, 32 columns per CTA: warp w adds parts w, w + 32, ... of every column (all its loads in flight),
// then the warps' sums of column w.  blockIdx.y: 0 dgamma, 1 dbeta.
constexpr int SUM_COLS = 32, SUM_LOADS = (LN_MAX_PARTS + 31) / 32;
template <typename TO>
__global__ void __launch_bounds__(SUM_COLS * 32)
k_layernorm_sum_parts(const float *__restrict__ part, int parts, int C, TO *__restrict__ dgamma, TO *__restrict__ dbeta)
{
    __shared__ float red[32][SUM_COLS + 1];
    pdl_enter();
    TO *dst = blockIdx.y ? dbeta : dgamma;
    if (dst == nullptr) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c = blockIdx.x * SUM_COLS + lane;
    float v[SUM_LOADS], s = 0.0f;
#pragma unroll
    for (int k = 0; k < SUM_LOADS; ++k) {
        const int q = warp + 32 * k;
        v[k] = q < parts && c < C ? part[((int64_t)q * 2 + blockIdx.y) * C + c] : 0.0f;
    }
#pragma unroll
    for (int k = 0; k < SUM_LOADS; ++k) s += v[k];
    red[warp][lane] = s;
    __syncthreads();
    s = warp_add(red[lane][warp]);
    const int out = blockIdx.x * SUM_COLS + warp;
    if (lane == 0 && out < C) dst[out] = from_f32<TO>(s);
}

// threads of a row group: enough for LN_NV vectors each, a whole number of warps
template <typename T> int group_threads(int C)
{
    const int vecs = C / Vec<T>::N;
    return ((vecs + LN_NV - 1) / LN_NV + 31) / 32 * 32;
}

constexpr int LN_MAX_DEVICES = 64;
cudaError_t device_sms(int &sms)
{
    static int by_dev[LN_MAX_DEVICES];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= LN_MAX_DEVICES) return cudaErrorInvalidDevice;
    if (by_dev[dev] == 0) {
        int n = 0;
        const cudaError_t e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
        if (e != cudaSuccess) return e;
        by_dev[dev] = n;
    }
    sms = by_dev[dev] < LN_MAX_PARTS ? by_dev[dev] : LN_MAX_PARTS;
    return cudaSuccess;
}

template <typename KernelT, typename... Args>
cudaError_t launch_smem(KernelT kern, dim3 grid, dim3 block, size_t smem, cudaStream_t s, Args... args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, args...);
}

// Resident CTAs of a forward launch: as many as registers and gamma and beta in shared memory allow.
template <typename T, bool ONE_WARP, bool FULL>
cudaError_t fwd_k(const T *x, const T *gamma, const T *beta, int64_t rows, int C, float eps, T *y, float *mean, float *rstd, int t,
                  cudaStream_t s)
{
    constexpr int WARP_ROWS = 8;
    int sms = 0;
    cudaError_t e = device_sms(sms);
    if (e != cudaSuccess) return e;
    const int groups = ONE_WARP ? WARP_ROWS : 1, threads = t * groups;
    const size_t smem = (size_t)2 * C * sizeof(T);
    if (smem > 32 * 1024) {
        e = cudaFuncSetAttribute(k_layernorm_fwd<T, ONE_WARP, FULL>, cudaFuncAttributeMaxDynamicSharedMemorySize, 2 * LN_MAX_C * 4);
        if (e != cudaSuccess) return e;
    }
    const int by_regs = 65536 / (threads * (sizeof(T) == 2 ? LN_FWD_REGS : LN_FWD_REGS_FP32)), by_smem = (int)(200 * 1024 / (smem + 2048));
    const int ctas = by_regs < by_smem ? (by_regs > 0 ? by_regs : 1) : (by_smem > 0 ? by_smem : 1);
    const int64_t need = (rows + groups - 1) / groups, most = (int64_t)sms * ctas;
    return launch_smem(k_layernorm_fwd<T, ONE_WARP, FULL>, dim3((unsigned)(need < most ? need : most)), dim3(t, groups), smem, s, x, gamma,
                       beta, rows, C, eps, y, mean, rstd);
}
template <typename T>
cudaError_t fwd_t(const T *x, const T *gamma, const T *beta, int64_t rows, int C, float eps, T *y, float *mean, float *rstd,
                  cudaStream_t s)
{
    const int t = group_threads<T>(C);
    const bool full = C == t * LN_NV * Vec<T>::N;
    if (t == 32) return full ? fwd_k<T, true, true>(x, gamma, beta, rows, C, eps, y, mean, rstd, t, s)
                             : fwd_k<T, true, false>(x, gamma, beta, rows, C, eps, y, mean, rstd, t, s);
    return full ? fwd_k<T, false, true>(x, gamma, beta, rows, C, eps, y, mean, rstd, t, s)
                : fwd_k<T, false, false>(x, gamma, beta, rows, C, eps, y, mean, rstd, t, s);
}

template <typename T>
cudaError_t bwd_t(const T *dy, const T *x, const T *gamma, const float *mean, const float *rstd, int64_t rows, int C, T *dx,
                  void *dgamma, void *dbeta, int dw_fp32, float *part, cudaStream_t s)
{
    int sms = 0;
    cudaError_t e = device_sms(sms);
    if (e != cudaSuccess) return e;
    const bool sums = dgamma != nullptr || dbeta != nullptr;
    const int t = (C + 32 * LN_BWD_COLS - 1) / (32 * LN_BWD_COLS) * 32;
    int parts;
    if (t <= LN_BWD_THREADS) {
        const int groups = LN_BWD_THREADS / t;
        const int64_t need = (rows + groups - 1) / groups;
        parts = (int)(need < sms ? (need > 0 ? need : 1) : sms);
        const size_t smem = LnBwd<T>::smem(C, t, groups);        // at most 225280 bytes: several groups only up to C = 5120
        const auto kern = C == t * LN_BWD_COLS ? k_layernorm_bwd<T, true> : k_layernorm_bwd<T, false>;   // every thread owns its columns
        e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, 225280);
        if (e != cudaSuccess) return e;
        e = launch_smem(kern, dim3(parts), dim3(t, groups), smem, s, dy, x, gamma, mean, rstd, rows, C, dx,
                        sums ? part : nullptr);
        if (e != cudaSuccess) return e;
    } else {
        parts = DG_CHUNKS;
        if (sums) {
            e = launch_pdl(k_layernorm_bwd_cols<T>, dim3((C + LN_COLS - 1) / LN_COLS, parts), dim3(LN_COLS * LN_LANES), s, dy, x, mean,
                           rstd, rows, C, part);
            if (e != cudaSuccess) return e;
        }
        if (rows > 0) {
            e = launch_pdl(k_layernorm_bwd_rows<T>, dim3((unsigned)rows), dim3(LN_LONG_THREADS), s, dy, x, gamma, mean, rstd, C, dx);
            if (e != cudaSuccess) return e;
        }
    }
    if (!sums) return cudaSuccess;
    const dim3 grid((C + SUM_COLS - 1) / SUM_COLS, 2), block(SUM_COLS * 32);
    return dw_fp32 ? launch_pdl(k_layernorm_sum_parts<float>, grid, block, s, part, parts, C, (float *)dgamma, (float *)dbeta)
                   : launch_pdl(k_layernorm_sum_parts<T>, grid, block, s, part, parts, C, (T *)dgamma, (T *)dbeta);
}

}  // namespace

cudaError_t launch_layernorm_forward(const void *x, const void *gamma, const void *beta, int64_t rows, int C, int dtype, float eps,
                                     void *y, float *mean, float *rstd, cudaStream_t s)
{
    if (rows <= 0) return cudaSuccess;
    return dtype == SKIPFFN_BF16 ? fwd_t((const bf16 *)x, (const bf16 *)gamma, (const bf16 *)beta, rows, C, eps, (bf16 *)y, mean, rstd, s)
                                 : fwd_t((const float *)x, (const float *)gamma, (const float *)beta, rows, C, eps, (float *)y, mean, rstd, s);
}

cudaError_t launch_layernorm_backward(const void *dy, const void *x, const void *gamma, const float *mean, const float *rstd,
                                      int64_t rows, int C, int dtype, void *dx, void *dgamma, void *dbeta, int dw_fp32, float *part,
                                      cudaStream_t s)
{
    return dtype == SKIPFFN_BF16
               ? bwd_t<bf16>((const bf16 *)dy, (const bf16 *)x, (const bf16 *)gamma, mean, rstd, rows, C, (bf16 *)dx, dgamma, dbeta, dw_fp32, part, s)
               : bwd_t<float>((const float *)dy, (const float *)x, (const float *)gamma, mean, rstd, rows, C, (float *)dx, dgamma, dbeta, 1, part, s);
}

}  // namespace skipffn
