// Packed attention with plain fused multiply-adds (fp32, and bf16 as an on-device second opinion), and
// the row statistics of the backward pass of both paths.  64 x 64 tiles in shared memory, 4 x 4 products per thread;
// the same row tiles as the tensor-core kernels (the heads of a group are rows), half as high.  Measured in fp32:
// backward of sequences of 33, 1 and 200 tokens, 8 / 2 heads, d = 64: 85 us a call (271 us with a CTA per tile instead of a
// cluster); bound by the latency of a tile's steps.
#include <cooperative_groups.h>

#include "attention.cuh"

namespace skipffn {

namespace cg = cooperative_groups;

namespace {

constexpr int SR = AT_SIMT_ROWS, SK = AT_SIMT_KEYS;
constexpr int ST_THREADS = 256;
constexpr int PITCH = AT_MAX_D + 4, PPITCH = SK + 4;     // shared-memory row pitches (floats): no bank conflicts
constexpr float LOG2E = 1.4426950408889634f;

// Thread (ty, tx) of the 16 x 16 grid owns rows 4 ty .. 4 ty + 3 and columns tx + 16 j of a 64 x 64 product,
// and rows 4 ty .. +3, columns 4 tx .. +3 and 64 + 4 tx .. +3 of a 64 x d accumulator.
struct Tile { int ty, tx; };
__device__ __forceinline__ Tile tile_of() { return {(int)threadIdx.x / 16, (int)threadIdx.x % 16}; }

struct Item { int start, len, t0, base, h; };
__device__ __forceinline__ Item item_of(const int4 *items, int hk, int block)
{
    const int4 e = items[block / hk];
    return {e.x, e.y, e.z, e.w, block % hk};
}

// 64 rows of a [tokens, heads, d] array as fp32: tile row r is token `token` + r / group, head h group + r % group;
// rows at or past `valid` read as zeros
template <typename T>
__device__ __forceinline__ void load_rows(float *dst, const T *src, int64_t ld, int64_t token, int head0, int group, int valid, int d)
{
    for (int i = threadIdx.x; i < SR * (AT_MAX_D / 4); i += ST_THREADS) {
        const int r = i / (AT_MAX_D / 4), c = 4 * (i % (AT_MAX_D / 4));
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (r < valid && c < d) load4(src + (token + r / group) * ld + (int64_t)(head0 + r % group) * d + c, v);
        store4(dst + r * PITCH + c, v);
    }
}
// s[i][j] = sum_d a[4 ty + i][d] b[tx + 16 j][d]
__device__ __forceinline__ void rows_rows(float (&s)[4][4], const float *a, const float *b, int d, Tile t)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] = 0.0f;
    for (int c = 0; c < d; c += 4) {
        float x[4][4], y[4][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { load4(a + (4 * t.ty + i) * PITCH + c, x[i]); load4(b + (t.tx + 16 * i) * PITCH + c, y[i]); }
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[i][j] = fmaf(x[i][e], y[j][e], s[i][j]);
    }
}
// acc[4 rows][4 NC columns] += w(row, k) b[k][columns], k < n; TR: w is stored [k][row], else [row][k].
// NC = 1 serves heads of up to 64 columns, 2 up to 128.
template <bool TR, int NC>
__device__ __forceinline__ void weights_rows(float (&acc)[4][4 * NC], const float *w, const float *b, int n, Tile t)
{
#pragma unroll 2
    for (int k = 0; k < n; ++k) {
        float x[4], y[NC][4];
        if (TR) load4(w + k * PPITCH + 4 * t.ty, x);
        else
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = w[(4 * t.ty + i) * PPITCH + k];
#pragma unroll
        for (int c = 0; c < NC; ++c) load4(b + k * PITCH + 64 * c + 4 * t.tx, y[c]);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 4 * NC; ++j) acc[i][j] = fmaf(x[i], y[j / 4][j % 4], acc[i][j]);
    }
}
template <typename T, int NC>
__device__ __forceinline__ void store_acc(T *row, const float (&v)[4 * NC], float f, int d, Tile t)
{
#pragma unroll
    for (int j = 0; j < NC; ++j)
        if (64 * j + 4 * t.tx < d) {
            const float o[4] = {v[4 * j] * f, v[4 * j + 1] * f, v[4 * j + 2] * f, v[4 * j + 3] * f};
            store4(row + 64 * j + 4 * t.tx, o);
        }
}
// The CTAs of a cluster share one item, each with every size-th step of its sum; this adds the accumulators of all
// ranks, in order, into every rank's own (through `buf`, 64 rows of shared memory per CTA that nothing else uses now).
template <int NC>
__device__ __forceinline__ void cluster_add(cg::cluster_group cl, float (&acc)[4][4 * NC], float *buf, Tile t)
{
    const int size = (int)cl.num_blocks();
    if (size == 1) return;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < NC; ++j) {
            const float o[4] = {acc[i][4 * j], acc[i][4 * j + 1], acc[i][4 * j + 2], acc[i][4 * j + 3]};
            store4(buf + (4 * t.ty + i) * PITCH + 64 * j + 4 * t.tx, o);
        }
    cl.sync();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4 * NC; ++j) acc[i][j] = 0.0f;
    for (int r = 0; r < size; ++r) {
        const float *src = cl.map_shared_rank(buf, r);
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < NC; ++j) {
                float v[4];
                load4(src + (4 * t.ty + i) * PITCH + 64 * j + 4 * t.tx, v);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][4 * j + e] += v[e];
            }
    }
    cl.sync();                               // nobody overwrites or leaves with a buffer that is still read
}
__device__ __forceinline__ float half_warp_max(float v)
{
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float half_warp_sum(float v)
{
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

template <typename T, int NC>
__global__ void __launch_bounds__(ST_THREADS)
k_attention_fwd_simt(const AttnArgs a)
{
    extern __shared__ float sm[];
    float *qs = sm, *kv = qs + SR * PITCH, *ps = kv + SK * PITCH;
    const Tile t = tile_of();
    const Item it = item_of(a.fwd_items, a.hk, blockIdx.x);
    const int valid = min(a.tokens, it.len - it.t0) * a.group;
    const int end = a.causal ? min(it.t0 + a.tokens, it.len) : it.len;
    load_rows(qs, (const T *)a.q, a.ldq, (int64_t)it.start + it.t0, it.h * a.group, a.group, valid, a.d);
    float m[4], l[4] = {0.0f, 0.0f, 0.0f, 0.0f}, acc[4][4 * NC] = {};
    int row_end[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = -INFINITY;
        row_end[i] = a.causal ? min(it.t0 + (4 * t.ty + i) / a.group + 1, it.len) : it.len;
    }
    for (int k0 = 0; k0 < end; k0 += SK) {
        __syncthreads();
        load_rows(kv, (const T *)a.k, a.ldk, (int64_t)it.start + k0, it.h, 1, min(SK, it.len - k0), a.d);
        __syncthreads();
        float s[4][4];
        rows_rows(s, qs, kv, a.d, t);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float bm = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[i][j] = k0 + t.tx + 16 * j < row_end[i] ? s[i][j] * a.scale : -INFINITY;
                bm = fmaxf(bm, s[i][j]);
            }
            // base: the maximum, or zero while a row has met nothing but minus infinity (its P and sum are zero then)
            const float mn = fmaxf(m[i], half_warp_max(bm)), base = mn == -INFINITY ? 0.0f : mn, f = expf(m[i] - base);
            float sum = 0.0f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float p = expf(s[i][j] - base);
                sum += p;
                ps[(4 * t.ty + i) * PPITCH + t.tx + 16 * j] = p;
            }
            l[i] = l[i] * f + half_warp_sum(sum);
            m[i] = mn;
#pragma unroll
            for (int j = 0; j < 4 * NC; ++j) acc[i][j] *= f;
        }
        __syncthreads();
        load_rows(kv, (const T *)a.v, a.ldv, (int64_t)it.start + k0, it.h, 1, min(SK, it.len - k0), a.d);
        __syncthreads();
        weights_rows<false, NC>(acc, ps, kv, min(SK, end - k0), t);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 4 * t.ty + i;
        if (r >= valid) continue;
        const int64_t tok = (int64_t)it.start + it.t0 + r / a.group;
        const int head = it.h * a.group + r % a.group;
        store_acc<T, NC>((T *)a.out + tok * a.ldo + (int64_t)head * a.d, acc[i], 1.0f / l[i], a.d, t);
        if (t.tx == 0) a.lse[tok * a.hq + head] = m[i] + logf(l[i]);
    }
}

// P and dS of one 64 x 64 tile into shared memory (rows = queries, columns = keys).  Where a row's keys are this one
// tile its delta is summed here, without the rounding of a bf16 `out`; that of a row that sees one key is this key's dP:
// its dS is zero (NaN where dP is not finite), not what two orders of summation differ by.
__device__ __forceinline__ void grad_tile(float *ps, float *ds, const float *qs, const float *gs, const float *ks, const float *vs,
                                          const float2 *stats, const AttnArgs &a, int t0, int len, int k0, Tile t)
{
    float s[4][4], dp[4][4];
    rows_rows(s, qs, ks, a.d, t);
    rows_rows(dp, gs, vs, a.d, t);
    const float c2 = a.scale * LOG2E;
    const bool whole = (a.causal ? min(t0 + a.tokens, len) : len) <= SK;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 4 * t.ty + i, row_end = a.causal ? min(t0 + r / a.group + 1, len) : len;
        const float2 st = stats[r];
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const bool on = k0 + t.tx + 16 * j < row_end;
            s[i][j] = on ? exp2f(fmaf(s[i][j], c2, -st.x)) : 0.0f;
            if (!on) dp[i][j] = 0.0f;
            sum = fmaf(s[i][j], dp[i][j], sum);
        }
        const float delta = whole ? half_warp_sum(sum) : st.y;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = t.tx + 16 * j;
            ps[r * PPITCH + c] = s[i][j];
            ds[r * PPITCH + c] = k0 + c < row_end ? s[i][j] * (dp[i][j] - (row_end == 1 ? dp[i][j] : delta)) : 0.0f;
        }
    }
}

// dK, dV of 64 keys by a cluster (see cluster_add): with one CTA per key tile a few short sequences would keep most
// of the GPU idle.
template <typename T, int NC>
__global__ void __launch_bounds__(ST_THREADS)
k_attention_bwd_kv_simt(const AttnArgs a)
{
    extern __shared__ float sm[];
    float *ks = sm, *vs = ks + SK * PITCH, *qs = vs + SK * PITCH, *gs = qs + SR * PITCH, *ps = gs + SR * PITCH, *ds = ps + SR * PPITCH;
    const Tile t = tile_of();
    cg::cluster_group cl = cg::this_cluster();
    const int rank = (int)cl.block_rank(), size = (int)cl.num_blocks();
    const Item it = item_of(a.key_items, a.hk, blockIdx.x / size);
    const int k0 = it.t0, keys = min(SK, it.len - k0);
    load_rows(ks, (const T *)a.k, a.ldk, (int64_t)it.start + k0, it.h, 1, keys, a.d);
    load_rows(vs, (const T *)a.v, a.ldv, (int64_t)it.start + k0, it.h, 1, keys, a.d);
    float dk[4][4 * NC] = {}, dv[4][4 * NC] = {};
    for (int tile = (a.causal ? k0 / a.tokens : 0) + rank; tile * a.tokens < it.len; tile += size) {
        const int t0 = tile * a.tokens, valid = min(a.tokens, it.len - t0) * a.group;
        __syncthreads();
        load_rows(qs, (const T *)a.q, a.ldq, (int64_t)it.start + t0, it.h * a.group, a.group, valid, a.d);
        load_rows(gs, (const T *)a.dout, a.lddo, (int64_t)it.start + t0, it.h * a.group, a.group, valid, a.d);
        __syncthreads();
        grad_tile(ps, ds, qs, gs, ks, vs, a.row_stats + ((int64_t)(it.base + tile) * a.hk + it.h) * SR, a, t0, it.len, k0, t);
        __syncthreads();
        weights_rows<true, NC>(dv, ps, gs, valid, t);
        weights_rows<true, NC>(dk, ds, qs, valid, t);
    }
    cluster_add<NC>(cl, dv, gs, t);
    cluster_add<NC>(cl, dk, qs, t);
    if (rank != 0) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int key = 4 * t.ty + i;
        if (key >= keys) continue;
        const int64_t tok = (int64_t)it.start + k0 + key;
        store_acc<T, NC>((T *)a.dk + tok * a.lddk + (int64_t)it.h * a.d, dk[i], a.scale, a.d, t);
        store_acc<T, NC>((T *)a.dv + tok * a.lddv + (int64_t)it.h * a.d, dv[i], 1.0f, a.d, t);
    }
}

template <typename T, int NC>
__global__ void __launch_bounds__(ST_THREADS)
k_attention_bwd_q_simt(const AttnArgs a)
{
    extern __shared__ float sm[];
    float *ks = sm, *vs = ks + SK * PITCH, *qs = vs + SK * PITCH, *gs = qs + SR * PITCH, *ps = gs + SR * PITCH, *ds = ps + SR * PPITCH;
    const Tile t = tile_of();
    cg::cluster_group cl = cg::this_cluster();
    const int rank = (int)cl.block_rank(), size = (int)cl.num_blocks();
    const Item it = item_of(a.row_items, a.hk, blockIdx.x / size);
    const int valid = min(a.tokens, it.len - it.t0) * a.group, end = a.causal ? min(it.t0 + a.tokens, it.len) : it.len;
    load_rows(qs, (const T *)a.q, a.ldq, (int64_t)it.start + it.t0, it.h * a.group, a.group, valid, a.d);
    load_rows(gs, (const T *)a.dout, a.lddo, (int64_t)it.start + it.t0, it.h * a.group, a.group, valid, a.d);
    const float2 *stats = a.row_stats + ((int64_t)(it.base + it.t0 / a.tokens) * a.hk + it.h) * SR;
    float dq[4][4 * NC] = {};
    for (int k0 = rank * SK; k0 < end; k0 += size * SK) {
        const int keys = min(SK, it.len - k0);
        __syncthreads();
        load_rows(ks, (const T *)a.k, a.ldk, (int64_t)it.start + k0, it.h, 1, keys, a.d);
        load_rows(vs, (const T *)a.v, a.ldv, (int64_t)it.start + k0, it.h, 1, keys, a.d);
        __syncthreads();
        grad_tile(ps, ds, qs, gs, ks, vs, stats, a, it.t0, it.len, k0, t);
        __syncthreads();
        weights_rows<false, NC>(dq, ds, ks, keys, t);
    }
    cluster_add<NC>(cl, dq, ks, t);
    if (rank != 0) return;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 4 * t.ty + i;
        if (r >= valid) continue;
        const int64_t tok = (int64_t)it.start + it.t0 + r / a.group;
        store_acc<T, NC>((T *)a.dq + tok * a.lddq + (int64_t)(it.h * a.group + r % a.group) * a.d, dq[i], a.scale, a.d, t);
    }
}

// (lse log2 e, delta = sum_d dout out) of every row of a row tile; rows that belong to no token get (infinity, 0),
// which makes their P and dS zero.  Reads out and dout once: HBM-bound.  A row of at most 128 columns is 16 (bf16)
// or 32 (fp32) lanes x 16 bytes; the loads of four rows of a lane are in flight at a time, with few enough registers
// for five CTAs on an SM.
template <typename T, int ROWS>
__global__ void __launch_bounds__(ST_THREADS, 5)
k_attention_row_stats(const AttnArgs a)
{
    constexpr int LANES = 128 * (int)sizeof(T) / 16, EL = 16 / (int)sizeof(T), STEP = ST_THREADS / LANES, N = ROWS / STEP;
    constexpr int BATCH = N < 4 ? N : 4;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const Item it = item_of(a.row_items, a.hk, blockIdx.x);
    const int valid = min(a.tokens, it.len - it.t0) * a.group;
    float2 *dst = a.row_stats + ((int64_t)(it.base + it.t0 / a.tokens) * a.hk + it.h) * ROWS;
    const int first = threadIdx.x / LANES, lane = threadIdx.x % LANES;
    const bool even = STEP % a.group == 0;       // a lane's rows then belong to one head, STEP / group tokens apart
    const int t_first = first / a.group, h_first = first - t_first * a.group, t_step = STEP / a.group;
#pragma unroll 1
    for (int k0 = 0; k0 < N; k0 += BATCH) {
        uint4 x[BATCH], y[BATCH];
        float l[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int r = first + (k0 + k) * STEP;
            const int t = even ? t_first + (k0 + k) * t_step : r / a.group, h = even ? h_first : r - t * a.group;
            x[k] = y[k] = make_uint4(0, 0, 0, 0);
            l[k] = 0.0f;
            if (r < valid && EL * lane < a.d) {
                const int64_t tok = (int64_t)it.start + it.t0 + t;
                const int head = it.h * a.group + h;
                x[k] = __ldcs(reinterpret_cast<const uint4 *>((const T *)a.out_in + tok * a.ldo + (int64_t)head * a.d + EL * lane));
                y[k] = __ldg(reinterpret_cast<const uint4 *>((const T *)a.dout + tok * a.lddo + (int64_t)head * a.d + EL * lane));
                if (lane == 0) l[k] = a.lse[tok * a.hq + head];
            }
        }
#pragma unroll
        for (int k = 0; k < BATCH; ++k) {
            const int r = first + (k0 + k) * STEP;
            float dot = 0.0f;
#pragma unroll
            for (int h = 0; h < EL / 4; ++h) {
                float u[4], v[4];
                load4(reinterpret_cast<const T *>(&x[k]) + 4 * h, u);
                load4(reinterpret_cast<const T *>(&y[k]) + 4 * h, v);
#pragma unroll
                for (int e = 0; e < 4; ++e) dot = fmaf(u[e], v[e], dot);
            }
#pragma unroll
            for (int o = LANES / 2; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
            if (lane == 0) dst[r] = r < valid ? make_float2(l[k] * LOG2E, dot) : make_float2(INFINITY, 0.0f);
        }
    }
}

constexpr int FWD_SMEM = (SR * PITCH + SK * PITCH + SR * PPITCH) * 4;
constexpr int BWD_SMEM = (2 * SR * PITCH + 2 * SK * PITCH + 2 * SR * PPITCH) * 4;

// n items, each by a cluster of 1, 2, 4 or 8 CTAs: as many as keep the grid within two waves of 148, and no more than
// the longest item has steps
template <typename Kernel>
static cudaError_t launch(Kernel kern, int n, int steps, int smem, const AttnArgs &a, cudaStream_t s)
{
    if (n <= 0) return cudaSuccess;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    int size = 1;
    while (size < 8 && 2 * size <= steps && (int64_t)n * 2 * size <= 296) size *= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)n * size); cfg.blockDim = dim3(ST_THREADS); cfg.dynamicSmemBytes = smem; cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = size; at[0].val.clusterDim.y = 1; at[0].val.clusterDim.z = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, a);
}

}  // namespace

template <typename T> static cudaError_t forward_t(const AttnArgs &a, cudaStream_t s)
{
    return a.d <= 64 ? launch(k_attention_fwd_simt<T, 1>, a.n_fwd * a.hk, 1, FWD_SMEM, a, s)
                     : launch(k_attention_fwd_simt<T, 2>, a.n_fwd * a.hk, 1, FWD_SMEM, a, s);
}
cudaError_t launch_attention_simt_forward(const AttnArgs &a, int dtype, cudaStream_t s)
{
    return dtype == SKIPFFN_BF16 ? forward_t<bf16>(a, s) : forward_t<float>(a, s);
}

template <typename T, int ROWS> static cudaError_t row_stats(const AttnArgs &a, cudaStream_t s)
{
    const int n = a.n_rows * a.hk;
    return n <= 0 ? cudaSuccess : launch_pdl(k_attention_row_stats<T, ROWS>, dim3((unsigned)n), dim3(ST_THREADS), s, a);
}
cudaError_t launch_attention_row_stats_tc(const AttnArgs &a, cudaStream_t s) { return row_stats<bf16, AT_TC_ROWS>(a, s); }

template <typename T> static cudaError_t backward_t(const AttnArgs &a, cudaStream_t s)
{
    cudaError_t e = row_stats<T, SR>(a, s);
    if (e != cudaSuccess) return e;
    const int row_steps = (a.max_len + a.tokens - 1) / a.tokens, key_steps = (a.max_len + SK - 1) / SK;
    e = a.d <= 64 ? launch(k_attention_bwd_kv_simt<T, 1>, a.n_keys * a.hk, row_steps, BWD_SMEM, a, s)
                  : launch(k_attention_bwd_kv_simt<T, 2>, a.n_keys * a.hk, row_steps, BWD_SMEM, a, s);
    if (e != cudaSuccess) return e;
    return a.d <= 64 ? launch(k_attention_bwd_q_simt<T, 1>, a.n_rows * a.hk, key_steps, BWD_SMEM, a, s)
                     : launch(k_attention_bwd_q_simt<T, 2>, a.n_rows * a.hk, key_steps, BWD_SMEM, a, s);
}
cudaError_t launch_attention_simt_backward(const AttnArgs &a, int dtype, cudaStream_t s)
{
    return dtype == SKIPFFN_BF16 ? backward_t<bf16>(a, s) : backward_t<float>(a, s);
}

}  // namespace skipffn
