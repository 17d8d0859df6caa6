// Attention over a paged cache and the weights of its rows with plain FMA: fp32, and a second opinion for bf16.
// Statistics and sums are fp32, in a fixed order.  Measured in fp32, 32 / 8 heads, head_dim 128: a chunk of 1000 tokens
// behind 3000 cached ones 2.5 ms (23 TFLOP/s of 72 on the FMA pipes, bound by what shared memory delivers to them), 12
// rows each of 24 conversations 326 us (487 MB; fp32 sequences of up to 8 rows have the kernel of few rows, 118 us).
#include "paged.cuh"

namespace skipffn {

namespace {

constexpr int KEYS = PG_SIMT_KEYS, THREADS = 256, PITCH = PG_MAX_D + 4, P_PITCH = KEYS + 4;
constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ uint32_t shared_address(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }
// 4 elements to shared memory as fp32: copied behind the thread's back where they are fp32 already
__device__ __forceinline__ void bring4(float *dst, const float *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(shared_address(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void bring4(float *dst, const bf16 *src)
{
    float v[4];
    load4(src, v);
    store4(dst, v);
}
__device__ __forceinline__ void brought() { asm volatile("cp.async.wait_all;" ::: "memory"); }

// N rows from j0 on of head h of sequence s; rows at or past `end`, and rows of pages that do not exist, as zeros
template <typename T, int N, int CTA> __device__ __forceinline__ void bring_keys(float (*dst)[PITCH], const PagedView &c, const char *base, int s, int h, int j0, int end)
{
    constexpr int PER = CTA / N;             // threads of a row
    const int r = threadIdx.x / PER;
    int64_t at = -1;
    if (j0 + r < end) {
        at = paged_row(c, s, j0 + r);
        if (at < 0) paged_report(c, SITE_PAGED_PAGE);
    }
    const T *src = at < 0 ? nullptr : (const T *)(base + at + h * c.head_stride);
    for (int e = 4 * (threadIdx.x % PER); e < c.d; e += 4 * PER) {
        if (src) bring4(&dst[r][e], src + e);
        else store4(&dst[r][e], {0.0f, 0.0f, 0.0f, 0.0f});
    }
}

// One CTA walks its run of units, a tile of 16 R rows x 64 keys each.  Threads are 16 x 16: (ty, tx) has rows R ty .. of
// the scores and sums, keys tx, tx + 16, .. of the scores and columns 4 tx .. and 64 + 4 tx .. of the sums, so that what a
// warp reads of keys and values together is 256 bytes without bank conflicts and what it reads of queries and weights is
// shared by half of it: with R = 4, 8 (scores) and 12 (sums) vectors of shared memory for 64 and 128 multiply-adds.
// Values arrive while scores are made, the next keys while sums are.  R = 4 for chunks; R = 1, two CTAs an SM, where no
// sequence has more than 16 rows, so that the rows that are not there cost less than reading the cache.
template <int R> struct SimtShape {
    static constexpr int ROWS = 16 * R, SMEM = (ROWS + 2 * KEYS) * PITCH * 4 + ROWS * P_PITCH * 4;
};
template <typename T, int R> __global__ void __launch_bounds__(THREADS, R == 1 ? 2 : 1) k_paged_simt(const PagedAttnArgs a)
{
    constexpr int ROWS = SimtShape<R>::ROWS;
    extern __shared__ __align__(16) float smem[];
    float(*qs)[PITCH] = reinterpret_cast<float(*)[PITCH]>(smem), (*ks)[PITCH] = qs + ROWS, (*vs)[PITCH] = ks + KEYS;
    float(*ps)[P_PITCH] = reinterpret_cast<float(*)[P_PITCH]>(vs + KEYS);
    pdl_enter();
    const PagedView &c = a.c;
    const int run = blockIdx.x;
    const Runs runs(*a.head, a.runs);
    const int64_t begin = runs.begin(run), end = runs.begin(run + 1);
    if (threadIdx.x == 0) a.cuts[run].pieces = 0;
    if (begin >= end) return;
    int t = a.starts[run];
    const int ty = threadIdx.x >> 4, tx = threadIdx.x & 15;
    const float c2 = a.scale * LOG2E;
    for (int64_t u = begin; u < end; ++t) {
        const PagedTile e = a.tiles[t];
        if (e.blocks == 0) continue;
        const int live = min(ROWS, e.n * a.group - e.r0), seg = e.blocks + PG_TILE_COST;
        for (int h = (int)((u - e.u0) / seg); h < c.heads && u < end; ++h) {
            const int64_t first = e.u0 + (int64_t)h * seg + PG_TILE_COST, last = first + e.blocks;   // units of the blocks
            const int b0 = (int)max((int64_t)0, u - first), b1 = (int)(min(end, last) - first);
            u = min(end, last);
            if (b1 <= b0) continue;          // the run ends before the tile's first block
            int limit[R];
#pragma unroll
            for (int i = 0; i < R; ++i) limit[i] = R * ty + i < live ? e.len - e.n + (e.r0 + R * ty + i) / a.group + 1 : 0;
            __syncthreads();                 // the tile before has been read
            for (int i = threadIdx.x; i < ROWS * (c.d / 4); i += THREADS) {
                const int qr = i / (c.d / 4), col = 4 * (i - qr * (c.d / 4));
                float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if (qr < live) {
                    const int64_t token = e.q0 + (e.r0 + qr) / a.group;
                    load4((const T *)a.q + token * a.ldq + (int64_t)(h * a.group + (e.r0 + qr) % a.group) * c.d + col, v);
                }
                store4(&qs[qr][col], v);
            }
            bring_keys<T, KEYS, THREADS>(ks, c, c.k, e.s, h, b0 * KEYS, e.len);
            float m[R], l[R], acc[R][2][4] = {};
#pragma unroll
            for (int i = 0; i < R; ++i) { m[i] = -INFINITY; l[i] = 0.0f; }
            for (int b = b0; b < b1; ++b) {
                const int j0 = b * KEYS;
                brought();
                __syncthreads();             // keys are there, values of the block before have been read
                bring_keys<T, KEYS, THREADS>(vs, c, c.v, e.s, h, j0, e.len);
                // four sums a score, over every fourth column: shorter chains, less rounding
                float s[R][4][4] = {};
#pragma unroll 2
                for (int x = 0; x < c.d; x += 4) {
                    float q[R][4], k[4][4];
#pragma unroll
                    for (int i = 0; i < R; ++i) load4(&qs[R * ty + i][x], q[i]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) load4(&ks[tx + 16 * i][x], k[i]);
#pragma unroll
                    for (int i = 0; i < R; ++i)
#pragma unroll
                        for (int j = 0; j < 4; ++j)
#pragma unroll
                            for (int y = 0; y < 4; ++y) {
                                float &d = R == 1 ? s[i][j][y] : s[i][j][y & 1];
                                d = fmaf(q[i][y], k[j][y], d);
                            }
                }
#pragma unroll
                for (int i = 0; i < R; ++i) {
                    float z[4], top = -INFINITY;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        z[j] = (s[i][j][0] + s[i][j][1]) + (R == 1 ? s[i][j][2] + s[i][j][3] : 0.0f);
                        if (j0 + tx + 16 * j >= limit[i]) z[j] = -INFINITY;
                        top = fmaxf(top, z[j]);
                    }
#pragma unroll
                    for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                    top = fmaxf(m[i], top);
                    const float f = top == m[i] ? 1.0f : exp2f((m[i] - top) * c2);
                    m[i] = top;
                    float sum = 0.0f;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float p = z[j] == -INFINITY ? 0.0f : exp2f((z[j] - top) * c2);
                        sum += p;
                        ps[R * ty + i][tx + 16 * j] = p;
                    }
                    l[i] = l[i] * f + sum;   // of this thread's keys; the sixteen of a row add up at the end
#pragma unroll
                    for (int y = 0; y < 8; ++y) acc[i][y >> 2][y & 3] *= f;
                }
                brought();
                __syncthreads();             // weights and values are there, keys have been read
                if (b + 1 < b1) bring_keys<T, KEYS, THREADS>(ks, c, c.k, e.s, h, j0 + KEYS, e.len);
#pragma unroll 2
                for (int j = 0; j < KEYS; j += 4) {
                    float p[R][4];
#pragma unroll
                    for (int i = 0; i < R; ++i) load4(&ps[R * ty + i][j], p[i]);
#pragma unroll
                    for (int y = 0; y < 4; ++y)
#pragma unroll
                        for (int z = 0; z < 2; ++z) {
                            const int col = 64 * z + 4 * tx;
                            if (col < c.d) {
                                float v[4];
                                load4(&vs[j + y][col], v);
#pragma unroll
                                for (int i = 0; i < R; ++i)
#pragma unroll
                                    for (int w = 0; w < 4; ++w) acc[i][z][w] = fmaf(p[i][y], v[w], acc[i][z][w]);
                            }
                        }
                }
            }
#pragma unroll
            for (int i = 0; i < R; ++i) {
#pragma unroll
                for (int o = 8; o > 0; o >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], o);
                const int row = R * ty + i, r = e.r0 + row;
                if (row >= live) continue;
                if (b0 == 0 && b1 == e.blocks) {
                    const int64_t token = e.q0 + r / a.group;
                    const int head = h * a.group + r % a.group;
                    const float inv = 1.0f / l[i];
                    const bool none = met_nothing(m[i], l[i]);
#pragma unroll
                    for (int z = 0; z < 2; ++z) {
                        const int col = 64 * z + 4 * tx;
                        if (col < c.d) {
                            float v[4];
#pragma unroll
                            for (int w = 0; w < 4; ++w) v[w] = none ? 0.0f : acc[i][z][w] * inv;
                            store4((T *)a.out + token * a.ldo + (int64_t)head * c.d + col, v);
                        }
                    }
                    if (tx == 0) a.lse[token * a.hq + head] = none ? -INFINITY : fmaf(m[i], a.scale, logf(l[i]));
                } else {
                    const int64_t at = (int64_t)(2 * run + (b0 == 0 ? 1 : 0)) * ROWS + row;
#pragma unroll
                    for (int z = 0; z < 2; ++z)
                        if (64 * z + 4 * tx < c.d) store4(a.part + at * PG_MAX_D + 64 * z + 4 * tx, acc[i][z]);
                    if (tx == 0) a.part_ml[at] = make_float2(m[i], l[i]);
                }
            }
            if (b0 == 0 && b1 < e.blocks && threadIdx.x == 0) {
                PagedCut cut = {};
                cut.q0 = e.q0; cut.r0 = e.r0; cut.rows = live; cut.h = h; cut.first = run;
                cut.pieces = runs.of(last - 1) - run + 1;
                a.cuts[run] = cut;
            }
        }
    }
}

// One CTA: 32 keys of one head of one sequence against all its new rows, 16 at a time; four threads a key, each with
// every fourth row, whose sums are added in a fixed order.
constexpr int W_THREADS = 128, W_ROWS = 16, W_KEYS = 32;
template <typename T> __global__ void __launch_bounds__(W_THREADS) k_paged_weights_simt(const PagedWeightsArgs a)
{
    __shared__ __align__(16) float qs[W_ROWS][PITCH], ks[W_KEYS][PITCH], lses[W_ROWS];
    pdl_enter();
    const PagedView &c = a.c;
    const int s = blockIdx.z, h = blockIdx.y, j0 = blockIdx.x * W_KEYS;
    const PagedSeq q = paged_seq(c, s, blockIdx.x == 0 && h == 0 && threadIdx.x == 0);
    if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0 && q.len > a.width) paged_report(c, SITE_PAGED_WIDTH);
    const int key = threadIdx.x >> 2, part = threadIdx.x & 3;    // four threads a key: every fourth row each
    const int rows = q.n * a.group, off = q.len - q.n;
    float total = 0.0f;
    if (j0 < q.len && rows > 0) {
        bring_keys<T, W_KEYS, W_THREADS>(ks, c, c.k, s, h, j0, q.len);
        brought();
        // the first row that sees any of these keys
        const int first = max(0, j0 - off) * a.group / W_ROWS * W_ROWS;
        for (int r0 = first; r0 < rows; r0 += W_ROWS) {
            __syncthreads();
            for (int i = threadIdx.x; i < W_ROWS * (c.d / 4); i += W_THREADS) {
                const int qr = i / (c.d / 4), col = 4 * (i - qr * (c.d / 4));
                float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if (r0 + qr < rows) {
                    const int64_t token = q.q0 + (r0 + qr) / a.group;
                    load4((const T *)a.q + token * a.ldq + (int64_t)(h * a.group + (r0 + qr) % a.group) * c.d + col, v);
                }
                store4(&qs[qr][col], v);
            }
            if (threadIdx.x < W_ROWS) {
                const int r = r0 + threadIdx.x;
                lses[threadIdx.x] = r < rows ? a.lse[(int64_t)(q.q0 + r / a.group) * a.hq + h * a.group + r % a.group] : -INFINITY;
            }
            __syncthreads();
            for (int i = part; i < W_ROWS; i += 4) {
                const int r = r0 + i;
                if (r >= rows || j0 + key > off + r / a.group || lses[i] == -INFINITY) continue;
                float d = 0.0f;
                for (int x = 0; x < c.d; x += 4) {
                    float u[4], k[4];
                    load4(&qs[i][x], u);
                    load4(&ks[key][x], k);
#pragma unroll
                    for (int y = 0; y < 4; ++y) d = fmaf(u[y], k[y], d);
                }
                total += exp2f(fmaf(d, a.scale, -lses[i]) * LOG2E);
            }
        }
    }
    total += __shfl_xor_sync(0xffffffffu, total, 1);
    total += __shfl_xor_sync(0xffffffffu, total, 2);
    const int j = j0 + key;
    if (part == 0 && j < a.width) {
        const int64_t at = ((int64_t)s * c.heads + h) * a.width + j;
        a.out[at] = j < q.len ? (a.prior ? a.prior[at] : 0.0f) + total : 0.0f;
    }
}

template <typename T, int R> cudaError_t simt(PagedAttnArgs a, cudaStream_t s)
{
    using Sh = SimtShape<R>;
    static bool ready[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (!ready[dev]) {
        const cudaError_t e = cudaFuncSetAttribute(k_paged_simt<T, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::SMEM);
        if (e != cudaSuccess) return e;
        ready[dev] = true;
    }
    a.runs = R == 1 ? PG_SIMT_RUNS : PG_SIMT_RUNS / 2;
    cudaError_t e = launch_paged_list(a, Sh::ROWS, KEYS, s);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.runs); cfg.blockDim = dim3(THREADS); cfg.dynamicSmemBytes = Sh::SMEM; cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, k_paged_simt<T, R>, a);
    return e != cudaSuccess ? e : launch_paged_join(a, Sh::ROWS, PG_MAX_D, s);
}

}  // namespace

cudaError_t launch_paged_simt(const PagedAttnArgs &a, int rows, cudaStream_t s)
{
    if (a.dtype == SKIPFFN_BF16) return rows <= 16 ? simt<bf16, 1>(a, s) : simt<bf16, 4>(a, s);
    return rows <= 16 ? simt<float, 1>(a, s) : simt<float, 4>(a, s);
}

cudaError_t launch_paged_weights_simt(const PagedWeightsArgs &a, cudaStream_t s)
{
    const dim3 grid((unsigned)((a.width + W_KEYS - 1) / W_KEYS), (unsigned)a.c.heads, (unsigned)a.c.n_seq);
    return a.dtype == SKIPFFN_BF16 ? launch_pdl(k_paged_weights_simt<bf16>, grid, dim3(W_THREADS), s, a)
                                   : launch_pdl(k_paged_weights_simt<float>, grid, dim3(W_THREADS), s, a);
}

}  // namespace skipffn
