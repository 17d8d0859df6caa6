// Attention over a paged cache and the weights of its rows with plain FMA: fp32, and a second opinion for bf16.
// One CTA of 128 threads walks its run of units (16 rows x 32 keys): a tile's rows are 16 groups of 8 threads, a thread
// has 4 keys of a row's scores and up to 16 columns of its sum.  Statistics and sums are fp32, in a fixed order.
#include "paged.cuh"

namespace skipffn {

namespace {

constexpr int ROWS = PG_SIMT_ROWS, KEYS = PG_SIMT_KEYS, THREADS = 128, PITCH = PG_MAX_D + 4;
constexpr float LOG2E = 1.4426950408889634f;

__device__ __forceinline__ float group8_max(float v)
{
    for (int o = 4; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float group8_sum(float v)
{
    for (int o = 4; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// rows j0 .. j0 + KEYS - 1 of head h of sequence s; rows at or past `end`, and rows of pages that do not exist, as zeros
template <typename T> __device__ void load_keys(float (*dst)[PITCH], const PagedView &c, const char *base, int s, int h, int j0, int end)
{
    const int r = threadIdx.x >> 2;          // 32 rows x 4 threads
    int64_t at = -1;
    if (j0 + r < end) {
        at = paged_row(c, s, j0 + r);
        if (at < 0) paged_report(c, SITE_PAGED_PAGE);
    }
    const T *src = at < 0 ? nullptr : (const T *)(base + at + h * c.head_stride);
    for (int e = 4 * (threadIdx.x & 3); e < c.d; e += 16) {
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (src) load4(src + e, v);
        store4(&dst[r][e], v);
    }
}

template <typename T> __global__ void __launch_bounds__(THREADS) k_paged_simt(const PagedAttnArgs a)
{
    __shared__ float qs[ROWS][PITCH], ks[KEYS][PITCH], vs[KEYS][PITCH], ps[ROWS][KEYS + 1];
    pdl_enter();
    const PagedView &c = a.c;
    const int tiles = a.head[0], run = blockIdx.x;
    const Runs runs(*(const int64_t *)(a.head + 2), a.runs);
    const int64_t begin = runs.begin(run), end = runs.begin(run + 1);
    if (threadIdx.x == 0) a.cuts[run].pieces = 0;
    if (begin >= end) return;
    int t = 0;
    for (int hi = tiles; hi - t > 1;) {      // largest tile with u0 <= begin
        const int mid = (t + hi) >> 1;
        if (a.tiles[mid].u0 <= begin) t = mid; else hi = mid;
    }
    const int row = threadIdx.x >> 3, part = threadIdx.x & 7;
    const float c2 = a.scale * LOG2E;
    for (int64_t u = begin; u < end; ++t) {
        const PagedTile e = a.tiles[t];
        if (e.blocks == 0) continue;
        const int live = min(ROWS, e.n * a.group - e.r0);
        const int seg = e.blocks + PG_TILE_COST;
        for (int h = (int)((u - e.u0) / seg); h < c.heads && u < end; ++h) {
            const int64_t first = e.u0 + (int64_t)h * seg + PG_TILE_COST, last = first + e.blocks;   // units of the blocks
            const int b0 = (int)max((int64_t)0, u - first), b1 = (int)(min(end, last) - first);
            u = min(end, last);
            if (b1 <= b0) continue;          // the run ends before the tile's first block
            const int r = e.r0 + row, limit = row < live ? e.len - e.n + r / a.group + 1 : 0;
            __syncthreads();
            for (int i = threadIdx.x; i < ROWS * (c.d / 4); i += THREADS) {
                const int qr = i / (c.d / 4), col = 4 * (i - qr * (c.d / 4));
                float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if (qr < live) {
                    const int64_t token = e.q0 + (e.r0 + qr) / a.group;
                    load4((const T *)a.q + token * a.ldq + (int64_t)(h * a.group + (e.r0 + qr) % a.group) * c.d + col, v);
                }
                store4(&qs[qr][col], v);
            }
            float m = -INFINITY, l = 0.0f, acc[4][4] = {};
            for (int b = b0; b < b1; ++b) {
                const int j0 = b * KEYS;
                __syncthreads();
                load_keys<T>(ks, c, c.k, e.s, h, j0, e.len);
                load_keys<T>(vs, c, c.v, e.s, h, j0, e.len);
                __syncthreads();
                float s[4] = {};
                for (int x = 0; x < c.d; x += 4) {
                    float q[4];
                    load4(&qs[row][x], q);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float k[4];
                        load4(&ks[part + 8 * i][x], k);
#pragma unroll
                        for (int y = 0; y < 4; ++y) s[i] = fmaf(q[y], k[y], s[i]);
                    }
                }
                float top = -INFINITY;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    if (j0 + part + 8 * i >= limit) s[i] = -INFINITY;
                    top = fmaxf(top, s[i]);
                }
                top = fmaxf(m, group8_max(top));
                const float f = top == m ? 1.0f : exp2f((m - top) * c2);
                m = top;
                l *= f;
                float sum = 0.0f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float p = s[i] == -INFINITY ? 0.0f : exp2f((s[i] - m) * c2);
                    sum += p;
                    ps[row][part + 8 * i] = p;
                }
                l += group8_sum(sum);
                __syncwarp();                // a row's eight threads are in one warp
#pragma unroll
                for (int x = 0; x < 4; ++x)
#pragma unroll
                    for (int y = 0; y < 4; ++y) acc[x][y] *= f;
                // rows past this row's last key may hold anything inside the tile of a longer row: they do not enter
                const int n = min(KEYS, limit - j0);
                for (int j = 0; j < n; ++j) {
                    const float p = ps[row][j];
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int col = 4 * part + 32 * x;
                        if (col < c.d) {
                            float v[4];
                            load4(&vs[j][col], v);
#pragma unroll
                            for (int y = 0; y < 4; ++y) acc[x][y] = fmaf(p, v[y], acc[x][y]);
                        }
                    }
                }
                __syncwarp();
            }
            if (row < live) {
                if (b0 == 0 && b1 == e.blocks) {
                    const int64_t token = e.q0 + r / a.group;
                    const int head = h * a.group + r % a.group;
                    const float inv = m == -INFINITY ? 0.0f : 1.0f / l;
#pragma unroll
                    for (int x = 0; x < 4; ++x) {
                        const int col = 4 * part + 32 * x;
                        if (col < c.d) {
                            float v[4];
#pragma unroll
                            for (int y = 0; y < 4; ++y) v[y] = m == -INFINITY ? 0.0f : acc[x][y] * inv;
                            store4((T *)a.out + token * a.ldo + (int64_t)head * c.d + col, v);
                        }
                    }
                    if (part == 0) a.lse[token * a.hq + head] = m == -INFINITY ? -INFINITY : fmaf(m, a.scale, logf(l));
                } else {
                    const int64_t at = (int64_t)(2 * run + (b0 == 0 ? 1 : 0)) * ROWS + row;
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        if (4 * part + 32 * x < c.d) store4(a.part + at * PG_MAX_D + 4 * part + 32 * x, acc[x]);
                    if (part == 0) a.part_ml[at] = make_float2(m, l);
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
template <typename T> __global__ void __launch_bounds__(THREADS) k_paged_weights_simt(const PagedWeightsArgs a)
{
    __shared__ float qs[ROWS][PITCH], ks[KEYS][PITCH], lses[ROWS];
    pdl_enter();
    const PagedView &c = a.c;
    const int s = blockIdx.z, h = blockIdx.y, j0 = blockIdx.x * KEYS;
    const PagedSeq q = paged_seq(c, s, blockIdx.x == 0 && h == 0 && threadIdx.x == 0);
    if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0 && q.len > a.width) paged_report(c, SITE_PAGED_WIDTH);
    const int key = threadIdx.x >> 2, part = threadIdx.x & 3;    // four threads a key: every fourth row each
    const int rows = q.n * a.group, off = q.len - q.n;
    float total = 0.0f;
    if (j0 < q.len && rows > 0) {
        load_keys<T>(ks, c, c.k, s, h, j0, q.len);
        // the first row that sees any of these keys
        const int first = max(0, j0 - off) * a.group / ROWS * ROWS;
        for (int r0 = first; r0 < rows; r0 += ROWS) {
            __syncthreads();
            for (int i = threadIdx.x; i < ROWS * (c.d / 4); i += THREADS) {
                const int qr = i / (c.d / 4), col = 4 * (i - qr * (c.d / 4));
                float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if (r0 + qr < rows) {
                    const int64_t token = q.q0 + (r0 + qr) / a.group;
                    load4((const T *)a.q + token * a.ldq + (int64_t)(h * a.group + (r0 + qr) % a.group) * c.d + col, v);
                }
                store4(&qs[qr][col], v);
            }
            if (threadIdx.x < ROWS) {
                const int r = r0 + threadIdx.x;
                lses[threadIdx.x] = r < rows ? a.lse[(int64_t)(q.q0 + r / a.group) * a.hq + h * a.group + r % a.group] : -INFINITY;
            }
            __syncthreads();
            for (int i = part; i < ROWS; i += 4) {
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

}  // namespace

cudaError_t launch_paged_simt(const PagedAttnArgs &args, cudaStream_t s)
{
    PagedAttnArgs a = args;
    a.runs = PG_SIMT_RUNS;
    cudaError_t e = launch_paged_list(a, ROWS, KEYS, s);
    if (e != cudaSuccess) return e;
    e = a.dtype == SKIPFFN_BF16 ? launch_pdl(k_paged_simt<bf16>, dim3(a.runs), dim3(THREADS), s, a)
                                : launch_pdl(k_paged_simt<float>, dim3(a.runs), dim3(THREADS), s, a);
    return e != cudaSuccess ? e : launch_paged_join(a, ROWS, PG_MAX_D, s);
}

cudaError_t launch_paged_weights_simt(const PagedWeightsArgs &a, cudaStream_t s)
{
    const dim3 grid((unsigned)((a.width + KEYS - 1) / KEYS), (unsigned)a.c.heads, (unsigned)a.c.n_seq);
    return a.dtype == SKIPFFN_BF16 ? launch_pdl(k_paged_weights_simt<bf16>, grid, dim3(THREADS), s, a)
                                   : launch_pdl(k_paged_weights_simt<float>, grid, dim3(THREADS), s, a);
}

}  // namespace skipffn
