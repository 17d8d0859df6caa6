// C-ABI entry points of the paged cache: argument checks, scratch, launch sequencing; the kernel that lists the tiles of
// a call and the one that joins the pieces of tiles that were cut.
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "arrays.cuh"
#include "paged.cuh"

namespace skipffn {

namespace {

struct Level { int64_t n, stride; };

// (page, row, head) levels of the pool, the inner ones first; levels of one entry do not count
int levels_of(const PagedView &c, int64_t page_size, Level (&l)[3])
{
    const Level all[3] = {{c.heads, c.head_stride}, {page_size, c.row_stride}, {c.n_pages, c.page_stride}};
    int n = 0;
    for (const Level &x : all)
        if (x.n > 1) l[n++] = x;
    std::sort(l, l + n, [](const Level &a, const Level &b) { return a.stride < b.stride; });
    return n;
}

}  // namespace

skipffn_status paged_view(const skipffn_paged_cache *c, int64_t N, PagedView *v)
{
    *v = PagedView{};
    if (!c || c->heads_kv <= 0 || c->head_dim <= 0 || (c->dtype != SKIPFFN_BF16 && c->dtype != SKIPFFN_FP32) || c->page_size <= 0 ||
        c->n_pages < 0 || c->n_seq < 0 || c->table_width < 0 || c->max_new < 0 || N < 0 || N > INT_MAX - 4096 ||
        (c->path != SKIPFFN_PATH_DEFAULT && c->path != SKIPFFN_PATH_SIMT) || !c->status || !is_aligned(c->status, 4))
        return SKIPFFN_EINVAL;
    if (c->head_dim % 8 || c->head_dim > PG_MAX_D || c->page_size % 8 || c->page_size > (1 << 30) || c->n_pages > INT_MAX || c->heads_kv > 65535 ||
        c->n_seq > PG_MAX_COUNT)
        return SKIPFFN_EUNSUPPORTED;
    const int64_t es = c->dtype == SKIPFFN_BF16 ? 2 : 4;
    for (const int64_t ld : {c->page_stride, c->row_stride, c->head_stride})
        if (ld < 0 || ld > (int64_t)1 << 36 || ld * es % 16) return SKIPFFN_EINVAL;
    v->k = (char *)c->k_pages; v->v = (char *)c->v_pages;
    v->page_stride = c->page_stride * es; v->row_stride = c->row_stride * es; v->head_stride = c->head_stride * es;
    v->table = c->page_table; v->cu = c->cu_new; v->lens = c->lens;
    v->table_stride = c->table_stride; v->n_pages = c->n_pages;
    v->n_seq = c->n_seq; v->heads = c->heads_kv; v->d = c->head_dim;
    v->capacity = c->n_pages == 0 ? 0 : (int32_t)std::min<int64_t>((int64_t)c->table_width * c->page_size, INT_MAX - 4096);
    v->N = N; v->max_new = c->max_new;
    v->page = make_divisor((uint32_t)c->page_size);
    v->status = c->status;
    if (c->n_seq > 0 && (!c->cu_new || !c->lens || !is_aligned(c->cu_new, 4) || !is_aligned(c->lens, 4))) return SKIPFFN_EINVAL;
    if (c->n_seq > 0 && c->table_width > 0 &&
        (!c->page_table || !is_aligned(c->page_table, 4) || (c->n_seq > 1 && c->table_stride < c->table_width) || c->table_stride > (int64_t)1 << 40))
        return SKIPFFN_EINVAL;
    if (c->n_pages > 0) {
        if (!v->k || !v->v || !is_aligned(v->k, 16) || !is_aligned(v->v, 16)) return SKIPFFN_EINVAL;
        // no two rows of the pool share a byte, and the pool's extent stays within 62 bits
        Level l[3];
        const int n = levels_of(*v, c->page_size, l);
        int64_t extent = (int64_t)c->head_dim * es;
        for (int i = 0; i < n; ++i) {
            if (l[i].stride < extent || l[i].stride > ((int64_t)1 << 60) / l[i].n) return SKIPFFN_EINVAL;
            extent += (l[i].n - 1) * l[i].stride;
        }
        v->extent = extent;
        // keys and values: two pools, or interleaved at one of the levels
        const int64_t off = v->v > v->k ? v->v - v->k : v->k - v->v;
        bool apart = off >= extent;
        extent = (int64_t)c->head_dim * es;
        for (int i = 0; i < n && !apart; ++i) {
            bool multiples = true;
            for (int j = i; j < n; ++j) multiples = multiples && l[j].stride % l[i].stride == 0;
            const int64_t at = off % l[i].stride;
            apart = multiples && at >= extent && at + extent <= l[i].stride;
            extent += (l[i].n - 1) * l[i].stride;
        }
        if (!apart) return SKIPFFN_EINVAL;
    }
    return SKIPFFN_OK;
}

bool paged_overlap(const PagedView &c, const void *p, int64_t bytes)
{
    const int64_t table = c.n_seq > 0 && c.capacity > 0 ? ((c.n_seq - 1) * c.table_stride + (c.capacity + (int64_t)c.page.d - 1) / c.page.d) * 4 : 0;
    return ranges_overlap(p, bytes, c.k, c.extent) || ranges_overlap(p, bytes, c.v, c.extent) || ranges_overlap(p, bytes, c.table, table) ||
           ranges_overlap(p, bytes, c.cu, c.n_seq > 0 ? (int64_t)(c.n_seq + 1) * 4 : 0) || ranges_overlap(p, bytes, c.lens, (int64_t)c.n_seq * 4) ||
           ranges_overlap(p, bytes, c.status, ST_WORDS * 4);
}

namespace {

constexpr int LIST_THREADS = 1024;

// sum over the threads before this one; `total` of all of them
__device__ int64_t block_exclusive(int64_t v, int64_t *warp_sums, int64_t &total)
{
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
    int64_t x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (lane >= o) x += y;
    }
    __syncthreads();                         // the sums of the previous call have been read
    if (lane == 31) warp_sums[w] = x;
    __syncthreads();
    int64_t before = 0;
    total = 0;
    for (int i = 0; i < LIST_THREADS / 32; ++i) {
        const int64_t y = warp_sums[i];
        if (i < w) before += y;
        total += y;
    }
    return before + x - v;
}

// Queries that see no row: zeros, and the logarithm of nothing.  A warp writes the rows first .. first + count - 1 of a sequence
// whose tokens begin at q0, for all heads.
template <typename T> __device__ void empty_rows(const PagedAttnArgs &a, int q0, int first, int count, int lane)
{
    for (int h = 0; h < a.c.heads; ++h)
        for (int r = first; r < first + count; ++r) {
            const int64_t token = q0 + r / a.group;
            const int head = h * a.group + r % a.group;
            for (int c = lane; c < a.c.d; c += 32) ((T *)a.out)[token * a.ldo + (int64_t)head * a.c.d + c] = from_f32<T>(0.0f);
            if (lane == 0) a.lse[token * a.hq + head] = -INFINITY;
        }
}

// Lists the tiles of the sequences with more than min_rows rows, in order of the batch, with their first units, and the tile
// that each run begins in.  One CTA: a list of 10 000 tiles takes 10 turns.  Searches go through shared memory while the
// sequences and tiles fit (a search through global memory costs 0.4 us a step).
constexpr int LIST_NEAR = 2048;
__global__ void __launch_bounds__(LIST_THREADS) k_paged_list(const PagedAttnArgs a, int rows, int block)
{
    __shared__ int64_t warp_sums[LIST_THREADS / 32], near_units[LIST_NEAR];
    __shared__ int near_tiles[LIST_NEAR];
    pdl_enter();
    const PagedView &c = a.c;
    int64_t carry = 0, total;
    for (int s0 = 0; s0 < c.n_seq; s0 += LIST_THREADS) {
        const int s = s0 + threadIdx.x;
        int64_t n = 0;
        if (s < c.n_seq) {
            const int64_t r = (int64_t)paged_seq(c, s, true).n * a.group;
            n = r > a.min_rows ? (r + rows - 1) / rows : 0;
        }
        const int64_t before = block_exclusive(n, warp_sums, total);
        if (s < c.n_seq) {
            const int first = (int)min(carry + before, (int64_t)a.max_tiles);
            a.seq_tiles[s] = first;
            if (s < LIST_NEAR) near_tiles[s] = first;
        }
        carry += total;
    }
    if (carry > a.max_tiles) {               // overlapping offsets: more rows than tokens
        if (threadIdx.x == 0) paged_report(c, SITE_PAGED_OFFSETS);
        carry = a.max_tiles;
    }
    const int tiles = (int)carry;
    __syncthreads();                         // the first tiles are read by every thread below
    const int *first_tile = c.n_seq <= LIST_NEAR ? near_tiles : a.seq_tiles;
    int64_t units = 0;
    for (int t0 = 0; t0 < tiles; t0 += LIST_THREADS) {
        const int t = t0 + threadIdx.x;
        PagedTile e = {};
        int empty = 0;                       // rows of a tile without keys
        if (t < tiles) {
            int lo = 0, hi = c.n_seq;        // largest s with first_tile[s] <= t
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (first_tile[mid] <= t) lo = mid; else hi = mid;
            }
            const PagedSeq q = paged_seq(c, lo, false);
            e.q0 = q.q0; e.n = q.n; e.len = q.len; e.s = lo;
            e.r0 = (t - first_tile[lo]) * rows;
            const int live = min(rows, q.n * a.group - e.r0);
            const int keys = max(0, q.len - q.n + (e.r0 + live - 1) / a.group + 1);
            e.blocks = (keys + block - 1) / block;
            if (keys == 0) empty = live;
        }
        for (unsigned todo = __ballot_sync(0xffffffffu, empty > 0); todo; todo &= todo - 1) {
            const int from = __ffs(todo) - 1, lane = threadIdx.x & 31;
            const int q0 = __shfl_sync(0xffffffffu, e.q0, from), r0 = __shfl_sync(0xffffffffu, e.r0, from), n = __shfl_sync(0xffffffffu, empty, from);
            if (a.dtype == SKIPFFN_BF16) empty_rows<bf16>(a, q0, r0, n, lane);
            else empty_rows<float>(a, q0, r0, n, lane);
        }
        const int64_t before = block_exclusive(e.blocks ? (int64_t)(e.blocks + PG_TILE_COST) * c.heads : 0, warp_sums, total);
        e.u0 = units + before;
        if (t < tiles) {
            a.tiles[t] = e;
            if (t < LIST_NEAR) near_units[t] = e.u0;
        }
        units += total;
    }
    if (threadIdx.x == 0) *(int64_t *)a.head = units;
    __syncthreads();
    const Runs runs(units, a.runs);
    for (int b = threadIdx.x; b < runs.n; b += LIST_THREADS) {
        const int64_t u = runs.begin(b);
        int lo = 0;
        for (int hi = tiles; hi - lo > 1;) { // largest tile with u0 <= u: it holds u
            const int mid = (lo + hi) >> 1;
            if ((tiles <= LIST_NEAR ? near_units[mid] : a.tiles[mid].u0) <= u) lo = mid; else hi = mid;
        }
        a.starts[b] = lo;
    }
}

// Adds the pieces of a cut tile up, in their order.  Listed tiles: cut blockIdx.x, ROWS = 4 rows a warp (SUBS = 1).  Few rows:
// the cut of (sequence, head) blockIdx.x, all warps of the CTA for row blockIdx.y, each with every SUBS-th piece: one long
// sequence leaves a hundred pieces a row.  Bound by the latency of two dependent reads, and by CTAs that find nothing to do.
constexpr int JOIN_THREADS = 256, JOIN_WARPS = JOIN_THREADS / 32;
template <typename T, int SUBS, int ROWS> __global__ void __launch_bounds__(JOIN_THREADS) k_paged_join(const PagedAttnArgs a, int slot_rows, int pitch)
{
    __shared__ float sums[SUBS > 1 ? JOIN_WARPS : 1][PG_MAX_D + 4];
    pdl_enter();
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = warp % SUBS;
    const int row = (blockIdx.y * (JOIN_WARPS / SUBS) + warp / SUBS) * ROWS;
    const PagedCut cut = a.cuts[blockIdx.x];
    if (SUBS > 1) {                          // sequences that another kernel has leave no word about their tiles
        const PagedSeq q = paged_seq(a.c, blockIdx.x / a.c.heads, false);
        if (row >= q.n * a.group || q.n * a.group > slot_rows) return;
    }
    if (row >= cut.rows || cut.pieces == 0) return;              // with several warps a row: the same for all
    const int rows = min(ROWS, cut.rows - row);
    auto slot = [&](int i) { return (int64_t)(i == 0 ? 2 * cut.first + 1 : 2 * (cut.first + i)) * slot_rows + row; };
    const float c2 = a.scale * 1.4426950408889634f;
    float top[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) top[r] = -INFINITY;
    for (int i = lane; i < cut.pieces; i += 32)
#pragma unroll
        for (int r = 0; r < ROWS; ++r)
            if (r < rows) top[r] = fmaxf(top[r], a.part_ml[slot(i) + r].x);
#pragma unroll
    for (int r = 0; r < ROWS; ++r)
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top[r] = fmaxf(top[r], __shfl_xor_sync(0xffffffffu, top[r], o));
    const bool mine = 4 * lane < a.c.d;
    float l[ROWS] = {}, acc[ROWS][4] = {};
    for (int i0 = sub; i0 < cut.pieces; i0 += 32 * SUBS) {
        // each lane looks up one piece's weights, then all walk through them
        const int i1 = i0 + lane * SUBS;
        float f[ROWS], fl[ROWS];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) {
            float2 ml = make_float2(-INFINITY, 0.0f);
            if (i1 < cut.pieces && r < rows) ml = a.part_ml[slot(i1) + r];
            f[r] = ml.x == -INFINITY ? ml.y : exp2f((ml.x - top[r]) * c2);    // without a maximum the sum is 0, or NaN
            fl[r] = f[r] * ml.y;
        }
        const int n = min(32, (cut.pieces - i0 + SUBS - 1) / SUBS);
#pragma unroll(ROWS == 1 ? 8 : 2)
        for (int i = 0; i < n; ++i) {
            const float *src = a.part + slot(i0 + i * SUBS) * pitch + 4 * lane;
#pragma unroll
            for (int r = 0; r < ROWS; ++r) {
                const float w = __shfl_sync(0xffffffffu, f[r], i);
                l[r] += __shfl_sync(0xffffffffu, fl[r], i);
                if (w != 0.0f && mine) {     // a piece without keys for this row has written no sums
                    float v[4];
                    load4(src + r * pitch, v);
#pragma unroll
                    for (int e = 0; e < 4; ++e) acc[r][e] = fmaf(w, v[e], acc[r][e]);
                }
            }
        }
    }
    if (SUBS > 1) {
        if (mine) store4(&sums[warp][4 * lane], acc[0]);
        if (lane == 0) sums[warp][PG_MAX_D] = l[0];
        __syncthreads();
        if (sub != 0) return;
        for (int i = 1; i < SUBS; ++i) {
            float v[4];
            load4(&sums[warp + i][4 * lane], v);
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[0][e] += v[e];
            l[0] += sums[warp + i][PG_MAX_D];
        }
    }
#pragma unroll
    for (int i = 0; i < ROWS; ++i) {
        if (i >= rows) break;
        const int r = cut.r0 + row + i;
        const int64_t token = cut.q0 + r / a.group;
        const int head = cut.h * a.group + r % a.group;
        const bool none = met_nothing(top[i], l[i]);
        if (mine) {
            const float inv = 1.0f / l[i];
#pragma unroll
            for (int e = 0; e < 4; ++e) acc[i][e] = none ? 0.0f : acc[i][e] * inv;
            store4((T *)a.out + token * a.ldo + (int64_t)head * a.c.d + 4 * lane, acc[i]);
        }
        if (lane == 0) a.lse[token * a.hq + head] = none ? -INFINITY : fmaf(top[i], a.scale, logf(l[i]));
    }
}

struct Scratch { size_t cuts, head, starts, seq_tiles, tiles, ml, part, total; int64_t max_tiles; };

bool simt(const skipffn_paged_cache *c) { return c->dtype == SKIPFFN_FP32 || c->path == SKIPFFN_PATH_SIMT; }

// rows of a sequence that the kernel of few rows takes (0: that kernel is not asked for)
int few_rows(const skipffn_paged_cache *c)
{
    return c->path == SKIPFFN_PATH_SIMT ? 0 : c->dtype == SKIPFFN_FP32 ? PG_FEW_ROWS_FP32 : PG_FEW_ROWS;
}

Scratch scratch_of(const skipffn_paged_cache *c, int group, int64_t N)
{
    const int64_t most = std::min<int64_t>(c->max_new, N) * group;
    const bool few = few_rows(c) > 0, listed = !few || most > few_rows(c);
    // the largest of the kernels that the call may launch
    const int64_t slots = std::max(few ? PG_FEW_SLOTS : 0, !listed ? 0 : simt(c) ? PG_SIMT_SLOTS : 2 * PG_TC_RUNS * PG_TC_ROWS);
    const int64_t tile = simt(c) ? (most <= 16 ? 16 : 64) : 2 * (128 / group) * group;
    const int64_t pitch = !simt(c) && c->head_dim <= 64 ? 64 : 128;
    const size_t cuts = std::max<size_t>(std::max(PG_SIMT_RUNS, PG_TC_RUNS), few ? (size_t)c->n_seq * c->heads_kv : 0);
    Scratch s;
    s.max_tiles = listed ? N * group / tile + c->n_seq + 1 : 0;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t o = at; at = (at + bytes + 255) & ~(size_t)255; return o; };
    s.cuts = take(cuts * sizeof(PagedCut));
    s.head = take(64);
    s.starts = take(std::max(PG_SIMT_RUNS, PG_TC_RUNS) * 4);
    s.seq_tiles = take(((size_t)c->n_seq + 1) * 4);
    s.tiles = take((size_t)s.max_tiles * sizeof(PagedTile));
    s.ml = take((size_t)slots * sizeof(float2));
    s.part = take((size_t)slots * pitch * sizeof(float));
    s.total = at;
    return s;
}

}  // namespace

cudaError_t launch_paged_list(const PagedAttnArgs &a, int rows, int block, cudaStream_t s)
{
    return launch_pdl(k_paged_list, dim3(1), dim3(LIST_THREADS), s, a, rows, block);
}

cudaError_t launch_paged_join(const PagedAttnArgs &a, int rows, int pitch, cudaStream_t s)
{
    const dim3 grid((unsigned)a.runs, (unsigned)((rows + 4 * JOIN_WARPS - 1) / (4 * JOIN_WARPS)));
    return a.dtype == SKIPFFN_BF16 ? launch_pdl(k_paged_join<bf16, 1, 4>, grid, dim3(JOIN_THREADS), s, a, rows, pitch)
                                   : launch_pdl(k_paged_join<float, 1, 4>, grid, dim3(JOIN_THREADS), s, a, rows, pitch);
}

cudaError_t launch_paged_join_few(const PagedAttnArgs &a, int rows, int pitch, cudaStream_t s)
{
    const int64_t most = std::max<int64_t>(1, std::min<int64_t>(a.c.max_new, a.c.N) * a.group), tiles = (int64_t)a.c.n_seq * a.c.heads;
    const dim3 grid((unsigned)tiles, (unsigned)std::min<int64_t>(most, rows));
    return a.dtype == SKIPFFN_BF16 ? launch_pdl(k_paged_join<bf16, JOIN_WARPS, 1>, grid, dim3(JOIN_THREADS), s, a, rows, pitch)
                                   : launch_pdl(k_paged_join<float, JOIN_WARPS, 1>, grid, dim3(JOIN_THREADS), s, a, rows, pitch);
}

}  // namespace skipffn

using namespace skipffn;

static skipffn_status check_heads(const PagedView &v, int32_t heads_q, float scale)
{
    if (heads_q <= 0 || heads_q % v.heads || !(scale > 0.0f) || !isfinite(scale)) return SKIPFFN_EINVAL;
    const int group = heads_q / v.heads;
    // the kernels count the rows of a sequence (new tokens x heads of a group) in 32 bits, and a tile or two beyond
    const int64_t rows = std::min<int64_t>(v.max_new, v.N) * group;
    return group > 64 || heads_q > 65535 || rows > INT_MAX - 4096 ? SKIPFFN_EUNSUPPORTED : SKIPFFN_OK;
}

extern "C" {

size_t skipffn_paged_attention_scratch_bytes(const skipffn_paged_cache *cache, int32_t heads_q, int64_t n)
{
    PagedView v;
    if (paged_view(cache, n, &v) != SKIPFFN_OK || check_heads(v, heads_q, 1.0f) != SKIPFFN_OK) return 0;
    return scratch_of(cache, heads_q / v.heads, n).total;
}

skipffn_status skipffn_paged_attention(const skipffn_paged_cache *cache, int32_t heads_q, float scale, int64_t n, const void *q, int64_t ldq,
                                       void *out, int64_t ldo, float *lse, void *scratch, size_t scratch_bytes, void *stream)
{
    PagedAttnArgs a = {};
    skipffn_status st = paged_view(cache, n, &a.c);
    if (st == SKIPFFN_OK) st = check_heads(a.c, heads_q, scale);
    if (st != SKIPFFN_OK || n == 0 || a.c.n_seq == 0) return st;
    if ((int64_t)a.c.n_seq * a.c.heads > INT_MAX) return SKIPFFN_EUNSUPPORTED;
    const int es = cache->dtype == SKIPFFN_BF16 ? 2 : 4;
    for (const int64_t ld : {ldq, ldo})
        if (ld < 0 || ld > (int64_t)1 << 36) return SKIPFFN_EINVAL;
    const int64_t w = (int64_t)heads_q * a.c.d * es, wl = (int64_t)heads_q * 4;
    const TokenArray Q{q, ldq * es, w}, O{out, ldo * es, w}, L{lse, wl, wl};
    if (!token_array_ok(Q, n) || !token_array_ok(O, n) || !lse || !is_aligned(lse, 4) || !scratch || !is_aligned(scratch, 16)) return SKIPFFN_EINVAL;
    const Scratch sc = scratch_of(cache, heads_q / a.c.heads, n);
    if (scratch_bytes < sc.total) return SKIPFFN_EWORKSPACE;
    if (tokens_overlap(O, Q, n) || tokens_overlap(L, Q, n) || tokens_overlap(L, O, n)) return SKIPFFN_EINVAL;
    for (const TokenArray &x : {Q, O, L})
        if (ranges_overlap(scratch, sc.total, x.p, token_bytes(x, n))) return SKIPFFN_EINVAL;
    for (const TokenArray &x : {O, L})
        if (paged_overlap(a.c, x.p, token_bytes(x, n))) return SKIPFFN_EINVAL;
    if (paged_overlap(a.c, scratch, sc.total)) return SKIPFFN_EINVAL;
    a.q = q; a.out = out; a.ldq = ldq; a.ldo = ldo; a.lse = lse;
    a.hq = heads_q; a.group = heads_q / a.c.heads; a.dtype = cache->dtype; a.simt = simt(cache); a.scale = scale;
    char *base = (char *)scratch;
    a.part = (float *)(base + sc.part); a.part_ml = (float2 *)(base + sc.ml); a.cuts = (PagedCut *)(base + sc.cuts);
    a.tiles = (PagedTile *)(base + sc.tiles); a.head = (int64_t *)(base + sc.head); a.starts = (int32_t *)(base + sc.starts); a.seq_tiles = (int32_t *)(base + sc.seq_tiles);
    a.max_tiles = (int32_t)std::min<int64_t>(sc.max_tiles, INT_MAX);
    cudaStream_t s = (cudaStream_t)stream;
    const int64_t most = std::min<int64_t>(cache->max_new, n) * a.group;
    cudaError_t e = cudaSuccess;
    // Sequences of few rows are bound by reading their keys and have a kernel of their own; a single sequence that may have
    // more is not worth the launches that would find nothing to do.
    const int rows = few_rows(cache);
    const bool listed = rows == 0 || most > rows, few = rows > 0 && (!listed || a.c.n_seq > 1);
    a.min_rows = few ? rows : 0;
    if (few) e = launch_paged_few(a, s);
    if (e == cudaSuccess && listed) e = a.simt ? launch_paged_simt(a, (int)std::min<int64_t>(most, 64), s) : launch_paged_tc(a, s);
    return e == cudaSuccess ? SKIPFFN_OK : SKIPFFN_ECUDA;
}

skipffn_status skipffn_paged_weights(const skipffn_paged_cache *cache, int32_t heads_q, float scale, int64_t n, const void *q, int64_t ldq,
                                     const float *lse, const float *prior, float *weights, int32_t width, void *stream)
{
    PagedWeightsArgs a = {};
    skipffn_status st = paged_view(cache, n, &a.c);
    if (st == SKIPFFN_OK) st = check_heads(a.c, heads_q, scale);
    if (st != SKIPFFN_OK) return st;
    if (width < 0) return SKIPFFN_EINVAL;
    if (a.c.n_seq == 0 || width == 0) return SKIPFFN_OK;
    if (a.c.n_seq > 65535 || width > PG_MAX_COUNT) return SKIPFFN_EUNSUPPORTED;
    const int es = cache->dtype == SKIPFFN_BF16 ? 2 : 4;
    const int64_t bytes = (int64_t)a.c.n_seq * a.c.heads * width * 4, wl = (int64_t)heads_q * 4;
    if (ldq < 0 || ldq > (int64_t)1 << 36 || !weights || !is_aligned(weights, 4) || !is_aligned(prior, 4)) return SKIPFFN_EINVAL;
    if (n > 0) {
        const TokenArray Q{q, ldq * es, (int64_t)heads_q * a.c.d * es};
        if (!token_array_ok(Q, n) || !lse || !is_aligned(lse, 4)) return SKIPFFN_EINVAL;
        if (ranges_overlap(weights, bytes, q, token_bytes(Q, n)) || ranges_overlap(weights, bytes, lse, n * wl)) return SKIPFFN_EINVAL;
    }
    if (paged_overlap(a.c, weights, bytes) || (prior != weights && ranges_overlap(prior, bytes, weights, bytes))) return SKIPFFN_EINVAL;
    a.q = q; a.ldq = ldq; a.lse = lse; a.prior = prior; a.out = weights; a.hq = heads_q; a.group = heads_q / a.c.heads;
    a.dtype = cache->dtype; a.width = width; a.simt = simt(cache); a.scale = scale;
    const cudaError_t e = a.simt ? launch_paged_weights_simt(a, (cudaStream_t)stream) : launch_paged_weights(a, (cudaStream_t)stream);
    return e == cudaSuccess ? SKIPFFN_OK : SKIPFFN_ECUDA;
}

skipffn_status skipffn_paged_evict(const skipffn_paged_cache *cache, const skipffn_paged_cache *into, const float *weights, int32_t width,
                                   int32_t budget, int32_t sinks, int32_t recent, int32_t *kept, int32_t *lens_out, float *weights_out,
                                   void *stream)
{
    PagedEvictArgs a = {};
    skipffn_status st = paged_view(cache, 0, &a.c);
    if (st != SKIPFFN_OK) return st;
    if (width < 0 || budget < 1 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget) return SKIPFFN_EINVAL;
    // the same pages through the same table are the same place, however they are named
    a.in_place = !into || (into->k_pages == cache->k_pages && into->v_pages == cache->v_pages && into->page_table == cache->page_table);
    a.dst = a.c;
    if (into) {
        st = paged_view(into, 0, &a.dst);
        if (st != SKIPFFN_OK) return st;
        if (into->dtype != cache->dtype || into->heads_kv != cache->heads_kv || into->head_dim != cache->head_dim || into->n_seq != cache->n_seq)
            return SKIPFFN_EINVAL;
        // one pool seen with other strides has no order in which its rows could move
        if (a.in_place && (into->page_stride != cache->page_stride || into->row_stride != cache->row_stride || into->head_stride != cache->head_stride ||
                           into->page_size != cache->page_size || into->table_stride != cache->table_stride))
            return SKIPFFN_EINVAL;
    }
    if (a.c.n_seq == 0) return SKIPFFN_OK;
    if (width > PG_MAX_COUNT || budget > PG_MAX_COUNT) return SKIPFFN_EUNSUPPORTED;
    const int64_t pairs = (int64_t)a.c.n_seq * a.c.heads, wb = pairs * width * 4, kb = pairs * budget * 4, lb = (int64_t)a.c.n_seq * 4;
    if (pairs > INT_MAX / 16) return SKIPFFN_EUNSUPPORTED;
    if ((width > 0 && !weights) || !kept || !lens_out || !weights_out) return SKIPFFN_EINVAL;
    for (const void *p : {(const void *)weights, (const void *)kept, (const void *)lens_out, (const void *)weights_out})
        if (!is_aligned(p, 4)) return SKIPFFN_EINVAL;
    const struct { const void *p; int64_t n; } res[3] = {{kept, kb}, {lens_out, lb}, {weights_out, kb}};
    for (int i = 0; i < 3; ++i) {
        if (ranges_overlap(res[i].p, res[i].n, weights, wb) || paged_overlap(a.c, res[i].p, res[i].n) || paged_overlap(a.dst, res[i].p, res[i].n))
            return SKIPFFN_EINVAL;
        for (int j = 0; j < i; ++j)
            if (ranges_overlap(res[i].p, res[i].n, res[j].p, res[j].n)) return SKIPFFN_EINVAL;
    }
    a.weights = weights; a.width = width; a.budget = budget; a.sinks = sinks; a.recent = recent;
    a.kept = kept; a.lens_out = lens_out; a.weights_out = weights_out;
    a.elem_bytes = cache->dtype == SKIPFFN_BF16 ? 2 : 4;
    return launch_paged_evict(a, (cudaStream_t)stream) == cudaSuccess ? SKIPFFN_OK : SKIPFFN_ECUDA;
}

skipffn_status skipffn_paged_poll(const skipffn_paged_cache *cache, void *stream, int32_t *site_out)
{
    if (!cache || !cache->status) return SKIPFFN_EINVAL;
    // on the caller's stream, not the default one: that may be busy, and a block cleared behind this call's back would lose what the
    // next one reports
    const cudaStream_t s = (cudaStream_t)stream;
    int32_t w[3] = {0, 0, 0};
    if (cudaMemcpyAsync(w, cache->status, sizeof(w), cudaMemcpyDeviceToHost, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess) return SKIPFFN_ECUDA;
    if (site_out) *site_out = w[ST_SITE];
    if (w[ST_STATUS] != 0 && (cudaMemsetAsync(cache->status + ST_STATUS, 0, 8, s) != cudaSuccess || cudaStreamSynchronize(s) != cudaSuccess)) return SKIPFFN_ECUDA;
    return (skipffn_status)w[ST_STATUS];
}

}  // extern "C"
