// Paged key / value cache: what the entry points (paged.cu) hand to the kernels, and how a kernel finds a row.
//
// Nothing that a kernel reads from device memory (offsets, lengths, page numbers) is trusted: offsets are cut to the
// tokens of the call, lengths to the rows the table has room for, and a page number outside the pool is a page that
// does not exist -- its rows read as zeros and are not written.  Each such repair leaves a status and a site.
#pragma once
#include "common.cuh"

namespace skipffn {

enum : int { SITE_PAGED_OFFSETS = 64, SITE_PAGED_LENGTH = 65, SITE_PAGED_PAGE = 66, SITE_PAGED_ROOM = 67, SITE_PAGED_WIDTH = 68 };

constexpr int PG_MAX_D = 128;
// sequences of a call, columns of weights, rows that eviction keeps: loops step past them by up to eight CTAs' threads
constexpr int PG_MAX_COUNT = 0x7fffffff - 8192;

// x / divisor for 0 <= x < 2^31 by one multiplication (divisor >= 2)
struct Divisor { uint32_t mul, shift, d; };
static inline Divisor make_divisor(uint32_t d)
{
    uint32_t sh = 1;
    while ((1ull << sh) < d) ++sh;                           // ceil(log2 d), at least 1
    return Divisor{(uint32_t)(((1ull << (31 + sh)) + d - 1) / d), sh - 1, d};
}

struct PagedView {
    char *k, *v;                             // row r of page p, head h: p * page_stride + r * row_stride + h * head_stride bytes
    int64_t page_stride, row_stride, head_stride;
    const int32_t *table, *cu, *lens;
    int64_t table_stride, n_pages;
    int32_t n_seq, heads, d, capacity;       // capacity: rows that a sequence's table has room for
    int64_t N, extent;                       // tokens of the call; bytes from the first to the last of a pool
    int32_t max_new;
    Divisor page;
    int32_t *status;
};

__device__ __forceinline__ int div_by(int x, const Divisor &d) { return (int)(__umulhi((uint32_t)x, d.mul) >> d.shift); }

__device__ __forceinline__ void paged_report(const PagedView &c, int site)
{
    if (atomicCAS(&c.status[ST_STATUS], 0, (int)SKIPFFN_EINVAL) == 0) c.status[ST_SITE] = site;
}

// One sequence: tokens q0 .. q0 + n - 1 of the call are its last n rows of `len`; token i sees rows j <= len - n + i.
struct PagedSeq { int q0, n, len; };
__device__ __forceinline__ PagedSeq paged_seq(const PagedView &c, int s, bool report)
{
    const int a = c.cu[s], b = c.cu[s + 1], l = c.lens[s];
    PagedSeq r;
    const int N = (int)c.N;
    r.q0 = min(max(a, 0), N);
    r.n = min(max(b, r.q0), N) - r.q0;
    r.len = min(max(l, 0), c.capacity);
    if (report) {
        if (r.q0 != a || r.q0 + r.n != b) paged_report(c, SITE_PAGED_OFFSETS);
        else if (r.n > c.max_new) paged_report(c, SITE_PAGED_OFFSETS);
        if (r.len != l) paged_report(c, SITE_PAGED_LENGTH);
    }
    if (r.n > c.max_new) r.n = 0;            // what the call was sized for does not hold: the sequence is left out
    return r;
}

// Does paged_seq take offsets a, b and length l as they are?
__device__ __forceinline__ bool paged_sound(const PagedView &c, int a, int b, int l)
{
    return a >= 0 && a <= b && b <= c.N && b - a <= c.max_new && l >= 0 && l <= c.capacity;
}

// Byte offset of row `row` (below the capacity), head 0, of sequence s; -1 if its page does not exist.
__device__ __forceinline__ int64_t paged_row(const PagedView &c, int s, int row)
{
    const int p = div_by(row, c.page);
    const int64_t e = c.table[(int64_t)s * c.table_stride + p];
    if (e < 0 || e >= c.n_pages) return -1;
    return e * c.page_stride + (int64_t)(row - p * (int)c.page.d) * c.row_stride;
}

// ---- work of the attention kernels over the cache
// A tile is up to `rows` consecutive rows of one sequence (row = token * group + head in group) of one kv head; its work
// is ceil(keys / block) blocks.  A line of units, PG_TILE_COST and then one for each block for every (tile, head), is cut into
// equal runs, one per CTA or group of warps: a run takes the end of one tile, some whole ones and the beginning of another.
// The units in front of a tile's blocks stand for what a tile costs beside them (measured about one block: without them
// the run that fell to a chunk of 500 tokens over 500 rows, 64 tiles of 1 to 4 blocks, took 150 us longer than the others).
// A tile inside one run is written at once; the pieces of a cut one go to the run's two slots -- the piece a run begins
// with (when it did not begin the tile) to slot 2b, the one it ends with to slot 2b + 1 -- and a second kernel adds them up
// in the order of the runs, from the one that holds the first block to the one that holds the last.
constexpr int PG_TILE_COST = 2;
struct PagedTile { int q0, n, r0, len, s, blocks; int64_t u0; };   // u0: first unit (of head 0)
struct PagedCut { int q0, r0, rows, h, pieces, first, pad[2]; };    // a tile that begins in run `first` and ends in a later one (pieces 0: none)

struct PagedAttnArgs {
    PagedView c;
    const void *q;
    void *out;
    int64_t ldq, ldo;
    float *lse;
    int32_t hq, group, dtype, simt;
    float scale;
    // scratch
    float *part;                             // [2 runs][rows][d or DP] unnormalised sums
    float2 *part_ml;                         // [2 runs][rows] maximum (of scores as they are) and sum
    PagedCut *cuts;                          // listed tiles: [runs]; few rows: [sequence][head]
    PagedTile *tiles;                        // listed tiles
    int64_t *head;                           // listed tiles: units
    int32_t *starts;                         // [runs] tile that a run begins in
    int32_t *seq_tiles;                      // [n_seq + 1] first tile of each sequence
    int32_t max_tiles;
    int32_t min_rows;                        // listed tiles: sequences of at most this many rows are another kernel's
    int32_t runs;
};

// Has a row with running maximum m and sum l met nothing but minus infinity?  The maximum alone does not say so: it passes NaN over, which
// the sum does not.
__device__ __forceinline__ bool met_nothing(float m, float l) { return m == -INFINITY && l == 0.0f; }

// Runs over `units` by at most `ctas` CTAs: no run is empty, since the pieces of a tile are counted by their runs.
struct Runs {
    int64_t units;
    int n;
    __host__ __device__ Runs(int64_t u, int ctas) : units(u), n(u < ctas ? (int)u : ctas) {}
    __host__ __device__ int64_t begin(int b) const { return b < n ? units * b / n : units; }
    __host__ __device__ int of(int64_t u) const { return (int)(((u + 1) * n - 1) / units); }     // the run that unit u lies in
};

struct PagedWeightsArgs {
    PagedView c;
    const void *q;
    int64_t ldq;
    const float *lse, *prior;
    float *out;
    int32_t hq, group, dtype, width, simt;
    float scale;
};

struct PagedEvictArgs {
    PagedView c, dst;
    const float *weights;                    // [n_seq, heads, width]
    int32_t width, budget, sinks, recent, in_place;
    int32_t *kept;                           // [n_seq, heads, budget]
    int32_t *lens_out;
    float *weights_out;                      // [n_seq, heads, budget]
    int32_t elem_bytes;
};

// rows of a tile, runs of a launch (these size the scratch): plain FMA, two CTAs an SM for 16 rows, one for 64; few rows,
// eight warps an SM
constexpr int PG_SIMT_KEYS = 64, PG_SIMT_RUNS = 296, PG_SIMT_SLOTS = 2 * 148 * 64;
constexpr int PG_FEW_ROWS = 16, PG_FEW_ROWS_FP32 = 8, PG_FEW_SMS = 160, PG_FEW_SLOTS = 2 * PG_FEW_SMS * 8 * PG_FEW_ROWS;
constexpr int PG_TC_RUNS = 160, PG_TC_ROWS = 256;     // tensor-core kernel: one run per SM, two row tiles

// paged.cu
// checks a cache for a call of N tokens and lays it out for the kernels
skipffn_status paged_view(const skipffn_paged_cache *c, int64_t N, PagedView *view);
// does a block of bytes touch the pages, or what the kernels read to find them?
bool paged_overlap(const PagedView &c, const void *p, int64_t bytes);
cudaError_t launch_paged_list(const PagedAttnArgs &a, int rows, int block, cudaStream_t s);
cudaError_t launch_paged_join(const PagedAttnArgs &a, int rows, int pitch, cudaStream_t s);
cudaError_t launch_paged_join_few(const PagedAttnArgs &a, int rows, int pitch, cudaStream_t s);
// paged_few.cu: sequences of at most PG_FEW_ROWS rows, bf16, or PG_FEW_ROWS_FP32
cudaError_t launch_paged_few(const PagedAttnArgs &a, cudaStream_t s);
// paged_tc.cu: sequences of more rows than that, bf16
cudaError_t launch_paged_tc(const PagedAttnArgs &a, cudaStream_t s);
// paged_simt.cu: sequences of more than min_rows and at most `rows` rows, any number, plain FMA
cudaError_t launch_paged_simt(const PagedAttnArgs &a, int rows, cudaStream_t s);
cudaError_t launch_paged_weights_simt(const PagedWeightsArgs &a, cudaStream_t s);
// paged_weights.cu (bf16)
cudaError_t launch_paged_weights(const PagedWeightsArgs &a, cudaStream_t s);
// paged_evict.cu
cudaError_t launch_paged_evict(const PagedEvictArgs &a, cudaStream_t s);

}  // namespace skipffn
