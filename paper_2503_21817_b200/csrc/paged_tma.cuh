// Tiles of 128 cache rows in shared memory: a row tile of one head comes from several pages, one TMA box of
// gcd(page_size, 128) rows from each, issued by the lanes of one warp.
#pragma once
#include "attention_tc.cuh"
#include "paged.cuh"

namespace skipffn {

namespace {

// This lane's part of a tile: its page's entry in the table, read a tile ahead and not looked at until then, and the row inside
// the page (-1: nothing to load)
struct PageBox { int page, row; };

struct PageBoxes {
    const PagedView &c;
    int box, lane;                           // rows of a box
    __device__ PageBox find(int s, int len, int j0) const
    {
        PageBox b = {0, -1};
        const int r = j0 + lane * box;
        if (lane < TILE / box && r < len) {
            const int k = div_by(r, c.page);
            b.page = c.table[(int64_t)s * c.table_stride + k];
            b.row = r - k * (int)c.page.d;
        }
        return b;
    }
    // a page that does not exist becomes the first one past the pool, which reads as zeros
    __device__ void check(PageBox &b) const
    {
        if (b.row >= 0 && (b.page < 0 || b.page >= c.n_pages)) {
            b.page = (int)c.n_pages;
            b.row = 0;
            paged_report(c, SITE_PAGED_PAGE);
        }
    }
    template <int DP> __device__ void load(uint32_t dst, const CUtensorMap *map, uint32_t bar, const PageBox &b, int head) const
    {
        const int n = __popc(__ballot_sync(0xffffffffu, b.row >= 0));
        if (lane == 0) mbar_expect_tx(bar, (uint32_t)(n * box * DP * 2));
        __syncwarp();
        if (b.row >= 0)
#pragma unroll
            for (int s = 0; s < DP / 64; ++s)
                asm volatile(
                    "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes "
                    "[%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst + s * (TILE * 128) + lane * box * 128),
                    "l"(map), "r"(64 * s), "r"(head), "r"(b.row), "r"(b.page), "r"(bar)
                    : "memory");
        __syncwarp();
    }
};

// ---- host
// rows of a box: gcd(page_size, 128), at least 8
int box_rows(const PagedView &c)
{
    int box = TILE;
    while ((int)c.page.d % box) box /= 2;
    return box;
}
// a pool of pages as [page][row][head][column]; box = 64 columns of `rows` rows of one head.  Without pages no row is ever
// loaded: any address (`spare`) will do.
bool pool_map(CUtensorMap *m, const void *base, const void *spare, const PagedView &c, int rows)
{
    EncodeTiledFn enc = get_encode();
    if (!enc) return false;
    // a level of one entry may carry any stride
    const int64_t width = (int64_t)c.d * 2, head = c.heads > 1 ? c.head_stride : width;
    const int64_t page = c.n_pages > 1 ? c.page_stride : (int64_t)1 << 30;
    cuuint64_t dims[4] = {(cuuint64_t)c.d, (cuuint64_t)c.heads, (cuuint64_t)c.page.d, (cuuint64_t)(c.n_pages > 0 ? c.n_pages : 1)};
    cuuint64_t strides[3] = {(cuuint64_t)head, (cuuint64_t)c.row_stride, (cuuint64_t)page};
    cuuint32_t box[4] = {64u, 1u, (cuuint32_t)rows, 1u}, es[4] = {1u, 1u, 1u, 1u};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void *>(c.n_pages > 0 ? base : spare), dims, strides, box, es,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

}  // namespace skipffn
