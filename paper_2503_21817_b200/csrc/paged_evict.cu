// Eviction: per sequence and kv head the `budget` rows with the largest weights stay (the first `sinks` and the last
// `recent` in any case), in their order, and move to the front of the same pages or to other ones.
//
// k_evict_select: one cluster of CTAs per (sequence, head).  The weight that separates kept from evicted rows is found by
// four counts of eight bits each over the weights' order-preserving integer form; the CTAs' counts are added up through
// distributed shared memory, one cluster barrier a count (two sets of bins take turns).  A CTA's part of the weights is read
// once and stays in registers (up to HELD x 512 weights; what is beyond comes from L2 again).  Then every CTA numbers the
// kept rows of its part.  Bound by the chain of barriers and shared-memory atomics: 16 381 rows of 8 heads in clusters of 16.
// k_evict_move: a warp takes up to 32 rows; its lanes look up their places in parallel, then 16-byte pieces of keys and
// values move, 8 in flight a lane.  Bound by memory.  In place, a pair's rows move in steps of its whole cluster: a row's
// destination is never behind it (order is kept), so it is enough that a step has read all its rows before it writes any --
// later steps read only rows behind this step's destinations.
#include "paged.cuh"
#include "ptx.cuh"

namespace skipffn {

namespace {

constexpr int THREADS = 512, WARPS = THREADS / 32, HELD = 8;         // select: weights that a thread holds
constexpr int SPAN = THREADS * HELD;
constexpr int MOVE_THREADS = 256, PIECES = 8;                        // move: 16-byte pieces a lane holds

// weights in ascending order as unsigned integers; NaN below everything, -0 = +0
__device__ __forceinline__ uint32_t order_of(float w)
{
    if (w != w) return 0u;
    const uint32_t b = __float_as_uint(w + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ uint32_t read_peer(const void *p, uint32_t rank)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(mapa_rank(smem_u32(p), rank)) : "memory");
    return v;
}

__global__ void __launch_bounds__(THREADS) k_evict_select(const PagedEvictArgs a, const int size)
{
    __shared__ uint32_t bins[2][256], all[256];
    __shared__ uint32_t counts[2], picked[2], turn_counts[2];
    __shared__ uint32_t warp_sums[HELD][WARPS][2];
    const PagedView &c = a.c;
    const uint32_t rank = cluster_ctarank();
    const int pair = blockIdx.x / size, s = pair / c.heads, h = pair - s * c.heads;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (tid < 256) bins[0][tid] = bins[1][tid] = 0;
    pdl_enter();
    const int asked = c.lens[s];
    int len = min(max(asked, 0), c.capacity);
    const int m_all = min(len, a.width);
    if (tid == 0 && rank == 0 && h == 0) {
        if (len != asked) paged_report(c, SITE_PAGED_LENGTH);
        else if (len > a.width) paged_report(c, SITE_PAGED_WIDTH);
        a.lens_out[s] = min(m_all, a.budget);
        if (min(m_all, a.budget) > a.dst.capacity) paged_report(a.dst, SITE_PAGED_ROOM);
    }
    len = m_all;
    const int m = min(len, a.budget);
    const float *w = a.weights + ((int64_t)s * c.heads + h) * a.width;
    int32_t *kept = a.kept + ((int64_t)s * c.heads + h) * a.budget;
    float *wout = a.weights_out + ((int64_t)s * c.heads + h) * a.budget;
    // rows of this CTA: a contiguous part, so that kept rows are numbered in order
    const int part = (len + size - 1) / size, lo = min(len, (int)rank * part), hi = min(len, lo + part);
    const bool cut = len > a.budget;
    const int first = a.sinks, past = len - a.recent;               // rows first .. past - 1 compete when there is a cut
    uint32_t key[HELD];
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int j = lo + i * THREADS + tid;
        key[i] = cut && j < hi ? order_of(w[j]) : 0u;
    }
    uint32_t limit = 0, equal = 0;                                  // kept: order above `limit`, and the first `equal` at it
    if (cut) {
        uint32_t want = (uint32_t)(a.budget - a.sinks - a.recent);  // of past - first > want competitors
        for (int shift = 24, turn = 0; shift >= 0; shift -= 8, turn ^= 1) {
            __syncthreads();                                        // the bins of this turn are zero
            const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
            auto count = [&](int j, uint32_t k) {
                if (j >= first && j < past && (k & mask) == limit) atomicAdd(&bins[turn][(k >> shift) & 255], 1u);
            };
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                const int j = lo + i * THREADS + tid;
                if (j < hi) count(j, key[i]);
            }
            for (int j = lo + SPAN + tid; j < hi; j += THREADS) count(j, order_of(w[j]));
            cluster_sync_all();
            if (tid < 256) {
                uint32_t n = 0;
                for (int r = 0; r < size; ++r) n += read_peer(&bins[turn][tid], r);
                all[tid] = n;
                // the other set was read before this barrier and is next to be counted into
                bins[turn ^ 1][tid] = 0;
            }
            __syncthreads();
            if (tid < 32) {                                         // the bin that holds the want-th from above
                uint32_t mine = 0;
                for (int i = 0; i < 8; ++i) mine += all[255 - 8 * tid - i];
                uint32_t above = mine;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const uint32_t x = __shfl_up_sync(0xffffffffu, above, o);
                    if (tid >= o) above += x;
                }
                above -= mine;
                // want = 0: nothing but the protected rows; the topmost bin, of which none is taken
                if (want == 0 ? tid == 0 : above < want && want <= above + mine) {
                    int b = 255 - 8 * tid;
                    while (want > 0 && above + all[b] < want) above += all[b--];
                    picked[0] = (uint32_t)b;
                    picked[1] = want - above;
                }
            }
            __syncthreads();
            limit |= picked[0] << shift;
            want = picked[1];
        }
        equal = want;
    }
    // every row's state: kept for certain (bit 0), at the limit (bit 1)
    auto state = [&](int j, uint32_t k) -> uint32_t {
        if (j >= hi) return 0u;
        if (!cut || j < first || j >= past) return 1u;
        return k > limit ? 1u : k == limit ? 2u : 0u;
    };
    uint32_t n0 = 0, n1 = 0;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const uint32_t x = state(lo + i * THREADS + tid, key[i]);
        n0 += x & 1; n1 += x >> 1;
    }
    for (int j = lo + SPAN + tid; j < hi; j += THREADS) {
        const uint32_t x = state(j, order_of(w[j]));
        n0 += x & 1; n1 += x >> 1;
    }
    n0 = __reduce_add_sync(0xffffffffu, n0);
    n1 = __reduce_add_sync(0xffffffffu, n1);
    if (tid == 0) counts[0] = counts[1] = 0;
    __syncthreads();
    if (lane == 0) { atomicAdd(&counts[0], n0); atomicAdd(&counts[1], n1); }
    cluster_sync_all();
    uint32_t base0 = 0, base1 = 0;
    for (uint32_t r = 0; r < rank; ++r) { base0 += read_peer(&counts[0], r); base1 += read_peer(&counts[1], r); }
    for (int j0 = lo; j0 < hi; j0 += SPAN) {                        // one turn when the part fits the registers
        uint32_t below0[HELD], below1[HELD];                        // within the warp
        __syncthreads();
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int j = j0 + i * THREADS + tid;
            if (j0 > lo) key[i] = j < hi ? order_of(w[j]) : 0u;
            const uint32_t x = state(j, key[i]);
            const uint32_t v0 = __ballot_sync(0xffffffffu, x & 1), v1 = __ballot_sync(0xffffffffu, x & 2), mask = (2u << lane) - 1;
            below0[i] = __popc(v0 & mask);
            below1[i] = __popc(v1 & mask);
            if (lane == 31) { warp_sums[i][warp][0] = below0[i]; warp_sums[i][warp][1] = below1[i]; }
        }
        __syncthreads();
        if (tid < 32) {                                             // sums before each (slice of 512 rows, warp), four a lane
            uint32_t *flat = &warp_sums[0][0][0];
            uint32_t v[4][2], t0 = 0, t1 = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[i][0] = flat[(4 * lane + i) * 2];
                v[i][1] = flat[(4 * lane + i) * 2 + 1];
                t0 += v[i][0]; t1 += v[i][1];
            }
            uint32_t x0 = t0, x1 = t1;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t y0 = __shfl_up_sync(0xffffffffu, x0, o), y1 = __shfl_up_sync(0xffffffffu, x1, o);
                if (lane >= o) { x0 += y0; x1 += y1; }
            }
            x0 -= t0; x1 -= t1;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                flat[(4 * lane + i) * 2] = x0;
                flat[(4 * lane + i) * 2 + 1] = x1;
                x0 += v[i][0]; x1 += v[i][1];
            }
            if (lane == 31) { turn_counts[0] = x0; turn_counts[1] = x1; }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int j = j0 + i * THREADS + tid;
            const uint32_t x = state(j, key[i]);
            const uint32_t at_limit = base1 + warp_sums[i][warp][1] + below1[i];         // rows at the limit up to this one
            if (x == 1u || (x == 2u && at_limit <= equal)) {
                const uint32_t r = base0 + warp_sums[i][warp][0] + below0[i] + min(at_limit, equal) - 1;
                kept[r] = j;
                wout[r] = w[j];
            }
        }
        base0 += turn_counts[0]; base1 += turn_counts[1];
    }
    for (int r = m + (int)rank * THREADS + tid; r < a.budget; r += size * THREADS) { kept[r] = -1; wout[r] = 0.0f; }
    cluster_sync_all();                                             // no CTA leaves while its counts are read
}

// pieces per row, rows of a warp's turn
struct MoveShape { Divisor pieces; int rows, turns; };

template <bool IN_PLACE> __global__ void __launch_bounds__(MOVE_THREADS, 3) k_evict_move(const PagedEvictArgs a, const MoveShape f, const int size)
{
    pdl_enter();
    const PagedView &c = a.c;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = MOVE_THREADS / 32, half = f.pieces.d / 2;
    // in place: one cluster per pair, which takes its turns together; else a warp takes one turn of one pair
    const int64_t id = (int64_t)blockIdx.x * warps + warp;
    const int pair = IN_PLACE ? blockIdx.x / size : (int)(id / f.turns);
    if (pair >= c.n_seq * c.heads) return;
    const int s = pair / c.heads, h = pair - s * c.heads;
    const int len = min(min(max(c.lens[s], 0), c.capacity), a.width), m = min(min(len, a.budget), a.dst.capacity);
    const int32_t *kept = a.kept + (int64_t)pair * a.budget;
    const int step = IN_PLACE ? size * warps * f.rows : 0x7fffffff;
    for (int64_t r0 = IN_PLACE ? 0 : (id - (int64_t)pair * f.turns) * f.rows; r0 < m; r0 += step) {
        const int64_t mine = r0 + (IN_PLACE ? ((int)(blockIdx.x % size) * warps + warp) * f.rows : 0);
        // a lane's row: where it stands and where it goes
        int64_t from = -1, dest = -1;
        const int64_t r = mine + lane;
        if (lane < f.rows && r < m) {
            const int j = kept[r];
            if (!IN_PLACE || j != r) {
                from = paged_row(c, s, j);
                dest = paged_row(a.dst, s, (int)r);
                if (from < 0) paged_report(c, SITE_PAGED_PAGE);
                if (dest < 0) paged_report(a.dst, SITE_PAGED_PAGE);
            }
        }
        uint4 v[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int x = lane + 32 * i, row = div_by(x, f.pieces), p = x - row * (int)f.pieces.d;
            const int64_t src = __shfl_sync(0xffffffffu, from, row & 31), to = __shfl_sync(0xffffffffu, dest, row & 31);
            v[i] = make_uint4(0, 0, 0, 0);
            if (row < f.rows && src >= 0 && to >= 0)
                v[i] = __ldcs(reinterpret_cast<const uint4 *>((p < half ? c.k : c.v) + src + h * c.head_stride + (p < half ? p : p - half) * 16));
        }
        if (IN_PLACE) cluster_sync_all();
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int x = lane + 32 * i, row = div_by(x, f.pieces), p = x - row * (int)f.pieces.d;
            const int64_t to = __shfl_sync(0xffffffffu, dest, row & 31);
            if (row < f.rows && to >= 0)
                *reinterpret_cast<uint4 *>((p < half ? a.dst.k : a.dst.v) + to + h * a.dst.head_stride + (p < half ? p : p - half) * 16) = v[i];
        }
    }
}

template <typename Kernel, typename... Args>
cudaError_t launch_clusters(Kernel kernel, int64_t ctas, int threads, int size, cudaStream_t s, const Args &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ctas); cfg.blockDim = dim3(threads); cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim = {(unsigned)size, 1, 1};
    cfg.attrs = at; cfg.numAttrs = size > 0 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

}  // namespace

cudaError_t launch_paged_evict(const PagedEvictArgs &a, cudaStream_t s)
{
    const int pairs = a.c.n_seq * a.c.heads;
    int size = 8;                            // CTAs of a cluster: eight, fewer when the pairs alone fill the SMs
    while (size > 1 && pairs * size / 2 >= 2 * 148) size /= 2;
    cudaError_t e = launch_clusters(k_evict_select, (int64_t)pairs * size, THREADS, size, s, a, size);
    if (e != cudaSuccess) return e;
    MoveShape f;
    const int pieces = 2 * (a.c.d * a.elem_bytes / 16);
    f.pieces = make_divisor((uint32_t)pieces);
    f.rows = 32 * PIECES / pieces < 32 ? 32 * PIECES / pieces : 32;
    f.turns = (a.budget + f.rows - 1) / f.rows;
    if (a.in_place) return launch_clusters(k_evict_move<true>, (int64_t)pairs * size, MOVE_THREADS, size, s, a, f, size);
    const int64_t warps = (int64_t)pairs * f.turns, ctas = (warps + MOVE_THREADS / 32 - 1) / (MOVE_THREADS / 32);
    if (ctas > 0x7fffffff) return cudaErrorInvalidValue;
    return launch_clusters(k_evict_move<false>, ctas, MOVE_THREADS, 0, s, a, f, 0);
}

}  // namespace skipffn
