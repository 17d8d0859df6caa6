// Eviction: per sequence and kv head the `budget` rows with the largest weights stay (the first `sinks` and the last
// `recent` in any case), in their order, and move to the front of the same pages or to other ones.
//
// k_evict_select: one cluster of CTAs per (sequence, head).  The weight that separates kept from evicted rows is found by
// three counts of 11, 11 and 10 bits over the weights' order-preserving integer form (with 8 bits first, sign and exponent
// alone, softmax weights crowd into a few bins and their atomic additions queue up).  A CTA counts its part, then adds its
// bins that are not empty to every CTA's sums in distributed shared memory: one cluster barrier a count.  A CTA's part of the
// weights is read once and stays in registers (up to HELD x 512; what is beyond comes from L2 again).  Then every CTA numbers
// the kept rows of its part.  Bound by this chain of counts and barriers: 22 us for 48 conversations of 37 to 8877 rows and 8
// heads (8-bit counts 36 us, with a barrier for every read of a peer's bins 33 us), 9 us for the 8 heads of one prompt.
// k_evict_move: a warp takes up to 32 rows; its lanes look up their places in parallel, then 16-byte pieces of keys and
// values move, 8 in flight a lane (4: 2 us less for the batch, 2 us more for one prompt; 16: 1 and 3 us more).  The three
// reads that find the next rows run behind the pieces of these.  Bound by memory: 61 us for the batch's 345 MB (5.7 TB/s;
// rows of a head are 256 bytes apart from their neighbours' in memory).  In place, a pair's rows move in steps of its whole cluster: a row's
// destination is never behind it (order is kept), so it is enough that a step has read all its rows before it writes any --
// later steps read only rows behind this step's destinations.  With its barriers the batch takes 95 us for 82, the one prompt 25 for 15.
#include <algorithm>
#include "paged.cuh"
#include "ptx.cuh"

namespace skipffn {

namespace {

constexpr int THREADS = 512, WARPS = THREADS / 32, HELD = 8;         // select: weights that a thread holds
constexpr int SPAN = THREADS * HELD, PER = HELD * WARPS / 32;
constexpr int BINS = 2048, OWN = BINS / THREADS;                     // bins of a count, of a thread
constexpr int MOVE_THREADS = 256, PIECES = 8;                        // move: 16-byte pieces a lane holds

// weights in ascending order as unsigned integers; NaN below everything, -0 = +0
__device__ __forceinline__ uint32_t order_of(float w)
{
    if (w != w) return 0u;
    const uint32_t b = __float_as_uint(w + 0.0f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// adds to the same word of CTA `rank` of the cluster
__device__ __forceinline__ void add_peer(uint32_t *p, uint32_t rank, uint32_t v)
{
    asm volatile("red.relaxed.cluster.shared::cluster.add.u32 [%0], %1;" ::"r"(mapa_rank(smem_u32(p), rank)), "r"(v) : "memory");
}
// inclusive sums over the lanes
__device__ __forceinline__ uint32_t lane_scan(uint32_t v, int lane)
{
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, v, o);
        if (lane >= o) v += x;
    }
    return v;
}

__global__ void __launch_bounds__(THREADS, 2) k_evict_select(const PagedEvictArgs a, const int size)
{
    static_assert(OWN == 4, "a thread's bins are one vector");
    __shared__ __align__(16) uint32_t bins[BINS], sums[3][BINS];    // of this CTA; of the cluster, one set a count
    __shared__ uint32_t before[2], picked[2], turn_counts[2], bin_sums[WARPS];
    __shared__ uint32_t warp_sums[HELD][WARPS][2];
    const PagedView &c = a.c;
    const uint32_t rank = cluster_ctarank();
    const int pair = blockIdx.x / size, s = pair / c.heads, h = pair - s * c.heads;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    auto own = [&](uint32_t *p) -> uint4 & { return *reinterpret_cast<uint4 *>(p + OWN * tid); };
    own(bins) = own(sums[0]) = own(sums[1]) = own(sums[2]) = make_uint4(0, 0, 0, 0);
    if (tid < 2) before[tid] = 0;
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");      // waited for before the first addition to a peer
    pdl_enter();
    const int asked = c.lens[s], all = min(min(max(asked, 0), c.capacity), a.width);
    if (tid == 0 && rank == 0 && h == 0) {
        if (asked < 0 || asked > c.capacity) paged_report(c, SITE_PAGED_LENGTH);
        else if (asked > a.width) paged_report(c, SITE_PAGED_WIDTH);
        a.lens_out[s] = min(all, a.budget);
        if (min(all, a.budget) > a.dst.capacity) paged_report(a.dst, SITE_PAGED_ROOM);
    }
    const int len = all, m = min(len, a.budget);
    const float *w = a.weights + ((int64_t)s * c.heads + h) * a.width;
    int32_t *kept = a.kept + ((int64_t)s * c.heads + h) * a.budget;
    float *wout = a.weights_out + ((int64_t)s * c.heads + h) * a.budget;
    // rows of this CTA: a contiguous part, so that kept rows are numbered in order
    const int part = (len + size - 1) / size, lo = min(len, (int)rank * part), hi = min(len, lo + part);
    const bool cut = len > a.budget;
    const int first = a.sinks, past = len - a.recent;               // rows first .. past - 1 compete when there is a cut
    float held[HELD];
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int j = lo + i * THREADS + tid;
        held[i] = j < hi ? w[j] : 0.0f;
    }
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
    uint32_t limit = 0, equal = 0;                                  // kept: order above `limit`, and the first `equal` at it
    if (cut) {
        uint32_t want = (uint32_t)(a.budget - a.sinks - a.recent);  // of past - first > want competitors
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
            const uint32_t mask = pass == 0 ? 0u : 0xffffffffu << (pass == 1 ? 21 : 10), digits = pass == 2 ? 1023 : 2047;
            uint32_t *mine = size == 1 ? sums[pass] : bins;
            auto count = [&](int j, float x) {
                const uint32_t k = order_of(x);
                if (j >= first && j < past && (k & mask) == limit) atomicAdd(&mine[(k >> shift) & digits], 1u);
            };
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                const int j = lo + i * THREADS + tid;
                if (j < hi) count(j, held[i]);
            }
#pragma unroll 4
            for (int j = lo + SPAN + tid; j < hi; j += THREADS) count(j, w[j]);
            __syncthreads();
            if (size > 1) {
                uint4 &v = own(bins);
#pragma unroll
                for (int i = 0; i < OWN; ++i) {
                    const uint32_t x = i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
                    if (x)
                        for (int r = 0; r < size; ++r) add_peer(&sums[pass][OWN * tid + i], r, x);
                }
                v = make_uint4(0, 0, 0, 0);
                cluster_sync_all();
            }
            // from above: thread 0 has the four highest bins
            const int top = BINS - OWN * (tid + 1);
            const uint4 n = *reinterpret_cast<const uint4 *>(&sums[pass][top]);
            const uint32_t here = n.x + n.y + n.z + n.w;
            uint32_t above = lane_scan(here, lane);
            if (lane == 31) bin_sums[warp] = above;
            __syncthreads();
            above -= here;
            for (int i = 0; i < warp; ++i) above += bin_sums[i];
            // the bin that holds the want-th from above; want = 0 (nothing but the protected rows): the topmost, none of it
            if (want == 0 ? tid == 0 : above < want && want <= above + here) {
                const uint32_t v[OWN] = {n.w, n.z, n.y, n.x};
                int b = 0;
#pragma unroll
                for (int i = 0; i < OWN - 1; ++i)
                    if (want > 0 && b == i && above + v[i] < want) { above += v[i]; ++b; }
                picked[0] = (uint32_t)(top + OWN - 1 - b) & digits;
                picked[1] = want - above;
            }
            __syncthreads();
            limit |= picked[0] << shift;
            want = picked[1];
        }
        equal = want;
    }
    // every row's state: kept for certain (bit 0), at the limit (bit 1)
    auto state = [&](int j, float x) -> uint32_t {
        if (j >= hi) return 0u;
        if (!cut || j < first || j >= past) return 1u;
        const uint32_t k = order_of(x);
        return k > limit ? 1u : k == limit ? 2u : 0u;
    };
    // rows kept before this CTA's part
    uint32_t base0 = 0, base1 = 0;
    if (size > 1) {
        uint32_t n0 = 0, n1 = 0;
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const uint32_t x = state(lo + i * THREADS + tid, held[i]);
            n0 += x & 1; n1 += x >> 1;
        }
#pragma unroll 4
        for (int j = lo + SPAN + tid; j < hi; j += THREADS) {
            const uint32_t x = state(j, w[j]);
            n0 += x & 1; n1 += x >> 1;
        }
        n0 = __reduce_add_sync(0xffffffffu, n0);
        n1 = __reduce_add_sync(0xffffffffu, n1);
        if (lane == 0)
            for (int r = rank + 1; r < size; ++r) { add_peer(&before[0], r, n0); add_peer(&before[1], r, n1); }
        cluster_sync_all();
        base0 = before[0];
        base1 = before[1];
    }
    for (int j0 = lo; j0 < hi; j0 += SPAN) {                        // one turn when the part fits the registers
        uint32_t below0[HELD], below1[HELD];                        // within the warp
        if (j0 > lo) {
#pragma unroll
            for (int i = 0; i < HELD; ++i) {
                const int j = j0 + i * THREADS + tid;
                held[i] = j < hi ? w[j] : 0.0f;
            }
            __syncthreads();                                        // the sums of the turn before have been read
        }
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const uint32_t x = state(j0 + i * THREADS + tid, held[i]);
            const uint32_t v0 = __ballot_sync(0xffffffffu, x & 1), v1 = __ballot_sync(0xffffffffu, x & 2), mask = (2u << lane) - 1;
            below0[i] = __popc(v0 & mask);
            below1[i] = __popc(v1 & mask);
            if (lane == 31) { warp_sums[i][warp][0] = below0[i]; warp_sums[i][warp][1] = below1[i]; }
        }
        __syncthreads();
        if (tid < 32) {                                             // sums before each (slice of rows, warp), PER a lane
            uint32_t *flat = &warp_sums[0][0][0];
            uint32_t v[PER][2], t0 = 0, t1 = 0;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                v[i][0] = flat[(PER * lane + i) * 2];
                v[i][1] = flat[(PER * lane + i) * 2 + 1];
                t0 += v[i][0]; t1 += v[i][1];
            }
            uint32_t x0 = lane_scan(t0, lane) - t0, x1 = lane_scan(t1, lane) - t1;
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                flat[(PER * lane + i) * 2] = x0;
                flat[(PER * lane + i) * 2 + 1] = x1;
                x0 += v[i][0]; x1 += v[i][1];
            }
            if (lane == 31) { turn_counts[0] = x0; turn_counts[1] = x1; }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
            const int j = j0 + i * THREADS + tid;
            const uint32_t x = state(j, held[i]);
            const uint32_t at_limit = base1 + warp_sums[i][warp][1] + below1[i];         // rows at the limit up to this one
            if (x == 1u || (x == 2u && at_limit <= equal)) {
                const uint32_t r = base0 + warp_sums[i][warp][0] + below0[i] + min(at_limit, equal) - 1;
                kept[r] = j;
                wout[r] = held[i];
            }
        }
        base0 += turn_counts[0]; base1 += turn_counts[1];
    }
    for (int r = m + (int)rank * THREADS + tid; r < a.budget; r += size * THREADS) { kept[r] = -1; wout[r] = 0.0f; }
}

// pieces per row, rows of a warp's turn
struct MoveShape { Divisor pieces; int rows, turns; };

template <bool IN_PLACE> __global__ void __launch_bounds__(MOVE_THREADS, 3) k_evict_move(const PagedEvictArgs a, const MoveShape f, const int size)
{
    pdl_enter();
    const PagedView &c = a.c;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = MOVE_THREADS / 32, half = f.pieces.d / 2;
    // In place, one cluster per pair, whose warps take `step` rows of it together.  Else the turns of all pairs are one line,
    // of which every warp has its share.
    const int64_t turns = (int64_t)c.n_seq * c.heads * f.turns, stride = (int64_t)gridDim.x * warps;
    const int step = size * warps * f.rows, own = IN_PLACE ? ((int)(blockIdx.x % size) * warps + warp) * f.rows : 0;
    int64_t at = IN_PLACE ? 0 : (int64_t)blockIdx.x * warps + warp;          // row of the pair; turn
    // a lane's row of a turn: where it stands and where it goes.  False behind the last turn.
    auto find = [&](int64_t t, int &h, int64_t &from, int64_t &dest) {
        from = dest = -1;
        if (!IN_PLACE && t >= turns) return false;
        const int pair = IN_PLACE ? blockIdx.x / size : (int)(t / f.turns), s = pair / c.heads;
        h = pair - s * c.heads;
        const int m = min(min(min(min(max(c.lens[s], 0), c.capacity), a.width), a.budget), a.dst.capacity);
        if (IN_PLACE && t >= m) return false;
        const int64_t r = (IN_PLACE ? t + own : (t - (int64_t)pair * f.turns) * f.rows) + lane;
        if (lane < f.rows && r < m) {
            const int j = a.kept[(int64_t)pair * a.budget + r];
            if (!IN_PLACE || j != r) {
                from = paged_row(c, s, j);
                dest = paged_row(a.dst, s, (int)r);
                if (from < 0) paged_report(c, SITE_PAGED_PAGE);
                if (dest < 0) paged_report(a.dst, SITE_PAGED_PAGE);
            }
        }
        return true;
    };
    int h, next_h = 0;
    int64_t from, dest, next_from, next_dest;
    bool more = find(at, h, from, dest);
    while (more) {
        uint4 v[PIECES];
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int x = lane + 32 * i, row = div_by(x, f.pieces), p = x - row * (int)f.pieces.d;
            const int64_t src = __shfl_sync(0xffffffffu, from, row & 31), to = __shfl_sync(0xffffffffu, dest, row & 31);
            v[i] = make_uint4(0, 0, 0, 0);
            if (row < f.rows && src >= 0 && to >= 0)
                v[i] = __ldcs(reinterpret_cast<const uint4 *>((p < half ? c.k : c.v) + src + h * c.head_stride + (p < half ? p : p - half) * 16));
        }
        at += IN_PLACE ? step : stride;
        more = find(at, next_h, next_from, next_dest);              // three reads, one after the other, behind those of the rows
        if (IN_PLACE) cluster_sync_all();
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int x = lane + 32 * i, row = div_by(x, f.pieces), p = x - row * (int)f.pieces.d;
            const int64_t to = __shfl_sync(0xffffffffu, dest, row & 31);
            if (row < f.rows && to >= 0)
                *reinterpret_cast<uint4 *>((p < half ? a.dst.k : a.dst.v) + to + h * a.dst.head_stride + (p < half ? p : p - half) * 16) = v[i];
        }
        h = next_h; from = next_from; dest = next_dest;
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
    return launch_clusters(k_evict_move<false>, std::min<int64_t>(ctas, 3 * 148), MOVE_THREADS, 0, s, a, f, 0);
}

}  // namespace skipffn
