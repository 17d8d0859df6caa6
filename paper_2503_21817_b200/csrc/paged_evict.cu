// Eviction: per sequence and kv head the `budget` rows with the largest weights stay (the first `sinks` and the last
// `recent` in any case), in their order, and move to the front of the same pages or to other ones.
//
// One cluster of CTAs per (sequence, head).  The weight that separates kept from evicted rows is found by four counts of
// eight bits each over the weights' order-preserving integer form, the counts of the CTAs added up through distributed
// shared memory; then every CTA numbers the kept rows of its part, and the rows move.  A row's destination is never
// behind it (order is kept), so in place it is enough that everything is read, in steps of the whole cluster, before what
// stands at the destinations of the same step is overwritten: later steps read only rows behind this step's destinations.
#include "paged.cuh"
#include "ptx.cuh"

namespace skipffn {

namespace {

constexpr int THREADS = 512, WARPS = THREADS / 32, HOLD = 4;         // 16-byte pieces a thread holds in a step of the move

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

// inclusive sums over the CTA of two counts
__device__ __forceinline__ uint2 block_scan(uint2 v, uint2 *warp_sums, uint2 &total)
{
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, v.x, o), y = __shfl_up_sync(0xffffffffu, v.y, o);
        if (lane >= o) { v.x += x; v.y += y; }
    }
    __syncthreads();
    if (lane == 31) warp_sums[w] = v;
    __syncthreads();
    total = make_uint2(0, 0);
    uint2 before = make_uint2(0, 0);
    for (int i = 0; i < WARPS; ++i) {
        const uint2 x = warp_sums[i];
        if (i < w) { before.x += x.x; before.y += x.y; }
        total.x += x.x; total.y += x.y;
    }
    return make_uint2(v.x + before.x, v.y + before.y);
}

__global__ void __launch_bounds__(THREADS) k_paged_evict(const PagedEvictArgs a, const int size)
{
    __shared__ uint32_t bins[256], all[256];
    __shared__ uint32_t counts[2];
    __shared__ uint32_t picked[2];
    __shared__ uint2 warp_sums[WARPS];
    pdl_enter();
    const PagedView &c = a.c;
    const uint32_t rank = cluster_ctarank();
    const int pair = blockIdx.x / size, s = pair / c.heads, h = pair - s * c.heads, tid = threadIdx.x;
    const int asked = c.lens[s];
    int len = min(max(asked, 0), c.capacity);
    if (tid == 0 && rank == 0 && h == 0) {
        if (len != asked) paged_report(c, SITE_PAGED_LENGTH);
        else if (len > a.width) paged_report(c, SITE_PAGED_WIDTH);
    }
    len = min(len, a.width);
    const int m = min(len, a.budget);
    const float *w = a.weights + ((int64_t)s * c.heads + h) * a.width;
    int32_t *kept = a.kept + ((int64_t)s * c.heads + h) * a.budget;
    float *wout = a.weights_out + ((int64_t)s * c.heads + h) * a.budget;
    if (h == 0 && rank == 0 && tid == 0) {
        a.lens_out[s] = m;
        if (m > a.dst.capacity) paged_report(a.dst, SITE_PAGED_ROOM);
    }
    // rows of this CTA: a contiguous part, so that kept rows are numbered in order
    const int part = (len + size - 1) / size, lo = min(len, (int)rank * part), hi = min(len, lo + part);
    const bool cut = len > a.budget;
    const int first = a.sinks, past = len - a.recent;               // rows first .. past - 1 compete when there is a cut
    uint32_t limit = 0, equal = 0;                                  // kept: order above `limit`, and the first `equal` at it
    if (cut) {
        uint32_t want = (uint32_t)(a.budget - a.sinks - a.recent);  // of past - first > want competitors
        uint32_t prefix = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
            for (int i = tid; i < 256; i += THREADS) bins[i] = 0;
            __syncthreads();
            const uint32_t mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
            for (int j = max(lo, first) + tid; j < min(hi, past); j += THREADS) {
                const uint32_t k = order_of(w[j]);
                if ((k & mask) == prefix) atomicAdd(&bins[(k >> shift) & 255], 1u);
            }
            cluster_sync_all();
            if (tid < 256) {
                uint32_t n = 0;
                for (int r = 0; r < size; ++r) n += read_peer(&bins[tid], r);
                all[tid] = n;
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
            cluster_sync_all();                                     // the bins have been read by every CTA
            prefix |= picked[0] << shift;
            want = picked[1];
        }
        limit = prefix;
        equal = want;
    }
    // every row's state: kept for certain (x), at the limit (y)
    auto state = [&](int j) {
        if (!cut || j < first || j >= past) return make_uint2(1, 0);
        const uint32_t k = order_of(w[j]);
        return make_uint2(k > limit ? 1 : 0, k == limit ? 1 : 0);
    };
    uint2 sum = make_uint2(0, 0), total;
    for (int j = lo + tid; j < hi; j += THREADS) { const uint2 x = state(j); sum.x += x.x; sum.y += x.y; }
    block_scan(sum, warp_sums, total);
    if (tid == 0) { counts[0] = total.x; counts[1] = total.y; }
    cluster_sync_all();
    uint2 base = make_uint2(0, 0);
    for (uint32_t r = 0; r < rank; ++r) { base.x += read_peer(&counts[0], r); base.y += read_peer(&counts[1], r); }
    for (int j0 = lo; j0 < hi; j0 += THREADS) {
        const int j = j0 + tid;
        const uint2 x = j < hi ? state(j) : make_uint2(0, 0);
        const uint2 upto = block_scan(x, warp_sums, total);
        const uint32_t at_limit = base.y + upto.y;                  // rows at the limit up to this one
        if (x.x || (x.y && at_limit <= equal)) {
            const uint32_t r = base.x + upto.x + min(at_limit, equal) - 1;
            kept[r] = j;
            wout[r] = w[j];
        }
        base.x += total.x; base.y += total.y;
    }
    for (int r = m + (int)rank * THREADS + tid; r < a.budget; r += size * THREADS) { kept[r] = -1; wout[r] = 0.0f; }
    cluster_sync_all();                                             // `kept` is complete for the whole cluster

    // ---- the move: pieces of 16 bytes, keys then values of a row
    const int pieces = c.d * a.elem_bytes / 16, per_row = 2 * pieces;
    const int64_t work = (int64_t)m * per_row, step = (int64_t)size * THREADS * HOLD;
    for (int64_t w0 = 0; w0 < work; w0 += step) {
        uint4 v[HOLD];
        char *to[HOLD];
#pragma unroll
        for (int i = 0; i < HOLD; ++i) {
            const int64_t x = w0 + ((int64_t)i * size + rank) * THREADS + tid;
            to[i] = nullptr;
            if (x >= work) continue;
            const int r = (int)(x / per_row), p = (int)(x - (int64_t)r * per_row), col = p < pieces ? p : p - pieces;
            const int j = kept[r];
            if (r >= a.dst.capacity || (a.in_place && j == r)) continue;
            const int64_t from = paged_row(c, s, j), dest = paged_row(a.dst, s, r);
            if (from < 0) paged_report(c, SITE_PAGED_PAGE);
            if (dest < 0) paged_report(a.dst, SITE_PAGED_PAGE);
            if (dest < 0) continue;
            v[i] = make_uint4(0, 0, 0, 0);
            if (from >= 0) v[i] = __ldcs(reinterpret_cast<const uint4 *>((p < pieces ? c.k : c.v) + from + h * c.head_stride + col * 16));
            to[i] = (p < pieces ? a.dst.k : a.dst.v) + dest + h * a.dst.head_stride + col * 16;
        }
        if (a.in_place) cluster_sync_all();
#pragma unroll
        for (int i = 0; i < HOLD; ++i)
            if (to[i]) *reinterpret_cast<uint4 *>(to[i]) = v[i];
    }
}

}  // namespace

cudaError_t launch_paged_evict(const PagedEvictArgs &a, cudaStream_t s)
{
    const int pairs = a.c.n_seq * a.c.heads;
    int size = 8;                            // CTAs of a cluster: eight, fewer when the pairs alone fill the SMs
    while (size > 1 && pairs * size / 2 >= 2 * 148) size /= 2;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(pairs * size)); cfg.blockDim = dim3(THREADS); cfg.stream = s;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim = {(unsigned)size, 1, 1};
    cfg.attrs = at; cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, k_paged_evict, a, size);
}

}  // namespace skipffn
