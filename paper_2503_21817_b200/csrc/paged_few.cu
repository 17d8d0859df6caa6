// Attention over a paged cache for sequences of few rows (tokens x query heads of a kv head <= 64), bf16: the token that
// is being answered, a handful of proposed ones.
//
//   s_rj = scale q_r . k_j,  out_r = sum_j softmax(s_r)_j v_j,  one pass over the keys with a running maximum and sum.
//
// Bound by reading the cache once: 512 bytes a key and kv head at head_dim 128 for 4 x rows x 128 flops, so the legacy
// matrix instructions (mma.sync, whose accumulators are registers and need no second kernel role) are far from their
// limit at 16 rows.  The keys of all sequences and heads, 64 to a unit, are one line that is cut into equal runs, one per
// CTA (two CTAs an SM): ragged batches and one long sequence load every SM alike.  A run streams its units through a ring
// of asynchronous 16-byte copies; rows come from their pages eight at a time (a page holds whole groups of eight).
// Warps share a unit by keys when there are at most 16 rows (each has its own maximum and sum, added up at the end of a
// tile), by rows when there are 64.
#include "paged.cuh"
#include "paged_mma.cuh"

namespace skipffn {

namespace {

constexpr int THREADS = 128, KEYS = 64, STAGES = 3;
constexpr float LOG2E = 1.4426950408889634f;

// Units of a sequence: blocks of keys of one head; a sequence without keys has one, which writes its empty rows.
__device__ __forceinline__ int few_blocks(const PagedSeq &q, int group, int rows)
{
    return q.n > 0 && q.n * group <= rows ? max(1, (q.len + KEYS - 1) / KEYS) : 0;
}

// A place in the line of units
struct Place {
    int s, h, b, blocks;
    PagedSeq q;
    // to the first unit of the next sequence that has any; there is one when a unit is left
    __device__ void next_seq(const PagedView &c, int group, int rows)
    {
        do {
            ++s;
            q = paged_seq(c, s, false);
            blocks = few_blocks(q, group, rows);
        } while (blocks == 0 && s + 1 < c.n_seq);
        h = b = 0;
    }
    __device__ void step(const PagedView &c, int group, int rows, bool more)
    {
        if (++b < blocks) return;
        b = 0;
        if (++h < c.heads) return;
        if (more) next_seq(c, group, rows);
    }
};

template <int DP, int WM> struct FewShape {
    static constexpr int ROW = DP * 2, TILE = KEYS * ROW, STAGE = 2 * TILE;     // keys, then values
    static constexpr int WK = 4 / WM;                                        // warps that share the keys of a unit
    static constexpr int MERGE = WK > 1 ? WM * 16 * DP * 4 : 0;
    static constexpr int SMEM = STAGES * STAGE + MERGE;
};

template <int DP, int WM>
__global__ void __launch_bounds__(THREADS, 2) k_paged_few(const PagedAttnArgs a)
{
    using Sh = FewShape<DP, WM>;
    constexpr int WK = Sh::WK, WKEYS = KEYS / WK, NT = WKEYS / 8, CHUNKS = DP / 8;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ int64_t scan[THREADS / 32];
    __shared__ int place[2];
    __shared__ float2 stats[4][16];
    const PagedView &c = a.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, run = blockIdx.x, ROWS = 16 * WM;
    pdl_enter();

    // ---- where this CTA's run lies: sums of units over the sequences
    auto units_of = [&](int s) { return s < c.n_seq ? (int64_t)few_blocks(paged_seq(c, s, run == 0), a.group, ROWS) * c.heads : 0; };
    auto block_sum = [&](int64_t v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        __syncthreads();
        if (lane == 0) scan[warp] = v;
        __syncthreads();
        return scan[0] + scan[1] + scan[2] + scan[3];
    };
    int64_t mine = 0;
    for (int s = tid; s < c.n_seq; s += THREADS) mine += units_of(s);
    const Runs runs(block_sum(mine), a.runs);
    const int64_t begin = runs.begin(run), end = runs.begin(run + 1);
    if (tid == 0) a.cuts[run].pieces = 0;
    if (begin >= end) return;
    int64_t before = 0;
    Place at;
    for (int s0 = 0;; s0 += THREADS) {
        const int64_t v = units_of(s0 + tid);
        int64_t x = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        const int64_t total = block_sum(v);
        int64_t lo = before + x - v;
        for (int i = 0; i < warp; ++i) lo += scan[i];
        if (v > 0 && lo <= begin && begin < lo + v) {
            place[0] = s0 + tid;
            place[1] = (int)(begin - lo);
        }
        before += total;
        if (before > begin) break;           // the same in every thread; ends, since begin < units
    }
    __syncthreads();
    at.s = place[0];
    at.q = paged_seq(c, at.s, false);
    at.blocks = few_blocks(at.q, a.group, ROWS);
    at.h = place[1] / at.blocks;
    at.b = place[1] - at.h * at.blocks;
    int64_t item = begin - at.b;             // first unit of the current tile

    // ---- the ring
    const uint32_t ring = smem_u32(smem);
    Place ahead = at;
    int64_t issued = begin;
    auto issue = [&]() {
        if (issued < end) {
            const uint32_t dst = ring + (uint32_t)((issued - begin) % STAGES) * Sh::STAGE;
            const int j0 = ahead.b * KEYS;
            // lane i < 8 finds the rows 8 i .. 8 i + 7 of the block; -1: not there
            int64_t base = -1;
            if (lane < KEYS / 8 && j0 + 8 * lane < ahead.q.len) {
                base = paged_row(c, ahead.s, j0 + 8 * lane);
                if (base >= 0) base += ahead.h * c.head_stride;
                else paged_report(c, SITE_PAGED_PAGE);
            }
            const int chunk = tid % CHUNKS, r0 = tid / CHUNKS;
            constexpr int STEP = THREADS / CHUNKS;
#pragma unroll
            for (int i = 0; i < KEYS / STEP; ++i) {
                const int r = r0 + i * STEP;
                const int64_t g = __shfl_sync(0xffffffffu, base, r >> 3);
                const bool on = g >= 0 && j0 + r < ahead.q.len && chunk * 8 < c.d;
                const int64_t off = on ? g + (r & 7) * c.row_stride + chunk * 16 : 0;
                const uint32_t to = dst + chunk_at<DP>(r, chunk);
                copy16(to, c.k + off, on);
                copy16(to + Sh::TILE, c.v + off, on);
            }
            ++issued;
            ahead.step(c, a.group, ROWS, issued < end);
        }
        copy_commit();
    };
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) issue();

    // ---- arithmetic: warp = (rows 16 wm .., keys wk * WKEYS ..); a thread has rows r0 and r0 + 8 of its 16
    const int wm = warp % WM, wk = warp / WM, r0 = wm * 16 + (lane >> 2);
    const float c2 = a.scale * LOG2E;
    uint32_t qf[DP / 16][4];
    float o[DP / 8][4], m[2], l[2];
    int limit[2] = {0, 0};
    for (int64_t u = begin; u < end; ++u) {
        if (u == begin || at.b == 0) {       // a new tile: its queries
            item = u - at.b;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = r0 + 8 * i;
                const bool live = r < at.q.n * a.group;
                limit[i] = live ? at.q.len - at.q.n + r / a.group + 1 : 0x7fffffff;   // a dead row's sums go nowhere
                const uint32_t *src = live ? (const uint32_t *)((const bf16 *)a.q + (int64_t)(at.q.q0 + r / a.group) * a.ldq +
                                                                (int64_t)(at.h * a.group + r % a.group) * c.d) : nullptr;
#pragma unroll
                for (int k = 0; k < DP / 16; ++k)
#pragma unroll
                    for (int x = 0; x < 2; ++x) {
                        const int col = 16 * k + 8 * x + 2 * (lane & 3);
                        qf[k][2 * x + i] = src && col < c.d ? src[col / 2] : 0u;
                    }
                m[i] = -INFINITY;
                l[i] = 0.0f;
            }
#pragma unroll
            for (int n = 0; n < DP / 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][e] = 0.0f;
        }
        copy_wait<STAGES - 2>();
        __syncthreads();                     // the unit is there for every warp, and the slot refilled next is free
        issue();
        const uint32_t kt = ring + (uint32_t)((u - begin) % STAGES) * Sh::STAGE + wk * WKEYS * Sh::ROW, vt = kt + Sh::TILE;
        const int j0 = at.b * KEYS + wk * WKEYS;
        float s[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] = 0.0f;
#pragma unroll
        for (int k = 0; k < DP / 16; ++k)
#pragma unroll
            for (int n = 0; n < NT; n += 2) {
                const int r = n * 8 + (lane >> 4) * 8 + (lane & 7), ch = 2 * k + ((lane >> 3) & 1);
                uint32_t b[4];
                ldsm_x4(kt + chunk_at<DP>(r, ch), b);
                mma_16x8(s[n], qf[k], b[0], b[1]);
                mma_16x8(s[n + 1], qf[k], b[2], b[3]);
            }
        // keys past a row's own
        if (j0 + WKEYS > min(limit[0], limit[1])) {
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (j0 + 8 * n + 2 * (lane & 3) + (e & 1) >= limit[e >> 1]) s[n][e] = -INFINITY;
        }
        float f[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float t = -INFINITY;
#pragma unroll
            for (int n = 0; n < NT; ++n) t = fmaxf(t, fmaxf(s[n][2 * i], s[n][2 * i + 1]));
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 1));
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2));
            t = fmaxf(t, m[i]);
            f[i] = t == m[i] ? 1.0f : fast_exp2((m[i] - t) * c2);
            m[i] = t;
            // a row that has met nothing but minus infinity has p = 2^(-inf) = 0 so far, not 2^(-inf + inf)
            const float shift = t == -INFINITY ? 0.0f : -t * c2;
            float sum = 0.0f;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float p = fast_exp2(fmaf(s[n][2 * i + e], c2, shift));
                    s[n][2 * i + e] = p;
                    sum += p;
                }
            l[i] = l[i] * f[i] + sum;        // of this thread's keys; the four threads of a row add up at the end
        }
        if (__any_sync(0xffffffffu, f[0] != 1.0f || f[1] != 1.0f)) {
#pragma unroll
            for (int n = 0; n < DP / 8; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) o[n][e] *= f[e >> 1];
        }
#pragma unroll
        for (int k = 0; k < NT / 2; ++k) {
            // p as operand of the second product: rounded to bf16, relative 2^-9 a term; the sum l takes it unrounded
            const uint32_t p[4] = {pack_bf16(s[2 * k][0], s[2 * k][1]), pack_bf16(s[2 * k][2], s[2 * k][3]),
                                   pack_bf16(s[2 * k + 1][0], s[2 * k + 1][1]), pack_bf16(s[2 * k + 1][2], s[2 * k + 1][3])};
#pragma unroll
            for (int n = 0; n < DP / 16; ++n) {
                const int r = 16 * k + (lane & 15), ch = 2 * n + (lane >> 4);
                uint32_t b[4];
                ldsm_x4_trans(vt + chunk_at<DP>(r, ch), b[0], b[1], b[2], b[3]);
                mma_16x8(o[2 * n], p, b[0], b[1]);
                mma_16x8(o[2 * n + 1], p, b[2], b[3]);
            }
        }
        if (u + 1 < end && at.b + 1 < at.blocks) { ++at.b; continue; }

        // ---- the end of this run's part of the tile
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
        }
        if (WK > 1) {
            // the warps of a row group: a common maximum, then their sums one after the other
            if ((lane & 3) == 0)
#pragma unroll
                for (int i = 0; i < 2; ++i) stats[warp][(lane >> 2) + 8 * i] = make_float2(m[i], l[i]);
            __syncthreads();
            float g[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float2 w[WK];
                float t = -INFINITY;
#pragma unroll
                for (int x = 0; x < WK; ++x) { w[x] = stats[x * WM + wm][(lane >> 2) + 8 * i]; t = fmaxf(t, w[x].x); }
                g[i] = m[i] == -INFINITY ? 0.0f : fast_exp2((m[i] - t) * c2);
                float sum = 0.0f;
#pragma unroll
                for (int x = 0; x < WK; ++x) sum += w[x].x == -INFINITY ? 0.0f : w[x].y * fast_exp2((w[x].x - t) * c2);
                m[i] = t;
                l[i] = sum;
            }
            float *merge = reinterpret_cast<float *>(smem + STAGES * Sh::STAGE) + wm * 16 * DP;
            for (int x = 1; x < WK; ++x) {
                if (wk == x)
#pragma unroll
                    for (int n = 0; n < DP / 8; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) merge[(4 * n + e) * 32 + lane] = o[n][e] * g[e >> 1];
                __syncthreads();
                if (wk == 0)
#pragma unroll
                    for (int n = 0; n < DP / 8; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[n][e] = (x == 1 ? o[n][e] * g[e >> 1] : o[n][e]) + merge[(4 * n + e) * 32 + lane];
                __syncthreads();
            }
        }
        const int64_t last = item + at.blocks;
        const bool whole = item >= begin && last <= end;
        if (wk == 0) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = r0 + 8 * i;
                if (r >= at.q.n * a.group) continue;
                const int64_t token = at.q.q0 + r / a.group;
                const int head = at.h * a.group + r % a.group;
                if (whole) {
                    bf16 *dst = (bf16 *)a.out + token * a.ldo + (int64_t)head * c.d;
                    const float inv = 1.0f / l[i];
                    const bool none = m[i] == -INFINITY;
#pragma unroll
                    for (int n = 0; n < DP / 8; ++n) {
                        const int col = 8 * n + 2 * (lane & 3);
                        if (col < c.d)
                            *reinterpret_cast<uint32_t *>(dst + col) = none ? 0u : pack_bf16(o[n][2 * i] * inv, o[n][2 * i + 1] * inv);
                    }
                    if ((lane & 3) == 0) a.lse[token * a.hq + head] = none ? -INFINITY : fmaf(m[i], a.scale, logf(l[i]));
                } else {
                    const int64_t to = (int64_t)(2 * run + (item >= begin ? 1 : 0)) * ROWS + r;
#pragma unroll
                    for (int n = 0; n < DP / 8; ++n)
                        *reinterpret_cast<float2 *>(a.part + to * DP + 8 * n + 2 * (lane & 3)) = make_float2(o[n][2 * i], o[n][2 * i + 1]);
                    if ((lane & 3) == 0) a.part_ml[to] = make_float2(m[i], l[i]);
                }
            }
        }
        if (item >= begin && last > end && tid == 0) {
            PagedCut cut = {};
            cut.q0 = at.q.q0; cut.rows = at.q.n * a.group; cut.h = at.h;
            cut.pieces = runs.of(last - 1) - run + 1;
            a.cuts[run] = cut;
        }
        at.step(c, a.group, ROWS, u + 1 < end);
    }
    copy_wait<0>();
}

template <int DP, int WM> cudaError_t few(const PagedAttnArgs &args, cudaStream_t s)
{
    using Sh = FewShape<DP, WM>;
    static int runs_of_device[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (runs_of_device[dev] == 0) {
        int sms = 0, per = 0;
        cudaError_t e = cudaFuncSetAttribute(k_paged_few<DP, WM>, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::SMEM);
        if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, k_paged_few<DP, WM>, THREADS, Sh::SMEM);
        if (e != cudaSuccess) return e;
        if (per < 1) return cudaErrorInvalidConfiguration;
        runs_of_device[dev] = sms * (per < 2 ? per : 2) < PG_MAX_RUNS ? sms * (per < 2 ? per : 2) : PG_MAX_RUNS;
    }
    PagedAttnArgs a = args;
    a.runs = runs_of_device[dev];
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)a.runs); cfg.blockDim = dim3(THREADS); cfg.dynamicSmemBytes = Sh::SMEM; cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, k_paged_few<DP, WM>, a);
    return e != cudaSuccess ? e : launch_paged_join(a, 16 * WM, DP, s);
}

}  // namespace

cudaError_t launch_paged_few(const PagedAttnArgs &a, int tile_rows, cudaStream_t s)
{
    if (a.c.d <= 64) return tile_rows == 16 ? few<64, 1>(a, s) : tile_rows == 32 ? few<64, 2>(a, s) : few<64, 4>(a, s);
    return tile_rows == 16 ? few<128, 1>(a, s) : tile_rows == 32 ? few<128, 2>(a, s) : few<128, 4>(a, s);
}

}  // namespace skipffn
