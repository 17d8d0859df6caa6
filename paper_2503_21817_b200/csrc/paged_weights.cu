// The softmax weight that every row of a paged cache gets from the new tokens of its sequence, per kv head, bf16:
//
//   weights[s, h, j] = prior + sum over new rows r of the head's group that see j of exp(scale q_r . k_j - lse_r)
//
// The forward's logarithms are given, so one pass over the keys suffices, and the sum over rows stays inside a warp: no
// atomics, a fixed order.  Work is a line of units (sequence, head, 64 keys) that is cut into runs of equal cost, one per
// CTA, two CTAs an SM; a CTA streams the steps of its units (64 keys x 32 rows; a unit's first step brings its keys, its
// last one its priors) through a ring of asynchronous copies.  Keys are the rows of the products' accumulators (mma.sync), so a thread
// adds its exponentials up as they come, and a warp's 16 keys stay in registers for all rows.  For few rows it is bound by
// reading the keys, for many by the products (legacy matrix instructions: 64 x 32 x d multiply-adds a step) and the
// exponentials.
#include "paged.cuh"
#include "paged_mma.cuh"

namespace skipffn {

namespace {

constexpr int THREADS = 128, KEYS = 64, ROWS = 32, ZERO_COLS = 1024;
constexpr float LOG2E = 1.4426950408889634f;

// What a stage of the ring holds, written when its copies are issued
struct StepInfo { int s, h, j0, r0, rows, off, len, first, last; };

template <int DP> struct WeightsShape {
    static constexpr int STAGES = DP == 128 ? 4 : 8;
    static constexpr int KEY_BYTES = KEYS * DP * 2, ROW_BYTES = ROWS * DP * 2;
    static constexpr int PRIOR = KEY_BYTES + ROW_BYTES, LSE = PRIOR + KEYS * 4, INFO = LSE + ROWS * 4, STAGE = INFO + 128;
    static constexpr int SMEM = STAGES * STAGE;
};

__device__ __forceinline__ void copy4(uint32_t dst, const void *src)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}

template <int DP> __global__ void __launch_bounds__(THREADS, 2) k_paged_weights(const PagedWeightsArgs a, const int runs)
{
    using Sh = WeightsShape<DP>;
    constexpr int CHUNKS = DP / 8, STEP = THREADS / CHUNKS;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ int64_t scan[THREADS / 32], place[2];
    pdl_enter();
    const PagedView &c = a.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, run = blockIdx.x;

    // ---- columns past a sequence's rows
    const int chunks = (a.width + ZERO_COLS - 1) / ZERO_COLS;
    for (int64_t i = run; i < (int64_t)c.n_seq * c.heads * chunks; i += runs) {
        const int64_t pair = i / chunks;
        const int j0 = (int)(i - pair * chunks) * ZERO_COLS, j1 = min(a.width, j0 + ZERO_COLS);
        const int len = min(max(c.lens[pair / c.heads], 0), c.capacity);
        for (int j = max(j0, len) + tid; j < j1; j += THREADS) a.out[pair * a.width + j] = 0.0f;
    }

    // ---- this CTA's run: units whose first step lies in it, in steps over the sequences
    auto steps_of = [&](const PagedSeq &q) { return max(1, (q.n * a.group + ROWS - 1) / ROWS); };        // of one unit
    auto blocks_of = [&](const PagedSeq &q) { return (min(q.len, a.width) + KEYS - 1) / KEYS; };
    auto cost_of = [&](int s) {
        if (s >= c.n_seq) return (int64_t)0;
        const PagedSeq q = paged_seq(c, s, run == 0);
        if (run == 0 && q.len > a.width) paged_report(c, SITE_PAGED_WIDTH);
        return (int64_t)blocks_of(q) * c.heads * steps_of(q);
    };
    auto block_sum = [&](int64_t v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        __syncthreads();
        if (lane == 0) scan[warp] = v;
        __syncthreads();
        return scan[0] + scan[1] + scan[2] + scan[3];
    };
    int64_t mine = 0;
    for (int s = tid; s < c.n_seq; s += THREADS) mine += cost_of(s);
    const Runs line(block_sum(mine), runs);
    const int64_t begin = line.begin(run), end = line.begin(run + 1);
    if (begin >= end) return;
    int64_t before = 0;
    for (int s0 = 0;; s0 += THREADS) {
        const int64_t v = cost_of(s0 + tid);
        int64_t x = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        const int64_t total = block_sum(v);
        int64_t lo = before + x - v;
        for (int i = 0; i < warp; ++i) lo += scan[i];
        if (v > 0 && lo <= begin && begin < lo + v) { place[0] = s0 + tid; place[1] = lo; }
        before += total;
        if (before > begin) break;           // the same in every thread; ends, since begin is inside the line
    }
    __syncthreads();

    // ---- the ring
    int s = (int)place[0], blocks, steps, unit, r0 = 0;
    int64_t at = place[1];                   // first step of the unit
    PagedSeq q;
    auto enter = [&]() { q = paged_seq(c, s, false); blocks = blocks_of(q); steps = steps_of(q); };
    auto first_row = [&](int j0) { return max(0, j0 - (q.len - q.n)) * a.group / ROWS * ROWS; };   // rows before it see none of the keys
    // to a unit that exists, when the run has one left
    auto settle = [&]() {
        while (unit == blocks * c.heads && at < end && s + 1 < c.n_seq) { ++s; enter(); unit = 0; }
        if (unit == blocks * c.heads) at = end;
        if (at < end) r0 = first_row(unit % blocks * KEYS);
    };
    enter();
    unit = (int)((begin - at + steps - 1) / steps);
    at += (int64_t)unit * steps;
    settle();
    const uint32_t ring = smem_u32(smem);
    int issued = 0;
    bool fresh = true;                       // the unit's first step
    auto issue = [&]() {
        if (at < end) {
            const int slot = issued % Sh::STAGES, h = unit / blocks, j0 = (unit - h * blocks) * KEYS, rows = q.n * a.group;
            const int len = min(q.len, a.width);
            const uint32_t dst = ring + slot * Sh::STAGE;
            const int chunk = tid % CHUNKS, t0 = tid / CHUNKS;
            const bool last = r0 + ROWS >= rows;
            if (fresh) {
                int64_t base = -1;           // lane i < 8: rows 8 i .. 8 i + 7
                if (lane < KEYS / 8 && j0 + 8 * lane < len && rows > 0) {
                    base = paged_row(c, s, j0 + 8 * lane);
                    if (base >= 0) base += h * c.head_stride;
                    else paged_report(c, SITE_PAGED_PAGE);
                }
#pragma unroll
                for (int i = 0; i < KEYS / STEP; ++i) {
                    const int r = t0 + i * STEP;
                    const int64_t g = __shfl_sync(0xffffffffu, base, r >> 3);
                    const bool on = g >= 0 && j0 + r < len && chunk * 8 < c.d;
                    copy16(dst + chunk_at<DP>(r, chunk), c.k + (on ? g + (r & 7) * c.row_stride + chunk * 16 : 0), on);
                }
            }
            if (last && a.prior && tid < KEYS && j0 + tid < len)
                copy4(dst + Sh::PRIOR + tid * 4, a.prior + ((int64_t)s * c.heads + h) * a.width + j0 + tid);
            const int live = min(ROWS, rows - r0);
#pragma unroll
            for (int i = 0; i < ROWS / STEP; ++i) {
                const int r = t0 + i * STEP;
                if (r >= ((live + 15) & ~15)) break;
                const bool on = r < live && chunk * 8 < c.d;
                const bf16 *src = (const bf16 *)a.q;
                if (on) src += (int64_t)(q.q0 + (r0 + r) / a.group) * a.ldq + (int64_t)(h * a.group + (r0 + r) % a.group) * c.d + chunk * 8;
                copy16(dst + Sh::KEY_BYTES + chunk_at<DP>(r, chunk), src, on);
            }
            if (tid < ROWS) {
                const int r = r0 + tid;
                if (tid < live) copy4(dst + Sh::LSE + tid * 4, a.lse + (int64_t)(q.q0 + r / a.group) * a.hq + h * a.group + r % a.group);
                else *reinterpret_cast<float *>(smem + slot * Sh::STAGE + Sh::LSE + tid * 4) = INFINITY;     // a row that is not there weighs nothing
            }
            if (tid == 0) *reinterpret_cast<StepInfo *>(smem + slot * Sh::STAGE + Sh::INFO) = StepInfo{s, h, j0, r0, rows, q.len - q.n, len, fresh, last};
            ++issued;
            fresh = last;
            r0 += ROWS;
            if (last) {
                ++unit;
                at += steps;
                settle();
            }
        }
        copy_commit();
    };
#pragma unroll
    for (int i = 0; i < Sh::STAGES - 1; ++i) issue();

    // ---- arithmetic: a warp has 16 keys, a thread keys `key` and `key` + 8 of them
    const int key = warp * 16 + (lane >> 2);
    uint32_t kf[DP / 16][4];
    float total[2] = {0.0f, 0.0f};
    for (int done = 0;; ++done) {
        if (done == issued) break;           // the ring is empty, and issue() had nothing to add
        copy_wait<Sh::STAGES - 2>();
        __syncthreads();                     // the step is there for every warp, and the slot refilled next is free
        issue();
        const int slot = done % Sh::STAGES;
        const uint32_t src = ring + slot * Sh::STAGE, rt = src + Sh::KEY_BYTES;
        const StepInfo t = *reinterpret_cast<const StepInfo *>(smem + slot * Sh::STAGE + Sh::INFO);
        const float *lse = reinterpret_cast<const float *>(smem + slot * Sh::STAGE + Sh::LSE);
        if (t.first) {
            total[0] = total[1] = 0.0f;
#pragma unroll
            for (int k = 0; k < DP / 16; ++k)
                // rows of a: lanes 0-15 keys 0-15 of eight columns, lanes 16-31 of the next eight
                ldsm_x4(src + chunk_at<DP>(warp * 16 + (lane & 15), 2 * k + (lane >> 4)), kf[k]);
        }
        // the first row of the step sees every key: no mask
        const bool masked = t.j0 + KEYS - 1 > t.off + t.r0 / a.group;
#pragma unroll
        for (int n = 0; n < ROWS / 8; n += 2) {
            if (t.r0 + 8 * n >= t.rows) break;
            float x[2][4] = {};
#pragma unroll
            for (int k = 0; k < DP / 16; ++k) {
                uint32_t b[4];
                ldsm_x4(rt + chunk_at<DP>(n * 8 + (lane >> 4) * 8 + (lane & 7), 2 * k + ((lane >> 3) & 1)), b);
                mma_16x8(x[0], kf[k], b[0], b[1]);
                mma_16x8(x[1], kf[k], b[2], b[3]);
            }
#pragma unroll
            for (int y = 0; y < 2; ++y) {
                const int i = 8 * (n + y) + 2 * (lane & 3);
                const float2 l2 = *reinterpret_cast<const float2 *>(lse + i);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float l = e & 1 ? l2.y : l2.x;
                    // the difference first: it is small where the weight counts, so its rounding is too
                    float w = fast_exp2(fmaf(x[y][e], a.scale, -l) * LOG2E);
                    // a token without a logarithm saw nothing
                    if (l == -INFINITY || (masked && t.j0 + key + 8 * (e >> 1) > t.off + (t.r0 + i + (e & 1)) / a.group)) w = 0.0f;
                    total[e >> 1] += w;
                }
            }
        }
        if (t.last) {
            const float *prior = reinterpret_cast<const float *>(smem + slot * Sh::STAGE + Sh::PRIOR);
            float *out = a.out + ((int64_t)t.s * c.heads + t.h) * a.width + t.j0;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                float w = total[i] + __shfl_xor_sync(0xffffffffu, total[i], 1);
                w += __shfl_xor_sync(0xffffffffu, w, 2);
                const int k = key + 8 * i;
                if ((lane & 3) == 0 && t.j0 + k < t.len) out[k] = a.prior ? prior[k] + w : w;
            }
        }
    }
    copy_wait<0>();
}

template <int DP> cudaError_t weights(const PagedWeightsArgs &a, cudaStream_t s)
{
    using Sh = WeightsShape<DP>;
    static int runs_of_device[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (runs_of_device[dev] == 0) {
        int sms = 0, per = 0;
        cudaError_t e = cudaFuncSetAttribute(k_paged_weights<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::SMEM);
        if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
        if (e == cudaSuccess) e = cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per, k_paged_weights<DP>, THREADS, Sh::SMEM);
        if (e != cudaSuccess) return e;
        if (per < 1) return cudaErrorInvalidConfiguration;
        runs_of_device[dev] = sms * (per < 2 ? per : 2);
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)runs_of_device[dev]); cfg.blockDim = dim3(THREADS); cfg.dynamicSmemBytes = Sh::SMEM; cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_paged_weights<DP>, a, runs_of_device[dev]);
}

}  // namespace

cudaError_t launch_paged_weights(const PagedWeightsArgs &a, cudaStream_t s) { return a.c.d <= 64 ? weights<64>(a, s) : weights<128>(a, s); }

}  // namespace skipffn
