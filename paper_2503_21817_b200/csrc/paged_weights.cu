// The softmax weight that every row of a paged cache gets from the new tokens of its sequence, per kv head, bf16:
//
//   weights[s, h, j] = prior + sum over new rows r of the head's group that see j of exp(scale q_r . k_j - lse_r)
//
// The forward's logarithms are given, so one pass over the keys suffices.  Scores are made with the keys on the
// accumulator's rows (tcgen05.mma, 128 keys x up to 128 rows of queries), so a thread of the epilogue has one key and adds
// its exponentials up in a register: no atomics, no shuffles, a fixed order.  Work is a line of units (sequence, head,
// 128 keys), each with a step for every tile of query rows, cut into runs of equal steps, one CTA per SM:
//   warp 0       key tiles through a ring (pages looked up a tile ahead), query tiles where they change
//   warp 1       one product per step into one of four accumulators
//   warps 2, 3   what needs no product: columns past a sequence's rows, sequences without new tokens
//   warps 4..11  two groups that take units in turn: exponentials and sums
// Bound by reading the keys for up to about 100 query rows a kv head, by the exponentials (16 a cycle and SM) beyond.  On the
// legacy matrix instructions a step of 64 keys x 32 rows took 2 us from its copies to its sums however it was cut, with eight
// warps an SM: 100 us for the batch of 48 conversations (238 MB), 250 us for 161 observing tokens of 40 heads.
#include "paged_tma.cuh"

namespace skipffn {

namespace {

constexpr int WARPS = 12, THREADS = 32 * WARPS, ACCS = 4, FIRST = 4, ZERO_COLS = 1024;

struct WeightsParams {
    PagedWeightsArgs a;
    int32_t tokens, box;                     // tokens of a tile of query rows; rows of a TMA box
};
struct alignas(64) WeightsMaps { CUtensorMap q, k; };

template <int DP> struct WeightsShape {
    static constexpr int T_BYTES = tile_bytes<DP>(), SLOTS = DP == 128 ? 4 : 8;
    static constexpr int SMEM = (2 + SLOTS) * T_BYTES + 2048;
};
struct alignas(8) WeightsCtl {
    uint64_t k_full[8], k_empty[8], q_full[2], q_empty[2], acc_full[ACCS], acc_empty[ACCS];
    int64_t scan[WARPS], place[2];
    uint32_t tmem_base;
    volatile int abort_flag;
    volatile uint32_t issued;
};

// One product: 128 keys from j0 on against `live` rows of queries, the tokens from t0 on
struct Step {
    int s, h, j0, t0, live, q0, off, len;    // len: rows that have a weight
    int unit, count;                         // of this run: units before this one, steps up to this one
    bool first, last, load_q;                // of the unit; other queries than the step before
};

// Walks the steps of this CTA's run, the same in every role
struct Line {
    const WeightsParams &p;
    int64_t at, end;                         // first step of the unit, end of the run
    int s, unit = 0, blocks, steps, tile = 0, units = 0, count = 0;
    int held_s = -1, held_h = -1;            // whose only tile of queries is in shared memory
    bool fresh = true;
    PagedSeq q;
    __device__ static int blocks_of(const PagedWeightsArgs &a, const PagedSeq &q) { return q.n > 0 ? (min(q.len, a.width) + TILE - 1) / TILE : 0; }
    __device__ static int64_t cost_of(const WeightsParams &p, const PagedSeq &q)
    {
        return (int64_t)blocks_of(p.a, q) * p.a.c.heads * ceil_div(q.n, p.tokens);
    }
    __device__ void enter()
    {
        q = paged_seq(p.a.c, s, false);
        blocks = blocks_of(p.a, q);
        steps = ceil_div(q.n, p.tokens);
    }
    // the run's units are those whose first step lies in it
    __device__ Line(const WeightsParams &p_, int64_t begin, int64_t end_, int seq, int64_t before) : p(p_), at(before), end(end_), s(seq)
    {
        if (begin >= end) { at = end; return; }
        enter();
        unit = (int)((begin - at + steps - 1) / steps);
        at += (int64_t)unit * steps;
        settle();
    }
    __device__ void settle()
    {
        while (unit == blocks * p.a.c.heads && at < end && s + 1 < p.a.c.n_seq) { ++s; enter(); unit = 0; }
        if (unit == blocks * p.a.c.heads) at = end;
        if (at < end) tile = max(0, unit % blocks * TILE - (q.len - q.n)) / p.tokens;     // tokens before it see none of the keys
    }
    __device__ bool next(Step &w)
    {
        if (at >= end) return false;
        w.s = s; w.h = unit / blocks; w.j0 = (unit - w.h * blocks) * TILE; w.t0 = tile * p.tokens;
        w.live = min(p.tokens, q.n - w.t0) * p.a.group;
        w.q0 = q.q0; w.off = q.len - q.n; w.len = min(q.len, p.a.width);
        w.unit = units; w.count = count++;
        w.first = fresh;
        w.last = fresh = ++tile == steps;
        w.load_q = steps > 1 || s != held_s || w.h != held_h;
        held_s = s; held_h = w.h;
        if (fresh) { ++unit; ++units; at += steps; settle(); }
        return true;
    }
};

template <int DP>
__global__ void __launch_bounds__(THREADS, 1) k_paged_weights(const __grid_constant__ WeightsMaps tm, const __grid_constant__ WeightsParams p)
{
    using Sh = WeightsShape<DP>;
    constexpr int T_BYTES = Sh::T_BYTES, SLOTS = Sh::SLOTS;
    extern __shared__ __align__(1024) uint8_t smem_raw[];
    // of each epilogue warp (so that none waits for another): logarithms of the tile's rows of queries, and the last key
    // that each sees, -1 for a row that gives nothing
    __shared__ __align__(16) float lses[WARPS - FIRST][TILE];
    __shared__ __align__(16) int sees[WARPS - FIRST][TILE];
    const uint32_t q_tile = smem_u32(smem_raw), ring = q_tile + 2 * T_BYTES;
    WeightsCtl *ctl = reinterpret_cast<WeightsCtl *>(smem_raw + (2 + SLOTS) * T_BYTES);
    const PagedWeightsArgs &a = p.a;
    const PagedView &c = a.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < SLOTS; ++i) { mbar_init(smem_u32(&ctl->k_full[i]), 1); mbar_init(smem_u32(&ctl->k_empty[i]), 1); }
        for (int i = 0; i < 2; ++i) { mbar_init(smem_u32(&ctl->q_full[i]), 1); mbar_init(smem_u32(&ctl->q_empty[i]), 1); }
        for (int i = 0; i < ACCS; ++i) { mbar_init(smem_u32(&ctl->acc_full[i]), 1); mbar_init(smem_u32(&ctl->acc_empty[i]), 4); }
        ctl->abort_flag = 0;
        ctl->issued = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    const int used = a.group * p.tokens;     // rows of a tile that a box fills; the others stay zero
    if (used < TILE) zero_smem(q_tile, 2 * T_BYTES);
    fence_proxy_async_smem();
    if (warp == 1) { tmem_alloc(smem_u32(&ctl->tmem_base), AT_TMEM_COLS); tmem_relinquish(); }
    pdl_enter();

    // ---- this CTA's run
    auto cost = [&](int s, bool report) {
        if (s >= c.n_seq) return (int64_t)0;
        const PagedSeq q = paged_seq(c, s, report);
        if (report && q.len > a.width) paged_report(c, SITE_PAGED_WIDTH);
        return Line::cost_of(p, q);
    };
    auto block_sum = [&](int64_t v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        __syncthreads();
        if (lane == 0) ctl->scan[warp] = v;
        __syncthreads();
        int64_t t = 0;
        for (int i = 0; i < WARPS; ++i) t += ctl->scan[i];
        return t;
    };
    int64_t mine = 0;
    for (int s = tid; s < c.n_seq; s += THREADS) mine += cost(s, blockIdx.x == 0);
    const Runs runs(block_sum(mine), (int)gridDim.x);
    const int64_t begin = runs.begin(blockIdx.x), end = runs.begin(blockIdx.x + 1);
    int64_t before = 0;
    for (int s0 = 0; s0 < c.n_seq && begin < end; s0 += THREADS) {
        const int64_t v = cost(s0 + tid, false);
        int64_t x = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        const int64_t total = block_sum(v);
        int64_t lo = before + x - v;
        for (int i = 0; i < warp; ++i) lo += ctl->scan[i];
        if (v > 0 && lo <= begin && begin < lo + v) { ctl->place[0] = s0 + tid; ctl->place[1] = lo; }
        before += total;
        if (before > begin) break;           // the same in every thread
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const Waits waits{&ctl->abort_flag, &ctl->issued, c.status, (uint32_t)WAIT_LIMIT_NS};
    bool ok = true;
    auto line = [&]() { return Line(p, begin, end, (int)ctl->place[0], ctl->place[1]); };

    if (warp == 0) {
        const PageBoxes boxes{c, p.box, lane};
        Line walk = line();
        Step w, n;
        uint32_t k = 0, q = 0;               // tiles of keys, of queries so far
        bool more = walk.next(w);
        PageBox box = {0, -1}, next = box;
        if (more) box = boxes.find(w.s, w.len, w.j0);
        while (more && ok) {
            const bool another = walk.next(n);
            if (another && n.first) next = boxes.find(n.s, n.len, n.j0);
            if (w.load_q) {
                const uint32_t s = q & 1;
                ok = wait_warp<true>(smem_u32(&ctl->q_empty[s]), ((q >> 1) & 1) ^ 1, waits, SITE_PRODUCER_EMPTY);
                if (!ok) break;
                if (lane == 0) {
                    mbar_expect_tx(smem_u32(&ctl->q_full[s]), (uint32_t)(used * DP * 2));
                    load_tile<DP>(q_tile + s * T_BYTES, &tm.q, w.h * a.group, w.q0 + w.t0, smem_u32(&ctl->q_full[s]));
                }
                ++q;
            }
            if (w.first) {
                boxes.check(box);
                const uint32_t s = k % SLOTS;
                ok = wait_warp<true>(smem_u32(&ctl->k_empty[s]), ((k / SLOTS) & 1) ^ 1, waits, SITE_PRODUCER_EMPTY);
                if (!ok) break;
                boxes.load<DP>(ring + s * T_BYTES, &tm.k, smem_u32(&ctl->k_full[s]), box, w.h);
                ++k;
                if (lane == 0) ctl->issued = k;
            }
            if (another && n.first) box = next;
            w = n;
            more = another;
        }
    } else if (warp == 1) {
        const uint32_t on = elect_one();     // the warp walks as one, one thread issues
        const uint32_t q_desc = desc_rows(q_tile), k_desc = desc_rows(ring);
        Line walk = line();
        Step w;
        uint32_t k = 0, q = 0;
        while (ok && walk.next(w)) {
            if (w.load_q) {
                // the queries before these have no product left to come
                if (q > 0) umma_commit_if(on, smem_u32(&ctl->q_empty[(q - 1) & 1]));
                ok = wait_warp<true>(smem_u32(&ctl->q_full[q & 1]), (q >> 1) & 1, waits, SITE_MMA_FULL);
                ++q;
            }
            if (w.first) {
                ok = ok && wait_warp<true>(smem_u32(&ctl->k_full[k % SLOTS]), (k / SLOTS) & 1, waits, SITE_MMA_FULL);
                ++k;
            }
            const uint32_t acc = w.count % ACCS, n = uniform(w.count) / ACCS;
            ok = ok && wait_warp<true>(smem_u32(&ctl->acc_empty[acc]), (n & 1) ^ 1, waits, SITE_MMA_TMEM_EMPTY);
            if (!ok) break;
            tc_fence_after();
            const uint32_t ks = uniform((int)((k - 1) % SLOTS)), qs = uniform((int)((q - 1) & 1));
            mma_rows_rows<DP>(on, tmem + uniform((int)acc) * TILE, k_desc + ks * (T_BYTES >> 4), q_desc + qs * (T_BYTES >> 4),
                              idesc_rows(uniform(mma_cols(w.live))));
            umma_commit_if(on, smem_u32(&ctl->acc_full[acc]));
            if (w.last) umma_commit_if(on, smem_u32(&ctl->k_empty[ks]));
        }
    } else if (warp < FIRST) {
        const int chunks = ceil_div(a.width, ZERO_COLS);
        for (int64_t i = blockIdx.x; i < (int64_t)c.n_seq * c.heads * chunks; i += gridDim.x) {
            const int64_t pair = i / chunks;
            const int j0 = (int)(i - pair * chunks) * ZERO_COLS, j1 = min(a.width, j0 + ZERO_COLS);
            const PagedSeq q = paged_seq(c, (int)(pair / c.heads), false);
            const int from = q.n > 0 ? max(j0, q.len) : j0;
            for (int j = from + tid - 64; j < j1; j += 64) {
                const int64_t at = pair * a.width + j;
                a.out[at] = j < q.len && a.prior ? a.prior[at] : 0.0f;
            }
        }
    } else {
        const int g = (warp - FIRST) >> 2, mine = (warp & 3) * 32 + lane;      // group, key of the unit
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        Line walk = line();
        Step w, n;
        auto next = [&](Step &x) {           // this group's units
            while (walk.next(x))
                if ((x.unit & 1) == g) return true;
            return false;
        };
        // a group sees every other unit: the queries are others when sequence, head or tile are
        int held_s = -1, held_h = -1, held_t = -1;
        auto changes = [&](const Step &x) { return x.s != held_s || x.h != held_h || x.t0 != held_t; };
        float ahead[4], total = 0.0f, prior = 0.0f, *ls = lses[warp - FIRST];
        int *see = sees[warp - FIRST];
        bool odd = false;                    // the tile has rows that give nothing
        auto look_up = [&](const Step &x) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = lane + 32 * i;
                ahead[i] = r < x.live ? a.lse[(int64_t)(x.q0 + x.t0 + r / a.group) * a.hq + x.h * a.group + r % a.group] : -INFINITY;
            }
        };
        bool more = next(w);
        if (more) look_up(w);
        while (more && ok) {
            if (changes(w)) {
                bool none = false;
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = lane + 32 * i;
                    const bool empty = ahead[i] == -INFINITY;
                    ls[r] = empty ? 0.0f : ahead[i];
                    see[r] = empty ? -1 : w.off + w.t0 + r / a.group;
                    none |= empty && r < w.live;
                }
                odd = __any_sync(0xffffffffu, none);
                __syncwarp();
                held_s = w.s; held_h = w.h; held_t = w.t0;
            }
            if (w.first) {
                total = 0.0f;
                prior = a.prior && w.j0 + mine < w.len ? a.prior[((int64_t)w.s * c.heads + w.h) * a.width + w.j0 + mine] : 0.0f;
            }
            const bool another = next(n);
            if (another && changes(n)) look_up(n);
            const uint32_t acc = w.count % ACCS;
            ok = wait_warp<true>(smem_u32(&ctl->acc_full[acc]), (w.count / ACCS) & 1, waits, SITE_EPI_TMEM_FULL);
            if (!ok) break;
            tc_fence_after();
            // every row of the tile sees every key, and gives something
            const bool plain = w.j0 + TILE - 1 <= w.off + w.t0 && !odd;
            const int key = w.j0 + mine;
#pragma unroll 1
            for (int c0 = 0; c0 < w.live; c0 += 16) {
                uint32_t x[16];
                tmem_ld16(tmem + lanes + acc * TILE + c0, x);
                tmem_ld_wait(x);
                float sum = 0.0f;
                // the difference first: it is small where the weight counts, so its rounding is too
                if (plain && c0 + 16 <= w.live) {
#pragma unroll
                    for (int e = 0; e < 16; e += 4) {
                        float l[4];
                        load4(ls + c0 + e, l);
#pragma unroll
                        for (int y = 0; y < 4; ++y) sum += fast_exp2(fmaf(__uint_as_float(x[e + y]), a.scale, -l[y]) * LOG2E);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float v = fast_exp2(fmaf(__uint_as_float(x[e]), a.scale, -ls[c0 + e]) * LOG2E);
                        sum += key <= see[c0 + e] ? v : 0.0f;
                    }
                }
                total += sum;
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctl->acc_empty[acc]));
            if (w.last && key < w.len) a.out[((int64_t)w.s * c.heads + w.h) * a.width + key] = prior + total;
            w = n;
            more = another;
        }
    }
    cta_teardown(waits.abort_flag, ctl->tmem_base, 1);
}

template <int DP> cudaError_t weights(const PagedWeightsArgs &a, cudaStream_t s)
{
    using Sh = WeightsShape<DP>;
    static int sms_of_device[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (sms_of_device[dev] == 0) {
        int n = 0;
        cudaError_t e = cudaFuncSetAttribute(k_paged_weights<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::SMEM);
        if (e == cudaSuccess) e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
        if (e != cudaSuccess) return e;
        sms_of_device[dev] = n;
    }
    WeightsParams p = {};
    p.a = a;
    p.tokens = TILE / a.group;
    p.box = box_rows(a.c);
    WeightsMaps tm = {};
    // a call without tokens has no products
    if (a.c.N > 0 && (!head_map(&tm.q, a.q, a.c.d, a.hq, a.c.N, a.ldq, a.group, p.tokens) || !pool_map(&tm.k, a.c.k, a.q, a.c, p.box)))
        return cudaErrorInvalidValue;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)sms_of_device[dev]); cfg.blockDim = dim3(THREADS); cfg.dynamicSmemBytes = Sh::SMEM; cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, k_paged_weights<DP>, tm, p);
}

}  // namespace

cudaError_t launch_paged_weights(const PagedWeightsArgs &a, cudaStream_t s) { return a.c.d <= 64 ? weights<64>(a, s) : weights<128>(a, s); }

}  // namespace skipffn
