// The softmax weight that every row of a paged cache gets from the new tokens of its sequence, per kv head, bf16:
//
//   weights[s, h, j] = prior + sum over new rows r of the head's group that see j of exp(scale q_r . k_j - lse_r)
//
// The forward's logarithms are given, so one pass over the keys suffices.  Scores are made with the keys on the
// accumulator's rows (tcgen05.mma, 128 keys x up to 128 rows of queries), so a thread of the epilogue has one key and adds
// its exponentials up in a register: no atomics, no shuffles, a fixed order.  Work is a line of units (sequence, head,
// 256 keys), each with a step for every tile of query rows, cut into runs of equal steps, one per CTA, one CTA per SM:
//   warps 0, 2   key tiles of the first and second half of a unit (pages looked up a unit ahead), query tiles
//   warp 1       the two products of a step
//   warp 3       what needs no product: columns past a sequence's rows, sequences without new tokens
//   warps 4..11  two groups, one for each half: exponentials and sums
// Bound by reading the keys for up to about 100 query rows a kv head, by the exponentials (16 a cycle and SM) beyond.  A TMA
// box costs its warp about 64 cycles whatever its size, so pages of 16 rows want the two warps (with units of 128 keys, 48
// conversations took 82 us from one warp, 71 us from two and 58 us from either with pages of 128 rows; with 256 it is 50 us
// for 238 MB at 16 rows a page as at 128).  161 observing tokens of 40 heads take 57 us, a chunk of 2000 tokens over a
// cache of 14 345 rows 518 us.  On the legacy matrix instructions a step of 64 keys x 32 rows
// took 2 us from its copies to its sums however it was cut, with eight warps an SM: 100 us for the batch of 48
// conversations (238 MB), 250 us for 161 observing tokens of 40 heads.
#include "paged_tma.cuh"

namespace skipffn {

namespace {

constexpr int WARPS = 12, THREADS = 32 * WARPS, FIRST = 4, FILL_COLS = 1024, UNIT = 2 * TILE;

struct WeightsParams {
    PagedWeightsArgs a;
    int32_t tokens, box;                     // tokens of a tile of query rows; rows of a TMA box
    int32_t q_slots, k_slots;                // tiles of queries, of each half's keys in shared memory
};
struct alignas(64) WeightsMaps { CUtensorMap q, k; };

template <int DP> struct WeightsShape {
    static constexpr int T_BYTES = tile_bytes<DP>(), SLOTS = DP == 128 ? 6 : 10;       // of keys and of queries
    static constexpr int SMEM = SLOTS * T_BYTES + 2048;
};
struct alignas(8) WeightsCtl {
    uint64_t full[10], empty[10], acc_full[2][2], acc_empty[2][2];      // accumulators of each group
    int64_t scan[WARPS], place[2];
    uint32_t tmem_base;
    volatile int abort_flag;
    volatile uint32_t issued;
};

// Up to 256 keys from j0 on against `live` rows of queries, the tokens from t0 on
struct Step {
    int s, h, j0, t0, live, q0, off, len;    // len: rows that have a weight
    bool first, last, load_q;                // of the unit; other queries than the step before
    __device__ bool half(int g) const { return j0 + g * TILE < len; }
};

// Walks the steps of this CTA's run, the same in every role
struct Line {
    const WeightsParams &p;
    int64_t at, end;                         // first step of the unit, end of the run
    int s, h = 0, b = 0, blocks, steps, tile = 0;
    bool fresh = true, moved = true;         // a new unit, another (sequence, head)
    PagedSeq q;
    __device__ static int blocks_of(const PagedWeightsArgs &a, const PagedSeq &q) { return q.n > 0 ? (min(q.len, a.width) + UNIT - 1) / UNIT : 0; }
    __device__ static int64_t cost_of(const WeightsParams &p, const PagedSeq &q)
    {
        return (int64_t)blocks_of(p.a, q) * p.a.c.heads * ceil_div(q.n, p.tokens);
    }
    __device__ void enter()
    {
        q = paged_seq(p.a.c, s, false);
        blocks = blocks_of(p.a, q);
        steps = ceil_div(q.n, p.tokens);
        h = b = 0;
    }
    // the run's units are those whose first step lies in it
    __device__ Line(const WeightsParams &p_, int64_t begin, int64_t end_, int seq, int64_t before) : p(p_), at(before), end(end_), s(seq)
    {
        if (begin >= end) { at = end; return; }
        enter();
        const int64_t unit = (begin - at + steps - 1) / steps;
        at += unit * steps;
        h = (int)(unit / blocks);
        b = (int)(unit - (int64_t)h * blocks);
        settle();
    }
    __device__ void settle()
    {
        if (b == blocks) { b = 0; ++h; moved = true; }
        if (h == p.a.c.heads) {
            do {
                if (at >= end || s + 1 >= p.a.c.n_seq) { at = end; return; }
                ++s;
                enter();
            } while (blocks == 0);
        }
        tile = max(0, b * UNIT - (q.len - q.n)) / p.tokens;           // tokens before it see none of the keys
    }
    __device__ bool next(Step &w)
    {
        if (at >= end) return false;
        w.s = s; w.h = h; w.j0 = b * UNIT; w.t0 = tile * p.tokens;
        w.live = min(p.tokens, q.n - w.t0) * p.a.group;
        w.q0 = q.q0; w.off = q.len - q.n; w.len = min(q.len, p.a.width);
        w.first = fresh;
        w.last = fresh = ++tile == steps;
        w.load_q = steps > 1 || moved;
        moved = false;
        if (fresh) { ++b; at += steps; settle(); }
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
    const uint32_t ring = smem_u32(smem_raw);                // tiles of queries, of first halves, of second halves
    WeightsCtl *ctl = reinterpret_cast<WeightsCtl *>(smem_raw + SLOTS * T_BYTES);
    const PagedWeightsArgs &a = p.a;
    const PagedView &c = a.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int i = 0; i < SLOTS; ++i) { mbar_init(smem_u32(&ctl->full[i]), 1); mbar_init(smem_u32(&ctl->empty[i]), 1); }
        for (int i = 0; i < 4; ++i) { mbar_init(smem_u32(&ctl->acc_full[i >> 1][i & 1]), 1); mbar_init(smem_u32(&ctl->acc_empty[i >> 1][i & 1]), 4); }
        ctl->abort_flag = 0;
        ctl->issued = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    const int used = a.group * p.tokens;     // rows of a tile that a box fills; the others stay zero
    if (used < TILE) zero_smem(ring, p.q_slots * T_BYTES);
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
    // a place in one of the rings (queries, first halves, second halves): slot and parity
    struct Ring {
        int first, slots, at = 0;
        uint32_t phase = 0;
        __device__ Ring(int f, int n) : first(f), slots(n) {}
        __device__ int slot() const { return first + at; }
        __device__ void next() { if (++at == slots) { at = 0; phase ^= 1; } }
    };
    auto full = [&](int slot) { return smem_u32(&ctl->full[slot]); };
    auto empty = [&](int slot) { return smem_u32(&ctl->empty[slot]); };
    auto queries = [&]() { return Ring(0, p.q_slots); };
    auto keys = [&](int g) { return Ring(p.q_slots + g * p.k_slots, p.k_slots); };
    auto line = [&]() { return Line(p, begin, end, (int)ctl->place[0], ctl->place[1]); };

    if (warp == 0 || warp == 2) {
        const PageBoxes boxes{c, p.box, lane};
        const int g = warp / 2;
        Line walk = line();
        Step w, n;
        Ring q = queries(), k = keys(g);
        uint32_t tiles = 0;
        bool more = walk.next(w);
        PageBox box = {0, -1}, next = box;
        if (more) box = boxes.find(w.s, w.len, w.j0 + g * TILE);
        while (more && ok) {
            const bool another = walk.next(n);
            if (another && n.first) next = boxes.find(n.s, n.len, n.j0 + g * TILE);
            if (w.load_q && g == 0) {
                const int s = q.slot();
                ok = wait_warp<true>(empty(s), q.phase ^ 1, waits, SITE_PRODUCER_EMPTY);
                if (!ok) break;
                if (lane == 0) {
                    mbar_expect_tx(full(s), (uint32_t)(used * DP * 2));
                    load_tile<DP>(ring + s * T_BYTES, &tm.q, w.h * a.group, w.q0 + w.t0, full(s));
                    ctl->issued = ++tiles;
                }
                q.next();
            }
            if (w.first && w.half(g)) {
                boxes.check(box);
                const int s = k.slot();
                ok = wait_warp<true>(empty(s), k.phase ^ 1, waits, SITE_PRODUCER_EMPTY);
                if (!ok) break;
                boxes.load<DP>(ring + s * T_BYTES, &tm.k, full(s), box, w.h);
                k.next();
                if (lane == 0 && g == 0) ctl->issued = ++tiles;
            }
            if (another && n.first) box = next;
            w = n;
            more = another;
        }
    } else if (warp == 1) {
        const uint32_t on = elect_one();     // the warp walks as one, one thread issues
        const uint32_t desc = desc_rows(ring);
        Line walk = line();
        Step w, n;
        Ring q = queries(), k[2] = {keys(0), keys(1)};
        int qs = 0, ks[2] = {0, 0};
        uint32_t count[2] = {0, 0};
        bool more = walk.next(w);
        while (more && ok) {
            const bool another = walk.next(n);
            if (w.load_q) {
                qs = uniform(q.slot());
                ok = wait_warp<true>(full(qs), q.phase, waits, SITE_MMA_FULL);
                q.next();
            }
            const uint32_t idesc = idesc_rows(uniform(mma_cols(w.live)));
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                if (!w.half(g)) continue;
                if (w.first) {
                    ks[g] = uniform(k[g].slot());
                    ok = ok && wait_warp<true>(full(ks[g]), k[g].phase, waits, SITE_MMA_FULL);
                    k[g].next();
                }
                const uint32_t acc = count[g] & 1;
                ok = ok && wait_warp<true>(smem_u32(&ctl->acc_empty[g][acc]), (count[g] >> 1 & 1) ^ 1, waits, SITE_MMA_TMEM_EMPTY);
                if (!ok) break;
                ++count[g];
                tc_fence_after();
                mma_rows_rows<DP>(on, tmem + (2 * g + acc) * TILE, desc + ks[g] * (T_BYTES >> 4), desc + qs * (T_BYTES >> 4), idesc);
                umma_commit_if(on, smem_u32(&ctl->acc_full[g][acc]));
                if (w.last) umma_commit_if(on, empty(ks[g]));
            }
            if (!ok) break;
            if (another && n.load_q) umma_commit_if(on, empty(qs));
            w = n;
            more = another;
        }
    } else if (warp == 3) {
        const int chunks = ceil_div(a.width, FILL_COLS);
        for (int64_t i = blockIdx.x; i < (int64_t)c.n_seq * c.heads * chunks; i += gridDim.x) {
            const int64_t pair = i / chunks;
            const int j0 = (int)(i - pair * chunks) * FILL_COLS, j1 = min(a.width, j0 + FILL_COLS);
            const PagedSeq q = paged_seq(c, (int)(pair / c.heads), false);
            const int from = q.n > 0 ? max(j0, q.len) : j0;
            for (int j = from + lane; j < j1; j += 32) {
                const int64_t at = pair * a.width + j;
                a.out[at] = j < q.len && a.prior ? a.prior[at] : 0.0f;
            }
        }
    } else {
        const int g = (warp - FIRST) >> 2, mine = g * TILE + (warp & 3) * 32 + lane;        // group, key of the unit
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        Line walk = line();
        Step w, n;
        auto next = [&](Step &x) {           // the steps in which this group has keys
            while (walk.next(x))
                if (x.half(g)) return true;
            return false;
        };
        // the lane looks after rows lane, lane + 32, .. of the queries: their tokens and heads in a tile
        int row_t[4], row_h[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) { row_t[i] = (lane + 32 * i) / a.group; row_h[i] = lane + 32 * i - row_t[i] * a.group; }
        // a group may pass steps over: the queries are others when sequence, head or tile are
        int held_s = -1, held_h = -1, held_t = -1;
        auto changes = [&](const Step &x) { return x.s != held_s || x.h != held_h || x.t0 != held_t; };
        float ahead[4], total = 0.0f, prior = 0.0f, prior_ahead = 0.0f, *ls = lses[warp - FIRST];
        int *see = sees[warp - FIRST];
        bool odd = false;                    // the tile has rows that give nothing
        uint32_t count = 0;
        auto look_up = [&](const Step &x) {
            const float *src = a.lse + (int64_t)(x.q0 + x.t0) * a.hq + x.h * a.group;
#pragma unroll
            for (int i = 0; i < 4; ++i) ahead[i] = lane + 32 * i < x.live ? src[(int64_t)row_t[i] * a.hq + row_h[i]] : -INFINITY;
        };
        auto prior_of = [&](const Step &x) {
            return a.prior && x.j0 + mine < x.len ? a.prior[((int64_t)x.s * c.heads + x.h) * a.width + x.j0 + mine] : 0.0f;
        };
        bool more = next(w);
        if (more) { look_up(w); prior_ahead = prior_of(w); }
        while (more && ok) {
            if (changes(w)) {
                bool none = false;
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int r = lane + 32 * i;
                    const bool empty = ahead[i] == -INFINITY;
                    ls[r] = empty ? 0.0f : ahead[i];
                    see[r] = empty ? -1 : w.off + w.t0 + row_t[i];
                    none |= empty && r < w.live;
                }
                odd = __any_sync(0xffffffffu, none);
                __syncwarp();
                held_s = w.s; held_h = w.h; held_t = w.t0;
            }
            if (w.first) {
                total = 0.0f;
                prior = prior_ahead;
            }
            // what the group's next step needs from memory arrives during this one
            const bool another = next(n);
            if (another && changes(n)) look_up(n);
            if (another && n.first) prior_ahead = prior_of(n);
            const uint32_t acc = count & 1;
            ok = wait_warp<true>(smem_u32(&ctl->acc_full[g][acc]), count >> 1 & 1, waits, SITE_EPI_TMEM_FULL);
            if (!ok) break;
            ++count;
            tc_fence_after();
            // every row of the tile sees every key, and gives something
            const bool plain = w.j0 + (g + 1) * TILE - 1 <= w.off + w.t0 && !odd;
            const int key = w.j0 + mine;
            const uint32_t src = tmem + lanes + (2 * g + acc) * TILE;
            // the difference first: it is small where the weight counts, so its rounding is too
            auto weight = [&](uint32_t x, float l) { return fast_exp2(fmaf(__uint_as_float(x), a.scale, -l) * LOG2E); };
            auto add_plain = [&](const uint32_t (&x)[32], int c0) {
                float sum[2] = {0.0f, 0.0f};
#pragma unroll
                for (int e = 0; e < 32; e += 4) {
                    float l[4];
                    load4(ls + c0 + e, l);
#pragma unroll
                    for (int y = 0; y < 4; ++y) sum[y & 1] += weight(x[e + y], l[y]);
                }
                total += sum[0] + sum[1];
            };
            int c0 = 0;
            if (plain) {                     // 64 columns a turn, the second half arrives while the first is worked on
                uint32_t x[32], y[32];
                if (w.live >= 32) tmem_ld32(src, x);
#pragma unroll 1
                for (; c0 + 64 <= w.live; c0 += 64) {
                    tmem_ld_wait(x);
                    tmem_ld32(src + c0 + 32, y);
                    add_plain(x, c0);
                    tmem_ld_wait(y);
                    if (c0 + 96 <= w.live) tmem_ld32(src + c0 + 64, x);
                    add_plain(y, c0 + 32);
                }
                if (c0 + 32 <= w.live) {
                    tmem_ld_wait(x);
                    add_plain(x, c0);
                    c0 += 32;
                }
            }
#pragma unroll 1
            for (; c0 < w.live; c0 += 16) {  // masks, and what is left
                uint32_t x[16];
                tmem_ld16(src + c0, x);
                tmem_ld_wait(x);
                float sum = 0.0f;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float v = weight(x[e], ls[c0 + e]);
                    sum += key <= see[c0 + e] ? v : 0.0f;
                }
                total += sum;
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctl->acc_empty[g][acc]));
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
    // queries that stay (one tile a head) need a place to change them ahead; a chunk's come with every step
    p.q_slots = a.c.max_new > p.tokens ? Sh::SLOTS - 2 : 2;
    p.k_slots = (Sh::SLOTS - p.q_slots) / 2;
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
