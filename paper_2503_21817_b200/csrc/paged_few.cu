// Attention over a paged cache for sequences of few rows (new tokens x query heads of a kv head; 16 in bf16, 8 in fp32): the
// token that is being answered, a few proposed ones.
//
//   s_rj = scale q_r . k_j,  out_r = sum_j softmax(s_r)_j v_j,  one pass over the keys with a running maximum and sum.
//
// Bound by reading the cache once: 512 bytes a key and kv head at head_dim 128 for 4 x rows x 128 flops, so the legacy
// matrix instructions (mma.sync, whose accumulators are registers and need no second kernel role) are far from their
// limit.  The keys of all sequences and heads, 16 to a unit, are one line that is cut into equal runs, one per WARP (eight
// an SM): ragged batches and one long sequence load every SM alike.  A warp brings its units through its own ring of
// asynchronous 16-byte copies and waits for no other: what the end of one tile costs (its sums written, the next queries
// fetched) does not hold up the rest of the SM.  Rows come from their pages eight at a time (a page holds whole groups of
// eight).  Measured, 48 conversations of 37 to 8877 rows, 32 / 8 heads, head_dim 128: 80 us (5.8 TB/s while it streams, 5.5
// over all); one of 130 001 rows 98 us.  Before, four warps shared a unit of 64 keys and merged their sums at a tile's end:
// 105 us.  Two or four warps with 16 rows each behind one ring were slower than the tensor-core kernel (32 rows 144 us
// against 128), which has everything beyond 16 rows.
// fp32 has the same walk with plain FMA, for 2, 4 or 8 rows by the most that a sequence of the call may have: single tokens
// of 24 conversations, 32 / 8 heads, head_dim 128 87 us (487 MB, 5.6 TB/s; with rows for 8 118 us, as 5 to 8 rows take; the
// kernel of 16 rows a tile 320 us), 16 / 16 heads 158 us, 40 / 40 heads of 64 columns over 13 336 rows 58 us.  Sixteen rows would
// need more registers for their queries than a thread has: the tiled kernel has them (326 us).
#include <algorithm>
#include "paged.cuh"
#include "paged_mma.cuh"

namespace skipffn {

namespace {

constexpr int WARPS = 8, THREADS = 32 * WARPS;
constexpr float LOG2E = 1.4426950408889634f;

// KEYS keys of DP columns and their values, the unit that a warp works on (8 KB, 4 KB of up to 64 columns); ROWS: rows of a
// sequence at most; PER: elements of 16 bytes.
template <typename T, int DP, int R> struct FewShape {
    static constexpr int ROWS = R, PER = 16 / (int)sizeof(T), KEYS = 2 * PER;
    static constexpr int TILE = KEYS * DP * (int)sizeof(T), STAGE = 2 * TILE;                 // keys, then values
    static constexpr int STAGES = DP == 128 ? 3 : 6;
    static constexpr int SMEM = WARPS * STAGES * STAGE;
    // where chunk ch of row r stands: matrix loads want eight rows on different banks, plain ones read a row's chunks together
    __device__ static uint32_t at(int r, int ch)
    {
        if constexpr (sizeof(T) == 2) return chunk_at<DP>(r, ch);
        else return (r * (DP / PER) + ch) * 16;
    }
    // Blocks of keys of a sequence, of one head; a sequence without keys has one, which writes its empty rows.
    __device__ static int blocks(const PagedSeq &q, int group)
    {
        return q.n > 0 && q.n * group <= ROWS ? max(1, (q.len + KEYS - 1) / KEYS) : 0;
    }
};

// A place in the line of units: block b of head h of sequence s
template <typename Sh> struct Place {
    int s, h, b, blocks;
    PagedSeq q;
    __device__ void enter(const PagedView &c, int group, int seq)
    {
        s = seq;
        q = paged_seq(c, s, false);
        blocks = Sh::blocks(q, group);
    }
    // to the next block; the units that lie between.  The sequences end where the line does.
    __device__ int step(const PagedView &c, int group)
    {
        if (++b < blocks) return 1;
        b = 0;
        if (++h == c.heads) {
            h = 0;
            do {
                if (s + 1 >= c.n_seq) break;
                enter(c, group, s + 1);
            } while (blocks == 0);
        }
        return 1 + PG_TILE_COST;
    }
};

// The rows of a tile on the matrix instructions: a thread has rows r0 and r0 + 8
template <int DP> struct MmaRows {
    using Sh = FewShape<bf16, DP, PG_FEW_ROWS>;
    static constexpr int KEYS = Sh::KEYS;
    uint32_t qf[DP / 16][4];
    float o[DP / 8][4], m[2], l[2];
    int limit[2] = {0, 0};

    __device__ void begin(const PagedAttnArgs &a, const Place<Sh> &at, int lane)
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = (lane >> 2) + 8 * i;
            const bool live = r < at.q.n * a.group;
            limit[i] = live ? at.q.len - at.q.n + r / a.group + 1 : 0x7fffffff;   // a dead row's sums go nowhere
            const uint32_t *src = live ? (const uint32_t *)((const bf16 *)a.q + (int64_t)(at.q.q0 + r / a.group) * a.ldq +
                                                            (int64_t)(at.h * a.group + r % a.group) * a.c.d) : nullptr;
#pragma unroll
            for (int k = 0; k < DP / 16; ++k)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int col = 16 * k + 8 * x + 2 * (lane & 3);
                    qf[k][2 * x + i] = src && col < a.c.d ? src[col / 2] : 0u;
                }
            m[i] = -INFINITY;
            l[i] = 0.0f;
        }
#pragma unroll
        for (int n = 0; n < DP / 8; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[n][e] = 0.0f;
    }

    // the unit of keys j0 .. in shared memory
    __device__ void unit(uint32_t kt, uint32_t vt, int j0, float c2, int lane)
    {
        float s[2][4] = {}, t2[2][4] = {};   // two chains a tile of eight keys
#pragma unroll
        for (int k = 0; k < DP / 16; ++k) {
            uint32_t b[4];
            ldsm_x4(kt + Sh::at((lane >> 4) * 8 + (lane & 7), 2 * k + ((lane >> 3) & 1)), b);
            mma_16x8(k & 1 ? t2[0] : s[0], qf[k], b[0], b[1]);
            mma_16x8(k & 1 ? t2[1] : s[1], qf[k], b[2], b[3]);
        }
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int e = 0; e < 4; ++e) s[n][e] += t2[n][e];
        // keys past a row's own
        if (j0 + KEYS > min(limit[0], limit[1])) {
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (j0 + 8 * n + 2 * (lane & 3) + (e & 1) >= limit[e >> 1]) s[n][e] = -INFINITY;
        }
        float f[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float t = fmaxf(fmaxf(s[0][2 * i], s[0][2 * i + 1]), fmaxf(s[1][2 * i], s[1][2 * i + 1]));
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 1));
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 2));
            t = fmaxf(t, m[i]);
            f[i] = t == m[i] ? 1.0f : fast_exp2((m[i] - t) * c2);
            m[i] = t;
            // a row that has met nothing but minus infinity has p = 2^(-inf) = 0 so far, not 2^(-inf + inf)
            const float shift = t == -INFINITY ? 0.0f : -t * c2;
            float sum = 0.0f;
#pragma unroll
            for (int n = 0; n < 2; ++n)
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
        // p as operand of the second product: rounded to bf16, at most 2^-8 of a term; the sum l takes it unrounded
        const uint32_t p[4] = {pack_bf16(s[0][0], s[0][1]), pack_bf16(s[0][2], s[0][3]), pack_bf16(s[1][0], s[1][1]), pack_bf16(s[1][2], s[1][3])};
#pragma unroll
        for (int n = 0; n < DP / 16; ++n) {
            uint32_t b[4];
            ldsm_x4_trans(vt + Sh::at(lane & 15, 2 * n + (lane >> 4)), b[0], b[1], b[2], b[3]);
            mma_16x8(o[2 * n], p, b[0], b[1]);
            mma_16x8(o[2 * n + 1], p, b[2], b[3]);
        }
    }

    // results of a tile that was `whole`ly this run's, else its sums to the slot's rows from `slot` on
    __device__ void end(const PagedAttnArgs &a, const Place<Sh> &at, bool whole, int64_t slot, int lane)
    {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
            l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
            const int r = (lane >> 2) + 8 * i;
            if (r >= at.q.n * a.group) continue;
            const int64_t token = at.q.q0 + r / a.group;
            const int head = at.h * a.group + r % a.group;
            if (whole) {
                bf16 *dst = (bf16 *)a.out + token * a.ldo + (int64_t)head * a.c.d;
                const float inv = 1.0f / l[i];
                const bool none = met_nothing(m[i], l[i]);
#pragma unroll
                for (int n = 0; n < DP / 8; ++n) {
                    const int col = 8 * n + 2 * (lane & 3);
                    if (col < a.c.d) *reinterpret_cast<uint32_t *>(dst + col) = none ? 0u : pack_bf16(o[n][2 * i] * inv, o[n][2 * i + 1] * inv);
                }
                if ((lane & 3) == 0) a.lse[token * a.hq + head] = none ? -INFINITY : fmaf(m[i], a.scale, logf(l[i]));
            } else {
#pragma unroll
                for (int n = 0; n < DP / 8; ++n)
                    *reinterpret_cast<float2 *>(a.part + (slot + r) * DP + 8 * n + 2 * (lane & 3)) = make_float2(o[n][2 * i], o[n][2 * i + 1]);
                if ((lane & 3) == 0) a.part_ml[slot + r] = make_float2(m[i], l[i]);
            }
        }
    }
};

// The rows of a tile in fp32 with plain FMA.  Scores: eight lanes a key, four keys at a time, a lane with every eighth chunk of
// the columns; sums: a lane has one chunk of the columns (of up to 64: half of the keys too).  Rows are registers, and a row that
// is not there costs as much as one that is: hence R = 2, 4, 8.
template <int DP, int R> struct FmaRows {
    using Sh = FewShape<float, DP, R>;
    static constexpr int KEYS = Sh::KEYS, CHUNKS = DP / 4, N = CHUNKS / 8, HALVES = 32 / CHUNKS, PASSES = KEYS / 4;
    uint64_t q[R][N][2], o[R][2];
    float m[R], l[R];
    int limit[R];

    __device__ static void load(uint32_t at, uint64_t (&v)[2]) { asm volatile("ld.shared.v2.b64 {%0, %1}, [%2];" : "=l"(v[0]), "=l"(v[1]) : "r"(at) : "memory"); }

    __device__ void begin(const PagedAttnArgs &a, const Place<Sh> &at, int lane)
    {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool live = r < at.q.n * a.group;
            limit[r] = live ? at.q.len - at.q.n + r / a.group + 1 : 0x7fffffff;   // a dead row's sums go nowhere
            const float *src = (const float *)a.q + (int64_t)(at.q.q0 + r / a.group) * a.ldq + (int64_t)(at.h * a.group + r % a.group) * a.c.d;
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const int col = 4 * (lane % 8 + 8 * i);
                const ulonglong2 v = live && col < a.c.d ? *reinterpret_cast<const ulonglong2 *>(src + col) : make_ulonglong2(0, 0);
                q[r][i][0] = v.x;
                q[r][i][1] = v.y;
            }
            o[r][0] = o[r][1] = 0;
            m[r] = -INFINITY;
            l[r] = 0.0f;
        }
    }

    __device__ void unit(uint32_t kt, uint32_t vt, int j0, float c2, int lane)
    {
        float s[PASSES][R];                  // of key 4 x pass + lane / 8
#pragma unroll
        for (int x = 0; x < PASSES; ++x) {
            const int key = 4 * x + lane / 8;
            uint64_t t[R] = {};
#pragma unroll
            for (int i = 0; i < N; ++i) {
                uint64_t k[2];
                load(kt + Sh::at(key, lane % 8 + 8 * i), k);
#pragma unroll
                for (int r = 0; r < R; ++r) t[r] = fma2(q[r][i][1], k[1], fma2(q[r][i][0], k[0], t[r]));
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float lo, hi;
                unpair2(t[r], lo, hi);
                lo += hi;
#pragma unroll
                for (int d = 1; d < 8; d <<= 1) lo += __shfl_xor_sync(0xffffffffu, lo, d);
                s[x][r] = j0 + key < limit[r] ? lo : -INFINITY;
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float t = m[r];
#pragma unroll
            for (int x = 0; x < PASSES; ++x) t = fmaxf(t, s[x][r]);
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 8));
            t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, 16));
            const float f = t == m[r] ? 1.0f : exp2f((m[r] - t) * c2);
            m[r] = t;
            l[r] *= f;                       // of this lane's keys
            o[r][0] = mul2(o[r][0], pair2(f, f));
            o[r][1] = mul2(o[r][1], pair2(f, f));
            // a row that has met nothing but minus infinity has p = 2^(-inf) = 0 so far, not 2^(-inf + inf)
            const float shift = t == -INFINITY ? 0.0f : t;
#pragma unroll
            for (int x = 0; x < PASSES; ++x) {
                s[x][r] = exp2f((s[x][r] - shift) * c2);
                l[r] += s[x][r];
            }
        }
        const int half = lane / CHUNKS;
#pragma unroll
        for (int i = 0; i < KEYS / HALVES; ++i) {
            const int key = HALVES * i + half;
            uint64_t v[2];
            load(vt + Sh::at(key, lane % CHUNKS), v);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float p = __shfl_sync(0xffffffffu, s[HALVES * i / 4][r], key % 4 * 8);
                const uint64_t pp = pair2(p, p);
                o[r][0] = fma2(pp, v[0], o[r][0]);
                o[r][1] = fma2(pp, v[1], o[r][1]);
            }
        }
    }

    __device__ void end(const PagedAttnArgs &a, const Place<Sh> &at, bool whole, int64_t slot, int lane)
    {
        const int col = 4 * (lane % CHUNKS);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (r >= at.q.n * a.group) break;                     // the same in every lane
            l[r] += __shfl_xor_sync(0xffffffffu, l[r], 8);
            l[r] += __shfl_xor_sync(0xffffffffu, l[r], 16);
            float v[4];
            unpair2(o[r][0], v[0], v[1]);
            unpair2(o[r][1], v[2], v[3]);
            if (HALVES == 2)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += __shfl_xor_sync(0xffffffffu, v[e], 16);
            const int64_t token = at.q.q0 + r / a.group;
            const int head = at.h * a.group + r % a.group;
            if (whole) {
                const bool none = met_nothing(m[r], l[r]);
                const float inv = 1.0f / l[r];
                if (lane < CHUNKS && col < a.c.d)
                    *reinterpret_cast<float4 *>((float *)a.out + token * a.ldo + (int64_t)head * a.c.d + col) =
                        none ? make_float4(0.0f, 0.0f, 0.0f, 0.0f) : make_float4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
                if (lane == 0) a.lse[token * a.hq + head] = none ? -INFINITY : fmaf(m[r], a.scale, logf(l[r]));
            } else {
                if (lane < CHUNKS) *reinterpret_cast<float4 *>(a.part + (slot + r) * DP + col) = make_float4(v[0], v[1], v[2], v[3]);
                if (lane == 0) a.part_ml[slot + r] = make_float2(m[r], l[r]);
            }
        }
    }
};
template <typename T, int DP, int R>
__global__ void __launch_bounds__(THREADS, 1) k_paged_few(const PagedAttnArgs a)
{
    using Sh = FewShape<T, DP, R>;
    using Rows = std::conditional_t<sizeof(T) == 2, MmaRows<DP>, FmaRows<DP, R>>;
    constexpr int CHUNKS = DP / Sh::PER, STEP = 32 / CHUNKS, STAGES = Sh::STAGES, KEYS = Sh::KEYS, ROWS = Sh::ROWS;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ int64_t scan[WARPS], place_in[WARPS];
    __shared__ int place_seq[WARPS];
    const PagedView &c = a.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, ctas = gridDim.x;
    pdl_enter();

    // ---- where the runs lie: sums of units over the sequences.  Run r is warp r / CTAs of CTA r % CTAs, so that a few runs are
    // spread over the SMs.
    auto units_of = [&](int s, bool report) {
        const int b = s < c.n_seq ? Sh::blocks(paged_seq(c, s, report), a.group) : 0;
        return b ? (int64_t)(b + PG_TILE_COST) * c.heads : 0;
    };
    auto block_sum = [&](int64_t v) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        __syncthreads();
        if (lane == 0) scan[warp] = v;
        __syncthreads();
        int64_t t = 0;
#pragma unroll
        for (int i = 0; i < WARPS; ++i) t += scan[i];
        return t;
    };
    int64_t mine = 0;
    for (int s = tid; s < c.n_seq; s += THREADS) mine += units_of(s, blockIdx.x == 0);
    const Runs runs(block_sum(mine), ctas * WARPS);
    if (runs.units == 0) return;
    int64_t before = 0;
    const int64_t last_begin = min(runs.begin((WARPS - 1) * ctas + (int)blockIdx.x), runs.units - 1);
    for (int s0 = 0; s0 < c.n_seq; s0 += THREADS) {
        const int64_t v = units_of(s0 + tid, false);
        int64_t x = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
            if (lane >= o) x += y;
        }
        const int64_t total = block_sum(v);
        int64_t lo = before + x - v;
        for (int i = 0; i < warp; ++i) lo += scan[i];
        for (int w = 0; w < WARPS; ++w) {
            const int64_t u = runs.begin(w * ctas + (int)blockIdx.x);
            if (lo <= u && u < lo + v) { place_seq[w] = s0 + tid; place_in[w] = u - lo; }
        }
        before += total;
        if (before > last_begin) break;      // the same in every thread
    }
    __syncthreads();
    const int run = warp * ctas + (int)blockIdx.x;
    const int64_t begin = runs.begin(run), end = runs.begin(run + 1);
    if (run >= runs.n) return;               // no barrier of the CTA below
    Place<Sh> at;
    at.enter(c, a.group, place_seq[warp]);
    const int seg = at.blocks + PG_TILE_COST;
    at.h = (int)(place_in[warp] / seg);
    at.b = (int)(place_in[warp] - (int64_t)at.h * seg) - PG_TILE_COST;
    int64_t u = begin;                       // of the next block
    if (at.b < 0) { u -= at.b; at.b = 0; }
    if (u >= end) return;                    // the run holds nothing but a tile's beginning
    int64_t item = u - at.b;                 // unit of the tile's first block

    // ---- the ring.  A unit's pages are looked up when the one before it is issued: lanes 0 and 1 keep the entries for its
    // rows 0 .. 7 and 8 .. 15 (fp32 has units of 8), which are touched a unit later.
    const uint32_t ring = smem_u32(smem) + warp * STAGES * Sh::STAGE;
    const int chunk = lane % CHUNKS, row0 = lane / CHUNKS;
    Place<Sh> ahead = at;
    int64_t issued = u;
    uint32_t fill = ring, use = ring;
    int entry = 0, inside = -1;              // page number, row inside the page (-1: no such row)
    auto find = [&]() {
        const int r = ahead.b * KEYS + 8 * lane;
        inside = -1;
        if (lane < KEYS / 8 && r < ahead.q.len) {
            const int p = div_by(r, c.page);
            entry = c.table[(int64_t)ahead.s * c.table_stride + p];
            inside = r - p * (int)c.page.d;
        }
    };
    auto issue = [&]() {
        if (issued < end) {
            const int left = ahead.q.len - ahead.b * KEYS;
            int64_t base = -1;
            if (inside >= 0) {
                if (entry < 0 || entry >= c.n_pages) paged_report(c, SITE_PAGED_PAGE);
                else base = entry * c.page_stride + inside * c.row_stride + ahead.h * c.head_stride;
            }
            const int64_t g[2] = {__shfl_sync(0xffffffffu, base, 0), __shfl_sync(0xffffffffu, base, 1)};
#pragma unroll
            for (int i = 0; i < KEYS / STEP; ++i) {
                const int r = row0 + i * STEP;
                const int64_t b = r < 8 ? g[0] : g[1];
                const bool on = b >= 0 && r < left && chunk * Sh::PER < c.d;
                const int64_t off = on ? b + (r & 7) * c.row_stride + chunk * 16 : 0;
                const uint32_t to = fill + Sh::at(r, chunk);
                copy16(to, c.k + off, on);
                copy16(to + Sh::TILE, c.v + off, on);
            }
            fill = fill == ring + (STAGES - 1) * Sh::STAGE ? ring : fill + Sh::STAGE;
            issued += ahead.step(c, a.group);
            if (issued < end) find();
        }
        copy_commit();
    };
    find();
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i) issue();

    // ---- arithmetic
    Rows rows;
    const float c2 = a.scale * LOG2E;
    for (bool fresh = true; u < end;) {
        if (fresh) {                         // a new tile: its queries
            fresh = false;
            item = u - at.b;
            rows.begin(a, at, lane);
        }
        copy_wait<STAGES - 2>();
        __syncwarp();                        // the unit is there for every lane, and the slot refilled next is free
        issue();
        const uint32_t kt = use, vt = use + Sh::TILE;
        use = use == ring + (STAGES - 1) * Sh::STAGE ? ring : use + Sh::STAGE;
        rows.unit(kt, vt, at.b * KEYS, c2, lane);
        if (u + 1 < end && at.b + 1 < at.blocks) { ++at.b; ++u; continue; }

        // ---- the end of this run's part of the tile
        const int64_t last = item + at.blocks;
        const bool whole = item >= begin && last <= end;
        rows.end(a, at, whole, (int64_t)(2 * run + (item >= begin ? 1 : 0)) * ROWS, lane);
        if (item >= begin && lane == 0) {    // the run that begins a tile says how many pieces it has
            PagedCut cut = {};
            cut.q0 = at.q.q0; cut.rows = at.q.n * a.group; cut.h = at.h; cut.first = run;
            cut.pieces = whole ? 0 : runs.of(last - 1) - run + 1;
            a.cuts[(int64_t)at.s * c.heads + at.h] = cut;
        }
        u += at.step(c, a.group);
        fresh = true;
    }
    copy_wait<0>();
}

template <typename T, int DP, int R> cudaError_t few(const PagedAttnArgs &a, cudaStream_t s)
{
    using Sh = FewShape<T, DP, R>;
    static int sms_of_device[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (sms_of_device[dev] == 0) {
        int n = 0;
        cudaError_t e = cudaFuncSetAttribute(k_paged_few<T, DP, R>, cudaFuncAttributeMaxDynamicSharedMemorySize, Sh::SMEM);
        if (e == cudaSuccess) e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
        if (e != cudaSuccess) return e;
        sms_of_device[dev] = n < PG_FEW_SMS ? n : PG_FEW_SMS;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)sms_of_device[dev]); cfg.blockDim = dim3(THREADS); cfg.dynamicSmemBytes = Sh::SMEM; cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, k_paged_few<T, DP, R>, a);
    return e != cudaSuccess ? e : launch_paged_join_few(a, R, DP, s);
}

}  // namespace

cudaError_t launch_paged_few(const PagedAttnArgs &a, cudaStream_t s)
{
    if (a.dtype == SKIPFFN_BF16) return a.c.d <= 64 ? few<bf16, 64, PG_FEW_ROWS>(a, s) : few<bf16, 128, PG_FEW_ROWS>(a, s);
    const int64_t most = std::min<int64_t>(a.c.max_new, a.c.N) * a.group;
    if (most <= 2) return a.c.d <= 64 ? few<float, 64, 2>(a, s) : few<float, 128, 2>(a, s);
    if (most <= 4) return a.c.d <= 64 ? few<float, 64, 4>(a, s) : few<float, 128, 4>(a, s);
    return a.c.d <= 64 ? few<float, 64, PG_FEW_ROWS_FP32>(a, s) : few<float, 128, PG_FEW_ROWS_FP32>(a, s);
}

}  // namespace skipffn
