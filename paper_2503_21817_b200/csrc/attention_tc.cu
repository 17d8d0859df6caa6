// Packed attention on the tensor cores (bf16, sm_100a): forward, query gradient, key / value gradient.
//
// All three are persistent (one CTA per SM) and warp-specialised: one lane issues the TMA loads, one warp the
// tcgen05 MMAs, 8 or 16 warps do the arithmetic between two products with scores in tensor memory, one warp
// zeroes what a load brought from behind a sequence's end.  The grouped heads of a key / value head are rows of
// the same 128-row tile, so K and V are read once for all of them and the gradient of a shared head is a sum over
// tile rows: no atomics, equal calls give equal bits.  The gradients take two kernels and seven products where
// one with atomic adds into dQ would take five; that buys a fixed order and no fp32 dQ buffer to clear and convert.
//
// Measured (B200, d = 128, 32 / 8 heads, causal; floor = flops at 1662 TFLOP/s; calls through the Python entry point on
// changing inputs, in brackets replays of a captured graph on the same ones):
//   forward   1 x 16381 tokens  2.02 ms (1.09 PFLOP/s, floor 1.32 ms; at the 1000 W cap, SM clock 1.6 GHz)
//             8 x 616 tokens    47 us   [41] (floor 15.5 us)
//   backward  16 documents, 26 k tokens  1.92 ms [1.80] for 1.06 TFLOP (floor 0.64 ms; at the power cap)
//             8 x 616 tokens    167 us  [144, row statistics 16 of it]
// What bounds them now: the round trips between a product and its arithmetic (forward: 3500 cycles per block and pair of
// tiles for 2048 cycles of products; dK / dV: 3300 for 2048), and the power limit on long sequences.
#include "attention.cuh"
#include "ptx.cuh"

namespace skipffn {

namespace {

constexpr int TILE = 128;                    // rows of a row tile = keys of a key tile
constexpr int AT_TMEM_COLS = 512;            // all of it, so the allocation starts at address 0
constexpr uint32_t tmem = 0;
// Warps of a CTA: TMA, MMA, tail cleaner, an idle one, then ARITH arithmetic warps.  At launch every thread has
// the same number of registers; the four service warps give some of theirs to the arithmetic warps.
//   forward : 8 (a row per thread)       384 x 168 = 128 x 88 + 256 x 208
//   backward: 16 (a quarter of a row) 640 x  96
template <int ARITH> struct Warps {
    static constexpr int THREADS = 32 * (ARITH + 4), TMA = 0, MMA = 1, TAIL = 2, FIRST = 4, COUNT = ARITH;   // FIRST of COUNT arithmetic warps
    static constexpr int REGS_SERVICE = ARITH == 8 ? 88 : 96, REGS_ARITH = ARITH == 8 ? 208 : 96;
};
using FwdWarps = Warps<8>;
using BwdWarps = Warps<16>;
constexpr float LOG2E = 1.4426950408889634f;
template <int N> __device__ __forceinline__ void regs_up() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ __forceinline__ void regs_down() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity)
{
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// Bounded waits, inlined: a kernel that moves registers between its warps cannot call functions.  A wait that runs
// out sets the CTA's abort flag and the status word; every other wait of the CTA then gives up as well.
// A warp may have nothing to do for most of the kernel (the tail warp until an item has a tail, the second row tile's
// softmax warps until an item has a second tile), so a warp's limit counts from the last tile that the TMA lane
// issued: it runs out only when the CTA stands still.  The lane itself stands still within a few tiles of whatever it
// waits for, and the tiles are finite, so every wait ends.
struct Waits { volatile int *abort_flag; volatile uint32_t *issued; int32_t *status; uint32_t limit_ns; };
__device__ __forceinline__ void expire(const Waits &w, int site)
{
    *w.abort_flag = 1;
    if (atomicCAS(&w.status[ST_STATUS], 0, (int)SKIPFFN_ETIMEOUT) == 0) w.status[ST_SITE] = site;
}
// of a single lane (the TMA issuer)
__device__ __forceinline__ bool wait_lane(uint32_t bar, uint32_t parity, const Waits &w, int site)
{
    if (mbar_test(bar, parity)) return true;
    const unsigned long long t0 = globaltimer_ns();
    for (uint32_t it = 1;; ++it) {
        if (mbar_test(bar, parity)) return true;
        if ((it & 0x3ff) == 0) {
            if (*w.abort_flag) return false;
            if (globaltimer_ns() - t0 > w.limit_ns) { expire(w, site); return false; }
        }
    }
}
// of a whole warp.  Every lane polls and a vote decides, so the answer is the same in every lane, and the warp is
// together, when whole-warp instructions follow (tcgen05.ld / st, votes, shuffles, the MMA warp's uniform registers):
// lane by lane, one lane could find the barrier complete and another its time up.  A form in which one lane polled for the
// others ended in an illegal access.  SPIN (the warps on the critical path) polls; the others let the hardware park
// the warp.
template <bool SPIN>
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, const Waits &w, int site)
{
    auto probe = [&] { return __all_sync(0xffffffffu, SPIN ? mbar_test(bar, parity) : mbar_try_wait(bar, parity)); };
    if (__builtin_expect(probe(), 1)) return true;
    unsigned long long t0 = globaltimer_ns();
    uint32_t seen = *w.issued;
    for (uint32_t it = 1;; ++it) {
        if (probe()) return true;
        if ((it & (SPIN ? 0x3ff : 0xf)) == 0) {
            const unsigned long long now = globaltimer_ns();
            if (*w.issued != seen) { seen = *w.issued; t0 = now; }
            const bool late = now - t0 > w.limit_ns;
            if (__any_sync(0xffffffffu, late || *w.abort_flag)) {
                if (late) expire(w, site);
                return false;
            }
        }
    }
}

__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

struct AtParams {
    const int4 *items;
    int32_t n_items;                         // list entries x kv heads
    int32_t hq, hk, group, tokens, d, causal;
    float scale, c2;                         // c2 = scale * log2 e
    int64_t ld0, ld1;                        // token strides of the outputs
    bf16 *out0, *out1;
    float *lse;
    float2 *row_stats;
    int32_t *status;
    uint32_t wait_ns;                        // limit of a wait
    uint32_t lose;                           // bytes that key tiles announce and that never come (failure path)
    int32_t wide;                            // dQ: every 16 columns of a row start on 32 bytes
};
struct alignas(64) AtMaps { CUtensorMap q, k, v, g; };

template <int DP> constexpr int tile_bytes() { return TILE * DP * 2; }

// Work items are sorted by falling work; CTA b takes items b, 2 grid - 1 - b, 2 grid + b, ... (the order of a
// round is reversed every other time), which evens out the sums.  The entry of the next item is fetched when
// the current one is taken.  WARP: used by a whole warp, whose copies are made uniform for the compiler.
__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }
template <typename Item, bool WARP> struct Feed {
    const AtParams &p;
    int round = 0, idx = -1, h = 0;
    int4 e = {};
    __device__ explicit Feed(const AtParams &p_) : p(p_) { fetch(); }
    __device__ void fetch()
    {
        const int g = (int)gridDim.x, b = (int)blockIdx.x;
        idx = round * g + ((round & 1) ? g - 1 - b : b);
        ++round;
        if (idx >= p.n_items) { idx = -1; return; }
        const int t = idx / p.hk;
        h = idx - t * p.hk;
        e = p.items[t];
    }
    __device__ bool take(Item &it)
    {
        if (idx < 0) return false;
        if (WARP) e = make_int4(uniform(e.x), uniform(e.y), uniform(e.z), uniform(e.w));
        it.set(p, h, e);
        fetch();
        return true;
    }
};

__device__ __forceinline__ int ceil_div(int a, int b) { return (a + b - 1) / b; }

// columns of a 128-wide tile that an MMA has to cover when `valid` of them (>= 1) mean something
__device__ __forceinline__ int mma_cols(int valid) { return valid >= TILE ? TILE : (valid + 15) & ~15; }

// Row r of a stored 128-byte-swizzled tile keeps its 128 bytes inside the row, so rows can be zeroed
// without undoing the swizzle.  One warp zeroes rows lo .. hi-1 of every 64-wide slab.
template <int DP> __device__ __forceinline__ void zero_rows(uint32_t tile, int lo, int hi, int lane)
{
    for (int i = lane; i < (hi - lo) * 8; i += 32)
#pragma unroll
        for (int s = 0; s < DP / 64; ++s)
            asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(tile + s * (TILE * 128) + lo * 128 + i * 16), "r"(0)
                         : "memory");
}
__device__ __forceinline__ void zero_smem(uint32_t addr, int bytes)
{
    for (int i = threadIdx.x * 16; i < bytes; i += blockDim.x * 16)
        asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};" ::"r"(addr + i), "r"(0) : "memory");
}

// A tile of [rows][head][token] boxes: one TMA box per 64-wide slab (columns past d read as zeros).
template <int DP>
__device__ __forceinline__ void load_tile(uint32_t dst, const CUtensorMap *map, int head, int token, uint32_t bar)
{
#pragma unroll
    for (int s = 0; s < DP / 64; ++s) tma_load_3d(dst + s * (TILE * 128), map, 64 * s, head, token, bar);
}

// The issuer's instructions are what a tile waits for, so they are kept few: descriptors are built as a constant
// upper word and a lower word that a stage or a K step moves by an addition (shared memory ends below 256 KiB,
// no carry leaves the address field).
constexpr uint32_t DESC_HI = (1024 >> 4) | 1u << 14 | 2u << 29;      // 8-row groups 1024 bytes apart, 128-byte swizzle
__device__ __forceinline__ uint64_t desc64(uint32_t lo)
{
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "n"(DESC_HI));
    return d;
}
__device__ __forceinline__ uint32_t desc_rows(uint32_t tile) { return tile >> 4 | (16u >> 4) << 16; }              // K-major
__device__ __forceinline__ uint32_t desc_across(uint32_t tile) { return tile >> 4 | (TILE * 128u >> 4) << 16; }    // MN-major
__device__ __forceinline__ uint32_t idesc_rows(int n) { return make_idesc(0, 0, 128, 0) | (uint32_t)n << 14; }

// D[128 x n] = A[128 x DP] B[n x DP]^T, both K-major in shared memory
template <int DP> __device__ __forceinline__ void mma_rows_rows(uint32_t on, uint32_t d_tmem, uint32_t a, uint32_t b, uint32_t idesc)
{
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
        const uint32_t off = (k / 4) * (TILE * 128 >> 4) + (k % 4) * 2;
        umma_bf16_if(on, d_tmem, desc64(a + off), desc64(b + off), idesc, k != 0);
    }
}
// D[128 x DP] (+)= A[128 x 16 K0..16 (K0 + KN) - 1] B[those rows x DP]: A in tensor memory, 16 of its rows in 8
// columns from `a` (every STRIDE steps 32 further on), B a stored tile read across its rows.  Steps at or past
// `steps` are left out.
template <int DP, int K0, int KN, int STRIDE>
__device__ __forceinline__ void mma_tmem_rows(uint32_t on, uint32_t d_tmem, uint32_t a, uint32_t b, int steps, uint32_t acc)
{
    constexpr uint32_t idesc = make_idesc(0, 1, 128, DP);
    if (steps >= K0 + KN) {
#pragma unroll
        for (int k = K0; k < K0 + KN; ++k)
            umma_bf16_ta_if(on, d_tmem, a + 32 * (k / STRIDE) + 8 * (k % STRIDE), desc64(b + k * (16 * 128 >> 4)), idesc, k == K0 ? acc : 1u);
    } else {
#pragma unroll
        for (int k = K0; k < K0 + KN - 1; ++k)
            if (k < steps)
                umma_bf16_ta_if(on, d_tmem, a + 32 * (k / STRIDE) + 8 * (k % STRIDE), desc64(b + k * (16 * 128 >> 4)), idesc, k == K0 ? acc : 1u);
    }
}

// 8 fp32 values times `f` as bf16
__device__ __forceinline__ uint4 pack8(const uint32_t *v, float f)
{
    return make_uint4(pack_bf16(__uint_as_float(v[0]) * f, __uint_as_float(v[1]) * f), pack_bf16(__uint_as_float(v[2]) * f, __uint_as_float(v[3]) * f),
                      pack_bf16(__uint_as_float(v[4]) * f, __uint_as_float(v[5]) * f), pack_bf16(__uint_as_float(v[6]) * f, __uint_as_float(v[7]) * f));
}
// Rows of a warp's accumulator to global memory: CHUNKS x 8 columns of one row per lane go through `stage`
// (32 x 16 CHUNKS bytes, slots XOR-swizzled by row: no bank conflicts), so that CHUNKS neighbouring lanes write one
// row's contiguous bytes.  Written straight from the lanes (32 rows, 16 bytes each per instruction) an
// item's output took 5000 cycles.  dst: this lane's row at the first column, null for a row that is not written;
// `chunks` of them lie inside the head.
template <int CHUNKS>
__device__ __forceinline__ void store_rows(uint32_t stage, int lane, const uint4 (&w)[CHUNKS], bf16 *dst, int chunks)
{
#pragma unroll
    for (int c = 0; c < CHUNKS; ++c)
        asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(stage + lane * (16 * CHUNKS) + ((c ^ (lane * CHUNKS / 8)) & (CHUNKS - 1)) * 16),
                     "r"(w[c].x), "r"(w[c].y), "r"(w[c].z), "r"(w[c].w)
                     : "memory");
    __syncwarp();
    const int c = lane & (CHUNKS - 1);
#pragma unroll
    for (int it = 0; it < CHUNKS; ++it) {
        const int row = it * (32 / CHUNKS) + lane / CHUNKS;
        uint4 v;
        asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                     : "r"(stage + row * (16 * CHUNKS) + ((c ^ (row * CHUNKS / 8)) & (CHUNKS - 1)) * 16)
                     : "memory");
        bf16 *d = (bf16 *)__shfl_sync(0xffffffffu, (unsigned long long)dst, row);
        if (d != nullptr && c < chunks) *reinterpret_cast<uint4 *>(d + 8 * c) = v;
    }
    __syncwarp();
}

// Ends of every kernel: drain after an abort, give the tensor memory back.
__device__ __forceinline__ void cta_teardown(volatile int *abort_flag, uint32_t tmem_base, int dealloc_warp)
{
    if (*abort_flag) {
        const unsigned long long t0 = globaltimer_ns();
        while (globaltimer_ns() - t0 < 200000ull) __nanosleep(1000);
    }
    tc_fence_before();
    __syncthreads();
    if ((int)(threadIdx.x >> 5) == dealloc_warp) {
        tc_fence_after();
        tmem_dealloc(tmem_base, AT_TMEM_COLS);
    }
}

}  // namespace

// ------------------------------------------------------------------------------------ forward
// One item = two row tiles (2 x 128 rows) of one kv head against the keys of their sequence, by one
// CTA; both tiles use every key / value tile that arrives.
//   warps 0..3 / 4..7  softmax of row tile 0 / 1, one row per thread: running maximum and sum in
//                      registers, P = 2^(c2 s - c2 m) packed to bf16 over the scores it came from
//   TMA warp           ring of key and value tiles, query tiles
//   MMA warp           S = Q K^T, O += P V (P read from tensor memory)
//   tail warp          zeroes value rows past the sequence's end inside the last 16-row step: their P is
//                      zero, but 0 * inf of a neighbour's (or of never-written) memory is not
// The output is rescaled only when the running maximum has grown by more than 2^8 since the last
// time (P stays below 2^8, far inside the range of bf16 and fp32).  Tried and slower: half a row per thread with
// the maxima exchanged (+5 %), an issuing warp per row tile (+21 %), P through shared memory so that scores run
// a block ahead (+10 %: one key tile fits then and its reload sets the pace).
template <int DP> struct FwdShape {
    static constexpr int T_BYTES = tile_bytes<DP>();
    static constexpr int SLOTS = DP == 128 ? 4 : 8;
    static constexpr int STAGE = 32 * 128;            // a warp's output rows, 64 columns at a time
    static constexpr int SMEM = (2 + SLOTS) * T_BYTES + 8 * STAGE + 512;
};
struct alignas(8) FwdCtl {
    uint64_t q_full[2], q_empty[2], kv_full[8], kv_empty[8], tail[8], s_full[2], p_full[2][2], o_full[2], o_free[2];   // p_full[g][half]
    uint32_t tmem_base;
    volatile int abort_flag;
    volatile uint32_t issued;        // tiles that the TMA lane has asked for
};

// Minus infinity into the columns of a row's scores at or past `limit`, from column `from` (a uniform lower bound of
// the warp's limits) up to `to`.  Done in tensor memory and as a loop: blocks that need it come once per item, and
// a second, masked copy of the softmax below would have to be fetched from L2 each time (measured: thousands
// of cycles on a busy memory system).
__device__ __forceinline__ void mask_scores(uint32_t t_s, int from, int to, int limit)
{
#pragma unroll 1
    for (int c = max(from, 0) & ~15; c < to; c += 16) {
        uint32_t r[16];
        tmem_ld16(t_s + c, r);
        tmem_ld_wait(r);
#pragma unroll
        for (int e = 0; e < 16; ++e)
            if (c + e >= limit) r[e] = 0xff800000u;
        tmem_st16(t_s + c, r);
    }
    tmem_st_wait();
}
__device__ __forceinline__ float max_chunk(const uint32_t (&r)[32], float m)
{
    float a = m, b = __uint_as_float(r[0]);
#pragma unroll
    for (int e = 1; e < 29; e += 4) {
        a = max3(a, __uint_as_float(r[e]), __uint_as_float(r[e + 1]));
        b = max3(b, __uint_as_float(r[e + 2]), __uint_as_float(r[e + 3]));
    }
    return max3(max3(a, b, __uint_as_float(r[29])), __uint_as_float(r[30]), __uint_as_float(r[31]));
}
// 32 scores of a row to P: 2^(c2 s - c2 m), summed, packed to bf16.  (Moving a quarter of the exponentials from
// the special-function unit to a polynomial on the FMA pipe was 2 % slower: the tile waits for latencies, not for
// that unit.)
__device__ __forceinline__ void exp_chunk(const uint32_t (&r)[32], uint64_t c2, uint64_t neg_mc, uint64_t (&sum)[2], uint32_t (&pk)[16])
{
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        float a, b;
        unpair2(fma2(pair2(__uint_as_float(r[2 * e]), __uint_as_float(r[2 * e + 1])), c2, neg_mc), a, b);
        a = fast_exp2(a);
        b = fast_exp2(b);
        sum[e & 1] = add2(sum[e & 1], pair2(a, b));
        // P enters the second product in bf16: relative 2^-8 per term, averaged over the row
        pk[e] = pack_bf16(a, b);
    }
}

// One block of scores of one row per thread: running maximum m and sum l, P over the scores.  Half of the
// scores is read twice (for the maximum, then again), which keeps a row's registers below what would spill.  P
// is handed over in two halves (p_full, p_full + 8), so that the second product starts while the second half
// is made.  `upper`: the block has columns past 63; `live`: this row is a query of the sequence.
template <int DP>
__device__ __forceinline__ void softmax_block(uint32_t t_s, uint32_t t_o, bool upper, bool live, float c2, bool first, float &m, float &l,
                                              uint32_t p_full, int lane)
{
    uint32_t x[32], y[32], u[32], v[32];
    float bm = -INFINITY;
    tmem_ld32(t_s, x);
    tmem_ld32(t_s + 32, y);
    if (upper) {
        tmem_ld32(t_s + 64, u);
        tmem_ld32(t_s + 96, v);
        tmem_ld_wait(u);
        tmem_ld_wait(v);
        bm = max_chunk(v, max_chunk(u, bm));
    }
    tmem_ld_wait(x);
    tmem_ld_wait(y);
    bm = max_chunk(y, max_chunk(x, bm));
    if (first) {
        m = bm;
    } else if (__any_sync(0xffffffffu, live && (bm - m) * c2 > 8.0f)) {
        // rows of other sequences in this tile have no say, so a sequence's bits depend on nothing else
        // the scores of this block were issued after the previous O += P V, so O is at rest
        const float mn = fmaxf(m, bm), f = m == mn ? 1.0f : fast_exp2((m - mn) * c2);    // both may be minus infinity
        m = mn;
        l *= f;
#pragma unroll 1
        for (int c = 0; c < DP; c += 16) {
            uint32_t o[16];
            tmem_ld16(t_o + c, o);
            tmem_ld_wait(o);
#pragma unroll
            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
            tmem_st16(t_o + c, o);
        }
    }
    // a row that has met nothing but minus infinity has P = 2^(-inf - 0) = 0 so far, not 2^(-inf + inf)
    const float neg_mc = m == -INFINITY ? 0.0f : -m * c2;
    const uint64_t c2p = pair2(c2, c2), mcp = pair2(neg_mc, neg_mc);
    uint64_t sum[2] = {0, 0};
    uint32_t pk[16];
    if (upper) tmem_ld32(t_s + 64, u);
    exp_chunk(x, c2p, mcp, sum, pk);
    tmem_st16(t_s, pk);
    exp_chunk(y, c2p, mcp, sum, pk);
    tmem_st16(t_s + 16, pk);
    tmem_st_wait();
    tc_fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(p_full);
    if (upper) {
        tmem_ld32(t_s + 96, v);
        tmem_ld_wait(u);
        exp_chunk(u, c2p, mcp, sum, pk);
        tmem_st16(t_s + 32, pk);
        tmem_ld_wait(v);
        exp_chunk(v, c2p, mcp, sum, pk);
        tmem_st16(t_s + 48, pk);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
    }
    if (lane == 0) mbar_arrive(p_full + 8);
    float a, b;
    unpair2(add2(sum[0], sum[1]), a, b);
    l += a + b;
}

struct FwdItem {
    int start, len, t0, h, nb0, nb1, end0, end1;   // key blocks and first key past the keys of the two tiles
    __device__ void set(const AtParams &p, int head, const int4 &e)
    {
        h = head;
        start = e.x; len = e.y; t0 = e.z;
        end0 = p.causal ? min(t0 + p.tokens, len) : len;
        end1 = t0 + p.tokens < len ? (p.causal ? min(t0 + 2 * p.tokens, len) : len) : 0;
        nb0 = ceil_div(end0, TILE);
        nb1 = ceil_div(end1, TILE);
    }
    __device__ int blocks() const { return max(nb0, nb1); }
    // the last value tile holds rows past the sequence that an MMA step would read
    __device__ bool dirty_tail() const { return (len & 15) != 0 && blocks() * TILE > len; }
};

template <int DP>
__global__ void __launch_bounds__(FwdWarps::THREADS, 1)
k_attention_fwd(const __grid_constant__ AtMaps tm, const AtParams p)
{
    constexpr int T_BYTES = FwdShape<DP>::T_BYTES, SLOTS = FwdShape<DP>::SLOTS;
    extern __shared__ __align__(1024) uint8_t smem_raw[];      // tiles need 1024 bytes
    const uint32_t tiles = smem_u32(smem_raw), q_tile = tiles, ring = tiles + 2 * T_BYTES;
    FwdCtl *ctl = reinterpret_cast<FwdCtl *>(smem_raw + (2 + SLOTS) * T_BYTES + 8 * FwdShape<DP>::STAGE);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&ctl->q_full[i]), 1);
            mbar_init(smem_u32(&ctl->q_empty[i]), 1);
            mbar_init(smem_u32(&ctl->s_full[i]), 1);
            mbar_init(smem_u32(&ctl->p_full[i][0]), 4);
            mbar_init(smem_u32(&ctl->p_full[i][1]), 4);
            mbar_init(smem_u32(&ctl->o_full[i]), 1);
            mbar_init(smem_u32(&ctl->o_free[i]), 4);
        }
        for (int i = 0; i < SLOTS; ++i) {
            mbar_init(smem_u32(&ctl->kv_full[i]), 1);
            mbar_init(smem_u32(&ctl->kv_empty[i]), 1);
            mbar_init(smem_u32(&ctl->tail[i]), 1);
        }
        ctl->abort_flag = 0;
        ctl->issued = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    const int used = p.group * p.tokens;     // rows of a tile that a box fills; the others stay zero
    if (used < TILE) zero_smem(q_tile, 2 * T_BYTES);
    fence_proxy_async_smem();
    if (warp == FwdWarps::MMA) { tmem_alloc(smem_u32(&ctl->tmem_base), AT_TMEM_COLS); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const Waits waits{&ctl->abort_flag, &ctl->issued, p.status, p.wait_ns};
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    if (warp < FwdWarps::FIRST) regs_down<FwdWarps::REGS_SERVICE>();
    if (warp == FwdWarps::TMA) {
        if (lane == 0) {
            uint32_t pos = 0, nq[2] = {0, 0};
            bool ok = true;
            auto acquire = [&]() {           // next ring slot, free to be written
                const uint32_t s = pos % SLOTS;
                ok = ok && wait_lane(smem_u32(&ctl->kv_empty[s]), ((pos / SLOTS) & 1) ^ 1, waits, SITE_PRODUCER_EMPTY);
                ++pos;
                return s;
            };
            auto load_q = [&](const FwdItem &it, int g) {
                ok = ok && wait_lane(smem_u32(&ctl->q_empty[g]), (nq[g] & 1) ^ 1, waits, SITE_PRODUCER_EMPTY);
                if (!ok) return;
                const uint32_t bar = smem_u32(&ctl->q_full[g]);
                mbar_expect_tx(bar, (uint32_t)(used * DP * 2));
                load_tile<DP>(q_tile + g * T_BYTES, &tm.q, it.h * p.group, it.start + it.t0 + g * p.tokens, bar);
                ++nq[g];
            };
            Feed<FwdItem, false> feed(p);
            FwdItem it;
            while (ok && feed.take(it)) {
                const int n = it.blocks();
                load_q(it, 0);
                for (int j = 0; j < n && ok; ++j) {
                    uint32_t s = acquire();
                    if (!ok) break;
                    uint32_t bar = smem_u32(&ctl->kv_full[s]);
                    mbar_expect_tx(bar, T_BYTES + p.lose);
                    load_tile<DP>(ring + s * T_BYTES, &tm.k, it.h, it.start + j * TILE, bar);
                    if (j == 0 && it.nb1) load_q(it, 1);
                    s = acquire();
                    if (!ok) break;
                    // the tail warp passes a tile with rows to zero on to the MMA warp
                    bar = smem_u32(j == n - 1 && it.dirty_tail() ? &ctl->tail[s] : &ctl->kv_full[s]);
                    mbar_expect_tx(bar, T_BYTES);
                    load_tile<DP>(ring + s * T_BYTES, &tm.v, it.h, it.start + j * TILE, bar);
                    ctl->issued = pos;
                }
            }
        }
    } else if (warp == FwdWarps::TAIL) {
        uint32_t pos = 0, seen = 0;          // bit s: parity of the tail events of slot s
        bool ok = true;
        Feed<FwdItem, true> feed(p);
        FwdItem it;
        while (ok && feed.take(it)) {
            const int n = it.blocks();
            pos += 2 * n;
            if (!it.dirty_tail()) continue;
            const uint32_t s = (pos - 1) % SLOTS;
            ok = wait_warp<false>(smem_u32(&ctl->tail[s]), (seen >> s) & 1, waits, SITE_PRODUCER_EMPTY);
            if (!ok) break;
            seen ^= 1u << s;
            const int valid = it.len - (n - 1) * TILE;
            zero_rows<DP>(ring + s * T_BYTES, valid, mma_cols(valid), lane);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctl->kv_full[s]));
        }
    } else if (warp == FwdWarps::MMA) {
        const uint32_t on = elect_one();     // the warp walks as one, one thread issues
        const uint32_t q_desc = desc_rows(q_tile), k_desc0 = desc_rows(ring), v_desc0 = desc_across(ring);
        const uint32_t kv_full = smem_u32(&ctl->kv_full[0]), kv_empty = smem_u32(&ctl->kv_empty[0]);
        uint32_t slot = 0, phase = 0, nq[2] = {0, 0}, np[2] = {0, 0};
        bool ok = true;
        auto wait_slot = [&]() { ok = ok && wait_warp<true>(kv_full + 8 * slot, phase, waits, SITE_MMA_FULL); };
        auto next_slot = [&]() {
            const uint32_t s = slot;
            if (++slot == SLOTS) { slot = 0; phase ^= 1; }
            return s;
        };
        Feed<FwdItem, true> feed(p);
        FwdItem it;
        while (ok && feed.take(it)) {
            const int n = it.blocks();
            const int nb[2] = {it.nb0, it.nb1};
            const int last_cols[2] = {mma_cols(it.end0 - (it.nb0 - 1) * TILE), mma_cols(it.end1 - (it.nb1 - 1) * TILE)};
            auto scores = [&](int g, int j, uint32_t k_slot) {
                mma_rows_rows<DP>(on, tmem + g * TILE, q_desc + g * (T_BYTES >> 4), k_desc0 + k_slot * (T_BYTES >> 4),
                                  idesc_rows(j == nb[g] - 1 ? last_cols[g] : TILE));
                umma_commit_if(on, smem_u32(&ctl->s_full[g]));
            };
            wait_slot();
            uint32_t ks = next_slot();
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                if (!ok || nb[g] == 0) break;
                ok = wait_warp<true>(smem_u32(&ctl->q_full[g]), nq[g] & 1, waits, SITE_MMA_FULL);
                if (!ok) break;
                ++nq[g];
                tc_fence_after();
                scores(g, 0, ks);
                if (nb[g] == 1) umma_commit_if(on, smem_u32(&ctl->q_empty[g]));
            }
            if (!ok) break;
            umma_commit_if(on, kv_empty + 8 * ks);
            for (int j = 0; j < n; ++j) {
                wait_slot();
                const uint32_t vs = next_slot();
                const bool more = j + 1 < n;
                if (more) { wait_slot(); ks = next_slot(); }
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    if (!ok) break;
                    if (j >= nb[g]) continue;
                    const uint32_t pt = tmem + g * TILE, ot = tmem + 2 * TILE + g * DP, vd = v_desc0 + vs * (T_BYTES >> 4);
                    const bool last = j == nb[g] - 1;
                    const int steps = last ? last_cols[g] / 16 : TILE / 16;
                    if (j == 0) ok = wait_warp<true>(smem_u32(&ctl->o_free[g]), (nq[g] - 1) & 1 ^ 1, waits, SITE_MMA_TMEM_EMPTY);
                    ok = ok && wait_warp<true>(smem_u32(&ctl->p_full[g][0]), np[g] & 1, waits, SITE_MMA_FULL);
                    if (!ok) break;
                    tc_fence_after();
                    mma_tmem_rows<DP, 0, 4, 8>(on, ot, pt, vd, steps, j > 0);
                    ok = wait_warp<true>(smem_u32(&ctl->p_full[g][1]), np[g] & 1, waits, SITE_MMA_FULL);
                    if (!ok) break;
                    ++np[g];
                    tc_fence_after();
                    mma_tmem_rows<DP, 4, 4, 8>(on, ot, pt, vd, steps, 1);
                    if (last) {
                        umma_commit_if(on, smem_u32(&ctl->o_full[g]));
                    } else {
                        scores(g, j + 1, ks);
                        if (j + 2 == nb[g]) umma_commit_if(on, smem_u32(&ctl->q_empty[g]));
                    }
                }
                if (!ok) break;
                umma_commit_if(on, kv_empty + 8 * vs);
                if (more) umma_commit_if(on, kv_empty + 8 * ks);
            }
        }
    } else if (warp >= FwdWarps::FIRST) {
        regs_up<FwdWarps::REGS_ARITH>();
        const int g = (warp - FwdWarps::FIRST) >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const uint32_t t_s = tmem + lanes + g * TILE, t_o = tmem + lanes + 2 * TILE + g * DP;
        const uint32_t s_full = smem_u32(&ctl->s_full[g]), p_full = smem_u32(&ctl->p_full[g][0]);
        uint32_t ns = 0, no = 0;
        bool ok = true;
        const int row_t = row / p.group, row_h = row - row_t * p.group;
        Feed<FwdItem, true> feed(p);
        FwdItem it;
        while (ok && feed.take(it)) {
            const int nb = g ? it.nb1 : it.nb0, end = g ? it.end1 : it.end0, t0 = it.t0 + g * p.tokens;
            if (nb == 0) continue;
            const int token = t0 + row_t;
            const int row_end = p.causal ? min(token + 1, it.len) : it.len;   // keys of this row
            const bool live = row < used && token < it.len;                   // a query of this sequence
            float m = -INFINITY, l = 0.0f;
            for (int j = 0; j < nb; ++j) {
                ok = wait_warp<true>(s_full, ns & 1, waits, SITE_EPI_TMEM_FULL);
                ++ns;
                if (!ok) break;
                tc_fence_after();
                // columns past the row's keys (or past the ones the MMA wrote) count as minus infinity
                const bool upper = end - j * TILE > 64;
                const int from = (p.causal ? t0 + 1 : it.len) - j * TILE, to = upper ? TILE : 64;
                if (from < to) mask_scores(t_s, from, to, row_end - j * TILE);
                softmax_block<DP>(t_s, t_o, upper, live, p.c2, j == 0, m, l, p_full, lane);
            }
            if (!ok) break;
            ok = wait_warp<true>(smem_u32(&ctl->o_full[g]), no & 1, waits, SITE_EPI_TMEM_FULL);
            ++no;
            if (!ok) break;
            tc_fence_after();
            const float inv = 1.0f / l;
            const int head = it.h * p.group + row_h;
            const int64_t tok = (int64_t)it.start + token;
            bf16 *dst = live ? p.out0 + tok * p.ld0 + (int64_t)head * p.d : nullptr;
            const uint32_t stage = ring + SLOTS * T_BYTES + (warp - FwdWarps::FIRST) * FwdShape<DP>::STAGE;
#pragma unroll 1
            for (int c = 0; c < DP; c += 64) {
                uint32_t o[32];
                uint4 w[8];
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    tmem_ld32(t_o + c + 32 * h, o);
                    tmem_ld_wait(o);
#pragma unroll
                    for (int k = 0; k < 4; ++k) w[4 * h + k] = pack8(o + 8 * k, inv);
                }
                store_rows<8>(stage, lane, w, dst ? dst + c : nullptr, (p.d - c) / 8);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctl->o_free[g]));
            if (live) p.lse[tok * p.hq + head] = fmaf(m, p.scale, logf(l));
        }
    }
    cta_teardown(waits.abort_flag, ctl->tmem_base, FwdWarps::MMA);
}

// ------------------------------------------------------------------------------------ dK, dV
// One item = one key tile (128 keys) of one kv head against the row tiles that attend to it.  The
// scores are computed transposed (keys on the accumulator rows), so that P^T and dS^T are already the
// tensor-memory operands of dV += P^T dO and dK += dS^T Q.  Four warpgroups share the rows, each
// with a quarter of the columns.  While the arithmetic warps turn scores into P, the tensor cores run the
// previous dK and the next dP; while they turn dP into dS, dV and the next scores.
// Sums over the query heads of a group are sums over tile rows: fixed order, no atomics.  P and dS lie over the
// scores they come from (tensor memory is full: S, dP, dV, dK), rounded to bf16 as operands; bound by the chain
// scores -> P -> dV -> next scores, 3300 cycles a step at d = 128 for 2048 of products.
template <int DP> struct KvShape {
    static constexpr int T_BYTES = tile_bytes<DP>();
    static constexpr int STAGES = 2;
    static constexpr int STAT_BYTES = TILE * 8;
    static constexpr int STAGE = 32 * 64;             // a warp's output rows, 32 columns at a time
    static constexpr int SMEM = (2 + 2 * STAGES) * T_BYTES + STAGES * STAT_BYTES + BwdWarps::COUNT * STAGE + 512;
};
struct alignas(8) KvCtl {
    uint64_t k_full, k_empty, v_full, v_empty, q_full[2], g_full[2], empty[2], q_tail[2], g_tail[2];
    uint64_t s_full, g_scores, p_ready, ds_ready, acc_full, acc_free;
    uint32_t tmem_base;
    volatile int abort_flag;
    volatile uint32_t issued;        // tiles that the TMA lane has asked for
};
struct KvItem {
    int start, len, k0, base, h, first, n;      // row tiles first .. first + n - 1 of the sequence
    __device__ void set(const AtParams &p, int head, const int4 &e)
    {
        h = head;
        start = e.x; len = e.y; k0 = e.z; base = e.w;
        first = p.causal ? k0 / p.tokens : 0;
        n = ceil_div(len, p.tokens) - first;
    }
    // tile rows that belong to tokens of the sequence (the others follow them)
    __device__ int valid(const AtParams &p, int tile) const { return min(p.tokens, len - tile * p.tokens) * p.group; }
    __device__ bool dirty(const AtParams &p, int tile) const
    {
        return len - tile * p.tokens < p.tokens && (valid(p, tile) & 15) != 0;
    }
};

template <int DP>
__global__ void __launch_bounds__(BwdWarps::THREADS, 1)
k_attention_bwd_kv(const __grid_constant__ AtMaps tm, const AtParams p)
{
    using Sh = KvShape<DP>;
    constexpr int T_BYTES = Sh::T_BYTES;
    extern __shared__ __align__(1024) uint8_t smem_raw[];      // tiles need 1024 bytes
    const uint32_t tiles = smem_u32(smem_raw);
    const uint32_t k_tile = tiles, v_tile = tiles + T_BYTES, q_ring = tiles + 2 * T_BYTES, g_ring = q_ring + 2 * T_BYTES;
    const uint32_t stats = g_ring + 2 * T_BYTES;
    uint8_t *after = smem_raw + (stats - smem_u32(smem_raw));
    KvCtl *ctl = reinterpret_cast<KvCtl *>(after + Sh::STAGES * Sh::STAT_BYTES + BwdWarps::COUNT * Sh::STAGE);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&ctl->q_full[i]), 1);
            mbar_init(smem_u32(&ctl->g_full[i]), 1);
            mbar_init(smem_u32(&ctl->q_tail[i]), 1);
            mbar_init(smem_u32(&ctl->g_tail[i]), 1);
            mbar_init(smem_u32(&ctl->empty[i]), 1);
        }
        mbar_init(smem_u32(&ctl->k_full), 1);
        mbar_init(smem_u32(&ctl->k_empty), 1);
        mbar_init(smem_u32(&ctl->v_full), 1);
        mbar_init(smem_u32(&ctl->v_empty), 1);
        mbar_init(smem_u32(&ctl->s_full), 1);
        mbar_init(smem_u32(&ctl->g_scores), 1);
        mbar_init(smem_u32(&ctl->p_ready), BwdWarps::COUNT);
        mbar_init(smem_u32(&ctl->ds_ready), BwdWarps::COUNT);
        mbar_init(smem_u32(&ctl->acc_full), 1);
        mbar_init(smem_u32(&ctl->acc_free), BwdWarps::COUNT);
        ctl->abort_flag = 0;
        ctl->issued = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    const int used = p.group * p.tokens;
    if (used < TILE) zero_smem(q_ring, 4 * T_BYTES);
    fence_proxy_async_smem();
    if (warp == BwdWarps::MMA) { tmem_alloc(smem_u32(&ctl->tmem_base), AT_TMEM_COLS); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const Waits waits{&ctl->abort_flag, &ctl->issued, p.status, p.wait_ns};
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t t_s = tmem, t_dp = tmem + TILE, t_dv = tmem + 2 * TILE, t_dk = t_dv + DP;

    if (warp < BwdWarps::FIRST) regs_down<BwdWarps::REGS_SERVICE>();
    if (warp == BwdWarps::TMA) {
        if (lane == 0) {
            uint32_t cnt = 0, items = 0;
            bool ok = true;
            Feed<KvItem, false> feed(p);
            KvItem it;
            for (; ok && feed.take(it); ++items) {
                for (int j = 0; j < it.n; ++j, ++cnt) {
                    const uint32_t s = cnt & 1;
                    const int tile = it.first + j, token = it.start + tile * p.tokens;
                    const bool dirty = it.dirty(p, tile);
                    const uint32_t qb = smem_u32(dirty ? &ctl->q_tail[s] : &ctl->q_full[s]);
                    const uint32_t gb = smem_u32(dirty ? &ctl->g_tail[s] : &ctl->g_full[s]);
                    if (j == 0) {
                        ok = wait_lane(smem_u32(&ctl->k_empty), (items & 1) ^ 1, waits, SITE_PRODUCER_EMPTY);
                        if (!ok) break;
                        mbar_expect_tx(smem_u32(&ctl->k_full), T_BYTES + p.lose);
                        load_tile<DP>(k_tile, &tm.k, it.h, it.start + it.k0, smem_u32(&ctl->k_full));
                    }
                    ok = wait_lane(smem_u32(&ctl->empty[s]), ((cnt >> 1) & 1) ^ 1, waits, SITE_PRODUCER_EMPTY);
                    if (!ok) break;
                    mbar_expect_tx(qb, (uint32_t)(used * DP * 2) + Sh::STAT_BYTES);
                    load_tile<DP>(q_ring + s * T_BYTES, &tm.q, it.h * p.group, token, qb);
                    bulk_load(stats + s * Sh::STAT_BYTES, p.row_stats + ((int64_t)(it.base + tile) * p.hk + it.h) * TILE, Sh::STAT_BYTES, qb);
                    mbar_expect_tx(gb, (uint32_t)(used * DP * 2));
                    load_tile<DP>(g_ring + s * T_BYTES, &tm.g, it.h * p.group, token, gb);
                    ctl->issued = cnt + 1;
                    if (j == 0) {
                        ok = wait_lane(smem_u32(&ctl->v_empty), (items & 1) ^ 1, waits, SITE_PRODUCER_EMPTY);
                        if (!ok) break;
                        mbar_expect_tx(smem_u32(&ctl->v_full), T_BYTES);
                        load_tile<DP>(v_tile, &tm.v, it.h, it.start + it.k0, smem_u32(&ctl->v_full));
                    }
                }
            }
        }
    } else if (warp == BwdWarps::TAIL) {
        uint32_t cnt = 0, seen = 0;
        bool ok = true;
        Feed<KvItem, true> feed(p);
        KvItem it;
        while (ok && feed.take(it)) {
            cnt += it.n;
            const int tile = it.first + it.n - 1;          // only a sequence's last row tile can be short
            if (!it.dirty(p, tile)) continue;
            const uint32_t s = (cnt - 1) & 1;
            const int valid = it.valid(p, tile);
            for (int w = 0; w < 2 && ok; ++w) {
                ok = wait_warp<false>(smem_u32(w ? &ctl->g_tail[s] : &ctl->q_tail[s]), (seen >> s) & 1, waits, SITE_PRODUCER_EMPTY);
                if (!ok) break;
                zero_rows<DP>((w ? g_ring : q_ring) + s * T_BYTES, valid, min(mma_cols(valid), used), lane);
                fence_proxy_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(w ? &ctl->g_full[s] : &ctl->q_full[s]));
            }
            seen ^= 1u << s;
        }
    } else if (warp == BwdWarps::MMA) {
        const uint32_t on = elect_one();
        const uint32_t k_desc = desc_rows(k_tile), v_desc = desc_rows(v_tile), q_desc = desc_rows(q_ring), g_desc = desc_rows(g_ring);
        const uint32_t q_across = desc_across(q_ring), g_across = desc_across(g_ring);
        uint32_t cnt = 0, items = 0;
        bool ok = true;
        Feed<KvItem, true> feed(p);
        KvItem it;
        for (; ok && feed.take(it); ++items) {
            auto cols_of = [&](int j) { return mma_cols(it.valid(p, it.first + j)); };
            auto scores = [&](int j, uint32_t c) {
                ok = ok && wait_warp<true>(smem_u32(&ctl->q_full[c & 1]), (c >> 1) & 1, waits, SITE_MMA_FULL);
                if (!ok) return;
                tc_fence_after();
                mma_rows_rows<DP>(on, t_s, k_desc, q_desc + (c & 1) * (T_BYTES >> 4), idesc_rows(cols_of(j)));
                umma_commit_if(on, smem_u32(&ctl->s_full));
                if (j == it.n - 1) umma_commit_if(on, smem_u32(&ctl->k_empty));
            };
            auto grad_scores = [&](int j, uint32_t c) {
                ok = ok && wait_warp<true>(smem_u32(&ctl->g_full[c & 1]), (c >> 1) & 1, waits, SITE_MMA_FULL);
                if (!ok) return;
                tc_fence_after();
                mma_rows_rows<DP>(on, t_dp, v_desc, g_desc + (c & 1) * (T_BYTES >> 4), idesc_rows(cols_of(j)));
                umma_commit_if(on, smem_u32(&ctl->g_scores));
                if (j == it.n - 1) umma_commit_if(on, smem_u32(&ctl->v_empty));
            };
            ok = wait_warp<true>(smem_u32(&ctl->k_full), items & 1, waits, SITE_MMA_FULL);
            scores(0, cnt);
            ok = ok && wait_warp<true>(smem_u32(&ctl->v_full), items & 1, waits, SITE_MMA_FULL);
            grad_scores(0, cnt);
            for (int j = 0; j < it.n && ok; ++j, ++cnt) {
                const uint32_t s = cnt & 1;
                ok = wait_warp<true>(smem_u32(&ctl->p_ready), cnt & 1, waits, SITE_MMA_FULL);
                if (ok && j == 0)
                    ok = wait_warp<true>(smem_u32(&ctl->acc_free), (items & 1) ^ 1, waits, SITE_MMA_TMEM_EMPTY);
                if (!ok) break;
                tc_fence_after();
                mma_tmem_rows<DP, 0, 8, 2>(on, t_dv, t_s, g_across + s * (T_BYTES >> 4), cols_of(j) / 16, j > 0);
                if (j + 1 < it.n) scores(j + 1, cnt + 1);
                ok = ok && wait_warp<true>(smem_u32(&ctl->ds_ready), cnt & 1, waits, SITE_MMA_FULL);
                if (!ok) break;
                tc_fence_after();
                mma_tmem_rows<DP, 0, 8, 2>(on, t_dk, t_dp, q_across + s * (T_BYTES >> 4), cols_of(j) / 16, j > 0);
                umma_commit_if(on, smem_u32(&ctl->empty[s]));
                if (j + 1 < it.n) grad_scores(j + 1, cnt + 1);
            }
            if (!ok) break;
            umma_commit_if(on, smem_u32(&ctl->acc_full));
        }
    } else if (warp >= BwdWarps::FIRST) {
        regs_up<BwdWarps::REGS_ARITH>();
        const int part = (warp - BwdWarps::FIRST) >> 2, row = (warp & 3) * 32 + lane, c0 = 32 * part;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        uint32_t cnt = 0, items = 0;
        bool ok = true;
        Feed<KvItem, true> feed(p);
        KvItem it;
        for (; ok && feed.take(it); ++items) {
            const int key = it.k0 + row;
            for (int j = 0; j < it.n; ++j, ++cnt) {
                const int tile = it.first + j, t0 = tile * p.tokens;
                const bool some = c0 < mma_cols(it.valid(p, tile));
                // causal: row (token, head) r of the tile sees this key if token >= key, r >= (key - t0) group
                const bool mask = p.causal && t0 < it.k0 + TILE - 1;
                const int from = mask ? (key - t0) * p.group - c0 : 0;
                const uint32_t st = stats + (cnt & 1) * Sh::STAT_BYTES + c0 * 8;
                ok = wait_warp<true>(smem_u32(&ctl->s_full), cnt & 1, waits, SITE_EPI_TMEM_FULL);
                if (!ok) break;
                tc_fence_after();
                uint32_t r[32], pk[16];
                if (some) {
                    tmem_ld32(t_s + lanes + c0, r);
                    tmem_ld_wait(r);
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float l0, d0, l1, d1;
                        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(l0), "=f"(d0), "=f"(l1), "=f"(d1) : "r"(st + e * 8));
                        float a = fast_exp2(fmaf(__uint_as_float(r[e]), p.c2, -l0));
                        float b = fast_exp2(fmaf(__uint_as_float(r[e + 1]), p.c2, -l1));
                        if (mask) {
                            a = e >= from ? a : 0.0f;
                            b = e + 1 >= from ? b : 0.0f;
                        }
                        r[e] = __float_as_uint(a);
                        r[e + 1] = __float_as_uint(b);
                        pk[e / 2] = pack_bf16(a, b);
                    }
                    tmem_st16(t_s + lanes + c0, pk);
                    tmem_st_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&ctl->p_ready));
                ok = wait_warp<true>(smem_u32(&ctl->g_scores), cnt & 1, waits, SITE_EPI_TMEM_FULL);
                if (!ok) break;
                tc_fence_after();
                if (some) {
                    uint32_t dp[32];
                    tmem_ld32(t_dp + lanes + c0, dp);
                    tmem_ld_wait(dp);
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float l0, d0, l1, d1;
                        asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(l0), "=f"(d0), "=f"(l1), "=f"(d1) : "r"(st + e * 8));
                        float a = __uint_as_float(r[e]) * (__uint_as_float(dp[e]) - d0);
                        float b = __uint_as_float(r[e + 1]) * (__uint_as_float(dp[e + 1]) - d1);
                        if (mask) {                // a masked product is zero even where dP is not finite
                            a = e >= from ? a : 0.0f;
                            b = e + 1 >= from ? b : 0.0f;
                        }
                        pk[e / 2] = pack_bf16(a, b);
                    }
                    tmem_st16(t_dp + lanes + c0, pk);
                    tmem_st_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&ctl->ds_ready));
            }
            if (!ok) break;
            ok = wait_warp<true>(smem_u32(&ctl->acc_full), items & 1, waits, SITE_EPI_TMEM_FULL);
            if (!ok) break;
            tc_fence_after();
            // parts 0, 1: the column halves of dV; 2, 3: of dK
            const bool live = key < it.len, is_k = part >= 2;
            const int col = (part & 1) * (DP / 2);
            bf16 *dst = (is_k ? p.out0 + ((int64_t)it.start + key) * p.ld0 : p.out1 + ((int64_t)it.start + key) * p.ld1) + (int64_t)it.h * p.d;
            const uint32_t stage = stats + Sh::STAGES * Sh::STAT_BYTES + (warp - BwdWarps::FIRST) * Sh::STAGE;
#pragma unroll 1
            for (int c = col; c < col + DP / 2; c += 32) {
                uint32_t o[32];
                uint4 w[4];
                tmem_ld32((is_k ? t_dk : t_dv) + lanes + c, o);
                tmem_ld_wait(o);
#pragma unroll
                for (int k = 0; k < 4; ++k) w[k] = pack8(o + 8 * k, is_k ? p.scale : 1.0f);
                store_rows<4>(stage, lane, w, live ? dst + c : nullptr, (p.d - c) / 8);
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctl->acc_free));
        }
    }
    cta_teardown(waits.abort_flag, ctl->tmem_base, BwdWarps::MMA);
}

// ------------------------------------------------------------------------------------ dQ
// One item = one row tile of one kv head against the keys of its sequence: S = Q K^T (two buffers),
// dP = dO V^T, dS over the scores, dQ += dS K.
// Two roundings would add up in dQ: dS to bf16, and the one of `out` that delta = do . out carries into every
// dS of the row (relative errors 1.6e-3 and 1.0e-3, next to 1.7e-3 of dQ's own rounding).  So dS enters the
// product as the sum of two bf16 numbers (eight more MMAs a block), which leaves the second.  The first is left in
// dK, whose kernel runs after this one, and the second is taken out there: the exact delta makes every row of
// dS sum to zero, so the row sums found here are added to delta.
// A row whose keys are one block has all of P and dP at hand: its delta is their sum in fp32 (short sequences, where
// the rounding of `out` was 1.6 to 5 times dQ's own), and where it sees one key, that key's dP: P = 1, and dS is zero
// (NaN where dP is not finite), not the difference of two orders of summation.  The kernel of dK and dV, whose dP is
// the same sum in the same order, gets these deltas too.
template <int DP> struct QShape {
    static constexpr int T_BYTES = tile_bytes<DP>();
    static constexpr int KS = 3, VS = 2;
    static constexpr int SUM_BYTES = 4 * TILE * 4;    // row sums of dS: [part][row]
    static constexpr int SMEM = (2 + KS + VS) * T_BYTES + SUM_BYTES + 512;
};
struct alignas(8) QCtl {
    uint64_t q_full, q_empty, g_full, g_empty, k_full[3], k_empty[3], k_tail[3], v_full[2], v_empty[2];
    uint64_t s_full[2], g_scores, ds_ready, acc_full, acc_free, sum_ready, sum_read;
    uint32_t tmem_base;
    volatile int abort_flag;
    volatile uint32_t issued;        // tiles that the TMA lane has asked for
};
struct QItem {
    int start, len, t0, tile, h, end, nb;
    __device__ void set(const AtParams &p, int head, const int4 &e)
    {
        h = head;
        start = e.x; len = e.y; t0 = e.z; tile = e.w + t0 / p.tokens;
        end = p.causal ? min(t0 + p.tokens, len) : len;
        nb = ceil_div(end, TILE);
    }
    __device__ bool dirty_tail() const { return (len & 15) != 0 && nb * TILE > len; }
};

template <int DP>
__global__ void __launch_bounds__(BwdWarps::THREADS, 1)
k_attention_bwd_q(const __grid_constant__ AtMaps tm, const AtParams p)
{
    using Sh = QShape<DP>;
    constexpr int T_BYTES = Sh::T_BYTES, KS = Sh::KS, VS = Sh::VS;
    extern __shared__ __align__(1024) uint8_t smem_raw[];      // tiles need 1024 bytes
    const uint32_t tiles = smem_u32(smem_raw);
    const uint32_t q_tile = tiles, g_tile = tiles + T_BYTES, k_ring = tiles + 2 * T_BYTES, v_ring = k_ring + KS * T_BYTES;
    const uint32_t sums = v_ring + VS * T_BYTES;
    QCtl *ctl = reinterpret_cast<QCtl *>(smem_raw + (2 + KS + VS) * T_BYTES + Sh::SUM_BYTES);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        mbar_init(smem_u32(&ctl->q_full), 1);
        mbar_init(smem_u32(&ctl->q_empty), 1);
        mbar_init(smem_u32(&ctl->g_full), 1);
        mbar_init(smem_u32(&ctl->g_empty), 1);
        for (int i = 0; i < KS; ++i) {
            mbar_init(smem_u32(&ctl->k_full[i]), 1);
            mbar_init(smem_u32(&ctl->k_empty[i]), 1);
            mbar_init(smem_u32(&ctl->k_tail[i]), 1);
        }
        for (int i = 0; i < VS; ++i) {
            mbar_init(smem_u32(&ctl->v_full[i]), 1);
            mbar_init(smem_u32(&ctl->v_empty[i]), 1);
        }
        mbar_init(smem_u32(&ctl->s_full[0]), 1);
        mbar_init(smem_u32(&ctl->s_full[1]), 1);
        mbar_init(smem_u32(&ctl->g_scores), 1);
        mbar_init(smem_u32(&ctl->ds_ready), BwdWarps::COUNT);
        mbar_init(smem_u32(&ctl->sum_ready), BwdWarps::COUNT);
        mbar_init(smem_u32(&ctl->sum_read), BwdWarps::COUNT);
        mbar_init(smem_u32(&ctl->acc_full), 1);
        mbar_init(smem_u32(&ctl->acc_free), BwdWarps::COUNT);
        ctl->abort_flag = 0;
        ctl->issued = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    const int used = p.group * p.tokens;
    if (used < TILE) zero_smem(q_tile, 2 * T_BYTES);
    fence_proxy_async_smem();
    if (warp == BwdWarps::MMA) { tmem_alloc(smem_u32(&ctl->tmem_base), AT_TMEM_COLS); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const Waits waits{&ctl->abort_flag, &ctl->issued, p.status, p.wait_ns};
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const uint32_t t_dp = tmem + 2 * TILE, t_dq = tmem + 3 * TILE;

    if (warp < BwdWarps::FIRST) regs_down<BwdWarps::REGS_SERVICE>();
    if (warp == BwdWarps::TMA) {
        if (lane == 0) {
            uint32_t cnt = 0, items = 0;
            bool ok = true;
            Feed<QItem, false> feed(p);
            QItem it;
            for (; ok && feed.take(it); ++items) {
                ok = wait_lane(smem_u32(&ctl->q_empty), (items & 1) ^ 1, waits, SITE_PRODUCER_EMPTY);
                if (!ok) break;
                mbar_expect_tx(smem_u32(&ctl->q_full), (uint32_t)(used * DP * 2));
                load_tile<DP>(q_tile, &tm.q, it.h * p.group, it.start + it.t0, smem_u32(&ctl->q_full));
                for (int j = 0; j < it.nb; ++j, ++cnt) {
                    const uint32_t ks = cnt % KS, vs = cnt % VS;
                    ok = wait_lane(smem_u32(&ctl->k_empty[ks]), ((cnt / KS) & 1) ^ 1, waits, SITE_PRODUCER_EMPTY);
                    if (!ok) break;
                    const uint32_t kb = smem_u32(j == it.nb - 1 && it.dirty_tail() ? &ctl->k_tail[ks] : &ctl->k_full[ks]);
                    mbar_expect_tx(kb, T_BYTES + p.lose);
                    load_tile<DP>(k_ring + ks * T_BYTES, &tm.k, it.h, it.start + j * TILE, kb);
                    if (j == 0) {
                        ok = wait_lane(smem_u32(&ctl->g_empty), (items & 1) ^ 1, waits, SITE_PRODUCER_EMPTY);
                        if (!ok) break;
                        mbar_expect_tx(smem_u32(&ctl->g_full), (uint32_t)(used * DP * 2));
                        load_tile<DP>(g_tile, &tm.g, it.h * p.group, it.start + it.t0, smem_u32(&ctl->g_full));
                    }
                    ok = wait_lane(smem_u32(&ctl->v_empty[vs]), ((cnt / VS) & 1) ^ 1, waits, SITE_PRODUCER_EMPTY);
                    if (!ok) break;
                    const uint32_t vb = smem_u32(&ctl->v_full[vs]);
                    mbar_expect_tx(vb, T_BYTES);
                    load_tile<DP>(v_ring + vs * T_BYTES, &tm.v, it.h, it.start + j * TILE, vb);
                    ctl->issued = cnt + 1;
                }
            }
        }
    } else if (warp == BwdWarps::TAIL) {
        uint32_t cnt = 0, seen = 0;
        bool ok = true;
        Feed<QItem, true> feed(p);
        QItem it;
        while (ok && feed.take(it)) {
            cnt += it.nb;
            if (!it.dirty_tail()) continue;
            const uint32_t s = (cnt - 1) % KS;
            ok = wait_warp<false>(smem_u32(&ctl->k_tail[s]), (seen >> s) & 1, waits, SITE_PRODUCER_EMPTY);
            if (!ok) break;
            seen ^= 1u << s;
            const int valid = it.len - (it.nb - 1) * TILE;
            zero_rows<DP>(k_ring + s * T_BYTES, valid, mma_cols(valid), lane);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctl->k_full[s]));
        }
    } else if (warp == BwdWarps::MMA) {
        const uint32_t on = elect_one();
        const uint32_t q_desc = desc_rows(q_tile), g_desc = desc_rows(g_tile), k_desc = desc_rows(k_ring), v_desc = desc_rows(v_ring);
        const uint32_t k_across = desc_across(k_ring);
        uint32_t cnt = 0, items = 0;
        bool ok = true;
        Feed<QItem, true> feed(p);
        QItem it;
        for (; ok && feed.take(it); ++items) {
            auto cols_of = [&](int j) { return mma_cols(it.end - j * TILE); };
            auto scores = [&](int j, uint32_t c) {
                ok = ok && wait_warp<true>(smem_u32(&ctl->k_full[c % KS]), (c / KS) & 1, waits, SITE_MMA_FULL);
                if (!ok) return;
                tc_fence_after();
                mma_rows_rows<DP>(on, tmem + (c & 1) * TILE, q_desc, k_desc + (c % KS) * (T_BYTES >> 4), idesc_rows(cols_of(j)));
                umma_commit_if(on, smem_u32(&ctl->s_full[c & 1]));
                if (j == it.nb - 1) umma_commit_if(on, smem_u32(&ctl->q_empty));
            };
            auto grad_scores = [&](int j, uint32_t c) {
                ok = ok && wait_warp<true>(smem_u32(&ctl->v_full[c % VS]), (c / VS) & 1, waits, SITE_MMA_FULL);
                if (!ok) return;
                tc_fence_after();
                mma_rows_rows<DP>(on, t_dp, g_desc, v_desc + (c % VS) * (T_BYTES >> 4), idesc_rows(cols_of(j)));
                umma_commit_if(on, smem_u32(&ctl->g_scores));
                umma_commit_if(on, smem_u32(&ctl->v_empty[c % VS]));
                if (j == it.nb - 1) umma_commit_if(on, smem_u32(&ctl->g_empty));
            };
            ok = wait_warp<true>(smem_u32(&ctl->q_full), items & 1, waits, SITE_MMA_FULL);
            scores(0, cnt);
            ok = ok && wait_warp<true>(smem_u32(&ctl->g_full), items & 1, waits, SITE_MMA_FULL);
            grad_scores(0, cnt);
            if (it.nb > 1) scores(1, cnt + 1);
            for (int j = 0; j < it.nb && ok; ++j, ++cnt) {
                ok = wait_warp<true>(smem_u32(&ctl->ds_ready), cnt & 1, waits, SITE_MMA_FULL);
                if (!ok) break;
                if (j + 1 < it.nb) grad_scores(j + 1, cnt + 1);
                if (ok && j == 0)
                    ok = wait_warp<true>(smem_u32(&ctl->acc_free), (items & 1) ^ 1, waits, SITE_MMA_TMEM_EMPTY);
                if (!ok) break;
                tc_fence_after();
                const uint32_t ds = tmem + (cnt & 1) * TILE;
                mma_tmem_rows<DP, 0, 8, 2>(on, t_dq, ds, k_across + (cnt % KS) * (T_BYTES >> 4), cols_of(j) / 16, j > 0);
                mma_tmem_rows<DP, 0, 8, 2>(on, t_dq, ds + 16, k_across + (cnt % KS) * (T_BYTES >> 4), cols_of(j) / 16, 1);
                umma_commit_if(on, smem_u32(&ctl->k_empty[cnt % KS]));
                if (j + 2 < it.nb) scores(j + 2, cnt + 2);
            }
            if (!ok) break;
            umma_commit_if(on, smem_u32(&ctl->acc_full));
        }
    } else if (warp >= BwdWarps::FIRST) {
        regs_up<BwdWarps::REGS_ARITH>();
        const int part = (warp - BwdWarps::FIRST) >> 2, row = (warp & 3) * 32 + lane, c0 = 32 * part;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        const int row_t = row / p.group, row_h = row - row_t * p.group;
        uint32_t cnt = 0, items = 0;
        bool ok = true;
        Feed<QItem, true> feed(p);
        QItem it;
        for (; ok && feed.take(it); ++items) {
            float2 *stats = p.row_stats + ((int64_t)it.tile * p.hk + it.h) * TILE + row;
            const float2 st = *stats;
            float sum = 0.0f, delta = st.y;  // sum: of this part's dS
            const int token = it.t0 + row_t, row_end = p.causal ? min(token + 1, it.len) : it.len;
            const bool live = row < used && token < it.len, whole = it.nb == 1;
            // The four parts' values of a row meet in `sums`: put in and, when all are there, added up.
            auto put = [&](float v) {
                ok = ok && wait_warp<true>(smem_u32(&ctl->sum_read), (items & 1) ^ 1, waits, SITE_EPI_EXCHANGE);
                if (!ok) return;
                asm volatile("st.shared.f32 [%0], %1;" ::"r"(sums + (part * TILE + row) * 4), "f"(v) : "memory");
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&ctl->sum_ready));
            };
            auto total = [&]() {
                ok = ok && wait_warp<true>(smem_u32(&ctl->sum_ready), items & 1, waits, SITE_EPI_EXCHANGE);
                if (!ok) return 0.0f;
                float s4[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) asm volatile("ld.shared.f32 %0, [%1];" : "=f"(s4[k]) : "r"(sums + (k * TILE + row) * 4) : "memory");
                return (s4[0] + s4[1]) + (s4[2] + s4[3]);
            };
            auto done = [&]() {
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&ctl->sum_read));
            };
            if (whole) {                     // ahead of the loop, which sees the same phases and looks at P and dP again
                ok = wait_warp<true>(smem_u32(&ctl->s_full[cnt & 1]), (cnt >> 1) & 1, waits, SITE_EPI_TMEM_FULL);
                ok = ok && wait_warp<true>(smem_u32(&ctl->g_scores), cnt & 1, waits, SITE_EPI_TMEM_FULL);
                if (!ok) break;
                tc_fence_after();
                float t = 0.0f, first = 0.0f;
#pragma unroll 1
                for (int c = c0; c < min(c0 + 32, mma_cols(it.end)); c += 16) {
                    uint32_t x[16], y[16];
                    tmem_ld16(tmem + lanes + (cnt & 1) * TILE + c, x);
                    tmem_ld16(t_dp + lanes + c, y);
                    tmem_ld_wait(x);
                    tmem_ld_wait(y);
                    if (c == 0) first = __uint_as_float(y[0]);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float v = fast_exp2(fmaf(__uint_as_float(x[e]), p.c2, -st.x)) * __uint_as_float(y[e]);
                        t += c + e < row_end ? v : 0.0f;
                    }
                }
                put(t);
                delta = total();
                if (!ok) break;
                done();
                if (row_end == 1) delta = first;
            }
            for (int j = 0; j < it.nb; ++j, ++cnt) {
                const int cols = mma_cols(it.end - j * TILE);
                const bool mask = cols < TILE || j * TILE + TILE > (p.causal ? it.t0 + 1 : it.len);
                const int limit = row_end - j * TILE - c0;
                ok = wait_warp<true>(smem_u32(&ctl->s_full[cnt & 1]), (cnt >> 1) & 1, waits, SITE_EPI_TMEM_FULL);
                ok = ok && wait_warp<true>(smem_u32(&ctl->g_scores), cnt & 1, waits, SITE_EPI_TMEM_FULL);
                if (!ok) break;
                tc_fence_after();
                if (c0 < cols) {
                    const uint32_t t_s = tmem + lanes + (cnt & 1) * TILE + c0;
                    uint32_t r[32], dp[32], hi[16], lo[16];
                    tmem_ld32(t_s, r);
                    tmem_ld32(t_dp + lanes + c0, dp);
                    tmem_ld_wait(r);
                    tmem_ld_wait(dp);
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float a = fast_exp2(fmaf(__uint_as_float(r[e]), p.c2, -st.x)) * (__uint_as_float(dp[e]) - delta);
                        float b = fast_exp2(fmaf(__uint_as_float(r[e + 1]), p.c2, -st.x)) * (__uint_as_float(dp[e + 1]) - delta);
                        if (mask) {
                            a = e < limit ? a : 0.0f;
                            b = e + 1 < limit ? b : 0.0f;
                        }
                        sum += a + b;
                        hi[e / 2] = pack_bf16(a, b);
                        lo[e / 2] = pack_bf16(a - __uint_as_float(hi[e / 2] << 16), b - __uint_as_float(hi[e / 2] & 0xffff0000u));
                    }
                    tmem_st16(t_s, hi);
                    tmem_st16(t_s + 16, lo);
                    tmem_st_wait();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&ctl->ds_ready));
            }
            if (!ok) break;
            ok = wait_warp<true>(smem_u32(&ctl->acc_full), items & 1, waits, SITE_EPI_TMEM_FULL);
            if (!ok) break;
            tc_fence_after();
            // part 0 puts the row's delta right for the kernel of dK and dV
            if (!whole) {
                put(sum);
                if (part == 0) delta += total();
                if (!ok) break;
                done();
            }
            if (part == 0 && live) stats->y = delta;
            if (c0 < DP) {
                uint32_t o[32];
                tmem_ld32(t_dq + lanes + c0, o);
                tmem_ld_wait(o);
                bf16 *dst = p.out0 + ((int64_t)it.start + token) * p.ld0 + (int64_t)(it.h * p.group + row_h) * p.d + c0;
#pragma unroll
                for (int k = 0; k < 4; k += 2) {
                    const uint4 a = pack8(o + 8 * k, p.scale), b = pack8(o + 8 * k + 8, p.scale);
                    if (live && c0 + 8 * k < p.d) {
                        if (p.wide)                  // 32 bytes per lane: whole sectors (there is no room to stage rows here)
                            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(dst + 8 * k), "r"(a.x), "r"(a.y),
                                         "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w)
                                         : "memory");
                        else {
                            *reinterpret_cast<uint4 *>(dst + 8 * k) = a;
                            if (c0 + 8 * k + 8 < p.d) *reinterpret_cast<uint4 *>(dst + 8 * k + 8) = b;
                        }
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_u32(&ctl->acc_free));
        }
    }
    cta_teardown(waits.abort_flag, ctl->tmem_base, BwdWarps::MMA);
}

// ------------------------------------------------------------------------------------ host
// [N, heads, d] bf16 with a token stride of `ld` elements; box = 64 columns x box_heads x box_tokens
static bool head_map(CUtensorMap *m, const void *base, int d, int heads, int64_t N, int64_t ld, int box_heads, int box_tokens)
{
    EncodeTiledFn enc = get_encode();
    if (!enc || !base) return false;
    cuuint64_t dims[3] = {(cuuint64_t)d, (cuuint64_t)heads, (cuuint64_t)N};
    cuuint64_t strides[2] = {(cuuint64_t)d * 2, (cuuint64_t)ld * 2};
    cuuint32_t box[3] = {64u, (cuuint32_t)box_heads, (cuuint32_t)box_tokens}, es[3] = {1u, 1u, 1u};
    return enc(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(base), dims, strides, box, es,
               CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

constexpr int AT_MAX_DEVICES = 64;

template <typename Kernel>
static cudaError_t launch_at(Kernel kern, int threads, int *sms_by_dev, int smem, const AtMaps &tm, const AtParams &p, cudaStream_t s)
{
    if (p.n_items <= 0) return cudaSuccess;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= AT_MAX_DEVICES) return cudaErrorInvalidDevice;
    if (sms_by_dev[dev] == 0) {
        int n = 0;
        cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
        if (e == cudaSuccess) e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
        if (e != cudaSuccess) return e;
        sms_by_dev[dev] = n;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.n_items < sms_by_dev[dev] ? p.n_items : sms_by_dev[dev]));
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, tm, p);
}

static AtParams params_of(const AttnArgs &a, const int4 *items, int n)
{
    AtParams p = {};
    p.items = items; p.n_items = n * a.hk;
    p.hq = a.hq; p.hk = a.hk; p.group = a.group; p.tokens = a.tokens; p.d = a.d; p.causal = a.causal;
    p.scale = a.scale; p.c2 = a.scale * LOG2E;
    p.status = a.status; p.row_stats = a.row_stats;
    p.wait_ns = (uint32_t)a.wait_us * 1000u; p.lose = a.lose_load ? 16 : 0;
    return p;
}

template <int DP> static cudaError_t forward_dp(const AttnArgs &a, cudaStream_t s)
{
    static int sms[AT_MAX_DEVICES];
    AtMaps tm;
    if (!head_map(&tm.q, a.q, a.d, a.hq, a.N, a.ldq, a.group, a.tokens) || !head_map(&tm.k, a.k, a.d, a.hk, a.N, a.ldk, 1, TILE) ||
        !head_map(&tm.v, a.v, a.d, a.hk, a.N, a.ldv, 1, TILE))
        return cudaErrorInvalidValue;
    tm.g = tm.q;
    AtParams p = params_of(a, a.fwd_items, a.n_fwd);
    p.out0 = (bf16 *)a.out; p.ld0 = a.ldo; p.lse = a.lse;
    return launch_at(k_attention_fwd<DP>, FwdWarps::THREADS, sms, FwdShape<DP>::SMEM, tm, p, s);
}

template <int DP> static cudaError_t backward_dp(const AttnArgs &a, cudaStream_t s)
{
    static int sms_kv[AT_MAX_DEVICES], sms_q[AT_MAX_DEVICES];
    AtMaps tm;
    if (!head_map(&tm.q, a.q, a.d, a.hq, a.N, a.ldq, a.group, a.tokens) || !head_map(&tm.k, a.k, a.d, a.hk, a.N, a.ldk, 1, TILE) ||
        !head_map(&tm.v, a.v, a.d, a.hk, a.N, a.ldv, 1, TILE) || !head_map(&tm.g, a.dout, a.d, a.hq, a.N, a.lddo, a.group, a.tokens))
        return cudaErrorInvalidValue;
    cudaError_t e = launch_attention_row_stats_tc(a, s);
    if (e != cudaSuccess) return e;
    AtParams p = params_of(a, a.row_items, a.n_rows);
    p.out0 = (bf16 *)a.dq; p.ld0 = a.lddq;
    p.wide = ((uintptr_t)a.dq & 31u) == 0 && a.lddq % 16 == 0 && a.d % 16 == 0;
    e = launch_at(k_attention_bwd_q<DP>, BwdWarps::THREADS, sms_q, QShape<DP>::SMEM, tm, p, s);
    if (e != cudaSuccess) return e;
    p = params_of(a, a.key_items, a.n_keys);
    p.out0 = (bf16 *)a.dk; p.ld0 = a.lddk; p.out1 = (bf16 *)a.dv; p.ld1 = a.lddv;
    return launch_at(k_attention_bwd_kv<DP>, BwdWarps::THREADS, sms_kv, KvShape<DP>::SMEM, tm, p, s);
}

cudaError_t launch_attention_tc_forward(const AttnArgs &a, cudaStream_t s)
{
    return a.d <= 64 ? forward_dp<64>(a, s) : forward_dp<128>(a, s);
}
cudaError_t launch_attention_tc_backward(const AttnArgs &a, cudaStream_t s)
{
    return a.d <= 64 ? backward_dp<64>(a, s) : backward_dp<128>(a, s);
}

}  // namespace skipffn
