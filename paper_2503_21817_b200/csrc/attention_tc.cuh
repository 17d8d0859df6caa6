// What the tensor-core attention kernels (attention_tc.cu, paged_tc.cu) share: roles and bounded waits, tiles in shared
// memory and their descriptors, products, the softmax of a block of scores in tensor memory, stores of whole lines.
#pragma once
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

struct alignas(64) AtMaps { CUtensorMap q, k, v, g; };

template <int DP> constexpr int tile_bytes() { return TILE * DP * 2; }

__device__ __forceinline__ int uniform(int v) { return __shfl_sync(0xffffffffu, v, 0); }
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

// ---- forward: two row tiles against a ring of key and value tiles
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

// ---- host
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

}  // namespace

}  // namespace skipffn
