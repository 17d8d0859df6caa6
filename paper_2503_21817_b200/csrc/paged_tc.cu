// Attention over a paged cache on the tensor cores (bf16): sequences with more than 16 rows, the chunks of a prompt.
//
// The softmax of two row tiles (2 x 128 rows: tokens x query heads of a kv head) against a ring of key and value tiles, as
// in the packed forward (roles, registers and the block's softmax are the same code).  What differs:
//   * a tile of 128 keys comes from several pages: the lanes of the TMA warp look their pages up a tile ahead and issue one
//     box each (gcd(page_size, 128) rows); a page that does not exist is a coordinate outside the pool, which reads as zeros
//   * a chunk is short and its cache long, so work is cut along the keys: the units (a tile pair's blocks of keys, over
//     all tiles and heads of the call, listed on the device by k_paged_list) are one line in equal runs, one per SM.  A pair
//     that lies in one run is written at once, pieces go to scratch in fp32 and are joined by k_paged_join.  The few pieces
//     at the ends of runs cost 256 rows x 512 bytes each; runs of whole pairs would leave up to half of the SMs idle
//     (32 pairs of rows and 8 heads on 148 SMs)
//   * tokens see up to their own row: only the last blocks of a pair are masked
// Bound by the chain of a block (product, softmax, product), as there.  Measured, 32 / 8 heads, head_dim 128: 2000 tokens
// over a cache of 16 345 rows 459 us with the list and the join (1.10 PFLOP/s), 16 381 tokens of one prompt 2.0 ms.  Sequences of
// one row tile (17 to 128 rows) have nothing beside its chain: 128 us for 48 conversations of 37 to 8877 rows, whatever
// their rows or pages.  Two blocks of such a tile at a time were slower (146 us): four tiles of keys and values in shared
// memory are then all in use, and none is left to load behind the products.
#include "paged_tma.cuh"

namespace skipffn {

namespace {

struct PagedTcParams {
    PagedAttnArgs a;
    int32_t tokens, box;                     // tokens of a row tile; rows of a TMA box
    float c2;
};
struct alignas(64) PagedMaps { CUtensorMap q, k, v; };

// A run's part of a tile pair: blocks b0 .. b1 - 1 of head h
struct Piece {
    int q0, n, len, s, t0, h, blocks, b0, b1;
    int nb0, nb1, end0, end1;                // of the row tiles: blocks in all, first key past the keys of their last token
    __device__ int past(int g) const { return g ? end1 : end0; }
    __device__ int all(int g) const { return g ? nb1 : nb0; }
    __device__ int count(int g) const { return max(0, min(all(g), b1) - b0); }
    __device__ int loads() const { return b1 - b0; }
    __device__ bool whole() const { return b0 == 0 && b1 == blocks; }
    // value rows past the sequence inside the last 16-row step of the last block
    __device__ bool dirty_tail() const { return (len & 15) != 0 && b1 * TILE > len; }
    // columns that the MMA covers in the last block of this piece for tile g
    __device__ int last_cols(int g) const { return b1 >= all(g) ? mma_cols(past(g) - (all(g) - 1) * TILE) : TILE; }
};

// Walks the pieces of this CTA's run, the same in every role
template <bool WARP> struct PieceFeed {
    const PagedTcParams &p;
    Runs runs;
    int64_t u, end;
    int t = 0;
    PagedTile e;
    __device__ explicit PieceFeed(const PagedTcParams &p_) : p(p_), runs(*p_.a.head, p_.a.runs)
    {
        u = runs.begin(blockIdx.x);
        end = runs.begin(blockIdx.x + 1);
        if (u >= end) return;
        t = p.a.starts[blockIdx.x];
        e = p.a.tiles[t];
    }
    __device__ bool take(Piece &w)
    {
        do {
            if (u >= end) return false;
            const int seg = e.blocks + PG_TILE_COST;
            const int64_t in = u - e.u0;
            if (e.blocks == 0 || in >= (int64_t)seg * p.a.c.heads) {
                e = p.a.tiles[++t];
                w.b0 = w.b1 = 0;
                continue;
            }
            w.blocks = pick(e.blocks);
            w.h = pick((int)(in / seg));
            const int p0 = pick((int)(in - (int64_t)w.h * seg)), p1 = pick((int)min((int64_t)seg, p0 + (end - u)));
            w.b0 = max(0, p0 - PG_TILE_COST);
            w.b1 = max(0, p1 - PG_TILE_COST);
            u += p1 - p0;
        } while (w.b1 <= w.b0);              // the run may end before the tile's first block
        w.q0 = pick(e.q0); w.n = pick(e.n); w.len = pick(e.len); w.s = pick(e.s);
        w.t0 = pick(e.r0 / p.a.group);
        const int t1 = w.t0 + p.tokens, off = w.len - w.n;
        w.end0 = max(0, off + min(t1, w.n));
        w.end1 = t1 < w.n ? max(0, off + min(t1 + p.tokens, w.n)) : 0;
        w.nb0 = ceil_div(w.end0, TILE);
        w.nb1 = ceil_div(w.end1, TILE);
        return true;
    }
    __device__ static int pick(int v) { return WARP ? uniform(v) : v; }
};

template <int DP>
__global__ void __launch_bounds__(FwdWarps::THREADS, 1)
k_paged_tc(const __grid_constant__ PagedMaps tm, const __grid_constant__ PagedTcParams p)
{
    constexpr int T_BYTES = FwdShape<DP>::T_BYTES, SLOTS = FwdShape<DP>::SLOTS;
    extern __shared__ __align__(1024) uint8_t smem_raw[];      // tiles need 1024 bytes
    const uint32_t tiles = smem_u32(smem_raw), q_tile = tiles, ring = tiles + 2 * T_BYTES;
    FwdCtl *ctl = reinterpret_cast<FwdCtl *>(smem_raw + (2 + SLOTS) * T_BYTES + 8 * FwdShape<DP>::STAGE);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const PagedAttnArgs &a = p.a;
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
    const int used = a.group * p.tokens;     // rows of a tile that a box fills; the others stay zero
    if (used < TILE) zero_smem(q_tile, 2 * T_BYTES);
    fence_proxy_async_smem();
    if (warp == FwdWarps::MMA) { tmem_alloc(smem_u32(&ctl->tmem_base), AT_TMEM_COLS); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const Waits waits{&ctl->abort_flag, &ctl->issued, a.c.status, (uint32_t)WAIT_LIMIT_NS};
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");

    if (warp < FwdWarps::FIRST) regs_down<FwdWarps::REGS_SERVICE>();
    if (warp == FwdWarps::TMA) {
        uint32_t pos = 0, nq[2] = {0, 0};
        bool ok = true;
        const PageBoxes boxes{a.c, p.box, lane};
        auto acquire = [&]() {               // next ring slot, free to be written
            const uint32_t s = pos % SLOTS;
            ok = ok && wait_warp<true>(smem_u32(&ctl->kv_empty[s]), ((pos / SLOTS) & 1) ^ 1, waits, SITE_PRODUCER_EMPTY);
            ++pos;
            return s;
        };
        auto load_q = [&](const Piece &it, int g) {
            ok = ok && wait_warp<true>(smem_u32(&ctl->q_empty[g]), (nq[g] & 1) ^ 1, waits, SITE_PRODUCER_EMPTY);
            if (!ok) return;
            if (lane == 0) {
                const uint32_t bar = smem_u32(&ctl->q_full[g]);
                mbar_expect_tx(bar, (uint32_t)(used * DP * 2));
                load_tile<DP>(q_tile + g * T_BYTES, &tm.q, it.h * a.group, it.q0 + it.t0 + g * p.tokens, bar);
            }
            ++nq[g];
        };
        PieceFeed<true> feed(p);
        Piece it;
        while (ok && feed.take(it)) {
            PageBox box = boxes.find(it.s, it.len, it.b0 * TILE), next = box;
            for (int j = it.b0; j < it.b1 && ok; ++j) {
                boxes.check(box);
                if (j == it.b0 && it.count(0)) load_q(it, 0);
                if (j + 1 < it.b1) next = boxes.find(it.s, it.len, (j + 1) * TILE);
                uint32_t s = acquire();
                if (!ok) break;
                boxes.load<DP>(ring + s * T_BYTES, &tm.k, smem_u32(&ctl->kv_full[s]), box, it.h);
                if (j == it.b0 && it.count(1)) load_q(it, 1);
                s = acquire();
                if (!ok) break;
                // the tail warp passes a tile with rows to zero on to the MMA warp
                boxes.load<DP>(ring + s * T_BYTES, &tm.v, smem_u32(j == it.b1 - 1 && it.dirty_tail() ? &ctl->tail[s] : &ctl->kv_full[s]), box, it.h);
                if (lane == 0) ctl->issued = pos;
                box = next;
            }
        }
    } else if (warp == FwdWarps::TAIL) {
        if (lane == 0) a.cuts[blockIdx.x].pieces = 0;
        uint32_t pos = 0, seen = 0;          // bit s: parity of the tail events of slot s
        bool ok = true;
        PieceFeed<true> feed(p);
        Piece it;
        while (ok && feed.take(it)) {
            const int n = it.loads();
            pos += 2 * n;
            if (it.b0 == 0 && it.b1 < it.blocks && lane == 0) {
                PagedCut cut = {};
                cut.q0 = it.q0; cut.r0 = it.t0 * a.group; cut.h = it.h; cut.first = blockIdx.x;
                cut.rows = min(2 * used, it.n * a.group - cut.r0);
                cut.pieces = feed.runs.of(feed.u + (it.blocks - it.b1) - 1) - (int)blockIdx.x + 1;
                a.cuts[blockIdx.x] = cut;
            }
            if (!it.dirty_tail()) continue;
            const uint32_t s = (pos - 1) % SLOTS;
            ok = wait_warp<false>(smem_u32(&ctl->tail[s]), (seen >> s) & 1, waits, SITE_PRODUCER_EMPTY);
            if (!ok) break;
            seen ^= 1u << s;
            const int valid = it.len - (it.b1 - 1) * TILE;
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
        PieceFeed<true> feed(p);
        Piece it;
        while (ok && feed.take(it)) {
            const int n = it.loads();
            const int nb[2] = {it.count(0), it.count(1)};
            const int last_cols[2] = {it.last_cols(0), it.last_cols(1)};
            auto scores = [&](int g, int j, uint32_t k_slot) {
                mma_rows_rows<DP>(on, tmem + g * TILE, q_desc + g * (T_BYTES >> 4), k_desc0 + k_slot * (T_BYTES >> 4),
                                  idesc_rows(j == nb[g] - 1 ? last_cols[g] : TILE));
                umma_commit_if(on, smem_u32(&ctl->s_full[g]));
            };
            wait_slot();
            uint32_t ks = next_slot();
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                if (!ok) break;
                if (nb[g] == 0) continue;
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
        const uint32_t stage = ring + SLOTS * T_BYTES + (warp - FwdWarps::FIRST) * FwdShape<DP>::STAGE;
        uint32_t ns = 0, no = 0;
        bool ok = true;
        const int row_t = row / a.group, row_h = row - row_t * a.group;
        PieceFeed<true> feed(p);
        Piece it;
        while (ok && feed.take(it)) {
            const int nb = it.count(g), t0 = it.t0 + g * p.tokens, token = t0 + row_t;
            const int off = it.len - it.n;
            const int row_end = min(off + token + 1, it.len);                 // keys of this row
            const bool live = row < used && token < it.n;                     // a query of this sequence
            const bool whole = it.whole();
            const int64_t tok = (int64_t)it.q0 + token;
            const int head = it.h * a.group + row_h;
            // where a piece's sums go
            const int64_t part = ((int64_t)(2 * blockIdx.x + (it.b0 == 0 ? 1 : 0)) * PG_TC_ROWS + g * used + row);
            float m = -INFINITY, l = 0.0f;
            if (nb > 0) {
                for (int j = 0; j < nb; ++j) {
                    ok = wait_warp<true>(s_full, ns & 1, waits, SITE_EPI_TMEM_FULL);
                    ++ns;
                    if (!ok) break;
                    tc_fence_after();
                    // columns past the row's keys (or past the ones the MMA wrote) count as minus infinity
                    const int j0 = (it.b0 + j) * TILE;
                    const bool upper = it.past(g) - j0 > 64;
                    const int from = off + t0 + 1 - j0, to = upper ? TILE : 64;
                    if (from < to) mask_scores(t_s, from, to, row_end - j0);
                    softmax_block<DP>(t_s, t_o, upper, live, p.c2, j == 0, m, l, p_full, lane);
                }
                if (!ok) break;
                ok = wait_warp<true>(smem_u32(&ctl->o_full[g]), no & 1, waits, SITE_EPI_TMEM_FULL);
                ++no;
                if (!ok) break;
                tc_fence_after();
            }
            const bool none = met_nothing(m, l);     // keys that it does not see among them
            if (whole) {
                const float inv = none ? 0.0f : 1.0f / l;
                bf16 *dst = live ? (bf16 *)a.out + tok * a.ldo + (int64_t)head * a.c.d : nullptr;
#pragma unroll 1
                for (int c = 0; c < DP; c += 64) {
                    uint32_t o[32];
                    uint4 w[8];
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        tmem_ld32(t_o + c + 32 * h, o);      // of the tile before, when no block was met: not used then
                        tmem_ld_wait(o);
#pragma unroll
                        for (int k = 0; k < 4; ++k) w[4 * h + k] = none ? make_uint4(0, 0, 0, 0) : pack8(o + 8 * k, inv);
                    }
                    store_rows<8>(stage, lane, w, dst ? dst + c : nullptr, (a.c.d - c) / 8);
                }
                if (live) a.lse[tok * a.hq + head] = none ? -INFINITY : fmaf(m, a.scale, logf(l));
            } else {
                if (nb > 0) {
                    float *dst = live ? a.part + part * DP : nullptr;
#pragma unroll 1
                    for (int c = 0; c < DP; c += 32) {
                        uint32_t o[32];
                        uint4 w[8];
                        tmem_ld32(t_o + c, o);
                        tmem_ld_wait(o);
#pragma unroll
                        for (int k = 0; k < 8; ++k) w[k] = make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
                        store_rows<8>(stage, lane, w, dst ? reinterpret_cast<bf16 *>(dst + c) : nullptr, 8);
                    }
                }
                if (live) a.part_ml[part] = make_float2(m, l);
            }
            if (nb > 0) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&ctl->o_free[g]));
            }
        }
    }
    cta_teardown(waits.abort_flag, ctl->tmem_base, FwdWarps::MMA);
}

template <int DP> cudaError_t tc(const PagedAttnArgs &args, cudaStream_t s)
{
    static int sms_of_device[64];
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= 64) return cudaErrorInvalidDevice;
    if (sms_of_device[dev] == 0) {
        int n = 0;
        cudaError_t e = cudaFuncSetAttribute(k_paged_tc<DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, FwdShape<DP>::SMEM);
        if (e == cudaSuccess) e = cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev);
        if (e != cudaSuccess) return e;
        sms_of_device[dev] = n < PG_TC_RUNS ? n : PG_TC_RUNS;
    }
    PagedTcParams p = {};
    p.a = args;
    p.a.runs = sms_of_device[dev];
    p.tokens = TILE / args.group;
    p.box = box_rows(args.c);
    p.c2 = args.scale * LOG2E;
    PagedMaps tm;
    if (!head_map(&tm.q, args.q, args.c.d, args.hq, args.c.N, args.ldq, args.group, p.tokens) || !pool_map(&tm.k, args.c.k, args.q, args.c, p.box) ||
        !pool_map(&tm.v, args.c.v, args.q, args.c, p.box))
        return cudaErrorInvalidValue;
    cudaError_t e = launch_paged_list(p.a, 2 * p.tokens * args.group, TILE, s);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.a.runs); cfg.blockDim = dim3(FwdWarps::THREADS); cfg.dynamicSmemBytes = FwdShape<DP>::SMEM; cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    e = cudaLaunchKernelEx(&cfg, k_paged_tc<DP>, tm, p);
    return e != cudaSuccess ? e : launch_paged_join(p.a, PG_TC_ROWS, DP, s);
}

}  // namespace

cudaError_t launch_paged_tc(const PagedAttnArgs &a, cudaStream_t s) { return a.c.d <= 64 ? tc<64>(a, s) : tc<128>(a, s); }

}  // namespace skipffn
