// The softmax weight that every row of a paged cache gets from the new tokens of its sequence, per kv head, bf16:
//
//   weights[s, h, j] = prior + sum over new rows r of the head's group that see j of exp(scale q_r . k_j - lse_r)
//
// The forward's logarithms are given, so one pass over the keys suffices, and the sum over rows stays inside a CTA: no
// atomics, a fixed order.  One CTA: 64 keys against all rows of its sequence, 32 rows at a time.  Keys are the rows of the
// products' accumulators (mma.sync: for one token per sequence the keys are read once for 2 x 4 flops a value, far from
// any matrix limit), so a thread adds its exponentials up as they come.  For few rows it is bound by reading the keys, with
// many CTAs an SM to keep loads in flight; for many by the exponentials (16 a cycle and SM).
#include "paged.cuh"
#include "paged_mma.cuh"

namespace skipffn {

namespace {

constexpr int THREADS = 128, KEYS = 64, ROWS = 32;

template <int DP> struct WeightsShape { static constexpr int KEY_BYTES = KEYS * DP * 2, ROW_BYTES = ROWS * DP * 2; };

template <int DP> __global__ void __launch_bounds__(THREADS) k_paged_weights(const PagedWeightsArgs a)
{
    using Sh = WeightsShape<DP>;
    constexpr int CHUNKS = DP / 8, STEP = THREADS / CHUNKS;
    __shared__ __align__(128) uint8_t keys[Sh::KEY_BYTES], rows_smem[2][Sh::ROW_BYTES];
    __shared__ float lses[2][ROWS];
    pdl_enter();
    const PagedView &c = a.c;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int s = blockIdx.z, h = blockIdx.y, j0 = blockIdx.x * KEYS;
    const bool reporter = blockIdx.x == 0 && h == 0 && tid == 0;
    const PagedSeq q = paged_seq(c, s, reporter);
    if (reporter && q.len > a.width) paged_report(c, SITE_PAGED_WIDTH);
    const int rows = q.n * a.group, off = q.len - q.n;
    const int64_t at = ((int64_t)s * c.heads + h) * a.width;
    float total[2] = {0.0f, 0.0f};                       // of this thread's two keys
    // the first row that sees any of these keys
    const int first = max(0, j0 - off) * a.group / ROWS * ROWS;
    if (j0 < q.len && first < rows) {
        const int chunk = tid % CHUNKS, r0 = tid / CHUNKS;
        int64_t base = -1;                               // lane i < 8: rows 8 i .. 8 i + 7
        if (lane < KEYS / 8 && j0 + 8 * lane < q.len) {
            base = paged_row(c, s, j0 + 8 * lane);
            if (base >= 0) base += h * c.head_stride;
            else paged_report(c, SITE_PAGED_PAGE);
        }
#pragma unroll
        for (int i = 0; i < KEYS / STEP; ++i) {
            const int r = r0 + i * STEP;
            const int64_t g = __shfl_sync(0xffffffffu, base, r >> 3);
            const bool on = g >= 0 && j0 + r < q.len && chunk * 8 < c.d;
            copy16(smem_u32(keys) + chunk_at<DP>(r, chunk), c.k + (on ? g + (r & 7) * c.row_stride + chunk * 16 : 0), on);
        }
        auto issue = [&](int t0, int buf) {
            if (t0 < rows) {
                for (int i = r0; i < ROWS; i += STEP) {
                    const int r = t0 + i;
                    const bool on = r < rows && chunk * 8 < c.d;
                    const bf16 *src = (const bf16 *)a.q;
                    if (on) src += (int64_t)(q.q0 + r / a.group) * a.ldq + (int64_t)(h * a.group + r % a.group) * c.d + chunk * 8;
                    copy16(smem_u32(rows_smem[buf]) + chunk_at<DP>(i, chunk), src, on);
                }
                if (tid < ROWS) {
                    // a row without a logarithm (it sees nothing) and a row that is not there weigh nothing
                    const int r = t0 + tid;
                    const float l = r < rows ? a.lse[(int64_t)(q.q0 + r / a.group) * a.hq + h * a.group + r % a.group] : INFINITY;
                    lses[buf][tid] = l == -INFINITY ? INFINITY : l;
                }
            }
            copy_commit();
        };
        issue(first, 0);
        uint32_t kf[DP / 16][4];
        const int key = warp * 16 + (lane >> 2);         // and key + 8
        for (int t0 = first, buf = 0; t0 < rows; t0 += ROWS, buf ^= 1) {
            issue(t0 + ROWS, buf ^ 1);
            copy_wait<1>();
            __syncthreads();
            if (t0 == first)
#pragma unroll
                for (int k = 0; k < DP / 16; ++k) {
                    // rows of a: lanes 0-7 keys 0-7, 8-15 keys 8-15 of the same columns, 16-31 the next eight columns
                    ldsm_x4(smem_u32(keys) + chunk_at<DP>(warp * 16 + (lane & 15), 2 * k + (lane >> 4)), kf[k]);
                }
            const bool masked = j0 + KEYS - 1 > off + t0 / a.group;
#pragma unroll
            for (int n = 0; n < ROWS / 8; n += 2) {
                if (t0 + 8 * n >= rows) break;
                float x[2][4] = {};
#pragma unroll
                for (int k = 0; k < DP / 16; ++k) {
                    uint32_t b[4];
                    ldsm_x4(smem_u32(rows_smem[buf]) + chunk_at<DP>(n * 8 + (lane >> 4) * 8 + (lane & 7), 2 * k + ((lane >> 3) & 1)), b);
                    mma_16x8(x[0], kf[k], b[0], b[1]);
                    mma_16x8(x[1], kf[k], b[2], b[3]);
                }
#pragma unroll
                for (int y = 0; y < 2; ++y)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int i = 8 * (n + y) + 2 * (lane & 3) + (e & 1);
                        // the difference first: it is small where the weight counts, so its rounding is too
                        float w = fast_exp2(fmaf(x[y][e], a.scale, -lses[buf][i]) * 1.4426950408889634f);
                        if (masked && j0 + key + 8 * (e >> 1) > off + (t0 + i) / a.group) w = 0.0f;
                        total[e >> 1] += w;
                    }
            }
            __syncthreads();                             // the rows have been read
        }
        copy_wait<0>();
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        total[i] += __shfl_xor_sync(0xffffffffu, total[i], 1);
        total[i] += __shfl_xor_sync(0xffffffffu, total[i], 2);
        const int j = j0 + warp * 16 + (lane >> 2) + 8 * i;
        if ((lane & 3) == 0 && j < a.width) a.out[at + j] = j < q.len ? (a.prior ? a.prior[at + j] : 0.0f) + total[i] : 0.0f;
    }
}

}  // namespace

cudaError_t launch_paged_weights(const PagedWeightsArgs &a, cudaStream_t s)
{
    const dim3 grid((unsigned)((a.width + KEYS - 1) / KEYS), (unsigned)a.c.heads, (unsigned)a.c.n_seq);
    return a.c.d <= 64 ? launch_pdl(k_paged_weights<64>, grid, dim3(THREADS), s, a) : launch_pdl(k_paged_weights<128>, grid, dim3(THREADS), s, a);
}

}  // namespace skipffn
