// Queries and keys of every head normalised (RMS norm) and rotated by position in one pass, its gradients, and the
// form that writes the rotated keys and the values into a paged cache.
//
//   n = x r gamma, r = 1 / sqrt(mean x^2 + eps)   (no gamma: n = x)
//   pair (a, b) of n -> (a cos t - b sin t, b cos t + a sin t),  t = position[axis of the pair] * frequency of the pair
//   backward: dn = the pair rotated by -t; dgamma = sum dn x r; u = dn gamma; dx = r (u - x r^2 mean(u x))
//
// Angles: a frequency is kept as turns per position in 64-bit fixed point (a fraction of a full turn), so position *
// frequency modulo one turn is one integer multiplication that drops what overflows: the angle's error does not grow
// with the position beyond that of the frequency's last bit (2^-65 of a turn each position).  The quadrant is taken from
// the top bits and the rest goes to sincospi.  A CTA computes the table of its tokens once, for all their heads.
//
// Bound by memory: every row is read and written once.  A group of lanes holds a row, each lane V pairs of it (two
// 16-byte vectors where the sizes allow), so the sums of a row are shuffles inside the group.
#include <math.h>

#include <initializer_list>
#include <new>

#include "arrays.cuh"
#include "paged.cuh"

namespace skipffn {

constexpr int RT_MAX_D = 256, RT_MAX_PAIRS = RT_MAX_D / 2, RT_MAX_AXES = 4;
constexpr int RT_THREADS = 256, RT_MAX_TOKENS = 16;          // tokens of a CTA's table
constexpr int RT_MAX_PARTS = 592;                            // CTAs of the backward: partial sums of the gains' gradients

struct RotaryTurns {                                         // by value in the kernels' parameters
    unsigned long long turns[RT_MAX_PAIRS];
    uint8_t axis[RT_MAX_PAIRS];
};

struct RotaryArgs {
    const void *q, *k, *v, *gq, *gk;                         // v: append only; gq, gk: gains or null
    const void *dyq, *dyk;                                   // backward
    void *oq, *ok;
    int64_t ldq, ldk, ldv, lddyq, lddyk, ldoq, ldok;
    const int32_t *pos;
    int64_t ldpos;
    int64_t n;
    int32_t hq, hk, d, rot, tokens, heads_per_cta;
    float eps;
    float *part;                                             // backward: [CTAs][2][d]
    PagedView c;
};

__device__ __forceinline__ float2 turn_to_cos_sin(unsigned long long a)
{
    const int t = (int)(a >> 32);                            // signed 2^-32 turns
    const unsigned quad = ((unsigned)t + (1u << 29)) >> 30;
    const int rest = t - (int)(quad << 30);                  // within an eighth of a turn
    float s, c;
    sincospif((float)rest * 4.656612873077393e-10f, &s, &c); // 2^-31: half turns
    if (quad & 1) { const float x = c; c = -s; s = x; }
    return quad & 2 ? make_float2(-c, -s) : make_float2(c, s);
}

template <typename T, int V> struct Vec;                     // V elements of T as one load
template <> struct Vec<bf16, 8> { typedef uint4 type; };
template <> struct Vec<bf16, 4> { typedef uint2 type; };
template <> struct Vec<float, 4> { typedef uint4 type; };

template <typename T, int V> __device__ __forceinline__ void unpack(const typename Vec<T, V>::type &w, float (&f)[V])
{
    const T *e = reinterpret_cast<const T *>(&w);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = to_f32(e[i]);
}
template <typename T, int V> __device__ __forceinline__ typename Vec<T, V>::type pack(const float (&f)[V])
{
    typename Vec<T, V>::type w;
    T *e = reinterpret_cast<T *>(&w);
#pragma unroll
    for (int i = 0; i < V; ++i) e[i] = from_f32<T>(f[i]);
    return w;
}

// Where a lane's V pairs are: elements e0 .. e0 + V - 1 and e1 .. e1 + V - 1 of the row, table entry p0 (below zero: columns
// behind the rotated ones, which are only normalised).
struct LanePairs { int e0, e1, p0; bool on; };
template <int V, bool INTER> __device__ __forceinline__ LanePairs lane_pairs(int c, int d, int rot)
{
    LanePairs l;
    const int turned = rot / (2 * V);
    l.on = c < d / (2 * V);
    if (c < turned) {
        l.p0 = c * V;
        l.e0 = INTER ? 2 * V * c : V * c;
        l.e1 = INTER ? l.e0 + V : rot / 2 + V * c;
    } else {
        l.p0 = -1;
        l.e0 = 2 * V * c;
        l.e1 = l.e0 + V;
    }
    return l;
}

// rotates the lane's pairs; sign -1 turns back
template <int V, bool INTER> __device__ __forceinline__ void rotate(float (&lo)[V], float (&hi)[V], const float2 *cs, float sign)
{
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float2 t = cs[i];
        float &a = INTER ? (2 * i < V ? lo[2 * i] : hi[2 * i - V]) : lo[i];
        float &b = INTER ? (2 * i < V ? lo[2 * i + 1] : hi[2 * i + 1 - V]) : hi[i];
        const float s = sign * t.y, x = a;
        a = x * t.x - b * s;
        b = b * t.x + x * s;
    }
}

template <int L> __device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// cos / sin of tokens t0 .. t0 + count - 1
__device__ __forceinline__ void fill_table(float2 *table, const RotaryArgs &a, const RotaryTurns &f, int64_t t0, int count)
{
    const int pairs = a.rot / 2;
    for (int i = threadIdx.x; i < count * pairs; i += RT_THREADS) {
        const int t = i / pairs, p = i - t * pairs;
        const long long pos = a.pos[f.axis[p] * a.ldpos + t0 + t];
        table[i] = turn_to_cos_sin((unsigned long long)pos * f.turns[p]);
    }
}

// Where the last row of a token's sequence puts it: byte offset of its cache row, -1 for none (token behind the last sequence: -2).
// One warp, every lane gets the answer.
__device__ __forceinline__ int64_t append_row(const PagedView &c, int64_t token, int lane)
{
    int lo = 0, hi = c.n_seq;                                // largest s with cu[s] <= token, 32 candidates at a time
    while (hi - lo > 1) {
        const int step = (hi - lo + 31) / 32, s = lo + lane * step;
        const unsigned below = __ballot_sync(0xffffffffu, s < hi && c.cu[s] <= token);
        const int k = 31 - __clz(below | 1u);
        const int first = lo + k * step;
        hi = min(hi, first + step);
        lo = first;
    }
    const int a = c.cu[lo], b = c.cu[lo + 1];
    if (token < a || token >= b) {
        // behind the last sequence is where rows may stand that belong to none
        if (lane == 0 && token < c.cu[c.n_seq]) paged_report(c, SITE_PAGED_OFFSETS);
        return -2;
    }
    const int64_t row = (int64_t)c.lens[lo] - b + token;
    if (row < 0 || row >= c.capacity) {
        if (lane == 0) paged_report(c, SITE_PAGED_ROOM);
        return -1;
    }
    const int64_t at = paged_row(c, lo, (int)row);
    if (at < 0 && lane == 0) paged_report(c, SITE_PAGED_PAGE);
    return at;
}

// Forward.  CTA: `tokens` tokens x heads blockIdx.y * heads_per_cta .. of the hq + hk (+ hk values) rows of each.
template <typename T, int V, int L, bool INTER, bool APPEND>
__global__ void __launch_bounds__(RT_THREADS)
k_rotary_fwd(const __grid_constant__ RotaryArgs a, const __grid_constant__ RotaryTurns f)
{
    typedef typename Vec<T, V>::type W;
    extern __shared__ float2 table[];
    __shared__ int64_t slot[RT_MAX_TOKENS];
    pdl_enter();
    const int64_t t0 = (int64_t)blockIdx.x * a.tokens;
    const int count = (int)min((int64_t)a.tokens, a.n - t0);
    const int h0 = blockIdx.y * a.heads_per_cta, all = a.hq + (APPEND ? 2 : 1) * a.hk, heads = min(a.heads_per_cta, all - h0);
    fill_table(table, a, f, t0, count);
    if (APPEND)
        for (int t = threadIdx.x >> 5; t < count; t += RT_THREADS / 32) {
            const int64_t r = append_row(a.c, t0 + t, threadIdx.x & 31);
            if ((threadIdx.x & 31) == 0) slot[t] = r;
        }
    __syncthreads();
    constexpr int GROUPS = RT_THREADS / L;
    const LanePairs l = lane_pairs<V, INTER>(threadIdx.x % L, a.d, a.rot);
    const float inv_d = 1.0f / a.d;
    int t = 0, h = threadIdx.x / L;
    while (h >= heads) { h -= heads; ++t; }
    // every lane of a warp takes part in the shuffles, so all walk the same number of rows
    for (int it = 0; it < (count * heads + GROUPS - 1) / GROUPS; ++it) {
        const bool live = t < count && l.on;
        const int head = h0 + h;
        const int64_t tok = t0 + t;
        const bool is_q = head < a.hq, is_v = APPEND && head >= a.hq + a.hk;
        const T *src = nullptr;
        T *dst = nullptr;
        if (live) {
            const int kh = is_q ? 0 : is_v ? head - a.hq - a.hk : head - a.hq;
            if (is_q) {
                src = (const T *)a.q + tok * a.ldq + (int64_t)head * a.d;
                dst = (T *)a.oq + tok * a.ldoq + (int64_t)head * a.d;
            } else {
                src = (is_v ? (const T *)a.v + tok * a.ldv : (const T *)a.k + tok * a.ldk) + (int64_t)kh * a.d;
                if (!APPEND) dst = (T *)a.ok + tok * a.ldok + (int64_t)kh * a.d;
            }
            if (APPEND) {
                const int64_t s = slot[t];
                if (s == -2) dst = nullptr;
                else if (!is_q) dst = s < 0 ? nullptr : (T *)((is_v ? a.c.v : a.c.k) + s + kh * a.c.head_stride);
            }
        }
        W w0 = {}, w1 = {};
        if (dst) {
            w0 = *reinterpret_cast<const W *>(src + l.e0);
            w1 = *reinterpret_cast<const W *>(src + l.e1);
        }
        const T *gamma = is_v ? nullptr : (const T *)(is_q ? a.gq : a.gk);
        float lo[V], hi[V];
        unpack<T, V>(w0, lo);
        unpack<T, V>(w1, hi);
        if (a.gq) {                                          // with a gain for q there is one for k
            float ss = 0.0f;
#pragma unroll
            for (int i = 0; i < V; ++i) ss = fmaf(lo[i], lo[i], fmaf(hi[i], hi[i], ss));
            const float r = rsqrtf(group_sum<L>(ss) * inv_d + a.eps);
            if (gamma && l.on) {
                float g0[V], g1[V];
                unpack<T, V>(*reinterpret_cast<const W *>(gamma + l.e0), g0);
                unpack<T, V>(*reinterpret_cast<const W *>(gamma + l.e1), g1);
#pragma unroll
                for (int i = 0; i < V; ++i) { lo[i] *= r * g0[i]; hi[i] *= r * g1[i]; }
            }
        }
        if (dst) {
            if (!is_v) {
                if (l.p0 >= 0) rotate<V, INTER>(lo, hi, table + t * (a.rot / 2) + l.p0, 1.0f);
                w0 = pack<T, V>(lo);
                w1 = pack<T, V>(hi);
            }
            *reinterpret_cast<W *>(dst + l.e0) = w0;
            *reinterpret_cast<W *>(dst + l.e1) = w1;
        }
        h += GROUPS;
        while (h >= heads) { h -= heads; ++t; }
    }
}

// Backward.  CTAs walk blocks of tokens; the gains' gradients are summed in registers (a lane's columns stay the
// same), over the CTA's groups in shared memory, then over the CTAs by k_rotary_sum: a fixed order throughout.
template <typename T, int V, int L, bool INTER>
__global__ void __launch_bounds__(RT_THREADS)
k_rotary_bwd(const __grid_constant__ RotaryArgs a, const __grid_constant__ RotaryTurns f)
{
    typedef typename Vec<T, V>::type W;
    extern __shared__ float2 table[];
    pdl_enter();
    constexpr int GROUPS = RT_THREADS / L;
    const LanePairs l = lane_pairs<V, INTER>(threadIdx.x % L, a.d, a.rot);
    const int heads = a.hq + a.hk;
    const float inv_d = 1.0f / a.d;
    float acc[2][2][V] = {};
    for (int64_t t0 = (int64_t)blockIdx.x * a.tokens; t0 < a.n; t0 += (int64_t)gridDim.x * a.tokens) {
        const int count = (int)min((int64_t)a.tokens, a.n - t0);
        __syncthreads();
        fill_table(table, a, f, t0, count);
        __syncthreads();
        int t = 0, h = threadIdx.x / L;
        while (h >= heads) { h -= heads; ++t; }
        for (int it = 0; it < (count * heads + GROUPS - 1) / GROUPS; ++it) {
            const bool live = t < count && l.on, is_q = h < a.hq;
            const int64_t tok = t0 + t;
            const int kh = is_q ? h : h - a.hq;
            W y0 = {}, y1 = {}, x0 = {}, x1 = {};
            if (live) {
                const T *dy = (is_q ? (const T *)a.dyq + tok * a.lddyq : (const T *)a.dyk + tok * a.lddyk) + (int64_t)kh * a.d;
                y0 = *reinterpret_cast<const W *>(dy + l.e0);
                y1 = *reinterpret_cast<const W *>(dy + l.e1);
                if (a.gq) {
                    const T *x = (is_q ? (const T *)a.q + tok * a.ldq : (const T *)a.k + tok * a.ldk) + (int64_t)kh * a.d;
                    x0 = *reinterpret_cast<const W *>(x + l.e0);
                    x1 = *reinterpret_cast<const W *>(x + l.e1);
                }
            }
            float lo[V], hi[V];
            unpack<T, V>(y0, lo);
            unpack<T, V>(y1, hi);
            if (live && l.p0 >= 0) rotate<V, INTER>(lo, hi, table + t * (a.rot / 2) + l.p0, -1.0f);
            if (a.gq) {
                const T *gamma = (const T *)(is_q ? a.gq : a.gk);
                float xl[V], xh[V], g0[V] = {}, g1[V] = {};
                unpack<T, V>(x0, xl);
                unpack<T, V>(x1, xh);
                if (l.on) {
                    unpack<T, V>(*reinterpret_cast<const W *>(gamma + l.e0), g0);
                    unpack<T, V>(*reinterpret_cast<const W *>(gamma + l.e1), g1);
                }
                float ss = 0.0f, ux = 0.0f;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    ss = fmaf(xl[i], xl[i], fmaf(xh[i], xh[i], ss));
                    ux = fmaf(lo[i] * g0[i], xl[i], fmaf(hi[i] * g1[i], xh[i], ux));
                }
                const float r = rsqrtf(group_sum<L>(ss) * inv_d + a.eps);
                const float m = group_sum<L>(ux) * inv_d * r * r;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float al = lo[i] * (xl[i] * r), ah = hi[i] * (xh[i] * r);
                    // a dead lane has zeros here
                    acc[0][0][i] += is_q ? al : 0.0f;
                    acc[0][1][i] += is_q ? ah : 0.0f;
                    acc[1][0][i] += is_q ? 0.0f : al;
                    acc[1][1][i] += is_q ? 0.0f : ah;
                    lo[i] = r * (lo[i] * g0[i] - xl[i] * m);
                    hi[i] = r * (hi[i] * g1[i] - xh[i] * m);
                }
            }
            if (live) {
                T *dx = (is_q ? (T *)a.oq + tok * a.ldoq : (T *)a.ok + tok * a.ldok) + (int64_t)kh * a.d;
                *reinterpret_cast<W *>(dx + l.e0) = pack<T, V>(lo);
                *reinterpret_cast<W *>(dx + l.e1) = pack<T, V>(hi);
            }
            h += GROUPS;
            while (h >= heads) { h -= heads; ++t; }
        }
    }
    if (!a.gq) return;
    float *sums = reinterpret_cast<float *>(table);           // [groups][d]
    for (int z = 0; z < 2; ++z) {
        __syncthreads();
        if (l.on)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                sums[(threadIdx.x / L) * a.d + l.e0 + i] = acc[z][0][i];
                sums[(threadIdx.x / L) * a.d + l.e1 + i] = acc[z][1][i];
            }
        __syncthreads();
        for (int c = threadIdx.x; c < a.d; c += RT_THREADS) {
            float s = 0.0f;
            for (int g = 0; g < GROUPS; ++g) s += sums[g * a.d + c];
            a.part[((int64_t)blockIdx.x * 2 + z) * a.d + c] = s;
        }
    }
}

// dgamma[z][c] = sum of the CTAs' parts: 32 columns a CTA, 32 rows of parts at a time
template <typename T> __global__ void __launch_bounds__(1024) k_rotary_sum(const float *__restrict__ part, int parts, int d, T *dgq, T *dgk)
{
    __shared__ float red[32][33];
    pdl_enter();
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;   // column of [2][d]
    float s = 0.0f;
    if (col < 2 * d)
        for (int p = w; p < parts; p += 32) s += part[(int64_t)p * 2 * d + col];
    red[w][lane] = s;
    __syncthreads();
    if (w == 0 && col < 2 * d) {
        float total = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) total += red[i][lane];
        T *dst = col < d ? dgq : dgk;
        if (dst) dst[col < d ? col : col - d] = from_f32<T>(total);
    }
}

template <typename... KArgs, typename... Args>
static cudaError_t launch_smem(void (*kernel)(KArgs...), dim3 grid, dim3 block, size_t smem, cudaStream_t s, const Args &...args)
{
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid; cfg.blockDim = block; cfg.dynamicSmemBytes = smem; cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at; cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}

static int lanes_of(int d, int V)
{
    int L = 1;
    while (L * 2 * V < d) L *= 2;
    return L;
}

template <typename T, int V, int L, bool INTER> static cudaError_t rotary_l(int mode, RotaryArgs a, const RotaryTurns &f, dim3 grid, cudaStream_t s)
{
    const size_t table = (size_t)a.tokens * (a.rot / 2) * sizeof(float2);
    if (mode == 0) return launch_smem(k_rotary_fwd<T, V, L, INTER, false>, grid, dim3(RT_THREADS), table, s, a, f);
    if (mode == 1) return launch_smem(k_rotary_fwd<T, V, L, INTER, true>, grid, dim3(RT_THREADS), table, s, a, f);
    const size_t sums = (size_t)(RT_THREADS / L) * a.d * sizeof(float);
    return launch_smem(k_rotary_bwd<T, V, L, INTER>, grid, dim3(RT_THREADS), table > sums ? table : sums, s, a, f);
}
template <typename T, int V, bool INTER> static cudaError_t rotary_v(int mode, const RotaryArgs &a, const RotaryTurns &f, dim3 grid, cudaStream_t s)
{
    switch (lanes_of(a.d, V)) {
    case 1: return rotary_l<T, V, 1, INTER>(mode, a, f, grid, s);
    case 2: return rotary_l<T, V, 2, INTER>(mode, a, f, grid, s);
    case 4: return rotary_l<T, V, 4, INTER>(mode, a, f, grid, s);
    case 8: return rotary_l<T, V, 8, INTER>(mode, a, f, grid, s);
    case 16: return rotary_l<T, V, 16, INTER>(mode, a, f, grid, s);
    default: return rotary_l<T, V, 32, INTER>(mode, a, f, grid, s);
    }
}
// Eight pairs a lane need halves and the columns behind the rotated ones to be multiples of 8 resp. 16; four always fit.
static cudaError_t rotary_launch(int mode, int dtype, bool inter, const RotaryArgs &a, const RotaryTurns &f, dim3 grid, cudaStream_t s)
{
    if (dtype == SKIPFFN_FP32) return inter ? rotary_v<float, 4, true>(mode, a, f, grid, s) : rotary_v<float, 4, false>(mode, a, f, grid, s);
    if (a.d % 16 == 0 && a.rot % 16 == 0)
        return inter ? rotary_v<bf16, 8, true>(mode, a, f, grid, s) : rotary_v<bf16, 8, false>(mode, a, f, grid, s);
    return inter ? rotary_v<bf16, 4, true>(mode, a, f, grid, s) : rotary_v<bf16, 4, false>(mode, a, f, grid, s);
}

// tokens of a CTA: up to 8, fewer while that leaves SMs without one; one token's heads are spread over CTAs when
// there are fewer tokens than SMs
static dim3 rotary_grid(RotaryArgs *a, int rows, int groups, bool split)
{
    int t = 8;
    while (t > 1 && (a->n + t - 1) / t < 4 * 148) t /= 2;
    a->tokens = t;
    a->heads_per_cta = rows;
    if (split && t == 1 && a->n < 148) a->heads_per_cta = groups < rows ? groups : rows;
    return dim3((unsigned)((a->n + t - 1) / t), (unsigned)((rows + a->heads_per_cta - 1) / a->heads_per_cta));
}

}  // namespace skipffn

using namespace skipffn;

struct skipffn_rotary {
    int32_t hq, hk, d, rot, inter, axes;
    float eps;
    RotaryTurns f;
};

namespace {

struct RotaryCall { int es; TokenArray q, k; };

skipffn_status check_call(const skipffn_rotary *h, int32_t dtype, int64_t n, const void *q, int64_t ldq, const void *k, int64_t ldk,
                          const int32_t *pos, int64_t ldpos, const void *gq, const void *gk, RotaryCall *c)
{
    if (!h || (dtype != SKIPFFN_BF16 && dtype != SKIPFFN_FP32) || n < 0 || n >= (int64_t)1 << 31) return SKIPFFN_EINVAL;
    if ((gq == nullptr) != (gk == nullptr) || !is_aligned(gq, 16) || !is_aligned(gk, 16)) return SKIPFFN_EINVAL;
    if (n == 0) return SKIPFFN_OK;
    c->es = dtype == SKIPFFN_BF16 ? 2 : 4;
    for (const int64_t ld : {ldq, ldk})
        if (ld < 0 || ld > (int64_t)1 << 36) return SKIPFFN_EINVAL;
    c->q = TokenArray{q, ldq * c->es, (int64_t)h->hq * h->d * c->es};
    c->k = TokenArray{k, ldk * c->es, (int64_t)h->hk * h->d * c->es};
    if (!token_array_ok(c->q, n) || !token_array_ok(c->k, n)) return SKIPFFN_EINVAL;
    if (h->rot > 0 && (!pos || !is_aligned(pos, 4) || (h->axes > 1 && (ldpos < n || ldpos > (int64_t)1 << 40)))) return SKIPFFN_EINVAL;
    return SKIPFFN_OK;
}

// `out` may be `same` (in place), every other overlap with what the call reads is refused
bool out_ok(const TokenArray &out, const TokenArray *same, std::initializer_list<TokenArray> in, const int32_t *pos, int64_t pos_bytes,
            const void *gq, const void *gk, int64_t g_bytes, int64_t n)
{
    if (!token_array_ok(out, n)) return false;
    for (const TokenArray &x : in) {
        if (same && x.p == same->p && x.ld == same->ld && out.p == x.p && out.ld == x.ld && out.width == x.width) continue;
        if (tokens_overlap(out, x, n)) return false;
    }
    const int64_t b = token_bytes(out, n);
    return !ranges_overlap(out.p, b, pos, pos_bytes) && !ranges_overlap(out.p, b, gq, g_bytes) && !ranges_overlap(out.p, b, gk, g_bytes);
}

int64_t pos_bytes(const skipffn_rotary *h, int64_t n, int64_t ldpos) { return h->rot ? ((h->axes - 1) * ldpos + n) * 4 : 0; }

RotaryArgs args_of(const skipffn_rotary *h, int64_t n, const void *q, int64_t ldq, const void *k, int64_t ldk, const int32_t *pos,
                   int64_t ldpos, const void *gq, const void *gk)
{
    RotaryArgs a = {};
    a.q = q; a.k = k; a.ldq = ldq; a.ldk = ldk; a.pos = pos; a.ldpos = ldpos; a.gq = gq; a.gk = gk; a.n = n;
    a.hq = h->hq; a.hk = h->hk; a.d = h->d; a.rot = h->rot; a.eps = h->eps;
    return a;
}

}  // namespace

extern "C" {

skipffn_status skipffn_rotary_create(skipffn_rotary **out, const skipffn_rotary_config *c)
{
    if (!out) return SKIPFFN_EINVAL;
    *out = nullptr;
    if (!c || c->heads_q <= 0 || c->heads_kv <= 0 || c->head_dim <= 0 || c->rotary_dim < 0 || c->rotary_dim > c->head_dim ||
        (c->interleaved != 0 && c->interleaved != 1) || c->axes < 1 || !(c->eps >= 0.0f) || !isfinite(c->eps))
        return SKIPFFN_EINVAL;
    if (c->rotary_dim > 0 && !c->inv_freq) return SKIPFFN_EINVAL;
    if (c->head_dim % 8 || c->head_dim > RT_MAX_D || c->rotary_dim % 8 || c->axes > RT_MAX_AXES || c->heads_q > 65535 || c->heads_kv > 65535)
        return SKIPFFN_EUNSUPPORTED;
    skipffn_rotary *h = new (std::nothrow) skipffn_rotary;
    if (!h) return SKIPFFN_EWORKSPACE;
    *h = skipffn_rotary{};
    h->hq = c->heads_q; h->hk = c->heads_kv; h->d = c->head_dim; h->rot = c->rotary_dim; h->inter = c->interleaved;
    h->axes = c->axes; h->eps = c->eps;
    for (int p = 0; p < c->rotary_dim / 2; ++p) {
        const int32_t axis = c->axis ? c->axis[p] : 0;
        if (axis < 0 || axis >= c->axes || !isfinite(c->inv_freq[p])) { delete h; return SKIPFFN_EINVAL; }
        const long double turn = (long double)c->inv_freq[p] / 6.283185307179586476925286766559L;
        h->f.axis[p] = (uint8_t)axis;
        // whole turns per position drop out: positions are whole numbers
        const long double scaled = roundl((turn - floorl(turn)) * 18446744073709551616.0L);
        h->f.turns[p] = scaled >= 18446744073709551616.0L ? 0ull : (unsigned long long)scaled;
    }
    *out = h;
    return SKIPFFN_OK;
}

void skipffn_rotary_destroy(skipffn_rotary *h) { delete h; }

skipffn_status skipffn_rotary_forward(const skipffn_rotary *h, int32_t dtype, int64_t n, const void *q, int64_t ldq, const void *k,
                                      int64_t ldk, const int32_t *positions, int64_t ldpos, const void *gamma_q, const void *gamma_k,
                                      void *q_out, int64_t ldqo, void *k_out, int64_t ldko, void *stream)
{
    RotaryCall c;
    const skipffn_status st = check_call(h, dtype, n, q, ldq, k, ldk, positions, ldpos, gamma_q, gamma_k, &c);
    if (st != SKIPFFN_OK || n == 0) return st;
    for (const int64_t ld : {ldqo, ldko})
        if (ld < 0 || ld > (int64_t)1 << 36) return SKIPFFN_EINVAL;
    const TokenArray oq{q_out, ldqo * c.es, c.q.width}, ok{k_out, ldko * c.es, c.k.width};
    const int64_t pb = pos_bytes(h, n, ldpos), gb = (int64_t)h->d * c.es;
    if (!out_ok(oq, &c.q, {c.q, c.k}, positions, pb, gamma_q, gamma_k, gb, n) ||
        !out_ok(ok, &c.k, {c.q, c.k}, positions, pb, gamma_q, gamma_k, gb, n) || tokens_overlap(oq, ok, n))
        return SKIPFFN_EINVAL;
    RotaryArgs a = args_of(h, n, q, ldq, k, ldk, positions, ldpos, gamma_q, gamma_k);
    a.oq = q_out; a.ok = k_out; a.ldoq = ldqo; a.ldok = ldko;
    const int V = dtype == SKIPFFN_BF16 && h->d % 16 == 0 && h->rot % 16 == 0 ? 8 : 4;
    const dim3 grid = rotary_grid(&a, h->hq + h->hk, RT_THREADS / lanes_of(h->d, V), true);
    return rotary_launch(0, dtype, h->inter, a, h->f, grid, (cudaStream_t)stream) == cudaSuccess ? SKIPFFN_OK : SKIPFFN_ECUDA;
}

size_t skipffn_rotary_scratch_bytes(const skipffn_rotary *h) { return h ? (size_t)RT_MAX_PARTS * 2 * h->d * sizeof(float) : 0; }

skipffn_status skipffn_rotary_backward(const skipffn_rotary *h, int32_t dtype, int64_t n, const void *dq_out, int64_t lddqo,
                                       const void *dk_out, int64_t lddko, const void *q, int64_t ldq, const void *k, int64_t ldk,
                                       const int32_t *positions, int64_t ldpos, const void *gamma_q, const void *gamma_k, void *dq,
                                       int64_t lddq, void *dk, int64_t lddk, void *dgamma_q, void *dgamma_k, int32_t dw_fp32,
                                       void *scratch, size_t scratch_bytes, void *stream)
{
    RotaryCall c;
    const skipffn_status st = check_call(h, dtype, n, q, ldq, k, ldk, positions, ldpos, gamma_q, gamma_k, &c);
    if (st != SKIPFFN_OK) return st;
    if (dw_fp32 != 0 && dw_fp32 != 1) return SKIPFFN_EINVAL;
    const int es = dtype == SKIPFFN_BF16 ? 2 : 4, gs = dw_fp32 || dtype == SKIPFFN_FP32 ? 4 : 2;
    const bool norm = gamma_q != nullptr;
    const size_t need = skipffn_rotary_scratch_bytes(h);
    if (norm) {
        if (!scratch || !is_aligned(scratch, 16) || !is_aligned(dgamma_q, gs) || !is_aligned(dgamma_k, gs)) return SKIPFFN_EINVAL;
        if (scratch_bytes < need) return SKIPFFN_EWORKSPACE;
        const int64_t b = (int64_t)h->d * gs;
        if (ranges_overlap(dgamma_q, b, dgamma_k, b) || ranges_overlap(dgamma_q, b, scratch, need) || ranges_overlap(dgamma_k, b, scratch, need))
            return SKIPFFN_EINVAL;
    }
    RotaryArgs a = args_of(h, n, q, ldq, k, ldk, positions, ldpos, gamma_q, gamma_k);
    dim3 grid(0, 1, 1);
    if (n > 0) {
        for (const int64_t ld : {lddqo, lddko, lddq, lddk})
            if (ld < 0 || ld > (int64_t)1 << 36) return SKIPFFN_EINVAL;
        const TokenArray gq{dq_out, lddqo * es, c.q.width}, gk{dk_out, lddko * es, c.k.width};
        const TokenArray oq{dq, lddq * es, c.q.width}, ok{dk, lddk * es, c.k.width};
        const int64_t pb = pos_bytes(h, n, ldpos), gb = (int64_t)h->d * es;
        if (!token_array_ok(gq, n) || !token_array_ok(gk, n)) return SKIPFFN_EINVAL;
        // a result may stand where its own row was read, the upstream gradient or the input
        const bool q_in = dq == q, k_in = dk == k;
        if (!out_ok(oq, q_in ? &c.q : &gq, {c.q, c.k, gq, gk}, positions, pb, gamma_q, gamma_k, gb, n) ||
            !out_ok(ok, k_in ? &c.k : &gk, {c.q, c.k, gq, gk}, positions, pb, gamma_q, gamma_k, gb, n) || tokens_overlap(oq, ok, n))
            return SKIPFFN_EINVAL;
        if (norm) {
            const int64_t b = (int64_t)h->d * gs;
            for (const TokenArray &x : {c.q, c.k, gq, gk, oq, ok}) {
                const int64_t xb = token_bytes(x, n);
                if (ranges_overlap(x.p, xb, dgamma_q, b) || ranges_overlap(x.p, xb, dgamma_k, b) || ranges_overlap(x.p, xb, scratch, need)) return SKIPFFN_EINVAL;
            }
            for (const void *g : {gamma_q, gamma_k})
                if (ranges_overlap(g, gb, dgamma_q, b) || ranges_overlap(g, gb, dgamma_k, b) || ranges_overlap(g, gb, scratch, need)) return SKIPFFN_EINVAL;
            if (ranges_overlap(positions, pb, dgamma_q, b) || ranges_overlap(positions, pb, dgamma_k, b) || ranges_overlap(positions, pb, scratch, need))
                return SKIPFFN_EINVAL;
        }
        a.dyq = dq_out; a.dyk = dk_out; a.lddyq = lddqo; a.lddyk = lddko;
        a.oq = dq; a.ok = dk; a.ldoq = lddq; a.ldok = lddk;
        a.part = (float *)scratch;
        grid = rotary_grid(&a, h->hq + h->hk, 0, false);
        if (grid.x > RT_MAX_PARTS) grid.x = RT_MAX_PARTS;
        if (rotary_launch(2, dtype, h->inter, a, h->f, grid, (cudaStream_t)stream) != cudaSuccess) return SKIPFFN_ECUDA;
    }
    if (!norm || (!dgamma_q && !dgamma_k)) return SKIPFFN_OK;
    const dim3 sum_grid((unsigned)((2 * h->d + 31) / 32));
    const cudaError_t e = gs == 4 ? launch_smem(k_rotary_sum<float>, sum_grid, dim3(1024), 0, (cudaStream_t)stream, (const float *)scratch,
                                                (int)grid.x, (int)h->d, (float *)dgamma_q, (float *)dgamma_k)
                                  : launch_smem(k_rotary_sum<bf16>, sum_grid, dim3(1024), 0, (cudaStream_t)stream, (const float *)scratch,
                                                (int)grid.x, (int)h->d, (bf16 *)dgamma_q, (bf16 *)dgamma_k);
    return e == cudaSuccess ? SKIPFFN_OK : SKIPFFN_ECUDA;
}

skipffn_status skipffn_rotary_append(const skipffn_rotary *h, const skipffn_paged_cache *cache, int64_t n, const void *q, int64_t ldq,
                                     const void *k, int64_t ldk, const void *v, int64_t ldv, const int32_t *positions, int64_t ldpos,
                                     const void *gamma_q, const void *gamma_k, void *q_out, int64_t ldqo, void *stream)
{
    RotaryCall c;
    PagedView view;
    skipffn_status st = paged_view(cache, n, &view);
    if (st != SKIPFFN_OK) return st;
    if (!h || h->hk != view.heads || h->d != view.d) return SKIPFFN_EINVAL;
    st = check_call(h, cache->dtype, n, q, ldq, k, ldk, positions, ldpos, gamma_q, gamma_k, &c);
    if (st != SKIPFFN_OK || n == 0 || view.n_seq == 0) return st;
    for (const int64_t ld : {ldv, ldqo})
        if (ld < 0 || ld > (int64_t)1 << 36) return SKIPFFN_EINVAL;
    const TokenArray va{v, ldv * c.es, c.k.width}, oq{q_out, ldqo * c.es, c.q.width};
    const int64_t pb = pos_bytes(h, n, ldpos), gb = (int64_t)h->d * c.es;
    if (!token_array_ok(va, n) || !out_ok(oq, &c.q, {c.q, c.k, va}, positions, pb, gamma_q, gamma_k, gb, n)) return SKIPFFN_EINVAL;
    for (const TokenArray &x : {c.q, c.k, va, oq})
        if (paged_overlap(view, x.p, token_bytes(x, n))) return SKIPFFN_EINVAL;
    if (paged_overlap(view, positions, pb) || paged_overlap(view, gamma_q, gb) || paged_overlap(view, gamma_k, gb)) return SKIPFFN_EINVAL;
    RotaryArgs a = args_of(h, n, q, ldq, k, ldk, positions, ldpos, gamma_q, gamma_k);
    a.v = v; a.ldv = ldv; a.oq = q_out; a.ldoq = ldqo; a.c = view;
    const int V = cache->dtype == SKIPFFN_BF16 && h->d % 16 == 0 && h->rot % 16 == 0 ? 8 : 4;
    const dim3 grid = rotary_grid(&a, h->hq + 2 * h->hk, RT_THREADS / lanes_of(h->d, V), true);
    return rotary_launch(1, cache->dtype, h->inter, a, h->f, grid, (cudaStream_t)stream) == cudaSuccess ? SKIPFFN_OK : SKIPFFN_ECUDA;
}

skipffn_status skipffn_paged_append(const skipffn_paged_cache *cache, int64_t n, const void *k, int64_t ldk, const void *v, int64_t ldv,
                                    void *stream)
{
    PagedView view;
    const skipffn_status st = paged_view(cache, n, &view);
    if (st != SKIPFFN_OK || n == 0 || view.n_seq == 0) return st;
    const int64_t es = cache->dtype == SKIPFFN_BF16 ? 2 : 4, w = (int64_t)view.heads * view.d * es;
    for (const int64_t ld : {ldk, ldv})
        if (ld < 0 || ld > (int64_t)1 << 36) return SKIPFFN_EINVAL;
    for (const TokenArray &x : {TokenArray{k, ldk * es, w}, TokenArray{v, ldv * es, w}})
        if (!token_array_ok(x, n) || paged_overlap(view, x.p, token_bytes(x, n))) return SKIPFFN_EINVAL;
    RotaryArgs a = {};                       // no queries, nothing turned
    a.k = k; a.v = v; a.ldk = ldk; a.ldv = ldv; a.n = n; a.hk = view.heads; a.d = view.d; a.c = view;
    const int V = cache->dtype == SKIPFFN_BF16 && view.d % 16 == 0 ? 8 : 4;
    const dim3 grid = rotary_grid(&a, 2 * a.hk, RT_THREADS / lanes_of(a.d, V), true);
    return rotary_launch(1, cache->dtype, false, a, RotaryTurns{}, grid, (cudaStream_t)stream) == cudaSuccess ? SKIPFFN_OK : SKIPFFN_ECUDA;
}

}  // extern "C"
