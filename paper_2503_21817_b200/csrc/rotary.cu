// Queries and keys of every head normalised (RMS norm) and rotated by position in one pass, its gradients, and the
// form that writes the rotated keys and the values into a paged cache.
//
//   n = x r gamma, r = 1 / sqrt(mean x^2 + eps)   (no gamma: n = x)
//   pair (a, b) of n -> (a cos t - b sin t, b cos t + a sin t),  t = position[axis of the pair] * frequency of the pair
//   backward: dn = the pair rotated by -t; dgamma = sum dn x r; u = dn gamma; dx = r (u - x r^2 mean(u x))
//
// Angles: a frequency is kept as turns per position in 64-bit fixed point (a fraction of a full turn), so position *
// frequency modulo one turn is one integer multiplication that drops what overflows: the angle's error does not grow
// with the position beyond that of the frequency's last bit (2^-65 of a turn each position).  A CTA computes the table of its tokens once, for all their heads.
//
// Bound by memory: every row is read and written once.  A group of lanes holds a row, each lane V pairs of it (two
// 16-byte vectors where the sizes allow), so the sums of a row are shuffles inside the group.  Measured: forward of 4928
// tokens, 32 / 8 heads, head_dim 128, normalised, bf16: 24 us for 101 MB (4.2 TB/s; 5.5 to 5.9 with four times the tokens; in
// a row 22.8 us, the norm alone 18.2, the rotation alone 20.8: nothing is loaded behind either); backward of four documents of
// 2344 tokens, 40 / 40 heads, 117 us (576 MB, 4.9 TB/s); one token a warp, its cosines in registers, was no faster (23.5 to 30
// and 128 us).  4096 tokens of a prompt into the cache: 26.4 us, in fp32 37.2.
#include <math.h>

#include <initializer_list>
#include <new>

#include "arrays.cuh"
#include "paged.cuh"

namespace skipffn {

constexpr int RT_MAX_D = 256, RT_MAX_PAIRS = RT_MAX_D / 2, RT_MAX_AXES = 4;
constexpr int RT_THREADS = 256, RT_MAX_TOKENS = 32;          // tokens of a CTA's table
constexpr int RT_FWD_ROWS = 2, RT_BWD_ROWS = 2;              // rows that a group of lanes has in flight
constexpr int RT_TURN = 8;                                   // rows of a group in a turn
constexpr int RT_MAX_PARTS = 296;                            // CTAs of the backward: partial sums of the gains' gradients

struct RotaryTurns {                                         // by value in the kernels' parameters
    unsigned long long turns[RT_MAX_PAIRS];
    uint8_t axis[RT_MAX_PAIRS];
};

// The rows of one kind: queries, keys, or values that are copied.  Each kind has its own CTAs, so that a CTA's rows share one
// gain and one set of strides, and `tokens` of them at a time.
struct RotaryRows {
    const void *x, *gamma, *dy;              // dy: backward
    void *out;
    int64_t ld, ldo, lddy;
    int32_t heads, tokens, ctas, pad;
};
struct RotaryArgs {
    RotaryRows rows[3];
    const int32_t *pos;
    int64_t ldpos, n;
    int32_t d, rot, axes;                    // axes: 0 without rotation
    float eps;
    float *part;                             // backward: [CTAs][d]
    PagedView c;
};

// cos and sin of a 2^-64 turns.  The quadrant is the top bits; the rest, within an eighth of a turn, goes to the functions'
// power series (terms 1 / n!): what they leave out is below 2^-29 there, so the error is that of the arithmetic, 4 x 2^-24.
__device__ __forceinline__ float2 turn_to_cos_sin(unsigned long long a)
{
    const int t = (int)(a >> 32);                            // signed 2^-32 turns
    const unsigned quad = ((unsigned)t + (1u << 29)) >> 30;
    const int rest = (int)((unsigned)t - (quad << 30));      // within 2^29 of zero; the difference of the signed ones would overflow
    const float x = (float)rest * 1.4629180792671596e-9f;    // 2 pi 2^-32
    const float z = x * x;
    float s = fmaf(z, 2.7557319e-6f, -1.9841270e-4f), c = fmaf(z, -2.7557319e-7f, 2.4801587e-5f);     // 1/9!, 1/7!; 1/10!, 1/8!
    s = fmaf(z, s, 8.3333333e-3f);                           // 1/5!
    s = fmaf(z, s, -1.6666667e-1f);                          // 1/3!
    s = fmaf(x * z, s, x);
    c = fmaf(z, c, -1.3888889e-3f);                          // 1/6!
    c = fmaf(z, c, 4.1666667e-2f);                           // 1/4!
    c = fmaf(z, c, -0.5f);
    c = fmaf(z, c, 1.0f);
    if (quad & 1) { const float y = c; c = -s; s = y; }
    return quad & 2 ? make_float2(-c, -s) : make_float2(c, s);
}

template <typename T, int V> struct Vec;                     // V elements of T as one load
template <> struct Vec<bf16, 8> { typedef uint4 type; };
template <> struct Vec<bf16, 4> { typedef uint2 type; };
template <> struct Vec<float, 4> { typedef uint4 type; };

// V elements as V / 2 pairs of fp32 (one instruction for two products or sums) and back, rounded once
__device__ __forceinline__ uint64_t widen(uint32_t w) { return pair2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ uint32_t narrow(uint64_t v)
{
    float a, b;
    unpair2(v, a, b);
    const __nv_bfloat162 t = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&t);
}
__device__ __forceinline__ void unpack(const uint4 &w, uint64_t (&f)[4]) { f[0] = widen(w.x); f[1] = widen(w.y); f[2] = widen(w.z); f[3] = widen(w.w); }
__device__ __forceinline__ void unpack(const uint2 &w, uint64_t (&f)[2]) { f[0] = widen(w.x); f[1] = widen(w.y); }
__device__ __forceinline__ void unpack(const uint4 &w, uint64_t (&f)[2])
{
    f[0] = pair2(__uint_as_float(w.x), __uint_as_float(w.y));
    f[1] = pair2(__uint_as_float(w.z), __uint_as_float(w.w));
}
__device__ __forceinline__ void pack(const uint64_t (&f)[4], uint4 &w) { w = make_uint4(narrow(f[0]), narrow(f[1]), narrow(f[2]), narrow(f[3])); }
template <typename T> __device__ __forceinline__ void pack(const uint64_t (&f)[2], uint2 &w) { w = make_uint2(narrow(f[0]), narrow(f[1])); }
template <typename T> __device__ __forceinline__ void pack(const uint64_t (&f)[2], uint4 &w)
{
    float a, b, c, d;
    unpair2(f[0], a, b);
    unpair2(f[1], c, d);
    w = make_uint4(__float_as_uint(a), __float_as_uint(b), __float_as_uint(c), __float_as_uint(d));
}
template <typename T> __device__ __forceinline__ void pack(const uint64_t (&f)[4], uint4 &w) { pack(f, w); }
__device__ __forceinline__ uint64_t both(float v) { return pair2(v, v); }
__device__ __forceinline__ float sum2(uint64_t v)
{
    float a, b;
    unpair2(v, a, b);
    return a + b;
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

// Where the cosine of pair p stands in a token's part of the table (its sine `pairs` further): four of a lane's pairs
// together, the lanes of a row side by side, so that a row's lanes read whole lines of banks.
template <int V> __device__ __forceinline__ int table_at(int p, int pairs) { return (p % V / 4 * (pairs / V) + p / V) * 4 + p % 4; }

// Rotates the lane's pairs, whose cosines start at `cs` (the place of the lane's first pair); sign -1 turns back.
template <int V, bool INTER> __device__ __forceinline__ void rotate(uint64_t (&lo)[V / 2], uint64_t (&hi)[V / 2], const float *cs, int pairs, float sign)
{
#pragma unroll
    for (int j = 0; j < V; j += 4) {
        float c[4], s[4];
        load4(cs + j * (pairs / V), c);
        load4(cs + j * (pairs / V) + pairs, s);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[e] *= sign;
        if (INTER) {                         // a pair stands in one register pair: (a, b) c + (-b, a) s
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint64_t &x = j + e < V / 2 ? lo[j + e] : hi[j + e - V / 2];
                float a, b;
                unpair2(x, a, b);
                x = fma2(pair2(-b, a), both(s[e]), mul2(x, both(c[e])));
            }
        } else {                             // two pairs in two register pairs
#pragma unroll
            for (int e = 0; e < 4; e += 2) {
                const int i = (j + e) / 2;
                const uint64_t c2 = pair2(c[e], c[e + 1]), x = lo[i];
                lo[i] = fma2(hi[i], pair2(-s[e], -s[e + 1]), mul2(x, c2));
                hi[i] = fma2(x, pair2(s[e], s[e + 1]), mul2(hi[i], c2));
            }
        }
    }
}

template <int L> __device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Cosines, then sines of the tokens whose positions stand at `pos` ([axis][RT_MAX_TOKENS]): a token's 2 x pairs floats.  A
// thread has one pair, whose frequency it reads once (parameters read at 32 different places take 32 turns).
template <int V> __device__ __forceinline__ void fill_table(float *table, const RotaryArgs &a, const RotaryTurns &f, const int *pos, int count)
{
    const int pairs = a.rot / 2;
    if (pairs == 0) return;
    const int step = RT_THREADS / pairs, first = threadIdx.x / pairs, p = threadIdx.x - first * pairs;
    if (first >= step) return;
    const int at = table_at<V>(p, pairs);
    const unsigned long long turns = f.turns[p];
    pos += f.axis[p] * RT_MAX_TOKENS;
    for (int t = first; t < count; t += step) {
        const float2 cs = turn_to_cos_sin((unsigned long long)(long long)pos[t] * turns);
        table[t * a.rot + at] = cs.x;
        table[t * a.rot + pairs + at] = cs.y;
    }
}

__device__ __forceinline__ void load_positions(int *pos, const RotaryArgs &a, int64_t t0, int count)
{
    const int i = threadIdx.x % RT_MAX_TOKENS, axis = threadIdx.x / RT_MAX_TOKENS;
    if (i < count && axis < a.axes) pos[threadIdx.x] = a.pos[axis * a.ldpos + t0 + i];
}

// Byte offset of the cache row of a token, -1 for none, -2 for none of a token that belongs to no sequence.  A sequence whose
// offsets or length are at fault has none for any of its tokens, since they may name older rows.  One warp, every lane gets
// the answer.
__device__ __forceinline__ int64_t append_row(const PagedView &c, int64_t token, int lane, bool report)
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
    int a = c.cu[lo], b = c.cu[lo + 1];
    const bool spanned = a <= token && token < b;
    // behind the last sequence is where rows may stand that belong to none
    if (!spanned && token >= c.cu[c.n_seq]) return -2;
    int len = c.lens[lo];
    if (!spanned || !paged_sound(c, a, b, len)) {            // the search wants ascending offsets: another may have the token
        unsigned has = 0;
        int s0 = -32;
        while (!has) {
            s0 += 32;
            if (s0 >= c.n_seq) break;
            lo = min(s0 + lane, c.n_seq - 1);
            a = c.cu[lo]; b = c.cu[lo + 1]; len = c.lens[lo];
            has = __ballot_sync(0xffffffffu, a <= token && token < b && paged_sound(c, a, b, len));
        }
        if (!has) {
            if (report && lane == 0 && !spanned) paged_report(c, SITE_PAGED_OFFSETS);
            return spanned ? -1 : -2;
        }
        lo = s0 + __ffs(has) - 1;
        b = c.cu[lo + 1]; len = c.lens[lo];
    }
    const int64_t row = (int64_t)len - b + token;
    if (row < 0) {
        if (report && lane == 0) paged_report(c, SITE_PAGED_ROOM);
        return -1;
    }
    const int64_t at = paged_row(c, lo, (int)row);
    if (report && at < 0 && lane == 0) paged_report(c, SITE_PAGED_PAGE);
    return at;
}

// Walks the (token, head) rows of a CTA, GROUPS apart
struct RowWalk {
    int t, h, heads, dt, dh;
    __device__ RowWalk(int first, int step, int heads_) : heads(heads_)
    {
        t = first / heads; h = first - t * heads;
        dt = step / heads; dh = step - dt * heads;
    }
    __device__ void next()
    {
        t += dt; h += dh;
        if (h >= heads) { h -= heads; ++t; }
    }
};

template <typename T, int V> struct Row { typename Vec<T, V>::type w0, w1; };
template <typename T, int V> __device__ __forceinline__ Row<T, V> load_row(const T *p, const LanePairs &l)
{
    typedef typename Vec<T, V>::type W;
    return Row<T, V>{*reinterpret_cast<const W *>(p + l.e0), *reinterpret_cast<const W *>(p + l.e1)};
}

// Forward.  Every group of lanes has several rows in flight: their loads are issued before any of them is worked on.
template <typename T, int V, int L, bool INTER, bool APPEND>
__global__ void __launch_bounds__(RT_THREADS, 4)
k_rotary_fwd(const __grid_constant__ RotaryArgs a, const __grid_constant__ RotaryTurns f)
{
    typedef typename Vec<T, V>::type W;
    extern __shared__ __align__(16) float table[];
    __shared__ int64_t slot[RT_MAX_TOKENS];
    __shared__ int pos[RT_MAX_AXES * RT_MAX_TOKENS];
    constexpr int GROUPS = RT_THREADS / L, U = RT_FWD_ROWS;
    int kind = 0, cta = blockIdx.x;
    while (cta >= a.rows[kind].ctas) cta -= a.rows[kind++].ctas;
    const RotaryRows &k = a.rows[kind];
    const int64_t t0 = (int64_t)cta * k.tokens;
    const int count = (int)min((int64_t)k.tokens, a.n - t0), rows = count * k.heads;
    const LanePairs l = lane_pairs<V, INTER>(threadIdx.x % L, a.d, a.rot);
    const float inv_d = 1.0f / a.d;
    RowWalk walk(threadIdx.x / L, GROUPS, k.heads);
    pdl_enter();
    uint64_t g0[V / 2] = {}, g1[V / 2] = {};
    if (k.gamma && l.on) {
        const Row<T, V> g = load_row<T, V>((const T *)k.gamma, l);
        unpack(g.w0, g0);
        unpack(g.w1, g1);
    }
    load_positions(pos, a, t0, kind < 2 ? count : 0);
    if (APPEND)
        for (int t = threadIdx.x >> 5; t < count; t += RT_THREADS / 32) {
            const int64_t r = append_row(a.c, t0 + t, threadIdx.x & 31, kind == 1);
            if ((threadIdx.x & 31) == 0) slot[t] = r;
        }
    __syncthreads();
    // every lane of a warp takes part in the shuffles, so all walk the same number of rows
    for (int r0 = 0; r0 < rows; r0 += U * GROUPS) {
        Row<T, V> x[U];
        int at[U];                           // token of the CTA, -1: no row
        int64_t to[U];                       // element offset of the result's row (append, keys and values: byte offset)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            at[u] = -1;
            to[u] = -1;
            x[u] = Row<T, V>{};
            if (walk.t < count && l.on) {
                const int64_t tok = t0 + walk.t;
                to[u] = tok * k.ldo + (int64_t)walk.h * a.d;
                if (APPEND) {
                    const int64_t s = slot[walk.t];
                    if (s == -2) to[u] = -1;
                    else if (kind > 0) to[u] = s < 0 ? -1 : s + walk.h * a.c.head_stride;
                }
                at[u] = walk.t;
                if (to[u] >= 0) x[u] = load_row<T, V>((const T *)k.x + tok * k.ld + (int64_t)walk.h * a.d, l);
            }
            walk.next();
        }
        if (r0 == 0 && kind < 2) {           // the table is made while the first rows arrive
            fill_table<V>(table, a, f, pos, count);
            __syncthreads();
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (kind < 2) {
                uint64_t lo[V / 2], hi[V / 2];
                unpack(x[u].w0, lo);
                unpack(x[u].w1, hi);
                if (k.gamma) {
                    uint64_t ss = 0;
#pragma unroll
                    for (int i = 0; i < V / 2; ++i) ss = fma2(lo[i], lo[i], fma2(hi[i], hi[i], ss));
                    const uint64_t r = both(rsqrtf(group_sum<L>(sum2(ss)) * inv_d + a.eps));
#pragma unroll
                    for (int i = 0; i < V / 2; ++i) { lo[i] = mul2(mul2(lo[i], g0[i]), r); hi[i] = mul2(mul2(hi[i], g1[i]), r); }
                }
                if (at[u] >= 0 && l.p0 >= 0) rotate<V, INTER>(lo, hi, table + at[u] * a.rot + l.p0 / V * 4, a.rot / 2, 1.0f);
                pack<T>(lo, x[u].w0);
                pack<T>(hi, x[u].w1);
            }
            if (to[u] >= 0) {
                T *dst = APPEND && kind > 0 ? (T *)((kind == 1 ? a.c.k : a.c.v) + to[u]) : (T *)k.out + to[u];
                *reinterpret_cast<W *>(dst + l.e0) = x[u].w0;
                *reinterpret_cast<W *>(dst + l.e1) = x[u].w1;
            }
        }
    }
    // offsets and lengths at fault are reported whether or not a token of this call meets them; the values' CTAs have no table to make
    if (APPEND && kind == 2 && cta == 0)
        for (int s = threadIdx.x; s < a.c.n_seq; s += RT_THREADS) paged_seq(a.c, s, true);
}

// Backward.  CTAs of a kind walk blocks of its tokens; the gain's gradient is summed in registers (a lane's columns stay
// the same), over the CTA's groups in shared memory, then over the CTAs by k_rotary_sum: a fixed order throughout.
template <typename T, int V, int L, bool INTER>
__global__ void __launch_bounds__(RT_THREADS, 2)
k_rotary_bwd(const __grid_constant__ RotaryArgs a, const __grid_constant__ RotaryTurns f)
{
    typedef typename Vec<T, V>::type W;
    extern __shared__ __align__(16) float table[];
    __shared__ int pos[RT_MAX_AXES * RT_MAX_TOKENS];
    constexpr int GROUPS = RT_THREADS / L, U = RT_BWD_ROWS;
    const int kind = blockIdx.x >= a.rows[0].ctas, cta = blockIdx.x - (kind ? a.rows[0].ctas : 0);
    const RotaryRows &k = a.rows[kind];
    const LanePairs l = lane_pairs<V, INTER>(threadIdx.x % L, a.d, a.rot);
    const float inv_d = 1.0f / a.d;
    pdl_enter();
    uint64_t acc[2][V / 2] = {}, g0[V / 2] = {}, g1[V / 2] = {};
    if (k.gamma && l.on) {
        const Row<T, V> g = load_row<T, V>((const T *)k.gamma, l);
        unpack(g.w0, g0);
        unpack(g.w1, g1);
    }
    for (int64_t t0 = (int64_t)cta * k.tokens; t0 < a.n; t0 += (int64_t)k.ctas * k.tokens) {
        const int count = (int)min((int64_t)k.tokens, a.n - t0), rows = count * k.heads;
        RowWalk walk(threadIdx.x / L, GROUPS, k.heads);
        load_positions(pos, a, t0, count);
        __syncthreads();                     // they are there, and the table has been read
        for (int r0 = 0; r0 < rows; r0 += U * GROUPS) {
            Row<T, V> y[U], x[U];
            int at[U], head[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                at[u] = -1;
                head[u] = walk.h;
                y[u] = x[u] = Row<T, V>{};
                if (walk.t < count && l.on) {
                    const int64_t tok = t0 + walk.t;
                    at[u] = walk.t;
                    y[u] = load_row<T, V>((const T *)k.dy + tok * k.lddy + (int64_t)walk.h * a.d, l);
                    if (k.gamma) x[u] = load_row<T, V>((const T *)k.x + tok * k.ld + (int64_t)walk.h * a.d, l);
                }
                walk.next();
            }
            if (r0 == 0) {
                fill_table<V>(table, a, f, pos, count);
                __syncthreads();
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                uint64_t lo[V / 2], hi[V / 2];
                unpack(y[u].w0, lo);
                unpack(y[u].w1, hi);
                if (at[u] >= 0 && l.p0 >= 0) rotate<V, INTER>(lo, hi, table + at[u] * a.rot + l.p0 / V * 4, a.rot / 2, -1.0f);
                if (k.gamma) {
                    uint64_t xl[V / 2], xh[V / 2], ss = 0, ux = 0;
                    unpack(x[u].w0, xl);
                    unpack(x[u].w1, xh);
#pragma unroll
                    for (int i = 0; i < V / 2; ++i) {
                        ss = fma2(xl[i], xl[i], fma2(xh[i], xh[i], ss));
                        ux = fma2(mul2(lo[i], g0[i]), xl[i], fma2(mul2(hi[i], g1[i]), xh[i], ux));
                    }
                    const float inv = rsqrtf(group_sum<L>(sum2(ss)) * inv_d + a.eps);
                    // lanes without a row add nothing: their zeros have no inverse norm when eps is 0
                    const float r = at[u] >= 0 ? inv : 0.0f;
                    const uint64_t r2 = both(r), m = both(-group_sum<L>(sum2(ux)) * inv_d * r * r);
#pragma unroll
                    for (int i = 0; i < V / 2; ++i) {
                        acc[0][i] = fma2(lo[i], mul2(xl[i], r2), acc[0][i]);
                        acc[1][i] = fma2(hi[i], mul2(xh[i], r2), acc[1][i]);
                        lo[i] = mul2(r2, fma2(xl[i], m, mul2(lo[i], g0[i])));
                        hi[i] = mul2(r2, fma2(xh[i], m, mul2(hi[i], g1[i])));
                    }
                }
                if (at[u] >= 0) {
                    T *dx = (T *)k.out + (t0 + at[u]) * k.ldo + (int64_t)head[u] * a.d;
                    W w0, w1;
                    pack<T>(lo, w0);
                    pack<T>(hi, w1);
                    *reinterpret_cast<W *>(dx + l.e0) = w0;
                    *reinterpret_cast<W *>(dx + l.e1) = w1;
                }
            }
        }
    }
    if (!k.gamma) return;
    float *sums = table;                     // [groups][d]
    __syncthreads();
    if (l.on)
#pragma unroll
        for (int i = 0; i < V / 2; ++i) {
            *reinterpret_cast<uint64_t *>(sums + (threadIdx.x / L) * a.d + l.e0 + 2 * i) = acc[0][i];
            *reinterpret_cast<uint64_t *>(sums + (threadIdx.x / L) * a.d + l.e1 + 2 * i) = acc[1][i];
        }
    __syncthreads();
    for (int c = threadIdx.x; c < a.d; c += RT_THREADS) {
        float s = 0.0f;
        for (int g = 0; g < GROUPS; ++g) s += sums[g * a.d + c];
        a.part[(int64_t)blockIdx.x * a.d + c] = s;
    }
}

// dgamma[c] = sum of the CTAs' parts, of parts 0 .. split - 1 for the queries' gain (blockIdx.y 0), the others for the
// keys': 32 columns a CTA, 32 parts at a time
template <typename T> __global__ void __launch_bounds__(1024) k_rotary_sum(const float *__restrict__ part, int split, int parts, int d, T *dgq, T *dgk)
{
    __shared__ float red[32][33];
    const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, col = blockIdx.x * 32 + lane;
    const int p0 = blockIdx.y ? split : 0, p1 = blockIdx.y ? parts : split;
    pdl_enter();
    float s = 0.0f;
    if (col < d) {
#pragma unroll 8
        for (int p = p0 + w; p < p1; p += 32) s += part[(int64_t)p * d + col];
    }
    red[w][lane] = s;
    __syncthreads();
    if (w == 0 && col < d) {
        float total = 0.0f;
#pragma unroll
        for (int i = 0; i < 32; ++i) total += red[i][lane];
        T *dst = blockIdx.y ? dgk : dgq;
        if (dst) dst[col] = from_f32<T>(total);
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

enum RotaryMode { RT_FORWARD, RT_APPEND, RT_BACKWARD };

template <typename T, int V, int L, bool INTER> static cudaError_t rotary_l(RotaryMode mode, const RotaryArgs &a, const RotaryTurns &f, cudaStream_t s)
{
    int tokens = 1, ctas = 0;
    for (const RotaryRows &k : a.rows) {
        if (k.ctas > 0 && k.tokens > tokens) tokens = k.tokens;
        ctas += k.ctas;
    }
    const size_t table = (size_t)tokens * a.rot * sizeof(float);
    const dim3 grid((unsigned)ctas), block(RT_THREADS);
    if (mode == RT_FORWARD) return launch_smem(k_rotary_fwd<T, V, L, INTER, false>, grid, block, table, s, a, f);
    if (mode == RT_APPEND) return launch_smem(k_rotary_fwd<T, V, L, INTER, true>, grid, block, table, s, a, f);
    const size_t sums = a.rows[0].gamma ? (size_t)(RT_THREADS / L) * a.d * sizeof(float) : 0;
    return launch_smem(k_rotary_bwd<T, V, L, INTER>, grid, block, table > sums ? table : sums, s, a, f);
}
template <typename T, int V, bool INTER> static cudaError_t rotary_v(RotaryMode mode, const RotaryArgs &a, const RotaryTurns &f, cudaStream_t s)
{
    switch (lanes_of(a.d, V)) {
    case 1: return rotary_l<T, V, 1, INTER>(mode, a, f, s);
    case 2: return rotary_l<T, V, 2, INTER>(mode, a, f, s);
    case 4: return rotary_l<T, V, 4, INTER>(mode, a, f, s);
    case 8: return rotary_l<T, V, 8, INTER>(mode, a, f, s);
    case 16: return rotary_l<T, V, 16, INTER>(mode, a, f, s);
    default: return rotary_l<T, V, 32, INTER>(mode, a, f, s);
    }
}
// Pairs of a lane: eight when halves and the columns behind the rotated ones are multiples of 8 resp. 16; four always fit.
static int pairs_per_lane(int dtype, int d, int rot) { return dtype == SKIPFFN_BF16 && d % 16 == 0 && rot % 16 == 0 ? 8 : 4; }
static cudaError_t rotary_launch(RotaryMode mode, int dtype, bool inter, const RotaryArgs &a, const RotaryTurns &f, cudaStream_t s)
{
    if (dtype == SKIPFFN_FP32) return inter ? rotary_v<float, 4, true>(mode, a, f, s) : rotary_v<float, 4, false>(mode, a, f, s);
    if (pairs_per_lane(dtype, a.d, a.rot) == 8) return inter ? rotary_v<bf16, 8, true>(mode, a, f, s) : rotary_v<bf16, 8, false>(mode, a, f, s);
    return inter ? rotary_v<bf16, 4, true>(mode, a, f, s) : rotary_v<bf16, 4, false>(mode, a, f, s);
}

// Tokens of a CTA's turn: as many as give every group of lanes RT_TURN rows, fewer while SMs would be left without work,
// never more than the table holds.
static void plan_rows(RotaryArgs *a, int dtype)
{
    const int groups = RT_THREADS / lanes_of(a->d, pairs_per_lane(dtype, a->d, a->rot));
    int64_t heads = 0, rows = (int64_t)RT_TURN * groups;
    for (const RotaryRows &k : a->rows) heads += k.heads;
    while (rows > groups && a->n * heads / rows < 4 * 148) rows /= 2;
    for (RotaryRows &k : a->rows) {
        if (k.heads == 0) continue;
        const int64_t t = rows / k.heads;
        k.tokens = (int32_t)(t < 1 ? 1 : t > RT_MAX_TOKENS ? RT_MAX_TOKENS : t);
        k.ctas = (int32_t)((a->n + k.tokens - 1) / k.tokens);
    }
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

// `out` may stand on an array of its `own` rows (in place: a row is read before it is written, by the same lanes); every other
// overlap with what the call reads is refused, also where an array of other rows is one of its own
bool out_ok(const TokenArray &out, std::initializer_list<TokenArray> own, std::initializer_list<TokenArray> others, const int32_t *pos,
            int64_t pos_bytes, const void *gq, const void *gk, int64_t g_bytes, int64_t n)
{
    if (!token_array_ok(out, n)) return false;
    for (const TokenArray &x : own)
        if (!(out.p == x.p && out.ld == x.ld && out.width == x.width) && tokens_overlap(out, x, n)) return false;
    for (const TokenArray &x : others)
        if (tokens_overlap(out, x, n)) return false;
    const int64_t b = token_bytes(out, n);
    return !ranges_overlap(out.p, b, pos, pos_bytes) && !ranges_overlap(out.p, b, gq, g_bytes) && !ranges_overlap(out.p, b, gk, g_bytes);
}

int64_t pos_bytes(const skipffn_rotary *h, int64_t n, int64_t ldpos) { return h->rot ? ((h->axes - 1) * ldpos + n) * 4 : 0; }

RotaryArgs args_of(const skipffn_rotary *h, int64_t n, const void *q, int64_t ldq, const void *k, int64_t ldk, const int32_t *pos,
                   int64_t ldpos, const void *gq, const void *gk, void *oq, int64_t ldoq, void *ok, int64_t ldok)
{
    RotaryArgs a = {};
    a.rows[0].x = q; a.rows[0].ld = ldq; a.rows[0].gamma = gq; a.rows[0].out = oq; a.rows[0].ldo = ldoq; a.rows[0].heads = h->hq;
    a.rows[1].x = k; a.rows[1].ld = ldk; a.rows[1].gamma = gk; a.rows[1].out = ok; a.rows[1].ldo = ldok; a.rows[1].heads = h->hk;
    a.pos = pos; a.ldpos = ldpos; a.n = n;
    a.d = h->d; a.rot = h->rot; a.axes = h->rot ? h->axes : 0; a.eps = h->eps;
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
    if (!out_ok(oq, {c.q}, {c.k}, positions, pb, gamma_q, gamma_k, gb, n) || !out_ok(ok, {c.k}, {c.q}, positions, pb, gamma_q, gamma_k, gb, n) ||
        tokens_overlap(oq, ok, n))
        return SKIPFFN_EINVAL;
    RotaryArgs a = args_of(h, n, q, ldq, k, ldk, positions, ldpos, gamma_q, gamma_k, q_out, ldqo, k_out, ldko);
    plan_rows(&a, dtype);
    return rotary_launch(RT_FORWARD, dtype, h->inter, a, h->f, (cudaStream_t)stream) == cudaSuccess ? SKIPFFN_OK : SKIPFFN_ECUDA;
}

size_t skipffn_rotary_scratch_bytes(const skipffn_rotary *h) { return h ? (size_t)RT_MAX_PARTS * h->d * sizeof(float) : 0; }

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
    RotaryArgs a = args_of(h, n, q, ldq, k, ldk, positions, ldpos, gamma_q, gamma_k, dq, lddq, dk, lddk);
    if (n > 0) {
        for (const int64_t ld : {lddqo, lddko, lddq, lddk})
            if (ld < 0 || ld > (int64_t)1 << 36) return SKIPFFN_EINVAL;
        const TokenArray gq{dq_out, lddqo * es, c.q.width}, gk{dk_out, lddko * es, c.k.width};
        const TokenArray oq{dq, lddq * es, c.q.width}, ok{dk, lddk * es, c.k.width};
        const int64_t pb = pos_bytes(h, n, ldpos), gb = (int64_t)h->d * es;
        if (!token_array_ok(gq, n) || !token_array_ok(gk, n)) return SKIPFFN_EINVAL;
        if (!out_ok(oq, {c.q, gq}, {c.k, gk}, positions, pb, gamma_q, gamma_k, gb, n) ||
            !out_ok(ok, {c.k, gk}, {c.q, gq}, positions, pb, gamma_q, gamma_k, gb, n) || tokens_overlap(oq, ok, n))
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
        a.rows[0].dy = dq_out; a.rows[0].lddy = lddqo;
        a.rows[1].dy = dk_out; a.rows[1].lddy = lddko;
        a.part = (float *)scratch;
        plan_rows(&a, dtype);
        // two CTAs an SM, shared out by the rows of a kind
        const int share = (int)((int64_t)RT_MAX_PARTS * h->hq / (h->hq + h->hk)), of_q = share < 1 ? 1 : share == RT_MAX_PARTS ? share - 1 : share;
        if (a.rows[0].ctas > of_q) a.rows[0].ctas = of_q;
        if (a.rows[1].ctas > RT_MAX_PARTS - of_q) a.rows[1].ctas = RT_MAX_PARTS - of_q;
        if (rotary_launch(RT_BACKWARD, dtype, h->inter, a, h->f, (cudaStream_t)stream) != cudaSuccess) return SKIPFFN_ECUDA;
    }
    if (!norm || (!dgamma_q && !dgamma_k)) return SKIPFFN_OK;
    const dim3 sum_grid((unsigned)((h->d + 31) / 32), 2);
    const int split = a.rows[0].ctas, parts = split + a.rows[1].ctas;         // none without tokens: zeros
    const cudaError_t e = gs == 4 ? launch_pdl(k_rotary_sum<float>, sum_grid, dim3(1024), (cudaStream_t)stream, (const float *)scratch, split, parts,
                                               (int)h->d, (float *)dgamma_q, (float *)dgamma_k)
                                  : launch_pdl(k_rotary_sum<bf16>, sum_grid, dim3(1024), (cudaStream_t)stream, (const float *)scratch, split, parts,
                                               (int)h->d, (bf16 *)dgamma_q, (bf16 *)dgamma_k);
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
    if (!token_array_ok(va, n) || !out_ok(oq, {c.q}, {c.k, va}, positions, pb, gamma_q, gamma_k, gb, n)) return SKIPFFN_EINVAL;
    for (const TokenArray &x : {c.q, c.k, va, oq})
        if (paged_overlap(view, x.p, token_bytes(x, n))) return SKIPFFN_EINVAL;
    if (paged_overlap(view, positions, pb) || paged_overlap(view, gamma_q, gb) || paged_overlap(view, gamma_k, gb)) return SKIPFFN_EINVAL;
    RotaryArgs a = args_of(h, n, q, ldq, k, ldk, positions, ldpos, gamma_q, gamma_k, q_out, ldqo, nullptr, 0);
    a.rows[2].x = v; a.rows[2].ld = ldv; a.rows[2].heads = h->hk;
    a.c = view;
    plan_rows(&a, cache->dtype);
    return rotary_launch(RT_APPEND, cache->dtype, h->inter, a, h->f, (cudaStream_t)stream) == cudaSuccess ? SKIPFFN_OK : SKIPFFN_ECUDA;
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
    a.rows[1].x = k; a.rows[1].ld = ldk; a.rows[1].heads = view.heads;
    a.rows[2].x = v; a.rows[2].ld = ldv; a.rows[2].heads = view.heads;
    a.n = n; a.d = view.d; a.c = view;
    plan_rows(&a, cache->dtype);
    return rotary_launch(RT_APPEND, cache->dtype, false, a, RotaryTurns{}, (cudaStream_t)stream) == cudaSuccess ? SKIPFFN_OK : SKIPFFN_ECUDA;
}

}  // extern "C"
