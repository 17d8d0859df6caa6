// C-ABI entry points of packed attention: argument checks, work lists, launch sequencing.
#include <limits.h>
#include <math.h>

#include <algorithm>
#include <initializer_list>
#include <new>
#include <vector>

#include "attention.cuh"

using namespace skipffn;

struct skipffn_attention {
    skipffn_attention_config cfg;
    int64_t N;
    int32_t group, tokens;               // query heads per kv head, tokens of a row tile
    int32_t n_fwd, n_rows, n_keys;       // entries of the work lists
    int32_t max_len;                     // of the longest sequence
    int32_t *status;                     // device: status block, then the lists
    const int4 *fwd_items, *row_items, *key_items;
    int32_t tune[SKIPFFN_ATTENTION_TUNE_COUNT];
};

namespace {

constexpr int32_t WAIT_US_DEFAULT = 1000000, WAIT_US_MAX = 4000000;      // the kernels count nanoseconds in 32 bits

bool simt(const skipffn_attention_config *c) { return c->dtype == SKIPFFN_FP32 || c->path == SKIPFFN_PATH_SIMT; }
int tile_rows(const skipffn_attention_config *c) { return simt(c) ? AT_SIMT_ROWS : AT_TC_ROWS; }
int tile_keys(const skipffn_attention_config *c) { return simt(c) ? AT_SIMT_KEYS : AT_TC_KEYS; }

skipffn_status check_cfg(const skipffn_attention_config *c)
{
    if (!c || c->heads_q <= 0 || c->heads_kv <= 0 || c->heads_q % c->heads_kv || c->head_dim <= 0 ||
        (c->dtype != SKIPFFN_BF16 && c->dtype != SKIPFFN_FP32) || (c->causal != 0 && c->causal != 1) ||
        (c->path != SKIPFFN_PATH_DEFAULT && c->path != SKIPFFN_PATH_SIMT) || !(c->scale > 0.0f) || !isfinite(c->scale))
        return SKIPFFN_EINVAL;
    if (c->head_dim % 8 || c->head_dim > AT_MAX_D || c->heads_q / c->heads_kv > AT_SIMT_ROWS || c->heads_q > 65535)
        return SKIPFFN_EUNSUPPORTED;
    return SKIPFFN_OK;
}

struct Counts { int64_t fwd, rows, keys; };

// lengths are differences of ascending offsets that start at 0; counts of the three work lists
skipffn_status check_offsets(const skipffn_attention_config *c, const int32_t *cu, int32_t n_seq, Counts *n)
{
    if (n_seq < 0 || !cu || cu[0] != 0) return SKIPFFN_EINVAL;
    const int64_t t = tile_rows(c) / (c->heads_q / c->heads_kv), f = simt(c) ? t : 2 * t, k = tile_keys(c);
    *n = Counts{0, 0, 0};
    for (int32_t i = 0; i < n_seq; ++i) {
        const int64_t len = (int64_t)cu[i + 1] - cu[i];
        if (len < 0) return SKIPFFN_EINVAL;
        n->fwd += (len + f - 1) / f;
        n->rows += (len + t - 1) / t;
        n->keys += (len + k - 1) / k;
    }
    // tokens of a tile past the end of the last sequence must not pass 32 bits, nor items x heads
    if (n_seq > 0 && cu[n_seq] > INT_MAX - 4096) return SKIPFFN_EUNSUPPORTED;
    if (std::max(n->rows, n->keys) * c->heads_kv > INT_MAX / 2) return SKIPFFN_EUNSUPPORTED;
    return SKIPFFN_OK;
}

size_t plan_bytes(const Counts &n) { return (size_t)ST_WORDS * 4 + (size_t)(n.fwd + n.rows + n.keys) * sizeof(int4); }

bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

// A [tokens, heads, d] array: base, token stride and extent of a token's heads in bytes
struct Array { const void *p; int64_t ld; int64_t width; };

// strides are bounded by what a tensor map takes and so that N of them stay within 64 bits
bool array_ok(const Array &a, int64_t N)
{
    return a.p && aligned16(a.p) && a.ld % 16 == 0 && a.ld >= a.width && a.ld <= (int64_t)1 << 38 && a.ld <= ((int64_t)1 << 60) / N;
}
// Do two arrays of N tokens share a byte?  Exact for equal strides (slices of one fused array), else by range.
bool overlap(const Array &x, const Array &y, int64_t N)
{
    const intptr_t a = (intptr_t)x.p, b = (intptr_t)y.p;
    if (a >= b + (N - 1) * y.ld + y.width || b >= a + (N - 1) * x.ld + x.width) return false;
    if (x.ld != y.ld) return true;
    const int64_t off = ((b - a) % x.ld + x.ld) % x.ld;      // y's columns relative to x's inside one stride
    return off < x.width || off + y.width > x.ld;
}

void fill_args(const skipffn_attention *h, AttnArgs *a)
{
    *a = AttnArgs{};
    a->fwd_items = h->fwd_items; a->row_items = h->row_items; a->key_items = h->key_items;
    a->n_fwd = h->n_fwd; a->n_rows = h->n_rows; a->n_keys = h->n_keys;
    a->N = h->N; a->max_len = h->max_len;
    a->hq = h->cfg.heads_q; a->hk = h->cfg.heads_kv; a->group = h->group; a->tokens = h->tokens;
    a->d = h->cfg.head_dim; a->causal = h->cfg.causal; a->scale = h->cfg.scale;
    a->status = h->status;
    a->wait_us = h->tune[SKIPFFN_ATTENTION_WAIT_US]; a->lose_load = h->tune[SKIPFFN_ATTENTION_LOSE_LOAD];
}

}  // namespace

extern "C" {

size_t skipffn_attention_plan_bytes(const skipffn_attention_config *cfg, const int32_t *cu_seqlens, int32_t n_seq)
{
    Counts n;
    if (check_cfg(cfg) != SKIPFFN_OK || check_offsets(cfg, cu_seqlens, n_seq, &n) != SKIPFFN_OK) return 0;
    return plan_bytes(n);
}

skipffn_status skipffn_attention_create(skipffn_attention **out, const skipffn_attention_config *cfg,
                                        const int32_t *cu_seqlens, int32_t n_seq, void *plan, size_t bytes, void *stream)
{
    if (!out) return SKIPFFN_EINVAL;
    *out = nullptr;
    skipffn_status st = check_cfg(cfg);
    if (st != SKIPFFN_OK) return st;
    Counts n;
    st = check_offsets(cfg, cu_seqlens, n_seq, &n);
    if (st != SKIPFFN_OK) return st;
    if (!plan || !aligned16(plan)) return SKIPFFN_EINVAL;
    if (bytes < plan_bytes(n)) return SKIPFFN_EWORKSPACE;
    skipffn_attention *h = new (std::nothrow) skipffn_attention;
    if (!h) return SKIPFFN_EWORKSPACE;
    h->cfg = *cfg;
    h->tune[SKIPFFN_ATTENTION_WAIT_US] = WAIT_US_DEFAULT;
    h->tune[SKIPFFN_ATTENTION_LOSE_LOAD] = 0;
    h->N = n_seq > 0 ? cu_seqlens[n_seq] : 0;
    h->group = cfg->heads_q / cfg->heads_kv;
    h->tokens = tile_rows(cfg) / h->group;
    h->n_fwd = (int32_t)n.fwd; h->n_rows = (int32_t)n.rows; h->n_keys = (int32_t)n.keys;
    h->max_len = 0;
    for (int32_t i = 0; i < n_seq; ++i) h->max_len = std::max(h->max_len, cu_seqlens[i + 1] - cu_seqlens[i]);
    h->status = (int32_t *)plan;
    int4 *lists = (int4 *)((char *)plan + ST_WORDS * 4);
    h->fwd_items = lists; h->row_items = lists + n.fwd; h->key_items = lists + n.fwd + n.rows;
    try {
        // the lists hold the longest work first (equal work in order of the batch), which is what
        // balances a grid that hands them out in order
        struct Entry { int4 e; int64_t work; };
        std::vector<char> host(plan_bytes(n), 0);
        int4 *dst = (int4 *)(host.data() + ST_WORDS * 4);
        std::vector<Entry> list;
        auto flush = [&]() {
            std::stable_sort(list.begin(), list.end(), [](const Entry &a, const Entry &b) { return a.work > b.work; });
            for (const Entry &e : list) *dst++ = e.e;
            list.clear();
        };
        const int t = h->tokens, f = simt(cfg) ? t : 2 * t, k = tile_keys(cfg);
        for (int kind = 0; kind < 3; ++kind) {
            const int step = kind == 0 ? f : kind == 1 ? t : k;
            int64_t base = 0;
            for (int32_t i = 0; i < n_seq; ++i) {
                const int len = cu_seqlens[i + 1] - cu_seqlens[i];
                for (int64_t t0 = 0; t0 < len; t0 += step) {
                    const int64_t seen = !cfg->causal ? len : kind == 2 ? len - t0 : std::min<int64_t>(len, t0 + step);
                    list.push_back({make_int4(cu_seqlens[i], len, (int)t0, (int)base), kind == 2 ? (seen + t - 1) / t : (seen + k - 1) / k});
                }
                base += (len + t - 1) / t;
            }
            flush();
        }
        cudaStreamCaptureStatus cap = cudaStreamCaptureStatusNone;
        if (cudaStreamIsCapturing((cudaStream_t)stream, &cap) != cudaSuccess) {
            (void)cudaGetLastError();
            st = SKIPFFN_ECUDA;
        } else if (cap != cudaStreamCaptureStatusNone) {
            st = SKIPFFN_EINVAL;              // a replay would copy from a host buffer that is gone
        } else if (cudaMemcpyAsync(plan, host.data(), host.size(), cudaMemcpyHostToDevice, (cudaStream_t)stream) != cudaSuccess ||
                   cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess) {
            (void)cudaGetLastError();
            st = SKIPFFN_ECUDA;
        }
    } catch (...) {
        st = SKIPFFN_EWORKSPACE;
    }
    if (st != SKIPFFN_OK) { delete h; return st; }
    *out = h;
    return SKIPFFN_OK;
}

skipffn_status skipffn_attention_tune(skipffn_attention *h, int32_t what, int32_t value)
{
    if (!h || what < 0 || what >= SKIPFFN_ATTENTION_TUNE_COUNT) return SKIPFFN_EINVAL;
    if (what == SKIPFFN_ATTENTION_WAIT_US ? value < 1 || value > WAIT_US_MAX : value != 0 && value != 1) return SKIPFFN_EINVAL;
    h->tune[what] = value;
    return SKIPFFN_OK;
}

void skipffn_attention_destroy(skipffn_attention *h) { delete h; }

skipffn_status skipffn_attention_forward(const skipffn_attention *h, const void *q, int64_t ldq, const void *k, int64_t ldk,
                                         const void *v, int64_t ldv, void *out, int64_t ldo, float *lse, void *stream)
{
    if (!h) return SKIPFFN_EINVAL;
    if (h->N == 0) return SKIPFFN_OK;
    const int es = h->cfg.dtype == SKIPFFN_BF16 ? 2 : 4;
    for (const int64_t ld : {ldq, ldk, ldv, ldo})
        if (ld < 0 || ld > (int64_t)1 << 36) return SKIPFFN_EINVAL;
    const int64_t wq = (int64_t)h->cfg.heads_q * h->cfg.head_dim * es, wk = (int64_t)h->cfg.heads_kv * h->cfg.head_dim * es;
    const int64_t wl = (int64_t)h->cfg.heads_q * 4;
    const Array in[3] = {{q, ldq * es, wq}, {k, ldk * es, wk}, {v, ldv * es, wk}}, O{out, ldo * es, wq}, L{lse, wl, wl};
    if (!array_ok(O, h->N) || !lse || ((uintptr_t)lse & 3u) || overlap(O, L, h->N)) return SKIPFFN_EINVAL;
    for (const Array &x : in)
        if (!array_ok(x, h->N) || overlap(O, x, h->N) || overlap(L, x, h->N)) return SKIPFFN_EINVAL;
    AttnArgs a;
    fill_args(h, &a);
    a.q = q; a.k = k; a.v = v; a.out = out; a.lse = lse;
    a.ldq = ldq; a.ldk = ldk; a.ldv = ldv; a.ldo = ldo;
    const cudaError_t e = simt(&h->cfg) ? launch_attention_simt_forward(a, h->cfg.dtype, (cudaStream_t)stream)
                                        : launch_attention_tc_forward(a, (cudaStream_t)stream);
    return e == cudaSuccess ? SKIPFFN_OK : SKIPFFN_ECUDA;
}

size_t skipffn_attention_scratch_bytes(const skipffn_attention *h)
{
    return h ? (size_t)h->n_rows * h->cfg.heads_kv * tile_rows(&h->cfg) * sizeof(float2) : 0;
}

skipffn_status skipffn_attention_backward(const skipffn_attention *h, const void *dout, int64_t lddo, const void *q, int64_t ldq,
                                          const void *k, int64_t ldk, const void *v, int64_t ldv, const void *out, int64_t ldo,
                                          const float *lse, void *dq, int64_t lddq, void *dk, int64_t lddk, void *dv, int64_t lddv,
                                          void *scratch, size_t scratch_bytes, void *stream)
{
    if (!h) return SKIPFFN_EINVAL;
    if (h->N == 0) return SKIPFFN_OK;
    const int es = h->cfg.dtype == SKIPFFN_BF16 ? 2 : 4;
    for (const int64_t ld : {lddo, ldq, ldk, ldv, ldo, lddq, lddk, lddv})
        if (ld < 0 || ld > (int64_t)1 << 36) return SKIPFFN_EINVAL;
    const int64_t wq = (int64_t)h->cfg.heads_q * h->cfg.head_dim * es, wk = (int64_t)h->cfg.heads_kv * h->cfg.head_dim * es;
    const Array in[5] = {{q, ldq * es, wq}, {k, ldk * es, wk}, {v, ldv * es, wk}, {out, ldo * es, wq}, {dout, lddo * es, wq}};
    const Array res[3] = {{dq, lddq * es, wq}, {dk, lddk * es, wk}, {dv, lddv * es, wk}};
    for (const Array &x : in)
        if (!array_ok(x, h->N)) return SKIPFFN_EINVAL;
    for (int i = 0; i < 3; ++i) {
        if (!array_ok(res[i], h->N)) return SKIPFFN_EINVAL;
        for (const Array &x : in)
            if (overlap(res[i], x, h->N)) return SKIPFFN_EINVAL;
        for (int j = 0; j < i; ++j)
            if (overlap(res[i], res[j], h->N)) return SKIPFFN_EINVAL;
    }
    if (!lse || ((uintptr_t)lse & 3u) || !scratch || !aligned16(scratch)) return SKIPFFN_EINVAL;
    const size_t need = skipffn_attention_scratch_bytes(h);
    if (scratch_bytes < need) return SKIPFFN_EWORKSPACE;
    // the row statistics are written before the arrays are read, and read while the results are written
    const int64_t wl = (int64_t)h->cfg.heads_q * 4;
    const Array L{lse, wl, wl};
    auto in_scratch = [&](const Array &x) {
        const uintptr_t s0 = (uintptr_t)scratch, x0 = (uintptr_t)x.p;
        return x0 < s0 + need && s0 < x0 + (h->N - 1) * x.ld + x.width;
    };
    if (in_scratch(L)) return SKIPFFN_EINVAL;
    for (const Array &x : in)
        if (in_scratch(x)) return SKIPFFN_EINVAL;
    for (const Array &x : res)
        if (in_scratch(x) || overlap(x, L, h->N)) return SKIPFFN_EINVAL;
    AttnArgs a;
    fill_args(h, &a);
    a.q = q; a.k = k; a.v = v; a.out_in = out; a.dout = dout; a.dq = dq; a.dk = dk; a.dv = dv;
    a.lse = const_cast<float *>(lse);
    a.ldq = ldq; a.ldk = ldk; a.ldv = ldv; a.ldo = ldo; a.lddo = lddo; a.lddq = lddq; a.lddk = lddk; a.lddv = lddv;
    a.row_stats = (float2 *)scratch;
    const cudaError_t e = simt(&h->cfg) ? launch_attention_simt_backward(a, h->cfg.dtype, (cudaStream_t)stream)
                                        : launch_attention_tc_backward(a, (cudaStream_t)stream);
    return e == cudaSuccess ? SKIPFFN_OK : SKIPFFN_ECUDA;
}

skipffn_status skipffn_attention_poll(const skipffn_attention *h, void *stream, int32_t *site_out)
{
    if (!h) return SKIPFFN_EINVAL;
    if (cudaStreamSynchronize((cudaStream_t)stream) != cudaSuccess) return SKIPFFN_ECUDA;
    int32_t w[3] = {0, 0, 0};
    if (cudaMemcpy(w, h->status, sizeof(w), cudaMemcpyDeviceToHost) != cudaSuccess) return SKIPFFN_ECUDA;
    if (site_out) *site_out = w[ST_SITE];
    if (w[ST_STATUS] != 0 && cudaMemset(h->status + ST_STATUS, 0, 8) != cudaSuccess) return SKIPFFN_ECUDA;
    return (skipffn_status)w[ST_STATUS];
}

}  // extern "C"
