// Packed attention: what the entry points (attention.cu) hand to the kernels (attention_tc.cu for
// bf16 on the tensor cores, attention_simt.cu for fp32 and as an on-device second opinion).
#pragma once
#include "common.cuh"

namespace skipffn {

// A row tile holds the queries of one key / value head: `group` query heads x `tokens` consecutive
// tokens, token-major (row = token * group + head in group), so that grouped heads share every key
// and value tile and the gradient of a shared head is a sum over tile rows.
// Plan entry (int4): {first token of the sequence, its length, first token or key of the tile inside
// the sequence, index of the sequence's first row tile}.
struct AttnArgs {
    const void *q, *k, *v, *dout;    // [tokens, heads, d], token strides below (elements)
    const void *out_in;              // backward: the forward's output
    void *out, *dq, *dk, *dv;
    float *lse;                      // [tokens, heads_q], natural logarithm
    int64_t ldq, ldk, ldv, lddo, ldo, lddq, lddk, lddv;
    const int4 *fwd_items, *row_items, *key_items;
    int32_t n_fwd, n_rows, n_keys;   // entries of the three lists
    int64_t N;                       // tokens of all sequences
    int32_t max_len;                 // of the longest sequence
    int32_t hq, hk, group, tokens, d, causal;
    float scale;
    float2 *row_stats;               // scratch: [row tile][kv head][rows of a tile] (lse log2 e, delta)
    int32_t *status;
    int32_t wait_us, lose_load;      // tensor-core kernels: see skipffn_attention_tune
};

constexpr int AT_TC_ROWS = 128, AT_TC_KEYS = 128;       // tile of the tensor-core kernels
constexpr int AT_SIMT_ROWS = 64, AT_SIMT_KEYS = 64;     // tile of the plain-FMA kernels
constexpr int AT_MAX_D = 128;

// attention_tc.cu (bf16)
cudaError_t launch_attention_tc_forward(const AttnArgs &a, cudaStream_t s);
cudaError_t launch_attention_tc_backward(const AttnArgs &a, cudaStream_t s);
// attention_simt.cu
cudaError_t launch_attention_simt_forward(const AttnArgs &a, int dtype, cudaStream_t s);
cudaError_t launch_attention_simt_backward(const AttnArgs &a, int dtype, cudaStream_t s);
// row statistics of the tensor-core backward (attention_simt.cu)
cudaError_t launch_attention_row_stats_tc(const AttnArgs &a, cudaStream_t s);

}  // namespace skipffn
