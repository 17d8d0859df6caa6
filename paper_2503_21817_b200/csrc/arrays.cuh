// Host checks of the arrays that entry points receive: alignment, extent, overlap.
#pragma once
#include <stdint.h>

namespace skipffn {

static inline bool is_aligned(const void *p, unsigned n) { return ((uintptr_t)p & (n - 1)) == 0; }

// A [tokens, heads, d] array: base, token stride and extent of a token's heads in bytes
struct TokenArray { const void *p; int64_t ld, width; };

// strides are bounded by what a tensor map takes and so that N of them stay within 64 bits
static inline bool token_array_ok(const TokenArray &a, int64_t N)
{
    return a.p && is_aligned(a.p, 16) && a.ld % 16 == 0 && a.ld >= a.width && a.ld <= (int64_t)1 << 38 && a.ld <= ((int64_t)1 << 60) / N;
}
// Do two arrays of N tokens share a byte?  Exact for equal strides (slices of one fused array), else by range.
static inline bool tokens_overlap(const TokenArray &x, const TokenArray &y, int64_t N)
{
    const intptr_t a = (intptr_t)x.p, b = (intptr_t)y.p;
    if (a >= b + (N - 1) * y.ld + y.width || b >= a + (N - 1) * x.ld + x.width) return false;
    if (x.ld != y.ld) return true;
    const int64_t off = ((b - a) % x.ld + x.ld) % x.ld;      // y's columns relative to x's inside one stride
    return off < x.width || off + y.width > x.ld;
}
// a contiguous block of bytes as an array of one token; null: no bytes
static inline bool ranges_overlap(const void *a, int64_t na, const void *b, int64_t nb)
{
    const uintptr_t p = (uintptr_t)a, q = (uintptr_t)b;
    return p && q && na > 0 && nb > 0 && p < q + nb && q < p + na;
}
static inline int64_t token_bytes(const TokenArray &a, int64_t N) { return N > 0 ? (N - 1) * a.ld + a.width : 0; }

}  // namespace skipffn
