// Where the rows of the paged 4-bit key/value cache lie.  Plain C++: the kernels use these functions, and so do host-side tests.
//
// A pool of n_pages pages of P = 2^shift tokens; per page and stored head (all of one page's heads behind one another):
//   key codes      [P][D/2]            a byte holds feature 2i (low half) and 2i + 1 (high half) of one token
//   value codes    [P/16][D/2][16]     likewise, but 16 tokens of one feature pair behind one another: the second product of
//                                      attention sums over tokens, and a lane loads what it multiplies as 16 bytes
//   key scales     [P][D/32]           a byte x stands for 2^(x - 127) and belongs to 32 features of a token; 255: NaN
//   value scales   [P/16][D/32][16]
// No byte belongs to two tokens: tokens are written one by one without reading their neighbours.
// Every array begins at a multiple of 16 bytes (P is a multiple of 16, D of 64).
#pragma once

#include <stddef.h>
#include <stdint.h>

#if defined(__HIPCC__)
#define ARL2_HD __host__ __device__ __forceinline__
#else
#define ARL2_HD inline
#endif

namespace arl2 {

struct KvPool {
    int shift;        // log2 of the tokens per page
    int heads;        // stored heads
    int n_pages;      // pages of the pool
    int max_pages;    // table entries per stream
};

ARL2_HD constexpr int kv_head_bytes(int shift, int D) { return (D + D / 16) << shift; }       // of one page
ARL2_HD constexpr size_t kv_pool_bytes(const KvPool &p, int D) { return (size_t)p.n_pages * p.heads * kv_head_bytes(p.shift, D); }

// Tokens that a stream's table row can place.
ARL2_HD int kv_capacity(const KvPool &p) { return p.max_pages << p.shift; }
ARL2_HD int kv_clamp(int n, int most) { return n < 0 ? 0 : n < most ? n : most; }

// Page of a token's position by the stream's table row, or -1: a position outside the table, an entry outside the pool.
// Nothing is stored there: no row is written, none is seen.
ARL2_HD int kv_page(const KvPool &p, const int32_t *row, int64_t pos)
{
    if (pos < 0 || pos >= (int64_t)kv_capacity(p)) return -1;
    const int32_t e = row[pos >> p.shift];
    return e >= 0 && e < p.n_pages ? e : -1;
}
// Offset of a page's bytes of one head in the pool.
ARL2_HD size_t kv_head_offset(const KvPool &p, int D, int page, int head)
{
    return ((size_t)page * p.heads + head) * (size_t)kv_head_bytes(p.shift, D);
}
// Offsets of the four arrays behind it, and of a token's entries in them: t the token's place in the page, i a feature pair,
// g a group of 32 features.
ARL2_HD int kv_key_codes(int t, int i, int D) { return t * (D / 2) + i; }
ARL2_HD int kv_value_codes(int shift, int t, int i, int D) { return ((D / 2) << shift) + ((t >> 4) * (D / 2) + i) * 16 + (t & 15); }
ARL2_HD int kv_key_scales(int shift, int t, int g, int D) { return (D << shift) + t * (D / 32) + g; }
ARL2_HD int kv_value_scales(int shift, int t, int g, int D) { return ((D + D / 32) << shift) + ((t >> 4) * (D / 32) + g) * 16 + (t & 15); }

}  // namespace arl2
