// What the kernels of attention over the paged 4-bit cache share: what a query row may see, bytes of codes and scales.
#pragma once

#include "arl2_device.h"

namespace arl2 {

constexpr int kKeys = 32;        // keys of a block
constexpr int kTileRows = 256;   // query rows of a workgroup of the tile kernel

// What one workgroup's query rows may see.  A row is a (query token, query head of the stored head's group).
struct Span {
    int klen, qn;        // stored tokens of the stream, its query tokens
    int rows;            // query rows there are
    __device__ __forceinline__ int limit(int row, const KvAttnArgs &a) const
    {
        return a.causal ? kv_clamp(klen - qn + row / a.G + 1, klen) : klen;
    }
};
__device__ __forceinline__ Span span_of(const KvAttnArgs &a, int b)
{
    Span s;
    s.klen = kv_clamp(a.kv_len[b], kv_capacity(a.pool));
    s.qn = a.q_len != nullptr ? kv_clamp(a.q_len[b], a.Lq) : a.Lq;
    s.rows = s.qn * a.G;
    return s;
}

// The first n bytes of a word, n any number; and its bytes of 255.
__device__ __forceinline__ uint32_t first_bytes(int n) { return n >= 4 ? ~0u : n <= 0 ? 0u : (1u << (8 * n)) - 1u; }
__device__ __forceinline__ uint32_t bytes_255(uint32_t w)
{
    uint32_t x = w & (w >> 4) & 0x0f0f0f0fu;
    x &= x >> 2 & 0x03030303u;
    x &= x >> 1 & 0x01010101u;
    return x * 255u;
}

// Scale byte b of a word as a conversion's scale operand, of which only the exponent bits count (measured for every exponent, with
// sign and mantissa bits set): the other bytes' bits need not be cleared.
template <int b>
__device__ __forceinline__ float scale_operand(uint32_t w)
{
    return __uint_as_float(b == 0 ? w << 23 : b == 1 ? w << 15 : b == 2 ? w << 7 : w >> 1);
}

hipError_t launch_kv_tile(const KvAttnArgs &a, unsigned groups, hipStream_t stream);

}  // namespace arl2
