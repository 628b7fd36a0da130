// What the kernels of attention over the paged 4-bit cache share: the query rows as operands, what a row may see.
#pragma once

#include "arl2_device.h"

namespace arl2 {

constexpr int kKeys = 32;        // keys of a block
constexpr int kTileRows = 256;   // query rows of a workgroup of the tile kernel
constexpr int kParts = 3;        // of a query feature

typedef __attribute__((ext_vector_type(6))) uint32_t u32x6;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(32))) __bf16 bf16x32;
typedef __attribute__((ext_vector_type(32))) float f32x32;

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

// Query features as B operands: lane (c, hh) has features 64 s + 32 hh .. + 31 of row c, as e2m1-scaled parts.
template <int D>
struct Query {
    static constexpr int STEPS = D / 64;
    u32x6 part[STEPS][kParts];
    uint32_t scale[STEPS];           // byte p: of part p
    __device__ __forceinline__ void load(const bf16_t *row, bool there)
    {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            union { u32x4 u[4]; bf16x32 v; } x;
#pragma unroll
            for (int i = 0; i < 4; ++i) x.u[i] = there ? *(const u32x4 *)(row + 64 * s + 8 * i) : u32x4{0, 0, 0, 0};
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) m = max(m, max(x.u[i][j] << 16 & 0x7fffffffu, x.u[i][j] & 0x7fff0000u));
            const bool finite = m < 0x7f800000u;
            const int e = finite ? max((int)(m >> 23) - 2, 27) : 127;      // largest magnitude in [4, 8) 2^(e - 127)
            scale[s] = (uint32_t)e | (uint32_t)(e - 4) << 8 | (uint32_t)(e - 8) << 16;
            if (!finite) scale[s] |= 255u;
#pragma unroll
            for (int p = 0; p < kParts; ++p) {
                const float unit = __uint_as_float((uint32_t)(e - 4 * p) << 23);
                part[s][p] = __builtin_amdgcn_cvt_scalef32_pk32_fp6_bf16(x.v, unit);
                const f32x32 taken = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(part[s][p], unit);
#pragma unroll
                for (int j = 0; j < 32; ++j) x.v[j] = to_bf16((float)x.v[j] - taken[j]);
            }
        }
    }
};

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
