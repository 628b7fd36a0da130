// How the rotation deals a token's rows to a workgroup's lanes, and the workspace that its weights' gradients take: host and kernels, no device code.
#pragma once

#include <stddef.h>

namespace arl2 {

constexpr int kRopeThreads = 256, kRopeChip = 256;               // lanes of a workgroup; CUs
constexpr int kRopeMostUnits = 1536;                             // of 16 features, queries and keys of a token together

// How tokens are dealt: lanes to a token, units to a lane, tokens of a lane at a time.
struct RopeShape { int lpt, nu, tok; };
constexpr RopeShape rope_shape(int units, bool f32, bool bwd)
{
    int lpt = 16;                                                 // (fewer would want more LDS for the turns of more tokens)
    while (lpt < units && lpt < kRopeThreads) lpt <<= 1;
    const int nu = units <= kRopeThreads ? 1 : units <= 2 * kRopeThreads ? 2 : units <= 3 * kRopeThreads ? 3 : 6;
    return {lpt, nu, bwd || nu > 2 || (nu == 2 && f32) ? 1 : 2};
}

// Wavefronts on a SIMD that the gradients' registers leave room for, and workgroups on a CU: with more, weights' gradients come in more parts.  One unit, 4680 tokens
// of 12 + 12 heads x 128: 3, 4, 5 wavefronts 38.6, 36.0, 37.2 us (the last with registers in scratch); two units, 32 + 8 heads: 3, 4 wavefronts 57.8, 54.5 us.
constexpr int rope_bwd_waves(int nu, bool f32) { return nu == 1 || (nu == 2 && !f32) ? 4 : 2; }

// Workgroups that have B L tokens among them, `most` at the most.
constexpr int rope_workgroups(int B, int L, const RopeShape &s, int most)
{
    const long long at_a_time = (long long)(kRopeThreads / s.lpt) * s.tok, n = ((long long)B * L + at_a_time - 1) / at_a_time;
    const long long rounds = (n + most - 1) / most;
    return (int)((n + rounds - 1) / rounds);                      // (as many tokens for each as can be)
}
constexpr int rope_bwd_workgroups(int B, int L, const RopeShape &s, bool f32) { return rope_workgroups(B, L, s, rope_bwd_waves(s.nu, f32) * kRopeChip); }

// A workgroup's part of the weights' gradients, in floats: the queries', then the keys' where there are keys; of a head's features (a norm by heads) or a row's.
constexpr int rope_part_queries(bool by_heads, int D, int H) { return by_heads ? D : H * D; }
constexpr int rope_part(bool by_heads, int D, int H, int Hk) { return rope_part_queries(by_heads, D, H) + (by_heads ? (Hk > 0 ? D : 0) : Hk * D); }

// Enough for either norm (a row is as wide as its heads, of which there is one at least for each part) and type (bf16 rows have the more workgroups).
constexpr size_t rope_parts_bytes(int B, int L, int D, int H, int Hk)
{
    const size_t n = (size_t)rope_bwd_workgroups(B, L, rope_shape((H + Hk) * (D / 16), false, true), false);
    return (n * rope_part(false, D, H, Hk) * sizeof(float) + 255) & ~(size_t)255;
}

}  // namespace arl2
