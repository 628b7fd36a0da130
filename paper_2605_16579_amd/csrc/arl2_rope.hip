// Queries and keys divided by their root mean square, weighted and rotated by positions on several axes, and the gradients (gfx950):
//
//   y = R(pos) (w . x r),  r = 1 / sqrt(mean x^2 + eps) over a head's features, over a token's row, or no norm and no weight
//   R turns the pair i of axis a by pos_a theta_a^(-i / m_a):  (x0, x1) -> (x0 c - x1 s, x0 s + x1 c)
//   z = R(-pos) dy,   dw = sum over tokens of z . x r,   g = w z,   dx = r (g - x r mean(g . x r))
//
// The angle in turns is position times the pair's turns in fp64 (exact to 2^-53 of it, so far positions lose nothing), its
// fraction goes to fp32; cosines and sines of a token are computed once and pass through LDS to the lanes.  Memory bounds both.
//
// A unit is 8 pairs of a head, 16 features: neighbours (2i, 2i + 1), or i and i + D / 2.  A token's units (queries, then keys) are dealt to
// LPT lanes of a workgroup, the least power of two from 16 on that holds them, 256 at the most and then NU to a lane; a head's units divide LPT, so
// a lane's units all have the same pairs.  A workgroup takes 256 / LPT tokens side by side and, forward, TOK of each in a row: their loads are all
// requested before the first sum, and their sums cross the wavefronts together.  The gradients hold twice the rows and the weights' sums: one token,
// turned back once, and more wavefronts on a SIMD (4680 tokens of 12 + 12 heads x 128 by rows, four tokens with their turns made twice and three wavefronts: 39.4 us,
// this one 34.9, 33.1 without selects for weights that are not there, missing tokens and pairs without an axis: 2.6 TB/s, 32760 tokens 143 us, 4.2 TB/s).  A weight's gradient
// stays with its lane.
#include "arl2_device.h"
#include "arl2_rope.h"

#include <algorithm>

namespace arl2 {
namespace {

constexpr int kThreads = kRopeThreads;
constexpr int kMostWorkgroups = 1 << 20;         // (a launch has room for 2^32 threads)
static_assert(kRopeChip == kNumCu, "the plan counts this chip's CUs");

template <class T> struct Raw;                    // 8 features as they lie in memory
template <> struct Raw<bf16_t> { u32x4 v; };
template <> struct Raw<float> { f32x4 v[2]; };

__device__ __forceinline__ Raw<bf16_t> load8(const bf16_t *p) { return {*reinterpret_cast<const u32x4 *>(p)}; }
__device__ __forceinline__ Raw<float> load8(const float *p) { return {{*reinterpret_cast<const f32x4 *>(p), *reinterpret_cast<const f32x4 *>(p + 4)}}; }
__device__ __forceinline__ float feature(const Raw<bf16_t> &r, int i) { return __uint_as_float(i % 2 ? r.v[i / 2] & 0xffff0000u : r.v[i / 2] << 16); }
__device__ __forceinline__ float feature(const Raw<float> &r, int i) { return r.v[i / 4][i % 4]; }
__device__ __forceinline__ void store8(bf16_t *p, const float *x)
{
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const bf16x2 r = {to_bf16(x[2 * i]), to_bf16(x[2 * i + 1])};
        v[i] = __builtin_bit_cast(uint32_t, r);
    }
    *reinterpret_cast<u32x4 *>(p) = v;
}
__device__ __forceinline__ void store8(float *p, const float *x)
{
    *reinterpret_cast<f32x4 *>(p) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4 *>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}

// 8 pairs: halves of a head apart, or neighbours (then `hi` follows `lo`).
template <class T> struct Unit { Raw<T> lo, hi; };
template <class T>
__device__ __forceinline__ Unit<T> load_unit(const T *p, int hi) { return {load8(p), load8(p + hi)}; }

// Place of a pair's two features among the unit's 16.
template <bool HALVES> __device__ __forceinline__ constexpr int first_of(int pair) { return HALVES ? pair : 2 * pair; }
template <bool HALVES> __device__ __forceinline__ constexpr int second_of(int pair) { return HALVES ? 8 + pair : 2 * pair + 1; }
template <class T>
__device__ __forceinline__ float feature(const Unit<T> &u, int i) { return i < 8 ? feature(u.lo, i) : feature(u.hi, i - 8); }

__device__ __forceinline__ void fill(Raw<bf16_t> &r, float x) { r.v = u32x4{} + (__float_as_uint(x) >> 16 | __float_as_uint(x)); }      // (x: 0 or 1)
__device__ __forceinline__ void fill(Raw<float> &r, float x) { r.v[0] = r.v[1] = f32x4{x, x, x, x}; }
template <class T>
__device__ __forceinline__ void fill(Unit<T> &u, float x) { fill(u.lo, x); fill(u.hi, x); }

// The compiler is to take these registers for new values: else it keeps what it has widened and turned of every token for the second
// time that they are used (the gradients of a row: 256 registers and 1 KB of scratch a lane).
__device__ __forceinline__ void forget(Raw<bf16_t> &r) { asm volatile("" : "+v"(r.v)); }
__device__ __forceinline__ void forget(Raw<float> &r) { asm volatile("" : "+v"(r.v[0]), "+v"(r.v[1])); }
template <class T>
__device__ __forceinline__ void forget(Unit<T> &u) { forget(u.lo); forget(u.hi); }

// f(pair, cosine, sine) for the unit's eight pairs, two after the other: what is on its way at a time decides how many registers it takes.
template <class F>
__device__ __forceinline__ void each_pair(const f32x2 *turn, F &&f)
{
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
        const f32x4 v = *reinterpret_cast<const f32x4 *>(turn + i);
        f(i, v[0], v[1]);
        f(i + 1, v[2], v[3]);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// What a lane knows of its units: unit u of a token is number li + 256 u.
struct Lane {
    int upt, units0, units, lpt, slots, slot, li;     // units per head, of queries, of a token; lanes per token, tokens side by side
    int in_head, at, hi;                              // which of its head's units; its first features' place there, the others' distance
};
__device__ __forceinline__ Lane lane_of(const RopeArgs &a, int lpt, bool halves)
{
    Lane m;
    m.upt = a.D / 16;
    m.units0 = a.heads[0] * m.upt;
    m.units = m.units0 + a.heads[1] * m.upt;
    m.lpt = lpt;
    m.slots = kThreads / lpt;
    m.slot = threadIdx.x / lpt;
    m.li = threadIdx.x & (lpt - 1);
    m.in_head = m.li & (m.upt - 1);
    m.hi = halves ? a.D / 2 : 8;
    m.at = m.in_head * (halves ? 8 : 16);
    return m;
}
// Which array (0, 1; 2: none) the lane's unit u lies in, and the offset of its features in that array's rows.
__device__ __forceinline__ int place(const RopeArgs &a, const Lane &m, int u, int &offset)
{
    int i = m.li + u * kThreads;
    const int which = i < m.units0 ? 0 : i < m.units ? 1 : 2;
    if (which) i -= m.units0;
    offset = i / m.upt * a.D + m.at;
    return which;
}

// Sum over the lanes of a head's units (8 at D = 128, 4 at D = 64).
__device__ __forceinline__ float head_sum(float x, int upt)
{
    x += dpp_peek<0xB1>(x);
    x += dpp_peek<0x4E>(x);
    return upt == 8 ? x + dpp_peek<0x141>(x) : x;
}
// Sum over aligned groups of `n` lanes, 16 to 64.
__device__ __forceinline__ float group_sum(float x, int n)
{
    x = lane_group_sum<16>(x);
    const auto sum = [](auto v) { return __uint_as_float(v[0]) + __uint_as_float(v[1]); };
    if (n >= 32) x = sum(__builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    if (n >= 64) x = sum(__builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false));
    return x;
}

// Sums over a token's lanes of N values of each of TOK tokens; `red` and a barrier where the token has several wavefronts.
template <int TOK, int N>
__device__ __forceinline__ void token_sums(float (*x)[N], const Lane &m, float (*red)[TOK * N])
{
    const int wave = threadIdx.x >> 6, n = min(m.lpt, 64);
#pragma unroll
    for (int t = 0; t < TOK; ++t)
#pragma unroll
        for (int i = 0; i < N; ++i) x[t][i] = group_sum(x[t][i], n);
    if (m.lpt <= 64) return;
    if ((threadIdx.x & 63) == 0)
#pragma unroll
        for (int t = 0; t < TOK; ++t)
#pragma unroll
            for (int i = 0; i < N; ++i) red[wave][t * N + i] = x[t][i];
    lds_barrier();
    const int w0 = m.lpt == 128 ? wave & 2 : 0;
#pragma unroll
    for (int t = 0; t < TOK; ++t)
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[t][i] = red[w0][t * N + i] + red[w0 + 1][t * N + i];
            if (m.lpt == 256) x[t][i] += red[2][t * N + i] + red[3][t * N + i];
        }
}

// Cosines and sines of all pairs of `tokens` tokens from `first` on, by all threads; a barrier has to follow.
__device__ __forceinline__ void turns_of(const RopeArgs &a, uint32_t first, uint32_t all, int tokens, f32x2 (*turns)[64])
{
    const int half = a.D / 2;
    for (int i = threadIdx.x; i < tokens * half; i += kThreads) {
        const int pair = i & (half - 1), t = i / half;
        float c = 1.f, s = 0.f;                                   // (also behind the last token: a weight's gradient takes zeros times these)
        if (pair < a.pairs && first + t < all) {
            const size_t at = a.pos_per_stream ? first + t : (first + t) % (uint32_t)a.L;
            const double turn = (double)a.pos[at * a.axes + a.axis[pair]] * a.turns[pair];
            sincospif(2.f * (float)(turn - ::rint(turn)), &s, &c);
        }
        turns[t][pair] = f32x2{c, s};
    }
}
// Is there such a token (of a sequence that goes so far)?
__device__ __forceinline__ bool token_there(const RopeArgs &a, uint32_t t, uint32_t all)
{
    if (t >= all) return false;
    if (a.len == nullptr) return true;
    const uint32_t b = t / (uint32_t)a.L;
    return (int)(t - b * a.L) < a.len[b];
}

// 1 over the root of the mean square; `over`: 1 over the number of features.
__device__ __forceinline__ float inverse_rms(float squares, float over, float eps) { return fast_rsqrt(fmaf(squares, over, eps)); }

template <class T, int NORM, bool HALVES, int NU, int TOK>
__global__ __launch_bounds__(kThreads, NU == 1 ? 4 : NU <= 3 ? 3 : 2) void rope_kernel(RopeArgs a, int lpt)
{
    extern __shared__ __align__(16) f32x2 turns[][64];            // of two rounds in turn
    __shared__ float red[2][4][TOK * 2];
    const Lane m = lane_of(a, lpt, HALVES);
    const bool partial = a.pairs < a.D / 2;
    const int at_a_time = m.slots * TOK, left = a.pairs - 8 * m.in_head;
    Unit<T> w[NU];
    int which[NU], off[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        which[u] = place(a, m, u, off[u]);
        fill(w[u], 1.f);
        if (NORM != kNormNone && which[u] < 2 && a.w[which[u]] != nullptr) w[u] = load_unit((const T *)a.w[which[u]] + (NORM == kNormHead ? m.at : off[u]), m.hi);
    }
    const uint32_t all = (uint32_t)a.B * a.L;                     // (2e9 at the most: no step past it wraps around)
    const float over_head = 1.f / (float)a.D, over_row[2] = {1.f / (float)(a.heads[0] * a.D), 1.f / (float)(max(a.heads[1], 1) * a.D)};
    int round = 0;
    for (uint32_t t0 = blockIdx.x * at_a_time; t0 < all; t0 += gridDim.x * at_a_time, round ^= 1) {
        bool there[TOK];
        Unit<T> x[TOK][NU];
#pragma unroll
        for (int t = 0; t < TOK; ++t) {
            const uint32_t tok = t0 + m.slot * TOK + t;
            there[t] = token_there(a, tok, all);
#pragma unroll
            for (int u = 0; u < NU; ++u)
                if (there[t] && which[u] < 2) x[t][u] = load_unit((const T *)a.x[which[u]] + (size_t)tok * a.heads[which[u]] * a.D + off[u], m.hi);
        }
        f32x2 (*const mine)[64] = turns + round * at_a_time;
        turns_of(a, t0, all, at_a_time, mine);
        float row[TOK][2];
        if constexpr (NORM == kNormRow) {
#pragma unroll
            for (int t = 0; t < TOK; ++t) {
                row[t][0] = row[t][1] = 0.f;
#pragma unroll
                for (int u = 0; u < NU; ++u) {
                    float s = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) { const float f = feature(x[t][u], i); s = fmaf(f, f, s); }
                    row[t][0] += which[u] == 0 ? s : 0.f;
                    row[t][1] += which[u] == 1 ? s : 0.f;
                }
            }
            token_sums<TOK, 2>(row, m, red[round]);
        }
        if (NORM != kNormRow || m.lpt <= 64) lds_barrier();
#pragma unroll
        for (int t = 0; t < TOK; ++t) {
            const f32x2 *const turn = &mine[m.slot * TOK + t][8 * m.in_head];
            if constexpr (NORM == kNormRow)
#pragma unroll
                for (int i = 0; i < 2; ++i) row[t][i] = inverse_rms(row[t][i], over_row[i], a.eps);
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                float r = 1.f, y[16];
                if constexpr (NORM == kNormHead) {
                    float s = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) { const float f = feature(x[t][u], i); s = fmaf(f, f, s); }
                    r = inverse_rms(head_sum(s, m.upt), over_head, a.eps);
                } else if constexpr (NORM == kNormRow) r = which[u] == 1 ? row[t][1] : row[t][0];
                forget(x[t][u]);
                if (NORM != kNormNone) forget(w[u]);
                each_pair(turn, [&](int i, float c, float s) {
                    const int j0 = first_of<HALVES>(i), j1 = second_of<HALVES>(i);
                    float f0 = feature(x[t][u], j0), f1 = feature(x[t][u], j1);
                    if constexpr (NORM != kNormNone) {
                        f0 *= r;
                        f1 *= r;
                        f0 *= feature(w[u], j0);
                        f1 *= feature(w[u], j1);
                    }
                    y[j0] = f0 * c - f1 * s;
                    y[j1] = f0 * s + f1 * c;
                    if (partial && i >= left) { y[j0] = f0; y[j1] = f1; }
                });
                if (!there[t] || which[u] == 2) continue;
                T *const to = (T *)a.y[which[u]] + (size_t)(t0 + m.slot * TOK + t) * a.heads[which[u]] * a.D + off[u];
                store8(to, y);
                store8(to + m.hi, y + 8);
            }
        }
    }
}

// Groups of a workgroup's wavefronts that have sums of the same weights' gradients.
__host__ __device__ constexpr int part_groups(bool by_heads, int lpt) { return !by_heads && lpt == 128 ? 2 : 4; }

// A weight's gradient is summed over all of a workgroup's tokens by the lanes that have its feature, joined among them at the end and written
// as this workgroup's part.
template <class T, int NORM, bool HALVES, int NU>
__global__ __launch_bounds__(kThreads, rope_bwd_waves(NU, std::is_same<T, float>::value)) void rope_bwd_kernel(RopeArgs a, int lpt)
{
    extern __shared__ __align__(16) f32x2 turns[][64];
    __shared__ float red[2][4][4];
    const Lane m = lane_of(a, lpt, HALVES);
    const bool partial = a.pairs < a.D / 2;
    const int left = a.pairs - 8 * m.in_head;
    Unit<T> w[NU];
    float dw[NU][16] = {};
    int which[NU], off[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        which[u] = place(a, m, u, off[u]);
        fill(w[u], 1.f);
        if (NORM != kNormNone && which[u] < 2 && a.w[which[u]] != nullptr) w[u] = load_unit((const T *)a.w[which[u]] + (NORM == kNormHead ? m.at : off[u]), m.hi);
    }
    const uint32_t all = (uint32_t)a.B * a.L;                     // (2e9 at the most: no step past it wraps around)
    const float over_head = 1.f / (float)a.D, over_row[2] = {1.f / (float)(a.heads[0] * a.D), 1.f / (float)(max(a.heads[1], 1) * a.D)};
    int round = 0;
    for (uint32_t t0 = blockIdx.x * m.slots; t0 < all; t0 += gridDim.x * m.slots, round ^= 1) {
        const uint32_t tok = t0 + m.slot;
        const bool there = token_there(a, tok, all);
        Unit<T> x[NU], d[NU];
#pragma unroll
        for (int u = 0; u < NU; ++u)
            if (there && which[u] < 2) {
                const size_t at = (size_t)tok * a.heads[which[u]] * a.D + off[u];
                d[u] = load_unit((const T *)a.dy[which[u]] + at, m.hi);
                if (NORM != kNormNone) x[u] = load_unit((const T *)a.x[which[u]] + at, m.hi);
            } else if (NORM != kNormNone) {                       // (adds nothing to a weight's gradient)
                fill(d[u], 0.f);
                fill(x[u], 0.f);
            }
        f32x2 (*const mine)[64] = turns + round * m.slots;
        turns_of(a, t0, all, m.slots, mine);
        lds_barrier();
        const f32x2 *const turn = &mine[m.slot][8 * m.in_head];
        // a pair of dy turned back, times the weights: z into z0, z1 and w z into the others
        auto back = [&](int u, int i, float c, float s, float &z0, float &z1, float &g0, float &g1) {
            const int j0 = first_of<HALVES>(i), j1 = second_of<HALVES>(i);
            const float d0 = feature(d[u], j0), d1 = feature(d[u], j1);
            z0 = d0 * c + d1 * s;
            z1 = d1 * c - d0 * s;
            if (partial) {
                asm volatile("");
                if (i >= left) { z0 = d0; z1 = d1; }
            }
            g0 = z0;
            g1 = z1;
            if (NORM != kNormNone) {
                g0 *= feature(w[u], j0);
                g1 *= feature(w[u], j1);
            }
        };
        // squares of the unit's features, and their products with w z
        auto sums = [&](int u, float &sq, float &dot) {
            float q = 0.f, p = 0.f;
            if (NU > 1) forget(w[u]);
            each_pair(turn, [&](int i, float c, float s) {
                float z0, z1, g0, g1;
                back(u, i, c, s, z0, z1, g0, g1);
                const float f0 = feature(x[u], first_of<HALVES>(i)), f1 = feature(x[u], second_of<HALVES>(i));
                q = fmaf(f0, f0, fmaf(f1, f1, q));
                p = fmaf(f0, g0, fmaf(f1, g1, p));
                asm volatile("" : "+v"(q), "+v"(p));
            });
            sq = q;
            dot = p;
        };
        float row[1][4] = {};                                     // squares of queries and keys, products with their gradients
        if constexpr (NORM == kNormRow) {
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                float s, p;
                sums(u, s, p);
                row[0][0] += which[u] == 0 ? s : 0.f;
                row[0][1] += which[u] == 1 ? s : 0.f;
                row[0][2] += which[u] == 0 ? p : 0.f;
                row[0][3] += which[u] == 1 ? p : 0.f;
            }
            token_sums<1, 4>(row, m, red[round]);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                row[0][i] = inverse_rms(row[0][i], over_row[i], a.eps);
                row[0][2 + i] *= row[0][i] * over_row[i];
            }
        }
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            float r = 1.f, p = 0.f, y[16];
            if constexpr (NORM == kNormHead) {
                float s;
                sums(u, s, p);
                r = inverse_rms(head_sum(s, m.upt), over_head, a.eps);
                p = head_sum(p, m.upt) * r * over_head;
            } else if constexpr (NORM == kNormRow) {
                r = which[u] == 1 ? row[0][1] : row[0][0];
                p = which[u] == 1 ? row[0][3] : row[0][2];
            }
            if (NU > 1) {
                forget(d[u]);
                if (NORM != kNormNone) {
                    forget(x[u]);
                    forget(w[u]);
                }
            }
            each_pair(turn, [&](int i, float c, float s) {
                const int j0 = first_of<HALVES>(i), j1 = second_of<HALVES>(i);
                float z0, z1, g0, g1;
                back(u, i, c, s, z0, z1, g0, g1);
                if constexpr (NORM != kNormNone) {
                    const float h0 = feature(x[u], j0) * r, h1 = feature(x[u], j1) * r;
                    dw[u][j0] = fmaf(z0, h0, dw[u][j0]);
                    dw[u][j1] = fmaf(z1, h1, dw[u][j1]);
                    asm volatile("" : "+v"(dw[u][j0]), "+v"(dw[u][j1]));      // (now, not where the next token needs them: z and h would be kept)
                    g0 = r * (g0 - h0 * p);
                    g1 = r * (g1 - h1 * p);
                }
                y[j0] = g0;
                y[j1] = g1;
                if (i % 2) asm volatile("" : "+v"(y[first_of<HALVES>(i - 1)]), "+v"(y[second_of<HALVES>(i - 1)]), "+v"(y[j0]), "+v"(y[j1]));
            });
            if (!there || which[u] == 2) continue;
            T *const to = (T *)a.y[which[u]] + (size_t)tok * a.heads[which[u]] * a.D + off[u];
            store8(to, y);
            store8(to + m.hi, y + 8);
        }
    }
    if (NORM == kNormNone || (a.dw[0] == nullptr && a.dw[1] == nullptr)) return;
    // this workgroup's part: [D] and, where there are keys, [D], or [heads D] and [heads D]
    const int width0 = rope_part_queries(NORM == kNormHead, a.D, a.heads[0]), width = rope_part(NORM == kNormHead, a.D, a.heads[0], a.heads[1]);
    float *const to = a.part + (size_t)blockIdx.x * width;
    if (NORM == kNormRow && m.lpt == kThreads) {                  // each of its elements is one lane's
#pragma unroll
        for (int u = 0; u < NU; ++u)
            if (which[u] < 2)
#pragma unroll
                for (int i = 0; i < 16; ++i) to[(which[u] ? width0 : 0) + off[u] + (i < 8 ? i : m.hi + i - 8)] = dw[u][i];
        return;
    }
    // sums of lanes with the same features in a wavefront, and of the wavefronts (or pairs of them that have a token together) in LDS
    float *const part = reinterpret_cast<float *>(&turns[0][0]);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, groups = part_groups(NORM == kNormHead, m.lpt);
    auto lanes_sum = [&](float (&x)[16], int from) {
        for (int s = from; s < 64; s <<= 1)
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] += __shfl_xor(x[i], s, kWave);
    };
    auto hand_over = [&](const float (&x)[16], float *at) {
#pragma unroll
        for (int i = 0; i < 16; ++i) at[i < 8 ? i : m.hi + i - 8] = x[i];
    };
    __syncthreads();                                              // the turns have been read
    if constexpr (NORM == kNormHead) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            if (k == 1 && width == width0) break;                 // there are no keys, and no room for them
            float sum[16] = {};
#pragma unroll
            for (int u = 0; u < NU; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) sum[i] += which[u] == k ? dw[u][i] : 0.f;
            lanes_sum(sum, m.upt);
            if (lane < m.upt) hand_over(sum, part + wave * width + (k ? width0 : 0) + m.at);
        }
    } else {                                                      // (NU is 1)
        lanes_sum(dw[0], m.lpt);
        if (lane < m.lpt && which[0] < 2) hand_over(dw[0], part + wave * groups / 4 * width + (which[0] ? width0 : 0) + off[0]);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < width; i += kThreads) {
        float s = 0.f;
        for (int g = 0; g < groups; ++g) s += part[g * width + i];
        to[i] = s;
    }
}

// Weights' gradients: 32 columns (128 bytes: with 16, halves of a line were read by two XCDs, 5.0 for 3.9 us and 936 parts of 12 KB) to a workgroup, the
// workgroups' parts in 32 groups added in order.
__global__ __launch_bounds__(1024) void rope_dw_kernel(RopeArgs a, int parts, int width0, int width)
{
    __shared__ float sums[32][33];
    const int c = threadIdx.x & 31, g = threadIdx.x >> 5, first = blockIdx.x * 32;
    float s = 0.f;
    for (int p0 = g; p0 < parts; p0 += 512) {                     // sixteen on their way at a time
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = p0 + 32 * i < parts ? a.part[(size_t)(p0 + 32 * i) * width + first + c] : 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) s += v[i];
    }
    sums[g][c] = s;
    __syncthreads();
    s = group_sum(sums[c][g], 32);                                // column g of the 32
    const int col = first + g;
    float *const to = col < width0 ? a.dw[0] : a.dw[1];
    if (to != nullptr && c == 0) to[col < width0 ? col : col - width0] = s;
}

template <class T, int NORM, bool HALVES, bool BWD>
hipError_t launch_shape(const RopeArgs &a, const RopeShape &s, dim3 grid, unsigned lds, hipStream_t stream)
{
    constexpr bool f32 = std::is_same<T, float>::value;
#define ARL2_ROPE(NU, TOK) launch_kernel_lds(BWD ? rope_bwd_kernel<T, NORM, HALVES, NU> : rope_kernel<T, NORM, HALVES, NU, TOK>, grid, dim3(kThreads), lds, stream, a, s.lpt)
    return s.nu == 1 ? ARL2_ROPE(1, 2) : s.nu == 2 ? ARL2_ROPE(2, f32 ? 1 : 2) : s.nu == 3 ? ARL2_ROPE(3, 1) : ARL2_ROPE(6, 1);
#undef ARL2_ROPE
}
template <class T, bool BWD>
hipError_t launch_norm(const RopeArgs &a, const RopeShape &s, dim3 grid, unsigned lds, hipStream_t stream)
{
    if (a.halves)
        return a.norm == kNormNone ? launch_shape<T, kNormNone, true, BWD>(a, s, grid, lds, stream)
             : a.norm == kNormHead ? launch_shape<T, kNormHead, true, BWD>(a, s, grid, lds, stream) : launch_shape<T, kNormRow, true, BWD>(a, s, grid, lds, stream);
    return a.norm == kNormNone ? launch_shape<T, kNormNone, false, BWD>(a, s, grid, lds, stream)
         : a.norm == kNormHead ? launch_shape<T, kNormHead, false, BWD>(a, s, grid, lds, stream) : launch_shape<T, kNormRow, false, BWD>(a, s, grid, lds, stream);
}
template <bool BWD>
hipError_t launch_any(const RopeArgs &a, const RopeShape &s, int grid, hipStream_t stream)
{
    // the turns of two rounds; at the end the weights' gradients of a workgroup's groups: a part each, or (several tokens side by side) 16 KB together at most
    const bool by_heads = a.norm == kNormHead;
    const int width = by_heads || s.lpt < kThreads ? part_groups(by_heads, s.lpt) * rope_part(by_heads, a.D, a.heads[0], a.heads[1]) : 0;
    const unsigned lds = (unsigned)std::max<size_t>(2 * (kThreads / s.lpt) * s.tok * 64 * sizeof(f32x2), BWD ? width * sizeof(float) : 0);
    return a.f32 ? launch_norm<float, BWD>(a, s, dim3(grid), lds, stream) : launch_norm<bf16_t, BWD>(a, s, dim3(grid), lds, stream);
}

}  // namespace

hipError_t launch_rope(const RopeArgs &a, hipStream_t stream)
{
    const RopeShape s = rope_shape((a.heads[0] + a.heads[1]) * (a.D / 16), a.f32, false);
    // Without weights to load a workgroup takes one round of tokens (up to 2^20 of them); else 4 x 10920 tokens of 32 + 8 heads x 128 (two units a lane) took 196, 209, 221 us
    // with at most 1024, 4096 and any number of workgroups, 7 x 4680 tokens of 12 + 12 heads (one unit) 101, 90, 97 us.
    const int most = a.norm == kNormNone ? kMostWorkgroups : s.nu == 1 ? 4096 : 1024;
    return launch_any<false>(a, s, rope_workgroups(a.B, a.L, s, most), stream);
}

hipError_t launch_rope_bwd(const RopeArgs &a, hipStream_t stream)
{
    const RopeShape s = rope_shape((a.heads[0] + a.heads[1]) * (a.D / 16), a.f32, true);
    const int n = a.norm == kNormNone ? rope_workgroups(a.B, a.L, s, kMostWorkgroups) : rope_bwd_workgroups(a.B, a.L, s, a.f32);
    const hipError_t e = launch_any<true>(a, s, n, stream);
    if (e != hipSuccess || a.norm == kNormNone || (a.dw[0] == nullptr && a.dw[1] == nullptr)) return e;
    const bool by_heads = a.norm == kNormHead;
    const int width0 = rope_part_queries(by_heads, a.D, a.heads[0]), width = rope_part(by_heads, a.D, a.heads[0], a.heads[1]);
    return launch_kernel(rope_dw_kernel, dim3(width / 32), dim3(1024), stream, a, n, width0, width);
}

}  // namespace arl2
