// The linear branch as a causal recurrence over tokens, and its gradients (gfx950).  Per (stream, head), k' and q' the normalised rows:
//
//   S_t = a_t S_{t-1} + k'_t^T v_t        out_t = q'_t S_t
//   G_t = a_{t+1} G_{t+1} + q'_t^T dout_t        dq'_t = S_t dout_t    dk'_t = G_t v_t    dv_t = G_t^T k'_t    dS0 = a_1 G_1
//   E_t = a_t <S_{t-1}, G_t> = E_{t+1} + q'_t . dq'_t - k'_t . dk'_t,  the gradient of log a_t;    E_{L+1} = <S_L, dS>
//
// All four row results are one walk over blocks of 64 tokens.  With c_t the sum of log2 a over the block's tokens up to t, rows
// X that ask, rows Y and Z that make the state, T the state that the block begins with, r_t = 2^(c_t):
//   row_t = r_t (X_t T + sum_{s <= t} (X_t . Y_s) Z_s / r_s),        T <- 2^(c_end) (T + sum_s Y_s^T Z_s / r_s)
//   out: X, Y, Z = q', k', v        dq': dout, v, k', the state transposed
//   and backwards in time (r_t = 2^(c_end - c_t), s >= t):    dv: k', q', dout        dk': v, dout, q', the state transposed
// E by the same blocks: with G_ts = 2^(c_t - c_s) (q'_t . k'_s)(dout_t . v_s) for s < t in a block, a_t the part of q'_t . dq'_t that comes from the state, b_t
// that of k'_t . dk'_t,
//   E_t = E_{t+1} + a_t - b_t + sum_s G_ts - sum_u G_ut:
// a pair's product goes in and out again as one fp32 value.  (q'.dq' - k'.dk' of the rows would do it too, but each holds that product rounded in its own way,
// and E is small against it where the memory is short: one head with gates of 0.8, 1024 tokens: E was off by 2.1e-5 in the 2-norm.)
// The state is held without the factor 2^(base + c_end) that its blocks so far have gathered: c counts on from block to block (as `base`), and
// only where it has run below -32 is the state multiplied by it, and c begins anew.  Where it runs below -64 in a block (gates of zero among
// them) 1 / r_s would leave the range: such a block's products take their decays 2^(c_t - c_s) pair by pair.
#include "arl2_device.h"
#include "arl2_scan.h"

#include <algorithm>

namespace arl2 {
namespace {

constexpr int kBlock = 64;                    // tokens
constexpr int kStepTokens = 8;
constexpr double kLog2e = 1.4426950408889634;
typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
constexpr float kZeroGate = -2839.f;           // below: a gate of zero (2^-4095.8, of which fp32 has nothing left), from which the gates' gradients begin anew

enum Mode { kOut, kDq, kDk, kDv, kSum, kSumBack };       // the last two make states and no rows

// One call's arrays in the workspace: states [B*H][nseg + 1][D][D], the way forth (state i: what segment i begins with) and back
// (state i: the gradient of what segment i - 1 ends with), the segments' decays, the parts
// of E by tokens [3][B*H][L] (a_t; -b_t; G's), and <state, its gradient> at the segments' borders [B*H][nseg + 1].
struct Work {
    float *forth, *back, *decay_forth, *decay_back, *parts, *anchor;
    int nseg, seg;
};

// A wavefront has 32 columns of the state, and all of its rows or (HALVES = 2) half of them: then twice as many wavefronts ask the state for
// half of the sums each and hand them on to the one of two that finishes a token's row.
template <int D, int HALVES>
struct Cfg {
    static constexpr int NC = D / 32, NW = HALVES * NC;
    static constexpr int NT = 64 * NW;
    static constexpr int TPW = NC / HALVES;               // 32 x 32 tiles of the state
    static constexpr int OWN = 2 / HALVES;                // of a block's two times 32 tokens: rows that a wavefront finishes
    static constexpr int LPR = D / 8;                     // lanes to a row of 16-byte pieces
    static constexpr int ROW = 2 * D;
    static constexpr int MAT = kBlock * ROW;
    static constexpr int PROW = 2 * kBlock;               // products: pieces lie as those of rows of 64 features
    static constexpr int PMAT = kBlock * PROW;
    // The 16-byte piece c of row r lies at place c ^ swizzle(r): 16 rows' pieces c are in different banks, and so are 64 bytes of each of four
    // rows 4 i .. 4 i + 3, which a transposing read of half a wavefront takes.
    static __device__ __forceinline__ int swizzle64(int r) { return (r >> 1 & 1) << 2 | (r >> 2 & 3); }
    static __device__ __forceinline__ int swizzle(int r) { return D == 128 ? (r & 3) << 2 | (r >> 2 & 3) : swizzle64(r); }
};

// What a block's tokens are multiplied with.  Exponents are taken apart into whole and fractional parts, whose differences lose nothing however
// far c runs; a gate of zero is 2^-4096 (which a block's other gates cannot bring back).
constexpr float kFold = -32.f, kPairs = -64.f;
template <int D>
struct Scalars {
    // by the gates alone, of two blocks in turn
    float whole[2][kBlock], frac[2][kBlock];              // c_t
    float row[2][kBlock], col[2][kBlock], enter[2][kBlock];     // r_t, 1 / r_s, and what rows enter the state with
    float fold[2];                                        // what the state is multiplied with before they do; 1: it is left
    int pairs[2];                                         // products take their decays pair by pair
    // with the norms of the rows
    float post[kBlock], pcol[kBlock], penter[kBlock], norm[kBlock];
    union {
        float red[D / 32][kBlock][3];
        struct { float later[3][32], earlier[3][32]; } pair;      // of the 32 x 32 pairs of a block: sums of G over s, over u
    };
    int unclean;                                          // the state has columns of NaNs
};

__device__ __forceinline__ int tokens_of(const ScanArgs &a, int b)
{
    if (a.len == nullptr) return a.L;
    return min(max(a.len[b], 0), a.L);
}

template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_add(double x)
{
    const unsigned long long u = __builtin_bit_cast(unsigned long long, x);
    const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xf, false);
    const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xf, false);
    return x + __builtin_bit_cast(double, ((unsigned long long)hi << 32) | lo);
}
// Sum over the lanes up to this one.
__device__ __forceinline__ double wave_prefix(double x)
{
    x = dpp_add<0x111, 0xf>(x);        // row_shr 1, 2, 4, 8
    x = dpp_add<0x112, 0xf>(x);
    x = dpp_add<0x114, 0xf>(x);
    x = dpp_add<0x118, 0xf>(x);
    x = dpp_add<0x142, 0xa>(x);        // row_bcast 15 to rows 1 and 3, 31 to rows 2 and 3
    return dpp_add<0x143, 0xc>(x);
}

__device__ __forceinline__ double log2_gate(float la)
{
    double x = (double)la * kLog2e;
    x = x > 0.0 ? 0.0 : x;
    return x < -4096.0 ? -4096.0 : x;                     // (a NaN stays one)
}

// 2^x, with the fraction's exponential scaled by the whole part: fp32's own precision whatever the size of x.
__device__ __forceinline__ float exp2_of(double x)
{
    const double w = __builtin_floor(fmax(x, -4096.0));
    const float f = __builtin_amdgcn_exp2f((float)(x - w));
    return x < -4096.0 ? 0.f : __builtin_ldexpf(f, (int)w);
}

// Two fp32 values as N bf16 each, whose sum is off by 2^(-8 N) of them at the most.
template <int N>
__device__ __forceinline__ void split_pair(float x, float y, uint32_t (&part)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const bf16x2 p = {to_bf16(x), to_bf16(y)};
        part[i] = __builtin_bit_cast(uint32_t, p);
        if (i + 1 < N) asm("" : "+v"(part[i]));           // (else the compiler rounds x once more for what is left of it)
        x -= __uint_as_float(part[i] << 16);
        y -= __uint_as_float(part[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma(u32x4 a, bf16x8 b, f32x16 c) { return mfma(__builtin_bit_cast(bf16x8, a), b, c); }

// Where two bf16 values are an infinity or a NaN: all bits of that half.
__device__ __forceinline__ uint32_t not_finite(uint32_t two) { return __builtin_bit_cast(uint32_t, __builtin_bit_cast(u16x2, two & 0x7fff7fffu) >= (u16x2)0x7f80); }

// Sum with the lane in the other half-wave, without LDS.
__device__ __forceinline__ float halves_sum(float x)
{
    const auto v = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(v[0]) + __uint_as_float(v[1]);
}
// Sums over the 32 lanes of a half-wave of each of 16 registers: lane l receives that of register l % 16.
__device__ __forceinline__ float lanes_sums(float (&v)[16], int lane)
{
    auto halve = [&](auto ctrl, int n, bool upper) {
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const float keep = upper ? v[i + n] : v[i], send = upper ? v[i] : v[i + n];
            v[i] = keep + dpp_peek<decltype(ctrl)::value>(send);
        }
    };
    halve(std::integral_constant<int, 0x140>{}, 8, lane & 8);          // row_mirror: lane 15 - l
    halve(std::integral_constant<int, 0x141>{}, 4, lane & 4);          // row_half_mirror: 7 - l of the 8
    halve(std::integral_constant<int, 0x1B>{}, 2, lane & 2);           // quad_perm [3,2,1,0]
    halve(std::integral_constant<int, 0xB1>{}, 1, lane & 1);           // quad_perm [1,0,3,2]
    const auto rows = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[0]), __float_as_uint(v[0]), false, false);
    return __uint_as_float(rows[0]) + __uint_as_float(rows[1]);
}

template <int D, int MODE, int HALVES>
struct Walk {
    using C = Cfg<D, HALVES>;
    static constexpr bool REV = MODE == kDk || MODE == kDv || MODE == kSumBack;
    static constexpr bool ROWS = MODE != kSum && MODE != kSumBack;
    static constexpr bool GRAD = MODE == kDq || MODE == kDk;      // rows through the normalisation
    // bf16 parts of the state that rows are asked of, and of the weighted rows that enter it.  Of the state: one, as the products of rows are rounded once and the
    // result; of what enters: two, the state is off by 2.5e-6 in the 2-norm.  Three of either where sums with q and k are parts of E, whose errors add up over a segment:
    // with two, heads with gates of 0.8 had E off by 9.1e-6, with three by 1.0e-6 (with three of one and two of the other 6e-6).
    static constexpr int ASKED = GRAD ? 3 : 1, ENTER = GRAD ? 3 : 2;
    static constexpr int GROUP = 4;                               // of D / 16 products of rows: operands requested together
    static constexpr int ROUND = C::NT / C::LPR, ROUNDS = kBlock / ROUND;    // rows that the threads stage at a time
    // Sums for the other half lie where X and Z were at D = 64, whose workgroups have to leave room for others.
    static constexpr bool HANDS_ON = ROWS && HALVES == 2, IN_PLACE = D == 64;
    static constexpr int LDS_ROWS = (ROWS ? 3 : 2) * C::MAT + (ROWS ? C::PMAT : 0) + (HANDS_ON && !IN_PLACE ? C::NW * 4096 : 0);

    // `lds`: LDS_ROWS bytes.  Segment `seg` of (stream, head) bh.  True (of kOut alone): it is to be walked once more, `careful`.  A token's products with later ones are zeros,
    // but zero times a NaN is not: a NaN or an infinity in a row of v makes its feature of earlier tokens of its 32 a NaN too, and its column of the state.  Where a state has come
    // out so, the second walk takes what is not finite in v as zeros, and then that token's feature, the later ones' and the state's column are made NaNs.  (Rows of q and k reach
    // the products of their own tokens and later ones alone.  To look at v's rows in every block took 3.5 to 4.5 % of the call.)
    static __device__ __forceinline__ bool run(const ScanArgs &a, const Work &wk, int bh, int seg, unsigned char *lds, Scalars<D> &sc, bool careful = false)
    {
        int tid = threadIdx.x;
        if (MODE == kOut) asm volatile("" : "+v"(tid), "+s"(bh), "+s"(seg));      // (else the first walk keeps the second one's addresses)
        int lane = tid & 63, l32 = lane & 31, hh = lane >> 5;
        const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), column = HALVES == 1 ? wave : wave % C::NC, half = HALVES == 1 ? 0 : wave / C::NC;
        const int b = bh / a.H, h = bh - b * a.H;
        const int tokens = tokens_of(a, b), n = careful ? __builtin_amdgcn_readfirstlane(tokens) : tokens;     // (behind the first walk's stores no scalar load)
        const int nblk = (n + kBlock - 1) / kBlock;
        const int blk0 = seg * wk.seg, blk1 = min(blk0 + wk.seg, nblk);
        const int nact = max(1, (nblk + wk.seg - 1) / wk.seg);
        if (seg >= nact) return false;                            // (without tokens the first segment hands its state on)

        const uint32_t rs = (uint32_t)a.H * D * 2;                // bytes from token to token
        const size_t stream = (size_t)b * a.L * rs;
        const uint32_t range = (uint32_t)n * rs;
        auto rows_of = [&](const void *p) { return make_rsrc((const char *)p + stream, range); };
        const auto rv = rows_of(MODE == kDv ? a.v : a.k);         // (for G)
        const auto rx = rows_of(MODE == kOut ? a.q : MODE == kDq ? a.dout : MODE == kDk ? a.v : a.k);
        const auto ry = rows_of(MODE == kOut || MODE == kSum ? a.k : MODE == kDq ? a.v : MODE == kDk ? a.dout : a.q);
        const auto rz = rows_of(MODE == kOut || MODE == kSum ? a.v : MODE == kDq ? a.k : MODE == kDk ? a.q : a.dout);
        const auto rla = make_rsrc(a.la + (a.la ? (size_t)b * a.L * a.H : 0), a.la ? (uint32_t)n * a.H * 4 : 0);

        unsigned char *const lx = lds, *const ly = lds + (ROWS ? C::MAT : 0), *const lz = ly + C::MAT, *const lp = lz + C::MAT;

        // ---- the state: register j of the wavefront's tile t is row r0 + 32 t + 16 (j / 8) + 8 hh + j % 8, column e0 + l32
        f32x16 st[C::TPW];
        const int e0 = 32 * column, r0 = 32 * C::TPW * half;
        // its product with its gradient, which lies there and is not transposed: the wavefronts' sums
        auto with_gradient = [&](const float *there) {
            there += (size_t)(e0 + l32) * D + r0 + 8 * hh;
            float dot = 0.f;
#pragma unroll
            for (int t = 0; t < C::TPW; ++t)
#pragma unroll
                for (int j = 0; j < 16; j += 4) {
                    const f32x4 x = *reinterpret_cast<const f32x4 *>(there + 32 * t + 16 * (j / 8) + j % 8);
#pragma unroll
                    for (int i = 0; i < 4; ++i) dot = fmaf(x[i], st[t][j + i], dot);
                }
#pragma unroll
            for (int m = 32; m > 0; m >>= 1) dot += __shfl_xor(dot, m, kWave);
            if (lane == 0) sc.red[column][half][0] = dot;
        };
        auto anchor = [&](int border, float factor) {             // by one lane, behind a barrier
            float dot = 0.f;
#pragma unroll
            for (int w = 0; w < C::NW; ++w) dot += sc.red[w % C::NC][w / C::NC][0];
            wk.anchor[(size_t)bh * (wk.nseg + 1) + border] = dot * factor;
        };
        {
            const float *from = nullptr;
            if (ROWS && wk.nseg == 1) {                           // one segment: what the call begins with
                from = REV ? a.dS : a.S0;
                if (from != nullptr) from += (size_t)bh * D * D;
            } else if (ROWS) from = (REV ? wk.back : wk.forth) + ((size_t)bh * (wk.nseg + 1) + seg + (REV ? 1 : 0)) * D * D;
            if (from == nullptr) {
#pragma unroll
                for (int t = 0; t < C::TPW; ++t) st[t] = f32x16{};
            } else if (GRAD) {                                    // transposed
#pragma unroll
                for (int t = 0; t < C::TPW; ++t)
#pragma unroll
                    for (int j = 0; j < 16; j += 4) {
                        const f32x4 x = *reinterpret_cast<const f32x4 *>(from + (size_t)(e0 + l32) * D + r0 + 32 * t + 16 * (j / 8) + 8 * hh + j % 8);
#pragma unroll
                        for (int i = 0; i < 4; ++i) st[t][j + i] = x[i];
                    }
                if (MODE == kDq && seg > 0 && a.dla != nullptr) with_gradient(wk.back + ((size_t)bh * (wk.nseg + 1) + seg) * D * D);
            } else {
#pragma unroll
                for (int t = 0; t < C::TPW; ++t)
#pragma unroll
                    for (int j = 0; j < 16; ++j) st[t][j] = from[(size_t)(r0 + 32 * t + 16 * (j / 8) + 8 * hh + j % 8) * D + e0 + l32];
            }
        }

        // ---- a block's rows on their way through registers, in 16-byte pieces
        const uint32_t piece0 = (uint32_t)(tid / C::LPR) * rs + (uint32_t)h * D * 2 + (tid % C::LPR) * 16;
        u32x4 gx[ROUNDS], gy[ROUNDS], gz[ROUNDS];
        float gla;
        auto fetch = [&](int blk) {
            const uint32_t o = piece0 + (uint32_t)blk * kBlock * rs;
            auto piece = [&](__amdgpu_buffer_rsrc_t r, int i) { return __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, o + (uint32_t)(ROUND * i) * rs, 0, 0)); };
#pragma unroll
            for (int i = 0; i < ROUNDS; ++i) {
                if (ROWS) gx[i] = piece(rx, i);
                gy[i] = piece(ry, i);
                gz[i] = piece(rz, i);
            }
        };
        auto fetch_gate = [&](int blk) {
            gla = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rla, ((uint32_t)(blk * kBlock + lane) * a.H + h) * 4u, 0, 0));
        };
        double seg_total = 0.0, base = 0.0;                       // (of the wavefront that does this)
        auto gates = [&](int buf) {
            const double c = wave_prefix(log2_gate(gla));
            const unsigned long long u = __builtin_bit_cast(unsigned long long, c);
            const double tot = __builtin_bit_cast(double, ((unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), 63) << 32) |
                                                           (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, 63));
            const double r = base + (REV ? tot - c : c), end = base + tot;
            const bool fold = !(end >= kFold), pairs = !(end >= kPairs);
            const double w = __builtin_floor(fmax(r, -4096.0));
            const float f = (float)(r - w);                       // (a NaN stays one)
            sc.row[buf][lane] = r < -4096.0 ? 0.f : __builtin_ldexpf(__builtin_amdgcn_exp2f(f), (int)w);
            float col = __builtin_ldexpf(__builtin_amdgcn_exp2f(-f), -(int)w);
            if (pairs) {
                sc.whole[buf][lane] = (float)__builtin_floor(c);
                sc.frac[buf][lane] = (float)(c - __builtin_floor(c));
                col = 0.f;
            }
            sc.col[buf][lane] = col;
            sc.enter[buf][lane] = col;
            float all = 1.f;
            if (fold) {
                sc.enter[buf][lane] = exp2_of(end - r);
                all = exp2_of(end);
            }
            if (lane == 0) {
                sc.fold[buf] = all;
                sc.pairs[buf] = pairs;
            }
            base = fold ? 0.0 : end;
            seg_total += tot;
        };
        // rows of one array to LDS
        auto stage = [&](const u32x4 *g, unsigned char *to) {
#pragma unroll
            for (int i = 0; i < ROUNDS; ++i) {
                const int row = ROUND * i + tid / C::LPR;
                *reinterpret_cast<u32x4 *>(to + row * C::ROW + (tid % C::LPR ^ C::swizzle(row)) * 16) = g[i];
            }
        };
        // norms of the rows that make the state and of those that ask, times their decays: lane r of a row's lanes finishes round r's
        auto norms = [&](const u32x4 *make, const u32x4 *ask, int buf) {
            int r = tid % C::LPR;
            if (ROWS && MODE != kOut) asm volatile("" : "+v"(r));  // (masks anew: the gradients' walks have no scalar registers left to keep them in)
            float mine = 0.f;
            auto squares = [&](const u32x4 *g, int first) {
                float x[ROUNDS];
#pragma unroll
                for (int i = 0; i < ROUNDS; ++i) {
                    x[i] = 0.f;
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const float x0 = __uint_as_float(g[i][j] << 16), x1 = __uint_as_float(g[i][j] & 0xffff0000u);
                        x[i] = fmaf(x0, x0, fmaf(x1, x1, x[i]));
                    }
                }
#pragma unroll
                for (int i = 0; i < ROUNDS; ++i) {
                    x[i] = lane_group_sum<C::LPR>(x[i]);
                    mine = r == first + i ? x[i] : mine;
                }
            };
            if (a.normalise) {
                squares(make, 0);
                if (!GRAD && ROWS) squares(ask, ROUNDS);
            }
            const float x = a.normalise ? fast_rsqrt(mine + a.eps) : 1.f;
            const int row = ROUND * (r & (ROUNDS - 1)) + tid / C::LPR;
            if (r < ROUNDS) {
                sc.pcol[row] = x * sc.col[buf][row];
                sc.penter[row] = x * sc.enter[buf][row];
                sc.norm[row] = x;
            } else if (!GRAD && ROWS && r < 2 * ROUNDS) sc.post[row] = sc.pairs[buf] ? x : x * sc.row[buf][row];
        };

        const int count = blk1 - blk0;
        auto block_at = [&](int i) { return REV ? blk1 - 1 - i : blk0 + i; };
        constexpr int GW = 3;                                     // the wavefront with the gates: it has fewest products
        if (count > 0) {
            fetch(block_at(0));
            fetch_gate(block_at(0));
            if (wave == GW) gates(0);
            if (MODE == kOut && tid == 0) sc.unclean = 0;
            if (count > 1) fetch_gate(block_at(1));
            lds_barrier();
            if (MODE == kDq && tid == 0 && seg > 0 && a.dla != nullptr) anchor(seg, 1.f);
        }
        // rows as operands: the lane's piece 2 m + hh of row l32 of a block's 32 lies at (row_at ^ 32 m); by columns, the lane's 8 bytes of
        // four of 16 tokens at tr_at[0], of the next four at tr_at[1], each ^ 64 per 32 columns.  For the state's step pieces 1 and 2 of four change
        // places: rows of its accumulator are then features 8 hh + j, as the operand of the rows' product with the state wants them.
        int row_at = l32 * C::ROW + 16 * (hh ^ C::swizzle(l32));
        int z_at[2], y_at[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int r = lane & 15, row = 8 * hh + 4 * k + (r >> 2), group = 2 * ((lane >> 4) & 1), swapped = (r & 1) << 1 | (r >> 1 & 1);
            z_at[k] = row * C::ROW + 16 * ((group + (r & 3) / 2) ^ C::swizzle(row)) + 8 * (r & 1);
            y_at[k] = row * C::ROW + 16 * ((group + swapped / 2) ^ C::swizzle(row)) + 8 * (swapped & 1);
        }
        auto by_columns = [&](const unsigned char *mat, const int (&at)[2], int tile, int m) {
            return __builtin_shufflevector(lds_read_tr(mat + (at[0] ^ 64 * tile) + 16 * m * C::ROW), lds_read_tr(mat + (at[1] ^ 64 * tile) + 16 * m * C::ROW), 0, 1, 2, 3, 4, 5, 6, 7);
        };
        auto by_rows = [&](const unsigned char *mat, int block, int m) { return *reinterpret_cast<const bf16x8 *>(mat + 32 * block * C::ROW + (row_at ^ 32 * m)); };
        int diagonal = 4 * hh - l32;                              // of a pair of 32 x 32 rows: row of Y less row of X, register 0
        for (int i = 0; i < count; ++i) {
            const int blk = block_at(i), buf = i & 1;
            // (the compiler is to compute what it makes of these anew: addresses and masks kept from block to block would take the registers of the state;
            // gradients of 8 x 4680 tokens with 33 registers in scratch and 147 of the scalar ones in lanes: 610 us, with none and 28: 551)
            asm volatile("" : "+v"(row_at), "+v"(y_at[0]), "+v"(y_at[1]), "+v"(z_at[0]), "+v"(z_at[1]), "+v"(diagonal));
            if (HALVES == 1) asm volatile("" : "+v"(tid), "+v"(lane), "+v"(l32), "+v"(hh));
            // Of the workgroups on a CU the one that is furthest in its block goes first: they are then not all at the same step.  With one priority gradients of 5 x 999
            // tokens of 24 heads x 64 took 76.5 us, so 71.4, of 8 x 4680 tokens of 12 heads x 128 547 and 535.
            __builtin_amdgcn_s_setprio(1);
            norms(GRAD ? gz : gy, gx, buf);
            if (MODE == kOut && careful)
#pragma unroll
                for (int r = 0; r < ROUNDS; ++r)
#pragma unroll
                    for (int j = 0; j < 4; ++j) gz[r][j] &= ~not_finite(gz[r][j]);
            if (ROWS) stage(gx, lx);
            stage(gy, ly);
            stage(gz, lz);
            if (!careful && i + 1 < count) fetch(block_at(i + 1));
            const bool pairs = __builtin_amdgcn_readfirstlane(sc.pairs[buf]) != 0;
            lds_barrier();

            __builtin_amdgcn_s_setprio(2);
            bf16x8 zf[4];                                         // Z^T of the wavefront's columns, 16 tokens each
            f32x16 acc[2] = {};                                   // rows of 32 tokens each, with two halves the wavefront's own ones first
            u32x2 own[C::OWN][4];                                 // the rows whose normalisation has a gradient
            float asked[C::OWN];                                  // their products with what the state gives
            // pairs of 32 x 32 rows: which of Y, which of X
            auto y_of = [](int t) { return REV ? (int)(t > 0) : (int)(t == 2); };
            auto x_of = [](int t) { return REV ? (int)(t == 2) : (int)(t > 0); };
            if constexpr (ROWS) {
                if (GRAD) {
                    const auto rg = rows_of(MODE == kDq ? a.q : a.k);
#pragma unroll
                    for (int o = 0; o < C::OWN; ++o)
#pragma unroll
                        for (int g = 0; g < 4; ++g)
                            own[o][g] = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rg, (uint32_t)(blk * kBlock + 32 * (o ^ half) + l32) * rs + (h * D + e0 + 8 * g + 4 * hh) * 2, 0, 0));
                }
                // the products of pair t, times their decays
                auto products = [&](int t) {
                    const int sb = y_of(t), tb = x_of(t);
                    f32x16 p = {};
#pragma unroll
                    for (int m0 = 0; m0 < D / 16; m0 += GROUP) {
                        bf16x8 yf[GROUP], xf[GROUP];
#pragma unroll
                        for (int m = 0; m < GROUP; ++m) {
                            yf[m] = by_rows(ly, sb, m0 + m);
                            xf[m] = by_rows(lx, tb, m0 + m);
                        }
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int m = 0; m < GROUP; ++m) p = mfma(yf[m], xf[m], p);
                    }
                    if (!pairs) {
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const f32x4 f = *reinterpret_cast<const f32x4 *>(&sc.pcol[32 * sb + 8 * g + 4 * hh]);
#pragma unroll
                            for (int j = 0; j < 4; ++j) p[4 * g + j] *= f[j];
                        }
                    } else {
                        const float wt = sc.whole[buf][32 * tb + l32], ft = sc.frac[buf][32 * tb + l32];
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const int s0 = 32 * sb + 8 * g + 4 * hh;
                            const f32x4 ws = *reinterpret_cast<const f32x4 *>(&sc.whole[buf][s0]), fs = *reinterpret_cast<const f32x4 *>(&sc.frac[buf][s0]),
                                        ys = *reinterpret_cast<const f32x4 *>(&sc.norm[s0]);
#pragma unroll
                            for (int j = 0; j < 4; ++j) p[4 * g + j] *= ys[j] * __builtin_amdgcn_exp2f(REV ? (ws[j] - wt) + (fs[j] - ft) : (wt - ws[j]) + (ft - fs[j]));
                        }
                    }
                    return p;
                };
                // ---- X.Y as rows of X in LDS, and from them G: products of k and q times those of dout, which lies in Z's place, and v
                if (wave < 3) {
                    const int t = wave, sb = y_of(t), tb = x_of(t);
                    constexpr int PIECES = MODE == kDv ? D / 16 : 1;
                    const bool pairs_too = MODE == kDv && a.dla != nullptr;
                    bf16x8 vf[PIECES];
                    if (pairs_too) {
                        const uint32_t row = (uint32_t)(blk * kBlock + 32 * tb + l32) * rs + (h * D + 8 * hh) * 2;
#pragma unroll
                        for (int m = 0; m < PIECES; ++m) vf[m] = __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rv, row + 32 * m, 0, 0));
                    }
                    f32x16 p = products(t);
                    if (sb == tb) {
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const int d = 8 * (j / 4) + j % 4 + diagonal;
                            p[j] = (REV ? d >= 0 : d <= 0) ? p[j] : 0.f;
                        }
                    }
                    unsigned char *const to = lp + (32 * tb + l32) * C::PROW + 8 * hh;
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const bf16x4 r = {to_bf16(p[4 * g]), to_bf16(p[4 * g + 1]), to_bf16(p[4 * g + 2]), to_bf16(p[4 * g + 3])};
                        *reinterpret_cast<bf16x4 *>(to + 16 * ((4 * sb + g) ^ C::swizzle64(l32))) = r;
                    }
                    if (pairs_too) {
                        f32x16 w = {};
#pragma unroll
                        for (int m = 0; m < PIECES; ++m) w = mfma(by_rows(lz, sb, m), vf[m], w);
                        const float post = sc.post[32 * tb + l32];
                        float v[16], sum = 0.f;
#pragma unroll
                        for (int j = 0; j < 16; ++j) {
                            const bool strictly = sb != tb || 8 * (j / 4) + j % 4 + diagonal > 0;
                            v[j] = strictly ? p[j] * post * w[j] : 0.f;   // (in this order: p has a decay taken out)
                            sum += v[j];
                        }
                        sum = halves_sum(sum);
                        if (hh == 0) sc.pair.earlier[t][l32] = sum;
                        const float of = lanes_sums(v, lane);
                        if ((lane & 16) == 0) sc.pair.later[t][8 * ((lane & 15) / 4) + 4 * hh + lane % 4] = of;
                    }
                }
                // ---- rows asked of the wavefront's part of the state
#pragma unroll
                for (int m = 0; m < 2 * C::TPW; ++m) {
                    u32x4 part[ASKED];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t w[ASKED];
                        split_pair(st[m / 2][8 * (m % 2) + 2 * j], st[m / 2][8 * (m % 2) + 2 * j + 1], w);
#pragma unroll
                        for (int k = 0; k < ASKED; ++k) part[k][j] = w[k];
                    }
                    const bf16x8 x0 = by_rows(lx, half, m + 2 * C::TPW * half), x1 = by_rows(lx, 1 - half, m + 2 * C::TPW * half);
#pragma unroll
                    for (int k = 0; k < ASKED; ++k) {
                        acc[0] = mfma(part[k], x0, acc[0]);
                        acc[1] = mfma(part[k], x1, acc[1]);
                    }
                }
                if (pairs) {
                    const float f0 = sc.row[buf][32 * half + l32], f1 = sc.row[buf][32 * (1 - half) + l32];
#pragma unroll
                    for (int j = 0; j < 16; ++j) { acc[0][j] *= f0; acc[1][j] *= f1; }
                }
                if (GRAD)
#pragma unroll
                    for (int o = 0; o < C::OWN; ++o) asked[o] = dot_of(own[o], acc[o]);
            }
#pragma unroll
            for (int m = 0; m < 4; ++m) zf[m] = by_columns(lz, z_at, column, m);
            if (i + 1 < count && wave == GW) gates(buf ^ 1);
            if (i + 2 < count) fetch_gate(block_at(i + 2));
            unsigned char *const exchange = !IN_PLACE ? lp + C::PMAT : column < C::NC / 2 ? lx : lz;
            const int place = IN_PLACE ? column % (C::NC / 2) * 2 : column * 2;
            auto hand_on = [&] {
                unsigned char *const to = exchange + (place + 1 - half) * 4096 + lane * 16;
#pragma unroll
                for (int g = 0; g < 4; ++g) *reinterpret_cast<f32x4 *>(to + 1024 * g) = f32x4{acc[1][4 * g], acc[1][4 * g + 1], acc[1][4 * g + 2], acc[1][4 * g + 3]};
            };
            if (HANDS_ON && !IN_PLACE) hand_on();
            __builtin_amdgcn_s_setprio(3);
            if (ROWS) lds_barrier();
            if (HANDS_ON && IN_PLACE) hand_on();                  // (nobody reads X and Z any more)

            // ---- and of the block's own rows
            if constexpr (ROWS)
#pragma unroll
                for (int o = 0; o < C::OWN; ++o) {
                    const int tb = o ^ half;
                    const unsigned char *const from = lp + (32 * tb + l32) * C::PROW;
                    auto tokens = [&](int m) { acc[o] = mfma(zf[m], *reinterpret_cast<const bf16x8 *>(from + 16 * ((2 * m + hh) ^ C::swizzle64(l32))), acc[o]); };
                    constexpr int same = REV ? 2 : 0;             // 32 tokens that all see, and those that the earlier or the later ones see
                    tokens(same);
                    tokens(same + 1);
                    if (tb == (REV ? 0 : 1)) {
                        tokens(2 - same);
                        tokens(3 - same);
                    }
                }

            // ---- the state's step: rows of Z times their weights
            const float fold = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(sc.fold[buf])));
            if (fold != 1.f) {
#pragma unroll
                for (int t = 0; t < C::TPW; ++t)
#pragma unroll
                    for (int j = 0; j < 16; ++j) st[t][j] *= fold;
            }
            {
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    constexpr bool FIRST = GRAD && HALVES == 2;   // requested before the split, where registers are left and it is long
                    bf16x8 y0;
                    if (FIRST) y0 = by_columns(ly, y_at, C::TPW * half, m);
                    const f32x4 w0 = *reinterpret_cast<const f32x4 *>(&sc.penter[16 * m + 8 * hh]), w1 = *reinterpret_cast<const f32x4 *>(&sc.penter[16 * m + 8 * hh + 4]);
                    const u32x4 zb = __builtin_bit_cast(u32x4, zf[m]);
                    u32x4 part[ENTER];
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t w[ENTER];
                        split_pair(__uint_as_float(zb[j] << 16) * (j < 2 ? w0[2 * j] : w1[2 * j - 4]), __uint_as_float(zb[j] & 0xffff0000u) * (j < 2 ? w0[2 * j + 1] : w1[2 * j - 3]), w);
#pragma unroll
                        for (int k = 0; k < ENTER; ++k) part[k][j] = w[k];
                    }
#pragma unroll
                    for (int t = 0; t < C::TPW; ++t) {
                        const bf16x8 yf = FIRST && t == 0 ? y0 : by_columns(ly, y_at, C::TPW * half + t, m);
#pragma unroll
                        for (int k = 0; k < ENTER; ++k) st[t] = mfma(yf, __builtin_bit_cast(bf16x8, part[k]), st[t]);
                    }
                }
            }

            __builtin_amdgcn_s_setprio(0);
            // ---- rows out
            if constexpr (ROWS) {
                if constexpr (HANDS_ON) {
                    if (IN_PLACE) lds_barrier();
                    const unsigned char *const from = exchange + (place + half) * 4096 + lane * 16;
                    f32x16 more;
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const f32x4 x = *reinterpret_cast<const f32x4 *>(from + 1024 * g);
#pragma unroll
                        for (int j = 0; j < 4; ++j) more[4 * g + j] = x[j];
                    }
                    if (GRAD) asked[0] += dot_of(own[0], more);
#pragma unroll
                    for (int j = 0; j < 16; ++j) acc[0][j] += more[j];
                }
                float scale[C::OWN], along[C::OWN];
#pragma unroll
                for (int o = 0; o < C::OWN; ++o) {
                    const int tok = 32 * (o ^ half) + l32;        // in the block
                    scale[o] = GRAD ? (pairs ? 1.f : sc.row[buf][tok]) : sc.post[tok];
                    if (GRAD) {
                        float ss = 0.f;
#pragma unroll
                        for (int g = 0; g < 4; ++g)
#pragma unroll
                            for (int j = 0; j < 2; ++j) {
                                const float x0 = __uint_as_float(own[o][g][j] << 16), x1 = __uint_as_float(own[o][g][j] & 0xffff0000u);
                                ss = fmaf(x0, x0, fmaf(x1, x1, ss));
                            }
                        ss = halves_sum(ss);
                        const float dot = halves_sum(dot_of(own[o], acc[o])), from_state = halves_sum(asked[o]);
                        if (hh == 0) {
                            sc.red[column][tok][0] = dot;
                            sc.red[column][tok][1] = from_state;
                            sc.red[column][tok][2] = ss;
                        }
                    }
                }
                float *const parts = wk.parts + ((MODE == kDq ? 0 : MODE == kDk ? (size_t)a.B * a.H : 2 * (size_t)a.B * a.H) + bh) * a.L + blk * kBlock;
                if (MODE == kDv && wave == 0 && blk * kBlock + lane < n && a.dla != nullptr)
                    parts[lane] = hh == 0 ? sc.pair.later[0][l32] - sc.pair.earlier[0][l32] - sc.pair.earlier[1][l32]
                                          : sc.pair.later[1][l32] + sc.pair.later[2][l32] - sc.pair.earlier[2][l32];
                lds_barrier();                                    // all have read the block's rows
                const auto ro = rows_of(MODE == kOut ? a.out : MODE == kDq ? a.dq : MODE == kDk ? a.dk : a.dv);
#pragma unroll
                for (int o = 0; o < C::OWN; ++o) {
                    const int tok = 32 * (o ^ half) + l32;
                    if (GRAD) {
                        float dot = 0.f, from_state = 0.f, ss = 0.f;
#pragma unroll
                        for (int w = 0; w < C::NC; ++w) {
                            dot += sc.red[w][tok][0];
                            from_state += sc.red[w][tok][1];
                            ss += sc.red[w][tok][2];
                        }
                        const float unit = a.normalise ? fast_rsqrt(ss + a.eps) : 1.f;
                        scale[o] *= unit;
                        along[o] = a.normalise ? -(dot * scale[o]) * unit * unit : 0.f;
                        if (column == 0 && hh == 0 && blk * kBlock + tok < n && a.dla != nullptr) parts[tok] = MODE == kDq ? from_state * scale[o] : -(from_state * scale[o]);
                    }
                    uint32_t w[4][2];
#pragma unroll
                    for (int g = 0; g < 4; ++g)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            float x0 = acc[o][4 * g + 2 * j] * scale[o], x1 = acc[o][4 * g + 2 * j + 1] * scale[o];
                            if (GRAD) {
                                x0 = fmaf(along[o], __uint_as_float(own[o][g][j] << 16), x0);
                                x1 = fmaf(along[o], __uint_as_float(own[o][g][j] & 0xffff0000u), x1);
                            }
                            const bf16x2 r = {to_bf16(x0), to_bf16(x1)};
                            w[g][j] = __builtin_bit_cast(uint32_t, r);
                        }
                    // 16 bytes of a row together: the half-waves hold 8 bytes each of four pieces
#pragma unroll
                    for (int g = 0; g < 2; ++g) {
                        const auto s0 = __builtin_amdgcn_permlane32_swap(w[g][0], w[g + 2][0], false, false);
                        const auto s1 = __builtin_amdgcn_permlane32_swap(w[g][1], w[g + 2][1], false, false);
                        const u32x4 v = {s0[0], s1[0], s0[1], s1[1]};
                        __builtin_amdgcn_raw_buffer_store_b128(v, ro, (uint32_t)(blk * kBlock + tok) * rs + (h * D + e0 + 16 * hh + 8 * g) * 2, 0, 0);
                    }
                }
            } else lds_barrier();
            if (careful && i + 1 < count) fetch(block_at(i + 1));     // (late: registers)
        }

        if (MODE == kOut && !careful && count > 0) {
            if (!(st[0][0] == st[0][0])) sc.unclean = 1;          // (what is not finite makes all rows of its column NaNs)
            lds_barrier();
            if (__builtin_amdgcn_readfirstlane(sc.unclean) != 0) {
                lds_barrier();
                return true;
            }
        }
        if (MODE == kOut && careful) {
            asm volatile("" : "+v"(l32), "+v"(hh));               // (addresses are made now)
            __threadfence();                                      // the rows have been written
            __syncthreads();
            const size_t column0 = ((size_t)b * a.L * a.H + h) * D + e0 + l32;
            const int last = min(blk1 * kBlock, n) - 1;
            bool seen = false;
            for (int t0 = blk0 * kBlock; t0 <= last; t0 += 8) {   // (the last token as often as it takes to make eight)
                uint16_t x[8];
#pragma unroll
                for (int t = 0; t < 8; ++t) x[t] = ((const uint16_t *)a.v)[column0 + (size_t)min(t0 + t, last) * a.H * D];
#pragma unroll
                for (int t = 0; t < 8; ++t) {
                    seen |= (x[t] & 0x7fff) >= 0x7f80;
                    if (seen && half == 0 && hh == 0) ((uint16_t *)a.out)[column0 + (size_t)min(t0 + t, last) * a.H * D] = 0x7fc0;
                }
            }
#pragma unroll
            for (int t = 0; t < C::TPW; ++t)
#pragma unroll
                for (int j = 0; j < 16; ++j) st[t][j] = seen ? __builtin_nanf("") : st[t][j];
        }

        // ---- the state at the end
        float *to = nullptr;
        if (MODE == kOut) to = seg == nact - 1 && a.S != nullptr ? a.S + (size_t)bh * D * D : nullptr;
        if (MODE == kDv) to = wk.nseg == 1 && a.dS0 != nullptr ? a.dS0 + (size_t)bh * D * D : nullptr;
        if (MODE == kSum) to = wk.forth + ((size_t)bh * (wk.nseg + 1) + seg + 1) * D * D;
        if (MODE == kSumBack) to = wk.back + ((size_t)bh * (wk.nseg + 1) + seg) * D * D;
        if (to != nullptr) {
            float gathered = 1.f;
            if (count > 0) {
                if (tid == 64 * GW) sc.fold[0] = exp2_of(base);   // (all have read it: a barrier ends every block)
                lds_barrier();
                gathered = sc.fold[0];
            }
#pragma unroll
            for (int t = 0; t < C::TPW; ++t)
#pragma unroll
                for (int j = 0; j < 16; ++j) to[(size_t)(r0 + 32 * t + 16 * (j / 8) + 8 * hh + j % 8) * D + e0 + l32] = st[t][j] * gathered;
        }
        if (MODE == kDq && seg == nact - 1 && a.dS != nullptr && a.dla != nullptr) {        // <S_L, dS>
            lds_barrier();                                        // all have read the last block's sums
            if (tid == 64 * GW) sc.fold[0] = count > 0 ? exp2_of(base) : 1.f;
            with_gradient(a.dS + (size_t)bh * D * D);
            lds_barrier();
            if (tid == 0) anchor(nact, sc.fold[0]);
        }
        if (!ROWS && tid == 64 * GW) (MODE == kSum ? wk.decay_forth : wk.decay_back)[(size_t)bh * wk.nseg + seg] = exp2_of(seg_total);
        return false;
    }

    // Product of 16 features of a row with the accumulator that lies over them.
    static __device__ __forceinline__ float dot_of(const u32x2 (&row)[4], const f32x16 &acc)
    {
        float dot = 0.f;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const uint32_t w = row[j / 4][(j / 2) % 2];
            dot = fmaf(__uint_as_float(j % 2 ? w & 0xffff0000u : w << 16), acc[j], dot);
        }
        return dot;
    }
};

// A block of 64 tokens takes 4.2 us (D = 128, one workgroup of eight wavefronts on a CU): the matrix cores are busy for 21 % of that, vector instructions take 39 % of the
// SIMDs' issue and LDS 26 % of its cycles, half of the wavefronts' time is waiting, for barriers, LDS and rows.  16 x 4096 tokens of 16 heads, one segment:
// 266 to 272 us, 4.1 TB/s, four fifths of a copy's; 32760 tokens of one stream, whose 21 segments are summed first: 107 + 58 + 7 us.  Two workgroups on a CU
// (128 registers, sums handed on in place): 168 for 172 us of the latter, 288 for 276 of the former, when a block took 4.4.
template <int D, int HALVES>
__global__ __launch_bounds__((Cfg<D, HALVES>::NT), D == 64 ? 3 : 2) void scan_out_kernel(ScanArgs a, Work wk)
{
    using W = Walk<D, kOut, HALVES>;
    __shared__ __align__(16) unsigned char lds[W::LDS_ROWS];
    __shared__ __align__(16) Scalars<D> sc;
    const int id = xcd_contiguous_id(blockIdx.x, gridDim.x);
    if (!W::run(a, wk, id / wk.nseg, id % wk.nseg, lds, sc)) return;
    // Once more, with the arguments read again: the first walk has no scalar registers left to keep them in (16 x 4096 tokens of 16 heads took 280 us for 269).
    struct Given { ScanArgs a; Work wk; };                        // (two arguments of like alignment lie so one behind the other)
    static_assert(alignof(ScanArgs) == alignof(Work) && sizeof(Given) == sizeof(ScanArgs) + sizeof(Work) && sizeof(Given) % 8 == 0, "");
    const __attribute__((address_space(4))) uint64_t *at = (const __attribute__((address_space(4))) uint64_t *)__builtin_amdgcn_kernarg_segment_ptr();
    int block = blockIdx.x;
    asm volatile("" : "+s"(at), "+s"(block));
    uint64_t words[sizeof(Given) / 8];
#pragma unroll
    for (int i = 0; i < (int)(sizeof(Given) / 8); ++i) words[i] = at[i];
    const Given given = __builtin_bit_cast(Given, words);
    const int unit = xcd_contiguous_id(block, gridDim.x);
    W::run(given.a, given.wk, unit / given.wk.nseg, unit % given.wk.nseg, lds, sc, true);
}

// Segments' own states, but for the last of the way forth.  `back`: the way back too, as every second workgroup; the first of the way back only where
// something reads it.
template <int D, int HALVES>
__global__ __launch_bounds__((Cfg<D, HALVES>::NT), 3) void scan_sum_kernel(ScanArgs a, Work wk, int back, int need_first)
{
    __shared__ __align__(16) unsigned char lds[Walk<D, kSum, HALVES>::LDS_ROWS];
    __shared__ __align__(16) Scalars<D> sc;
    const int id = xcd_contiguous_id(blockIdx.x, gridDim.x);
    const int unit = back ? id >> 1 : id;
    const int bh = unit / wk.nseg, seg = unit % wk.nseg;
    const int blocks = (tokens_of(a, bh / a.H) + kBlock - 1) / kBlock, nact = max(1, (blocks + wk.seg - 1) / wk.seg);
    if (back && (id & 1)) {
        if (seg > 0 || need_first) Walk<D, kSumBack, HALVES>::run(a, wk, bh, seg, lds, sc);
    } else if (seg < nact - 1) Walk<D, kSum, HALVES>::run(a, wk, bh, seg, lds, sc);
}

// States at the segments' borders from the segments' own: each its decay times the one before, plus its own.
__global__ __launch_bounds__(256) void scan_join_kernel(ScanArgs a, Work wk, int need_first)
{
    const int nn = a.D * a.D, per = nn / 1024, unit = blockIdx.x / per;
    const int e = ((blockIdx.x - unit * per) * 256 + threadIdx.x) * 4;
    const bool back = unit >= a.B * a.H;
    const int bh = back ? unit - a.B * a.H : unit;
    const int blocks = (tokens_of(a, bh / a.H) + kBlock - 1) / kBlock, nact = max(1, (blocks + wk.seg - 1) / wk.seg);
    float *const base = (back ? wk.back : wk.forth) + (size_t)bh * (wk.nseg + 1) * nn + e;
    const float *const decay = (back ? wk.decay_back : wk.decay_forth) + (size_t)bh * wk.nseg;
    const float *const start = back ? a.dS : a.S0;
    f32x4 x = {};
    if (start != nullptr) x = *reinterpret_cast<const f32x4 *>(start + (size_t)bh * nn + e);
    *reinterpret_cast<f32x4 *>(base + (size_t)(back ? nact : 0) * nn) = x;
    const int steps = nact - 1 + (back ? need_first : 0);
    constexpr int AHEAD = 16;                                     // states on their way at a time
    for (int i0 = 0; i0 < steps; i0 += AHEAD) {
        f32x4 own[AHEAD];
        float d[AHEAD];
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int step = min(i0 + i, steps - 1), seg = back ? nact - 1 - step : step;
            own[i] = *reinterpret_cast<const f32x4 *>(base + (size_t)(back ? seg : seg + 1) * nn);
            d[i] = decay[seg];
        }
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            if (i0 + i >= steps) break;
            const int seg = back ? nact - 1 - (i0 + i) : i0 + i;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = fmaf(d[i], x[j], own[i][j]);
            *reinterpret_cast<f32x4 *>(base + (size_t)(back ? seg : seg + 1) * nn) = x;
        }
    }
    if (back && a.dS0 != nullptr) *reinterpret_cast<f32x4 *>(a.dS0 + (size_t)bh * nn + e) = x;
}

// The rows' gradients: three walks of a segment by three workgroups that follow one another.  At D = 128 a wavefront has all rows of its columns, and two workgroups of four share a
// CU: 8 x 4680 tokens of 12 heads take 385 to 400 us in three times 15 blocks, 8.7 us for two workgroups' blocks; vector instructions take 51 % of the SIMDs' issue (half of them
// takes states and rows apart into bf16 parts), the matrix cores are busy for a third of the time, wavefronts wait for a third of it.
template <int D, int HALVES>
__global__ __launch_bounds__((Cfg<D, HALVES>::NT), D == 64 ? 3 : 2) void scan_grad_kernel(ScanArgs a, Work wk)
{
    __shared__ __align__(16) unsigned char lds[Walk<D, kDq, HALVES>::LDS_ROWS];
    __shared__ __align__(16) Scalars<D> sc;
    const int id = xcd_contiguous_id(blockIdx.x, gridDim.x);
    const int unit = id / 3, which = id - 3 * unit;
    const int bh = unit / wk.nseg, seg = unit % wk.nseg;
    if (which == 0) Walk<D, kDv, HALVES>::run(a, wk, bh, seg, lds, sc);
    else if (which == 1) Walk<D, kDk, HALVES>::run(a, wk, bh, seg, lds, sc);
    else Walk<D, kDq, HALVES>::run(a, wk, bh, seg, lds, sc);
}

// The gates' gradients of a segment: from <state, gradient of the state> at its end backwards, a sum that a gate of zero begins anew.
__global__ __launch_bounds__(256) void scan_gate_kernel(ScanArgs a, Work wk)
{
    constexpr int PER = 4;                                        // tokens of a thread: 1024 of a workgroup, which a segment has at the most
    __shared__ double ends[4];
    __shared__ int cuts[4];
    const int bh = blockIdx.x / wk.nseg, seg = blockIdx.x % wk.nseg, b = bh / a.H, h = bh - b * a.H;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int n = tokens_of(a, b), blocks = (n + kBlock - 1) / kBlock, nact = max(1, (blocks + wk.seg - 1) / wk.seg);
    const int t0 = seg * wk.seg * kBlock, t1 = min(n, t0 + wk.seg * kBlock);
    if (t0 >= t1) return;
    // this thread's tokens from late to early, later tokens in lower lanes
    double v[PER];
    int cut = 0;                                                  // bit i: a gate of zero; what lies behind it does not reach what lies before
    const int last = t0 + PER * 256 - 1 - PER * tid;
    const size_t rows = (size_t)a.B * a.H * a.L;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int t = last - i;
        const float *const p = wk.parts + (size_t)bh * a.L + t;
        v[i] = t < t1 ? (double)p[0] + p[rows] + p[2 * rows] : 0.0;
        if (t < t1 && a.la[((size_t)b * a.L + t) * a.H + h] < kZeroGate) cut |= 1 << i;
    }
    const double end = seg < nact - 1 || a.dS != nullptr ? wk.anchor[(size_t)bh * (wk.nseg + 1) + seg + 1] : 0.f;
    // sums within the thread, over the lanes before it, over the wavefronts before that
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        if (cut & 1 << i) v[i] = 0.0;
        else if (i > 0) v[i] += v[i - 1];
    }
    double run = v[PER - 1];
    int any = cut != 0;
#pragma unroll
    for (int m = 1; m < 64; m <<= 1) {
        const double u = __shfl_up(run, m, kWave);
        const int c = __shfl_up(any, m, kWave);
        if (lane >= m) {
            if (!any) run += u;
            any |= c;
        }
    }
    if (lane == 63) { ends[wave] = run; cuts[wave] = any; }
    __syncthreads();
    double before = end;
    for (int w = 0; w < wave; ++w) before = cuts[w] ? ends[w] : before + ends[w];
    const double lanes = __shfl_up(run, 1, kWave);
    const int lane_cut = __shfl_up(any, 1, kWave);
    if (lane > 0) before = lane_cut ? lanes : before + lanes;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int t = last - i;
        if ((cut & ((2 << i) - 1)) == 0) v[i] += before;          // (no gate of zero among this thread's tokens from the last to this one)
        if (t < t1) a.dla[((size_t)b * a.L + t) * a.H + h] = (float)v[i];
    }
}

// ---- few tokens: the state once in and out, by elements; 32 columns to a workgroup, 8 lanes to a row of them.  Bound by memory: one token of 16 streams of 12 heads x 128
// moves 25 MB in 7.2 us.
template <int D>
__global__ __launch_bounds__(256) void scan_step_kernel(ScanArgs a)
{
    constexpr int RPT = D / 32;                                   // rows per thread
    __shared__ __align__(16) float sq[kStepTokens][D], sk[kStepTokens][D], sv[kStepTokens][32];
    __shared__ float gate[kStepTokens];
    __shared__ __align__(16) float part[kStepTokens][4][32];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int e0 = 32 * (blockIdx.x % (D / 32)), bh = blockIdx.x / (D / 32), b = bh / a.H, h = bh - b * a.H;
    const int n = tokens_of(a, b);
    const int c4 = 4 * (tid & 7), r0 = tid >> 3;
    const size_t at = (size_t)bh * D * D + (size_t)r0 * D + e0 + c4;
    f32x4 st[RPT];
#pragma unroll
    for (int i = 0; i < RPT; ++i) st[i] = a.S0 != nullptr ? *reinterpret_cast<const f32x4 *>(a.S0 + at + (size_t)32 * i * D) : f32x4{};
    // one wavefront to a row of q or k
    for (int r = wave; r < 2 * n; r += 4) {
        const int t = r >> 1;
        const bf16_t *const src = (const bf16_t *)(r & 1 ? a.k : a.q) + (((size_t)b * a.L + t) * a.H + h) * D;
        const float x0 = lane < D / 2 ? (float)src[2 * lane] : 0.f, x1 = lane < D / 2 ? (float)src[2 * lane + 1] : 0.f;
        float s = x0 * x0 + x1 * x1;
#pragma unroll
        for (int m = 32; m > 0; m >>= 1) s += __shfl_xor(s, m, kWave);
        const float inv = a.normalise ? fast_rsqrt(s + a.eps) : 1.f;
        if (lane < D / 2) *reinterpret_cast<f32x2 *>(&(r & 1 ? sk : sq)[t][2 * lane]) = f32x2{x0 * inv, x1 * inv};
    }
    if (tid < 32 * n) sv[tid >> 5][tid & 31] = (float)((const bf16_t *)a.v)[(((size_t)b * a.L + (tid >> 5)) * a.H + h) * D + e0 + (tid & 31)];
    if (tid < n) gate[tid] = a.la == nullptr ? 1.f : (float)::exp2(log2_gate(a.la[((size_t)b * a.L + tid) * a.H + h]));
    __syncthreads();
    for (int t = 0; t < n; ++t) {
        const float g = gate[t];
        const f32x4 v = *reinterpret_cast<const f32x4 *>(&sv[t][c4]);
        f32x4 o = {};
#pragma unroll
        for (int i = 0; i < RPT; ++i) {
            const float k = sk[t][r0 + 32 * i], q = sq[t][r0 + 32 * i];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                st[i][j] = fmaf(k, v[j], g * st[i][j]);
                o[j] = fmaf(q, st[i][j], o[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int m = 8; m < 64; m <<= 1) o[j] += __shfl_xor(o[j], m, kWave);
        if (lane < 8) *reinterpret_cast<f32x4 *>(&part[t][wave][c4]) = o;
    }
    if (a.S != nullptr)
#pragma unroll
        for (int i = 0; i < RPT; ++i) *reinterpret_cast<f32x4 *>(a.S + at + (size_t)32 * i * D) = st[i];
    __syncthreads();
    if (tid < 32 * n) {
        const int t = tid >> 5, e = tid & 31;
        const float o = (part[t][0][e] + part[t][1][e]) + (part[t][2][e] + part[t][3][e]);
        ((bf16_t *)a.out)[(((size_t)b * a.L + t) * a.H + h) * D + e0 + e] = to_bf16(o);
    }
}

Work work_of(const ScanArgs &a, const ScanPlan &p)
{
    char *const w = (char *)a.workspace;
    const size_t decays = (size_t)a.B * a.H * p.nseg, rows = (size_t)a.B * a.H * a.L;
    Work wk;
    wk.forth = (float *)w;
    wk.back = (float *)(w + p.back);
    wk.decay_forth = (float *)(w + p.decay);
    wk.decay_back = wk.decay_forth + decays;
    wk.parts = (float *)(w + p.dots);
    wk.anchor = wk.parts + 3 * rows;
    wk.nseg = p.nseg;
    wk.seg = p.seg;
    return wk;
}

template <int D>
hipError_t launch_sums(const ScanArgs &a, const ScanPlan &p, const Work &wk, bool back, int first, hipStream_t stream)
{
    if (p.nseg == 1) return hipSuccess;
    const int bh = a.B * a.H, ways = back ? 2 : 1;
    const hipError_t e = launch_kernel(scan_sum_kernel<D, 2>, dim3(ways * bh * p.nseg), dim3(Cfg<D, 2>::NT), stream, a, wk, (int)back, first);
    if (e != hipSuccess) return e;
    return launch_kernel(scan_join_kernel, dim3(ways * bh * (D * D / 1024)), dim3(256), stream, a, wk, first);
}

template <int D>
hipError_t launch_fwd(const ScanArgs &a, const ScanPlan &p, hipStream_t stream)
{
    const int bh = a.B * a.H;
    if (p.step) return launch_kernel(scan_step_kernel<D>, dim3(bh * (D / 32)), dim3(256), stream, a);
    const Work wk = work_of(a, p);
    const hipError_t e = launch_sums<D>(a, p, wk, false, 0, stream);
    if (e != hipSuccess) return e;
    return launch_kernel(scan_out_kernel<D, 2>, dim3(bh * p.nseg), dim3(Cfg<D, 2>::NT), stream, a, wk);
}

template <int D, int HALVES>
hipError_t launch_bwd(const ScanArgs &a, const ScanPlan &p, hipStream_t stream)
{
    const int bh = a.B * a.H;
    const Work wk = work_of(a, p);
    hipError_t e = launch_sums<D>(a, p, wk, true, a.dS0 != nullptr, stream);
    if (e != hipSuccess) return e;
    e = launch_kernel(scan_grad_kernel<D, HALVES>, dim3(3 * bh * p.nseg), dim3(Cfg<D, HALVES>::NT), stream, a, wk);
    if (e != hipSuccess || a.dla == nullptr) return e;
    return launch_kernel(scan_gate_kernel, dim3(bh * p.nseg), dim3(256), stream, a, wk);
}

size_t align256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace

// Segments: enough workgroups for the chip, no more states than that takes.  Time is counted in hundredths of a block of a full chip, which has `per_cu` workgroups
// on a CU (one alone takes 70 and 60 hundredths of two's and three's); a second part of the sequence costs the sums of the segments (a block half of one), what joins them,
// by segment, and two launches.  12 heads x 128: 1560 tokens in 7, 9, 13 (taken), 25 segments 31.4, 27.6, 24.9, 32.7 us; 32760 in 15, 21 (taken), 32, 42: 210,
// 169, 188, 176 us; gradients of 1560 in 3, 7, 13 (taken), 25: 84, 52.5, 48.5, 64 us; of 8 x 4680 in 5 (taken), 6, 8, 10: 518, 554, 564, 577 us; 24 heads x 64: 5 x 2999 in
// 4, 6 (taken), 8: 71, 60.4, 67 us; gradients of 5 x 999 in 1 (taken), 2, 4: 61.7, 68.3, 71.9 us.  All pairs have the same number of segments, and some counts of pairs fit
// the chip badly: 4096 tokens of 96, 128, 192, 256, 257, 320, 384, 448, 512 pairs x 128 take 177, 206, 243, 271, 430, 486, 486, 508, 534 us.
ScanPlan scan_plan(int B, int H, int L, int D, bool backward)
{
    ScanPlan p = {};
    const int blocks = (L + kBlock - 1) / kBlock, per_cu = D == 64 ? 3 : backward ? 2 : 1;
    const long long bh = (long long)B * H, walks = (backward ? 3 : 1) * bh;
    p.nseg = 1;
    if (!backward && L <= kStepTokens) {
        p.step = 1;
        return p;
    }
    double best = 0.0;
    for (int r = 0; r <= 2 * per_cu + 2; ++r) {                   // segments for r workgroups on each CU
        const long long want = r == 0 ? 1 : std::min<long long>(r * kNumCu / walks, blocks);
        if (want < 1) continue;
        const int seg = std::min((int)((blocks + want - 1) / want), backward ? 16 : blocks), nseg = (blocks + seg - 1) / seg;
        const long long all = walks * nseg, full = all / (per_cu * kNumCu), rest = (all % (per_cu * kNumCu) + kNumCu - 1) / kNumCu;
        double cost = seg * (100.0 * full + (rest ? 40.0 + 60.0 * rest / per_cu : 0.0));
        if (nseg > 1) cost += 50.0 * seg * ((bh * nseg + kNumCu - 1) / kNumCu) + 8.0 * nseg + 150.0;
        if (best == 0.0 || cost < best) {
            best = cost;
            p.seg = seg;
            p.nseg = nseg;
        }
    }
    const size_t states = p.nseg > 1 ? align256((size_t)bh * (p.nseg + 1) * D * D * sizeof(float)) : 0;
    const size_t decays = p.nseg > 1 ? align256((size_t)2 * bh * p.nseg * sizeof(float)) : 0;
    p.back = states;
    p.decay = backward ? 2 * states : states;
    p.dots = p.decay + decays;
    p.bytes = p.dots + (backward ? align256((size_t)bh * (3 * (size_t)L + p.nseg + 1) * sizeof(float)) : 0);
    return p;
}

hipError_t launch_scan_fwd(const ScanArgs &a, const ScanPlan &p, hipStream_t stream)
{
    return a.D == 128 ? launch_fwd<128>(a, p, stream) : launch_fwd<64>(a, p, stream);
}

hipError_t launch_scan_bwd(const ScanArgs &a, const ScanPlan &p, hipStream_t stream)
{
    return a.D == 128 ? launch_bwd<128, 1>(a, p, stream) : launch_bwd<64, 2>(a, p, stream);
}

}  // namespace arl2
