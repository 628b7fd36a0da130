// Attention over the paged 4-bit key/value cache (gfx950):
//   out_i = sum_j softmax_j(sm_scale * q_i.K_j) V_j      over the stored tokens j of the stream, all or (causal) up to query i
//
// Here: the kernel for few query rows (single tokens, drafts: up to 64 rows of a stored head), the join of what several workgroups
// found for the same rows, and the choice between this kernel and that of arl2_kv_tile.hip.
//
// Few rows: reading the cache is all there is to do (136 bytes of a token and head at D = 128 against 2 D multiplications).  Workgroups
// of four wavefronts take 32 rows (columns of the matrix products; one is as good as 32) and a split of the tokens.  A wavefront
// works alone on every fourth block of 32 tokens: it copies blocks straight into an LDS ring of its own, two ahead of the one it is
// on, and waits on nothing but its own loads.  13 KB per wavefront, three workgroups per CU: 104 KB of a CU on their way.  Keys and values are
// converted to bf16, in which they are exact.  At the end the wavefronts' results, each with its own maximum and sum, are added.
// Measured: 131001 tokens of 8 stored heads, 32 query heads: 33 us (4.3 TB/s; a copy of 1 GiB moves 4.85 TB/s) and 5 us for the
// join; 64 streams of 1 to 7122 tokens 31 us, of which a workgroup's fixed part (lengths, table, first blocks, ending: 5 us) and
// splits that turn out empty are most.  Two workgroups per CU with a block more ahead: 38.5 and 39.6 us instead of 38.4 and 35.2 in all.
#include "arl2_kv_attn.h"

#include <limits.h>

#include <algorithm>

namespace arl2 {
namespace {

constexpr int kRows = 32;        // query rows of a workgroup
constexpr int kWaves = 4;
constexpr int kSlots = 3 * kNumCu;     // workgroups that run at a time at D = 128 (D = 64: four of them find room on a CU; divided alike)

// LDS of a wavefront: a ring of blocks of 32 tokens as they are stored, per 16-token group key codes [16-byte piece of a row][token],
// value codes, key scales, value scales.
template <int D>
struct Stream {
    static constexpr int STEPS = D / 64, OB = D / 32;
    static constexpr int CODES = 16 * D / 2, SCALES = 16 * D / 32;         // of a group: keys', and values'
    static constexpr int GROUP = 2 * CODES + 2 * SCALES, BLOCK = 2 * GROUP;
    static constexpr int STAGES = 3, AHEAD = STAGES - 1;                   // blocks on their way while one is worked on
    static constexpr int LOADS = D == 128 ? 6 : 4;                         // instructions per block
    static constexpr int ENDING = kRows * (64 + 4) * 4;                    // outputs on their way to the join: 64 features of 32 rows, 128 of 16
    static constexpr int RING = STAGES * BLOCK > ENDING ? STAGES * BLOCK : ENDING;
};

// Waits until at most n of this wavefront's requests of LOADS loads each are on their way, n <= 2.
template <int LOADS>
__device__ __forceinline__ void wait_requests(int n)
{
    static_assert(2 * LOADS <= 63, "vmcnt has 6 bits");
    if (n == 2) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * LOADS) : "memory");
    else if (n == 1) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

template <int D>
__global__ __launch_bounds__(64 * kWaves, 3) void kv_stream_kernel(KvAttnArgs a)
{
    using C = Stream<D>;
    constexpr int STEPS = C::STEPS, OB = C::OB, KS = D / 16;
    __shared__ __attribute__((aligned(16))) unsigned char ring[kWaves][C::RING];
    __shared__ float sm_ml[kWaves][2][kRows];

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 31, hh = lane >> 5;
    // All first splits, then all second ones, ..: consecutive workgroups go to different XCDs, and the later splits are empty for
    // the shorter streams.  Query tiles of one stored head stay on one XCD where the heads divide evenly.
    const int split = (int)blockIdx.x / a.units, u = (int)blockIdx.x % a.units;
    const bool by_xcd = a.n_tiles > 1 && a.units / a.n_tiles % kNumXcd == 0;
    const int qt = (by_xcd ? u / kNumXcd : u) % a.n_tiles, bh = by_xcd ? u / kNumXcd / a.n_tiles * kNumXcd + u % kNumXcd : u / a.n_tiles;
    const int h = bh % a.pool.heads, b = bh / a.pool.heads, unit = bh * a.n_tiles + qt;
    const int kbeg = split * a.chunk;

    // ---- blocks: wavefront w takes blocks w, w + kWaves, .. of the split, straight into its ring
    // (the block table, like the lengths, is read through the scalar cache: a vector load's wait would wait for the copies too)
    typedef const __attribute__((address_space(4))) int32_t *scalar_ptr;
    const scalar_ptr table = (scalar_ptr)(uintptr_t)(a.table + (size_t)b * a.pool.max_pages);
    const int shift = a.pool.shift, in_page = (1 << shift) - 1, capacity = kv_capacity(a.pool);
    const unsigned char *head_base = (const unsigned char *)a.cache + (size_t)h * kv_head_bytes(shift, D);
    const uint32_t page_bytes = (uint32_t)a.pool.heads * (uint32_t)kv_head_bytes(shift, D);
    unsigned char *mine = ring[wave];
    const uint32_t lds0 = lds_address(mine);
    auto key_of = [&](int m) { return kbeg + (wave + kWaves * m) * kKeys; };        // first key of the wavefront's block m
    auto page_of = [&](int pos) -> int {          // kv_page, for a position that is not negative
        const int e = table[min(pos >> shift, a.pool.max_pages - 1)];
        return pos < capacity && (uint32_t)e < (uint32_t)a.pool.n_pages ? e : -1;
    };
    int page[2];                                  // of the two groups of the next block to request
    uint32_t placed = 0;                          // whether the groups of the blocks requested have one, two bits each, the last block lowest
    auto lookup = [&](int m) {
        page[0] = page_of(key_of(m));
        page[1] = page_of(key_of(m) + 16);
    };
    const uint32_t codes_at = D == 128 ? (lane & 15) * (D / 2) + 16 * (lane >> 4)                        // keys (D = 64: and values)
                                       : lane < 32 ? (lane & 15) * (D / 2) + 16 * (lane >> 4) : 16 * (lane - 32) + ((D / 2) << shift);
    const uint32_t scales_at = (D << shift) + (lane < D / 32 ? 16 * lane : 16 * (lane - D / 32) + ((D / 32) << shift));
    auto request = [&](int m) {                   // `page` holds the block's
#pragma unroll
        for (int g = 0; g < 2; ++g) {
            const __amdgpu_buffer_rsrc_t rsrc = make_rsrc(head_base + (uint64_t)(uint32_t)max(page[g], 0) * page_bytes, (uint32_t)kv_head_bytes(shift, D));
            const uint32_t t = (uint32_t)(key_of(m) + 16 * g) & in_page, dst = lds0 + m % C::STAGES * C::BLOCK + g * C::GROUP;
            load_to_lds(rsrc, codes_at + t * (D / 2), dst);
            if constexpr (D == 128) load_to_lds(rsrc, 16 * lane + ((D / 2) << shift) + t * (D / 2), dst + C::CODES);
            if (lane < D / 16) load_to_lds(rsrc, scales_at + t * (D / 32), dst + 2 * C::CODES);
        }
        placed = placed << 2 | (page[0] >= 0 ? 1u : 0u) | (page[1] >= 0 ? 2u : 0u);
    };
    if (split == 0) lookup(0);           // (beside the lengths; later splits are often empty and first see whether they are)

    const Span sp = span_of(a, b);
    const int row0 = qt * a.tile_rows;
    if (row0 >= sp.rows) return;
    const int n_rows = min(a.tile_rows, sp.rows - row0);
    const int lim_min = sp.limit(row0, a), lim_max = sp.limit(row0 + n_rows - 1, a);
    const int kend = min(lim_max, kbeg + a.chunk);
    if (kbeg >= kend && split > 0) return;
    const bool whole = lim_max <= a.chunk;                    // this workgroup sees all that its rows see
    if (split > 0) lookup(0);
    const int n_blocks = (kend - kbeg + kKeys - 1) / kKeys, n = (n_blocks - wave + kWaves - 1) / kWaves;      // of the split, of the wavefront
    for (int m = 0; m < C::AHEAD; ++m) {
        if (m < n) {
            request(m);
            lookup(m + 1);
        } else {
            placed <<= 2;
        }
    }

    const int row = row0 + c;
    const bool row_there = c < n_rows;
    const int lim = row_there ? sp.limit(row, a) : sp.klen;
    const size_t q_row = (((size_t)b * a.Lq + row / a.G) * a.H + (size_t)h * a.G + row % a.G) * D;
    // k-step t of the first product takes features (D / 2) hh + 8 t .. + 7 in half-wave hh, for the keys as they lie in a row
    bf16x8 qf[KS];
#pragma unroll
    for (int t = 0; t < KS; ++t) qf[t] = row_there ? *(const bf16x8 *)((const bf16_t *)a.q + q_row + (D / 2) * hh + 8 * t) : bf16x8{};

    f32x16 o[OB];                // O^T: block 2 s + e holds features 64 s + 2 i + e, i the accumulator's row
#pragma unroll
    for (int i = 0; i < OB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    bool sees = false;           // whether the row sees one of the wavefront's tokens (this half-wave's of them)
    const f32x16 zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    int nan_key[STEPS];          // first key with a NaN value among those that not all rows see
#pragma unroll
    for (int s = 0; s < STEPS; ++s) nan_key[s] = INT_MAX;

#pragma unroll 1
    for (int m = 0; m < n; ++m) {
        if (m + C::AHEAD < n) {
            request(m + C::AHEAD);
            lookup(m + C::AHEAD + 1);
        } else {
            placed <<= 2;
        }
        static_assert(C::AHEAD == 2, "the counts that wait_requests knows");
        wait_requests<C::LOADS>(min(n - 1 - m, C::AHEAD));
        const unsigned char *blk = mine + m % C::STAGES * C::BLOCK;
        const int key0 = key_of(m);
        const uint32_t groups = placed >> (2 * C::AHEAD) & 3u;

        // ---- logits: row c of the product is key c, so that accumulator r of half-wave hh is key 8 (r / 4) + 4 hh + r % 4
        u32x4 kf[STEPS];                                       // codes of features (D / 2) hh ..
        const unsigned char *kg = blk + (c >> 4) * C::GROUP;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) kf[s] = *(const u32x4 *)(kg + (STEPS * hh + s) * 256 + (c & 15) * 16);
        uint32_t ks;                                           // their scales
        if constexpr (D == 128) ks = *(const uint16_t *)(kg + 2 * C::CODES + 4 * (c & 15) + 2 * hh);
        else ks = kg[2 * C::CODES + 2 * (c & 15) + hh];
        // value codes and scales of the same keys: feature pair 32 s + c, tokens 16 u + 8 x + 4 hh ..
        uint32_t vc[STEPS][2][2], vs[STEPS][2][2];
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    vc[s][u][x] = *(const uint32_t *)(blk + u * C::GROUP + C::CODES + (32 * s + c) * 16 + 8 * x + 4 * hh);
                    vs[s][u][x] = *(const uint32_t *)(blk + u * C::GROUP + 2 * C::CODES + C::SCALES + (2 * s + (c >> 4)) * 16 + 8 * x + 4 * hh);
                }
        f32x16 s_acc = zero;
        static_for<0, KS>([&](auto t_) {
            constexpr int t = decltype(t_)::value;
            union { uint32_t u[4]; bf16x8 v; } x;
            static_for<0, 4>([&](auto i_) {
                constexpr int i = decltype(i_)::value;
                x.u[i] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(kf[t >> 2][t & 3], scale_operand<(t >> 2)>(ks), i));
            });
            s_acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x.v, qf[t], s_acc, 0, 0, 0);
        });
        if (__builtin_expect(key0 + kKeys > min(lim_min, kend) || groups != 3u, 0)) {
            const int left = min(lim, kend) - (key0 + 4 * hh);
            const int left0 = groups & 1u ? left : INT_MIN, left1 = groups & 2u ? left : INT_MIN;
            sees |= left0 > 0 || left1 > 16;
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (8 * (r >> 2) + (r & 3) >= (r < 8 ? left0 : left1)) s_acc[r] = -INFINITY;
            // values that no row of the workgroup sees are not to reach the product, whatever they are; a NaN among those that
            // some see goes to these rows alone, at the end
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int x = 0; x < 2; ++x) {
                    const int key = key0 + 16 * u + 8 * x + 4 * hh;
                    const uint32_t seen = first_bytes((groups >> u & 1u ? kend : 0) - key), by_all = first_bytes(lim_min - key);
#pragma unroll
                    for (int s = 0; s < STEPS; ++s) {
                        const uint32_t nan = bytes_255(vs[s][u][x]) & ~by_all, gone = ~seen | nan;
                        if ((nan & seen) != 0) nan_key[s] = min(nan_key[s], key + (__ffs(nan & seen) - 1) / 8);
                        vc[s][u][x] &= ~gone;
                        vs[s][u][x] = (vs[s][u][x] & ~gone) | (gone & 0x7f7f7f7fu);
                    }
                }
        } else {
            sees = true;
        }

        // ---- softmax
        float mx = s_acc[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s_acc[r]);
        const auto other = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);      // both half-waves'
        mx = fmaxf(__uint_as_float(other[0]), __uint_as_float(other[1])) * a.scale_log2;
        const float m_new = fmaxf(m_run, mx);
        const float m_ref = fmaxf(m_new, -FLT_MAX);
        if (__any(m_new > m_run)) {
            const float alpha = __builtin_amdgcn_exp2f(m_run - m_ref);
            l_run *= alpha;
#pragma unroll
            for (int i = 0; i < OB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[i][r] *= alpha;
            m_run = m_new;
        }
        bf16x8 pf[2];
#pragma unroll
        for (int r = 0; r < 16; ++r) {
            const float p = __builtin_amdgcn_exp2f(fmaf(s_acc[r], a.scale_log2, -m_ref));
            l_run += p;
            pf[r >> 3][r & 7] = to_bf16(p);
        }

        // ---- output
        static_for<0, STEPS>([&](auto s_) {
            constexpr int s = decltype(s_)::value;
            static_for<0, 2>([&](auto u_) {
                constexpr int u = decltype(u_)::value;
                uint32_t w[8];
                static_for<0, 8>([&](auto j_) {
                    constexpr int j = decltype(j_)::value;
                    w[j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(vc[s][u][j >> 2], scale_operand<(j & 3)>(vs[s][u][j >> 2]), j & 3));
                });
                union { u32x4 u; bf16x8 v; } even, odd;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    even.u[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x05040100);
                    odd.u[i] = __builtin_amdgcn_perm(w[2 * i + 1], w[2 * i], 0x07060302);
                }
                o[2 * s] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(even.v, pf[u], o[2 * s], 0, 0, 0);
                o[2 * s + 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(odd.v, pf[u], o[2 * s + 1], 0, 0, 0);
            });
        });
    }

    // ---- the wavefronts' results, each relative to its own maximum
    if (n > 0) {             // zero times the query row: NaN where it is not finite, which logits of -inf alone would not show
        f32x16 nil = zero;
#pragma unroll
        for (int t = 0; t < KS; ++t) nil = __builtin_amdgcn_mfma_f32_32x32x16_bf16(bf16x8{}, qf[t], nil, 0, 0, 0);
        if (sees) l_run += nil[0];       // (a row that sees nothing is zero, whatever it holds)
    }
    l_run = xhalf_sum(l_run);
    bool any_nan = false;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) any_nan |= nan_key[s] != INT_MAX;
    if (__any(any_nan)) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            int k = nan_key[s];                        // of features 64 s + 32 (c / 16) ..
            for (int d = 1; d < 16; d *= 2) k = min(k, __shfl_xor(k, d, kWave));
            k = min(k, __shfl_xor(k, 32, kWave));
            const int k_lo = __shfl(k, 0, kWave), k_hi = __shfl(k, 16, kWave);
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (lim > (r < 8 ? k_lo : k_hi)) o[2 * s][r] = o[2 * s + 1][r] = NAN;
        }
    }
    if (hh == 0) {
        sm_ml[wave][0][c] = m_run;
        sm_ml[wave][1][c] = l_run;
    }
    // The outputs take the ring's place (nothing is on its way into it any more): up to 16 rows at once, more 64 features at a time.
    auto put = [&](int orw, int first) {
        if (row_there) {
            static_for<0, STEPS>([&](auto s_) {
                constexpr int s = decltype(s_)::value;
                if (first < 0 || first == 64 * s) {
                    float *dst = (float *)mine + c * orw + (first < 0 ? 64 * s : 0);
#pragma unroll
                    for (int g = 0; g < 4; ++g)
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            *(f32x4 *)(dst + 16 * g + 8 * hh + 4 * i) = f32x4{o[2 * s][4 * g + 2 * i], o[2 * s + 1][4 * g + 2 * i], o[2 * s][4 * g + 2 * i + 1], o[2 * s + 1][4 * g + 2 * i + 1]};
                }
            });
        }
        __syncthreads();
    };
    auto join = [&](int orw, int first, int pieces) {  // 16-byte pieces of a row
        for (int e = tid; e < n_rows * pieces; e += 64 * kWaves) {
            const int rr = e / pieces, d = 4 * (e % pieces);
            float mw[kWaves], m = -INFINITY, l = 0.f;
            f32x4 y[kWaves], sum = {0, 0, 0, 0};
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                mw[w] = sm_ml[w][0][rr];
                y[w] = *(const f32x4 *)((const float *)ring[w] + rr * orw + d);
                m = fmaxf(m, mw[w]);
            }
            const float m_ref = fmaxf(m, -FLT_MAX);
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const float f = __builtin_amdgcn_exp2f(mw[w] - m_ref);
                l = fmaf(sm_ml[w][1][rr], f, l);
#pragma unroll
                for (int i = 0; i < 4; ++i) sum[i] = fmaf(y[w][i], f, sum[i]);
            }
            if (whole) {
                const float inv = l == 0.f ? 0.f : 1.f / l;          // a row that sees nothing is zero
                const int orow = row0 + rr;
                bf16x4 z;
#pragma unroll
                for (int i = 0; i < 4; ++i) z[i] = to_bf16(sum[i] * inv);
                *(bf16x4 *)((bf16_t *)a.out + (((size_t)b * a.Lq + orow / a.G) * a.H + (size_t)h * a.G + orow % a.G) * D + first + d) = z;
            } else {
                const size_t slot = ((size_t)unit * a.nsplit + split) * a.tile_rows + rr;
                *(f32x4 *)(a.part_o + slot * D + first + d) = sum;
                if (first + d == 0) *(f32x2 *)(a.part_ml + slot * 2) = f32x2{m, l};
            }
        }
    };
    if (D == 64 || n_rows <= 16) {
        put(D + 4, -1);
        join(D + 4, 0, D / 4);
    } else {
        for (int f = 0; f < D; f += 64) {
            if (f > 0) __syncthreads();
            put(64 + 4, f);
            join(64 + 4, f, 16);
        }
    }
}

// Adds the partial results of splits `first`, first + step, .. (up to n) of a row into (m, l, sum): four features from d on, four
// splits at a time, whose loads do not wait for one another.
template <int D>
__device__ __forceinline__ void add_splits(const KvAttnArgs &a, size_t slot0, int first, int step, int n, int d, float &m, float &l, f32x4 &sum)
{
    constexpr int AT_ONCE = 4;
    for (int s0 = first; s0 < n; s0 += step * AT_ONCE) {
        f32x2 ml[AT_ONCE];
        f32x4 y[AT_ONCE];
        float m_new = m;
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const int s = s0 + step * k;
            const size_t slot = slot0 + (size_t)min(s, n - 1) * a.tile_rows;
            ml[k] = *(const f32x2 *)(a.part_ml + slot * 2);
            y[k] = *(const f32x4 *)(a.part_o + slot * D + d);
            if (s >= n) ml[k] = f32x2{-INFINITY, 0.f}, y[k] = f32x4{0, 0, 0, 0};
        }
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) m_new = fmaxf(m_new, ml[k][0]);
        const float m_ref = fmaxf(m_new, -FLT_MAX), f0 = __builtin_amdgcn_exp2f(m - m_ref);
        l *= f0;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] *= f0;
#pragma unroll
        for (int k = 0; k < AT_ONCE; ++k) {
            const float f1 = __builtin_amdgcn_exp2f(ml[k][0] - m_ref);
            l = fmaf(ml[k][1], f1, l);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = fmaf(y[k][i], f1, sum[i]);
        }
        m = m_new;
    }
}

// Joins the partial results of rows that more than one workgroup worked on.  Up to kFewSplits splits: D / 4 lanes to a row, in the
// order of the splits.  More: a workgroup to a row, 1024 / D splits side by side, then these in order.
// Whole calls, lanes and workgroups to a row: 18720 rows of 3 splits 103 and 119 us, 2048 of up to 8 34.6 and 35.4 us.
constexpr int kFewSplits = 8;
template <int D, bool FEW>
__global__ __launch_bounds__(256) void kv_join_kernel(KvAttnArgs a)
{
    constexpr int LANES = D / 4, GROUPS = 256 / LANES;
    const int g = threadIdx.x / LANES, d = 4 * (threadIdx.x % LANES);
    const int per_unit = FEW ? (a.tile_rows + GROUPS - 1) / GROUPS : a.tile_rows;
    const int unit = blockIdx.x / per_unit, rr = FEW ? (int)(blockIdx.x % per_unit) * GROUPS + g : blockIdx.x % per_unit;
    const int qt = unit % a.n_tiles, bh = unit / a.n_tiles, h = bh % a.pool.heads, b = bh / a.pool.heads;
    const Span sp = span_of(a, b);
    const int row0 = qt * a.tile_rows, row = row0 + rr;
    if (rr >= a.tile_rows || row >= sp.rows) return;
    const int lim_max = sp.limit(min(row0 + a.tile_rows, sp.rows) - 1, a);
    if (lim_max <= a.chunk) return;                    // written by the one workgroup that saw it all
    const int n = (lim_max + a.chunk - 1) / a.chunk;
    const size_t slot0 = (size_t)unit * a.nsplit * a.tile_rows + rr;
    float m = -INFINITY, l = 0.f;
    f32x4 sum = {0, 0, 0, 0};
    add_splits<D>(a, slot0, FEW ? 0 : g, FEW ? 1 : GROUPS, n, d, m, l, sum);
    if constexpr (!FEW) {
        __shared__ __attribute__((aligned(16))) float sm_o[GROUPS][D];
        __shared__ float sm_ml[GROUPS][2];
        *(f32x4 *)&sm_o[g][d] = sum;
        if (d == 0) {
            sm_ml[g][0] = m;
            sm_ml[g][1] = l;
        }
        __syncthreads();
        if (g > 0) return;
        m = sm_ml[0][0];
#pragma unroll
        for (int i = 1; i < GROUPS; ++i) m = fmaxf(m, sm_ml[i][0]);
        const float m_ref = fmaxf(m, -FLT_MAX);
        sum = f32x4{0, 0, 0, 0};
        l = 0.f;
#pragma unroll
        for (int i = 0; i < GROUPS; ++i) {
            const float f = __builtin_amdgcn_exp2f(sm_ml[i][0] - m_ref);
            l = fmaf(sm_ml[i][1], f, l);
#pragma unroll
            for (int j = 0; j < 4; ++j) sum[j] = fmaf(sm_o[i][d + j], f, sum[j]);
        }
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    bf16x4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = to_bf16(sum[i] * inv);
    *(bf16x4 *)((bf16_t *)a.out + (((size_t)b * a.Lq + row / a.G) * a.H + (size_t)h * a.G + row % a.G) * D + d) = y;
}

template <int D>
hipError_t launch_join(const KvAttnArgs &a, hipStream_t stream)
{
    constexpr int GROUPS = 1024 / D;
    if (a.nsplit > kFewSplits) return launch_kernel(kv_join_kernel<D, false>, dim3((unsigned)a.units * a.tile_rows), dim3(256), stream, a);
    return launch_kernel(kv_join_kernel<D, true>, dim3((unsigned)a.units * ((a.tile_rows + GROUPS - 1) / GROUPS)), dim3(256), stream, a);
}

}  // namespace

// How a call is divided, from its sizes alone.
// The kernel.  In us, few rows and many: 12 heads x 128 over 32760 tokens 64 rows 37 and 36, 96 rows 48 and 38; 8 streams x 8 heads over 4096,
// causal, 64 rows 28 and 27, 96 rows 32 and 29; 64 x 8 over 1024 64 rows 36 and 40, 96 rows 49 and 44; x 64, 16 x 12 over 2000 64 rows 25 and 31,
// 96 rows 34 and 32.  (Where either finds few workgroups the first stays ahead: 12 heads over 4680, 256 rows 27 and 32.)
// Many rows: the splits that the measured cost of a tile, of a workgroup's ends and of partial results make the cheapest; e.g. 12 heads,
// 1560 rows over 10920: 1 to 6 splits 236, 143, 110, 152, 133, 122 us; 4680 rows over 4680: 119 without, 146 with two.
// Few rows: one round of workgroups; with several streams, whose lengths the host does not know, at most an eighth of the table's length or
// 1024 tokens (64 streams of 1 to 7122 tokens, a table for 7136: 512, 1024, 1408, 2048 tokens 39, 36.5, 36, 44 us).
// Both go by what the table could hold, and many rows by all of it for every row, causal or not.
KvAttnPlan kv_attn_plan(int B, int Lq, int G, const KvPool &pool, int D)
{
    KvAttnPlan p = {};
    const long long rows = (long long)Lq * G, cap = kv_capacity(pool), heads = (long long)B * pool.heads;
    p.tiled = rows > 64;
    p.tile_rows = p.tiled ? kTileRows : (int)(rows < kRows ? rows : kRows);
    p.n_tiles = (rows + p.tile_rows - 1) / p.tile_rows;
    p.units = heads * p.n_tiles;
    long long chunk = 256;
    if (p.tiled) {
        double best = 1e30;
        for (int n = 1; n <= 64; ++n) {
            const long long tokens = std::max((cap + n - 1) / n + 63, 256LL) / 64 * 64;
            if (n > 1 && (cap + tokens - 1) / tokens < n) continue;
            const double rounds = (double)((p.units * n + kNumCu - 1) / kNumCu);
            const double us = rounds * (tokens / 64 * (D == 128 ? 1.42 : 1.0) + 7) + (n > 1 ? 5 + (double)heads * rows * n * D * 8 / 4.5e6 : 0);
            if (us < best) { best = us; chunk = tokens; }
        }
    } else {
        const long long one_round = (cap * p.units + kSlots - 1) / kSlots;
        chunk = B == 1 ? one_round : std::min(one_round, std::max(1024LL, cap / 8));
        chunk = (std::max(chunk, 256LL) + 127) / 128 * 128;
    }
    p.nsplit = (int)((cap + chunk - 1) / chunk);
    p.chunk = (int)chunk;
    const size_t slots = (size_t)p.units * p.nsplit * p.tile_rows;
    p.o_bytes = p.nsplit > 1 ? slots * D * sizeof(float) : 0;
    p.bytes = p.nsplit > 1 ? p.o_bytes + slots * 2 * sizeof(float) : 0;
    return p;
}

hipError_t launch_kv_attn(KvAttnArgs a, const KvAttnPlan &p, void *workspace, hipStream_t stream)
{
    a.n_tiles = (int)p.n_tiles;
    a.units = (int)p.units;
    a.nsplit = p.nsplit;
    a.chunk = p.chunk;
    a.tile_rows = p.tile_rows;
    a.part_o = (float *)workspace;
    a.part_ml = (float *)((unsigned char *)workspace + p.o_bytes);
    const dim3 grid((unsigned)(p.units * p.nsplit)), block(64 * kWaves);
    hipError_t e = p.tiled ? launch_kv_tile(a, grid.x, stream) : a.D == 128 ? launch_kernel(kv_stream_kernel<128>, grid, block, stream, a) : launch_kernel(kv_stream_kernel<64>, grid, block, stream, a);
    if (e != hipSuccess || p.nsplit == 1) return e;
    return a.D == 128 ? launch_join<128>(a, stream) : launch_join<64>(a, stream);
}

}  // namespace arl2
