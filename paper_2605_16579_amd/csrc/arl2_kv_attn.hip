// Attention over the paged 4-bit key/value cache (gfx950):
//   out_i = sum_j softmax_j(sm_scale * q_i.K_j) V_j      over the stored tokens j of the stream, all or (causal) up to query i
#include "arl2_kv_attn.h"

#include <limits.h>

namespace arl2 {
namespace {

constexpr int kRows = 32;        // query rows of a workgroup
constexpr int kWaves = 4;

// One block of 32 stored tokens in registers.
template <int D>
struct Block {
    static constexpr int STEPS = D / 64;
    u32x4 k[STEPS];          // lane (c, hh): key row i = c, features 64 s + 32 hh .. + 31
    uint32_t ks;             // the row's scales from feature 32 hh on
    u32x4 v[STEPS], vs[STEPS];     // feature pair 32 x + c, tokens 16 hh .. + 15: codes, and scales of the pair's group
    int page;                // of tokens 16 hh .. + 15, or -1
};

template <int D>
__global__ __launch_bounds__(64 * kWaves, 2) void kv_stream_kernel(KvAttnArgs a)
{
    constexpr int STEPS = D / 64, OB = D / 32;
    __shared__ __attribute__((aligned(16))) float sm_o[kWaves][kRows][D + 4];
    __shared__ float sm_ml[kWaves][2][kRows];

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 31, hh = lane >> 5;
    uint32_t id = blockIdx.x;
    const int split = id % a.nsplit;
    const int unit = id / a.nsplit;
    const int qt = unit % a.n_tiles, bh = unit / a.n_tiles, h = bh % a.pool.heads, b = bh / a.pool.heads;
    const Span sp = span_of(a, b);
    const int row0 = qt * kRows;
    if (row0 >= sp.rows) return;
    const int n_rows = min(kRows, sp.rows - row0);
    const int lim_min = sp.limit(row0, a), lim_max = sp.limit(row0 + n_rows - 1, a);
    const int kbeg = split * a.chunk, kend = min(lim_max, kbeg + a.chunk);
    if (kbeg >= kend && split > 0) return;
    const bool whole = lim_max <= a.chunk;                    // this workgroup sees all that its rows see

    const int row = row0 + c;
    const bool row_there = c < n_rows;
    const int lim = row_there ? sp.limit(row, a) : sp.klen;
    const size_t q_row = (((size_t)b * a.Lq + row / a.G) * a.H + (size_t)h * a.G + row % a.G) * D;
    Query<D> q;
    q.load((const bf16_t *)a.q + q_row + 32 * hh, row_there);

    // Keys are dealt to the rows of the first product so that the logits of lane (c, hh) belong to keys 16 hh .. 16 hh + 15 of the
    // block in order: accumulator r of half-wave hh is row 8 (r / 4) + 4 hh + r % 4.
    const int row_key = 16 * ((c >> 2) & 1) + 8 * (c >> 4) + 4 * ((c >> 3) & 1) + (c & 3);
    const int32_t *table = a.table + (size_t)b * a.pool.max_pages;
    const unsigned char *pool = (const unsigned char *)a.cache;
    const int shift = a.pool.shift, in_page = (1 << shift) - 1;
    auto head = [&](int page) { return pool + kv_head_offset(a.pool, D, page < 0 ? 0 : page, h); };
    auto load = [&](Block<D> &x, int key0, int page_k, int page_v) {
        const unsigned char *kb = head(page_k), *vb = head(page_v);
        const int tk = (key0 + row_key) & in_page, tv = (key0 + 16 * hh) & in_page;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) x.k[s] = *(const u32x4 *)(kb + kv_key_codes(tk, 32 * s + 16 * hh, D));
        if constexpr (D == 128) x.ks = *(const uint32_t *)(kb + kv_key_scales(shift, tk, 0, D)) >> (8 * hh);
        else x.ks = *(const uint16_t *)(kb + kv_key_scales(shift, tk, 0, D)) >> (8 * hh);
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            x.v[s] = *(const u32x4 *)(vb + kv_value_codes(shift, tv, 32 * s + c, D));
            x.vs[s] = *(const u32x4 *)(vb + kv_value_scales(shift, tv, 2 * s + (c >> 4), D));
        }
        x.page = page_v;
    };

    f32x16 o[OB];                // O^T: block 2 s + e holds features 64 s + 2 i + e, i the accumulator's row
#pragma unroll
    for (int i = 0; i < OB; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
    float m_run = -INFINITY, l_run = 0.f;
    int nan_key[STEPS];          // first key with a NaN value among those that not all rows see
#pragma unroll
    for (int s = 0; s < STEPS; ++s) nan_key[s] = INT_MAX;

    auto process = [&](Block<D> &x, int key0, auto masked_) {
        constexpr bool MASKED = decltype(masked_)::value;
        f32x16 s_acc = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
        static_for<0, STEPS>([&](auto s_) {
            constexpr int s = decltype(s_)::value;
            const i32x8 ka = {(int)x.k[s][0], (int)x.k[s][1], (int)x.k[s][2], (int)x.k[s][3], 0, 0, 0, 0};
            static_for<0, kParts>([&](auto p_) {
                constexpr int p = decltype(p_)::value;
                const u32x6 w = q.part[s][p];
                const i32x8 qb = {(int)w[0], (int)w[1], (int)w[2], (int)w[3], (int)w[4], (int)w[5], 0, 0};
                s_acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ka, qb, s_acc, 4, 2, 2 * s, (int)x.ks, p, (int)q.scale[s]);
            });
        });
        if constexpr (MASKED) {
            const int left = (x.page < 0 ? 0 : lim) - (key0 + 16 * hh);
#pragma unroll
            for (int r = 0; r < 16; ++r)
                if (r >= left) s_acc[r] = -INFINITY;
            // values that no row of the workgroup sees are not to reach the product, whatever they are; a NaN among those that
            // some see goes to these rows alone, at the end
            const int left_v = (x.page < 0 ? 0 : lim_max) - (key0 + 16 * hh), left_all = lim_min - (key0 + 16 * hh);
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
#pragma unroll
                for (int t = 0; t < 16; ++t) {
                    const uint32_t byte = 255u << (8 * (t & 3));
                    const bool nan = (x.vs[s][t >> 2] & byte) == byte;
                    if (t >= left_v || (nan && t >= left_all)) {
                        x.v[s][t >> 2] &= ~byte;
                        x.vs[s][t >> 2] = (x.vs[s][t >> 2] & ~byte) | (byte & 0x7f7f7f7fu);
                        if (t < left_v) nan_key[s] = min(nan_key[s], key0 + 16 * hh + t);
                    }
                }
        }
        float mx = s_acc[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s_acc[r]);
        mx = xhalf_max(mx) * a.scale_log2;
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
        static_for<0, STEPS>([&](auto s_) {
            constexpr int s = decltype(s_)::value;
            static_for<0, 2>([&](auto u_) {
                constexpr int u = decltype(u_)::value;
                uint32_t w[8];
                static_for<0, 8>([&](auto j_) {
                    constexpr int j = decltype(j_)::value, t = 8 * u + j;
                    w[j] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x.v[s][t >> 2], scale_operand<(t & 3)>(x.vs[s][t >> 2]), t & 3));
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
    };

    {
        const int n_blocks = (kend - kbeg + kKeys - 1) / kKeys;
        int blk = wave;
        Block<D> x, y;
        auto pages = [&](int blk, int &pk, int &pv) {
            const int key0 = kbeg + blk * kKeys;
            pk = kv_page(a.pool, table, key0 + row_key);
            pv = kv_page(a.pool, table, key0 + 16 * hh);
        };
        int pk = 0, pv = 0;
        if (blk < n_blocks) {
            pages(blk, pk, pv);
            load(x, kbeg + blk * kKeys, pk, pv);
            pages(blk + kWaves, pk, pv);
        }
        while (blk < n_blocks) {
            const int next = blk + kWaves;
            if (next < n_blocks) {
                load(y, kbeg + next * kKeys, pk, pv);
                pages(next + kWaves, pk, pv);
            }
            const int key0 = kbeg + blk * kKeys;
            if (key0 + kKeys > lim_min || __any(x.page < 0)) process(x, key0, std::true_type{});
            else process(x, key0, std::false_type{});
            x = y;
            blk = next;
        }
    }

    // ---- the wavefronts' results, each relative to its own maximum
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
    if (c < n_rows) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int i = 8 * (r >> 2) + 4 * hh + (r & 3);
                *(f32x2 *)&sm_o[wave][c][64 * s + 2 * i] = f32x2{o[2 * s][r], o[2 * s + 1][r]};
            }
    }
    __syncthreads();
    constexpr int PER = D / 4;                         // 16-byte pieces of a row
    for (int e = tid; e < n_rows * PER; e += 64 * kWaves) {
        const int rr = e / PER, d = 4 * (e % PER);
        float m = sm_ml[0][0][rr];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) m = fmaxf(m, sm_ml[w][0][rr]);
        const float m_ref = fmaxf(m, -FLT_MAX);
        f32x4 sum = {0, 0, 0, 0};
        float l = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float f = __builtin_amdgcn_exp2f(sm_ml[w][0][rr] - m_ref);
            const f32x4 y = *(const f32x4 *)&sm_o[w][rr][d];
            l = fmaf(sm_ml[w][1][rr], f, l);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = fmaf(y[i], f, sum[i]);
        }
        if (whole) {
            const float inv = l == 0.f ? 0.f : 1.f / l;          // a row that sees nothing is zero
            const int orow = row0 + rr;
            bf16x4 y;
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = to_bf16(sum[i] * inv);
            *(bf16x4 *)((bf16_t *)a.out + (((size_t)b * a.Lq + orow / a.G) * a.H + (size_t)h * a.G + orow % a.G) * D + d) = y;
        } else {
            const size_t slot = ((size_t)unit * a.nsplit + split) * a.tile_rows + rr;
            *(f32x4 *)(a.part_o + slot * D + d) = sum;
            if (d == 0) *(f32x2 *)(a.part_ml + slot * 2) = f32x2{m, l};
        }
    }
}

// Joins a row's partial results, in the order of the splits within each of 8 groups and then of the groups.
template <int D>
__global__ __launch_bounds__(256) void kv_join_kernel(KvAttnArgs a)
{
    constexpr int LANES = D / 4, GROUPS = 256 / LANES;
    __shared__ __attribute__((aligned(16))) float sm_o[GROUPS][D];
    __shared__ float sm_ml[GROUPS][2];
    const int unit = blockIdx.x / a.tile_rows, rr = blockIdx.x % a.tile_rows;
    const int qt = unit % a.n_tiles, bh = unit / a.n_tiles, h = bh % a.pool.heads, b = bh / a.pool.heads;
    const Span sp = span_of(a, b);
    const int row0 = qt * a.tile_rows, row = row0 + rr;
    if (row >= sp.rows) return;
    const int lim_max = sp.limit(min(row0 + a.tile_rows, sp.rows) - 1, a);
    if (lim_max <= a.chunk) return;                    // written by the one workgroup that saw it all
    const int n = (lim_max + a.chunk - 1) / a.chunk;
    const int g = threadIdx.x / LANES, d = 4 * (threadIdx.x % LANES);
    float m = -INFINITY, l = 0.f;
    f32x4 sum = {0, 0, 0, 0};
    for (int s = g; s < n; s += GROUPS) {
        const size_t slot = ((size_t)unit * a.nsplit + s) * a.tile_rows + rr;
        const f32x2 ml = *(const f32x2 *)(a.part_ml + slot * 2);
        const f32x4 y = *(const f32x4 *)(a.part_o + slot * D + d);
        const float m_new = fmaxf(m, ml[0]), m_ref = fmaxf(m_new, -FLT_MAX);
        const float f0 = __builtin_amdgcn_exp2f(m - m_ref), f1 = __builtin_amdgcn_exp2f(ml[0] - m_ref);
        l = l * f0 + ml[1] * f1;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] = sum[i] * f0 + y[i] * f1;
        m = m_new;
    }
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
    const float inv = l == 0.f ? 0.f : 1.f / l;
    bf16x4 y;
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = to_bf16(sum[i] * inv);
    *(bf16x4 *)((bf16_t *)a.out + (((size_t)b * a.Lq + row / a.G) * a.H + (size_t)h * a.G + row % a.G) * D + d) = y;
}

}  // namespace

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
        // the fewest rounds of one workgroup per CU, each split paying for its partial results
        double best = 1e30;
        for (int s = 1; s <= 32; ++s) {
            const long long tokens = ((cap + s - 1) / s + 255) / 256 * 256;
            const long long n = (cap + tokens - 1) / tokens;
            const double rounds = (double)((p.units * n + kNumCu - 1) / kNumCu);
            const double us = rounds * (tokens / 64 * 1.4 + 8) + (n > 1 ? 5 + (double)heads * rows * n * D * 8 / 4.5e6 : 0);
            if (us < best) { best = us; chunk = tokens; }
        }
    } else {
        while (chunk < 2048 && p.units * ((cap + chunk - 1) / chunk) > 1024) chunk *= 2;
        if (p.units >= 1024) chunk = cap;
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
    a.nsplit = p.nsplit;
    a.chunk = p.chunk;
    a.tile_rows = p.tile_rows;
    a.part_o = (float *)workspace;
    a.part_ml = (float *)((unsigned char *)workspace + p.o_bytes);
    const dim3 grid((unsigned)(p.units * p.nsplit)), block(64 * kWaves);
    hipError_t e = p.tiled ? launch_kv_tile(a, grid.x, stream) : a.D == 128 ? launch_kernel(kv_stream_kernel<128>, grid, block, stream, a) : launch_kernel(kv_stream_kernel<64>, grid, block, stream, a);
    if (e != hipSuccess || p.nsplit == 1) return e;
    const dim3 jgrid((unsigned)(p.units * p.tile_rows));
    return a.D == 128 ? launch_kernel(kv_join_kernel<128>, jgrid, dim3(256), stream, a) : launch_kernel(kv_join_kernel<64>, jgrid, dim3(256), stream, a);
}

}  // namespace arl2
