// Attention over the paged 4-bit key/value cache for many query rows (gfx950): chunks and prompts, from 65 rows on.
//
// A row is a (query token, query head of the stored head's group).  A workgroup has 256 of them, eight wavefronts 32 each, and walks
// over its tokens in tiles of 64, everything transposed:
//   S^T[key][row] = K[key][:] . Q[row][:]      keys as they are stored, 4 bits with a scale per 32 features: operands of the scaled
//                                              matrix instruction as they lie; queries as sums of 6-bit floats (`Query`)
//   O^T[d][row]  += V^T[d][key] . P^T[key][row]     values as bf16, in which they are exact; probabilities rounded to bf16 (2^-9 on the
//                                              average of the result's size, as in every product of bf16 matrices)
// Values cannot go into the scaled instruction: its scales belong to 32 terms of a sum, which runs over tokens here, and the cache
// scales values per token so that single tokens can be appended.  So they are converted, once per workgroup and tile (28 vector
// instructions per thread), into an LDS tile that the second product reads in 16-byte pieces without bank conflicts.  The codes are read
// 4 bytes a lane, 16 apart, with conflicts: the 11.2 M cycles counted in the launch below are 6 for each of these 1.87 M reads.
//
// Tiles come straight from memory into LDS as they are stored (8.7 KB; a bf16 tile is 32 KB), requested three intervals before their
// values are converted; the block table's entries pass through LDS as well.  Per tile a wavefront requests one of eight pieces.  Waits
// count this wavefront's loads, one barrier per tile publishes them all.  What belongs to a request is spread over the first steps
// of a slot, beside products in flight: behind the barrier all eight wavefronts did it at once (682 -> 646 us on zeros).
//
// The unit of the schedule is a slot, the softmax of one 32-key block beside the first product of the next block and the second
// product of the previous one.  Softmax: probabilities relative to a running maximum that starts as the first block's and is
// raised only where a lane's share of a block's sum shows that a logit passed it by about 2^7; then the block is done again.
// Masks (the last tile, causal rows' ends, groups without a page) are branches around the slots, not variants of them: two variants
// in one loop doubled the accumulators (344 bytes of scratch).
//
// What bounds it: vector instructions and the power of the matrix cores together.  12 heads x 128, 4680 queries over 32760 keys: 677
// to 726 us by card (942 GFLOP: 1.30 to 1.39 PFLOP/s), on zeros, where power does not bound it, 629 us; the matrix instructions alone
// would take 390 us.  The bf16 readout over a dense bf16 cache takes 760 to 818 us on the same cards.  24 heads x 64, as many operations:
// 1032 us (0.91 PFLOP/s), with as many exponentials for half the products.
#include "arl2_kv_attn.h"

#include <limits.h>

// (the lambdas of the main loop have two users each)
#define INLINE __attribute__((always_inline))

namespace arl2 {
namespace {

typedef __attribute__((ext_vector_type(6))) uint32_t u32x6;
typedef __attribute__((ext_vector_type(8))) int i32x8;
typedef __attribute__((ext_vector_type(32))) __bf16 bf16x32;
typedef __attribute__((ext_vector_type(32))) float f32x32;

constexpr int kParts = 3;         // of a query feature, at most
constexpr int kTile = 64;         // keys of a tile
constexpr int kNT = 512;          // threads: eight wavefronts of 32 query rows
constexpr int kStages = 4;        // of each LDS ring
constexpr int kWindow = 64;       // tiles whose block-table entries are held in LDS at a time, twice

template <int D>
struct Tile {
    static constexpr int STEPS = D / 64, OB = D / 32;
    static constexpr int PVN = 2 * OB;              // products of a block's output
    static constexpr int RING = 4, PF = RING - 1;   // V fragments in flight from LDS
    static constexpr int T = D / 16;                // tokens of a feature pair that a thread converts
    // as stored: key codes [16-key group][16-byte piece of a row][key], value codes as in the cache, key scales, value scales
    static constexpr int CODES = kTile * D / 2, SCALES = kTile * D / 32;
    static constexpr int RAW = 2 * CODES + 2 * SCALES;
    static constexpr int V_BYTES = kTile * D * 2;   // values as bf16, [even or odd features][8-key chunk][feature pair]
    static constexpr int V_OFF = kStages * RAW, TC_OFF = V_OFF + kStages * V_BYTES;
    static constexpr int SMEM = TC_OFF + 2 * kWindow * 4 * 4;
    static_assert(PVN % RING == 0, "the fragment ring runs across slots");
};

// A query row as B operands of the scaled matrix instruction: lane (c, hh) has features 64 s + 32 hh .. + 31 of row c, each as the
// sum of up to three 6-bit floats (e2m3: 4 significant bits, steps of 1/8 below 2, 1/4 below 4, 1/2 up to 7.5) at units u, u / 32 and
// u / 256, the largest of the 32 in (3.75, 7.5] u.  6-bit operands run at four times bf16's rate: two parts take half the time of
// one bf16 product, three parts three quarters.  Three parts are within 2^-12 u of a bf16 feature and exact from u / 8 on; two are
// exact from u / 2 on (but for 2^-6 u where the first leaves just half a step of 1/2).  Two are enough where what they leave of
// the row is no longer than 2^-9 of it, half of what one rounding to bf16 may take; a wavefront spares the third product where all its
// rows have enough.  Rows of normal values leave 2^-10.9, the longest of 32 rarely more than 2^-9.1; rows with a feature far above the
// others' size get the third part.
// (4680 queries over 32760 keys: 712 us with two parts, 759 us with three on one card.)
// That is decided from sums of squares in fp32, out of whose range they fall for features below 2^-63 and rows from 2^64 on: a row shorter
// than 2^-30 or longer than 2^64 keeps three parts.  u is 2^-100 at least, where three parts are within 2^-112 of a feature.
template <int D>
struct Query {
    static constexpr int STEPS = D / 64;
    u32x6 part[STEPS][kParts];
    uint32_t scale[STEPS];           // byte p: of part p; 255, a NaN, in the place of the first where a feature is not finite
    bool two;                        // whether two parts are enough; the third is then zero
    __device__ __forceinline__ void load(const bf16_t *row, bool there)
    {
        float all = 0.f, left = 0.f;
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
            const int e = finite ? max((int)((m + 0xfffffu) >> 23) - 2, 27) : 127;       // one more from above 7.5 on
            scale[s] = (uint32_t)e | (uint32_t)(e - 5) << 8 | (uint32_t)(e - 8) << 16;
            if (!finite) scale[s] |= 255u;
            left += m != 0 ? 0x1p-78f : 0.f;      // (above 2^-18 of the squares of a row shorter than 2^-30; nothing beside those of others)
#pragma unroll
            for (int p = 0; p < kParts; ++p) {
                const float unit = __uint_as_float((uint32_t)(e - (p == 0 ? 0 : p == 1 ? 5 : 8)) << 23);
                bf16x32 from = x.v;
                // (features whose nearest 6-bit float is 2^128, beyond fp32: cut to the one below, which leaves up to 7.5 of the second's units)
                if (p == 0 && __builtin_expect(__any(m > 0x7f700000u), 0)) {
#pragma unroll
                    for (int j = 0; j < 32; ++j) from[j] = to_bf16(fminf(fmaxf((float)from[j], -0x1.ep127f), 0x1.ep127f));
                }
                part[s][p] = __builtin_amdgcn_cvt_scalef32_pk32_fp6_bf16(from, unit);
                const f32x32 taken = __builtin_amdgcn_cvt_scalef32_pk32_f32_fp6(part[s][p], unit);
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    const float f = (float)x.v[j], r = f - taken[j];              // (exact: fewer bits than the feature has)
                    if (p == 0) all = fmaf(f, f, all);
                    if (p == 1) left = fmaf(r, r, left);
                    x.v[j] = to_bf16(r);
                }
            }
        }
        all = xhalf_sum(all);
        two = xhalf_sum(left) <= 0x1p-18f * all && all <= FLT_MAX;
        // (if another row of the wavefront needs the third part, this one's is zero: its result is the same in whatever company)
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int i = 0; i < 6; ++i) part[s][2][i] = two ? 0u : part[s][2][i];
    }
};

// Workgroup barrier after all but the last N of this wavefront's loads into LDS have arrived, and all but the last M of its LDS
// operations, which end in the order they were issued in.
template <int N, int M = 0>
__device__ __forceinline__ void wait_barrier()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(%1)\n\ts_barrier" ::"n"(N), "n"(M) : "memory");
}

template <int D>
__global__ __launch_bounds__(kNT, 2) void kv_tile_kernel(KvAttnArgs a)
{
    using C = Tile<D>;
    constexpr int STEPS = C::STEPS, OB = C::OB;
    __shared__ __attribute__((aligned(16))) unsigned char smem[C::SMEM];
    __shared__ int nan_key[D / 32];      // first key with a NaN value among those that not all rows see

    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, c = lane & 31, hh = lane >> 5;
    // The last query tiles first: of causal rows they see the most.  Heads innermost, so that every XCD has work of every stream
    // (a stored head of 4000 tokens is 0.5 MB: that several L2s read it costs less than an idle XCD).
    const int heads = a.units / a.n_tiles, bh = (int)blockIdx.x % heads;
    const int split = (int)blockIdx.x / heads % a.nsplit, qt = a.n_tiles - 1 - (int)blockIdx.x / heads / a.nsplit;
    const int h = bh % a.pool.heads, b = bh / a.pool.heads;
    const Span sp = span_of(a, b);
    const int row0 = qt * a.tile_rows;
    if (row0 >= sp.rows) return;
    const int n_rows = min(a.tile_rows, sp.rows - row0);
    const int lim_min = sp.limit(row0, a), lim_max = sp.limit(row0 + n_rows - 1, a);
    const int kbeg = split * a.chunk, kend = min(lim_max, kbeg + a.chunk);
    if (kbeg >= kend && split > 0) return;
    const bool whole = lim_max <= a.chunk;                    // this workgroup sees all that its rows see

    const int q0 = 32 * wave, row = row0 + q0 + c;
    const bool active = q0 < n_rows, row_there = q0 + c < n_rows;
    const int lim = row_there ? sp.limit(row, a) : sp.klen;
    auto row_offset = [&](int r) { return (((size_t)b * a.Lq + r / a.G) * a.H + (size_t)h * a.G + r % a.G) * D; };
    if (tid < D / 32) nan_key[tid] = INT_MAX;

    // ---- tiles
    const int32_t *table = a.table + (size_t)b * a.pool.max_pages;
    const unsigned char *pool = (const unsigned char *)a.cache;
    const int shift = a.pool.shift, in_page = (1 << shift) - 1;
    const int tile0 = kbeg / kTile, n = max(2, (kend - kbeg + kTile - 1) / kTile);       // (a second, empty tile where there is one)
    const uint32_t lds0 = lds_address(smem);
    // The block table: entries of the 16-token groups of a window of tiles, one per thread.
    int *tc = (int *)(smem + C::TC_OFF);
    auto window_entry = [&](int w) { return kv_page(a.pool, table, ((int64_t)(tile0 + w * kWindow) * 4 + (tid & 255)) * 16); };
    auto window_store = [&](int w, int entry) {
        if (tid < 256) tc[(w & 1) * 256 + tid] = entry;
    };
    // Of the tiles requested, the last one lowest: which of its groups have a page (4 bits), and whether care is due (1 bit): a group
    // has no page, or not every row sees all of the tile.
    uint32_t placed = 0, careful = 0;
    const int first_careful = min(lim_min, kend) / kTile - tile0;
    // Requests a tile, straight into LDS: wavefront w moves group w / 2, its keys (even w) or values, codes and scales.  In three steps.
    const int part = wave & 1, grp = wave >> 1;
    const unsigned char *head_base = pool + (size_t)h * kv_head_bytes(shift, D);
    const uint32_t page_bytes = (uint32_t)a.pool.heads * (uint32_t)kv_head_bytes(shift, D);      // (the host sees to it that they are below 2^32)
    const uint32_t code_src = (part ? 16 * lane : (lane & 15) * (D / 2) + 16 * (lane >> 4)) + (part ? (D / 2) << shift : 0);
    const uint32_t scale_src = 16 * lane + (D << shift) + (part ? (D / 32) << shift : 0);
    const uint32_t code_dst = lds0 + part * C::CODES + grp * (C::CODES / 4), scale_dst = lds0 + 2 * C::CODES + part * C::SCALES + grp * (C::SCALES / 4);
    int group_entry;                 // of 16-token group lane & 3 of the next tile to request
    __amdgpu_buffer_rsrc_t page_rsrc;
    auto entry_fetch = [&](int tile) INLINE { group_entry = tc[((tile / kWindow) & 1) * 256 + (tile % kWindow) * 4 + (lane & 3)]; };
    auto request = [&](int tile, auto step_) INLINE {
        constexpr int step = decltype(step_)::value;
        const uint32_t t = (uint32_t)((tile0 + tile) * kTile + 16 * grp) & in_page, stage = (tile & (kStages - 1)) * C::RAW;
        if constexpr (step == 0) {
            const uint32_t ok = (uint32_t)__ballot(group_entry >= 0) & 15u;
            placed = placed << 4 | ok;
            careful = careful << 1 | (ok != 15u || tile >= first_careful ? 1u : 0u);
            const uint32_t page = (uint32_t)max(__builtin_amdgcn_readlane(group_entry, grp), 0);
            page_rsrc = make_rsrc(head_base + (uint64_t)page * page_bytes, (uint32_t)kv_head_bytes(shift, D));
        } else if constexpr (step == 1) {
            if (D == 128 || lane < D / 2) load_to_lds(page_rsrc, code_src + t * (D / 2), code_dst + stage);
        } else {
            if (lane < D / 32) load_to_lds(page_rsrc, scale_src + t * (D / 32), scale_dst + stage);
        }
    };
    auto request_all = [&](int tile) { static_for<0, 3>([&](auto step_) { request(tile, step_); }); };
    // Converts values: feature pair dp of tokens 16 g + 8 x + 4 hv .. + 3, x both 0 and 1 (D = 64: one of them), which are an 8-key
    // chunk of the second product: the keys that half-wave hv's logits belong to.
    const int dp = tid % (D / 2), vg = (tid / (D / 2)) & 3, hv = (tid / (D / 2) >> 2) & 1, vx = D == 64 ? tid >> 8 : 0;
    const int v_src = C::CODES + (vg * (D / 2) + dp) * 16 + 8 * vx + 4 * hv;
    const int vs_src = 2 * C::CODES + C::SCALES + (vg * (D / 32) + (dp >> 4)) * 16 + 8 * vx + 4 * hv;
    const int v_dst = C::V_OFF + ((4 * (vg >> 1) + 2 * hv + (vg & 1)) * (D / 2) + dp) * 16 + 8 * vx;
    uint32_t vc[C::T / 4], vs[C::T / 4];
    auto values_fetch = [&](int tile) INLINE {
        const unsigned char *raw = smem + (tile & (kStages - 1)) * C::RAW;
#pragma unroll
        for (int i = 0; i < C::T / 4; ++i) {
            vc[i] = *(const uint32_t *)(raw + v_src + 8 * i);
            vs[i] = *(const uint32_t *)(raw + vs_src + 8 * i);
        }
    };
    // Values that no row of the workgroup sees are not to reach the product, whatever they are; a NaN among those that some see
    // goes to these rows alone, at the end.
    auto take_out = [&](int tile, uint32_t groups) INLINE {
        const bool ok = groups >> vg & 1u;
#pragma unroll
        for (int i = 0; i < C::T / 4; ++i) {
            const int key = (tile0 + tile) * kTile + 16 * vg + 8 * (vx + i) + 4 * hv;
            const uint32_t seen = first_bytes((ok ? kend : 0) - key), by_all = first_bytes(lim_min - key);
            const uint32_t nan = bytes_255(vs[i]) & ~by_all;
            if ((nan & seen) != 0) atomicMin(&nan_key[dp >> 4], key + (__ffs(nan & seen) - 1) / 8);
            const uint32_t gone = ~seen | nan;
            vc[i] &= ~gone;
            vs[i] = (vs[i] & ~gone) | (gone & 0x7f7f7f7fu);
        }
    };
    uint32_t w[C::T];
    auto convert = [&](auto t_) INLINE {
        constexpr int t = decltype(t_)::value;
        w[t] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(vc[t >> 2], scale_operand<(t & 3)>(vs[t >> 2]), t & 3));
    };
    auto values_store = [&](int tile, auto odd_) INLINE {       // of the pair's even or odd feature
        constexpr bool odd = decltype(odd_)::value;
        constexpr uint32_t sel = odd ? 0x07060302 : 0x05040100;
        unsigned char *dst = smem + v_dst + (tile & (kStages - 1)) * C::V_BYTES + (odd ? C::V_BYTES / 2 : 0);
        if constexpr (D == 128)
            *(u32x4 *)dst = u32x4{__builtin_amdgcn_perm(w[1], w[0], sel), __builtin_amdgcn_perm(w[3], w[2], sel), __builtin_amdgcn_perm(w[5], w[4], sel), __builtin_amdgcn_perm(w[7], w[6], sel)};
        else
            *(u32x2 *)dst = u32x2{__builtin_amdgcn_perm(w[1], w[0], sel), __builtin_amdgcn_perm(w[3], w[2], sel)};
    };
    auto values = [&](int tile, bool care, uint32_t groups) INLINE {        // all of it at once
        values_fetch(tile);
        if (care) take_out(tile, groups);
        static_for<0, C::T>(convert);
        values_store(tile, std::false_type{});
        values_store(tile, std::true_type{});
    };

    // ---- query rows, running softmax state, accumulators
    f32x16 o[OB];                // O^T: block 2 x + e holds features 64 x + 2 i + e, i the accumulator's row
    f32x16 s_acc[2];             // S^T of the key block whose softmax runs, and of the next one
    bf16x8 pf[2][2];             // P^T fragments: two per key block
    u32x4 kf[STEPS];             // K fragments of a key block
    uint32_t kscale[2];
    bf16x8 fr[C::RING];          // V^T fragments in flight from LDS
    float m_run, l_run = 0.f;
    Query<D> q;

    // Block j is half j % 2 of tile j / 2; its key c is row c of the first product.
    auto k_fetch = [&](int j, auto s_) INLINE {
        constexpr int s = decltype(s_)::value;
        const unsigned char *p = smem + ((j >> 1) & (kStages - 1)) * C::RAW + (j & 1) * (C::CODES / 2);
        kf[s] = *(const u32x4 *)(p + (c >> 4) * (C::CODES / 4) + (2 * s + hh) * 256 + (c & 15) * 16);
    };
    auto ks_fetch = [&](auto par_, int j) INLINE {
        constexpr int P = decltype(par_)::value;
        const unsigned char *p = smem + ((j >> 1) & (kStages - 1)) * C::RAW + 2 * C::CODES + (j & 1) * (C::SCALES / 2);
        if constexpr (D == 128) kscale[P] = *(const uint32_t *)(p + 4 * c) >> (8 * hh);
        else kscale[P] = *(const uint16_t *)(p + 2 * c) >> (8 * hh);
    };
    auto v_frag = [&](int j, auto p_) INLINE -> bf16x8 {       // of the block's product p: 16-key step p / OB, features p % OB
        constexpr int p = decltype(p_)::value, u = p / OB, x = p % OB / 2, e = p % OB % 2;
        const unsigned char *v = smem + C::V_OFF + ((j >> 1) & (kStages - 1)) * C::V_BYTES + e * (C::V_BYTES / 2);
        return *(const bf16x8 *)(v + ((4 * (j & 1) + 2 * hh + u) * (D / 2) + 32 * x + c) * 16);
    };
    auto s_mfma = [&](auto parts_, auto par_, auto n_) INLINE {        // product n of the logits: features 64 (n / parts) .., part n % parts
        constexpr int PARTS = decltype(parts_)::value, P = decltype(par_)::value, nn = decltype(n_)::value, s = nn / PARTS, p = nn % PARTS;
        const i32x8 ka = {(int)kf[s][0], (int)kf[s][1], (int)kf[s][2], (int)kf[s][3], 0, 0, 0, 0};
        const u32x6 w6 = q.part[s][p];
        const i32x8 qb = {(int)w6[0], (int)w6[1], (int)w6[2], (int)w6[3], (int)w6[4], (int)w6[5], 0, 0};
        const f32x16 zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
        if constexpr (nn == 0) s_acc[P] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ka, qb, zero, 4, 2, 2 * s, (int)kscale[P], p, (int)q.scale[s]);
        else s_acc[P] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(ka, qb, s_acc[P], 4, 2, 2 * s, (int)kscale[P], p, (int)q.scale[s]);
    };
    auto pv_mfma = [&](auto par_, auto p_) INLINE {
        constexpr int P = decltype(par_)::value, p = decltype(p_)::value;
        o[p % OB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[p % C::RING], pf[P][p / OB], o[p % OB], 0, 0, 0);
    };
    auto mask = [&](auto par_, int j, uint32_t groups) INLINE {        // logits of block j of keys that the row does not see
        constexpr int P = decltype(par_)::value;
        const uint32_t ok = groups >> (2 * (j & 1));
        const int key0 = tile0 * kTile + 32 * j + 4 * hh, left = min(lim, kend) - key0;
        const int left0 = ok & 1u ? left : INT_MIN, left1 = ok & 2u ? left : INT_MIN;
#pragma unroll
        for (int r = 0; r < 16; ++r)
            if (8 * (r >> 2) + (r & 3) >= (r < 8 ? left0 : left1)) s_acc[P][r] = -INFINITY;
    };

    // One slot, on key block j (logits in s_acc[j % 2]): S(j+1) = K_{j+1} Q^T and O^T += V_{j-1}^T P_{j-1}^T on the matrix cores beside
    // the softmax of block j on the vector ALU; on the way the K fragments of block j + 2 and, at the end, the first V fragments
    // of block j.  STAGE 1: tile `tile` is requested; 2: its values (in vc, vs) are converted.
    auto slot = [&](auto parts_, auto par_, auto has_s_, auto has_pv_, auto next_k_, bool masked, uint32_t groups, auto stage_, int j, int tile) INLINE {
        constexpr int P = decltype(par_)::value;
        constexpr bool HAS_S = decltype(has_s_)::value, HAS_PV = decltype(has_pv_)::value, NEXT_K = decltype(next_k_)::value;
        constexpr int STAGE = decltype(stage_)::value;
        constexpr int PARTS = decltype(parts_)::value, SN = STEPS * PARTS;     // products of a block's logits
        constexpr int SL = HAS_S ? SN : 0, NS = SL + (HAS_PV ? C::PVN : 0);
        if (__builtin_expect(masked, 0)) mask(par_, j, groups);
        float x[16], ps0 = 0.f, ps1 = 0.f;
        auto op_scale = [&](auto v_) {
            constexpr int v = decltype(v_)::value;
            if constexpr (v < 16) x[v] = fmaf(s_acc[P][v], a.scale_log2, -m_run);
        };
        auto op_exp = [&](auto v_) {
            constexpr int v = decltype(v_)::value;
            if constexpr (v < 16) x[v] = __builtin_amdgcn_exp2f(x[v]);
        };
        auto op_sum = [&](auto v_) {
            constexpr int v = decltype(v_)::value;
            if constexpr (v & 1) {
                ps1 += x[v];
                bf16x2 pk = {to_bf16(x[v - 1]), to_bf16(x[v])};
                asm volatile("" : "+v"(pk));
                pf[P][v >> 3][(v & 7) - 1] = pk[0];
                pf[P][v >> 3][v & 7] = pk[1];
            } else {
                ps0 += x[v];
            }
        };
        auto is_s = [](int n) constexpr { return HAS_S && (!HAS_PV || ((n & 1) == 0 && n < 2 * SL)); };
        auto idx = [](int n) constexpr { return HAS_S && HAS_PV ? (n < 2 * SL ? n >> 1 : n - SL) : n; };
        op_scale(std::integral_constant<int, 0>{});
        op_scale(std::integral_constant<int, 1>{});
        op_exp(std::integral_constant<int, 0>{});
        static_for<0, NS>([&](auto n_) {
            constexpr int n = decltype(n_)::value;
            if constexpr (is_s(n)) {
                s_mfma(parts_, std::integral_constant<int, P ^ 1>{}, std::integral_constant<int, idx(n)>{});
                // (a fragment's last product: the next block's takes its place)
                if constexpr (NEXT_K && idx(n) % PARTS == PARTS - 1) k_fetch(j + 2, std::integral_constant<int, idx(n) / PARTS>{});
            } else {
                constexpr int p = idx(n);
                if constexpr (p + C::PF < C::PVN) fr[(p + C::PF) % C::RING] = v_frag(j - 1, std::integral_constant<int, p + C::PF>{});
                else fr[(p + C::PF) % C::RING] = v_frag(j, std::integral_constant<int, p + C::PF - C::PVN>{});
                pv_mfma(std::integral_constant<int, P ^ 1>{}, std::integral_constant<int, p>{});
            }
            if constexpr (NEXT_K && n == 1) ks_fetch(par_, j + 2);
            if constexpr (STAGE == 1) {          // (beside products in flight: behind the barrier every wavefront would do it at once)
                if constexpr (n == 1) request(tile, std::integral_constant<int, 0>{});
                if constexpr (n == 3) request(tile, std::integral_constant<int, 1>{});
                static_assert(NS > 5, "a step for each");
                if constexpr (n == 4) request(tile, std::integral_constant<int, 2>{});
                if constexpr (n == 5) {
                    entry_fetch(tile + 1);
                    values_fetch(tile - 2);
                }
            }
            if constexpr (STAGE == 2) {
                static_for<C::T * n / (NS - 4), (n < NS - 4 ? C::T * (n + 1) / (NS - 4) : 0)>(convert);
                if constexpr (n == NS - 4) values_store(tile, std::false_type{});
                if constexpr (n == NS - 3) values_store(tile, std::true_type{});
            }
            static_for<16 * n / NS, 16 * (n + 1) / NS>([&](auto v_) {
                constexpr int v = decltype(v_)::value;
                op_scale(std::integral_constant<int, v + 2>{});
                op_exp(std::integral_constant<int, v + 1>{});
                op_sum(v_);
            });
            __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (!HAS_PV)
            static_for<0, C::PF>([&](auto p_) { fr[decltype(p_)::value] = v_frag(j, p_); });
        // Rarely a logit exceeded the running maximum by more than the threshold: raise it, rescale, redo the block.  Rows of the wavefront
        // without need keep their maximum and find the same probabilities and sums again, bit for bit.
        ps0 += ps1;
        if (__builtin_expect(__any(!(ps0 < 4096.0f)), 0)) {
            // (a use on this path too: the products of block j + 1 would otherwise be moved behind the branch, away from the softmax)
            if constexpr (HAS_S) asm volatile("" : "+v"(s_acc[P ^ 1]));
            float mx = s_acc[P][0];
            static_for<1, 16>([&](auto r_) { mx = fmaxf(mx, s_acc[P][decltype(r_)::value]); });
            mx = xhalf_max(mx) * a.scale_log2;
            const bool need = xhalf_max(ps0 < 4096.0f ? 0.f : 1.f) > 0.f;
            const float m_new = need ? fmaxf(m_run, mx) : m_run;
            const float alpha = m_new == m_run ? 1.0f : __builtin_amdgcn_exp2f(m_run - m_new);
            m_run = m_new;
            l_run *= alpha;
            if constexpr (HAS_PV)
                static_for<0, OB>([&](auto i_) { static_for<0, 16>([&](auto r_) { o[decltype(i_)::value][decltype(r_)::value] *= alpha; }); });
            ps0 = ps1 = 0.f;
            static_for<0, 16>([&](auto r_) {
                constexpr int r = decltype(r_)::value;
                const float p = __builtin_amdgcn_exp2f(fmaf(s_acc[P][r], a.scale_log2, -m_run));
                (r & 1 ? ps1 : ps0) += p;
                pf[P][r >> 3][r & 7] = to_bf16(p);
            });
            ps0 += ps1;
        }
        l_run += ps0;
    };

    const std::false_type no{};
    const std::true_type yes{};
    const std::integral_constant<int, 0> par0{};
    const std::integral_constant<int, 1> par1{};
    const std::integral_constant<int, 0> stage0{};
    const std::integral_constant<int, 1> stage1{};
    const std::integral_constant<int, 2> stage2{};

    // ---- prologue: the block table's first window, tiles 0 to 2 requested, the values of tile 0
    int entry = window_entry(0);
    window_store(0, entry);
    if (active) q.load((const bf16_t *)a.q + row_offset(row) + 32 * hh, row_there);
    __syncthreads();
    static_for<0, 3>([&](auto t_) {
        entry_fetch(decltype(t_)::value);
        request_all(decltype(t_)::value);
    });
    entry_fetch(3);
    wait_barrier<4>();                   // tile 0 is there
    values(0, careful >> 2 & 1u, placed >> 8);

    // Interval i holds the slots of blocks 2 i and 2 i + 1.  They read the keys of tile i + 1 and the values of tiles i - 1 and i; the
    // values of tile i + 1 are converted and tile i + 3 is requested.  The barrier at its end publishes the values and makes sure
    // that tile i + 2, requested an interval before, is there.
    auto table_ahead = [&](int i) INLINE {
        if (__builtin_expect((i & (kWindow - 5)) == 8, 0)) {          // 8 or 12 of 64
            if ((i & 4) == 0) entry = window_entry(i / kWindow + 1);
            else window_store(i / kWindow + 1, entry);
        }
    };
    auto attend = [&](auto parts_) INLINE {
        asm volatile("" ::: "memory");       // (the first fragments are read here, not before the choice of parts and kept for both)
        ks_fetch(par0, 0);
        ks_fetch(par1, 1);
        static_for<0, STEPS>([&](auto s_) { k_fetch(0, s_); });
        static_for<0, STEPS * decltype(parts_)::value>([&](auto n_) { s_mfma(parts_, par0, n_); });
        static_for<0, STEPS>([&](auto s_) { k_fetch(1, s_); });
        mask(par0, 0, placed >> 8);
        float mx = s_acc[0][0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s_acc[0][r]);
        m_run = fmaxf(xhalf_max(mx) * a.scale_log2, -FLT_MAX);
        wait_barrier<2>();
        {
            const uint32_t groups = placed >> 8, next = placed >> 4;
            const bool care_next = careful >> 1 & 1u;
            request_all(3);
            entry_fetch(4);
            slot(parts_, par0, yes, no, yes, true, groups, stage0, 0, 0);
#pragma unroll
            for (int i = 0; i < OB; ++i)
#pragma unroll
                for (int r = 0; r < 16; ++r) o[i][r] = 0.f;
            values_fetch(1);
            if (care_next) take_out(1, next);
            slot(parts_, par1, yes, yes, yes, true, groups, stage2, 1, 1);
            wait_barrier<2>();
        }
#pragma unroll 1
        for (int i = 1; i < n - 1; ++i) {
            table_ahead(i);
            const uint32_t groups = placed >> 8, next = placed >> 4;
            const bool masked = careful >> 2 & 1u, care_next = careful >> 1 & 1u;
            slot(parts_, par0, yes, yes, yes, masked, groups, stage1, 2 * i, i + 3);
            if (__builtin_expect(care_next, 0)) take_out(i + 1, next);
            slot(parts_, par1, yes, yes, yes, masked, groups, stage2, 2 * i + 1, i + 1);
            wait_barrier<2, 2>();        // (two fragments were requested after the values' last store)
        }
        const int j = 2 * (n - 1);
        slot(parts_, par0, yes, yes, no, true, placed >> 8, stage0, j, 0);
        slot(parts_, par1, no, yes, no, true, placed >> 8, stage0, j + 1, 0);
        static_for<0, C::PVN>([&](auto p_) {
            constexpr int p = decltype(p_)::value;
            if constexpr (p + C::PF < C::PVN) fr[(p + C::PF) % C::RING] = v_frag(j + 1, std::integral_constant<int, p + C::PF>{});
            pv_mfma(par1, p_);
        });
    };
    if (active) {
        if (__all(q.two)) attend(std::integral_constant<int, 2>{});
        else attend(std::integral_constant<int, 3>{});
    } else {                             // no rows: moves the tiles only
        m_run = 0.f;
        wait_barrier<2>();
#pragma unroll 1
        for (int i = 0; i < n - 1; ++i) {
            table_ahead(i);
            const uint32_t next = placed >> 4;
            const bool care_next = careful >> 1 & 1u;
            request_all(i + 3);
            entry_fetch(i + 4);
            values(i + 1, care_next, next);
            wait_barrier<2>();
        }
    }

    // ---- results
    wait_barrier<0>();                   // (nan_key of every wavefront; nothing is on its way into LDS)
    if (!active) return;
    l_run = xhalf_sum(l_run);
    static_for<0, STEPS>([&](auto s_) {
        constexpr int s = decltype(s_)::value;
        if (lim > nan_key[2 * s])
            for (int r = 0; r < 8; ++r) o[2 * s][r] = o[2 * s + 1][r] = NAN;
        if (lim > nan_key[2 * s + 1])
            for (int r = 8; r < 16; ++r) o[2 * s][r] = o[2 * s + 1][r] = NAN;
    });
    if (!row_there) return;
    if (whole) {
        const float inv = l_run == 0.f ? 0.f : 1.f / l_run;          // a row that sees nothing is zero
        int out_row = row;
        asm volatile("" : "+v"(out_row));                            // (its offset is worked out here, not kept from the beginning)
        bf16_t *out = (bf16_t *)a.out + row_offset(out_row);
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                bf16x8 y;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    y[2 * i] = to_bf16(o[2 * s][4 * g + i] * inv);
                    y[2 * i + 1] = to_bf16(o[2 * s + 1][4 * g + i] * inv);
                }
                *(bf16x8 *)(out + 64 * s + 16 * g + 8 * hh) = y;
            }
    } else {
        const size_t slot_ = ((size_t)(bh * (size_t)a.n_tiles + qt) * a.nsplit + split) * a.tile_rows + q0 + c;
        float *out = a.part_o + slot_ * D;
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int g = 0; g < 4; ++g)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    *(f32x4 *)(out + 64 * s + 16 * g + 8 * hh + 4 * i) = f32x4{o[2 * s][4 * g + 2 * i], o[2 * s + 1][4 * g + 2 * i], o[2 * s][4 * g + 2 * i + 1], o[2 * s + 1][4 * g + 2 * i + 1]};
        if (hh == 0) *(f32x2 *)(a.part_ml + slot_ * 2) = f32x2{m_run, l_run};
    }
}

}  // namespace

hipError_t launch_kv_tile(const KvAttnArgs &a, unsigned groups, hipStream_t stream)
{
    return a.D == 128 ? launch_kernel(kv_tile_kernel<128>, dim3(groups), dim3(kNT), stream, a) : launch_kernel(kv_tile_kernel<64>, dim3(groups), dim3(kNT), stream, a);
}

}  // namespace arl2
