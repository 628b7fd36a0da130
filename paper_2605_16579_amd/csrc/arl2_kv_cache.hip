// Paged 4-bit key/value cache (gfx950): appending rows, with the position rotation applied to the keys, and reading rows back.
//
//   append:  k'_p = RoPE_p(k_p) (pairs (2i, 2i + 1)), then k'_p and v_p per 32 features as  2^e * c,  c from e2m1
//            = {0, 1/2, 1, 3/2, 2, 3, 4, 6, and negative}, e the least exponent with max |x| <= 7 * 2^e
//   read:    the values 2^e * c as bf16, which holds them exactly (2 significant bits)
//
// The rotation is computed in fp64: products of a bf16 feature and an fp32 cosine are exact there (32 of 53 bits), so the sum of
// two of them is rounded the same whatever the order, and the fp32 value it is rounded to does not depend on how it was
// computed; a code next to a rounding border would otherwise come out differently here and there.  4680 tokens of 12 heads x 128 in a
// loop of appends: 10.3 us, with fp32 products instead 9.4, without tables and rotation 7.7.
// e: 7 2^e rather than 6 2^e is the border because values between 6 and 7 are off by at most 1 when stored as 6, half of the step
// between 4 and 6; at twice the scale every other value of the group would lose a bit.
// The conversion to e2m1 is the hardware's (round to nearest even, saturating).
//
// One thread: 8 features of four tokens at positions 4 m .. 4 m + 3, keys and values: 16-byte loads, a row by D / 8 consecutive
// lanes, the group's maximum by two exchanges between four lanes.  Four neighbouring threads groups make a 16-token group; the
// heads of a group follow one another, so that a workgroup's heads find the rotation tables in its CU's cache.  The four tokens of
// a value pair are one 4-byte store (they are neighbours in the cache), at D = 128 the whole group's 16 tokens one 16-byte store after
// an exchange between lanes; where the call has only some of the tokens they are stored byte by byte.
//
// What bounds them: memory, and the loads that wait for one another (lengths, then rows and page, then stores); append's rotation and
// tables besides (every head loads these anew, and all workgroups are in the same phase).  4680 tokens of 12 heads x 128, append and read in
// turn: 12.2 us (38.7 MB: 3.2 TB/s) and 8.8 us (36.4 MB: 4.1 TB/s); reading 4 x 1560 tokens 11.2 us (48.5 MB: 4.3 TB/s); a copy of 1 GiB
// moves 4.85 TB/s.  One token of 16 streams: 4.8 and 3.2 us, which is launch and latency.
#include "arl2_device.h"

namespace arl2 {
namespace {

constexpr int kThreads = 256;
constexpr uint32_t kScaleMin = 7, kScaleMax = 252, kScaleNan = 255;    // 2^-120 (half of it is a normal number) .. 2^125 (6 times it is finite)

// Maximum over aligned groups of four lanes.
__device__ __forceinline__ uint32_t quad_max(uint32_t x)
{
    x = max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0xB1, 0xf, 0xf, true));      // quad_perm [1,0,3,2]
    return max(x, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, 0x4E, 0xf, 0xf, true));   // quad_perm [2,3,0,1]
}

// Codes of 8 features (4 bytes) and the scale of the 32 that four lanes hold together.
__device__ __forceinline__ uint32_t quantise(const float *y, uint32_t &scale)
{
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(y[j]) & 0x7fffffffu);     // (as integers in the order of magnitudes, NaN above all)
    m = quad_max(m);
    // max |x| = f 2^(E - 126) with f in [1/2, 1): e = E - 129, one more from f > 7/8 on; as a byte e + 127
    const int e = (int)((m + 0x1fffffu) >> 23) - 2;
    scale = m >= 0x7f800000u ? kScaleNan : (uint32_t)min(max(e, (int)kScaleMin), (int)kScaleMax);
    const float s = __uint_as_float(min(scale, kScaleMax) << 23);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[0], y[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[2], y[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[4], y[5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, y[6], y[7], s, 3);
    return scale == kScaleNan ? 0 : c;
}

__device__ __forceinline__ u32x4 dequantise(uint32_t codes, uint32_t scale)
{
    const float s = __uint_as_float(scale << 23);          // (255: NaN out of the conversion)
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0));
    r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1));
    r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2));
    r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3));
    return r;
}

// 4 x 4 bytes: byte j of r[i] is byte i of x[j].
__device__ __forceinline__ u32x4 transpose_bytes(u32x4 x)
{
    const uint32_t a = __builtin_amdgcn_perm(x[1], x[0], 0x05010400), b = __builtin_amdgcn_perm(x[3], x[2], 0x05010400);     // 0,0' 1,1'
    const uint32_t c = __builtin_amdgcn_perm(x[1], x[0], 0x07030602), d = __builtin_amdgcn_perm(x[3], x[2], 0x07030602);     // 2,2' 3,3'
    u32x4 r;
    r[0] = __builtin_amdgcn_perm(b, a, 0x05040100);
    r[1] = __builtin_amdgcn_perm(b, a, 0x07060302);
    r[2] = __builtin_amdgcn_perm(d, c, 0x05040100);
    r[3] = __builtin_amdgcn_perm(d, c, 0x07060302);
    return r;
}

// Words I and J become (I's lower and J's lower half-wave, I's upper and J's upper one); the same with every 16 lanes and the next.
template <int I, int J>
__device__ __forceinline__ void swap32(u32x4 &x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(x[I], x[J], false, false);
    x[I] = r[0];
    x[J] = r[1];
}
template <int I, int J>
__device__ __forceinline__ void swap16(u32x4 &x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(x[I], x[J], false, false);
    x[I] = r[0];
    x[J] = r[1];
}

// What a thread works on.
struct Item {
    int b, h, chunk;        // stream, head, 8-feature chunk
    int64_t pos;            // its four positions begin here (a multiple of four)
    int64_t first;          // the call's first position
    int count;              // the call's tokens of this stream
    int page;               // page of the positions, or -1
    __device__ bool has(int i) const { return pos + i >= first && pos + i < first + count; }
    __device__ bool has_all() const { return pos >= first && pos + 4 <= first + count; }
    __device__ bool has_any() const { return pos + 4 > first && pos < first + count; }
    __device__ size_t row(int i, int L, int H) const { return ((size_t)b * L + (size_t)(pos + i - first)) * H + h; }
};

template <int D>
__device__ __forceinline__ bool item_of(const KvRowsArgs &a, Item &it)
{
    constexpr int CPR = D / 8;
    const uint32_t id = blockIdx.x * kThreads + threadIdx.x;
    it.chunk = id % CPR;
    uint32_t rest = id / CPR;
    const uint32_t quad = rest & 3, groups = (uint32_t)(a.L + 15) / 16 + 1;
    rest >>= 2;
    it.h = rest % a.pool.heads;
    rest /= a.pool.heads;
    const uint32_t group = rest % groups;
    it.b = rest / groups;
    if (it.b >= a.B) return false;
    it.first = a.start[it.b];
    it.count = a.count != nullptr ? kv_clamp(a.count[it.b], a.L) : a.L;
    it.pos = ((it.first >> 4) + group) * 16 + 4 * quad;    // (a negative position has no page)
    if (!it.has_any()) return false;
    it.page = kv_page(a.pool, a.table + (size_t)it.b * a.pool.max_pages, it.pos);
    return true;
}

template <int D>
__global__ __launch_bounds__(kThreads) void kv_append_kernel(KvRowsArgs a)
{
    Item it;
    if (!item_of<D>(a, it)) return;
    const int shift = a.pool.shift, t = (int)it.pos & ((1 << shift) - 1), H = a.pool.heads;
    u32x4 kx[4], vx[4];
    f32x4 cs[4], sn[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        kx[i] = vx[i] = u32x4{0, 0, 0, 0};
        if (!it.has(i)) continue;
        const size_t off = it.row(i, a.L, H) * D + 8 * it.chunk;
        kx[i] = *(const u32x4 *)((const bf16_t *)a.k + off);
        vx[i] = *(const u32x4 *)((const bf16_t *)a.v + off);
        if (a.cs != nullptr && it.pos + i >= 0 && it.pos + i < kv_capacity(a.pool)) {       // (the tables' rows)
            cs[i] = *(const f32x4 *)(a.cs + (size_t)(it.pos + i) * (D / 2) + 4 * it.chunk);
            sn[i] = *(const f32x4 *)(a.sn + (size_t)(it.pos + i) * (D / 2) + 4 * it.chunk);
        }
    }
    // The rows are on their way before the page is known to exist: they are there in any case.  The four lanes of a group have the same
    // page and leave together.
    asm volatile("" ::: "memory");
    if (it.page < 0) return;
    unsigned char *base = (unsigned char *)a.cache + kv_head_offset(a.pool, D, it.page, it.h);
    u32x4 vcodes;
    uint32_t vscale[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float y[8], w[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            y[2 * j] = __uint_as_float(kx[i][j] << 16);
            y[2 * j + 1] = __uint_as_float(kx[i][j] & 0xffff0000u);
            w[2 * j] = __uint_as_float(vx[i][j] << 16);
            w[2 * j + 1] = __uint_as_float(vx[i][j] & 0xffff0000u);
            if (a.cs != nullptr && it.has(i)) {
                const double x0 = y[2 * j], x1 = y[2 * j + 1], c = cs[i][j], s = sn[i][j];
                y[2 * j] = (float)(x0 * c - x1 * s);
                y[2 * j + 1] = (float)(x0 * s + x1 * c);
            }
        }
        uint32_t kscale;
        const uint32_t kcodes = quantise(y, kscale);
        vcodes[i] = quantise(w, vscale[i]);
        if (it.has(i)) {
            *(uint32_t *)(base + kv_key_codes(t + i, 4 * it.chunk, D)) = kcodes;
            if ((it.chunk & 3) == 0) base[kv_key_scales(shift, t + i, it.chunk >> 2, D)] = (unsigned char)kscale;
        }
    }
    if (it.has_all()) {
        u32x4 r = transpose_bytes(vcodes);
        if (D == 128 && __popcll(__ballot(true)) == kWave) {
            // The wavefront has all of a 16-token group.  Lane 16 q + i holds tokens 4 q .. of feature pairs 4 i + j in word j; after the
            // exchange it holds all tokens of pair 4 i + q.
            swap32<0, 2>(r);
            swap32<1, 3>(r);
            swap16<0, 1>(r);
            swap16<2, 3>(r);
            *(u32x4 *)(base + kv_value_codes(shift, t & ~15, 4 * it.chunk + ((threadIdx.x >> 4) & 3), D)) = r;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) *(uint32_t *)(base + kv_value_codes(shift, t, 4 * it.chunk + j, D)) = r[j];
        }
        if ((it.chunk & 3) == 0)
            *(uint32_t *)(base + kv_value_scales(shift, t, it.chunk >> 2, D)) = vscale[0] | vscale[1] << 8 | vscale[2] << 16 | vscale[3] << 24;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (it.has(i)) {
#pragma unroll
            for (int j = 0; j < 4; ++j) base[kv_value_codes(shift, t + i, 4 * it.chunk + j, D)] = (unsigned char)(vcodes[i] >> (8 * j));
            if ((it.chunk & 3) == 0) base[kv_value_scales(shift, t + i, it.chunk >> 2, D)] = (unsigned char)vscale[i];
        }
}

// The rows' values; zeros where nothing is stored.
template <int D>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(KvRowsArgs a)
{
    Item it;
    if (!item_of<D>(a, it)) return;
    const int shift = a.pool.shift, t = (int)it.pos & ((1 << shift) - 1), H = a.pool.heads;
    const unsigned char *base = (const unsigned char *)a.cache + kv_head_offset(a.pool, D, it.page < 0 ? 0 : it.page, it.h);
    u32x4 kc = {0, 0, 0, 0}, vc = kc, ks = kc, vs = kc;
    if (it.page >= 0) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            kc[i] = *(const uint32_t *)(base + kv_key_codes(t + i, 4 * it.chunk, D));
            vc[i] = *(const uint32_t *)(base + kv_value_codes(shift, t, 4 * it.chunk + i, D));
            ks[i] = base[kv_key_scales(shift, t + i, it.chunk >> 2, D)];
        }
        const uint32_t w = *(const uint32_t *)(base + kv_value_scales(shift, t, it.chunk >> 2, D));
#pragma unroll
        for (int i = 0; i < 4; ++i) vs[i] = (w >> (8 * i)) & 255u;
    }
    vc = transpose_bytes(vc);
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (it.has(i)) {
            const size_t off = it.row(i, a.L, H) * D + 8 * it.chunk;
            *(u32x4 *)((bf16_t *)a.k_out + off) = dequantise(kc[i], ks[i]);
            *(u32x4 *)((bf16_t *)a.v_out + off) = dequantise(vc[i], vs[i]);
        }
}

unsigned row_groups(const KvRowsArgs &a, int D)
{
    const long long n = (long long)a.B * a.pool.heads * ((a.L + 15) / 16 + 1) * 4 * (D / 8);
    return (unsigned)((n + kThreads - 1) / kThreads);
}

}  // namespace

hipError_t launch_kv_append(const KvRowsArgs &a, hipStream_t stream)
{
    const dim3 grid(row_groups(a, a.D)), block(kThreads);
    return a.D == 128 ? launch_kernel(kv_append_kernel<128>, grid, block, stream, a) : launch_kernel(kv_append_kernel<64>, grid, block, stream, a);
}

hipError_t launch_kv_read(const KvRowsArgs &a, hipStream_t stream)
{
    const dim3 grid(row_groups(a, a.D)), block(kThreads);
    return a.D == 128 ? launch_kernel(kv_read_kernel<128>, grid, block, stream, a) : launch_kernel(kv_read_kernel<64>, grid, block, stream, a);
}

}  // namespace arl2
