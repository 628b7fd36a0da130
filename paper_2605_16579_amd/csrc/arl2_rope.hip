// Queries and keys divided by their root mean square, weighted and rotated by positions on several axes, and the gradients (gfx950):
//
//   y = R(pos) (w . x r),  r = 1 / sqrt(mean x^2 + eps) over a head's features, over a token's row, or no norm and no weight
//   R turns the pair i of axis a by pos_a theta_a^(-i / m_a):  (x0, x1) -> (x0 c - x1 s, x0 s + x1 c)
//   z = R(-pos) dy,   dw = sum over tokens of z . x r,   g = w z,   dx = r (g - x r mean(g . x r))
//
// The angle in turns is position times the pair's turns in fp64 (exact to 2^-53 of it, so far positions lose nothing), its
// fraction goes to fp32; a wavefront's lanes compute one pair each and hand cosine and sine on through LDS.  Memory bounds both.
//
// A unit is 8 pairs of a head, 16 features: neighbours (2i, 2i + 1), or i and i + D / 2.  A token's units (queries, then keys) are
// dealt to the lanes of WPT wavefronts, NU to a lane; 64 is a multiple of a head's units, so a lane's units all have the same pairs.
#include "arl2_device.h"
#include "arl2_rope.h"

namespace arl2 {
namespace {

constexpr int kThreads = 256;
constexpr int kMostWorkgroups = 2048;
constexpr int kGradWorkgroups = 512;

template <class T> struct Raw;                    // 8 features as they lie in memory
template <> struct Raw<bf16_t> { u32x4 v; };
template <> struct Raw<float> { f32x4 v[2]; };

__device__ __forceinline__ Raw<bf16_t> load8(const bf16_t *p) { return {*reinterpret_cast<const u32x4 *>(p)}; }
__device__ __forceinline__ Raw<float> load8(const float *p) { return {{*reinterpret_cast<const f32x4 *>(p), *reinterpret_cast<const f32x4 *>(p + 4)}}; }
__device__ __forceinline__ void widen(const Raw<bf16_t> &r, float *x)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) { x[2 * i] = __uint_as_float(r.v[i] << 16); x[2 * i + 1] = __uint_as_float(r.v[i] & 0xffff0000u); }
}
__device__ __forceinline__ void widen(const Raw<float> &r, float *x)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = r.v[i / 4][i % 4];
}
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

template <class T> struct Unit { Raw<T> lo, hi; };

// 16 features as floats in memory order (neighbours: 16 in a row; halves: 8 and, D / 2 further, 8)
template <class T>
__device__ __forceinline__ void widen(const Unit<T> &u, float *x) { widen(u.lo, x); widen(u.hi, x + 8); }

struct Turn { float c[8], s[8]; };

// The unit's pairs turned, backwards with SIGN -1; pairs from `pairs` on (counted from the unit's first) stay.
template <int SIGN>
__device__ __forceinline__ void turn_unit(float *x, const Turn &t, bool halves, bool partial, int pairs)
{
    auto one = [&](float &x0, float &x1, int i) {
        const float s = SIGN * t.s[i], y0 = x0 * t.c[i] - x1 * s, y1 = x0 * s + x1 * t.c[i];
        const bool stays = partial && i >= pairs;
        x0 = stays ? x0 : y0;
        x1 = stays ? x1 : y1;
    };
    if (halves) {
#pragma unroll
        for (int i = 0; i < 8; ++i) one(x[i], x[8 + i], i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) one(x[2 * i], x[2 * i + 1], i);
    }
}

// What a lane knows of its units: unit u of a token is number u * 64 * WPT + (lane among the token's).
struct Lane {
    int upt, units[2], first, step, in_head, hi;     // units per head, of queries and keys; its first, from one to the next; place in the head
};

template <int WPT>
__device__ __forceinline__ Lane lane_of(const RopeArgs &a)
{
    Lane m;
    m.upt = a.D / 16;
    m.units[0] = a.heads[0] * m.upt;
    m.units[1] = a.heads[1] * m.upt;
    m.first = WPT == 1 ? threadIdx.x & 63 : threadIdx.x;
    m.step = 64 * WPT;
    m.in_head = m.first & (m.upt - 1);
    m.hi = a.halves ? a.D / 2 : 8;
    return m;
}
// Which array (0, 1; 2: none) the lane's unit u lies in, and the offset of its features in that array's rows.
__device__ __forceinline__ int place(const RopeArgs &a, const Lane &m, int u, int &offset)
{
    int i = m.first + u * m.step;
    const int which = i < m.units[0] ? 0 : i < m.units[0] + m.units[1] ? 1 : 2;
    if (which) i -= m.units[0];
    offset = i / m.upt * a.D + m.in_head * (a.halves ? 8 : 16);
    return which;
}

template <class T>
__device__ __forceinline__ Unit<T> load_unit(const T *p, int hi) { return {load8(p), load8(p + hi)}; }

// Sum over the lanes of a head's units (8 at D = 128, 4 at D = 64).
__device__ __forceinline__ float head_sum(float x, int upt)
{
    x += dpp_peek<0xB1>(x);
    x += dpp_peek<0x4E>(x);
    return upt == 8 ? x + dpp_peek<0x141>(x) : x;
}
__device__ __forceinline__ float wave_sum(float x)
{
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) x += __shfl_xor(x, m, kWave);
    return x;
}

// Sums over a token's lanes of two values; `red` and two barriers where the token has several wavefronts.
template <int WPT>
__device__ __forceinline__ void token_sums(float &x, float &y, float (*red)[2])
{
    x = wave_sum(x);
    y = wave_sum(y);
    if constexpr (WPT > 1) {
        if ((threadIdx.x & 63) == 0) { red[threadIdx.x >> 6][0] = x; red[threadIdx.x >> 6][1] = y; }
        __syncthreads();
        x = y = 0.f;
#pragma unroll
        for (int w = 0; w < WPT; ++w) { x += red[w][0]; y += red[w][1]; }
        __syncthreads();
    }
}

// Cosines and sines of the lane's eight pairs at a token (b, l).
__device__ __forceinline__ Turn turns_of(const RopeArgs &a, const Lane &m, double step, int axis, int b, int l, f32x2 *own)
{
    const int lane = threadIdx.x & 63;
    if (lane < a.D / 2) {
        const int32_t p = a.pos[((a.pos_per_stream ? (size_t)b * a.L : 0) + l) * a.axes + axis];
        const double t = (double)p * step;
        float s, c;
        sincospif(2.f * (float)(t - ::rint(t)), &s, &c);
        own[lane] = f32x2{c, s};
    }
    __builtin_amdgcn_wave_barrier();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    Turn r;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const f32x4 v = *reinterpret_cast<const f32x4 *>(&own[8 * m.in_head + 2 * i]);
        r.c[2 * i] = v[0]; r.s[2 * i] = v[1]; r.c[2 * i + 1] = v[2]; r.s[2 * i + 1] = v[3];
    }
    __builtin_amdgcn_wave_barrier();
    return r;
}

template <class T, int NU, int WPT>
__global__ __launch_bounds__(kThreads) void rope_kernel(RopeArgs a)
{
    __shared__ __align__(16) f32x2 turns[4][64];
    __shared__ float red[4][2];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const Lane m = lane_of<WPT>(a);
    const bool partial = a.pairs < a.D / 2;
    const double step = lane < a.D / 2 ? a.turns[lane] : 0.0;
    const int axis = lane < a.D / 2 ? a.axis[lane] : 0;
    Unit<T> w[NU];
    int which[NU], off[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        which[u] = place(a, m, u, off[u]);
        if (which[u] < 2 && a.w[which[u]] != nullptr)
            w[u] = load_unit((const T *)a.w[which[u]] + (a.norm == kNormHead ? off[u] % a.D : off[u]), m.hi);
    }
    const long long tokens = (long long)a.B * a.L;
    for (long long t = WPT == 1 ? (long long)blockIdx.x * 4 + wave : blockIdx.x; t < tokens; t += (long long)gridDim.x * (WPT == 1 ? 4 : 1)) {
        const int b = (int)(t / a.L), l = (int)(t - (long long)b * a.L);
        if (a.len != nullptr && l >= a.len[b]) continue;
        Unit<T> x[NU];
#pragma unroll
        for (int u = 0; u < NU; ++u)
            if (which[u] < 2) x[u] = load_unit((const T *)a.x[which[u]] + (size_t)t * a.heads[which[u]] * a.D + off[u], m.hi);
        const Turn turn = turns_of(a, m, step, axis, b, l, turns[wave]);
        float row[2] = {1.f, 1.f};
        if (a.norm == kNormRow) {
            row[0] = row[1] = 0.f;
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                float f[16], s = 0.f;
                widen(x[u], f);
#pragma unroll
                for (int i = 0; i < 16; ++i) s = fmaf(f[i], f[i], s);
                row[0] += which[u] == 0 ? s : 0.f;
                row[1] += which[u] == 1 ? s : 0.f;
            }
            token_sums<WPT>(row[0], row[1], red);
#pragma unroll
            for (int i = 0; i < 2; ++i) row[i] = 1.f / sqrtf(row[i] / (float)(a.heads[i] * a.D) + a.eps);
        }
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            float f[16];
            widen(x[u], f);
            float r = which[u] == 1 ? row[1] : row[0];
            if (a.norm == kNormHead) {
                float s = 0.f;
#pragma unroll
                for (int i = 0; i < 16; ++i) s = fmaf(f[i], f[i], s);
                s = head_sum(s, m.upt);
                r = 1.f / sqrtf(s / (float)a.D + a.eps);
            }
            if (which[u] == 2) continue;
            if (a.norm != kNormNone) {
#pragma unroll
                for (int i = 0; i < 16; ++i) f[i] *= r;
                if (a.w[which[u]] != nullptr) {
                    float g[16];
                    widen(w[u], g);
#pragma unroll
                    for (int i = 0; i < 16; ++i) f[i] *= g[i];
                }
            }
            turn_unit<1>(f, turn, a.halves, partial, a.pairs - 8 * m.in_head);
            T *const to = (T *)a.y[which[u]] + (size_t)t * a.heads[which[u]] * a.D + off[u];
            store8(to, f);
            store8(to + m.hi, f + 8);
        }
    }
}

// Sums of weights' gradients stay with their lane over all of a workgroup's tokens (one axis of the units for weights of a head's
// features), are joined in LDS and written as this workgroup's part.
template <class T, int NU, int WPT>
__global__ __launch_bounds__(kThreads) void rope_bwd_kernel(RopeArgs a)
{
    __shared__ __align__(16) f32x2 turns[4][64];
    __shared__ float red[4][2];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const Lane m = lane_of<WPT>(a);
    const bool partial = a.pairs < a.D / 2;
    const double step = lane < a.D / 2 ? a.turns[lane] : 0.0;
    const int axis = lane < a.D / 2 ? a.axis[lane] : 0;
    Unit<T> w[NU];
    float dw[NU][16] = {};
    int which[NU], off[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
        which[u] = place(a, m, u, off[u]);
        if (which[u] < 2 && a.w[which[u]] != nullptr)
            w[u] = load_unit((const T *)a.w[which[u]] + (a.norm == kNormHead ? off[u] % a.D : off[u]), m.hi);
    }
    const long long tokens = (long long)a.B * a.L;
    for (long long t = WPT == 1 ? (long long)blockIdx.x * 4 + wave : blockIdx.x; t < tokens; t += (long long)gridDim.x * (WPT == 1 ? 4 : 1)) {
        const int b = (int)(t / a.L), l = (int)(t - (long long)b * a.L);
        if (a.len != nullptr && l >= a.len[b]) continue;
        Unit<T> x[NU], d[NU];
#pragma unroll
        for (int u = 0; u < NU; ++u)
            if (which[u] < 2) {
                const size_t at = (size_t)t * a.heads[which[u]] * a.D + off[u];
                d[u] = load_unit((const T *)a.dy[which[u]] + at, m.hi);
                if (a.norm != kNormNone) x[u] = load_unit((const T *)a.x[which[u]] + at, m.hi);
            }
        const Turn turn = turns_of(a, m, step, axis, b, l, turns[wave]);
        float row[2] = {0.f, 0.f}, dot[2] = {0.f, 0.f};
        if (a.norm == kNormRow) {
#pragma unroll
            for (int u = 0; u < NU; ++u) {
                float f[16], g[16], wf[16], s = 0.f, p = 0.f;
                widen(x[u], f);
                widen(d[u], g);
                turn_unit<-1>(g, turn, a.halves, partial, a.pairs - 8 * m.in_head);
                const bool weighted = which[u] < 2 && a.w[which[u]] != nullptr;
                if (weighted) widen(w[u], wf);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s = fmaf(f[i], f[i], s);
                    p = fmaf(f[i], weighted ? g[i] * wf[i] : g[i], p);
                }
                row[0] += which[u] == 0 ? s : 0.f;
                row[1] += which[u] == 1 ? s : 0.f;
                dot[0] += which[u] == 0 ? p : 0.f;
                dot[1] += which[u] == 1 ? p : 0.f;
            }
            token_sums<WPT>(row[0], row[1], red);
            token_sums<WPT>(dot[0], dot[1], red);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float over = 1.f / (float)(a.heads[i] * a.D);
                row[i] = 1.f / sqrtf(row[i] * over + a.eps);
                dot[i] *= row[i] * over;
            }
        }
#pragma unroll
        for (int u = 0; u < NU; ++u) {
            float g[16];
            widen(d[u], g);
            turn_unit<-1>(g, turn, a.halves, partial, a.pairs - 8 * m.in_head);
            if (a.norm != kNormNone) {
                float f[16], wf[16];
                widen(x[u], f);
                const bool weighted = which[u] < 2 && a.w[which[u]] != nullptr;
                if (weighted) widen(w[u], wf);
                float r = which[u] == 1 ? row[1] : row[0], p = which[u] == 1 ? dot[1] : dot[0];
                if (a.norm == kNormHead) {
                    float s = 0.f;
                    p = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        s = fmaf(f[i], f[i], s);
                        p = fmaf(f[i], weighted ? g[i] * wf[i] : g[i], p);
                    }
                    s = head_sum(s, m.upt);
                    p = head_sum(p, m.upt);
                    r = 1.f / sqrtf(s / (float)a.D + a.eps);
                    p *= r / (float)a.D;
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float xh = f[i] * r;
                    if (which[u] < 2) dw[u][i] = fmaf(g[i], xh, dw[u][i]);
                    g[i] = r * ((weighted ? g[i] * wf[i] : g[i]) - xh * p);
                }
            }
            if (which[u] == 2) continue;
            T *const to = (T *)a.y[which[u]] + (size_t)t * a.heads[which[u]] * a.D + off[u];
            store8(to, g);
            store8(to + m.hi, g + 8);
        }
    }
    if (a.norm == kNormNone || (a.dw[0] == nullptr && a.dw[1] == nullptr)) return;
    // this workgroup's part: [D] and [D], or [heads D] and [heads D]
    extern __shared__ __align__(16) float part[];
    const int width0 = a.norm == kNormHead ? a.D : a.heads[0] * a.D, width = width0 + (a.norm == kNormHead ? a.D : a.heads[1] * a.D);
    if (WPT > 1 && a.norm == kNormRow) {                          // each of its elements is one lane's
        float *const to = a.part + (size_t)blockIdx.x * width;
#pragma unroll
        for (int u = 0; u < NU; ++u)
            if (which[u] < 2)
#pragma unroll
                for (int i = 0; i < 16; ++i) to[(which[u] ? width0 : 0) + off[u] + (i < 8 ? i : m.hi + i - 8)] = dw[u][i];
        return;
    }
    for (int i = threadIdx.x; i < width; i += kThreads) part[i] = 0.f;
    __syncthreads();
    if (a.norm == kNormHead) {
        // lanes of the same place in their heads, units of a lane: one sum of each array
        float sum[2][16] = {};
#pragma unroll
        for (int u = 0; u < NU; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                sum[0][i] += which[u] == 0 ? dw[u][i] : 0.f;
                sum[1][i] += which[u] == 1 ? dw[u][i] : 0.f;
            }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                for (int s = m.upt; s < 64; s <<= 1) sum[k][i] += __shfl_xor(sum[k][i], s, kWave);
        for (int v = 0; v < 4; ++v) {
            if (wave == v && lane < m.upt)
#pragma unroll
                for (int k = 0; k < 2; ++k)
#pragma unroll
                    for (int i = 0; i < 16; ++i) part[(k ? width0 : 0) + m.in_head * (a.halves ? 8 : 16) + (i < 8 ? i : m.hi + i - 8)] += sum[k][i];
            __syncthreads();
        }
    } else {
        for (int v = 0; v < 4; ++v) {
            if (wave == v)
#pragma unroll
                for (int u = 0; u < NU; ++u)
                    if (which[u] < 2)
#pragma unroll
                        for (int i = 0; i < 16; ++i) part[(which[u] ? width0 : 0) + off[u] + (i < 8 ? i : m.hi + i - 8)] += dw[u][i];
            __syncthreads();
        }
    }
    for (int i = threadIdx.x; i < width; i += kThreads) a.part[(size_t)blockIdx.x * width + i] = part[i];
}

// Weights' gradients: 16 columns to a workgroup, the workgroups' parts in 16 groups added in order.
__global__ __launch_bounds__(256) void rope_dw_kernel(RopeArgs a, int parts, int width0, int width)
{
    __shared__ float sums[16][17];
    const int c = threadIdx.x & 15, g = threadIdx.x >> 4, col = blockIdx.x * 16 + c;
    float s = 0.f;
    for (int p = g; p < parts; p += 16) s += a.part[(size_t)p * width + col];
    sums[g][c] = s;
    __syncthreads();
    if (g > 0) return;
    s = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) s += sums[i][c];
    float *const to = col < width0 ? a.dw[0] : a.dw[1];
    if (to != nullptr) to[col < width0 ? col : col - width0] = s;
}

// Wavefronts to a token and units to a lane: one wavefront while five units do.
struct Shape { int wpt, nu; };
Shape shape_of(int units)
{
    if (units <= 320) return {1, units <= 64 ? 1 : units <= 128 ? 2 : units <= 192 ? 3 : 5};
    return {4, units <= 512 ? 2 : units <= 768 ? 3 : 6};
}

template <class T, bool BWD>
hipError_t launch_shape(const RopeArgs &a, dim3 grid, unsigned lds, hipStream_t stream)
{
    const Shape s = shape_of((a.heads[0] + a.heads[1]) * (a.D / 16));
#define ARL2_ROPE(NU, WPT) launch_kernel_lds(BWD ? rope_bwd_kernel<T, NU, WPT> : rope_kernel<T, NU, WPT>, grid, dim3(kThreads), lds, stream, a)
    if (s.wpt == 1) return s.nu == 1 ? ARL2_ROPE(1, 1) : s.nu == 2 ? ARL2_ROPE(2, 1) : s.nu == 3 ? ARL2_ROPE(3, 1) : ARL2_ROPE(5, 1);
    return s.nu == 2 ? ARL2_ROPE(2, 4) : s.nu == 3 ? ARL2_ROPE(3, 4) : ARL2_ROPE(6, 4);
#undef ARL2_ROPE
}

int workgroups(int B, int L, int units, int most)
{
    const long long tokens = (long long)B * L, n = shape_of(units).wpt == 1 ? (tokens + 3) / 4 : tokens;
    return (int)(n < most ? n : most);
}

}  // namespace

int rope_workgroups(int B, int L, int D, int heads) { return workgroups(B, L, heads * (D / 16), kGradWorkgroups); }

size_t rope_workspace_bytes(int B, int L, int D, int heads)
{
    return (((size_t)rope_workgroups(B, L, D, heads) * heads * D * sizeof(float)) + 255) & ~(size_t)255;
}

hipError_t launch_rope(const RopeArgs &a, hipStream_t stream)
{
    const dim3 grid(workgroups(a.B, a.L, (a.heads[0] + a.heads[1]) * (a.D / 16), kMostWorkgroups));
    return a.f32 ? launch_shape<float, false>(a, grid, 0, stream) : launch_shape<bf16_t, false>(a, grid, 0, stream);
}

hipError_t launch_rope_bwd(const RopeArgs &a, hipStream_t stream)
{
    const int n = rope_workgroups(a.B, a.L, a.D, a.heads[0] + a.heads[1]);
    const bool weights = a.norm != kNormNone && (a.dw[0] != nullptr || a.dw[1] != nullptr);
    const int width0 = a.norm == kNormHead ? a.D : a.heads[0] * a.D, width = a.norm == kNormHead ? 2 * a.D : (a.heads[0] + a.heads[1]) * a.D;
    const bool direct = a.norm == kNormRow && shape_of((a.heads[0] + a.heads[1]) * (a.D / 16)).wpt > 1;
    const unsigned lds = weights && !direct ? (unsigned)(width * sizeof(float)) : 0;        // 20 KB at the most
    const hipError_t e = a.f32 ? launch_shape<float, true>(a, dim3(n), lds, stream) : launch_shape<bf16_t, true>(a, dim3(n), lds, stream);
    if (e != hipSuccess || !weights) return e;
    return launch_kernel(rope_dw_kernel, dim3(width / 16), dim3(256), stream, a, n, width0, width);
}

}  // namespace arl2
