// Host side of the C ABI declared in include/arl2.h: argument validation, dispatch to the
// gfx950 kernels, error reporting.  Nothing here allocates device memory or synchronises.
#include "../../include/arl2.h"
#include "arl2_device.h"
#include "arl2_rope.h"
#include "arl2_scan.h"

#include <atomic>
#include <cmath>
#include <cstdio>
#include <cstring>
#include <initializer_list>

namespace {

thread_local char g_err[256] = "";

arl2_status fail(arl2_status s, const char *fmt, const char *detail = "")
{
    std::snprintf(g_err, sizeof(g_err), fmt, detail);
    return s;
}

bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Do the byte ranges [a, a + na) and [b, b + nb) share a byte?  (NULL pointers overlap nothing.)
bool overlaps(const void *a, size_t na, const void *b, size_t nb)
{
    if (a == nullptr || b == nullptr || na == 0 || nb == 0) return false;
    const uintptr_t pa = reinterpret_cast<uintptr_t>(a), pb = reinterpret_cast<uintptr_t>(b);
    return pa < pb + nb && pb < pa + na;
}

size_t elem_bytes(int dtype) { return dtype == ARL2_BF16 ? 2 : 4; }
size_t q_bytes(const arl2_desc *d) { return (size_t)d->B * d->Lq * d->H * d->D * elem_bytes(d->io_dtype); }
size_t kv_bytes(const arl2_desc *d) { return (size_t)d->B * d->Lkv * d->H * d->D * elem_bytes(d->io_dtype); }
size_t state_bytes(const arl2_desc *d) { return (size_t)d->B * d->H * d->D * d->D * sizeof(float); }
size_t g_bytes(const arl2_desc *d)
{
    const size_t per_token = d->g_mode == ARL2_GATE_PER_TOKEN ? 1 : d->g_mode == ARL2_GATE_PER_ELEMENT ? (size_t)d->H * d->D : (size_t)d->H;
    return (size_t)d->B * d->Lq * per_token * elem_bytes(d->g_dtype);
}
size_t table_bytes(const arl2_desc *d) { return (size_t)d->Lq * (d->D / 2) * sizeof(float); }
size_t wmap_bytes(const arl2_desc *d) { return (size_t)d->H * d->D * d->D * 2; }

// The fp32 kernels span up to 32 rows of [H][D] with 32-bit byte offsets, which this bound on H keeps below 2 GiB; the bound on
// B is part of the interface.
bool f32_sizes_ok(const arl2_desc *d) { return d->io_dtype != ARL2_F32 || (d->H <= 65535 && d->B <= 65535); }

// Checks everything that does not depend on which call is made.
arl2_status check_desc(const arl2_desc *d)
{
    if (d == nullptr) return fail(ARL2_ERR_INVALID_ARG, "desc is NULL");
    if (d->B < 1 || d->H < 1 || d->Lq < 1 || d->Lkv < 1)
        return fail(ARL2_ERR_INVALID_ARG, "B, H, Lq, Lkv must all be >= 1");
    if (d->io_dtype != ARL2_F32 && d->io_dtype != ARL2_BF16)
        return fail(ARL2_ERR_INVALID_ARG, "io_dtype is not an arl2_dtype");
    if (d->g_dtype != ARL2_F32 && d->g_dtype != ARL2_BF16)
        return fail(ARL2_ERR_INVALID_ARG, "g_dtype is not an arl2_dtype");
    if (d->g_mode != ARL2_GATE_PER_HEAD && d->g_mode != ARL2_GATE_PER_ELEMENT && d->g_mode != ARL2_GATE_PER_TOKEN)
        return fail(ARL2_ERR_INVALID_ARG, "g_mode is not an arl2_gate_mode");
    if (d->D != 64 && d->D != 128) return fail(ARL2_ERR_UNSUPPORTED, "D must be 64 or 128");
    if (!(d->sm_scale >= 0.f) || !(d->l2_eps >= 0.f))
        return fail(ARL2_ERR_INVALID_ARG, "sm_scale and l2_eps must be >= 0 (0 selects the default)");
    // element counts must stay addressable with the kernels' index arithmetic
    const double tokens = (double)d->B * (double)(d->Lq > d->Lkv ? d->Lq : d->Lkv);
    if (tokens > 2.0e9 || (double)d->B * d->H > 1.0e6)
        return fail(ARL2_ERR_UNSUPPORTED, "problem too large (B*L must stay below 2e9, B*H below 1e6)");
    return ARL2_OK;
}

// The kernels address one stream's [L][H][D] slice (and the feature map / gate projection the whole
// [B][L][H][D] array) with 32-bit byte offsets.
bool fits_32bit(double elems, int elem_bytes) { return elems * elem_bytes <= 2147483647.0; }

float resolved_eps(const arl2_desc *d) { return d->l2_eps > 0.f ? d->l2_eps : 1e-6f; }

// Workspace of the commits: one D x D partial sum per token split, of which the delta rule may take more than the plain rule.
// The fp32 commit reads and writes none of it; its size is part of the interface.
size_t commit_workspace_of(const arl2_desc *d, int nsplit)
{
    if (d->io_dtype == ARL2_BF16) return (size_t)d->B * d->H * nsplit * d->D * d->D * sizeof(float);
    return (size_t)d->B * d->Lq * d->H * sizeof(float);
}
size_t commit_workspace(const arl2_desc *d) { return commit_workspace_of(d, arl2::commit_delta_max_nsplit(d->B, d->H, d->Lq)); }
size_t commit_workspace_plain(const arl2_desc *d) { return commit_workspace_of(d, arl2::commit_nsplit(d->B, d->H, d->Lq)); }

// ---- paged 4-bit key/value cache

arl2_status check_kv_desc(const arl2_kv_desc *d)
{
    if (d == nullptr) return fail(ARL2_ERR_INVALID_ARG, "desc is NULL");
    if (d->B < 1 || d->Hkv < 1 || d->Lq < 1 || d->n_pages < 1 || d->max_pages < 1)
        return fail(ARL2_ERR_INVALID_ARG, "B, Hkv, Lq, n_pages and max_pages must all be >= 1");
    if (d->D != 64 && d->D != 128) return fail(ARL2_ERR_UNSUPPORTED, "D must be 64 or 128");
    if (d->page_size < 16 || d->page_size > 256 || (d->page_size & (d->page_size - 1)))
        return fail(ARL2_ERR_UNSUPPORTED, "page_size must be 16, 32, 64, 128 or 256");
    if ((double)d->max_pages * d->page_size > 1073741824.0)
        return fail(ARL2_ERR_UNSUPPORTED, "max_pages * page_size must stay below 2^30");
    if ((double)d->Hkv * d->page_size * (d->D + d->D / 16) > 4294967295.0) return fail(ARL2_ERR_UNSUPPORTED, "a page must stay below 4 GiB");
    if ((double)d->B * d->Lq > 2.0e9 || (double)d->B * d->Hkv > 1.0e6 || (double)d->n_pages * d->Hkv > 2.0e9)
        return fail(ARL2_ERR_UNSUPPORTED, "problem too large (B*Lq and n_pages*Hkv must stay below 2e9, B*Hkv below 1e6)");
    return ARL2_OK;
}

// The same with what attention needs beyond it.
arl2_status check_kv_attn_desc(const arl2_kv_desc *d)
{
    const arl2_status st = check_kv_desc(d);
    if (st != ARL2_OK) return st;
    if (d->H < 1 || d->H % d->Hkv) return fail(ARL2_ERR_INVALID_ARG, "H must be a positive multiple of Hkv");
    if (d->causal != 0 && d->causal != 1) return fail(ARL2_ERR_INVALID_ARG, "causal must be 0 or 1");
    // (the kernels multiply by sm_scale * log2(e), which is to be finite too)
    if (!(d->sm_scale >= 0.f) || d->sm_scale > 0x1p127f) return fail(ARL2_ERR_INVALID_ARG, "sm_scale must be >= 0 (0 selects the default) and at most 2^127");
    if ((double)d->B * d->H > 1.0e6 || (double)d->Lq * d->H > 2.0e9 || (double)d->B * d->H * d->Lq > 68719476736.0)
        return fail(ARL2_ERR_UNSUPPORTED, "problem too large (B*H must stay below 1e6, Lq*H below 2e9, B*H*Lq below 2^36)");
    return ARL2_OK;
}

arl2::KvPool kv_pool(const arl2_kv_desc *d)
{
    arl2::KvPool p;
    p.shift = 0;
    while ((1 << p.shift) < d->page_size) ++p.shift;
    p.heads = d->Hkv;
    p.n_pages = d->n_pages;
    p.max_pages = d->max_pages;
    return p;
}
size_t kv_rows_bytes(const arl2_kv_desc *d, int heads) { return (size_t)d->B * d->Lq * heads * d->D * 2; }
size_t kv_table_bytes(const arl2_kv_desc *d) { return (size_t)d->B * d->max_pages * sizeof(int32_t); }
arl2::KvAttnPlan kv_plan(const arl2_kv_desc *d) { return arl2::kv_attn_plan(d->B, d->Lq, d->H / d->Hkv, kv_pool(d), d->D); }

struct Range { const void *p; size_t n; };

// Does `out` share a byte with one of the inputs?
template <int N>
bool overlaps_any(Range out, const Range (&in)[N])
{
    for (const Range &r : in)
        if (overlaps(out.p, out.n, r.p, r.n)) return true;
    return false;
}
bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

// The kernels give a thread to 8 features of four tokens.
bool kv_rows_fit(const arl2_kv_desc *d) { return (double)d->B * d->Hkv * ((d->Lq + 15.0) / 16 + 1) * (d->D / 2) <= 2147483000.0; }

arl2::KvRowsArgs kv_rows_args(const arl2_kv_desc *d, const int32_t *table, const int32_t *start, const int32_t *count)
{
    arl2::KvRowsArgs a = {};
    a.table = table; a.start = start; a.count = count;
    a.pool = kv_pool(d);
    a.B = d->B; a.L = d->Lq; a.D = d->D;
    return a;
}

// Rows of zeros, those behind a sequence's end among them, are multiplied by 1 / sqrt(eps) and by decays of up to 2^64 that are taken out: with
// smaller epsilons by an infinity.
constexpr float kLeastEps = 1e-30f;
bool epsilon_ok(float eps) { return eps == 0.f || eps >= kLeastEps; }

// ---- the causal recurrence

arl2_status check_scan_desc(const arl2_scan_desc *d)
{
    if (d == nullptr) return fail(ARL2_ERR_INVALID_ARG, "desc is NULL");
    if (d->B < 1 || d->H < 1 || d->L < 1) return fail(ARL2_ERR_INVALID_ARG, "B, H and L must all be >= 1");
    if (d->D != 64 && d->D != 128) return fail(ARL2_ERR_UNSUPPORTED, "D must be 64 or 128");
    if (d->raw_rows != 0 && d->raw_rows != 1) return fail(ARL2_ERR_INVALID_ARG, "raw_rows must be 0 or 1");
    if (!epsilon_ok(d->l2_eps)) return fail(ARL2_ERR_INVALID_ARG, "l2_eps must be 0 (it selects the default) or >= 1e-30");
    // A stream's rows are addressed with 32-bit byte offsets, which may point 64 rows past the last.
    if ((double)d->L * d->H * d->D >= 1073741824.0 || 64.0 * d->H * d->D >= 1073741824.0)
        return fail(ARL2_ERR_UNSUPPORTED, "problem too large (L*H*D and 64*H*D must stay below 2^30)");
    if ((double)d->B * d->H > 1.0e6 || (double)d->B * d->H * ((d->L + 63.0) / 64) * 3 > 2147483000.0)
        return fail(ARL2_ERR_UNSUPPORTED, "problem too large (B*H must stay below 1e6, B*H*L below 2^35)");
    return ARL2_OK;
}
size_t scan_rows_bytes(const arl2_scan_desc *d) { return (size_t)d->B * d->L * d->H * d->D * 2; }
size_t scan_gate_bytes(const arl2_scan_desc *d) { return (size_t)d->B * d->L * d->H * sizeof(float); }
size_t scan_state_bytes(const arl2_scan_desc *d) { return (size_t)d->B * d->H * d->D * d->D * sizeof(float); }
arl2::ScanArgs scan_args(const arl2_scan_desc *d, const void *q, const void *k, const void *v, const float *log_alpha, const int32_t *seq_len, const float *S0)
{
    arl2::ScanArgs a = {};
    a.q = q; a.k = k; a.v = v; a.la = log_alpha; a.len = seq_len; a.S0 = S0;
    a.workspace = d->workspace;
    a.B = d->B; a.H = d->H; a.L = d->L; a.D = d->D;
    a.normalise = !d->raw_rows;
    a.eps = d->l2_eps > 0.f ? d->l2_eps : 1e-6f;
    return a;
}

// ---- rotary positions

arl2_status check_rope_desc(const arl2_rope_desc *d)
{
    if (d == nullptr) return fail(ARL2_ERR_INVALID_ARG, "desc is NULL");
    if (d->B < 1 || d->H < 1 || d->L < 1 || d->Hk < 0) return fail(ARL2_ERR_INVALID_ARG, "B, H and L must all be >= 1, Hk >= 0");
    if (d->D != 64 && d->D != 128) return fail(ARL2_ERR_UNSUPPORTED, "D must be 64 or 128");
    if (d->io_dtype != ARL2_F32 && d->io_dtype != ARL2_BF16) return fail(ARL2_ERR_INVALID_ARG, "io_dtype is not an arl2_dtype");
    if (d->norm != ARL2_NORM_NONE && d->norm != ARL2_NORM_HEAD && d->norm != ARL2_NORM_ROW) return fail(ARL2_ERR_INVALID_ARG, "norm is not an arl2_norm_mode");
    if ((d->halves != 0 && d->halves != 1) || (d->pos_per_stream != 0 && d->pos_per_stream != 1))
        return fail(ARL2_ERR_INVALID_ARG, "halves and pos_per_stream must be 0 or 1");
    if (d->n_axes < 1 || d->n_axes > 4) return fail(ARL2_ERR_INVALID_ARG, "n_axes must be 1 to 4");
    long long pairs = 0;
    for (int a = 0; a < d->n_axes; ++a) {
        if (d->axis_pairs[a] < 1) return fail(ARL2_ERR_INVALID_ARG, "axis_pairs must be >= 1");
        if (!(d->theta[a] >= 0.0) || d->theta[a] > 1e30 || (d->theta[a] > 0.0 && d->theta[a] < 1e-3))
            return fail(ARL2_ERR_INVALID_ARG, "theta must lie in [1e-3, 1e30] (0 selects the default)");
        pairs += d->axis_pairs[a];
    }
    if (pairs > d->D / 2) return fail(ARL2_ERR_INVALID_ARG, "axis_pairs must be D / 2 at most together");
    if (!epsilon_ok(d->norm_eps)) return fail(ARL2_ERR_INVALID_ARG, "norm_eps must be 0 (it selects the default) or >= 1e-30");
    if (((double)d->H + d->Hk) * (d->D / 16) > arl2::kRopeMostUnits) return fail(ARL2_ERR_UNSUPPORTED, "(H + Hk) * D must be 24576 at most");
    if ((double)d->B * d->L > 2.0e9) return fail(ARL2_ERR_UNSUPPORTED, "problem too large (B*L must stay below 2e9)");
    return ARL2_OK;
}
size_t rope_rows_bytes(const arl2_rope_desc *d, int heads) { return (size_t)d->B * d->L * heads * d->D * elem_bytes(d->io_dtype); }
size_t rope_weight_bytes(const arl2_rope_desc *d, int heads) { return (size_t)(d->norm == ARL2_NORM_HEAD ? 1 : heads) * d->D * elem_bytes(d->io_dtype); }
size_t rope_pos_bytes(const arl2_rope_desc *d) { return (size_t)(d->pos_per_stream ? d->B : 1) * d->L * d->n_axes * sizeof(int32_t); }

// What both directions check; `keys`: the arrays of keys' rows, which are there exactly where there are keys.
arl2_status check_rope_call(const arl2_rope_desc *d, std::initializer_list<const void *> keys, const void *wq, const void *wk, const int32_t *pos, const int32_t *seq_len)
{
    const arl2_status st = check_rope_desc(d);
    if (st != ARL2_OK) return st;
    for (const void *k : keys)
        if ((k != nullptr) != (d->Hk > 0)) return fail(ARL2_ERR_INVALID_ARG, "keys must be given exactly where Hk > 0");
    if (pos == nullptr) return fail(ARL2_ERR_INVALID_ARG, "pos must not be NULL");
    if ((wq || wk) && d->norm == ARL2_NORM_NONE) return fail(ARL2_ERR_INVALID_ARG, "rows without a norm have no weights");
    if (wk && d->Hk == 0) return fail(ARL2_ERR_INVALID_ARG, "wk must be NULL where there are no keys");
    if (!aligned16(wq) || !aligned16(wk)) return fail(ARL2_ERR_INVALID_ARG, "wq and wk must be 16-byte aligned");
    if (!aligned4(pos) || !aligned4(seq_len)) return fail(ARL2_ERR_INVALID_ARG, "pos and seq_len must be 4-byte aligned");
    return ARL2_OK;
}

arl2::RopeArgs rope_args(const arl2_rope_desc *d, const void *q, const void *k, const void *wq, const void *wk, const int32_t *pos, const int32_t *seq_len)
{
    arl2::RopeArgs a = {};
    a.x[0] = q; a.x[1] = k; a.w[0] = wq; a.w[1] = wk; a.pos = pos; a.len = seq_len;
    a.B = d->B; a.L = d->L; a.D = d->D; a.heads[0] = d->H; a.heads[1] = d->Hk;
    a.axes = d->n_axes; a.pos_per_stream = d->pos_per_stream; a.halves = d->halves;
    a.norm = d->norm == ARL2_NORM_NONE ? arl2::kNormNone : d->norm == ARL2_NORM_HEAD ? arl2::kNormHead : arl2::kNormRow;
    a.f32 = d->io_dtype == ARL2_F32;
    a.eps = d->norm_eps > 0.f ? d->norm_eps : 1e-6f;
    for (int x = 0; x < d->n_axes; ++x) {
        const double theta = d->theta[x] > 0.0 ? d->theta[x] : 10000.0;
        for (int i = 0; i < d->axis_pairs[x]; ++i, ++a.pairs) {
            a.axis[a.pairs] = (uint8_t)x;
            a.turns[a.pairs] = std::pow(theta, -(double)i / d->axis_pairs[x]) * 0.15915494309189535;      // 1 / 2 pi
        }
    }
    return a;
}

}  // namespace

extern "C" {

size_t arl2_workspace_bytes(const arl2_desc *desc)
{
    if (check_desc(desc) != ARL2_OK) return 0;
    return commit_workspace(desc);
}

arl2_status arl2_hybrid_attn_fwd_ex(const arl2_desc *desc, const void *q, const void *k, const void *v,
                                    const void *q_lin, const float *S, const void *g, void *out)
{
    arl2_status st = check_desc(desc);
    if (st != ARL2_OK) return st;
    if (!q || !k || !v || !out) return fail(ARL2_ERR_INVALID_ARG, "q, k, v and out must not be NULL");
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(S) || !aligned16(q_lin))
        return fail(ARL2_ERR_INVALID_ARG, "q, k, v, q_lin, S and out must be 16-byte aligned");
    if (g && (reinterpret_cast<uintptr_t>(g) & 3u))
        return fail(ARL2_ERR_INVALID_ARG, "g must be 4-byte aligned");
    if (g && desc->g_mode == ARL2_GATE_PER_ELEMENT && !aligned16(g))
        return fail(ARL2_ERR_INVALID_ARG, "an element-wise g must be 16-byte aligned");
    if (S != nullptr && desc->Lkv != desc->Lq)
        return fail(ARL2_ERR_INVALID_ARG, "Lkv must equal Lq when a state is given");
    if (!f32_sizes_ok(desc)) return fail(ARL2_ERR_UNSUPPORTED, "fp32 inputs: H and B must stay below 65536");
    if (desc->io_dtype == ARL2_BF16 && !fits_32bit(((double)desc->Lkv + 256.0) * desc->H * desc->D, 2))
        return fail(ARL2_ERR_UNSUPPORTED, "one stream's k (or v) must stay below 2 GiB");
    {
        const size_t nq = q_bytes(desc), nkv = kv_bytes(desc);
        if (overlaps(out, nq, q, nq) || overlaps(out, nq, k, nkv) || overlaps(out, nq, v, nkv) || overlaps(out, nq, q_lin, nq) ||
            overlaps(out, nq, S, state_bytes(desc)) || overlaps(out, nq, g, g_bytes(desc)))
            return fail(ARL2_ERR_INVALID_ARG, "out must not overlap an input");
    }

    arl2::FwdArgs a;
    a.q = q; a.k = k; a.v = v; a.S = S; a.g = (S != nullptr) ? g : nullptr; a.out = out;
    a.q_lin = (S != nullptr) ? q_lin : nullptr;
    a.xq = nullptr; a.Wq = nullptr; a.cs = nullptr; a.sn = nullptr;
    a.B = desc->B; a.H = desc->H; a.Lq = desc->Lq; a.Lkv = desc->Lkv; a.D = desc->D;
    a.g_is_bf16 = desc->g_dtype == ARL2_BF16;
    a.g_per_element = desc->g_mode == ARL2_GATE_PER_ELEMENT;
    a.g_per_token = desc->g_mode == ARL2_GATE_PER_TOKEN;
    a.sm_scale = desc->sm_scale > 0.f ? desc->sm_scale : 1.0f / sqrtf((float)desc->D);
    a.l2_eps = resolved_eps(desc);
    hipStream_t stream = reinterpret_cast<hipStream_t>(desc->stream);
    const hipError_t e = desc->io_dtype == ARL2_BF16 ? arl2::launch_fwd_bf16(a, stream)
                                                     : arl2::launch_fwd_f32(a, stream);
    if (e != hipSuccess) return fail(ARL2_ERR_DEVICE, "fwd launch failed: %s", hipGetErrorString(e));
    return ARL2_OK;
}

arl2_status arl2_hybrid_attn_fwd(const arl2_desc *desc, const void *q, const void *k, const void *v,
                                 const float *S, const void *g, void *out)
{
    return arl2_hybrid_attn_fwd_ex(desc, q, k, v, nullptr, S, g, out);
}

arl2_status arl2_hybrid_attn_fwd_fm(const arl2_desc *desc, const void *q, const void *k, const void *v,
                                    const void *xq, const void *Wq, const float *rope_cos, const float *rope_sin,
                                    const float *S, const void *g, void *out)
{
    arl2_status st = check_desc(desc);
    if (st != ARL2_OK) return st;
    if (!q || !k || !v || !out || !xq || !Wq || !S)
        return fail(ARL2_ERR_INVALID_ARG, "q, k, v, xq, Wq, S and out must not be NULL");
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(S) || !aligned16(xq) || !aligned16(Wq))
        return fail(ARL2_ERR_INVALID_ARG, "q, k, v, xq, Wq, S and out must be 16-byte aligned");
    if ((rope_cos == nullptr) != (rope_sin == nullptr))
        return fail(ARL2_ERR_INVALID_ARG, "rope_cos and rope_sin must be given together");
    if ((reinterpret_cast<uintptr_t>(rope_cos) & 7u) || (reinterpret_cast<uintptr_t>(rope_sin) & 7u))
        return fail(ARL2_ERR_INVALID_ARG, "rope_cos and rope_sin must be 8-byte aligned");
    if (g && (reinterpret_cast<uintptr_t>(g) & 3u)) return fail(ARL2_ERR_INVALID_ARG, "g must be 4-byte aligned");
    if (g && desc->g_mode == ARL2_GATE_PER_ELEMENT && !aligned16(g))
        return fail(ARL2_ERR_INVALID_ARG, "an element-wise g must be 16-byte aligned");
    if (desc->Lkv != desc->Lq) return fail(ARL2_ERR_INVALID_ARG, "Lkv must equal Lq when a state is given");
    if (desc->io_dtype != ARL2_BF16) return fail(ARL2_ERR_UNSUPPORTED, "arl2_hybrid_attn_fwd_fm takes bf16 inputs only");
    if (!fits_32bit(((double)desc->Lkv + 256.0) * desc->H * desc->D, 2))
        return fail(ARL2_ERR_UNSUPPORTED, "one stream's k (or v) must stay below 2 GiB");
    {
        const size_t nq = q_bytes(desc), nkv = kv_bytes(desc);
        if (overlaps(out, nq, q, nq) || overlaps(out, nq, k, nkv) || overlaps(out, nq, v, nkv) || overlaps(out, nq, xq, nq) ||
            overlaps(out, nq, Wq, wmap_bytes(desc)) || overlaps(out, nq, S, state_bytes(desc)) || overlaps(out, nq, g, g_bytes(desc)) ||
            overlaps(out, nq, rope_cos, table_bytes(desc)) || overlaps(out, nq, rope_sin, table_bytes(desc)))
            return fail(ARL2_ERR_INVALID_ARG, "out must not overlap an input");
    }

    arl2::FwdArgs a;
    a.q = q; a.k = k; a.v = v; a.S = S; a.g = g; a.out = out; a.q_lin = nullptr;
    a.xq = xq; a.Wq = Wq; a.cs = rope_cos; a.sn = rope_sin;
    a.B = desc->B; a.H = desc->H; a.Lq = desc->Lq; a.Lkv = desc->Lkv; a.D = desc->D;
    a.g_is_bf16 = desc->g_dtype == ARL2_BF16;
    a.g_per_element = desc->g_mode == ARL2_GATE_PER_ELEMENT;
    a.g_per_token = desc->g_mode == ARL2_GATE_PER_TOKEN;
    a.sm_scale = desc->sm_scale > 0.f ? desc->sm_scale : 1.0f / sqrtf((float)desc->D);
    a.l2_eps = resolved_eps(desc);
    const hipError_t e = arl2::launch_fwd_bf16(a, reinterpret_cast<hipStream_t>(desc->stream));
    if (e != hipSuccess) return fail(ARL2_ERR_DEVICE, "fwd launch failed: %s", hipGetErrorString(e));
    return ARL2_OK;
}

arl2_status arl2_feature_map(const arl2_desc *desc, const void *x, const void *W,
                             const float *rope_cos, const float *rope_sin, void *y)
{
    arl2_status st = check_desc(desc);
    if (st != ARL2_OK) return st;
    if (!x || !W || !y) return fail(ARL2_ERR_INVALID_ARG, "x, W and y must not be NULL");
    if (!aligned16(x) || !aligned16(W) || !aligned16(y))
        return fail(ARL2_ERR_INVALID_ARG, "x, W and y must be 16-byte aligned");
    if ((rope_cos == nullptr) != (rope_sin == nullptr))
        return fail(ARL2_ERR_INVALID_ARG, "rope_cos and rope_sin must be given together");
    if ((reinterpret_cast<uintptr_t>(rope_cos) & 7u) || (reinterpret_cast<uintptr_t>(rope_sin) & 7u))
        return fail(ARL2_ERR_INVALID_ARG, "rope_cos and rope_sin must be 8-byte aligned");
    if (desc->io_dtype != ARL2_BF16) return fail(ARL2_ERR_UNSUPPORTED, "arl2_feature_map takes bf16 x, W only");
    if (!fits_32bit((double)desc->B * desc->Lq * desc->H * desc->D, 2))
        return fail(ARL2_ERR_UNSUPPORTED, "x must stay below 2 GiB");
    {
        const size_t nx = q_bytes(desc);
        if (overlaps(y, nx, x, nx) || overlaps(y, nx, W, wmap_bytes(desc)) || overlaps(y, nx, rope_cos, table_bytes(desc)) ||
            overlaps(y, nx, rope_sin, table_bytes(desc)))
            return fail(ARL2_ERR_INVALID_ARG, "y must not overlap an input");
    }

    arl2::FmapArgs a;
    a.x = x; a.W = W; a.cs = rope_cos; a.sn = rope_sin; a.y = y;
    a.B = desc->B; a.H = desc->H; a.L = desc->Lq; a.D = desc->D;
    const hipError_t e = arl2::launch_feature_map_bf16(a, reinterpret_cast<hipStream_t>(desc->stream));
    if (e != hipSuccess) return fail(ARL2_ERR_DEVICE, "feature map launch failed: %s", hipGetErrorString(e));
    return ARL2_OK;
}

arl2_status arl2_gate_proj(const arl2_desc *desc, const void *x, const void *Wg, void *g)
{
    arl2_status st = check_desc(desc);
    if (st != ARL2_OK) return st;
    if (!x || !Wg || !g) return fail(ARL2_ERR_INVALID_ARG, "x, Wg and g must not be NULL");
    if (!aligned16(x) || !aligned16(Wg)) return fail(ARL2_ERR_INVALID_ARG, "x and Wg must be 16-byte aligned");
    if (reinterpret_cast<uintptr_t>(g) & 3u) return fail(ARL2_ERR_INVALID_ARG, "g must be 4-byte aligned");
    if (desc->io_dtype != ARL2_BF16) return fail(ARL2_ERR_UNSUPPORTED, "arl2_gate_proj takes bf16 x, Wg only");
    if (!fits_32bit((double)desc->B * desc->Lq * desc->H * desc->D, 2))
        return fail(ARL2_ERR_UNSUPPORTED, "x must stay below 2 GiB");
    const int n_out = desc->g_mode == ARL2_GATE_PER_TOKEN ? 1 : desc->g_mode == ARL2_GATE_PER_ELEMENT ? desc->H * desc->D : desc->H;
    if (!fits_32bit((double)n_out * desc->H * desc->D, 2))
        return fail(ARL2_ERR_UNSUPPORTED, "Wg must stay below 2 GiB");
    {
        const size_t nx = (size_t)desc->B * desc->Lq * desc->H * desc->D * 2;
        const size_t rows = desc->g_mode == ARL2_GATE_PER_TOKEN ? 1 : desc->g_mode == ARL2_GATE_PER_ELEMENT ? (size_t)desc->H * desc->D : (size_t)desc->H;
        if (overlaps(g, g_bytes(desc), x, nx) || overlaps(g, g_bytes(desc), Wg, rows * desc->H * desc->D * 2))
            return fail(ARL2_ERR_INVALID_ARG, "g must not overlap an input");
    }

    arl2::GateArgs a;
    a.x = x; a.Wg = Wg; a.g = g;
    a.B = desc->B; a.H = desc->H; a.L = desc->Lq; a.dm = desc->H * desc->D;
    a.n_out = n_out;
    a.g_is_bf16 = desc->g_dtype == ARL2_BF16;
    const hipError_t e = arl2::launch_gate_proj_bf16(a, reinterpret_cast<hipStream_t>(desc->stream));
    if (e != hipSuccess) return fail(ARL2_ERR_DEVICE, "gate projection launch failed: %s", hipGetErrorString(e));
    return ARL2_OK;
}

static arl2_status commit_common(const arl2_desc *desc, const void *k, const void *v, const float *gate,
                                 const float *beta, bool delta, float *S)
{
    arl2_status st = check_desc(desc);
    if (st != ARL2_OK) return st;
    if (!k || !v || !gate || !S || (delta && !beta))
        return fail(ARL2_ERR_INVALID_ARG, "k, v, gate%s and S must not be NULL", delta ? ", beta" : "");
    if (!aligned16(k) || !aligned16(v) || !aligned16(S))
        return fail(ARL2_ERR_INVALID_ARG, "k, v and S must be 16-byte aligned");
    if ((reinterpret_cast<uintptr_t>(gate) & 3u) || (reinterpret_cast<uintptr_t>(beta) & 3u))
        return fail(ARL2_ERR_INVALID_ARG, "gate and beta must be 4-byte aligned");
    if (desc->Lkv != desc->Lq) return fail(ARL2_ERR_INVALID_ARG, "Lkv must equal Lq in a state commit");
    if (delta && desc->io_dtype != ARL2_BF16)
        return fail(ARL2_ERR_UNSUPPORTED, "arl2_state_commit_delta takes bf16 k, v only");
    if (desc->io_dtype == ARL2_BF16 && !fits_32bit(((double)desc->Lq + 256.0) * desc->H * desc->D, 2))
        return fail(ARL2_ERR_UNSUPPORTED, "one stream's k (or v) must stay below 2 GiB");
    const size_t need = delta ? commit_workspace(desc) : commit_workspace_plain(desc);
    if (desc->workspace == nullptr || desc->workspace_bytes < need)
        return fail(ARL2_ERR_WORKSPACE, "workspace is NULL or smaller than arl2_workspace_bytes()");
    if (!aligned16(desc->workspace)) return fail(ARL2_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    if (!f32_sizes_ok(desc)) return fail(ARL2_ERR_UNSUPPORTED, "fp32 inputs: H and B must stay below 65536");
    {
        const size_t ns = state_bytes(desc), nkv = kv_bytes(desc), ngate = (size_t)desc->B * desc->H * sizeof(float);
        if (overlaps(S, ns, k, nkv) || overlaps(S, ns, v, nkv) || overlaps(S, ns, gate, ngate) || overlaps(S, ns, beta, ngate) ||
            overlaps(S, ns, desc->workspace, need))
            return fail(ARL2_ERR_INVALID_ARG, "S must not overlap k, v, the gates or the workspace");
        if (overlaps(desc->workspace, need, k, nkv) || overlaps(desc->workspace, need, v, nkv) ||
            overlaps(desc->workspace, need, gate, ngate) || overlaps(desc->workspace, need, beta, ngate))
            return fail(ARL2_ERR_INVALID_ARG, "the workspace must not overlap an input");
    }

    arl2::CommitArgs a;
    a.k = k; a.v = v; a.gate = gate; a.beta = delta ? beta : nullptr; a.S = S; a.workspace = desc->workspace;
    a.B = desc->B; a.H = desc->H; a.L = desc->Lq; a.D = desc->D;
    a.nsplit = delta ? arl2::commit_delta_max_nsplit(desc->B, desc->H, desc->Lq) : arl2::commit_nsplit(desc->B, desc->H, desc->Lq);
    a.l2_eps = resolved_eps(desc);
    hipStream_t stream = reinterpret_cast<hipStream_t>(desc->stream);
    const hipError_t e = desc->io_dtype == ARL2_BF16 ? arl2::launch_commit_bf16(a, stream)
                                                     : arl2::launch_commit_f32(a, stream);
    if (e != hipSuccess) return fail(ARL2_ERR_DEVICE, "commit launch failed: %s", hipGetErrorString(e));
    return ARL2_OK;
}

arl2_status arl2_state_commit(const arl2_desc *desc, const void *k, const void *v, const float *gate, float *S)
{
    return commit_common(desc, k, v, gate, nullptr, false, S);
}

arl2_status arl2_state_commit_delta(const arl2_desc *desc, const void *k, const void *v, const float *gate,
                                    const float *beta, float *S)
{
    return commit_common(desc, k, v, gate, beta, true, S);
}

arl2_status arl2_state_commit_fm(const arl2_desc *desc, const void *xk, const void *Wk,
                                 const float *rope_cos, const float *rope_sin,
                                 const void *xv, const void *Wv, const float *gate, float *S)
{
    arl2_status st = check_desc(desc);
    if (st != ARL2_OK) return st;
    if (!xk || !Wk || !xv || !Wv || !gate || !S)
        return fail(ARL2_ERR_INVALID_ARG, "xk, Wk, xv, Wv, gate and S must not be NULL");
    if (!aligned16(xk) || !aligned16(Wk) || !aligned16(xv) || !aligned16(Wv) || !aligned16(S))
        return fail(ARL2_ERR_INVALID_ARG, "xk, Wk, xv, Wv and S must be 16-byte aligned");
    if ((rope_cos == nullptr) != (rope_sin == nullptr))
        return fail(ARL2_ERR_INVALID_ARG, "rope_cos and rope_sin must be given together");
    if ((reinterpret_cast<uintptr_t>(rope_cos) & 7u) || (reinterpret_cast<uintptr_t>(rope_sin) & 7u))
        return fail(ARL2_ERR_INVALID_ARG, "rope_cos and rope_sin must be 8-byte aligned");
    if (reinterpret_cast<uintptr_t>(gate) & 3u) return fail(ARL2_ERR_INVALID_ARG, "gate must be 4-byte aligned");
    if (desc->Lkv != desc->Lq) return fail(ARL2_ERR_INVALID_ARG, "Lkv must equal Lq in a state commit");
    if (desc->io_dtype != ARL2_BF16) return fail(ARL2_ERR_UNSUPPORTED, "arl2_state_commit_fm takes bf16 inputs only");
    if (!fits_32bit(((double)desc->Lq + 256.0) * desc->H * desc->D, 2))
        return fail(ARL2_ERR_UNSUPPORTED, "one stream's xk (or xv) must stay below 2 GiB");
    const size_t need = commit_workspace_plain(desc);
    if (desc->workspace == nullptr || desc->workspace_bytes < need)
        return fail(ARL2_ERR_WORKSPACE, "workspace is NULL or smaller than arl2_workspace_bytes()");
    if (!aligned16(desc->workspace)) return fail(ARL2_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    {
        const size_t ns = state_bytes(desc), nx = kv_bytes(desc), ngate = (size_t)desc->B * desc->H * sizeof(float);
        const size_t nw = wmap_bytes(desc), nt = table_bytes(desc);
        const void *in[] = {xk, xv, Wk, Wv, rope_cos, rope_sin, gate};
        const size_t nb[] = {nx, nx, nw, nw, nt, nt, ngate};
        for (int i = 0; i < 7; ++i) {
            if (overlaps(S, ns, in[i], nb[i])) return fail(ARL2_ERR_INVALID_ARG, "S must not overlap an input");
            if (overlaps(desc->workspace, need, in[i], nb[i]))
                return fail(ARL2_ERR_INVALID_ARG, "the workspace must not overlap an input");
        }
        if (overlaps(S, ns, desc->workspace, need)) return fail(ARL2_ERR_INVALID_ARG, "S must not overlap the workspace");
    }

    arl2::CommitFmArgs a;
    a.xk = xk; a.xv = xv; a.Wk = Wk; a.Wv = Wv; a.cs = rope_cos; a.sn = rope_sin;
    a.gate = gate; a.S = S; a.workspace = desc->workspace;
    a.B = desc->B; a.H = desc->H; a.L = desc->Lq; a.D = desc->D;
    a.nsplit = arl2::commit_nsplit(desc->B, desc->H, desc->Lq);
    a.l2_eps = resolved_eps(desc);
    const hipError_t e = arl2::launch_commit_fm_bf16(a, reinterpret_cast<hipStream_t>(desc->stream));
    if (e != hipSuccess) return fail(ARL2_ERR_DEVICE, "commit launch failed: %s", hipGetErrorString(e));
    return ARL2_OK;
}

size_t arl2_gdn_workspace_bytes(const arl2_desc *desc)
{
    if (check_desc(desc) != ARL2_OK) return 0;
    return arl2::gdn_workspace_bytes(desc->B, desc->H, desc->Lq, desc->D);
}

arl2_status arl2_state_commit_gdn(const arl2_desc *desc, const void *k, const void *v, const float *alpha,
                                  const float *beta, float *S)
{
    arl2_status st = check_desc(desc);
    if (st != ARL2_OK) return st;
    if (!k || !v || !alpha || !beta || !S)
        return fail(ARL2_ERR_INVALID_ARG, "k, v, alpha, beta and S must not be NULL");
    if (!aligned16(k) || !aligned16(v) || !aligned16(S))
        return fail(ARL2_ERR_INVALID_ARG, "k, v and S must be 16-byte aligned");
    if ((reinterpret_cast<uintptr_t>(alpha) & 3u) || (reinterpret_cast<uintptr_t>(beta) & 3u))
        return fail(ARL2_ERR_INVALID_ARG, "alpha and beta must be 4-byte aligned");
    if (desc->Lkv != desc->Lq) return fail(ARL2_ERR_INVALID_ARG, "Lkv must equal Lq in a state commit");
    if (desc->io_dtype != ARL2_BF16)
        return fail(ARL2_ERR_UNSUPPORTED, "arl2_state_commit_gdn takes bf16 k, v only");
    if (!fits_32bit(((double)desc->Lq + 256.0) * desc->H * desc->D, 2))
        return fail(ARL2_ERR_UNSUPPORTED, "one stream's k (or v) must stay below 2 GiB");
    const size_t need = arl2::gdn_workspace_bytes(desc->B, desc->H, desc->Lq, desc->D);
    if (desc->workspace == nullptr || desc->workspace_bytes < need)
        return fail(ARL2_ERR_WORKSPACE, "workspace is NULL or smaller than arl2_gdn_workspace_bytes()");
    if (!aligned16(desc->workspace)) return fail(ARL2_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    {
        const size_t ns = state_bytes(desc), nkv = kv_bytes(desc), ngate = (size_t)desc->B * desc->Lq * desc->H * sizeof(float);
        if (overlaps(S, ns, k, nkv) || overlaps(S, ns, v, nkv) || overlaps(S, ns, alpha, ngate) || overlaps(S, ns, beta, ngate) ||
            overlaps(S, ns, desc->workspace, need))
            return fail(ARL2_ERR_INVALID_ARG, "S must not overlap k, v, the gates or the workspace");
        if (overlaps(desc->workspace, need, k, nkv) || overlaps(desc->workspace, need, v, nkv) ||
            overlaps(desc->workspace, need, alpha, ngate) || overlaps(desc->workspace, need, beta, ngate))
            return fail(ARL2_ERR_INVALID_ARG, "the workspace must not overlap an input");
    }

    arl2::GdnArgs a;
    a.k = k; a.v = v; a.alpha = alpha; a.beta = beta; a.S = S; a.workspace = desc->workspace;
    a.B = desc->B; a.H = desc->H; a.L = desc->Lq; a.D = desc->D;
    a.l2_eps = resolved_eps(desc);
    const hipError_t e = arl2::launch_commit_gdn_bf16(a, reinterpret_cast<hipStream_t>(desc->stream));
    if (e != hipSuccess) return fail(ARL2_ERR_DEVICE, "gdn commit launch failed: %s", hipGetErrorString(e));
    return ARL2_OK;
}

// ---- entry point that allocates nothing ---------------------------------------------------------------
// The commit's token-split partial sums go to a fixed device array instead of a caller's workspace.  Every
// GPU the library runs on holds its own copy of the array (at its own address) until the process ends.
constexpr size_t kStaticScratchBytes = (size_t)16 << 20;
static __device__ __align__(256) unsigned char scratch[kStaticScratchBytes];

namespace {

constexpr int kMaxDevices = 64;
std::atomic<void *> g_scratch_ptr[kMaxDevices];   // device address of `scratch` per device, looked up once

// The array's name is a host-side stand-in, not a device address: the address on the current device comes
// from the runtime, once per device, and only that pointer is ever handed to a kernel.
arl2_status static_scratch(void **out)
{
    int dev = -1;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return fail(ARL2_ERR_DEVICE, "hipGetDevice failed: %s", hipGetErrorString(e));
    if (dev < 0 || dev >= kMaxDevices) return fail(ARL2_ERR_UNSUPPORTED, "device ordinal beyond the static scratch table");
    void *p = g_scratch_ptr[dev].load(std::memory_order_acquire);
    if (p == nullptr) {
        e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
        if (e != hipSuccess || p == nullptr)
            return fail(ARL2_ERR_DEVICE, "hipGetSymbolAddress(scratch) failed: %s", hipGetErrorString(e));
        g_scratch_ptr[dev].store(p, std::memory_order_release);   // every thread would look up the same address
    }
    *out = p;
    return ARL2_OK;
}

}  // namespace

size_t arl2_static_scratch_bytes(void) { return kStaticScratchBytes; }

arl2_status arl2_state_commit_static(const arl2_desc *desc, const void *k, const void *v, const float *gate, float *S)
{
    arl2_status st = check_desc(desc);
    if (st != ARL2_OK) return st;
    const size_t need = commit_workspace_plain(desc);
    if (need > kStaticScratchBytes)
        return fail(ARL2_ERR_UNSUPPORTED, "problem needs more scratch than the static array holds (arl2_static_scratch_bytes)");
    void *ptr = nullptr;
    st = static_scratch(&ptr);
    if (st != ARL2_OK) return st;
    arl2_desc d = *desc;
    d.workspace = ptr;
    d.workspace_bytes = kStaticScratchBytes;
    return commit_common(&d, k, v, gate, nullptr, false, S);
}

// ---- paged 4-bit key/value cache ----------------------------------------------------------------------
size_t arl2_kv_cache_bytes(const arl2_kv_desc *desc)
{
    return check_kv_desc(desc) == ARL2_OK ? arl2::kv_pool_bytes(kv_pool(desc), desc->D) : 0;
}

size_t arl2_kv_workspace_bytes(const arl2_kv_desc *desc)
{
    return check_kv_attn_desc(desc) == ARL2_OK ? kv_plan(desc).bytes : 0;
}

arl2_status arl2_kv_append(const arl2_kv_desc *desc, const void *k, const void *v, const float *rope_cos, const float *rope_sin,
                           const int32_t *block_table, const int32_t *start, const int32_t *count, void *cache)
{
    const arl2_status st = check_kv_desc(desc);
    if (st != ARL2_OK) return st;
    if (!k || !v || !block_table || !start || !cache)
        return fail(ARL2_ERR_INVALID_ARG, "k, v, block_table, start and cache must not be NULL");
    if ((rope_cos == nullptr) != (rope_sin == nullptr))
        return fail(ARL2_ERR_INVALID_ARG, "rope_cos and rope_sin must be given together");
    if (!aligned16(k) || !aligned16(v) || !aligned16(cache) || !aligned16(rope_cos) || !aligned16(rope_sin))
        return fail(ARL2_ERR_INVALID_ARG, "k, v, cache, rope_cos and rope_sin must be 16-byte aligned");
    if (!aligned4(block_table) || !aligned4(start) || !aligned4(count))
        return fail(ARL2_ERR_INVALID_ARG, "block_table, start and count must be 4-byte aligned");
    if (!kv_rows_fit(desc)) return fail(ARL2_ERR_UNSUPPORTED, "problem too large (B * Hkv * Lq * D must stay below 2^36)");
    const size_t rows = kv_rows_bytes(desc, desc->Hkv), lens = desc->B * sizeof(int32_t);
    const size_t rope = (size_t)desc->max_pages * desc->page_size * (desc->D / 2) * sizeof(float);
    const Range in[] = {{k, rows}, {v, rows}, {rope_cos, rope}, {rope_sin, rope}, {block_table, kv_table_bytes(desc)}, {start, lens}, {count, lens}};
    if (overlaps_any({cache, arl2_kv_cache_bytes(desc)}, in)) return fail(ARL2_ERR_INVALID_ARG, "the cache must not overlap an input");

    arl2::KvRowsArgs a = kv_rows_args(desc, block_table, start, count);
    a.k = k; a.v = v; a.cs = rope_cos; a.sn = rope_sin; a.cache = cache;
    const hipError_t e = arl2::launch_kv_append(a, reinterpret_cast<hipStream_t>(desc->stream));
    if (e != hipSuccess) return fail(ARL2_ERR_DEVICE, "append launch failed: %s", hipGetErrorString(e));
    return ARL2_OK;
}

arl2_status arl2_kv_read(const arl2_kv_desc *desc, const void *cache, const int32_t *block_table, const int32_t *start, const int32_t *count,
                         void *k, void *v)
{
    const arl2_status st = check_kv_desc(desc);
    if (st != ARL2_OK) return st;
    if (!k || !v || !block_table || !start || !cache)
        return fail(ARL2_ERR_INVALID_ARG, "cache, block_table, start, k and v must not be NULL");
    if (!aligned16(k) || !aligned16(v) || !aligned16(cache)) return fail(ARL2_ERR_INVALID_ARG, "cache, k and v must be 16-byte aligned");
    if (!aligned4(block_table) || !aligned4(start) || !aligned4(count))
        return fail(ARL2_ERR_INVALID_ARG, "block_table, start and count must be 4-byte aligned");
    if (!kv_rows_fit(desc)) return fail(ARL2_ERR_UNSUPPORTED, "problem too large (B * Hkv * Lq * D must stay below 2^36)");
    const size_t rows = kv_rows_bytes(desc, desc->Hkv), lens = desc->B * sizeof(int32_t);
    const Range in[] = {{cache, arl2_kv_cache_bytes(desc)}, {block_table, kv_table_bytes(desc)}, {start, lens}, {count, lens}};
    if (overlaps_any({k, rows}, in) || overlaps_any({v, rows}, in) || overlaps(k, rows, v, rows))
        return fail(ARL2_ERR_INVALID_ARG, "k and v must overlap neither an input nor each other");

    arl2::KvRowsArgs a = kv_rows_args(desc, block_table, start, count);
    a.cache = const_cast<void *>(cache); a.k_out = k; a.v_out = v;
    const hipError_t e = arl2::launch_kv_read(a, reinterpret_cast<hipStream_t>(desc->stream));
    if (e != hipSuccess) return fail(ARL2_ERR_DEVICE, "read launch failed: %s", hipGetErrorString(e));
    return ARL2_OK;
}

arl2_status arl2_kv_attn_fwd(const arl2_kv_desc *desc, const void *q, const void *cache, const int32_t *block_table, const int32_t *kv_len,
                             const int32_t *q_len, void *out)
{
    const arl2_status st = check_kv_attn_desc(desc);
    if (st != ARL2_OK) return st;
    if (!q || !cache || !block_table || !kv_len || !out)
        return fail(ARL2_ERR_INVALID_ARG, "q, cache, block_table, kv_len and out must not be NULL");
    if (!aligned16(q) || !aligned16(cache) || !aligned16(out)) return fail(ARL2_ERR_INVALID_ARG, "q, cache and out must be 16-byte aligned");
    if (!aligned4(block_table) || !aligned4(kv_len) || !aligned4(q_len))
        return fail(ARL2_ERR_INVALID_ARG, "block_table, kv_len and q_len must be 4-byte aligned");
    const arl2::KvAttnPlan plan = kv_plan(desc);
    if ((double)plan.units * plan.nsplit > 2147483000.0 || (double)plan.units * plan.tile_rows > 2147483000.0)
        return fail(ARL2_ERR_UNSUPPORTED, "problem too large for one launch");
    if (plan.bytes > 0 && (desc->workspace == nullptr || desc->workspace_bytes < plan.bytes))
        return fail(ARL2_ERR_WORKSPACE, "workspace is NULL or smaller than arl2_kv_workspace_bytes()");
    if (!aligned16(desc->workspace)) return fail(ARL2_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    const size_t rows = kv_rows_bytes(desc, desc->H), lens = desc->B * sizeof(int32_t);
    const Range in[] = {{q, rows}, {cache, arl2_kv_cache_bytes(desc)}, {block_table, kv_table_bytes(desc)}, {kv_len, lens}, {q_len, lens}};
    const Range ws = {desc->workspace, plan.bytes};
    if (overlaps_any({out, rows}, in)) return fail(ARL2_ERR_INVALID_ARG, "out must not overlap an input");
    if (overlaps_any(ws, in) || overlaps(ws.p, ws.n, out, rows))
        return fail(ARL2_ERR_INVALID_ARG, "the workspace must overlap neither an input nor out");

    arl2::KvAttnArgs a = {};
    a.q = q; a.cache = cache; a.table = block_table; a.kv_len = kv_len; a.q_len = q_len; a.out = out;
    a.pool = kv_pool(desc);
    a.B = desc->B; a.H = desc->H; a.Lq = desc->Lq; a.D = desc->D; a.G = desc->H / desc->Hkv;
    a.causal = desc->causal;
    a.scale_log2 = (desc->sm_scale > 0.f ? desc->sm_scale : 1.0f / sqrtf((float)desc->D)) * 1.4426950408889634f;
    const hipError_t e = arl2::launch_kv_attn(a, plan, desc->workspace, reinterpret_cast<hipStream_t>(desc->stream));
    if (e != hipSuccess) return fail(ARL2_ERR_DEVICE, "attention launch failed: %s", hipGetErrorString(e));
    return ARL2_OK;
}

// ---- the causal recurrence ----------------------------------------------------------------------------
size_t arl2_scan_workspace_bytes(const arl2_scan_desc *desc)
{
    return check_scan_desc(desc) == ARL2_OK ? arl2::scan_plan(desc->B, desc->H, desc->L, desc->D, false).bytes : 0;
}

size_t arl2_scan_bwd_workspace_bytes(const arl2_scan_desc *desc)
{
    return check_scan_desc(desc) == ARL2_OK ? arl2::scan_plan(desc->B, desc->H, desc->L, desc->D, true).bytes : 0;
}

arl2_status arl2_scan_fwd(const arl2_scan_desc *desc, const void *q, const void *k, const void *v, const float *log_alpha,
                          const int32_t *seq_len, const float *S0, void *out, float *S)
{
    const arl2_status st = check_scan_desc(desc);
    if (st != ARL2_OK) return st;
    if (!q || !k || !v || !out) return fail(ARL2_ERR_INVALID_ARG, "q, k, v and out must not be NULL");
    if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(S0) || !aligned16(S))
        return fail(ARL2_ERR_INVALID_ARG, "q, k, v, S0, out and S must be 16-byte aligned");
    if (!aligned4(log_alpha) || !aligned4(seq_len)) return fail(ARL2_ERR_INVALID_ARG, "log_alpha and seq_len must be 4-byte aligned");
    const arl2::ScanPlan plan = arl2::scan_plan(desc->B, desc->H, desc->L, desc->D, false);
    if (plan.bytes > 0 && (desc->workspace == nullptr || desc->workspace_bytes < plan.bytes))
        return fail(ARL2_ERR_WORKSPACE, "workspace is NULL or smaller than arl2_scan_workspace_bytes()");
    if (!aligned16(desc->workspace)) return fail(ARL2_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    const size_t rows = scan_rows_bytes(desc), gates = scan_gate_bytes(desc), state = scan_state_bytes(desc), lens = desc->B * sizeof(int32_t);
    const Range ws = {desc->workspace, plan.bytes};
    const Range in[] = {{q, rows}, {k, rows}, {v, rows}, {log_alpha, gates}, {seq_len, lens}, {S0, state}};
    const Range in_but_S0[] = {{q, rows}, {k, rows}, {v, rows}, {log_alpha, gates}, {seq_len, lens}, {S == S0 ? nullptr : S0, state}};
    if (overlaps_any({out, rows}, in) || overlaps_any({S, state}, in_but_S0) || overlaps(out, rows, S, state))
        return fail(ARL2_ERR_INVALID_ARG, "out and S must overlap neither an input nor each other (S may be S0)");
    if (overlaps_any(ws, in) || overlaps(ws.p, ws.n, out, rows) || overlaps(ws.p, ws.n, S, state))
        return fail(ARL2_ERR_INVALID_ARG, "the workspace must overlap no other argument");

    arl2::ScanArgs a = scan_args(desc, q, k, v, log_alpha, seq_len, S0);
    a.out = out; a.S = S;
    const hipError_t e = arl2::launch_scan_fwd(a, plan, reinterpret_cast<hipStream_t>(desc->stream));
    if (e != hipSuccess) return fail(ARL2_ERR_DEVICE, "scan launch failed: %s", hipGetErrorString(e));
    return ARL2_OK;
}

arl2_status arl2_scan_bwd(const arl2_scan_desc *desc, const void *q, const void *k, const void *v, const float *log_alpha,
                          const int32_t *seq_len, const float *S0, const void *dout, const float *dS,
                          void *dq, void *dk, void *dv, float *dlog_alpha, float *dS0)
{
    const arl2_status st = check_scan_desc(desc);
    if (st != ARL2_OK) return st;
    if (!q || !k || !v || !dout || !dq || !dk || !dv) return fail(ARL2_ERR_INVALID_ARG, "q, k, v, dout, dq, dk and dv must not be NULL");
    for (const void *p : {q, k, v, dout, (const void *)dq, (const void *)dk, (const void *)dv, (const void *)S0, (const void *)dS, (const void *)dS0})
        if (!aligned16(p)) return fail(ARL2_ERR_INVALID_ARG, "rows, states and their gradients must be 16-byte aligned");
    if (!aligned4(log_alpha) || !aligned4(seq_len) || !aligned4(dlog_alpha))
        return fail(ARL2_ERR_INVALID_ARG, "log_alpha, dlog_alpha and seq_len must be 4-byte aligned");
    if (dlog_alpha != nullptr && log_alpha == nullptr) return fail(ARL2_ERR_INVALID_ARG, "dlog_alpha is of a log_alpha that is NULL");
    const arl2::ScanPlan plan = arl2::scan_plan(desc->B, desc->H, desc->L, desc->D, true);
    if (desc->workspace == nullptr || desc->workspace_bytes < plan.bytes)
        return fail(ARL2_ERR_WORKSPACE, "workspace is NULL or smaller than arl2_scan_bwd_workspace_bytes()");
    if (!aligned16(desc->workspace)) return fail(ARL2_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    const size_t rows = scan_rows_bytes(desc), gates = scan_gate_bytes(desc), state = scan_state_bytes(desc), lens = desc->B * sizeof(int32_t);
    const Range in[] = {{q, rows}, {k, rows}, {v, rows}, {log_alpha, gates}, {seq_len, lens}, {S0, state}, {dout, rows}, {dS, state}};
    const Range made[] = {{dq, rows}, {dk, rows}, {dv, rows}, {dlog_alpha, gates}, {dS0, state}, {desc->workspace, plan.bytes}};
    for (const Range &m : made) {
        for (const Range &i : in)
            if (overlaps(m.p, m.n, i.p, i.n)) return fail(ARL2_ERR_INVALID_ARG, "gradients and the workspace must not overlap an input");
        for (const Range &o : made)
            if (&o != &m && overlaps(m.p, m.n, o.p, o.n)) return fail(ARL2_ERR_INVALID_ARG, "gradients and the workspace must not overlap each other");
    }

    arl2::ScanArgs a = scan_args(desc, q, k, v, log_alpha, seq_len, S0);
    a.dout = dout; a.dS = dS; a.dq = dq; a.dk = dk; a.dv = dv; a.dla = dlog_alpha; a.dS0 = dS0;
    const hipError_t e = arl2::launch_scan_bwd(a, plan, reinterpret_cast<hipStream_t>(desc->stream));
    if (e != hipSuccess) return fail(ARL2_ERR_DEVICE, "scan gradient launch failed: %s", hipGetErrorString(e));
    return ARL2_OK;
}

// ---- rotary positions ---------------------------------------------------------------------------------
size_t arl2_rope_workspace_bytes(const arl2_rope_desc *desc)
{
    return check_rope_desc(desc) == ARL2_OK ? arl2::rope_parts_bytes(desc->B, desc->L, desc->D, desc->H, desc->Hk) : 0;
}

arl2_status arl2_rope_fwd(const arl2_rope_desc *desc, const void *q, const void *k, const void *wq, const void *wk,
                          const int32_t *pos, const int32_t *seq_len, void *yq, void *yk)
{
    const arl2_status st = check_rope_call(desc, {k, yk}, wq, wk, pos, seq_len);
    if (st != ARL2_OK) return st;
    if (!q || !yq) return fail(ARL2_ERR_INVALID_ARG, "q and yq must not be NULL");
    for (const void *p : {q, k, (const void *)yq, (const void *)yk})
        if (!aligned16(p)) return fail(ARL2_ERR_INVALID_ARG, "rows must be 16-byte aligned");
    const size_t nq = rope_rows_bytes(desc, desc->H), nk = rope_rows_bytes(desc, desc->Hk);
    const Range fixed[] = {{wq, rope_weight_bytes(desc, desc->H)}, {wk, rope_weight_bytes(desc, desc->Hk)}, {pos, rope_pos_bytes(desc)}, {seq_len, desc->B * sizeof(int32_t)}};
    if (overlaps_any({yq, nq}, fixed) || overlaps_any({yk, nk}, fixed) || overlaps(yq, nq, yk, nk) || overlaps(yq, nq, k, nk) || overlaps(yk, nk, q, nq) ||
        (yq != q && overlaps(yq, nq, q, nq)) || (yk != k && overlaps(yk, nk, k, nk)))
        return fail(ARL2_ERR_INVALID_ARG, "yq and yk must overlap neither an input nor each other (yq may be q, yk may be k)");

    arl2::RopeArgs a = rope_args(desc, q, k, wq, wk, pos, seq_len);
    a.y[0] = yq; a.y[1] = yk;
    const hipError_t e = arl2::launch_rope(a, reinterpret_cast<hipStream_t>(desc->stream));
    if (e != hipSuccess) return fail(ARL2_ERR_DEVICE, "rotation launch failed: %s", hipGetErrorString(e));
    return ARL2_OK;
}

arl2_status arl2_rope_bwd(const arl2_rope_desc *desc, const void *q, const void *k, const void *wq, const void *wk,
                          const int32_t *pos, const int32_t *seq_len, const void *dyq, const void *dyk,
                          void *dq, void *dk, float *dwq, float *dwk)
{
    const arl2_status st = check_rope_call(desc, {dyk, dk}, wq, wk, pos, seq_len);
    if (st != ARL2_OK) return st;
    if (!dyq || !dq) return fail(ARL2_ERR_INVALID_ARG, "dyq and dq must not be NULL");
    const bool norm = desc->norm != ARL2_NORM_NONE;
    if (norm && (!q || (desc->Hk > 0 && !k))) return fail(ARL2_ERR_INVALID_ARG, "q and k must not be NULL where rows have a norm");
    if ((dwq || dwk) && !norm) return fail(ARL2_ERR_INVALID_ARG, "rows without a norm have no weights and no gradients of weights");
    if (dwk && desc->Hk == 0) return fail(ARL2_ERR_INVALID_ARG, "dwk must be NULL where there are no keys");
    for (const void *p : {q, k, dyq, dyk, (const void *)dq, (const void *)dk})
        if (!aligned16(p)) return fail(ARL2_ERR_INVALID_ARG, "rows must be 16-byte aligned");
    if (!aligned4(dwq) || !aligned4(dwk)) return fail(ARL2_ERR_INVALID_ARG, "dwq and dwk must be 4-byte aligned");
    const size_t need = dwq || dwk ? arl2_rope_workspace_bytes(desc) : 0;
    if (need > 0 && (desc->workspace == nullptr || desc->workspace_bytes < need))
        return fail(ARL2_ERR_WORKSPACE, "workspace is NULL or smaller than arl2_rope_workspace_bytes()");
    if (!aligned16(desc->workspace)) return fail(ARL2_ERR_INVALID_ARG, "workspace must be 16-byte aligned");
    const size_t nq = rope_rows_bytes(desc, desc->H), nk = rope_rows_bytes(desc, desc->Hk), w = sizeof(float);
    const size_t elem = elem_bytes(desc->io_dtype);
    const Range in[] = {{norm ? q : nullptr, nq}, {norm ? k : nullptr, nk}, {wq, rope_weight_bytes(desc, desc->H)}, {wk, rope_weight_bytes(desc, desc->Hk)},
                        {pos, rope_pos_bytes(desc)}, {seq_len, desc->B * sizeof(int32_t)}, {dyq, nq}, {dyk, nk}};
    const Range made[] = {{dq, nq}, {dk, nk}, {dwq, rope_weight_bytes(desc, desc->H) / elem * w}, {dwk, rope_weight_bytes(desc, desc->Hk) / elem * w}, {desc->workspace, need}};
    for (const Range &m : made) {
        for (const Range &i : in)
            if (overlaps(m.p, m.n, i.p, i.n) && !(m.p == dq && i.p == dyq && dq == dyq) && !(m.p == dk && i.p == dyk && dk == dyk))
                return fail(ARL2_ERR_INVALID_ARG, "gradients and the workspace must not overlap an input (dq may be dyq, dk may be dyk)");
        for (const Range &o : made)
            if (&o != &m && overlaps(m.p, m.n, o.p, o.n)) return fail(ARL2_ERR_INVALID_ARG, "gradients and the workspace must not overlap each other");
    }

    arl2::RopeArgs a = rope_args(desc, q, k, wq, wk, pos, seq_len);
    a.dy[0] = dyq; a.dy[1] = dyk; a.y[0] = dq; a.y[1] = dk; a.dw[0] = dwq; a.dw[1] = dwk; a.part = (float *)desc->workspace;
    const hipError_t e = arl2::launch_rope_bwd(a, reinterpret_cast<hipStream_t>(desc->stream));
    if (e != hipSuccess) return fail(ARL2_ERR_DEVICE, "rotation gradient launch failed: %s", hipGetErrorString(e));
    return ARL2_OK;
}

const char *arl2_status_string(arl2_status s)
{
    switch (s) {
    case ARL2_OK: return "ARL2_OK";
    case ARL2_ERR_INVALID_ARG: return "ARL2_ERR_INVALID_ARG";
    case ARL2_ERR_UNSUPPORTED: return "ARL2_ERR_UNSUPPORTED";
    case ARL2_ERR_WORKSPACE: return "ARL2_ERR_WORKSPACE";
    case ARL2_ERR_DEVICE: return "ARL2_ERR_DEVICE";
    }
    return "ARL2_ERR_UNKNOWN";
}

const char *arl2_last_error(void) { return g_err; }

int arl2_version(void) { return 100; }

}  // extern "C"
