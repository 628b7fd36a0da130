"""Plain 64-bit forms of the paged 4-bit cache's operations (CPU, numpy): the format, the rotation, attention with its error bound."""
import numpy as np
import torch

GRID = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantise(x):
    """Values [..., D] (fp32) -> what is stored for them, in float64; groups with a NaN or an infinity are NaN."""
    x = np.asarray(x, dtype=np.float32).astype(np.float64)
    g = x.reshape(x.shape[:-1] + (-1, 32))
    finite = np.isfinite(g).all(-1, keepdims=True)
    g = np.where(finite, g, 0.0)
    amax = np.abs(g).max(-1, keepdims=True)
    m, x2 = np.frexp(amax)                                      # amax = m 2^x2, m in [1/2, 1): within 7 2^e from e = x2 - 3 on, or x2 - 2
    e = np.clip(np.where(amax == 0, -120, x2 - 3 + (m > 0.875)), -120, 125)
    u = g / 2.0 ** e.astype(np.float64)
    a = np.abs(u)
    # nearest of the grid, ties to the even code
    d = np.abs(a[..., None] - GRID)
    best = d.min(-1, keepdims=True)
    near = d == best
    even = near & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), near.argmax(-1))
    y = np.copysign(GRID[code], u) * 2.0 ** e.astype(np.float64)
    return np.where(finite, y, np.nan).reshape(x.shape)


def rotate(x, cos, sin):
    """x [L, H, D] by tables [L, D/2], pairs (2i, 2i + 1), rounded once to fp32."""
    x = x.astype(np.float64)
    c, s = cos.astype(np.float64)[:, None], sin.astype(np.float64)[:, None]
    y = np.empty_like(x)
    y[..., 0::2] = x[..., 0::2] * c - x[..., 1::2] * s
    y[..., 1::2] = x[..., 0::2] * s + x[..., 1::2] * c
    with np.errstate(over="ignore"):
        return y.astype(np.float32)


def attend(q, k, v, limit, scale, seen=None):
    """One stream: q [n, H, D], k, v [T, Hkv, D] (float64), query i sees keys j < limit[i] (and seen[j]).

    Returns the outputs [n, H, D] and how far a kernel may be from them, for a kernel that rounds probabilities and outputs to bf16
    (2^-8 relative each), takes a query row to within 1.07 * 2^-12 of the largest of each 32 features, feature by feature, or to within
    2^-9 of its length (see below) and otherwise computes in fp32:

      |error| <= 2^-8 (sum_j p_j |v_j| + |out|)  +  2 dl sum_j p_j |v_j|,
      dl, the error of a logit: scale * max(sum_d 1.07 * 2^-12 amax_32(q) |k_d|, 2^-9 |q| |k|)  +  2^-18 (1 + |largest logit|)
      (fp32: sums of up to 128 products, a scaling, and an exponential's argument, each a few 2^-24 of the operands)

    A query feature is taken as three 6-bit floats (4 significant bits, steps of 1/2 at most below 8) at units u, u/32, u/256
    with the largest magnitude in (3.75, 7.5] u: the first leaves at most half its largest step, u/4, the second of that (up to
    7.5 units) u/64, the third at most half its largest step, 2^-10 u <= 2^-12 * 1.07 amax; 1.07 is in the factor of the sum below.
    The third is left out only where the two leave no more than 2^-9 of the row's length, in the Euclidean norm: the error of its
    product with a key is then at most 2^-9 |q| |k| by Cauchy and Schwarz.
    """
    n, H, D = q.shape
    T, Hkv, _ = k.shape
    G = H // Hkv
    out, bound = np.zeros((n, H, D)), np.zeros((n, H, D))
    see = np.arange(T)[None, :] < np.asarray(limit)[:, None]
    if seen is not None:
        see &= seen[None, :]
    for h in range(H):
        kk, vv = k[:, h // G], v[:, h // G]
        with np.errstate(invalid="ignore"):
            logit = (q[:, h] @ np.where(np.isnan(kk), 0.0, kk).T) * scale
        logit = np.where(np.isnan(kk).any(-1)[None, :], np.nan, logit)
        logit = np.where(see, logit, -np.inf)
        top = np.where(see.any(-1), np.max(logit, -1, initial=-np.inf), 0.0)
        p = np.where(see, np.exp(logit - top[:, None]), 0.0)
        s = p.sum(-1, keepdims=True)
        p = np.divide(p, s, out=np.zeros_like(p), where=s != 0)
        nan_v = np.isnan(vv)
        v0 = np.where(nan_v, 0.0, vv)
        o = p @ v0
        touched = (see.astype(np.float64) @ nan_v.astype(np.float64)) > 0          # a NaN value that the row sees
        out[:, h] = np.where(touched, np.nan, o)
        mag = p @ np.abs(v0)
        amax = np.abs(q[:, h]).reshape(n, D // 32, 32).max(-1).repeat(32, -1)
        k0 = np.where(np.isnan(kk), 0.0, kk)
        by_feature, by_length = 1.07 * 2.0 ** -12 * (amax @ np.abs(k0).max(0, initial=0.0)), 2.0 ** -9 * np.linalg.norm(q[:, h], axis=-1) * np.linalg.norm(k0, axis=-1).max(initial=0.0)
        dl = scale * np.maximum(by_feature, by_length) + 2.0 ** -18 * (1 + np.abs(np.where(see, logit, 0.0)).max(-1, initial=0.0))
        bound[:, h] = 2.0 ** -8 * (mag + np.abs(o)) * 1.01 + 2 * dl[:, None] * mag + 2.0 ** -120
    return out, bound


class Paged:
    """A pool on the GPU next to the values that it is to hold: streams of rows placed by a shuffled block table."""

    def __init__(self, A, B, Hkv, D, page, tokens, seed=0, spare=3, fill=0xFF):
        self.A, self.B, self.Hkv, self.D, self.page = A, B, Hkv, D, page
        self.width = max(1, -(-tokens // page))
        self.n_pages = B * self.width + spare
        r = np.random.default_rng(seed)
        self.table = r.permutation(self.n_pages)[:B * self.width].reshape(B, self.width).astype(np.int32)
        self.table_dev = torch.from_numpy(self.table).cuda()
        self.cache = A.alloc_kv_cache(self.n_pages, Hkv, page, D)
        self.cache.fill_(fill)                                   # whatever unused memory holds: NaN scales
        cap = self.width * page
        self.k = np.full((B, cap, Hkv, D), np.nan)
        self.v = np.full((B, cap, Hkv, D), np.nan)
        ang = r.uniform(-np.pi, np.pi, (cap, D // 2))
        self.cos, self.sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)

    def append(self, k, v, start, count=None, rope=True):
        """k, v bf16 CPU tensors [B, L, Hkv, D]; start, count lists."""
        L = k.shape[1]
        self.A.arl2_kv_append(k.cuda(), v.cuda(), self.cache, self.table_dev, ints(start), count=None if count is None else ints(count),
                              rope_cos=torch.from_numpy(self.cos).cuda() if rope else None, rope_sin=torch.from_numpy(self.sin).cuda() if rope else None)
        kn, vn = k.float().numpy(), v.float().numpy()
        if rope:
            at = np.clip(np.asarray(start, dtype=np.int64)[:, None] + np.arange(L), 0, self.width * self.page - 1)
            kn = np.stack([rotate(kn[b], self.cos[at[b]], self.sin[at[b]]) for b in range(self.B)])
        kn, vn = quantise(kn), quantise(vn)
        for b in range(self.B):
            n = L if count is None else min(max(count[b], 0), L)
            for i in range(n):
                p = start[b] + i
                if 0 <= p < self.width * self.page and 0 <= self.table[b, p // self.page] < self.n_pages:
                    self.k[b, p], self.v[b, p] = kn[b, i], vn[b, i]

    def fill_with(self, lens, seed=1, std=1.0, chunk=512):
        """Appends normal rows until stream b holds lens[b] tokens."""
        g = torch.Generator().manual_seed(seed)
        for at in range(0, max(lens), chunk):
            L = min(chunk, max(lens) - at)
            k = (torch.randn((self.B, L, self.Hkv, self.D), generator=g) * std).bfloat16()
            v = torch.randn((self.B, L, self.Hkv, self.D), generator=g).bfloat16()
            self.append(k, v, [at] * self.B, [min(max(n - at, 0), L) for n in lens], rope=False)

    def set_table(self, table):
        self.table = np.asarray(table, dtype=np.int32)
        self.table_dev = torch.from_numpy(self.table).cuda()

    def seen(self, b):
        ok = (self.table[b] >= 0) & (self.table[b] < self.n_pages)
        return ok.repeat(self.page)


def ints(x):
    return torch.tensor(list(x), dtype=torch.int32).cuda()


def bf16_normal(shape, seed, std=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * std).bfloat16()


def check_attention(A, pool, q, kv_len, q_len=None, causal=False, sm_scale=0.0, out_fill=7.0):
    """Runs the kernel on `pool` and holds every output to its bound; rows past q_len to their old contents.  Returns the output."""
    B, L, H, D = q.shape
    out = torch.full(q.shape, out_fill, dtype=torch.bfloat16, device="cuda")
    ws = A.alloc_kv_workspace(B, H, pool.Hkv, L, D, pool.page, pool.width)
    A.arl2_kv_attn_fwd(q.cuda(), pool.cache, pool.table_dev, ints(kv_len), out, q_len=None if q_len is None else ints(q_len), causal=causal,
                       sm_scale=sm_scale, workspace=ws)
    torch.cuda.synchronize()
    got = out.float().cpu().numpy().astype(np.float64)
    scale = sm_scale or D ** -0.5
    for b in range(B):
        n = L if q_len is None else min(max(q_len[b], 0), L)
        T = min(max(kv_len[b], 0), pool.width * pool.page)
        limit = [min(max(T - n + i + 1, 0), T) if causal else T for i in range(n)]
        ref, bound = attend(q[b, :n].float().numpy().astype(np.float64), pool.k[b, :T], pool.v[b, :T], limit, scale, pool.seen(b)[:T])
        nan = np.isnan(ref)
        assert np.array_equal(np.isnan(got[b, :n]), nan), (b, np.argwhere(np.isnan(got[b, :n]) != nan)[:4])
        off = np.abs(got[b, :n] - ref)
        bad = (off > bound) & ~nan
        assert not bad.any(), (b, np.argwhere(bad)[:4], off[bad][:4], bound[bad][:4])
        assert (got[b, n:] == out_fill).all(), "rows past the last query were written"
    return out
