"""Attention over the 4-bit cache held to what its roundings amount to, tight enough that a lost or an unwanted key shows.

`kv_reference.attend` bounds the worst case: every rounding at its largest and all of one sign.  Here the query is taken exactly as the
kernel takes it, so that only roundings of many independent terms are left, and these are bounded by their sum of squares:

    error of an output = sum_j p_j v_j r_j + sum_j p_j (v_j - out) d_j + out r,    |r_j|, |r| <= 2^-8 (bf16),  |d_j| <= 2^-18 (1 + |largest logit|) (fp32)

  one output      <= 2^-8 |out| + min(6.5 sqrt(sum_j c_j^2), sum_j c_j),   c_j = 2^-8 p_j |v_j| + d p_j |v_j - out|:
                     by Hoeffding's inequality independent terms of mean zero and at most c_j pass 6.5 sqrt(sum c_j^2) once in 7 * 10^8
  all of a head   <= sqrt(sum over its outputs of (2^-8 out)^2 + sum_j c_j^2) in the Euclidean norm, and a third of that square from 16
                     rows on: a rounding is uniform between -2^-8 and 2^-8 of the smallest value of its binade at most, of which the
                     mean square is a third (a bit over half of that on the values of a whole binade, which is the margin)
"""
import numpy as np

import kv_reference as R

LEAST_UNIT, PARTS = 27 - 127, (0, 5, 8)


def _e2m3(x):
    """Nearest 6-bit floats, ties to even, 7.5 at the most."""
    a = np.abs(x)
    step = np.where(a < 2, 0.125, np.where(a < 4, 0.25, 0.5))
    return np.copysign(np.minimum(np.rint(a / step) * step, 7.5), x)


def taken_query(q):
    """What calls of more than 64 rows take for query rows [..., D] of finite bf16 values: per 32 features the sum of 6-bit floats at units u,
    u / 32 and u / 256, the largest in (3.75, 7.5] u, u >= 2^-100; without the third where two leave at most 2^-9 of the row's length
    and its square is in fp32's reach (not above it; what is left counts 2^-78 more in every 32 features, in the square)."""
    g = q.reshape(q.shape[:-1] + (-1, 32)).astype(np.float64)
    amax = np.abs(g).max(-1, keepdims=True)
    m, e = np.frexp(amax)                                           # amax = m 2^e, m in [1/2, 1): 3.75 < amax / u <= 7.5
    e = np.maximum(np.where(amax == 0, LEAST_UNIT, np.where(m > 0.9375, e - 2, e - 3)), LEAST_UNIT)
    left, sums = g, []
    for p in PARTS:
        unit = 2.0 ** (e - p)
        # (the largest that rounds to a finite value: beyond it the first part is cut, and the second holds the rest)
        part = _e2m3(np.clip(left, -3.75 * 2.0 ** 126, 3.75 * 2.0 ** 126) / unit) * unit
        left = left - part
        sums.append(part if not sums else sums[-1] + part)
    length = np.square(g).sum((-1, -2), keepdims=True)
    left = np.square(g - sums[1]).sum((-1, -2), keepdims=True) + 2.0 ** -78 * (amax > 0).sum(-2, keepdims=True)
    two = (left <= 2.0 ** -18 * length) & (length < 2.0 ** 128)
    return np.where(two, sums[1], sums[2]).reshape(q.shape)


def expected(q, k, v, limit, scale, seen=None):
    """One stream and query head: q [n, D] as taken, k, v [T, D]; query i sees keys j < limit[i] (and seen[j]).  Probabilities [n, T], outputs
    [n, D], and the terms' squares and sums that the limits are made of."""
    see = np.arange(k.shape[0])[None, :] < np.asarray(limit)[:, None]
    if seen is not None:
        see = see & seen[None, :]
    k, v = np.where(see.any(0)[:, None], k, 0.0), np.where(see.any(0)[:, None], v, 0.0)
    logit = np.where(see, (q @ k.T) * scale, -np.inf)
    top = np.where(see.any(-1), logit.max(-1, initial=-np.inf), 0.0)
    p = np.exp(logit - top[:, None])
    total = p.sum(-1, keepdims=True)
    p = np.divide(p, total, out=np.zeros_like(p), where=total != 0)
    out = p @ v
    d = 2.0 ** -18 * (1 + np.abs(np.where(see, logit, 0.0)).max(-1, initial=0.0))[:, None]
    # sum_j of c_j^2, of which each term's vector has its length and the sum at most both, and of c_j with |v - out| <= |v| + |out|
    square = 2.0 ** -16 * (p ** 2 @ v ** 2)
    spread = d ** 2 * (p ** 2 @ v ** 2 - 2 * out * (p ** 2 @ v) + (p ** 2).sum(-1, keepdims=True) * out ** 2)
    # What was summed up to a running maximum is lost where a later one is 2^126 times as much; many rows raise theirs where a block's
    # probabilities add up to 2^12.
    gone = 2.0 ** -114 * (see @ np.abs(v))
    both = np.square(np.sqrt(square) + np.sqrt(np.maximum(spread, 0.0)) + gone)
    return p, out, both, (2.0 ** -8 + d) * (p @ np.abs(v)) + d * np.abs(out) + gone


def misses(got, out, square, total):
    """How far outputs [n, D] of a head are beyond their limits: the largest ratio of one output's error, and that of all together."""
    off = np.abs(got - out)
    one = 2.0 ** -8 * np.abs(out) + np.minimum(6.5 * np.sqrt(square), total) + 2.0 ** -120
    norm = np.sqrt((2.0 ** -16 * out ** 2 + square).sum() * (1 / 3 if got.shape[0] >= 16 else 1)) + 2.0 ** -120
    return (off / one).max(initial=0.0), np.sqrt((off ** 2).sum()) / norm


def check(A, pool, q, kv_len, q_len=None, causal=False, sm_scale=0.0, heads=None):
    """Runs the kernel on `pool` (finite rows) and holds all outputs of `heads` to the limits.  Returns the output."""
    import torch
    B, L, H, D = q.shape
    G = H // pool.Hkv
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    ws = A.alloc_kv_workspace(B, H, pool.Hkv, L, D, pool.page, pool.width)
    A.arl2_kv_attn_fwd(q.cuda(), pool.cache, pool.table_dev, R.ints(kv_len), out, q_len=None if q_len is None else R.ints(q_len), causal=causal,
                       sm_scale=sm_scale, workspace=ws)
    torch.cuda.synchronize()
    got, rows = out.float().cpu().numpy().astype(np.float64), q.float().numpy().astype(np.float64)
    if L * G > 64:
        rows = taken_query(rows)
    for b in range(B):
        n = L if q_len is None else min(max(q_len[b], 0), L)
        T = min(max(kv_len[b], 0), pool.width * pool.page)
        limit = [min(max(T - n + i + 1, 0), T) if causal else T for i in range(n)]
        for h in range(H) if heads is None else heads:
            _, ref, square, total = expected(rows[b, :n, h], pool.k[b, :T, h // G], pool.v[b, :T, h // G], limit, sm_scale or D ** -0.5, pool.seen(b)[:T])
            one, norm = misses(got[b, :n, h], ref, square, total)
            assert one <= 1 and norm <= 1, (b, h, one, norm)
    return out
