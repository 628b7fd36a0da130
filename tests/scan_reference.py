"""The causal recurrence and its gradients, token by token in fp64 (numpy), with the same sums over magnitudes, from which the limits of
the kernels' roundings follow."""
import numpy as np
import torch

EPS = 1e-6
BLOCK, LONGEST = 64, 1024        # tokens of a block; of a segment of the gradients' walk at the most

# One rounding to bf16 is off by at most U16 of the value.  A value in two bf16 parts is off by U16 of U16, fp32 arithmetic on the way (norms,
# decays, products, sums of up to some hundred terms) by less than another 2^-17 of the terms' magnitudes.  A block's own products
# (dout.v for dq and dk) are rounded to bf16 before they multiply rows of the block: U16 of each term's magnitude more, `near` below.
# For out (from 9 tokens on) and dv these products and the state's features that the block's rows are multiplied with both are: a term is one of
# the two, so that U16 of all magnitudes comes in.
# A value below the normal numbers of both types, 2^-126, may come as zero: off by less than TINY (half of bf16's smallest step would be 2^-134).
U16 = 2.0 ** -8
TINY = 2.0 ** -126
TWO = U16 * U16 + 2.0 ** -17


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(torch.bfloat16)


def wide(t):
    return t.detach().float().cpu().numpy().astype(np.float64)


class Case:
    """Inputs of one call, on the host: rows as bf16 hold them, and the results from the definition."""

    def __init__(self, B, H, L, D, seed=0, normalise=True, lens=None, start=True, gates="sigmoid", rows=1.0):
        g = np.random.Generator(np.random.Philox(seed))
        self.B, self.H, self.L, self.D, self.normalise = B, H, L, D, normalise
        self.lens = [L] * B if lens is None else list(lens)
        self.q, self.k, self.v, self.do = (bf16(g.standard_normal((B, L, H, D)) * rows) for _ in range(4))
        z = g.standard_normal((B, L, H)) + np.linspace(0.0, 6.0, H)
        la = -np.log1p(np.exp(-z))
        if gates == "resets":
            la[g.random((B, L, H)) < 0.05] = -np.inf
        elif gates == "small":
            la = -g.random((B, L, H)) * 300.0
        elif gates == "one":
            la = np.zeros((B, L, H))
        self.la = torch.from_numpy(la.astype(np.float32)) if gates != "none" else None
        state = (B, H, D, D)
        self.S0 = torch.from_numpy(g.standard_normal(state).astype(np.float32)) if start else None
        self.dS = torch.from_numpy(g.standard_normal(state).astype(np.float32)) if start else None

    def lens_device(self):
        return None if all(n == self.L for n in self.lens) else torch.tensor(self.lens, dtype=torch.int32, device="cuda")

    # -- in fp64

    def _inputs(self):
        q, k, v, do = (wide(x) for x in (self.q, self.k, self.v, self.do))
        iq, ik = (1.0 / np.sqrt((x * x).sum(-1, keepdims=True) + EPS) if self.normalise else np.ones_like(x[..., :1]) for x in (q, k))
        a = np.ones(q.shape[:3]) if self.la is None else np.exp(np.minimum(self.la.numpy().astype(np.float64), 0.0))
        zero = np.zeros((self.B, self.H, self.D, self.D))
        S0, dS = (zero.copy() if x is None else x.numpy().astype(np.float64) for x in (self.S0, self.dS))
        return q, k, v, do, iq, ik, a, S0, dS

    def forward(self):
        """out, S, and their limits."""
        q, k, v, do, iq, ik, a, S, _ = self._inputs()
        q, k = q * iq, k * ik
        out, most = np.zeros_like(q), np.zeros_like(q)
        M = np.abs(S)                                     # magnitudes
        for t in range(self.L):
            on = np.array([t < n for n in self.lens])
            for X, f in ((S, lambda x: x), (M, np.abs)):
                X[on] = a[on, t, :, None, None] * X[on] + f(k[on, t])[..., :, None] * f(v[on, t])[..., None, :]
            out[on, t] = np.einsum("bhd,bhde->bhe", q[on, t], S[on])
            most[on, t] = np.einsum("bhd,bhde->bhe", np.abs(q[on, t]), M[on])
        few = self.L <= 8
        return out, S, U16 * np.abs(out) + (0.0 if few else U16) * most + TWO * most + TINY, TWO * M + 1e-30

    def backward(self):
        """dq, dk, dv, dla, dS0, and their limits."""
        q0, k0, v, do, iq, ik, a, S, G = self._inputs()
        q, k = q0 * iq, k0 * ik
        B, L = self.B, self.L
        dq, dk, dv = np.zeros_like(q), np.zeros_like(q), np.zeros_like(q)
        mq, mk, mv, nq, nk = (np.zeros_like(q) for _ in range(5))
        E, ME, MS = np.zeros(q.shape[:3]), np.zeros(q.shape[:3]), [None] * L
        states, M, near = [None] * L, np.abs(S), np.zeros_like(S)
        for t in range(L):
            on = np.array([t < n for n in self.lens])
            if t % BLOCK == 0:
                near[:] = 0.0
            near[on] = a[on, t, :, None, None] * near[on] + np.abs(k[on, t])[..., :, None] * np.abs(v[on, t])[..., None, :]
            nq[on, t] = np.einsum("bhe,bhde->bhd", np.abs(do[on, t]), near[on])
            states[t], MS[t] = S.copy(), M.copy()         # before the token
            S[on] = a[on, t, :, None, None] * S[on] + k[on, t][..., :, None] * v[on, t][..., None, :]
            M[on] = a[on, t, :, None, None] * M[on] + np.abs(k[on, t])[..., :, None] * np.abs(v[on, t])[..., None, :]
            dq[on, t] = np.einsum("bhe,bhde->bhd", do[on, t], S[on])
            mq[on, t] = np.einsum("bhe,bhde->bhd", np.abs(do[on, t]), M[on])
        N = np.abs(G)
        near[:] = 0.0
        for t in reversed(range(L)):
            on = np.array([t < n for n in self.lens])
            if t % BLOCK == BLOCK - 1:
                near[:] = 0.0
            near[on] += np.abs(q[on, t])[..., :, None] * np.abs(do[on, t])[..., None, :]
            nk[on, t] = np.einsum("bhe,bhde->bhd", np.abs(v[on, t]), near[on])
            near[on] *= a[on, t, :, None, None]
            G[on] += q[on, t][..., :, None] * do[on, t][..., None, :]
            N[on] += np.abs(q[on, t])[..., :, None] * np.abs(do[on, t])[..., None, :]
            dk[on, t], mk[on, t] = np.einsum("bhe,bhde->bhd", v[on, t], G[on]), np.einsum("bhe,bhde->bhd", np.abs(v[on, t]), N[on])
            dv[on, t], mv[on, t] = np.einsum("bhd,bhde->bhe", k[on, t], G[on]), np.einsum("bhd,bhde->bhe", np.abs(k[on, t]), N[on])
            E[on, t] = (a[on, t, :, None, None] * states[t][on] * G[on]).sum((-1, -2))
            ME[on, t] = (a[on, t, :, None, None] * MS[t][on] * N[on]).sum((-1, -2))
            G[on] *= a[on, t, :, None, None]
            N[on] *= a[on, t, :, None, None]
        # E is summed from the segment's end: its error is that of the later tokens' products
        each = (np.abs(q) * mq).sum(-1) + (np.abs(k) * mk).sum(-1)
        along = np.zeros_like(E)
        for t in range(L):
            along[:, t] = each[:, t:t + LONGEST].sum(1)
        ends = ME.max(1, keepdims=True) + (np.abs(self.dS.numpy().astype(np.float64)) * M).sum((-1, -2))[:, None] if self.dS is not None else ME.max(1, keepdims=True)
        limits = []
        for d, m, c, x, i in ((dq, mq, nq, q, iq), (dk, mk, nk, k, ik)):
            if self.normalise:
                d[:] = i * (d - x * (x * d).sum(-1, keepdims=True))
                for y in (m, c):
                    y[:] = i * (y + np.abs(x) * (np.abs(x) * y).sum(-1, keepdims=True))
            limits.append(U16 * (np.abs(d) + c) + 2.0 * TWO * m + TINY)
        limits += [U16 * (np.abs(dv) + mv) + TWO * mv + TINY, 2.0 * TWO * (along + ends) + 1e-30, TWO * N + 1e-30]
        return (dq, dk, dv, E, G), limits


def run_forward(A, c, S0="own", out=None, S=None, in_place=False, stream=None, **kw):
    dev = lambda x: None if x is None else x.cuda()       # noqa: E731
    S0 = dev(c.S0) if isinstance(S0, str) else S0
    out = torch.full((c.B, c.L, c.H, c.D), 7.0, dtype=torch.bfloat16, device="cuda") if out is None else out
    S = S0 if in_place else torch.full((c.B, c.H, c.D, c.D), 7.0, device="cuda") if S is None else S
    ws = A.alloc_scan_workspace(c.B, c.H, c.L, c.D)
    if ws is not None:
        ws.fill_(0xff)                                    # NaN everywhere
    A.arl2_scan_fwd(dev(c.q), dev(c.k), dev(c.v), dev(c.la), S0, out, S, seq_len=c.lens_device(), normalise=c.normalise, workspace=ws, **kw)
    torch.cuda.synchronize()
    return out, S


def run_backward(A, c, want_gates=True, want_start=True, **kw):
    dev = lambda x: None if x is None else x.cuda()       # noqa: E731
    rows = [torch.full((c.B, c.L, c.H, c.D), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    dla = torch.full((c.B, c.L, c.H), 7.0, device="cuda") if want_gates and c.la is not None else None
    dS0 = torch.full((c.B, c.H, c.D, c.D), 7.0, device="cuda") if want_start else None
    ws = A.alloc_scan_workspace(c.B, c.H, c.L, c.D, backward=True)
    ws.fill_(0xff)
    A.arl2_scan_bwd(dev(c.q), dev(c.k), dev(c.v), dev(c.la), dev(c.S0), dev(c.do), dev(c.dS), *rows, dla, dS0, seq_len=c.lens_device(),
                    normalise=c.normalise, workspace=ws, **kw)
    torch.cuda.synchronize()
    return (*rows, dla, dS0)


def check(name, got, want, limit, lens=None):
    """`got` within `limit` of `want`; rows from lens[b] on untouched (7)."""
    got = wide(got)
    if lens is not None:
        for b, n in enumerate(lens):
            assert (got[b, n:] == 7.0).all(), f"{name}: rows behind the sequence of stream {b}"
        there = np.arange(got.shape[1])[None] < np.array(lens)[:, None]
        got, want, limit = got[there], want[there], limit[there]
    if not got.size:
        return
    assert np.isfinite(got).all(), name
    off = np.abs(got - want)
    bad = off > limit
    assert not bad.any(), f"{name}: {bad.sum()} values, first {np.argwhere(bad)[0]}: off by {off[bad][0]:.3g}, limit {limit[bad][0]:.3g}"
