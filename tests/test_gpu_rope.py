"""Rotary positions on several axes with the norm before them, and the gradients, against fp64 within the limits of the roundings."""
import itertools

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

# One rounding to the output's type is off by at most half a step of the value; fp32 arithmetic (the norm's sum, root, products,
# the turn, whose cosine and sine are off by 2^-22) by less than 2^-19 of the magnitudes that meet in a value.
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
F32 = 2.0 ** -19


@pytest.fixture(scope="module")
def A():
    import paper_2605_16579_amd as A
    A.load_library()
    return A


class Case:
    def __init__(self, B, H, Hk, L, D, dtype=torch.bfloat16, norm="row", halves=False, axis_pairs=None, theta=None, weights=True,
                 per_stream=False, lens=None, far=0, seed=0):
        g = torch.Generator().manual_seed(seed)
        self.B, self.heads, self.L, self.D, self.dtype, self.norm, self.halves = B, (H, Hk), L, D, dtype, norm, halves
        self.axis_pairs = axis_pairs or [D // 2 - 2 * (D // 6), D // 6, D // 6]
        self.theta = theta
        n = len(self.axis_pairs)
        self.x = [torch.randn((B, L, h, D), generator=g).to(dtype) if h else None for h in self.heads]
        self.dy = [torch.randn((B, L, h, D), generator=g).to(dtype) if h else None for h in self.heads]
        width = [D if norm == "head" else h * D for h in self.heads]
        self.w = [(1 + 0.3 * torch.randn(m, generator=g)).to(dtype) if weights and norm != "none" and m and h else None for m, h in zip(width, self.heads)]
        self.pos = torch.randint(-5, 200, (B, L, n) if per_stream else (L, n), generator=g, dtype=torch.int32) + far
        self.lens = lens

    def kw(self):
        return dict(axis_pairs=self.axis_pairs, theta=self.theta, halves=self.halves, norm=self.norm,
                    seq_len=None if self.lens is None else torch.tensor(self.lens, dtype=torch.int32, device="cuda"))

    # -- in fp64
    def _turn(self, x, sign):
        angle = np.zeros((*self.pos.shape[:-1], self.D // 2))
        at = 0
        for a, m in enumerate(self.axis_pairs):
            theta = (self.theta or [10000.0] * 4)[a] or 10000.0
            for i in range(m):
                angle[..., at + i] = self.pos[..., a].numpy().astype(np.float64) * theta ** (-i / m)
            at += m
        angle = np.broadcast_to(angle, (self.B, self.L, self.D // 2))[:, :, None]
        c, s = np.cos(angle), sign * np.sin(angle)
        y = np.empty_like(x)
        i0, i1 = (slice(0, self.D // 2), slice(self.D // 2, None)) if self.halves else (slice(0, None, 2), slice(1, None, 2))
        y[..., i0], y[..., i1] = x[..., i0] * c - x[..., i1] * s, x[..., i0] * s + x[..., i1] * c
        size = np.empty_like(x)
        size[..., i0] = size[..., i1] = np.hypot(x[..., i0], x[..., i1])      # what meets in the pair's values
        return y, size

    def _norm(self, x):
        if self.norm == "none":
            return np.ones_like(x[..., :1])
        return 1.0 / np.sqrt((x * x).mean((-1, -2) if self.norm == "row" else -1, keepdims=True) + 1e-6)

    def _wide(self, i):
        x = self.x[i].double().numpy()
        w = 1.0 if self.w[i] is None else self.w[i].double().numpy().reshape(-1, self.D)
        return x, w, self._norm(x)

    def forward(self):
        for i in range(2):
            if self.x[i] is None:
                yield None, None
                continue
            x, w, r = self._wide(i)
            y, size = self._turn(x * r * w, 1)
            yield y, HALF[self.dtype] * np.abs(y) + F32 * size

    def backward(self):
        """(dx, limit, dw, limit) of queries and keys."""
        there = np.arange(self.L)[None] < np.array(self.lens if self.lens is not None else [self.L] * self.B)[:, None]
        for i in range(2):
            if self.x[i] is None:
                yield (None,) * 4
                continue
            x, w, r = self._wide(i)
            z, size = self._turn(self.dy[i].double().numpy(), -1)
            z, size = z * there[..., None, None], size * there[..., None, None]
            xh = x * r
            over = (-1, -2) if self.norm == "row" else -1
            dw = (z * xh).sum((0, 1) if self.norm == "row" else (0, 1, 2)).reshape(-1)
            dwm = (size * np.abs(xh)).sum((0, 1) if self.norm == "row" else (0, 1, 2)).reshape(-1)
            g, gm = z * w, size * np.abs(w)
            if self.norm == "none":
                dx, m = g, gm
            else:
                dx = r * (g - xh * (g * xh).mean(over, keepdims=True))
                m = r * (gm + np.abs(xh) * (gm * np.abs(xh)).mean(over, keepdims=True))
            yield dx, HALF[self.dtype] * np.abs(dx) + F32 * m, dw, F32 * dwm


def dev(x):
    return None if x is None else x.cuda()


def check(name, got, want, limit, lens=None):
    got = got.double().cpu().numpy()
    if lens is not None:
        for b, n in enumerate(lens):
            assert (got[b, n:] == 7.0).all(), name
        there = np.arange(got.shape[1])[None] < np.array(lens)[:, None]
        got, want, limit = got[there], want[there], limit[there]
    off = np.abs(got - want)
    bad = ~(off <= limit)
    assert not bad.any(), f"{name}: {bad.sum()} values, first {np.argwhere(bad)[0]}: off by {off[bad][0]:.3g}, limit {limit[bad][0]:.3g}"


def run_forward(A, c, in_place=False):
    x = [dev(t) for t in c.x]
    y = x if in_place else [None if t is None else torch.full_like(t, 7.0) for t in x]
    A.arl2_rope_fwd(*x, dev(c.w[0]), dev(c.w[1]), dev(c.pos), *y, **c.kw())
    torch.cuda.synchronize()
    return y


def run_backward(A, c, in_place=False, weights=True):
    x, dy = [dev(t) for t in c.x], [dev(t) for t in c.dy]
    dx = dy if in_place else [None if t is None else torch.full_like(t, 7.0) for t in dy]
    dw = [torch.full((t.numel(),), 7.0, device="cuda") if t is not None and weights else None for t in c.w]
    ws = A.alloc_rope_workspace(c.B, *c.heads, c.L, c.D)
    ws.fill_(0xff)
    A.arl2_rope_bwd(*x, dev(c.w[0]), dev(c.w[1]), dev(c.pos), *dy, *dx, *dw, workspace=ws, **c.kw())
    torch.cuda.synchronize()
    return dx, dw


def both(A, c):
    for name, got, (want, limit) in zip(("yq", "yk"), run_forward(A, c), c.forward()):
        if got is not None:
            check(name, got, want, limit, c.lens)
    dx, dw = run_backward(A, c)
    for name, gx, gw, (wx, lx, ww, lw) in zip("qk", dx, dw, c.backward()):
        if gx is not None:
            check("d" + name, gx, wx, lx, c.lens)
        if gw is not None:
            check("dw" + name, gw, ww, lw)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("norm,halves", itertools.product(("none", "head", "row"), (False, True)))
@pytest.mark.parametrize("D", [64, 128])
def test_norms_and_pairings(A, D, norm, halves, dtype):
    both(A, Case(2, 3, 2, 37, D, dtype, norm, halves))


@pytest.mark.parametrize("norm", ["none", "head", "row"])
@pytest.mark.parametrize("H,Hk,D", [(1, 0, 64), (1, 1, 128), (7, 7, 128), (12, 12, 128), (24, 6, 64), (32, 8, 128), (40, 8, 128), (33, 31, 128), (64, 64, 64), (96, 12, 128), (96, 96, 128)])
def test_widths(A, norm, H, Hk, D):
    """Every number of units to a lane, one wavefront to a token and four, rows that leave lanes without a unit."""
    both(A, Case(1, H, Hk, 9, D, torch.float32 if H % 2 else torch.bfloat16, norm, bool(H % 3)))


@pytest.mark.parametrize("B,L", [(1, 1), (1, 4), (3, 1), (2, 3000), (1, 9001)])
@pytest.mark.parametrize("norm", ["head", "row"])
def test_lengths(A, B, L, norm):
    both(A, Case(B, 3, 1, L, 64, norm=norm, per_stream=L == 3000))


@pytest.mark.parametrize("H,D", [(3, 64), (48, 128)])
@pytest.mark.parametrize("norm", ["none", "head", "row"])
def test_sequences_of_different_lengths(A, H, D, norm):
    both(A, Case(4, H, 2, 21, D, norm=norm, lens=[0, 21, 5, 1], per_stream=True))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_no_weights_and_few_pairs(A, dtype):
    both(A, Case(2, 3, 3, 20, 128, dtype, "head", True, [5, 1, 7, 2], [10000.0, 100.0, 0.0, 5e5], weights=False))
    both(A, Case(2, 3, 3, 20, 64, dtype, "row", False, [3], [1e6], weights=False))


@pytest.mark.parametrize("far", [0, 1000000, 2 ** 31 - 300, -(2 ** 31) + 300])
def test_far_positions(A, far):
    """Angles of 2^31 radians: fp32 would have nothing left of them."""
    both(A, Case(1, 2, 2, 30, 128, torch.float32, "none", far=far, axis_pairs=[64]))


def test_features_that_no_axis_turns_stay_as_they_are(A):
    c = Case(1, 2, 1, 8, 64, torch.float32, "none", True, [4])
    c.x[0][0, 2, 1, 20] = float("inf")
    c.x[0][0, 3, 1, 52] = float("nan")
    y = run_forward(A, c)[0].cpu()
    still = [i for i in range(64) if i % 32 >= 4]
    assert torch.equal(y[..., still].nan_to_num(1.5), c.x[0][..., still].nan_to_num(1.5))


def test_in_place_and_again(A):
    for norm, H in (("row", 5), ("head", 5), ("none", 5), ("row", 70)):
        c = Case(2, H, 3, 50, 128, norm=norm)
        y, (dx, dw) = run_forward(A, c), run_backward(A, c)
        assert all(torch.equal(a, b) for a, b in zip(y, run_forward(A, c, in_place=True)))
        dx2, dw2 = run_backward(A, c, in_place=True)
        assert all(torch.equal(a, b) for a, b in zip(dx, dx2))
        assert all(a is None or torch.equal(a, b) for a, b in zip(dw, dw2))
        dx3, _ = run_backward(A, c, weights=False)
        assert all(torch.equal(a, b) for a, b in zip(dx, dx3))


def test_zero_rows(A):
    c = Case(1, 2, 2, 6, 64, norm="head")
    c.x[0][0, 2] = 0
    both(A, c)


def test_captured_with_the_recurrence(A):
    """Rotation, recurrence and the gradients of both as a training step has them, captured and replayed on new inputs."""
    B, H, L, D = 2, 3, 150, 64
    bf = dict(dtype=torch.bfloat16, device="cuda")
    x = [torch.randn((B, L, H, D), **bf) for _ in range(2)]
    w = [torch.rand(H * D, **bf) + 0.5 for _ in range(2)]
    v, do = torch.randn((B, L, H, D), **bf), torch.randn((B, L, H, D), **bf)
    la = torch.nn.functional.logsigmoid(torch.randn((B, L, H), device="cuda") + 2)
    pos = torch.randint(0, 50, (L, 3), dtype=torch.int32, device="cuda")
    r, d = [torch.empty_like(v) for _ in range(2)], [torch.empty_like(v) for _ in range(3)]
    out, S, dla = torch.empty_like(v), torch.empty((B, H, D, D), device="cuda"), torch.empty_like(la)
    dw = [torch.empty(H * D, device="cuda") for _ in range(2)]
    how = dict(axis_pairs=[12, 10, 10], norm="row")
    ws, wb, wr = A.alloc_scan_workspace(B, H, L, D), A.alloc_scan_workspace(B, H, L, D, backward=True), A.alloc_rope_workspace(B, H, H, L, D)

    def step():
        A.arl2_rope_fwd(*x, *w, pos, *r, **how)
        A.arl2_scan_fwd(*r, v, la, None, out, S, workspace=ws)
        A.arl2_scan_bwd(*r, v, la, None, do, None, *d, dla, None, workspace=wb)
        A.arl2_rope_bwd(*x, *w, pos, d[0], d[1], d[0], d[1], *dw, workspace=wr, **how)

    # the same, one after the other, in fp64
    def double():
        leaves = [t.double().cpu().requires_grad_() for t in (*x, *w, v, la)]
        xq, xk, wq, wk, vv, g = leaves
        angle = torch.cat([pos[:, a:a + 1].double().cpu() * 10000.0 ** (-torch.arange(m).double() / m) for a, m in enumerate((12, 10, 10))], 1)[None, :, None]
        rows = []
        for t, u in ((xq, wq), (xk, wk)):
            y = t * (t.square().mean((-1, -2), keepdim=True) + 1e-6) ** -0.5 * u.view(H, D)
            y = torch.stack((y[..., 0::2] * angle.cos() - y[..., 1::2] * angle.sin(), y[..., 0::2] * angle.sin() + y[..., 1::2] * angle.cos()), -1).flatten(-2)
            rows.append(y / (y.square().sum(-1, keepdim=True) + 1e-6).sqrt())
        state, outs = torch.zeros((B, H, D, D), dtype=torch.float64), []
        for t in range(L):
            state = g[:, t].exp()[..., None, None] * state + rows[1][:, t, :, :, None] * vv[:, t, :, None]
            outs.append((rows[0][:, t, :, :, None] * state).sum(-2))
        torch.stack(outs, 1).backward(do.double().cpu())
        return torch.stack(outs, 1).detach(), [t.grad for t in leaves]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    written = (out, S, d[0], d[1], d[2], dla, *dw)
    for i in range(3):
        for t in (*x, v, do):
            t.copy_(torch.randn_like(t))
        step()
        torch.cuda.synchronize()
        want = [t.clone() for t in written]
        for t in written:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(written, want)), i
    ref, grads = double()
    # rounded to bf16: the rotated rows, a block's products and the result (or the rotated rows' gradients and theirs), each at most
    # 2^-8 of a value and independent of one another: three in the 2-norm, with what a normalised row's roundings add to its length
    for got, r64 in ((out, ref), (d[0], grads[0]), (d[1], grads[1]), (d[2], grads[4]), (dla, grads[5]), (dw[0], grads[2]), (dw[1], grads[3])):
        e = (got.double().cpu() - r64).norm() / r64.norm()
        assert e <= 3 * 2.0 ** -8, float(e)


@pytest.mark.parametrize("norm", ["head", "row"])
def test_one_weight_and_one_gradient(A, norm):
    """Weights of one of the arrays, gradients of one of them, keys' or queries': what the others get does not change."""
    c = Case(2, 5, 3, 40, 64, norm=norm, lens=[33, 40])
    full, fw = run_backward(A, c)
    for i in range(2):
        x, dy = [dev(t) for t in c.x], [dev(t) for t in c.dy]
        dx, dw = [torch.full_like(t, 7.0) for t in dy], [None, None]
        dw[i] = torch.full_like(fw[i], 7.0)
        ws = A.alloc_rope_workspace(c.B, *c.heads, c.L, c.D)
        A.arl2_rope_bwd(*x, dev(c.w[0]), dev(c.w[1]), dev(c.pos), *dy, *dx, *dw, workspace=ws, **c.kw())
        assert all(torch.equal(a, b) for a, b in zip((*dx, dw[i]), (*full, fw[i])))
        one = Case(2, 5, 3, 40, 64, norm=norm, lens=[33, 40])
        one.w[1 - i] = None
        both(A, one)


def test_without_norm_the_rows_are_not_needed(A):
    c = Case(2, 3, 2, 30, 128, norm="none", per_stream=True)
    want, _ = run_backward(A, c)
    dy = [dev(t) for t in c.dy]
    got = [torch.full_like(t, 7.0) for t in dy]
    A.arl2_rope_bwd(None, None, None, None, dev(c.pos), *dy, *got, None, None, **c.kw())
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    only = Case(2, 3, 0, 30, 128, norm="none")
    both(A, only)


@pytest.mark.parametrize("norm", ["head", "row"])
def test_missing_rows_add_nothing_to_a_weights_gradient(A, norm):
    """The last workgroup has room for tokens that there are not, in memory that a call before left NaNs in."""
    bad = torch.full((64, 200, 12, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    out, ws = torch.empty_like(bad), A.alloc_scan_workspace(64, 12, 200, 128)
    for B, H, Hk, L in ((1, 2, 1, 1), (1, 2, 1, 17), (3, 4, 2, 5), (1, 8, 8, 77)):
        c = Case(B, H, Hk, L, 64, norm=norm)
        A.arl2_scan_fwd(bad, bad, bad, None, None, out, None, workspace=ws)
        _, dw = run_backward(A, c)
        for name, gw, (_, _, ww, lw) in zip("qk", dw, c.backward()):
            check("dw" + name, gw, ww, lw)


def test_lengths_are_cut(A):
    c = Case(3, 3, 2, 30, 64, norm="row", lens=[0, 30, 30])
    given = torch.tensor([-7, 31, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    kw = c.kw()
    c.kw = lambda: {**kw, "seq_len": given}
    both(A, c)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_a_bad_row_reaches(A, bad):
    """Its own token (its head's rows, or the row's), and the weights' gradients; nothing from behind a sequence."""
    for norm in ("head", "row"):
        c = Case(2, 3, 2, 30, 64, norm=norm, lens=[20, 30])
        y, (dx, dw) = run_forward(A, c), run_backward(A, c)
        for t in (*c.x, *c.dy):
            t[0, 25] = bad
        y2, (dx2, dw2) = run_forward(A, c), run_backward(A, c)
        assert all(torch.equal(a, b) for a, b in zip((*y, *dx, *dw), (*y2, *dx2, *dw2)))
        c.x[0][1, 7, 1, 3] = bad
        y3, (dx3, _) = run_forward(A, c), run_backward(A, c)
        for a, b in zip((*y, *dx), (*y3, *dx3)):
            a, b = a.clone(), b.clone()
            assert not torch.isfinite(b[1, 7].float()).all() or b.shape[2] == 2
            a[1, 7], b[1, 7] = 0, 0
            assert torch.equal(a, b)


def test_offsets_past_32_bits(A):
    B, L, D = 2, 8400011, 128
    x, dy = (torch.empty((B, L, 1, D), dtype=torch.bfloat16, device="cuda").normal_() for _ in range(2))
    pos = torch.arange(L, dtype=torch.int32, device="cuda")[:, None].contiguous()
    y, dx, dw = torch.empty_like(x), torch.empty_like(x), torch.empty(D, device="cuda")
    kw = dict(axis_pairs=[64], norm="head")
    A.arl2_rope_fwd(x, None, None, None, pos, y, None, **kw)
    A.arl2_rope_bwd(x, None, None, None, pos, dy, None, dx, None, dw, None, workspace=A.alloc_rope_workspace(B, 1, 0, L, D), **kw)
    c = Case(1, 1, 0, 50, D, norm="head", axis_pairs=[64], weights=False)
    c.x[0], c.dy[0], c.pos = x[-1:, -50:].cpu(), dy[-1:, -50:].cpu(), pos[-50:].cpu()
    (want, limit), _ = c.forward()
    check("y", y[-1:, -50:], want, limit)
    want, limit, _, _ = next(c.backward())
    check("dx", dx[-1:, -50:], want, limit)
    # the weight's gradient over all tokens: a sum of 2^24 terms of unit size in fp64 by halves of the streams
    angle = pos.double() * 10000.0 ** (-torch.arange(64, device="cuda").double() / 64)
    want = torch.zeros(D, dtype=torch.float64, device="cuda")
    most = torch.zeros_like(want)
    for b in range(B):
        for a in range(0, L, 1 << 21):
            u, d, t = x[b, a:a + (1 << 21), 0].double(), dy[b, a:a + (1 << 21), 0].double(), angle[a:a + (1 << 21)]
            u = u * (u.square().mean(-1, keepdim=True) + 1e-6) ** -0.5
            z = torch.empty_like(d)
            z[:, 0::2], z[:, 1::2] = d[:, 0::2] * t.cos() + d[:, 1::2] * t.sin(), d[:, 1::2] * t.cos() - d[:, 0::2] * t.sin()
            want += (z * u).sum(0)
            most += (z * u).abs().sum(0)
    # a lane adds L B / (1024 workgroups 16) tokens one by one in fp32: 2^-24 of the sum so far each, 1026 terms, beside the terms' own F32
    check("dw", dw, want.cpu().numpy(), ((1026 * 2.0 ** -24 + F32) * most).cpu().numpy())
