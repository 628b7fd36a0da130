"""The causal recurrence and its gradients against fp64, element by element within the limits of the roundings."""
import numpy as np
import pytest
import torch

import scan_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2605_16579_amd as A
    A.load_library()
    return A


def check_forward(A, c, **kw):
    out, S, lo, ls = c.forward()
    got, state = R.run_forward(A, c, **kw)
    R.check("out", got, out, lo, c.lens)
    R.check("S", state, S, ls)
    # in the 2-norm the roundings of out and of a block's products are independent: U16 / sqrt(3) each at the most
    there = np.arange(c.L)[None] < np.array(c.lens)[:, None]
    if there.any() and np.linalg.norm(out[there]) > 0:
        assert np.linalg.norm(R.wide(got)[there] - out[there]) <= R.U16 * np.linalg.norm(out[there])
        assert np.linalg.norm(R.wide(state) - S) <= R.TWO * np.linalg.norm(S) + 1e-30
    return got, state


def check_backward(A, c, **kw):
    want, limits = c.backward()
    got = R.run_backward(A, c, **kw)
    for name, g, w, l, rows in zip(("dq", "dk", "dv", "dlog_alpha", "dS0"), got, want, limits, (True, True, True, True, False)):
        if g is not None:
            R.check(name, g, w, l, c.lens if rows else None)
    return got


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L", [1, 2, 8, 9, 63, 64, 65, 128, 200, 513])
def test_lengths(A, D, L):
    c = R.Case(2, 3, L, D, seed=L)
    check_forward(A, c)
    check_backward(A, c)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L,lens", [(5, [0, 1, 5, 3]), (70, [0, 1, 70, 64]), (300, [300, 0, 129, 192])])
@pytest.mark.parametrize("start", [False, True])
def test_ragged(A, D, L, lens, start):
    c = R.Case(4, 2, L, D, seed=L, lens=lens, start=start)
    check_forward(A, c)
    check_backward(A, c)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("gates", ["none", "one", "small", "resets"])
@pytest.mark.parametrize("L", [7, 150])
def test_gates(A, D, gates, L):
    c = R.Case(2, 3, L, D, seed=3, gates=gates)
    check_forward(A, c)
    dla = check_backward(A, c)[3]
    if gates == "resets":
        assert (dla.cpu()[torch.isinf(c.la)] == 0).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L", [4, 100])
def test_rows_as_they_are(A, D, L):
    c = R.Case(2, 3, L, D, seed=5, normalise=False, rows=0.3)
    check_forward(A, c)
    check_backward(A, c)


def test_rows_of_zeros(A):
    c = R.Case(1, 2, 100, 64, seed=6)
    for x in (c.q, c.k):
        x[0, 3:70:5] = 0
    check_forward(A, c)
    check_backward(A, c)


@pytest.mark.parametrize("D,H,L", [(128, 2, 3000), (64, 300, 140), (128, 520, 70), (64, 1, 2500)])
def test_many_segments_and_many_heads(A, D, H, L):
    """One stream of many segments, and more heads than there is room for at once; sampled heads."""
    full = R.Case(1, H, L, D, seed=H)
    out, S = R.run_forward(A, full)
    grads = R.run_backward(A, full)
    for h in sorted({0, H // 2, H - 1}):
        c = R.Case(1, 1, L, D, seed=1)
        for n in ("q", "k", "v", "do", "la"):
            setattr(c, n, getattr(full, n)[:, :, h:h + 1])
        c.S0, c.dS = full.S0[:, h:h + 1], full.dS[:, h:h + 1]
        w, ws, lo, ls = c.forward()
        R.check("out", out[:, :, h:h + 1], w, lo)
        R.check("S", S[:, h:h + 1], ws, ls)
        want, limits = c.backward()
        for name, g, x, l in zip(("dq", "dk", "dv", "dlog_alpha"), grads, want, limits):
            R.check(name, g[:, :, h:h + 1], x, l)
        R.check("dS0", grads[4][:, h:h + 1], want[4], limits[4])


@pytest.mark.parametrize("L", [1, 6, 90])
def test_state_in_place_and_not_wanted(A, L):
    c = R.Case(2, 2, L, 128, seed=8)
    out, S = R.run_forward(A, c)
    again, S2 = R.run_forward(A, c, in_place=True)
    assert torch.equal(out, again) and torch.equal(S, S2)
    none = torch.empty_like(out)
    ws = A.alloc_scan_workspace(c.B, c.H, c.L, c.D)
    A.arl2_scan_fwd(c.q.cuda(), c.k.cuda(), c.v.cuda(), c.la.cuda(), c.S0.cuda(), none, None, workspace=ws)
    assert torch.equal(none, out)


def test_gradients_that_are_not_wanted(A):
    c = R.Case(2, 2, 150, 64, seed=9)
    full = R.run_backward(A, c)
    for gates in (False, True):
        for start in (False, True):
            got = R.run_backward(A, c, want_gates=gates, want_start=start)
            for x, y in zip(got, full):
                assert x is None or torch.equal(x, y)


def test_token_by_token_is_the_whole(A):
    """A prompt, then single tokens in place, against one call over all of them."""
    c = R.Case(2, 3, 140, 128, seed=11)
    out, S, lo, ls = c.forward()
    dev = [x.cuda() for x in (c.q, c.k, c.v, c.la)]
    state = c.S0.cuda()
    got = torch.empty_like(dev[0])

    def part(a, b):
        o = torch.empty_like(got[:, a:b].contiguous())
        A.arl2_scan_fwd(*(x[:, a:b].contiguous() for x in dev), state, o, state, workspace=A.alloc_scan_workspace(2, 3, b - a, 128))
        got[:, a:b] = o

    part(0, 100)
    for t in range(100, 134):
        part(t, t + 1)
    part(134, 140)
    R.check("out", got, out, lo + R.U16 * np.abs(out))
    R.check("S", state, S, 2 * ls)


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_what_a_bad_row_reaches(A, bad):
    """Nothing before its block of 64 tokens, no other head or stream, nothing where it lies behind the sequence."""
    for at, lens in ((130, [200, 200]), (150, [140, 200])):
        c = R.Case(2, 2, 200, 64, seed=12, lens=lens)
        clean, cs = R.run_forward(A, c)
        grads = R.run_backward(A, c)
        for x in (c.q, c.k, c.v, c.do):
            x[0, at, 1, 5] = bad
        got, gs = R.run_forward(A, c)
        g2 = R.run_backward(A, c)
        if at >= lens[0]:
            assert torch.equal(got, clean) and torch.equal(gs, cs)
            assert all(torch.equal(x, y) for x, y in zip(g2, grads))
            continue
        assert torch.equal(got[:, :128], clean[:, :128]) and torch.equal(got[1], clean[1]) and torch.equal(got[0, :, 0], clean[0, :, 0])
        assert not torch.isfinite(got[0, at, 1].float()).all() and not torch.isfinite(gs[0, 1]).all()
        assert all(torch.equal(x[1], y[1]) for x, y in zip(g2, grads))


def test_a_reset_forgets_infinite_gates_sums(A):
    """A gate of zero, and gates beside it whose product underflows."""
    c = R.Case(1, 2, 130, 64, seed=13)
    c.la[0, 40:60] = -80.0
    c.la[0, 60] = -float("inf")
    c.la[0, 61:90] = -1e-4
    c.la[0, 100] = -3000.0
    check_forward(A, c)
    check_backward(A, c)


def test_repeats_bit_for_bit_and_streams(A):
    c = R.Case(3, 5, 700, 128, seed=14)
    first, grads = R.run_forward(A, c), R.run_backward(A, c)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        second, grads2 = R.run_forward(A, c), R.run_backward(A, c)
    third = R.run_forward(A, c, stream=side.cuda_stream)
    for x, y in zip((*first, *grads), (*second, *grads2)):
        assert torch.equal(x, y)
    assert all(torch.equal(x, y) for x, y in zip(first, third))


def test_captured_and_replayed(A):
    """A step of training and single tokens in one graph, replayed on new inputs beside eager work."""
    c = R.Case(2, 2, 300, 64, seed=15)
    t = {n: getattr(c, n).cuda() for n in ("q", "k", "v", "la", "S0", "do", "dS")}
    out, S = torch.empty_like(t["q"]), torch.empty_like(t["S0"])
    rows, dla, dS0 = [torch.empty_like(t["q"]) for _ in range(3)], torch.empty_like(t["la"]), torch.empty_like(t["S0"])
    one = [t[n][:, :1].contiguous() for n in ("q", "k", "v", "la")]
    o1 = torch.empty_like(one[0])
    lens = torch.tensor([300, 210], dtype=torch.int32, device="cuda")
    ws, wb = A.alloc_scan_workspace(2, 2, 300, 64), A.alloc_scan_workspace(2, 2, 300, 64, backward=True)

    def step():
        A.arl2_scan_fwd(t["q"], t["k"], t["v"], t["la"], t["S0"], out, S, seq_len=lens, workspace=ws)
        A.arl2_scan_fwd(*one, S, o1, S)
        A.arl2_scan_bwd(t["q"], t["k"], t["v"], t["la"], t["S0"], t["do"], t["dS"], *rows, dla, dS0, seq_len=lens, workspace=wb)

    written = (out, S, o1, *rows, dla, dS0)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(3):
        for n in ("q", "v", "do"):
            t[n].copy_(torch.randn_like(t[n]))
        lens.copy_(torch.tensor([300 - 64 * i, 100 + i], dtype=torch.int32))
        for x in written:
            x.zero_()
        step()
        torch.cuda.synchronize()
        want = [x.clone() for x in written]
        for x in written:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(written, want)), i


def test_gradients_against_differences(A):
    """The fp64 forward along random directions of every argument, against the kernels' gradients."""
    c = R.Case(1, 2, 90, 64, seed=16)
    grads = [R.wide(x) for x in R.run_backward(A, c)]
    g = np.random.Generator(np.random.Philox(17))
    names = ("q", "k", "v", "la", "S0")

    def value():
        out, S, _, _ = c.forward()
        return (out * R.wide(c.do)).sum() + (S * c.dS.numpy().astype(np.float64)).sum()

    for name, grad in zip(names, grads):
        x = getattr(c, name)
        d = g.standard_normal(tuple(x.shape))
        h = 2.0 ** -12
        vals = []
        for s in (1, -1):
            moved = torch.from_numpy(R.wide(x) + s * h * d)        # in fp64: no rounding of the step
            setattr(c, name, moved)
            c_wide, R.wide = R.wide, lambda t: t.detach().cpu().to(torch.float64).numpy()
            try:
                vals.append(value())
            finally:
                R.wide = c_wide
        setattr(c, name, x)
        got = (vals[0] - vals[1]) / (2 * h)
        want = (grad * d).sum()
        # gradients rounded to bf16 (rows) or off by 2^-14 (others), and the step's third order
        scale = U = np.linalg.norm(grad) * (R.U16 if name in "qkv" else 2.0 ** -14) * 4
        assert abs(got - want) <= scale + 1e-4 * abs(want), (name, got, want, U)
