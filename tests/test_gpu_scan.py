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
        assert np.linalg.norm(R.wide(got)[there] - out[there]) <= R.U16 * np.linalg.norm(out[there]) + R.TINY * out[there].size ** 0.5
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


@pytest.mark.parametrize("gate", [None, -0.4, -0.65, -3.0])
@pytest.mark.parametrize("normalise,rows", [(True, 2.0 ** 13), (True, 2.0 ** -50), (False, 2.0 ** 13), (False, 2.0 ** -25)])
def test_large_and_small_rows(A, normalise, rows, gate):
    """Decays are taken out of rows and states, up to 2^60 of a block here: what they are multiplied with in between has room."""
    for L in (5, 200):
        c = R.Case(1, 3, L, 64, seed=23, normalise=normalise, rows=rows, start=False)
        if gate is not None:
            c.la[:] = gate
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


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("B,H,L,lens", [(1, 2, 9, None), (2, 3, 65, [65, 1]), (3, 2, 130, [0, 130, 70]), (2, 12, 1560, [1560, 33])])
def test_what_a_call_before_left_in_fast_memory(A, D, B, H, L, lens):
    """Results behind calls on rows of NaNs are the same bits."""
    bad = torch.full((64, 200, 12, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    out, ws = torch.empty_like(bad), A.alloc_scan_workspace(64, 12, 200, 128)
    c = R.Case(B, H, L, D, seed=L, lens=lens)
    first = (*R.run_forward(A, c), *R.run_backward(A, c))
    A.arl2_scan_fwd(bad, bad, bad, None, None, out, None, workspace=ws)
    second = R.run_forward(A, c)
    A.arl2_scan_fwd(bad, bad, bad, None, None, out, None, workspace=ws)
    for x, y in zip(first, (*second, *R.run_backward(A, c))):
        assert torch.equal(x, y)


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


@pytest.mark.parametrize("eps", [1e-12, 1e-3, 4.0])
@pytest.mark.parametrize("L", [5, 140])
def test_epsilons(A, monkeypatch, eps, L):
    monkeypatch.setattr(R, "EPS", float(np.float32(eps)))
    c = R.Case(2, 2, L, 64, seed=18, rows=0.05)
    check_forward(A, c, l2_eps=eps)
    check_backward(A, c, l2_eps=eps)


@pytest.mark.parametrize("L", [6, 130])
def test_gates_above_one_are_one_and_lengths_are_cut(A, L):
    c = R.Case(3, 2, L, 64, seed=19, lens=[0, L, L])
    c.la[:, ::3] = 0.7
    given = torch.tensor([-5, L + 9, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    c.lens_device = lambda: given
    check_forward(A, c)
    check_backward(A, c)


def test_two_calls_at_once(A):
    """Two streams, a workspace each, against the same calls one after the other."""
    cases = [R.Case(2, 4, 900, 128, seed=20), R.Case(3, 2, 700, 64, seed=21, lens=[700, 0, 333])]
    alone = [(*R.run_forward(A, c), *R.run_backward(A, c)) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    dev = [{n: getattr(c, n).cuda() for n in ("q", "k", "v", "la", "S0", "do", "dS")} for c in cases]
    lens = [c.lens_device() for c in cases]
    rows = [[torch.full_like(d["q"], 7.0) for _ in range(4)] for d in dev]
    states = [[torch.full_like(d["S0"], 7.0) for _ in range(2)] for d in dev]
    dla = [torch.full_like(d["la"], 7.0) for d in dev]
    ws = [[A.alloc_scan_workspace(c.B, c.H, c.L, c.D, backward=b) for b in (False, True)] for c in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        for i, s in enumerate(streams):
            d, r = dev[i], rows[i]
            with torch.cuda.stream(s):
                A.arl2_scan_fwd(d["q"], d["k"], d["v"], d["la"], d["S0"], r[0], states[i][0], seq_len=lens[i], workspace=ws[i][0])
                A.arl2_scan_bwd(d["q"], d["k"], d["v"], d["la"], d["S0"], d["do"], d["dS"], *r[1:], dla[i], states[i][1], seq_len=lens[i], workspace=ws[i][1])
    torch.cuda.synchronize()
    for i, (out, S, dq, dk, dv, g, dS0) in enumerate(alone):
        for x, y in zip((out, S, dq, dk, dv, g, dS0), (rows[i][0], states[i][0], *rows[i][1:], dla[i], states[i][1])):
            assert torch.equal(x, y), i


def test_offsets_past_32_bits(A):
    """Streams of 2 GB of rows each, of which the last one's end is looked at: gates of exp(-0.5) leave nothing of what lies 128 tokens back."""
    B, L, D, window, seen = 3, 8000037, 128, 384, 256
    g = torch.Generator(device="cuda").manual_seed(22)
    q, k, v, do = (torch.empty((B, L, 1, D), dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(4))
    la = torch.full((B, L, 1), -0.5, device="cuda")
    dS = torch.randn((B, 1, D, D), generator=g, device="cuda")
    out, rows, dla = torch.empty_like(q), [torch.empty_like(q) for _ in range(3)], torch.empty_like(la)
    S, dS0 = torch.empty_like(dS), torch.empty_like(dS)
    A.arl2_scan_fwd(q, k, v, la, None, out, S, workspace=A.alloc_scan_workspace(B, 1, L, D))
    A.arl2_scan_bwd(q, k, v, la, None, do, dS, *rows, dla, dS0, workspace=A.alloc_scan_workspace(B, 1, L, D, backward=True))
    c = R.Case(1, 1, window, D, start=False)
    for n, x in (("q", q), ("k", k), ("v", v), ("do", do), ("la", la)):
        setattr(c, n, x[-1:, -window:].cpu())
    c.dS = dS[-1:].cpu()
    want, state, lo, ls = c.forward()
    R.check("out", out[-1:, -seen:], want[:, -seen:], lo[:, -seen:])
    R.check("S", S[-1:], state, ls)
    for name, x, w, l in zip(("dq", "dk", "dv", "dlog_alpha"), (*rows, dla), *c.backward()):
        R.check(name, x[-1:, -seen:], w[:, -seen:], l[:, -seen:])
    for n, x in (("q", q), ("k", k), ("v", v), ("do", do), ("la", la)):
        setattr(c, n, x[-1:, :window].cpu())
    c.dS = None
    want, limits = c.backward()
    R.check("dS0", dS0[-1:], want[4], limits[4])


# ---- the binding's two ways

class Checked(torch.Tensor):
    """A tensor that is no plain torch.Tensor: a call with it is marshalled in Python."""


def test_compiled_and_checked_calls_agree(A, monkeypatch):
    from paper_2605_16579_amd import binding
    seen, host_call = [], binding._host_call

    def recorded(*args):
        seen.append(host_call(*args))
        return seen[-1]

    monkeypatch.setattr(binding, "_host_call", recorded)
    B, H, L, D = 2, 3, 90, 64
    q, k, v, do = (torch.randn((B, L, H, D), device="cuda").bfloat16() for _ in range(4))
    la, S0, dS = -torch.rand((B, L, H), device="cuda"), torch.randn((B, H, D, D), device="cuda"), torch.randn((B, H, D, D), device="cuda")
    lens = torch.tensor([90, 50], dtype=torch.int32, device="cuda")
    x, w, dy = torch.randn((B, L, 2, D), device="cuda").bfloat16(), torch.rand(D, device="cuda").bfloat16(), torch.randn((B, L, 2, D), device="cuda").bfloat16()
    pos = torch.randint(0, 99, (L, 2), dtype=torch.int32, device="cuda")
    ws, wr = A.alloc_scan_workspace(B, H, L, D, backward=True), A.alloc_rope_workspace(B, H, 2, L, D)
    how = dict(axis_pairs=[20, 12], theta=[500.0, 0], halves=True, norm="head", norm_eps=1e-3, seq_len=lens)

    def run(wrap, **kw):
        out, rows, yq, yk, dq, dk = torch.zeros_like(q), [torch.zeros_like(q) for _ in range(3)], torch.zeros_like(q), torch.zeros_like(x), torch.zeros_like(q), torch.zeros_like(x)
        S, dS0, dla, dw = torch.zeros_like(S0), torch.zeros_like(S0), torch.zeros_like(la), [torch.zeros(D, device="cuda") for _ in range(2)]
        A.arl2_scan_fwd(wrap(q), k, v, la, S0, out, S, seq_len=lens, normalise=False, l2_eps=1e-3, workspace=ws, **kw)
        A.arl2_scan_bwd(wrap(q), k, v, la, S0, do, dS, *rows, dla, dS0, seq_len=lens, l2_eps=1e-3, workspace=ws, **kw)
        A.arl2_rope_fwd(wrap(q), x, w, None, pos, yq, yk, **how, **kw)
        A.arl2_rope_bwd(wrap(q), x, w, None, pos, do, dy, dq, dk, *dw, workspace=wr, **how, **kw)
        torch.cuda.synchronize()
        return out, *rows, S, dS0, dla, yq, yk, dq, dk, *dw

    plain = run(lambda t: t)
    assert seen == [0] * 4
    seen.clear()
    checked = run(lambda t: t.as_subclass(Checked))
    assert seen == [None] * 4
    on_stream = run(lambda t: t, stream=torch.cuda.current_stream().cuda_stream)
    for a, b, c in zip(plain, checked, on_stream):
        assert torch.equal(a, b) and torch.equal(a, c) and a.any()
    # what the compiled way does not take is refused by the other
    out, S = torch.empty_like(q), torch.empty_like(S0)
    for bad in (dict(k=k[:, :-1].contiguous()), dict(v=v.float()), dict(la=la[..., None]), dict(la=la.double()), dict(S0=S0[:, :1].contiguous()), dict(out=out.transpose(1, 2)),
                dict(S=S.cpu()), dict(lens=lens.long()), dict(lens=lens[:1]), dict(q=q[0]), dict(workspace=ws.cpu())):
        a = dict(q=q, k=k, v=v, la=la, S0=S0, out=out, S=S, lens=lens, workspace=ws)
        a.update(bad)
        seen.clear()
        with pytest.raises((ValueError, TypeError)):
            A.arl2_scan_fwd(a["q"], a["k"], a["v"], a["la"], a["S0"], a["out"], a["S"], seq_len=a["lens"], workspace=a["workspace"])
        assert seen == [None], bad
    y, z = torch.empty_like(q), torch.empty_like(x)
    for bad in (dict(k=None), dict(z=None), dict(k=x[..., :32].contiguous()), dict(w=w.float()), dict(w=w.repeat(3)), dict(pos=pos.long()), dict(pos=pos[:, :1].contiguous()),
                dict(pos=pos[None].repeat(3, 1, 1)), dict(y=y.float()), dict(lens=lens.cpu()), dict(q=q[0]), dict(norm="layer"), dict(axis_pairs=[]), dict(theta=[1.0])):
        a = dict(q=q, k=x, w=w, pos=pos, y=y, z=z, lens=lens, norm="head", axis_pairs=[20, 12], theta=None)
        a.update(bad)
        seen.clear()
        with pytest.raises((ValueError, TypeError, A.Arl2Error)):
            A.arl2_rope_fwd(a["q"], a["k"], a["w"], None, a["pos"], a["y"], a["z"], seq_len=a["lens"], norm=a["norm"], axis_pairs=a["axis_pairs"], theta=a["theta"])
        assert seen == [None] or bad == dict(z=None), bad
    with pytest.raises(A.Arl2Error, match="workspace"):
        A.arl2_rope_bwd(q, x, w, None, pos, do, dy, y, z, torch.zeros(D, device="cuda"), None, workspace=wr[:-256], **how)
