"""The linear branch as a causal recurrence over tokens and the rotation of its queries and keys, as measurable cases.

    scan    S_t = a_t S_{t-1} + k'_t^T v_t, out_t = q'_t S_t for t = 1 .. L, with k' = L2Norm(k), q' = L2Norm(q) (Eq. (3) of the
            paper; or the rows as they are) and a gate a_t = exp(log_alpha_t) for each token and head
    grad    the gradients of a scan
    rope    queries and keys divided by their root mean square (of a head's features, of a token's whole row, or not at all), times
            a weight, and rotated by positions on one or several axes
    unrope  the gradients of that

    own               whether run() calls the package's kernels or computes the plain form
    listed()          the cases that are always measured
    draw(rng)         one more case from the ranges that the listed ones stand for
    prepare(case, s)  what the user's program holds before the call, on the GPU, from the seed alone
    run(state)        one pass
    work(case)        bytes and operations that the pass cannot do without
    exact(case, s)    the outputs from the definition, in 64 bits
"""
import math

import torch

own = False


def listed():
    return [
        # One more token for each of many streams, the states updated in place: latency.
        dict(name="scan_token", kind="scan", B=16, H=12, D=128, L=1, norm=True, start=True, resets=False, ragged=False),
        # One latent frame of one stream behind what came before.
        dict(name="scan_frame", kind="scan", B=1, H=12, D=128, L=1560, norm=True, start=True, resets=False, ragged=False),
        # A whole video of 21 frames, one stream.
        dict(name="scan_video", kind="scan", B=1, H=12, D=128, L=32760, norm=True, start=False, resets=False, ragged=False),
        # Narrow heads, sequences of different lengths, rows as they are, states reset where a sequence's scenes begin.
        dict(name="scan_ragged", kind="scan", B=5, H=24, D=64, L=2999, norm=False, start=True, resets=True, ragged=True),
        # A training batch: more streams and heads than the chip has room for at once.
        dict(name="scan_batch", kind="scan", B=16, H=16, D=128, L=4096, norm=True, start=False, resets=False, ragged=False),
        # The gradients of one latent frame.
        dict(name="grad_frame", kind="grad", B=1, H=12, D=128, L=1560, norm=True, start=True, resets=False, ragged=False),
        # The gradients of sequences of different lengths, narrow heads.
        dict(name="grad_ragged", kind="grad", B=5, H=24, D=64, L=999, norm=False, start=True, resets=True, ragged=True),
        # The gradients of a training batch: a chunk of three latent frames for each of eight streams.
        dict(name="grad_batch", kind="grad", B=8, H=12, D=128, L=4680, norm=True, start=False, resets=False, ragged=False),
        # A chunk's queries and keys, normalised over the whole row, rotated by frame, row and column.
        dict(name="rope_chunk", kind="rope", B=1, H=12, Hk=12, D=128, L=4680, axes=3, halves=False, norm="row", bits=16, ragged=False),
        # Long sequences, four query heads to a key head, normalised head by head, one axis.
        dict(name="rope_long", kind="rope", B=4, H=32, Hk=8, D=128, L=10920, axes=1, halves=True, norm="head", bits=16, ragged=False),
        # The gradients of the chunk's rotation, with those of the weights.
        dict(name="unrope_chunk", kind="unrope", B=1, H=12, Hk=12, D=128, L=4680, axes=3, halves=False, norm="row", bits=16, ragged=False),
        # Gradients in single precision, narrow heads, sequences of different lengths.
        dict(name="unrope_ragged", kind="unrope", B=6, H=24, Hk=8, D=64, L=1777, axes=2, halves=True, norm="head", bits=32, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Counts are spread over their logarithm; a drawn case asks for less work than the largest listed one of its kind."""
    most = {"scan": 16 * 4096 * 16 * 128, "grad": 8 * 4680 * 12 * 128, "rope": 4 * 10920 * 40 * 128, "unrope": 4680 * 24 * 128}
    while True:
        c = dict(kind=rng.choice(("scan", "scan", "grad", "grad", "rope", "unrope")), B=_log_int(rng, 1, 64),
                 H=rng.choice((1, 2, 3, 5, 8, 12, 16)), D=rng.choice((64, 128, 128)), ragged=rng.random() < 0.4)
        heads = c["H"]
        if c["kind"] in ("scan", "grad"):
            c["L"] = rng.choice((_log_int(rng, 1, 64), _log_int(rng, 64, 32760)))
            c.update(norm=rng.random() < 0.6, start=rng.random() < 0.5, resets=rng.random() < 0.3)
        else:
            c["L"] = _log_int(rng, 1, 32760)
            c.update(Hk=c["H"], axes=rng.choice((1, 2, 3)), halves=rng.random() < 0.5, norm=rng.choice(("row", "head", "none")),
                     bits=rng.choice((16, 16, 32)))
            c["H"] *= rng.choice((1, 1, 4))
            heads = c["H"] + c["Hk"]
        if c["B"] * c["L"] * heads * c["D"] <= most[c["kind"]] and c["B"] * c["H"] <= 512:
            return c


def _lengths(case):
    """Tokens of each stream."""
    if not case["ragged"]:
        return [case["L"]] * case["B"]
    return [max(1, min(case["L"], int(round(case["L"] * ((0.5 + 0.6180339887 * b) % 1.0) + 0.5)))) for b in range(case["B"])]


def _axis_pairs(case):
    """Pairs that each axis rotates; with two axes some features are left as they are."""
    half = case["D"] // 2
    return {1: [half], 2: [half // 4, half // 2 - 3], 3: [half - 2 * (half // 3), half // 3, half // 3]}[case["axes"]]


_THETA = {1: [500000.0], 2: [10000.0, 100.0], 3: [10000.0] * 3}


def prepare(case, seed):
    B, L, H, D = case["B"], case["L"], case["H"], case["D"]
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape, dtype=torch.bfloat16, scale=1.0):
        return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)

    s = dict(case=case, len=torch.tensor(_lengths(case), dtype=torch.int32, device="cuda") if case["ragged"] else None)
    if case["kind"] in ("rope", "unrope"):
        t = torch.bfloat16 if case["bits"] == 16 else torch.float32
        shapes = ((B, L, H, D), (B, L, case["Hk"], D))
        s["x"] = [normal(*n, dtype=t) for n in shapes]
        s["w"] = [None, None]
        if case["norm"] != "none":
            s["w"] = [(1.0 + normal(n[2] * D if case["norm"] == "row" else D, dtype=torch.float32, scale=0.2)).to(t) for n in shapes]
        l = torch.arange(L, device="cuda")
        grid = torch.stack((l // 1560, (l // 52) % 30, l % 52), 1)          # frame, row and column of a 30 x 52 grid
        if case["axes"] == 1:                                               # places in texts, far ones among them
            grid = l[None, :, None] + torch.randint(0, 120000, (B, 1, 1), generator=g, device="cuda")
        s["pos"] = grid[..., 3 - case["axes"]:].to(torch.int32).contiguous() if case["axes"] > 1 else grid.to(torch.int32).contiguous()
        s["y"] = [torch.zeros_like(x) for x in s["x"]]
        if case["kind"] == "unrope":
            s["dy"] = [normal(*n, dtype=t) for n in shapes]
            s["dw"] = [None if w is None else torch.zeros(w.shape, device="cuda") for w in s["w"]]
            if own:      # the scratch that a training program keeps for its calls of these sizes
                import paper_2605_16579_amd as A
                s["ws"] = A.alloc_rope_workspace(B, H, case["Hk"], L, D)
        return s
    row = 1.0 if case["norm"] else D ** -0.5
    s["q"], s["k"], s["v"] = normal(B, L, H, D, scale=row), normal(B, L, H, D, scale=row), normal(B, L, H, D)
    # gates as a sigmoid gives them: from head to head a memory of a few to about a thousand tokens
    z = 1.5 + 5.5 * torch.arange(H, device="cuda") / max(1, H - 1) + normal(B, L, H, dtype=torch.float32, scale=0.7)
    s["la"] = torch.nn.functional.logsigmoid(z)
    if case["resets"]:
        s["la"][torch.rand((B, L, H), generator=g, device="cuda") < 0.003] = -math.inf
    s["S0"] = normal(B, H, D, D, dtype=torch.float32, scale=0.5) if case["start"] else None
    if case["kind"] == "scan":
        s["out"] = torch.zeros_like(s["q"])
        s["S"] = s["S0"] if case["start"] and L <= 8 else torch.zeros((B, H, D, D), device="cuda")     # a few tokens: in place
    else:
        s["do"] = normal(B, L, H, D)
        s["dS"] = normal(B, H, D, D, dtype=torch.float32, scale=0.3) if case["start"] else None
        s["dq"], s["dk"], s["dv"] = (torch.zeros_like(s["q"]) for _ in range(3))
        s["dla"] = torch.zeros_like(s["la"])
        s["dS0"] = torch.zeros((B, H, D, D), device="cuda") if case["start"] else None
    if own:
        import paper_2605_16579_amd as A
        s["ws"] = A.alloc_scan_workspace(B, H, L, D, backward=case["kind"] == "grad")
    return s


def _there(s):
    """Which tokens there are, [B, L]."""
    L = s["case"]["L"]
    i = torch.arange(L, device="cuda")
    return (i < s["len"][:, None]) if s["len"] is not None else (i < L).expand(s["case"]["B"], L)


_BLOCK = 64


def _blocks(x, there):
    """[B, L, H, ...] with zeros where there is no token -> [B, H, blocks, tokens of a block, ...]."""
    x = torch.where(there.view(*there.shape, *[1] * (x.dim() - 2)), x, 0.0)
    pad = -x.shape[1] % _BLOCK
    x = torch.cat((x, x.new_zeros((x.shape[0], pad, *x.shape[2:]))), 1)
    return x.unflatten(1, (-1, _BLOCK)).movedim(3, 1)


def _unblock(x, old, there):
    x = x.movedim(1, 3).flatten(1, 2)[:, :old.shape[1]]
    old.copy_(torch.where(there.view(*there.shape, *[1] * (old.dim() - 2)), x.to(old.dtype), old))
    return old


def _plain_parts(s):
    """What a scan and its gradients share: the blocks' rows, their decays, the states that blocks begin with."""
    there, norm = _there(s), s["case"]["norm"]

    def rows(x):
        x = x.float()
        return _blocks(x / torch.sqrt((x * x).sum(-1, keepdim=True) + 1e-6) if norm else x, there)

    q, k, v = rows(s["q"]), rows(s["k"]), _blocks(s["v"].float(), there)
    c = _blocks(s["la"].double().clamp(min=-1e4), there).cumsum(-1)          # exp(-1e4) is zero
    lower = torch.ones((_BLOCK, _BLOCK), dtype=torch.bool, device="cuda").tril()
    p = dict(there=there, q=q, k=k, v=v, decay=torch.where(lower, (c[..., :, None] - c[..., None, :]).clamp(max=0.0).exp(), 0.0).float(),
             first=c.exp().float()[..., None], last=(c[..., -1:] - c).exp().float()[..., None])
    # from the end of block m to the beginning of block n > m: the blocks between them; from the first state: all before n
    total = torch.cat((torch.zeros_like(c[..., :1, -1]), c[..., -1].cumsum(-1)), -1)             # [B, H, blocks + 1]
    n = total.shape[-1]
    i = torch.arange(n, device="cuda")
    span = (total[..., :, None] - total[..., None, 1:]).clamp(max=0.0).exp()                      # [n, m]: begin n, end of m
    p["span"] = torch.where(i[:, None] > i[None, :-1], span, 0.0).float()
    p["whole"] = total.exp().float()
    own_sum = torch.matmul((k * p["last"]).transpose(-1, -2).contiguous(), v)                     # [B, H, blocks, D, D]
    states = torch.matmul(p["span"], own_sum.flatten(-2)).unflatten(-1, own_sum.shape[-2:])
    if s["S0"] is not None:
        states = states + p["whole"][..., None, None] * s["S0"][:, :, None]
    p["states"] = states                                                                          # [B, H, blocks + 1, D, D]
    return p


def _plain_scan(s):
    p = _plain_parts(s)
    scores = torch.matmul(p["q"], p["k"].transpose(-1, -2).contiguous()) * p["decay"]
    out = torch.matmul(scores, p["v"]) + torch.matmul(p["q"], p["states"][:, :, :-1]) * p["first"]
    _unblock(out, s["out"], p["there"])
    s["S"].copy_(p["states"][:, :, -1])
    return [s["out"], s["S"]]


def _plain_grad(s):
    p = _plain_parts(s)
    q, k, v, S = p["q"], p["k"], p["v"], p["states"][:, :, :-1]
    do = _blocks(s["do"].float(), p["there"])

    def t(x):
        return x.transpose(-1, -2).contiguous()

    # gradients of the states that blocks end with
    own_sum = torch.matmul(t(q * p["first"]), do)
    back = t(p["span"])
    # span[n, m]: from the end of block m to the beginning of block n; a block's gradient of its beginning reaches the ends before it
    R = torch.matmul(back[..., :, :-1], own_sum.flatten(-2)).unflatten(-1, own_sum.shape[-2:])
    dS0 = torch.matmul(p["whole"][..., None, :-1], own_sum.flatten(-2)).unflatten(-1, own_sum.shape[-2:])[:, :, 0]
    if s["dS"] is not None:
        R = R + back[..., -1][..., None, None] * s["dS"][:, :, None]
        dS0 = dS0 + p["whole"][..., -1][..., None, None] * s["dS"]
    A = torch.matmul(q, t(k)) * p["decay"]
    Bm = torch.matmul(do, t(v)) * p["decay"]
    dq_in, dk_in = torch.matmul(do, t(S)) * p["first"], torch.matmul(v, t(R)) * p["last"]
    dq, dk = torch.matmul(Bm, k) + dq_in, torch.matmul(t(Bm), q) + dk_in
    dv = torch.matmul(t(A), do) + torch.matmul(k, R) * p["last"]
    # a gate's gradient: the pairs of tokens on either side of it, in its block and beyond
    pairs = torch.matmul(q, t(k)).double() * Bm
    pairs = pairs.cumsum(-1) - pairs
    pairs = pairs.flip(-2).cumsum(-2).flip(-2).diagonal(dim1=-2, dim2=-1)
    a, b = (q * dq_in).sum(-1).double(), (k * dk_in).sum(-1).double()
    whole = (S.double() * R).sum((-1, -2)) * (p["first"][..., -1, 0].double())
    dla = pairs + a.flip(-1).cumsum(-1).flip(-1) + b.cumsum(-1) - b + whole[..., None]
    if s["case"]["norm"]:
        for name, r, d in (("q", q, dq), ("k", k, dk)):
            x = _blocks(s[name].float(), p["there"])
            d.sub_(r * (r * d).sum(-1, keepdim=True)).div_(torch.sqrt((x * x).sum(-1, keepdim=True) + 1e-6))
    got = [_unblock(x, s[n], p["there"]) for x, n in ((dq, "dq"), (dk, "dk"), (dv, "dv"), (dla, "dla"))]
    if s["dS0"] is not None:
        got.append(s["dS0"].copy_(dS0))
    return got


def _turns(s):
    """Cosines and sines [L or B, L, 1, pairs] of all pairs, in fp32 from angles in fp64, and how many pairs there are."""
    angles = [s["pos"][..., a, None].double() * th ** (-torch.arange(m, device="cuda").double() / m)
              for a, (m, th) in enumerate(zip(_axis_pairs(s["case"]), _THETA[s["case"]["axes"]]))]
    angle = torch.cat(angles, -1).unsqueeze(-2)
    return angle.cos().float(), angle.sin().float(), angle.shape[-1]


def _rotate(x, cos, sin, n, halves):
    """The pairs (i, i + D/2) or (2i, 2i + 1) for i < n turned, the others as they are."""
    D = x.shape[-1]
    x0, x1 = (x[..., :D // 2], x[..., D // 2:]) if halves else (x[..., 0::2], x[..., 1::2])
    a, b = x0[..., :n], x1[..., :n]
    x0 = torch.cat((a * cos - b * sin, x0[..., n:]), -1)
    x1 = torch.cat((a * sin + b * cos, x1[..., n:]), -1)
    return torch.cat((x0, x1), -1) if halves else torch.stack((x0, x1), -1).flatten(-2)


def _normalised(x, norm):
    """x over its root mean square, and 1 over that."""
    if norm == "none":
        return x, torch.ones_like(x[..., :1])
    m = (x * x).mean((-1, -2) if norm == "row" else -1, keepdim=True)
    r = torch.rsqrt(m + 1e-6)
    return x * r, r


def _plain_rope(s):
    case = s["case"]
    cos, sin, n = _turns(s)
    keep = _there(s)[..., None, None]
    for x, w, y in zip(s["x"], s["w"], s["y"]):
        z, _ = _normalised(x.float(), case["norm"])
        if w is not None:
            z = z * w.float().view(*((x.shape[2], -1) if case["norm"] == "row" else (-1,)))
        y.copy_(torch.where(keep, _rotate(z, cos, sin, n, case["halves"]).to(y.dtype), y))
    return s["y"]


def _plain_unrope(s):
    case = s["case"]
    cos, sin, n = _turns(s)
    keep = _there(s)[..., None, None]
    for x, w, dy, dw, y in zip(s["x"], s["w"], s["dy"], s["dw"], s["y"]):
        z = _rotate(dy.float(), cos, -sin, n, case["halves"])
        xh, r = _normalised(x.float(), case["norm"])
        d = z
        if w is not None:
            dw.copy_(torch.where(keep, z * xh, 0.0).sum((0, 1) if case["norm"] == "row" else (0, 1, 2)).view_as(dw))
            d = z * w.float().view(*((x.shape[2], -1) if case["norm"] == "row" else (-1,)))
        if case["norm"] != "none":
            d = r * (d - xh * (d * xh).mean((-1, -2) if case["norm"] == "row" else -1, keepdim=True))
        y.copy_(torch.where(keep, d.to(y.dtype), y))
    return [*s["y"], *s["dw"]]


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        import paper_2605_16579_amd as A
        if kind == "scan":
            A.arl2_scan_fwd(s["q"], s["k"], s["v"], s["la"], s["S0"], s["out"], s["S"], seq_len=s["len"], normalise=case["norm"], workspace=s["ws"])
            return [s["out"], s["S"]]
        if kind == "grad":
            A.arl2_scan_bwd(s["q"], s["k"], s["v"], s["la"], s["S0"], s["do"], s["dS"], s["dq"], s["dk"], s["dv"], s["dla"], s["dS0"],
                            seq_len=s["len"], normalise=case["norm"], workspace=s["ws"])
            return [s["dq"], s["dk"], s["dv"], s["dla"]] + ([s["dS0"]] if s["dS0"] is not None else [])
        how = dict(axis_pairs=_axis_pairs(case), theta=_THETA[case["axes"]], halves=case["halves"], norm=case["norm"], seq_len=s["len"])
        if kind == "rope":
            A.arl2_rope_fwd(*s["x"], *s["w"], s["pos"], *s["y"], **how)
            return s["y"]
        A.arl2_rope_bwd(*s["x"], *s["w"], s["pos"], *s["dy"], *s["y"], *s["dw"], workspace=s["ws"], **how)
        return [*s["y"], *s["dw"]]
    return {"scan": _plain_scan, "grad": _plain_grad, "rope": _plain_rope, "unrope": _plain_unrope}[kind](s)


def work(case):
    B, H, D, n = case["B"], case["H"], case["D"], sum(_lengths(case))
    if case["kind"] in ("rope", "unrope"):
        rows, w = n * (H + case["Hk"]) * D, case["bits"] // 8
        positions = case["axes"] * 4 * (n if case["axes"] == 1 else case["L"])
        return {"bytes": rows * w * (2 if case["kind"] == "rope" else 3) + positions, "flops": rows * (7 if case["kind"] == "rope" else 14)}
    rows, state = n * H, B * H * D * D * 4
    if case["kind"] == "scan":
        return {"bytes": rows * (4 * D * 2 + 4) + state * (1 + case["start"]), "flops": rows * 4 * D * D}
    return {"bytes": rows * (7 * D * 2 + 8) + state * 3 * case["start"], "flops": rows * 10 * D * D}


def _exact_scan(case, s):
    """The recurrence token by token."""
    B, L, H, D = case["B"], case["L"], case["H"], case["D"]
    n = torch.tensor(_lengths(case), device="cuda")

    def unit(x):
        x = x.double()
        return x * torch.rsqrt(x.square().sum(-1, keepdim=True) + 1e-6) if case["norm"] else x

    q, k, v, gate = unit(s["q"]), unit(s["k"]), s["v"].double(), s["la"].double().exp()
    after = torch.arange(L, device="cuda")[None] >= n[:, None]
    # a token that is not there changes nothing and has no output
    gate[after] = 1.0
    q[after], k[after], v[after] = 0.0, 0.0, 0.0
    S = torch.zeros((B, H, D, D), dtype=torch.float64, device="cuda") if s["S0"] is None else s["S0"].double()

    def steps(S, order, first, second, read, transposed):
        """S <- gate S + first^T second, rows read S (or its transpose); the gate before or behind the sum as `order` runs."""
        got = torch.zeros_like(q)
        for i in order:
            S.mul_(gate[:, i, :, None, None]).addcmul_(first[:, i, :, :, None], second[:, i, :, None, :])
            got[:, i] = (S * read[:, i, :, None, :]).sum(-1) if transposed else (S * read[:, i, :, :, None]).sum(-2)
        return got

    if case["kind"] == "scan":
        out = steps(S, range(L), k, v, q, False)
        return [out, S]
    do = s["do"].double()
    do[after] = 0.0
    dq = steps(S, range(L), k, v, do, True)
    G = torch.zeros((B, H, D, D), dtype=torch.float64, device="cuda") if s["dS"] is None else s["dS"].double()
    E = (S * G).sum((-1, -2))
    dk, dv, dla = torch.zeros_like(q), torch.zeros_like(q), torch.zeros((B, L, H), dtype=torch.float64, device="cuda")
    for i in reversed(range(L)):
        G.addcmul_(q[:, i, :, :, None], do[:, i, :, None, :])
        dk[:, i] = (G * v[:, i, :, None, :]).sum(-1)
        dv[:, i] = (G * k[:, i, :, :, None]).sum(-2)
        E = E + (q[:, i] * dq[:, i]).sum(-1) - (k[:, i] * dk[:, i]).sum(-1)
        E = torch.where(gate[:, i] == 0.0, 0.0, E)
        dla[:, i] = E
        G.mul_(gate[:, i, :, None, None])
    dla[after] = 0.0
    if case["norm"]:
        for x, r, d in ((s["q"], q, dq), (s["k"], k, dk)):
            d.sub_(r * (r * d).sum(-1, keepdim=True)).mul_(torch.rsqrt(x.double().square().sum(-1, keepdim=True) + 1e-6))
    return [dq, dk, dv, dla] + ([G] if s["dS0"] is not None else [])


def _exact_rope(case, s):
    """Features as complex numbers; the gradients by the adjoints of the three steps."""
    B, L, D = case["B"], case["L"], case["D"]
    there = torch.arange(L, device="cuda")[None] < torch.tensor(_lengths(case), device="cuda")[:, None]
    turn = torch.ones((*s["pos"].shape[:-1], D // 2), dtype=torch.complex128, device="cuda")
    at = 0
    for a, (m, th) in enumerate(zip(_axis_pairs(case), _THETA[case["axes"]])):
        angle = s["pos"][..., a, None].double() * torch.exp(-math.log(th) * torch.arange(m, device="cuda").double() / m)
        turn[..., at:at + m] = torch.polar(torch.ones_like(angle), angle)
        at += m
    turn = turn.expand(B, L, D // 2)[:, :, None]

    def to(x):
        return torch.complex(x[..., :D // 2].contiguous(), x[..., D // 2:].contiguous()) if case["halves"] else torch.complex(x[..., ::2].contiguous(), x[..., 1::2].contiguous())

    def back(z):
        return torch.cat((z.real, z.imag), -1) if case["halves"] else torch.view_as_real(z).flatten(-2)

    ys, dws = [], []
    for i in range(2):
        x = s["x"][i].double()
        over = (2, 3) if case["norm"] == "row" else (3,)
        size = case["D"] * (x.shape[2] if case["norm"] == "row" else 1)
        r = torch.ones_like(x[..., :1]) if case["norm"] == "none" else (x.square().sum(over, keepdim=True) / size + 1e-6) ** -0.5
        w = 1.0 if s["w"][i] is None else s["w"][i].double().view(1, 1, -1, D)
        if case["kind"] == "rope":
            ys.append(torch.where(there[..., None, None], back(to(x * r * w) * turn), 0.0))
            continue
        z = torch.where(there[..., None, None], back(to(s["dy"][i].double()) * turn.conj()), 0.0)
        if s["w"][i] is not None:
            dw = (z * x * r).sum((0, 1))
            dws.append(dw.flatten() if case["norm"] == "row" else dw.sum(0))
        z = z * w
        ys.append(z if case["norm"] == "none" else r * z - x * r ** 3 * ((z * x).sum(over, keepdim=True) / size))
    return ys + dws


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_rope(case, s) if case["kind"] in ("rope", "unrope") else _exact_scan(case, s)
