"""The paged 4-bit key/value cache of a softmax layer, as measurable cases: appending to it, reading rows back, attending to it.

A layer that keeps softmax (Eq. (1) of the paper) holds the keys and values of everything generated so far.  Here they
lie in pages of a pool, in 4 bits (e2m1) with one power-of-two scale per 32 features of a (token, head) row:

    append    rotates the new keys by their positions' tables, quantises keys and values, writes them into their pages
    read      gives the values that stored rows stand for
    attend    softmax(q K^T / sqrt(D)) V over a stream's stored tokens, all of them or those up to the query's position

    own               whether run() calls the package's kernels or computes the plain form
    listed()          the cases that are always measured
    draw(rng)         one more case from the ranges that the listed ones stand for
    prepare(case, s)  what the user's program holds before the call, on the GPU, from the seed alone
    run(state)        one pass
    work(case)        bytes and operations that the pass cannot do without
    exact(case, s)    the outputs from the definition, in 64 bits

Bytes of a page and head, P tokens of D features: key codes [P][D/2], value codes [P/16][D/2][16 tokens], key scales
[P][D/32], value scales [P/16][D/32][16 tokens].  A byte of codes holds feature 2i in its low and 2i + 1 in its high
half; a scale byte x stands for 2^(x - 127).
"""
import math

import torch

own = False

# magnitudes of the codes 0 .. 7; code 8 + i is the negative of code i
_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # Single tokens appended for a batch of streams of different lengths: latency.
        dict(name="append_tokens", kind="append", B=16, H=12, D=128, L=1, page=64, top=4096, ragged=True),
        # A clean pass of the usual layer: one chunk of three latent frames behind the six chunks before it.
        dict(name="append_chunk", kind="append", B=1, H=12, D=128, L=4680, page=64, top=32760, ragged=False),
        # Narrow heads, small pages, streams that get different numbers of tokens at odd positions.
        dict(name="append_ragged", kind="append", B=8, H=24, D=64, L=999, page=16, top=5000, ragged=True),
        # The frame before last of four streams, read back to be committed to the linear memory.
        dict(name="read_frame", kind="read", B=4, H=12, D=128, L=1560, page=64, top=10920, ragged=False),
        # A few tokens of many streams of different lengths, narrow heads.
        dict(name="read_ragged", kind="read", B=32, H=24, D=64, L=77, page=32, top=3000, ragged=True),
        # The smallest attention there is in use: one token, a short history.
        dict(name="token_short", kind="attend", B=1, H=12, Hkv=12, D=128, L=1, page=16, top=199, causal=True, ragged=False),
        # One token over a long history, four query heads to a stored head.
        dict(name="token_long", kind="attend", B=1, H=32, Hkv=8, D=128, L=1, page=64, top=131001, causal=True, ragged=False),
        # A serving step: one token for each of many streams whose histories differ a hundredfold.
        dict(name="token_batch", kind="attend", B=64, H=32, Hkv=8, D=128, L=1, page=32, top=8192, causal=True, ragged=True),
        # A few tokens at once (drafts to be verified), narrow heads.
        dict(name="tokens_narrow", kind="attend", B=16, H=24, Hkv=12, D=64, L=5, page=16, top=4000, causal=True, ragged=True),
        # Frame-by-frame generation: one latent frame against seven, itself included.
        dict(name="frame", kind="attend", B=1, H=12, Hkv=12, D=128, L=1560, page=64, top=10920, causal=False, ragged=False),
        # The layer that keeps softmax at the end of a 21-frame video: a chunk against everything.
        dict(name="chunk", kind="attend", B=1, H=12, Hkv=12, D=128, L=4680, page=64, top=32760, causal=False, ragged=False),
        # Prompts of different lengths behind a stored beginning, causal, grouped heads.
        dict(name="prompt", kind="attend", B=3, H=16, Hkv=4, D=128, L=2222, page=128, top=6001, causal=True, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """Counts are spread over their logarithm; a drawn case asks for less work than the largest listed one of its kind."""
    while True:
        kind = rng.choice(("append", "read", "attend", "attend", "attend"))
        c = dict(kind=kind, B=_log_int(rng, 1, 64), H=rng.choice((2, 3, 5, 8, 12, 16)), D=rng.choice((64, 128, 128)),
                 page=rng.choice((16, 32, 64, 128, 256)), ragged=rng.random() < 0.5)
        if kind == "attend":
            c["Hkv"] = c["H"]
            c["H"] *= rng.choice((1, 1, 2, 4, 7))
            c["L"] = rng.choice((1, _log_int(rng, 2, 64), _log_int(rng, 64, 4680)))
            c["causal"] = c["L"] == 1 or rng.random() < 0.5
        else:
            c["L"] = _log_int(rng, 1, 4680)
        c["top"] = max(c["L"], _log_int(rng, 20, 130000))
        pairs = c["B"] * c["L"] * c["H"] * c["D"] * (c["top"] if kind == "attend" else 1)
        rows = c["B"] * c["top"] * c.get("Hkv", c["H"]) * c["D"]
        if rows <= 3 * 2 ** 27 and c["B"] * c["L"] * c["H"] * c["D"] <= 2 ** 25 and pairs <= 4680 * 32760 * 12 * 128:
            return c


def _lengths(case):
    """Per stream: tokens stored in the end, and those that the call appends, reads or asks about."""
    total, new = [], []
    for b in range(case["B"]):
        u = (0.5 + 0.6180339887 * b) % 1.0 if case["ragged"] else 1.0      # spread evenly over (0, 1)
        n = int(round(case["top"] ** u * min(case["L"], case["top"]) ** (1.0 - u) * (0.5 + 0.5 * u)))
        n = max(1, min(case["top"], n))
        total.append(n)
        new.append(max(1, min(n, int(round(case["L"] * (0.3 + 0.7 * u))))))
    return total, new


def _kv_heads(case):
    return case.get("Hkv", case["H"])


def _tables(positions, D):
    """Cosines and sines of a three-axis rotation over (latent frame, row, column) of a 30 x 52 grid of tokens."""
    l = torch.arange(positions, device="cuda")
    pos = torch.stack([l // 1560, (l // 52) % 30, l % 52], dim=1).double()
    half = D // 2
    n = half // 3
    ang = torch.cat([pos[:, a:a + 1] * (10000.0 ** (-torch.arange(m, device="cuda").double() / m))[None]
                     for a, m in enumerate((half - 2 * n, n, n))], dim=1)
    return ang.cos().float().contiguous(), ang.sin().float().contiguous()


def prepare(case, seed):
    B, H, D, L, P = case["B"], _kv_heads(case), case["D"], case["L"], case["page"]
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)

    total, new = _lengths(case)
    width = (max(total) + P - 1) // P                   # table entries per stream
    n_pages = B * width + 3
    order = torch.randperm(n_pages, generator=g, device="cuda")[:B * width].view(B, width)
    used = torch.arange(width, device="cuda")[None, :] * P < torch.tensor(total, device="cuda")[:, None]
    s = dict(case=case, table=torch.where(used, order, -1).to(torch.int32).contiguous(),
             total=torch.tensor(total, dtype=torch.int32, device="cuda"), new=torch.tensor(new, dtype=torch.int32, device="cuda"))
    s["start"] = s["total"] - s["new"]
    # What is stored: rows of normal values, quantised.  Codes and scales are drawn as such values have them (the largest of
    # 32 is 2.1 on the average, so the scale is 2^-2 or 2^-1); this fills any number of pages quickly.
    s["cache"] = torch.empty((n_pages, H, P, 2 * (D // 2 + D // 32)), dtype=torch.uint8, device="cuda")
    flat = s["cache"].view(n_pages, H, P * 2 * (D // 2 + D // 32))
    nc = 2 * P * (D // 2)
    flat[:, :, nc:] = torch.randint(125, 127, (n_pages, H, 2 * P * (D // 32)), generator=g, device="cuda", dtype=torch.uint8)
    drawn = _codes(torch.randn(1 << 22, generator=g, device="cuda") * 3.0)
    drawn = drawn[0::2] | (drawn[1::2] << 4)
    step = max(1, (1 << 28) // (H * nc))
    for p in range(0, n_pages, step):
        m = min(step, n_pages - p)
        flat[p:p + m, :, :nc] = drawn[torch.randint(0, drawn.numel(), (m, H, nc), generator=g, device="cuda")]
    if case["kind"] == "attend":
        s["q"], s["out"] = normal(B, L, case["H"], D), torch.zeros((B, L, case["H"], D), dtype=torch.bfloat16, device="cuda")
        if own:      # the scratch that a serving program keeps for its calls of these sizes
            import paper_2605_16579_amd as A
            s["ws"] = A.alloc_kv_workspace(B, case["H"], H, L, D, P, width)
        return s
    if case["kind"] == "append":
        s["k"], s["v"] = normal(B, L, H, D), normal(B, L, H, D)
        s["cos"], s["sin"] = _tables(width * P, D)
    s["k_out"], s["v_out"] = (torch.zeros((B, L, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    return s


def _codes(t):
    """e2m1 codes of values that are already divided by their scale: the nearest, ties to the even code, 6 at the most."""
    a = t.abs()
    c = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    return c.to(torch.uint8) | (t < 0).to(torch.uint8) << 3


def _power(e):
    """2^e for whole e in [-126, 127], exactly, in fp32."""
    return ((e + 127).to(torch.int32) << 23).view(torch.float32)


def _quantise(x):
    """fp32 rows [..., D] -> codes [..., D/2] and scales [..., D/32]."""
    groups = x.unflatten(-1, (-1, 32))
    bits = groups.abs().amax(-1).view(torch.int32)
    scale = (((bits + 0x1fffff) >> 23) - 2).clamp(7, 252)            # the least with no value beyond 7 times it
    c = _codes(groups.double() * _power(127 - scale)[..., None]).flatten(-2)
    return c[..., 0::2] | (c[..., 1::2] << 4), scale.to(torch.uint8)


def _dequantise(codes, scales):
    """The fp32 values of codes [..., D/2] with scales [..., D/32]."""
    value = torch.tensor(_VALUES + tuple(-v for v in _VALUES), device=codes.device)
    x = torch.stack((value[(codes & 15).long()], value[(codes >> 4).long()]), -1).flatten(-2).unflatten(-1, (-1, 32))
    return (x * _power(scales.int() - 127)[..., None]).flatten(-2)


def _parts(blocks, P, D):
    """Views of pages' bytes [..., bytes]: key codes [..., P, D/2], value codes, key scales [..., P, D/32], value scales."""
    kc, vc, ks, vs = blocks.split((P * (D // 2), P * (D // 2), P * (D // 32), P * (D // 32)), -1)
    return (kc.unflatten(-1, (P, D // 2)), vc.unflatten(-1, (P // 16, D // 2, 16)).transpose(-1, -2).flatten(-3, -2),
            ks.unflatten(-1, (P, D // 32)), vs.unflatten(-1, (P // 16, D // 32, 16)).transpose(-1, -2).flatten(-3, -2))


def _stored(s):
    """All rows of every stream, [B, tokens, H, D] each for keys and values, in fp32."""
    case = s["case"]
    P, D = case["page"], case["D"]
    blocks = s["cache"].flatten(2)[s["table"].clamp(min=0).long()]                   # [B, width, H, bytes]
    kc, vc, ks, vs = _parts(blocks, P, D)
    return tuple(_dequantise(c, x).transpose(2, 3).flatten(1, 2) for c, x in ((kc, ks), (vc, vs)))


def _token_index(s, L):
    """Positions [B, L] of the call's tokens, which of them there are, their pages and places there."""
    i = torch.arange(L, device="cuda")
    pos = (s["start"][:, None] + i).long()
    there = i < s["new"][:, None]
    pos = torch.where(there, pos, 0)
    P = s["case"]["page"]
    return pos, there, s["table"].long().gather(1, pos // P), pos % P


def _plain_append(s):
    case = s["case"]
    L, P, D = case["L"], case["page"], case["D"]
    pos, there, page, place = _token_index(s, L)
    c, n = s["cos"][pos].double()[:, :, None], s["sin"][pos].double()[:, :, None]
    x0, x1 = s["k"][..., 0::2].double(), s["k"][..., 1::2].double()
    rotated = torch.stack((x0 * c - x1 * n, x0 * n + x1 * c), -1).flatten(-2).float()
    kc, ks = _quantise(rotated)
    vc, vs = _quantise(s["v"].float())
    H = s["k"].shape[2]
    h = torch.arange(H, device="cuda")
    flat = s["cache"].flatten(2)
    b, i = there.nonzero(as_tuple=True)
    page, place = page[b, i][:, None, None], place[b, i][:, None, None]

    def put(first, row, values):          # row: offsets [tokens, 1 or H, n] behind `first`
        flat[page, h[None, :, None], first + row] = values

    d, r = torch.arange(D // 2, device="cuda"), torch.arange(D // 32, device="cuda")
    nc, ns = P * (D // 2), P * (D // 32)
    put(0, place * (D // 2) + d, kc[b, i])
    put(nc, (place // 16 * (D // 2) + d) * 16 + place % 16, vc[b, i])
    put(2 * nc, place * (D // 32) + r, ks[b, i])
    put(2 * nc + ns, (place // 16 * (D // 32) + r) * 16 + place % 16, vs[b, i])


def _plain_read(s):
    case = s["case"]
    pos, there, page, place = _token_index(s, case["L"])
    P, D = case["page"], case["D"]
    H = s["cache"].shape[1]
    h = torch.arange(H, device="cuda")[:, None]
    flat = s["cache"].flatten(2)
    page, place = page.clamp(min=0)[..., None, None], place[..., None, None]
    d, r = torch.arange(D // 2, device="cuda"), torch.arange(D // 32, device="cuda")
    nc, ns = P * (D // 2), P * (D // 32)
    k = _dequantise(flat[page, h, place * (D // 2) + d], flat[page, h, 2 * nc + place * (D // 32) + r])
    v = _dequantise(flat[page, h, nc + (place // 16 * (D // 2) + d) * 16 + place % 16],
                    flat[page, h, 2 * nc + ns + (place // 16 * (D // 32) + r) * 16 + place % 16])
    keep = there[..., None, None]
    s["k_out"].copy_(torch.where(keep, k, s["k_out"].float()))
    s["v_out"].copy_(torch.where(keep, v, s["v_out"].float()))


def _plain_attend(s):
    case = s["case"]
    B, L, H, D, Hkv = case["B"], case["L"], case["H"], case["D"], case["Hkv"]
    k, v = (x.transpose(1, 2).contiguous() for x in _stored(s))                      # [B, Hkv, tokens, D]
    q = s["q"].float().view(B, L, Hkv, H // Hkv, D).permute(0, 2, 1, 3, 4).flatten(2, 3)
    logits = torch.matmul(q, k.transpose(-1, -2).contiguous()) / math.sqrt(D)
    i = torch.arange(L, device="cuda")
    limit = s["total"][:, None].expand(B, L)
    if case["causal"]:
        limit = torch.minimum(limit, s["total"][:, None] - s["new"][:, None] + i + 1)
    limit = limit.repeat_interleave(H // Hkv, 1)[:, None, :, None]
    seen = torch.arange(k.shape[2], device="cuda") < limit
    logits.masked_fill_(~seen, -math.inf)
    top = logits.amax(-1, keepdim=True).clamp(min=-3e38)
    p = logits.sub_(top).exp_()
    o = torch.matmul(p, v) / p.sum(-1, keepdim=True)
    o = o.unflatten(2, (L, H // Hkv)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    s["out"].copy_(torch.where((i < s["new"][:, None])[..., None, None], o, s["out"].float()))


def run(s):
    kind = s["case"]["kind"]
    if own:
        import paper_2605_16579_amd as A
        if kind == "attend":
            A.arl2_kv_attn_fwd(s["q"], s["cache"], s["table"], s["total"], s["out"], q_len=s["new"], causal=s["case"]["causal"], workspace=s["ws"])
            return s["out"]
        if kind == "append":
            A.arl2_kv_append(s["k"], s["v"], s["cache"], s["table"], s["start"], count=s["new"], rope_cos=s["cos"], rope_sin=s["sin"])
        A.arl2_kv_read(s["cache"], s["table"], s["start"], s["k_out"], s["v_out"], count=s["new"])
        return [s["k_out"], s["v_out"]]
    if kind == "attend":
        _plain_attend(s)
        return s["out"]
    if kind == "append":
        _plain_append(s)
    _plain_read(s)           # what is stored comes back as the values that it stands for
    return [s["k_out"], s["v_out"]]


def work(case):
    B, D, H, Hkv = case["B"], case["D"], case["H"], _kv_heads(case)
    total, new = _lengths(case)
    row = 2 * (D // 2 + D // 32) * Hkv                      # a stored token, keys and values
    if case["kind"] == "attend":
        pairs = sum(n * t - (n * (n - 1) // 2 if case["causal"] else 0) for t, n in zip(total, new))
        return {"bytes": sum(total) * row + 2 * sum(new) * H * D * 2 + 4 * sum(-(-t // case["page"]) for t in total),
                "flops": 4 * pairs * H * D}
    rows = sum(new) * H * D
    if case["kind"] == "read":
        return {"bytes": sum(new) * row + 2 * rows * 2, "flops": 2 * rows}
    # the new rows in, the stored ones out and in again, their values out; the tables' rows of all positions touched
    touched = max(total) - min(t - n for t, n in zip(total, new))
    return {"bytes": 4 * rows * 2 + 2 * sum(new) * row + min(sum(new), touched) * D * 4, "flops": 10 * rows}


def exact(case, seed):
    s = prepare(case, seed)
    B, L, D, P = case["B"], case["L"], case["D"], case["page"]
    total, new = _lengths(case)
    nc, ns = P * (D // 2), P * (D // 32)
    feature = torch.arange(D, device="cuda")
    shift = 4 * (feature % 2)

    def two_to(e):
        return ((e + 1023) << 52).view(torch.float64)

    def values(code, exponent):
        """e2m1 by its fields: sign, two exponent bits (0: subnormal), one mantissa bit."""
        e, m = (code >> 1) & 3, (code & 1).double()
        mag = torch.where(e > 0, (1 + m / 2) * two_to(e.long() - 1), m / 2)
        return torch.where(code >= 8, -mag, mag) * two_to(exponent.long() - 127)

    def rows(b, h, first, n):
        """Keys and values [n, D] of stream b, stored head h, tokens first .. first + n - 1."""
        pos = torch.arange(first, first + n, device="cuda")
        at = s["cache"][:, h].flatten(1)[s["table"][b].long()[pos // P]]             # [n, bytes] of each token's page
        t = (pos % P)[:, None]
        k = values((at.gather(1, t * (D // 2) + feature // 2) >> shift) & 15, at.gather(1, 2 * nc + t * (D // 32) + feature // 32))
        v = values((at.gather(1, nc + (t // 16) * (8 * D) + feature // 2 * 16 + t % 16) >> shift) & 15,
                   at.gather(1, 2 * nc + ns + (t // 16) * (D // 2) + feature // 32 * 16 + t % 16))
        return k, v

    if case["kind"] == "attend":
        H, Hkv = case["H"], case["Hkv"]
        G = H // Hkv
        if 4 * sum(total) * L * H * D > 8e13 or B * Hkv > 1024:
            return None
        out = torch.zeros((B, L, H, D), dtype=torch.float64, device="cuda")
        for b in range(B):
            n, t = new[b], total[b]
            for h in range(Hkv):
                parts = [rows(b, h, f, min(8192, t - f)) for f in range(0, t, 8192)]
                k, v = torch.cat([p[0] for p in parts]), torch.cat([p[1] for p in parts])
                for x in range(h * G, (h + 1) * G):
                    logit = (s["q"][b, :n, x].double() @ k.T) * D ** -0.5
                    if case["causal"]:
                        logit.masked_fill_(torch.ones_like(logit, dtype=torch.bool).triu_(t - n + 1), -math.inf)
                    out[b, :n, x] = torch.softmax(logit, -1) @ v
        return out
    k_out = torch.zeros((B, L, case["H"], D), dtype=torch.float64, device="cuda")
    v_out = torch.zeros_like(k_out)
    for b in range(B):
        n, first = new[b], total[b] - new[b]
        if case["kind"] == "read":
            for h in range(case["H"]):
                k_out[b, :n, h], v_out[b, :n, h] = rows(b, h, first, n)
            continue
        turn = torch.complex(s["cos"][first:first + n].double(), s["sin"][first:first + n].double())[:, None]
        k = torch.view_as_real(torch.view_as_complex(s["k"][b, :n].double().unflatten(-1, (D // 2, 2)).contiguous()) * turn).flatten(-2)
        for x, y in ((k.float().double(), k_out), (s["v"][b, :n].double(), v_out)):
            w = x.unflatten(-1, (D // 32, 32))
            mantissa, power = torch.frexp(w.abs().amax(-1, keepdim=True))            # amax = mantissa 2^power, mantissa in [1/2, 1)
            unit = two_to((power.long() - 3 + (mantissa > 0.875)).clamp(-120, 125))
            u = w / unit
            # the grid's step is 1/2 below 2, 1 below 4, 2 beyond; rounding half to even is that of e2m1's codes
            grid = torch.where(u.abs() < 2, 0.5, torch.where(u.abs() < 4, 1.0, 2.0))
            y[b, :n] = ((u / grid).round() * grid).clamp(-6, 6).mul(unit).flatten(-2)
    return [k_out, v_out]
