"""The recurrence and the rotation with a workspace of exactly the stated size: what lies before and behind it stays as it was."""
import pytest
import torch

pytestmark = pytest.mark.gpu

GUARD = 1 << 16


@pytest.fixture(scope="module")
def A():
    import paper_2605_16579_amd as A
    A.load_library()
    return A


class Guarded:
    """`n` bytes of NaNs among bytes of 0x5a, as many more behind them as the call could mean to use twice."""

    def __init__(self, n):
        self.n = n
        self.all = torch.full((GUARD + 2 * n + GUARD,), 0x5a, dtype=torch.uint8, device="cuda")
        self.part = self.all[GUARD:GUARD + n]
        self.part.fill_(0xff)

    def check(self):
        torch.cuda.synchronize()
        assert (self.all[:GUARD] == 0x5a).all(), "before the workspace"
        assert (self.all[GUARD + self.n:] == 0x5a).all(), "behind the workspace"


@pytest.mark.parametrize("norm", ["head", "row"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,Hk,D,L", [(1, 0, 64, 9), (1, 0, 128, 1), (1, 0, 128, 4680), (2, 0, 64, 333), (5, 0, 128, 77), (1, 1, 64, 2000), (12, 12, 128, 500), (40, 8, 128, 300)])
def test_rotation_gradients(A, H, Hk, D, L, dtype, norm):
    g = torch.Generator(device="cuda").manual_seed(H)
    rows = [torch.randn((2, L, h, D), generator=g, device="cuda").to(dtype) if h else None for h in (H, Hk, H, Hk)]
    pos = torch.arange(L, dtype=torch.int32, device="cuda")[:, None].contiguous()
    widths = [D if norm == "head" else h * D for h in (H, Hk)]

    def run(ws):
        dx = [None if t is None else torch.zeros_like(t) for t in rows[:2]]
        dw = [torch.zeros(w, device="cuda") if h else None for w, h in zip(widths, (H, Hk))]
        A.arl2_rope_bwd(*rows[:2], None, None, pos, *rows[2:], *dx, *dw, axis_pairs=[D // 2], norm=norm, workspace=ws)
        return [t for t in (*dx, *dw) if t is not None]

    guarded = Guarded(A.arl2_rope_workspace_bytes(2, H, Hk, L, D))
    got = run(guarded.part)
    guarded.check()
    roomy = torch.empty(4 * guarded.n + 4096, dtype=torch.uint8, device="cuda")
    assert all(torch.equal(a, b) and torch.isfinite(a).all() for a, b in zip(got, run(roomy)))


@pytest.mark.parametrize("B,H,L,D", [(1, 1, 9, 64), (2, 3, 200, 64), (1, 1, 3000, 128), (1, 12, 1560, 128), (5, 24, 999, 64), (1, 300, 140, 64), (3, 2, 65, 128)])
def test_recurrence(A, B, H, L, D):
    g = torch.Generator(device="cuda").manual_seed(L)
    q, k, v, do = (torch.randn((B, L, H, D), generator=g, device="cuda").bfloat16() for _ in range(4))
    la = torch.nn.functional.logsigmoid(torch.randn((B, L, H), generator=g, device="cuda") + 3.0)
    S0, dS = (torch.randn((B, H, D, D), generator=g, device="cuda") for _ in range(2))
    lens = torch.tensor([L, max(1, L // 3), 0, L - 1, 1][:B], dtype=torch.int32, device="cuda")

    def forward(ws):
        out, S = torch.zeros_like(q), torch.zeros_like(S0)
        A.arl2_scan_fwd(q, k, v, la, S0, out, S, seq_len=lens, workspace=ws)
        return out, S

    def backward(ws):
        rows, dla, dS0 = [torch.zeros_like(q) for _ in range(3)], torch.zeros_like(la), torch.zeros_like(S0)
        A.arl2_scan_bwd(q, k, v, la, S0, do, dS, *rows, dla, dS0, seq_len=lens, workspace=ws)
        return (*rows, dla, dS0)

    for call, n in ((forward, A.arl2_scan_workspace_bytes(B, H, L, D)), (backward, A.arl2_scan_bwd_workspace_bytes(B, H, L, D))):
        guarded = Guarded(n)
        got = call(guarded.part if n else None)
        guarded.check()
        roomy = torch.empty(4 * n + 4096, dtype=torch.uint8, device="cuda")
        assert all(torch.equal(a, b) and torch.isfinite(a.float()).all() for a, b in zip(got, call(roomy)))
