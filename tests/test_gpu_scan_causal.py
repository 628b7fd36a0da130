"""What is not finite in a token's rows or gate reaches that token's outputs and later ones alone: the others are those of the call without it, bit for bit (behind a
gate that is a NaN a block takes its decays pair by pair: within the limits of its roundings)."""
import pytest
import torch

import scan_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2605_16579_amd as A
    A.load_library()
    return A


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("gates", ["sigmoid", "resets", "none"])
@pytest.mark.parametrize("row,bad", [("v", float("nan")), ("v", float("inf")), ("v", -float("inf")), ("k", float("nan")), ("k", float("inf")), ("q", float("nan")), ("la", float("nan"))])
@pytest.mark.parametrize("L,ats", [(6, [0, 3, 5]), (200, [0, 1, 31, 32, 63, 64, 100, 127, 150, 191, 192, 199]), (1560, [777, 1559])])
def test_nothing_before_the_token(A, L, ats, row, bad, gates, D):
    if row == "la" and gates == "none":
        return
    clean = R.Case(2, 2, L, D, seed=61, gates=gates, lens=[L, L - 1])
    out, S = R.run_forward(A, clean)
    want, _, limit, _ = clean.forward() if row == "la" else [None] * 4
    for at in ats:
        c = R.Case(2, 2, L, D, seed=61, gates=gates, lens=[L, L - 1])
        x = getattr(c, row)
        if row == "la":
            x[0, at, 1] = bad
        else:
            x[0, at, 1, 5 + at % 50] = bad
        got, state = R.run_forward(A, c)
        if row == "la":
            R.check("out", got[:1, :at, 1:], want[:1, :at, 1:], limit[:1, :at, 1:])
        else:
            assert torch.equal(got[0, :at], out[0, :at]), at
        assert torch.equal(got[0, :, 0], out[0, :, 0]) and torch.equal(got[1], out[1]) and torch.equal(state[0, 0], S[0, 0]) and torch.equal(state[1], S[1])
        if not (row == "k" and bad == float("inf")):      # (a normalised row with an infinity: NaN there, zeros beside it)
            assert not torch.isfinite(got[0, at, 1].float()).all(), at
        if row == "v":                                    # other features are as they were
            others = [e for e in range(D) if e != 5 + at % 50]
            assert torch.equal(got[..., others], out[..., others]) and torch.equal(state[..., others], S[..., others])


@pytest.mark.parametrize("D", [64, 128])
def test_several_in_one_block(A, D):
    """The first of them in each feature counts."""
    c, clean = (R.Case(1, 1, 130, D, seed=62) for _ in range(2))
    out, _ = R.run_forward(A, clean)
    where = {3: [70, 90], 17: [64], 40: [127, 80], 63: [129]}
    for e, tokens in where.items():
        for t in tokens:
            c.v[0, t, 0, e] = float("nan") if t % 2 else float("inf")
    got, state = R.run_forward(A, c)
    again, in_place = R.run_forward(A, c, in_place=True)  # (the second walk begins with the state that the first has not written over)
    assert torch.equal(got.view(torch.int16), again.view(torch.int16)) and torch.equal(state.isnan(), in_place.isnan())
    assert torch.equal(state.nan_to_num(0.5), in_place.nan_to_num(0.5)) and state.isnan().all(2)[0, 0].nonzero().flatten().tolist() == sorted(where)
    for e in range(D):
        first = min(where.get(e, [130]))
        assert torch.equal(got[0, :first, 0, e], out[0, :first, 0, e]), e
        assert not torch.isfinite(got[0, first:, 0, e].float()).any(), e
