"""The recurrence's gradients in the 2-norm, head by head and segment by segment."""
import pytest
import torch

import scan_norms as N
import scan_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2605_16579_amd as A
    A.load_library()
    return A


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L", [1, 2, 9, 64, 65, 200, 513])
@pytest.mark.parametrize("normalise", [True, False])
def test_lengths(A, D, L, normalise):
    c = R.Case(2, 3, L, D, seed=40 + L, normalise=normalise, rows=1.0 if normalise else 0.3)
    N.check_gradients(c, c.backward()[0], R.run_backward(A, c))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("gates", ["none", "one", "small", "resets"])
@pytest.mark.parametrize("L,lens", [(150, None), (300, [300, 0, 129, 192]), (1300, [1300, 7])])
def test_gates(A, D, gates, L, lens):
    c = R.Case(2 if lens is None else len(lens), 2, L, D, seed=41, gates=gates, lens=lens, start=gates != "small")
    N.check_gradients(c, c.backward()[0], R.run_backward(A, c))


@pytest.mark.parametrize("D,H,L", [(128, 1, 3000), (64, 1, 2500), (128, 12, 1560), (64, 300, 140), (128, 520, 70)])
def test_many_segments_and_many_heads(A, D, H, L):
    """One stream of many segments, and more heads than there is room for at once; sampled heads."""
    full = R.Case(1, H, L, D, seed=42)
    grads = R.run_backward(A, full)
    for h in sorted({0, H // 2, H - 1}):
        c = R.Case(1, 1, L, D, seed=1)
        for n in ("q", "k", "v", "do", "la"):
            setattr(c, n, getattr(full, n)[:, :, h:h + 1])
        c.S0, c.dS = full.S0[:, h:h + 1], full.dS[:, h:h + 1]
        N.check_gradients(c, c.backward()[0], [x[:, :, h:h + 1] for x in grads[:4]] + [grads[4][:, h:h + 1]])


def test_short_memory_over_long_sequences(A):
    """Gates of 0.8: what a gate's gradient is small against."""
    for D in (64, 128):
        c = R.Case(1, 1, 4200, D, seed=43)
        c.la[:] = torch.log(torch.tensor(0.8))
        N.check_gradients(c, c.backward()[0], R.run_backward(A, c))
