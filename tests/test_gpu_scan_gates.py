"""Gates that count as zero: the gradients of their logarithms are zeros, to the last bit."""
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


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("gate", [float(np.nextafter(np.float32(-2839), np.float32(-3000))), -2839.05, -2839.1, -2839.15, -2839.2, -2840.0, -1e30, -float("inf")])
def test_zero_at_a_gate_of_zero(A, D, gate):
    c = R.Case(1, 3, 150, D, seed=3)
    c.la[0, 10:140:9] = gate
    want, limits = c.backward()
    got = R.run_backward(A, c)
    for name, g, w, l in zip(("dq", "dk", "dv", "dlog_alpha", "dS0"), got, want, limits):
        R.check(name, g, w, l)
    assert (got[3].cpu()[0, 10:140:9] == 0).all()
