"""Rows at the ends of the ranges that the header states, with decays whose reciprocals are as large as they come."""
import math

import pytest
import torch

import scan_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2605_16579_amd as A
    A.load_library()
    return A


def case(L, D, normalise, rows):
    """All features alike, so that every sum is as large as it can be; the first gate of each block is 2^-63.9."""
    c = R.Case(1, 1, L, D, seed=51, normalise=normalise, start=False)
    for x in (c.q, c.k, c.v, c.do):
        x.fill_(rows)
    c.la.zero_()
    c.la[:, ::R.BLOCK] = -63.9 * math.log(2.0)
    return c


@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L", [64, 130])
def test_forward(A, L, D, normalise):
    c = case(L, D, normalise, 65280.0)
    out, S, lo, ls = c.forward()
    got, state = R.run_forward(A, c)
    R.check("out", got, out, lo)
    R.check("S", state, S, ls)


@pytest.mark.parametrize("normalise", [True, False])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("L", [64, 130])
def test_gradients(A, L, D, normalise):
    c = case(L, D, normalise, 32640.0)
    want, limits = c.backward()
    for name, g, w, l in zip(("dq", "dk", "dv", "dlog_alpha", "dS0"), R.run_backward(A, c), want, limits):
        R.check(name, g, w, l)
