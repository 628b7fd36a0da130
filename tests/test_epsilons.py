"""The least epsilons of the recurrence and the rotation: smaller ones are refused, with the least one rows of zeros stay finite."""
import ctypes

import numpy as np
import pytest
import torch

import scan_reference as R
from helpers import built_package
from test_gpu_rope import Case, both
from test_scan_rope_refusals import rope, scan

LEAST = 1e-30


@pytest.fixture(scope="module")
def A():
    A = built_package()
    A.load_library()
    return A


@pytest.mark.parametrize("eps", [1e-45, 1e-40, 1e-38, 9.9e-31])
def test_smaller_ones_are_refused(A, eps):
    for bwd in (False, True):
        st, why = scan(A, bwd, l2_eps=eps)
        assert st == 1 and "l2_eps" in why
        st, why = rope(A, bwd, norm_eps=eps)
        assert st == 1 and "norm_eps" in why


def test_what_is_accepted(A):
    lib = A.load_library()
    for eps in (0.0, LEAST * 1.0001, 1e-12, 1.0):
        assert lib.arl2_scan_workspace_bytes(ctypes.byref(A.arl2_scan_desc(B=1, H=1, L=1000, D=64, l2_eps=eps))) > 0
        d = A.arl2_rope_desc(B=1, H=1, L=1000, D=64, io_dtype=1, norm=1, n_axes=1, norm_eps=eps)
        d.axis_pairs[0] = 1
        assert lib.arl2_rope_workspace_bytes(ctypes.byref(d)) > 0


def test_the_binding_does_not_turn_one_into_the_default(A):
    rows, pos = torch.zeros((1, 4, 2, 64), dtype=torch.bfloat16), torch.zeros((4, 1), dtype=torch.int32)
    with pytest.raises(ValueError, match="single precision"):
        A.binding._scan_desc(1, 2, 4, 64, l2_eps=1e-50, stream=0)
    with pytest.raises(ValueError, match="single precision"):
        A.arl2_rope_fwd(rows, None, None, None, pos, rows, None, axis_pairs=[32], norm="head", norm_eps=1e-50, stream=0)


@pytest.mark.gpu
def test_the_binding_does_not_turn_one_into_the_default_on_the_device(A):
    rows = torch.ones((1, 9, 2, 64), dtype=torch.bfloat16, device="cuda")
    pos = torch.zeros((9, 1), dtype=torch.int32, device="cuda")
    out = torch.empty_like(rows)
    with pytest.raises(ValueError, match="single precision"):
        A.arl2_scan_fwd(rows, rows, rows, None, None, out, None, l2_eps=1e-50)
    with pytest.raises(ValueError, match="single precision"):
        A.arl2_rope_fwd(rows, None, None, None, pos, out, None, axis_pairs=[32], norm="head", norm_eps=1e-50)


@pytest.mark.gpu
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("gate", [-1e-3, -0.4, -0.68])
@pytest.mark.parametrize("L,lens", [(5, None), (100, None), (200, [200, 70, 1])])
def test_rows_of_zeros_with_the_least_one(A, monkeypatch, L, lens, gate, D):
    """Blocks' gates of 2^-63 together; rows of zeros within the sequences and behind their ends."""
    eps = float(np.nextafter(np.float32(LEAST), np.float32(1)))
    monkeypatch.setattr(R, "EPS", eps)
    c = R.Case(3, 2, L, D, seed=31, lens=lens)
    c.la[:] = gate
    for x in (c.q, c.k):
        x[:, 2::7] = 0
    out, S, lo, ls = c.forward()
    got, state = R.run_forward(A, c, l2_eps=eps)
    R.check("out", got, out, lo, c.lens)
    R.check("S", state, S, ls)
    want, limits = c.backward()
    for name, g, w, l in zip(("dq", "dk", "dv", "dlog_alpha", "dS0"), R.run_backward(A, c, l2_eps=eps), want, limits):
        R.check(name, g, w, l, c.lens if name != "dS0" else None)


@pytest.mark.gpu
@pytest.mark.parametrize("norm", ["head", "row"])
def test_rotation_with_the_least_one(A, monkeypatch, norm):
    """Rows of zeros and rows behind the sequences' ends (whose weights' gradients are finite)."""
    eps = float(np.nextafter(np.float32(LEAST), np.float32(1)))
    c = Case(3, 4, 2, 21, 64, norm=norm, lens=[21, 5, 0])
    for x in c.x:
        x[:, 3] = 0
    over = (-1, -2) if norm == "row" else -1
    c._norm = lambda x: 1.0 / np.sqrt((x * x).mean(over, keepdims=True) + eps)
    kw = c.kw()
    c.kw = lambda: {**kw, "norm_eps": eps}
    both(A, c)
