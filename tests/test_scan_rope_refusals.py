"""What the recurrence and the rotation refuse before any launch (no GPU needed), and the reference's gradients against differences."""
import ctypes
import os
import re

import numpy as np
import pytest
import torch

import scan_reference as R
from helpers import built_package

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
# (never dereferenced: the calls fail validation before any launch)
PTR = [0x100000000 * i for i in range(1, 15)]
WS = 0x7f0000000000


@pytest.fixture(scope="module")
def A():
    A = built_package()
    A.load_library()
    return A


@pytest.mark.parametrize("name", ["arl2_scan_desc", "arl2_rope_desc"])
def test_descriptors_match_the_header(A, name):
    header = open(os.path.join(ROOT, "include", "arl2.h")).read()
    body = re.search(r"typedef struct \{([^{}]*)\} %s;" % name, header, flags=re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    names = [n.split("[")[0].strip(" *") for line in body.split(";") if line.strip() for n in re.sub(r"^\s*\w+\s", "", line.strip()).split(",")]
    assert names == [f[0] for f in getattr(A, name)._fields_]


def scan(A, bwd=False, at=(), **kw):
    d = A.arl2_scan_desc(**{**dict(B=2, H=3, L=1000, D=64, workspace=WS, workspace_bytes=1 << 40), **kw})
    p = PTR[:13 if bwd else 8]
    for i, x in dict(at).items():
        p[i] = x
    lib = A.load_library()
    st = (lib.arl2_scan_bwd if bwd else lib.arl2_scan_fwd)(ctypes.byref(d), *p)
    return st, lib.arl2_last_error().decode()


@pytest.mark.parametrize("bwd", [False, True])
def test_scan_sizes(A, bwd):
    lib = A.load_library()
    for bad in (dict(B=0), dict(H=0), dict(L=0), dict(raw_rows=2), dict(raw_rows=-1), dict(l2_eps=-1.0), dict(l2_eps=float("nan"))):
        assert scan(A, bwd, **bad)[0] == 1, bad
        assert lib.arl2_scan_workspace_bytes(ctypes.byref(A.arl2_scan_desc(**{**dict(B=2, H=3, L=1000, D=64), **bad}))) == 0
    for bad in (dict(D=96), dict(D=256), dict(L=1 << 23), dict(H=1 << 18, L=1), dict(B=1 << 20)):
        assert scan(A, bwd, **bad)[0] == 2, bad
    need = (lib.arl2_scan_bwd_workspace_bytes if bwd else lib.arl2_scan_workspace_bytes)(ctypes.byref(A.arl2_scan_desc(B=2, H=3, L=1000, D=64)))
    assert need > 0
    for bad in (dict(workspace=None), dict(workspace_bytes=need - 1)):
        assert scan(A, bwd, **bad)[0] == 3, bad
    assert scan(A, bwd, workspace=WS + 8)[0] == 1


def test_scan_arguments(A):
    for i in (0, 1, 2, 6):                                    # rows that have to be there
        assert scan(A, at={i: None})[0] == 1
    for i in (0, 1, 2, 5, 6, 7):                              # 16 bytes
        assert scan(A, at={i: PTR[i] + 8})[0] == 1
    for i in (3, 4):
        assert scan(A, at={i: PTR[i] + 2})[0] == 1
    rows, state = 2 * 1000 * 3 * 64 * 2, 2 * 3 * 64 * 64 * 4
    for i, n in ((0, rows), (1, rows), (2, rows), (3, 2 * 1000 * 3 * 4), (4, 8), (5, state), (7, state)):
        st, why = scan(A, at={6: (PTR[i] + n - 1) // 16 * 16})
        assert st == 1 and "overlap" in why, i                # out's first bytes are the argument's last
    st, why = scan(A, at={7: PTR[5] + 16})                    # S may be S0, not a part of it
    assert st == 1 and "overlap" in why
    st, why = scan(A, workspace=PTR[1] + 256)
    assert st == 1 and "workspace" in why
    for i in (0, 1, 2, 6, 8, 9, 10):
        assert scan(A, True, at={i: None})[0] == 1
    for i in (0, 1, 2, 5, 6, 7, 8, 9, 10, 12):
        assert scan(A, True, at={i: PTR[i] + 4})[0] == 1
    st, why = scan(A, True, at={3: None})                     # the gradient of gates that are not there
    assert st == 1 and "dlog_alpha" in why
    for i in (8, 9, 10, 11, 12):
        for j in (0, 1, 2, 3, 5, 6, 7):
            st, why = scan(A, True, at={i: PTR[j]})           # (dS0 is not dS either: other workgroups still read it)
            assert st == 1 and "overlap" in why, (i, j)
        for j in (8, 9, 10, 11, 12):
            if i != j:
                st, why = scan(A, True, at={i: PTR[j]})
                assert st == 1 and "overlap" in why, (i, j)
    st, why = scan(A, True, at={12: PTR[7] + 16})
    assert st == 1 and "overlap" in why


def rope(A, bwd=False, at=(), **kw):
    axes = kw.pop("axis_pairs", [10, 11, 11, 0])
    theta = kw.pop("theta", [0.0] * 4)
    d = A.arl2_rope_desc(**{**dict(B=2, H=3, L=10, D=64, Hk=1, io_dtype=1, norm=2, n_axes=3, workspace=WS, workspace_bytes=1 << 40), **kw})
    for i in range(4):
        d.axis_pairs[i], d.theta[i] = axes[i], theta[i]
    p = PTR[:12 if bwd else 8]
    for i, x in dict(at).items():
        p[i] = x
    lib = A.load_library()
    st = (lib.arl2_rope_bwd if bwd else lib.arl2_rope_fwd)(ctypes.byref(d), *p)
    return st, lib.arl2_last_error().decode()


@pytest.mark.parametrize("bwd", [False, True])
def test_rope_sizes(A, bwd):
    for bad in (dict(B=0), dict(H=0), dict(L=0), dict(Hk=-1), dict(io_dtype=2), dict(norm=3), dict(norm=-1), dict(halves=2), dict(pos_per_stream=2), dict(n_axes=0), dict(n_axes=5),
                dict(axis_pairs=[32, 1, 1, 0]), dict(axis_pairs=[0, 1, 1, 0]), dict(axis_pairs=[2 ** 31 - 1] * 4, n_axes=4), dict(theta=[-1.0, 0, 0, 0]),
                dict(theta=[float("nan"), 0, 0, 0]), dict(theta=[float("inf"), 0, 0, 0]), dict(theta=[1e-9, 0, 0, 0]), dict(norm_eps=-1.0), dict(norm_eps=float("nan"))):
        assert rope(A, bwd, **bad)[0] == 1, bad
    for bad in (dict(D=80), dict(H=400), dict(H=2 ** 31 - 1), dict(B=1 << 20, L=1 << 20)):
        assert rope(A, bwd, **bad)[0] == 2, bad


def test_rope_arguments(A):
    q, k, wq, wk, pos, lens, yq, yk = range(8)
    for i in (q, k, pos, yq, yk):
        assert rope(A, at={i: None})[0] == 1, i
    for i in (q, k, wq, wk, yq, yk):
        assert rope(A, at={i: PTR[i] + 8})[0] == 1, i
    for i in (pos, lens):
        assert rope(A, at={i: PTR[i] + 1})[0] == 1, i
    assert rope(A, Hk=0)[0] == 1 and rope(A, Hk=0, at={k: None, yk: None})[0] == 1      # keys, and their weights, without heads
    assert rope(A, norm=0)[0] == 1                                                    # weights without a norm
    for i, j in ((yq, k), (yk, q), (yq, wq), (yk, wk), (yq, pos), (yk, lens), (yq, yk)):
        st, why = rope(A, at={i: PTR[j]})
        assert st == 1 and "overlap" in why, (i, j)
    for i, j in ((yq, q), (yk, k)):
        st, why = rope(A, at={i: PTR[j] + 16})
        assert st == 1 and "overlap" in why, (i, j)
    q, k, wq, wk, pos, lens, dyq, dyk, dq, dk, dwq, dwk = range(12)
    for i in (q, k, pos, dyq, dyk, dq, dk):
        assert rope(A, True, at={i: None})[0] == 1, i
    assert rope(A, True, at={dwq: PTR[dwq] + 2})[0] == 1
    assert rope(A, True, norm=0, at={wq: None, wk: None})[0] == 1                      # their gradients without a norm
    for bad in (dict(workspace=None), dict(workspace_bytes=16)):
        assert rope(A, True, **bad)[0] == 3
    for i in (dq, dk, dwq, dwk):
        for j in (q, k, wq, wk, pos, lens, dyq, dyk):
            if (i, j) not in ((dq, dyq), (dk, dyk)):
                st, why = rope(A, True, at={i: PTR[j]})
                assert st == 1 and "overlap" in why, (i, j)
    st, why = rope(A, True, at={dq: PTR[dyq] + 16})
    assert st == 1 and "overlap" in why


def test_binding_checks_tensors_before_the_call(A):
    rows, gates, state = torch.zeros((1, 4, 2, 64), dtype=torch.bfloat16), torch.zeros((1, 4, 2)), torch.zeros((1, 2, 64, 64))
    with pytest.raises(ValueError, match="q must live in device memory"):
        A.arl2_scan_fwd(rows, rows, rows, gates, state, rows, state)
    with pytest.raises(ValueError, match="device memory"):
        A.arl2_scan_bwd(rows, rows, rows, gates, state, rows, state, rows, rows, rows, gates, state)
    with pytest.raises(ValueError, match="device memory"):
        A.arl2_rope_fwd(rows, None, None, None, torch.zeros((4, 1), dtype=torch.int32), rows, None, axis_pairs=[32])
    with pytest.raises(ValueError, match="norm"):
        A.arl2_rope_fwd(rows, None, None, None, torch.zeros((4, 1), dtype=torch.int32), rows, None, axis_pairs=[32], norm="layer")
    with pytest.raises(ValueError, match="axes"):
        A.arl2_rope_fwd(rows, None, None, None, torch.zeros((4, 1), dtype=torch.int32), rows, None, axis_pairs=[1] * 5)
    with pytest.raises(ValueError, match="heads"):
        A.arl2_rope_fwd(rows[0], None, None, None, torch.zeros((4, 1), dtype=torch.int32), rows, None, axis_pairs=[32])


@pytest.mark.parametrize("normalise", [True, False])
def test_the_references_gradients_against_differences(normalise, monkeypatch):
    """Central differences of the fp64 recurrence along random directions: third order of the step and fp64's own roundings."""
    c = R.Case(2, 2, 9, 64, seed=1, normalise=normalise, lens=[9, 4])
    monkeypatch.setattr(R, "wide", lambda t: t.detach().to(torch.float64).numpy())
    grads = c.backward()[0]
    do, dS = c.do.double().numpy(), c.dS.double().numpy()
    g = np.random.Generator(np.random.Philox(2))
    for name, grad in zip(("q", "k", "v", "la", "S0"), grads):
        x = getattr(c, name)
        d, h, vals = g.standard_normal(tuple(x.shape)), 2.0 ** -14, []
        for s in (1, -1):
            setattr(c, name, x.double() + s * h * torch.from_numpy(d))
            out, S, _, _ = c.forward()
            vals.append((out * do).sum() + (S * dS).sum())
        setattr(c, name, x)
        want = (grad * d).sum()
        assert abs((vals[0] - vals[1]) / (2 * h) - want) <= 1e-5 * (abs(want) + np.abs(grad * d).sum() ** 0.5), name
