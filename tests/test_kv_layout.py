"""The paged 4-bit cache on the host: where rows lie and what bad tables lead to (the functions that the kernels use, compiled for
the CPU), what the C ABI and the binding refuse."""
import ctypes
import os
import subprocess

import numpy as np
import pytest
import torch

import kv_reference as R
from helpers import built_package

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2605_16579_amd", "csrc")
SOURCE = r'''
#include "arl2_kv_layout.h"
extern "C" {
int page_of(int shift, int n_pages, int max_pages, const int32_t *row, long long pos) { return arl2::kv_page({shift, 1, n_pages, max_pages}, row, pos); }
int clamp(int n, int most) { return arl2::kv_clamp(n, most); }
int head_bytes(int shift, int D) { return arl2::kv_head_bytes(shift, D); }
long long head_offset(int shift, int heads, int D, int page, int head) { return (long long)arl2::kv_head_offset({shift, heads, 1 << 30, 1}, D, page, head); }
int offset(int what, int shift, int t, int i, int D)
{
    return what == 0 ? arl2::kv_key_codes(t, i, D) : what == 1 ? arl2::kv_value_codes(shift, t, i, D)
         : what == 2 ? arl2::kv_key_scales(shift, t, i, D) : arl2::kv_value_scales(shift, t, i, D);
}
}
'''


@pytest.fixture(scope="module")
def layout(tmp_path_factory):
    d = tmp_path_factory.mktemp("kv_layout")
    (d / "shim.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wall", "-Werror", "-I", CSRC, "-o", str(d / "shim.so"), str(d / "shim.cpp")], check=True)
    lib = ctypes.CDLL(str(d / "shim.so"))
    lib.page_of.argtypes = [ctypes.c_int] * 3 + [ctypes.POINTER(ctypes.c_int32), ctypes.c_longlong]
    lib.head_offset.restype = ctypes.c_longlong
    return lib


@pytest.fixture(scope="module")
def A():
    A = built_package()
    A.load_library()
    return A


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shift", [4, 5, 6, 7, 8])
def test_every_byte_of_a_page_belongs_to_one_token(layout, shift, D):
    n = layout.head_bytes(shift, D)
    assert n == (1 << shift) * 2 * (D // 2 + D // 32) and n % 16 == 0
    owner = np.full(n, -1)
    for t in range(1 << shift):
        for what, count in ((0, D // 2), (1, D // 2), (2, D // 32), (3, D // 32)):
            for i in range(count):
                o = layout.offset(what, shift, t, i, D)
                assert 0 <= o < n and owner[o] == -1
                owner[o] = t
    assert (owner >= 0).all()
    # what the kernels load as 16, 4 or 2 bytes starts at a multiple of them
    for t in range(0, 1 << shift, 16):
        for i in range(D // 2):
            assert layout.offset(1, shift, t, i, D) % 16 == 0
        for g in range(D // 32):
            assert layout.offset(3, shift, t, g, D) % 16 == 0
    for t in range(1 << shift):
        assert layout.offset(0, shift, t, 0, D) % 32 == 0 and layout.offset(2, shift, t, 0, D) % (D // 32) == 0
    assert all(layout.offset(what, shift, 0, 0, D) % 16 == 0 for what in range(4))


@pytest.mark.parametrize("shift", [4, 6, 8])
def test_positions_without_a_place_have_no_page(layout, shift):
    P = 1 << shift
    row = (ctypes.c_int32 * 8)(5, -1, 6, 7, 2 ** 31 - 1, -2 ** 31, 0, 99)
    guard = (ctypes.c_int32 * 5)(*row[:5])                      # a row of five entries
    for pos in (-1, -P, -2 ** 31, 5 * P, 5 * P + 1, 2 ** 31, 2 ** 40, -2 ** 40):
        assert layout.page_of(shift, 7, 5, guard, pos) == -1    # (the row's end is never passed)
    want = [5, -1, 6, -1, -1, -1, 0, -1]                        # entries outside [0, 7)
    for i, w in enumerate(want):
        for t in (0, 1, P - 1):
            assert layout.page_of(shift, 7, 8, row, i * P + t) == w
    assert [layout.clamp(n, 5) for n in (-2 ** 31, -1, 0, 1, 5, 6, 2 ** 31 - 1)] == [0, 0, 0, 1, 5, 5, 5]


def test_offsets_pass_32_bits(layout):
    assert layout.head_offset(8, 16, 128, 10 ** 6, 15) == (10 ** 6 * 16 + 15) * 256 * 136 > 2 ** 39


def test_quantise_reference_on_worked_values():
    x = np.zeros((6, 32), dtype=np.float32)
    x[0, :8] = [7.0, 6.5, 5.0, 5.1, 2.5, 3.5, 0.25, -0.26]      # largest 7: unit 1
    x[1, :3] = [7.5, 7.0, 0.5]                                  # beyond 7: unit 2
    x[2, :2] = [2.0 ** -125, 1e-40]                             # below the least unit
    x[3, :2] = [3.0e38, -3.4e38]                                # beyond the largest: 6 * 2^125
    x[4, 0] = np.inf
    x[5, :2] = [1.75, 1.25]                                     # unit 1/4: 7 and 5
    y = R.quantise(x)
    assert y[0, :8].tolist() == [6.0, 6.0, 4.0, 6.0, 2.0, 4.0, 0.0, -0.5]
    assert y[1, :3].tolist() == [8.0, 8.0, 0.0]
    assert y[2, :2].tolist() == [0.0, 0.0]
    assert y[3, :2].tolist() == [6 * 2.0 ** 125, -6 * 2.0 ** 125]
    assert np.isnan(y[4]).all()
    assert y[5, :2].tolist() == [1.5, 1.0]


def test_attend_reference_against_torch():
    r = np.random.default_rng(0)
    q, k, v = r.normal(size=(5, 4, 64)), r.normal(size=(9, 2, 64)), r.normal(size=(9, 2, 64))
    out, bound = R.attend(q, k, v, [5, 6, 7, 8, 9], 0.125)
    t = [torch.from_numpy(x).transpose(0, 1) for x in (q, k.repeat(2, 1), v.repeat(2, 1))]
    mask = torch.ones(5, 9, dtype=torch.bool).tril(4)
    want = torch.softmax((t[0] @ t[1].transpose(1, 2) * 0.125).masked_fill(~mask, -np.inf), -1) @ t[2]
    assert np.abs(out - want.transpose(0, 1).numpy()).max() < 1e-14 and (bound > 0).all()
    out, _ = R.attend(q, k, v, [0, 1, 1, 0, 0], 0.125)
    assert (out[0] == 0).all() and np.allclose(out[1, 0], v[0, 0]) and np.allclose(out[2, 3], v[0, 1])


def _desc(A, **kw):
    d = dict(B=2, H=8, Hkv=2, Lq=4, D=128, page_size=64, n_pages=9, max_pages=4, causal=0, sm_scale=0.0, workspace=None, workspace_bytes=0, stream=None)
    d.update(kw)
    return A.arl2_kv_desc(*[d[f[0]] for f in A.arl2_kv_desc._fields_])


# the pointers are never dereferenced: every call below must fail validation before any launch
PTR = [0x10000000 * i for i in range(1, 9)]


def _append(A, d, k=PTR[0], v=PTR[1], c=PTR[2], s=PTR[3], t=PTR[4], st=PTR[5], n=PTR[6], cache=PTR[7]):
    return A.load_library().arl2_kv_append(ctypes.byref(d), k, v, c, s, t, st, n, cache)


def _read(A, d, cache=PTR[0], t=PTR[1], st=PTR[2], n=PTR[3], k=PTR[4], v=PTR[5]):
    return A.load_library().arl2_kv_read(ctypes.byref(d), cache, t, st, n, k, v)


def _attn(A, d, q=PTR[0], cache=PTR[1], t=PTR[2], kl=PTR[3], ql=PTR[4], out=PTR[5]):
    return A.load_library().arl2_kv_attn_fwd(ctypes.byref(d), q, cache, t, kl, ql, out)


def test_kv_desc_struct_matches_header(A):
    import re
    header = open(os.path.join(os.path.dirname(CSRC), "..", "include", "arl2.h")).read()
    body = header[:header.index("} arl2_kv_desc;")]
    body = re.sub(r"/\*.*?\*/", "", body[body.rindex("typedef struct {"):], flags=re.S)
    assert re.findall(r"\b(\w+)\s*;", body) == [f[0] for f in A.arl2_kv_desc._fields_]
    assert ctypes.sizeof(A.arl2_kv_desc) == 64


def test_refusals_of_the_descriptor(A):
    lib = A.load_library()
    for call in (_append, _read, _attn):
        for bad in (dict(B=0), dict(Hkv=0), dict(Lq=0), dict(Lq=-3), dict(n_pages=0), dict(max_pages=0)):
            assert call(A, _desc(A, **bad)) == 1, (call, bad)
        for bad in (dict(D=96), dict(D=256), dict(page_size=8), dict(page_size=48), dict(page_size=512), dict(max_pages=2 ** 25), dict(B=10 ** 6), dict(n_pages=2 ** 31 - 1),
                    dict(B=1, Hkv=130000, H=130000, page_size=256)):
            assert call(A, _desc(A, **bad)) == 2, (call, bad)
    for bad in (dict(H=0), dict(H=7), dict(causal=2), dict(sm_scale=-1.0), dict(sm_scale=float("nan")), dict(sm_scale=float("inf"))):
        assert _attn(A, _desc(A, **bad)) == 1, bad
    assert _attn(A, _desc(A, H=2 * 600000)) == 2
    huge = _desc(A, B=90000, H=10, Hkv=1, Lq=20000, max_pages=2 ** 22, page_size=256)
    assert _attn(A, huge) == 2 and lib.arl2_kv_workspace_bytes(ctypes.byref(huge)) == 0
    assert _append(A, _desc(A, B=1000, Hkv=900, Lq=10 ** 6)) == 2 and _read(A, _desc(A, B=1000, Hkv=900, Lq=10 ** 6)) == 2
    assert lib.arl2_kv_append(None, *PTR) == 1 and lib.arl2_kv_read(None, *PTR[:6]) == 1 and lib.arl2_kv_attn_fwd(None, *PTR[:6]) == 1
    assert lib.arl2_kv_cache_bytes(ctypes.byref(_desc(A))) == 9 * 2 * 64 * 136
    assert lib.arl2_kv_cache_bytes(ctypes.byref(_desc(A, D=64))) == 9 * 2 * 64 * 68
    assert lib.arl2_kv_cache_bytes(ctypes.byref(_desc(A, D=80))) == 0
    assert lib.arl2_kv_cache_bytes(ctypes.byref(_desc(A, n_pages=10 ** 6, page_size=256))) == 10 ** 6 * 2 * 256 * 136
    assert lib.arl2_kv_workspace_bytes(ctypes.byref(_desc(A, H=7))) == 0


def test_refusals_of_pointers(A):
    d = _desc(A)
    for name in ("k", "v", "t", "st", "cache"):
        assert _append(A, d, **{name: None}) == 1, name
    for name in ("k", "v", "c", "s", "cache"):
        assert _append(A, d, **{name: PTR[0] + 0x7000008}) == 1, name
    for name in ("t", "st", "n"):
        assert _append(A, d, **{name: PTR[0] + 0x7000002}) == 1, name
    assert _append(A, d, c=None) == 1 and _append(A, d, s=None) == 1                  # one table without the other
    size = 9 * 2 * 64 * 136
    for name in ("k", "v", "c", "s", "t", "st", "n"):                                 # the cache's last bytes are an input's first
        assert _append(A, d, **{name: PTR[7] + size - 16}) == 1, name
        assert b"overlap" in A.load_library().arl2_last_error()
    for name in ("cache", "t", "st", "k", "v"):
        assert _read(A, d, **{name: None}) == 1, name
    assert _read(A, d, v=PTR[4] + 256) == 1 and _read(A, d, k=PTR[0] + 256) == 1      # outputs that overlap
    for name in ("q", "cache", "t", "kl", "out"):
        assert _attn(A, d, **{name: None}) == 1, name
    assert _attn(A, d, out=PTR[0] + 256) == 1 and _attn(A, d, out=PTR[1] + 512) == 1 and _attn(A, d, q=PTR[0] + 2) == 1


def test_attention_asks_for_its_workspace(A):
    lib = A.load_library()
    d = _desc(A, max_pages=2048)                       # a long table: the key axis is split
    need = lib.arl2_kv_workspace_bytes(ctypes.byref(d))
    assert need > 0
    assert _attn(A, d) == 3
    short = _desc(A, max_pages=2048, workspace=0x90000000, workspace_bytes=need - 1)
    assert _attn(A, short) == 3 and b"arl2_kv_workspace_bytes" in lib.arl2_last_error()
    assert _attn(A, _desc(A, max_pages=2048, workspace=0x90000008, workspace_bytes=need)) == 1        # misaligned
    assert _attn(A, _desc(A, max_pages=2048, workspace=PTR[5], workspace_bytes=need)) == 1            # on top of out
    assert A.arl2_kv_workspace_bytes(2, 8, 2, 4, 128, 64, 2048) == need


def test_binding_refuses_what_does_not_fit(A):
    cache = torch.zeros((9, 2, 64, 136), dtype=torch.uint8)
    k = torch.zeros((2, 4, 2, 128), dtype=torch.bfloat16)
    table, start = torch.zeros((2, 4), dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError, match="cache must be uint8"):
        A.arl2_kv_append(k, k, cache[..., :68].contiguous(), table, start)
    with pytest.raises(ValueError, match="cache must be uint8"):
        A.arl2_kv_append(k, k, cache.float(), table, start)
    with pytest.raises(ValueError, match="heads"):
        A.arl2_kv_append(k[:, :, :1].contiguous(), k, cache, table, start)
    with pytest.raises(ValueError, match="block_table"):
        A.arl2_kv_append(k, k, cache, table[:1], start)
    with pytest.raises(ValueError, match=r"\[B, L, heads, D\]"):
        A.arl2_kv_read(cache, table, start, k[0], k[0])
    with pytest.raises(ValueError, match="device memory"):
        A.arl2_kv_attn_fwd(k, cache, table, start, k.clone())
    assert A.alloc_kv_cache(9, 2, 64, 128, device="cpu").shape == cache.shape


def test_cache_kernels_use_no_scratch(A):
    from test_kernel_resources import scratch_per_kernel
    kernels = {name: n for name, n in scratch_per_kernel(A.binding.LIB_PATH).items() if "kv_" in name}
    # append, read, attention for few and for many rows, and two joins, for two head dimensions each
    assert len(kernels) == 12, sorted(kernels)
    assert not any(kernels.values()), {name: n for name, n in kernels.items() if n}
