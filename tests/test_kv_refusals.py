"""What attention over the 4-bit cache refuses of its logit scale."""
import ctypes

import pytest

from helpers import built_package

# (never dereferenced: the calls fail validation before any launch)
PTR = [0x10000000 * i for i in range(1, 7)]


@pytest.fixture(scope="module")
def A():
    A = built_package()
    A.load_library()
    return A


@pytest.mark.parametrize("scale", [2.0 ** 127 * (1 + 2.0 ** -23), 2.4e38, 3.0e38, 3.4028234663852886e38, float("inf"), float("nan"), -1.0])
def test_scales_whose_base_two_form_is_not_finite(A, scale):
    """sm_scale * log2(e) overflows from 1.39 * 2^127 on: logits of zero would become NaN."""
    lib = A.load_library()
    d = A.arl2_kv_desc(B=2, H=8, Hkv=2, Lq=4, D=128, page_size=64, n_pages=9, max_pages=4, sm_scale=scale)
    assert lib.arl2_kv_attn_fwd(ctypes.byref(d), *PTR) == 1
    assert b"sm_scale" in lib.arl2_last_error()
    assert lib.arl2_kv_workspace_bytes(ctypes.byref(d)) == 0


def test_the_largest_scale_is_taken(A):
    lib = A.load_library()
    d = A.arl2_kv_desc(B=2, H=8, Hkv=2, Lq=4, D=128, page_size=64, n_pages=9, max_pages=2048, sm_scale=2.0 ** 127)
    assert lib.arl2_kv_workspace_bytes(ctypes.byref(d)) > 0
