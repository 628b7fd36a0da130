"""What attention over the 4-bit cache makes of a query row: of any size that bf16 has, and of that row alone."""
import pytest
import torch

import kv_checks as C
import kv_reference as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2605_16579_amd as A
    A.load_library()
    return A


def one_feature_rows(L, H, D, seed):
    """Rows of one feature of 4.25 among small ones: its first 6-bit part leaves half a step and its second part half of one of its own,
    2^-8.1 of the row, so that it takes a third."""
    q = R.bf16_normal((1, L, H, D), seed, 0.02)
    for i in range(L):
        for h in range(H):
            q[0, i, h, (7 * i + 3 * h) % D] = 4.25 * (-1) ** i
    return q


@pytest.mark.parametrize("L,G", [(64, 1), (65, 1), (40, 3)])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("power", [-106, -98, -90, -76, -62, -31, 0, 40, 62, 100])
def test_rows_of_every_size(A, D, L, G, power):
    """(Logits are the same for every power: sm_scale is its reciprocal.)"""
    pool = R.Paged(A, 1, 1, D, 64, 300)
    pool.fill_with([300])
    q = (one_feature_rows(L, G, D, 1).float() * 2.0 ** power).bfloat16()
    C.check(A, pool, q, [300], sm_scale=2.0 ** (1 - power))
    # without the one feature, and rows of zeros among them
    q = (R.bf16_normal((1, L, G, D), 2).float() * 2.0 ** power).bfloat16()
    q[0, 3:40:5] = 0.0
    C.check(A, pool, q, [300], causal=True, sm_scale=2.0 ** -(power + 3))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("L,G", [(9, 2), (100, 2), (70, 4), (300, 1)])
@pytest.mark.parametrize("D", [64, 128])
def test_a_row_depends_on_itself_alone(A, D, L, G, causal):
    """A query that is changed changes no other: neither those of other tokens, earlier causal ones above all, nor of other heads."""
    pool = R.Paged(A, 1, 2, D, 32, 900)
    pool.fill_with([900], std=1.5)
    q = R.bf16_normal((1, L, 2 * G, D), 4)
    out = torch.full((5,) + tuple(q.shape[1:]), 7.0, dtype=torch.bfloat16, device="cuda")
    ws = A.alloc_kv_workspace(1, 2 * G, 2, L, D, 32, pool.width)
    changed = torch.zeros((L, 2 * G), dtype=torch.bool)
    for i in range(5, L, 16):
        changed[i, i // 16 % (2 * G)] = True
    for n, row in enumerate((None, one_feature_rows(1, 1, D, 3)[0, 0, 0], 40.0, float("nan"), 0.0)):
        x = q.clone()
        if n > 0:
            x[0, changed] = row if n == 1 else x[0, changed] * row
        A.arl2_kv_attn_fwd(x.cuda(), pool.cache, pool.table_dev, R.ints([900]), out[n:n + 1], causal=causal, workspace=ws)
    out = out.cpu().view(torch.int16)
    for n in range(1, 5):
        assert torch.equal(out[n][~changed], out[0][~changed]), n
        assert not torch.equal(out[n][changed], out[0][changed]), n


@pytest.mark.parametrize("L,G", [(64, 1), (65, 1), (33, 4)])
@pytest.mark.parametrize("D", [64, 128])
def test_the_largest_features(A, D, L, G):
    """Features next to the largest of bf16, whose nearest 6-bit float is 2^128."""
    pool = R.Paged(A, 1, 1, D, 64, 300)
    pool.fill_with([300], std=2.0 ** -9)
    q = (R.bf16_normal((1, L, G, D), 1).float().clamp(-3, 3) * 2.0 ** 124).bfloat16()
    for i in range(L):
        q[0, i, :, i % D] = (-1) ** i * (255 - i % 16) * 2.0 ** 120
    C.check(A, pool, q, [300], sm_scale=2.0 ** -118)


@pytest.mark.parametrize("L", [1, 64, 65])
def test_the_largest_scale(A, L):
    pool = R.Paged(A, 1, 1, 128, 64, 300)
    pool.fill_with([300], std=2.0 ** -40)
    q = (R.bf16_normal((1, L, 1, 128), 2).float() * 2.0 ** -90).bfloat16()
    C.check(A, pool, q, [300], sm_scale=2.0 ** 127)
