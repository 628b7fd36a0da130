"""The paged 4-bit key/value cache on the GPU: appending, reading back and attention against plain 64-bit forms (tests/kv_reference.py)."""
import numpy as np
import pytest
import torch

import kv_reference as R
import workloads as W
from helpers import rel_err_per_head, to_np

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def A():
    import paper_2605_16579_amd as A
    A.load_library()
    return A


def read(A, pool, start, L, count=None, fill=3.0):
    k, v = (torch.full((pool.B, L, pool.Hkv, pool.D), fill, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    A.arl2_kv_read(pool.cache, pool.table_dev, R.ints(start), k, v, count=None if count is None else R.ints(count))
    return k.float().cpu().numpy().astype(np.float64), v.float().cpu().numpy().astype(np.float64)


def check_rows(A, pool):
    """Every row of the pool as the model has it, bit for bit (never-written ones are NaN in both)."""
    cap = pool.width * pool.page
    k, v = read(A, pool, [0] * pool.B, cap)
    placed = np.stack([pool.seen(b) for b in range(pool.B)])[:, :, None, None]
    np.testing.assert_array_equal(k, np.where(placed, pool.k, 0.0))
    np.testing.assert_array_equal(v, np.where(placed, pool.v, 0.0))


# ---- append and read

@pytest.mark.parametrize("D,Hkv,page", [(128, 1, 16), (128, 12, 64), (128, 3, 256), (64, 1, 16), (64, 5, 32), (64, 2, 128)])
def test_rows_are_stored_as_the_format_says(A, D, Hkv, page):
    pool = R.Paged(A, 3, Hkv, D, page, 300, seed=D + page)
    for n, (L, start, count, rope) in enumerate([(1, [0, 17, 299], None, True), (37, [5, 40, 250], [37, 0, 36], True), (64, [64, 128, 16], [63, 64, 1], False),
                                                 (3, [100, 101, 102], [-4, 99, 2], True), (50, [255, 256, 257], None, True)]):
        k, v = R.bf16_normal((3, L, Hkv, D), 10 * n, 1.0 + n), R.bf16_normal((3, L, Hkv, D), 10 * n + 1, 0.1)
        pool.append(k, v, start, count, rope)
        check_rows(A, pool)


def test_an_append_touches_its_rows_alone(A):
    pool = R.Paged(A, 2, 2, 128, 64, 200)
    pool.fill_with([200, 180])
    before = pool.cache.clone()
    pool.append(R.bf16_normal((2, 9, 2, 128), 5), R.bf16_normal((2, 9, 2, 128), 6), [61, 30], [9, 0])
    changed = (pool.cache != before).flatten(2)                       # [page, head, byte]
    pages = {int(pool.table[0, 0]): range(61, 64), int(pool.table[0, 1]): range(0, 6)}
    for p in range(pool.n_pages):
        if p not in pages:
            assert not changed[p].any()
            continue
        mine = np.zeros(64 * 136, dtype=bool)
        for t in pages[p]:
            mine[t * 64:(t + 1) * 64] = True
            mine[64 * 64 + (t // 16) * 1024 + np.arange(64) * 16 + t % 16] = True
            mine[64 * 128 + t * 4:64 * 128 + t * 4 + 4] = True
            mine[64 * 132 + (t // 16) * 64 + np.arange(4) * 16 + t % 16] = True
        assert not (changed[p].cpu().numpy() & ~mine).any()
    check_rows(A, pool)


def test_special_values(A):
    D, n = 128, 12
    x = R.bf16_normal((1, n, 2, D), 3)
    x[0, 0, 0] = 0.0
    x[0, 1, 0, :32] = 0.0
    x[0, 2, 0, 5] = float("inf")
    x[0, 3, 0, 40] = float("nan")
    x[0, 4, 1, 127] = float("-inf")
    x[0, 5, 0] *= 2.0 ** -126                                          # below the least unit
    x[0, 6, 0] = 3.3e38
    x[0, 7, 0] *= 2.0 ** 120
    x[0, 8, 0, :8] = torch.tensor([7.0, 6.5, 5.0, 2.5, 3.5, 0.25, -0.75, -1.25])   # ties
    x[0, 8, 0, 8:32] = 0.5
    x[0, 9, 0, :4] = torch.tensor([7.03125, 7.0, 3.0, -1.0])           # just beyond 7
    x[0, 9, 0, 4:32] = 0.0
    x[0, 10, 0] = 2.0 ** -133                                          # bf16 denormals
    x[0, 11, 0] = torch.tensor([-0.0, 1.0]).repeat(64)
    pool = R.Paged(A, 1, 2, D, 16, n)
    pool.append(x, x.flip(1), [0], rope=False)
    check_rows(A, pool)
    pool.append(x, x.flip(1), [0], rope=True)
    check_rows(A, pool)


def test_rotation_next_to_rounding_borders(A):
    """Rotated values that lie on or next to the borders between codes: cosines and sines that make them so."""
    D, n = 64, 64
    pool = R.Paged(A, 1, 1, D, 64, n)
    r = np.random.default_rng(1)
    x = torch.zeros((1, n, 1, D), dtype=torch.bfloat16)
    x[0, :, 0, 0::2] = 1.0
    borders = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], dtype=np.float32)
    near = borders[r.integers(0, 7, (n, D // 2))]
    steps = r.integers(-1, 2, near.shape)
    pool.cos = np.where(steps < 0, np.nextafter(near, np.float32(0)), np.where(steps > 0, np.nextafter(near, np.float32(9)), near)).astype(np.float32)
    pool.cos[:, 0] = 6.0
    pool.cos[:, 16] = 4.0
    pool.sin = (r.normal(size=near.shape) * 0.5).astype(np.float32)
    pool.append(x, x, [0])
    check_rows(A, pool)


@pytest.mark.parametrize("D", [64, 128])
def test_tables_that_lead_nowhere(A, D):
    pool = R.Paged(A, 2, 2, D, 32, 32 * 5)
    pool.fill_with([160, 160])
    table = pool.table.copy()
    table[0, 1], table[0, 3], table[1, 0], table[1, 4] = -1, pool.n_pages, 2 ** 31 - 1, -2 ** 31
    old = pool.table
    pool.set_table(table)
    check_rows(A, pool)                                                 # zeros there
    pool.append(R.bf16_normal((2, 200, 2, D), 1), R.bf16_normal((2, 200, 2, D), 2), [-20, 7])
    check_rows(A, pool)
    for start in ([2 ** 31 - 1, -2 ** 31], [160, 1000], [-200, 2 ** 30]):
        before = pool.cache.clone()
        pool.append(R.bf16_normal((2, 200, 2, D), 3), R.bf16_normal((2, 200, 2, D), 4), start)
        if start[0] > 0:
            assert torch.equal(pool.cache, before)
        k, v = read(A, pool, start, 200)
        assert start[0] < 0 or ((k == 0).all() and (v == 0).all())
    pool.set_table(old)
    check_rows(A, pool)


def test_read_leaves_rows_past_the_count(A):
    pool = R.Paged(A, 3, 2, 64, 16, 50)
    pool.fill_with([50, 50, 50])
    k, v = read(A, pool, [3, 0, 40], 12, [5, 0, 12], fill=9.0)
    for b, (s, n) in enumerate([(3, 5), (0, 0), (40, 12)]):
        m = min(n, max(0, 50 - s))
        np.testing.assert_array_equal(k[b, :m], pool.k[b, s:s + m])
        np.testing.assert_array_equal(v[b, :m], pool.v[b, s:s + m])
        assert (k[b, n:] == 9.0).all() and (v[b, n:] == 9.0).all()


# ---- attention

LENS = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 129, 255, 256, 257, 300]


@pytest.mark.parametrize("D,page", [(128, 16), (128, 64), (64, 32), (64, 256)])
@pytest.mark.parametrize("G", [1, 3])
def test_one_token_over_every_length(A, D, page, G):
    pool = R.Paged(A, len(LENS), 2, D, page, 300, seed=page)
    pool.fill_with(LENS)
    q = R.bf16_normal((len(LENS), 1, 2 * G, D), 7, 1.5)
    R.check_attention(A, pool, q, LENS)
    R.check_attention(A, pool, q, LENS, causal=True)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D,G,page,L", [(128, 1, 16, 5), (128, 4, 64, 9), (128, 7, 32, 40), (64, 2, 16, 33), (64, 1, 128, 130), (128, 1, 64, 300), (128, 2, 64, 257), (64, 3, 64, 290)])
def test_several_queries(A, D, G, page, L, causal):
    lens = [0, 1, 33, 64, 100, 290, 600, 611]
    q_len = [L, 3, L, 0, 1, L - 1, L, L + 5]
    pool = R.Paged(A, len(lens), 2, D, page, 611, seed=L)
    pool.fill_with(lens)
    q = R.bf16_normal((len(lens), L, 2 * G, D), L)
    R.check_attention(A, pool, q, lens, q_len, causal)
    R.check_attention(A, pool, q, lens, None, causal, sm_scale=0.3)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D,L,G", [(128, 1, 4), (64, 6, 1), (128, 200, 1), (64, 300, 2)])
def test_long_and_short_streams_in_one_call(A, D, L, G, causal):
    lens = [2500, 3, 700, 5000]
    pool = R.Paged(A, 4, 1, D, 64, 5000, seed=2)
    pool.fill_with(lens)
    R.check_attention(A, pool, R.bf16_normal((4, L, G, D), 1), lens, [L, min(L, 2), L, L], causal)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D,Hkv,splits", [(64, 8, 1), (128, 8, 1), (64, 4, 2)])
def test_many_rows_over_long_caches(A, D, Hkv, splits, causal):
    """Workgroups that walk over more tiles than one or two portions of the block table hold, past pages that were dropped."""
    G, L, page, T = 32, 250, 16, 9003
    pool = R.Paged(A, 1, Hkv, D, page, T)
    pool.fill_with([T])
    table = pool.table.copy()
    for at in (4095, 4096, 4544, 8191, 8192, 8992):                          # pages that end and begin portions, or lie about them
        table[0, at // page] = -1
    pool.set_table(table)
    slots = A.arl2_kv_workspace_bytes(1, G * Hkv, Hkv, L, D, page, pool.width) // (4 * (D + 2))
    assert slots == (0 if splits == 1 else Hkv * -(-G * L // 256) * 256 * splits)
    q = R.bf16_normal((1, L, G * Hkv, D), 3)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    ws = A.alloc_kv_workspace(1, G * Hkv, Hkv, L, D, page, pool.width)
    A.arl2_kv_attn_fwd(q.cuda(), pool.cache, pool.table_dev, R.ints([T]), out, causal=causal, workspace=ws)
    got = out.float().cpu().numpy().astype(np.float64)[0]
    limit = [T - L + i + 1 if causal else T for i in range(L)]
    for h in (0, G + 7, G * Hkv - 1):
        one = slice(h // G, h // G + 1)
        ref, bound = R.attend(q[0, :, h:h + 1].double().numpy(), pool.k[0, :T, one], pool.v[0, :T, one], limit, D ** -0.5, pool.seen(0)[:T])
        off = np.abs(got[:, h:h + 1] - ref)
        assert (off <= bound).all(), (h, np.argwhere(~(off <= bound))[:4])


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("B,L", [(200, 1), (70, 66)])
def test_many_streams(A, B, L, causal):
    lens = [(37 * b) % 131 for b in range(B)]
    pool = R.Paged(A, B, 1, 64, 16, 130)
    pool.fill_with(lens)
    R.check_attention(A, pool, R.bf16_normal((B, L, 1, 64), 1), lens, [(5 * b) % (L + 1) for b in range(B)], causal)


def test_lengths_beyond_the_table_are_cut(A):
    pool = R.Paged(A, 3, 1, 128, 16, 48)
    pool.fill_with([48, 48, 48])
    R.check_attention(A, pool, R.bf16_normal((3, 2, 1, 128), 1), [2 ** 31 - 1, -5, 49], [2 ** 31 - 1, 2, -1])


@pytest.mark.parametrize("L", [1, 300])
@pytest.mark.parametrize("std", [0.01, 4.0, 40.0])
def test_small_and_large_logits(A, std, L):
    pool = R.Paged(A, 1, 2, 128, 64, 700)
    pool.fill_with([700], std=std)
    R.check_attention(A, pool, R.bf16_normal((1, L, 2, 128), 3, std), [700])


@pytest.mark.parametrize("L", [1, 260])
def test_growing_logits_raise_the_maximum_again_and_again(A, L):
    """Keys whose logits grow from token to token: every block lies above what the ones before it have seen."""
    pool = R.Paged(A, 1, 1, 64, 32, 900)
    k = torch.ones((1, 900, 1, 64)) * torch.linspace(0.1, 30.0, 900)[None, :, None, None]
    pool.append(k.bfloat16(), R.bf16_normal((1, 900, 1, 64), 1), [0], rope=False)
    R.check_attention(A, pool, torch.ones((1, L, 1, 64)).bfloat16(), [900])
    R.check_attention(A, pool, -torch.ones((1, L, 1, 64)).bfloat16(), [900], causal=True)


@pytest.mark.parametrize("L", [1, 260])
def test_one_feature_far_above_the_others(A, L):
    """The query's parts: features of one group that differ a thousandfold."""
    pool = R.Paged(A, 1, 1, 128, 64, 400)
    pool.fill_with([400])
    q = R.bf16_normal((1, L, 1, 128), 1)
    q[..., 7] *= 30
    q[..., 40:44] *= 0.01
    q[..., 100] = 0.0
    q[:, :1, :, 64:] = 0.0
    R.check_attention(A, pool, q, [400])


@pytest.mark.parametrize("L", [3, 300])
def test_queries_that_are_not_finite_give_nan(A, L):
    pool = R.Paged(A, 1, 2, 128, 64, 100)
    pool.fill_with([100])
    q = R.bf16_normal((1, L, 2, 128), 1)
    q[0, 0, 0, 3], q[0, 1, 1, 99], q[0, L - 1, 0, 64] = float("nan"), float("inf"), float("-inf")
    out = torch.empty(q.shape, dtype=torch.bfloat16, device="cuda")
    A.arl2_kv_attn_fwd(q.cuda(), pool.cache, pool.table_dev, R.ints([100]), out, workspace=A.alloc_kv_workspace(1, 2, 2, L, 128, 64, pool.width))
    nan = torch.isnan(out).cpu()
    want = torch.zeros(1, L, 2, 128, dtype=torch.bool)
    want[0, 0, 0] = want[0, 1, 1] = want[0, L - 1, 0] = True
    assert torch.equal(nan, want)


@pytest.mark.parametrize("L", [3, 300])
@pytest.mark.parametrize("tokens", [0, 20, 600])
def test_queries_that_are_not_finite_and_see_nothing_give_zeros(A, tokens, L):
    pool = R.Paged(A, 2, 1, 128, 16, 640)
    pool.fill_with([tokens, 640])
    table = pool.table.copy()
    table[0] = -1                                                            # stream 0: every page dropped
    table[1, 1:] = -1
    pool.set_table(table)
    q = R.bf16_normal((2, L, 2, 128), 1)
    q[:, 0, 0, 5], q[:, 1, 1, 127], q[:, 2, 0, 64] = float("nan"), float("inf"), -float("inf")
    out = R.check_attention(A, pool, q, [tokens, 640])
    assert (out[0] == 0).all() and out[1].isnan().any()
    # causal, more queries than tokens: the first queries see nothing
    pool = R.Paged(A, 1, 1, 128, 16, 640)
    pool.fill_with([2])
    out = R.check_attention(A, pool, q[:1], [min(2, L - 2)], causal=True)
    assert (out[0, :2] == 0).all()


@pytest.mark.parametrize("L", [5, 300])
@pytest.mark.parametrize("where", ["key", "value"])
def test_rows_that_are_not_finite_reach_only_queries_that_see_them(A, where, L):
    T = 333
    for at in (T - L // 2, T - L, 3, T - 1):
        pool = R.Paged(A, 1, 1, 128, 64, 400)
        k, v = R.bf16_normal((1, T, 1, 128), 1), R.bf16_normal((1, T, 1, 128), 2)
        (k if where == "key" else v)[0, at, 0, 70] = float("inf")
        pool.append(k, v, [0], rope=False)
        out = R.check_attention(A, pool, R.bf16_normal((1, L, 1, 128), 3), [T], causal=True)
        first = max(0, at - (T - L))                                   # the first query that sees it
        nan = torch.isnan(out)[0, :, 0].cpu()
        assert not nan[:first].any() and nan[first:, 64:96].all() and (where == "key") == bool(nan[first:, :64].all())


@pytest.mark.parametrize("L,D", [(1, 128), (6, 64), (290, 128), (270, 64)])
@pytest.mark.parametrize("page", [16, 64])
def test_dropped_pages_are_not_seen(A, L, D, page):
    pool = R.Paged(A, 4, 1, D, page, 1300)
    pool.fill_with([1300, 1300, 500, 1300])
    table = pool.table.copy()
    table[0, 3:9] = -1                                                  # a window with the first pages kept
    table[1, :] = -1                                                    # nothing left
    table[2, ::2] = pool.n_pages + 5
    table[3, 512 // page] = -7
    pool.set_table(table)
    for causal in (False, True):
        R.check_attention(A, pool, R.bf16_normal((4, L, 2, D), 1), [1300, 1300, 500, 1290], causal=causal)


def test_streams_may_share_pages(A):
    pool = R.Paged(A, 2, 2, 128, 64, 256)
    pool.fill_with([256, 256])
    table = pool.table.copy()
    table[1, :2] = table[0, :2]
    table[1, 3] = table[1, 2]                                           # and a page may stand in a row twice
    pool.set_table(table)
    pool.k[1, :128], pool.v[1, :128] = pool.k[0, :128], pool.v[0, :128]
    pool.k[1, 192:], pool.v[1, 192:] = pool.k[1, 128:192], pool.v[1, 128:192]
    R.check_attention(A, pool, R.bf16_normal((2, 3, 4, 128), 1), [256, 250])


@pytest.mark.parametrize("L", [1, 140])
def test_a_pool_beyond_four_gigabytes(A, L):
    heads, D, page = 8, 128, 256
    n_pages = (1 << 32) // (heads * page * 136) + 40
    pool = R.Paged(A, 1, heads, D, page, 600)
    pool.cache = A.alloc_kv_cache(n_pages, heads, page, D)
    assert pool.cache.nbytes > 1 << 32
    pool.n_pages = n_pages
    pool.set_table([[n_pages - 1, 0, n_pages - 17]])
    pool.fill_with([600])
    k, v = read(A, pool, [0], 600)
    np.testing.assert_array_equal(k, pool.k[:, :600])
    np.testing.assert_array_equal(v, pool.v[:, :600])
    R.check_attention(A, pool, R.bf16_normal((1, L, heads, D), 1), [600])


def test_attention_without_its_workspace_is_refused(A):
    pool = R.Paged(A, 1, 1, 64, 16, 4096)
    q = R.bf16_normal((1, 1, 1, 64), 1).cuda()
    assert A.arl2_kv_workspace_bytes(1, 1, 1, 1, 64, 16, pool.width) > 0
    with pytest.raises(A.Arl2Error, match="workspace"):
        A.arl2_kv_attn_fwd(q, pool.cache, pool.table_dev, R.ints([5]), torch.empty_like(q))


def test_binding_checks_device_tensors(A):
    pool = R.Paged(A, 1, 1, 64, 16, 64)
    q = R.bf16_normal((1, 2, 1, 64), 1).cuda()
    lens = R.ints([5])
    for bad in (dict(q=q.float()), dict(q=q.transpose(0, 1)), dict(kv_len=lens.long()), dict(kv_len=R.ints([5, 5])), dict(out=q[:, :1]), dict(kv_len=lens.cpu())):
        a = dict(q=q, kv_len=lens, out=torch.empty_like(q), **{})
        a.update(bad)
        with pytest.raises((ValueError, TypeError)):
            A.arl2_kv_attn_fwd(a["q"], pool.cache, pool.table_dev, a["kv_len"], a["out"])
    with pytest.raises(ValueError, match="rope_cos"):
        A.arl2_kv_append(q, q, pool.cache, pool.table_dev, lens, rope_cos=torch.zeros(2, 32, device="cuda"), rope_sin=torch.zeros(64, 32, device="cuda"))
    with pytest.raises(A.Arl2Error, match="together"):
        A.arl2_kv_append(q, q, pool.cache, pool.table_dev, lens, rope_cos=torch.zeros(64, 32, device="cuda"))


@pytest.mark.parametrize("L,B", [(1, 3), (300, 1)])
def test_runs_are_bit_identical_and_streams_independent(A, L, B):
    pool = R.Paged(A, B, 2, 128, 64, 3000)
    lens = [3000, 17, 1234][:B]
    pool.fill_with(lens)
    q = R.bf16_normal((B, L, 4, 128), 1)
    a = R.check_attention(A, pool, q, lens, causal=True)
    for _ in range(3):
        assert torch.equal(a, R.check_attention(A, pool, q, lens, causal=True))


@pytest.mark.parametrize("L", [1, 300])
def test_captured_calls_follow_their_indexes(A, L):
    """A graph of append, attention and read replayed for growing streams, next to eager calls with a workspace of their own."""
    B, H, D, page, cap = 2, 2, 128, 32, 2048
    pool, twin = (R.Paged(A, B, H, D, page, cap, seed=4) for _ in range(2))
    for p in (pool, twin):
        p.fill_with([100, 1])
    k, v, q = (torch.zeros((B, L, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(3))
    out, rk, rv = (torch.zeros_like(q) for _ in range(3))
    out2, rk2, rv2 = (torch.zeros_like(q) for _ in range(3))
    cos, sin = torch.from_numpy(pool.cos).cuda(), torch.from_numpy(pool.sin).cuda()
    lens = R.ints([100, 1])
    ws, ws2 = (A.alloc_kv_workspace(B, H, H, L, D, page, pool.width) for _ in range(2))
    assert ws is not None

    def step(p, lens_, out_, rk_, rv_, w):
        A.arl2_kv_append(k, v, p.cache, p.table_dev, lens_, rope_cos=cos, rope_sin=sin)
        new = lens_ + L
        A.arl2_kv_attn_fwd(q, p.cache, p.table_dev, new, out_, causal=True, workspace=w)
        A.arl2_kv_read(p.cache, p.table_dev, lens_, rk_, rv_)
        lens_.copy_(new)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(pool, lens.clone(), out, rk, rv, ws)                        # (rows that the first replay writes again)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(pool, lens, out, rk, rv, ws)
    eager = R.ints([100, 1])
    for n in range(4):
        for x, s in ((k, 1), (v, 2), (q, 3)):
            x.copy_(R.bf16_normal((B, L, H, D), 10 * n + s))
        graph.replay()
        step(twin, eager, out2, rk2, rv2, ws2)
        torch.cuda.synchronize()
        assert torch.equal(lens, eager) and torch.equal(out, out2) and torch.equal(rk, rk2) and torch.equal(rv, rv2)
        assert torch.isfinite(out).all() and out.abs().max() > 0


def test_calls_on_another_stream(A):
    pool = R.Paged(A, 1, 2, 128, 64, 2000)
    pool.fill_with([2000])
    q = R.bf16_normal((1, 4, 2, 128), 1).cuda()
    want = torch.empty_like(q)
    ws = A.alloc_kv_workspace(1, 2, 2, 4, 128, 64, pool.width)
    A.arl2_kv_attn_fwd(q, pool.cache, pool.table_dev, R.ints([2000]), want, workspace=ws)
    lens, got, s = R.ints([2000]), torch.empty_like(q), torch.cuda.Stream()
    torch.cuda.synchronize()
    A.arl2_kv_attn_fwd(q, pool.cache, pool.table_dev, lens, got, workspace=ws, stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(got, want)
    got.zero_()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        A.arl2_kv_attn_fwd(q, pool.cache, pool.table_dev, lens, got, workspace=ws)
    s.synchronize()
    assert torch.equal(got, want)


def test_two_calls_at_once(A):
    """On two streams, with a workspace each."""
    pool = R.Paged(A, 1, 2, 128, 64, 4000)
    pool.fill_with([4000])
    q = [R.bf16_normal((1, 8, 4, 128), i).cuda() for i in range(2)]
    ws = [A.alloc_kv_workspace(1, 4, 2, 8, 128, 64, pool.width) for _ in range(2)]
    lens = [R.ints([4000]), R.ints([3210])]
    want = [torch.empty_like(x) for x in q]
    for i in range(2):
        A.arl2_kv_attn_fwd(q[i], pool.cache, pool.table_dev, lens[i], want[i], workspace=ws[0])
    got = [torch.empty_like(x) for x in q]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for i in range(2):
            A.arl2_kv_attn_fwd(q[i], pool.cache, pool.table_dev, lens[i], got[i], workspace=ws[i], stream=streams[i].cuda_stream)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


# ---- together

def test_a_chunk_goes_from_the_softmax_cache_into_the_linear_memory(A, oracle):
    """What a layer does chunk by chunk: append, attend to everything, then hand the oldest chunk to the state and drop its pages."""
    w = W.WORKLOADS["ragged_small"]
    B, H, L, D, page = w.B, w.H, w.L, w.D, 32
    pool = R.Paged(A, B, H, D, page, 3 * L)
    cos, sin = pool.cos, pool.sin
    S = torch.zeros((B, H, D, D), dtype=torch.float32, device="cuda")
    S_ref = np.zeros((B, H, D, D))
    cws = A.alloc_workspace(B, H, L, D, torch.bfloat16)
    for c in range(3):
        k, v, gate = W.clean_inputs(w, c)
        q = W.pass_inputs(w, c, 0)[0]
        pool.append(k, v, [c * L] * B)
        R.check_attention(A, pool, q, [(c + 1) * L] * B)
        if c == 0:
            continue
        rk, rv = (torch.empty((B, L, H, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        A.arl2_kv_read(pool.cache, pool.table_dev, R.ints([(c - 1) * L] * B), rk, rv)
        A.arl2_state_commit(rk, rv, gate.cuda(), S, cws)
        S_ref = oracle.commit(pool.k[:, (c - 1) * L:c * L].astype(np.float32), pool.v[:, (c - 1) * L:c * L].astype(np.float32), W.as_f32_numpy(gate), S_ref)
        assert rel_err_per_head(to_np(S), S_ref) <= 1e-4
        table = pool.table.copy()
        table[:, :c * L // page] = -1                                   # whole pages of what the state now holds
        pool.set_table(table)
    assert (cos == pool.cos).all() and (sin == pool.sin).all()


# ---- the binding's two ways

class Checked(torch.Tensor):
    """A tensor that is no plain torch.Tensor: a call with it is marshalled in Python."""


def test_compiled_and_checked_calls_agree(A, monkeypatch):
    from paper_2605_16579_amd import binding
    seen, host_call = [], binding._host_call

    def recorded(*args):
        seen.append(host_call(*args))
        return seen[-1]

    monkeypatch.setattr(binding, "_host_call", recorded)
    B, Hkv, H, L, D, page, width = 2, 2, 6, 5, 64, 32, 20
    table = torch.randperm(B * width).view(B, width).int().cuda()
    k, v = (R.bf16_normal((B, L, Hkv, D), i).cuda() for i in range(2))
    q, start, count, lens = R.bf16_normal((B, L, H, D), 3).cuda(), R.ints([0, 600]), R.ints([5, 3]), R.ints([5, 603])
    cs, sn = torch.rand(width * page, D // 2, device="cuda"), torch.rand(width * page, D // 2, device="cuda")
    ws = A.alloc_kv_workspace(B, H, Hkv, L, D, page, width)
    assert ws is not None

    def run(wrap, **kw):
        cache = torch.zeros((B * width, Hkv, page, 68), dtype=torch.uint8, device="cuda")
        out, rk, rv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
        for f in (lambda: A.arl2_kv_append(wrap(k), v, cache, table, start, count=count, rope_cos=cs, rope_sin=sn, **kw),
                  lambda: A.arl2_kv_read(cache, table, start, wrap(rk), rv, count=count, **kw),
                  lambda: A.arl2_kv_attn_fwd(wrap(q), cache, table, lens, out, q_len=count, causal=True, sm_scale=0.2, workspace=ws, **kw)):
            f()
        torch.cuda.synchronize()
        return cache, out, rk, rv

    plain = run(lambda t: t)
    assert seen == [0, 0, 0]
    seen.clear()
    checked = run(lambda t: t.as_subclass(Checked))
    assert seen == [None] * 3
    on_stream = run(lambda t: t, stream=torch.cuda.current_stream().cuda_stream)
    for a, b, c in zip(plain, checked, on_stream):
        assert torch.equal(a, b) and torch.equal(a, c) and a.any()
    # what the compiled way does not take is refused by the other
    cache = plain[0]
    for bad in (dict(cache=cache[:, :1].contiguous()), dict(cache=cache.int()), dict(table=table[:1]), dict(start=start.long()), dict(start=R.ints([1])),
                dict(k=k.float()), dict(v=v[:, :2].contiguous()), dict(cs=cs[:-1]), dict(start=start.cpu()), dict(k=k.transpose(1, 2))):
        a = dict(k=k, v=v, cache=cache, table=table, start=start, cs=cs)
        a.update(bad)
        seen.clear()
        with pytest.raises((ValueError, TypeError)):
            A.arl2_kv_append(a["k"], a["v"], a["cache"], a["table"], a["start"], rope_cos=a["cs"], rope_sin=sn)
        assert seen == [None], bad
    with pytest.raises(A.Arl2Error, match="workspace"):
        A.arl2_kv_attn_fwd(q, cache, table, lens, torch.empty_like(q), workspace=ws[:-16])


def test_bench_runs_the_stack_on_the_cache(A):
    import bench
    dev = torch.device("cuda:0")
    dense, four = (bench.stack_execute(A, W, torch, dev, layers=4, hybrid_layers=2, chunks=2, kv_cache=c) for c in ("bf16", "4bit"))
    assert four["softmax_stack"]["readout_calls"] == dense["softmax_stack"]["readout_calls"]
    # 136 bytes of a stored token and head where bf16 takes 512; the workspace is shared by the layers
    assert four["softmax_stack"]["peak_memory_bytes"] < 0.5 * dense["softmax_stack"]["peak_memory_bytes"]
