"""Attention over the 4-bit cache held to the limits of its roundings (tests/kv_checks.py), to single keys that matter, and to the stream
that it belongs to."""
import numpy as np
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


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D,G,page,L", [(128, 1, 16, 1), (64, 4, 32, 1), (128, 7, 32, 9), (64, 2, 16, 33), (128, 2, 64, 32), (64, 1, 128, 130), (128, 1, 64, 300), (128, 4, 64, 257), (64, 3, 64, 290)])
def test_ragged_streams(A, D, G, page, L, causal):
    lens = [1, 33, 100, 290, 600, 1411]
    pool = R.Paged(A, len(lens), 2, D, page, 1411, seed=L)
    pool.fill_with(lens)
    q = R.bf16_normal((len(lens), L, 2 * G, D), L)
    C.check(A, pool, q, lens, [L, 3, L, 1, max(L - 1, 1), L + 5], causal)
    C.check(A, pool, q, lens, None, causal, sm_scale=0.3)


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D,Hkv,L,G", [(64, 8, 250, 32), (128, 8, 250, 32), (64, 4, 250, 32), (128, 12, 100, 1), (128, 2, 1, 8), (64, 2, 6, 4)])
def test_long_caches_with_dropped_pages(A, D, Hkv, L, G, causal):
    """Splits of the key axis and none, workgroups of several portions of the block table, pages missing about the portions' ends."""
    page, T = 16, 9003
    pool = R.Paged(A, 1, Hkv, D, page, T)
    pool.fill_with([T])
    table = pool.table.copy()
    for at in (0, 4095, 4096, 4544, 8191, 8192, 8992):
        table[0, at // page] = -1
    pool.set_table(table)
    C.check(A, pool, R.bf16_normal((1, L, G * Hkv, D), 3), [T], causal=causal, heads=sorted({0, min(G + 7, G * Hkv - 1), G * Hkv - 1}))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("D,G,L", [(128, 1, 1), (64, 4, 1), (128, 2, 6), (128, 1, 64), (128, 1, 70), (64, 4, 20), (64, 2, 140)])
def test_single_keys_that_matter(A, D, G, L, causal):
    """Each stream has one key that takes most of the weight of a row that sees it: first and last ones, at the ends of pages, tiles and
    splits, past the limit, in dropped pages and beside them."""
    T, cap, page = 1500, 1700, 16
    drop = {40, 41, 80}
    at = [0, 1, 15, 16, 31, 32, 63, 64, 127, 128, 191, 192, 255, 256, 511, 512, 639, 640, 650, 671, 672, 1023, 1024, 1279, 1280, 1295, 1296,
          T - L - 1, T - L, T - L + 1, T - 2, T - 1, T, T + 1, cap - 1]
    B = len(at)
    pool = R.Paged(A, B, 1, D, page, cap)
    pool.fill_with([cap] * B)
    d = torch.sign(R.bf16_normal((D,), 11).float())
    for b, p in enumerate(at):
        k, v = (torch.zeros((B, 1, 1, D), dtype=torch.bfloat16) for _ in range(2))
        k[b, 0, 0], v[b, 0, 0] = (d * (64 / D)).bfloat16(), 6.0
        pool.append(k, v, [p] * B, [int(x == b) for x in range(B)], rope=False)
    table = pool.table.copy()
    table[:, sorted(drop)] = -1
    pool.set_table(table)
    q = (d + 0.25 * R.bf16_normal((B, L, G, D), 5).float()).bfloat16()
    C.check(A, pool, q, [T] * B, causal=causal, sm_scale=0.3)
    limit = np.array([T - L + i + 1 if causal else T for i in range(L)])
    for b, p in enumerate(at):                                        # a row that sees the key gives it weight, ten times the limits and more
        if p // page not in drop and (p < limit).any():
            weight = C.expected(q[b, :, 0].double().numpy(), pool.k[b, :T, 0], pool.v[b, :T, 0], limit, 0.3, pool.seen(b)[:T])[0]
            assert (weight[p < limit, p] > 0.1).all(), (b, p)


@pytest.mark.parametrize("L", [1, 40, 300])
@pytest.mark.parametrize("D", [64, 128])
def test_streams_do_not_reach_each_other(A, D, L):
    """Whatever another stream's queries, lengths, pages and rows are, a stream's output, and what it reads, keep their bits."""
    pool = R.Paged(A, 3, 2, D, 32, 2000)
    lens = [1999, 1400, 3]
    pool.fill_with(lens)
    q = R.bf16_normal((3, L, 4, D), 1).cuda()
    ws = A.alloc_kv_workspace(3, 4, 2, L, D, 32, pool.width)

    def run(x, kv_len, q_len=None, table=pool.table):
        out, k, v = (torch.full(s, 7.0, dtype=torch.bfloat16, device="cuda") for s in ((3, L, 4, D), (3, 50, 2, D), (3, 50, 2, D)))
        dev = torch.from_numpy(np.ascontiguousarray(table)).cuda()
        A.arl2_kv_attn_fwd(x, pool.cache, dev, R.ints(kv_len), out, q_len=None if q_len is None else R.ints(q_len), causal=True, workspace=ws)
        A.arl2_kv_read(pool.cache, dev, R.ints([max(n - 50, 0) for n in kv_len]), k, v)
        return out.cpu(), k.cpu(), v.cpu()

    base = run(q, lens)

    def same(got, *streams):
        for b in streams:
            assert all(torch.equal(x[b].view(torch.int16), y[b].view(torch.int16)) for x, y in zip(got, base)), b

    x = q.clone()
    x[1] *= -30
    x[1, 0, 0, 0] = float("nan")
    same(run(x, lens), 0, 2)
    same(run(q, [1999, 0, 3]), 0, 2)
    same(run(q, [1999, 2 ** 31 - 1, 3], [L, L // 2, L]), 0, 2)
    table = pool.table.copy()
    table[1] = -1
    same(run(q, lens, table=table), 0, 2)
    table[1] = pool.table[0]
    same(run(q, lens, table=table), 0, 2)
    assert not torch.equal(run(q, lens, table=table)[0][1], base[0][1])
    k = R.bf16_normal((3, 60, 2, D), 9)
    k[1, 5] = float("inf")
    pool.append(k, k, [0, 0, 0], [0, 60, 0])
    got = run(q, lens)
    same(got, 0, 2)
    assert got[0][1].isnan().all()
