"""The limits that attention over the 4-bit cache is held to (tests/kv_checks.py): outputs with the kernels' roundings pass, outputs with a
mistake do not."""
import numpy as np
import pytest
import torch

import kv_checks as C
import kv_reference as R


def bf16(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).double().numpy()


def inputs(n, T, D, seed=0):
    r = np.random.default_rng(seed)
    return bf16(r.normal(size=(n, D))), R.quantise(r.normal(size=(T, D))), R.quantise(r.normal(size=(T, D)))


def rounded(q, k, v, limit, scale, seen=None, reference=0.0):
    """Outputs as the kernels round them: probabilities relative to some logit near the largest, outputs."""
    see = np.arange(k.shape[0])[None, :] < np.asarray(limit)[:, None]
    if seen is not None:
        see = see & seen[None, :]
    logit = np.where(see, q @ k.T * scale, -np.inf)
    top = np.where(see.any(-1), logit.max(-1, initial=-np.inf), 0.0)[:, None] - reference
    p = np.exp(logit - top)
    total = p.sum(-1, keepdims=True)
    return bf16(np.divide(bf16(p) @ v, total, out=np.zeros(q.shape), where=total != 0))


@pytest.mark.parametrize("reference", [0.0, 0.3, 3.1])
@pytest.mark.parametrize("n,T,D", [(1, 1, 64), (1, 17, 128), (1, 9003, 128), (5, 3, 128), (16, 2, 64), (20, 257, 64), (250, 1, 128), (250, 40, 64), (250, 9003, 128)])
@pytest.mark.parametrize("std", [0.01, 1.0, 30.0])
def test_roundings_stay_within_the_limits(n, T, D, std, reference):
    q, k, v = inputs(n, T, D, T)
    q = bf16(q * std)
    limit = [max(T - n + i + 1, 0) for i in range(n)]
    _, ref, square, total = C.expected(q, k, v, limit, D ** -0.5)
    one, norm = C.misses(rounded(q, k, v, limit, D ** -0.5, reference=reference), ref, square, total)
    assert one <= 1 and norm <= 1, (one, norm)


@pytest.mark.parametrize("n,T,D", [(1, 600, 128), (20, 700, 64), (250, 9003, 128), (250, 9003, 64)])
def test_mistakes_do_not(n, T, D):
    q, k, v = inputs(n, T, D, 1)
    limit, scale = np.array([T - n + i + 1 for i in range(n)]), D ** -0.5
    seen = np.ones(T, dtype=bool)
    seen[T // 2:T // 2 + 16] = False
    _, ref, square, total = C.expected(q, k, v, limit, scale, seen)
    right = rounded(q, k, v, limit, scale, seen)
    assert max(C.misses(right, ref, square, total)) <= 1
    page = seen | (np.arange(T) // 16 == (T // 2 + 5) // 16)
    lost = seen & ~((np.arange(T) >= 128) & (np.arange(T) < 384))
    other = np.roll(np.arange(T), 16)                                # pages in another order: keys of one token, values of another
    wrong = {"a dropped page seen": rounded(q, k, v, limit, scale, page), "a split lost": rounded(q, k, v, limit, scale, lost),
             "values of other tokens": rounded(q, k, v[other], limit, scale, seen), "scale": rounded(q, k, v, limit, scale * 1.1, seen),
             "nothing": np.zeros_like(right)}
    if n > 1:
        wrong["the last key lost"] = rounded(q, k, v, limit - 1, scale, seen)
        wrong["the first key lost"] = rounded(q, k, v, limit, scale, seen & (np.arange(T) > 0))
        wrong["one key too many"] = rounded(q, k, v, np.minimum(limit + 1, T), scale, seen)
        wrong["not causal"] = rounded(q, k, v, np.full(n, T), scale, seen)
        wrong["one row of another"] = np.concatenate((right[1:2], right[1:]))
    for name, got in wrong.items():
        assert max(C.misses(got, ref, square, total)) > 1, name


@pytest.mark.parametrize("T", [600, 9003])
def test_a_key_that_matters_is_missed_in_a_single_row(T):
    """One row, one key with a quarter of the weight: lost, or seen past the limit."""
    q, k, v = inputs(1, T, 128, 2)
    k[5] = 0.0
    k[5, :32] = np.sign(q[0, :32])
    scale = np.log(0.25 * np.exp(0.5) * T) / (q[0] @ k[5])            # (about: the others' logits are of size one half at most)
    _, ref, square, total = C.expected(q, k, v, [T], scale)
    assert max(C.misses(rounded(q, k, v, [T], scale), ref, square, total)) <= 1
    assert max(C.misses(rounded(q, k, v, [T], scale, np.arange(T) != 5), ref, square, total)) > 1
    _, ref, square, total = C.expected(q, k, v, [T], scale, np.arange(T) != 5)
    assert max(C.misses(rounded(q, k, v, [T], scale), ref, square, total)) > 1


def test_the_query_as_it_is_taken():
    """Worked values, and what the parts leave at most."""
    q = np.zeros((6, 64))
    q[0, :3] = [7.5, 0.234375, 2.0 ** -9]                             # u = 1: two parts leave the last one, less than 2^-9 of the row
    q[1, :2] = [7.53125, 1.0]                                         # beyond 7.5: u = 2
    q[2, :2] = [2.0 ** -105, 2.0 ** -112]                             # the least unit, 2^-100; the last at half the third's step: to even
    q[3, :2] = [255 * 2.0 ** 120, -249 * 2.0 ** 120]                  # the largest of bf16
    q[4, 0] = 2.0 ** -40                                              # short, and exact
    q[5, :32] = 2.0 ** -75 * np.where(np.arange(32) == 0, 1000.0, 1.0078125)
    t = C.taken_query(q)
    assert np.array_equal(t[0, :3], [7.5, 0.234375, 0]) and np.array_equal(t[1], q[1]) and np.array_equal(t[3:5], q[3:5])
    assert t[2, 0] == q[2, 0] and t[2, 1] == 0
    assert t[5, 0] == q[5, 0] and (t[5, 1:32] == 2.0 ** -75).all()    # u = 2^-67: the third part's steps are 2^-78, to even at half of one
    r = np.random.default_rng(0)
    x = bf16(r.normal(size=(4000, 128)) * 2.0 ** r.integers(-90, 100, (4000, 1)) * np.where(r.random((4000, 128)) < 0.02, 300, 1))
    length, rest = np.linalg.norm(x, axis=-1), np.linalg.norm(C.taken_query(x) - x, axis=-1)
    assert (rest <= 2.0 ** -9 * length).all() and rest.max() > 0
    # rows of normal values keep two parts, which leave 2^-10.9 of them in the root of the mean square
    x = bf16(r.normal(size=(4000, 128)))
    left = np.square(C.taken_query(x) - x).sum(-1) / np.square(x).sum(-1)
    assert 2.0 ** -11.0 < np.sqrt(left.mean()) < 2.0 ** -10.8
