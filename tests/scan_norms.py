"""Limits in the 2-norm, head by head, for the recurrence's gradients: those element by element allow for every rounding at its worst and in one direction."""
import numpy as np

import scan_reference as R

# dq, dk, dv: a block's products (for dv also the state's features, which other terms have) and the result are rounded to bf16, each off by U16 of a value at the
# most: were all of them that, in one direction, 2 U16.
ROWS = 2.0 * R.U16
# dS0: rows enter in two parts, each off by TWO of a value at the most, in directions of their own.
STATE = R.TWO
# dlog_alpha: a token adds the state's part of q'.dq' and of k'.dk', and pairs' products that go in and out again as one fp32 value.  The state and what enters it are
# in three parts (2^-25) and fp32 sums, so that a token's is off by 2^-22 of what a token has to do with the state, at least its product with itself, E's own
# size or more; up to 1024 such errors add up in directions of their own, by 2^5: 2^-17 of the two in the 2-norm.  Three times that is 2^-15.4: TWO is 2^-15.4.
# Not for gates that leave next to nothing of the state where dS is given: a token's product with dS, which goes in and out again, has nothing to do with the two.
GATES = R.TWO


def own_products(c):
    """(q'.k') (v.dout) of each token with itself."""
    q, k, v, do, iq, ik, _, _, _ = c._inputs()
    return (q * iq * k * ik).sum(-1) * (v * do).sum(-1)


def gates_limit(c, E):
    """[(b, h, first, last, limit)]: of the 2-norm of dlog_alpha's error over the tokens of a segment at its longest."""
    own = own_products(c)
    return [(b, h, t, min(t + R.LONGEST, n), GATES * float(np.sqrt((E[b, t:min(t + R.LONGEST, n), h] ** 2 + own[b, t:min(t + R.LONGEST, n), h] ** 2).sum())))
            for b, n in enumerate(c.lens) for h in range(c.H) for t in range(0, n, R.LONGEST)]


def gates_off(c, E, got):
    """The largest error in units of its limit."""
    return max((float(np.linalg.norm((got - E)[b, t0:t1, h])) / limit for b, h, t0, t1, limit in gates_limit(c, E)), default=0.0)


def rows_off(c, want, got):
    worst = 0.0
    for b, n in enumerate(c.lens):
        for h in range(c.H):
            x, y = want[b, :n, h], got[b, :n, h]
            if n:
                worst = max(worst, float(np.linalg.norm(y - x) / (ROWS * np.linalg.norm(x) + R.TINY * x.size ** 0.5)))
    return worst


def state_off(want, got):
    return max(float(np.linalg.norm(got[i] - want[i]) / (STATE * np.linalg.norm(want[i]) + 1e-30)) for i in np.ndindex(want.shape[:2]))


def check_gradients(c, want, got):
    """dq, dk, dv, dlog_alpha (or None), dS0 (or None) on the device against those in fp64."""
    got = [None if x is None else R.wide(x) for x in got]
    off = {n: rows_off(c, w, g) for n, w, g in zip(("dq", "dk", "dv"), want, got)}
    if got[3] is not None:
        off["dlog_alpha"] = gates_off(c, want[3], got[3])
    if got[4] is not None:
        off["dS0"] = state_off(want[4], got[4])
    assert max(off.values()) <= 1.0, off
