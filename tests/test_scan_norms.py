"""The limits in the 2-norm reject what the limits element by element let through (mistakes planted in the reference's gradients; no GPU needed)."""
import numpy as np
import pytest

import scan_norms as N
import scan_reference as R

CASES = [dict(B=1, H=1, L=3000, D=128), dict(B=2, H=3, L=513, D=64), dict(B=1, H=1, L=2500, D=64), dict(B=4, H=2, L=300, D=64, lens=[300, 0, 129, 192]),
         dict(B=2, H=2, L=150, D=64, gates="resets"), dict(B=2, H=2, L=150, D=64, gates="one")]


@pytest.mark.parametrize("kw", CASES, ids=str)
def test_gates_gradients_without_what_crosses_a_segments_border(kw):
    c = R.Case(**kw, seed=42)
    E = c.backward()[0][3]
    assert N.gates_off(c, E, E) == 0.0
    for blocks in (1, 16):
        seg, wrong = 64 * blocks, E.copy()
        if seg >= c.L:
            continue
        for t in range(0, c.L - seg, seg):
            wrong[:, t:t + seg] -= E[:, t + seg:t + seg + 1]
        assert N.gates_off(c, E, wrong) > 100.0
    for wrong in (np.zeros_like(E), 1.1 * E, 1.001 * E):
        assert N.gates_off(c, E, wrong) > 10.0
    # at the accuracy that the header states
    noise = np.random.Generator(np.random.Philox(1)).standard_normal(E.shape)
    assert N.gates_off(c, E, E + 4.3e-6 * noise * np.sqrt((E ** 2).mean(1, keepdims=True))) <= 1.0


def test_rows_and_states():
    c = R.Case(2, 2, 150, 64, seed=42)
    dq, dk, dv, _, dS0 = c.backward()[0]
    for x in (dq, dk, dv):
        assert N.rows_off(c, x, x) == 0.0 and N.rows_off(c, x, R.wide(R.bf16(x))) <= 0.5
        for wrong in (0.0 * x, 0.98 * x, np.where(np.arange(150)[:, None, None] == 77, 0.0, x)):
            assert N.rows_off(c, x, wrong) > 1.0
    assert N.state_off(dS0, dS0) == 0.0 and N.state_off(dS0, 0.9999 * dS0) > 1.0
