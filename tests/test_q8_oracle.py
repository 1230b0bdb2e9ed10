"""Pins of the 8-bit oracle (oracle/q8_oracle.py) against independent statements of what it computes."""
import numpy as np
import pytest

from oracle import q8_oracle as orc


def test_rows_against_scalar_loops():
    rng = np.random.default_rng(1)
    v = rng.standard_normal((7, 40)) * 10.0 ** rng.integers(-3, 4, (7, 1))
    q, s = orc.rows8(v)
    for i in range(7):
        top = max(abs(float(t)) for t in v[i])
        assert s[i] == pytest.approx(top / 127, rel=1e-15)
        for j in range(40):
            exact = float(v[i, j]) * 127 / top
            assert abs(q[i, j] - exact) <= 0.5 + 1e-12
    assert np.abs(q).max(-1).tolist() == [127] * 7
    assert np.all(np.abs(orc.values(q, s) - v) <= s[:, None] * (0.5 + 1e-12))


def test_whole_steps_ties_and_signs():
    q, s = orc.rows8(np.array([[127.0, -127.0, 3.0, 2.5, 3.5, -2.5, 0.0, 0.49]]))
    assert s.tolist() == [1.0] and q.tolist() == [[127, -127, 3, 2, 4, -2, 0, 0]]


def test_zero_and_nonfinite_rows():
    v = np.array([[0.0, -0.0, 0.0], [1.0, np.nan, 2.0], [1.0, -np.inf, 2.0], [1.0, 2.0, 4.0]])
    q, s = orc.rows8(v)
    assert s[0] == 0 and np.isnan(s[1]) and np.isnan(s[2]) and s[3] == 4 / 127
    assert q[:3].tolist() == [[0] * 3] * 3


def test_linear_in_python_integers():
    rng = np.random.default_rng(2)
    xq, wq = rng.integers(-128, 128, (3, 33), dtype=np.int8), rng.integers(-128, 128, (5, 33), dtype=np.int8)
    xs, ws, b = rng.random(3), rng.random(5), rng.standard_normal(5)
    y = orc.linear_fwd(xq, xs, wq, ws, b)
    for i in range(3):
        for j in range(5):
            total = sum(int(p) * int(q) for p, q in zip(xq[i], wq[j]))
            assert y[i, j] == pytest.approx(total * xs[i] * ws[j] + b[j], rel=1e-13, abs=1e-13)


def test_modulation_without_residual_and_tangent():
    rng = np.random.default_rng(3)
    x, a, b = rng.standard_normal((2, 3, 8)), rng.standard_normal((2, 8)), rng.standard_normal((2, 8))
    z, tz, y, ty = orc.gate_adaln_fwd(x, None, None, None, None, None, a, None, b, None, 1e-6)
    n = lambda v: v / np.sqrt((v * v).mean(-1, keepdims=True) + 1e-6)
    assert np.array_equal(z, x) and not tz.any() and not ty.any()
    assert np.allclose(y, n(x) * n(a)[:, None] + n(b)[:, None], rtol=1e-13)
