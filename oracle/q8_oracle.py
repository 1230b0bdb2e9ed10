"""Float64 CPU oracle for 8-bit rows (int8 values with one scale per row) and the linear layer on them.

TEST INFRASTRUCTURE ONLY.  Imported by tests/ and nothing else; it shares no code with the HIP kernels and never calls them.

A row v: s = max|v| / 127, q = v 127 / max|v| rounded to the nearest integer, ties to even; it stands for q s.  Zero rows have s = 0 and
q = 0; rows with a NaN or an infinity s = NaN and q = 0.  The operators whose outputs are such rows (the MLP's activation, the
gated residual with the modulation behind it) are the other oracles' functions, then `rows8`.

Pins (tests/test_q8_oracle.py, tests/test_q8_ties_oracle.py): scalar loops, the largest error of a step's half, rows whose values are whole steps, ties, zero
rows, non-finite rows; the linear layer against its definition in Python integers.
"""
import numpy as np

from oracle import adaln_oracle, gate_oracle


def steps(v):
    """(v in steps of its row, not rounded; s).  v: [..., C] float64."""
    v = np.asarray(v, dtype=np.float64)
    m = np.abs(v).max(-1)
    s = np.where(np.isfinite(m), m / 127, np.nan)
    with np.errstate(divide="ignore", invalid="ignore"):
        # (not v / s, whose s is rounded: max / 2 is a tie whatever max is; 127 v is exact for float32 values)
        t = np.where((m > 0)[..., None] & np.isfinite(m)[..., None], v * 127 / m[..., None], 0.0)
    return t, s


def rows8(v):
    """(q, s): int8 [..., C], float64 [...]."""
    t, s = steps(v)
    return np.rint(t).astype(np.int8), s


def values(q, s):
    return q.astype(np.float64) * np.asarray(s, dtype=np.float64)[..., None]


def linear_fwd(xq, xs, wq, ws, bias=None):
    """xq [R, K], wq [F, K] int8: (sum_k xq wq) xs ws + bias; the sums are exact (below 2^53)."""
    y = (xq.astype(np.float64) @ wq.astype(np.float64).T) * np.asarray(xs, np.float64)[:, None] * np.asarray(ws, np.float64)
    return y if bias is None else y + np.asarray(bias, np.float64)


def gate_adaln_fwd(x, tx, h, th, c, tc, a, ta, b, tb, eps):
    """(z, tz, y, ty) before y and ty become 8-bit rows.  h None: z = x.  tx None: tangents of zero."""
    zero = lambda t, like: np.zeros_like(like) if t is None else t
    tx, ta, tb = zero(tx, x), zero(ta, a), zero(tb, b)
    z, tz = x, tx
    if h is not None:
        z, tz = gate_oracle.gate_jvp_fwd(x, tx, h, zero(th, h), c, zero(tc, c), eps)
    return (z, tz) + tuple(adaln_oracle.adaln_jvp_fwd(z, tz, a, ta, b, tb, eps))
