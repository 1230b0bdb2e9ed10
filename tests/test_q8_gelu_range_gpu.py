"""The activation into 8-bit rows where u is far from zero: rows whose largest value is tiny, and values whose square leaves float32.

Reference in float64 with the activation as u s, s = t / (1 + t) or 1 / (1 + t) from t = exp(-2|w|), w = sqrt(2/pi) (u + 0.044715 u^3):
no difference of numbers near 1, so that its relative error stays at 2^-45 down to exp's underflow.  (0.5 u (1 + tanh w) in float64
has lost everything at u = -9.)
Tolerances.  What the kernel rounds is the exponent 2 w log2 e, at most 110 here: three float32 roundings and those of two constants,
relative 3.5 2^-24, make 110 ln 2 3.5 2^-24 < 2^-15.9 of t, and the rest a few 2^-24.  A row's values and its largest are then
off by 2^-15.8 each, 127 2 2^-15.8 < 0.005 steps, and its scale by 2^-15.8: 0.51 steps and 2^-15 are asserted.
"""
import numpy as np
import pytest
import torch

import paper_2511_19797_amd as tvm
from paper_2511_19797_amd import workloads as wl
from tests.test_q8_gpu import check_rows, say

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def reference(u, tu):
    k = np.sqrt(2 / np.pi)
    with np.errstate(over="ignore", under="ignore"):
        t = np.exp(-2 * k * (np.abs(u) + 0.044715 * np.abs(u) ** 3))
        s, so = np.where(u < 0, t, 1.0) / (1 + t), t / (1 + t) ** 2
        slope = np.where(so > 0, u * so * 2 * k * (1 + 0.134145 * u ** 2), 0.0) + s
    return u * s, slope * tu


def rows(seed, R, C, centre, spread, dtype):
    rng = np.random.default_rng(seed)
    u = torch.from_numpy((centre + spread * rng.uniform(-1, 1, (R, C))).astype(np.float32)).to(DT[dtype])
    return u, torch.from_numpy(rng.standard_normal((R, C)).astype(np.float32)).to(DT[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [1152, 4608])
@pytest.mark.parametrize("centre", [-3.0, -4.5, -6.0, -9.0])
def test_rows_of_negative_values(centre, C, dtype):
    say("gelu_q8 around", centre, C, dtype)
    u, tu = rows(int(-10 * centre) + C, 6, C, centre, 0.2, dtype)
    a, ta = reference(wl.to_f64(u), wl.to_f64(tu))
    q, s, tq, ts = tvm.tvmattn_gelu_jvp_fwd_q8(u.cuda(), tu.cuda())
    check_rows(q, s, a)
    check_rows(tq, ts, ta)
    q0, s0, _, _ = tvm.tvmattn_gelu_jvp_fwd_q8(u.cuda())
    assert torch.equal(q0, q) and torch.equal(s0, s)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_tangents_that_live_at_negative_values_only(dtype):
    """An ordinary row of activations whose tangent is zero but for entries far on the negative side."""
    u, tu = rows(3, 5, 1152, 0.0, 2.0, dtype)
    far, tfar = rows(4, 5, 30, -5.5, 0.5, dtype)
    tu.zero_()
    u[:, 17:1152:38], tu[:, 17:1152:38] = far, tfar
    a, ta = reference(wl.to_f64(u), wl.to_f64(tu))
    q, s, tq, ts = tvm.tvmattn_gelu_jvp_fwd_q8(u.cuda(), tu.cuda())
    check_rows(q, s, a)
    check_rows(tq, ts, ta)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [1e13, 1e20, 3e38, -1e13, -1e20, -3e38])
def test_values_whose_powers_leave_float32(value, dtype):
    """The activation is u or 0 there and its derivative 1 or 0: the row's other tangents stay what they are."""
    u, tu = rows(5, 3, 1152, 0.0, 2.0, dtype)
    u[1, 700] = value
    a, ta = reference(wl.to_f64(u), wl.to_f64(tu))
    assert np.isfinite(a).all() and np.isfinite(ta).all()
    q, s, tq, ts = tvm.tvmattn_gelu_jvp_fwd_q8(u.cuda(), tu.cuda())
    check_rows(q, s, a)
    check_rows(tq, ts, ta)


def test_values_that_are_not_finite():
    """NaN and infinities: the tangent's row is NaN like the row itself, and no other row is touched."""
    u, tu = rows(6, 8, 1152, 0.0, 2.0, "f32")
    clean = [t.cpu() for t in tvm.tvmattn_gelu_jvp_fwd_q8(u.cuda(), tu.cuda())]
    u[1, 3], u[4, 1151], u[6, 64] = float("nan"), float("inf"), float("-inf")
    q, s, tq, ts = (t.cpu() for t in tvm.tvmattn_gelu_jvp_fwd_q8(u.cuda(), tu.cuda()))
    for r in range(8):
        if r in (1, 4, 6):
            assert torch.isnan(s[r]) and torch.isnan(ts[r]) and not q[r].any() and not tq[r].any()
        else:
            for got, want in zip((q, s, tq, ts), clean):
                assert torch.equal(got[r], want[r])
