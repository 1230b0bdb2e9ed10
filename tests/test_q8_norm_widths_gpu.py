"""The norm with 8-bit rows at widths of five to eight chunks per lane that are not full: idle lanes in a chunk, whole chunks past the
row's end, quads past the vectors' end; rows that do not fill the last workgroup.  Tolerances: test_q8_gpu.py."""
import numpy as np
import pytest

from paper_2511_19797_amd import workloads as wl
from oracle import q8_oracle as orc
from tests.test_q8_gpu import EPS, ORDER, check_close, check_rows, norm_call, norm_inputs, say

pytestmark = pytest.mark.gpu
WIDTHS = [(2, 5, 2056, "bf16"), (1, 7, 2600, "bf16"), (3, 3, 3592, "bf16"), (2, 6, 4088, "bf16"), (2, 5, 1028, "f32"), (1, 7, 1540, "f32"),
          (2, 3, 2044, "f32")]


@pytest.mark.parametrize("gate,tangent", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("B,T,C,dtype", WIDTHS)
def test_ragged_wide_rows(B, T, C, dtype, gate, tangent):
    say("gate_adaln_q8 wide", B, T, C, dtype, gate, tangent)
    t = norm_inputs(B, T, C, dtype, B + T + C)
    z, tz, q, s, tq, ts = norm_call(t, gate, tangent)
    f = {n: wl.to_f64(v) if (gate or n not in ("h", "th", "c", "tc")) and (tangent or not n.startswith("t")) else None for n, v in t.items()}
    rz, rtz, ry, rty = orc.gate_adaln_fwd(*(f[n] for n in ORDER), EPS)
    check_rows(q, s, ry)
    if tangent:
        check_rows(tq, ts, rty, off=0.55, scale=2.0 ** -13)
    if gate:
        n = lambda v: v / np.sqrt((v * v).mean(-1, keepdims=True) + EPS)
        check_close(z, rz, dtype, np.abs(f["x"]) + np.abs(n(f["c"])[:, None] * f["h"]))
        if tangent:
            big = 4 * (np.abs(f["tx"]) + np.abs(f["h"]).max() * (np.abs(f["tc"]).max() + np.abs(f["c"]).max()) + np.abs(f["th"]) * np.abs(f["c"]).max())
            check_close(tz, rtz, dtype, big)
