"""The 8-bit linear layer with scales at the ends of float32's range: a sum times its row's scale is far outside it, the result is not.
Tolerances: three float32 roundings of the product (2^-24 each; 2^-20 asserted), half a step of the result's type, as in test_q8_gpu.py."""
import numpy as np
import pytest
import torch

import paper_2511_19797_amd as tvm
from tests.test_q8_gpu import DT, linear_check, linear_inputs, say

pytestmark = pytest.mark.gpu
SHAPES = [(3, 1152, 200), (100, 1152, 200), (512, 1152, 4608), (1000, 1152, 3456), (4096, 1152, 1152)]   # each kernel


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("big,small", [(120, -110), (-95, 100)])
@pytest.mark.parametrize("R,K,F", SHAPES)
def test_scales_at_the_ends_of_the_range(R, K, F, big, small, dtype):
    say("linear_q8 scales", R, K, F, big, small, dtype)
    t = linear_inputs(R, K, F, R + F)
    for n, e in (("xs", big), ("txs", big), ("ws", small)):
        t[n] = t[n] * 2.0 ** e
        assert torch.isfinite(t[n]).all() and (t[n] > 2.0 ** -126).all()
    d = {n: v.cuda() for n, v in t.items()}
    y, ty = tvm.tvmattn_linear_jvp_fwd_q8(d["xq"], d["xs"], d["txq"], d["txs"], d["wq"], d["ws"], d["bias"].to(DT[dtype]), dtype=DT[dtype])
    some = torch.arange(0, R, max(1, R // 60))
    part = {n: (v[some] if n in ("xq", "xs", "txq", "txs") else v) for n, v in t.items()}
    linear_check(part, y[some.cuda()], ty[some.cuda()], dtype, True)


def test_rows_near_the_largest_value():
    """End to end: bf16 tokens of up to 2^120, a weight that brings them down."""
    rng = np.random.default_rng(1)
    x = torch.from_numpy(rng.standard_normal((40, 1152), dtype=np.float32)) * 2.0 ** 117
    w = torch.from_numpy(rng.standard_normal((72, 1152), dtype=np.float32)) * 2.0 ** -60
    xq, xs, _, _ = tvm.tvmattn_rowquant_fwd(x.bfloat16().cuda())
    wq, ws, _, _ = tvm.tvmattn_rowquant_fwd(w.bfloat16().cuda())
    y, _ = tvm.tvmattn_linear_jvp_fwd_q8(xq, xs, None, None, wq, ws)
    ref = (xq.double().cpu() @ wq.double().cpu().t()) * xs.double().cpu()[:, None] * ws.double().cpu()
    assert torch.isfinite(y).all() and ((y.double().cpu() - ref).abs() <= 2.0 ** -8 * ref.abs() + 2.0 ** -20 * ref.abs()).all()
