"""The 8-bit linear layer at the very ends of what a row's scale can be: the quantiser's smallest (2^-100 / 127) and its largest (the largest
finite value / 127), with the largest sums there are.  Bounds: 2^-17 of the result for the smallest scales (2^-18 for xs 2^-24, a denormal
number, and three roundings), 2^-22 elsewhere (three float32 roundings of 2^-24 each)."""
import pytest
import torch

import paper_2511_19797_amd as tvm
from tests.test_q8_gpu import linear_inputs, say

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R,K,F", [(3, 65536, 16), (70, 65536, 16), (512, 1152, 4608), (1000, 1152, 3456), (4096, 1152, 1152)])
@pytest.mark.parametrize("xs,ws,bound", [(2.0 ** -100 / 127, 2.0 ** 60, 2.0 ** -17), (3.4028234e38 / 127, 2.0 ** -60, 2.0 ** -22),
                                         (1.37, 1.99 * 2.0 ** 90, 2.0 ** -22)])
def test_ends_of_the_range(R, K, F, xs, ws, bound):
    say("linear_q8 range", R, K, F, xs, ws)
    t = linear_inputs(R, K, F, R + F)
    t["xq"][0], t["wq"][0], t["wq"][-1] = 127, 127, -127
    t["xs"], t["ws"] = torch.full((R,), xs), torch.full((F,), ws)
    assert torch.isfinite(t["xs"]).all() and (t["xs"] > 0).all()
    d = {n: v.cuda() for n, v in t.items()}
    y, _ = tvm.tvmattn_linear_jvp_fwd_q8(d["xq"], d["xs"], None, None, d["wq"], d["ws"], dtype=torch.float32)
    some = torch.arange(0, R, max(1, R // 50))
    ref = (t["xq"][some].double() @ t["wq"].double().t()) * t["xs"][some].double()[:, None] * t["ws"].double()
    got = y[some.cuda()].double().cpu()
    assert torch.isfinite(y).all() and ((got - ref).abs() <= bound * ref.abs()).all(), ((got - ref).abs() / ref.abs().clamp_min(1e-300)).max()
