"""The 8-bit linear layer where a workgroup works on several output tiles of 256 rows, one behind the other.

Each result is exact sums, one product, one fused multiply-add and one rounding, whatever the tiles: the whole call is compared bit
for bit with calls on a few rows at a time, which take the small tiles, and sampled rows with the float64 oracle (tolerances of test_q8_gpu.py).
"""
import pytest
import torch

import paper_2511_19797_amd as tvm
from paper_2511_19797_amd import block, workloads as wl
from tests.test_q8_gpu import DT, EPS, linear_check, linear_inputs, say
from tests.test_q8_rounds_host import PART, ROUNDS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("sets,R,K,F", list(ROUNDS))
def test_several_output_tiles(sets, R, K, F, dtype):
    say("linear_q8 rounds", sets, R, K, F, dtype)
    t = linear_inputs(R, K, F, R + K + F)
    d = {n: v.cuda() for n, v in t.items()}
    bias = d["bias"].to(DT[dtype])
    tan = lambda n, rows: d[n][rows] if sets == 2 else None
    call = lambda rows: tvm.tvmattn_linear_jvp_fwd_q8(d["xq"][rows], d["xs"][rows], tan("txq", rows), tan("txs", rows), d["wq"], d["ws"], bias,
                                                      dtype=DT[dtype])
    y, ty = call(slice(None))
    for r in range(0, R, PART):
        py, pty = call(slice(r, r + PART))
        assert torch.equal(y[r:r + PART], py), r
        assert sets == 1 or torch.equal(ty[r:r + PART], pty), r
    some = torch.unique(torch.cat([torch.arange(0, R, 163), torch.arange(R - 5, R)]))
    part = {n: (v[some] if n in ("xq", "xs", "txq", "txs") else v) for n, v in t.items()}
    linear_check(part, y[some.cuda()], ty[some.cuda()] if sets == 2 else None, dtype, True)


def test_captured_with_256_row_tiles():
    """A block whose linear layers take the 256-row tiles, in a graph: replays on new inputs against eager calls, bit for bit."""
    B, T, H, d, hidden = 4, 1024, 16, 72, 4608
    x, tx, mods, tmods, params, _, _ = wl.make_block_inputs(B, T, H, d, hidden, seed=5)
    dev = lambda m: {k: v.cuda() for k, v in m.items()}
    x, tx, mods, tmods, p = x.cuda(), tx.cuda(), dev(mods), dev(tmods), block.block_q8_params(dev(params))
    call = lambda: block.block_jvp_fwd_q8(x, tx, mods, tmods, p, H, EPS, EPS)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        z, tz = call()
    gen = torch.Generator(device="cuda").manual_seed(6)
    for n in range(4):
        x.copy_(torch.randn(B, T, H * d, generator=gen, device="cuda"))
        tx.copy_(torch.randn(B, T, H * d, generator=gen, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        got = z.clone(), tz.clone()
        ref = call()
        torch.cuda.synchronize()
        assert torch.isfinite(ref[0]).all() and torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1]), n
