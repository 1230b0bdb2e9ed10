"""The 8-bit operators on the GPU against the float64 oracle, element by element.

Tolerances.  8-bit rows: the kernel's value before rounding is off by a few float32 roundings (2^-24) of the row's largest
magnitude, and a sum of C <= 32768 squares by less than 2^-18 of itself: below 2^-16 of the largest magnitude, 127 2^-16 < 0.002 steps.
A step is then off by 1/2 + 0.002 at most, a scale by 2^-16 relative; 0.51 and 2^-15 are asserted.  (Tangents of the norms are
differences of terms a few times their size: 0.55 and 2^-13.)  Floating outputs: half a step of the type (bf16 2^-8, float32
2^-24) of the result, and 2^-20 of the terms that it is the sum of.
"""
import sys

import numpy as np
import pytest
import torch

import paper_2511_19797_amd as tvm
from oracle import block_oracle, gelu_oracle, q8_oracle as orc
from paper_2511_19797_amd import block, workloads as wl
from tests import parity_util as pu

pytestmark = pytest.mark.gpu
EPS = 1e-6
DT = {"f32": torch.float32, "bf16": torch.bfloat16}
HALF = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8}


def say(*a):
    print("[case]", *a, flush=True)
    sys.stdout.flush()


def draw(rng, *shape, dtype="f32", std=1.0):
    return torch.from_numpy(rng.standard_normal(shape, dtype=np.float32) * np.float32(std)).to(DT[dtype])


def check_rows(q, s, ref, off=0.51, scale=2.0 ** -15):
    t, rs = orc.steps(ref)
    q, s = q.cpu().numpy().astype(np.float64), s.cpu().numpy().astype(np.float64)
    assert q.shape == t.shape and s.shape == rs.shape
    worst = float(np.abs(q - t).max())
    assert worst <= off, f"a value is {worst} steps off"
    assert np.all(np.abs(s - rs) <= scale * rs), float(np.abs(s / np.where(rs > 0, rs, 1) - 1).max())
    assert np.abs(q).max() <= 127


def check_close(got, ref, dtype, terms):
    got = got.float().cpu().numpy().astype(np.float64)
    off = np.abs(got - ref) - HALF[dtype] * np.abs(ref) - 2.0 ** -20 * terms
    assert np.isfinite(got).all() and off.max() <= 0, float(off.max())


# ---- rows as they are, and through the activation
ROWS = [
    (1, 8, "bf16"), (1, 4, "f32"), (1, 1152, "bf16"),
    (3, 504, "bf16"), (5, 516, "f32"),           # one chunk per lane and its edge
    (130, 1152, "bf16"), (129, 412, "f32"),
    (7, 2048, "bf16"), (6, 1024, "f32"),         # the widest row of one wave
    (7, 2056, "bf16"), (6, 1028, "f32"),         # one chunk more
    (33, 4608, "bf16"), (9, 8192, "bf16"), (9, 8200, "bf16"), (5, 4100, "f32"),
    (3, 32768, "bf16"), (2, 16384, "f32"),       # the widest of all
]


@pytest.mark.parametrize("tangent", [False, True])
@pytest.mark.parametrize("R,C,dtype", ROWS)
def test_rowquant(R, C, dtype, tangent):
    say("rowquant", R, C, dtype, tangent)
    rng = np.random.default_rng(R + C)
    x, tx = draw(rng, R, C, dtype=dtype), draw(rng, R, C, dtype=dtype, std=30.0)
    q, s, tq, ts = tvm.tvmattn_rowquant_fwd(x.cuda(), tx.cuda() if tangent else None)
    check_rows(q, s, wl.to_f64(x))
    if tangent:
        check_rows(tq, ts, wl.to_f64(tx))
    else:
        assert tq is None and ts is None


@pytest.mark.parametrize("tangent", [False, True])
@pytest.mark.parametrize("R,C,dtype", ROWS)
def test_gelu(R, C, dtype, tangent):
    say("gelu_q8", R, C, dtype, tangent)
    rng = np.random.default_rng(R + C + 1)
    u, tu = draw(rng, R, C, dtype=dtype, std=2.0), draw(rng, R, C, dtype=dtype)
    q, s, tq, ts = tvm.tvmattn_gelu_jvp_fwd_q8(u.cuda(), tu.cuda() if tangent else None)
    a, ta = gelu_oracle.gelu_jvp_fwd(wl.to_f64(u), wl.to_f64(tu))
    check_rows(q, s, a)
    if tangent:
        check_rows(tq, ts, ta)


def test_rows_with_a_pitch_of_a_wider_buffer():
    rng = np.random.default_rng(3)
    wide, twide = draw(rng, 60, 3 * 1152, dtype="bf16"), draw(rng, 60, 3 * 1152, dtype="bf16")
    for at in (0, 1152, 2304):
        x, tx = wide.cuda()[:, at:at + 1152], twide.cuda()[:, at:at + 1152]
        q, s, tq, ts = tvm.tvmattn_rowquant_fwd(x, tx)
        assert q.is_contiguous()
        check_rows(q, s, wl.to_f64(wide[:, at:at + 1152]))
        check_rows(tq, ts, wl.to_f64(twide[:, at:at + 1152]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("C", [1152, 4608])
def test_zero_tiny_and_nonfinite_rows_stay_by_themselves(dtype, C):
    rng = np.random.default_rng(4)
    x = draw(rng, 12, C, dtype=dtype)
    clean = x.clone()
    x[1] = 0
    x[2] = -0.0
    x[3, 5], x[4, C - 1], x[5, 0] = float("nan"), float("inf"), float("-inf")
    x[6] *= 2.0 ** -110                         # below 2^-100: nothing to represent
    x[7] *= 2.0 ** -90
    x[8] *= 2.0 ** 100
    x[9] = torch.finfo(DT[dtype]).max
    bad = (3, 4, 5)
    q, s, _, _ = (None if t is None else t.cpu() for t in tvm.tvmattn_rowquant_fwd(x.cuda()))
    for r in range(12):
        if r in bad:
            assert torch.isnan(s[r]) and not q[r].any()
        elif r in (1, 2, 6):
            assert s[r] == 0 and not q[r].any()
        else:
            check_rows(q[r:r + 1], s[r:r + 1], wl.to_f64(x[r:r + 1]))
    # what is made of such rows: NaN in their own rows, the others as if they were not there
    wq, ws = tvm.tvmattn_rowquant_fwd(draw(rng, 64, C, dtype=dtype).cuda())[:2]
    y = tvm.tvmattn_linear_jvp_fwd_q8(q.cuda(), s.cuda(), None, None, wq, ws)[0].cpu()
    q0, s0, _, _ = tvm.tvmattn_rowquant_fwd(clean.cuda())
    y0 = tvm.tvmattn_linear_jvp_fwd_q8(q0, s0, None, None, wq, ws)[0].cpu()
    assert all(torch.isnan(y[r]).all() for r in bad) and not y[1].any() and not y[6].any()
    assert torch.equal(y[10:], y0[10:]) and torch.equal(y[0], y0[0])


def test_every_bf16_value_against_the_largest():
    """All finite bf16 magnitudes above 2^-100 as the row's largest: scale and steps in float32's whole range."""
    bits = torch.arange(0x0d80, 0x7f80, 7, dtype=torch.int32).to(torch.int16)
    top = bits.view(torch.bfloat16)
    x = (top.double()[:, None] * torch.tensor([1.0, -1.0, 0.5, 0.25, -0.125, 1 / 127, 0.75, 0.0], dtype=torch.float64)).to(torch.bfloat16)
    q, s, _, _ = tvm.tvmattn_rowquant_fwd(x.cuda())
    check_rows(q, s, wl.to_f64(x))
    assert (q[:, 0] == 127).all() and (q[:, 1] == -127).all()


# ---- the gated residual and the modulation
NORMS = [
    (1, 1, 8, "bf16"), (1, 1, 4, "f32"), (1, 3, 1152, "bf16"), (2, 5, 72, "bf16"),
    (3, 130, 412, "f32"), (2, 250, 768, "bf16"), (1, 256, 1152, "bf16"), (16, 4, 1152, "bf16"),
    (2, 37, 2048, "bf16"), (2, 9, 4096, "bf16"), (2, 9, 2048, "f32"), (1, 4500, 64, "bf16"), (70, 1, 520, "f32"),
]


def norm_inputs(B, T, C, dtype, seed):
    rng = np.random.default_rng(seed)
    t = {n: draw(rng, B, T, C, dtype=dtype) for n in ("x", "tx", "h", "th")}
    return t | {n: draw(rng, B, C) for n in ("c", "tc", "a", "ta", "b", "tb")}


ORDER = ("x", "tx", "h", "th", "c", "tc", "a", "ta", "b", "tb")


def norm_call(t, gate=True, tangent=True, **kw):
    use = lambda n: (gate or n not in ("h", "th", "c", "tc")) and (tangent or not n.startswith("t"))
    return tvm.tvmattn_gate_adaln_jvp_fwd_q8(*(t[n].cuda() if use(n) else None for n in ORDER), EPS, **kw)


@pytest.mark.parametrize("gate,tangent", [(True, True), (True, False), (False, True), (False, False)])
@pytest.mark.parametrize("B,T,C,dtype", NORMS)
def test_gate_adaln(B, T, C, dtype, gate, tangent):
    say("gate_adaln_q8", B, T, C, dtype, gate, tangent)
    t = norm_inputs(B, T, C, dtype, 5 * B + T + C)
    z, tz, q, s, tq, ts = norm_call(t, gate, tangent)
    f = {n: wl.to_f64(v) if (gate or n not in ("h", "th", "c", "tc")) and (tangent or not n.startswith("t")) else None for n, v in t.items()}
    rz, rtz, ry, rty = orc.gate_adaln_fwd(*(f[n] for n in ORDER), EPS)
    check_rows(q, s, ry)
    if tangent:
        check_rows(tq, ts, rty, off=0.55, scale=2.0 ** -13)
    else:
        assert tz is None and tq is None and ts is None
    if gate:
        n = lambda v: v / np.sqrt((v * v).mean(-1, keepdims=True) + EPS)
        check_close(z, rz, dtype, np.abs(f["x"]) + np.abs(n(f["c"])[:, None] * f["h"]))
        if tangent:
            big = 4 * (np.abs(f["tx"]) + np.abs(f["h"]).max() * (np.abs(f["tc"]).max() + np.abs(f["c"]).max()) + np.abs(f["th"]) * np.abs(f["c"]).max())
            check_close(tz, rtz, dtype, big)


def test_gate_adaln_in_place_and_into_given_outputs():
    t = norm_inputs(2, 70, 1152, "bf16", 9)
    ref = norm_call(t)
    x, tx = t["x"].cuda(), t["tx"].cuda()
    args = [x, tx] + [t[n].cuda() for n in ORDER[2:]]
    out = (x, tx, torch.empty(2, 70, 1152, dtype=torch.int8, device="cuda"), torch.empty(2, 70, device="cuda"),
           torch.empty(2, 70, 1152, dtype=torch.int8, device="cuda"), torch.empty(2, 70, device="cuda"))
    got = tvm.tvmattn_gate_adaln_jvp_fwd_q8(*args, EPS, out=out)
    assert got[0] is x and got[1] is tx
    for a, b in zip(got, ref):
        assert torch.equal(a, b)


def test_gate_adaln_rows_stay_by_themselves():
    t = norm_inputs(2, 9, 1152, "bf16", 10)
    ref = [r.cpu() for r in norm_call(t)]
    t["x"][1, 4, 7] = float("inf")
    t["th"][0, 2, 3] = float("nan")
    got = [r.cpu() for r in norm_call(t)]
    assert torch.isnan(got[3][1, 4]) and not got[2][1, 4].any() and torch.isnan(got[5][1, 4])
    assert torch.isnan(got[5][0, 2]) and not got[4][0, 2].any() and torch.equal(got[2][0], ref[2][0])
    keep = torch.ones(2, 9, dtype=torch.bool)
    keep[1, 4] = keep[0, 2] = False
    for a, b in zip(got, ref):
        assert torch.equal(a[keep], b[keep])


def test_gate_adaln_with_a_modulation_that_is_not_finite():
    """z is NaN where the two separate operators make it so, and nowhere else; rows that take such a vector are NaN."""
    for at, v in ((1151, float("inf")), (3, float("-inf")), (700, float("nan"))):
        t = norm_inputs(2, 6, 1152, "bf16", 11)
        t["c"][1, at] = v
        z, tz, q, s, tq, ts = norm_call(t)
        ref, tref = tvm.tvmattn_gate_jvp_fwd(*(t[n].cuda() for n in ("x", "tx", "h", "th", "c", "tc")), EPS)
        assert torch.equal(torch.isnan(z), torch.isnan(ref)) and torch.equal(torch.isnan(tz), torch.isnan(tref))
        assert torch.isnan(s[1]).all() and not q[1].any() and torch.isfinite(s[0]).all() and torch.isfinite(z[0]).all()


def test_gate_adaln_against_the_two_operators():
    """z and the modulated tokens of the bf16 operators: z to one rounding, the 8-bit rows to half a step and the roundings between."""
    t = {n: v.cuda() for n, v in norm_inputs(4, 100, 1152, "bf16", 12).items()}
    z, tz, q, s, tq, ts = norm_call(t)
    rz, rtz = tvm.tvmattn_gate_jvp_fwd(*(t[n] for n in ORDER[:6]), EPS)
    y, ty = tvm.tvmattn_adaln_jvp_fwd(rz, rtz, *(t[n] for n in ORDER[6:]), EPS)
    assert torch.allclose(z.float(), rz.float(), rtol=2 ** -7, atol=1e-6) and torch.allclose(tz.float(), rtz.float(), rtol=2 ** -7, atol=1e-5)
    for r, k, v in ((q, s, y), (tq, ts, ty)):
        assert ((r.float() * k.unsqueeze(-1) - v.float()).abs() <= 0.5 * k.unsqueeze(-1) + 2 ** -6 * v.float().abs().amax(-1, keepdim=True)).all()


# ---- the linear layer
LINEAR = [
    (1, 16, 8), (1, 1152, 6912), (2, 48, 40), (7, 4608, 1152), (16, 1152, 1160), (17, 1168, 72), (33, 32, 8),
    (64, 128, 64), (65, 144, 72), (250, 768, 2304), (256, 1152, 1152), (500, 400, 1000), (129, 112, 136),
    (300, 4624, 264), (1000, 1152, 3456), (1030, 2320, 520), (2100, 64, 2056), (4000, 1152, 1152), (70, 65536, 16),
    (9000, 64, 1160), (9000, 112, 1160), (9000, 208, 1160),   # several output tiles per workgroup, of one and two contraction tiles
    (1000, 1168, 3456), (600, 1024, 5000), (530, 2048, 3480),  # 256 x 128 tiles, rows in 64-byte pieces and not
    (9, 1152, 40), (8, 2064, 1160), (16, 4608, 200),           # a handful of rows, two sets of them and one; 4 waves and 8
]


def linear_inputs(R, K, F, seed, extreme=False):
    rng = np.random.default_rng(seed)
    ints = lambda *s: torch.from_numpy(rng.integers(-128 if extreme else -127, 128, s, dtype=np.int8))
    t = {"xq": ints(R, K), "txq": ints(R, K), "wq": ints(F, K)}
    if extreme:                                      # the largest sum there is
        t["xq"][0], t["wq"][0], t["wq"][-1] = -128, -128, 127
    t |= {n: torch.from_numpy((0.01 + rng.random(k)).astype(np.float32)) for n, k in (("xs", R), ("txs", R), ("ws", F))}
    return t | {"bias": torch.from_numpy(rng.standard_normal(F).astype(np.float32) * 1000)}


def linear_check(t, y, ty, dtype, bias):
    n = {k: v.numpy() for k, v in t.items()}
    b = wl.to_f64(t["bias"].to(DT[dtype])) if bias else None
    plain = orc.linear_fwd(n["xq"], n["xs"], n["wq"], n["ws"])
    check_close(y, plain if b is None else plain + b, dtype, np.abs(plain) + (0 if b is None else np.abs(b)))
    if ty is not None:
        ref = orc.linear_fwd(n["txq"], n["txs"], n["wq"], n["ws"])
        check_close(ty, ref, dtype, np.abs(ref))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("tangent,bias", [(True, True), (False, False)])
@pytest.mark.parametrize("R,K,F", LINEAR)
def test_linear(R, K, F, dtype, tangent, bias):
    say("linear_q8", R, K, F, dtype, tangent, bias)
    t = linear_inputs(R, K, F, R + K + F, extreme=K == 65536)
    d = {n: v.cuda() for n, v in t.items()}
    y, ty = tvm.tvmattn_linear_jvp_fwd_q8(d["xq"], d["xs"], d["txq"] if tangent else None, d["txs"] if tangent else None, d["wq"],
                                          d["ws"], d["bias"].to(DT[dtype]) if bias else None, dtype=DT[dtype])
    assert y.dtype == DT[dtype] and (ty is None) == (not tangent)
    linear_check(t, y, ty, dtype, bias)


@pytest.mark.parametrize("R,K,F", [(1, 1152, 96), (40, 160, 96), (300, 1152, 520), (1500, 400, 1000)])
def test_linear_with_pitches_leaves_the_rest_alone(R, K, F):
    t = linear_inputs(R, K, F, 3)
    d = {n: v.cuda() for n, v in t.items()}
    wide = torch.full((2, R, K + 48), 77, dtype=torch.int8, device="cuda")
    wide[0, :, 16:16 + K], wide[1, :, 16:16 + K] = d["xq"], d["txq"]
    for dtype in ("bf16", "f32"):
        out = torch.full((2, R + 2, 3 * F), 5.0, dtype=DT[dtype], device="cuda")
        y, ty = (o[1:R + 1, F:2 * F] for o in out)
        tvm.tvmattn_linear_jvp_fwd_q8(wide[0, :, 16:16 + K], d["xs"], wide[1, :, 16:16 + K], d["txs"], d["wq"], d["ws"],
                                      d["bias"].to(DT[dtype]), dtype=DT[dtype], out=(y, ty))
        linear_check(t, y, ty, dtype, True)
        out[:, 1:R + 1, F:2 * F] = 5.0
        assert (out == 5.0).all()


def test_linear_batched_rows_and_row_ranges():
    t = linear_inputs(60, 1152, 256, 5)
    d = {n: v.cuda() for n, v in t.items()}
    whole, _ = tvm.tvmattn_linear_jvp_fwd_q8(d["xq"], d["xs"], None, None, d["wq"], d["ws"])
    y, _ = tvm.tvmattn_linear_jvp_fwd_q8(d["xq"].view(3, 20, 1152), d["xs"].view(3, 20), None, None, d["wq"], d["ws"])
    assert y.shape == (3, 20, 256) and torch.equal(y.view(60, 256), whole)
    part, _ = tvm.tvmattn_linear_jvp_fwd_q8(d["xq"][7:40], d["xs"][7:40], None, None, d["wq"], d["ws"])  # scales aligned to 4 bytes
    assert torch.equal(part, whole[7:40])


# ---- together
def fake8(v):
    return orc.values(*orc.rows8(v))


@pytest.mark.parametrize("B,T,H,d,hidden", [(2, 200, 4, 72, 1152), (1, 130, 2, 64, 256), (1, 256, 16, 72, 4608), (1, 1, 2, 64, 512)])
def test_block(B, T, H, d, hidden, monkeypatch):
    """One block's forward with its linear layers in 8 bits against the chained float64 oracles whose linear layers take the values
    of 8-bit rows.  The stages between them round to bf16 (2^-8 each, ten stages: the bound of the bf16 chain, 4e-2), and where that
    moves a value over the border between two steps, one product's operand differs by a step, 2^-7 of its row's largest: of the same size, and rare."""
    say("block_q8", B, T, H, d, hidden)
    x, tx, mods, tmods, params, _, _ = wl.make_block_inputs(B, T, H, d, hidden, seed=17 + T)
    dev = lambda m: {k: v.cuda() for k, v in m.items()}
    z, tz = block.block_jvp_fwd_q8(x.cuda(), tx.cuda(), dev(mods), dev(tmods), block.block_q8_params(dev(params)), H, EPS, EPS)
    f = wl.to_f64
    ff = lambda m: {k: f(v) for k, v in m.items()}
    lin = block_oracle.linear_oracle.linear_jvp_fwd
    monkeypatch.setattr(block_oracle.linear_oracle, "linear_jvp_fwd", lambda x, tx, w, b: lin(fake8(x), fake8(tx), fake8(w), b))
    rz, rtz = block_oracle.block_jvp_fwd(f(x), f(tx), ff(mods), ff(tmods), ff(params), H, EPS, EPS)
    err = {n: pu.rel_err(g.float().cpu().numpy(), r) for n, g, r in (("z", z, rz), ("tz", tz, rtz))}
    print("   max|err|/max|ref|:", err, flush=True)
    assert max(err.values()) <= 4e-2, err


def test_captured_and_replayed():
    """A block in a graph, replayed on new inputs with eager work and synchronisations between, against eager calls, bit for bit."""
    B, T, H, d, hidden = 1, 100, 2, 64, 256
    x, tx, mods, tmods, params, _, _ = wl.make_block_inputs(B, T, H, d, hidden, seed=3)
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
    for n in range(4):
        x.copy_(torch.randn(B, T, H * d))
        tx.copy_(torch.randn(B, T, H * d))
        graph.replay()
        torch.cuda.synchronize()
        got = z.clone(), tz.clone()
        ref = call()
        torch.cuda.synchronize()
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1]), n


def test_two_streams_at_once():
    t = [linear_inputs(300, 1152, 520, s) for s in (1, 2)]
    d = [{n: v.cuda() for n, v in u.items()} for u in t]
    run = lambda e: tvm.tvmattn_linear_jvp_fwd_q8(e["xq"], e["xs"], e["txq"], e["txs"], e["wq"], e["ws"])
    ref = [run(e) for e in d]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [None, None]
    for _ in range(5):
        for n, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[n] = run(d[n])
    torch.cuda.synchronize()
    for a, b in zip(got, ref):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


# ---- the binding: native and Python ways, what it refuses
def binding_calls():
    t = norm_inputs(2, 5, 64, "bf16", 1)
    d = {n: v.cuda() for n, v in t.items()}
    x = d["x"].view(10, 64)
    e = {n: v.cuda() for n, v in linear_inputs(10, 64, 40, 2).items()}
    b = e["bias"].bfloat16()
    wide = torch.randn(10, 192, device="cuda")
    return {
        "rowquant": (tvm.tvmattn_rowquant_fwd, [(x, None), (x, x), (wide[:, 64:128], wide[:, :64]), (d["x"], None)]),
        "gelu_q8": (tvm.tvmattn_gelu_jvp_fwd_q8, [(x, None), (x, x), (wide[:, 64:128], wide[:, :64])]),
        "gate_adaln_q8": (tvm.tvmattn_gate_adaln_jvp_fwd_q8, [
            [d[n] for n in ORDER] + [EPS], [d["x"], d["tx"]] + [None] * 4 + [d[n] for n in ORDER[6:]] + [EPS],
            [d["x"], None, d["h"], None, d["c"], None, d["a"], None, d["b"], None, EPS], [d["x"]] + [None] * 5 + [d["a"], None, d["b"], None, EPS]]),
        "linear_q8": (tvm.tvmattn_linear_jvp_fwd_q8, [
            [e["xq"], e["xs"], e["txq"], e["txs"], e["wq"], e["ws"], b], [e["xq"], e["xs"], None, None, e["wq"], e["ws"]],
            [e["xq"].view(2, 5, 64), e["xs"].view(2, 5), None, None, e["wq"], e["ws"], e["bias"], torch.float32]]),
    }


@pytest.mark.parametrize("name", ["rowquant", "gelu_q8", "gate_adaln_q8", "linear_q8"])
def test_native_calls_against_the_python(monkeypatch, name):
    from tests.test_fastcall import both
    fn, calls = binding_calls()[name]
    for a in calls:
        both(monkeypatch, name, "native", fn, *a)
    if name != "linear_q8":
        fn, calls = binding_calls()[name]
        a = [t.double() if isinstance(t, torch.Tensor) and t.dtype == torch.bfloat16 else t for t in calls[0]]
        both(monkeypatch, name, "python", fn, *a)


def refused(fn, *a, **kw):
    with pytest.raises((ValueError, tvm.TvmattnError)):
        fn(*a, **kw)


def test_refusals():
    q = tvm.tvmattn_rowquant_fwd
    x = torch.randn(6, 64, device="cuda")
    refused(q, x.half())
    refused(q, x.expand(6, 64)[:1].expand(6, 64))        # rows that overlap
    refused(q, x.t())
    refused(q, x[:, 1:61])                               # misaligned
    refused(q, x[:, :62])
    refused(q, x, x[:, :32])
    refused(q, x, x.bfloat16())
    refused(q, x.view(2, 3, 64)[:, :, :32])              # a non-contiguous view of three dimensions
    refused(q, torch.empty(0, 64, device="cuda"))
    refused(q, torch.empty(4, 0, device="cuda"))
    refused(q, x, out=(torch.empty(6, 64, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda"),
                       torch.empty(6, 64, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda")))
    refused(q, x, out=(torch.empty(6, 32, dtype=torch.int8, device="cuda"), torch.empty(6, device="cuda"), None, None))
    t = {n: v.cuda() for n, v in norm_inputs(2, 3, 64, "bf16", 1).items()}
    full = [t[n] for n in ORDER]
    for n in range(10):                                  # each of them missing, each of them of another shape
        refused(tvm.tvmattn_gate_adaln_jvp_fwd_q8, *full[:n], None, *full[n + 1:], EPS) if n else None
        refused(tvm.tvmattn_gate_adaln_jvp_fwd_q8, *full[:n], full[n][:1], *full[n + 1:], EPS)
    refused(tvm.tvmattn_gate_adaln_jvp_fwd_q8, *full, -1.0)
    e = {n: v.cuda() for n, v in linear_inputs(6, 64, 40, 1).items()}
    args = [e["xq"], e["xs"], e["txq"], e["txs"], e["wq"], e["ws"], e["bias"]]
    f = lambda *a, **kw: tvm.tvmattn_linear_jvp_fwd_q8(*a, dtype=torch.float32, **kw)
    for n in range(7):
        refused(f, *args[:n], args[n].double(), *args[n + 1:])
        refused(f, *args[:n], args[n][:-1], *args[n + 1:])
    refused(f, *args[:2], None, *args[3:])
    refused(f, *args[:3], None, *args[4:])
    refused(tvm.tvmattn_linear_jvp_fwd_q8, *args, dtype=torch.float16)
    refused(tvm.tvmattn_linear_jvp_fwd_q8, *args)        # a float32 bias with bfloat16 results
    refused(f, *args, out=(torch.empty(6, 40, device="cuda"), None))
    refused(f, *args, out=(torch.empty(5, 40, device="cuda"), torch.empty(5, 40, device="cuda")))
    y = torch.empty(6, 40, device="cuda")
    refused(f, *args, out=(y, y))


def test_another_device_than_the_current_one_is_refused(monkeypatch):
    x = torch.randn(6, 64, device="cuda")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    monkeypatch.setattr(tvm.binding, "_fast", tvm.binding._PythonOnly())
    refused(tvm.tvmattn_rowquant_fwd, x)
    refused(tvm.tvmattn_gate_adaln_jvp_fwd_q8, x.view(1, 6, 64), None, None, None, None, None, x[:1], None, x[:1], None, EPS)


def test_results_do_not_depend_on_what_was_there_before():
    """Every output element is written: outputs of a poisoned allocator pool against those of a clean one."""
    t = norm_inputs(3, 33, 72, "bf16", 4)
    e = {n: v.cuda() for n, v in linear_inputs(77, 144, 200, 5).items()}
    def all_calls():
        z = norm_call(t)
        q = tvm.tvmattn_rowquant_fwd(t["x"].cuda(), t["tx"].cuda())
        y = tvm.tvmattn_linear_jvp_fwd_q8(e["xq"], e["xs"], e["txq"], e["txs"], e["wq"], e["ws"])
        return [r.clone() for r in (*z, *q, *y)]
    first = all_calls()
    for _ in range(3):
        for n in (64, 1 << 10, 1 << 14, 1 << 16):
            torch.full((n,), float("nan"), device="cuda")
        for a, b in zip(all_calls(), first):
            assert torch.equal(a, b)


# ---- offsets past 32 bits: the last rows of a wide or long buffer as in a small call, bit for bit
def test_wide_pitches():
    rng = np.random.default_rng(6)
    x = draw(rng, 40, 64, dtype="bf16").cuda()
    buf = torch.empty(70000, 65536, dtype=torch.bfloat16, device="cuda")          # 9 GB
    buf[:, :64] = 0
    buf[-40:, :64] = x
    for fn in (tvm.tvmattn_rowquant_fwd, tvm.tvmattn_gelu_jvp_fwd_q8):
        q, s, _, _ = fn(buf[:, :64])
        rq, rs, _, _ = fn(x)
        assert torch.equal(q[-40:], rq) and torch.equal(s[-40:], rs) and not q[:-40].any() and not s[:-40].any()
    del buf


@pytest.mark.parametrize("K,F", [(64, 1152), (144, 72)])
def test_linear_with_wide_pitches(K, F):
    R, keep, wide = 5000, 300, 1 << 20
    t = {n: v.cuda() for n, v in linear_inputs(keep, K, F, 8).items()}
    xq = torch.empty(R, wide, dtype=torch.int8, device="cuda")                    # 5 GB
    xq[:, :K] = 0
    xq[-keep:, :K] = t["xq"]
    xs = torch.ones(R, device="cuda")
    xs[-keep:] = t["xs"]
    y = torch.empty(R, wide, dtype=torch.bfloat16, device="cuda")                 # 10 GB
    y[:, F] = 3.0
    bias = t["bias"].bfloat16()
    tvm.tvmattn_linear_jvp_fwd_q8(xq[:, :K], xs, None, None, t["wq"], t["ws"], bias, out=(y[:, :F], None))
    ref, _ = tvm.tvmattn_linear_jvp_fwd_q8(t["xq"], t["xs"], None, None, t["wq"], t["ws"], bias)
    assert torch.equal(y[-keep:, :F], ref) and (y[:-keep, :F] == bias).all() and (y[:, F] == 3.0).all()


def test_long_streams():
    B, T, C = 17, 65536, 2048                                                     # 2.3 G values: 4.6 GB a tensor
    t = norm_inputs(1, 30, C, "bf16", 13)
    x, h = (torch.zeros(B, T, C, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    x[-1, -30:], h[-1, -30:] = t["x"][0].cuda(), t["h"][0].cuda()
    mods = [torch.ones(B, C, device="cuda") for _ in range(3)]
    for m, n in zip(mods, ("c", "a", "b")):
        m[-1] = t[n][0].cuda()
    z, _, q, s, _, _ = tvm.tvmattn_gate_adaln_jvp_fwd_q8(x, None, h, None, mods[0], None, mods[1], None, mods[2], None, EPS)
    rz, _, rq, rs, _, _ = norm_call(t, True, False)
    assert torch.equal(z[-1, -30:], rz[0]) and torch.equal(q[-1, -30:], rq[0]) and torch.equal(s[-1, -30:], rs[0])
    assert (q[0, ::997] == 127).all() and not z[0, ::997].any()                   # rows of zeros: y is the shift, all ones


def test_many_rows():
    """More workgroups than one dimension of a launch holds."""
    R = (1 << 22) + 9
    x = torch.zeros(R, 8, dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.arange(24, device="cuda").view(3, 8).bfloat16()
    q, s, _, _ = tvm.tvmattn_rowquant_fwd(x)
    check_rows(q[-3:], s[-3:], x[-3:].double().cpu().numpy())
    assert not q[:-3].any() and not s[:-3].any()


def test_longest_stream():
    """The row counter steps past the last row, and must not come back as a negative one."""
    T, C = (1 << 31) - 1, 8                                                       # 34 GB
    t = norm_inputs(1, 30, C, "bf16", 14)
    x = torch.zeros(1, T, C, dtype=torch.bfloat16, device="cuda")
    x[:, -30:] = t["x"].cuda()
    a, b = t["a"].cuda(), t["b"].cuda()
    _, _, q, s, _, _ = tvm.tvmattn_gate_adaln_jvp_fwd_q8(x, None, None, None, None, None, a, None, b, None, EPS)
    _, _, rq, rs, _, _ = norm_call(t, False, False)
    assert torch.equal(q[:, -30:], rq) and torch.equal(s[:, -30:], rs)
    assert (q[0, :-30:9973] == q[0, 0]).all() and (s[0, :-30:9973] == s[0, 0]).all() and q[0, 0].abs().max() == 127
