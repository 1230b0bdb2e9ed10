"""The 8-bit operators around the block's linear layers, as timed cases.

A network that is run and not trained (sampling in a few steps, the target network of the training loss) takes its linear
layers in 8-bit integers: every token row and every output channel of a weight is int8 with one float32 scale.  Four
operators, each with an optional tangent:

* "norm": the gated residual and the normalised modulation behind it, z = x + n(c) h, y = n(z) n(a) + n(b) with
  n(v) = v / sqrt(mean(v^2) + eps), y in 8 bits (`tvmattn_gate_adaln_jvp_fwd_q8`); without h it is the block's entry, z = x.
* "gelu": the MLP's activation (tanh form), its output in 8 bits (`tvmattn_gelu_jvp_fwd_q8`).
* "quant": rows to 8 bits, weights or the attention's output (`tvmattn_rowquant_fwd`).
* "linear": y = (xq wq^T) xs ws + bias on 8-bit rows (`tvmattn_linear_jvp_fwd_q8`).

8-bit rows: s = max|row| / 127, q = round(row / s) to the nearest, ties to even.  They are returned as the values q s that
they stand for, in bfloat16, with the scales.  Sizes are those of the DiT-XL/2 block at 256 and 512 px, ragged ones and small ones.
"""
import math

import torch

own = False

EPS = 1e-6
_DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def _norm(name, B, T, C, dtype="bf16", tangent=True, gate=True):
    return {"name": name, "kind": "norm", "B": B, "T": T, "C": C, "dtype": dtype, "tangent": tangent, "gate": gate}


def _gelu(name, R, C, dtype="bf16", tangent=True):
    return {"name": name, "kind": "gelu", "R": R, "C": C, "dtype": dtype, "tangent": tangent}


def _quant(name, R, C, pitch, dtype="bf16", tangent=True):
    return {"name": name, "kind": "quant", "R": R, "C": C, "pitch": pitch, "dtype": dtype, "tangent": tangent}


def _linear(name, R, K, F, dtype="bf16", tangent=True, bias=True):
    return {"name": name, "kind": "linear", "R": R, "K": K, "F": F, "dtype": dtype, "tangent": tangent, "bias": bias}


def listed():
    return [
        # one image at 256 px behind the attention, forward with tangent: what one call costs when there is little work
        _norm("norm_one_image", 1, 256, 1152),
        # a DiT-XL/2 block at 512 px, the batch one GPU takes, behind the attention
        _norm("norm_512px", 16, 1024, 1152),
        # a block's entry in float32, a cropped batch, a narrow model, sampling (no tangent)
        _norm("norm_entry_ragged", 7, 130, 412, dtype="f32", tangent=False, gate=False),
        # the MLP's activation of that block at 512 px
        _gelu("gelu_512px", 16 * 1024, 4608),
        # a small model's activation in float32, one cropped image, sampling
        _gelu("gelu_small", 250, 1536, dtype="f32", tangent=False),
        # a weight of the MLP's first layer, once per loaded network
        _quant("quant_weight", 4608, 1152, 1152, tangent=False),
        # the attention's output at 512 px, laid out like its queries: rows of a fused [3, C] buffer
        _quant("quant_attention", 16 * 1024, 1152, 3456),
        # the six modulation vectors of one image from its time embedding, float32 out: one row, the weight is all there is to read
        _linear("linear_one_row", 1, 1152, 6912, dtype="f32", tangent=False),
        # the output projection for one image at 256 px, with tangent
        _linear("linear_one_image", 256, 1152, 1152),
        # widths and a row count that no tile divides, float32 out, with tangent
        _linear("linear_ragged", 500, 400, 1000, dtype="f32", bias=False),
        # the MLP's second layer, 32 images at 256 px, sampling
        _linear("linear_mlp_256px", 32 * 256, 4608, 1152, tangent=False),
        # the fused q, k, v projection at 512 px, with tangent
        _linear("linear_qkv_512px", 16 * 1024, 1152, 3456),
    ]


# A drawn case costs no more than the largest listed one of its kind.
_MOST_NORM = 16 * 1024 * 1152
_MOST_GELU = 16 * 1024 * 4608
_MOST_QUANT = 16 * 1024 * 1152
_MOST_LINEAR = 16 * 1024 * 1152 * 3456


def _spread(rng, lo, hi):
    """An integer in [lo, hi], its logarithm evenly spread."""
    return min(hi, max(lo, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _width(rng, unit, lo, hi):
    """A multiple of `unit` in [lo, hi]."""
    return unit * _spread(rng, -(-lo // unit), hi // unit)


def draw(rng):
    kind = rng.choice(["norm", "gelu", "quant", "linear", "linear"])
    f32, tangent = rng.random() < 0.25, rng.random() < 0.5
    dtype, unit, share = ("f32", 4, 2) if f32 else ("bf16", 8, 1)
    if kind == "norm":
        C = _width(rng, unit, 64, 2048)
        T = _spread(rng, 1, min(4096, _MOST_NORM // share // C))
        B = _spread(rng, 1, max(1, min(32, _MOST_NORM // share // C // T)))
        case = _norm("", B, T, C, dtype, tangent, rng.random() < 0.7)
    elif kind == "gelu":
        C = _width(rng, unit, 128, 8192)
        case = _gelu("", _spread(rng, 1, min(16384, _MOST_GELU // share // C)), C, dtype, tangent)
    elif kind == "quant":
        C = _width(rng, unit, 64, 8192)
        R = _spread(rng, 1, min(16384, _MOST_QUANT // share // C))
        case = _quant("", R, C, C * rng.choice([1, 1, 3]), dtype, tangent)
    else:
        K, F = _width(rng, 16, 64, 4608), _width(rng, 8, 64, 6912)
        R = _spread(rng, 1, min(16384, _MOST_LINEAR // (K * F)))
        case = _linear("", R, K, F, dtype, tangent, rng.random() < 0.7)
    return {k: v for k, v in case.items() if k != "name"}


def _to_rows8(t):
    """int8 rows and their scales of a float32 tensor: what a program holds of a weight or of a layer's input."""
    m = t.abs().amax(-1, keepdim=True)
    return torch.round(t * (127 / m.clamp_min(1e-30))).to(torch.int8), (m / 127).squeeze(-1)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    kind, dt = case["kind"], _DT[case["dtype"]]

    def normal(*shape, std=1.0, dtype=torch.float32):
        return (torch.randn(*shape, generator=gen, device="cuda") * std).to(dtype)

    def tokens(*shape, dtype=dt):
        """Activations: rows of different size, a few channels larger than the others."""
        t = torch.randn(*shape, generator=gen, device="cuda")
        t *= torch.exp(0.5 * torch.randn(*shape[:-1], 1, generator=gen, device="cuda"))
        t[..., ::61] *= 4
        return t.to(dtype)

    tangent = case["tangent"]
    if kind == "norm":
        B, T, C = case["B"], case["T"], case["C"]
        t = {"x": tokens(B, T, C), "a": normal(B, C), "b": normal(B, C)}
        if case["gate"]:
            t |= {"h": normal(B, T, C, dtype=dt), "c": normal(B, C)}
        if tangent:
            t |= {"t" + n: normal(*v.shape, dtype=v.dtype) for n, v in list(t.items())}
    elif kind == "gelu":
        t = {"u": normal(case["R"], case["C"], dtype=dt)}
        if tangent:
            t["tu"] = normal(case["R"], case["C"], dtype=dt)
    elif kind == "quant":
        t = {n: tokens(case["R"], case["pitch"])[:, :case["C"]] for n in (("x", "tx") if tangent else ("x",))}
    else:
        R, K, F = case["R"], case["K"], case["F"]
        t = {}
        t["wq"], t["ws"] = _to_rows8(normal(F, K, std=K ** -0.5))
        t["xq"], t["xs"] = _to_rows8(tokens(R, K, dtype=torch.float32))
        if tangent:
            t["txq"], t["txs"] = _to_rows8(tokens(R, K, dtype=torch.float32))
        if case["bias"]:
            t["bias"] = normal(F, std=0.1, dtype=dt)
    return {"case": case, "t": t}


# ---- the framework's calls
def _values(q, s):
    """What int8 rows stand for."""
    return torch.mul(q, s.unsqueeze(-1), out=torch.empty(q.shape, dtype=torch.bfloat16, device=q.device))


def _rows8_out(q, s, tq, ts):
    out = {"y": _values(q, s), "s": s}
    return out if tq is None else out | {"ty": _values(tq, ts), "ts": ts}


def _run_own(case, t):
    import paper_2511_19797_amd as tvm
    kind, get = case["kind"], t.get
    if kind == "norm":
        z, tz, *rows = tvm.tvmattn_gate_adaln_jvp_fwd_q8(t["x"], get("tx"), get("h"), get("th"), get("c"), get("tc"), t["a"], get("ta"),
                                                         t["b"], get("tb"), EPS)
        out = _rows8_out(*rows)
        if case["gate"]:
            out["z"] = z
            if case["tangent"]:
                out["tz"] = tz
        return out
    if kind == "gelu":
        return _rows8_out(*tvm.tvmattn_gelu_jvp_fwd_q8(t["u"], get("tu")))
    if kind == "quant":
        return _rows8_out(*tvm.tvmattn_rowquant_fwd(t["x"], get("tx")))
    y, ty = tvm.tvmattn_linear_jvp_fwd_q8(t["xq"], t["xs"], get("txq"), get("txs"), t["wq"], t["ws"], get("bias"), dtype=_DT[case["dtype"]])
    return {"y": y, "ty": ty} if case["tangent"] else {"y": y}


# ---- the plain forms: elementary operations in float32
def _plain_rows8(y):
    """(the values that the 8-bit rows stand for, the scales)."""
    m = y.abs().amax(-1, keepdim=True)
    s = m / 127
    q = torch.round(y * torch.where(m > 0, 127 / m, 0.0))
    return (q * s).to(torch.bfloat16), s.squeeze(-1)


def _plain_unit(v, tv):
    """v / sqrt(mean(v^2) + eps) and its tangent."""
    r = 1 / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS)
    return v * r, None if tv is None else tv * r - v * (r * r * r) * (v * tv).mean(-1, keepdim=True)


def _plain(case, t):
    kind, tangent = case["kind"], case["tangent"]
    if kind == "linear":
        w = t["wq"].float().t()
        y = (t["xq"].float() @ w) * t["xs"].unsqueeze(-1) * t["ws"]
        if case["bias"]:
            y = y + t["bias"].float()
        out = {"y": y.to(_DT[case["dtype"]])}
        if tangent:
            out["ty"] = ((t["txq"].float() @ w) * t["txs"].unsqueeze(-1) * t["ws"]).to(_DT[case["dtype"]])
        return out
    out = {}
    if kind == "norm":
        f = {n: (v.float() if v.dim() == 3 else v.unsqueeze(1)) for n, v in t.items()}
        a, ta = _plain_unit(f["a"], f.get("ta"))
        b, tb = _plain_unit(f["b"], f.get("tb"))
        z, tz = f["x"], f.get("tx")
        if case["gate"]:
            c, tc = _plain_unit(f["c"], f.get("tc"))
            z = z + c * f["h"]
            out["z"] = z.to(t["x"].dtype)
            if tangent:
                tz = tz + c * f["th"] + tc * f["h"]
                out["tz"] = tz.to(t["x"].dtype)
        n, tn = _plain_unit(z, tz)
        y = n * a + b
        ty = tn * a + n * ta + tb if tangent else None
    elif kind == "gelu":
        u = t["u"].float()
        k = math.sqrt(2 / math.pi)
        th = torch.tanh(k * (u + 0.044715 * u * u * u))
        y = 0.5 * u * (1 + th)
        ty = (0.5 * (1 + th) + 0.5 * u * (1 - th * th) * k * (1 + 3 * 0.044715 * u * u)) * t["tu"].float() if tangent else None
    else:
        y, ty = t["x"].float(), t["tx"].float() if tangent else None
    out["y"], out["s"] = _plain_rows8(y)
    if tangent:
        out["ty"], out["ts"] = _plain_rows8(ty)
    return out


def run(state):
    return _run_own(state["case"], state["t"]) if own else _plain(state["case"], state["t"])


def work(case):
    e, sets = (2 if case["dtype"] == "bf16" else 4), (2 if case["tangent"] else 1)
    if case["kind"] == "linear":
        R, K, F = case["R"], case["K"], case["F"]
        return {"bytes": sets * R * (K + 4 + F * e) + F * K + 4 * F + (F * e if case["bias"] else 0), "flops": 2 * sets * R * K * F}
    if case["kind"] == "norm":
        R, C = case["B"] * case["T"], case["C"]
        tensors = 3 if case["gate"] else 1  # x, h, z: bytes per element; the 8-bit rows; the modulation vectors
        return {"bytes": sets * (R * C * (tensors * e + 1) + 4 * R + 4 * case["B"] * C * (3 if case["gate"] else 2)), "flops": 12 * sets * R * C}
    R, C = case["R"], case["C"]
    return {"bytes": sets * R * (C * (e + 1) + 4), "flops": sets * R * C * (20 if case["kind"] == "gelu" else 3)}


# ---- the definitions in float64
def _rows8_64(y):
    s = y.abs().max(-1).values / 127
    steps = torch.round(y / s.clamp_min(1e-300).unsqueeze(-1))
    return steps * s.unsqueeze(-1), s


def _unit64(v, tv):
    """u = v / N with N = sqrt(mean(v^2) + eps): du = (dv - u dN) / N with dN = mean(v dv) / N."""
    size = torch.sqrt((v ** 2).sum(-1, keepdim=True) / v.shape[-1] + EPS)
    u = v / size
    if tv is None:
        return u, None
    return u, (tv - u * ((v * tv).sum(-1, keepdim=True) / v.shape[-1] / size)) / size


def exact(case, seed):
    t = {n: v.double() for n, v in prepare(case, seed)["t"].items()}
    tangent = case["tangent"]
    if case["kind"] == "linear":
        out = {}
        for y, q, s in (("y", "xq", "xs"), ("ty", "txq", "txs")):
            if q in t:
                out[y] = torch.matmul(t[q] * t[s][:, None], (t["wq"] * t["ws"][:, None]).t())
        if case["bias"]:
            out["y"] += t["bias"]
        return out
    out, ty = {}, None
    if case["kind"] == "norm":
        each = lambda n: t[n][:, None, :] if n in t else None
        z, tz = t["x"], t.get("tx")
        if case["gate"]:
            c, tc = _unit64(each("c"), each("tc"))
            if tangent:
                out["tz"] = tz = tz + tc * t["h"] + c * t["th"]
            out["z"] = z = z + c * t["h"]
        (n, tn), (a, ta), (b, tb) = _unit64(z, tz), _unit64(each("a"), each("ta")), _unit64(each("b"), each("tb"))
        y = b + a * n
        if tangent:
            ty = tb + ta * n + a * tn
    elif case["kind"] == "gelu":
        # gelu(u) = u sigmoid(2 w), w = sqrt(2/pi) (u + 0.044715 u^3)
        u, k = t["u"], math.sqrt(2 / math.pi)
        sig = torch.sigmoid(2 * k * (u + 0.044715 * u ** 3))
        y = u * sig
        if tangent:
            ty = t["tu"] * (sig + u * sig * (1 - sig) * 2 * k * (1 + 0.134145 * u ** 2))
    else:
        y, ty = t["x"], t.get("tx")
    out["y"], out["s"] = _rows8_64(y)
    if tangent:
        out["ty"], out["ts"] = _rows8_64(ty)
    return out
