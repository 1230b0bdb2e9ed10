"""8-bit rows of values as they are: q = v 127 / max|v| to the nearest integer and ties to even, exactly, for every float32 and bf16 row.

The expected integers are worked out with Python's: v and max are whole multiples of one power of two, 254 v and (2 n + 1) max are
compared as they are.  No tolerance: there is one right integer.
"""
import sys

import numpy as np
import pytest
import torch

import paper_2511_19797_amd as tvm

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "bf16": torch.bfloat16}


def whole(v):
    """float32 values as integers times one power of two: an object array of Python integers."""
    frac, exp = np.frexp(v.astype(np.float64))
    low = int(exp[v != 0].min()) - 24
    return np.array([int(f * (1 << 24)) << (int(e) - 24 - low) if f else 0 for f, e in zip(frac, exp)], dtype=object)


def expected(row):
    """The row's int8 values by integer arithmetic."""
    n = whole(row)
    m = max(abs(int(t)) for t in n)
    out = []
    for t in n:
        a = abs(int(t)) * 254
        down = a // (2 * m)                           # floor of |v| 127 / m
        twice = a - 2 * m * down                      # against m: below, at or above the half
        q = down + (twice > m or (twice == m and down & 1))
        out.append(q if t >= 0 else -q)
    return np.array(out, dtype=np.int8)


def check(x, place):
    """x: [R, k] rows of candidates, each row's largest value in its first column; `place`: the width they are spread over, zeros between."""
    R, k = x.shape
    wide = torch.zeros(R, place, dtype=x.dtype)
    at = torch.linspace(0, place - 1, k).round().long()
    assert at.unique().numel() == k
    wide[:, at] = x
    q, s, tq, ts = tvm.tvmattn_rowquant_fwd(wide.cuda(), (-wide).cuda())
    want = np.stack([expected(r) for r in x.float().numpy()])
    got, tgot = q.cpu()[:, at].numpy(), tq.cpu()[:, at].numpy()
    assert np.array_equal(got, want), [(x[i, j].item(), x[i, 0].item(), int(got[i, j]), int(want[i, j])) for i, j in np.argwhere(got != want)[:5]]
    assert np.array_equal(tgot, -want)
    assert torch.equal(s, ts) and torch.equal(s.cpu(), x[:, 0].float().abs() / 127)
    rest = q.cpu().clone()
    rest[:, at] = 0
    assert not rest.any()


@pytest.mark.parametrize("place", [64, 1152, 2064, 8200])          # a wave per row, one chunk of lanes and more; 4 waves; 16
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_half_of_the_largest(dtype, place):
    """max / 2 stands at 63.5 steps whatever max is, and goes to 64: all bf16 mantissas, and float32 ones."""
    print("[case]", dtype, place, flush=True)
    sys.stdout.flush()
    rng = np.random.default_rng(place)
    top = torch.arange(128, 256).float() if dtype == "bf16" else torch.from_numpy((1 + rng.random(500)).astype(np.float32))
    top = torch.cat([top * 2.0 ** e for e in (0, -90, 60)])
    x = torch.stack([top, top / 2, -top / 2, top / 4, -top], 1).to(DT[dtype])
    assert torch.equal(x[:, 0].float(), top)
    check(x, place)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_every_half_step(dtype):
    """Rows whose steps are powers of two: every half of a step is a value, and all of them are ties."""
    half = torch.arange(-254, 255).float() / 2
    if dtype == "bf16":
        assert torch.equal(half.bfloat16().float(), half)
    half = torch.cat([torch.tensor([127.0]), half])
    check(torch.stack([half * 2.0 ** e for e in (0, -50, 3)]).to(DT[dtype]), 1152)


@pytest.mark.parametrize("place", [2048, 2056])
def test_next_to_every_border(place):
    """float32 values on either side of every border between two steps, as near as float32 has them."""
    rng = np.random.default_rng(place)
    top = np.concatenate([(1 + rng.random(60)) * 2.0 ** rng.integers(-80, 80, 60), [127.0, 254.0, 1.0, np.nextafter(np.float32(2), np.float32(0))]]).astype(np.float32)
    border = ((2 * np.arange(127) + 1) * top[:, None].astype(np.float64) / 254).astype(np.float32)
    up, down = np.nextafter(border, np.float32(np.inf)), np.nextafter(border, np.float32(0))
    x = np.concatenate([top[:, None], border, -border, up, down, -up, np.minimum(down, top[:, None])], 1)
    check(torch.from_numpy(x), place)
