"""The 8-bit operators without a GPU: what the entry points refuse, the host code under the sanitizers, the rule that chooses the
linear layer's kernels, the instruction streams, and the native calls in front of entry points that do nothing."""
import ctypes
import os
import subprocess
import tempfile

import pytest
import torch

import paper_2511_19797_amd as tvm
from paper_2511_19797_amd import binding, build
from tests import test_isa_hazards as isa
from tests.test_linear_pipe import generated, lds_load_violations

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, UNSUPPORTED = 0, -1, -2
G = 1 << 40   # between fake buffers; nothing reads them: every call below is refused


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(binding.LIB_PATH):
        build.build()
    return binding.lib()


def rows(L, entry="tvmattn_rowquant_fwd", R=4, C=64, dtype=1, ld=0, x=G, tx=2 * G, q=3 * G, s=4 * G, tq=5 * G, ts=6 * G):
    return getattr(L, entry)(R, C, dtype, x, tx, ld, q, s, tq, ts, None)


@pytest.mark.parametrize("entry", ["tvmattn_rowquant_fwd", "tvmattn_gelu_jvp_fwd_q8"])
@pytest.mark.parametrize("kw,status", [
    (dict(R=0), INVALID), (dict(C=0), INVALID), (dict(R=-1), INVALID), (dict(ld=-1), INVALID), (dict(ld=32), INVALID),
    (dict(dtype=2), UNSUPPORTED), (dict(C=60), UNSUPPORTED), (dict(ld=68), UNSUPPORTED), (dict(C=32776), UNSUPPORTED),
    (dict(C=62, dtype=0), UNSUPPORTED), (dict(C=16388, dtype=0), UNSUPPORTED),
    (dict(x=None), INVALID), (dict(q=None), INVALID), (dict(s=None), INVALID),
    (dict(tx=None), INVALID), (dict(tq=None), INVALID), (dict(ts=None), INVALID), (dict(tx=None, tq=None), INVALID),
    (dict(x=G + 8), INVALID), (dict(q=3 * G + 8), INVALID), (dict(s=4 * G + 2), INVALID),
    (dict(q=G + 256), INVALID), (dict(s=3 * G + 252), INVALID), (dict(tq=3 * G + 128), INVALID),   # overlaps
])
def test_rows_refusals(L, entry, kw, status):
    assert rows(L, entry, **kw) == status


def norm(L, B=2, T=3, C=64, dtype=1, eps=1e-6, **kw):
    names = ("x", "tx", "h", "th", "c", "tc", "a", "ta", "b", "tb", "z", "tz", "q", "s", "tq", "ts")
    p = {n: (i + 1) * G for i, n in enumerate(names)} | kw
    return L.tvmattn_gate_adaln_jvp_fwd_q8(B, T, C, dtype, *(p[n] for n in names[:10]), eps, *(p[n] for n in names[10:]), None)


@pytest.mark.parametrize("kw,status", [
    (dict(B=0), INVALID), (dict(T=0), INVALID), (dict(C=0), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID),
    (dict(eps=float("inf")), INVALID), (dict(dtype=9), UNSUPPORTED), (dict(C=68), UNSUPPORTED), (dict(C=4104), UNSUPPORTED),
    (dict(C=2052, dtype=0), UNSUPPORTED), (dict(B=65536), UNSUPPORTED), (dict(B=65535, T=65535), UNSUPPORTED),
    *[({n: None}, INVALID) for n in ("x", "tx", "h", "th", "c", "tc", "a", "ta", "b", "tb", "z", "tz", "q", "s", "tq", "ts")],
    (dict(h=None, c=None, z=None), INVALID),                     # th, tc, tz left over
    (dict(tx=None, ta=None, tb=None, tq=None, ts=None), INVALID),
    (dict(z=3 * G), INVALID), (dict(z=2 * G), INVALID), (dict(tz=G), INVALID), (dict(z=G + 16), INVALID), (dict(q=G), INVALID),
    (dict(a=7 * G + 4), INVALID), (dict(ts=14 * G), INVALID),
])
def test_norm_refusals(L, kw, status):
    assert norm(L, **kw) == status


def linear(L, R=40, K=64, F=32, dtype=1, ldx=0, ldy=0, **kw):
    names = ("xq", "xs", "txq", "txs", "wq", "ws", "bias", "y", "ty")
    p = {n: (i + 1) * G for i, n in enumerate(names)} | kw
    return L.tvmattn_linear_jvp_fwd_q8(R, K, F, dtype, *(p[n] for n in names[:4]), ldx, *(p[n] for n in names[4:]), ldy, None)


@pytest.mark.parametrize("kw,status", [
    (dict(R=0), INVALID), (dict(K=0), INVALID), (dict(F=0), INVALID), (dict(ldx=48), INVALID), (dict(ldy=24), INVALID), (dict(ldx=-16), INVALID),
    (dict(dtype=3), UNSUPPORTED), (dict(K=72), UNSUPPORTED), (dict(F=36), UNSUPPORTED), (dict(K=65552), UNSUPPORTED),
    (dict(ldx=72), UNSUPPORTED), (dict(ldy=36), UNSUPPORTED), (dict(ldx=(1 << 20) + 16), UNSUPPORTED), (dict(F=(1 << 20) + 8), UNSUPPORTED),
    (dict(R=(1 << 30) + 1, F=8), UNSUPPORTED), (dict(R=1 << 24, F=1 << 15), UNSUPPORTED),
    *[({n: None}, INVALID) for n in ("xq", "xs", "txq", "txs", "wq", "ws", "y", "ty")],
    (dict(txq=None, txs=None), INVALID), (dict(txq=None, ty=None), INVALID),
    (dict(xq=G + 8), INVALID), (dict(xs=2 * G + 2), INVALID), (dict(ws=6 * G + 4), INVALID), (dict(bias=7 * G + 2), INVALID),
    (dict(y=G), INVALID), (dict(ty=8 * G), INVALID), (dict(ty=8 * G + 64, ldy=32), INVALID), (dict(y=5 * G + 16), INVALID),
])
def test_linear_refusals(L, kw, status):
    assert linear(L, **kw) == status


def test_host_code_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "q8_checks")
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined",
           "-Xarch_host", "-fno-sanitize-recover=all"]
    cmd = ["hipcc", "--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-x", "hip", "-Xclang", "-target-feature", "-Xclang",
           "-packed-fp32-ops", "-Wno-unused-command-line-argument", *san, os.path.join(isa.CSRC, "q8_api.hip"),
           os.path.join(ROOT, "tests", "host_sanitize", "q8_driver.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=120)
    out = r.stdout + r.stderr
    assert r.returncode == 0 and "host checks ok" in r.stdout and "runtime error" not in out, out[-3000:]


def test_tile_shapes():
    """The measured sides of the rule's borders, and that a launch can hold what is chosen."""
    cases = {(1, 64, 1152, 4608): (64, 64), (2, 256, 1152, 1152): (64, 64), (1, 512, 4608, 1152): (128, 128), (2, 642, 2248, 4528): (128, 128),
             (2, 1000, 3456, 1152): (256, 128), (2, 4096, 1152, 1152): (256, 192), (2, 16384, 3456, 1152): (256, 192),
             (1, 8192, 1152, 4608): (256, 192), (1, 17, 8, 16): (64, 64), (2, 1 << 30, 8, 16): (256, 128), (1, 1 << 18, 1 << 20, 16): (256, 128)}
    src = '#include "linear_q8_plan.h"\n#include <cstdio>\nint main(){int s,R,F,K; while(std::scanf("%d %d %d %d",&s,&R,&F,&K)==4)' \
          '{int n=tvm::pick_shape_q8(s,R,F,K); long long t=s*tvm::tiles_q8(n,R,F);' \
          'std::printf("%d %d %d\\n",tvm::kTileRowsQ8[n],tvm::kTileColsQ8[n],(int)(tvm::grid_fits_q8(n,t)&&t<(1ll<<31)));}}'
    with tempfile.TemporaryDirectory() as tmp:
        open(os.path.join(tmp, "p.cpp"), "w").write(src)
        exe = os.path.join(tmp, "p")
        r = subprocess.run(["g++", "-O1", "-fsanitize=undefined", "-fno-sanitize-recover=all", f"-I{isa.CSRC}", os.path.join(tmp, "p.cpp"), "-o", exe],
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        r = subprocess.run([exe], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert [tuple(map(int, l.split())) for l in r.stdout.splitlines()] == [(*tile, 1) for tile in cases.values()]


def broadcast_violations(asm_text):
    """A data-parallel-primitive operand must not be a register that a VALU instruction wrote in one of the two slots before."""
    ins, bad = list(isa.instructions(asm_text)), []
    for i, (op, ops) in enumerate(ins):
        if "row_newbcast" not in " ".join(ops):
            continue
        src, slots, j = isa.regs(ops[1].split()[0]), 0, i - 1
        while j >= 0 and slots < 2:
            pop, pops = ins[j]
            if pop.startswith("v_") and isa.regs(pops[0]) & src:
                bad.append((i, pop, op))
            slots += int(pops[0], 0) + 1 if pop == "s_nop" else 1
            j -= 1
    return bad


def test_broadcast_check_sees_a_planted_hazard():
    bad = "v_mov_b32 v9, v1\n s_mov_b32 s0, 1\n v_mov_b32_dpp v2, v9 row_newbcast:3 row_mask:0xf bank_mask:0xf"
    assert len(broadcast_violations(bad)) == 1
    assert broadcast_violations(bad.replace("s_mov_b32 s0, 1", "s_nop 1")) == []


def test_instruction_streams():
    """The rules that no interlock keeps, in the hand-scheduled kernel; the loads into LDS in the small tiles' too; nothing spills."""
    text = generated("linear_q8_pipe.hip")
    assert text.count("v_mfma_i32") > 2 * (48 + 32) and text.count("offen lds") > 60 and text.count("row_newbcast") > 300
    assert isa.violations(text) == [] and isa.result_violations(text) == [] and broadcast_violations(text) == []
    for name in ("linear_q8_pipe.hip", "linear_q8.hip"):
        text = generated(name)
        assert lds_load_violations(text) == [] and isa.m0_violations(text) == [] and isa.scalar_violations(text) == []
        assert text.count("offen lds") > 60 and "scratch_" not in text
    for name in ("linear_q8_few.hip", "rows_q8.hip"):
        assert "scratch_" not in generated(name)


@pytest.mark.parametrize("call", [
    lambda x: tvm.tvmattn_rowquant_fwd(x), lambda x: tvm.tvmattn_gelu_jvp_fwd_q8(x, x),
    lambda x: tvm.tvmattn_gate_adaln_jvp_fwd_q8(x.view(1, 4, 64), None, None, None, None, None, x[:1], None, x[:1], None, 1e-6),
    lambda x: tvm.tvmattn_linear_jvp_fwd_q8(x.char(), x[:, 0], None, None, x.char(), x[:, 0]),
])
def test_host_tensors_are_refused(call):
    with pytest.raises(ValueError):
        call(torch.zeros(4, 64))


NATIVE = """
import torch, _fastcall
z = lambda *s, t=torch.float32: torch.zeros(*s, dtype=t)
x, m, q, s = z(2, 4, 16), z(2, 16), z(6, 32, t=torch.int8), z(6)
calls = {
    "rowquant": [x, x], "gelu_q8": [x, x],
    "gate_adaln_q8": [x] * 4 + [m] * 6 + [1e-6],
    "linear_q8": [q, s, q, s, z(64, 32, t=torch.int8), z(64), z(64), False],
}
plain = {"rowquant": [x, None], "gelu_q8": [x, None], "gate_adaln_q8": [x] + [None] * 5 + [m, None, m, None, 1e-6],
         "linear_q8": [q, s, None, None, z(64, 32, t=torch.int8), z(64), None, True]}
for name, args in plain.items():
    out = getattr(_fastcall, name)(*args)
    assert out is not None and sum(o is None for o in out) >= 1, name
calls = {n: [t.clone() if isinstance(t, torch.Tensor) else t for t in a] for n, a in calls.items()}
for name, args in calls.items():
    assert getattr(_fastcall, name)(*args) is not None, name
    for i, t in enumerate(args):
        if isinstance(t, torch.Tensor):
            locked = t.clone()
            torch._C._set_throw_on_mutable_data_ptr(locked)
            print(name, i, flush=True)
            try:
                getattr(_fastcall, name)(*args[:i], locked, *args[i + 1:])
            except RuntimeError as e:
                assert "Cannot access data pointer" in str(e)
            else:
                raise AssertionError((name, i))
            wrong = t.double()
            assert getattr(_fastcall, name)(*args[:i], wrong, *args[i + 1:]) is None, (name, i)
            if name != "rowquant" and name != "gelu_q8":
                assert getattr(_fastcall, name)(*args[:i], t[..., :4], *args[i + 1:]) is None, (name, i)
"""


def test_native_calls_take_and_leave_what_they_should():
    """Built to take CPU tensors, in front of entry points that do nothing: complete and plain calls are taken, a tensor that refuses
    access raises, other types and shapes are left to the Python."""
    from tests import test_fastcall_host as host
    here = "t.get_device() == c10::hip::current_device()"
    with tempfile.TemporaryDirectory() as tmp:
        text = open(os.path.join(host.CSRC, "fastcall.cpp")).read()
        for real, instead in (("!t.is_cuda()", "!t.is_cpu()"), ("(void*)c10::hip::getCurrentHIPStream().stream()", "nullptr"), (here, "t.is_cpu()"),
                              ('"../../include/tvmattn.h"', f'"{os.path.join(ROOT, "include", "tvmattn.h")}"')):
            assert real in text
            text = text.replace(real, instead)
        src, stubs = os.path.join(tmp, "fastcall.cpp"), os.path.join(tmp, "stubs.cpp")
        open(src, "w").write(text)
        import re
        open(stubs, "w").write("".join(f'extern "C" long {n}() {{ return 0; }}\n' for n in sorted(set(re.findall(r"\b(tvmattn_\w+)\b(?=[(,])", text)))))
        r = subprocess.run(build.fastcall_command(src, os.path.join(tmp, "_fastcall.so"), [stubs]), capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
        import sys
        r = subprocess.run([sys.executable, "-X", "faulthandler", "-c", NATIVE], capture_output=True, text=True, timeout=110,
                           env={**os.environ, "PYTHONPATH": tmp})
    assert r.returncode == 0, r.stdout[-300:] + r.stderr[-3000:]
