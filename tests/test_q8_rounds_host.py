"""Which kernels the cases of test_q8_rounds_gpu.py reach: a change of the rule that chooses tiles may not empty them."""
import os
import subprocess
import tempfile

from tests import test_isa_hazards as isa

# sets, R, K, F -> columns of the 256-row tiles, contraction tiles.  A workgroup of each has two output tiles at least.
ROUNDS = {
    (2, 9000, 64, 1152): (192, 1), (2, 9000, 144, 1152): (192, 2), (2, 9000, 384, 1152): (192, 3), (2, 9000, 400, 1152): (192, 4),
    (2, 9000, 1152, 1152): (192, 9), (2, 9000, 384, 1160): (192, 3), (2, 9000, 400, 1000): (192, 4), (2, 9000, 1168, 1160): (192, 10),
    (2, 9000, 64, 768): (128, 1), (2, 9000, 144, 768): (128, 2), (2, 9000, 384, 768): (128, 3), (2, 9000, 400, 768): (128, 4),
    (2, 9000, 1152, 768): (128, 9), (2, 9000, 64, 760): (128, 1), (2, 9000, 384, 760): (128, 3), (2, 9000, 1168, 760): (128, 10),
    (2, 4500, 384, 1528): (128, 3), (1, 9000, 400, 1536): (128, 4),
    (2, 16384, 400, 1152): (192, 4), (2, 16384, 400, 1024): (128, 4),           # three rounds and four
    (1, 16384, 1152, 3456): (128, 9), (2, 16384, 1152, 3456): (192, 9),         # the fused projection of 16384 tokens: seven and nine
    (1, 8192, 4608, 1152): (192, 36), (2, 8192, 4608, 1152): (192, 36),         # the MLP's second layer: one round and two
}
PART = 300   # rows at a time, which take the small tiles


def test_the_cases_are_what_they_are_meant_to_be():
    src = '#include "linear_q8_plan.h"\n#include <cstdio>\nint main(){int s,R,K,F; while(std::scanf("%d %d %d %d",&s,&R,&K,&F)==4)' \
          '{int n=tvm::pick_shape_q8(s,R,F,K); std::printf("%d %d %lld %d\\n",tvm::kTileRowsQ8[n],tvm::kTileColsQ8[n],' \
          's*tvm::tiles_q8(n,R,F),(K+tvm::kBKQ-1)/tvm::kBKQ);}}'
    cases = list(ROUNDS) + [(s, PART, K, F) for s, _, K, F in ROUNDS]
    with tempfile.TemporaryDirectory() as tmp:
        open(os.path.join(tmp, "p.cpp"), "w").write(src)
        exe = os.path.join(tmp, "p")
        r = subprocess.run(["g++", "-O1", f"-I{isa.CSRC}", os.path.join(tmp, "p.cpp"), "-o", exe], capture_output=True, text=True)
        assert r.returncode == 0, r.stderr
        r = subprocess.run([exe], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True)
    got = [tuple(map(int, l.split())) for l in r.stdout.splitlines()]
    for (case, (cols, steps)), (rows, c, tiles, nct) in zip(ROUNDS.items(), got):
        rounds = -(-(-(-tiles // 8)) // 32)                                     # of an XCD's share, 32 workgroups at a time
        assert (rows, c, nct) == (256, cols, steps) and rounds >= (1 if case[:2] == (1, 8192) else 2), (case, rows, c, tiles, nct)
    assert all(rows < 256 for rows, *_ in got[len(ROUNDS):])
    # second output tiles with 1, 2, 3, 4 and more contraction tiles, on both shapes, results streamed (bf16 rows of whole 64 bytes) and not
    for cols in (192, 128):
        assert {1, 2, 3, 4, 9} <= {n for c, (w, n) in ROUNDS.items() if w == cols and c[3] * 2 % 64 == 0}
        assert any(n >= 3 for c, (w, n) in ROUNDS.items() if w == cols and c[3] * 2 % 64)
