"""What the block's forward in 8 bits refuses, before any of its operators is called."""
import pytest
import torch

from paper_2511_19797_amd import block


def test_block_refusals():
    x, m = torch.zeros(1, 4, 64, dtype=torch.bfloat16), {n: torch.zeros(1, 64) for n in block.MODS}
    for args, what in (((x, None, m, m), "tangent"), ((x, x, m, None), "tangent"), ((x.float(), x.float(), m, m), "bfloat16")):
        with pytest.raises(ValueError, match=what):
            block.block_jvp_fwd_q8(*args, {}, 1, 1e-6, 1e-6)
