"""Sizes that do not fit the library's 32-bit arguments are refused by the binding: as they are passed they would be taken modulo 2^32
(4 rows for 2^32 + 4, the others left unwritten)."""
import ctypes

import pytest
import torch

import paper_2511_19797_amd as tvm


class Device:
    """What the binding asks a tensor about its layout, for a contiguous device tensor of any size."""
    is_cuda, device = True, torch.device("cuda", 0)

    def __init__(self, *shape, dtype=torch.bfloat16):
        self.shape, self.dtype = torch.Size(shape), dtype

    def dim(self):
        return len(self.shape)

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def stride(self, i=None):
        st, n = [], 1
        for s in reversed(self.shape):
            st.insert(0, n)
            n *= s
        return tuple(st) if i is None else st[i]

    def is_contiguous(self):
        return True


LONG = (1 << 32) + 4
f32 = torch.float32


def test_what_a_32_bit_argument_makes_of_it():
    assert ctypes.c_int(LONG).value == 4


@pytest.mark.parametrize("call", [
    lambda: tvm.tvmattn_rowquant_fwd(Device(LONG, 8)),
    lambda: tvm.tvmattn_rowquant_fwd(Device(1 << 16, 1 << 16, 8)),
    lambda: tvm.tvmattn_rowquant_fwd(Device(4, 1 << 31)),
    lambda: tvm.tvmattn_gelu_jvp_fwd_q8(Device(1 << 31, 8), Device(1 << 31, 8)),
    lambda: tvm.tvmattn_gate_adaln_jvp_fwd_q8(Device(1, LONG, 8), None, None, None, None, None, Device(1, 8, dtype=f32), None, Device(1, 8, dtype=f32),
                                              None, 1e-6),
    lambda: tvm.tvmattn_gate_adaln_jvp_fwd_q8(Device(LONG, 1, 8), None, None, None, None, None, Device(LONG, 8, dtype=f32), None,
                                              Device(LONG, 8, dtype=f32), None, 1e-6),
    lambda: tvm.tvmattn_linear_jvp_fwd_q8(Device(LONG, 16, dtype=torch.int8), Device(LONG, dtype=f32), None, None, Device(8, 16, dtype=torch.int8),
                                          Device(8, dtype=f32)),
    lambda: tvm.tvmattn_linear_jvp_fwd_q8(Device(4, 16, dtype=torch.int8), Device(4, dtype=f32), None, None, Device(LONG, 16, dtype=torch.int8),
                                          Device(LONG, dtype=f32)),
])
def test_long_tensors_are_refused(call, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    with pytest.raises(ValueError, match="2\\^31"):
        call()
