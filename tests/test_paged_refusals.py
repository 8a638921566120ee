"""Refusals of the C entry points that come before anything touches a GPU, on a machine without one: a context of zeros but for its shape."""
import ctypes

import pytest
import torch

from paper_2503_00540_amd import rekv

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="a call that is not refused would launch")
SOME = 4096                     # an address that is 16- and 256-byte aligned and that no call here follows
UNSUPPORTED, INVALID, NO_GPU = 2, 1, 4


class Context:
    def __init__(self, hq=14, hkv=2, d=64, dtype=rekv.REKV_BF16):
        self.memory = ctypes.create_string_buffer(1 << 14)          # larger than a context, whose first member is the shape
        shape = rekv.RekvShape(hq, hkv, d, 16, dtype, 0.0)
        ctypes.memmove(self.memory, ctypes.byref(shape), ctypes.sizeof(shape))
        self.h = ctypes.addressof(self.memory)

    def error(self):
        return rekv.lib().rekv_last_error(self.h).decode()


def rotary(pairs=32):
    return ctypes.byref(rekv.RekvRotary(1e4, 0, 0, 0, 1, (ctypes.c_int32 * 4)(pairs)))


@pytest.mark.parametrize("tokens,heads", [(1, (1 << 31) - 1), (1, 1 << 30), (1 << 30, 1)])
def test_rotations_whose_heads_or_tokens_do_not_fit_32_bit_steps(tokens, heads):
    c, L = Context(), rekv.lib()
    assert L.rekv_rotate(c.h, rotary(), SOME, heads * 64, tokens, heads, SOME, tokens, SOME, heads * 64, None) == UNSUPPORTED
    assert "too many" in c.error()
    assert L.rekv_rotate(c.h, rotary(), SOME, 64, 1, 1, SOME, 1, SOME, 64, None) == NO_GPU
