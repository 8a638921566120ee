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


def workspace(c, tokens, seqs, max_kv, window=-1, sinks=0, prefix=0):
    n = ctypes.c_int64(-1)
    assert rekv.lib().rekv_attention_paged_workspace(c.h, tokens, seqs, max_kv, window, sinks, prefix, ctypes.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("heads", [(28, 4, 128), (14, 2, 64)])
@pytest.mark.parametrize("tokens,seqs,max_kv,prefix", [(4, 4, 20000, 5000), (64, 64, 9000, 25088), (200, 2, 30000, 4000), (1, 1, 60000, 300)])
def test_a_prefix_has_no_window_in_the_workspace_query_either(heads, tokens, seqs, max_kv, prefix):
    """rekv_attention_shared_prefix takes none, so a query that names one answers for the call that there is."""
    c, L = Context(*heads), rekv.lib()
    need = workspace(c, tokens, seqs, max_kv, prefix=prefix)
    assert need > 0
    cache = rekv.RekvPaged(SOME, SOME, SOME, SOME, SOME, 1000, 1000, 9000, 64, seqs, tokens)
    for window, sinks in ((0, 0), (1, 0), (100, 30), (3000, 4)):
        said = workspace(c, tokens, seqs, max_kv, window, sinks, prefix)
        assert said == need
        assert L.rekv_attention_shared_prefix(c.h, ctypes.byref(cache), SOME, SOME, prefix, max_kv, SOME, SOME, said, None) == NO_GPU


@pytest.mark.parametrize("heads,dtype", [((14, 2, 64), rekv.REKV_BF16), ((28, 4, 128), rekv.REKV_BF16), ((4, 1, 64), rekv.REKV_F32)])
@pytest.mark.parametrize("max_kv,prefix", [(60000, 0), (40, 5000)])
def test_workspaces_that_are_short_missing_or_misaligned(heads, dtype, max_kv, prefix):
    c, L = Context(*heads, dtype), rekv.lib()
    cache = rekv.RekvPaged(SOME, SOME, SOME, SOME, SOME, 1000, 1000, 9000, 64, 2, 4)
    need = workspace(c, 4, 2, max_kv, prefix=prefix)
    assert need > 0

    def call(p, n):
        if prefix:
            return L.rekv_attention_shared_prefix(c.h, ctypes.byref(cache), SOME, SOME, prefix, max_kv, SOME, p, n, None)
        return L.rekv_attention_paged(c.h, ctypes.byref(cache), SOME, max_kv, -1, 0, SOME, p, n, None)
    for p, n in ((None, need), (SOME, need - 1), (SOME, 0), (SOME + 16, need)):
        assert call(p, n) == INVALID and "workspace" in c.error()
    assert call(SOME, need) == NO_GPU
