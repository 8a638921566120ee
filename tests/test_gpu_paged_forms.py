"""Blocks of 128 rows of either head size with windows and sinks, written straight and from split keys, and the workspace checks: each test
says which launch its sizes plan, so that a change of the plan shows."""
import ctypes

import pytest
import torch

from paged_cases import Batch, ints
from paper_2503_00540_amd import rekv
from paper_2503_00540_amd.rekv import Rekv
from test_gpu_paged import attend
from test_paged_plan import H05, H7, ROWS, plan

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("heads", [H05, H7])
@pytest.mark.parametrize("window,sinks,page", [(None, 0, 5), (None, 0, 48), (700, 20, 16), (700, 0, 144), (1400, 40, 7), (1, 0, 64), (90, 130, 32)])
def test_blocks_of_128_rows_that_write_their_output(heads, window, sinks, page):
    new, kv = [2600, 300, 1], [2900, 410, 700]
    p = plan(heads, sum(new), len(new), max(kv), -1 if window is None else window, sinks)
    assert p["how"] == ROWS and p["bytes"] == 0, p
    b = Batch(new, kv, page, *heads, pad=4)
    if window is not None:
        b.lost_pages(window, sinks)
    attend(b, window, sinks, max_kv=max(kv), every=97)


@pytest.mark.parametrize("heads", [H05, H7])
@pytest.mark.parametrize("window,sinks,page", [(None, 0, 16), (2500, 30, 10), (2500, 30, 196)])
def test_blocks_of_128_rows_over_split_keys(heads, window, sinks, page):
    new, kv = ([1200, 200], [6000, 3000]) if heads == H05 else ([900, 196], [5000, 3000])
    p = plan(heads, sum(new), len(new), max(kv), -1 if window is None else window, sinks)
    assert p["how"] == ROWS and p["splits"] > 1, p
    b = Batch(new, kv, page, *heads, pad=4)
    if window is not None:
        b.lost_pages(window, sinks)
    attend(b, window, sinks, max_kv=max(kv), every=97)


@pytest.mark.parametrize("heads", [(14, 2, 64, "bf16"), (28, 4, 128, "bf16"), (4, 1, 64, "f32")])
def test_workspaces_that_are_short_missing_or_misaligned(heads):
    """Both calls refuse them before anything is launched; nothing is written."""
    b = Batch([1, 3], [40, 20], 16, *heads, n_prefix=5000)
    r, (q, kp, vp, start, kv, table), pre = Rekv(*heads[:3], 16, b.dtype), b.device(), ints(b.prefix_pages)
    L, out = rekv.lib(), torch.full_like(q, 7.0)
    cache = r._paged(kp, vp, start, kv, table, 4)
    for n_prefix, max_kv, call in (
            (0, 60000, lambda p, n: L.rekv_attention_paged(r._h, ctypes.byref(cache), q.data_ptr(), 60000, -1, 0, out.data_ptr(), p, n, None)),
            (5000, 40, lambda p, n: L.rekv_attention_shared_prefix(r._h, ctypes.byref(cache), q.data_ptr(), pre.data_ptr(), 5000, 40, out.data_ptr(),
                                                                   p, n, None))):
        need = ctypes.c_int64()
        assert L.rekv_attention_paged_workspace(r._h, 4, 2, max_kv, -1, 0, n_prefix, ctypes.byref(need)) == 0 and need.value > 0
        ws = torch.empty(need.value + 512, dtype=torch.uint8, device="cuda:0")
        for p, n in ((None, need.value), (ws.data_ptr(), need.value - 1), (ws.data_ptr(), 0), (ws.data_ptr() + 16, need.value)):
            assert call(p, n) == 1 and b"workspace" in L.rekv_last_error(r._h)
        torch.cuda.synchronize()
        assert (out == 7).all()
