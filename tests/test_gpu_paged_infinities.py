"""Rows whose scores are all -infinity, in every form of the paged attention: zeros, whatever the values are."""
import numpy as np
import pytest
import torch

from paged_cases import Batch, dev, ints
from paper_2503_00540_amd.rekv import Rekv
from test_paged_plan import KEYS, ROWS, STREAMED, plan

pytestmark = pytest.mark.gpu
H05, H7, F32 = (14, 2, 64, "bf16"), (28, 4, 128, "bf16"), (4, 1, 64, "f32")


@pytest.mark.parametrize("value", [np.inf, np.nan])
@pytest.mark.parametrize("heads,new,kv,prefix,window,form", [
    (H05, [2600, 300, 1], [2900, 410, 700], 0, None, (ROWS, False)), (H7, [1200, 300, 1], [1500, 410, 700], 0, None, (ROWS, False)),
    (H05, [40, 3], [300, 90], 0, None, (KEYS, False)), (H7, [60, 3], [600, 90], 0, 130, (KEYS, False)), (H7, [1, 1], [9000, 700], 0, None, (STREAMED, True)),
    (H7, [1] * 40, [20] * 40, 6000, None, (STREAMED, True)), (F32, [40, 3], [200, 90], 0, None, (0, False)), (F32, [40, 3], [300, 90], 0, None, (0, True)),
    (F32, [1, 1], [5000, 90], 0, None, (0, True))])
def test_scores_of_minus_infinity(heads, new, kv, prefix, window, form, value):
    b = Batch(new, kv, 16, *heads, n_prefix=prefix)
    r = Rekv(*heads[:3], 16, b.dtype)
    p = plan(heads[:3], b.n_tokens, len(new), max(kv), -1 if window is None else window, 0, prefix, int(b.dtype == "bf16"))
    assert (p["how"], p["bytes"] > 0) == form, p
    b.q[..., 0] = np.abs(b.q[..., 0]) + 0.25          # times -infinity: -infinity
    q, kp, vp, start, lens, table = b.device()

    def run():
        if prefix:
            return r.attention_shared_prefix(q, kp, vp, ints(b.prefix_pages), prefix, start, lens, table, max_kv=max(kv))
        return r.attention_paged(q, kp, vp, start, lens, table, max_kv=max(kv), window=window)
    plain = run()
    g = heads[0] // heads[1]
    kp[:, :, 0, 0] = float("-inf")
    assert not run()[:, :g].any()
    some = [t[i // 16] for t, n in zip(b.table, kv) for i in range(0, n, 11)] + list(b.prefix_pages[::3])
    for row in (0, 7):
        vp[some, row, 0, 3] = value
        vp[some, row, 0, heads[2] - 1] = -value
    got = run()
    assert not got[:, :g].any(), "not zeros"          # NaN counts as any
    assert torch.equal(got[:, g:], plain[:, g:])
