"""Unusual but valid arguments of the paged-cache calls, through both halves of the binding."""
import numpy as np
import pytest
import torch

from paged_cases import Batch, dev, ints, rounded
from paper_2503_00540_amd import rekv
from paper_2503_00540_amd.rekv import Rekv

pytestmark = pytest.mark.gpu


def halves(r):
    """The native half and the Python methods, one after the other."""
    native = r._fast
    yield "native"
    r._fast = rekv._NoNative()
    yield "python"
    r._fast = native


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,kv", [([1, 3], [40, 20]), ([1], [33])])
def test_positions_expanded_over_the_axes(dtype, new, kv):
    """As text has them: the same position on every axis, without a copy per axis.  What they say counts, not the index."""
    b = Batch(new, kv, 16, 14, 2, 64, dtype)
    r, (q, kp, vp, start, lens, table) = Rekv(14, 2, 64, 16, dtype), b.device()
    g = np.random.default_rng(3)
    k, v = (dev(rounded(g.standard_normal((b.n_tokens, 2, 64)), dtype), dtype) for _ in range(2))
    row = ints(g.integers(1000, 99999, b.n_tokens).tolist())
    args = dict(sections=[8, 12, 12], order="turns")
    want_k, want_v = kp.clone(), vp.clone()
    want_q = r.append_kv(k, v, want_k, want_v, start, lens, table, q=q, positions=row.repeat(3, 1), **args)
    own = kp.clone()
    r.append_kv(k, v, own, vp.clone(), start, lens, table, **args)
    assert not torch.equal(own.nan_to_num(9.0), want_k.nan_to_num(9.0))
    want = r.rotate(q, row.repeat(3, 1), **args)
    for half in halves(r):
        for base in (10000.0, 10000):            # (a whole number is left to the Python method)
            a, c = kp.clone(), vp.clone()
            got = r.append_kv(k, v, a, c, start, lens, table, q=q, positions=row.expand(3, -1), base=base, **args)
            assert torch.equal(got, want_q) and torch.equal(a.nan_to_num(9.0), want_k.nan_to_num(9.0)), (half, base)
            assert torch.equal(c.nan_to_num(9.0), want_v.nan_to_num(9.0))
            assert torch.equal(r.rotate(q, row.expand(3, -1), base=base, **args), want), (half, base)
