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


def test_views_that_leave_one_element_with_a_stride():
    """One token of one sequence whose positions, length and page number are cut out of larger tensors."""
    b = Batch([1], [33], 64, 14, 2, 64)
    r, (q, kp, vp, start, lens, table) = Rekv(14, 2, 64, 64), b.device()
    k, v = (torch.randn((1, 2, 64), device="cuda:0").to(torch.bfloat16) for _ in range(2))
    pos = ints([[7, 800, 31]])
    cut_lens, cut_table = ints([[0, 33], [5, 6]])[:1, 1], table.T.as_strided((1, 1), (1, 9))
    args = dict(sections=[8, 12, 12], q=q)
    want_k = kp.clone()
    want_q = r.append_kv(k, v, want_k, vp.clone(), start, lens, table, positions=pos.T.clone(memory_format=torch.contiguous_format), **args)
    want = r.attention_paged(q, kp, vp, start, lens, table)
    for half in halves(r):
        a = kp.clone()
        got = r.append_kv(k, v, a, vp.clone(), start, cut_lens, cut_table, positions=pos.T, **args)
        assert torch.equal(got, want_q) and torch.equal(a.nan_to_num(9.0), want_k.nan_to_num(9.0)), half
        assert torch.equal(r.attention_paged(q, kp, vp, start, cut_lens, cut_table), want), half
