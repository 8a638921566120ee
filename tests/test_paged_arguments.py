"""What the Python methods of the paged-cache calls hand to the C calls, without a GPU: a stand-in for the library records it."""

import pytest
import torch

from paper_2503_00540_amd import rekv


class Recorded(rekv.Rekv):
    """The Python methods on host tensors, before a library that notes its arguments and succeeds."""

    def __init__(self, monkeypatch):
        monkeypatch.setattr(rekv, "_stream", lambda: 0)
        self.n_q_heads, self.n_kv_heads, self.head_dim, self.tokens_per_frame, self.torch_dtype = 4, 2, 64, 16, torch.bfloat16
        self._h, self._fast, self._lib, self.calls = None, rekv._NoNative(), self, []

    def __getattr__(self, name):
        if not name.startswith("rekv_"):
            raise AttributeError(name)

        def call(*args):
            self.calls.append((name, args))
            return 0
        return call

    def _here(self, **tensors):
        pass

    def _dev(self, t, dtype=None, last=None, name="tensor"):
        return t.data_ptr()


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


@pytest.fixture
def r(monkeypatch):
    return Recorded(monkeypatch)


@pytest.mark.parametrize("n", [1, 5])
def test_one_row_of_positions_expanded_over_the_axes_is_handed_on(r, n):
    row = i32(n)
    for pos, stride in ((row.expand(3, -1), 0), (row.repeat(3, 1), n), (i32(3, n + 2)[:, :n], n + 2)):
        r.append_kv(bf(n, 2, 64), bf(n, 2, 64), bf(5, 16, 2, 64), bf(5, 16, 2, 64), i32(2), i32(1), i32(1, 3), positions=pos, sections=[8, 12, 12])
        r.rotate(bf(n, 4, 64), pos, sections=[8, 12, 12])
        (_, append), (_, rotate) = r.calls[-2:]
        assert append[-3] == pos.data_ptr() and append[-2] == stride
        assert rotate[6] == pos.data_ptr() and rotate[7] == stride
    r.append_kv(bf(n, 2, 64), bf(n, 2, 64), bf(5, 16, 2, 64), bf(5, 16, 2, 64), i32(2), i32(1), i32(1, 3))
    assert r.calls[-1][1][-3] is None


def test_a_single_element_has_no_neighbour(r):
    """A view leaves a dimension of one element any stride, which contiguous() does not change either."""
    pos = i32(1, 3).T
    lens, table = i32(2, 7)[:1, 3], i32(1, 1).as_strided((1, 1), (1, 5))
    assert pos.stride() == (1, 3) and pos.contiguous().stride(1) == 3 and lens.stride() == (7,)
    r.append_kv(bf(1, 2, 64), bf(1, 2, 64), bf(5, 16, 2, 64), bf(5, 16, 2, 64), i32(2), lens, table, positions=pos, sections=[8, 12, 12])
    assert r.calls[-1][1][-3] == pos.data_ptr() and r.calls[-1][1][-2] == 1
    r.rotate(bf(1, 4, 64), pos, sections=[8, 12, 12])
    with pytest.raises(ValueError, match="side by side"):
        r.append_kv(bf(2, 2, 64), bf(2, 2, 64), bf(5, 16, 2, 64), bf(5, 16, 2, 64), i32(3), i32(2, 7)[:, 3], i32(2, 1))


def test_sizes_beyond_32_bits_are_refused(r):
    """Of tensors without storage; a wrapped number of tokens or pages would serve a part of them and report success."""
    def meta(*shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device="meta")

    big = (1 << 32) + 1
    ok = dict(n=3, pages=5, page=16, seqs=1, table=3)
    for name, size in ok.items():
        a = dict(ok, **{name: big})
        kp = meta(a["pages"], a["page"], 2, 64)
        batch = (kp, kp, meta(a["seqs"] + 1, dtype=torch.int32), meta(a["seqs"], dtype=torch.int32), meta(a["seqs"], a["table"], dtype=torch.int32))
        k, q = meta(a["n"], 2, 64), meta(a["n"], 4, 64)
        for call in (lambda: r.append_kv(k, k, *batch), lambda: r.attention_paged(q, *batch),
                     lambda: r.attention_shared_prefix(q, kp, kp, meta(2, dtype=torch.int32), 20, *batch[2:])):
            with pytest.raises(ValueError, match="2.31"):
                call()
    for shape in ((big, 1, 64), (1, big, 64)):
        with pytest.raises(ValueError, match="2.31"):
            r.rotate(meta(*shape), meta(shape[0], dtype=torch.int32))
    assert not r.calls
