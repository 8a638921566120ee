"""The fp64 definitions of the paged-cache operators against other formulations: complex numbers, one dense masked softmax, torch's
attention."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as P


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("order", ["blocks", "turns"])
def test_rotation_is_multiplication_by_a_unit_complex_number(layout, order):
    g = np.random.default_rng(1)
    x, pos, sections, base = g.standard_normal((5, 3, 16)), g.integers(0, 99999, (3, 5)), (2, 3, 3), 1e4
    axis = [0, 0, 1, 1, 1, 2, 2, 2] if order == "blocks" else [0, 1, 2, 0, 1, 2, 1, 2]
    z = x[..., :8] + 1j * x[..., 8:] if layout == "half" else x[..., 0::2] + 1j * x[..., 1::2]
    z = z * np.exp(1j * pos[axis].T * base ** (-np.arange(8) / 8))[:, None]
    want = np.concatenate((z.real, z.imag), -1) if layout == "half" else np.stack((z.real, z.imag), -1).reshape(5, 3, 16)
    got = P.rotate(x, pos, sections, base, layout, order)
    assert np.abs(got - want).max() < 1e-10
    assert np.abs(P.rotate(got, pos, sections, base, layout, order, inverse=True) - x).max() < 1e-10


def test_one_axis_for_all_pairs_is_the_same_as_equal_positions_on_every_axis():
    g = np.random.default_rng(2)
    x, pos = g.standard_normal((4, 2, 8)), g.integers(0, 1000, 4)
    one = P.rotate(x, pos[None], (4,), 1e4, "half")
    for order in ("blocks", "turns"):
        assert np.array_equal(one, P.rotate(x, np.stack([pos] * 3), (1, 0, 3), 1e4, "half", order))


@pytest.mark.parametrize("window,sinks", [(None, 0), (5, 0), (5, 3), (1, 0), (0, 2), (0, 0), (100, 4)])
def test_attention_over_pages_is_the_dense_masked_softmax(window, sinks):
    g = np.random.default_rng(3)
    size, hq, hkv, d = 3, 4, 2, 8
    token_start, kv_len, table = [0, 4, 4, 9], [11, 5, 5], [[7, 1, 4, 0], [2, 3, -1, -1], [6, 5, -1, -1]]
    kp, vp = g.standard_normal((2, 9, size, hkv, d))
    q = g.standard_normal((9, hq, d))
    out, spread = P.attention(q, kp, vp, token_start, kv_len, table, 0.3, window, sinks)
    for s in (0, 2):
        n = token_start[s + 1] - token_start[s]
        k, v = (np.concatenate([x[pg] for pg in table[s] if pg >= 0])[:kv_len[s]] for x in (kp, vp))
        p, j = np.arange(kv_len[s] - n, kv_len[s])[:, None], np.arange(kv_len[s])
        see = (j <= p) & ((p - j < (10 ** 9 if window is None else window)) | (j < sinks))
        for h in range(hq):
            e = np.where(see, np.exp(q[token_start[s]:token_start[s + 1], h] @ k[:, h // 2].T * 0.3), 0)
            want = (e @ v[:, h // 2]) / np.maximum(e.sum(1, keepdims=True), 1e-300)
            assert np.abs(out[token_start[s]:token_start[s + 1], h] - want).max() < 1e-12
    assert (spread >= np.abs(out) - 1e-12).all()


def test_a_shared_prefix_is_the_start_of_every_sequence():
    g = np.random.default_rng(4)
    size, hq, hkv, d, n_prefix = 4, 2, 1, 8, 6
    kp, vp = g.standard_normal((2, 6, size, hkv, d))
    q = g.standard_normal((3, hq, d))
    out, _ = P.attention(q, kp, vp, [0, 1, 3], [3, 2], [[4, -1], [5, -1]], 0.4, prefix_pages=[3, 0], n_prefix=n_prefix)
    for s, (rows, own) in enumerate((((0, 1), 3), ((1, 3), 2))):
        k, v = (torch.from_numpy(np.concatenate([x[3], x[0][:2], x[4 + s][:own]])[:, 0]) for x in (kp, vp))
        qs = torch.from_numpy(q[rows[0]:rows[1]]).transpose(0, 1)
        n = rows[1] - rows[0]
        mask = torch.arange(n_prefix + own) <= torch.arange(n_prefix + own - n, n_prefix + own)[:, None]
        want = torch.nn.functional.scaled_dot_product_attention(qs, k.expand(hq, -1, -1), v.expand(hq, -1, -1), attn_mask=mask, scale=0.4)
        assert np.abs(out[rows[0]:rows[1]] - want.transpose(0, 1).numpy()).max() < 1e-12


def test_append_writes_the_new_rows_and_skips_what_has_no_place():
    pages = np.zeros((3, 2, 1, 1))
    rows = np.arange(1.0, 8.0).reshape(7, 1, 1)
    out = P.append(pages, rows, [0, 3, 5, 6], [3, 1, 5], [[2, 0], [1, 1], [-1, 7]])
    # sequence 0: indexes 0..2; sequence 1: -1 (skipped) and 0; sequence 2: index 4, behind its table
    assert out[2, :, 0, 0].tolist() == [1, 2] and out[0, :, 0, 0].tolist() == [3, 0] and out[1, :, 0, 0].tolist() == [5, 0]
