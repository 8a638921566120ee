"""How attention over a paged cache is dispatched and split, without a GPU."""
import ctypes
import itertools

import pytest

from paper_2503_00540_amd import rekv

ROWS, KEYS, STREAMED = 0, 1, 2


def plan(heads, tokens, seqs, max_kv, window=-1, sinks=0, prefix=0, dtype=1):
    out = (ctypes.c_int64 * 8)()
    rekv.lib().rekv_internal_paged_plan(dtype, *heads, tokens, seqs, max_kv, window, sinks, prefix, out)
    names = ("how", "rows", "blocks", "splits", "prefix_blocks", "prefix_splits", "bytes", "workgroups")
    return dict(zip(names, out))


H7, H05, H72 = (28, 4, 128), (14, 2, 64), (64, 8, 128)


@pytest.mark.parametrize("heads,dtype", [(H7, 1), (H05, 1), (H72, 1), ((8, 8, 64), 1), ((1, 1, 128), 1), ((64, 1, 128), 1), ((4, 1, 64), 0),
                                         ((6, 2, 20), 0)])
def test_every_row_has_a_block_and_the_workspace_holds_every_part(heads, dtype):
    hq, hkv, d = heads
    for tokens, seqs, max_kv, prefix in itertools.product((1, 2, 63, 64, 1000, 50000), (1, 7, 64, 3000), (1, 31, 4096, 10 ** 6, 2 ** 30), (0, 1, 5000, 10 ** 6)):
        p = plan(heads, tokens, seqs, max_kv, prefix=prefix, dtype=dtype)
        rows, g = p["rows"], hq // hkv
        assert p["blocks"] >= -(-tokens * g // rows) and p["splits"] >= 1, p
        # the worst raggedness still finds its blocks: every sequence may leave one unfilled
        assert p["blocks"] == tokens * g // rows + seqs
        slots = p["splits"] + (p["prefix_splits"] if p["prefix_blocks"] else 0)
        assert p["bytes"] == (tokens * hq * slots * (d + 2) * 4 if slots > 1 else 0)
        assert (p["prefix_blocks"] > 0) == (p["prefix_splits"] > 0) and (not p["prefix_blocks"] or prefix > 0)
        assert p["workgroups"] < 2 ** 31
        if tokens <= 1000 and seqs <= 64:
            assert p["bytes"] <= 1 << 30, (tokens, seqs, max_kv, prefix, p)


def test_partial_results_of_many_rows_stay_few():
    for heads in (H7, H72, H05):
        for tokens in (4096, 8192, 50000):
            assert plan(heads, tokens, 1, tokens)["bytes"] == 0                      # a long prompt writes its output itself


@pytest.mark.parametrize("heads,tokens,seqs,kv,window,how", [
    (H72, 64, 64, 8192, -1, STREAMED), (H7, 1, 1, 50000, 15000, STREAMED),          # decode steps
    (H7, 196, 1, 196, -1, KEYS), (H7, 1000, 1, 1000, -1, KEYS), (H7, 16, 1, 3016, -1, KEYS), (H05, 196, 1, 12196, 3136, KEYS),
    (H7, 240, 8, 3060, -1, KEYS), (H7, 8192, 1, 8192, -1, ROWS), (H72, 2000, 1, 2000, -1, ROWS), (H72, 576, 4, 12144, 2304, ROWS),
    (H7, 610, 8, 12196, 3136, ROWS), (H7, 270, 32, 3016, -1, ROWS), (H7, 900, 30, 60, -1, ROWS), (H7, 900, 30, 460, -1, KEYS)])
def test_which_blocks_take_a_launch(heads, tokens, seqs, kv, window, how):
    assert plan(heads, tokens, seqs, kv, window)["how"] == how


@pytest.mark.parametrize("tokens,seqs,own,prefix,at_once", [
    (64, 64, 400, 25088, True), (6, 6, 91, 3136, True), (40, 40, 40, 6000, True), (64, 64, 400, 100, False), (1, 1, 4, 5216, False), (64 * 12, 64, 12, 4608, True), (64 * 32, 64, 32, 4608, True), (24 * 40, 24, 40, 4608, True),
    (64 * 512, 64, 512, 4608, False), (4 * 8, 4, 8, 4608, False)])
def test_which_prefixes_are_computed_at_once(tokens, seqs, own, prefix, at_once):
    assert (plan(H7, tokens, seqs, own, prefix=prefix)["prefix_blocks"] > 0) == at_once


def test_splits_fill_the_chip_and_no_more():
    p = plan(H7, 1, 1, 50000, 15000, 4)
    assert p["splits"] == 59                                                         # of two tiles a wavefront
    p = plan(H7, 64, 64, 400, prefix=25088)
    assert p["prefix_blocks"] == 4 and p["prefix_splits"] == 24                      # beside 256 workgroups of own keys
    assert plan(H72, 64, 64, 8192)["splits"] == 4 and plan(H72, 64, 64, 10 ** 9)["splits"] == 64


def test_a_short_prefix_takes_one_launch():
    for heads, tokens, own, prefix in ((H7, 64, 40, 100), (H72, 64, 13, 157), (H05, 20, 1, 15), ((8, 8, 64), 5, 9, 4)):
        p = plan(heads, tokens, tokens, own, prefix=prefix)
        assert p["how"] == KEYS and p["splits"] == 1 and p["bytes"] == 0


@pytest.mark.parametrize("dtype,heads", [(1, H7), (1, H05), (1, H72), (1, (8, 8, 64)), (1, (64, 1, 128)), (1, (5, 5, 128)), (0, (4, 1, 64)),
                                         (0, (14, 2, 64)), (0, (6, 2, 20)), (0, (8, 8, 256))])
def test_one_workspace_holds_every_smaller_batch(dtype, heads):
    """The header's bound: of all batches of at most so many tokens, whatever their sequences, lengths and windows."""
    import math
    import random
    rng = random.Random(7)
    hq, _, d = heads

    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    near = [0, 0]
    for _ in range(4000):
        tokens = log_int(1, 100000)
        seqs = rng.choice([1, tokens, log_int(1, tokens), log_int(1, 5000)])
        max_kv, window, prefix = log_int(1, 1 << 30), rng.choice([-1, -1, log_int(1, 1 << 20)]), rng.choice([0, log_int(1, 1 << 29)])
        r = tokens * hq
        s = max(1 << 16, min(64 * r, 1 << 22))
        bound = 4 * (d + 2) * (s if prefix == 0 else max(s, r) + max(r, min(512 * r, (1 << 27) // (d + 2))))
        need = plan(heads, tokens, seqs, max_kv, window if prefix == 0 else -1, 0, prefix, dtype)["bytes"]
        assert need <= bound, (tokens, seqs, max_kv, window, prefix, need, bound)
        near[prefix > 0] = max(near[prefix > 0], need / bound)
    assert dtype == 0 or min(near) > 0.25, near          # and it is of their size
