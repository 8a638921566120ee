"""Attention over a paged cache against its fp64 definition: ragged batches, pages of any size, windows and sinks, shared prefixes."""
import numpy as np
import pytest
import torch

from paged_cases import TYPES, Batch, check, dev, ints
from paper_2503_00540_amd.rekv import Rekv

pytestmark = pytest.mark.gpu

HEADS = [(14, 2, 64, "bf16"), (28, 4, 128, "bf16"), (8, 8, 64, "bf16"), (4, 1, 64, "f32"), (6, 2, 20, "f32"), (8, 2, 128, "f32"),
         (6, 2, 80, "f32"), (2, 1, 256, "f32")]


LONG = 10 ** 6          # as a hint: launches of few rows are no longer taken for short ones


def attend(b, window=None, sinks=0, max_kv=None, r=None, every=1):
    r = r or Rekv(b.hq, b.hkv, b.d, b.page, b.dtype)
    q, kp, vp, start, kv, table = b.device()
    out = torch.full_like(q, 7.0)
    if b.n_prefix:
        got = r.attention_shared_prefix(q, kp, vp, ints(b.prefix_pages), b.n_prefix, start, kv, table, max_kv=max_kv, out=out)
    else:
        got = r.attention_paged(q, kp, vp, start, kv, table, max_kv=max_kv, window=window, sinks=sinks, out=out)
    torch.cuda.synchronize()
    assert got is out
    check(out, b, window, sinks, before=torch.full_like(q, 7.0), every=every)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("page", [1, 5, 16, 32, 48, 196])
def test_ragged_batches(heads, page):
    # decode steps, short and longer new parts, a sequence without new tokens, one without any, the whole sequence new
    b = Batch([1, 7, 0, 40, 0, 1, 33], [1, 130, 50, 40, 0, 300, 65], page, *heads, pad=3)
    attend(b)
    attend(b, max_kv=LONG)


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("window,sinks", [(1, 0), (0, 3), (0, 0), (17, 0), (64, 4), (100, 33), (33, 100), (31, 32), (10 ** 6, 5)])
def test_windows_and_sinks(heads, window, sinks):
    for page in (10, 64):
        b = Batch([1, 20, 70, 2], [250, 140, 70, 400], page, *heads, pad=2, seed=window)
        b.lost_pages(window, sinks)
        attend(b, window, sinks)


@pytest.mark.parametrize("heads", [HEADS[1], HEADS[0], HEADS[3]])
@pytest.mark.parametrize("new,kv,page", [(1, 9000, 64), (1, 2500, 7), (3, 4099, 196), (200, 5000, 144)])
def test_long_sequences_are_split(heads, new, kv, page):
    b, every = Batch([new], [kv], page, *heads), 1 if new < 10 else 19
    attend(b, every=every)
    attend(b, max_kv=1, every=every)                  # the hint splits the work, nothing else
    attend(b, max_kv=10 ** 9, every=every)
    b.lost_pages(1500, 40)
    attend(b, 1500, 40, every=every)


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[1]])
@pytest.mark.parametrize("page", [5, 16, 48, 144])
def test_many_rows(heads, page):
    """Enough rows for blocks of 128 whose results go straight to the output: prompts, windows inside and beyond a block, sinks."""
    b = Batch([1200, 300, 1], [1500, 410, 700], page, *heads, pad=4)
    attend(b, every=61)
    attend(b, 700, 20, every=61)
    attend(b, 1400, 0, every=61)


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[1]])
@pytest.mark.parametrize("seqs,new,n_prefix,page", [(3, 200, 5000, 64), (40, 30, 2100, 144), (24, 100, 2500, 7), (70, 3, 3000, 16)])
def test_prefixes_of_many_rows(heads, seqs, new, n_prefix, page):
    """Prefixes at once in several pieces and walked, over more tiles than are placed at a time, sequences of more than a lane each."""
    b = Batch([new if s % 3 else max(new // 2, 1) for s in range(seqs)], [new + s for s in range(seqs)], page, *heads, n_prefix=n_prefix, pad=2)
    attend(b, every=max(new // 2, 2))


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("n_prefix,page", [(1, 16), (31, 5), (500, 196), (2000, 64)])
def test_shared_prefixes(heads, n_prefix, page):
    attend(Batch([1] * 9, [1, 2, 0, 40, 33, 64, 5, 100, 31], page, *heads, n_prefix=n_prefix, pad=1))       # one row per user
    attend(Batch([40, 0, 18, 1], [40, 0, 30, 1], page, *heads, n_prefix=n_prefix))                          # questions


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[1]])
def test_many_sequences(heads):
    g = np.random.default_rng(5)
    for n in (64, 65, 130, 5000):
        new = [int(x) for x in g.integers(0, 3, n)]
        kv = [int(x) + m for x, m in zip(g.integers(0, 20, n), new)]
        attend(Batch(new, kv, 16, *heads[:3], "bf16", pad=5))


@pytest.mark.parametrize("page", [16, 20, 64])
def test_many_users_single_tokens_after_a_long_prefix(page):
    """Long enough to be computed for the batch at once; a short one is walked by every user's block."""
    for prefix in (6000, 100):
        attend(Batch([1] * 40, [1 + 7 * i % 40 for i in range(40)], page, 28, 4, 128, n_prefix=prefix, pad=2), every=1 if prefix < 1000 else 9)


def test_negative_indexes_and_lengths_beyond_the_table():
    # more new tokens than tokens in all: the first ones have no index, see nothing and get zeros
    for heads in (HEADS[0], HEADS[3]):
        attend(Batch([5, 2], [3, 2], 16, *heads))
        # a length beyond what the table holds: the keys that there are
        b = Batch([2, 1], [64, 20], 16, *heads)
        b.kv_len = [70, 20]
        attend(b)


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[1], HEADS[3]])
@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
def test_values_that_are_not_finite_stay_with_the_rows_that_see_them(heads, value):
    b = Batch([60, 30], [200, 60], 16, *heads)
    page, row = b.table[0][170 // 16], 170 % 16
    b.v_pages[page, row, 0, 3] = value
    want, spread = b.want()
    r = Rekv(*heads[:3], 16, b.dtype)
    q, kp, vp, start, kv, table = b.device()
    fine = np.isfinite(want)
    assert not fine.all()
    for max_kv in (None, LONG):
        got = r.attention_paged(q, kp, vp, start, kv, table, max_kv=max_kv).double().cpu().numpy()
        assert np.array_equal(np.isfinite(got), fine) and np.array_equal(np.isnan(got), np.isnan(want))
        assert (np.abs(got[fine] - want[fine]) <= b.tolerance(want, np.abs(spread))[fine]).all()


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[1], HEADS[3]])
def test_a_key_that_is_nan_stays_with_the_rows_that_see_it(heads):
    b = Batch([60], [200], 16, *heads)
    b.k_pages[b.table[0][170 // 16], 170 % 16, 0] = np.nan
    r = Rekv(*heads[:3], 16, b.dtype)
    q, kp, vp, start, kv, table = b.device()
    g = heads[0] // heads[1]
    for max_kv in (None, LONG):
        got = r.attention_paged(q, kp, vp, start, kv, table, max_kv=max_kv)
        assert torch.isfinite(got[:30]).all() and torch.isnan(got[30:, :g]).all() and torch.isfinite(got[30:, g:]).all()


@pytest.mark.parametrize("heads", [HEADS[0], HEADS[1], HEADS[3]])
@pytest.mark.parametrize("new,kv,prefix", [([1, 2], [5000, 900], 0), ([40, 3], [5000, 900], 0), ([1, 1, 1], [9, 40, 200], 3000), ([40, 30], [300, 90], 3000)])
def test_rows_of_nothing_but_nan_scores_are_nan(heads, new, kv, prefix):
    """A query that is NaN, and a lone key that is: however the keys are split, the row does not pass for one that sees nothing."""
    b = Batch(new, kv, 16, *heads, n_prefix=prefix)
    bad = new[0] - 1                                 # the first sequence's last token
    b.q[bad, -1, 5] = np.nan
    r = Rekv(*heads[:3], 16, b.dtype)
    q, kp, vp, start, kv_len, table = b.device()
    pages = ints(b.prefix_pages) if prefix else None
    for max_kv in (None, LONG):
        got = r.attention_shared_prefix(q, kp, vp, pages, prefix, start, kv_len, table, max_kv=max_kv) if prefix else \
            r.attention_paged(q, kp, vp, start, kv_len, table, max_kv=max_kv)
        nan = torch.isnan(got)
        assert nan[bad, -1].all() and int(nan.sum()) == heads[2]
    if not prefix:
        b.k_pages[b.table[0][(kv[0] - 1) // 16], (kv[0] - 1) % 16, 0] = np.nan
        for sinks in (0, 30):
            got = r.attention_paged(q, dev(b.k_pages, b.dtype), vp, start, kv_len, table, max_kv=LONG, window=1, sinks=sinks)
            assert torch.isnan(got[bad, :heads[0] // heads[1]]).all() and torch.isfinite(got[new[0]:]).all()


def test_large_scores():
    for heads in (HEADS[1], HEADS[3]):
        # scores of hundreds: a single key takes the row; the running maximum moves far
        b = Batch([3, 50], [300, 120], 48, *heads, scale=4.0)
        out, spread = b.want()
        r = Rekv(*heads[:3], 48, b.dtype)
        q, kp, vp, start, kv, table = b.device()
        got = r.attention_paged(q, kp, vp, start, kv, table).double().cpu().numpy()
        # scores of 16 x sigma^2 sqrt(D) about: their fp32 roundings count D * 256 as above
        bound = b.tolerance(out, spread) if b.dtype == "bf16" else 2.0 ** -24 * (2 * 256 * b.d + 400) * spread
        assert (np.abs(got - out) <= bound + (2.0 ** -24 * 2 * 256 * b.d * spread if b.dtype == "bf16" else 0)).all()


def test_pages_beyond_4_gib():
    hq, hkv, d, page = 8, 8, 128, 256                # 512 KB a page and tensor
    n_pages = 9000                                   # 4.7 GB each
    r = Rekv(hq, hkv, d, page)
    g = torch.Generator(device="cuda:0").manual_seed(1)
    kp, vp = torch.zeros((2, n_pages, page, hkv, d), dtype=torch.bfloat16, device="cuda:0").unbind(0)
    table = ints([[8999, 3, 8500], [8200, 8998, 1]])
    kv, start = ints([700, 520]), ints([0, 1, 3])
    for row in table.tolist():
        for pg in row:
            kp[pg] = torch.randn((page, hkv, d), device="cuda:0", generator=g)
            vp[pg] = torch.randn((page, hkv, d), device="cuda:0", generator=g)
    q = torch.randn((3, hq, d), device="cuda:0", generator=g).to(torch.bfloat16)
    got = r.attention_paged(q, kp, vp, start, kv, table)
    small = table.flatten().long()
    again = r.attention_paged(q, kp[small].contiguous(), vp[small].contiguous(), start, kv, ints([[0, 1, 2], [3, 4, 5]]))
    assert torch.equal(got, again)
    k, v = torch.zeros((2, 3, hkv, d), dtype=torch.bfloat16, device="cuda:0").unbind(0)
    k += 1
    v += 2
    r.append_kv(k, v, kp, vp, start, ints([513, 258]), table, rotate=False)
    assert (kp[8500, 0] == 1).all() and (kp[8998, 0:2] == 1).all() and (vp[8998, 0:2] == 2).all() and (vp[8500, 0] == 2).all()


def test_bad_page_numbers_are_not_followed():
    b = Batch([1, 4], [100, 60], 16, 14, 2, 64)
    r = Rekv(14, 2, 64, 16)
    q, kp, vp, start, kv, table = b.device()
    kp.nan_to_num_(0.0)
    vp.nan_to_num_(0.0)
    table = ints([[10 ** 9] * 7, [-5] * 7])
    assert torch.isfinite(r.attention_paged(q, kp, vp, start, kv, table)).all()
    old = kp.clone(), vp.clone()
    k = torch.ones((5, 2, 64), dtype=torch.bfloat16, device="cuda:0")
    r.append_kv(k, k, kp, vp, start, kv, table)
    assert torch.equal(kp, old[0]) and torch.equal(vp, old[1])


def test_results_are_the_same_every_time():
    for window in (None, 900):
        b = Batch([1, 5, 1], [3000, 1200, 77], 64, 28, 4, 128)
        r = Rekv(28, 4, 128, 64)
        q, kp, vp, start, kv, table = b.device()
        first = r.attention_paged(q, kp, vp, start, kv, table, window=window)
        for _ in range(4):
            assert torch.equal(first, r.attention_paged(q, kp, vp, start, kv, table, window=window))


def test_a_page_per_frame_is_the_dense_window_of_the_stream():
    """encode_chunk's cache seen as pages of one frame: with the window anchored alike (a chunk of one token) both agree."""
    nf, frames = 24, 9
    r = Rekv(14, 2, 64, nf)
    g = torch.Generator(device="cuda:0").manual_seed(3)
    k, v = (torch.randn((frames * nf, 2, 64), device="cuda:0", generator=g).to(torch.bfloat16) for _ in range(2))
    q = torch.randn((1, 14, 64), device="cuda:0", generator=g).to(torch.bfloat16)
    t = frames * nf - 1
    dense = r.encode_chunk(q, k, v, t, 1, 1, 3 * nf)
    paged = r.attention_paged(q, k.view(frames, nf, 2, 64), v.view(frames, nf, 2, 64), ints([0, 1]), ints([t + 1]), ints([list(range(frames))]),
                              window=3 * nf + 1)
    assert (dense.float() - paged.float()).abs().max() <= 2 * 2.0 ** -8 * dense.float().abs().max() + 2 * 2.0 ** -8 * v.float().abs().max()


def test_the_dtype_and_the_outputs_own_buffer():
    b = Batch([2], [40], 16, 14, 2, 64)
    r = Rekv(14, 2, 64, 16)
    q, kp, vp, start, kv, table = b.device()
    out = r.attention_paged(q, kp, vp, start, kv, table)
    assert out.dtype is TYPES["bf16"] and out.data_ptr() != q.data_ptr()
    big = ints([[0] * 5 + b.table[0] + [0] * 2])[:, 5:5 + len(b.table[0])]      # a table inside a larger one
    assert torch.equal(out, r.attention_paged(q, kp, vp, start, kv, big))
    assert dev(b.q, "bf16").equal(q)
