"""How the paged-cache calls behave as calls: refusals, both halves of the binding, streams, captured graphs, and a run of all of them."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as P
from paged_cases import Batch, check, dev, ints, rounded
from paper_2503_00540_amd import rekv
from paper_2503_00540_amd.rekv import Rekv, RekvError

pytestmark = pytest.mark.gpu


def small(dtype="bf16", **kw):
    b = Batch([1, 3], [40, 20], 16, 14, 2, 64, dtype, **kw)
    return b, Rekv(14, 2, 64, 16, dtype), b.device()


def test_wrong_arguments_are_refused():
    b, r, (q, kp, vp, start, kv, table) = small(n_prefix=20)
    pre = ints(b.prefix_pages)
    ok = dict(q=q, kp=kp, vp=vp, start=start, kv=kv, table=table, pre=pre, n=20)

    def both(match, **kw):
        a = dict(ok, **kw)
        batch = (a["start"], a["kv"], a["table"])
        for call in (lambda: r.attention_paged(a["q"], a["kp"], a["vp"], *batch),
                     lambda: r.attention_shared_prefix(a["q"], a["kp"], a["vp"], a["pre"], a["n"], *batch)):
            with pytest.raises((ValueError, RekvError), match=match):
                call()
    both("q", q=q.float())
    both("q", q=q[:, :12].contiguous())
    both("q", q=q[None])
    both("n_tokens=0", q=q[:0])
    both("k_pages", kp=kp[:-1])
    both("pages", kp=kp.transpose(0, 1), vp=vp.transpose(0, 1))
    both("token_start", start=start[:-1])
    both("token_start", start=start.long())
    both("kv_len", kv=kv[:, None])
    both("page_table", table=table.T.contiguous().T)
    both("max_pages=0", table=table[:, :0])
    both("CUDA", kv=kv.cpu())
    for n, pages in ((0, pre), (33, pre), (20, pre[None]), (20, pre.long())):
        with pytest.raises((ValueError, RekvError), match="prefix"):
            r.attention_shared_prefix(q, kp, vp, pages, n, start, kv, table)
    for kw in (dict(window=-1), dict(window=5, sinks=-1), dict(out=q[:2])):
        with pytest.raises((ValueError, RekvError), match="window|sinks|out"):
            r.attention_paged(q, kp, vp, start, kv, table, **kw)

    k = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda:0")
    batch = (kp, vp, start, kv, table)
    for kw, match in ((dict(sections=[8, 8]), "pairs"), (dict(sections=[40, -8]), "pairs"), (dict(base=1.0), "base"), (dict(sections=[]), "axes"),
                      (dict(sections=[32, 1 << 32]), "pairs"), (dict(rotate=False, positions=ints([0] * 4)), "without"),
                      (dict(positions=torch.zeros(3, dtype=torch.int32, device="cuda:0")), "positions"), (dict(q_out=q), "q_out"),
                      (dict(q=q[:3]), "q"), (dict(q=q, q_out=q[:, :, :32]), "q_out")):
        with pytest.raises((ValueError, RekvError), match=match):
            r.append_kv(k, k, *batch, **kw)
    with pytest.raises((ValueError, RekvError), match="v"):
        r.append_kv(k, k[:3], *batch)
    wide = torch.zeros((4, 2 * 64 + 4), dtype=torch.bfloat16, device="cuda:0")[:, :128].unflatten(1, (2, 64))
    with pytest.raises(RekvError, match="stride"):
        r.append_kv(wide, k, *batch)
    with pytest.raises(RekvError, match="stride"):
        r.rotate(wide, ints([0] * 4))
    with pytest.raises(RekvError, match="head_dim"):
        Rekv(4, 2, 20, 16, "f32").rotate(torch.zeros((1, 4, 20), device="cuda:0"), ints([0]))
    assert torch.equal(kp.nan_to_num(), dev(b.k_pages, "bf16").nan_to_num())


def test_launches_that_are_too_large_are_refused():
    r = Rekv(64, 8, 128, 16)
    for n_tokens, n_seqs, n_prefix in ((2, (1 << 24) - 1, 0), ((1 << 24) - 1, 1 << 23, 5000)):
        need = rekv.c_int64(7)
        assert r._lib.rekv_attention_paged_workspace(r._h, n_tokens, n_seqs, 5000, -1, 0, n_prefix, rekv.byref(need)) == 2     # not supported
        assert need.value == 0 and b"parts of the batch" in r._lib.rekv_last_error(r._h)
    many = torch.zeros((1, 1, 1 << 20, 64), dtype=torch.bfloat16, device="cuda:0")
    with pytest.raises(RekvError, match="64 MiB"):
        Rekv(1 << 20, 1 << 20, 64, 16).attention_paged(many[0], many, many, ints([0, 1]), ints([1]), ints([[0]]))
    need = rekv.c_int64(7)
    assert r._lib.rekv_attention_paged_workspace(r._h, 1 << 20, 1000, 5000, -1, 0, 0, rekv.byref(need)) == 0 and need.value == 0


def test_arguments_beyond_32_bits_do_not_wrap():
    b, r, (q, kp, vp, start, kv, table) = small()
    want = r.attention_paged(q, kp, vp, start, kv, table)
    for kw in (dict(window=1 << 32), dict(window=(1 << 31) - 1), dict(window=1 << 40, sinks=1 << 33), dict(max_kv=1 << 33), dict(max_kv=-5),
               dict(window=1 << 30, max_kv=1 << 32)):
        assert torch.equal(want, r.attention_paged(q, kp, vp, start, kv, table, **kw)), kw
    narrow = r.attention_paged(q, kp, vp, start, kv, table, window=0, sinks=1 << 40)
    assert torch.equal(want, narrow)
    with pytest.raises((ValueError, RekvError)):
        r.attention_shared_prefix(q, kp, vp, ints([1, 2]), (1 << 32) + 20, start, kv, table)


def test_the_workspace_stays_bounded_by_a_wild_hint():
    import ctypes
    r = Rekv(28, 4, 128, 64)
    L, n = rekv.lib(), ctypes.c_int64()
    for tokens, seqs in ((1, 1), (64, 64), (196, 1), (500, 500)):
        for max_kv in (1, 10 ** 4, 10 ** 6, (1 << 31) - 1):
            for prefix in (0, 10 ** 6):
                assert L.rekv_attention_paged_workspace(r._h, tokens, seqs, max_kv, -1, 0, prefix, ctypes.byref(n)) == 0
                assert n.value <= 1 << 30, (tokens, seqs, max_kv, prefix, n.value)


def test_a_small_workspace_is_refused_by_the_c_call():
    import ctypes
    b, r, (q, kp, vp, start, kv, table) = small(n_prefix=20)
    cache = r._paged(kp, vp, start, kv, table, 4)
    need = ctypes.c_int64()
    L = rekv.lib()
    assert L.rekv_attention_paged_workspace(r._h, 4, 2, 40, -1, 0, 20, ctypes.byref(need)) == 0
    ws = torch.empty(need.value + 512, dtype=torch.uint8, device="cuda:0")
    args = (r._h, ctypes.byref(cache), q.data_ptr(), ints(b.prefix_pages).data_ptr(), 20, 40, q.data_ptr())
    if need.value:
        for p, n in ((None, need.value), (ws.data_ptr(), need.value - 1), (ws.data_ptr() + 16, need.value)):
            assert L.rekv_attention_shared_prefix(*args, p, n, None) == 1
            assert b"workspace" in L.rekv_last_error(r._h)
    assert L.rekv_attention_paged_workspace(r._h, 0, 2, 40, -1, 0, 0, ctypes.byref(need)) == 1 and need.value == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_native_half_and_python_methods_do_the_same(dtype):
    b, r, (q, kp, vp, start, kv, table) = small(dtype, n_prefix=20, pad=1)
    g = np.random.default_rng(0)
    k, v = (dev(rounded(g.standard_normal((5, 2, 64)), dtype), dtype) for _ in range(2))
    pos = ints(g.integers(0, 9999, (3, 5)).tolist())
    native = r._fast
    results, taken = [], []
    for fast in (native, rekv._NoNative()):
        class Counting:
            def __getattr__(self, name):
                def call(*args):
                    got = getattr(fast, name)(*args)
                    taken.append((name, got is not None))
                    return got
                return call
        r._fast = Counting()
        a, c = kp.clone(), vp.clone()
        zero = torch.zeros_like(q)
        got = [r.rotate(q, pos, sections=[8, 12, 12], base=1e5, layout="interleaved", order="turns", inverse=True),
               r.rotate(q, pos[0], out=zero.clone()),
               r.append_kv(k, v, a, c, start, kv, table, q=q, positions=pos, sections=(8, 12, 12), q_out=zero.clone()),
               r.append_kv(k, v, a, c, start, kv, table), a, c,
               r.append_kv(k, v, a, c, start, kv, table, rotate=False),
               r.attention_paged(q, kp, vp, start, kv, table, window=9, sinks=2, out=zero.clone()),
               r.attention_paged(q, kp, vp, start, kv, table, max_kv=40, out=zero.clone()),
               r.attention_shared_prefix(q, kp, vp, ints(b.prefix_pages), 20, start, kv, table, out=zero.clone())]
        results.append(got)
    r._fast = native
    for x, y in zip(*results):
        assert (x is None and y is None) or torch.equal(x.nan_to_num(9.0), y.nan_to_num(9.0))
    half = len(taken) // 2
    assert all(t for _, t in taken[:half]) and not any(t for _, t in taken[half:]), taken


def test_calls_of_one_context_on_two_streams_at_once():
    b1, b2 = Batch([1], [6000], 64, 28, 4, 128, n_prefix=0), Batch([1, 1], [50, 4000], 64, 28, 4, 128, seed=1)
    r = Rekv(28, 4, 128, 64)
    d1, d2 = b1.device(), b2.device()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = [], []
    for _ in range(10):
        for s, d, o in zip(streams, (d1, d2), outs):
            with torch.cuda.stream(s):
                o.append(r.attention_paged(*d))
    torch.cuda.synchronize()
    for o, b in zip(outs, (b1, b2)):
        check(o[0], b)
        assert all(torch.equal(o[0], x) for x in o[1:])


def test_captured_calls_replay_with_other_lengths_beside_eager_ones():
    """Two graphs of one context, each with a workspace of its own; lengths, tables and inputs change between the replays."""
    r = Rekv(28, 4, 128, 64)
    b = Batch([1, 1, 1], [900, 2500, 3], 64, 28, 4, 128, pad=1)
    p = Batch([1, 1], [30, 100], 64, 28, 4, 128, n_prefix=1500, seed=2)
    dp, pre = p.device(), ints(p.prefix_pages)
    q, kp, vp, start, kv, table = b.device()
    k, v = (torch.zeros((4, 4, 128), dtype=torch.bfloat16, device="cuda:0") for _ in range(2))
    q_rot, out, out2 = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(dp[0])

    def step():
        r.append_kv(k, v, kp, vp, start, kv, table, q=q, q_out=q_rot)
        r.attention_paged(q_rot, kp, vp, start, kv, table, max_kv=4096, window=2000, sinks=4, out=out)

    def step2():
        r.attention_shared_prefix(dp[0], dp[1], dp[2], pre, 1500, dp[3], dp[4], dp[5], max_kv=128, out=out2)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step(), step2()
    torch.cuda.synchronize()
    g1, g2 = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(g1):
        step()
    with torch.cuda.graph(g2):
        step2()
    gen = torch.Generator(device="cuda:0").manual_seed(4)
    for i in range(4):
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, device="cuda:0", generator=gen))
        lens = [900 - 40 * i, 2500 - 300 * i, 3 + i]
        kv.copy_(ints(lens))
        before = kp.clone(), vp.clone()
        out.fill_(7.0), out2.fill_(7.0)
        g1.replay(), g2.replay()
        torch.cuda.synchronize()
        got, got2 = out.clone(), out2.clone()
        large = r.attention_paged(torch.cat([q] * 9), kp, vp, ints(list(range(28)) + [30]), kv.repeat(10)[:28], table.repeat(10, 1)[:28])
        assert torch.isfinite(large[:3]).all()
        check(got2, p)
        kp2, vp2 = before
        want_q = r.append_kv(k, v, kp2, vp2, start, kv, table, q=q, q_out=torch.zeros_like(q))
        assert torch.equal(kp2.nan_to_num(9), kp.nan_to_num(9)) and torch.equal(vp2.nan_to_num(9), vp.nan_to_num(9))
        want = r.attention_paged(want_q, kp2, vp2, start, kv, table, max_kv=4096, window=2000, sinks=4, out=torch.full_like(q, 7.0))
        assert torch.equal(got, want) and (got[3] == 7).all()
        b.q[:3] = want_q[:3].double().cpu().numpy()
        b.k_pages, b.v_pages, b.kv_len = kp.double().cpu().numpy(), vp.double().cpu().numpy(), lens
        check(got, b, 2000, 4)


@pytest.mark.parametrize("heads", [(14, 2, 64, "bf16"), (28, 4, 128, "bf16"), (4, 1, 64, "f32")])
def test_streams_and_questions_in_one_cache(heads):
    """Two live streams write frames with three position axes into pages of a frame and attend through a window; the frames'
    vectors and a question's retrieval work on the same arena; then two users answer token by token over the retrieved frames
    as a shared prefix, their own tokens in pages of their own."""
    hq, hkv, d, dtype = heads
    nf, frames, top = 24, 5, 2
    r = Rekv(hq, hkv, d, nf, dtype)
    g = np.random.default_rng(11)
    sections = [d // 2 - 2 * (d // 6), d // 6, d // 6]
    n_pages = 1 + 2 * frames + 3
    kp, vp = (torch.full((n_pages, nf, hkv, d), float("nan"), dtype=r.torch_dtype, device="cuda:0") for _ in range(2))
    table = [list(range(1, 1 + frames)), list(range(1 + frames, 1 + 2 * frames))]
    state = Batch([nf, nf], [nf, nf], nf, hq, hkv, d, dtype)                # carries the definitions' view
    state.table, state.k_pages, state.v_pages = table, np.full(kp.shape, np.nan), np.full(vp.shape, np.nan)
    for f in range(frames):
        q, k, v = (rounded(g.standard_normal((2 * nf, h, d)), dtype) for h in (hq, hkv, hkv))
        i = np.tile(np.arange(nf), 2)
        pos = np.stack([np.full(2 * nf, f), i // 6, i % 6]).astype(np.int32)
        start, kv = ints([0, nf, 2 * nf]), ints([(f + 1) * nf] * 2)
        qr = r.append_kv(dev(k, dtype), dev(v, dtype), kp, vp, start, kv, ints(table), q=dev(q, dtype), positions=dev(pos), sections=sections)
        out = r.attention_paged(qr, kp, vp, start, kv, ints(table), window=2 * nf, sinks=5)
        state.kv_len, state.q = [(f + 1) * nf] * 2, qr.double().cpu().numpy()
        state.k_pages = P.append(state.k_pages, P.rotate(k, pos, sections, 1e4, "half"), state.token_start, state.kv_len, table)
        state.v_pages = P.append(state.v_pages, v, state.token_start, state.kv_len, table)
        got_k = kp.double().cpu().numpy()
        err = np.abs(np.nan_to_num(got_k) - np.nan_to_num(state.k_pages))
        assert err.max() <= (2.0 ** -8 if dtype == "bf16" else 2.0 ** -20) * np.nanmax(np.abs(state.k_pages))
        state.k_pages = got_k
        check(out, state, 2 * nf, 5)
    stream = kp[1:1 + frames].reshape(frames * nf, hkv, d)                  # stream 0's arena of frames, as it lies
    fk = r.frame_keys(stream, frames)
    idx, n_sel, _ = r.retrieve_topk(fk, frames, dev(rounded(g.standard_normal((1, 4, hq, d)), dtype), dtype), top)
    assert n_sel.tolist() == [top]
    prefix = idx[0] + 1                                                     # pages of the retrieved frames
    users = Batch([1, 1], [1, 1], nf, hq, hkv, d, dtype)
    users.table, users.prefix_pages, users.n_prefix = [[n_pages - 1], [n_pages - 2]], prefix.tolist(), top * nf
    for t in range(4):
        q, k, v = (dev(rounded(g.standard_normal((2, h, d)), dtype), dtype) for h in (hq, hkv, hkv))
        start, kv = ints([0, 1, 2]), ints([t + 1, t + 1])
        qr = r.append_kv(k, v, kp, vp, start, kv, ints(users.table), q=q, positions=ints([top * nf + t] * 2))
        out = r.attention_shared_prefix(qr, kp, vp, prefix, top * nf, start, kv, ints(users.table))
        users.kv_len, users.q = [t + 1, t + 1], qr.double().cpu().numpy()
        users.k_pages, users.v_pages = kp.double().cpu().numpy(), vp.double().cpu().numpy()
        check(out, users)
