"""Ragged batches over a paged cache for the tests, with NaN wherever nothing may be read."""
from __future__ import annotations

import numpy as np
import torch

from oracle import paged_oracle as P

EPS = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}           # half a step, relative
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def rounded(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(TYPES[dtype]).double().numpy()


def dev(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x))
    return (t if dtype is None else t.float().to(TYPES[dtype])).to("cuda:0")


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda:0")


class Batch:
    """Sequences of new[s] new tokens and kv[s] in all.  Page 0 and all rows that hold no token are NaN; table entries past a
    sequence's pages are -1 (taken as page 0 if ever read)."""

    def __init__(self, new, kv, page, hq, hkv, d, dtype="bf16", n_prefix=0, pad=0, seed=0, spare=1, scale=1.0):
        g = np.random.default_rng([seed, page, hq, d, sum(kv)])
        self.new, self.kv_len, self.page, self.d, self.dtype, self.n_prefix = list(new), list(kv), page, d, dtype, n_prefix
        self.hq, self.hkv = hq, hkv
        self.token_start = [0, *np.cumsum(new).tolist()]
        self.total, self.n_tokens = self.token_start[-1], self.token_start[-1] + pad
        need, pre = [-(-max(k, 0) // page) for k in kv], -(-n_prefix // page)
        n_pages = 1 + sum(need) + pre + spare
        order = (1 + g.permutation(n_pages - 1)).tolist()
        self.prefix_pages, at, self.table = order[:pre], pre, []
        width = max(max(need), 1)
        for n in need:
            self.table.append(order[at:at + n] + [-1] * (width - n))
            at += n
        shape = (n_pages, page, hkv, d)
        self.k_pages, self.v_pages = np.full(shape, np.nan), np.full(shape, np.nan)
        for rows, n in [*zip(self.table, kv), (self.prefix_pages, n_prefix)]:
            for i, pg in enumerate(rows):
                m = min(page, n - i * page)
                if m > 0:
                    self.k_pages[pg, :m] = rounded(scale * g.standard_normal((m, hkv, d)), dtype)
                    self.v_pages[pg, :m] = rounded(g.standard_normal((m, hkv, d)) + 0.5, dtype)
        self.q = rounded(scale * g.standard_normal((self.n_tokens, hq, d)), dtype)
        self.q[self.total:] = np.nan

    def lost_pages(self, window, sinks):
        """Gives back the pages that no new token sees any more: their table entries become -1."""
        for s, (n, kv) in enumerate(zip(self.new, self.kv_len)):
            lo = max(0, kv - n + 1 - window)
            for i in range(len(self.table[s])):
                if i * self.page >= sinks and (i + 1) * self.page <= lo:
                    self.table[s][i] = -1

    def device(self):
        return (dev(self.q, self.dtype), dev(self.k_pages, self.dtype), dev(self.v_pages, self.dtype), ints(self.token_start), ints(self.kv_len),
                ints(self.table))

    def want(self, window=None, sinks=0, every=1):
        return P.attention(self.q, self.k_pages, self.v_pages, self.token_start, self.kv_len, self.table, self.d ** -0.5, window, sinks,
                           self.prefix_pages, self.n_prefix, every)

    def tolerance(self, out, spread, keys=None):
        """Per element.  bf16: the output's own rounding, that of each probability (weighted: spread), and 2^-11 of spread for scores
        and sums in fp32.  fp32: scores of D products of sizes up to 6 sigma^2 each sum to about D^(1/2) |q||k| < 16 after scaling, so
        D * 16 roundings move a probability at most; sums over the keys one rounding each; 64 more for the exponential."""
        if self.dtype == "bf16":
            return EPS["bf16"] * np.abs(out) + (EPS["bf16"] + 2.0 ** -11) * spread
        n = max(self.kv_len) + self.n_prefix
        return EPS["f32"] * (2 * 16 * self.d + n + 64) * spread + 1e-30


def check(got, batch, window=None, sinks=0, before=None, every=1):
    """The batch's rows against the definition (of `every`-th tokens); rows of no sequence as they were."""
    out, spread = batch.want(window, sinks, every)
    got = got.double().cpu().numpy()
    n = batch.total
    assert np.isfinite(got[:n]).all(), "not finite"
    at = np.isfinite(out[:n, 0, 0])
    assert at.all() or every > 1
    err = np.abs(got[:n][at] - out[:n][at])
    bad = err - batch.tolerance(out[:n][at], spread[:n][at])
    assert (bad <= 0).all(), f"off by {err.max():.3g}, {int((bad > 0).sum())} of {bad.size} beyond the bound"
    if before is not None:
        assert np.array_equal(got[n:], before.double().cpu().numpy()[n:], equal_nan=True)
