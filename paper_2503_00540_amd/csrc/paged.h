// Device pieces of the paged cache: which sequence a token or a row block belongs to, which page a key lies in, and what the
// rows of a block see.
#pragma once

#include "common.h"

namespace rekv {

// A uniform word of a table that no kernel in flight writes, through the scalar cache.
__device__ inline int32_t scalar_word(const int32_t* p, int64_t i) {
    typedef const __attribute__((address_space(4))) int32_t* constant_ptr;
    return reinterpret_cast<constant_ptr>(reinterpret_cast<uintptr_t>(p))[i];
}

__device__ inline int clamped(int v, int lo, int hi) { return v < lo ? lo : v < hi ? v : hi; }

struct Sequence {
    int i, start, end, kv;      // its number, token rows [start, end) and length, within their bounds
};

// The last sequence i whose off(i, token_start[i]) is at most `target`; off does not decrease, and that of sequence 0 counts as
// reached.  A wavefront narrows 64 to one at a time, and reads what the last 64 hold with the same round trip.
template <class Off>
__device__ inline Sequence find_sequence(const PagedBatch& b, int lane, int target, Off off) {
    int lo = 0, n = b.n_seqs;
    while (n > 64) {
        const int step = (n + 63) / 64, i = lane * step;
        const bool reached = i == 0 || (i < n && off(lo + i, b.token_start[i < n ? lo + i : lo]) <= target);
        const int last = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(reached));
        lo += last * step;
        n = n - last * step < step ? n - last * step : step;
    }
    const int j = lane < n ? lo + lane : lo;
    const int start = b.token_start[j], end = b.token_start[j + 1], kv = b.kv_len[j];
    const bool reached = lane == 0 || (lane < n && off(j, start) <= target);
    const int last = 63 - __builtin_clzll(__builtin_amdgcn_ballot_w64(reached));
    Sequence s;
    s.i = lo + last;
    s.start = clamped(__builtin_amdgcn_readlane(start, last), 0, b.n_tokens);
    s.end = clamped(__builtin_amdgcn_readlane(end, last), s.start, b.n_tokens);
    s.kv = clamped(__builtin_amdgcn_readlane(kv, last), 0, 1 << 30);
    return s;
}

// The batch's token rows that belong to sequences: [first, end).
struct TokenRange {
    int first, end;
};
__device__ inline TokenRange token_range(const PagedBatch& b) {
    const int first = clamped(scalar_word(b.token_start, 0), 0, b.n_tokens);
    return TokenRange{first, clamped(scalar_word(b.token_start, b.n_seqs), first, b.n_tokens)};
}

// What a row block attends to.  Its rows are (token, query head of the KV head's group), token by token.
//   own keys:  the token at index p sees j < hi(p) = min(p + 1, capacity) with j > p - window or j < sinks
//   prefix:    all of it
struct Job {
    const int32_t* table;   // own pages
    int split, slot, n_splits;
    int row0, n_rows;       // first row of the block, rows of the sequence (or of all sequences: the prefix job)
    int token0;             // token row of row 0
    int p0;                 // index of that token in its sequence
    int n_prefix;           // prefix tokens this block sees, 0: none
    bool own;               // whether it sees own keys
};

// Block r of a launch (of one KV head): first the prefix jobs, where the prefix is computed for the batch at once, then the own ones,
// row blocks fastest.  False: no work.
template <int ROWS>
__device__ inline bool find_prefix_job(const PagedProblem& p, int prefix_blocks, int prefix_splits, int r, Job* job) {
    // (rows of no sequence too: the merge leaves them out, and nothing has to be looked up)
    const int G = p.n_q_heads / p.n_kv_heads;
    job->split = job->slot = r / prefix_blocks;
    job->n_splits = prefix_splits;
    job->row0 = (r - job->split * prefix_blocks) * ROWS;
    job->n_rows = p.b.n_tokens * G;
    job->token0 = 0;
    job->p0 = 0;
    job->n_prefix = p.n_prefix;
    job->own = false;
    job->table = p.prefix_pages;
    return job->row0 < job->n_rows;
}
template <int ROWS>
__device__ inline bool find_own_job(const PagedProblem& p, int prefix_blocks, int prefix_splits, int blocks, int splits, int r, int lane, Job* job) {
    const int G = p.n_q_heads / p.n_kv_heads;
    const PagedBatch& b = p.b;
    r -= prefix_blocks * prefix_splits;
    job->split = r / blocks;
    job->slot = job->split + (prefix_blocks > 0 ? prefix_splits : 0);
    job->n_splits = splits;
    // A sequence's blocks start at floor(start * G / ROWS) + its number: at least as many as it needs, some stay empty.
    // The last blocks first: of a long prompt they have the most keys.
    const int blk = blocks - 1 - (r - job->split * blocks);
    auto first_block = [&](int i, int start) { return clamped(start, 0, b.n_tokens) * G / ROWS + i; };
    const Sequence s = find_sequence(b, lane, blk, first_block);
    job->row0 = (blk - first_block(s.i, s.start)) * ROWS;
    job->n_rows = (s.end - s.start) * G;
    job->token0 = s.start;
    job->p0 = s.kv - (s.end - s.start);
    job->n_prefix = prefix_blocks > 0 ? 0 : p.n_prefix;
    job->own = true;
    job->table = b.page_table + s.i * b.table_stride;
    return job->row0 >= 0 && job->row0 < job->n_rows;
}

// The keys of a block as a list of tiles of T keys: the prefix's, those of the first tokens, those of the window.  Tiles of own keys
// start at multiples of T, whatever the window; where the two parts would overlap there is one, from key 0 on.
template <int T>
struct Tiles {
    int n_prefix_tiles, n_sink_tiles, n;
    int n_prefix, sinks, first, hi, lo;       // own: the window part starts at key `first`; keys some row sees: [0, sinks) and [lo, hi)
    // tiles that all rows see whole: [0, a) of the prefix, [n_prefix_tiles, b) of the first tokens, [c, d) of the window part
    int a, b, c, d;

    __device__ Tiles(const PagedProblem& p, const Job& j, int first_tok, int last_tok) {
        n_prefix = j.n_prefix;
        n_prefix_tiles = (n_prefix + T - 1) / T;
        a = n_prefix / T;
        n_sink_tiles = first = lo = 0;
        sinks = 0;
        hi = 0;
        b = c = d = n = n_prefix_tiles;
        if (!j.own) return;
        const int cap = p.b.capacity;
        const int hi_all = clamped(j.p0 + first_tok + 1, 0, cap);        // keys below that every row sees, but for the window
        hi = clamped(j.p0 + last_tok + 1, 0, cap);
        int lo_all = 0;
        if (p.window >= 0) {
            lo = j.p0 + first_tok + 1 - p.window;
            lo_all = j.p0 + last_tok + 1 - p.window;
            lo = clamped(lo, 0, hi > 0 ? hi - 1 : 0);
            lo_all = lo_all < 0 ? 0 : lo_all;
            sinks = p.sinks < hi ? p.sinks : hi;
        }
        const int sink_tiles = (sinks + T - 1) / T;
        if (lo / T > sink_tiles) {
            n_sink_tiles = sink_tiles;
            first = lo / T * T;
        }
        const int own0 = n_prefix_tiles + n_sink_tiles;
        n = own0 + (hi > first ? (hi - first + T - 1) / T : 0);
        b = n_sink_tiles > 0 ? n_prefix_tiles + (sinks < hi_all ? sinks : hi_all) / T : n_prefix_tiles;
        c = own0 + (lo_all > first ? lo_all - first + T - 1 : 0) / T;
        d = own0 + (hi_all > first ? hi_all - first : 0) / T;
    }
    __device__ bool in_prefix(int t) const { return t < n_prefix_tiles; }
    __device__ int key0(int t) const {
        if (t < n_prefix_tiles) return t * T;
        t -= n_prefix_tiles;
        return t < n_sink_tiles ? t * T : first + (t - n_sink_tiles) * T;
    }
    // rows of tile t that are fetched, relative to its first key; the others repeat the nearest of these
    __device__ void rows(int t, int* r0, int* r1) const {
        const int k0 = key0(t);
        *r0 = 0;
        int end = n_prefix;
        if (t >= n_prefix_tiles) {
            const bool sink = t < n_prefix_tiles + n_sink_tiles;
            end = sink ? sinks : hi;
            if (!sink && first > 0 && lo > k0) *r0 = lo - k0;
        }
        *r1 = end - k0 < T ? end - k0 - 1 : T - 1;
    }
    // whether all rows see tile t whole
    __device__ bool whole(int t) const { return t < a || (t >= n_prefix_tiles && t < b) || (t >= c && t < d); }
};

// What a row sees of a part: keys [lo, hi) and those below `first`.
struct Seen {
    int lo, hi, first;
    __device__ bool operator()(int key) const { return (uint32_t)(key - lo) < (uint32_t)(hi - lo) | key < first; }
};
// Of the own keys, for the token at index pos.
__device__ inline Seen seen_by(const PagedProblem& p, int pos) {
    Seen s = {0, clamped(pos + 1, 0, p.b.capacity), 0};
    if (p.window >= 0) {
        s.lo = clamped(pos + 1 - p.window, 0, s.hi);
        s.first = p.sinks < s.lo ? p.sinks : s.lo;
    }
    return s;
}

}  // namespace rekv
