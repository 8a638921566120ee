// Attention of a ragged batch over a paged cache, bf16: sliding windows with first tokens that stay visible, and batches that
// share a long prefix.
//
//   o = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m),  s_j = scale q.k_j,  over the keys j a token sees (paged.h)
//
// in one pass with a running maximum m and sum in fp32; probabilities are rounded to bf16 for the second product (their
// sum is taken before), which adds to an output's own rounding about as much again.  Where the keys of a row are split over workgroups,
// or between a prefix and the row's own keys, each part leaves (m, sum, O) in fp32 and a second launch joins them.
//
// Rows are stacked as in attention_bf16.hip, the G query heads of a KV head token by token, so a K/V tile in LDS
// serves them all; a prefix shared by the batch is walked by blocks of all sequences' rows, so that one user's few rows do not
// read it for themselves.  Operand layouts, the four LDS stages per tensor and the order of a step are those of attention_bf16.hip.
// What differs is where tiles come from: 32 keys lie in one or two pages, whose numbers come through the scalar cache a
// step before the loads that need them.
#include "attention_mfma.h"
#include "paged.h"

namespace rekv {
namespace {

constexpr int STAGES = 4;
constexpr int WAVES = 4;
constexpr int WM = 32;
constexpr int BM = WAVES * WM;

struct PagedArgs {
    PagedProblem p;
    int32_t prefix_blocks, prefix_splits, blocks, splits, min_tiles, n_slots;
    float* part_o;        // [slot][token * Hq + head][D]
    float* part_ml;       // [slot][token * Hq + head][2]: maximum (of base-2 exponents), sum
};

template <int N>
__device__ inline void step_barrier() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// As dma16 (attention_mfma.h), from a 64-bit address per lane.
__device__ inline void dma16_at(uint64_t addr, uint32_t lds_addr) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
                 ::"v"(addr), "s"(__builtin_amdgcn_readfirstlane(lds_addr)) : "memory", "m0");
}

// Page numbers of a tile's first key and of the page after it.
struct Entries {
    int32_t a, b;
};
// A tile in the pages: byte offsets (from k_pages or v_pages) of its row 0 as the first page has it and as the next one would,
// and how many rows lie in the first.
struct Place {
    int64_t a, b;
    int rows_a;
    bool whole;             // all rows see the tile whole
};

// TWO_PAGES: 32 keys from a multiple of 32 on lie in two pages at most (pages of 32 tokens or more, or of 16); otherwise every
// lane looks its rows' pages up.
template <int D, bool TWO_PAGES>
__global__ __launch_bounds__(WAVES * 64, 2) void attn_paged_kernel(PagedArgs a) {
    constexpr int CH = D / 8;                 // 16-byte chunks per key row
    constexpr int RPI = 64 / CH;              // key rows one 1 KB wave-wide load covers
    constexpr int N_DMA = BN / RPI / WAVES;   // such loads per wave, tile and tensor
    constexpr uint32_t TILE_B = BN * D * 2;
    __shared__ __attribute__((aligned(1024))) bf16_t lds[2 * STAGES * BN * D];
    __shared__ int sh_dropped;

    const PagedProblem& p = a.p;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int col = lane & 31, hh = lane >> 5;
    const int G = p.n_q_heads / p.n_kv_heads;

    // KV heads fastest: workgroups are dealt to the eight XCDs in turn, so that one of them sees few heads' keys
    const int L = blockIdx.x / p.n_kv_heads, kvh = blockIdx.x - L * p.n_kv_heads;
    Job job;
    if (!find_job<BM>(p, a.prefix_blocks, a.prefix_splits, a.blocks, a.splits, L, lane, &job)) return;

    const int row = job.row0 + wave * WM + col;
    const bool row_ok = row < job.n_rows;
    const int tok = row / G;
    const int first_tok = job.row0 / G;
    int last_tok = (job.row0 + BM - 1) / G;
    const int n_tok = job.n_rows / G;
    last_tok = last_tok < n_tok ? last_tok : n_tok - 1;
    const bool wave_active = job.row0 + wave * WM < job.n_rows;
    const Tiles<BN> tiles(p, job, first_tok, last_tok);
    int per_split = (tiles.n + job.n_splits - 1) / job.n_splits;
    per_split = per_split > a.min_tiles ? per_split : a.min_tiles;
    const int t_begin = job.split * per_split;
    const int t_end = t_begin + per_split < tiles.n ? t_begin + per_split : tiles.n;
    const int pos = job.p0 + tok;                                       // this row's token: its index, the keys below it
    const int row_hi = clamped(pos + 1, 0, p.b.capacity);

    const uint32_t row_b = (uint32_t)p.n_kv_heads * D * 2u;             // bytes of a token's keys
    const char* k_base = static_cast<const char*>(p.b.k_pages) + kvh * D * 2;
    const char* v_base = static_cast<const char*>(p.b.v_pages) + kvh * D * 2;
    const int page = (int)p.b.by_page.d;

    // ---- lane-constant addressing, as in attention_bf16.hip
    const uint32_t lds0 = lds_addr_of(lds);
    const int dma_row = wave * N_DMA * RPI + lane / CH;
    const int dma_p = lane % CH;
    uint32_t dma_coff[N_DMA], dma_off[N_DMA];
#pragma unroll
    for (int j = 0; j < N_DMA; ++j) {
        dma_coff[j] = (uint32_t)(dma_p ^ swz<D>(dma_row + j * RPI)) * 16u;
        dma_off[j] = (uint32_t)(dma_row + j * RPI) * row_b + dma_coff[j];
    }
    const uint32_t dma_lds = lds0 + (uint32_t)(wave * N_DMA) * 1024u;
    uint32_t k_addr[D / 16];
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
        k_addr[ks] = lds0 + (uint32_t)(col * D + (((ks * 2 + hh) ^ swz<D>(col)) * 8)) * 2u;
    uint32_t v_addr[2][D / 32];
    {
        const int gq = lane >> 4, i16 = lane & 15, qd = i16 & 3, jk = i16 >> 2;
        const int cl = (gq & 1) * 2 + (qd >> 1), half = qd & 1;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int keyl = r * 8 + hh * 4 + jk;
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
                v_addr[r][db] = lds0 + STAGES * TILE_B + (uint32_t)(keyl * D + (((db * 4 + cl) ^ swz<D>(keyl)) * 8) + half * 4) * 2u;
        }
    }

    // ---- pages
    auto table_of = [&](int t) { return tiles.in_prefix(t) ? p.prefix_pages : job.table; };
    auto last_slot_of = [&](int t) {
        return tiles.in_prefix(t) ? (int)quot((uint32_t)(tiles.n_prefix - 1), p.b.by_page) : p.b.max_pages - 1;
    };
    auto in_list = [&](int t) { return t < t_end ? t : t_end - 1; };
    auto entries = [&](int t) {              // t is in the list
        const int slot = (int)quot((uint32_t)tiles.key0(t), p.b.by_page), last = last_slot_of(t);
        const int32_t* table = table_of(t);
        return Entries{scalar_word(table, slot), scalar_word(table, slot < last ? slot + 1 : last)};
    };
    auto place = [&](int t, Entries e) {
        const int k0 = tiles.key0(t), within = k0 - (int)quot((uint32_t)k0, p.b.by_page) * page;
        const int pa = clamped(e.a, 0, p.b.n_pages - 1), pb = clamped(e.b, 0, p.b.n_pages - 1);
        return Place{((int64_t)pa * page + within) * row_b, ((int64_t)pb * page + within - page) * row_b, page - within, tiles.whole(t, 1)};
    };
    // Row r of a tile, by the page it lies in: lanes of either page take a load of their own, from a uniform address (where a
    // load has lanes of both, one more is in flight than step_barrier counts, which only makes it wait longer).
    auto dma_row_of = [&](const char* base, const Place& at, int r, uint32_t off, uint32_t dst) {
        if (r < at.rows_a) dma16<false>(base + at.a, off, dst);
        else dma16<false>(base + at.b, off, dst);
    };
    // Tile t; the rows that no row of the block sees repeat the nearest that one does.
    auto dma_tile = [&](const char* base, int t, const Place& at, uint32_t stage_b) {
        if (TWO_PAGES) {
            if (at.whole && at.rows_a >= BN) {
#pragma unroll
                for (int j = 0; j < N_DMA; ++j) dma16<false>(base + at.a, dma_off[j], dma_lds + stage_b + j * 1024u);
                return;
            }
            int r0 = 0, r1 = BN - 1;
            if (!at.whole) tiles.rows(t, &r0, &r1);
#pragma unroll
            for (int j = 0; j < N_DMA; ++j) {
                const int r = clamped(dma_row + j * RPI, r0, r1);
                dma_row_of(base, at, r, (uint32_t)r * row_b + dma_coff[j], dma_lds + stage_b + j * 1024u);
            }
        } else {
            const int32_t* table = table_of(t);
            const int k0 = tiles.key0(t);
            int r0, r1;
            tiles.rows(t, &r0, &r1);
            uint64_t from[N_DMA];
#pragma unroll
            for (int j = 0; j < N_DMA; ++j) {
                const int key = k0 + clamped(dma_row + j * RPI, r0, r1), slot = (int)quot((uint32_t)key, p.b.by_page);
                const int pg = clamped(table[slot], 0, p.b.n_pages - 1);
                from[j] = reinterpret_cast<uint64_t>(base) + (uint64_t)((int64_t)pg * page + (key - slot * page)) * row_b + dma_coff[j];
            }
#pragma unroll
            for (int j = 0; j < N_DMA; ++j) dma16_at(from[j], dma_lds + stage_b + j * 1024u);
        }
    };
    constexpr int DMA_PER_STEP = 2 * N_DMA;

    bf16x8 qf[D / 16];
    const int64_t q_row = (int64_t)(job.token0 + tok) * p.n_q_heads + kvh * G + (row - tok * G);     // over (token, head)
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) {
        u32x4 v = {0u, 0u, 0u, 0u};
        if (row_ok) v = *reinterpret_cast<const u32x4*>(static_cast<const bf16_t*>(p.q) + q_row * D + ks * 16 + hh * 8);
        qf[ks] = __builtin_bit_cast(bf16x8, v);
    }

    f32x16 o[D / 32];
#pragma unroll
    for (int i = 0; i < D / 32; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    float m_ref = -INFINITY, l_part = 0.f;
    const float sc = p.scale * 1.4426950408889634f;

    auto qk = [&](const bf16x8 (&kf)[D / 16], f32x16& s) {
#pragma unroll
        for (int j = 0; j < 16; ++j) s[j] = 0.f;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[ks], s, 0, 0, 0);
    };
    auto load_k = [&](uint32_t stage_b, bf16x8 (&kf)[D / 16]) {
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) kf[ks] = *reinterpret_cast<LDS_AS const bf16x8*>(k_addr[ks] + stage_b);
    };

    // Entries of tile t + 5 and places of tiles t + 4 and t + 3, as step t needs them.
    Entries e_next;
    Place at_k, at_v;

    // A tile that not every row sees whole: probabilities of 0 keep a value out only if it is finite, so its infinities and NaNs
    // become 0 in LDS (every wavefront sees to that for itself, before it reads the tile) and are added after the loop.
    auto drop_nonfinite = [&](uint32_t stage_b) {
        const uint32_t at = lds0 + STAGES * TILE_B + stage_b + lane * 16u;
        uint32_t any = 0;
#pragma unroll
        for (uint32_t i = 0; i < TILE_B; i += 1024) {
            const u32x4 w = *reinterpret_cast<LDS_AS const u32x4*>(at + i);
#pragma unroll
            for (int k = 0; k < 4; ++k) any |= (w[k] & 0x7f807f80u) + 0x00800080u;      // bit 15 of a half: its exponent is all ones
        }
        if (__builtin_amdgcn_ballot_w64((any & 0x80008000u) != 0) == 0) return;
        sh_dropped = 1;
#pragma unroll 1
        for (uint32_t i = 0; i < TILE_B; i += 1024) {
            u32x4 w = *reinterpret_cast<LDS_AS const u32x4*>(at + i);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if ((w[k] & 0x7f80u) == 0x7f80u) w[k] &= 0xffff0000u;
                if ((w[k] & 0x7f800000u) == 0x7f800000u) w[k] &= 0x0000ffffu;
            }
            *reinterpret_cast<LDS_AS u32x4*>(at + i) = w;
        }
    };

    // One step, as in attention_bf16.hip.
    auto step = [&](int t, f32x16& s_cur, f32x16& s_next, auto kn, auto kl, auto vc, auto vl) __attribute__((always_inline)) {
        constexpr uint32_t KN = decltype(kn)::value * TILE_B, KL = decltype(kl)::value * TILE_B;
        constexpr uint32_t VC = decltype(vc)::value * TILE_B, VL = decltype(vl)::value * TILE_B;
        if (TWO_PAGES) {
            at_v = at_k;
            at_k = place(in_list(t + 4), e_next);
        }
        dma_tile(k_base, in_list(t + 4), at_k, KL);
        dma_tile(v_base, in_list(t + 3), at_v, STAGES * TILE_B + VL);
        if (TWO_PAGES) e_next = entries(in_list(t + 5));
        if (!tiles.whole(t, 1)) {
            const int k0 = tiles.key0(t);
            const bool pre = tiles.in_prefix(t);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int key = k0 + (j >> 2) * 8 + hh * 4 + (j & 3);
                s_cur[j] = (pre ? key < tiles.n_prefix : sees(p, pos, row_hi, key)) ? s_cur[j] : -INFINITY;
            }
            drop_nonfinite(VC);
        }
        bf16x8 kf[D / 16];
        load_k(KN, kf);
        bf16x8 vf[2][D / 32];
        auto load_v = [&](int g16) {
#pragma unroll
            for (int db = 0; db < D / 32; ++db) {
                const tr4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
                    reinterpret_cast<LDS_AS tr4_t*>(v_addr[0][db] + VC + g16 * 16 * D * 2));
                const tr4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(
                    reinterpret_cast<LDS_AS tr4_t*>(v_addr[1][db] + VC + g16 * 16 * D * 2));
                vf[g16][db] = __builtin_shufflevector(__builtin_bit_cast(bf16x4, lo),
                                                      __builtin_bit_cast(bf16x4, hi), 0, 1, 2, 3, 4, 5, 6, 7);
            }
        };
        load_v(0);
        __builtin_amdgcn_sched_barrier(0);
        float mx = s_cur[0];
#pragma unroll
        for (int j = 1; j < 16; ++j) mx = fmaxf(mx, s_cur[j]);
        mx = pair_max(mx);
        const float mt2 = mx * sc;
        if (__builtin_amdgcn_ballot_w64(mt2 > m_ref + RESCALE_GAP) != 0) {
            const float m_new = fmaxf(m_ref, mt2);
            const float alpha = (m_new == -INFINITY) ? 1.f : __builtin_amdgcn_exp2f(m_ref - m_new);
            l_part *= alpha;
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[i][j] *= alpha;
            m_ref = m_new;
        }
        const float mr = (m_ref == -INFINITY) ? 0.f : m_ref;
        __builtin_amdgcn_s_setprio(3);
        qk(kf, s_next);            // past the last tile this works on a stale stage and is unused
        load_v(1);
#pragma unroll
        for (int g16 = 0; g16 < 2; ++g16) {
            float e[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                e[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s_cur[g16 * 8 + j], sc, -mr));
                l_part += e[j];
            }
            bf16x8 pf;
#pragma unroll
            for (int j = 0; j < 8; j += 2) {
                const bf16x2 b2 = __builtin_convertvector((f32x2{e[j], e[j + 1]}), bf16x2);
                pf[j] = b2[0];
                pf[j + 1] = b2[1];
            }
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
                o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[g16][db], pf, o[db], 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (i < 8) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
        }
        __builtin_amdgcn_s_setprio(0);
        step_barrier<2 * DMA_PER_STEP>();
    };

    if (t_begin < t_end) {
        if (tid == 0) sh_dropped = 0;        // before the first barrier
        f32x16 s_a, s_b;
        constexpr uint32_t VB = STAGES * TILE_B;
#pragma unroll
        for (int i = 0; i < 4; ++i) {        // K of four tiles, V of three
            const int t = in_list(t_begin + i);
            if (TWO_PAGES) at_k = place(t, entries(t));
            dma_tile(k_base, t, at_k, i * TILE_B);
            if (i < 3) dma_tile(v_base, t, at_k, VB + i * TILE_B);
        }
        if (TWO_PAGES) e_next = entries(in_list(t_begin + 4));
        step_barrier<0>();
        if (wave_active) {
            bf16x8 kf0[D / 16];
            load_k(0, kf0);
            qk(kf0, s_a);
        }
        step_barrier<0>();
        wait_vmem();                         // the Q fragments have landed, as the compiler sees it
        int t = t_begin;
        if (!wave_active) {
            for (; t < t_end; ++t) {         // the same loads into the same stages as the steps below
                const uint32_t i4 = (uint32_t)(t - t_begin) & 3u;
                if (TWO_PAGES) {
                    at_v = at_k;
                    at_k = place(in_list(t + 4), e_next);
                }
                dma_tile(k_base, in_list(t + 4), at_k, i4 * TILE_B);
                dma_tile(v_base, in_list(t + 3), at_v, VB + ((i4 + 3u) & 3u) * TILE_B);
                if (TWO_PAGES) e_next = entries(in_list(t + 5));
                step_barrier<2 * DMA_PER_STEP>();
            }
        }
        while (t < t_end) {
            step(t, s_a, s_b, IC<1>{}, IC<0>{}, IC<0>{}, IC<3>{});
            if (++t == t_end) break;
            step(t, s_b, s_a, IC<2>{}, IC<1>{}, IC<1>{}, IC<0>{});
            if (++t == t_end) break;
            step(t, s_a, s_b, IC<3>{}, IC<2>{}, IC<2>{}, IC<1>{});
            if (++t == t_end) break;
            step(t, s_b, s_a, IC<0>{}, IC<3>{}, IC<3>{}, IC<2>{});
            ++t;
        }
        wait_vmem();               // no load may still be writing LDS when the workgroup retires
    }

    // The values left out, for the rows that do see them: from memory, key by key.  (A step's last barrier is behind every write.)
    if (t_begin < t_end && sh_dropped != 0 && row_ok) {
        const float mr = (m_ref == -INFINITY) ? 0.f : m_ref;
        const bf16_t* qr = static_cast<const bf16_t*>(p.q) + q_row * D;
#pragma unroll 1
        for (int t = t_begin; t < t_end; ++t) {
            if (tiles.whole(t, 1)) continue;
            const bool pre = tiles.in_prefix(t);
            const int32_t* table = table_of(t);
#pragma unroll 1
            for (int key = tiles.key0(t); key < tiles.key0(t) + BN; ++key) {
                if (!(pre ? key < tiles.n_prefix : sees(p, pos, row_hi, key))) continue;
                const int slot = (int)quot((uint32_t)key, p.b.by_page);
                const int pg = clamped(table[slot], 0, p.b.n_pages - 1);
                const int64_t at = ((int64_t)pg * page + (key - slot * page)) * row_b;
                const bf16_t* kr = reinterpret_cast<const bf16_t*>(k_base + at);
                const bf16_t* vr = reinterpret_cast<const bf16_t*>(v_base + at);
                float s = 0.f;
#pragma unroll 1
                for (int d = 0; d < D; ++d) s = fmaf((float)kr[d], (float)qr[d], s);
                const float e = __builtin_amdgcn_exp2f(fmaf(s, sc, -mr));
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        const float v = (float)vr[db * 32 + (j >> 2) * 8 + hh * 4 + (j & 3)];
                        if (!(__builtin_fabsf(v) < INFINITY)) o[db][j] = fmaf(e, v, o[db][j]);
                    }
            }
        }
    }

    const float l_tot = pair_sum(l_part);
    if (!row_ok) return;
    if (a.n_slots == 1) {
        const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;      // a row that sees nothing: zeros
        bf16_t* orow = static_cast<bf16_t*>(p.out) + q_row * D;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int j4 = 0; j4 < 4; ++j4) {
                u32x2 w;
                w.x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{o[db][j4 * 4] * inv, o[db][j4 * 4 + 1] * inv}), bf16x2));
                w.y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{o[db][j4 * 4 + 2] * inv, o[db][j4 * 4 + 3] * inv}), bf16x2));
                *reinterpret_cast<u32x2*>(orow + db * 32 + j4 * 8 + hh * 4) = w;
            }
    } else {
        const int64_t at = (int64_t)job.slot * p.b.n_tokens * p.n_q_heads + q_row;
        if (l_tot != 0.f) {
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int j4 = 0; j4 < 4; ++j4)
                    *reinterpret_cast<f32x4*>(a.part_o + at * D + db * 32 + j4 * 8 + hh * 4) =
                        f32x4{o[db][j4 * 4], o[db][j4 * 4 + 1], o[db][j4 * 4 + 2], o[db][j4 * 4 + 3]};
        }
        if (hh == 0) *reinterpret_cast<f32x2*>(a.part_ml + at * 2) = f32x2{l_tot != 0.f ? m_ref : -INFINITY, l_tot};
    }
}

// Joins the partial results of the rows (token, head).  TPR threads own four dimensions each of a row; the slots of a row are
// spread over a.n_slots / per_group thread groups, whose sums meet in LDS, so that a few rows of many slots (one user) are not
// read one after the other.  Slots of no keys hold the maximum -inf and are not read.
constexpr int MERGE_THREADS = 256;
template <bool BF16>
__global__ __launch_bounds__(MERGE_THREADS) void attn_paged_merge_kernel(PagedArgs a, int tpr, int groups, int rows_per_block) {
    __shared__ float red_m[MERGE_THREADS], red_l[MERGE_THREADS];
    __shared__ f32x4 red_o[MERGE_THREADS];
    const PagedProblem& p = a.p;
    const int D = p.head_dim, tid = threadIdx.x;
    const int unit = tid / tpr, dq = tid - unit * tpr;           // (row of the block, group), dimensions 4 dq ..
    const int r = unit / groups, g = unit - r * groups;
    const int64_t n_rows = (int64_t)p.b.n_tokens * p.n_q_heads;
    const int64_t row = (int64_t)blockIdx.x * rows_per_block + r;
    const TokenRange range = token_range(p.b);
    const bool ok = r < rows_per_block && row >= (int64_t)range.first * p.n_q_heads && row < (int64_t)range.end * p.n_q_heads;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    if (ok) {
        constexpr int U = 4;
        for (int s0 = g; s0 < a.n_slots; s0 += U * groups) {
            f32x2 ml[U];
            f32x4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int s = s0 + u * groups;
                ml[u] = f32x2{-INFINITY, 0.f};
                v[u] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (s < a.n_slots) ml[u] = *reinterpret_cast<const f32x2*>(a.part_ml + ((int64_t)s * n_rows + row) * 2);
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (ml[u][0] != -INFINITY) v[u] = *reinterpret_cast<const f32x4*>(a.part_o + ((int64_t)(s0 + u * groups) * n_rows + row) * D + dq * 4);
            float m_new = m;
#pragma unroll
            for (int u = 0; u < U; ++u) m_new = fmaxf(m_new, ml[u][0]);
            const float ref = m_new == -INFINITY ? 0.f : m_new, f = __builtin_amdgcn_exp2f(m - ref);
            l *= f;
            acc *= f;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (ml[u][0] == -INFINITY) continue;
                const float w = __builtin_amdgcn_exp2f(ml[u][0] - ref);
                l += ml[u][1] * w;
                acc += v[u] * w;
            }
            m = m_new;
        }
    }
    if (groups > 1) {
        red_o[tid] = acc;
        red_m[tid] = m;
        red_l[tid] = l;
        __syncthreads();
        if (!ok || g != 0) return;
        float m_all = m;
        for (int i = 1; i < groups; ++i) m_all = fmaxf(m_all, red_m[tid + i * tpr]);
        const float ref = m_all == -INFINITY ? 0.f : m_all;
        acc = f32x4{0.f, 0.f, 0.f, 0.f};
        l = 0.f;
        for (int i = 0; i < groups; ++i) {
            if (red_m[tid + i * tpr] == -INFINITY) continue;
            const float w = __builtin_amdgcn_exp2f(red_m[tid + i * tpr] - ref);
            acc += red_o[tid + i * tpr] * w;
            l += red_l[tid + i * tpr] * w;
        }
    }
    if (!ok) return;
    acc *= l == 0.f ? 0.f : 1.f / l;
    if (BF16) {
        u32x2 w;
        w.x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{acc[0], acc[1]}), bf16x2));
        w.y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{acc[2], acc[3]}), bf16x2));
        *reinterpret_cast<u32x2*>(static_cast<bf16_t*>(p.out) + row * D + dq * 4) = w;
    } else {
        *reinterpret_cast<f32x4*>(static_cast<float*>(p.out) + row * D + dq * 4) = acc;
    }
}

// ---- fp32: plain vector-ALU code, one wavefront per row.  The keys a row sees are numbered through, first tokens, then window (or the
// prefix), and a split takes a run of them; 64 keys at a time each lane scores one, then the lanes own output dimensions.
constexpr int F32_ROWS = 4;
constexpr int MAX_D = 256;
__device__ inline float wave_max(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}
__device__ inline float wave_sum(float v) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o);
    return v;
}

__global__ __launch_bounds__(F32_ROWS * 64) void attn_paged_f32_kernel(PagedArgs a) {
    __shared__ float q_lds[F32_ROWS][MAX_D];
    __shared__ float p_lds[F32_ROWS][64];
    __shared__ int64_t at_lds[F32_ROWS][64];
    const PagedProblem& p = a.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int D = p.head_dim, G = p.n_q_heads / p.n_kv_heads;
    const int L = blockIdx.x / p.n_kv_heads, kvh = blockIdx.x - L * p.n_kv_heads;
    Job job;
    if (!find_job<F32_ROWS>(p, a.prefix_blocks, a.prefix_splits, a.blocks, a.splits, L, lane, &job)) return;
    const int row = job.row0 + wave;
    if (row >= job.n_rows) return;           // whole wavefront leaves; nothing below waits for the workgroup
    const int tok = row / G, pos = job.p0 + tok;
    const int64_t q_row = (int64_t)(job.token0 + tok) * p.n_q_heads + kvh * G + (row - tok * G);
    const float* q = static_cast<const float*>(p.q) + q_row * D;
    for (int d = lane; d < D; d += 64) q_lds[wave][d] = q[d];
    __builtin_amdgcn_wave_barrier();

    // key i of the row's list: prefix, first tokens, window
    int hi = 0, lo = 0, n_first = 0;
    if (job.own) {
        hi = clamped(pos + 1, 0, p.b.capacity);
        if (p.window >= 0) {
            lo = clamped(pos + 1 - p.window, 0, hi);
            n_first = p.sinks < lo ? p.sinks : lo;
        }
    }
    const int n_keys = job.n_prefix + n_first + (hi - lo);
    int per_split = (n_keys + job.n_splits - 1) / job.n_splits;
    per_split = per_split > a.min_tiles * BN ? per_split : a.min_tiles * BN;
    const int begin = job.split * per_split, end = begin + per_split < n_keys ? begin + per_split : n_keys;

    const int page = (int)p.b.by_page.d;
    float o[MAX_D / 64] = {0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    const float sc = p.scale * 1.4426950408889634f;
    for (int j0 = begin; j0 < end; j0 += 64) {
        int j = j0 + lane;
        float s = -INFINITY;
        if (j < end) {
            const bool pre = j < job.n_prefix;
            const int32_t* table = pre ? p.prefix_pages : job.table;
            if (!pre) {
                j -= job.n_prefix;
                if (j >= n_first) j += lo - n_first;
            }
            const int slot = (int)quot((uint32_t)j, p.b.by_page);
            const int64_t at = (((int64_t)clamped(table[slot], 0, p.b.n_pages - 1) * page + (j - slot * page)) * p.n_kv_heads + kvh) * D;
            at_lds[wave][lane] = at;
            const float* k = static_cast<const float*>(p.b.k_pages) + at;
            float acc = 0.f;
            for (int d = 0; d < D; d += 4) {
                const f32x4 x = *reinterpret_cast<const f32x4*>(k + d);
#pragma unroll
                for (int i = 0; i < 4; ++i) acc = fmaf(x[i], q_lds[wave][d + i], acc);
            }
            s = acc * sc;
        }
        const float m_new = fmaxf(m, wave_max(s)), ref = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m - ref);
        const float e = j0 + lane < end ? __builtin_amdgcn_exp2f(s - ref) : 0.f;
        l = l * alpha + wave_sum(e);
        m = m_new;
        p_lds[wave][lane] = e;
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < MAX_D / 64; ++i) o[i] *= alpha;
        const int n = end - j0 < 64 ? end - j0 : 64;
        for (int jj = 0; jj < n; ++jj) {
            const float* v = static_cast<const float*>(p.b.v_pages) + at_lds[wave][jj];
            const float e_j = p_lds[wave][jj];
#pragma unroll
            for (int i = 0; i < MAX_D / 64; ++i)
                if (lane + 64 * i < D) o[i] = fmaf(e_j, v[lane + 64 * i], o[i]);
        }
        __builtin_amdgcn_wave_barrier();
    }
    const int64_t at = (int64_t)job.slot * p.b.n_tokens * p.n_q_heads + q_row;
    const float inv = a.n_slots > 1 ? 1.f : l == 0.f ? 0.f : 1.f / l;
    float* out = a.n_slots > 1 ? a.part_o + at * D : static_cast<float*>(p.out) + q_row * D;
#pragma unroll
    for (int i = 0; i < MAX_D / 64; ++i)
        if (lane + 64 * i < D) out[lane + 64 * i] = o[i] * inv;
    if (a.n_slots > 1 && lane == 0) *reinterpret_cast<f32x2*>(a.part_ml + at * 2) = f32x2{l != 0.f ? m : -INFINITY, l};
}

int64_t up(int64_t n, int64_t d) { return (n + d - 1) / d; }

}  // namespace

PagedPlan attn_paged_plan(int dtype, int n_q_heads, int n_kv_heads, int head_dim, int64_t n_tokens, int64_t n_seqs, int64_t max_kv,
                          int64_t window, int64_t sinks, int64_t n_prefix) {
    const int64_t G = n_q_heads / n_kv_heads;
    PagedPlan plan;
    plan.rows = dtype == REKV_BF16 ? BM : F32_ROWS;
    plan.blocks = (int32_t)(n_tokens * G / plan.rows + n_seqs);
    plan.min_tiles = 4;
    const int64_t places = dtype == REKV_BF16 ? 512 : 1024;
    auto splits_of = [&](int64_t blocks, int64_t keys) {
        const int64_t most = keys / (BN * plan.min_tiles) > 1 ? keys / (BN * plan.min_tiles) : 1, s = places / (blocks * n_kv_heads);
        return (int32_t)(s < 1 ? 1 : s < most ? s : most);
    };
    plan.prefix_blocks = plan.prefix_splits = 0;
    int64_t keys = window < 0 || window + sinks > max_kv ? max_kv : window + sinks;
    // Rows that fill blocks by themselves walk the prefix in their own blocks.
    const bool together = n_prefix > 0 && n_tokens * G < n_seqs * (plan.rows / 2);
    if (together) {
        plan.prefix_blocks = (int32_t)up(n_tokens * G, plan.rows);
        plan.prefix_splits = splits_of(plan.prefix_blocks, n_prefix);
    } else {
        keys += n_prefix;
    }
    plan.splits = splits_of(plan.blocks, keys);
    plan.workspace_bytes = plan.slots() > 1 ? n_tokens * n_q_heads * plan.slots() * (head_dim + 2) * 4 : 0;
    return plan;
}

hipError_t attn_paged_launch(const PagedProblem& p, const PagedPlan& plan, int dtype, void* workspace, hipStream_t stream) {
    PagedArgs a;
    a.p = p;
    a.prefix_blocks = plan.prefix_blocks; a.prefix_splits = plan.prefix_splits;
    a.blocks = plan.blocks; a.splits = plan.splits; a.min_tiles = plan.min_tiles;
    a.n_slots = plan.slots();
    const int64_t rows = (int64_t)p.b.n_tokens * p.n_q_heads;
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = a.n_slots > 1 ? a.part_o + rows * a.n_slots * p.head_dim : nullptr;
    const int64_t jobs = (int64_t)plan.prefix_blocks * plan.prefix_splits + (int64_t)plan.blocks * plan.splits;
    const dim3 grid((unsigned)(jobs * p.n_kv_heads));
    const uint32_t page = p.b.by_page.d;
    const bool two = page >= BN || page == 16;
    if (dtype == REKV_F32)
        hipLaunchKernelGGL(attn_paged_f32_kernel, grid, dim3(F32_ROWS * 64), 0, stream, a);
    else if (p.head_dim == 128 && two)
        hipLaunchKernelGGL((attn_paged_kernel<128, true>), grid, dim3(WAVES * 64), 0, stream, a);
    else if (p.head_dim == 128)
        hipLaunchKernelGGL((attn_paged_kernel<128, false>), grid, dim3(WAVES * 64), 0, stream, a);
    else if (two)
        hipLaunchKernelGGL((attn_paged_kernel<64, true>), grid, dim3(WAVES * 64), 0, stream, a);
    else
        hipLaunchKernelGGL((attn_paged_kernel<64, false>), grid, dim3(WAVES * 64), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.n_slots == 1) return e;
    const int tpr = p.head_dim / 4, units = MERGE_THREADS / tpr;
    int groups = 1;                           // of at most four slots each, as far as a block has threads
    while (groups * 2 <= units && groups * 4 < a.n_slots) groups *= 2;
    const int per_block = units / groups;
    const dim3 merge_grid((unsigned)up(rows, per_block));
    if (dtype == REKV_F32)
        hipLaunchKernelGGL(attn_paged_merge_kernel<false>, merge_grid, dim3(MERGE_THREADS), 0, stream, a, tpr, groups, per_block);
    else
        hipLaunchKernelGGL(attn_paged_merge_kernel<true>, merge_grid, dim3(MERGE_THREADS), 0, stream, a, tpr, groups, per_block);
    return hipGetLastError();
}

}  // namespace rekv
