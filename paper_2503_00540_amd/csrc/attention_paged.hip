// Attention of a ragged batch over a paged cache: sliding windows with first tokens that stay visible, and batches that share a
// long prefix.
//
//   o = sum_j e^(s_j - m) v_j / sum_j e^(s_j - m),  s_j = scale q.k_j,  over the keys j a token sees (paged.h)
//
// in one pass with a running maximum m and sum in fp32; probabilities are rounded to bf16 for the second product (their
// sum is taken before), which adds to an output's own rounding about as much again.  Where the keys of a row are split over workgroups,
// or between a prefix and the row's own keys, each part leaves (m, sum, O) in fp32 and a second launch joins them.
//
// Rows are stacked as in attention_bf16.hip, the G query heads of a KV head token by token, so a K/V tile in LDS
// serves them all; a long prefix shared by the batch is walked by blocks of all sequences' rows, so that one user's few rows do
// not read it for themselves (a short one they do, which saves the second launch).  Operand layouts, the four LDS stages per tensor and the order of a step are those of attention_bf16.hip.
// What differs is where tiles come from: 32 keys lie in one or two pages, and the places of 64 tiles are worked out at once.
//
// What bounds it (28/4/128, pages of 64 to 256 unless said).  Long prompts: the matrix cores at the clock the chip grants them,
// 1.02 to 1.07 PFLOP/s for 8,192 tokens (451 to 473 us; a library GEMM of 8,192^3 reaches 1.24), as attention_bf16.hip.  Many users' decode
// steps: HBM, 5.5 TB/s for 64 users of 1 to 8,192 tokens at 64/8/128 (199 us), 6.1 where all have 4,096.  One user's: round trips; a
// workgroup of a 15,000-token window spends (us) 0.4 on finding its sequence, 1.3 on the page table, 0.8 to the first tile, 3.0 on two tiles
// per wavefront and 1.2 on the merge in LDS, the joining launch 3.9, 15.7 in all.  A live frame over 3,136 keys: 0.8, 0.8 and 3.4 to the
// first tiles, 0.97 per tile with two workgroups per CU (0.67 with one), 1.8 to write.
#include <float.h>

#include "attention_mfma.h"
#include "paged.h"

namespace rekv {
namespace {

constexpr int WAVES = 4;
constexpr int THREADS = WAVES * 64;
constexpr int WM = 32;                // rows of a wavefront
constexpr int BM = WAVES * WM;        // rows of a block whose wavefronts share the tiles
constexpr int STAGES = 4;             // of such a block, per tensor
enum { ROW_BLOCKS, KEY_BLOCKS, STREAMED };

struct PagedArgs {
    PagedProblem p;
    int32_t prefix_blocks, prefix_splits, blocks, splits, min_tiles, min_prefix_tiles, n_slots;
    float* part_o;        // [slot][token * Hq + head][D]
    float* part_ml;       // [slot][token * Hq + head][2]: maximum (of base-2 exponents), sum
};

// As dma16 (attention_mfma.h), from a 64-bit address per lane.
__device__ inline void dma16_at(uint64_t addr, uint32_t lds_addr) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
                 ::"v"(addr), "s"(__builtin_amdgcn_readfirstlane(lds_addr)) : "memory", "m0");
}

// Where a tile lies.  Pages of 32 tokens or more, or of 16 (TWO_PAGES): the cache's row (page * page_size + row) that the tile's
// row 0 is in its first page and would be in its next, and how many rows lie in the first (32: all).  Smaller pages: every
// lane's row.  whole: all rows of the block see the tile whole.
struct Place {
    int a, b, rows_a;
    bool whole;
};
// The places of 64 tiles from t0 on, one per lane.  Worked out at once, with one wait for the page table, they cost a step two or
// three lane reads, where following the list step by step cost it about 80 scalar instructions.
struct Places {
    int t0, a, b, rows_whole;
};

// A block's tiles and their way into LDS, by LOADERS wavefronts together.
template <int D, bool TWO_PAGES, int LOADERS, bool STREAM>
struct Source {
    static constexpr int CH = D / 8;                       // 16-byte chunks per key row
    static constexpr int RPI = 64 / CH;                    // key rows one 1 KB wave-wide load covers
    static constexpr int N_DMA = BN / RPI / LOADERS;       // such loads per wave, tile and tensor
    static constexpr int N_OFF = N_DMA < 16 / RPI ? N_DMA : 16 / RPI;      // the swizzle repeats every 16 rows
    static constexpr uint32_t TILE_B = BN * D * 2;         // bytes of a tile

    const PagedProblem& p;
    const Job& job;
    const Tiles<BN>& tiles;
    int t_end, lane, loader;
    const char *k_base, *v_base;
    uint32_t row_b;                                        // bytes of a token's keys
    int first_row;                                         // of this lane
    uint32_t off[N_OFF];                                   // byte offset in a whole tile of what load j fetches

    __device__ Source(const PagedProblem& p_, const Job& job_, const Tiles<BN>& tiles_, int t_end_, int kvh, int lane_, int loader_)
        : p(p_), job(job_), tiles(tiles_), t_end(t_end_), lane(lane_), loader(loader_) {
        row_b = (uint32_t)p.n_kv_heads * D * 2u;
        k_base = static_cast<const char*>(p.b.k_pages) + kvh * D * 2;
        v_base = static_cast<const char*>(p.b.v_pages) + kvh * D * 2;
        first_row = loader * N_DMA * RPI + lane / CH;
#pragma unroll
        for (int j = 0; j < N_OFF; ++j) off[j] = (uint32_t)(first_row + j * RPI) * row_b + chunk(first_row + j * RPI);
    }
    __device__ uint32_t chunk(int row) const { return (uint32_t)((lane % CH) ^ swz<D>(row)) * 16u; }
    __device__ int in_list(int t) const { return t < t_end ? t : t_end - 1; }

    __device__ __attribute__((always_inline)) void fill(Places& at, int t0) const {
        at.t0 = t0;
        if (!TWO_PAGES) return;
        const int t = in_list(t0 + lane), page = (int)p.b.by_page.d, k0 = tiles.key0(t);
        const bool pre = tiles.in_prefix(t);
        const int32_t* table = pre ? p.prefix_pages : job.table;
        const int last = pre ? (int)quot((uint32_t)(tiles.n_prefix - 1), p.b.by_page) : p.b.max_pages - 1;
        const int slot = (int)quot((uint32_t)k0, p.b.by_page), within = k0 - slot * page;
        const int a = clamped(table[slot], 0, p.b.n_pages - 1), b = clamped(table[slot < last ? slot + 1 : last], 0, p.b.n_pages - 1);
        const int rows_a = page - within < BN ? page - within : BN;
        at.a = a * page + within;
        at.b = b * page + within - page;
        at.rows_whole = rows_a * 2 + tiles.whole(t);
    }
    // Of tile t; the 64 tiles move on where it is behind them.
    __device__ __attribute__((always_inline)) Place place(Places& from, int t) const {
        Place at;
        if (t - from.t0 >= 64) fill(from, t);
        if (TWO_PAGES) {
            const int i = t - from.t0, rw = __builtin_amdgcn_readlane(from.rows_whole, i);
            at.a = __builtin_amdgcn_readlane(from.a, i);
            at.b = __builtin_amdgcn_readlane(from.b, i);
            at.rows_a = rw >> 1;
            at.whole = rw & 1;
        } else {
            at.whole = tiles.whole(t);
            int r0, r1;
            tiles.rows(t, &r0, &r1);
            const int k0 = tiles.key0(t), page = (int)p.b.by_page.d;
            const int32_t* table = tiles.in_prefix(t) ? p.prefix_pages : job.table;
            if (LOADERS > 1) {               // eight rows of this wavefront: lane i (of eight) gets the place of row i
                const int base = loader * N_DMA * RPI;
                static_assert(LOADERS == 1 || N_DMA * RPI == 8, "below");
                at.a = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) {      // through the scalar cache: waiting for it does not wait for tile loads
                    const int key = k0 + clamped(base + i, r0, r1), slot = (int)quot((uint32_t)key, p.b.by_page);
                    const int row = clamped(scalar_word(table, slot), 0, p.b.n_pages - 1) * page + (key - slot * page);
                    at.a = (lane & 7) == i ? row : at.a;
                }
            } else {
                const int key = k0 + clamped(lane & 31, r0, r1), slot = (int)quot((uint32_t)key, p.b.by_page);
                at.a = clamped(table[slot], 0, p.b.n_pages - 1) * page + (key - slot * page);
            }
        }
        return at;
    }
    // This wavefront's share of a tile.  Rows that no row of the block sees repeat the nearest that one does.
    __device__ __attribute__((always_inline)) void fetch(const char* base, int t, const Place& at, uint32_t dst) const {
        dst += (uint32_t)(loader * N_DMA) * 1024u;
        if (!TWO_PAGES) {
#pragma unroll
            for (int j = 0; j < N_DMA; ++j) {
                const int r = first_row + j * RPI, row = __shfl(at.a, LOADERS > 1 ? r & 7 : r);
                dma16_at(reinterpret_cast<uint64_t>(base) + (uint64_t)(uint32_t)row * row_b + chunk(r), dst + j * 1024u);
            }
            return;
        }
        const char* in_a = base + (int64_t)at.a * row_b;
        if (at.whole && at.rows_a >= BN) {
#pragma unroll
            for (int j = 0; j < N_DMA; ++j) dma16<STREAM>(in_a + (uint32_t)(j / N_OFF * 16) * row_b, off[j % N_OFF], dst + j * 1024u);
            return;
        }
        // Lanes of either page take a load of their own, from a uniform address.  Where a load has lanes of both, one more is in
        // flight than is counted, which only makes a wait longer.
        const char* in_b = base + (int64_t)at.b * row_b;
        auto row_of = [&](int r, uint32_t o, uint32_t to) __attribute__((always_inline)) {
            if (r < at.rows_a) dma16<STREAM>(in_a, o, to);
            else dma16<STREAM>(in_b, o, to);
        };
        if (at.whole) {
#pragma unroll
            for (int j = 0; j < N_DMA; ++j) {
                const int first = (loader * N_DMA + j) * RPI;                      // of the load's rows
                const uint32_t on = (uint32_t)(j / N_OFF * 16) * row_b, to = dst + j * 1024u;
                if (first + RPI <= at.rows_a) dma16<STREAM>(in_a + on, off[j % N_OFF], to);
                else if (first >= at.rows_a) dma16<STREAM>(in_b + on, off[j % N_OFF], to);
                else row_of(first_row + j * RPI, off[j % N_OFF] + on, to);
            }
            return;
        }
        int r0, r1;
        tiles.rows(t, &r0, &r1);
#pragma unroll 1
        for (int j = 0; j < N_DMA; ++j) {
            const int r = clamped(first_row + j * RPI, r0, r1);
            row_of(r, (uint32_t)r * row_b + chunk(first_row + j * RPI), dst + j * 1024u);
        }
    }
};

// Operand addresses in LDS, for a K tile at k0 and a V tile at v0 (see attention_bf16.hip).
template <int D>
struct Operands {
    uint32_t k[D / 16], v[2][D / 32];
    __device__ Operands(uint32_t k0, uint32_t v0, int lane) {
        const int col = lane & 31, hh = lane >> 5;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) k[ks] = k0 + (uint32_t)(col * D + (((ks * 2 + hh) ^ swz<D>(col)) * 8)) * 2u;
        const int gq = lane >> 4, i16 = lane & 15, qd = i16 & 3, jk = i16 >> 2;
        const int cl = (gq & 1) * 2 + (qd >> 1), half = qd & 1;
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            const int keyl = r * 8 + hh * 4 + jk;
#pragma unroll
            for (int db = 0; db < D / 32; ++db) v[r][db] = v0 + (uint32_t)(keyl * D + (((db * 4 + cl) ^ swz<D>(keyl)) * 8) + half * 4) * 2u;
        }
    }
    __device__ void load_k(uint32_t stage_b, bf16x8 (&kf)[D / 16]) const {
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) kf[ks] = *reinterpret_cast<LDS_AS const bf16x8*>(k[ks] + stage_b);
    }
    __device__ void load_v(uint32_t stage_b, int g16, bf16x8 (&vf)[D / 32]) const {
#pragma unroll
        for (int db = 0; db < D / 32; ++db) {
            const tr4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(reinterpret_cast<LDS_AS tr4_t*>(v[0][db] + stage_b + g16 * 16 * D * 2));
            const tr4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16(reinterpret_cast<LDS_AS tr4_t*>(v[1][db] + stage_b + g16 * 16 * D * 2));
            vf[db] = __builtin_shufflevector(__builtin_bit_cast(bf16x4, lo), __builtin_bit_cast(bf16x4, hi), 0, 1, 2, 3, 4, 5, 6, 7);
        }
    }
};

// A wavefront's 32 rows (a query per lane pair): the running softmax and output.
template <int D>
struct Rows {
    bf16x8 qf[D / 16];
    f32x16 o[D / 32];
    float m_ref, l, sc;
    int pos;                // index of this row's token
    bool ok;
    int64_t q_row;          // over (token, head)

    __device__ Rows(const PagedProblem& p, const Job& job, int row, int kvh, int G, int hh) {
        ok = row < job.n_rows;
        const int tok = row / G;
        pos = job.p0 + tok;
        sc = p.scale * 1.4426950408889634f;
        m_ref = -INFINITY;
        l = 0.f;
        q_row = (int64_t)(job.token0 + tok) * p.n_q_heads + kvh * G + (row - tok * G);
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) {
            u32x4 v = {0u, 0u, 0u, 0u};
            if (ok) v = *reinterpret_cast<const u32x4*>(static_cast<const bf16_t*>(p.q) + q_row * D + ks * 16 + hh * 8);
            qf[ks] = __builtin_bit_cast(bf16x8, v);
        }
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    }
    __device__ __attribute__((always_inline)) void qk(const bf16x8 (&kf)[D / 16], f32x16& s) const {
#pragma unroll
        for (int j = 0; j < 16; ++j) s[j] = 0.f;
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[ks], qf[ks], s, 0, 0, 0);
    }
    __device__ __attribute__((always_inline)) void mask(const PagedProblem& p, const Tiles<BN>& tiles, int t, int hh, f32x16& s) const {
        const int k0 = tiles.key0(t) + hh * 4;
        const Seen sees = tiles.in_prefix(t) ? Seen{0, tiles.n_prefix, 0} : seen_by(p, pos);
#pragma unroll
        for (int j = 0; j < 16; ++j) s[j] = sees(k0 + (j >> 2) * 8 + (j & 3)) ? s[j] : -INFINITY;
    }
    // The running maximum over a tile's scores (lazily: O is rescaled when it has moved by more than 2^8); returns what the
    // exponents refer to.
    __device__ __attribute__((always_inline)) float maximum(const f32x16& s) {
        float mx = s[0];
#pragma unroll
        for (int j = 1; j < 16; ++j) mx = fmaxf(mx, s[j]);
        mx = pair_max(mx);
        const float mt2 = mx * sc;
        if (__builtin_amdgcn_ballot_w64(mt2 > m_ref + RESCALE_GAP) != 0) {
            const float m_new = fmaxf(m_ref, mt2);
            const float alpha = (m_new == -INFINITY) ? 1.f : __builtin_amdgcn_exp2f(m_ref - m_new);
            l *= alpha;
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
#pragma unroll
                for (int j = 0; j < 16; ++j) o[i][j] *= alpha;
            m_ref = m_new;
        }
        return (m_ref == -INFINITY) ? 0.f : m_ref;
    }
    // Half a tile's probabilities, summed and rounded to bf16 for the product with V.
    __device__ __attribute__((always_inline)) bf16x8 probabilities(const f32x16& s, int g16, float mr) {
        bf16x8 pf;
        float e[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            e[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[g16 * 8 + j], sc, -mr));
            l += e[j];
        }
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const bf16x2 b2 = __builtin_convertvector((f32x2{e[j], e[j + 1]}), bf16x2);
            pf[j] = b2[0];
            pf[j + 1] = b2[1];
        }
        return pf;
    }
    __device__ __attribute__((always_inline)) void pv(const bf16x8 (&vf)[D / 32], const bf16x8& pf) {
#pragma unroll
        for (int db = 0; db < D / 32; ++db) o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[db], pf, o[db], 0, 0, 0);
    }

    // A row whose scores are all -infinity has the sum 0, and its output is 0 whatever its values are: an infinity or a NaN among them has
    // made the products with probabilities of 0 NaN.
    __device__ __attribute__((always_inline)) void clear_empty(float l_tot) {
        if (l_tot != 0.f) return;
#pragma unroll
        for (int i = 0; i < D / 32; ++i)
#pragma unroll
            for (int j = 0; j < 16; ++j) o[i][j] = 0.f;
    }

    // The values that drop_nonfinite took out of tiles [t0, t1), for the rows that do see them: from memory, key by key.
    __device__ __attribute__((always_inline)) void add_nonfinite(const PagedProblem& p, const Job& job, const Tiles<BN>& tiles, int t0, int t1,
                                                                 int kvh, int hh) {
        if (!ok) return;
        const float mr = (m_ref == -INFINITY) ? 0.f : m_ref;
        const int page = (int)p.b.by_page.d;
        const bf16_t* qr = static_cast<const bf16_t*>(p.q) + q_row * D;
#pragma unroll 1
        for (int t = t0; t < t1; ++t) {
            if (tiles.whole(t)) continue;
            const bool pre = tiles.in_prefix(t);
            const int32_t* table = pre ? p.prefix_pages : job.table;
            const Seen sees = pre ? Seen{0, tiles.n_prefix, 0} : seen_by(p, pos);
#pragma unroll 1
            for (int key = tiles.key0(t); key < tiles.key0(t) + BN; ++key) {
                if (!sees(key)) continue;
                const int slot = (int)quot((uint32_t)key, p.b.by_page);
                const int64_t row = (int64_t)clamped(table[slot], 0, p.b.n_pages - 1) * page + (key - slot * page);
                const int64_t at = (row * p.n_kv_heads + kvh) * D;
                const bf16_t* kr = static_cast<const bf16_t*>(p.b.k_pages) + at;
                const bf16_t* vr = static_cast<const bf16_t*>(p.b.v_pages) + at;
                float s = 0.f;
#pragma unroll 1
                for (int d = 0; d < D; ++d) s = fmaf((float)kr[d], (float)qr[d], s);
                const float e = __builtin_amdgcn_exp2f(fmaf(s, sc, -mr));
#pragma unroll
                for (int db = 0; db < D / 32; ++db)
#pragma unroll
                    for (int j = 0; j < 16; j += 4) {
                        const bf16x4 v = *reinterpret_cast<const bf16x4*>(vr + db * 32 + j * 2 + hh * 4);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float x = (float)v[i];
                            o[db][j + i] = fmaf(e, __builtin_fabsf(x) < INFINITY ? 0.f : x, o[db][j + i]);
                        }
                    }
            }
        }
    }
};

// A tile that not every row sees whole: probabilities of 0 keep a value out only if it is finite, so the V tile's infinities and NaNs
// become 0 in LDS.  Every wavefront that reads the tile calls this itself, before it reads; true if it found any.
template <int D>
__device__ inline bool drop_nonfinite(uint32_t v_tile, int lane) {
    constexpr uint32_t TILE_B = BN * D * 2;
    const uint32_t at = v_tile + lane * 16u;
    uint32_t any = 0;
#pragma unroll
    for (uint32_t i = 0; i < TILE_B; i += 1024) {
        const u32x4 w = *reinterpret_cast<LDS_AS const u32x4*>(at + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) any |= (w[k] & 0x7f807f80u) + 0x00800080u;      // bit 15 of a half: its exponent is all ones
    }
    if (__builtin_amdgcn_ballot_w64((any & 0x80008000u) != 0) == 0) return false;
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
    return true;
}

// What a partial result's exponents refer to: -inf where it has no keys, and only there.  Scores that are all NaN leave a NaN sum under
// no maximum, which must not pass for none.
__device__ inline float part_max(float m, float l) { return l == 0.f ? -INFINITY : fmaxf(m, -FLT_MAX); }

// The tiles [begin, end) of split `job.split`; `runs` wavefronts divide them.
__device__ inline void split_range(const PagedArgs& a, const Job& job, int n_tiles, int runs, int* begin, int* end) {
    int n = (n_tiles + job.n_splits - 1) / job.n_splits;
    const int least = job.own ? a.min_tiles : a.min_prefix_tiles;
    n = n > least ? n : least;
    n = (n + runs - 1) / runs * runs;
    *begin = job.split * n;
    *end = *begin + n < n_tiles ? *begin + n : n_tiles;
}
template <int ROWS>
__device__ inline Tiles<BN> tiles_of(const PagedProblem& p, const Job& job, int G) {
    const int n_tok = job.n_rows / G, last = (job.row0 + ROWS - 1) / G;
    return Tiles<BN>(p, job, job.row0 / G, last < n_tok ? last : n_tok - 1);
}

__device__ inline void store4(bf16_t* to, f32x4 v) {
    u32x2 w;
    w.x = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{v[0], v[1]}), bf16x2));
    w.y = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{v[2], v[3]}), bf16x2));
    *reinterpret_cast<u32x2*>(to) = w;
}

template <int N>
__device__ inline void step_barrier() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
    __builtin_amdgcn_sched_barrier(0);
}

// A block of 128 rows: its four wavefronts share the tiles.  Order of a step, stages and operand reads as in attention_bf16.hip.
template <int D, bool TWO_PAGES>
__device__ __attribute__((always_inline)) void rows_block(const PagedArgs& a, const Job& job, int kvh, uint32_t lds0, int* sh_dropped) {
    typedef Source<D, TWO_PAGES, WAVES, false> Src;
    constexpr uint32_t TILE_B = Src::TILE_B, VB = STAGES * TILE_B;
    const PagedProblem& p = a.p;
    const int tid = threadIdx.x, lane = tid & 63, hh = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = p.n_q_heads / p.n_kv_heads;
    const bool wave_active = job.row0 + wave * WM < job.n_rows;
    const Tiles<BN> tiles = tiles_of<BM>(p, job, G);
    int t_begin, t_end;
    split_range(a, job, tiles.n, 1, &t_begin, &t_end);
    const Src src(p, job, tiles, t_end, kvh, lane, wave);
    Places places;
    if (t_begin < t_end) src.fill(places, t_begin);      // (before the queries' loads, whose wait this one would be otherwise)
    const Operands<D> at(lds0, lds0 + VB, lane);
    Rows<D> r(p, job, job.row0 + wave * WM + (lane & 31), kvh, G, hh);

    Place at_k, at_v;                        // of tiles t + 4 and t + 3 in step t
    uint32_t whole = 0;                      // bit i: all rows see tile t + i whole
    auto fetch = [&](int t, uint32_t kl, uint32_t vl) __attribute__((always_inline)) {      // the loads of step t
        at_v = at_k;
        at_k = src.place(places, src.in_list(t + 4));
        src.fetch(src.k_base, src.in_list(t + 4), at_k, lds0 + kl);
        src.fetch(src.v_base, src.in_list(t + 3), at_v, lds0 + VB + vl);
    };
    constexpr int DMA_PER_STEP = 2 * Src::N_DMA;
    auto step = [&](int t, f32x16& s_cur, f32x16& s_next, auto kn, auto kl, auto vc, auto vl) __attribute__((always_inline)) {
        constexpr uint32_t KN = decltype(kn)::value * TILE_B, KL = decltype(kl)::value * TILE_B;
        constexpr uint32_t VC = decltype(vc)::value * TILE_B, VL = decltype(vl)::value * TILE_B;
        fetch(t, KL, VL);
        if (!(whole & 1)) {
            r.mask(p, tiles, t, hh, s_cur);
            if (drop_nonfinite<D>(lds0 + VB + VC, lane)) *sh_dropped = 1;
        }
        whole = (whole >> 1) | ((uint32_t)at_k.whole << 3);
        bf16x8 kf[D / 16], vf[2][D / 32];
        at.load_k(KN, kf);
        at.load_v(VC, 0, vf[0]);
        __builtin_amdgcn_sched_barrier(0);
        const float mr = r.maximum(s_cur);
        __builtin_amdgcn_s_setprio(3);
        r.qk(kf, s_next);            // past the last tile this works on a stale stage and is unused
        at.load_v(VC, 1, vf[1]);
#pragma unroll
        for (int g16 = 0; g16 < 2; ++g16) r.pv(vf[g16], r.probabilities(s_cur, g16, mr));
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
        if (tid == 0) *sh_dropped = 0;       // before the first barrier
        f32x16 s_a, s_b;
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {        // K of four tiles, V of three
            const int t = src.in_list(t_begin + i);
            at_k = src.place(places, t);
            whole |= (uint32_t)at_k.whole << i;
            src.fetch(src.k_base, t, at_k, lds0 + i * TILE_B);
            if (i < 3) src.fetch(src.v_base, t, at_k, lds0 + VB + i * TILE_B);
        }
        step_barrier<0>();
        if (wave_active) {
            bf16x8 kf0[D / 16];
            at.load_k(0, kf0);
            r.qk(kf0, s_a);
        }
        step_barrier<0>();
        wait_vmem();                         // the Q fragments have landed, as the compiler sees it
        int t = t_begin;
        if (!wave_active) {
            for (; t < t_end; ++t) {         // the same loads into the same stages as the steps below
                const uint32_t i4 = (uint32_t)(t - t_begin) & 3u;
                fetch(t, i4 * TILE_B, ((i4 + 3u) & 3u) * TILE_B);
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
        // (a step's last barrier is behind every write of the flag)
        if (*sh_dropped != 0) r.add_nonfinite(p, job, tiles, t_begin, t_end, kvh, hh);
    }

    const float l_tot = pair_sum(r.l);
    if (!r.ok) return;
    r.clear_empty(l_tot);
    if (a.n_slots == 1) {
        const float inv = l_tot == 0.f ? 0.f : 1.f / l_tot;      // a row that sees nothing: zeros
        bf16_t* out = static_cast<bf16_t*>(p.out) + r.q_row * D + hh * 4;
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int j = 0; j < 16; j += 4)
                store4(out + db * 32 + j * 2, f32x4{r.o[db][j] * inv, r.o[db][j + 1] * inv, r.o[db][j + 2] * inv, r.o[db][j + 3] * inv});
    } else {
        const int64_t to = (int64_t)job.slot * p.b.n_tokens * p.n_q_heads + r.q_row;
        float* out = a.part_o + to * D + hh * 4;
        if (l_tot != 0.f) {
#pragma unroll
            for (int db = 0; db < D / 32; ++db)
#pragma unroll
                for (int j = 0; j < 16; j += 4)
                    *reinterpret_cast<f32x4*>(out + db * 32 + j * 2) = f32x4{r.o[db][j], r.o[db][j + 1], r.o[db][j + 2], r.o[db][j + 3]};
        }
        if (hh == 0) *reinterpret_cast<f32x2*>(a.part_ml + to * 2) = f32x2{part_max(r.m_ref, l_tot), l_tot};
    }
}

// A block of 32 rows, as a decode step's: its four wavefronts divide the KEYS, each walks its run of tiles through a K and a V tile
// of its own in LDS without a barrier, and their results meet in LDS.  STREAM: non-temporal loads, where nobody else reads the keys (64
// users' decode step 201 us so, 224 with cached loads; a live frame over 3,136 keys, which 43 blocks read, 40 and 31).  Pages below 32
// tokens other than 16, whose rows are fetched by 64-bit addresses, have cached loads only.
template <int D, bool TWO_PAGES, bool STREAM>
__device__ __attribute__((always_inline)) void keys_block(const PagedArgs& a, const Job& job, int kvh, unsigned char* lds, f32x2 (*ml)[WM]) {
    typedef Source<D, TWO_PAGES, 1, STREAM> Src;
    constexpr uint32_t TILE_B = Src::TILE_B;
    constexpr int N_DMA = Src::N_DMA, CPR = D / 4;       // 16-byte fp32 chunks per output row
    const PagedProblem& p = a.p;
    const int tid = threadIdx.x, lane = tid & 63, hh = lane >> 5, col = lane & 31;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int G = p.n_q_heads / p.n_kv_heads;
    const Tiles<BN> tiles = tiles_of<WM>(p, job, G);
    int begin, end;
    split_range(a, job, tiles.n, WAVES, &begin, &end);
    const int n = end > begin ? end - begin : 0, each = n / WAVES, rest = n - each * WAVES;      // the first `rest` runs are one longer
    const int t_begin = begin + each * wave + (wave < rest ? wave : rest), t_end = t_begin + each + (wave < rest);
    const uint32_t k_tile = lds_addr_of(lds) + (uint32_t)wave * 2u * TILE_B, v_tile = k_tile + TILE_B;
    const Src src(p, job, tiles, t_end, kvh, lane, 0);
    Places places;
    Place now, next;                         // of tiles t and t + 1
    if (t_begin < t_end) {                   // the first tile's loads leave before anything else is set up
        src.fill(places, t_begin);
        now = src.place(places, t_begin);
        src.fetch(src.k_base, t_begin, now, k_tile);
        src.fetch(src.v_base, t_begin, now, v_tile);
        next = src.place(places, src.in_list(t_begin + 1));
    }
    Rows<D> r(p, job, job.row0 + col, kvh, G, hh);
    const Operands<D> at(k_tile, v_tile, lane);
    wait_vmem();                             // the Q fragments have landed, as the compiler sees it
    bool dropped = false;
    auto reads_done = [] {                   // operands are in registers: their tile may be overwritten
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    auto wait_newest = [](auto k) { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(decltype(k)::value) : "memory"); };
    for (int t = t_begin; t < t_end; ++t) {
        const bool more = t + 1 < t_end;
        wait_newest(IC<N_DMA>{});            // K(t); V(t)'s loads are the only newer ones
        bf16x8 kf[D / 16], vf[2][D / 32];
        f32x16 s;
        at.load_k(0, kf);
        reads_done();
        if (more) src.fetch(src.k_base, t + 1, next, k_tile);
        r.qk(kf, s);
        const bool whole = now.whole;
        if (!whole) r.mask(p, tiles, t, hh, s);
        const float mr = r.maximum(s);
        const bf16x8 p0 = r.probabilities(s, 0, mr), p1 = r.probabilities(s, 1, mr);
        if (more) wait_newest(IC<N_DMA>{});  // V(t); K(t+1)'s loads are newer
        else wait_newest(IC<0>{});
        if (!whole) dropped |= drop_nonfinite<D>(v_tile, lane);
        at.load_v(0, 0, vf[0]);
        at.load_v(0, 1, vf[1]);
        reads_done();
        if (more) {
            src.fetch(src.v_base, t + 1, next, v_tile);
            now = next;
            next = src.place(places, src.in_list(t + 2));
        }
        r.pv(vf[0], p0);
        r.pv(vf[1], p1);
    }
    if (dropped) r.add_nonfinite(p, job, tiles, t_begin, t_end, kvh, hh);

    // ---- the wavefronts' results meet in LDS, each scaled to the common maximum, in its own tiles; 16-byte chunk c of row i lies at
    // chunk position c ^ i, so that writes (a row per lane) and reads (a row per CPR lanes) touch all banks
    const float l_tot = pair_sum(r.l);
    if (hh == 0) ml[wave][col] = f32x2{part_max(r.m_ref, l_tot), l_tot};
    __syncthreads();
    const int n_rows = job.n_rows - job.row0 < WM ? job.n_rows - job.row0 : WM;
    if (r.ok) {
        r.clear_empty(l_tot);
        float m_all = ml[0][col][0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) m_all = fmaxf(m_all, ml[w][col][0]);
        const float f = l_tot == 0.f ? 0.f : __builtin_amdgcn_exp2f(part_max(r.m_ref, l_tot) - m_all);
        f32x4* mine = reinterpret_cast<f32x4*>(lds + (size_t)wave * 2 * TILE_B);
#pragma unroll
        for (int db = 0; db < D / 32; ++db)
#pragma unroll
            for (int j4 = 0; j4 < 4; ++j4) {
                const int c = db * 8 + j4 * 2 + hh;
                mine[col * CPR + (c ^ (col & (CPR - 1)))] =
                    f32x4{r.o[db][j4 * 4] * f, r.o[db][j4 * 4 + 1] * f, r.o[db][j4 * 4 + 2] * f, r.o[db][j4 * 4 + 3] * f};
            }
    }
    __syncthreads();
    for (int e = tid; e < n_rows * CPR; e += THREADS) {
        const int i = e / CPR, c = e % CPR, row = job.row0 + i, tok = row / G;
        const int64_t q_row = (int64_t)(job.token0 + tok) * p.n_q_heads + kvh * G + (row - tok * G);
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += *reinterpret_cast<const f32x4*>(lds + (size_t)w * 2 * TILE_B + (i * CPR + (c ^ (i & (CPR - 1)))) * 16);
        float m_all = ml[0][i][0], l_all = 0.f;
#pragma unroll
        for (int w = 1; w < WAVES; ++w) m_all = fmaxf(m_all, ml[w][i][0]);
#pragma unroll
        for (int w = 0; w < WAVES; ++w)
            if (ml[w][i][1] != 0.f) l_all += ml[w][i][1] * __builtin_amdgcn_exp2f(ml[w][i][0] - m_all);
        if (a.n_slots == 1) {
            store4(static_cast<bf16_t*>(p.out) + q_row * D + c * 4, v * (l_all == 0.f ? 0.f : 1.f / l_all));
        } else {
            const int64_t to = (int64_t)job.slot * p.b.n_tokens * p.n_q_heads + q_row;
            if (l_all != 0.f) *reinterpret_cast<f32x4*>(a.part_o + to * D + c * 4) = v;
            if (c == 0) *reinterpret_cast<f32x2*>(a.part_ml + to * 2) = f32x2{m_all, l_all};
        }
    }
}

// ROW_BLOCKS: all by blocks of 128 rows.  KEY_BLOCKS, STREAMED: the sequences' own keys by blocks of 32 rows, a prefix computed
// for the batch at once still by blocks of 128 (42 rows over 3,136 tokens take 11.1 us so, 10.8 to 11.6 by blocks of 32).
template <int D, bool TWO_PAGES, int HOW>
__global__ __launch_bounds__(THREADS, 2) void attn_paged_kernel(PagedArgs a) {
    constexpr bool FEW = HOW != ROW_BLOCKS;
    __shared__ __attribute__((aligned(1024))) unsigned char lds[2 * STAGES * BN * D * 2];
    __shared__ f32x2 ml[FEW ? WAVES : 1][WM];
    __shared__ int sh_dropped;
    // KV heads fastest: workgroups are dealt to the eight XCDs in turn, so that one of them sees few heads' keys
    const int L = blockIdx.x / a.p.n_kv_heads, kvh = blockIdx.x - L * a.p.n_kv_heads, lane = threadIdx.x & 63;
    const bool prefix = L < a.prefix_blocks * a.prefix_splits;
    Job job;
    if (FEW && !prefix) {
        if (find_own_job<WM>(a.p, a.prefix_blocks, a.prefix_splits, a.blocks, a.splits, L, lane, &job))
            keys_block<D, TWO_PAGES, HOW == STREAMED>(a, job, kvh, lds, ml);
        return;
    }
    if (prefix ? find_prefix_job<BM>(a.p, a.prefix_blocks, a.prefix_splits, L, &job)
               : find_own_job<BM>(a.p, a.prefix_blocks, a.prefix_splits, a.blocks, a.splits, L, lane, &job))
        rows_block<D, TWO_PAGES>(a, job, kvh, lds_addr_of(lds), &sh_dropped);
}

// Joins the partial results of the rows (token, head).  tpr threads own four dimensions each of a row; the slots of a row are
// spread over `groups` sets of them, whose sums meet in LDS, so that a few rows of many slots (one user) are not read one after the
// other: 28 rows of 58 slots 9.3 us with 256 threads a row and a maximum waited for before its sums, 3.9 so.  Slots of no keys hold the
// maximum -inf; what else they hold is not used.
constexpr int MOST_MERGE_THREADS = 1024;
template <bool BF16>
__global__ __launch_bounds__(MOST_MERGE_THREADS) void attn_paged_merge_kernel(PagedArgs a, int tpr, int groups, int rows_per_block) {
    __shared__ float red_m[MOST_MERGE_THREADS], red_l[MOST_MERGE_THREADS];
    __shared__ f32x4 red_o[MOST_MERGE_THREADS];
    const PagedProblem& p = a.p;
    const int D = p.head_dim, tid = threadIdx.x;
    const int unit = tid / tpr, dq = tid - unit * tpr;           // (row of the block, group), dimensions 4 dq ..
    const int r = unit / groups, g = unit - r * groups;
    const int64_t n_rows = (int64_t)p.b.n_tokens * p.n_q_heads;
    const int64_t row = (int64_t)blockIdx.x * rows_per_block + r;
    const TokenRange range = token_range(p.b);       // (looked at when the partial results are on their way)
    bool ok = r < rows_per_block && row < n_rows;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    if (ok) {
        constexpr int U = 4;
        for (int s0 = g; s0 < a.n_slots; s0 += U * groups) {
            f32x2 ml[U];
            f32x4 v[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {        // all loads leave together; what an empty slot holds is not used
                const int s = s0 + u * groups;
                ml[u] = f32x2{-INFINITY, 0.f};
                if (s < a.n_slots) {
                    ml[u] = *reinterpret_cast<const f32x2*>(a.part_ml + ((int64_t)s * n_rows + row) * 2);
                    v[u] = *reinterpret_cast<const f32x4*>(a.part_o + ((int64_t)s * n_rows + row) * D + dq * 4);
                }
            }
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
    ok = ok && row >= (int64_t)range.first * p.n_q_heads && row < (int64_t)range.end * p.n_q_heads;
    if (groups > 1) {
        red_o[tid] = acc;
        red_m[tid] = m;
        red_l[tid] = l;
        __syncthreads();
        if (!ok || g != 0) return;
        float m_all = m;
#pragma unroll 8
        for (int i = 1; i < groups; ++i) m_all = fmaxf(m_all, red_m[tid + i * tpr]);
        const float ref = m_all == -INFINITY ? 0.f : m_all;
        acc = f32x4{0.f, 0.f, 0.f, 0.f};
        l = 0.f;
#pragma unroll 8
        for (int i = 0; i < groups; ++i) {       // (a group of no keys has the weight 0 and sums of 0)
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

// ---- fp32: true fp32 products and sums on the matrix cores, operands straight from memory as in attention_f32.hip.  Head sizes between
// 64, 128 and 256 (D_MAX) are padded with zeros in the registers.  A workgroup's four wavefronts share 16 stacked rows and take the
// 32-key tiles in turn; their (maximum, sum, O) meet in LDS.  Bound, at the sizes that fp32 serves, by the round trips to the first key.  The tiny configuration's ragged batch
// (5 sequences, window 77) takes 8.1 us, 21.5 on the vector ALU.
constexpr int F32_ROWS = 16;

// All four lanes (q, q + 16, q + 32, q + 48) of a query combine a value.
template <bool MAX>
__device__ inline float quad_combine(float v) {
    auto op = [](uint32_t a, uint32_t b) {
        const float x = __uint_as_float(a), y = __uint_as_float(b);
        return MAX ? fmaxf(x, y) : x + y;
    };
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = op(r[0], r[1]);
    const auto t = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return op(t[0], t[1]);
}

template <int D_MAX, bool PADDED>
__global__ __launch_bounds__(THREADS, D_MAX > 128 ? 1 : 2) void attn_paged_f32_kernel(PagedArgs a) {
    constexpr int QD = D_MAX / 4;                 // dims per lane of a Q or K row
    constexpr int VB = D_MAX / 64;                // 64-dim blocks of V and O
    const int D = PADDED ? a.p.head_dim : D_MAX;
    auto load4 = [&](const float* v, int dim) { return !PADDED || dim < D ? *reinterpret_cast<const f32x4*>(v + dim) : f32x4{0.f, 0.f, 0.f, 0.f}; };
    __shared__ f32x4 o_lds[WAVES][VB * 4][64];
    __shared__ float m_lds[WAVES][F32_ROWS], l_lds[WAVES][F32_ROWS];
    const PagedProblem& p = a.p;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r = lane & 15, g = lane >> 4, G = p.n_q_heads / p.n_kv_heads, page = (int)p.b.by_page.d;
    const int L = blockIdx.x / p.n_kv_heads, kvh = blockIdx.x - L * p.n_kv_heads;
    Job job;
    if (!(L < a.prefix_blocks * a.prefix_splits ? find_prefix_job<F32_ROWS>(p, a.prefix_blocks, a.prefix_splits, L, &job)
                                                : find_own_job<F32_ROWS>(p, a.prefix_blocks, a.prefix_splits, a.blocks, a.splits, L, lane, &job)))
        return;
    const Tiles<BN> tiles = tiles_of<F32_ROWS>(p, job, G);
    int t_begin, t_end;
    split_range(a, job, tiles.n, WAVES, &t_begin, &t_end);
    const int row = job.row0 + r, tok = row / G, pos = job.p0 + tok;
    const bool row_ok = row < job.n_rows;
    const int64_t q_row = (int64_t)(job.token0 + tok) * p.n_q_heads + kvh * G + (row - tok * G);
    // lane l (of 32): the cache's row (over tokens and heads) of key l of a tile
    auto places = [&](int t) -> int64_t {
        int r0, r1;
        tiles.rows(t, &r0, &r1);
        const int key = tiles.key0(t) + clamped(lane & 31, r0, r1), slot = (int)quot((uint32_t)key, p.b.by_page);
        const int32_t* table = tiles.in_prefix(t) ? p.prefix_pages : job.table;
        return ((int64_t)clamped(table[slot], 0, p.b.n_pages - 1) * page + (key - slot * page)) * p.n_kv_heads + kvh;
    };
    auto of_lane = [](int64_t v, int from) -> int64_t {
        return (int64_t)((uint64_t)(uint32_t)__shfl((int)(v >> 32), from) << 32 | (uint32_t)__shfl((int)v, from));
    };
    const float* qp = static_cast<const float*>(p.q) + q_row * D;
    f32x4 qf[QD / 4];
#pragma unroll
    for (int i = 0; i < QD / 4; ++i) qf[i] = row_ok ? load4(qp, g * QD + i * 4) : f32x4{0.f, 0.f, 0.f, 0.f};
    f32x4 o[VB][4];
#pragma unroll
    for (int b = 0; b < VB; ++b)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[b][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;
    const float sc = p.scale * 1.4426950408889634f;
    bool dropped = false;
    int64_t next = t_begin + wave < t_end ? places(t_begin + wave) : 0;
    for (int t = t_begin + wave; t < t_end; t += WAVES) {
        const int64_t at = next;
        f32x4 kf[2][QD / 4], vf[2][4][VB];
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            const float* k = static_cast<const float*>(p.b.k_pages) + of_lane(at, kb * 16 + r) * D;
#pragma unroll
            for (int i = 0; i < QD / 4; ++i) kf[kb][i] = load4(k, g * QD + i * 4);
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int jj = 0; jj < 4; ++jj) {
                const float* v = static_cast<const float*>(p.b.v_pages) + of_lane(at, kb * 16 + g * 4 + jj) * D;
#pragma unroll
                for (int b = 0; b < VB; ++b) vf[kb][jj][b] = load4(v, b * 64 + r * 4);
            }
        if (t + WAVES < t_end) next = places(t + WAVES);
        __builtin_amdgcn_sched_barrier(0);       // the loads leave together
        const int k0 = tiles.key0(t) + g * 4;
        const bool whole = tiles.whole(t);
        const Seen sees = whole ? Seen{0, 0x7fffffff, 0} : tiles.in_prefix(t) ? Seen{0, tiles.n_prefix, 0} : seen_by(p, pos);
        f32x4 s[2];
        float mx = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
            f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = {0.f, 0.f, 0.f, 0.f};     // two chains
#pragma unroll
            for (int i = 0; i < QD / 4; ++i)
#pragma unroll
                for (int c = 0; c < 4; c += 2) {
                    s0 = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[kb][i][c], qf[i][c], s0, 0, 0, 0);
                    s1 = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[kb][i][c + 1], qf[i][c + 1], s1, 0, 0, 0);
                }
#pragma unroll
            for (int jj = 0; jj < 4; ++jj) {
                s[kb][jj] = sees(k0 + kb * 16 + jj) ? (s0[jj] + s1[jj]) * sc : -INFINITY;
                mx = fmaxf(mx, s[kb][jj]);
            }
        }
        mx = quad_combine<true>(mx);
        const float m_new = fmaxf(m, mx), ref = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m - ref);
        m = m_new;
        l *= alpha;
#pragma unroll
        for (int b = 0; b < VB; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[b][e] *= alpha;
        // Where not every row sees every key, a probability of 0 keeps a value out only if that value is finite: the others are left
        // out here and added after the loop.
        if (!whole) {
            float nan_or_0 = 0.f;
#pragma unroll
            for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                for (int jj = 0; jj < 4; ++jj)
#pragma unroll
                    for (int b = 0; b < VB; ++b)
#pragma unroll
                        for (int e = 0; e < 4; ++e) nan_or_0 = fmaf(vf[kb][jj][b][e], 0.f, nan_or_0);
            if (__builtin_amdgcn_ballot_w64(nan_or_0 != 0.f) != 0) {
                dropped = true;
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int jj = 0; jj < 4; ++jj)
#pragma unroll
                        for (int b = 0; b < VB; ++b)
#pragma unroll
                            for (int e = 0; e < 4; ++e)
                                vf[kb][jj][b][e] = __builtin_fabsf(vf[kb][jj][b][e]) < INFINITY ? vf[kb][jj][b][e] : 0.f;
            }
        }
#pragma unroll
        for (int kb = 0; kb < 2; ++kb)
#pragma unroll
            for (int jj = 0; jj < 4; ++jj) {
                const float pj = __builtin_amdgcn_exp2f(s[kb][jj] - ref);
                l += pj;
#pragma unroll
                for (int b = 0; b < VB; ++b)
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[b][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[kb][jj][b][e], pj, o[b][e], 0, 0, 0);
            }
    }
    // lane (q = r, g), register i of block e of o[b]: dim b*64 + 4*(4g + i) + e
    if (dropped && row_ok) {
        const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll 1
        for (int t = t_begin + wave; t < t_end; t += WAVES) {
            if (tiles.whole(t)) continue;
            const bool pre = tiles.in_prefix(t);
            const int32_t* table = pre ? p.prefix_pages : job.table;
            const Seen sees = pre ? Seen{0, tiles.n_prefix, 0} : seen_by(p, pos);
#pragma unroll 1
            for (int key = tiles.key0(t); key < tiles.key0(t) + BN; ++key) {
                if (!sees(key)) continue;
                const int slot = (int)quot((uint32_t)key, p.b.by_page);
                const int64_t at = (((int64_t)clamped(table[slot], 0, p.b.n_pages - 1) * page + (key - slot * page)) * p.n_kv_heads + kvh) * D;
                const float *kr = static_cast<const float*>(p.b.k_pages) + at, *vr = static_cast<const float*>(p.b.v_pages) + at;
                float s = 0.f;
#pragma unroll 1
                for (int d = 0; d < D; ++d) s = fmaf(kr[d], qp[d], s);
                const float pj = __builtin_amdgcn_exp2f(s * sc - ref);
#pragma unroll
                for (int b = 0; b < VB; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const f32x4 v = load4(vr, b * 64 + g * 16 + i * 4);
#pragma unroll
                        for (int e = 0; e < 4; ++e) o[b][e][i] = fmaf(pj, __builtin_fabsf(v[e]) < INFINITY ? 0.f : v[e], o[b][e][i]);
                    }
            }
        }
    }
    l = quad_combine<false>(l);
#pragma unroll
    for (int b = 0; b < VB; ++b)
#pragma unroll
        for (int i = 0; i < 4; ++i) o_lds[wave][b * 4 + i][lane] = f32x4{o[b][0][i], o[b][1][i], o[b][2][i], o[b][3][i]};
    if (g == 0) {
        m_lds[wave][r] = part_max(m, l);
        l_lds[wave][r] = l;
    }
    __syncthreads();
    if (!row_ok) return;
    float m_all = m_lds[0][r], l_all = 0.f, w[WAVES];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) m_all = fmaxf(m_all, m_lds[i][r]);
#pragma unroll
    for (int i = 0; i < WAVES; ++i) {
        w[i] = l_lds[i][r] == 0.f ? 0.f : __builtin_amdgcn_exp2f(m_lds[i][r] - m_all);
        l_all += l_lds[i][r] * w[i];
    }
    const int64_t to = (int64_t)job.slot * p.b.n_tokens * p.n_q_heads + q_row;
    const float inv = a.n_slots > 1 ? 1.f : l_all == 0.f ? 0.f : 1.f / l_all;
    float* out = (a.n_slots > 1 ? a.part_o + to * D : static_cast<float*>(p.out) + q_row * D);
    for (int c = wave; c < VB * 4; c += WAVES) {          // a wavefront each four dims of a 64-dim block
        const int dim = c / 4 * 64 + g * 16 + c % 4 * 4;
        if (PADDED && dim >= D) continue;
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < WAVES; ++i)
            if (w[i] != 0.f) v += o_lds[i][c][lane] * w[i];
        *reinterpret_cast<f32x4*>(out + dim) = v * inv;
    }
    if (a.n_slots > 1 && wave == 0 && g == 0) *reinterpret_cast<f32x2*>(a.part_ml + to * 2) = f32x2{m_all, l_all};
}

int64_t up(int64_t n, int64_t d) { return (n + d - 1) / d; }
constexpr int64_t MOST_PARTIALS = (int64_t)512 << 20;      // bytes of a prefix's partial results
constexpr int64_t PLACES = 512;       // workgroups of a bf16 launch that the chip holds: two per CU

}  // namespace

PagedPlan attn_paged_plan(int dtype, int n_q_heads, int n_kv_heads, int head_dim, int64_t n_tokens, int64_t n_seqs, int64_t max_kv,
                          int64_t window, int64_t sinks, int64_t n_prefix) {
    const int64_t G = n_q_heads / n_kv_heads, all_rows = n_tokens * G;
    const bool bf16 = dtype == REKV_BF16;
    PagedPlan plan;
    const int64_t keys = window < 0 || window + sinks > max_kv ? max_kv : window + sinks;
    // Blocks of 32 rows start and end sooner but fetch every tile four times as often: they take the sequences' own keys where few rows of
    // a sequence share them, and where the chip holds them in two rounds and has no more than SMALL tiles of 128 rows per place to do (causal
    // ones half).  Blocks of 128 and of 32 rows at 28/4/128 (us): a prompt of 196 tokens 13.8 and 8.6, of 1,000 28 and 16, a live frame over
    // 3,136 at 14/2/64 22.1 and 16.8, 8 x 60 tokens over 3,000 37 and 26; the other way 32 x 16 over 3,000 36 and 44 (23 tiles a place), 8
    // x 160 through a window of 3,200 51 and 70 (26), in more than two rounds a prompt of 2,000 at 64/8/128 48 and 79, 80 x 50 tokens over 400 39 and 46.
    // In the second round they need something to do: of 30 x 60 tokens over nothing 16 and 20, over 400 37 and 28.  On the 250 random batches that
    // it was fitted to the choice takes 1.007 of the better time, one by tiles alone 1.054; on 500 others 1.010, blocks of 32 rows always 1.013, of
    // 128 always 1.15.  Beside a prefix, which larger batches have computed for all at once, SMALL is 7.
    const int64_t SMALL = n_prefix > 0 ? 7 : 20;
    const int64_t row_blocks = up(all_rows, BM) > n_seqs ? up(all_rows, BM) : n_seqs;
    const int64_t key_jobs = (up(all_rows, WM) > n_seqs ? up(all_rows, WM) : n_seqs) * n_kv_heads;
    const bool lone = all_rows <= n_seqs * WM;
    const int64_t causal = n_tokens / n_seqs < keys ? n_tokens / n_seqs : keys;
    const bool rounds = key_jobs <= PLACES || (key_jobs <= 2 * PLACES && (head_dim < 128 || keys + n_prefix > 4 * BN));
    const bool small = rounds && row_blocks * n_kv_heads * up(keys + n_prefix - causal / 2, BN) <= SMALL * PLACES;
    const bool few = bf16 && (lone || small);

    // Blocks of 128 rows in `jobs` times n workgroups over `tiles` tiles, in us: rounds of workgroups, each of about 8 us and tau a tile; and
    // what a partial result of every row takes to write and read again.
    const double tau = head_dim == 128 ? 0.8 : 0.5, slot_us = (double)(n_tokens * n_q_heads * (head_dim + 2)) * 8.0 / 3.5e6;
    auto rows_us = [&](double jobs, int64_t tiles, int64_t n) { return ceil(jobs * (double)n / PLACES) * ((double)tiles / (double)n * tau + 8.0); };
    // blocks that ragged sequences fill, about; uneven over the XCDs
    const double own_jobs = (n_seqs == 1 ? (double)row_blocks : 1.15 * ((double)all_rows / BM + 0.5 * (double)n_seqs)) * (double)n_kv_heads;

    // Blocks of 32 rows: in how many splits, of at most so many as fill the chip and two tiles a wavefront at least (a user's window of
    // 15,000 tokens at 28/4/128 takes 16.7 us so, 18.7 with one, 17.5 with three), and in about how many us.  A round of workgroups takes 7
    // and a wavefront's tiles, 1.4 times as long with two workgroups on a CU, or what its blocks' reads of a prefix take from the caches at 10
    // TB/s; splits take the joining launch, if nothing else does, and the partial results (28/4/128, unsplit and filling the chip, us: a user's 450 tokens 9.2 and 9.8, 700 10.8 and 9.8, 2,000 19.0 and 10.7; 300
    // tokens over 1,400 20.1 and 22.5; 8 x 60 over 1,000 18.7 and 26.6).
    constexpr int64_t FEW_TILES = 2 * WAVES;
    const double few_jobs = (double)key_jobs;
    auto few_us = [&](int64_t tiles, int64_t prefix, bool joined, int64_t* splits) {
        double best = 1e30;
        const double reads = few_jobs * (double)(prefix * head_dim * 4) / 10e6;
        for (int64_t n = 1; n == 1 || (n * key_jobs <= PLACES && n <= up(tiles, FEW_TILES)); ++n) {
            const double step = (head_dim == 128 ? 1.0 : 0.6) * (2.0 * few_jobs * (double)n > PLACES ? 1.4 : 1.0);
            const double in_turn = ceil(few_jobs * (double)n / PLACES), walk = in_turn * (double)tiles / (double)(WAVES * n) * step;
            const double us = in_turn * 7.0 + (walk > reads ? walk : reads) + (n > 1 ? (joined ? 0.0 : 3.0) + (double)n * slot_us : 0.0);
            if (us < best) {
                best = us;
                *splits = n;
            }
        }
        return best;
    };
    int64_t few_splits = 1;

    // A prefix is computed for the batch at once, by full blocks of all sequences' rows whose results are joined with the own keys', or
    // walked by each sequence's own blocks.  Measured, walked and at once (us, 28/4/128, a prefix of 4,608): 64 sequences of 12 tokens 119
    // and 77, of 24 211 and 132, of 32 228 and 158, of 48 260 and 249, of 64 280 and 305, 24 of 40 128 and 86, 16 of 12 45 and 36.  The estimate is off
    // by a tenth where the two are alike: of these it takes the slower one at 48 and at 64 tokens.  On 260 random batches that it was not fitted to
    // it takes 1.030 of the better time, at once always 1.23, walked always 1.12.
    plan.prefix_blocks = plan.prefix_splits = 0;
    plan.min_prefix_tiles = 4;
    // (fp32: lone rows walk a prefix of up to F32_SHORT tiles, and up to F32_WHOLE tiles are not split.  30 users' tokens after five tiles at
    // 14/2/64 take 10.5 us at once, 9.5 walked in two splits, 8.0 in one; after 13 tiles 11.1, 11.1 and 13.1; after 32 11.1 and 15.2.  Users of eight
    // rows or more walk every prefix, which long ones make dear: 8 users of 28/4/128 with 13 tokens after 4,000 take 39 us, 26 at once.  The splits of a
    // prefix at once come from the estimate for bf16 blocks; on 81 batches they take 1.031 of the best power of two's time, 1.20 at worst.)
    constexpr int64_t F32_SHORT = 16, F32_WHOLE = 8;
    bool together = !bf16 && all_rows < n_seqs * (F32_ROWS / 2) && n_prefix > F32_SHORT * BN;
    const int64_t prefix_rows = bf16 ? BM : F32_ROWS, prefix_tiles = up(n_prefix, BN);
    if (n_prefix > 0 && (together || (bf16 && (lone || !small)))) {
        plan.prefix_blocks = (int32_t)up(all_rows, prefix_rows);
        plan.prefix_splits = 1;
        const double jobs = (double)plan.prefix_blocks * (double)n_kv_heads;
        // Lone rows' workgroups are short and run beside these: half a place each (64 users over 25,088 tokens at 28/4/128, us: 48.5 with 24
        // splits, as this gives, 56.0 with 32, 50.6 with 16).
        const double beside = lone ? 0.5 * (double)(n_seqs * n_kv_heads) : 0.0;
        double best = 1e30;
        const int64_t most = MOST_PARTIALS / (n_tokens * n_q_heads * (head_dim + 2) * 4);
        for (int64_t n = 1; n == 1 || (n <= PLACES && n <= most && n * plan.min_prefix_tiles <= prefix_tiles); ++n) {
            const double us = rows_us(jobs + beside / (double)n, prefix_tiles, n) + (double)n * slot_us;
            if (us < best) {
                best = us;
                plan.prefix_splits = (int32_t)n;
            }
        }
        if (bf16 && lone) {
            // (of the 125 random batches it was fitted to 1.015 of the better time, all at once 1.26, all walked 1.08; of 260 others 1.023, 1.13, 1.14)
            const double own = few_us(up(keys, BN), 0, true, &few_splits);
            together = (best > own ? best : own) + slot_us + 1.0 < few_us(up(keys + n_prefix, BN), n_prefix, false, &few_splits);
        } else if (!together) {
            const int64_t s = PLACES / (row_blocks * n_kv_heads), tiles = up(keys + n_prefix, BN);
            const double walked = rows_us(own_jobs, tiles, s > 1 ? s : 1) + (s > 1 ? (double)s * slot_us + 4.0 : 0.0);
            together = best + rows_us(own_jobs, up(keys, BN), 1) + slot_us + 4.0 < walked;
        }
        if (!together) plan.prefix_blocks = plan.prefix_splits = 0;
    }

    plan.how = !few ? ROW_BLOCKS : lone && (together || n_prefix == 0 || n_seqs == 1) ? STREAMED : KEY_BLOCKS;     // (a walked prefix is shared)
    plan.rows = !bf16 ? F32_ROWS : few ? WM : BM;
    plan.blocks = (int32_t)(all_rows / plan.rows + n_seqs);
    const int64_t places = bf16 ? PLACES : 1024, busy = up(all_rows, plan.rows) > n_seqs ? up(all_rows, plan.rows) : n_seqs;
    const int64_t tiles = up(together ? keys : keys + n_prefix, BN);
    plan.min_tiles = few ? FEW_TILES : 4;
    int64_t s = places / (busy * n_kv_heads);
    if (s > up(tiles, plan.min_tiles)) s = up(tiles, plan.min_tiles);
    if (!bf16 && tiles <= F32_WHOLE) s = 1;
    if (few) {
        few_us(tiles, together ? 0 : n_prefix, together, &few_splits);
        s = few_splits;
    }
    // Where lone rows all but fill it, their lengths differ: pieces of one size, LONG tiles, spread the longer ones (64 users of 1 to 8,192
    // tokens at 64/8/128: 221 us whole, 207, 199, 199, 205 in pieces of 96, 64, 48, 32).
    constexpr int64_t LONG = 64, MOST_PIECES = 64;
    if (few && s < 8 && s < tiles / LONG && busy * n_kv_heads < 4 * PLACES) {
        s = tiles / LONG < MOST_PIECES ? tiles / LONG : MOST_PIECES;
        plan.min_tiles = (int32_t)LONG;
    }
    plan.splits = (int32_t)(s < 1 ? 1 : s);
    plan.workspace_bytes = plan.slots() > 1 ? n_tokens * n_q_heads * plan.slots() * (head_dim + 2) * 4 : 0;
    return plan;
}

template <int D, bool TWO_PAGES>
void launch_bf16(const PagedArgs& a, int how, dim3 grid, hipStream_t stream) {
    if (TWO_PAGES && how == STREAMED) hipLaunchKernelGGL((attn_paged_kernel<D, TWO_PAGES, TWO_PAGES ? STREAMED : KEY_BLOCKS>), grid, dim3(THREADS), 0, stream, a);
    else if (how != ROW_BLOCKS) hipLaunchKernelGGL((attn_paged_kernel<D, TWO_PAGES, KEY_BLOCKS>), grid, dim3(THREADS), 0, stream, a);
    else hipLaunchKernelGGL((attn_paged_kernel<D, TWO_PAGES, ROW_BLOCKS>), grid, dim3(THREADS), 0, stream, a);
}

hipError_t attn_paged_launch(const PagedProblem& p, const PagedPlan& plan, int dtype, void* workspace, hipStream_t stream) {
    PagedArgs a;
    a.p = p;
    a.prefix_blocks = plan.prefix_blocks; a.prefix_splits = plan.prefix_splits;
    a.blocks = plan.blocks; a.splits = plan.splits; a.min_tiles = plan.min_tiles; a.min_prefix_tiles = plan.min_prefix_tiles;
    a.n_slots = plan.slots();
    const int64_t rows = (int64_t)p.b.n_tokens * p.n_q_heads;
    a.part_o = static_cast<float*>(workspace);
    a.part_ml = a.n_slots > 1 ? a.part_o + rows * a.n_slots * p.head_dim : nullptr;
    const int64_t jobs = (int64_t)plan.prefix_blocks * plan.prefix_splits + (int64_t)plan.blocks * plan.splits;
    const dim3 grid((unsigned)(jobs * p.n_kv_heads));
    const bool two_pages = p.b.by_page.d >= BN || p.b.by_page.d == 16;
    if (dtype == REKV_F32) {
        const int d = p.head_dim;
        hipLaunchKernelGGL((d == 64    ? attn_paged_f32_kernel<64, false>
                            : d == 128 ? attn_paged_f32_kernel<128, false>
                            : d < 64   ? attn_paged_f32_kernel<64, true>
                            : d < 128  ? attn_paged_f32_kernel<128, true>
                                       : attn_paged_f32_kernel<256, true>),
                           grid, dim3(THREADS), 0, stream, a);
    }
    else if (p.head_dim == 128) (two_pages ? launch_bf16<128, true> : launch_bf16<128, false>)(a, plan.how, grid, stream);
    else (two_pages ? launch_bf16<64, true> : launch_bf16<64, false>)(a, plan.how, grid, stream);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.n_slots == 1) return e;
    const int tpr = p.head_dim / 4, threads = a.n_slots > 32 ? MOST_MERGE_THREADS : 256, units = threads / tpr;
    int groups = 1;                           // of at most four slots each, as far as a block has threads
    while (groups * 2 <= units && groups * 4 < a.n_slots) groups *= 2;
    const int per_block = units / groups;
    const dim3 merge_grid((unsigned)up(rows, per_block));
    if (dtype == REKV_F32) hipLaunchKernelGGL(attn_paged_merge_kernel<false>, merge_grid, dim3(threads), 0, stream, a, tpr, groups, per_block);
    else hipLaunchKernelGGL(attn_paged_merge_kernel<true>, merge_grid, dim3(threads), 0, stream, a, tpr, groups, per_block);
    return hipGetLastError();
}

}  // namespace rekv
