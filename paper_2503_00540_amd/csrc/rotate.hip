// Rotary positions with several axes, and the append of new keys and values to a paged cache with the rotation on the way.
//
//   (x_a, x_b) -> (x_a cos t - x_b sin t, x_a sin t + x_b cos t),  t = position[axis of the pair] * base^(-2i / D)
//
// Bound: HBM for many tokens (50,176 x 28 heads of 128 out of a fused projection 121 us = 5.95 TB/s, a plain copy 5.96; append of
// 26,800 tokens at 28/4/128 with their queries 92 us = 5.4 TB/s), the launch and its round trips for few (64 users 4.8 us).  A unit of work is one 16-byte chunk of a head
// vector and its partner half a vector on, which hold both members of their pairs in either layout.  A lane keeps one
// chunk position of one token and walks that token's heads, so that its angles (formed in double precision, reduced to within
// an eighth of a turn there) are worked out once for all of them.
#include "common.h"
#include "paged.h"

namespace rekv {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
constexpr int WAVES = 4;
// Few tokens: their heads are divided until there are so many wavefronts (64 tokens of 64/8/128 with keys and values 1.1 us less with ten a
// token than with four, of 4.8).
constexpr int FILL_WAVES = 4096;
// At most so many wavefronts; the tokens beyond are walked.  Rotation of 50,176 x 28 heads of 128 (us): 128 with 8,192, 123 with 20,480, 121 with
// 40,960, 153 with one per token; append of 24 streams' 26,800 tokens at 28/4/128: 93.3, 92.6, 94.5, 108.
constexpr int MOST_WAVES[2] = {40960, 20480};

// Sine and cosine of t quarter turns, |t| < 2^31: the angle less a multiple q of a quarter turn (exact) lies within pi / 4, where the
// Taylor series to y^9 and y^10 are off by less than 2^-28.  The angle is rounded to fp32 once, there, as late as it can be (2^-25 at most): with
// the roundings of the sums both results are within 1.4 x 2^-24, rms 1.7e-8; from a fraction of a whole turn in fp32 it were 2.4 x 2^-24, rms 3.4e-8.
__device__ inline void sin_cos_quarters(double t, float* sn, float* cs) {
    const double qd = rint(t);
    const float y = (float)((t - qd) * 1.5707963267948966), z = y * y;
    float s = fmaf(z, 2.7557319e-6f, -1.9841270e-4f), c = fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
    s = fmaf(z, s, 8.3333333e-3f);
    c = fmaf(z, c, -1.3888889e-3f);
    s = fmaf(z, s, -0.16666667f);
    c = fmaf(z, c, 4.1666667e-2f);
    s = fmaf(z * y, s, y);
    c = fmaf(z, fmaf(z, c, -0.5f), 1.f);
    const int q = (int)qd;
    const float u = q & 1 ? c : s, v = q & 1 ? s : c;
    *sn = __uint_as_float(__float_as_uint(u) ^ ((uint32_t)(q & 2) << 30));
    *cs = __uint_as_float(__float_as_uint(v) ^ ((uint32_t)((q + 1) & 2) << 30));
}

// A wavefront takes part `part` of `parts` of a token's head vectors (queries, then keys, then values), 64 / cpr of them at a time,
// of every n_waves / parts-th token; what its pairs turn by per position stays in its registers.
template <bool BF16, bool APPEND>
__global__ __launch_bounds__(WAVES * 64) void rotate_kernel(RotateArgs a, int parts, int tokens_apart) {
    constexpr int EPC = BF16 ? 8 : 4;            // elements per 16-byte chunk
    constexpr int ES = BF16 ? 2 : 4;
    constexpr int BATCH = APPEND ? 2 : 4;        // head vectors of a lane whose loads leave together
    const int lane = threadIdx.x & 63;
    const uint32_t w = blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int first_tok = (int)(w / (uint32_t)parts), part = (int)(w - (uint32_t)first_tok * (uint32_t)parts);
    const PagedBatch& b = a.b;
    if (first_tok >= tokens_apart) return;       // of the last workgroup: the tokens are others'
    int tok_begin = 0, tok_end = a.n_tokens;
    if (APPEND) {
        const TokenRange range = token_range(b);
        tok_begin = range.first;
        tok_end = range.end;
    }
    const int half = a.head_dim / 2, cpr = half / EPC;           // chunk pairs per head vector
    const int per_wave = 64 / cpr, c = lane % cpr;
    const int n_q = a.q ? a.n_q_heads : 0, n_heads = APPEND ? n_q + 2 * a.n_kv_heads : n_q;
    const int step = per_wave * parts, base = part * per_wave;   // of the wavefront's heads
    const int mine = lane / cpr < per_wave ? base + lane / cpr : n_heads;
    const size_t at = (size_t)c * 16, head_b = (size_t)a.head_dim * ES;

    const bool turn = a.r.n_axes > 0;
    double turns[EPC];
    uint32_t axes = 0;                           // two bits a pair
    if (turn) {
#pragma unroll
        for (int e = 0; e < EPC; e += 2) {
            // pairs e and e + 1 of this lane's two chunks: elements of both, or neighbours, the first half of them in the first chunk; i is even
            const uint32_t i = a.r.interleaved ? (e >= EPC / 2 ? half / 2 : 0) + c * (EPC / 2) + e % (EPC / 2) : c * EPC + e;
            const double coarse = a.r.coarse[i / 8];
            turns[e] = coarse * a.r.fine[i % 8];
            turns[e + 1] = coarse * a.r.fine[i % 8 + 1];
            axes |= (a.r.axes[i / 16] >> (2 * (i % 16)) & 15u) << (2 * e);
        }
    }
    const int last = base + per_wave - 1;        // of the first heads; the wavefront's last ones are a multiple of step on
    const bool has_kv = APPEND && last + (n_heads - 1 - base) / step * step >= n_q;

    for (int tok = first_tok; tok < a.n_tokens; tok += tokens_apart) {
        const char* q = static_cast<const char*>(a.q) + (int64_t)tok * a.q_stride * ES + at;
        const char* k = static_cast<const char*>(a.k) + (int64_t)tok * a.k_stride * ES + at;
        const char* v = static_cast<const char*>(a.v) + (int64_t)tok * a.v_stride * ES + at;
        char* q_out = static_cast<char*>(a.q_out) + (int64_t)tok * a.q_out_stride * ES + at;

        u32x4 lo[BATCH], hi[BATCH];
        auto load = [&](int h0) {
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int h = h0 + i * step;
                if (h >= n_heads) continue;
                const char* src = h < n_q ? q + h * head_b : h < n_q + a.n_kv_heads ? k + (h - n_q) * head_b : v + (h - n_q - a.n_kv_heads) * head_b;
                lo[i] = *reinterpret_cast<const u32x4*>(src);
                hi[i] = *reinterpret_cast<const u32x4*>(src + half * ES);
            }
        };
        load(mine);                              // the first batch is under way before anything else is looked up
        if (tok < tok_begin || tok >= tok_end) continue;

        // the token's place in the pages, where this wavefront has keys or values, or where its index is its position
        char *k_row = nullptr, *v_row = nullptr;
        int index = 0;
        bool keep = false;
        if (APPEND && (has_kv || (turn && !a.positions))) {
            const Sequence s = find_sequence(b, lane, tok, [](int, int start) { return start; });
            index = s.kv - s.end + tok;
            if (index >= 0 && index < b.capacity) {
                const int slot = (int)quot((uint32_t)index, b.by_page), page = scalar_word(b.page_table + s.i * b.table_stride, slot);
                keep = page >= 0 && page < b.n_pages;
                const int64_t row = ((int64_t)page * b.by_page.d + (index - slot * (int)b.by_page.d)) * a.n_kv_heads * a.head_dim * ES;
                k_row = static_cast<char*>(b.k_pages) + row + at;
                v_row = static_cast<char*>(b.v_pages) + row + at;
            }
        }

        float cs[EPC], sn[EPC];
        if (turn) {
            int pos[MAX_AXES] = {index, index, index, index};
            if (!APPEND || a.positions)
#pragma unroll
                for (int x = 0; x < MAX_AXES; ++x) pos[x] = x < a.r.n_axes ? scalar_word(a.positions + x * a.positions_stride, tok) : 0;
#pragma unroll
            for (int e = 0; e < EPC; ++e) {
                const uint32_t x = axes >> (2 * e) & 3;
                const double t = (double)(x == 0 ? pos[0] : x == 1 ? pos[1] : x == 2 ? pos[2] : pos[3]) * turns[e];
                sin_cos_quarters(t, &sn[e], &cs[e]);
            }
        }
        auto rotate = [&](u32x4& l, u32x4& r) {
            float x[2 * EPC];                        // first chunk, then its partner
    #pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (BF16) {
                    x[2 * i] = __uint_as_float(l[i] << 16);
                    x[2 * i + 1] = __uint_as_float(l[i] & 0xffff0000u);
                    x[EPC + 2 * i] = __uint_as_float(r[i] << 16);
                    x[EPC + 2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
                } else {
                    x[i] = __uint_as_float(l[i]);
                    x[EPC + i] = __uint_as_float(r[i]);
                }
            }
            if (a.r.interleaved) {
    #pragma unroll
                for (int e = 0; e < EPC; ++e) {      // the chunks one after the other
                    const float y = x[2 * e], z = x[2 * e + 1];
                    x[2 * e] = y * cs[e] - z * sn[e];
                    x[2 * e + 1] = y * sn[e] + z * cs[e];
                }
            } else {
    #pragma unroll
                for (int e = 0; e < EPC; ++e) {
                    const float y = x[e], z = x[EPC + e];
                    x[e] = y * cs[e] - z * sn[e];
                    x[EPC + e] = y * sn[e] + z * cs[e];
                }
            }
    #pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (BF16) {
                    l[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[2 * i], x[2 * i + 1]}), bf16x2));
                    r[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[EPC + 2 * i], x[EPC + 2 * i + 1]}), bf16x2));
                } else {
                    l[i] = __float_as_uint(x[i]);
                    r[i] = __float_as_uint(x[EPC + i]);
                }
            }
        };
        for (int h0 = mine; h0 < n_heads; h0 += BATCH * step) {
            if (h0 != mine) load(h0);
#pragma unroll
            for (int i = 0; i < BATCH; ++i) {
                const int h = h0 + i * step;
                if (h >= n_heads) continue;
                if (turn && h < n_q + a.n_kv_heads) rotate(lo[i], hi[i]);
                if (h >= n_q && !keep) continue;
                char* dst = h < n_q ? q_out + h * head_b : h < n_q + a.n_kv_heads ? k_row + (h - n_q) * head_b : v_row + (h - n_q - a.n_kv_heads) * head_b;
                __builtin_nontemporal_store(lo[i], reinterpret_cast<u32x4*>(dst));
                __builtin_nontemporal_store(hi[i], reinterpret_cast<u32x4*>(dst + half * ES));
            }
        }
    }
}

}  // namespace

hipError_t rotate_launch(const RotateArgs& a, int dtype, hipStream_t stream) {
    const int per_wave = 64 / (a.head_dim / 2 / (dtype == REKV_BF16 ? 8 : 4));
    const int heads = (a.q ? a.n_q_heads : 0) + (a.k ? 2 * a.n_kv_heads : 0), most = (heads + per_wave - 1) / per_wave;
    // Many tokens: a wavefront has a whole token, and its angles serve all heads.  Few: as many wavefronts as the chip has places for.
    int parts = FILL_WAVES / a.n_tokens;
    parts = parts < 1 ? 1 : parts < most ? parts : most;
    int64_t waves = (int64_t)a.n_tokens * parts;
    const int64_t most_waves = MOST_WAVES[a.k != nullptr] / parts * parts;
    waves = waves < most_waves ? waves : most_waves;
    const int apart = (int)(waves / parts);
    const dim3 grid((unsigned)((waves + WAVES - 1) / WAVES)), block(WAVES * 64);
    if (dtype == REKV_BF16) {
        if (a.k) hipLaunchKernelGGL((rotate_kernel<true, true>), grid, block, 0, stream, a, parts, apart);
        else hipLaunchKernelGGL((rotate_kernel<true, false>), grid, block, 0, stream, a, parts, apart);
    } else {
        if (a.k) hipLaunchKernelGGL((rotate_kernel<false, true>), grid, block, 0, stream, a, parts, apart);
        else hipLaunchKernelGGL((rotate_kernel<false, false>), grid, block, 0, stream, a, parts, apart);
    }
    return hipGetLastError();
}

}  // namespace rekv
