// Rotary positions with several axes, and the append of new keys and values to a paged cache with the rotation on the way.
//
//   (x_a, x_b) -> (x_a cos t - x_b sin t, x_a sin t + x_b cos t),  t = position[axis of the pair] * base^(-2i / D)
//
// Bound: HBM for many tokens, the launch and one or two round trips for few.  A unit of work is one 16-byte chunk of a head
// vector and its partner half a vector on, which hold both members of their pairs in either layout.  A lane keeps one
// chunk position of one token and walks that token's heads, so that its angles (formed in double precision, reduced to a
// fraction of a turn) are worked out once for all of them.
#include "common.h"
#include "paged.h"

namespace rekv {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
constexpr int WAVES = 4;

// waves_per_token: the wavefronts of a workgroup that share a token's heads (1, 2 or 4).
template <bool BF16, bool APPEND>
__global__ __launch_bounds__(WAVES * 64) void rotate_kernel(RotateArgs a, int waves_per_token) {
    constexpr int EPC = BF16 ? 8 : 4;            // elements per 16-byte chunk
    constexpr int ES = BF16 ? 2 : 4;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tokens_per_block = WAVES / waves_per_token;
    const int64_t tok64 = (int64_t)blockIdx.x * tokens_per_block + wave / waves_per_token;
    if (tok64 >= a.n_tokens) return;
    const int tok = (int)tok64;
    const int half = a.head_dim / 2, cpr = half / EPC;           // chunk pairs per head vector
    const int per_wave = 64 / cpr;                               // heads a wavefront takes at a time
    const int c = lane % cpr;
    int h0 = lane / cpr;
    const bool idle = h0 >= per_wave;
    h0 += (wave % waves_per_token) * per_wave;

    char *k_row = nullptr, *v_row = nullptr;
    int index = 0;
    bool keep = false;                                           // whether the token goes into a page
    if (APPEND) {
        const PagedBatch& b = a.b;
        if (tok < scalar_word(b.token_start, 0) || tok >= scalar_word(b.token_start, b.n_seqs)) return;
        const int s = find_sequence(b, lane, tok, [](int, int start) { return start; });
        index = clamped(scalar_word(b.kv_len, s), 0, 1 << 30) - scalar_word(b.token_start, s + 1) + tok;
        if (index >= 0 && index < b.capacity) {
            const int slot = (int)quot((uint32_t)index, b.by_page), page = scalar_word(b.page_table + s * b.table_stride, slot);
            keep = page >= 0 && page < b.n_pages;
            const int64_t row = ((int64_t)page * b.by_page.d + (index - slot * (int)b.by_page.d)) * a.n_kv_heads * a.head_dim * ES;
            k_row = static_cast<char*>(b.k_pages) + row;
            v_row = static_cast<char*>(b.v_pages) + row;
        }
    }
    if (idle) return;

    const bool turn = a.r.n_axes > 0;
    float cs[EPC], sn[EPC];
#pragma unroll
    for (int e = 0; e < EPC; ++e) {
        cs[e] = 1.f;
        sn[e] = 0.f;
        if (!turn) continue;
        // pair e of this lane's two chunks: element e of both, or neighbours, the first half of them in the first chunk
        const int i = a.r.interleaved ? (e >= EPC / 2 ? half / 2 : 0) + c * (EPC / 2) + e % (EPC / 2) : c * EPC + e;
        const int pos = APPEND && !a.positions ? index : a.positions[a.r.axis[i] * a.positions_stride + tok];
        const double turns = (double)pos * a.r.turns[i];
        const float fr = (float)(turns - rint(turns));           // in [-0.5, 0.5]
        sincospif(2.f * fr, &sn[e], &cs[e]);
    }
    auto rotate = [&](const char* src, char* dst) {
        u32x4 lo = *reinterpret_cast<const u32x4*>(src), hi = *reinterpret_cast<const u32x4*>(src + half * ES);
        if (turn) {
            float x[2 * EPC];                    // first chunk, then its partner
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (BF16) {
                    x[2 * i] = __uint_as_float(lo[i] << 16);
                    x[2 * i + 1] = __uint_as_float(lo[i] & 0xffff0000u);
                    x[EPC + 2 * i] = __uint_as_float(hi[i] << 16);
                    x[EPC + 2 * i + 1] = __uint_as_float(hi[i] & 0xffff0000u);
                } else {
                    x[i] = __uint_as_float(lo[i]);
                    x[EPC + i] = __uint_as_float(hi[i]);
                }
            }
            if (a.r.interleaved) {
#pragma unroll
                for (int e = 0; e < EPC; ++e) {
                    const int ia = 2 * e;        // the chunks one after the other
                    const float p = x[ia], q = x[ia + 1];
                    x[ia] = p * cs[e] - q * sn[e];
                    x[ia + 1] = p * sn[e] + q * cs[e];
                }
            } else {
#pragma unroll
                for (int e = 0; e < EPC; ++e) {
                    const float p = x[e], q = x[EPC + e];
                    x[e] = p * cs[e] - q * sn[e];
                    x[EPC + e] = p * sn[e] + q * cs[e];
                }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if (BF16) {
                    lo[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[2 * i], x[2 * i + 1]}), bf16x2));
                    hi[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{x[EPC + 2 * i], x[EPC + 2 * i + 1]}), bf16x2));
                } else {
                    lo[i] = __float_as_uint(x[i]);
                    hi[i] = __float_as_uint(x[EPC + i]);
                }
            }
        }
        *reinterpret_cast<u32x4*>(dst) = lo;
        *reinterpret_cast<u32x4*>(dst + half * ES) = hi;
    };
    const int step = per_wave * waves_per_token;
    const size_t at = (size_t)c * 16, head_b = (size_t)a.head_dim * ES;
    if (a.q) {
        const char* src = static_cast<const char*>(a.q) + (int64_t)tok * a.q_stride * ES + at;
        char* dst = static_cast<char*>(a.q_out) + (int64_t)tok * a.q_out_stride * ES + at;
        for (int h = h0; h < a.n_q_heads; h += step) rotate(src + h * head_b, dst + h * head_b);
    }
    if (APPEND && keep) {
        const char* ks = static_cast<const char*>(a.k) + (int64_t)tok * a.k_stride * ES + at;
        const char* vs = static_cast<const char*>(a.v) + (int64_t)tok * a.v_stride * ES + at;
        for (int h = h0; h < a.n_kv_heads; h += step) {
            rotate(ks + h * head_b, k_row + at + h * head_b);
            const u32x4 lo = *reinterpret_cast<const u32x4*>(vs + h * head_b), hi = *reinterpret_cast<const u32x4*>(vs + h * head_b + half * ES);
            *reinterpret_cast<u32x4*>(v_row + at + h * head_b) = lo;
            *reinterpret_cast<u32x4*>(v_row + at + h * head_b + half * ES) = hi;
        }
    }
}

}  // namespace

hipError_t rotate_launch(const RotateArgs& a, int dtype, hipStream_t stream) {
    const int wpt = a.n_tokens >= 2048 ? 1 : WAVES;
    const dim3 grid((unsigned)(((int64_t)a.n_tokens * wpt + WAVES - 1) / WAVES)), block(WAVES * 64);
    if (dtype == REKV_BF16) {
        if (a.k) hipLaunchKernelGGL((rotate_kernel<true, true>), grid, block, 0, stream, a, wpt);
        else hipLaunchKernelGGL((rotate_kernel<true, false>), grid, block, 0, stream, a, wpt);
    } else {
        if (a.k) hipLaunchKernelGGL((rotate_kernel<false, true>), grid, block, 0, stream, a, wpt);
        else hipLaunchKernelGGL((rotate_kernel<false, false>), grid, block, 0, stream, a, wpt);
    }
    return hipGetLastError();
}

}  // namespace rekv
