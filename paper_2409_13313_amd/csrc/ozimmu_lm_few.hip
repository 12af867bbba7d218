// The loss of few tokens, or over few words: sums straight from memory, without tiles (ozimmu_lm.h, launch_few_loss).
#include "ozimmu_lm.h"
#include <type_traits>

namespace {

using namespace mxk;
using lmk::FewLoss;

constexpr float LOG2E = 1.44269504088896341f;

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

template <int TYPE> __device__ inline v4f mfma(v4i x, v4i w, v4f c)
{
    if constexpr (TYPE == BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, x), __builtin_bit_cast(v8bf, w), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, x), __builtin_bit_cast(v8h, w), c, 0, 0, 0);
}

// over a row of 16 lanes
template <class F> __device__ inline float over_sixteen(float v, F&& f)
{
    auto moved = [&](auto CTRL) {
        return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), decltype(CTRL)::value, 0xf, 0xf, false));
    };
    v = f(v, moved(std::integral_constant<int, 0xb1>{}));   // lane ^ 1
    v = f(v, moved(std::integral_constant<int, 0x4e>{}));   // lane ^ 2
    v = f(v, moved(std::integral_constant<int, 0x141>{}));  // the other four of eight
    return f(v, moved(std::integral_constant<int, 0x140>{}));  // the other eight of sixteen
}

// A workgroup has 16 MF tokens and 16 PF words.  Its waves share the inner dimension, 64 elements (a whole line of a row) at a time, one piece on its way
// while the other is multiplied; operands come from memory into registers as the matrix instruction wants them, from rows that begin
// anywhere.  The waves' sums meet in LDS in a fixed order, and 16 lanes make a row's part of them.
//
// Bound by reading W: 1 x 4096 x 32768 43 us, 268 MB at 6.2 TB/s, what a kernel that only reads reaches.
//
// ODD: rows may begin at odd elements.  A load of 16 bytes takes twice as long where it does not begin at a whole word, so whole words are loaded, one more
// where the elements begin in the middle of one, and shifted when they are multiplied (1 x 4096 x 32768, rows 4097 apart: 73 us, else 113; 4098 apart 68).
// (A word that is loaded holds an element of the row: what lies beside it in that word, also before the first row or behind the last, is shifted out.)
template <int TYPE, int MF, int PF, int WAVES, bool ODD> __global__ __launch_bounds__(64 * WAVES) void k_few_loss(FewLoss g)
{
    typedef typename Elem<TYPE>::Bits Bits;
    constexpr int PIECE = 64, COLUMNS = 16 * PF, PITCH = COLUMNS + 4;
    __shared__ __align__(16) float sums[WAVES][16 * MF][PITCH];
    const int t = threadIdx.x, lane = t & 63;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t row0 = (int64_t)blockIdx.y * (16 * MF), col0 = (int64_t)blockIdx.x * COLUMNS;
    const Bits* x_at[MF];
    const Bits* w_at[PF];
    // (rows behind the last one: the last one again; what they give is not stored, or masked)
#pragma unroll
    for (int i = 0; i < MF; ++i) x_at[i] = (const Bits*)g.X + min(row0 + 16 * i + (lane & 15), g.m - 1) * g.ldx + (lane >> 4) * 8;
#pragma unroll
    for (int f = 0; f < PF; ++f) w_at[f] = (const Bits*)g.W + min(col0 + 16 * f + (lane & 15), g.p - 1) * g.ldw + (lane >> 4) * 8;
    // ODD: to the word that the row begins in, and the bits in front of it there
    uint32_t x_shift[MF], w_shift[PF];
    if constexpr (ODD) {
        auto to_word = [](const Bits*& p, uint32_t& shift) {
            shift = (uint32_t)(uintptr_t)p % 4 * 8;
            p -= shift / 16;
        };
#pragma unroll
        for (int i = 0; i < MF; ++i) to_word(x_at[i], x_shift[i]);
#pragma unroll
        for (int f = 0; f < PF; ++f) to_word(w_at[f], w_shift[f]);
    }
    const int n = (int)g.n, left = n - (lane >> 4) * 8, pieces = (n + PIECE - 1) / PIECE;

    v4f acc[MF][PF];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int f = 0; f < PF; ++f) acc[i][f] = v4f{0, 0, 0, 0};
    struct Piece {
        v4i x[MF][2], w[PF][2];
        uint32_t x_last[MF][2], w_last[PF][2];  // ODD
    };
    // (no further word where the eight end with the fourth)
    auto last_word = [](const Bits* p, uint32_t shift) {
        uint32_t last;
        __builtin_memcpy(&last, p + (shift ? 8 : 6), 4);
        return last;
    };
    auto shifted = [](v4i v, uint32_t last, uint32_t shift) {
        if constexpr (!ODD) return v;
        const uint32_t a = (uint32_t)v[0], b = (uint32_t)v[1], c = (uint32_t)v[2], d = (uint32_t)v[3];
        return v4i{(int)__builtin_amdgcn_alignbit(b, a, shift), (int)__builtin_amdgcn_alignbit(c, b, shift), (int)__builtin_amdgcn_alignbit(d, c, shift),
                   (int)__builtin_amdgcn_alignbit(last, d, shift)};
    };
    auto load = [&](int piece, Piece& o) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = piece * PIECE + 32 * h;
            const bool there = left - k >= 8;  // (the rest of a row: below)
#pragma unroll
            for (int f = 0; f < PF; ++f) {
                o.w[f][h] = v4i{0, 0, 0, 0};
                if constexpr (ODD) o.w_last[f][h] = 0;
                if (there) {
                    __builtin_memcpy(&o.w[f][h], w_at[f] + k, 16);
                    if constexpr (ODD) o.w_last[f][h] = last_word(w_at[f] + k, w_shift[f]);
                }
            }
#pragma unroll
            for (int i = 0; i < MF; ++i) {
                o.x[i][h] = v4i{0, 0, 0, 0};
                if constexpr (ODD) o.x_last[i][h] = 0;
                if (there) {
                    __builtin_memcpy(&o.x[i][h], x_at[i] + k, 16);
                    if constexpr (ODD) o.x_last[i][h] = last_word(x_at[i] + k, x_shift[i]);
                }
            }
        }
    };
    auto multiply = [&](const Piece& o) __attribute__((always_inline)) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            v4i w[PF];
#pragma unroll
            for (int f = 0; f < PF; ++f) w[f] = shifted(o.w[f][h], o.w_last[f][h], w_shift[f]);
#pragma unroll
            for (int i = 0; i < MF; ++i) {
                const v4i x = shifted(o.x[i][h], o.x_last[i][h], x_shift[i]);
#pragma unroll
                for (int f = 0; f < PF; ++f) acc[i][f] = mfma<TYPE>(x, w[f], acc[i][f]);
            }
        }
    };
    Piece o[2];
    if (wave < pieces) load(wave, o[0]);
    for (int piece = wave; piece < pieces; piece += 2 * WAVES) {
        if (piece + WAVES < pieces) load(piece + WAVES, o[1]);
        multiply(o[0]);
        if (piece + WAVES < pieces) {
            if (piece + 2 * WAVES < pieces) load(piece + 2 * WAVES, o[0]);
            multiply(o[1]);
        }
    }
    // the eight elements that a row ends in, where they are not whole: zeros for the others
    if (n % 8 != 0 && wave == (pieces - 1) % WAVES) {
        if constexpr (ODD) {  // (one by one, and nothing to shift)
            auto to_row = [](const Bits*& p, uint32_t& shift) {
                p += shift / 16;
                shift = 0;
            };
#pragma unroll
            for (int i = 0; i < MF; ++i) to_row(x_at[i], x_shift[i]);
#pragma unroll
            for (int f = 0; f < PF; ++f) to_row(w_at[f], w_shift[f]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int k = (pieces - 1) * PIECE + 32 * h, here = left - k;
            auto rest = [&](const Bits* p) __attribute__((always_inline)) {
                Bits e[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) e[q] = here < 8 && q < here ? p[k + q] : 0;
                v4i v;
                __builtin_memcpy(&v, e, 16);
                return v;
            };
#pragma unroll
            for (int f = 0; f < PF; ++f) o[0].w[f][h] = rest(w_at[f]);
#pragma unroll
            for (int i = 0; i < MF; ++i) o[0].x[i][h] = rest(x_at[i]);
        }
        multiply(o[0]);
    }
    // lane l: word l % 16 of fragment f, tokens 4 (l / 16) + r of fragment i
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int f = 0; f < PF; ++f)
#pragma unroll
            for (int r = 0; r < 4; ++r) sums[wave][16 * i + (lane >> 4) * 4 + r][16 * f + (lane & 15)] = acc[i][f][r];
    __syncthreads();
    const float none = -__builtin_inff();
    for (int at = t >> 4; at < 16 * MF; at += 4 * WAVES) {
        const int64_t row = row0 + at;
        const int64_t y = g.targets.y[min(row, g.m - 1) * g.targets.stride];
        float z[PF], m = none;
#pragma unroll
        for (int f = 0; f < PF; ++f) {
            const int c = 16 * f + (t & 15);
            float v = sums[0][at][c];
#pragma unroll
            for (int w = 1; w < WAVES; ++w) v += sums[w][at][c];
            if (col0 + c >= g.p) {
                v = none;
            } else if (col0 + c == y && y != g.targets.ignore) {
                // (left out of the part)
                g.at_target[row] = v;
                v = none;
            }
            z[f] = v;
            m = fmaxf(m, v);
        }
        m = over_sixteen(m, [](float p, float q) { return fmaxf(p, q); }) * LOG2E;
        const float base = m == none ? 0.0f : m;
        float s = 0.0f;
#pragma unroll
        for (int f = 0; f < PF; ++f) s += __builtin_amdgcn_exp2f(__builtin_fmaf(z[f], LOG2E, -base));
        s = over_sixteen(s, [](float p, float q) { return p + q; });
        if ((t & 15) == 0) g.parts[row * g.parts_ld + blockIdx.x] = make_float2(m, s);
    }
}

template <int TYPE, int MF, int PF, int WAVES> void run(const FewLoss& g, hipStream_t st)
{
    const dim3 grid((unsigned)((g.p + 16 * PF - 1) / (16 * PF)), (unsigned)((g.m + 16 * MF - 1) / (16 * MF)));
    const bool odd = (((uintptr_t)g.X | (uintptr_t)g.W) % 4 | (g.ldx | g.ldw) % 2) != 0;
    odd ? k_few_loss<TYPE, MF, PF, WAVES, true><<<grid, dim3(64 * WAVES), 0, st>>>(g) : k_few_loss<TYPE, MF, PF, WAVES, false><<<grid, dim3(64 * WAVES), 0, st>>>(g);
}
template <int TYPE> void run(const FewLoss& g, const lmk::FewPlan& plan, hipStream_t st)
{
    if (plan.rows == 16 && plan.columns == 16) run<TYPE, 1, 1, 8>(g, st);
    if (plan.rows == 16 && plan.columns == 64) run<TYPE, 1, 4, 8>(g, st);
    if (plan.rows == 32 && plan.columns == 16) run<TYPE, 2, 1, 8>(g, st);
    if (plan.rows == 32 && plan.columns == 64) run<TYPE, 2, 4, 4>(g, st);
    if (plan.rows == 64 && plan.columns == 16) run<TYPE, 4, 1, 4>(g, st);
    if (plan.rows == 64 && plan.columns == 64) run<TYPE, 4, 4, 4>(g, st);
}

}  // namespace

namespace lmk {

hipError_t launch_few_loss(int type, const FewLoss& g, const FewPlan& plan, hipStream_t st)
{
    if (type == BF16) run<BF16>(g, plan, st);
    if (type == F16) run<F16>(g, plan, st);
    return hipGetLastError();
}

}  // namespace lmk
