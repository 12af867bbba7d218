// Weights in 4 bits with a scale per group (ozimmu_lm.h): quantisation, reading back, the plain layout, and the product of rows of 16 bits with
// them straight from the stored form.
#include "ozimmu_lm.h"
#include <type_traits>

namespace {

using namespace mxk;
using namespace lml;
using lmk::Linear;
using lmk::Weights;

typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));

constexpr int64_t COMPUTE_UNITS = 256;

template <int I, int N, class F> __device__ __attribute__((always_inline)) inline void static_for(F&& f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        static_for<I + 1, N>(f);
    }
}

// eight codes, element e at bits 4 e, and the order they are stored in
__device__ inline uint32_t stored_order(uint32_t w)
{
    uint32_t r = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) r |= (w >> (4 * e) & 15u) << (e % 2 * 16 + e / 2 * 4);
    return r;
}
__device__ inline uint32_t plain_order(uint32_t w)
{
    uint32_t r = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) r |= (w >> (e % 2 * 16 + e / 2 * 4) & 15u) << (4 * e);
    return r;
}
__device__ inline int code_at(uint32_t stored, int e) { return (int)(stored >> (e % 2 * 16 + e / 2 * 4) & 15u); }

__device__ inline float scale_float(int stype, uint16_t s) { return stype == BF16 ? to_float<BF16>(s) : to_float<F16>(s); }

// The place of a wave: a block of 16 rows x 128 elements, of which lane l has row l % 16 and 8 elements at 32 j + 8 (l / 16), j < 4
struct Place {
    int64_t block, row, col;
    int lane;
    __device__ inline Place(const Shape& s, int64_t wave) : block(wave), lane(threadIdx.x & 63)
    {
        const int64_t kb = s.inner_blocks();
        row = wave / kb * ROWS + (lane & 15);
        col = wave % kb * INNER + (lane >> 4) * 8;
    }
    __device__ inline int64_t codes() const { return block * BLOCK_BYTES + lane * 16; }
    __device__ inline int64_t scale(const Shape& s, int group) const { return (block * ROWS + (lane & 15)) * s.groups() + group; }  // number
};

__device__ inline float over_lanes_max(float v)
{
    v = fmaxf(v, __shfl_xor(v, 16));
    return fmaxf(v, __shfl_xor(v, 32));
}

// ---- quantisation: a wave a block, so that a group's elements are in four lanes ----
template <int TYPE, int GROUP>
__global__ __launch_bounds__(256) void k_lm_quantize(Shape s, int stype, const typename Elem<TYPE>::Bits* W, int64_t ldw, uint8_t* out)
{
    typedef typename Elem<TYPE>::Bits Bits;
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (wave >= s.blocks()) return;
    const Place at(s, wave);
    const bool inside = at.row < s.p;
    float x[4][8];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        Bits raw[8];
        load_row<TYPE, 8>(W + at.row * ldw + at.col + 32 * j, inside ? s.n - at.col - 32 * j : 0, raw);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[j][e] = to_float<TYPE>(raw[e]);
    }
    constexpr int STEPS = GROUP / 32, GROUPS = 4 / STEPS;
    v4i codes;
    uint16_t scales[GROUPS];
    uint8_t zeros[GROUPS];
#pragma unroll
    for (int q = 0; q < GROUPS; ++q) {
        float hi = 0.0f, lo = 0.0f;
        bool finite = true;
#pragma unroll
        for (int j = q * STEPS; j < (q + 1) * STEPS; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                hi = fmaxf(hi, x[j][e]);
                lo = fminf(lo, x[j][e]);
                finite &= fabsf(x[j][e]) < __builtin_inff();
            }
        hi = over_lanes_max(hi);
        lo = -over_lanes_max(-lo);
        finite = over_lanes_max(finite ? 0.0f : 1.0f) == 0.0f;
        const float range = s.zeros ? (hi - lo) / 15.0f : fmaxf(hi, -lo) / 7.0f;
        // (a range that the type cannot hold: its largest number)
        if (stype == BF16) {
            scales[q] = from_float<BF16>(range);
            if (scales[q] == 0x7f80u) scales[q] = 0x7f7fu;
            if (!finite) scales[q] = 0x7fc0u;
        } else {
            scales[q] = from_float<F16>(range);
            if (scales[q] == 0x7c00u) scales[q] = 0x7bffu;
            if (!finite) scales[q] = 0x7e00u;
        }
        const float scale = scale_float(stype, scales[q]);
        const bool some = scale > 0.0f;
        const float zero = s.zeros ? (some ? fminf(fmaxf(rintf(-lo / scale), 0.0f), 15.0f) : 0.0f) : 8.0f;
        zeros[q] = (uint8_t)zero;
#pragma unroll
        for (int j = q * STEPS; j < (q + 1) * STEPS; ++j) {
            uint32_t w = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float c = some ? fminf(fmaxf(rintf(x[j][e] / scale) + zero, 0.0f), 15.0f) : zero;
                w |= (uint32_t)(at.col + 32 * j + e < s.n ? (int)c : 0) << (e % 2 * 16 + e / 2 * 4);
            }
            codes[j] = (int)w;
        }
        if (at.col - (at.lane >> 4) * 8 + q * GROUP >= s.n) scales[q] = 0;
    }
    if (!inside) return;
    *(v4i*)(out + at.codes()) = codes;
    if (at.lane < 16) {
#pragma unroll
        for (int q = 0; q < GROUPS; ++q) {
            ((uint16_t*)(out + s.scales_at()))[at.scale(s, q)] = scales[q];
            if (s.zeros) (out + s.zeros_at())[at.scale(s, q)] = zeros[q];
        }
    }
}

// ---- reading back ----
template <int TYPE>
__global__ __launch_bounds__(256) void k_lm_dequantize(Weights w, int64_t row0, int64_t rows, int64_t cols, typename Elem<TYPE>::Bits* X, int64_t ldx)
{
    typedef typename Elem<TYPE>::Bits Bits;
    const Shape& s = w.shape;
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6) + row0 / ROWS * s.inner_blocks();  // (row0: a multiple of 16)
    if (wave >= (row0 + rows + ROWS - 1) / ROWS * s.inner_blocks()) return;
    const Place at(s, wave);
    if (at.row >= row0 + rows) return;
    const v4i codes = *(const v4i*)(w.data + at.codes());
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int q = j * 32 / s.group;
        const float scale = scale_float(w.stype, ((const uint16_t*)(w.data + s.scales_at()))[at.scale(s, q)]);
        const int zero = s.zeros ? (w.data + s.zeros_at())[at.scale(s, q)] : 8;
        Bits x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e)
            x[e] = at.col + 32 * j + e < s.n ? from_float<TYPE>((float)(code_at((uint32_t)codes[j], e) - zero) * scale) : 0;
        store_row<TYPE, 8>(X + (at.row - row0) * ldx + at.col + 32 * j, cols - at.col - 32 * j, x);
    }
}

// ---- the plain layout ----
__global__ __launch_bounds__(256) void k_lm_pack(Shape s, const uint8_t* codes, int64_t ldc, const uint16_t* scales, int64_t lds, const uint8_t* zeros,
                                                 int64_t ldz, uint8_t* out)
{
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (wave >= s.blocks()) return;
    const Place at(s, wave);
    if (at.row >= s.p) return;
    v4i words;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t w = 0;
        const int64_t col = at.col + 32 * j;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            if (col + 2 * b >= s.n) break;
            uint32_t c = codes[at.row * ldc + col / 2 + b];
            if (col + 2 * b + 1 >= s.n) c &= 15u;
            w |= c << (8 * b);
        }
        words[j] = (int)stored_order(w);
    }
    *(v4i*)(out + at.codes()) = words;
    if (at.lane < 16) {
        const int64_t first = (at.col - (at.lane >> 4) * 8) / s.group, all = (s.n + s.group - 1) / s.group;
        for (int q = 0; q < s.groups(); ++q) {
            const bool real = first + q < all;
            ((uint16_t*)(out + s.scales_at()))[at.scale(s, q)] = real ? scales[at.row * lds + first + q] : 0;
            if (s.zeros) (out + s.zeros_at())[at.scale(s, q)] = real ? zeros[at.row * ldz + first + q] & 15 : 0;
        }
    }
}

__global__ __launch_bounds__(256) void k_lm_unpack(Shape s, const uint8_t* in, uint8_t* codes, int64_t ldc, uint16_t* scales, int64_t lds, uint8_t* zeros,
                                                   int64_t ldz)
{
    const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (wave >= s.blocks()) return;
    const Place at(s, wave);
    if (at.row >= s.p) return;
    const v4i words = *(const v4i*)(in + at.codes());
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t w = plain_order((uint32_t)words[j]);
        const int64_t col = at.col + 32 * j;
#pragma unroll
        for (int b = 0; b < 4; ++b)
            if (col + 2 * b < s.n) codes[at.row * ldc + col / 2 + b] = (uint8_t)(w >> (8 * b));
    }
    if (at.lane < 16) {
        const int64_t first = (at.col - (at.lane >> 4) * 8) / s.group, all = (s.n + s.group - 1) / s.group;
        for (int q = 0; q < s.groups() && first + q < all; ++q) {
            scales[at.row * lds + first + q] = ((const uint16_t*)(in + s.scales_at()))[at.scale(s, q)];
            if (s.zeros) zeros[at.row * ldz + first + q] = (in + s.zeros_at())[at.scale(s, q)];
        }
    }
}

// ---- D <- alpha X W^T + beta D from the stored form: 16 MF rows of X and 16 PF of W by a workgroup ----
//
// A code becomes a 16-bit number by one mask and one or: 128 + q as BF16, 1024 + q as FP16, both exact.  FP16 pairs then have 1024 + zero
// taken off, again exactly; BF16 has no such instruction, so its groups are summed with the 128 and (128 + zero) times the sum of X, which one more
// matrix instruction a step gives, is taken off the group's sum in FP32.  So no weight is rounded: a group's sum is multiplied by its scale in FP32.
// The waves share the blocks of 128 inner elements; their sums meet in LDS in a fixed order.
template <int XTYPE> __device__ inline v4f mfma(v4i x, v4i w, v4f c)
{
    if constexpr (XTYPE == BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8bf, x), __builtin_bit_cast(v8bf, w), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8h, x), __builtin_bit_cast(v8h, w), c, 0, 0, 0);
}

template <int XTYPE> __device__ inline v4i numbers(uint32_t w, float zero)
{
    v4i r;
    if constexpr (XTYPE == BF16) {
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = (int)((w >> (4 * i) & 0x000f000fu) | 0x43004300u);
    } else {
        const _Float16 off = (_Float16)(-1024.0f - zero);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const v2h v = __builtin_bit_cast(v2h, (w >> (4 * i) & 0x000f000fu) | 0x64006400u) + v2h{off, off};
            r[i] = __builtin_bit_cast(int, v);
        }
    }
    return r;
}

// FOUR: at most four rows, row i at place 4 i of the fragment, so that a lane's first sum is the one that counts
template <int XTYPE, int GROUP, int MF, int PF, int WAVES, int BLOCKS, bool FOUR>
__global__ __launch_bounds__(64 * WAVES) void k_lm_direct(Linear g, Weights w)
{
    static_assert(!FOUR || MF == 1, "four rows are one fragment");
    typedef typename Elem<XTYPE>::Bits Bits;
    constexpr int STEPS = GROUP / 32, GROUPS = 4 / STEPS, R = FOUR ? 1 : 4;
    __shared__ __align__(16) float sums[WAVES][MF][PF][64][R];
    const Shape& s = w.shape;
    const int t = threadIdx.x, lane = t & 63;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int64_t KB = s.inner_blocks(), last_rows = s.row_blocks() - 1;
    const int64_t pb0 = (int64_t)blockIdx.x * PF, row0 = (int64_t)blockIdx.y * (16 * MF);
    const uint8_t* code_at[PF];
    const uint8_t* scale_at[PF];
    const uint8_t* zero_at[PF];
#pragma unroll
    for (int f = 0; f < PF; ++f) {
        // (blocks of rows behind the last one: the last one again, not stored)
        const int64_t block = (pb0 + f < last_rows ? pb0 + f : last_rows) * KB;
        code_at[f] = w.data + block * BLOCK_BYTES + lane * 16;
        scale_at[f] = w.data + s.scales_at() + (block * ROWS + (lane & 15)) * (GROUPS * 2);
        zero_at[f] = w.data + s.zeros_at() + (block * ROWS + (lane & 15)) * GROUPS;
    }
    const Bits* x_at[MF];
#pragma unroll
    for (int i = 0; i < MF; ++i) {
        const int64_t row = row0 + 16 * i + (FOUR ? (lane & 15) >> 2 : lane & 15);
        x_at[i] = (const Bits*)g.X + (row < g.m ? row : g.m - 1) * g.ldx + (lane >> 4) * 8;
    }
    const int64_t left = s.n - (lane >> 4) * 8;  // elements of a row from this lane's first on

    float acc[MF][PF][R];
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int f = 0; f < PF; ++f)
#pragma unroll
            for (int r = 0; r < R; ++r) acc[i][f][r] = 0.0f;

    struct Stored {
        v4i code;
        uint16_t scale[GROUPS];
        uint8_t zero[GROUPS];
    };
    auto load = [&](int f, int64_t kb, Stored& o) __attribute__((always_inline)) {
        o.code = *(const v4i*)(code_at[f] + kb * BLOCK_BYTES);
        __builtin_memcpy(o.scale, __builtin_assume_aligned(scale_at[f] + kb * (ROWS * GROUPS * 2), 2 * GROUPS), sizeof(o.scale));
        if (s.zeros)
            __builtin_memcpy(o.zero, __builtin_assume_aligned(zero_at[f] + kb * (ROWS * GROUPS), GROUPS), sizeof(o.zero));
        else
#pragma unroll
            for (int q = 0; q < GROUPS; ++q) o.zero[q] = 8;
    };
    const v4i ones = {0x3f803f80, 0x3f803f80, 0x3f803f80, 0x3f803f80};
    auto multiply = [&](const Stored (&o)[PF], const v4i (&x)[MF][4]) __attribute__((always_inline)) {
        static_for<0, GROUPS>([&](auto Q) __attribute__((always_inline)) {
            constexpr int q = decltype(Q)::value;
            v4f xs[MF];
            if constexpr (XTYPE == BF16)
#pragma unroll
                for (int i = 0; i < MF; ++i) {
                    xs[i] = v4f{0, 0, 0, 0};
#pragma unroll
                    for (int j = q * STEPS; j < (q + 1) * STEPS; ++j) xs[i] = mfma<XTYPE>(x[i][j], ones, xs[i]);
                }
#pragma unroll
            for (int f = 0; f < PF; ++f) {
                const float scale = scale_float(w.stype, o[f].scale[q]), zero = (float)o[f].zero[q];
                v4f c[MF];
#pragma unroll
                for (int i = 0; i < MF; ++i) c[i] = v4f{0, 0, 0, 0};
#pragma unroll
                for (int j = q * STEPS; j < (q + 1) * STEPS; ++j) {
                    const v4i b = numbers<XTYPE>((uint32_t)o[f].code[j], zero);
#pragma unroll
                    for (int i = 0; i < MF; ++i) c[i] = mfma<XTYPE>(x[i][j], b, c[i]);
                }
#pragma unroll
                for (int i = 0; i < MF; ++i)
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const float sum = XTYPE == BF16 ? __builtin_fmaf(-128.0f - zero, xs[i][r], c[i][r]) : c[i][r];
                        acc[i][f][r] = __builtin_fmaf(scale, sum, acc[i][f][r]);
                    }
            }
        });
    };

    for (int64_t kb0 = wave; kb0 < KB; kb0 += WAVES * BLOCKS) {
        Stored o[BLOCKS][PF];
        v4i x[BLOCKS][MF][4];
#pragma unroll
        for (int u = 0; u < BLOCKS; ++u) {
            // (a block behind the last one: the last one again, with zeros for X)
            const int64_t kb = kb0 + u * WAVES, there = kb < KB ? kb : KB - 1;
#pragma unroll
            for (int f = 0; f < PF; ++f) load(f, there, o[u][f]);
#pragma unroll
            for (int i = 0; i < MF; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    x[u][i][j] = v4i{0, 0, 0, 0};
                    if (kb < KB && left - kb * INNER - 32 * j >= 8) __builtin_memcpy(&x[u][i][j], x_at[i] + kb * INNER + 32 * j, 16);
                }
        }
#pragma unroll
        for (int u = 0; u < BLOCKS; ++u) multiply(o[u], x[u]);
    }
    // the eight elements that a row ends in, where they are not whole: zeros for the others
    if (s.n % 8 != 0 && wave == (int)((KB - 1) % WAVES)) {
        Stored o[PF];
        v4i x[MF][4];
#pragma unroll
        for (int f = 0; f < PF; ++f) load(f, KB - 1, o[f]);
#pragma unroll
        for (int i = 0; i < MF; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t here = left - (KB - 1) * INNER - 32 * j;
                Bits e[8];
#pragma unroll
                for (int n = 0; n < 8; ++n) e[n] = here < 8 && n < here ? x_at[i][(KB - 1) * INNER + 32 * j + n] : 0;
                __builtin_memcpy(&x[i][j], e, 16);
            }
        multiply(o, x);
    }
#pragma unroll
    for (int i = 0; i < MF; ++i)
#pragma unroll
        for (int f = 0; f < PF; ++f)
#pragma unroll
            for (int r = 0; r < R; ++r) sums[wave][i][f][lane][r] = acc[i][f][r];
    __syncthreads();
    // lane l: column l % 16 of fragment f, rows 4 (l / 16) + r (FOUR: row l / 16)
    for (int at = t; at < MF * PF * 64; at += 64 * WAVES) {
        const int l = at & 63, f = at / 64 % PF, i = at / (64 * PF);
        const int64_t col = (pb0 + f) * ROWS + (l & 15);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float v = sums[0][i][f][l][r];
#pragma unroll
            for (int u = 1; u < WAVES; ++u) v += sums[u][i][f][l][r];
            const int64_t row = row0 + 16 * i + (FOUR ? l >> 4 : (l >> 4) * 4 + r);
            if (row >= g.m || col >= s.p) continue;
            const int64_t to = row * g.ldd + col;
            auto out = [&](auto D) {
                constexpr int DTYPE = decltype(D)::value;
                typedef typename Elem<DTYPE>::Bits Out;
                Out* const d = (Out*)g.D + to;
                *d = from_float<DTYPE>(g.beta != 0.0f ? g.alpha * v + g.beta * to_float<DTYPE>(*d) : g.alpha * v);
            };
            if (g.dtype == F32) out(std::integral_constant<int, F32>{});
            if (g.dtype == BF16) out(std::integral_constant<int, BF16>{});
            if (g.dtype == F16) out(std::integral_constant<int, F16>{});
        }
    }
}

template <int XTYPE, int GROUP, int MF, int PF, int WAVES, int BLOCKS, bool FOUR> void direct(const Linear& g, const Weights& w, hipStream_t st)
{
    const dim3 grid((unsigned)((w.shape.row_blocks() + PF - 1) / PF), (unsigned)((g.m + 16 * MF - 1) / (16 * MF)));
    k_lm_direct<XTYPE, GROUP, MF, PF, WAVES, BLOCKS, FOUR><<<grid, dim3(64 * WAVES), 0, st>>>(g, w);
}

template <int XTYPE, int GROUP> void direct(const Linear& g, const Weights& w, hipStream_t st)
{
    const int64_t units = w.shape.row_blocks();
    if (g.m <= 4) {
        if (units <= COMPUTE_UNITS) return direct<XTYPE, GROUP, 1, 1, 16, 2, true>(g, w, st);
        if (units <= 2 * COMPUTE_UNITS) return direct<XTYPE, GROUP, 1, 2, 16, 1, true>(g, w, st);
        return direct<XTYPE, GROUP, 1, 4, 8, 1, true>(g, w, st);
    }
    if (g.m <= 16) {
        if (units <= COMPUTE_UNITS) return direct<XTYPE, GROUP, 1, 1, 8, 2, false>(g, w, st);
        if (units <= 2 * COMPUTE_UNITS) return direct<XTYPE, GROUP, 1, 2, 8, 2, false>(g, w, st);
        return direct<XTYPE, GROUP, 1, 4, 8, 1, false>(g, w, st);
    }
    if (g.m <= 32) return direct<XTYPE, GROUP, 2, 2, 8, 1, false>(g, w, st);
    return direct<XTYPE, GROUP, 4, 2, 8, 1, false>(g, w, st);
}
template <int XTYPE> void direct(const Linear& g, const Weights& w, hipStream_t st)
{
    if (w.shape.group == 32) direct<XTYPE, 32>(g, w, st);
    if (w.shape.group == 64) direct<XTYPE, 64>(g, w, st);
    if (w.shape.group == 128) direct<XTYPE, 128>(g, w, st);
}

inline unsigned four_waves_each(int64_t waves) { return (unsigned)((waves + 3) / 4); }

template <int TYPE> void quantize(const void* W, int64_t ldw, const Shape& s, int stype, void* packed, hipStream_t st)
{
    const dim3 grid(four_waves_each(s.blocks()));
    const auto* w = (const typename Elem<TYPE>::Bits*)W;
    if (s.group == 32) k_lm_quantize<TYPE, 32><<<grid, dim3(256), 0, st>>>(s, stype, w, ldw, (uint8_t*)packed);
    if (s.group == 64) k_lm_quantize<TYPE, 64><<<grid, dim3(256), 0, st>>>(s, stype, w, ldw, (uint8_t*)packed);
    if (s.group == 128) k_lm_quantize<TYPE, 128><<<grid, dim3(256), 0, st>>>(s, stype, w, ldw, (uint8_t*)packed);
}

}  // namespace

namespace lmk {

hipError_t launch_quantize(int type, const void* W, int64_t ldw, const Shape& s, int stype, void* packed, hipStream_t st)
{
    if (type == F32) quantize<F32>(W, ldw, s, stype, packed, st);
    if (type == BF16) quantize<BF16>(W, ldw, s, stype, packed, st);
    if (type == F16) quantize<F16>(W, ldw, s, stype, packed, st);
    return hipGetLastError();
}

hipError_t launch_dequantize(int type, const Weights& w, int64_t row0, int64_t rows, int64_t cols, void* X, int64_t ldx, hipStream_t st)
{
    const dim3 grid(four_waves_each(((row0 + rows + ROWS - 1) / ROWS - row0 / ROWS) * w.shape.inner_blocks()));
    if (type == F32) k_lm_dequantize<F32><<<grid, dim3(256), 0, st>>>(w, row0, rows, cols, (uint32_t*)X, ldx);
    if (type == BF16) k_lm_dequantize<BF16><<<grid, dim3(256), 0, st>>>(w, row0, rows, cols, (uint16_t*)X, ldx);
    if (type == F16) k_lm_dequantize<F16><<<grid, dim3(256), 0, st>>>(w, row0, rows, cols, (uint16_t*)X, ldx);
    return hipGetLastError();
}

hipError_t launch_pack(const Shape& s, const uint8_t* codes, int64_t ldc, const void* scales, int64_t lds, const uint8_t* zeros, int64_t ldz, void* packed,
                       hipStream_t st)
{
    k_lm_pack<<<dim3(four_waves_each(s.blocks())), dim3(256), 0, st>>>(s, codes, ldc, (const uint16_t*)scales, lds, zeros, ldz, (uint8_t*)packed);
    return hipGetLastError();
}

hipError_t launch_unpack(const Shape& s, const void* packed, uint8_t* codes, int64_t ldc, void* scales, int64_t lds, uint8_t* zeros, int64_t ldz,
                         hipStream_t st)
{
    k_lm_unpack<<<dim3(four_waves_each(s.blocks())), dim3(256), 0, st>>>(s, (const uint8_t*)packed, codes, ldc, (uint16_t*)scales, lds, zeros, ldz);
    return hipGetLastError();
}

hipError_t launch_direct(const Linear& l, const Weights& w, hipStream_t st)
{
    if (l.xtype == BF16) direct<BF16>(l, w, st);
    if (l.xtype == F16) direct<F16>(l, w, st);
    return hipGetLastError();
}

}  // namespace lmk
