// What stands around the products of the cross entropy (ozimmu_lm_tile.hip): targets, the join of the parts of a row, the slopes' factors, the
// states' gradient.  All of it is bound by memory or by launches.
#include "ozimmu_lm.h"

namespace {

using namespace mxk;
using lmk::BAD_TARGET;
using lmk::NO_TARGET;

constexpr float LN2 = 0.693147180559945309f, LOG2E = 1.44269504088896341f;

__device__ inline int target_of(int64_t y, int64_t words, int64_t ignore) { return y == ignore ? NO_TARGET : (y >= 0 && y < words ? (int)y : BAD_TARGET); }

// 8 elements a thread; `width` is a multiple of 8 and Y's rows are 16-byte aligned
template <int TYPE>
__global__ __launch_bounds__(256) void k_lay_out(int64_t rows, int64_t cols, const uint16_t* X, int64_t ldx, const float* ratio, uint16_t* Y, int64_t ldy,
                                                 int64_t width)
{
    const int64_t eights = width / 8, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= rows * eights) return;
    const int64_t row = at / eights, col = at % eights * 8;
    uint16_t x[8];
    load_row<TYPE, 8>(X + row * ldx + col, cols - col, x);
    if (ratio) {
        const float r = ratio[row];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = r == 0.0f ? 0 : from_float<TYPE>(r * to_float<TYPE>(x[e]));
    }
    __builtin_memcpy(Y + row * ldy + col, x, 16);
}

__global__ __launch_bounds__(256) void k_targets(int64_t rows, int64_t padded, int64_t words, const int64_t* y, int64_t stride, int64_t ignore, int* targets)
{
    const int64_t t = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (t < padded) targets[t] = t < rows ? target_of(y[t * stride], words, ignore) : NO_TARGET;
}

// (m, s) stands for s 2^m; the sum of two of them.  A part of nothing is (-inf, 0).
__device__ inline float2 join(float2 a, float2 b)
{
    const float m = fmaxf(a.x, b.x), m0 = m == -__builtin_inff() ? 0.0f : m;
    return make_float2(m, a.y * exp2f(a.x - m0) + b.y * exp2f(b.x - m0));
}

// 16 rows a workgroup, their parts shared by 64 threads each, joined in a fixed order.  The parts leave out the target's own exponential, so that
// loss = log(1 + others / own) keeps its digits where the target has nearly all of the row.
__global__ __launch_bounds__(1024) void k_join(int64_t rows, int64_t blocks, const float2* parts, int64_t parts_ld, const int* targets, const float* at_target,
                                               float* loss, float* lse)
{
    __shared__ float2 of_wave[16][16];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int64_t row = (int64_t)blockIdx.x * 16 + (lane & 15);  // (parts have rows of whole tiles)
    float2 sum = make_float2(-__builtin_inff(), 0.0f);
    for (int64_t b = t >> 4; b < blocks; b += 64) sum = join(sum, parts[b * parts_ld + row]);
    for (int far = 16; far < 64; far *= 2) {
        const float2 other = make_float2(__shfl_xor(sum.x, far), __shfl_xor(sum.y, far));
        sum = lane & far ? join(other, sum) : join(sum, other);
    }
    if (lane < 16) of_wave[wave][lane] = sum;
    __syncthreads();
    if (t >= 16 || row >= rows) return;
    sum = of_wave[0][t];
    for (int w = 1; w < 16; ++w) sum = join(sum, of_wave[w][t]);
    const int target = targets[row];
    if (target >= 0) {
        const float own = at_target[row];
        const float x = LN2 * ((sum.x - own * LOG2E) + log2f(sum.y));  // log(others / own)
        const float l = x > 0.0f ? x + log1pf(expf(-x)) : log1pf(expf(x));
        loss[row] = l;
        lse[row] = own + l;
    } else {
        loss[row] = target == BAD_TARGET ? __builtin_nanf("") : 0.0f;
        lse[row] = LN2 * (sum.x + log2f(sum.y));
    }
}

// One workgroup: the largest |g| is the same for all.  (With it in front, the slopes and each row's share of it lie in -1 .. 1, and a g that is
// the same for all rows costs no rounding.)
__global__ __launch_bounds__(1024) void k_slopes(int64_t rows, int64_t padded, int64_t words, const int64_t* y, int64_t stride, int64_t ignore, const float* g,
                                                 int64_t g_stride, const float* lse, int* targets, float* lse2, float* ratio, float* largest)
{
    __shared__ float of_wave[16];
    const int t = threadIdx.x;
    float most = 0.0f;
    for (int64_t r = t; r < padded; r += 1024) {
        const int target = r < rows ? target_of(y[r * stride], words, ignore) : NO_TARGET;
        targets[r] = target;
        lse2[r] = target == BAD_TARGET ? __builtin_nanf("") : (target == NO_TARGET ? 0.0f : lse[r] * LOG2E);
        if (target != NO_TARGET) most = fmaxf(most, fabsf(g[r * g_stride]));
    }
    for (int far = 1; far < 64; far *= 2) most = fmaxf(most, __shfl_xor(most, far));
    if ((t & 63) == 0) of_wave[t >> 6] = most;
    __syncthreads();
    for (int w = 0; w < 16; ++w) most = fmaxf(most, of_wave[w]);
    if (t == 0) *largest = most;
    for (int64_t r = t; r < rows; r += 1024) {
        const float own = g[r * g_stride];
        ratio[r] = targets[r] == NO_TARGET || own == 0.0f ? 0.0f : own / most;
    }
}

template <int TYPE>
__global__ __launch_bounds__(256) void k_states(int64_t rows, int64_t cols, const float* parts, int64_t ld, int splits, int64_t split_stride, const float* g,
                                                int64_t g_stride, const int* targets, float scale, void* dX, int64_t ldx)
{
    typedef typename Elem<TYPE>::Bits Bits;
    const int64_t eights = (cols + 7) / 8, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= rows * eights) return;
    const int64_t row = at / eights, col = at % eights * 8;
    Bits x[8];
    if (targets[row] == NO_TARGET) {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = 0;
    } else {
        const float* const p = parts + row * ld + col;
        v4f lo = *(const v4f*)p, hi = *(const v4f*)(p + 4);
        for (int s = 1; s < splits; ++s) {
            lo += *(const v4f*)(p + s * split_stride);
            hi += *(const v4f*)(p + s * split_stride + 4);
        }
        const float f = g[row * g_stride] * scale;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = from_float<TYPE>(f * (e < 4 ? lo[e] : hi[e - 4]));
    }
    store_row<TYPE, 8>((Bits*)dX + row * ldx + col, cols - col, x);
}

template <int TYPE> __global__ __launch_bounds__(256) void k_scale(int64_t rows, int64_t cols, float beta, typename Elem<TYPE>::Bits* X, int64_t ldx)
{
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < rows * cols; at += (int64_t)gridDim.x * 256) {
        typename Elem<TYPE>::Bits* const x = X + at / cols * ldx + at % cols;
        *x = beta == 0.0f ? 0 : from_float<TYPE>(beta * to_float<TYPE>(*x));
    }
}

inline unsigned blocks_of(int64_t threads) { return (unsigned)((threads + 255) / 256); }

}  // namespace

namespace lmk {

hipError_t launch_lay_out(int type, int64_t rows, int64_t cols, const void* X, int64_t ldx, const float* ratio, void* Y, int64_t ldy, int64_t width,
                          hipStream_t st)
{
    const dim3 grid(blocks_of(rows * (width / 8)));
    if (type == BF16) k_lay_out<BF16><<<grid, dim3(256), 0, st>>>(rows, cols, (const uint16_t*)X, ldx, ratio, (uint16_t*)Y, ldy, width);
    if (type == F16) k_lay_out<F16><<<grid, dim3(256), 0, st>>>(rows, cols, (const uint16_t*)X, ldx, ratio, (uint16_t*)Y, ldy, width);
    return hipGetLastError();
}

hipError_t launch_targets(int64_t rows, int64_t padded, int64_t words, const int64_t* y, int64_t stride, int64_t ignore, int* targets, hipStream_t st)
{
    k_targets<<<dim3(blocks_of(padded)), dim3(256), 0, st>>>(rows, padded, words, y, stride, ignore, targets);
    return hipGetLastError();
}

hipError_t launch_join(int64_t rows, int64_t blocks, const float2* parts, int64_t parts_ld, const int* targets, const float* at_target, float* loss,
                       float* lse, hipStream_t st)
{
    k_join<<<dim3((unsigned)((rows + 15) / 16)), dim3(1024), 0, st>>>(rows, blocks, parts, parts_ld, targets, at_target, loss, lse);
    return hipGetLastError();
}

hipError_t launch_slopes(int64_t rows, int64_t padded, int64_t words, const int64_t* y, int64_t stride, int64_t ignore, const float* g, int64_t g_stride,
                         const float* lse, int* targets, float* lse2, float* ratio, float* largest, hipStream_t st)
{
    k_slopes<<<dim3(1), dim3(1024), 0, st>>>(rows, padded, words, y, stride, ignore, g, g_stride, lse, targets, lse2, ratio, largest);
    return hipGetLastError();
}

hipError_t launch_states(int type, int64_t rows, int64_t cols, const float* parts, int64_t ld, int splits, int64_t split_stride, const float* g,
                         int64_t g_stride, const int* targets, float scale, void* dX, int64_t ldx, hipStream_t st)
{
    const dim3 grid(blocks_of(rows * ((cols + 7) / 8)));
    if (type == F32) k_states<F32><<<grid, dim3(256), 0, st>>>(rows, cols, parts, ld, splits, split_stride, g, g_stride, targets, scale, dX, ldx);
    if (type == BF16) k_states<BF16><<<grid, dim3(256), 0, st>>>(rows, cols, parts, ld, splits, split_stride, g, g_stride, targets, scale, dX, ldx);
    if (type == F16) k_states<F16><<<grid, dim3(256), 0, st>>>(rows, cols, parts, ld, splits, split_stride, g, g_stride, targets, scale, dX, ldx);
    return hipGetLastError();
}

hipError_t launch_scale(int type, int64_t rows, int64_t cols, float beta, void* X, int64_t ldx, hipStream_t st)
{
    const dim3 grid(2048);
    if (type == F32) k_scale<F32><<<grid, dim3(256), 0, st>>>(rows, cols, beta, (uint32_t*)X, ldx);
    if (type == BF16) k_scale<BF16><<<grid, dim3(256), 0, st>>>(rows, cols, beta, (uint16_t*)X, ldx);
    if (type == F16) k_scale<F16><<<grid, dim3(256), 0, st>>>(rows, cols, beta, (uint16_t*)X, ldx);
    return hipGetLastError();
}

}  // namespace lmk
