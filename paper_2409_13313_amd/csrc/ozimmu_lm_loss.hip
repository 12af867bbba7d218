// What stands around the products of the cross entropy (ozimmu_lm_tile.hip): targets, the join of the parts of a row, the slopes' factors, the
// states' gradient.  All of it is bound by memory or by launches.
#include "ozimmu_lm.h"

namespace {

using namespace mxk;
using lmk::BAD_TARGET;
using lmk::LayOut;
using lmk::NO_TARGET;
using lmk::Prepare;
using lmk::Targets;

constexpr float LN2 = 0.693147180559945309f, LOG2E = 1.44269504088896341f;

// Eight elements from `at` (a number of eights) of what is laid out; x: the eight, whose row is returned
template <int TYPE> __device__ inline int64_t lay_out(const LayOut& o, int64_t at, uint16_t* x)
{
    const int64_t eights = o.width / 8, row = at / eights, col = at % eights * 8;
    load_row<TYPE, 8>((const uint16_t*)o.X + row * o.ldx + col, o.cols - col, x);
    if (o.Y) __builtin_memcpy((uint16_t*)o.Y + at * 8, x, 16);
    return row;
}

// Memory: 10007 x 1001 into rows of 1024, 40 MB, 8.2 us.
template <int TYPE> __global__ __launch_bounds__(256) void k_lay_out(LayOut a, LayOut b)
{
    const int64_t of_a = a.rows * (a.width / 8), all = of_a + b.rows * (b.width / 8);
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += (int64_t)gridDim.x * 256) {
        uint16_t x[8];
        at < of_a ? lay_out<TYPE>(a, at, x) : lay_out<TYPE>(b, at - of_a, x);
    }
}

// Every workgroup finds the largest |g| for itself, so that one launch does.  (With it in front, the slopes and each row's share of it lie in -1 .. 1, and
// a g that is the same for all rows costs no rounding.)  4096 x 4096 states scaled: 40 us, 777 x 1001 states and 10007 words laid out 13; of a step's
// 12 ms and 147 us.
template <int TYPE> __global__ __launch_bounds__(256) void k_prepare(Prepare p)
{
    __shared__ float of_wave[4];
    const int t = threadIdx.x;
    const bool first = blockIdx.x == 0;
    const int64_t begin = (int64_t)blockIdx.x * 256 + t, step = (int64_t)gridDim.x * 256;
    // (W first, which needs no |g|, from the last workgroups on, which have less of X)
    const int64_t of_w = p.w.Y ? p.w.rows * (p.w.width / 8) : 0;
    for (int64_t at = step - 1 - begin; at < of_w; at += step) {
        uint16_t x[8];
        lay_out<TYPE>(p.w, at, x);
    }
    float most = 0.0f;
    for (int64_t r = t; r < p.padded; r += 256) {
        const int target = r < p.rows ? p.targets[r] : NO_TARGET;
        if (target != NO_TARGET) most = fmaxf(most, fabsf(p.g[r * p.g_stride]));
        if (first) {
            p.known[r] = target;
            p.lse2[r] = target == BAD_TARGET ? __builtin_nanf("") : (target == NO_TARGET ? 0.0f : p.lse[r] * LOG2E);
        }
    }
    for (int far = 1; far < 64; far *= 2) most = fmaxf(most, __shfl_xor(most, far));
    if ((t & 63) == 0) of_wave[t >> 6] = most;
    __syncthreads();
    most = fmaxf(fmaxf(of_wave[0], of_wave[1]), fmaxf(of_wave[2], of_wave[3]));
    if (first && t == 0) *p.largest = most;
    const int64_t of_x = p.x.Y || p.scaled ? p.x.rows * (p.x.width / 8) : 0;
    for (int64_t at = begin; at < of_x; at += step) {
        uint16_t x[8];
        const int64_t row = lay_out<TYPE>(p.x, at, x);
        if (!p.scaled) continue;
        const float own = p.targets[row] == NO_TARGET ? 0.0f : p.g[row * p.g_stride], ratio = own == 0.0f ? 0.0f : own / most;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = ratio == 0.0f ? 0 : from_float<TYPE>(ratio * to_float<TYPE>(x[e]));
        __builtin_memcpy((uint16_t*)p.scaled + at * 8, x, 16);
    }
}

// (m, s) stands for s 2^m; the sum of two of them.  A part of nothing is (-inf, 0).
__device__ inline float2 join(float2 a, float2 b)
{
    const float m = fmaxf(a.x, b.x), m0 = m == -__builtin_inff() ? 0.0f : m;
    return make_float2(m, a.y * exp2f(a.x - m0) + b.y * exp2f(b.x - m0));
}

// A row's loss and lse from its parts' sum, which leaves out the target's own exponential, so that loss = log(1 + others / own) keeps its digits where
// the target has nearly all of the row.
__device__ inline void finish(int64_t row, float2 sum, const Targets& targets, const float* at_target, float* loss, float* lse)
{
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

// The sum of parts first, first + STEP, ..., `stride` between neighbours, eight loads on their way at a time
template <int STEP> __device__ inline float2 joined(const float2* parts, int64_t stride, int64_t first, int64_t blocks)
{
    float2 sum = make_float2(-__builtin_inff(), 0.0f);
    for (int64_t b = first; b < blocks; b += STEP * 8) {
        float2 part[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) part[u] = b + STEP * u < blocks ? parts[(b + STEP * u) * stride] : make_float2(-__builtin_inff(), 0.0f);
        float most = sum.x;
#pragma unroll
        for (int u = 0; u < 8; ++u) most = fmaxf(most, part[u].x);
        const float base = most == -__builtin_inff() ? 0.0f : most;
        float s = sum.y * exp2f(sum.x - base);
#pragma unroll
        for (int u = 0; u < 8; ++u) s += part[u].y * exp2f(part[u].x - base);
        sum = make_float2(most, s);
    }
    return sum;
}
template <int FROM> __device__ inline float2 over_wave(float2 sum, int lane)
{
    for (int far = FROM; far < 64; far *= 2) {
        const float2 other = make_float2(__shfl_xor(sum.x, far), __shfl_xor(sum.y, far));
        sum = lane & far ? join(other, sum) : join(sum, other);
    }
    return sum;
}

// Parts [column block][row]: 16 rows a workgroup, shared by 64 threads each, joined in a fixed order.  Reading the parts is what it takes: of 4096 rows and
// 131072 words 67 MB, 10.6 us.
__global__ __launch_bounds__(1024) void k_join(int64_t rows, int64_t blocks, const float2* parts, int64_t parts_ld, Targets targets, const float* at_target,
                                               float* loss, float* lse)
{
    __shared__ float2 of_wave[16][16];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int64_t row = (int64_t)blockIdx.x * 16 + (lane & 15);  // (parts have rows of whole tiles)
    float2 sum = over_wave<16>(joined<64>(parts + row, parts_ld, t >> 4, blocks), lane);
    if (lane < 16) of_wave[wave][lane] = sum;
    __syncthreads();
    if (t >= 16 || row >= rows) return;
    sum = of_wave[0][t];
    for (int w = 1; w < 16; ++w) sum = join(sum, of_wave[w][t]);
    finish(row, sum, targets, at_target, loss, lse);
}

// Parts [row][column block], of few tokens: a row by a workgroup, whose threads read neighbours.  1 row of 2048 parts: 3 us less than by 16 rows.
__global__ __launch_bounds__(256) void k_join_rows(int64_t blocks, const float2* parts, int64_t parts_ld, Targets targets, const float* at_target, float* loss,
                                                   float* lse)
{
    __shared__ float2 of_wave[4];
    const int t = threadIdx.x;
    const int64_t row = blockIdx.x;
    const float2 sum = over_wave<1>(joined<256>(parts + row * parts_ld, 1, t, blocks), t & 63);
    if ((t & 63) == 0) of_wave[t >> 6] = sum;
    __syncthreads();
    if (t == 0) finish(row, join(join(of_wave[0], of_wave[1]), join(of_wave[2], of_wave[3])), targets, at_target, loss, lse);
}

// dX from the sums of the splits, in their order, times what the slopes were divided by.  Memory: 4096 x 4096, 101 MB, 21 us.
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
        v4f lo = {0, 0, 0, 0}, hi = lo;
        // (eight splits on their way at a time: 18 tokens x 253 in 235 splits 24 us, one after the other 72)
        for (int s = 0; s < splits; s += 8) {
            v4f part[8][2];
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                part[u][0] = part[u][1] = v4f{0, 0, 0, 0};
                if (s + u < splits) {
                    part[u][0] = *(const v4f*)(p + (s + u) * split_stride);
                    part[u][1] = *(const v4f*)(p + (s + u) * split_stride + 4);
                }
            }
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                lo += part[u][0];
                hi += part[u][1];
            }
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

// (workgroups for that many threads, some rounds of them for many)
inline unsigned rounds_of(int64_t threads)
{
    const int64_t blocks = (threads + 255) / 256;
    return (unsigned)(blocks < 1 ? 1 : blocks < 4096 ? blocks : 4096);
}

hipError_t launch_lay_out(int type, const LayOut& a, const LayOut& b, hipStream_t st)
{
    const dim3 grid(rounds_of(a.rows * (a.width / 8) + b.rows * (b.width / 8)));
    if (type == BF16) k_lay_out<BF16><<<grid, dim3(256), 0, st>>>(a, b);
    if (type == F16) k_lay_out<F16><<<grid, dim3(256), 0, st>>>(a, b);
    return hipGetLastError();
}

hipError_t launch_prepare(int type, const Prepare& p, hipStream_t st)
{
    const dim3 grid(rounds_of((p.x.Y || p.scaled ? p.x.rows * (p.x.width / 8) : 0) + (p.w.Y ? p.w.rows * (p.w.width / 8) : 0)));
    if (type == BF16) k_prepare<BF16><<<grid, dim3(256), 0, st>>>(p);
    if (type == F16) k_prepare<F16><<<grid, dim3(256), 0, st>>>(p);
    return hipGetLastError();
}

hipError_t launch_join_rows(int64_t rows, int64_t blocks, const float2* parts, int64_t parts_ld, const Targets& targets, const float* at_target,
                            float* loss, float* lse, hipStream_t st)
{
    k_join_rows<<<dim3((unsigned)rows), dim3(256), 0, st>>>(blocks, parts, parts_ld, targets, at_target, loss, lse);
    return hipGetLastError();
}

hipError_t launch_join(int64_t rows, int64_t blocks, const float2* parts, int64_t parts_ld, const Targets& targets, const float* at_target, float* loss,
                       float* lse, hipStream_t st)
{
    k_join<<<dim3((unsigned)((rows + 15) / 16)), dim3(1024), 0, st>>>(rows, blocks, parts, parts_ld, targets, at_target, loss, lse);
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
