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

// The largest finite |x| of each row in FP16: a wave a row.  Memory: 4096 x 4096 in FP16, 34 MB, 9 to 10 us.
__global__ __launch_bounds__(256) void k_row_peaks(int64_t rows, int64_t cols, const uint16_t* X, int64_t ldx, float* peaks)
{
    const int lane = threadIdx.x & 63;
    const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (row >= rows) return;
    int most = 0;
    for (int64_t col = lane * 8; col < cols; col += 64 * 8) {
        uint16_t x[8];
        load_row<F16, 8>(X + row * ldx + col, cols - col, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int magnitude = x[e] & 0x7fff;
            most = max(most, magnitude < 0x7c00 ? magnitude : 0);
        }
    }
    for (int far = 1; far < 64; far *= 2) most = max(most, __shfl_xor(most, far));
    if (lane == 0) peaks[row] = to_float<F16>((uint16_t)most);
}

// dW in FP16.  A row of X times its share of the largest |g| may lie anywhere below the numbers of FP16, so what is held is X times the share times 2^up: the
// largest of all lies in 2^14 .. 2^15 then, and 2^-up times the largest |g| stands in front of the sums.  (No more than leaves 2^-15 times that, which is what
// the sums are multiplied by, a normal number.)
__device__ inline int share_exponent(float most, float peak)
{
    if (!(most > 0.0f && most < __builtin_inff())) return 0;
    // (a peak that is none of FP32's normal numbers says nothing; without it nothing can overflow)
    const int up = peak >= 0x1p-100f && peak < __builtin_inff() ? 15 - __builtin_amdgcn_frexp_expf(peak / most) : 0;
    return min(up, 110 + __builtin_amdgcn_frexp_expf(most));
}
// Rows whose largest element lies 2^18 or more below that are not held so: what FP16 cuts off there, 2^-25, is more than 2^-21 of it.  They are added to dW in
// FP32 (k_far).  A row that is not made smaller than X itself loses nothing that X has.
__device__ inline bool is_far(float own, float share, float peak)
{
    return own != 0.0f && peak > 0.0f && fabsf(share) < 1.0f && fabsf(share) * peak < 0x1p-4f;
}

// Every workgroup finds the largest |g| for itself, so that one launch does.  (With it in front, the slopes and each row's share of it lie in -1 .. 1, and
// a g that is the same for all rows costs no rounding.)  4096 x 4096 states scaled: 35 us in BF16, 41 in FP16; 777 x 1001 states and 10007 words laid
// out 13 and 16; of a step's 12 ms and 151 and 161 us.  (That walk over all rows grows as rows times workgroups.)
template <int TYPE> __global__ __launch_bounds__(256) void k_prepare(Prepare p)
{
    __shared__ float of_wave[4], of_wave_peak[4];
    const int t = threadIdx.x;
    const bool first = blockIdx.x == 0, raised = TYPE == F16 && p.scaled;
    const int64_t begin = (int64_t)blockIdx.x * 256 + t, step = (int64_t)gridDim.x * 256;
    // (W first, which needs no |g|, from the last workgroups on, which have less of X)
    const int64_t of_w = p.w.Y ? p.w.rows * (p.w.width / 8) : 0;
    for (int64_t at = step - 1 - begin; at < of_w; at += step) {
        uint16_t x[8];
        lay_out<TYPE>(p.w, at, x);
    }
    float most = 0.0f, peak = 0.0f;
    for (int64_t r = t; r < p.padded; r += 256) {
        const int target = r < p.rows ? p.targets[r] : NO_TARGET;
        if (target != NO_TARGET) {
            const float own = fabsf(p.g[r * p.g_stride]);
            most = fmaxf(most, own);
            if (raised) peak = fmaxf(peak, own * p.peaks[r]);
        }
        if (first) {
            p.known[r] = target;
            p.lse2[r] = target == BAD_TARGET ? __builtin_nanf("") : (target == NO_TARGET ? 0.0f : p.lse[r] * LOG2E);
        }
    }
    for (int far = 1; far < 64; far *= 2) {
        most = fmaxf(most, __shfl_xor(most, far));
        if (raised) peak = fmaxf(peak, __shfl_xor(peak, far));
    }
    if ((t & 63) == 0) {
        of_wave[t >> 6] = most;
        of_wave_peak[t >> 6] = peak;
    }
    __syncthreads();
    most = fmaxf(fmaxf(of_wave[0], of_wave[1]), fmaxf(of_wave[2], of_wave[3]));
    peak = fmaxf(fmaxf(of_wave_peak[0], of_wave_peak[1]), fmaxf(of_wave_peak[2], of_wave_peak[3]));
    const int up = raised ? share_exponent(most, peak) : 0;
    if (first && t == 0) *p.largest = ldexpf(most, -up);
    // g, times 2^up over the largest |g|
    auto share_of = [&](float own) { return own == 0.0f ? 0.0f : ldexpf(own / most, up); };
    if (first && raised) {
        // the rows that are added in FP32, in their order
        __shared__ int of_wave_far[4];
        int count = 0;
        for (int64_t base = 0; base < p.rows; base += 256) {
            const int64_t r = base + t;
            bool far = false;
            if (r < p.rows && p.targets[r] != NO_TARGET) {
                const float own = p.g[r * p.g_stride];
                far = is_far(own, share_of(own), p.peaks[r]);
            }
            const uint64_t all = __ballot(far);
            if ((t & 63) == 0) of_wave_far[t >> 6] = __popcll(all);
            __syncthreads();
            int at = count + __popcll(all & (((uint64_t)1 << (t & 63)) - 1));
            for (int w = 0; w < 4; ++w) {
                if (w < t >> 6) at += of_wave_far[w];
                count += of_wave_far[w];
            }
            if (far) p.far[at] = (int)r;
            __syncthreads();
        }
        if (t == 0) *p.far_count = count;
    }
    const int64_t of_x = p.x.Y || p.scaled ? p.x.rows * (p.x.width / 8) : 0;
    for (int64_t at = begin; at < of_x; at += step) {
        uint16_t x[8];
        const int64_t row = lay_out<TYPE>(p.x, at, x);
        if (!p.scaled) continue;
        const float own = p.targets[row] == NO_TARGET ? 0.0f : p.g[row * p.g_stride];
        float share = share_of(own);
        if (raised && is_far(own, share, p.peaks[row])) share = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = share == 0.0f ? 0 : from_float<TYPE>(share * to_float<TYPE>(x[e]));
        __builtin_memcpy((uint16_t*)p.scaled + at * 8, x, 16);
    }
}

// What the rows in `far` give to a piece of dW, added to it in FP32 and rounded once more.  Slopes are held times SLOPE_SCALE_F16, their rows whole tiles; a thread
// has eight words and eight columns.  Mostly there are no such rows, and all it takes is a launch, 4.6 us; 100 of 4096 tokens, 16384 words x 4096: 610 us.
template <int DTYPE>
__global__ __launch_bounds__(256) void k_far(int64_t words, int64_t cols, const uint16_t* slopes, int64_t lds, const uint16_t* X, int64_t ldx, const float* g,
                                             int64_t g_stride, const int* far, const int* far_count, typename Elem<DTYPE>::Bits* dW, int64_t ldw)
{
    const int count = *far_count;
    if (count == 0) return;
    const int64_t eights = (cols + 7) / 8, all = (words + 7) / 8 * eights;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < all; at += (int64_t)gridDim.x * 256) {
        const int64_t word = at / eights * 8, col = at % eights * 8;
        float sum[8][8] = {};
        for (int i = 0; i < count; ++i) {
            const int64_t row = far[i];
            const float own = g[row * g_stride];
            uint16_t slope[8], x[8];
            __builtin_memcpy(slope, slopes + row * lds + word, 16);
            load_row<F16, 8>(X + row * ldx + col, cols - col, x);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float of_x = own * to_float<F16>(x[e]);
#pragma unroll
                for (int w = 0; w < 8; ++w) sum[w][e] = __builtin_fmaf(to_float<F16>(slope[w]), of_x, sum[w][e]);
            }
        }
#pragma unroll
        for (int w = 0; w < 8; ++w) {
            if (word + w >= words) break;
            typename Elem<DTYPE>::Bits y[8];
            load_row<DTYPE, 8>(dW + (word + w) * ldw + col, cols - col, y);
#pragma unroll
            for (int e = 0; e < 8; ++e) y[e] = from_float<DTYPE>(__builtin_fmaf(sum[w][e], 1.0f / lmk::SLOPE_SCALE_F16, to_float<DTYPE>(y[e])));
            store_row<DTYPE, 8>(dW + (word + w) * ldw + col, cols - col, y);
        }
    }
}

// (m, s) stands for s 2^m; the sum of two of them.  A part of nothing is (-inf, 0).
__device__ inline float2 join(float2 a, float2 b)
{
    const float m = fmaxf(a.x, b.x), m0 = m == -__builtin_inff() ? 0.0f : m;
    return make_float2(m, a.y * exp2f(a.x - m0) + b.y * exp2f(b.x - m0));
}

// A row's loss and lse from its parts' sum, which leaves out the target's own exponential, so that loss = log(1 + others / own) keeps its digits where
// the target has nearly all of the row.  lse is made from the larger of the two, not as own + loss: a target far below the others (a word that may not be
// taken, at -1e9 or at -infinity) would leave it the digits of its own magnitude, and the gradient takes exponentials of what is off.
__device__ inline void finish(int64_t row, float2 sum, const Targets& targets, const float* at_target, float* loss, float* lse)
{
    const int target = targets[row];
    const float others = LN2 * (sum.x + log2f(sum.y));
    if (target >= 0) {
        const float own = at_target[row];
        const float x = LN2 * ((sum.x - own * LOG2E) + log2f(sum.y));  // log(others / own)
        // (a logit of infinity has no share: infinity less infinity, as among the others)
        const float rest = own == __builtin_inff() ? __builtin_nanf("") : log1pf(expf(-fabsf(x)));
        loss[row] = x > 0.0f ? x + rest : rest;
        lse[row] = (x > 0.0f ? others : own) + rest;
    } else {
        loss[row] = target == BAD_TARGET ? __builtin_nanf("") : 0.0f;
        lse[row] = others;
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

// dX from the sums of the splits, in their order, times what the slopes were divided by.  Memory: 4096 x 4096, 101 MB, 22 to 24 us.
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

hipError_t launch_row_peaks(int64_t rows, int64_t cols, const void* X, int64_t ldx, float* peaks, hipStream_t st)
{
    k_row_peaks<<<dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, st>>>(rows, cols, (const uint16_t*)X, ldx, peaks);
    return hipGetLastError();
}

hipError_t launch_far(int type, int64_t words, int64_t cols, const uint16_t* slopes, int64_t lds, const void* X, int64_t ldx, const float* g, int64_t g_stride,
                      const int* far, const int* far_count, void* dW, int64_t ldw, hipStream_t st)
{
    // (few workgroups: mostly all that they do is to begin and end)
    const unsigned blocks = rounds_of((words + 7) / 8 * ((cols + 7) / 8));
    const dim3 grid(blocks < 512 ? blocks : 512);
    const auto* const x = (const uint16_t*)X;
    if (type == F32) k_far<F32><<<grid, dim3(256), 0, st>>>(words, cols, slopes, lds, x, ldx, g, g_stride, far, far_count, (uint32_t*)dW, ldw);
    if (type == BF16) k_far<BF16><<<grid, dim3(256), 0, st>>>(words, cols, slopes, lds, x, ldx, g, g_stride, far, far_count, (uint16_t*)dW, ldw);
    if (type == F16) k_far<F16><<<grid, dim3(256), 0, st>>>(words, cols, slopes, lds, x, ldx, g, g_stride, far, far_count, (uint16_t*)dW, ldw);
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
