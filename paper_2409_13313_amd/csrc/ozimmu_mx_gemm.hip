// Product of microscaled 4-bit matrices on the matrix cores: D <- alpha A B^T + beta D (include/ozimmu_mx.h).
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 by 128 x 16 elements of 4 bits, every block of 32 with its scale, and adds
// to 16 x 16 FP32 sums: 16 cycles of a SIMD, 4096 operations a cycle.  The fragments of B are its first operand, so that a lane's four
// sums are four neighbouring columns of one row of D.
#include "ozimmu_mx_convert.h"

namespace {

using namespace mxk;
using namespace mxl;

__device__ inline v8i operand(v4i x) { return __builtin_shufflevector(x, x, 0, 1, 2, 3, -1, -1, -1, -1); }

template <int SEL_B, int SEL_A> __device__ inline v4f mfma(v4i b, int sb, v4i a, int sa, v4f acc)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(b), operand(a), acc, 4, 4, SEL_B, sb, SEL_A, sa);
}

// v: N sums of one row, from column col on, into D
template <int TYPE, int N> __device__ inline void finish(const Gemm& g, int64_t row, int64_t col, const float* v)
{
    typedef typename Elem<TYPE>::Bits Bits;
    if (row >= g.m || col >= g.p) return;
    Bits* const out = (Bits*)g.D + row * g.ldd + col;
    const int64_t left = g.p - col;
    Bits x[N];
    if (g.beta != 0.0f) {
        load_row<TYPE, N>(out, left, x);
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = from_float<TYPE>(g.alpha * v[e] + g.beta * to_float<TYPE>(x[e]));
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = from_float<TYPE>(g.alpha * v[e]);
    }
    store_row<TYPE, N>(out, left, x);
}

// 64 x 64 outputs by four waves, each a quarter of the inner tiles straight from memory into registers; their sums meet in LDS.
template <int TYPE> __global__ __launch_bounds__(256) void k_mx_direct(Gemm g, int64_t KT)
{
    constexpr int PITCH = 64 + 4;  // floats between the rows of a wave's sums: 16 rows fall on different banks
    __shared__ __align__(16) float sums[4 * 64 * PITCH];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int64_t row0 = (int64_t)blockIdx.y * 64, col0 = (int64_t)blockIdx.x * 64;
    const uint8_t* const A = g.A + row0 / TILE_R * KT * TILE_BYTES;
    const uint8_t* const B = g.B + col0 / TILE_R * KT * TILE_BYTES;
    const int qa = (int)(row0 % TILE_R) / 64, qb = (int)(col0 % TILE_R) / 64;
    v4f acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = v4f{0, 0, 0, 0};
    for (int64_t kt = wave; kt < KT; kt += 4) {
        const uint8_t* const ta = A + kt * TILE_BYTES;
        const uint8_t* const tb = B + kt * TILE_BYTES;
        v4i fa[4], fb[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            fa[i] = *(const v4i*)(ta + (4 * qa + i) * FRAGMENT_BYTES + lane * 16);
            fb[i] = *(const v4i*)(tb + (4 * qb + i) * FRAGMENT_BYTES + lane * 16);
        }
        const int sa = *(const int*)(ta + CODE_BYTES + qa * 256 + lane * 4);
        const int sb = *(const int*)(tb + CODE_BYTES + qb * 256 + lane * 4);
#define ROW(I)                                                \
    acc[I][0] = mfma<0, I>(fb[0], sb, fa[I], sa, acc[I][0]); \
    acc[I][1] = mfma<1, I>(fb[1], sb, fa[I], sa, acc[I][1]); \
    acc[I][2] = mfma<2, I>(fb[2], sb, fa[I], sa, acc[I][2]); \
    acc[I][3] = mfma<3, I>(fb[3], sb, fa[I], sa, acc[I][3]);
        ROW(0) ROW(1) ROW(2) ROW(3)
#undef ROW
    }
    // lane l holds columns 4 (l / 16) .. + 3 of row l % 16 of every 16 x 16 tile
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
            *(v4f*)(sums + (wave * 64 + i * 16 + (lane & 15)) * PITCH + j * 16 + 4 * (lane >> 4)) = acc[i][j];
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int r = u * 16 + t / 16, c = (t % 16) * 4;
        v4f s = *(const v4f*)(sums + r * PITCH + c);
#pragma unroll
        for (int w = 1; w < 4; ++w) s += *(const v4f*)(sums + (w * 64 + r) * PITCH + c);
        const float v[4] = {s[0], s[1], s[2], s[3]};
        finish<TYPE, 4>(g, row0 + r, col0 + c, v);
    }
}

template <int TYPE> void direct(const Gemm& g, hipStream_t st)
{
    const dim3 grid((unsigned)((g.p + 63) / 64), (unsigned)((g.m + 63) / 64));
    hipLaunchKernelGGL(k_mx_direct<TYPE>, grid, dim3(256), 0, st, g, inner_tiles(g.n));
}

}  // namespace

namespace mxk {

hipError_t launch_gemm(const Gemm& g, hipStream_t st)
{
    if (g.dtype == F32) direct<F32>(g, st);
    if (g.dtype == BF16) direct<BF16>(g, st);
    if (g.dtype == F16) direct<F16>(g, st);
    return hipGetLastError();
}

}  // namespace mxk
