// Quantisation to the microscaled 4-bit form, reading back, and the plain layout of checkpoints (include/ozimmu_mx.h).
//
// All of it moves memory: an element is read in 2 or 4 bytes and written in 17/32 of one (or the other way round), with two
// dozen operations for eight elements between.
#include "ozimmu_mx_convert.h"

namespace {

using namespace mxk;
using namespace mxl;

// Blocks along the rows.  A workgroup takes 64 rows x 128 columns (a quarter of a tile): thread t the eight elements t % 16 of
// the four rows at place t / 16 of the fragments, so that 16 lanes read 128 columns of a row side by side; four lanes hold a block and
// share its maximum.
template <int TYPE> __device__ inline void quantize_rows(const typename Elem<TYPE>::Bits (&x)[4][8], int64_t row0, int64_t rows, uint8_t* tile, int chunk)
{
    const int c = chunk >> 2, sub = chunk & 3;
    uint32_t scales = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        uint32_t amax = max_magnitude<TYPE, 8>(x[i]);
#pragma unroll
        for (int d = 1; d < 4; d *= 2) {
            const uint32_t o = (uint32_t)__shfl_xor((int)amax, d);
            amax = o > amax ? o : amax;
        }
        const uint32_t b = scale_byte(f32_bits<TYPE>(amax));
        scales |= b << (8 * i);
        const int64_t row = row0 + row_of(i, 0);
        if (row < rows) *(uint32_t*)(tile + code_offset((int)(row % TILE_R), c) + 4 * sub) = codes8<TYPE>(x[i], scale_value(b));
    }
    // (the scales of rows that are not there are those of zeros)
    if (sub == 0 && row0 < rows) *(uint32_t*)(tile + scale_offset((int)(row0 % TILE_R), c)) = scales;
}

template <int TYPE>
__global__ __launch_bounds__(256) void k_mx_quantize_rows(int64_t rows, int64_t n, const typename Elem<TYPE>::Bits* X, int64_t ldx,
                                                          uint8_t* out, int64_t KT)
{
    typename Elem<TYPE>::Bits x[4][8];
    const int t = threadIdx.x, chunk = t & 15;
    const int64_t kt = blockIdx.x, row0 = (int64_t)blockIdx.y * 64 + row_of(0, t >> 4), col = kt * TILE_K + chunk * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t row = row0 + row_of(i, 0);
        load_row<TYPE, 8>(X + row * ldx + col, row < rows ? n - col : 0, x[i]);
    }
    quantize_rows<TYPE>(x, row0, rows, out + ((row0 / TILE_R) * KT + kt) * TILE_BYTES, chunk);
}

// Blocks along the columns, and along the rows too where by_row is given.  A workgroup takes 128 rows x 128 columns, read as above (rows
// quantised on the way) and left in LDS as they are; then wave w takes block w of all columns, lane l columns 2 l and 2 l + 1: it reads
// their 32 rows one after the other, 64 lanes a row side by side, so that a block is one lane's.
template <int TYPE>
__global__ __launch_bounds__(256) void k_mx_quantize_cols(int64_t rows, int64_t n, const typename Elem<TYPE>::Bits* X, int64_t ldx,
                                                          uint8_t* by_row, uint8_t* by_col, int64_t KT_row, int64_t KT_col)
{
    typedef typename Elem<TYPE>::Bits Bits;
    __shared__ __align__(16) Bits held[128 * 128];
    const int t = threadIdx.x, chunk = t & 15;
    // (one number for both: there may be more row tiles than a grid has in its second dimension)
    const uint32_t tiles = (uint32_t)((n + 127) / 128), tile_col = blockIdx.x % tiles, tile_row = blockIdx.x / tiles;
    const int64_t col0 = (int64_t)tile_col * 128, first = (int64_t)tile_row * 128;
    Bits x[2][4][8];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int64_t row = first + h * 64 + row_of(i, t >> 4);
            load_row<TYPE, 8>(X + row * ldx + col0 + chunk * 8, row < rows ? n - col0 - chunk * 8 : 0, x[h][i]);
        }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < 4; ++i) __builtin_memcpy(held + (h * 64 + row_of(i, t >> 4)) * 128 + chunk * 8, x[h][i], 8 * sizeof(Bits));
        const int64_t row0 = first + h * 64 + row_of(0, t >> 4);
        if (by_row) quantize_rows<TYPE>(x[h], row0, rows, by_row + ((row0 / TILE_R) * KT_row + tile_col) * TILE_BYTES, chunk);
    }
    __syncthreads();
    const int c = t >> 6, lane = t & 63;
    Bits y[2][BLOCK];
#pragma unroll
    for (int r = 0; r < BLOCK; ++r) {
        Bits pair[2];
        __builtin_memcpy(pair, held + (c * BLOCK + r) * 128 + 2 * lane, sizeof(pair));
        y[0][r] = pair[0];
        y[1][r] = pair[1];
    }
    uint8_t* const tile = by_col + ((col0 / TILE_R) * KT_col + tile_row) * TILE_BYTES;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const uint32_t b = scale_byte(f32_bits<TYPE>(max_magnitude<TYPE, BLOCK>(y[j])));
        const float s = scale_value(b);
        v4i codes;
#pragma unroll
        for (int q = 0; q < 4; ++q) codes[q] = (int)codes8<TYPE>(y[j] + 8 * q, s);
        const int64_t col = col0 + 2 * lane + j;
        if (col < n) {
            *(v4i*)(tile + code_offset((int)(col % TILE_R), c)) = codes;
            tile[scale_offset((int)(col % TILE_R), c)] = (uint8_t)b;
        }
    }
}

// Reading back: the same threads as k_mx_quantize_rows.
template <int TYPE>
__global__ __launch_bounds__(256) void k_mx_dequantize(int64_t rows, int64_t n, const uint8_t* in, typename Elem<TYPE>::Bits* X,
                                                       int64_t ldx, int64_t KT)
{
    typedef typename Elem<TYPE>::Bits Bits;
    const int t = threadIdx.x, chunk = t & 15, c = chunk >> 2, sub = chunk & 3;
    const int64_t kt = blockIdx.x, row0 = (int64_t)blockIdx.y * 64 + row_of(0, t >> 4);
    const int64_t col = kt * TILE_K + chunk * 8;
    if (row0 >= rows || col >= n) return;
    const uint8_t* const tile = in + ((row0 / TILE_R) * KT + kt) * TILE_BYTES;
    const uint32_t scales = *(const uint32_t*)(tile + scale_offset((int)(row0 % TILE_R), c));
    uint32_t codes[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) codes[i] = *(const uint32_t*)(tile + code_offset((int)(row0 % TILE_R) + row_of(i, 0), c) + 4 * sub);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int64_t row = row0 + row_of(i, 0);
        if (row >= rows) break;
        Bits x[8];
        values8<TYPE>(codes[i], (scales >> (8 * i)) & 255u, x);
        store_row<TYPE, 8>(X + row * ldx + col, n - col, x);
    }
}

// Plain layout -> packed and back: one thread a block.
__global__ __launch_bounds__(256) void k_mx_pack(int64_t rows, int64_t n, const uint8_t* codes, int64_t ldc, const uint8_t* scales,
                                                 int64_t lds, uint8_t* out, int64_t KT)
{
    const int t = threadIdx.x, c = t & 3;
    const int64_t kt = blockIdx.x, row = (int64_t)blockIdx.y * 64 + (t >> 2);
    if (row >= rows) return;
    const int64_t block = kt * 4 + c, left = n - block * BLOCK;  // elements from the block's first one to the row's end
    uint32_t w[4] = {0, 0, 0, 0};
    uint8_t b = 0;
    if (left > 0) {
        __builtin_memcpy(w, codes + row * ldc + block * 16, 16);
        b = scales[row * lds + block];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const int64_t keep = left - 8 * q;  // codes of this word
            w[q] = keep >= 8 ? w[q] : (keep <= 0 ? 0u : w[q] & ((1u << (4 * (int)keep)) - 1u));
        }
    }
    uint8_t* const tile = out + ((row / TILE_R) * KT + kt) * TILE_BYTES;
    *(v4i*)(tile + code_offset((int)(row % TILE_R), c)) = v4i{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
    tile[scale_offset((int)(row % TILE_R), c)] = b;
}

__global__ __launch_bounds__(256) void k_mx_unpack(int64_t rows, int64_t n, const uint8_t* in, uint8_t* codes, int64_t ldc,
                                                   uint8_t* scales, int64_t lds, int64_t KT)
{
    const int t = threadIdx.x, c = t & 3;
    const int64_t kt = blockIdx.x, row = (int64_t)blockIdx.y * 64 + (t >> 2);
    const int64_t block = kt * 4 + c;
    if (row >= rows || block * BLOCK >= n) return;
    const uint8_t* const tile = in + ((row / TILE_R) * KT + kt) * TILE_BYTES;
    const v4i w = *(const v4i*)(tile + code_offset((int)(row % TILE_R), c));
    __builtin_memcpy(codes + row * ldc + block * 16, &w, 16);
    scales[row * lds + block] = tile[scale_offset((int)(row % TILE_R), c)];
}

template <int TYPE>
void quantize(int64_t rows, int64_t n, const void* X, int64_t ldx, void* by_row, void* by_col, hipStream_t st)
{
    typedef typename Elem<TYPE>::Bits Bits;
    if (by_col)
        hipLaunchKernelGGL(k_mx_quantize_cols<TYPE>, dim3((unsigned)(inner_tiles(n) * inner_tiles(rows))), dim3(256), 0, st, rows, n,
                           (const Bits*)X, ldx, (uint8_t*)by_row, (uint8_t*)by_col, inner_tiles(n), inner_tiles(rows));
    else
        hipLaunchKernelGGL(k_mx_quantize_rows<TYPE>, dim3((unsigned)inner_tiles(n), (unsigned)((rows + 63) / 64)), dim3(256), 0, st,
                           rows, n, (const Bits*)X, ldx, (uint8_t*)by_row, inner_tiles(n));
}

template <int TYPE> void dequantize(int64_t rows, int64_t n, const void* packed, void* X, int64_t ldx, hipStream_t st)
{
    hipLaunchKernelGGL(k_mx_dequantize<TYPE>, dim3((unsigned)inner_tiles(n), (unsigned)((rows + 63) / 64)), dim3(256), 0, st, rows, n,
                       (const uint8_t*)packed, (typename Elem<TYPE>::Bits*)X, ldx, inner_tiles(n));
}

}  // namespace

namespace mxk {

hipError_t launch_quantize(int type, int64_t rows, int64_t n, const void* X, int64_t ldx, void* by_row, void* by_col, hipStream_t st)
{
    if (type == F32) quantize<F32>(rows, n, X, ldx, by_row, by_col, st);
    if (type == BF16) quantize<BF16>(rows, n, X, ldx, by_row, by_col, st);
    if (type == F16) quantize<F16>(rows, n, X, ldx, by_row, by_col, st);
    return hipGetLastError();
}

hipError_t launch_dequantize(int type, int64_t rows, int64_t n, const void* packed, void* X, int64_t ldx, hipStream_t st)
{
    if (type == F32) dequantize<F32>(rows, n, packed, X, ldx, st);
    if (type == BF16) dequantize<BF16>(rows, n, packed, X, ldx, st);
    if (type == F16) dequantize<F16>(rows, n, packed, X, ldx, st);
    return hipGetLastError();
}

hipError_t launch_pack(int64_t rows, int64_t n, const uint8_t* codes, int64_t ldc, const uint8_t* scales, int64_t lds, void* packed,
                       hipStream_t st)
{
    hipLaunchKernelGGL(k_mx_pack, dim3((unsigned)inner_tiles(n), (unsigned)((rows + 63) / 64)), dim3(256), 0, st, rows, n, codes, ldc,
                       scales, lds, (uint8_t*)packed, inner_tiles(n));
    return hipGetLastError();
}

hipError_t launch_unpack(int64_t rows, int64_t n, const void* packed, uint8_t* codes, int64_t ldc, uint8_t* scales, int64_t lds,
                         hipStream_t st)
{
    hipLaunchKernelGGL(k_mx_unpack, dim3((unsigned)inner_tiles(n), (unsigned)((rows + 63) / 64)), dim3(256), 0, st, rows, n,
                       (const uint8_t*)packed, codes, ldc, scales, lds, inner_tiles(n));
    return hipGetLastError();
}

}  // namespace mxk
