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
// (largest of the four lanes of a quad, in all of them)
__device__ inline uint32_t quad_max(uint32_t m)
{
    const uint32_t a = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, true);  // lanes 1 0 3 2
    m = a > m ? a : m;
    const uint32_t b = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 0xf, 0xf, true);  // lanes 2 3 0 1
    return b > m ? b : m;
}

// COUNT (2 or 4) of the four fragments' rows at a place, from fragment `first` on
template <int TYPE, int COUNT>
__device__ inline void quantize_rows(const typename Elem<TYPE>::Bits (*x)[8], int64_t row0, int first, int64_t rows, uint8_t* tile, int chunk)
{
    const int c = chunk >> 2, sub = chunk & 3;
    uint32_t scales = 0;
#pragma unroll
    for (int i = 0; i < COUNT; ++i) {
        const uint32_t b = scale_byte(f32_bits<TYPE>(quad_max(max_magnitude<TYPE, 8>(x[i]))));
        scales |= b << (8 * i);
        const int64_t row = row0 + row_of(first + i, 0);
        if (row < rows) *(uint32_t*)(tile + code_offset((int)(row % TILE_R), c) + 4 * sub) = codes8<TYPE>(x[i], scale_value(b));
    }
    // (the scales of rows that are not there are those of zeros)
    if (sub == 0 && row0 + row_of(first, 0) < rows) {
        uint8_t* const at = tile + scale_offset((int)(row0 % TILE_R), c) + first;
        if constexpr (COUNT == 4)
            *(uint32_t*)at = scales;
        else
            *(uint16_t*)at = (uint16_t)scales;
    }
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
    quantize_rows<TYPE, 4>(x, row0, 0, rows, out + ((row0 / TILE_R) * KT + kt) * TILE_BYTES, chunk);
}

// Blocks along the columns, and along the rows too where by_row is given.  A workgroup takes 32 rows x 128 columns, read as above (rows
// quantised on the way) and left in LDS as they are; then 128 threads take a column each, whose 32 rows they read one after the other, 64 lanes a
// row side by side, so that a block is one lane's.  (Two and four blocks of rows a workgroup: 8192 x 8192 bf16 both ways 43.6 and 44.1 us, one
// block 41.0, 205 MB at 5.0 TB/s as a large copy; 513 x 1001 4.2 and 6.3 us, one block 3.3.)
template <int TYPE> struct Columns {
    typedef typename Elem<TYPE>::Bits Bits;
    const Bits* X;
    int64_t rows, n, ldx;
    uint8_t *by_row, *by_col;  // by_row: nullptr where it is not wanted
    int64_t KT_row, KT_col;

    // tile_col: 128 columns; block: 32 rows (all of the packed rows' inner tiles have to be taken, so that their padding is written)
    __device__ inline void run(int64_t tile_col, int64_t block, Bits* held) const
    {
        const int t = threadIdx.x, chunk = t & 15;
        const int64_t col0 = tile_col * 128;
        // half a quarter of the rows: fragments 0 and 1, or 2 and 3
        const int64_t row0 = block / 2 * 64 + row_of(0, t >> 4);
        const int first = (int)(block % 2) * 2;
        Bits x[2][8];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int64_t row = row0 + row_of(first + i, 0);
            load_row<TYPE, 8>(X + row * ldx + col0 + chunk * 8, row < rows ? n - col0 - chunk * 8 : 0, x[i]);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) __builtin_memcpy(held + row_of(i, t >> 4) * 128 + chunk * 8, x[i], 8 * sizeof(Bits));
        if (by_row) quantize_rows<TYPE, 2>(x, row0, first, rows, by_row + ((row0 / TILE_R) * KT_row + tile_col) * TILE_BYTES, chunk);
        __syncthreads();
        const int64_t col = col0 + t;
        if (t >= 128 || col >= n) return;
        Bits y[BLOCK];
#pragma unroll
        for (int r = 0; r < BLOCK; ++r) y[r] = held[r * 128 + t];
        const uint32_t b = scale_byte(f32_bits<TYPE>(max_magnitude<TYPE, BLOCK>(y)));
        const float s = scale_value(b);
        v4i codes;
#pragma unroll
        for (int q = 0; q < 4; ++q) codes[q] = (int)codes8<TYPE>(y + 8 * q, s);
        uint8_t* const tile = by_col + ((col0 / TILE_R) * KT_col + block / 4) * TILE_BYTES;
        *(v4i*)(tile + code_offset((int)(col % TILE_R), (int)(block % 4))) = codes;
        tile[scale_offset((int)(col % TILE_R), (int)(block % 4))] = (uint8_t)b;
    }
};

constexpr int64_t BLOCKS_Y = 32768;  // (there may be more blocks of rows than a grid has in its second dimension)
template <int TYPE> __global__ __launch_bounds__(256) void k_mx_quantize_cols(Columns<TYPE> c)
{
    __shared__ __align__(16) typename Elem<TYPE>::Bits held[BLOCK * 128];
    const int64_t block = (int64_t)blockIdx.z * BLOCKS_Y + blockIdx.y;
    if (block < 4 * c.KT_col) c.run(blockIdx.x, block, held);
}

// Two matrices in one launch: what a small one takes is the launch (a gradient's G both ways and X by columns: 777 x 513 and 777 x 1001, FP32, 3.3
// and 3.0 us one after the other).
template <int TYPE> __global__ __launch_bounds__(256) void k_mx_quantize_cols2(Columns<TYPE> a, Columns<TYPE> b, uint32_t blocks_a)
{
    __shared__ __align__(16) typename Elem<TYPE>::Bits held[BLOCK * 128];
    const uint32_t at = blockIdx.x < blocks_a ? blockIdx.x : blockIdx.x - blocks_a;
    const Columns<TYPE>& c = blockIdx.x < blocks_a ? a : b;
    const uint32_t tiles = (uint32_t)((c.n + 127) / 128);
    c.run(at % tiles, at / tiles, held);
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

template <int TYPE> Columns<TYPE> columns(const Quantize& q)
{
    return {(const typename Elem<TYPE>::Bits*)q.X, q.rows, q.n, q.ldx, (uint8_t*)q.by_row, (uint8_t*)q.by_col, inner_tiles(q.n), inner_tiles(q.rows)};
}

template <int TYPE> void quantize(const Quantize& q, hipStream_t st)
{
    if (q.by_col) {
        const int64_t blocks = 4 * inner_tiles(q.rows);
        const dim3 grid((unsigned)inner_tiles(q.n), (unsigned)(blocks < BLOCKS_Y ? blocks : BLOCKS_Y), (unsigned)((blocks + BLOCKS_Y - 1) / BLOCKS_Y));
        k_mx_quantize_cols<TYPE><<<grid, dim3(256), 0, st>>>(columns<TYPE>(q));
    } else {
        k_mx_quantize_rows<TYPE><<<dim3((unsigned)inner_tiles(q.n), (unsigned)((q.rows + 63) / 64)), dim3(256), 0, st>>>(
            q.rows, q.n, (const typename Elem<TYPE>::Bits*)q.X, q.ldx, (uint8_t*)q.by_row, inner_tiles(q.n));
    }
}

template <int TYPE> void quantize2(const Quantize& a, const Quantize& b, hipStream_t st)
{
    const int64_t blocks_a = 4 * inner_tiles(a.rows) * inner_tiles(a.n), blocks_b = 4 * inner_tiles(b.rows) * inner_tiles(b.n);
    k_mx_quantize_cols2<TYPE><<<dim3((unsigned)(blocks_a + blocks_b)), dim3(256), 0, st>>>(columns<TYPE>(a), columns<TYPE>(b), (uint32_t)blocks_a);
}

template <int TYPE> void dequantize(int64_t rows, int64_t n, const void* packed, void* X, int64_t ldx, hipStream_t st)
{
    hipLaunchKernelGGL(k_mx_dequantize<TYPE>, dim3((unsigned)inner_tiles(n), (unsigned)((rows + 63) / 64)), dim3(256), 0, st, rows, n,
                       (const uint8_t*)packed, (typename Elem<TYPE>::Bits*)X, ldx, inner_tiles(n));
}

}  // namespace

namespace mxk {

hipError_t launch_quantize(int type, const Quantize& q, hipStream_t st)
{
    if (type == F32) quantize<F32>(q, st);
    if (type == BF16) quantize<BF16>(q, st);
    if (type == F16) quantize<F16>(q, st);
    return hipGetLastError();
}

hipError_t launch_quantize2(int type, const Quantize& a, const Quantize& b, hipStream_t st)
{
    // (work items of a launch are counted in 32 bits)
    if (4 * (inner_tiles(a.rows) * inner_tiles(a.n) + inner_tiles(b.rows) * inner_tiles(b.n)) >= (int64_t)1 << 24) {
        const hipError_t e = launch_quantize(type, a, st);
        return e != hipSuccess ? e : launch_quantize(type, b, st);
    }
    if (type == F32) quantize2<F32>(a, b, st);
    if (type == BF16) quantize2<BF16>(a, b, st);
    if (type == F16) quantize2<F16>(a, b, st);
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
