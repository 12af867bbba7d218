// Quantisation to the microscaled 4-bit form, reading back, and the plain layout of checkpoints (include/ozimmu_mx.h).
//
// All of it moves memory: an element is read in 2 or 4 bytes and written in 17/32 of one (or the other way round), with two
// dozen operations for eight elements between.
#include "ozimmu_mx_convert.h"

namespace {

using namespace mxk;
using namespace mxl;

// (largest of the four lanes of a quad, in all of them)
__device__ inline uint32_t quad_max(uint32_t m)
{
    const uint32_t a = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xb1, 0xf, 0xf, true);  // lanes 1 0 3 2
    m = a > m ? a : m;
    const uint32_t b = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4e, 0xf, 0xf, true);  // lanes 2 3 0 1
    return b > m ? b : m;
}

constexpr int64_t BLOCKS_Y = 32768;  // (there may be more blocks of rows than a grid has in its second dimension)
inline dim3 grid_of(int64_t cols, int64_t blocks)
{
    return dim3((unsigned)cols, (unsigned)(blocks < BLOCKS_Y ? blocks : BLOCKS_Y), (unsigned)((blocks + BLOCKS_Y - 1) / BLOCKS_Y));
}

// Blocks along the rows.  A workgroup takes 32 rows x 128 columns (half a quarter of a tile, its fragments 0 and 1 or 2 and 3): thread t the
// eight elements t % 16 of the two rows at place t / 16, so that 16 lanes read 128 columns of a row side by side; four lanes hold a block and
// share its maximum.  (8192 x 8192 bf16 30.5 us, 170 MB at 5.6 TB/s, a large copy moves 5.0.)
struct RowsAt {
    int64_t row0;  // the place's row in fragment 0 of the quarter
    int first;     // the first of the two fragments
    __device__ inline RowsAt(int64_t block) : row0(block / 2 * 64 + row_of(0, (int)threadIdx.x >> 4)), first((int)(block % 2) * 2) {}
    __device__ inline int64_t row(int i) const { return row0 + row_of(first + i, 0); }
};
template <int TYPE>
__device__ inline void load_rows(typename Elem<TYPE>::Bits (&x)[2][8], const typename Elem<TYPE>::Bits* X, int64_t ldx, int64_t rows, int64_t n,
                                 const RowsAt& at, int64_t col)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) load_row<TYPE, 8>(X + at.row(i) * ldx + col, at.row(i) < rows ? n - col : 0, x[i]);
}
template <int TYPE>
__device__ inline void quantize_rows(const typename Elem<TYPE>::Bits (&x)[2][8], const RowsAt& at, int64_t rows, uint8_t* row_tiles, int64_t KT, int64_t kt)
{
    const int chunk = threadIdx.x & 15, c = chunk >> 2, sub = chunk & 3;
    uint8_t* const tile = row_tiles + ((at.row0 / TILE_R) * KT + kt) * TILE_BYTES;
    uint32_t scales = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t b = scale_byte(f32_bits<TYPE>(quad_max(max_magnitude<TYPE, 8>(x[i]))));
        scales |= b << (8 * i);
        if (at.row(i) < rows) *(uint32_t*)(tile + code_offset((int)(at.row(i) % TILE_R), c) + 4 * sub) = codes8<TYPE>(x[i], scale_value(b));
    }
    // (the scale of a row that is not there is that of zeros)
    if (sub == 0 && at.row(0) < rows) *(uint16_t*)(tile + scale_offset((int)(at.row(0) % TILE_R), c)) = (uint16_t)scales;
}

template <int TYPE>
__global__ __launch_bounds__(256) void k_mx_quantize_rows(int64_t rows, int64_t n, const typename Elem<TYPE>::Bits* X, int64_t ldx,
                                                          uint8_t* out, int64_t KT)
{
    typename Elem<TYPE>::Bits x[2][8];
    const RowsAt at((int64_t)blockIdx.z * BLOCKS_Y + blockIdx.y);
    load_rows<TYPE>(x, X, ldx, rows, n, at, (int64_t)blockIdx.x * TILE_K + (threadIdx.x & 15) * 8);
    quantize_rows<TYPE>(x, at, rows, out, KT, blockIdx.x);
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
        const RowsAt at(block);
        Bits x[2][8];
        load_rows<TYPE>(x, X, ldx, rows, n, at, col0 + chunk * 8);
#pragma unroll
        for (int i = 0; i < 2; ++i) __builtin_memcpy(held + row_of(i, t >> 4) * 128 + chunk * 8, x[i], 8 * sizeof(Bits));
        if (by_row) quantize_rows<TYPE>(x, at, rows, by_row, KT_row, tile_col);
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

// Reading back: a lane makes 16 bytes, E elements, of a row, side by side with its neighbours (FP32: half of the eight codes that it loads; 32 bytes a
// lane in two stores: 16384 x 8192 183 us, so 154, today 84).  A workgroup takes 16 rows x 128 columns (64 rows: 4096 x 4096 FP32 13.6 us, 16 rows 11.5;
// 513 x 1001 3.6 and 2.9; 16384 x 8192 85.7 and 84.5).  STREAM, where rows begin at multiples of 16 bytes: stores
// past the caches (16384 x 8192 FP32 84.5 us = 7.2 TB/s, a large fill writes 6.9; bf16 47.7 and 64).  What reads X right behind them loses up to 5 %
// of the two, and gains where X is large (past the caches and plain, bf16: read back and a product of 16 rows with it, 4096 x 4096 27.1 and 26.3 us,
// 8192 x 8192 63 and 69, 16384 x 8192 132 and 137; read back and 1 added to it, 22.9 and 21.8, 79 and 76, 154 and 162).  Rows that begin anywhere: plain
// stores (1001 x 4099 bf16 4.2 us, past the caches 5.6), in FP32 of 8 bytes (1001 x 4099 6.0 us; 4, 16 bytes: 7.4, 7.0; bf16 of 2, 4, 8, 16 bytes: 6.9, 5.3, 4.7, 4.2).
constexpr int BACK_ROWS = 16;
template <int TYPE, bool STREAM>
__global__ __launch_bounds__(256) void k_mx_dequantize(int64_t rows, int64_t n, const uint8_t* in, typename Elem<TYPE>::Bits* X,
                                                       int64_t ldx, int64_t KT)
{
    typedef typename Elem<TYPE>::Bits Bits;
    constexpr int E = TYPE != F32 ? 8 : STREAM ? 4 : 2, LANES = 128 / E, PLACES = 256 / LANES;  // lanes to a row, places of a fragment at a time
    constexpr int STEPS = BACK_ROWS / PLACES;                                                   // rows of a thread
    const int t = threadIdx.x, lane = t % LANES, first = lane * E, chunk = first / 8, c = chunk >> 2, sub = chunk & 3;
    const int64_t block = ((int64_t)blockIdx.z * BLOCKS_Y + blockIdx.y) * BACK_ROWS, quarter = block / 64 * 64;
    const int64_t kt = blockIdx.x, col = kt * TILE_K + first;
    if (block >= (rows + 63) / 64 * 64 || col >= n) return;
    const uint8_t* const tile = in + ((quarter / TILE_R) * KT + kt) * TILE_BYTES;
    const int step0 = (int)(block % 64) / PLACES;
    uint32_t scales[STEPS], codes[STEPS];
    // step: four fragments of the places at hand, then the next places
    const auto row_at = [&](int step) { return row_of(step % 4, step / 4 * PLACES + t / LANES); };
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int r = (int)(quarter % TILE_R) + row_at(step0 + s);
        scales[s] = tile[scale_offset(r, c)];
        codes[s] = *(const uint32_t*)(tile + code_offset(r, c) + 4 * sub) >> (first % 8 * 4);
    }
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
        const int64_t row = quarter + row_at(step0 + s);
        if (row >= rows) continue;
        Bits x[8];
        values8<TYPE>(codes[s], scales[s], x);
        if (STREAM && n - col >= E) {
            v4i y;
            __builtin_memcpy(&y, x, 16);
            __builtin_nontemporal_store(y, (v4i*)(X + row * ldx + col));
        } else {
            store_row<TYPE, E>(X + row * ldx + col, n - col, x);
        }
    }
}

// Plain layout -> packed and back: one thread a block.  (16384 x 8192: 35 and 28 us, 143 MB at 4.1 and 5.0 TB/s.)
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
    if (q.by_col)
        k_mx_quantize_cols<TYPE><<<grid_of(inner_tiles(q.n), 4 * inner_tiles(q.rows)), dim3(256), 0, st>>>(columns<TYPE>(q));
    else
        k_mx_quantize_rows<TYPE><<<grid_of(inner_tiles(q.n), (q.rows + BLOCK - 1) / BLOCK), dim3(256), 0, st>>>(
            q.rows, q.n, (const typename Elem<TYPE>::Bits*)q.X, q.ldx, (uint8_t*)q.by_row, inner_tiles(q.n));
}

template <int TYPE> void quantize2(const Quantize& a, const Quantize& b, hipStream_t st)
{
    const int64_t blocks_a = 4 * inner_tiles(a.rows) * inner_tiles(a.n), blocks_b = 4 * inner_tiles(b.rows) * inner_tiles(b.n);
    k_mx_quantize_cols2<TYPE><<<dim3((unsigned)(blocks_a + blocks_b)), dim3(256), 0, st>>>(columns<TYPE>(a), columns<TYPE>(b), (uint32_t)blocks_a);
}

template <int TYPE> void dequantize(int64_t rows, int64_t n, const void* packed, void* X, int64_t ldx, hipStream_t st)
{
    typedef typename Elem<TYPE>::Bits Bits;
    const dim3 grid = grid_of(inner_tiles(n), (rows + 63) / 64 * (64 / BACK_ROWS));
    if (((uintptr_t)X | (uintptr_t)(ldx * (int64_t)sizeof(Bits))) % 16 == 0)
        k_mx_dequantize<TYPE, true><<<grid, dim3(256), 0, st>>>(rows, n, (const uint8_t*)packed, (Bits*)X, ldx, inner_tiles(n));
    else
        k_mx_dequantize<TYPE, false><<<grid, dim3(256), 0, st>>>(rows, n, (const uint8_t*)packed, (Bits*)X, ldx, inner_tiles(n));
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
    // (large ones one after the other: 8192 x 8192 both ways and 8192 x 4096 by columns 57 us, in one launch 71)
    if (4 * (inner_tiles(a.rows) * inner_tiles(a.n) + inner_tiles(b.rows) * inner_tiles(b.n)) > 4096) {
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
