// Packed layout of microscaled 4-bit matrices and the launchers of their kernels (ozimmu_mx_*.hip).
//
// Rows are padded to a multiple of TILE_R, the inner index to a multiple of TILE_K.  A tile of TILE_R rows x TILE_K inner
// elements is one contiguous piece of TILE_BYTES; the tiles of one row block follow each other along the inner dimension, so that
// a workgroup streams consecutive memory whatever the row length is.  A tile is four quarters of 64 rows, each 256 bytes of scales and
// four fragments of 1 KiB of codes - what one wave copies to LDS, or takes from memory, as it is:
//   row r of a quarter belongs to fragment 2 (r / 32) + (r / 4) % 2 and there to place (r / 8) % 4 * 4 + r % 4: a lane's four sums of a
//           product come from four places in a row, so that in two fragments it holds 8 neighbouring columns of the result - 16 bytes
//           in a 16-bit type, and the four lanes of a row 64
//   codes   of a fragment: 16 bytes for each lane l of a wave, the 32 codes of block l / 16 (of the tile's four) of the row at
//           place l % 16 - the operand of v_mfma_scale_f32_16x16x128_f8f6f4 as the lanes hold it, one 16-byte load a lane from
//           memory or from LDS, in order, without a swizzle
//   scales  4 bytes for each lane, byte f the scale of that lane's block of fragment f; the matrix instruction picks the byte, so
//           one register serves four fragments
// Inner padding is code 0 with scale byte 0 (exact zeros).  Padding rows are not written: what the memory held is multiplied, and
// the results, which touch no other row, are not stored.
#pragma once
#include <hip/hip_runtime.h>
#include <cstddef>
#include <cstdint>

namespace mxl {

constexpr int TILE_R = 256, TILE_K = 128, BLOCK = 32;
constexpr int QUARTER_R = 64, FRAGMENT_BYTES = 1024, SCALE_BYTES = 256;
constexpr int QUARTER_BYTES = SCALE_BYTES + 4 * FRAGMENT_BYTES, TILE_BYTES = 4 * QUARTER_BYTES;  // 4352 and 17 KiB

__host__ __device__ inline int64_t row_tiles(int64_t rows) { return (rows + TILE_R - 1) / TILE_R; }
__host__ __device__ inline int64_t inner_tiles(int64_t n) { return (n + TILE_K - 1) / TILE_K; }
__host__ __device__ inline int64_t packed_bytes(int64_t rows, int64_t n) { return row_tiles(rows) * inner_tiles(n) * TILE_BYTES; }

// place of row r (0 .. 255 of its tile)
__host__ __device__ inline int fragment_of(int r) { return r / 32 % 2 * 2 + r / 4 % 2; }
__host__ __device__ inline int place_of(int r) { return r / 8 % 4 * 4 + r % 4; }
// row (0 .. 63 of its quarter) at a place of a fragment
__host__ __device__ constexpr int row_of(int fragment, int place) { return fragment / 2 * 32 + place / 4 * 8 + fragment % 2 * 4 + place % 4; }
// byte offsets inside a tile of row r, block c (0 .. 3)
__host__ __device__ inline int code_offset(int r, int c)
{
    return r / QUARTER_R * QUARTER_BYTES + SCALE_BYTES + fragment_of(r) * FRAGMENT_BYTES + (c * 16 + place_of(r)) * 16;
}
__host__ __device__ inline int scale_offset(int r, int c) { return r / QUARTER_R * QUARTER_BYTES + (c * 16 + place_of(r)) * 4 + fragment_of(r); }

}  // namespace mxl

namespace mxk {

enum Type { F32 = 0, BF16 = 1, F16 = 2 };

// X of rows x n, and where it goes (nullptr: not wanted; at least one of them)
struct Quantize {
    int64_t rows, n;
    const void* X;
    int64_t ldx;
    void *by_row, *by_col;
};
hipError_t launch_quantize(int type, const Quantize& q, hipStream_t st);
hipError_t launch_quantize2(int type, const Quantize& a, const Quantize& b, hipStream_t st);  // in one launch; both with by_col
hipError_t launch_dequantize(int type, int64_t rows, int64_t n, const void* packed, void* X, int64_t ldx, hipStream_t st);
hipError_t launch_pack(int64_t rows, int64_t n, const uint8_t* codes, int64_t ldc, const uint8_t* scales, int64_t lds, void* packed,
                       hipStream_t st);
hipError_t launch_unpack(int64_t rows, int64_t n, const void* packed, uint8_t* codes, int64_t ldc, uint8_t* scales, int64_t lds,
                         hipStream_t st);

// D <- alpha A B^T + beta D
struct Gemm {
    int64_t m, n, p;
    const uint8_t* A;
    const uint8_t* B;
    void* D;
    int64_t ldd;
    int dtype;
    float alpha, beta;
    bool read_later = false;  // D is not what the next work reads (a gradient of weights)
};
// How a product is run (OZIMMU_MX_WAY_*); WAY_AUTO: choose() says
enum { WAY_AUTO = -1, WAY_DIRECT = 0, WAY_TILE = 1, WAY_HALF = 2 };
int choose(int64_t m, int64_t n, int64_t p, int64_t ldd);
bool way_fits(int way, int64_t m, int64_t n, int64_t p, int64_t ldd);
hipError_t launch_gemm(const Gemm& g, int way, hipStream_t st);
hipError_t launch_gemm2(const Gemm& a, const Gemm& b, hipStream_t st);  // both; neither waits for the other
// D <- alpha Q(X) B^T + beta D in one launch (g.A is not looked at); few_rows(m, p): what this is for
bool few_rows(int64_t m, int64_t p);
hipError_t launch_few(const Gemm& g, int xtype, const void* X, int64_t ldx, hipStream_t st);

}  // namespace mxk
