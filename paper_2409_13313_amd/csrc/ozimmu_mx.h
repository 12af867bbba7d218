// Packed layout of microscaled 4-bit matrices and the launchers of their kernels (ozimmu_mx_*.hip).
//
// Rows are padded to a multiple of TILE_R, the inner index to a multiple of TILE_K.  A tile of TILE_R rows x TILE_K inner
// elements is one contiguous piece of TILE_BYTES: 16 KiB of codes, then 1 KiB of scales; the tiles of one row block follow each
// other along the inner dimension, so that a workgroup streams consecutive memory whatever the row length is.
//   codes   fragment f (rows 16 f .. 16 f + 15 of the tile) is 1 KiB: 16 bytes for each lane l of a wave, the 32 codes of
//           block l / 16 (of the tile's four) of row l % 16 - the operand of v_mfma_scale_f32_16x16x128_f8f6f4 as the lanes
//           hold it, so that a fragment is one 16-byte load a lane from memory or from LDS, in order, without a swizzle
//   scales  quarter q (fragments 4 q .. 4 q + 3) is 256 bytes: 4 bytes for each lane, byte f % 4 the scale of that lane's block
//           of fragment f; the matrix instruction picks the byte, so one register serves four fragments
// Inner padding is code 0 with scale byte 0 (exact zeros).  Padding rows are not written: what the memory held is multiplied, and
// the results, which touch no other row, are not stored.
#pragma once
#include <hip/hip_runtime.h>
#include <cstddef>
#include <cstdint>

namespace mxl {

constexpr int TILE_R = 256, TILE_K = 128, BLOCK = 32;
constexpr int FRAGMENT_BYTES = 1024, CODE_BYTES = TILE_R * TILE_K / 2, SCALE_BYTES = TILE_R * TILE_K / BLOCK;
constexpr int TILE_BYTES = CODE_BYTES + SCALE_BYTES;  // 17 KiB

__host__ __device__ inline int64_t row_tiles(int64_t rows) { return (rows + TILE_R - 1) / TILE_R; }
__host__ __device__ inline int64_t inner_tiles(int64_t n) { return (n + TILE_K - 1) / TILE_K; }
__host__ __device__ inline int64_t packed_bytes(int64_t rows, int64_t n) { return row_tiles(rows) * inner_tiles(n) * TILE_BYTES; }

// byte offsets inside a tile of row r (0 .. 255), block c (0 .. 3)
__host__ __device__ inline int code_offset(int r, int c) { return (r / 16) * FRAGMENT_BYTES + (c * 16 + r % 16) * 16; }
__host__ __device__ inline int scale_offset(int r, int c) { return CODE_BYTES + (r / 64) * 256 + (c * 16 + r % 16) * 4 + (r / 16) % 4; }

}  // namespace mxl

namespace mxk {

enum Type { F32 = 0, BF16 = 1, F16 = 2 };

hipError_t launch_quantize(int type, int64_t rows, int64_t n, const void* X, int64_t ldx, void* by_row, void* by_col, hipStream_t st);
hipError_t launch_dequantize(int type, int64_t rows, int64_t n, const void* packed, void* X, int64_t ldx, hipStream_t st);
hipError_t launch_pack(int64_t rows, int64_t n, const uint8_t* codes, int64_t ldc, const uint8_t* scales, int64_t lds, void* packed,
                       hipStream_t st);
hipError_t launch_unpack(int64_t rows, int64_t n, const void* packed, uint8_t* codes, int64_t ldc, uint8_t* scales, int64_t lds,
                         hipStream_t st);

// D <- alpha A B^T + beta D; with X (of xtype, m x n, ldx) in the place of A: quantised on the way
struct Gemm {
    int64_t m, n, p;
    const uint8_t* A;
    const uint8_t* B;
    void* D;
    int64_t ldd;
    int dtype;
    float alpha, beta;
};
hipError_t launch_gemm(const Gemm& g, hipStream_t st);

}  // namespace mxk
