// Operators around a model's output layer (include/ozimmu_lm.h): the stored form of 4-bit weights and the launchers of their kernels
// (ozimmu_lm_*.hip).
//
// Weights in 4 bits, p rows of n elements.  Codes come in blocks of 16 rows x 128 elements, 1 KiB each, the blocks of 16 rows one behind the
// other along the row: 16 bytes for each lane l of a wave, the codes of row l % 16 that it holds in four matrix instructions (16x16x32).
// Word j of them (j < 4) is elements 32 j + 8 (l / 16) .. + 7, element 2 i at bits 4 i and 2 i + 1 at bits 16 + 4 i, so that one mask
// and one or makes a pair of 16-bit numbers of two neighbouring elements.
// Behind the codes of all blocks comes a record for each of their rows, [block][row]: 128 / group scales of 16 bits (0 behind the end of a row), then,
// where the weights have zero points, as many of these as bytes; so a lane has what its row needs beside the codes in one load.  Codes behind the
// end of a row are 0.  Padding rows are not written: what they give is not stored.
#pragma once
#include "ozimmu_mx_convert.h"

namespace lml {

constexpr int ROWS = 16, INNER = 128, BLOCK_BYTES = 1024;

struct Shape {
    int64_t p, n;
    int group;   // 32, 64 or 128
    bool zeros;
    __host__ __device__ inline int64_t row_blocks() const { return (p + ROWS - 1) / ROWS; }
    __host__ __device__ inline int64_t inner_blocks() const { return (n + INNER - 1) / INNER; }
    __host__ __device__ inline int64_t blocks() const { return row_blocks() * inner_blocks(); }
    __host__ __device__ inline int groups() const { return INNER / group; }  // of a block's row
    __host__ __device__ inline int record() const { return groups() * (zeros ? 3 : 2); }
    __host__ __device__ inline int64_t records_at() const { return blocks() * BLOCK_BYTES; }
    // (16 bytes more: records are read as whole dwords)
    __host__ __device__ inline int64_t bytes() const { return blocks() ? records_at() + (blocks() * ROWS * record() + 16 + 255) / 256 * 256 : 0; }
};

}  // namespace lml

namespace lmk {

using mxk::BF16;
using mxk::F16;
using mxk::F32;

struct Weights {
    lml::Shape shape;
    int stype;            // type of the scales: BF16 or F16
    const uint8_t* data;
};

hipError_t launch_quantize(int type, const void* W, int64_t ldw, const lml::Shape& s, int stype, void* packed, hipStream_t st);
// rows row0 .. row0 + rows - 1 into X (of `type`); columns n .. cols - 1 (no more than whole blocks have) become zeros; through: for
// a reader right behind it (k_lm_dequantize).  peaks (nullptr: without; else FP16 from scales in BF16, `through`, X's rows 16-byte aligned): room for
// SCALE_PEAKS + 1 numbers; X is held times a power of two then, and the last of them is what the products have to be multiplied by
constexpr int SCALE_PEAKS = 256;
hipError_t launch_dequantize(int type, const Weights& w, int64_t row0, int64_t rows, int64_t cols, void* X, int64_t ldx, bool through, float* peaks,
                             hipStream_t st);
hipError_t launch_pack(const lml::Shape& s, const uint8_t* codes, int64_t ldc, const void* scales, int64_t lds, const uint8_t* zeros, int64_t ldz,
                       void* packed, hipStream_t st);
hipError_t launch_unpack(const lml::Shape& s, const void* packed, uint8_t* codes, int64_t ldc, void* scales, int64_t lds, uint8_t* zeros,
                         int64_t ldz, hipStream_t st);

// D <- alpha X W^T + beta D straight from the stored weights (m rows of X)
struct Linear {
    int64_t m;
    const void* X;
    int64_t ldx;
    int xtype;
    void* D;
    int64_t ldd;
    int dtype;
    float alpha, beta;
};
hipError_t launch_direct(const Linear& l, const Weights& w, hipStream_t st);
// The same with X in LDS: rows (32, 64) x columns (128, 256) a workgroup, the inner dimension in `splits` parts, whose sums meet in `parts`
// (splits > 1: that many matrices of whole workgroups in FP32)
struct SharedPlan {
    int rows, columns, splits;
};
hipError_t launch_shared(const Linear& l, const Weights& w, const SharedPlan& plan, float* parts, hipStream_t st);

// ---- products of 16-bit matrices in tiles of 256 x 256 (ozimmu_lm_tile.hip) ----

// What is made of the sums C (m x p, over the inner dimension n):
enum Kind {
    LINEAR,   // A: m x n, B: p x n.  D <- alpha C + beta D
    LOSS,     // A: m x n, B: p x n.  per row and part_columns: log2(e) times the largest sum, and the sum of 2^(log2(e) c - that) (without the target's)
    SLOPE,    // A: m x n, B: p x n.  D <- exp(C - lse) - [column = target] in 16 bits (0 in rows without a target)
    STATES,   // A: m x n, B: n x p.  D (FP32, one for each split of n) <- C, or C + D
    WEIGHTS,  // A: n x m, B: n x p.  D <- alpha C + beta D, alpha from the device
};

constexpr int NO_TARGET = -1, BAD_TARGET = -2;  // an ignored row; a target that no column has

struct Targets {
    const int64_t* y;
    int64_t stride, ignore, words;
    __device__ inline int operator[](int64_t row) const
    {
        const int64_t v = y[row * stride];
        return v == ignore ? NO_TARGET : (v >= 0 && v < words ? (int)v : BAD_TARGET);
    }
};

enum TileShape { TILE_256, TILE_128_256, TILE_128 };  // sums a workgroup: 256 x 256, 128 x 256, 128 x 128

struct Tile {
    int kind, type;       // type: of A and B
    int shape = TILE_256;
    int64_t m, n, p;
    const void *A, *B;    // 16-byte aligned; leading dimensions multiples of 8 elements; where rows lie along n, n a multiple of 8
    int64_t lda, ldb;
    int64_t b_rows;       // of B: p, or where its rows lie across n how many of n there are (the others count as zeros)
    void* D = nullptr;
    int64_t ldd = 0;
    int dtype = 0;
    float alpha = 1, beta = 0;
    const float* alpha_at = nullptr;   // WEIGHTS, and LINEAR of FP16 where it is given: alpha is multiplied by this
    int splits = 1;                    // STATES: of the inner dimension
    int64_t split_stride = 0;          // STATES: elements between the D of splits
    Targets targets{};                 // LOSS
    const int* known = nullptr;        // SLOPE: targets per row of whole tiles, as target_of has them
    int column0 = 0;                   // LOSS, SLOPE: what number the first column is to them
    const float* lse2 = nullptr;       // SLOPE: log2(e) lse per row of whole tiles
    float* at_target = nullptr;        // LOSS: the sums at the targets
    float2* parts = nullptr;           // LOSS: [part_columns][row]
    int64_t parts_ld = 0;
};
bool tile_fits(const Tile& t);
int tile_shape(int64_t m, int64_t n, int64_t p, int splits);   // the one that takes the least time, by an estimate
int tile_splits(int64_t m, int64_t n, int64_t p);             // STATES: the number of splits that does
inline int part_columns(int shape) { return shape == TILE_128 ? 64 : 128; }  // LOSS: columns of a part
hipError_t launch_tile(const Tile& t, hipStream_t st);
hipError_t launch_tile_1(const Tile& t, hipStream_t st);  // BF16
hipError_t launch_tile_2(const Tile& t, hipStream_t st);  // F16

// ---- the loss without tiles (ozimmu_lm_few.hip) ----

struct FewLoss {
    int64_t m, n, p;
    const void* X;
    int64_t ldx;
    const void* W;
    int64_t ldw;
    Targets targets;
    float* at_target;
    float2* parts;   // [row][columns of the plan], rows of whole workgroups
    int64_t parts_ld;
};
// tokens (16, 32, 64) and words (16, 64) a workgroup; rows == 0: by tiles
struct FewPlan {
    int rows, columns;
};
hipError_t launch_few_loss(int type, const FewLoss& g, const FewPlan& plan, hipStream_t st);

// ---- what stands around them in the loss (ozimmu_lm_loss.hip) ----

constexpr float SLOPE_SCALE_F16 = 32768.0f;     // slopes in FP16 are held times this: most of them are far below 2^-14

// rows x cols of X (16 bits) into Y (nullptr: not wanted), columns cols .. width - 1 zeros (width: a multiple of 8; Y's rows 16-byte aligned)
struct LayOut {
    int64_t rows, cols;
    const void* X;
    int64_t ldx;
    void* Y;
    int64_t width;
};
hipError_t launch_lay_out(int type, const LayOut& a, const LayOut& b, hipStream_t st);  // both, of one type
hipError_t launch_join_rows(int64_t rows, int64_t blocks, const float2* parts, int64_t parts_ld, const Targets& targets, const float* at_target,
                            float* loss, float* lse, hipStream_t st);
hipError_t launch_join(int64_t rows, int64_t blocks, const float2* parts, int64_t parts_ld, const Targets& targets, const float* at_target, float* loss,
                       float* lse, hipStream_t st);
// FP16: the largest finite magnitude of each row of X
hipError_t launch_row_peaks(int64_t rows, int64_t cols, const void* X, int64_t ldx, float* peaks, hipStream_t st);
// What the gradient begins with: targets and log2(e) lse (NaN where the target is bad) per row, `padded` of them, the largest |g| of rows with a
// target, X laid out (as x says) and, in `scaled` (nullptr: not wanted), X times each row's share of that |g|, zeros in rows without a target; and W laid out.
// FP16 with `scaled`: that times a power of two, which `largest` is divided by; zeros also in rows too small for it, whose numbers are in `far` (as many as
// the gradient has tokens at the most)
struct Prepare {
    int64_t rows, padded;
    Targets targets;
    const float* g;
    int64_t g_stride;
    const float* lse;
    int* known;
    float *lse2, *largest;
    const float* peaks;   // FP16 with `scaled`: of launch_row_peaks
    int *far, *far_count;
    LayOut x;
    void* scaled;
    LayOut w;
};
hipError_t launch_prepare(int type, const Prepare& p, hipStream_t st);
// dX <- g (the sum of the splits) / scale, zeros in rows without a target
hipError_t launch_states(int type, int64_t rows, int64_t cols, const float* parts, int64_t ld, int splits, int64_t split_stride, const float* g,
                         int64_t g_stride, const int* targets, float scale, void* dX, int64_t ldx, hipStream_t st);
// FP16: dW (of `type`) += what the rows in `far` give, from slopes (times SLOPE_SCALE_F16), X and g
hipError_t launch_far(int type, int64_t words, int64_t cols, const uint16_t* slopes, int64_t lds, const void* X, int64_t ldx, const float* g, int64_t g_stride,
                      const int* far, const int* far_count, void* dW, int64_t ldw, hipStream_t st);
// X <- beta X (beta == 0: zeros)
hipError_t launch_scale(int type, int64_t rows, int64_t cols, float beta, void* X, int64_t ldx, hipStream_t st);

}  // namespace lmk
