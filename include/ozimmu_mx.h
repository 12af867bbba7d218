/*
 * ozimmu_mx.h - C ABI of the microscaled 4-bit operators of the library (gfx950 / MI355X): quantisation, reading back,
 * product, and a linear layer with its gradient.
 *
 * The form.  A matrix of `rows` rows and n columns is cut along its rows into blocks of 32 elements (the last block of a
 * row may be shorter).  A block has one scale 2^(b - 127), b a byte of 0 .. 254, and 32 elements of 4 bits: a sign (bit 3)
 * and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 (bits 0 .. 2).  b = 255 makes every element of the block NaN.
 * Quantisation of a block whose largest magnitude is amax:
 *     b = max(0, floor(log2 amax) - 2 + 127)   (0 for a block of zeros),    element = x / 2^(b - 127)
 * rounded to the nearest of those values, ties to the even code, magnitudes above 6 to 6.  (amax / 2^(b - 127) is below 8: an
 * element of 7 and more becomes 6.)  A block that holds a NaN or an infinity gets b = 255: four bits have neither.
 * Q(X) below is X quantised and read back.
 *
 * Conventions are those of ozimmu.h: row-major matrices with leading dimensions counted in elements, device pointers owned by the
 * caller, no allocation, all work enqueued on `stream`, OZIMMU_OK or a negative status, nothing enqueued when a check fails.
 * Rows may begin at any element: leading dimensions (below 2^40, and rows x leading dimension below 2^60) and pointers need the
 * alignment of their element type only.  Inputs and outputs of a call must not overlap.  No state is kept between calls, and
 * every call may be captured into a HIP graph.  Results do not depend on timing: the same call gives the same bits.
 */
#ifndef OZIMMU_MX_H
#define OZIMMU_MX_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* element types of unpacked matrices */
enum { OZIMMU_MX_F32 = 0, OZIMMU_MX_BF16 = 1, OZIMMU_MX_F16 = 2 };

/* Bytes of the packed form of a matrix of `rows` rows and n columns; 0 for sizes out of range (rows > 2^22 - 256, n > 2^29).
 * The packed layout is private to the library (see ozimmu_mx_pack / ozimmu_mx_unpack for the plain one); a packed matrix lies at a
 * 256-byte aligned address and may be copied as plain bytes.  Host, pure. */
size_t ozimmu_mx_bytes(int64_t rows, int64_t n);

/* X (device, rows x n, ldx >= n, of type `type`) quantised:
 *   by_row  device, ozimmu_mx_bytes(rows, n) bytes, or NULL: the packed form of X, blocks along its rows
 *   by_col  device, ozimmu_mx_bytes(n, rows) bytes, or NULL: the packed form of the transpose of X, blocks along its columns.
 * With both, X is read once.  At least one of them must be given. */
int ozimmu_mx_quantize(int type, int64_t rows, int64_t n, const void *X, int64_t ldx, void *by_row, void *by_col, void *stream);

/* X <- the values of a packed matrix (of rows x n), rounded to `type` where it cannot hold them. */
int ozimmu_mx_dequantize(int type, int64_t rows, int64_t n, const void *packed, void *X, int64_t ldx, void *stream);

/* From and to the plain layout that checkpoints hold: per row ceil(n / 32) blocks of 16 bytes, two codes a byte, the first of
 * the two in bits 0 .. 3, and ceil(n / 32) scale bytes.  Codes behind the end of a row (n not a multiple of 32) are not looked at by
 * ozimmu_mx_pack and written as zeros by ozimmu_mx_unpack.  ldc, lds: bytes between the rows of codes and of scales. */
int ozimmu_mx_pack(int64_t rows, int64_t n, const uint8_t *codes, int64_t ldc, const uint8_t *scales, int64_t lds, void *packed,
                   void *stream);
int ozimmu_mx_unpack(int64_t rows, int64_t n, const void *packed, uint8_t *codes, int64_t ldc, uint8_t *scales, int64_t lds,
                     void *stream);

/* Bytes of device workspace (256-byte aligned, contents irrelevant) that ozimmu_mx_linear needs for X of m x n and D of m x p, 0 where it
 * takes one launch and needs none (workspace may be NULL then), and ozimmu_mx_linear_backward for X of m x n and G of m x p (one size,
 * whichever of the gradients are asked for).  Calls that may run at the same time must not share one.  0 for sizes out of range.  Host, pure. */
size_t ozimmu_mx_workspace_bytes(int64_t m, int64_t n, int64_t p);
size_t ozimmu_mx_backward_workspace_bytes(int64_t m, int64_t n, int64_t p);

/* D <- alpha A B^T + beta D: A packed m x n, B packed p x n, D (device, m x p, ldd >= p) of type `type`.
 * Sums are formed in FP32 on the matrix cores; alpha and beta are applied in FP32 and D is rounded once.  beta == 0: the old D is
 * not read.  n == 0: the product is zero. */
int ozimmu_mx_gemm(int64_t m, int64_t n, int64_t p, float alpha, const void *A, const void *B, float beta, int type, void *D,
                   int64_t ldd, void *stream);

/* The same, run in a given way instead of the library's choice (OZIMMU_ERR_WAY where it cannot run so); and that choice.  Debug / test
 * helpers; the second one is host, pure. */
enum { OZIMMU_MX_WAY_AUTO = -1,
       OZIMMU_MX_WAY_DIRECT = 0,    /* 64 rows and 16 to 64 columns a workgroup, operands from memory into registers */
       OZIMMU_MX_WAY_TILE = 1,      /* 256 x 256 outputs a workgroup at a time, operands through LDS; inner dimensions above 384 */
       OZIMMU_MX_WAY_HALF = 2 };    /* 256 x 128; inner dimensions above 640 */
int ozimmu_mx_gemm_way(int way, int64_t m, int64_t n, int64_t p, float alpha, const void *A, const void *B, float beta, int type,
                       void *D, int64_t ldd, void *stream);
int ozimmu_mx_choose(int64_t m, int64_t n, int64_t p, int64_t ldd);

/* The forward pass of a linear layer: D <- alpha Q(X) W^T + beta D, X (device, m x n, ldx >= n) of type `xtype`, W packed
 * p x n, D of type `dtype`.  The product that ozimmu_mx_quantize(X) and ozimmu_mx_gemm make; for few rows in one launch, whose FP32 sums are
 * formed in another order (the last bits of D may differ from theirs). */
int ozimmu_mx_linear(int64_t m, int64_t n, int64_t p, float alpha, int xtype, const void *X, int64_t ldx, const void *W, float beta,
                     int dtype, void *D, int64_t ldd, void *workspace, size_t workspace_bytes, void *stream);

/* Its gradient, from the gradient G (m x p) of its output, each operand quantised along the dimension that is summed over:
 *   dX <- alpha Q(G) Wt^T + beta_x dX      (m x n; Wt packed n x p: by_col of ozimmu_mx_quantize for the weights, p x n)
 *   dW <- alpha Q(G^T) Q(X^T)^T + beta_w dW  (p x n)
 * X and G are of type `type`, dX of dx_type, dW of dw_type.  dX or dW may be NULL (Wt, or X, is not looked at then).
 * (The rounding of the quantisation counts as the identity: the gradient of the layer with the operands it multiplied.) */
int ozimmu_mx_linear_backward(int64_t m, int64_t n, int64_t p, float alpha, int type, const void *G, int64_t ldg, const void *X,
                              int64_t ldx, const void *Wt, float beta_x, int dx_type, void *dX, int64_t lddx, float beta_w,
                              int dw_type, void *dW, int64_t lddw, void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* OZIMMU_MX_H */
