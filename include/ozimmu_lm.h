/*
 * ozimmu_lm.h - C ABI of the operators around a model's output layer (gfx950 / MI355X): a linear layer whose weights are stored in 4 bits
 * with a scale per group, and the cross entropy of a linear layer's outputs over a large vocabulary, with its gradient.
 *
 * Weights in 4 bits.  A matrix of p rows and n columns is cut along its rows into groups of 32, 64 or 128 elements (the last of a row may be
 * shorter).  A group has a scale of 16 bits and, if the matrix has zero points, a zero point of 0 .. 15 (else 8); an element is a code q of
 * 0 .. 15 and stands for scale (q - zero).  Quantisation of a group:
 *     without zero points   scale = max|x| / 7
 *     with them             scale = (hi - lo) / 15, zero = round(-lo / scale) within 0 .. 15, hi = max(0, max x), lo = min(0, min x)
 *     q = round(x / scale) + zero, within 0 .. 15
 * Differences and quotients are FP32 numbers, each rounded once; the scale is rounded to its type (where that overflows: its largest number);
 * roundings to whole numbers take ties to the even one.  Where the scale is 0 every code is the zero point (0 with zero points).  A group that holds
 * a NaN or an infinity gets a NaN as its scale.
 *
 * Cross entropy.  With logits z = X W^T (X: m tokens x n, W: p words x n), lse_t = log sum_v exp z_tv and target y_t:
 *     loss_t = lse_t - z_t,y_t,
 *     d_tv = g_t (exp(z_tv - lse_t) - [v = y_t]),   dX = d W,   dW = d^T X        (g_t: the gradient of loss_t)
 * A row whose target is `ignore` has loss 0, a row of zeros in dX and no part in dW, whatever X and g hold there.  A target that is neither `ignore` nor
 * one of 0 .. p - 1 has a NaN as its loss, in its row of dX and in all of dW.  z is never stored: the loss takes it a tile at a time, the gradient
 * computes it again, a piece of the vocabulary at a time.  X and W are of one 16-bit type.  Products are summed in FP32; the slopes
 * exp(z - lse) - [v = y] are rounded to 16 bits (FP16: times 2^15) before they are multiplied, as gradients of 16-bit logits are.  For dW, X g / max|g| is
 * rounded to 16 bits too: in BF16 to 8 digits; in FP16 to 11, or to 2^-21 of the largest |x| of its row where that is more, whatever g is (tokens whose |x g| is
 * far below the largest are added in FP32, to a dW that is rounded twice then).
 *
 * Conventions are those of ozimmu_mx.h: row-major matrices with leading dimensions counted in elements, device pointers owned by the caller, no
 * allocation, all work enqueued on `stream`, OZIMMU_OK or a negative status, nothing enqueued when a check fails; rows may begin at any element of
 * their type; inputs and outputs of a call must not overlap; no state between calls; every call may be captured into a HIP graph; the same call
 * gives the same bits.  Workspaces are 256-byte aligned and their contents irrelevant; calls that may run at the same time must not share one.
 * Numbers of rows (m, p) are at most 2^22 - 256, inner dimensions n at most 2^20, leading dimensions below 2^40.
 */
#ifndef OZIMMU_LM_H
#define OZIMMU_LM_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* element types: those of ozimmu_mx.h */
enum { OZIMMU_LM_F32 = 0, OZIMMU_LM_BF16 = 1, OZIMMU_LM_F16 = 2 };

/* Bytes of the packed form of 4-bit weights of p rows and n columns; 0 for sizes out of range or a group that is not 32, 64 or 128.  The
 * layout is private to the library; a packed matrix lies at a 256-byte aligned address and may be copied as plain bytes.  Host, pure. */
size_t ozimmu_lm_bytes(int64_t p, int64_t n, int group, int zeros);

/* W (device, p x n, of type `type`) quantised; scales of type scale_type (BF16 or F16). */
int ozimmu_lm_quantize(int type, int64_t p, int64_t n, const void *W, int64_t ldw, int group, int zeros, int scale_type, void *packed,
                       void *stream);

/* W <- the values of packed weights, rounded to `type` where it cannot hold them. */
int ozimmu_lm_dequantize(int type, int64_t p, int64_t n, int group, int zeros, int scale_type, const void *packed, void *W, int64_t ldw,
                         void *stream);

/* From and to the plain layout that checkpoints hold: per row ceil(n / 2) bytes of two codes each, the first in bits 0 .. 3, ceil(n / group)
 * scales of 16 bits and, with zero points, as many bytes of 0 .. 15 (NULL: without; bits 4 .. 7 are not looked at).  A code behind the end
 * of a row (odd n) is not looked at by ozimmu_lm_pack and written as zero by ozimmu_lm_unpack.  ldc, ldz: bytes between rows; lds: scales. */
int ozimmu_lm_pack(int64_t p, int64_t n, int group, const uint8_t *codes, int64_t ldc, const void *scales, int64_t lds, const uint8_t *zeros,
                   int64_t ldz, void *packed, void *stream);
int ozimmu_lm_unpack(int64_t p, int64_t n, int group, const void *packed, uint8_t *codes, int64_t ldc, void *scales, int64_t lds,
                     uint8_t *zeros, int64_t ldz, void *stream);

/* D <- alpha X W^T + beta D: X (device, m x n, of type xtype: BF16 or F16), W packed p x n, D (device, m x p, of type dtype).
 * Sums in FP32, alpha and beta applied in FP32, D rounded once; beta == 0: the old D is not read.  There are two forms.  In the first, always taken up to 16
 * rows, the codes are multiplied as they are and nothing else is rounded.  In BF16 it sums x (128 + q) and takes (128 + zero) times the sum of x off again: what
 * passes through the FP32 sums is up to ten times larger than the values, and a row of X that holds an infinity, or numbers of 2^113 and more, may give NaN.
 * In the second the weights are read back in the type of X, a piece at a time, each rounded once.  In FP16 with scales in BF16 they are held times a power of
 * two, so that no scale is out of its range (those below 2^-28 of the piece's largest lose digits); with scales in FP16 weights beyond 65504 become infinite.
 * The library takes the first up to 512 rows, or up to m p = 2^21 where that is more of them, and the second beyond (ozimmu_lm_linear_choose
 * tells); results whose roundings may not depend on the number of rows are had from ozimmu_lm_linear_way.
 * n is 1 at the least (nothing is stored of n = 0).
 * Workspace: 0 bytes (workspace may be NULL then) up to 16 rows, and for more of them where the codes are multiplied without splitting the sums. */
size_t ozimmu_lm_linear_workspace_bytes(int64_t m, int64_t n, int64_t p);
int ozimmu_lm_linear(int64_t m, int64_t n, int64_t p, float alpha, int xtype, const void *X, int64_t ldx, int group, int zeros, int scale_type,
                     const void *W, float beta, int dtype, void *D, int64_t ldd, void *workspace, size_t workspace_bytes, void *stream);

/* The same, run in a given way instead of the library's choice (OZIMMU_ERR_WAY where there is no such way), with the workspace that
 * way needs; and that choice.  Debug / test helpers; the last two are host, pure. */
enum { OZIMMU_LM_WAY_AUTO = -1,
       OZIMMU_LM_WAY_DIRECT = 0,   /* from the stored codes into registers */
       OZIMMU_LM_WAY_TILE = 1,     /* weights read back, tiles of 128 x 128 to 256 x 256 outputs a workgroup at a time */
       OZIMMU_LM_WAY_SHARED = 2 }; /* from the stored codes, rows of X shared in LDS, the inner dimension split where outputs are few */
int ozimmu_lm_linear_way(int way, int64_t m, int64_t n, int64_t p, float alpha, int xtype, const void *X, int64_t ldx, int group, int zeros,
                         int scale_type, const void *W, float beta, int dtype, void *D, int64_t ldd, void *workspace, size_t workspace_bytes,
                         void *stream);
size_t ozimmu_lm_linear_way_workspace_bytes(int way, int64_t m, int64_t n, int64_t p);
int ozimmu_lm_linear_choose(int64_t m, int64_t n, int64_t p);

/* loss and lse (device, FP32, m each) of X (m x n), W (p x n) of type `type` and targets (device, m, y_stride elements apart).  n and p are 1 at the
 * least, and m times n, each rounded up to a multiple of 256, is below 2^31 - 2^20.  A row with a logit of +infinity has a NaN as its lse (and, unless it is
 * ignored, as its loss).  Workspace bytes: 0 for sizes out of range. */
size_t ozimmu_lm_cross_entropy_workspace_bytes(int64_t m, int64_t n, int64_t p);
int ozimmu_lm_cross_entropy(int type, int64_t m, int64_t n, int64_t p, const void *X, int64_t ldx, const void *W, int64_t ldw, const int64_t *y,
                            int64_t y_stride, int64_t ignore, float *loss, float *lse, void *workspace, size_t workspace_bytes, void *stream);

/* Its gradient, from the gradient g (device, FP32, m, g_stride elements apart; 0: one for all) of the losses and the lse of the forward pass:
 *   dX <- d W               (m x n, of type dx_type)
 *   dW <- d^T X + beta dW   (p x n, of type dw_type; beta == 0: the old dW is not read)
 * dX or dW may be NULL. */
size_t ozimmu_lm_cross_entropy_backward_workspace_bytes(int64_t m, int64_t n, int64_t p);
int ozimmu_lm_cross_entropy_backward(int type, int64_t m, int64_t n, int64_t p, const float *g, int64_t g_stride, const void *X, int64_t ldx,
                                     const void *W, int64_t ldw, const int64_t *y, int64_t y_stride, int64_t ignore, const float *lse, int dx_type,
                                     void *dX, int64_t lddx, float beta, int dw_type, void *dW, int64_t lddw, void *workspace,
                                     size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* OZIMMU_LM_H */
