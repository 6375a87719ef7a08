/*
 * polyq_fp4.h - C ABI of the 4-bit floating-point linear layer and of the
 * gated feed-forward block for GB300 (sm_103a).
 *
 * Beside the integer widths of polyq.h the library holds tensors in
 * microscaled 4-bit floating point, multiplies two of them on the block-scaled
 * tensor cores, and runs a decoder layer's gated feed-forward block
 * h = silu(x gate^T) * (x up^T) in one kernel, on 4-bit operands (serving) or
 * on 16-bit ones with its backward pass (quantisation-aware training).
 *
 * The conventions of polyq.h hold: return codes and polyq_last_error(), caller
 * owns every buffer, GPU entry points check their arguments on the host, never
 * allocate device memory and never synchronise, `stream` is a cudaStream_t.
 * Every entry works on the current device.  Sizes are at least 1: an empty
 * tensor is POLYQ_EINVAL.  Outputs must not overlap inputs or each other
 * unless stated otherwise.
 *
 * A 4-bit tensor [rows][K]:
 *   codes   uint8 [rows][code_stride]: element k of a row in bits 4*(k%2).. of
 *           byte k/2; a code is sign, two exponent bits and one mantissa bit
 *           (e2m1): 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives.  With an
 *           odd K the last byte's upper half is 0.  Bytes past (K+1)/2 of a row
 *           do not matter (an entry point that writes codes may set them to 0).
 *   scales  one byte per block of a row: 32 consecutive elements and a power
 *           of two 2^(byte-127) (e8m0; 255 is NaN) for POLYQ_FP4_MX, 16
 *           consecutive elements and a non-negative e4m3 number (bit 7 clear;
 *           0x7F is NaN) for POLYQ_FP4_NV.  They are stored as the tensor cores take them: the
 *           scale of block b of row r is byte
 *             ((r/128)*A + b/4)*512 + (r%32)*16 + ((r/32)%4)*4 + b%4
 *           with A = ceil(blocks per row / 4).  Bytes of blocks past a row's
 *           last must be 0 for the rows that exist; those of rows past the last
 *           are not read.
 *   An element is e2m1 * scale * tensor_scale (tensor_scale is 1 for
 *   POLYQ_FP4_MX).
 */
#ifndef POLYQ_FP4_H
#define POLYQ_FP4_H

#include "polyq.h"

#ifdef __cplusplus
extern "C" {
#endif

#define POLYQ_FP4_MX 0 /* blocks of 32, e8m0 scales */
#define POLYQ_FP4_NV 1 /* blocks of 16, e4m3 scales, a scale per tensor */

/* Element types of dense tensors. */
#define POLYQ_F32 0
#define POLYQ_BF16 1
#define POLYQ_F16 2

typedef struct {
  uint8_t* codes;       /* device, 16-byte aligned */
  uint8_t* scales;      /* device, 16-byte aligned */
  int64_t rows, K;      /* 1..2^24 each */
  int64_t code_stride;  /* bytes, a multiple of 16, at least (K+1)/2 */
  int32_t format;       /* POLYQ_FP4_* */
  float tensor_scale;   /* positive and finite; 1 for POLYQ_FP4_MX */
} polyq_fp4;

/* A dense tensor: rows of K elements, `stride` elements apart. */
typedef struct {
  void* data;      /* device, aligned to its element size */
  int64_t stride;  /* elements, at least the row's length */
  int32_t type;    /* POLYQ_F32, POLYQ_BF16 or POLYQ_F16 */
} polyq_dense;

/* Code bytes per row (16-byte rows) and bytes of the scales of a tensor. */
int polyq_fp4_bytes(int64_t rows, int64_t K, int32_t format, int64_t* code_stride,
                    int64_t* scale_bytes);

/* Quantise x [rows][K] (any type; rows and K from *out) into out->codes and
 * out->scales.
 * POLYQ_FP4_MX: a block's scale is 2^e, e = floor(log2(largest |x|)) - 2 (at
 * least -127), each element the e2m1 number nearest to x / 2^e (ties to the
 * even code, values beyond 6 to 6).
 * POLYQ_FP4_NV: t = fp32(x / tensor_scale); a block's scale s is the e4m3
 * number nearest to fp32(largest |t| / 6) (ties to even, at most 448), each
 * element the e2m1 number nearest to the exact t / s, 0 where s is 0.
 * A block that holds an infinity or a NaN (POLYQ_FP4_NV: in t, which a small
 * tensor scale may take beyond fp32) gets the scale NaN, and codes 0.
 * One launch. */
int polyq_fp4_quantize(const polyq_dense* x, const polyq_fp4* out, void* stream);

/* y[r][k] = the tensor's value, rounded once to y's type.  One launch. */
int polyq_fp4_dequantize(const polyq_fp4* t, const polyq_dense* y, void* stream);

/* Bytes of the workspace of the products below on the current device (it
 * grows with its SM count): a status word in its first 4 bytes (read it with
 * polyq_workspace_status), counters, and the parts of output tiles that several
 * SMs share.  Its first POLYQ_FP4_WORKSPACE_ZERO bytes must be zero before its
 * first use, and again after a wait that gave up.  A workspace may serve
 * consecutive calls on one stream but not calls that run at the same time. */
#define POLYQ_FP4_WORKSPACE_ZERO 16640
int polyq_fp4_workspace_bytes(size_t* bytes);

/* y[m][n] = residual[m][n] + sum_k x[m][k] w[n][k]: x [M][K] and w [N][K] in
 * one 4-bit format, whose tensor scales' product is a normal fp32 number, y
 * [M][N] of any type; residual NULL or [M][N] of y's type (its data may be y's,
 * with y's stride).  Products are exact and summed in fp32; one rounding to y's
 * type.  One launch; the result does not change from
 * run to run. */
int polyq_fp4_linear(const polyq_fp4* x, const polyq_fp4* w, const polyq_dense* residual,
                     const polyq_dense* y, void* workspace, size_t workspace_bytes, void* stream);

/* h[m][f] = silu(a) * u, a = sum_k x[m][k] gate[f][k], u = sum_k x[m][k]
 * up[f][k], silu(a) = a / (1 + exp(-a)): x [M][K], gate and up [F][K] in one
 * 4-bit format.  a, u and the activation stay in fp32, the activation by fast
 * exponential and quotient (off by up to (8 + 1.2 |a|) 2^-23 of h; below a = -87,
 * where exp(-a) nears fp32's largest number, it may be 0); exactly one of the
 * outputs is given: h [M][F] of any type, or hq [M][F] in 4 bits (either
 * format), which is h in fp32 quantised as polyq_fp4_quantize does.  One
 * launch; the result does not change from run to run. */
int polyq_fp4_ffn(const polyq_fp4* x, const polyq_fp4* gate, const polyq_fp4* up,
                  const polyq_dense* h, const polyq_fp4* hq, void* workspace,
                  size_t workspace_bytes, void* stream);

/* The gated block on 16-bit operands, for training.  x [T][K], gate and up
 * [F][K], all POLYQ_BF16 or all POLYQ_F16, 16-byte aligned with strides that
 * are multiples of 8 elements; h [T][F] of the same type.
 *   a = x gate^T, u = x up^T, h = silu(a) * u
 * in one launch.  saved: NULL, or device memory of polyq_ffn_saved_bytes,
 * 32-byte aligned, which receives a and u for the backward pass, each rounded to
 * 16 significant bits in fp32's range. */
int polyq_ffn_saved_bytes(int64_t T, int64_t F, size_t* bytes);
int polyq_ffn_forward(const polyq_dense* x, const polyq_dense* gate, const polyq_dense* up,
                      int64_t T, int64_t F, int64_t K, const polyq_dense* h, void* saved,
                      void* workspace, size_t workspace_bytes, void* stream);

/* Workspace of the backward pass on the current device: that of the products,
 * which it begins with, and the gradients of a and u. */
int polyq_ffn_backward_workspace_bytes(int64_t T, int64_t F, size_t* bytes);

/* Gradients of the block for the gradient dh [T][F] of h (x's type) and the
 * `saved` of its forward pass:
 *   s = 1/(1+exp(-a)), da = dh u s (1 + a (1-s)), du = dh a s
 *   dx [T][K] = da gate + du up, dgate [F][K] = da^T x, dup [F][K] = du^T x
 * s is as exact as the activation of polyq_fp4_ffn; da and du are rounded once to
 * x's type (as the tensor cores take them), also for gradients in fp32; sums are
 * in fp32.  Any of dx, dgate, dup may be NULL (not wanted; dgate and dup
 * both or neither); each is of x's type or POLYQ_F32, dgate and dup of one type
 * and stride (else POLYQ_EINVAL).  One launch for da and du, one for dx, one for
 * dgate and dup.  The result does not change from run to run. */
int polyq_ffn_backward(const polyq_dense* x, const polyq_dense* gate, const polyq_dense* up,
                       int64_t T, int64_t F, int64_t K, const void* saved, const polyq_dense* dh,
                       const polyq_dense* dx, const polyq_dense* dgate, const polyq_dense* dup,
                       void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* POLYQ_FP4_H */
