/*
 * polyq_finetune.h - C ABI of the operators that fine-tune a quantised model on
 * GB300 (sm_103a) and serve the result: layer norm, AdamW and low-rank adapters.
 *
 * They stand around the products of polyq.h and polyq_fp4.h: the norm before a
 * projection with its gradients, the adapters of many requests (or of a training
 * step) beside a projection whose quantised weights stay as they are, and the
 * optimiser's step over all trained tensors at once.
 *
 * The conventions of polyq.h hold: return codes and polyq_last_error(), caller
 * owns every buffer, entry points check their arguments on the host, never
 * allocate device memory and never synchronise, `stream` is a cudaStream_t.
 * Every entry works on the current device and may be captured in a CUDA graph.
 * Sizes are at least 1 (an empty tensor is POLYQ_EINVAL), rows and widths at most 2^24.  Outputs must not
 * overlap inputs or each other unless stated otherwise.  A workspace may serve
 * consecutive calls on one stream, but not calls that run at the same time.  Results do not change from run to run.
 */
#ifndef POLYQ_FINETUNE_H
#define POLYQ_FINETUNE_H

#include "polyq_fp4.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- layer norm ---- */

#define POLYQ_NORM_MAX_K 24576 /* widest row */

/* y[r][k] = hat[r][k] weight[k] + bias[k] of x [rows][K],
 *   hat = (x - mean) rstd, rstd = 1 / sqrt(mean of (x - mean)^2 + eps),
 *   mean = the row's mean with center != 0 (layer norm), else 0 (RMS norm).
 * x and y of any type and row stride; y may be x itself where both have one type
 * and stride (another one is POLYQ_EINVAL).  weight, bias: K elements (their
 * stride does not matter) of any type, each may be NULL (1 and 0).  stats: NULL,
 * or device memory of 2*rows floats, 8-byte aligned, which receives (mean, rstd)
 * of every row for the backward pass.  The row is held in fp32, its mean is taken
 * before the squares of what is left are summed (their sum must stay within fp32),
 * and one rounding makes y.  One launch.
 * K above POLYQ_NORM_MAX_K is POLYQ_EUNSUPPORTED. */
int polyq_layernorm_forward(const polyq_dense* x, int64_t rows, int64_t K, const polyq_dense* weight,
                            const polyq_dense* bias, float eps, int center, const polyq_dense* y,
                            float* stats, void* stream);

int polyq_layernorm_workspace_bytes(int64_t rows, int64_t K, size_t* bytes);

/* Gradients for the gradient dy [rows][K] of y and the stats of the forward pass:
 *   g = dy weight,  dx = residual + rstd (g - [mean of g] - hat mean of (g hat)),
 *   dweight = sum over rows of dy hat, dbias = sum over rows of dy
 * with the mean of g only where center != 0.  dx NULL (not wanted) or of x's type;
 * residual NULL or [rows][K] of dx's type (the gradient that reaches x beside the
 * norm; its data may be dx's, with dx's stride); dweight, dbias: NULL or K
 * elements of any type; at least one of the three is wanted.  dx may be dy's
 * memory where both have one type and stride.  (Other strides or types in place are
 * POLYQ_EINVAL; a single row's stride does not matter.)
 * The workspace (polyq_layernorm_workspace_bytes, 16-byte aligned) is needed with
 * dweight or dbias: every SM's sums over its rows, which a second launch adds in
 * a fixed order. */
int polyq_layernorm_backward(const polyq_dense* x, int64_t rows, int64_t K, const polyq_dense* weight,
                             const float* stats, int center, const polyq_dense* dy,
                             const polyq_dense* residual, const polyq_dense* dx,
                             const polyq_dense* dweight, const polyq_dense* dbias, void* workspace,
                             size_t workspace_bytes, void* stream);

/* ---- AdamW ---- */

#define POLYQ_ADAMW_BLOCK 256 /* elements of an 8-bit state that share a scale */

/* A trained tensor of n elements without gaps: its parameters, its gradient and,
 * where `copy` is not NULL, a second place for the new parameters in another type
 * (16-bit weights made of fp32 ones).  Each aligned to its element size.  Its state
 * begins at element `at` of the state's buffers, a multiple of POLYQ_ADAMW_BLOCK;
 * tensors' states must not overlap, nor may any other buffers. */
typedef struct {
  void* p;
  const void* grad;
  void* copy;
  int64_t n;    /* 1..2^38 */
  int64_t at;   /* 0..2^38 */
  float decay;  /* of the decoupled weight decay, >= 0 */
  float rate;   /* factor of the learning rate, >= 0 */
} polyq_adamw_tensor;

/* The moments of all tensors.  bits 32: m and v are fp32, 16-byte aligned; m_scales
 * and v_scales do not matter.  bits 8: m and v are uint8 codes, 16-byte aligned, with
 * one scale byte per block of POLYQ_ADAMW_BLOCK elements, 2^(byte-127) (255 is NaN):
 *   m        sign in bit 7, bits 0..6 a magnitude of 4 exponent and 3 mantissa bits
 *   v        the root of the second moment, 4 exponent and 4 mantissa bits
 * A magnitude with exponent bits E and mantissa F (a fraction) is F for E = 0 and
 * (1 + F) 2^(E-1) else, so that its highest binade begins at 2^14.  A tensor's last
 * block belongs to it whole: what lies past its n elements is set to 0. */
typedef struct {
  void* m;
  void* v;
  uint8_t* m_scales;
  uint8_t* v_scales;
  int64_t n;  /* elements of m and of v, a multiple of POLYQ_ADAMW_BLOCK */
  int32_t bits;
} polyq_adamw_state;

typedef struct {
  double lr, beta1, beta2, eps; /* lr >= 0, 0 <= beta < 1, 2^-126 <= eps <= 1e30 */
  int64_t step;                 /* 1, 2, ...: this step's number */
  uint64_t seed;                /* of the rounding of 8-bit states: another one for each step, or the
                                   same elements are rounded the same way every time and small
                                   moments never change.  (`step` does not enter; step_dev does.) */
  /* Device values, read when the step runs (so that a captured step can take new
   * ones); each may be NULL. */
  const float* lr_dev;          /* the learning rate in place of lr */
  const int64_t* step_dev;      /* the step's number in place of step (below 1 counts as 1), also
                                   added to the seed */
  const float* grad_scale;      /* factor of every gradient; the step leaves everything as it
                                   was where it is not finite */
} polyq_adamw_hyper;

/* One step of all tensors:
 *   m = beta1 m + (1-beta1) g,  v = beta2 v + (1-beta2) g^2   (g the scaled gradient)
 *   p = p (1 - lr rate decay) - lr rate / (1-beta1^t) m / (sqrt(v / (1-beta2^t)) + eps)
 * in fp32, p rounded once to its type, copy once from p; m and v as (beta1 m) + ((1-beta1) g)
 * and (beta2 v) + (((1-beta2) g) g), each operation rounded, and the root to nearest.  All tensors of a call have one
 * type of p, one of the gradient and one of the copies (any of POLYQ_F32, POLYQ_BF16,
 * POLYQ_F16).
 * 8-bit states are rounded after p has been computed: a block's scale is the smallest with
 * which its largest magnitude is at most the largest code, and a magnitude is rounded down
 * after adding a fraction u of its last place (up with a probability that equals the part
 * cut off, so that a moment's slow changes are not lost; a root that is not 0 is at least
 * the smallest code).  u takes 16 bits of a hash of the seed and the element's
 * place in the state, m the low and v the high half:
 *   mix(h):  h = (h ^ h >> 16) * 0x9E2D58A5;  h = (h ^ h >> 15) * 0x6C62272D   (mod 2^32)
 *   key = mix(mix(block ^ mix(seed + 1)) ^ block >> 32 ^ seed >> 32)
 *   h = mix(key + 0x9E3779B1 * (element % 256));  bits = h ^ h >> 16
 * A block with an infinity or a NaN gets the scale NaN and codes 0.
 * Up to 640 tensors a launch. */
int polyq_adamw_step(const polyq_adamw_tensor* tensors, int32_t n_tensors, int32_t p_type,
                     int32_t grad_type, int32_t copy_type, const polyq_adamw_state* state,
                     const polyq_adamw_hyper* hyper, void* stream);

/* The values of an 8-bit state: m and the root of v, each NULL or state->n elements of any type, rounded
 * once (bf16 and fp32 hold them exactly).  One launch. */
int polyq_adamw_values(const polyq_adamw_state* state, const polyq_dense* m, const polyq_dense* root,
                       void* stream);

/* ---- low-rank adapters ---- */

#define POLYQ_ADAPTERS_MAX_RANK 128

/* n adapters beside a projection from K to N channels, in one 16-bit type (POLYQ_BF16 or
 * POLYQ_F16): a [n][R][K] and b [n][N][R], 16-byte aligned, rows of a_stride and b_stride
 * elements, a_next and b_next elements from one adapter to the next, all multiples of 8 (many
 * rows are fastest where a_next and b_next are 0 or multiples of the rows' stride that hold a matrix).
 * R is a multiple of 8 (above POLYQ_ADAPTERS_MAX_RANK POLYQ_EUNSUPPORTED); an adapter of a
 * smaller rank has it in `ranks`, and what a and b hold past it does not matter.
 * Beside a layer of polyq.h, a's columns are in the order of the x that both read (the layer
 * gathers by itself), and b's rows in that of the y that it emits: the channels' own, or that of
 * polyq_layer_permute_rows, whose permutation b's rows then take as well. */
typedef struct {
  const void* a;
  const void* b;
  int64_t a_stride, a_next, b_stride, b_next;
  int64_t K, N;
  int32_t n, R, type;
  const float* scales;   /* device [n], or NULL: 1 */
  const int32_t* ranks;  /* device [n], 0..R, or NULL: R */
} polyq_adapters;

/* Which rows go through which adapter: segment i is rows offsets[i] .. offsets[i+1] - 1
 * (ascending) and adapter ids[i]; a number outside 0..n-1 is none.  Segments may be empty,
 * several may have one adapter, and rows before the first and behind the last are left
 * as they are.  Both are device arrays, read when the call runs; offsets outside the
 * tensors' rows are taken as their ends, and where they fall the rows that segments share
 * are unspecified. */
typedef struct {
  const int32_t* offsets;  /* [n+1] */
  const int32_t* ids;      /* [n] */
  int32_t n;
} polyq_segments;

/* Bytes of the workspace of the calls below for T rows: a status word in its first 4 bytes
 * (read it with polyq_workspace_status), and v or dv.  Its first
 * POLYQ_ADAPTERS_WORKSPACE_ZERO bytes must be zero before its first use, and again after a
 * wait that gave up; 16-byte aligned. */
#define POLYQ_ADAPTERS_WORKSPACE_ZERO 256
int polyq_adapters_workspace_bytes(int64_t T, int32_t R, size_t* bytes);

/* y[t][n] = residual[t][n] + s sum_j v[t][j] b[n][j],  v[t][j] = sum_k x[t][k] a[j][k]
 * of the row's adapter (scale s); rows of segments without one get the residual.  x [T][K] of the
 * adapters' type (fastest where it is 16-byte aligned with a stride that is a multiple of 8); y
 * [T][N] of that type or POLYQ_F32; residual NULL (0) or of y's type: the projection's result, its
 * data may be y's, with y's stride.  Products of x and a are exact and their sums in
 * fp32, as v is; v enters the second product with 16 (bf16) or 21 (fp16: down to 2^-17 of
 * its row's largest finite magnitude, from there on to 2^-39 of that) significant bits; one
 * rounding to y's type.  saved: NULL, or device memory of T*R floats, 16-byte
 * aligned, which receives v [T][R] for the backward pass (rows without an adapter are left
 * as they were).  Two launches. */
int polyq_adapters_forward(const polyq_dense* x, int64_t T, const polyq_adapters* adapters,
                           const polyq_segments* segments, const polyq_dense* residual,
                           const polyq_dense* y, float* saved, void* workspace,
                           size_t workspace_bytes, void* stream);

/* Gradients for the gradient dy [T][N] of y (of the adapters' type, best aligned as x) and the `saved`
 * of the forward pass:
 *   dv[t][j] = s sum_n dy[t][n] b[n][j],  dx[t][k] = residual[t][k] + sum_j dv[t][j] a[j][k]
 *   da[j][k] = sum over the adapter's rows of dv[t][j] x[t][k]
 *   db[n][j] = s sum over the adapter's rows of dy[t][n] v[t][j]
 * dx NULL or as y, with its residual (the gradient that reaches x through the
 * projection); da [n][R][K] and db [n][N][R] without gaps, of grad_type (the adapters'
 * type or POLYQ_F32), each may be NULL.  All adapters' gradients are written: zeros where no row
 * has the adapter, and past its rank.  At least one of the three is wanted; saved
 * may be NULL without db.  dv is in fp32, and enters its products as v does (fp16, da and db:
 * the largest magnitude is that of up to 64 rows).  Up to three
 * launches. */
int polyq_adapters_backward(const polyq_dense* x, int64_t T, const polyq_adapters* adapters,
                            const polyq_segments* segments, const float* saved,
                            const polyq_dense* dy, const polyq_dense* residual,
                            const polyq_dense* dx, void* da, void* db, int32_t grad_type,
                            void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* POLYQ_FINETUNE_H */
