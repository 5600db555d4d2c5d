/*
 * zf_layer.h -- the operators around the weights that libzf updates: the RMS
 * norm in front of a linear layer, its products in 8-bit floating point, and
 * the AdamW step of the parameters that are not split by channel (norm gains,
 * biases, embeddings).
 *
 *   zf_quantize_fp8      activations, gradients or weights to 8 bits
 *   zf_matmul_fp8        product of two 8-bit operands; forward pass, input
 *                        gradient and weight gradient of a linear layer
 *   zf_rmsnorm_forward   residual addition, RMS norm, 8-bit output
 *   zf_rmsnorm_backward  its gradients
 *   zf_adamw_*           AdamW over many tensors, states in 32 or 8 bits
 *
 * Conventions (device pointers, caller-owned memory, stream ordering, status
 * codes, validation before anything is enqueued) are those of zf.h.  Strides
 * (ld_*) count elements between rows.  Two buffers of one call may overlap
 * only where the call says so; ZF_EINVAL otherwise.
 *
 * The 8-bit format
 * ----------------
 * Elements are OCP e4m3 (largest magnitude 448).  Each group of elements
 * shares a scale 2^(code - 127), kept as the 8-bit code (OCP e8m0).  Groups
 * are 128 consecutive elements of a row (group 1), or blocks of 128 rows by
 * 128 columns (group 128); groups at the edges are smaller.  The code is the
 * least one with which the group's largest magnitude is at most 448 scales,
 * an element is its value over the scale rounded to nearest, ties to even.  A
 * group that holds an infinity or a NaN gets code 255 (NaN) and zero
 * elements: every product it enters is NaN.
 * Scales are powers of two because the conversions of gfx950 apply
 * such scales themselves, and dividing by one is exact.
 * An operand of `rows` rows and `cols` columns is stored as
 *   data   [rows][ld_data], ld_data >= cols a multiple of 16, 16-byte aligned;
 *          the ceil(cols / 16) * 16 first bytes of every row must be
 *          readable, those past cols may hold anything;
 *   scale  [ceil(rows / group)][ld_scale], ld_scale >= ceil(cols / 128) a
 *          multiple of 4, 4-byte aligned; the ceil(cols / 512) * 4 first
 *          bytes of every row must be readable.
 */
#ifndef ZF_LAYER_H
#define ZF_LAYER_H

#include <stddef.h>
#include <stdint.h>

#include "zf.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum zf_dtype { ZF_BF16 = 0, ZF_F32 = 1 } zf_dtype;

/* ---- 8-bit operands ------------------------------------------------------ */

/* HOST struct of DEVICE pointers: an operand in the format above. */
typedef struct zf_fp8 {
  uint8_t* data;
  int64_t ld_data;
  uint8_t* scale;
  int64_t ld_scale;
  int32_t group; /* 1 or 128 */
} zf_fp8;

/* x [rows][ld_x] (bf16 or fp32) to 8 bits: `out` receives x, `out_t` its
 * transpose (an operand of cols rows and rows columns, whose groups run along
 * x's rows).  Either may be NULL, not both; they share one `group`.  With
 * group 128 both hold the same values.  rows, cols < 2^30, fewer than 2^24
 * tiles of 128 x 128.  Bytes of the outputs past their columns are not written. */
zf_status zf_quantize_fp8(const void* x, int32_t x_dtype, int64_t rows, int64_t cols,
                          int64_t ld_x, const zf_fp8* out, const zf_fp8* out_t,
                          zf_stream stream);

/* Workspace bytes zf_matmul_fp8 needs for these sizes (0 for most). */
size_t zf_matmul_fp8_workspace_bytes(int64_t m, int64_t n, int64_t k);

/* out[i][j] = sum over l < k of a[i][l] * b[j][l], a an operand of m rows and
 * k columns, b of n rows and k columns, each with its own group; products
 * summed in fp32 and rounded once to out_dtype (bf16 or fp32).  k = 0 writes
 * zeros.  With W [n][k] a linear layer's weight:
 *   forward          y  [t][n] = matmul(x, W)
 *   input gradient   dx [t][k] = matmul(dy, W's transposed copy)
 *   weight gradient  dW [n][k] = matmul(dy's transposed copy, x's transposed
 *                    copy), the row-major gradient of zf.h; the two swapped
 *                    give the channel-major one.
 * Products and sums are fp32 with either result type, and their order depends on
 * m, n and k only: equal calls give equal bits, and a bf16 result is the fp32
 * one rounded.  Scales may lie anywhere in their range: a value of a or b (an
 * element times its scale) is held to within 2^-118 times the largest scale of
 * its row.  m, n < 2^30; k and, with more than one row, the strides of data
 * and scale < 2^23; fewer than 2^24 tiles of 128 x 128.  ws:
 * zf_matmul_fp8_workspace_bytes(m, n, k) bytes, 16-byte aligned (may be NULL if
 * that is 0), contents overwritten. */
zf_status zf_matmul_fp8(const zf_fp8* a, const zf_fp8* b, int64_t m, int64_t n, int64_t k,
                        void* out, int32_t out_dtype, int64_t ld_out, void* ws, size_t ws_bytes,
                        zf_stream stream);

/* ---- RMS norm ------------------------------------------------------------ */

/* For every row i:
 *   h[i]    = round(x[i] + residual[i])   (residual NULL: h = x, h may be NULL)
 *   rstd[i] = 1 / sqrt(mean over the row of h^2 + eps)
 *   y[i][j] = round((h[i][j] * rstd[i]) * gain[j])
 * x, residual, h, y in `dtype` (bf16 or fp32), gain in gain_dtype; the
 * arithmetic in fp32.  h is required with a residual and may be x or the
 * residual itself (the same address and stride).  y and q may each be NULL;
 * q receives y in 8 bits (group 1).  rstd: [rows] fp32, required (the
 * backward pass reads it); with cols = 0 it is 1 / sqrt(eps).  eps finite and
 * >= 0.  rows, cols < 2^30. */
zf_status zf_rmsnorm_forward(const void* x, int64_t ld_x, const void* residual,
                             int64_t ld_residual, int32_t dtype, int64_t rows, int64_t cols,
                             const void* gain, int32_t gain_dtype, double eps, void* h,
                             int64_t ld_h, void* y, int64_t ld_y, const zf_fp8* q, float* rstd,
                             zf_stream stream);

/* Workspace bytes of zf_rmsnorm_backward. */
size_t zf_rmsnorm_backward_workspace_bytes(int64_t rows, int64_t cols);

/* With hh = h * rstd, t = dy * gain, c[i] = mean over row i of t * hh:
 *   dx[i]    = round(rstd[i] * (t[i] - hh[i] * c[i]) + dresidual[i])
 *   dgain[j] = sum over i of dy[i][j] * hh[i][j]            (fp32)
 * dx is the gradient of x and of the residual alike; dresidual (may be NULL)
 * is the gradient that reaches h from elsewhere (the residual stream).  dy,
 * h, dresidual, dx in `dtype`; dx may be dy or dresidual itself (the same
 * address and stride).  The 8-bit output's rounding counts as the identity.
 * dgain: [cols], or NULL where it is not wanted; the rows are summed in an
 * order that depends on rows and cols only.  rows = 0 writes zeros to dgain.
 * ws: zf_rmsnorm_backward_workspace_bytes(rows, cols) bytes, 16-byte
 * aligned; NULL with dgain NULL. */
zf_status zf_rmsnorm_backward(const void* dy, int64_t ld_dy, const void* h, int64_t ld_h,
                              int32_t dtype, int64_t rows, int64_t cols, const void* gain,
                              int32_t gain_dtype, const float* rstd, const void* dresidual,
                              int64_t ld_dresidual, void* dx, int64_t ld_dx, float* dgain,
                              void* ws, size_t ws_bytes, zf_stream stream);

/* ---- AdamW over many tensors ---------------------------------------------- */

/* HOST struct of DEVICE pointers: one parameter of n contiguous elements.
 * States in 32 bits (scales NULL): exp_avg, exp_avg_sq are fp32 [n].
 * States in 8 bits (both scales given): exp_avg holds e4m3 codes of the first
 * moment, exp_avg_sq e4m3 codes of the second moment's square root, in blocks
 * of 128 consecutive elements with one fp32 scale each
 * ([ceil(n / 128)]); a code stands for its e4m3 value times the scale.  A
 * block is stored with scale = max / 448 and code = round(x * (448 / max)) to
 * nearest even, max its largest magnitude (each operation one fp32
 * operation); a square root that is not zero never gets code 0, so that no
 * step divides by eps alone; a block whose max is below 2^-100 is stored as
 * zeros; an infinity or NaN turns its whole block to NaN.
 * All zero bytes are the states of a fresh parameter in either form. */
typedef struct zf_adamw_tensor {
  int64_t n;
  const void* grad;
  int32_t grad_dtype; /* zf_dtype */
  float* master;
  uint16_t* weight; /* bf16 copy of the master, or NULL */
  void* exp_avg;
  void* exp_avg_sq;
  float* exp_avg_scale;
  float* exp_avg_sq_scale;
} zf_adamw_tensor;

typedef struct zf_adamw_plan zf_adamw_plan;

/* Device bytes of a plan over these tensors (its tables).  tensors: HOST
 * array of count >= 1; 32- and 8-bit states and both gradient types may be
 * mixed.  Every pointer is aligned to its element; no two buffers overlap.
 * One launch takes fewer than 2^24 blocks of 1024 elements, a tensor's last one
 * partly filled: the sum of ceil(n / 1024) over the tensors is below 2^24. */
zf_status zf_adamw_plan_query(const zf_adamw_tensor* tensors, int32_t count,
                              size_t* device_bytes);

/* Builds the plan in caller-provided device memory (at least
 * zf_adamw_plan_query's bytes, 256-byte aligned), as zf_plan_create does: the
 * upload is enqueued on `stream`, the handle is the only allocation. */
zf_status zf_adamw_plan_create(const zf_adamw_tensor* tensors, int32_t count, void* device_mem,
                               size_t device_bytes, zf_stream stream, zf_adamw_plan** out);

/* Frees the plan's host handle; no device call, no synchronisation. */
void zf_adamw_plan_destroy(zf_adamw_plan* plan);

/* One AdamW step of every tensor, in one launch: the element sequence of
 * zf_adam_selected with g = grad, or grad * *grad_scale (one fp32
 * multiplication) where grad_scale, a DEVICE scalar, is not NULL (gradient
 * clipping, loss scaling).  step >= 1. */
zf_status zf_adamw_step(zf_adamw_plan* plan, const zf_adam_hparams* hp, int64_t step,
                        const float* grad_scale, zf_stream stream);

#ifdef __cplusplus
}
#endif

#endif /* ZF_LAYER_H */
