/*
 * hetsim_ops.h -- C ABI of the layer operators: hand-written gfx950 kernels
 * for the dense part of a transformer layer's training and serving step.
 *
 * The evaluator of hetsim.h takes each device type's TFLOP/s and GB/s as
 * given, where the paper profiles the layers themselves on every device type
 * (Sec. 4.2 "Workload layer", [C1]).  These operators run such a layer on the
 * card at hand, so that the rates of a device type can be measured
 * (paper_2508_05370_amd/calibrate.py) and a layer's step be timed:
 *
 *   sim_op_quantize      a matrix into 8-bit floating point with a scale for
 *                        each block of 128
 *   sim_op_matmul        the product of two such matrices
 *   sim_op_linear        activations in 16 or 32 bits times a weight that is
 *                        held in 8 bits (serving)
 *   sim_op_norm          the norm of a block's output, its gate and residual
 *                        scale, and the norm of the sum
 *   sim_op_norm_backward its gradients
 *   sim_op_adamw         one AdamW step over many tensors, moments in 32 or
 *                        in 8 bits
 *
 * paper_2508_05370_amd/ops.py offers them on torch tensors.
 *
 * All pointers are device memory of the caller unless said otherwise; calls
 * only enqueue work on `stream` (a hipStream_t; NULL = null stream) of the
 * current device, allocate nothing, keep nothing between calls and may be
 * recorded into a HIP graph.  Workspaces are the caller's and need no
 * preparation; two calls that may overlap in time need two.  Return codes
 * are hetsim.h's: SIM_EINVAL for a NULL or misaligned pointer, a size or
 * stride out of range or an unknown type, SIM_EHIP if a launch fails.
 * Results do not depend on the timing of a launch: no sum is made by
 * atomics.
 */
#ifndef HETSIM_OPS_H
#define HETSIM_OPS_H

#include <stddef.h>
#include <stdint.h>

#include "hetsim.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types */
#define SIM_BF16 0
#define SIM_FP16 1
#define SIM_FP32 2
#define SIM_NONE 3

/* kinds of norm */
#define SIM_NORM_NONE 0
#define SIM_NORM_RMS 1     /* v / sqrt(mean(v^2) + eps) */
#define SIM_NORM_LAYER 2   /* (v - mean(v)) / sqrt(mean((v - mean(v))^2) + eps) */

#define SIM_BLOCK 128                /* elements to a scale */
#define SIM_MATMUL_MAX_K (1 << 23)   /* longest sum sim_op_matmul makes */
#define SIM_NORM_MAX_HIDDEN 32768    /* longest row sim_op_norm takes */

/*
 * The 8-bit block form of a matrix X [rows, cols]:
 *   codes  [rows][ld]        OCP e4m3 (largest value 448); ld is a multiple
 *                            of 16 and at least cols rounded up to 128, the
 *                            codes past cols are zero; 16-byte aligned
 *   scales [cols/128][ld_s]  one 32-bit scale for each 128 columns (the last
 *                            block may be shorter) of one row (block_rows 1,
 *                            ld_s >= rows) or of 128 rows (block_rows 128,
 *                            ld_s >= rows/128), both rounded up
 * X[r][c] = code[r][c] * scale[c/128][r/block_rows].  With a the largest
 * absolute value of a block, or 2^-110 where that is larger, and f the 32-bit
 * quotient 448/a, an element's code is its 32-bit product with f rounded to
 * nearest even, and the scale is the 32-bit quotient a/448.  An infinity
 * makes its block's elements NaN; a NaN makes itself one.
 */
typedef struct {
  uint8_t* codes;
  int64_t ld;
  float* scales;
  int64_t ld_s;
  uint32_t block_rows;   /* 1 or 128 */
} sim_blocks;

/*
 * X [rows, cols] (dtype SIM_BF16, SIM_FP16 or SIM_FP32, row stride ld
 * elements, any alignment of its own type) into the block form `q` and, in
 * the same pass, its transpose [cols, rows] into `qt`.  Either may have
 * codes == NULL: not wanted.  Both have the same block_rows: with 1 the
 * transpose's blocks are 128 rows of one column of X; with 128 both share
 * the codes and the scales are transposed.  rows = 0 or cols = 0: no-op.
 * rows and cols are below 2^31; 2^31 - 128 columns are the most, unless rows
 * alone are wanted with block_rows 1.
 */
int sim_op_quantize(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, const sim_blocks* q,
                    const sim_blocks* qt, void* stream);

/*
 * C[m][n] = sum over k of A[m][k] B[n][k], A [m, k] and B [n, k] in the block
 * form; C of type c_dtype (row stride ldc elements) is overwritten, or added
 * to with `accumulate`.  The products of a block of 128 are summed by the
 * matrix cores, whose alignment of the 8-bit products keeps about 16 bits
 * below the largest product (measured: 1.3e-5 of the result on normal
 * inputs), the blocks' sums in 32 bits.  k = 0 gives zeros; k and the
 * operands' ld are at most SIM_MATMUL_MAX_K.
 * `workspace` holds the partial sums of products that are split over k:
 * sim_op_matmul_workspace(m, n, k) bytes (it may be 0), 16-byte aligned.
 */
size_t sim_op_matmul_workspace(int64_t m, int64_t n, int64_t k);
int sim_op_matmul(const sim_blocks* a, const sim_blocks* b, int64_t m, int64_t n, int64_t k, void* c, int c_dtype,
                  int64_t ldc, int accumulate, void* workspace, size_t workspace_bytes, void* stream);

/*
 * y = x W^T: x [tokens, k] of type dtype (row stride ldx) is brought to the
 * block form with a scale for each row and 128 columns, W [n, k] is in the
 * block form already; y [tokens, n] has type dtype, row stride ldy.  The
 * result is that of sim_op_quantize and sim_op_matmul, bit for bit where both
 * sum in the same order.  workspace: sim_op_linear_workspace bytes, 16-byte
 * aligned.
 */
size_t sim_op_linear_workspace(int64_t tokens, int64_t n, int64_t k);
int sim_op_linear(const void* x, int dtype, int64_t ldx, const sim_blocks* w, int64_t tokens, int64_t n, int64_t k,
                  void* y, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The end of one block of a transformer and the beginning of the next, for
 * `rows` tokens of `hidden` channels:
 *   n = post(y) * post_weight + post_bias          (n = y with post = NONE)
 *   r = alpha * h + beta * gate * n                (r = h with y = NULL)
 *   h_out = r                                      (rounded to h's type)
 *   x = pre(r) * pre_weight + pre_bias             (with pre = NONE: none)
 * computed in 32 bits.  Weights and biases are [hidden], 32 bits, NULL = one
 * and zero.  gate is [ceil(rows / rows_per_gate)][hidden], contiguous, of
 * type act: token t takes row t / rows_per_gate (rows_per_gate >= rows: one
 * row for all); NULL = one.
 * y and x have type act, h and h_out type res (act or SIM_FP32); ld_* are
 * row strides in elements.  h_out may be h, or NULL where it is not wanted.
 * x goes to `x` or, with xq, into the block form with block_rows 1.
 * post_stats and pre_stats ([2][rows]: means, then reciprocal deviations) are
 * what the backward pass needs; NULL = not wanted.  hidden is at most
 * SIM_NORM_MAX_HIDDEN.
 */
typedef struct {
  int64_t rows, hidden;
  int act, res;                    /* element types */
  int post, pre;                   /* kinds of norm */
  float alpha, beta, eps;
  const void* h;       int64_t ld_h;
  const void* y;       int64_t ld_y;
  const void* gate;    int64_t rows_per_gate;
  const float* post_weight;
  const float* post_bias;
  const float* pre_weight;
  const float* pre_bias;
  void* h_out;         int64_t ld_h_out;
  void* x;             int64_t ld_x;
  const sim_blocks* xq;            /* host struct */
  float* post_stats;
  float* pre_stats;
} sim_norm_args;

int sim_op_norm(const sim_norm_args* args, void* stream);

/*
 * Gradients of sim_op_norm from those of h_out (dh_out, type res) and of x
 * (dx, type act; read where pre != NONE).  h is the forward pass's h_out, y,
 * gate, weights, statistics and constants are its own.  Written: dh (type
 * res), dy (type act), and in 32 bits dgate (gate's shape), dpost_weight,
 * dpost_bias, dpre_weight, dpre_bias ([hidden]); any of them NULL = not
 * wanted.  dh may be dh_out.  With y = NULL in the forward pass: y = NULL,
 * dy = NULL, and dh is r's gradient.  workspace:
 * sim_op_norm_backward_workspace bytes (rows_per_gate: rows, without a gate),
 * 16-byte aligned.
 */
typedef struct {
  int64_t rows, hidden;
  int act, res;
  int post, pre;
  float alpha, beta;
  const void* dh_out;  int64_t ld_dh_out;   /* NULL = zero */
  const void* dx;      int64_t ld_dx;
  const void* h;       int64_t ld_h;
  const void* y;       int64_t ld_y;
  const void* gate;    int64_t rows_per_gate;
  const float* post_weight;
  const float* post_bias;
  const float* pre_weight;
  const float* post_stats;
  const float* pre_stats;
  void* dh;            int64_t ld_dh;
  void* dy;            int64_t ld_dy;
  float* dgate;
  float* dpost_weight;
  float* dpost_bias;
  float* dpre_weight;
  float* dpre_bias;
} sim_norm_grad_args;

size_t sim_op_norm_backward_workspace(int64_t rows, int64_t hidden, int64_t rows_per_gate);
int sim_op_norm_backward(const sim_norm_grad_args* args, void* workspace, size_t workspace_bytes, void* stream);

/*
 * One AdamW step over `n` tensors (host array; the pointers in it are device
 * memory, each aligned to its element type):
 *   g = grad * grad_scale
 *   m = beta1 m + (1 - beta1) g;  v = beta2 v + (1 - beta2) g g
 *   p = p (1 - lr weight_decay) - lr / (1 - beta1^step) m
 *                                / (sqrt(v / (1 - beta2^step)) + eps)
 * in 32 bits; p (p_dtype) is rounded to its type, and `copy` (copy_dtype,
 * SIM_NONE = none) gets p too.  Every operation of the moments is rounded by
 * itself (no fused multiply-add), so that their codes are reproducible.
 * state_bits 32: m and v are float [n].
 * state_bits 8: m and v are e4m3 codes [n] with a scale for each 128 elements
 * (m_scale, v_scale [ceil(n/128)]); v holds sqrt(v).  Scales are those of the
 * block form; the codes are rounded down or up with the probability of the
 * distance (nearest rounding would freeze v: one step moves sqrt(v) by less
 * than half of a code's spacing).  The probabilities are compared with 16-bit
 * numbers each from a counter: with mix() the 32-bit function
 *   x ^= x >> 16; x *= 0x9E3779B9; x ^= x >> 15; x *= 0x85A308D3; x ^= x >> 16
 * and key = mix(mix(mix(seed low) ^ seed high) ^ step), element i of a tensor
 * whose `first` is f (a multiple of 128) takes bits = mix(mix(key ^ high(f + i)) ^ low(f + i)),
 * the lower half for m and the upper half for v.  sqrt(v) > 0 gets the
 * smallest code at least, so that an element's update stays bounded.
 * grad_scale (one float, NULL = 1) multiplies every gradient; where *skip is
 * not zero (NULL = never) the whole step changes nothing.
 */
typedef struct {
  void* p;
  const void* grad;
  void* m;
  void* v;
  float* m_scale;
  float* v_scale;
  void* copy;
  int64_t n;
  uint64_t first;
  float weight_decay;
} sim_adamw_tensor;

typedef struct {
  int p_dtype, grad_dtype, copy_dtype, state_bits;
  double lr, beta1, beta2, eps;
  int64_t step;             /* 1 for the first step */
  uint64_t seed;
  const float* grad_scale;
  const uint32_t* skip;
} sim_adamw_args;

int sim_op_adamw(const sim_adamw_tensor* tensors, int64_t n, const sim_adamw_args* args, void* stream);

#ifdef __cplusplus
}
#endif
#endif
