/*
 * act8.h - C ABI of libslide for layers whose activations are kept in 8 bits: activation checkpoints, linear layers that multiply
 * out of them (forward, input gradient, weight gradient), and group normalisation with its activation, channels last.
 *
 * What limits a slide held in memory is the activations (paper, Method: tiles per device); 8 bits hold twice the tiles of
 * bfloat16.  A matrix in 8 bits ("act8") has one e4m3 code per value and one power of two per row and block of 128 columns:
 *     value[r][c] = code[r][c] * 2^(scale[r][c / 128] - 127)
 * The power is the smallest that brings the block's largest finite magnitude to 448, the largest e4m3 number, or below (not below
 * 2^-127; 1 for a block of zeros), so packing rounds each value once, to the nearest code, and never clips.  What is not finite becomes a NaN and does not
 * count for the block's power.  Every value is exactly a bfloat16 unless it is below 2^-133, and the matrix cores take the powers as they are.
 *
 * Conventions as in slide.h: device pointers unless a comment says "host"; `hip_stream` is a hipStream_t passed as void*, of the
 * current device; every call only enqueues work and returns; the library never allocates device memory: work space is the
 * caller's, needs no clearing, is 256-byte aligned, holds nothing from one call to the next, and must not be shared by calls
 * that may run at the same time.  Return value 0 or a negative SLIDE_E* code.  `dtype` is 0 = float32, 1 = bfloat16.
 * Strides ("ld") count elements between rows and may be larger than the row.  Unless a comment allows it, outputs must not
 * overlap inputs or each other.
 */
#ifndef SLIDE_ACT8_H_
#define SLIDE_ACT8_H_

#include "slide.h"

#ifdef __cplusplus
extern "C" {
#endif

/* A matrix in 8 bits (the struct itself: host).  codes: 16-byte aligned, ldc a multiple of 16 and >= cols; a row's bytes from
 * `cols` up to the next multiple of 16 are zero (slide_act8_pack and slide_group_norm_fwd write them so).  scales: [rows][lds],
 * lds >= ceil(cols / 128).  rows < 2^31, cols < 2^24. */
typedef struct slide_act8 {
  uint8_t* codes;  int64_t ldc;
  uint8_t* scales; int64_t lds;
  int64_t rows, cols;
} slide_act8;

/* Activation of a layer. */
#define SLIDE_ACT_NONE 0
#define SLIDE_ACT_RELU 1
#define SLIDE_ACT_SILU 2   /* u / (1 + exp(-u)) */
#define SLIDE_ACT_GELU 3   /* u / 2 (1 + erf(u / sqrt 2)) */

/* out = x in 8 bits.  transpose == 0: x is [out.rows][out.cols]; transpose != 0: x is [out.cols][out.rows] and its transpose is
 * packed (a weight matrix for the input gradient).  ldx: elements between x's rows. */
int slide_act8_pack(const void* x, int dtype, int64_t ldx, int transpose, const slide_act8* out, void* hip_stream);

/* y [a.rows][a.cols] = the values of a; one rounding (of values below 2^-133) where y is bfloat16, none else. */
int slide_act8_unpack(const slide_act8* a, void* y, int dtype, int64_t ldy, void* hip_stream);

/* Linear layer: y[m][n] = act(sum_k x8[m][k] w8[n][k] + bias[n]) + residual[m][n].
 * x: [x8.rows][x8.cols] of dtype, packed into x8 first (x8 is then the layer's checkpoint); NULL: x8 already holds its values.
 * w8: [out][in], in = x8.cols.  bias [out] float32 and residual [x8.rows][out] of dtype may be NULL.  y: [x8.rows][out] of dtype;
 * y may be the residual itself (same pointer and stride), and the residual may be x.
 * The input gradient of the layer is the same call with the output gradient for x and the packed transpose of the weights
 * for w8.  bfloat16: products and sums on the matrix cores' 8-bit instruction.  It adds eight neighbouring products (columns 8 i .. 8 i + 7)
 * with 13 bits below the largest of them and cuts off what is smaller; from there on the sums are float32.  A result is off by
 * 7 * 2^-13 of the eights' largest products at most, 2e-5 to 8e-5 of its size on activations, where its rounding costs up to 2^-9.
 * float32: products and sums as exact as float32 sums are (operands below 2^-133 are rounded to bfloat16's). */
int slide_act8_linear(const void* x, int dtype, int64_t ldx, const slide_act8* x8, const slide_act8* w8, const float* bias,
                      int act, const void* residual, int64_t ldr, void* y, int64_t ldy, void* hip_stream);

/* Weight gradient of the layer out of the checkpoint of its input: dW[n][k] = sum_m dy[m][n] x8[m][k], db[n] = sum_m dy[m][n],
 * written (accumulate == 0) or added to what is there.  dy: [x8.rows][out] of dtype; dW: float32, lddw between rows; db: [out]
 * float32 or NULL.  Sums in float32, over slabs of rows that are then added in a fixed order: the same bits on every run.  float32 gradients count
 * with all their bits, whatever their size; where a result is not finite, or past 2^80 on the way, its part is summed again, more slowly.
 * work: slide_act8_wgrad_workspace_bytes(x8.rows, out, x8.cols) bytes (0 for sizes that are refused).  SLIDE_EUNSUPPORTED for those and
 * where rows of x8's codes or scales are more than 2^24 bytes apart. */
size_t slide_act8_wgrad_workspace_bytes(int64_t rows, int64_t out, int64_t in);
int slide_act8_wgrad(const void* dy, int dtype, int64_t lddy, int64_t out, const slide_act8* x8, float* dW, int64_t lddw,
                     float* db_or_null, int accumulate, void* work, size_t work_bytes, void* hip_stream);

/* Group normalisation over n tiles (plain data, host): a tile is [hw][channels], channels last; each tile's groups of
 * channels / groups channels are normalised by themselves, so no tile depends on another. */
typedef struct slide_group_norm {
  int64_t n, hw;
  int32_t channels, groups;   /* channels % groups == 0, channels <= 65536 */
  int32_t dtype, act;
  float   eps;
  int32_t reserved;           /* must be 0 */
} slide_group_norm;

/* Bytes of work space of the two calls below (0: the shape is refused). */
size_t slide_group_norm_workspace_bytes(const slide_group_norm* s);

/* xhat = (x - mean) rstd over the hw x channels / groups values of a group, rstd = 1 / sqrt(var + eps) with the variance
 * of those values; y = act(gamma xhat + beta + residual).  x, y, residual (may be NULL): [n * hw][channels] of dtype; y may be x or
 * the residual (same pointer and stride).  gamma, beta: [channels] float32.  mean, rstd: [n][groups] float32, written.
 * x8 (may be NULL): also put x away in 8 bits, for the backward. */
int slide_group_norm_fwd(const slide_group_norm* s, const void* x, int64_t ldx, const float* gamma, const float* beta,
                         const void* residual, int64_t ldr, void* y, int64_t ldy, const slide_act8* x8, float* mean,
                         float* rstd, void* work, size_t work_bytes, void* hip_stream);

/* Gradients at dy, with mean and rstd as the forward left them: dx, dresidual (may be NULL) [n * hw][channels] of dtype;
 * dgamma, dbeta [channels] float32, written (accumulate == 0) or added to.  The input is x, or x8 where x is NULL (exactly one of
 * them): from x8 the formulas are those of the forward with the checkpoint's values in x's place, so next to zero a rectifier may let
 * another value through than the forward did.  residual as in the forward: the
 * activation's slope is taken at the same sum; which side of zero a rectifier's input is on is settled in 64 bits.
 * dx or dresidual may be dy (same pointer and stride), not both; neither may be x or the residual. */
int slide_group_norm_bwd(const slide_group_norm* s, const void* dy, int64_t lddy, const void* x, int64_t ldx,
                         const slide_act8* x8, const float* gamma, const float* beta, const void* residual, int64_t ldr,
                         const float* mean, const float* rstd, void* dx, int64_t lddx, void* dresidual, int64_t lddr,
                         float* dgamma, float* dbeta, int accumulate, void* work, size_t work_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* SLIDE_ACT8_H_ */
