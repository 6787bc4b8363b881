/*
 * eden_layers.h -- C ABI of the layer operators: a linear layer that is trained from 8-bit activation checkpoints.
 *
 * A sender's vector is usually a gradient.  These calls compute one on the same device: the forward pass of a linear layer with
 * its bias, activation and residual, the activations it keeps for the backward pass in 8 bits, and the backward pass that reads
 * them.  Weight and bias gradients are fp32 and may be written straight into (a part of) the vector that eden_encode takes.
 *
 * Conventions are those of eden.h: 0 or a negative eden_status is returned, nothing throws or aborts; pointers are HIP device
 * pointers on the current device; the caller owns every buffer and the library keeps no pointer after the call; a call only
 * launches kernels on `stream` (no allocation, no memset, no host synchronisation), so it may be captured in a HIP graph.
 * Nothing is kept from one call to the next: calls may run on any streams at once if their buffers do not overlap.
 *
 * Matrices are row-major with unit distance between the columns; ld* is the distance between rows in elements, at least the
 * number of columns (any value if there is at most one row).  Pointers are aligned to their element type; rows that start at
 * multiples of 16 bytes are read fastest.  Every size may be 0 (nothing is written where there is no output; a sum over nothing is 0), and
 * is at most 2^30; a product's result has less than 2^24 tiles of 128 x 128, and rows (cols / 2048 + 1) of an element-wise call
 * is below 2^31 (beyond any device's memory, and refused).  Outputs must not overlap inputs, except that eden_linear's y and eden_linear_input_grad's dx may be the
 * residual itself and eden_activation_grad's dz may be dy itself (same pointer, same distance).
 *
 * Sums are held in fp32 and results rounded once, to nearest even.  The products of fp16 and bf16 operands are exact.  fp32
 * operands are taken as three bf16 terms (exact down to 2^-133); in eden_linear and eden_linear_input_grad, where both operands are fp32,
 * the smallest products of terms are left out, less than 2^-22 of the whole product and of either sign, and an infinity among
 * the operands gives NaN in the results it reaches.  (A call with at most 16 rows in eden_linear multiplies in fp32 and has no such exception.)
 *
 * Checkpoint of an m x c matrix: blocks of 32 consecutive columns of a row, the last one filled up with zeros.  A block has an
 * exponent byte t and 32 codes q of -127 .. 127, which stand for q 2^(t - 127).  t = max(1, e - 6), e = exponent field of the fp32
 * number max |x|; q = x 2^(127 - t) rounded to the nearest even whole number and clipped.  A block that holds an infinity or a NaN has
 * t = 255 and stands for 32 NaN.  q 2^(t - 127) has seven significant bits and is exact in bf16: the backward pass multiplies the values themselves.
 * Layout: m rows of 32 ceil(c/32) signed bytes, then m rows of ceil(c/32) exponent bytes.  Buffers are 16-byte aligned.
 */
#ifndef EDEN_LAYERS_H
#define EDEN_LAYERS_H

#include "eden.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum eden_dtype { EDEN_F32 = 0, EDEN_F16 = 1, EDEN_BF16 = 2 } eden_dtype;

/* relu: max(z, 0), slope 0 at 0; gelu: z Phi(z); gelu_tanh: z (1 + tanh(sqrt(2/pi) (z + 0.044715 z^3))) / 2; silu: z / (1 + exp(-z)) */
typedef enum eden_activation { EDEN_ACT_NONE = 0, EDEN_ACT_RELU = 1, EDEN_ACT_GELU = 2, EDEN_ACT_GELU_TANH = 3, EDEN_ACT_SILU = 4 } eden_activation;

/* Bytes of the checkpoint of a rows x cols matrix; 0 if a size is above 2^30. */
size_t eden_checkpoint_bytes(uint64_t rows, uint64_t cols);

/* x (rows x cols, dtype) -> checkpoint. */
int eden_checkpoint_save(const void *x, uint64_t ldx, uint64_t rows, uint64_t cols, uint32_t dtype, void *checkpoint,
                         size_t capacity, void *stream);

/* checkpoint -> the values it stands for, rounded to dtype. */
int eden_checkpoint_restore(const void *checkpoint, uint64_t rows, uint64_t cols, uint32_t dtype, void *x, uint64_t ldx, void *stream);

/* Workspace with which the following three calls split a long sum over workgroups where the result alone would leave most of the
 * device idle.  They work with any smaller one, NULL among them, and then split less; the split sets the order of the
 * fp32 additions, so results may differ in their last bits from those with another workspace size.  16-byte aligned; what it
 * holds before or after a call does not matter.
 *   rows x cols   size of the result;  depth   length of the sums
 * (eden_linear: m, n, k;  eden_linear_weight_grad: n, k, m;  eden_linear_input_grad: m, k, n).
 * eden_linear of up to 4 rows, in fp32 up to 16, uses none. */
size_t eden_layers_workspace_bytes(uint64_t rows, uint64_t cols, uint64_t depth, uint32_t dtype);

/* The same and, for large products, room for copies of both operands: a call whose operands' rows do not all start at multiples of
 * 16 bytes and hold whole 16-byte pieces then copies those that do not before it multiplies, which is faster.  Equal to eden_layers_workspace_bytes
 * where that is not worth it; no use where all rows are so. */
size_t eden_layers_copying_bytes(uint64_t rows, uint64_t cols, uint64_t depth, uint32_t dtype);

/* y = act(z) + residual, z = x w^T + bias.
 *   x m x k, w n x k, bias n or NULL, residual m x n or NULL, y m x n, all of dtype
 *   z_checkpoint   NULL, or a buffer of eden_checkpoint_bytes(m, n) that gets the checkpoint of z (taken from the fp32 z) */
int eden_linear(const void *x, uint64_t ldx, const void *w, uint64_t ldw, const void *bias, const void *residual, uint64_t ldr,
                void *y, uint64_t ldy, void *z_checkpoint, size_t z_capacity, uint64_t m, uint64_t n, uint64_t k, uint32_t dtype,
                uint32_t activation, void *workspace, size_t workspace_bytes, void *stream);

/* dw = dy^T x^ (n x k, fp32), x^ the values of x's checkpoint; bias_grad (n, fp32, or NULL) = sum of dy over its rows.
 *   dy m x n of dtype; x_checkpoint of an m x k matrix; accumulate != 0: added to what dw and bias_grad hold */
int eden_linear_weight_grad(const void *dy, uint64_t ldy, const void *x_checkpoint, float *dw, uint64_t ldw, float *bias_grad,
                            uint64_t m, uint64_t n, uint64_t k, uint32_t dtype, int accumulate, void *workspace,
                            size_t workspace_bytes, void *stream);

/* dx = (dz w) * act'(z^) + residual (m x k), z^ the values of z_checkpoint (of an m x k matrix: the input of the activation in
 * front of this layer).
 *   dz m x n, w n x k, residual m x k or NULL, dx m x k, all of dtype; z_checkpoint is NULL iff activation is EDEN_ACT_NONE */
int eden_linear_input_grad(const void *dz, uint64_t ldz, const void *w, uint64_t ldw, const void *z_checkpoint, uint32_t activation,
                           const void *residual, uint64_t ldr, void *dx, uint64_t ldx, uint64_t m, uint64_t n, uint64_t k,
                           uint32_t dtype, void *workspace, size_t workspace_bytes, void *stream);

/* dz = dy * act'(z^), z^ the values of z_checkpoint; all rows x cols. */
int eden_activation_grad(const void *dy, uint64_t ldy, const void *z_checkpoint, uint32_t activation, void *dz, uint64_t ldz,
                         uint64_t rows, uint64_t cols, uint32_t dtype, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* EDEN_LAYERS_H */
