/*
 * eden_mx4.h -- C ABI of 4-bit operands and their products: a linear layer's forward pass and gradients on the card's 4-bit matrix cores.
 *
 * Conventions are those of eden_layers.h: status codes, device pointers, row-major matrices with a distance between rows, streams, no allocation, no memset,
 * no synchronisation; a call may be captured in a HIP graph, and calls may run on any streams at once if their buffers do not overlap.  Any size may be 0.
 *
 * 4 bits of an r x c matrix: blocks of 32 consecutive columns of a row, the last one filled up with zeros.  A block has an exponent byte t and 32 codes of a sign and
 * three bits, 0 .. 7 for 0, 1/2, 1, 3/2, 2, 3, 4, 6 times 2^(t - 127).  2^(t - 127) is the smallest power of two, from t = 0 on, that reaches the largest |x| of the block with a
 * 6: nothing is clipped.  A block that holds an infinity or a NaN has t = 255 and stands for 32 NaN, here and in every product.
 * Rounding is to the nearest, ties to the even code; or stochastic: a value between two codes goes to the upper one (in size) if d + 1/2 < 65536 s, where s is the
 * share of the way it has gone and d 16 bits of the hash (row i, column j of what is rounded, as in eden_blocks.h, with a stream of its own): its expectation is x, to 2^-17 of a
 * step, and what is a code's value stays.
 * Layout: r rows of 128 ceil(c / 256) bytes, two codes to a byte, the even column's in the low half, zeros behind the last column; then, for each 256 columns, eight
 * exponent bytes of each row, for an even number of rows (what those of a row too many hold does not matter).  Exponents behind the last block are 0.  Buffers
 * are 16-byte aligned; r is at most 2^27, c at most 2^22.
 *
 * Products of codes are exact, sums fp32, results rounded once to nearest even.  Outputs must not overlap inputs, except that eden_mx4_linear's y and eden_mx4_input_grad's dx may be the
 * residual itself (same pointer, same distance).
 */
#ifndef EDEN_MX4_H
#define EDEN_MX4_H

#include "eden_blocks.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Bytes of the 4 bits of a rows x cols matrix; 0 if a size is out of range. */
size_t eden_mx4_bytes(uint64_t rows, uint64_t cols);

/* x (rows x cols, dtype) -> its 4 bits, or those of its transpose (cols x rows) if transpose != 0.
 *   rounding   NULL: to the nearest; else stochastic (threshold is not used)
 *   sums       NULL, or cols numbers: the sums of x's columns in fp32 (the bias gradient, where x is dy); with transpose only.  accumulate != 0: added to what they
 *              hold.  They are split over workgroups as far as the workspace reaches (16-byte aligned, NULL: not at all); the split sets the order of the additions. */
int eden_mx4_quantize(const void *x, uint64_t ldx, uint64_t rows, uint64_t cols, uint32_t dtype, int transpose, const eden_random *rounding, void *packed,
                      size_t capacity, float *sums, int accumulate, void *workspace, size_t workspace_bytes, void *stream);

/* Workspace of the sums of a rows x cols matrix. */
size_t eden_mx4_sums_bytes(uint64_t rows, uint64_t cols);

/* 4 bits -> the values they stand for, rounded to dtype. */
int eden_mx4_restore(const void *packed, uint64_t rows, uint64_t cols, uint32_t dtype, void *x, uint64_t ldx, void *stream);

/* Workspace with which the following three calls split a long sum over workgroups where the result alone would leave most of the device idle.  They work with
 * any smaller one, NULL among them, and then split less; the split sets the order of the fp32 additions.  16-byte aligned.
 *   rows x cols   size of the result;  depth   length of the sums
 * quantize != 0: eden_mx4_linear with x as a matrix, whose 4 bits come first in the workspace: that much is needed unless eden_mx4_linear says otherwise. */
size_t eden_mx4_workspace_bytes(uint64_t rows, uint64_t cols, uint64_t depth, int quantize);

/* y = act(z) + residual, z = x^ w^T + bias.
 *   x^ m x k: x_packed, or x (dtype) rounded to the nearest; the other one is NULL.  With x the workspace has to have room for eden_mx4_bytes(m, k), unless m is
 *   at most EDEN_MX4_ROWS and m k at most EDEN_MX4_VALUES (EDEN_ERR_CAPACITY)
 *   w_packed n x k, bias n or NULL, residual m x n or NULL, y m x n of dtype
 *   z_checkpoint   NULL, or a buffer of eden_checkpoint_bytes(m, n) that gets the 8-bit checkpoint of z */
#define EDEN_MX4_ROWS 16
#define EDEN_MX4_VALUES 16384
int eden_mx4_linear(const void *x, uint64_t ldx, const void *x_packed, const void *w_packed, const void *bias, const void *residual, uint64_t ldr, void *y,
                    uint64_t ldy, void *z_checkpoint, size_t z_capacity, uint64_t m, uint64_t n, uint64_t k, uint32_t dtype, uint32_t activation,
                    void *workspace, size_t workspace_bytes, void *stream);

/* dx = (dz w) * act'(z^) + residual (m x k of dtype): dz_packed m x n, wt_packed the 4 bits of w's transpose, k x n; z_checkpoint and activation as in
 * eden_linear_input_grad. */
int eden_mx4_input_grad(const void *dz_packed, const void *wt_packed, const void *z_checkpoint, uint32_t activation, const void *residual, uint64_t ldr,
                        void *dx, uint64_t ldx, uint64_t m, uint64_t n, uint64_t k, uint32_t dtype, void *workspace, size_t workspace_bytes, void *stream);

/* dw = dy^T x (n x k, fp32): the 4 bits of both transposes, dyt_packed n x m and xt_packed k x m; accumulate != 0: added to what dw holds. */
int eden_mx4_weight_grad(const void *dyt_packed, const void *xt_packed, float *dw, uint64_t ldw, uint64_t m, uint64_t n, uint64_t k, int accumulate,
                         void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* EDEN_MX4_H */
