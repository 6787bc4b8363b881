/*
 * eden_blocks.h -- C ABI of the operators around a residual block: dropout, norms, and the join of a block's two branches with the norm of the next.
 *
 * A trained block is r = x + f(norm(x)).  These calls do what stands around its layers (eden_layers.h, eden_mx4.h), forward and
 * backward: the norm in front of it, a norm behind its branch, dropout, the gate, both scales and the sum, in one pass over the rows.
 *
 * Conventions are those of eden_layers.h: status codes, device pointers, row-major matrices with a distance between rows, streams,
 * no allocation, no memset, no synchronisation; a call may be captured in a HIP graph, and calls may run on any streams at once if their buffers
 * do not overlap.  Rows have up to EDEN_MOST_COLUMNS columns, there are up to 2^30 of them; either may be 0.
 * Values, statistics and sums are fp32; a row's mean square has to be in its range, the sum of its squares need not.  Every result is rounded once, to nearest even.
 *
 * Random numbers: the words of the hash of eden.h.  Row i, column j of a matrix of c columns has bits 16 (j mod 4) .. + 15 of word
 * i ceil(c / 4) + floor(j / 4) of the stream's key for (seed, id).  Nothing is stored: the backward pass names the same seed and id.
 */
#ifndef EDEN_BLOCKS_H
#define EDEN_BLOCKS_H

#include "eden_layers.h"

#ifdef __cplusplus
extern "C" {
#endif

#define EDEN_MOST_COLUMNS 16384

/* Where random numbers come from.  seed_at: NULL, or a device pointer (8-byte aligned) to a number that the kernels add to seed when they run, so that
 * a captured call draws new ones in every replay. */
typedef struct eden_random {
    uint64_t seed;
    const uint64_t *seed_at;
    uint32_t id;
    uint32_t threshold;            /* dropout: a value is dropped if its 16 bits are below; 65536 p, at most 65535; 0: none */
} eden_random;

/* rms: v / sqrt(mean(v^2) + eps) * weight;  layer: (v - mean(v)) / sqrt(mean((v - mean(v))^2) + eps) * weight + bias */
typedef enum eden_norm_kind { EDEN_NORM_NONE = 0, EDEN_NORM_RMS = 1, EDEN_NORM_LAYER = 2 } eden_norm_kind;
typedef struct eden_norm {
    uint32_t kind;
    float eps;                     /* finite, not negative */
    const void *weight, *bias;     /* cols each, dtype; NULL: ones, zeros; an rms norm has no bias */
} eden_norm;

/* y = x 65536 / (65536 - threshold) where kept, 0 elsewhere, whatever x is there.  Its gradient is the same call on that of y.  y may be x (same pointer, same distance). */
int eden_dropout(const void *x, uint64_t ldx, void *y, uint64_t ldy, uint64_t rows, uint64_t cols, uint32_t dtype, const eden_random *random,
                 void *stream);

/*   r = x_scale x + scale gate * dropout(post(f))         h = pre(r)
 * Without f: h = pre(x), and there is neither gate nor post nor dropout nor r.
 *   gate: gates x cols; row i of x has gate i / (rows / gates), gates divides rows; NULL: ones
 *   r: may be NULL if only h is wanted; h: NULL iff pre.kind is EDEN_NORM_NONE.  pre takes r as it is before it is rounded.
 * r may be x or f, h may be x or f (same pointer, same distance); they must not overlap anything else. */
typedef struct eden_join_args {
    uint64_t rows, cols;
    const void *x, *f, *gate;
    void *r, *h;
    uint64_t ldx, ldf, ld_gate, ldr, ldh;
    uint64_t gates;
    eden_norm post, pre;
    eden_random random;
    float x_scale, scale;          /* finite, scale 65536 / (65536 - threshold) too */
    uint32_t dtype;
} eden_join_args;
int eden_join(const eden_join_args *args, void *stream);

/* The gradients of the join from those of r (dr) and h (dh); either may be NULL for zeros, dh is if pre.kind is EDEN_NORM_NONE:
 *   d = dr + (gradient of pre at r);  dx = x_scale d;  df, gate_grad, and those of the norms' weights and biases: behind d.
 * r: the sum as eden_join wrote it (without a branch x), read if dh is there.  f: read if post is there or gate_grad is wanted; `branch` says whether the join had one:
 * without it there are no gate, post, dropout and df, and dh has to be there.
 * dx, df and every sum may be NULL.  Sums are fp32: gate_grad gates x cols at distance ld_gate_grad, the others cols; accumulate != 0: added
 * to what they hold.  dx may be dr, dh or r, df may be f (same pointer, same distance); outputs must not overlap anything else.
 * Sums over rows are split over workgroups as far as the workspace reaches (NULL: not at all, which is slow); the split sets the order of the
 * fp32 additions.  16-byte aligned. */
typedef struct eden_join_grad_args {
    uint64_t rows, cols;
    const void *dr, *dh, *r, *f, *gate;
    void *dx, *df;
    uint64_t lddr, lddh, ldr, ldf, ld_gate, lddx, lddf;
    uint64_t gates;
    float *gate_grad, *post_weight_grad, *post_bias_grad, *pre_weight_grad, *pre_bias_grad;
    uint64_t ld_gate_grad;
    eden_norm post, pre;
    eden_random random;
    float x_scale, scale;
    uint32_t dtype, branch, accumulate;
    void *workspace;
    size_t workspace_bytes;
} eden_join_grad_args;
int eden_join_grad(const eden_join_grad_args *args, void *stream);

/* Workspace with which eden_join_grad splits its sums over as many workgroups as fill the device; 0 where there is nothing to split or a size is out of range. */
size_t eden_join_workspace_bytes(uint64_t rows, uint64_t cols, uint64_t gates, uint32_t dtype);

#ifdef __cplusplus
}
#endif
#endif /* EDEN_BLOCKS_H */
