/*
 * vms_ops: the operators of a training block beside the allocators, as kernels for
 * one AMD MI355X (gfx950): dropout whose mask is never stored, layer norm with the
 * residual sum on the way in, and low-rank adapters of many requests beside a shared
 * projection, each with its backward pass.  None of them keeps a mask or any other
 * tensor of its own between forward and backward but what the header names, so that a
 * recomputed forward pass makes the same numbers again and the allocation stream of a
 * training loop holds nothing but the program's tensors.
 *
 * Matrices are row-major with a row stride in elements (ld*); the columns of a row are
 * consecutive, rows and pointers need no more than the alignment of their type.  A row
 * stride of an input may be 0 (the same row for all), that of an output is at least the
 * number of columns.  Element types are VMS_F32, VMS_F16 and VMS_BF16, the same for all
 * tensors of a call; every sum is kept in 32 bits.  rows = 0 is allowed and does nothing
 * but clear the gradients of weights.
 *
 * Outputs overlap neither each other nor an input, but where an entry point says so.
 *
 * Pointers named d_* are DEVICE pointers owned by the caller, on the current HIP device.
 * Calls are asynchronous on `stream` (a hipStream_t of that device), allocate nothing,
 * keep nothing and can be captured into a graph.  They return VMS_OK or a negative VMS_E*
 * code of vms_replay.h and never throw; nothing is launched when the arguments are wrong.
 * Workspaces are 16-byte aligned, need not be cleared and are free again when the call's
 * kernels are done: two calls that may run at the same time need two.
 */
#ifndef VMS_OPS_H
#define VMS_OPS_H

#include <stddef.h>
#include <stdint.h>

#include "vms_replay.h"

#ifdef __cplusplus
extern "C" {
#endif

#define VMS_F32  0
#define VMS_F16  1
#define VMS_BF16 2

/* Which elements a dropout drops.  Philox-4x32 with ten rounds (Salmon, Moraes, Dror and Shaw,
 * 2011) turns the counter (column / 8, row, call low word, call high word) under the key `seed`
 * into eight 16-bit numbers, the low half of each word first; number (column mod 8) is the
 * element's.  An element is dropped where its number is below p * 65536, rounded to a whole number
 * T, and multiplied by 65536 / (65536 - T) where it is kept: p is taken in steps of 2^-16, and the
 * expected value is that of the input for the p that was taken.  The mask depends on nothing else:
 * neither on strides nor on the type.                                                             */
typedef struct vms_dropout_mask {
    double   p;                  /* 0 <= p <= 1                                                     */
    uint64_t seed;               /* used if d_seed is NULL                                          */
    const uint64_t *d_seed;      /* nullable: the seed in device memory, read when the kernel runs  */
    uint64_t call;               /* number of the call: one for each dropout under a seed           */
} vms_dropout_mask;

/* y = residual + dropout(x); residual may be NULL.  The backward pass is the same call with the
 * gradient for x and no residual.  y may be x or residual themselves (same stride), but not
 * overlap them otherwise.                                                                         */
typedef struct vms_dropout_args {
    uint32_t struct_size;        /* sizeof(vms_dropout_args)                                        */
    uint32_t dtype;
    uint64_t rows, cols;         /* each below 2^31                                                 */
    const void *d_x;
    const void *d_residual;
    void *d_y;
    uint64_t ldx, ldr, ldy;
    vms_dropout_mask mask;
} vms_dropout_args;
int vms_dropout(const vms_dropout_args *a, void *stream);

/* s = residual + dropout(x), or x without a residual (then p must be 0 and d_s NULL);
 * y = (s - mean) * rstd * weight + bias over each row, rstd = 1 / sqrt(variance + eps).
 * y goes by s before it is rounded to the type.  d_weight and d_bias may each be NULL, and d_s where no
 * backward pass follows.  d_stats (nullable) receives two floats for each row, for the backward pass:
 * mean and rstd of s as it is stored.                                                             */
typedef struct vms_layernorm_args {
    uint32_t struct_size;        /* sizeof(vms_layernorm_args)                                      */
    uint32_t dtype;
    uint64_t rows, cols;         /* rows below 2^31, cols from 1 to 2^26 - 1                        */
    const void *d_x, *d_residual, *d_weight, *d_bias;
    void *d_y, *d_s;
    float *d_stats;
    uint64_t ldx, ldr, ldy, lds;
    double eps;                  /* >= 0                                                            */
    vms_dropout_mask mask;
} vms_layernorm_args;
int vms_layernorm(const vms_layernorm_args *a, void *stream);

/* The backward pass, from dy (gradient of y) and ds (gradient that arrives at s elsewhere; NULL: none),
 * the s of the forward pass (x where there was no residual) and its statistics:
 *   d_dres  gradient of s, which is that of the residual;
 *   d_dx    gradient of x behind the dropout; NULL where p is 0 (it is d_dres then);
 *   d_dweight, d_dbias: gradients of the weights, each nullable.
 * The sums over the rows are joined in a fixed order: the same call gives the same bits.           */
typedef struct vms_layernorm_backward_args {
    uint32_t struct_size;        /* sizeof(vms_layernorm_backward_args)                             */
    uint32_t dtype;
    uint64_t rows, cols;
    const void *d_dy, *d_ds, *d_s, *d_weight;
    const float *d_stats;
    void *d_dres, *d_dx, *d_dweight, *d_dbias;
    uint64_t lddy, ldds, lds, lddres, lddx;
    vms_dropout_mask mask;
    void *d_workspace;           /* vms_layernorm_backward_workspace_bytes; NULL if that is 0       */
    uint64_t workspace_bytes;
} vms_layernorm_backward_args;
size_t vms_layernorm_backward_workspace_bytes(const vms_layernorm_backward_args *a);   /* reads sizes and which gradients are asked for */
int vms_layernorm_backward(const vms_layernorm_backward_args *a, void *stream);

/* Low-rank adapters beside a shared projection.  out = y + scale * (x a^T) b^T for the rows of every
 * request, with the a [rank, in] and b [out, rank] of the request's adapter; out = y elsewhere.
 *
 * Requests are packed one behind the other: request i has rows d_starts[i] .. d_starts[i + 1] - 1 of
 * adapter d_which[i] (outside 0 .. n_adapters - 1: none).  d_starts has n_requests + 1 numbers that do not
 * decrease, from 0 .. rows; rows before the first and behind the last belong to no request.  Numbers
 * that break this are never followed out of the tensors, but the values of `out` are then undefined.
 * d_starts = NULL: all rows are one request of adapter 0.
 * d_y = d_out (same stride): the sum is made in place, and rows of no request are not touched.
 *
 * d_hidden (vms_lowrank_hidden_bytes, 16-byte aligned) receives scale * x a^T: workspace of the forward
 * pass, and what the backward pass reads, in a layout of the library's own.  In 16 bits a value is kept as
 * two numbers of the type (what the first leaves in the second): to 2^-16 of it in bfloat16, to 2^-22 or
 * 2^-25 in float16, where one beyond 65504 is an infinity, as in a program that stores it.             */
#define VMS_LOWRANK_MAX_RANK 128
typedef struct vms_lowrank_args {
    uint32_t struct_size;        /* sizeof(vms_lowrank_args)                                        */
    uint32_t dtype;
    uint64_t rows, in, out;      /* rows < 2^28 (2^27 with ranks above 64), in and out in 1 .. 2^22 - 1;
                                    refused where a launch cannot have as many workgroups           */
    uint32_t rank;               /* 1 .. VMS_LOWRANK_MAX_RANK                                       */
    uint32_t n_adapters;         /* 1 .. 65535                                                      */
    uint32_t n_requests;         /* < 2^16; ignored if d_starts is NULL                             */
    float scale;                 /* used if d_scales is NULL                                        */
    const float *d_scales;       /* nullable: one for each adapter                                  */
    const void *d_x, *d_y, *d_a, *d_b;      /* a and b without gaps                                 */
    const int32_t *d_starts, *d_which;
    void *d_out;
    uint64_t ldx, ldy, ldo;      /* each below 2^23, here and in the backward pass                  */
    void *d_hidden;
    uint64_t hidden_bytes;
} vms_lowrank_args;
size_t vms_lowrank_hidden_bytes(const vms_lowrank_args *a);             /* reads the sizes only; 0 if they are wrong */
int vms_lowrank(const vms_lowrank_args *a, void *stream);

/* The backward pass: from `dout` the gradients d_dx (0 in rows of no request), d_da and d_db, each
 * nullable; the gradient of y is dout itself.  An adapter's gradients sum over all its requests, in a
 * fixed order; those of an adapter without rows are 0.  f.d_hidden is the forward pass's, f.d_y, f.d_out and
 * their strides are not used.                                                                     */
typedef struct vms_lowrank_backward_args {
    uint32_t struct_size;        /* sizeof(vms_lowrank_backward_args)                               */
    uint32_t reserved0;
    vms_lowrank_args f;          /* the forward pass                                                */
    const void *d_dout;
    void *d_dx, *d_da, *d_db;
    uint64_t lddout, lddx;
    void *d_workspace;           /* vms_lowrank_backward_workspace_bytes                            */
    uint64_t workspace_bytes;
} vms_lowrank_backward_args;
size_t vms_lowrank_backward_workspace_bytes(const vms_lowrank_backward_args *a);       /* reads sizes and which gradients are asked for */
int vms_lowrank_backward(const vms_lowrank_backward_args *a, void *stream);

#ifdef __cplusplus
}
#endif
#endif
