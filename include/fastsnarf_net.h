/*
 * fastsnarf_net.h -- the layers of the networks on either side of the search: the skinning network, whose values on the grid's nodes give
 * W (fastsnarf.h), and the occupancy network, evaluated at the roots.
 *
 * X [rows, inputs], weight [outputs, inputs], bias [outputs]; residual, Y, Z and their gradients [rows, outputs]:
 *
 *   Z = X weight^T + bias
 *   Y = residual + drop(act(Z))
 *   act:  z,  max(z, 0),  z Phi(z),  z / (1 + e^-z),  ln(1 + e^(beta z)) / beta       (Phi: the normal distribution's)
 *   drop: element e = row * columns + column is kept and multiplied by 1 / (1 - p) where word e mod 4 of Philox4x32-10 with counter
 *         (e div 4, offset) and key `seed`, both of 64 bits with the low word first, is at least round(p 2^32); otherwise it is 0,
 *         whatever it was
 *
 * and backward, from G = dL/dY (dL/dresidual is G itself):
 *
 *   dZ = drop(G act'(Z)),  dbias = sum of dZ over the rows,  dX = dZ weight,  dweight = dZ^T X
 *
 * No mask is stored: the backward pass makes it anew.  Philox4x32-10: Salmon et al., "Parallel random numbers: as easy as 1, 2, 3" (2011).
 *
 * Arithmetic: sums in fp32, dbias over the rows in 64 bits (columns may cancel); results rounded once, to nearest even.
 *  - Where the type has 16 bits, dZ is rounded to it for the products that read it (not for dbias, which is summed before that).  Where that would not average
 *    out, dZ goes in as two parts of 16 bits: in products of at most 4096 results or from at most 4096 values of dZ, and in layers of at most 128 inputs, 128
 *    outputs and 131072 values of dZ.  fp16's range does not matter for it: dZ is scaled by a power of two on the way, and its rounding steps are at most 2^-38
 *    of the largest finite |G| / (1 - p).
 *  - Z is kept for the backward pass in the bias's type, or in fp32 by FS_Z_FULL: an fp32 bias gets a gradient that is good to fp32.  fp16 keeps finite Z
 *    within +-65504 and positive Z positive, which changes no slope but that of softplus with beta below 2^-11 (take FS_Z_FULL for that).
 *  - fp32 operands of the products go in as three bf16 parts each (24 bits together), of whose nine products the six largest are added: what is left out is
 *    below 2^-23 of |x w|, as fp32 rounds a product to 2^-24.  Operands below 2^-102 lose digits (the parts are normal numbers no more).
 *  - Results are the same from call to call on a device: no atomics.
 *  - NaN and infinities go through as the formulas say.  Blocks of fp32 results among which there are any are made twice: up to some ten times as long, where all are.
 *
 * Conventions of fastsnarf.h hold (device pointers, nothing synchronises, status codes, no exceptions or aborts), with these differences:
 *  - No context: the calls keep nothing.  They run on the current device and on the stream that is given, in memory that is given.  Calls that may
 *    overlap in time need workspaces of their own; any number of threads may call.
 *  - Pointers are aligned to their own element type, the workspace to 256 bytes.  A row's elements lie one after another; rows are `ld` elements
 *    apart: at least the row's length in what is written, 0 or more in what is read.
 *  - What a call writes overlaps neither what it reads nor what else it writes, with one exception: Y may be the residual (or X, in fs_dropout)
 *    itself, with the same ld.
 *  - The calls can be captured into graphs.  A graph's calls keep the addresses, also those of the workspace.
 */
#ifndef FASTSNARF_NET_H
#define FASTSNARF_NET_H

#include "fastsnarf_train.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { FS_ACT_NONE = 0, FS_ACT_RELU = 1, FS_ACT_GELU = 2, FS_ACT_SILU = 3, FS_ACT_SOFTPLUS = 4, FS_Z_FULL = 256 };

typedef struct {
    double p;               /* 0 .. 1: the chance of being dropped; 0: nothing is, and the rest is not looked at */
    uint64_t seed, offset;  /* where d_seed is NULL */
    const int64_t *d_seed;  /* two words on the device, seed and offset, read in their place when the call runs (8-byte aligned), or NULL */
} fs_drop;

typedef struct {
    int64_t rows;           /* 0 .. 5 10^8 */
    int64_t inputs;         /* 0 .. 2^24 */
    int64_t outputs;        /* 0 .. 2^24 */
    int32_t type;           /* FS_FLOAT_*: X, weight, residual, Y, and their gradients */
    int32_t bias_type;      /* that type or FS_FLOAT_FULL: bias, dbias and Z */
    int32_t act;            /* FS_ACT_*; + FS_Z_FULL: Z is fp32 whatever the bias is */
    float beta;             /* of softplus: > 0, finite */
    fs_drop drop;
} fs_linear;

/* A product of 2^23 tiles of its result or more (of 128 by 128; 64 by 64 where there are few, or either side is at most 64) is refused: FS_E_SHAPE. */

/* Bytes of workspace that fs_linear_forward (backward = 0) or fs_linear_backward (1) needs on the current device; -1 if `layer` is refused.
 * Depends on the layer alone, not on seeds or addresses. */
int64_t fs_linear_bytes(const fs_linear *layer, int32_t backward);

/* d_y, and d_z for the backward pass (or NULL).  d_bias and d_r may be NULL.  d_work: fs_linear_bytes() bytes (NULL if 0). */
fs_status fs_linear_forward(const fs_linear *layer, const void *d_x, int64_t ldx, const void *d_w, int64_t ldw, const void *d_bias,
                            const void *d_r, int64_t ldr, void *d_y, int64_t ldy, void *d_z, int64_t ldz,
                            void *d_work, int64_t work_bytes, void *hip_stream);

/* Any of d_dx, d_dw, d_dbias may be NULL: it is not computed.  d_z as fs_linear_forward wrote it (not looked at, and may be NULL, where act is
 * FS_ACT_NONE); d_w may be NULL where d_dx is, d_x where d_dw is. */
fs_status fs_linear_backward(const fs_linear *layer, const void *d_g, int64_t ldg, const void *d_x, int64_t ldx, const void *d_w, int64_t ldw,
                             const void *d_z, int64_t ldz, void *d_dx, int64_t lddx, void *d_dw, int64_t lddw, void *d_dbias,
                             void *d_work, int64_t work_bytes, void *hip_stream);

/* Y = residual + drop(X), [rows, columns] of FS_FLOAT_* `type`, up to 2^40 elements (d_r may be NULL); the backward pass is drop(G), the same call. */
fs_status fs_dropout(int32_t type, int64_t rows, int64_t columns, const fs_drop *drop, const void *d_x, int64_t ldx, const void *d_r, int64_t ldr,
                     void *d_y, int64_t ldy, void *hip_stream);

/* Message for the last non-OK status that a call of this header returned to this thread ("" if none). */
const char *fs_net_error(void);

#ifdef __cplusplus
}
#endif
#endif /* FASTSNARF_NET_H */
