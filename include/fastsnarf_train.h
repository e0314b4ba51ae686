/*
 * fastsnarf_train.h -- what a training step does with gradients: their global norm, clipping, and the AdamW update.
 *
 * fs_grad (fastsnarf.h) leaves dL/dW and dL/dB; a program that learns a skinning field adds the gradients of the networks
 * around it.  The calls below work on the whole list of tensors at once, whatever their number, sizes and types:
 *
 *   norm    s sqrt(sum_i sum_j g_ij^2), or s max |g_ij|, s = grad_scale (the inverse of a loss scale, usually 1)
 *   coef    s min(1, max_norm / (norm + 1e-6)); a norm that is NaN gives NaN.  max_norm = INFINITY: s
 *   clip    out_ij = g_ij coef
 *   AdamW   t = steps done + 1, g' = g coef, l = lr lr_scale_i:
 *             m = beta1 m + (1 - beta1) g',  v = beta2 v + (1 - beta2) g'^2
 *             p = p (1 - l weight_decay decay_scale_i) - l / (1 - beta1^t) m / (sqrt(v / (1 - beta2^t)) + eps)
 *
 * Magnitudes are squared and added in 64 bits, and the norm stays in 64 bits until it is written: for the coefficient, and for whether it is
 * finite.  The norm of any finite fp32 gradients is, also where the fp32 that is written is infinity.  A norm that is given has 32 bits.  The
 * coefficient and the bias corrections are computed in 64 bits, the update in fp32 (an eps that fp32 rounds to 0 is its smallest number).  16-bit
 * results are rounded once, to nearest even.  Sums run in an order that depends on the list (with its addresses) and on the device only: results
 * are the same from call to call.  NaN and infinities go through as the formulas say.
 *
 * Conventions of fastsnarf.h hold (device pointers, nothing synchronises, status codes, no exceptions or aborts), with one
 * difference: the pointers of a list are aligned to their own element type, no more, so tensors may be views into a packed buffer.
 */
#ifndef FASTSNARF_TRAIN_H
#define FASTSNARF_TRAIN_H

#include "fastsnarf.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct fs_tensors fs_tensors; /* opaque: a list of tensors, its copy on the device and the scratch of its sums */

enum { FS_FLOAT_FULL = 0, FS_FLOAT_BRAIN = 1, FS_FLOAT_HALF = 2 }; /* fp32, bf16, fp16 */
enum { FS_NORM_TWO = 0, FS_NORM_MAX = 1 };
enum { FS_MAX_TENSORS = 1 << 20 };

/* One tensor: n elements in memory one after another, in the same order in every array.  A call checks that the arrays it
 * needs are there; the others may be NULL.  n == 0: the tensor takes part in nothing and its pointers are not looked at. */
typedef struct {
    void *grad;           /* dL/dp; written only by an fs_grad_clip in place                                     */
    void *out;            /* of fs_grad_clip, grad's type; NULL: in place.  Either grad itself or apart from it  */
    void *param;          /* p; where there is a master, it is only written                                      */
    float *master;        /* p in fp32, or NULL: p itself is read, updated in fp32 and rounded to its type      */
    float *exp_avg;       /* m                                                                                   */
    float *exp_avg_sq;    /* v                                                                                   */
    int64_t n;            /* 0 .. 2^40                                                                           */
    int32_t grad_type;    /* FS_FLOAT_*                                                                          */
    int32_t param_type;   /* FS_FLOAT_*                                                                          */
    float lr_scale;       /* factors of this tensor on lr and weight_decay (0 for biases, say); finite           */
    float decay_scale;
} fs_tensor;

typedef struct {
    double lr;            /* finite                                                                              */
    double beta1, beta2;  /* 0 <= beta < 1                                                                       */
    double eps;           /* >= 0                                                                                */
    double weight_decay;  /* finite                                                                              */
    double max_norm;      /* >= 0, INFINITY: no clipping                                                         */
    double grad_scale;    /* > 0, finite                                                                         */
    int32_t norm_given;   /* 0: d_norm is computed (2-norm) and written.  1: it is read (a norm over several GPUs, say)  */
    int32_t skip_nonfinite; /* 1: where the norm is NaN or infinite (in 64 bits) nothing is written but the norm: no update, no step */
    const float *d_lr;    /* a word on the device that is read in place of lr (a schedule under graph capture), or NULL */
} fs_adamw;

/* Make a list of `count` tensors (0 .. FS_MAX_TENSORS) on the current device.  `list` is host memory and is not kept; the
 * tensors' memory stays the caller's and has to stay where it is while calls on the list are made.  Tensors that a call writes must
 * not overlap one another or what it reads otherwise.  Allocates 84 bytes per tensor and 25 KiB.  On failure *out is NULL. */
fs_status fs_tensors_create(const fs_tensor *list, int32_t count, void *hip_stream, fs_tensors **out);

/* The same in memory of the caller's, for callers that cannot allocate (graph capture): fs_tensors_bytes(count) bytes (0 for a count out of range) of the current
 * device, aligned to 256.  The memory stays the caller's, and has to be there until the calls on the list are done, those of graphs that are replayed included.
 * On a stream that records a graph, the list is brought to the device whenever the graph runs. */
int64_t fs_tensors_bytes(int32_t count);
fs_status fs_tensors_create_noalloc(const fs_tensor *list, int32_t count, void *hip_stream, void *workspace, int64_t bytes, fs_tensors **out);

/* Free what the list owns.  Where it owns memory of the device, its stream is synchronised first; where that memory cannot be freed (as
 * while a graph is captured), the list stays, and the call can be made again.  NULL is allowed. */
fs_status fs_tensors_destroy(fs_tensors *t);

/* Other addresses, sizes or types for the same number of tensors, for the calls after this one (a program whose gradients move from
 * step to step).  A list that is refused changes nothing; after FS_E_DEVICE, calls return FS_E_STATE until another update has succeeded.
 * A stream that records a graph records the update: it is for the calls behind it in the same graph, and any other call returns FS_E_STATE until
 * another update has succeeded where that call is made.  A graph's calls read the list as it is on the device when they are replayed: a list that
 * a graph uses is neither updated outside of it nor destroyed while the graph is. */
fs_status fs_tensors_update(fs_tensors *t, const fs_tensor *list, int32_t count);

/* FS_OK if a call on the list would find it on the device now, FS_E_STATE if another update is needed before. */
fs_status fs_tensors_ready(fs_tensors *t);

/* The stream of the calls after this one.  The list's scratch is shared by all its calls, fs_grad_norm's included: the caller orders this stream behind the
 * one before.  A graph that may be replayed beside other calls needs a list of its own. */
fs_status fs_tensors_set_stream(fs_tensors *t, void *hip_stream);

/* d_norm [1] = norm of all gradients (kind: FS_NORM_TWO or FS_NORM_MAX); of an empty list 0. */
fs_status fs_grad_norm(fs_tensors *t, int32_t kind, double grad_scale, float *d_norm);

/* Scaled gradients into the tensors' `out`, or in place, where a coefficient of 1 leaves the memory untouched.
 * norm_given = 0: d_norm [1] is computed as by fs_grad_norm; 1: it is read (kind is then not looked at). */
fs_status fs_grad_clip(fs_tensors *t, int32_t kind, double max_norm, double grad_scale, int32_t norm_given, float *d_norm);

/* One AdamW step.  d_step [1]: steps done before, one more after (8-byte aligned).  d_norm [1] may be NULL if max_norm is INFINITY and
 * skip_nonfinite 0: then no norm is computed. */
fs_status fs_adamw_step(fs_tensors *t, const fs_adamw *how, int64_t *d_step, float *d_norm);

/* Message for the last non-OK status returned on this list ("" if none). */
const char *fs_tensors_error(const fs_tensors *t);

#ifdef __cplusplus
}
#endif
#endif /* FASTSNARF_TRAIN_H */
