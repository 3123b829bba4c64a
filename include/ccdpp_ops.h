/*
 * ccdpp_ops.h -- operators of the CCD++ library on DEVICE memory (MI355X, gfx950).
 *
 * ccdpp.h learns factors W (users) and H (items) from squared error.  The calls
 * here train and judge such factors, or any rows against any table, as a choice
 * among all items: the softmax cross entropy of rows x_t over a whole table
 * e_v with its gradients, without holding the t x v logits (a training pass
 * over many columns keeps up to 1 GiB of them for its gradients, and all calls
 * those of up to 128 rows, or up to 64 MiB of partial ones of small problems),
 * and the global norm of many gradient tensors with their clipping.
 *
 * Conventions for every call:
 *  - Array arguments are DEVICE memory on the current HIP device, owned by the
 *    caller (tables of pointers and sizes, and the structures, are host memory
 *    and read during the call), aligned to its type.  Outputs must not overlap inputs or the
 *    workspace unless a call says so.
 *  - Calls enqueue their work on `stream` (a hipStream_t; NULL: the null
 *    stream) and return; nothing waits for the device, nothing is allocated,
 *    and no state is kept between calls.  They may be captured in a HIP graph.
 *  - Temporaries live in a workspace given by the caller: at least as many
 *    bytes as the matching *_workspace call says, aligned to 256 bytes.  Its
 *    contents need no initialisation and mean nothing afterwards.  Calls that
 *    may run at the same time need workspaces of their own.
 *  - Calls return CCDPP_OK or a negative status of ccdpp.h: EINVAL for a bad
 *    argument, found before any work is enqueued, and EDEVICE where a launch
 *    fails or no device is there.  ccdpp_ops_last_error() says why.
 *  - Results are the same, bit for bit, from run to run.
 */
#ifndef CCDPP_OPS_H
#define CCDPP_OPS_H

#include <stdint.h>

#include "ccdpp.h"

#ifdef __cplusplus
extern "C" {
#endif

enum ccdpp_dtype {
    CCDPP_F32 = 0,
    CCDPP_BF16 = 1,
    CCDPP_F16 = 2
};

/*
 * Rows against a table.  Logits z_tv = scale * (x_t . e_v) + offset_v.
 *   t, v, d  : rows (0 <= t < 2^26), table length (1 <= v < 2^28), factors
 *              (1 <= d <= 65536); t * v < 2^39
 *   dtype    : enum ccdpp_dtype of x, table and their gradients
 *   x, ldx   : t rows of d values, ldx >= d values apart
 *   table, ldt : v rows of d values, ldt >= d values apart
 *   target, target_bits : t integers of 32 or 64 bits.  0 <= target < v; a negative one
 *              marks an ignored row (loss 0, no part in any gradient, whatever its
 *              x holds); one >= v makes the row's loss, and with it the gradients, NaN
 *   scale    : finite
 *   offset   : float[v], or NULL for zeros; a constant (no gradient).  -inf, or
 *              anything below -1e38, excludes the item: its probability and its
 *              gradient are 0 whatever its table row holds.  A row whose target is
 *              excluded has loss +inf and is left out of the gradients.  Where
 *              every item is excluded, lse is -inf and probabilities are 0.
 * Products of 16-bit values are exact and summed in 32 bits.  32-bit values are
 * multiplied as they are for t <= 32 (for the logits also t <= 128 where d > 128), and as
 * sums of two halves with 11 bits each otherwise: 22 bits of every value down to 2^-17 of
 * the largest of its row (of x or of the table), and 2^-39 of that largest below it.  (With
 * d <= 128, of the table's largest, or to what is some 5e-7 of a logit, where x is small enough for that.)
 * A logit's and a probability's relative error are some 5e-7 (1 + |z|), what a logit and
 * its lse have in 32 bits.
 */
typedef struct ccdpp_softmax {
    int64_t t, v;
    int32_t d;
    int32_t dtype;
    const void *x;
    int64_t ldx;
    const void *table;
    int64_t ldt;
    const void *target;
    int32_t target_bits;
    float scale;
    const float *offset;
} ccdpp_softmax_t;

enum ccdpp_softmax_call {
    CCDPP_SOFTMAX_LOSS = 0,   /* ccdpp_softmax_loss */
    CCDPP_SOFTMAX_GRAD = 1,   /* ccdpp_softmax_loss_grad */
    CCDPP_SOFTMAX_TRAIN = 2   /* ccdpp_softmax_loss_train */
};

/* Bytes of workspace of `call` (enum ccdpp_softmax_call) on this problem: of its
 * sizes and dtype; no pointer of p is read. */
int ccdpp_softmax_workspace(const ccdpp_softmax_t *p, int32_t call, int64_t *bytes);

/* loss[i] = lse[i] - z[i, target_i] and lse[i] = log sum_v exp z_iv, float[t] each. */
int ccdpp_softmax_loss(const ccdpp_softmax_t *p, float *loss, float *lse, void *workspace,
                       int64_t workspace_bytes, void *stream);

/* Gradients of sum_t grad_t loss_t, from the lse of ccdpp_softmax_loss on the same problem (a
 * lower one gives terms beyond their weight, which overflow to infinities and NaN from 8 times on):
 *   dx_t = scale sum_v G_tv e_v,  dtable_v = scale sum_t G_tv x_t,
 *   G_tv = grad_t (exp(z_tv - lse_t) - [v = target_t]).
 *   grad          : float[t], or NULL for ones
 *   dx, lddx      : t rows of d values of p->dtype, lddx >= d values apart; may be NULL
 *   dtable, lddt  : v rows likewise; may be NULL
 * Sums are held in 32 bits and rounded once to p->dtype.  The terms G_tv are rounded to 11 bits
 * for 16-bit types with d > 128 and t > 32, to 16 at least for other 16-bit ones, and to 22 for 32-bit
 * types (t <= 32: as they are), but none by more than 2^-29 of its row's weight for dx and 2^-19 of its
 * item's largest term for dtable: light rows and unlikely items keep their digits.  32-bit x and
 * tables have 22 bits of each value down to 2^-17 of the largest of all, 2^-39 of that below it. */
int ccdpp_softmax_loss_grad(const ccdpp_softmax_t *p, const float *lse, const float *grad,
                            void *dx, int64_t lddx, void *dtable, int64_t lddt,
                            void *workspace, int64_t workspace_bytes, void *stream);

/* Both in one call: loss and lse as ccdpp_softmax_loss, then the gradients. */
int ccdpp_softmax_loss_train(const ccdpp_softmax_t *p, float *loss, float *lse, const float *grad,
                             void *dx, int64_t lddx, void *dtable, int64_t lddt,
                             void *workspace, int64_t workspace_bytes, void *stream);

/* Bytes of workspace of ccdpp_grad_norm and ccdpp_clip_grads (the same for any tensors). */
int ccdpp_grad_norm_workspace(int64_t *bytes);

/* norm[0] = sqrt(sum of the squares of all values of n tensors), summed in 64 bits.
 *   tensors, sizes, dtypes : host arrays of n device pointers, lengths (>= 0) and
 *                            enum ccdpp_dtype; each tensor is contiguous
 *   n >= 0 (the norm of nothing is 0) */
int ccdpp_grad_norm(int32_t n, const void *const *tensors, const int64_t *sizes,
                    const int32_t *dtypes, float *norm, void *workspace, int64_t workspace_bytes,
                    void *stream);

/* The norm as above, and out_i = c * tensor_i with c = min(1, max_norm / (norm + eps)).
 *   out      : host array of n device pointers; out[i] == tensors[i] clips in place (no
 *              other overlap).  In place, tensors are not written where c is 1.
 *   max_norm : >= 0 (may be infinite); eps : >= 0
 * A norm that is NaN makes every output NaN; one that is infinite makes c = 0 (1 where max_norm is, too).
 * Tensors that share memory with one another are not clipped twice but undefined. */
int ccdpp_clip_grads(int32_t n, const void *const *tensors, void *const *out, const int64_t *sizes,
                     const int32_t *dtypes, float max_norm, float eps, float *norm, void *workspace,
                     int64_t workspace_bytes, void *stream);

/* Message of the last failed call of this header on this thread.  Never NULL. */
const char *ccdpp_ops_last_error(void);

#ifdef __cplusplus
}
#endif
#endif
