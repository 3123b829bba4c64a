/*
 * ccdpp_seq.h -- operators of the CCD++ library on sequences of choices, in
 * DEVICE memory (MI355X, gfx950).
 *
 * ccdpp_ops.h takes every choice by itself.  The calls here take what a user
 * chose one after another: a gated linear recurrence turns the rows of a
 * sequence (the factors of the items that were taken, hidden states) into the
 * row that the softmax over all items is made from, with its gradients for
 * training and a call of one row for serving; a selection of beams answers with
 * the best next items and puts the beams' states in their order; dropout stands
 * between them in training.
 *
 * The conventions are those of ccdpp_ops.h (device memory, streams, workspaces,
 * statuses, graphs; the message is ccdpp_ops_last_error()), and types are its
 * enum ccdpp_dtype.  Results are the same, bit for bit, from run to run.
 */
#ifndef CCDPP_SEQ_H
#define CCDPP_SEQ_H

#include "ccdpp_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

enum ccdpp_scan_mode {
    CCDPP_SCAN_GIVEN = 0,    /* a = gate,             u = x           */
    CCDPP_SCAN_SIGMOID = 1   /* a = 1 / (1 + e^-gate), u = (1 - a) x  */
};

/*
 * Gated recurrences over sequences that lie one after another ("packed") in n rows:
 *   h_t = a_t h_(t-1) + u_t, each column by itself, h before a sequence's first row its
 *   initial state.
 *   n, s, d  : rows (0 <= n < 2^31), sequences (0 <= s < 2^31), columns (1 <= d <= 65536)
 *   dtype    : of x, gate, y and their gradients; states and their gradients are float
 *   mode     : enum ccdpp_scan_mode
 *   x, ldx   : n rows of d values, ldx >= d values apart; gate, ldg likewise
 *   starts, starts_bits : s + 1 integers of 32 or 64 bits, ascending: sequence q has rows
 *              starts[q] to starts[q + 1] - 1, and none where they are equal.  Rows before
 *              starts[0] and from starts[s] on belong to no sequence: they are not read, and
 *              outputs are 0 there.  (Values are held within [0, n]; where they do not
 *              ascend, results are undefined, but nothing else is read or written.)
 *   initial  : float, s rows of d, or NULL for zeros
 * States, products of decays and their gradients are held in 32 bits and rounded once to dtype;
 * SIGMOID has a and 1 - a to some 2^-21 of themselves.
 * (GIVEN decays above 1: also the product of those of any rows one after another has to lie
 * within the range of 32 bits.  Where that of many rows is below it, what the state before them
 * adds behind them may be 0, and NaN where the state is infinite.)  A value that is not finite stays
 * within its column and its sequence.
 */
typedef struct ccdpp_scan {
    int64_t n, s;
    int32_t d;
    int32_t dtype;
    int32_t mode;
    int32_t starts_bits;
    const void *x;
    int64_t ldx;
    const void *gate;
    int64_t ldg;
    const void *starts;
    const float *initial;
} ccdpp_scan_t;

enum ccdpp_scan_call {
    CCDPP_SCAN_FORWARD = 0,  /* ccdpp_gated_scan */
    CCDPP_SCAN_GRAD = 1      /* ccdpp_gated_scan_grad */
};

/* Bytes of workspace of `call` (enum ccdpp_scan_call), and of the states that the forward
 * call keeps for the gradients: of sizes, dtype and mode; no pointer of p is read. */
int ccdpp_scan_workspace(const ccdpp_scan_t *p, int32_t call, int64_t *bytes);
int ccdpp_scan_kept(const ccdpp_scan_t *p, int64_t *bytes);

/* y_t = h_t, and last_q = the state behind sequence q's last row (its initial state where it
 * has none).
 *   y, ldy : n rows of d values of dtype, ldy >= d values apart
 *   last   : float, s rows of d, or NULL; not `initial` itself
 *   kept   : ccdpp_scan_kept bytes, aligned to 16, or NULL: one state in 8 rows */
int ccdpp_gated_scan(const ccdpp_scan_t *p, void *y, int64_t ldy, float *last, void *kept,
                     void *workspace, int64_t workspace_bytes, void *stream);

/* Gradients of sum_t dy_t y_t + sum_q dlast_q last_q.  With l_t = dy_t + a_(t+1) l_(t+1)
 * (dlast_q behind the last row):
 *   GIVEN:   dx_t = l_t,            dgate_t = l_t h_(t-1)
 *   SIGMOID: dx_t = (1 - a_t) l_t,  dgate_t = l_t (h_(t-1) - x_t) a_t (1 - a_t)
 *   dinitial_q = a l of the first row (dlast_q where there is none)
 *   dy, lddy : n rows likewise;  dlast : float, s rows of d, or NULL for zeros
 *   kept     : what ccdpp_gated_scan left for the same problem
 *   dx, dgate : n rows likewise;  dinitial : float, s rows of d, or NULL; not `dlast` itself */
int ccdpp_gated_scan_grad(const ccdpp_scan_t *p, const void *dy, int64_t lddy, const float *dlast,
                          const void *kept, void *dx, int64_t lddx, void *dgate, int64_t lddg,
                          float *dinitial, void *workspace, int64_t workspace_bytes, void *stream);

/* One more row of n sequences: state = a state + u in place, y = state.
 *   n, d, dtype, mode, x, gate, y : as above;  state, lds : float, n rows, lds >= d values apart */
int ccdpp_gated_scan_step(int64_t n, int32_t d, int32_t dtype, int32_t mode, const void *x,
                          int64_t ldx, const void *gate, int64_t ldg, float *state, int64_t lds,
                          void *y, int64_t ldy, void *stream);

/*
 * The best continuations of beams.  Each of `groups` groups has `beams` beams with a score;
 * beam b continued by item i has the score
 *   score_b + z_bi - log sum_j exp z_bj,   z_bi = logits_bi + offset_i (in 32 bits).
 * The exponentials and parts of their sums have 32 bits, and the log sum is within 2^-17 of the
 * exact one; all else is in 64 bits, and scores are rounded once.  The k greatest of a group are taken,
 * in descending order; of equal ones the lowest beam goes first, and of a beam the greatest z, then the
 * lowest item.  The order within a beam is exact; of beams whose exact scores differ by less
 * than their log sums may be off, either may go first.
 *   groups, beams, k, v : 0 <= groups < 2^24, 1 <= beams <= 64, 1 <= k <= 64, 1 <= v < 2^28
 *   logits, ld : groups * beams rows of v values of dtype, ld >= v values apart
 *   score  : float per beam; -inf: there is no such beam, and its logits are not read
 *   offset : float[v], or NULL for zeros; -inf, or anything below -1e38, excludes the item,
 *            whatever its logits hold (so does a z of -inf)
 *   done   : one byte per beam, or NULL for zeros.  A beam with one other than 0 is at its end:
 *            its logits are not read, and it goes on as itself, with the item `end` and its score
 *   end    : the item that ends a beam, or -1
 * Among z, NaN counts as +inf; all continuations of a beam that has one of them have the score NaN, and
 * NaN counts as the greatest score.
 */
typedef struct ccdpp_beam {
    int64_t groups, v;
    int32_t beams, k;
    int32_t dtype;
    int32_t reserved; /* 0 */
    const void *logits;
    int64_t ld;
    const float *score;
    const float *offset;
    const uint8_t *done;
    int64_t end;
} ccdpp_beam_t;

/* Bytes of workspace: of sizes and dtype; no pointer of p is read. */
int ccdpp_beam_workspace(const ccdpp_beam_t *p, int64_t *bytes);

/* groups x k each: the scores, the beams (within the group) and the items; where there are
 * fewer than k continuations -inf, -1 and -1.
 *   out_done : one byte each, or NULL: 1 where the item is `end` or -1 */
int ccdpp_beam_select(const ccdpp_beam_t *p, float *out_score, int64_t *parent, int64_t *item,
                      uint8_t *out_done, void *workspace, int64_t workspace_bytes, void *stream);

/* out row (g, j) = in row (g, parent[g, j]) of n tensors; zeros where parent is not in [0, beams).
 *   in, in_stride : host arrays: groups * beams rows each, and how many bytes they are apart
 *   out, row_bytes : host arrays: groups * k rows each, one after another, of so many bytes (>= 0)
 * Pointers need no alignment. */
int ccdpp_beam_reorder(int64_t groups, int32_t beams, int32_t k, const int64_t *parent, int32_t n,
                       const void *const *in, const int64_t *in_stride, void *const *out,
                       const int64_t *row_bytes, void *stream);

/* y = [residual +] x * [r >= p 2^32] / (1 - p): 1 / (1 - p), its product with x and the sum with the
 * residual are rounded to 32 bits each, and y to dtype.  r is word j mod 4 of Philox4x32 with
 * 7 rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) of
 * counter (j / 4, i, i >> 32, 0) and key (seed, seed >> 32), for column j and row
 * i = first_row + the row's number: the mask is never stored, and the gradient is the same call
 * on dy.  Values that are dropped go nowhere, whatever they hold.
 *   n, d   : 0 <= n < 2^31, 1 <= d < 2^31;  x, residual (or NULL), y : n rows, ld* >= d apart
 *   y      : may be x or residual itself (the same pointer and stride; no other overlap)
 *   p      : 0 <= p <= 1, taken as round(p 2^32) / 2^32 for the mask; 1 drops everything
 *   seed   : the key, or, where seed_at is not NULL, *seed_at in device memory when the call runs
 *   first_row : >= 0 */
int ccdpp_dropout(int64_t n, int64_t d, int32_t dtype, const void *x, int64_t ldx,
                  const void *residual, int64_t ldr, void *y, int64_t ldy, double p, uint64_t seed,
                  const uint64_t *seed_at, int64_t first_row, void *stream);

#ifdef __cplusplus
}
#endif
#endif
