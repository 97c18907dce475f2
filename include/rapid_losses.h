/*
 * rapid_losses.h -- further losses over the policy's logits, each with its gradient by the logits, as CUDA kernels for NVIDIA
 * B200 (sm_100a).  They stand beside the policy-gradient loss of rapid_pg.h, on the same padded token grid:
 *
 *   rapid_clip_loss_*        clipped importance ratios for every token, with an optional KL term to a reference policy
 *   rapid_preference_loss_*  pairs of generations, one preferred to the other
 *   rapid_distill_loss_*     a teacher's top logits for every token
 *
 * (The paper compares its method to group-relative training with a KL term, to clipped variants of it and to training on a
 * teacher's output; these are the losses of such runs.)
 *
 * The conventions are those of rapid_pg.h: plain scalars and descriptors are HOST memory, every array is a DEVICE pointer valid
 * on the current device; the calls only enqueue work on `stream` (several launches, all capturable in a CUDA graph), allocate
 * nothing and keep nothing between calls; what the host can see is checked before the first launch and returned as a status;
 * what only the device can see never traps.  Calls that use one workspace must not overlap on the device.  No result depends
 * on the order in which blocks run: the same inputs give the same bits.
 *
 * Common arguments:
 *   logits     [T, ld] of desc->dtype, only the first `vocab` entries of a row are used.  Entries may be -inf or the dtype's
 *              lowest finite value (probability and gradient exactly 0) as long as every live row has a finite entry.  The largest
 *              other entry of a row (and with a teacher's log-sum-exp the largest outside the list) over the temperature has to lie
 *              within +-2^27.  Beyond that, and with +inf and NaN, results are unspecified, but memory-safe.  Rows that do not
 *              count are never read.
 *   targets    [T] int32, the token y_r; a row whose token lies outside [0, vocab) counts as masked and is counted in stats
 *   mask       [T] uint8, non-zero = the row counts; NULL = all ones
 *   dlogits    [T, ld_grad] out, the type of the logits: the gradient of `loss`, rounded once.  Rows that do not count are
 *              written as zeros, columns >= vocab are not touched.  May be `logits` itself (in place, ld_grad == ld); no other
 *              overlap is allowed.  NULL = no gradient (the logits are read once and nothing of their size is written)
 *   loss       [1] float out
 *   stats      out, may be NULL
 *   workspace  256-byte aligned, of the size that the operator's *_workspace_bytes gives; need not be initialised
 * Bases of logits and dlogits are 16-byte aligned and their pitches multiples of 16 bytes; int32 and float arrays lie on 4-byte
 * boundaries, stats on an 8-byte one.  `scale` multiplies the loss and its gradient.
 *
 * Sums over the vocabulary are formed in float pieces that are added in double, everything of one value a row, a pair or a generation is
 * double (sums over a generation's pairs, where there are many, whole numbers of 2^-83 of the largest of them).
 */
#ifndef RAPID_LOSSES_H
#define RAPID_LOSSES_H

#include "rapid_pg.h"

#ifdef __cplusplus
extern "C" {
#endif

enum {
    /* rapid_clip_loss: every generation weighs the same: row r of generation n has the weight 1 / (N len_n), len_n its rows  */
    /* that count, instead of 1 / (rows that count).  A generation without such rows still counts in N.                       */
    RAPID_LOSS_NORM_SEQ = 1u,
    /* The number of rows, of generations (with RAPID_LOSS_NORM_SEQ) or of pairs to divide by is desc->norm_z: the global one */
    /* where a mini-batch is spread over several GPUs, so that the losses and gradients of the parts add up.                  */
    RAPID_LOSS_NORM_GIVEN = 2u,
    /* rapid_clip_loss: adv is [T], an advantage for each row, instead of [N], one for each generation.                       */
    RAPID_CLIP_ADV_TOKEN = 4u,
    /* rapid_preference_loss: max(0, 1 - h), or (h - 1/2)^2, in place of the logistic form (at most one of the two).          */
    RAPID_PREF_HINGE = 16u,
    RAPID_PREF_SQUARED = 32u,
    /* rapid_preference_loss: s_n is the mean over the generation's rows that count instead of their sum.                     */
    RAPID_PREF_TOKEN_MEAN = 64u
};

/* Side statistics (DEVICE memory, 48 bytes like rapid_stats_t; what an operator does not name is zero). */
typedef struct rapid_loss_stats {
    int64_t n_tokens;      /* rows that count                                                                        */
    int32_t n_clipped;     /* clip: rows whose ratio's gradient the clip cuts off                                    */
    int32_t n_bad;         /* rows with the mask set but a token (distill: a list) that is not valid                 */
    int32_t n_pairs;       /* preference: valid pairs                                                                */
    int32_t status;        /* RAPID_OK, or RAPID_ERR_TIMEOUT when a bounded wait gave up (outputs then unspecified)  */
    double mean_log_ratio; /* clip: mean over rows of log rho; preference: mean over pairs of h                      */
    double mean_kl;        /* clip: mean over rows of the KL estimate; preference: share of pairs with h > 0         */
    double loss;           /* the loss in double                                                                     */
} rapid_loss_stats_t;

/* ---- clipped policy loss ----------------------------------------------------------------------------------- */

typedef struct rapid_clip_desc {
    int32_t n_seq, seq_len;   /* N generations of L padded positions, T = N * L rows (at most 2^31 - 1024)           */
    int32_t vocab;            /* V                                                                                   */
    int32_t dtype;            /* rapid_dtype_t of logits and dlogits                                                 */
    int64_t ld, ld_grad;      /* row pitches, in elements, of logits and dlogits, >= vocab                           */
    uint32_t flags;           /* RAPID_LOSS_* and RAPID_CLIP_* bits                                                  */
    int32_t reserved;         /* 0                                                                                   */
    double eps_low, eps_high; /* >= 0; the ratio is clipped to [1 - eps_low, 1 + eps_high] (+inf: not on that side)  */
    double kl_beta;           /* >= 0, finite                                                                        */
    double scale;             /* finite                                                                              */
    double norm_z;            /* > 0, finite with RAPID_LOSS_NORM_GIVEN; else ignored                                */
} rapid_clip_desc_t;

/* Scratch of rapid_clip_loss: 25 bytes a row and 16 for each begun 16 KB of its logits (up to four times), 4 a generation with           */
/* RAPID_LOSS_NORM_SEQ, and 73 KB. */
rapid_status_t rapid_clip_loss_workspace_bytes(const rapid_clip_desc_t* desc, size_t* bytes);

/*
 *     lp_r = z[r, y_r] - log sum_v exp z[r, v],   rho_r = exp(lp_r - old_logp_r),   d_r = ref_logp_r - lp_r
 *     loss = sum_r w_r ( max(-rho_r A_r, -clip(rho_r, 1 - eps_low, 1 + eps_high) A_r) + kl_beta (exp(d_r) - d_r - 1) )
 *     dlogits[r, v] = g_r (softmax(z[r, .])_v - 1[v == y_r])
 *     g_r = w_r ( rho_r A_r [where the first of the two is not the smaller] + kl_beta (exp(d_r) - 1) )
 * over the rows that count; w_r = scale / (their number), see the flags.
 *   old_logp   [T] float, log-probabilities of the tokens under the policy that sampled them
 *   ref_logp   [T] float, under the reference policy; may be NULL when kl_beta is 0
 *   adv        [N] float, or [T] with RAPID_CLIP_ADV_TOKEN
 *   token_logp [T] float out, lp_r (0 on rows that do not count); may be NULL
 */
rapid_status_t rapid_clip_loss(const rapid_clip_desc_t* desc, const void* logits, const int32_t* targets, const uint8_t* mask,
                               const float* old_logp, const float* ref_logp, const float* adv, void* dlogits, float* loss,
                               float* token_logp, rapid_loss_stats_t* stats, void* workspace, size_t workspace_bytes,
                               void* stream);

/* ---- preference loss --------------------------------------------------------------------------------------- */

typedef struct rapid_pref_desc {
    int32_t n_seq, seq_len, vocab, dtype; /* as above                                                                */
    int64_t ld, ld_grad;
    uint32_t flags;          /* RAPID_LOSS_NORM_GIVEN and RAPID_PREF_* bits                                          */
    int32_t n_pairs;         /* P >= 1, at most 2^20                                                                 */
    double beta;             /* > 0, finite                                                                          */
    double margin;           /* finite                                                                               */
    double label_smoothing;  /* 0 .. 0.5, the probability that a pair is the wrong way round (logistic form only)    */
    double scale, norm_z;    /* as above                                                                             */
} rapid_pref_desc_t;

/* Scratch of rapid_preference_loss: that of rapid_clip_loss, 32 bytes a generation and 8 a pair. */
rapid_status_t rapid_preference_loss_workspace_bytes(const rapid_pref_desc_t* desc, size_t* bytes);

/*
 *     s_n = sum over the rows of generation n that count of (lp_r - ref_logp_r)
 *     h_p = beta (s_c - s_j) - margin for pair p = (c, j), c preferred to j
 *     loss = scale / P sum_p f(h_p),  f(h) = -(1 - e) log sigmoid(h) - e log sigmoid(-h), e = label_smoothing (or see the flags)
 *     dlogits[r, v] = g_n (softmax(z[r, .])_v - 1[v == y_r]),   g_n = - d loss / d s_n  (/ len_n with RAPID_PREF_TOKEN_MEAN)
 * (The squared form is that of the margin h itself; published forms that take (s_c - s_j - 1 / (2 beta))^2 are 1 / beta^2 of it.)
 * A generation may be in any number of pairs.  A pair with an index outside [0, N) is left out (P is then the number of the
 * others); a generation without rows that count has s_n = 0.
 *   pairs      [P][2] int32: preferred, other
 *   ref_logp   [T] float; NULL = no reference policy (zeros)
 *   margins    [P] float out, h_p (NaN for a pair that is left out); may be NULL
 *   token_logp [T] float out; may be NULL
 * The logits are read a second time for the gradient, once all rows of a pair are known.
 */
rapid_status_t rapid_preference_loss(const rapid_pref_desc_t* desc, const void* logits, const int32_t* targets,
                                     const uint8_t* mask, const int32_t* pairs, const float* ref_logp, void* dlogits,
                                     float* loss, float* margins, float* token_logp, rapid_loss_stats_t* stats,
                                     void* workspace, size_t workspace_bytes, void* stream);

/* ---- distillation from a teacher's top logits --------------------------------------------------------------- */

typedef struct rapid_distill_desc {
    int64_t n_rows;      /* T, 1 .. 2^31 - 1024                                                                      */
    int32_t vocab;       /* V                                                                                        */
    int32_t k;           /* K, entries of a row's list, 1 .. 256                                                     */
    int64_t ld, ld_grad; /* as above                                                                                 */
    int64_t ld_top;      /* row pitch, in elements, of top_index and top_logit, >= k                                 */
    int32_t dtype;       /* rapid_dtype_t of logits and dlogits                                                      */
    uint32_t flags;      /* RAPID_LOSS_NORM_GIVEN                                                                    */
    double temperature;  /* tau, 1e-3 .. 1e3                                                                         */
    double scale, norm_z;
} rapid_distill_desc_t;

/* Scratch of rapid_distill_loss: 29 bytes a row and 73 KB. */
rapid_status_t rapid_distill_loss_workspace_bytes(const rapid_distill_desc_t* desc, size_t* bytes);

/*
 * With q = softmax(z[r, .] / tau) over the whole vocabulary and the row's entries j = (index i_j, teacher's logit t_j):
 *   top_lse == NULL:  p = softmax(t / tau) over the list,         loss_r = sum_j p_j (log p_j - log q_{i_j})
 *   top_lse given:    p_j = exp(t_j / tau - top_lse_r), and all other tokens are one outcome more with p_0 = 1 - sum_j p_j (0 if
 *                     that is negative) and q_0 = sum of q_v outside the list:  loss_r += p_0 (log p_0 - log q_0)
 *     loss = w sum_r loss_r over the rows that count,  w = scale / (their number)
 *     dlogits[r, v] = w / tau (q_v - p_j [v == i_j]),  and w / tau q_v (1 - p_0 / q_0) outside the list where top_lse is given
 *     (where top_lse is below the list's own log-sum-exp and sum_j p_j = m > 1: w / tau (m q_v - p_j [v == i_j]))
 * (tau^2, the usual factor of a softened loss, goes into `scale`.)  Where the student has nothing outside the list (q_0 = 0: it holds the
 * whole vocabulary, or the rest is masked), a p_0 within 2^-21 max(1, |top_lse_r|), what a float leaves of 0, counts as 0; a larger
 * one is an infinite loss.
 *   top_index  [T, ld_top] int32; a negative index is a place without an entry, whatever its logit
 *   top_logit  [T, ld_top] float; -inf is an entry of probability 0
 *   top_lse    [T] float, log sum over the teacher's whole vocabulary of exp(t / tau)
 *   token_loss [T] float out, loss_r (0 on rows that do not count); may be NULL
 * A row whose list has no entry, or (top_lse == NULL) none with a finite logit, counts as masked; so does a row whose list has an
 * index >= vocab or one index twice, or a logit that is NaN or +inf, or a top_lse that is not finite: those are counted in stats->n_bad.
 */
rapid_status_t rapid_distill_loss(const rapid_distill_desc_t* desc, const void* logits, const int32_t* top_index,
                                  const float* top_logit, const float* top_lse, const uint8_t* mask, void* dlogits,
                                  float* loss, float* token_loss, rapid_loss_stats_t* stats, void* workspace,
                                  size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* RAPID_LOSSES_H */
