/*
 * rapid_policy_ops.h -- the operators of a policy network that lie between the sampled tokens and the hidden states
 * that rapid_pg_loss_fused_head turns into the loss, each with its gradient, as CUDA kernels for NVIDIA B200 (sm_100a):
 *
 *   rapid_embedding_*      token embedding with scaling; its gradient, summed over sorted tokens
 *   rapid_qk_norm_rope_*   root-mean-square norm of every query and key head and the rotation by position, in one pass
 *   rapid_attention_*      causal attention over the padded token grid; its gradient, from recomputed probabilities
 *
 * The conventions are those of rapid_pg.h: plain scalars and descriptors are HOST memory, every array is a DEVICE
 * pointer valid on the current device; the calls only enqueue work on `stream` (several launches may be enqueued, all
 * capturable in a CUDA graph), allocate nothing and keep nothing between calls; what the host can see is checked before
 * the first launch and returned as a status; what only the device can see never traps.  Calls that use one workspace must
 * not overlap on the device.  No result depends on the order in which blocks run: the same inputs give the same bits.
 *
 * Arrays of int32 and float lie on 4-byte boundaries, stats on 8-byte ones, matrices and pitches as each operator says.
 *
 * Rows are those of the padded token grid: row r = n * seq_len + t is position t of generation n.
 */
#ifndef RAPID_POLICY_OPS_H
#define RAPID_POLICY_OPS_H

#include "rapid_pg.h"

#ifdef __cplusplus
extern "C" {
#endif

/* ---- token embedding ------------------------------------------------------------------------------------- */

enum {
    /* rapid_embedding_bwd: dtable is [vocab, ld_table] bf16 instead of float (dtype must be RAPID_BF16). */
    RAPID_EMBED_DTABLE_BF16 = 1u,
    /* rapid_embedding_bwd: add to dtable (rows of tokens that do not occur are neither read nor written) instead of  */
    /* overwriting all of it.  The sum over a token's rows is formed in float and added with one rounding.            */
    RAPID_EMBED_ACCUMULATE = 2u
};

typedef struct rapid_embed_desc {
    int64_t n_rows;   /* T >= 1 (at most 2^31 - 1)                                                         */
    int32_t vocab;    /* V: rows of the table, 1 .. 2^27 - 2                                               */
    int32_t dim;      /* D: columns                                                                        */
    int64_t ld_table; /* row pitch of table / dtable in elements of their own type, >= dim                 */
    int64_t ld_rows;  /* row pitch of out / dout in elements, >= dim                                       */
    int32_t dtype;    /* rapid_dtype_t of table, out and dout                                              */
    uint32_t flags;   /* RAPID_EMBED_* bits                                                                */
    float scale;      /* s, finite                                                                         */
    int32_t reserved; /* 0                                                                                 */
} rapid_embed_desc_t;

/*
 * out[r, :] = s * table[tokens[r], :], the product in float, rounded once.  Rows that are masked, or whose token lies
 * outside [0, vocab), come out as zeros.
 *   tokens [T] int32;  mask [T] uint8, non-zero = live, NULL = all live;  table [V, ld_table];  out [T, ld_rows]
 *   stats  may be NULL; n_tokens = live rows with a valid token, n_bad_token = live rows with another; the rest zero
 * Row pitches are multiples of 16 bytes and bases are 16-byte aligned; columns >= dim are neither read nor written, so matrices of
 * one pitch (in bytes) may lie side by side in the same rows.  Other matrices have to be apart altogether.
 */
rapid_status_t rapid_embedding_fwd(const rapid_embed_desc_t* desc, const int32_t* tokens, const uint8_t* mask,
                                   const void* table, void* out, rapid_stats_t* stats, void* stream);

/* Scratch of rapid_embedding_bwd: 32 bytes a row at most, 4 bytes a token, 4 bytes per 32 elements of dout, and 128 KB. */
rapid_status_t rapid_embedding_bwd_workspace_bytes(const rapid_embed_desc_t* desc, size_t* bytes);

/*
 * dtable[v, :] (+)= s * sum of dout[r, :] over the live rows r with tokens[r] == v, summed in float.  The order of the additions
 * is fixed by tokens and mask: the rows are sorted by token (stable); a token with at most 8 rows has them added in row order; of
 * another, whole pieces (sorted positions 32 j .. 32 j + 31) are summed in row order first, then seven runs each add a seventh of the
 * rows before the first whole piece, of those behind the last one, and of the pieces, and the seven sums are added in order.
 * Where a piece begins depends on the rows of smaller tokens, so they can change a sum's last bits.  Masked rows of dout, and
 * rows with a token outside [0, vocab), are never read.  Without RAPID_EMBED_ACCUMULATE every row of dtable is written (zeros
 * where a token does not occur).
 *   dtable [V, ld_table] float (bf16 with RAPID_EMBED_DTABLE_BF16);  workspace 256-byte aligned
 */
rapid_status_t rapid_embedding_bwd(const rapid_embed_desc_t* desc, const int32_t* tokens, const uint8_t* mask,
                                   const void* dout, void* dtable, void* workspace, size_t workspace_bytes, void* stream);

/* ---- norms of queries and keys for each head, with the rotation by position ------------------------------- */

enum {
    RAPID_QK_NO_NORM = 1u,     /* rotation only: weights are not used (may be NULL)                              */
    RAPID_QK_UNIT_OFFSET = 2u, /* the norm multiplies by 1 + weight instead of weight                            */
    RAPID_QK_INTERLEAVED = 4u  /* pair i is elements (2i, 2i + 1) of a head instead of (i, i + rot_dim / 2)      */
};

typedef struct rapid_qk_desc {
    int32_t n_seq, seq_len;        /* T = n_seq * seq_len rows                                                 */
    int32_t n_q_heads, n_k_heads;  /* both >= 1                                                                */
    int32_t head_dim;              /* a multiple of 16, at most 256                                            */
    int32_t rot_dim;               /* elements of a head that rotate: a multiple of 16, 16 .. head_dim         */
    int64_t ld_q, ld_k;            /* row pitch, in elements, of q and of k                                    */
    int64_t ld_q_out, ld_k_out;    /* of q_out and dq_out, and of k_out and dk_out                             */
    int64_t ld_dq, ld_dk;          /* of dq and of dk (rapid_qk_norm_rope_bwd only)                            */
    int32_t dtype;                 /* rapid_dtype_t of the matrices                                            */
    uint32_t flags;                /* RAPID_QK_* bits                                                          */
    float eps;                     /* >= 0, finite                                                             */
    int32_t reserved;              /* 0                                                                        */
} rapid_qk_desc_t;

/*
 * For every head x of a row's queries (weight q_weight) and keys (k_weight), with p the row's position:
 *     n = x * (mean_j x_j^2 + eps)^(-1/2) * weight                       (n = x with RAPID_QK_NO_NORM)
 *     y_a = n_a cos(p f_i) - n_b sin(p f_i),  y_b = n_a sin(p f_i) + n_b cos(p f_i)    for pair i = (a, b), i < rot_dim / 2
 *     y_j = n_j                                                          for the elements that do not rotate
 * in float, rounded once; the angles p f_i are formed and reduced in double.
 *   q [T, ld_q], k [T, ld_k]   heads side by side: head h of row r starts at r * ld + h * head_dim
 *   q_weight, k_weight [head_dim] float;  inv_freq [rot_dim / 2] float, f_i
 *   positions [T] int32, p of each row; NULL = t, the place in the generation
 *   mask [T] uint8, non-zero = live, NULL = all live: masked rows are never read and come out as zeros
 *   q_out, k_out   may be q and k themselves (in place, with equal pitches); no other overlap is allowed
 * Bases are 16-byte aligned and row pitches are multiples of 16 bytes.
 */
rapid_status_t rapid_qk_norm_rope_fwd(const rapid_qk_desc_t* desc, const void* q, const void* k, const float* q_weight,
                                      const float* k_weight, const float* inv_freq, const int32_t* positions,
                                      const uint8_t* mask, void* q_out, void* k_out, void* stream);

/* Scratch of rapid_qk_norm_rope_bwd: partial sums of the two weight gradients. */
rapid_status_t rapid_qk_norm_rope_bwd_workspace_bytes(const rapid_qk_desc_t* desc, size_t* bytes);

/*
 * The gradient of the above, from the inputs q and k and the gradients dq_out, dk_out of its outputs; the norms are
 * recomputed.  With y' = the gradient rotated back, xh = x * rstd and w the factor of the norm:
 *     dx = rstd * (w y' - xh * mean_j(w_j y'_j xh_j)),    dweight = sum over rows and heads of y' * xh
 *   dq [T, ld_dq], dk [T, ld_dk]   masked rows are written as zeros; may be dq_out and dk_out themselves (equal pitches)
 *   dq_weight, dk_weight [head_dim] float, summed over all live rows and heads (not written with RAPID_QK_NO_NORM, and
 *                                  may then be NULL)
 */
rapid_status_t rapid_qk_norm_rope_bwd(const rapid_qk_desc_t* desc, const void* q, const void* k, const float* q_weight,
                                      const float* k_weight, const float* inv_freq, const int32_t* positions,
                                      const uint8_t* mask, const void* dq_out, const void* dk_out, void* dq, void* dk,
                                      float* dq_weight, float* dk_weight, void* workspace, size_t workspace_bytes,
                                      void* stream);

/* ---- causal attention ------------------------------------------------------------------------------------- */

typedef struct rapid_attn_desc {
    int32_t n_seq, seq_len;       /* T = n_seq * seq_len rows                                                     */
    int32_t n_heads, n_kv_heads;  /* n_heads a multiple of n_kv_heads; query head h reads key head h / (n_heads / n_kv_heads) */
    int32_t head_dim;             /* a multiple of 8, 8 .. 128                                                    */
    int32_t window;               /* 0 = none; w > 0: position i sees the keys j with i - w < j <= i              */
    int64_t ld_q, ld_k, ld_v;     /* row pitch, in elements, of q, k and v                                        */
    int64_t ld_out, ld_dout;      /* of out and dout                                                              */
    int64_t ld_dq, ld_dk, ld_dv;  /* of the gradients (ld_dout too: rapid_attention_bwd only)                     */
    int32_t dtype;                /* RAPID_BF16                                                                   */
    uint32_t flags;               /* 0                                                                            */
    double scale;                 /* factor of the scores, > 0 (1 / sqrt(head_dim) as a rule); it and its product with log2(e) */
                                  /* are used as floats and have to be normal ones                                */
} rapid_attn_desc_t;

/*
 * For every generation n and head h, over the live positions b0 <= t < b1 of n:
 *     s_ij = scale * q_i . k_j  for j <= i (and i - j < window),   lse_i = log sum_j exp s_ij,
 *     out_i = sum_j exp(s_ij - lse_i) v_j
 *   q [T, ld_q], k [T, ld_k], v [T, ld_v], out [T, ld_out]  bf16, heads side by side (head h of row r starts at
 *            r * ld + h * head_dim); bases 16-byte aligned, pitches multiples of 8 elements
 *   bounds [n_seq][2] int32: b0, b1 of each generation (padding may lie on either side); NULL = 0, seq_len.  Values are
 *            clipped to [0, seq_len]; b1 <= b0 leaves the generation without a live position
 *   out      rows outside the bounds are written as zeros
 *   lse      [n_seq, n_heads, seq_len] float out, natural logarithm, -infinity outside the bounds; may be NULL
 *   stats    may be NULL; only status is meaningful: RAPID_OK, or RAPID_ERR_TIMEOUT when a bounded wait gave up (the
 *            outputs are then unspecified).  Nothing else reports that: without stats a call that gave up looks like any other
 * Rows outside the bounds may hold anything (infinities and NaN too) and influence nothing.  Rows inside must be finite, and so must be
 * the scores of pairs that see each other, in float.
 * The products run on the tensor cores in bf16 with float accumulation; scores, maximum and sum of the softmax are float;
 * the probabilities are rounded to bf16 for their product with v (half a step, a relative error of at most 2^-8 each).
 */
rapid_status_t rapid_attention_fwd(const rapid_attn_desc_t* desc, const void* q, const void* k, const void* v,
                                   const int32_t* bounds, void* out, float* lse, rapid_stats_t* stats, void* stream);

/*
 * Scratch of rapid_attention_bwd: two floats for each head and position of the tiles, which are 128 positions of one generation or, where
 * generations have at most 64 positions, as many whole generations as fit; each of the two arrays in whole 8 KB.
 */
rapid_status_t rapid_attention_bwd_workspace_bytes(const rapid_attn_desc_t* desc, size_t* bytes);

/*
 * The gradient, from the inputs, out and lse of the forward call and the gradient dout of out:
 *     p_ij = exp(s_ij - lse_i),  delta_i = dout_i . out_i,  ds_ij = scale * p_ij * (dout_i . v_j - delta_i)
 *     dq_i = sum_j ds_ij k_j,   dk_j = sum_i ds_ij q_i,   dv_j = sum_i p_ij dout_i    (dk, dv summed over the heads that
 * share a key head).  Rows outside the bounds are written as zeros and read from nowhere.  p and ds are rounded to bf16 for
 * the last three products; the sums are float, each gradient is rounded once.
 *   dout [T, ld_dout], dq [T, ld_dq], dk [T, ld_dk], dv [T, ld_dv] bf16;  workspace 256-byte aligned
 * Refused (RAPID_ERR_UNSUPPORTED): more than 2^20 pairs of a query tile of 128 positions that sees one key and a head that shares it.
 */
rapid_status_t rapid_attention_bwd(const rapid_attn_desc_t* desc, const void* q, const void* k, const void* v,
                                   const int32_t* bounds, const void* out, const float* lse, const void* dout, void* dq,
                                   void* dk, void* dv, rapid_stats_t* stats, void* workspace, size_t workspace_bytes,
                                   void* stream);

#ifdef __cplusplus
}
#endif
#endif /* RAPID_POLICY_OPS_H */
