/*
 * aspis_worker.h -- the two ends of the model whose gradient a worker computes:
 * the embedding of tokens with its gradient, dropout, and the clipped policy
 * loss with a KL term from logits to their gradient.
 *
 *   dropout    y = residual + keep * x * 65536 / (65536 - t)                aspis_dropout
 *   embedding  y[i] = drop( scale * table[token_i] )                         aspis_embed
 *   gradient   dtable[v] = scale * sum over i with token_i = v of drop( dy[i] )  aspis_embed_grad
 *   scoring    logp_i = a z_i[y_i] - log sum_j exp( a z_i[j] )               aspis_token_logp
 *   loss       sum_i scale w_i ( max(-A_i rho_i, -A_i clip(rho_i)) + beta k_i ), and dz  aspis_policy_loss
 *
 * aspis_check compares the copies of a file's gradient bit by bit, so r workers that
 * compute the same file have to get the same bits.  All calls here give them: sums have
 * an order that the arguments fix (none depends on which block ends first), and a dropout mask is a
 * function of a seed, a stream and the element's number, of nothing that the device remembers.
 * One thing is left to the caller: aspis_token_logp and aspis_policy_loss add a row's logits in an order that depends on its
 * address modulo 32.  So a file's workers place its logits alike, each row at the same remainder (the same ld, and
 * logits that begin at multiples of 32 bytes or equally far behind one); else honest copies may differ in last bits.
 *
 * Conventions, beside those of aspis.h:
 *   - Matrices are rows of `cols` elements of fp32, bf16 or fp16 (aspis_dtype), ld >= cols
 *     elements apart, at any address that is a multiple of the element's size.  Offsets are
 *     64 bits wide.  Fastest are rows whose addresses are multiples of 16 bytes (fp32: 32).
 *   - Tokens are int32 or int64 without gaps.  A token outside 0 .. vocabulary - 1 (-1, -100)
 *     is padding: an embedding of zeros, no gradient, no loss, a zero row of dz.
 *   - Arithmetic is in fp32 (the loss's sums over the rows as pairs of fp32 numbers, 48 bits), and each result is
 *     rounded to its type once.
 *   - What a call writes must not overlap what it reads, nor another of its outputs, except
 *     where it is said to; rows that lie between one another (parts of one wider matrix)
 *     are told apart where their distances ld are equal, else refused as overlapping.
 *   - work is device memory, 16-byte aligned, of at least the bytes that the call's
 *     ..._workspace_bytes gives.  Nothing in it has to be kept or cleared between calls; calls that may
 *     overlap on the GPU, and graphs that may replay at the same time, need one each.
 *   - No call differentiates by itself: aspis_dropout on the gradient, aspis_embed_grad and aspis_policy_loss's grad are the backward
 *     passes, which a program calls.
 *   - No call allocates, copies from the host or waits; all can be captured in a graph.
 */
#ifndef ASPIS_WORKER_H
#define ASPIS_WORKER_H

#include "aspis_optim.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { ASPIS_I32 = 0, ASPIS_I64 = 1 } aspis_itype;

/* A dropout mask.  Element number e (modulo 2^64; first + i * cols + j for row i, column j) takes the 16
 * bits number e % 8, low bits of low words first, of block e / 8 of Philox 4x32 with ten
 * rounds (Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", SC 2011), whose key is `seed` and
 * whose counter is (e / 8, stream + *step), each 64 bits with the low word first.  It stays where
 * they are no less than t = p * 65536 rounded to nearest, and is then scaled by 65536 / (65536 - t), so that the
 * mean is kept exactly.  p below 2^-17 keeps all, p above 1 - 2^-17 drops all.
 * The mask is stored nowhere: a backward pass gives the same mask again.  A part of a
 * tensor has the tensor's mask if first is the number of its first element. */
typedef struct {
    double p;                    /* in [0, 1] */
    uint64_t seed;
    uint64_t stream;             /* the mask's own number: the layer, the step, the file */
    uint64_t first;
    const uint64_t *step;        /* device, or NULL for 0: added to stream when the kernel runs, so that a
                                    graph that counts it up has another mask each time */
} aspis_drop;

/* out = residual + keep * x * 65536 / (65536 - t), rounded once.  A dropped x counts as 0 whatever
 * it was.  The gradient of x is the same call on that of out.
 *   residual  of out's type, or NULL for none
 *   out       may be x (same address, type and ld) or residual
 * rows or cols 0: nothing is done.  ASPIS_E_RANGE (here and in aspis_embed): rows x ceil((cols + 7) / 248) beyond 2^31. */
aspis_status aspis_dropout(const void *x, int x_type, int64_t ldx, const void *residual, int64_t ldr,
                           void *out, int out_type, int64_t ldo, int64_t rows, int64_t cols,
                           const aspis_drop *drop, void *stream);

/* out[i] = drop( scale * table[token_i] ) for i < T.
 *   table  [V][width], ld_table apart
 *   drop   or NULL; element (i, j) of out has number first + i * width + j
 *   scale  finite; ASPIS_E_RANGE where drop leaves values and scale * 65536 / (65536 - t) is neither 0 nor a normal
 *          number of fp32 */
aspis_status aspis_embed(const void *table, int table_type, int64_t ld_table, int64_t V, const void *tokens,
                         int token_type, int64_t T, int64_t width, float scale, const aspis_drop *drop,
                         void *out, int out_type, int64_t ld_out, void *stream);

/* Device bytes that aspis_embed_grad needs for up to T tokens, V rows and that width; 0 where
 * the call would refuse them.  Host only. */
size_t aspis_embed_workspace_bytes(int64_t T, int64_t V, int64_t width);

/* table_grad[v] = scale * sum over i with token_i = v of drop( grad[i] ), in fp32 in an order that T, V, width
 * and the tokens alone fix, rounded once.  Tokens are sorted (stably) and each run of equal ones is summed in pieces.
 *   accumulate  0: all V rows are written, zeros where no token is
 *               1: table_grad + the sum replaces it, in the rows that tokens name; no other is touched
 *   scale, drop as in aspis_embed
 *   work        ASPIS_E_RANGE where work_bytes is too small
 * T, V < 2^31; T = 0 is allowed (grad, tokens and work may then be NULL). */
aspis_status aspis_embed_grad(const void *grad, int grad_type, int64_t ld_grad, const void *tokens,
                              int token_type, int64_t T, int64_t V, int64_t width, float scale,
                              const aspis_drop *drop, int accumulate, void *table_grad, int table_type,
                              int64_t ld_table, void *work, size_t work_bytes, void *stream);

/* logp[i] = a z_i[y_i] - log sum_j exp( a z_i[j] ), with the maximum taken out first; 0 for a
 * padding token.  logits [T][V], ld apart; a = logit_scale (1 / temperature), finite and > 0.
 * IEEE-754 through the formula: a logit of -infinity has probability 0, a row of nothing else, or with
 * a NaN or +infinity in it, gives NaN.  Never above 0, and exactly 0 (with a gradient of 0 in aspis_policy_loss) where all but
 * y_i have probability 0.  T = 0 is allowed. */
aspis_status aspis_token_logp(const void *logits, int type, int64_t ld, const void *tokens, int token_type,
                              int64_t T, int64_t V, float logit_scale, float *logp, void *stream);

typedef struct {
    const void *logits;          /* device [T][V], ld apart */
    void *grad;                  /* device [T][V] of the same type, ld_grad apart: d(loss * grad_scale) / d logits.
                                    May be logits (with the same ld).  NULL: none */
    const void *tokens;          /* device [T]: y */
    const float *old_logp;       /* device [T], or NULL: logp itself (the ratio is 1, and has a gradient) */
    const float *ref_logp;       /* device [T], or NULL: no KL term */
    const float *advantages;     /* device [T]: A */
    const float *weights;        /* device [T]: w, or NULL for 1.  Rows of weight 0 are not read: their logits
                                    may be anything; dz is 0 there, and so is logp */
    float *logp;                 /* device [T], out, or NULL */
    float *sums;                 /* device [4], out: the loss, its policy term, its KL term (without beta), and
                                    the clipped tokens, each sum_i scale w_i (...) */
    void *work;
    size_t work_bytes;
    int64_t T, V, ld, ld_grad;
    int32_t type, token_type;    /* aspis_dtype, aspis_itype */
    float logit_scale;           /* a, finite and > 0 */
    float clip_low, clip_high;   /* rho is clipped to [1 - clip_low, 1 + clip_high]; in [0, 1] and >= 0, high may be infinite */
    float kl_coef;               /* beta, finite and >= 0; 0: k is summed, and has no other part */
    float scale;                 /* finite: 1 / the tokens of the whole batch, not of this file alone */
    float grad_scale;            /* finite: a loss scale, which only dz is multiplied by.  With grad, ASPIS_E_RANGE where
                                    grad_scale * scale * logit_scale is neither 0 nor a normal number of fp32 */
} aspis_policy_args;

/* Device bytes that aspis_policy_loss needs for T tokens; 0 where T is out of range.  Host only. */
size_t aspis_policy_workspace_bytes(int64_t T);

/* The clipped policy loss with a KL term, and its gradient, in one pass over the logits:
 *     rho_i = exp(logp_i - old_i)
 *     L_i   = max( -A_i rho_i, -A_i min(max(rho_i, 1 - clip_low), 1 + clip_high) )    (0 where A_i is 0)
 *     k_i   = exp(ref_i - logp_i) - (ref_i - logp_i) - 1
 *     dz_i[j] = grad_scale scale w_i a s_i ( [j = y_i] - softmax(a z_i)[j] ),
 *     s_i   = ( -A_i rho_i where that is the maximum, else 0 ) + beta (1 - exp(ref_i - logp_i))
 * The same call gives the same bits each time; a row at another address modulo 32 may be summed in another
 * order (grad's place changes nothing).  T = 0 gives sums of 0. */
aspis_status aspis_policy_loss(const aspis_policy_args *args, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* ASPIS_WORKER_H */
