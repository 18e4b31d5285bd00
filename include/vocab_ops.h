/*
 * vocab_ops.h -- C ABI of the operators over the vocabulary for MI355X (gfx950): what stands at the two ends of a
 * model over words, beside lstm_stack.h and attn_softmax.h.
 *
 *   vocab_embed    x[n,:] = scale * table[ids[n],:], and the table's gradient
 *   vocab_xent     softmax cross-entropy of h W^T + b against word ids, and the gradients of h, W and b, without keeping
 *                  the logits: they are made a piece of the vocabulary at a time, in both passes
 *   vocab_distill  the same products with a teacher's top K logits per position as a second, soft target
 *   vocab_verify   which of the words that a small model drafted the large model's probabilities accept, and the word behind them
 *
 * Used together they make a language model of lstm_stack.h: ids -> vocab_embed_fwd -> lstm_stack_fwd -> vocab_xent_fwd,
 * vocab_xent_bwd -> lstm_stack_bwd -> vocab_embed_bwd; with a tied table (W = table, H = I) vocab_embed_bwd accumulates
 * onto dW.
 *
 * Conventions as in attn_softmax.h: every data pointer is DEVICE memory owned by the caller, dense row-major, 16-byte
 * aligned; calls only enqueue on hip_stream (NULL = default stream), on the calling thread's current device, which must be
 * the stream's; the library allocates nothing; calls that share a workspace must be ordered on one stream, and so must replays of
 * graphs captured with it; errors are returned as as_status codes (attn_softmax_last_error() has the message),
 * host-checkable faults before any launch.  Outputs are overwritten unless said otherwise, and no two arguments overlap.  Results do not
 * depend on the launch: the same call on the same inputs gives the same bits.
 *
 * dtype is the storage type of table, x, h, W and b: AS_F32 or AS_BF16 (which requires I % 8 == 0, H % 8 == 0).
 * grad_dtype is that of dy and of all gradients: AS_F32 always, or AS_BF16 where dtype is AS_BF16 too.  Sums are kept in
 * fp32 and rounded once on the way out.  Losses are float whatever the types.
 *   AS_F32 / AS_F32    fp32 products: operands as the sum of three bf16 terms, six products on the bf16 matrix cores
 *   AS_BF16 / AS_F32   the derivative of the logits as the sum of three bf16 terms, h and W as they are: fp32 products
 *   AS_BF16 / AS_BF16  the derivative of the logits as the sum of two bf16 terms (2^-17 of it; up to 16 positions and H <= 2048: fp32)
 *
 * Padding: a position whose id (target) equals pad_id or lies outside [0,V) is padding (pad_id = -1: only the latter).  Its row of
 * table, dy, h and of the teacher is not read (it may hold anything, NaN too), its output row is 0, and it contributes
 * nothing to losses, counts and gradients.
 */
#ifndef VOCAB_OPS_H
#define VOCAB_OPS_H

#include "attn_softmax.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef struct {
  int32_t N;          /* positions, 1 .. 2^24 */
  int32_t I;          /* width of the embedding, 1 .. 2^16 */
  int32_t V;          /* vocabulary, 1 .. 2^28; V * I < 2^40 */
  int32_t pad_id;     /* -1 <= pad_id < V */
  int32_t dtype;      /* as_dtype of table and x */
  int32_t grad_dtype; /* as_dtype of dy and d_table */
  float scale;        /* finite */
} vo_embed;

/* Bytes of workspace vocab_embed_bwd needs; 0 if the shape is invalid.  (The forward pass needs none.) */
size_t vocab_embed_workspace_bytes(const vo_embed* shape);

/* x [N,I] dtype = scale * table [V,I] dtype at ids [N] int32, rounded once; rows of 0 at padding. */
as_status vocab_embed_fwd(const vo_embed* shape, const void* table, const int32_t* ids, void* x, void* hip_stream);

/*
 * d_table [V,I] grad_dtype = scale * (sum of the rows of dy [N,I] grad_dtype per word), all V rows, zeros where no
 * position has the word.  accumulate (0 or 1): added to what d_table holds instead; rows of other words are then left as they are.
 * The positions are sorted by word and each word's rows added in a fixed order.
 */
as_status vocab_embed_bwd(const vo_embed* shape, const int32_t* ids, const void* dy, void* d_table, int accumulate,
                          void* workspace, size_t workspace_bytes, void* hip_stream);

typedef struct {
  int32_t N;          /* positions, 1 .. 2^24 */
  int32_t H;          /* width of h, 1 .. 2^16 */
  int32_t V;          /* vocabulary, 1 .. 2^26; V * H < 2^40 */
  int32_t pad_id;     /* -1 <= pad_id < V */
  int32_t dtype;      /* as_dtype of h, W and b */
  int32_t grad_dtype; /* as_dtype of dh, dW and db */
  float grad_scale;   /* g: gradients are those of g * loss_sum (+ s * distill_sum) */
} vo_shape;

/* A teacher's top logits.  Entries whose id lies outside [0,V) or whose logit is -inf are absent; an id may come twice. */
typedef struct {
  int32_t K;          /* entries per position, 1 .. 256; V <= 2^20 then */
  float temperature;  /* tau >= 2^-10 (fp32 logits over less have no digits left); tau^2 and s tau are finite */
  float scale;        /* s */
} vo_teacher;

/* Bytes of workspace the forward and backward pass need; 0 if the shape is invalid.  teacher: NULL for vocab_xent. */
size_t vocab_xent_workspace_bytes(const vo_shape* shape, const vo_teacher* teacher);

/*
 * Forward: l = h W^T + b, loss[n] = log sum_v exp l[n,v] - l[n,targets[n]].
 *   h [N,H] dtype   W [V,H] dtype   b [V] dtype or NULL (zeros)   targets [N] int32
 *   loss_sum [1] float   sum of the losses (not scaled by g)
 *   n_tok    [1] int32   number of positions that are not padding
 *   tok_loss [N] float   (optional) per position, 0 at padding
 *   argmax   [N] int32   (optional) lowest id attaining the row maximum of the fp32 logits; pad_id at padding
 * The workspace keeps what the backward pass needs (no logits): the rows of words of h, log-sum-exps.
 */
as_status vocab_xent_fwd(const vo_shape* shape, const void* h, const void* W, const void* b, const int32_t* targets,
                         float* loss_sum, int32_t* n_tok, float* tok_loss, int32_t* argmax,
                         void* workspace, size_t workspace_bytes, void* hip_stream);

/*
 * Backward of g * loss_sum: the W and b of the forward call and the workspace as that call left it (any number of
 * backward calls may follow one forward call) -> dh [N,H] (rows of 0 at padding), dW [V,H], db [V] (NULL if not wanted).
 */
as_status vocab_xent_bwd(const vo_shape* shape, const void* W, const void* b, void* workspace, size_t workspace_bytes,
                         void* dh, void* dW, void* db, void* hip_stream);

/*
 * Forward of both losses: the above, and per position that is not padding and has an entry at least
 *   p[k] = softmax over the position's entries of teacher_logits[n,k] / tau,  q = softmax over the vocabulary of l[n,:] / tau
 *   distill[n] = tau^2 * sum_k p[k] (log p[k] - log q[teacher_ids[n,k]])        (0 elsewhere)
 *   teacher_ids [N,K] int32   teacher_logits [N,K] float
 *   distill_sum [1] float   tok_distill [N] float (optional)
 */
as_status vocab_distill_fwd(const vo_shape* shape, const vo_teacher* teacher, const void* h, const void* W, const void* b,
                            const int32_t* targets, const int32_t* teacher_ids, const float* teacher_logits,
                            float* loss_sum, int32_t* n_tok, float* distill_sum, float* tok_loss, float* tok_distill,
                            void* workspace, size_t workspace_bytes, void* hip_stream);

/* Backward of g * loss_sum + s * distill_sum, as vocab_xent_bwd.  (g = 0: distillation alone.) */
as_status vocab_distill_bwd(const vo_shape* shape, const vo_teacher* teacher, const void* W, const void* b,
                            void* workspace, size_t workspace_bytes, void* dh, void* dW, void* db, void* hip_stream);

/*
 * Verification of drafted words (speculative sampling): with p[t] = softmax(target[b,t,:] / tau) and q[t] = softmax(draft[b,t,:] / tau),
 * the words drafted[b,t], t = 0, 1, .., are accepted as long as they lie in [0,V) and u_accept[b,t] q[t][word] < p[t][word].  Of n accepted
 * words the next one is drawn from p[n] where there is no word at n (n = T, or it lies outside [0,V): a shorter draft), and
 * from max(p[n] - q[n], 0) where that word was refused (from p[n] should this be 0 throughout): it is the lowest v whose weights up
 * to and including v add up to more than u_next[b] times all of them (the last v of a weight above 0, should rounding leave none).
 * If the drafted words were drawn from q, the words are distributed as if all were drawn from p.
 *   target [B,T+1,V] dtype, rows ld_target elements apart   draft [B,T,V] dtype, rows ld_draft apart (multiples of 16 bytes, >= V; what is
 *   between rows is not read into results)   drafted [B,T] int32   u_accept [B,T] float, u_next [B] float: uniform in [0,1)
 *   n_accepted [B] int32   words [B,T+1] int32: the accepted ones, the next one, -1 behind it
 * A logit of -inf has the probability 0.  A row that holds a NaN or +inf, or nothing but -inf, is no distribution: where one of them is
 * asked for, the words before are accepted and the next one is -1.  Probabilities and their sums are computed in 64 bits.
 */
typedef struct {
  int32_t B;          /* sequences, 1 .. 2^16 */
  int32_t T;          /* drafted words of each, 1 .. 64 */
  int32_t V;          /* vocabulary, 1 .. 2^20 */
  int32_t dtype;      /* as_dtype of the logits */
  float temperature;  /* tau, 2^-10 .. 2^10 */
} vo_verify;

/* Bytes of workspace vocab_verify needs; 0 if the shape is invalid. */
size_t vocab_verify_workspace_bytes(const vo_verify* shape);

as_status vocab_verify(const vo_verify* shape, const void* target, int64_t ld_target, const void* draft, int64_t ld_draft,
                       const int32_t* drafted, const float* u_accept, const float* u_next, int32_t* n_accepted, int32_t* words,
                       void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* VOCAB_OPS_H */
