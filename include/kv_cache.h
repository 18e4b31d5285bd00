/*
 * kv_cache.h -- C ABI of a paged cache of keys and values and of the attention that reads it, for MI355X (gfx950): the serving
 * form of a model that looks back at what it has written so far, one or a few tokens of each sequence at a time.
 *
 *   kv_cache_write  keys and values of new tokens into the pages of their sequences, as they are or in 8 bits
 *   kv_cache_read   places of the cache back as dense rows
 *   kv_cache_attn   attention of each sequence's newest T tokens over its cached ones
 *
 * Where attn_softmax.h's per-step mode attends to a block of states that is the same for a whole batch, here sequences of any length
 * come and go: each holds pages of a common pool, named by its row of a table.  Pages may be shared (a common beginning).
 * Drafted words (vocab_verify in vocab_ops.h) are written and attended to like any others, T of them at once; those that are not
 * accepted leave by counting the sequence's length back.
 *
 * Conventions as in attn_softmax.h: every data pointer is DEVICE memory owned by the caller, 16-byte aligned; calls only enqueue
 * on hip_stream (NULL = default stream), on the calling thread's current device, which must be the stream's; the library
 * allocates nothing; calls that share a workspace must be ordered on one stream, and so must replays of graphs captured with it;
 * errors are returned as as_status codes (attn_softmax_last_error() has the message), host-checkable faults before any launch.
 * Outputs are overwritten, and an output overlaps no other argument.  Results do not depend on the launch: the same call on the
 * same inputs gives the same bits.
 *
 * The pool, for keys and for values: pages [pages, heads, page, D] of cache_type, and in 8 bits scales [pages, heads, page] float.
 * Token `pos` of sequence b lies in page page_table[b, pos / page] at place pos % page.  A page outside [0, pages) is no page: what
 * would lie there is not written, reads as 0, and is not attended to.
 *
 * 8 bits: each token's row of each head has a scale s = max(max |x| * (1 / Q), 2^-120), Q = 127 (KC_INT8) or 448 (KC_E4M3), and
 * holds the codes x * (1 / s), the float product rounded to the nearest code, ties to even; it stands for code * s.  (All
 * steps in fp32, 1 / Q among them.)  The error is at most half a code and a few roundings of fp32: max |x| / 254, or 2^-4 of
 * the value above max |x| 2^-15.  A row that holds an infinity or a NaN has the scale NaN and reads as NaN.
 */
#ifndef KV_CACHE_H
#define KV_CACHE_H

#include "attn_softmax.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  KC_F32 = 0,   /* = AS_F32  */
  KC_BF16 = 1,  /* = AS_BF16 */
  KC_INT8 = 2,
  KC_E4M3 = 3   /* 8-bit float with 4 bits of exponent, largest value 448 */
} kc_type;

typedef struct {
  int32_t pages;      /* of the pool, >= 1; pages * page < 2^31 */
  int32_t page;       /* tokens of a page: a multiple of 16, 16 .. 4096 */
  int32_t heads;      /* of keys and values, 1 .. 1024 */
  int32_t D;          /* width of a head: a multiple of 16, 16 .. 256 */
  int32_t dtype;      /* as_dtype of k, v, q and out */
  int32_t cache_type; /* kc_type: dtype's, KC_INT8 or KC_E4M3 */
  int32_t B;          /* sequences, 1 .. 2^16 */
  int32_t max_pages;  /* columns of page_table [B, max_pages] int32, >= 1; B * max_pages < 2^31 */
} kc_cache;

/*
 * Rows n of k and v [N, heads, D] dtype, ld_k and ld_v elements apart (at least heads * D, a multiple of 16 bytes), to token pos[n] of sequence
 * seq[n].  Rows whose seq lies outside [0,B), whose pos lies outside [0, max_pages * page) or whose page is none are not
 * written, and their k and v play no part (they may hold anything).  The places of a call differ: of rows with the same one any may be
 * left, in parts.  k_scales, v_scales: in 8 bits only (else NULL).  N in 1 .. 2^24.
 * k_pages and v_pages differ here.
 */
as_status kv_cache_write(const kc_cache* cache, int32_t N, const void* k, int64_t ld_k, const void* v, int64_t ld_v,
                         const int32_t* seq, const int32_t* pos, const int32_t* page_table,
                         void* k_pages, void* v_pages, float* k_scales, float* v_scales, void* hip_stream);

/* k and v [N, heads, D] dtype, dense: what the cache stands for at token pos[n] of sequence seq[n], rounded once; rows of 0 where
 * kv_cache_write would not write. */
as_status kv_cache_read(const kc_cache* cache, int32_t N, const void* k_pages, const void* v_pages, const float* k_scales,
                        const float* v_scales, const int32_t* seq, const int32_t* pos, const int32_t* page_table,
                        void* k, void* v, void* hip_stream);

typedef struct {
  int32_t T;        /* new tokens of each sequence, 1 .. 64: one for decoding, drafted ones and one for verification */
  int32_t q_heads;  /* heads of queries, a multiple of the cache's; head i reads head i / (q_heads / heads); T * q_heads / heads <= 1024 */
  int32_t max_len;  /* no sequence is longer, 1 .. max_pages * page and below 2^28: lengths are clamped to [0, max_len] */
  int32_t window;   /* > 0: a token sees itself and the window - 1 ahead of it; 0: all */
  float scale;      /* of the products q . k; finite, and 1.45 times it too */
} kc_attn;

/* Bytes of workspace kv_cache_attn needs (it may need none: then 16); 0 if the shape is invalid.  B * heads * ceil(T q_heads / heads / 64)
 * is at most 2^22, and less than 2^30 times that with max_len / 16 + 1. */
size_t kv_cache_attn_workspace_bytes(const kc_cache* cache, const kc_attn* attn);

/*
 * The newest T tokens of each sequence, whose keys and values the cache holds already: token t of sequence b has the position
 * lengths[b] - T + t, sees cached tokens up to and including it, and
 *   a[i] = scale * q . k[i],  out = sum_i softmax(a)[i] v[i],  lse = log sum_i exp a[i]   over the tokens i that it sees.
 *   q   [B, T, q_heads, D] dtype, rows b T + t being ld_q elements apart (at least q_heads * D, a multiple of 16 bytes)
 *   out [B, T, q_heads, D] dtype, dense     lse [B, T, q_heads] float (optional)
 * A token that sees none (its position is negative: the sequence has fewer than T tokens; or all of its pages are none) gives 0 and -inf.
 * Tokens that are not seen, and what lies behind a sequence's end in its last page, may hold anything.  What a seen value's
 * infinity makes of its column of out is unspecified (an infinity or NaN).  k_pages and v_pages may be the same.
 * Scores may be of any size: q . k, in 8 bits of q and the codes, has to lie within 2^126 of zero (sums, and differences of sums, are fp32).
 * Sums are divided by the sum of their weights at the end, and weights go up to 2^8: values above 2^120 divided by the number of tokens may
 * leave fp32's range on the way and give infinities.
 * Products and sums are fp32 or better: fp32 caches on the fp32 matrix instructions; bf16 and 8-bit codes, which bf16 holds, with
 * the probabilities as two (dtype AS_BF16) or three bf16 terms and fp32 queries as three.
 */
as_status kv_cache_attn(const kc_cache* cache, const kc_attn* attn, const void* q, int64_t ld_q,
                        const void* k_pages, const void* v_pages, const float* k_scales, const float* v_scales,
                        const int32_t* page_table, const int32_t* lengths, void* out, float* lse,
                        void* workspace, size_t workspace_bytes, void* hip_stream);

#ifdef __cplusplus
}
#endif
#endif /* KV_CACHE_H */
