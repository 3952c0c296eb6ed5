/*
 * taps_attention.h -- C ABI of the operators that run one device's share of
 * an attention block (libtaps_attention.so, built beside libtaps.so).
 *
 * A strategy that splits the batch, head and query axes of the projection,
 * score, softmax and context operators leaves each device with some of the
 * heads and a chunk of the tokens.  These calls run that share:
 *
 *   1. taps_norm_rotate, taps_norm_rotate_backward -- the RMS norm of every
 *      query and key head and the rotation by the token's position, in one
 *      pass, and their gradients;
 *   2. taps_cache_append -- the new tokens' keys (normed and rotated on the
 *      way if asked for) and values into a paged cache;
 *   3. taps_attend -- attention of the new tokens over that cache: prompts,
 *      chunks of a prompt and single tokens, in one call.
 *
 * Conventions
 *   - A tensor of heads (taps_heads) is device memory with element (b, t, h, i)
 *     at data + b stride[0] + t stride[1] + h stride[2] + i, in elements: rows
 *     of head_dim elements are contiguous, everything else has a stride.
 *   - Sums, norms, scores and softmax statistics are held in 32 bits; outputs
 *     are rounded once to the tensors' type.  Attention rounds the softmax
 *     numerators to the cache's type for the product with the values.
 *   - A rotation table is device memory float [n_positions][2][rotary_dim / 2]:
 *     per position the cosines and the sines of its angles.
 *   - The rotated pairs of a head are (i, i + rotary_dim / 2), or with
 *     interleaved (2 i, 2 i + 1), i < rotary_dim / 2: (a, b) becomes
 *     (a cos - b sin, b cos + a sin).  Elements from rotary_dim on stay.
 *   - A paged cache is two tensors of n_pages pages: key head h of slot j of
 *     page g is the head_dim elements at data + g stride[0] + h stride[1] +
 *     j stride[2] (taps_heads with that meaning of its strides).
 *   - Work is asynchronous on `stream` (a hipStream_t, NULL = the null
 *     stream); no call allocates, synchronises or keeps a pointer.  Calls can
 *     be captured into a HIP graph.  Results do not depend on the order in
 *     which workgroups run.
 *   - Errors are those of taps.h: arguments are validated before any GPU work
 *     and nothing is written on a validation error;
 *     taps_attention_last_error() describes the calling thread's last failure.
 */
#ifndef TAPS_ATTENTION_H
#define TAPS_ATTENTION_H

#include "taps.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TAPS_BF16 0
#define TAPS_F16 1
#define TAPS_F32 2

#define TAPS_MAX_HEAD_DIM 256   /* norm_rotate, cache_append */
#define TAPS_MAX_ATTEND_DIM 128 /* attend: a multiple of 8 up to this */
/* taps_norm_rotate_backward never needs more bytes of workspace */
#define TAPS_NORM_ROTATE_WORKSPACE(head_dim) (8192u * (head_dim))
#define TAPS_MIN_PAGE 16        /* slots of a page: a power of two, 16 .. 4096 */
#define TAPS_MAX_PAGE 4096

/* Tensor of heads: see the conventions. */
typedef struct {
    void *data;
    int64_t stride[3];
} taps_heads;

/* What taps_norm_rotate does to which shapes. */
typedef struct {
    uint32_t batch, tokens, q_heads, k_heads; /* k_heads 0: queries only */
    uint32_t head_dim;                        /* 1 .. TAPS_MAX_HEAD_DIM */
    uint32_t rotary_dim;                      /* even, 0 .. head_dim */
    uint32_t dtype;                           /* of q, k, the outputs and gradients */
    uint32_t weight_dtype;                    /* of the weights: dtype or TAPS_F32 */
    uint32_t interleaved;
    float eps;
    const void *q_weight, *k_weight; /* device [head_dim]; NULL: that side is only rotated */
    const float *table;              /* device; may be NULL if rotary_dim is 0 */
    uint32_t n_positions;            /* rows of the table */
    uint32_t position_bytes;         /* 4 or 8: type of positions */
    const void *positions;           /* device [batch][tokens] integers, or NULL: token t of
                                        every sequence is at first_position + t */
    int64_t first_position;
} taps_norm_rotate_args;

/* q_out = rotate(norm(q)), k_out = rotate(norm(k)), with
 *   norm(x)_i = x_i (mean_j x_j^2 + eps)^(-1/2) weight_i.
 * k and k_out are not looked at (and may be NULL) if k_heads is 0.
 * q_out may be q and k_out k (the same data and strides); otherwise outputs
 * overlap nothing.  first_position .. first_position + tokens - 1 must be
 * rows of the table (TAPS_ERR_ARG); a value of `positions` that is not one
 * makes that token's outputs NaN (in the gradients: those of its inputs and
 * of the weights); a table without rows is refused (TAPS_ERR_ARG). */
taps_status taps_norm_rotate(const taps_norm_rotate_args *args, const taps_heads *q,
                             const taps_heads *k, const taps_heads *q_out, const taps_heads *k_out,
                             void *stream);

/* The gradients of taps_norm_rotate: from those of its outputs (dq_out,
 * dk_out) and its inputs (q, k) to those of its inputs (dq, dk) and weights
 * (device [head_dim] in weight_dtype, each NULL exactly if the weight is).
 * dq may be dq_out and dk dk_out.  The weights' gradients are sums over all
 * rows, held in 32 bits and added in an order that only the sizes determine.
 * `workspace` (device, 16-byte aligned) holds partial sums; with workspace
 * NULL the call only writes the bytes it needs to *workspace_bytes, otherwise
 * *workspace_bytes says how many there are (TAPS_ERR_CAPACITY if too few). */
taps_status taps_norm_rotate_backward(const taps_norm_rotate_args *args, const taps_heads *dq_out,
                                      const taps_heads *dk_out, const taps_heads *q,
                                      const taps_heads *k, const taps_heads *dq,
                                      const taps_heads *dk, void *q_weight_grad,
                                      void *k_weight_grad, void *workspace,
                                      uint64_t *workspace_bytes, void *stream);

/* The sequences of one step.  After the append of its q_lens[s] new tokens,
 * sequence s has kv_lens[s] keys; key j is in page
 * pages[s * pages_stride + j / page_size], slot j % page_size.  New token i is
 * at position kv_lens[s] - q_lens[s] + i.  The new tokens of all sequences
 * lie one after the other in the tensors of heads (their stride[1]; stride[0]
 * is not used). */
typedef struct {
    uint32_t n_seqs, page_size, n_pages, pages_stride;
    const int32_t *q_lens, *kv_lens; /* host [n_seqs], >= 0 */
    const int32_t *kv_starts;        /* host [n_seqs] or NULL (zeros), 0 .. kv_lens: keys before
                                        it are gone or were never there (padding): nothing sees
                                        them, none is appended, their pages may be anything */
    const int32_t *pages;            /* host [n_seqs][pages_stride] */
    uint32_t q_heads, kv_heads;      /* q_heads a multiple of kv_heads */
    uint32_t head_dim;
    uint32_t causal;                 /* a token sees keys up to its own position, else all */
    uint32_t window;                 /* causal: only the last `window` of those; 0: all */
} taps_paged_batch;

/* Lays a step out for taps_cache_append and taps_attend: every token's slot,
 * and the work of attention cut into pieces of like size for `cus` compute
 * units (0: 256).  A plan serves every layer of the step and any cache with
 * its page size, at least its pages and its heads.  `plan` is host memory,
 * 16-byte aligned, of *plan_bytes bytes (NULL: only the needed size is
 * written); the caller copies it to the device and passes both copies on,
 * unchanged.  *workspace_bytes is what taps_attend needs.  TAPS_ERR_ARG also
 * for a page number outside 0 .. n_pages - 1 where a key is or is to be
 * written, for lengths above 2^30, 2^31 or more tokens or slots in all, and if
 * a page is to be written from two places of the page table.
 * A sequence with kv_lens < q_lens can be attended (tokens at negative
 * positions see nothing), not appended. */
taps_status taps_paged_plan(const taps_paged_batch *batch, uint32_t cus, void *plan,
                            uint64_t *plan_bytes, uint64_t *workspace_bytes);

/* Norm and rotation of appended keys. */
typedef struct {
    uint32_t dtype, weight_dtype, rotary_dim, interleaved;
    float eps;
    const void *k_weight; /* device [head_dim]; NULL: no norm */
    const float *table;   /* device; rows for every new token's position */
    uint32_t n_positions;
} taps_append_args;

/* Writes the new tokens' keys, rotate(norm(k)) as in taps_norm_rotate, and
 * values into the cache.  TAPS_ERR_ARG if a token's position is not a row of the
 * table or the plan has a sequence with kv_lens < q_lens. */
taps_status taps_cache_append(const taps_append_args *args, const void *plan,
                              const void *plan_device, const taps_heads *k, const taps_heads *v,
                              const taps_heads *k_cache, const taps_heads *v_cache,
                              void *stream);

/* out = softmax(scale q k^T) v over the keys each token sees; query head h
 * reads key head h / (q_heads / kv_heads).  A token that sees no key gets
 * zeros, and -inf in lse; one that sees only keys with scores of -inf gets NaN in both.
 *   dtype  TAPS_BF16 or TAPS_F16, of q, the cache and out.
 *   scale  positive and finite.
 *   lse    device float [tokens][q_heads] or NULL: log of the sum of
 *          exp(scale q k) of every token and head.
 *   workspace  device, 16-byte aligned, workspace_bytes as the plan said.
 * Every data pointer must be 16-byte aligned and every stride of an axis longer
 * than one a multiple of 8; a cache's slots must be less than 2^26 elements apart. */
taps_status taps_attend(uint32_t dtype, const void *plan, const void *plan_device,
                        const taps_heads *q, const taps_heads *k_cache, const taps_heads *v_cache,
                        float scale, const taps_heads *out, float *lse, void *workspace,
                        uint64_t workspace_bytes, void *stream);

/* Description of the calling thread's last failure ("" if none). */
const char *taps_attention_last_error(void);

#ifdef __cplusplus
}
#endif

#endif /* TAPS_ATTENTION_H */
