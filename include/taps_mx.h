/*
 * taps_mx.h -- C ABI of the paged cache in microscaling formats
 * (libtaps_attention.so, beside taps_attention.h, whose conventions, plans and
 * errors hold here too).
 *
 * Keys and values held in 4 or 8 bits take 4.25 or 8.25 bits an element where
 * the 16-bit cache of taps_cache_append takes 16: sequences four or two times as
 * long fit, and single tokens, whose attention reads the cache and does little
 * else, wait for a quarter or half of the bytes.
 *
 *   1. taps_mx_append -- taps_cache_append into such a cache: keys normed and
 *      rotated on the way if asked for, keys and values rounded as they are written;
 *   2. taps_mx_read -- any slots read back to 16 or 32 bits;
 *   3. taps_mx_attend -- taps_attend over such a cache.
 *
 * The formats are those of the OCP Microscaling Formats (MX) specification 1.0
 * (blocks of 32 elements that share a power of two; elements of 4 bits, E2M1, or
 * of 8 bits, E4M3; scales of 8 bits, E8M0), with one rule for the scale:
 *   - Blocks are of 32 neighbouring elements of a head; the last one of a head
 *     whose size is no multiple of 32 is filled up with zeros.
 *   - a block's scale is 2^e, e the smallest integer from -110 on with
 *     a <= L 2^e; a is its largest magnitude, L = 7 (4 bits) or 464 (8 bits), the
 *     largest that is rounded to the format's largest number (6, 448) and not
 *     past it.  It is held as the byte e + 127.
 *   - an element x is held as the code nearest to x 2^-e, the even one of two.
 *     So it is off by at most 2^(e-2), 2^(e-1) or 2^e in 4 bits (below 2, from 2, from 4
 *     times 2^e) and by 2^-4 of itself or 2^(e-10) in 8.
 *   - a block with an infinite or NaN element has the byte 255 and zeros for
 *     codes, and is read as NaN.
 *   - Magnitudes that would be rounded past the largest number of the type that
 *     is appended are taken for 49152 (4 bits) or 61440 (8 bits) in TAPS_F16, 6 x 2^125
 *     or 15 x 2^124 in TAPS_BF16 and TAPS_F32.
 */
#ifndef TAPS_MX_H
#define TAPS_MX_H

#include "taps_attention.h"

#ifdef __cplusplus
extern "C" {
#endif

#define TAPS_MX_BLOCK 32
#define TAPS_MX_NAN 255u          /* scale of a block that is read as NaN */
#define TAPS_MX_BLOCKS(head_dim) (((head_dim) + 31u) / 32u)
/* bytes of a slot's codes for one head */
#define TAPS_MX_CODES(head_dim, bits) (TAPS_MX_BLOCKS(head_dim) * 4u * (bits))

/* Pages of keys, or of values: for key head h of slot j of page g, codes lie at
 * codes + g codes_stride[0] + h codes_stride[1] + j codes_stride[2], scales
 * likewise (strides in bytes).  A slot's codes are TAPS_MX_CODES(head_dim, bits)
 * bytes: element 2 i in the low half of byte i, 2 i + 1 in the high half (4 bits), or
 * element i in byte i; those beyond head_dim must be zeros.  Its scales are
 * TAPS_MX_BLOCKS(head_dim) bytes.  Codes start at multiples of 16 bytes (the data
 * and every stride of an axis longer than one); scales may start anywhere.  Slots
 * must be less than 2^27 bytes apart. */
typedef struct {
    void *codes;
    int64_t codes_stride[3];
    void *scales;
    int64_t scales_stride[3];
} taps_mx_pages;

/* taps_cache_append into pages of `bits` (4 or 8) bits: writes the new tokens'
 * codes, those that fill the last block up among them, and scales, and nothing
 * else.  args and plan as for taps_cache_append; head_dim a multiple of 8 up to
 * TAPS_MAX_ATTEND_DIM.  The norm's sum and root are taken in 64 bits and every
 * other step is rounded to 32, so that codes do not depend on the order of a sum:
 *   n_i = round(round(x_i rstd) weight_i),  (a, b) -> round(round(a cos) -+ round(b sin)). */
taps_status taps_mx_append(const taps_append_args *args, uint32_t bits, const void *plan,
                           const void *plan_device, const taps_heads *k, const taps_heads *v,
                           const taps_mx_pages *k_cache, const taps_mx_pages *v_cache,
                           void *stream);

/* What taps_mx_read reads. */
typedef struct {
    uint32_t dtype, bits;   /* dtype: of what is written */
    uint32_t tokens, kv_heads, head_dim;
    uint32_t page_size;     /* a power of two, as in a plan */
    uint32_t n_pages;
    uint32_t slot_bytes;    /* 4 or 8: type of slots */
    const void *slots;      /* device [tokens]: page * page_size + slot; the same one may be
                               asked for more than once */
} taps_mx_read_args;

/* Reads slots back: token t of k and v (stride[1]; stride[0] is not used) becomes the keys
 * and values of slots[t], rounded to dtype once.  A number that is no slot of the cache
 * makes its token NaN.  k and v overlap nothing. */
taps_status taps_mx_read(const taps_mx_read_args *args, const taps_mx_pages *k_cache,
                         const taps_mx_pages *v_cache, const taps_heads *k, const taps_heads *v,
                         void *stream);

/* taps_attend over pages of `bits` (4 or 8) bits, with its arguments, results and
 * conditions: out = softmax(scale q k^T) v with keys and values as taps_mx_read
 * gives them in dtype (those beyond its range are infinite).  Masked keys' codes and
 * scales may be anything. */
taps_status taps_mx_attend(uint32_t dtype, uint32_t bits, const void *plan, const void *plan_device,
                           const taps_heads *q, const taps_mx_pages *k_cache,
                           const taps_mx_pages *v_cache, float scale, const taps_heads *out,
                           float *lse, void *workspace, uint64_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif

#endif /* TAPS_MX_H */
