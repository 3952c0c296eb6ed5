// taps_mx_api.hip -- the C ABI of taps_mx.h: validation and launches.
#include <cmath>

#include "taps_attention_checks.h"
#include "taps_mx_internal.h"

using namespace taps_checks;

namespace {

taps_status check_format(uint32_t bits, uint32_t dim) {
    if (bits != 4 && bits != 8) return fail(TAPS_ERR_ARG, "bits %u is neither 4 nor 8", bits);
    if (dim < 8 || dim % 8 || dim > TAPS_MAX_ATTEND_DIM)
        return fail(TAPS_ERR_ARG, "head_dim %u is not a multiple of 8 up to %u", dim,
                    TAPS_MAX_ATTEND_DIM);
    return TAPS_OK;
}

// lengths: of the axes page, head and slot; one of a single step is not stepped along.
taps_status check_pages(const taps_mx_pages *t, const char *what, uint32_t pages, uint32_t heads,
                        taps_mx_place *to) {
    if (!t || !t->codes || !t->scales) return fail(TAPS_ERR_ARG, "%s is NULL", what);
    const uint32_t lengths[3] = {pages, heads, 2};
    bool fits = aligned(t->codes, 16);
    for (int i = 0; i < 3; ++i) fits = fits && (lengths[i] < 2 || t->codes_stride[i] % 16 == 0);
    if (!fits)
        return fail(TAPS_ERR_ARG, "%s: codes do not start at multiples of 16 bytes", what);
    // 16 slots' offsets are held in 32 bits
    for (const int64_t s : {t->codes_stride[2], t->scales_stride[2]})
        if (s < 0 || s >= (1 << 27))
            return fail(TAPS_ERR_ARG, "%s: slots are 2^27 bytes or more apart", what);
    to->codes = (char *)t->codes, to->scales = (char *)t->scales;
    for (int i = 0; i < 3; ++i)
        to->code_stride[i] = t->codes_stride[i], to->scale_stride[i] = t->scales_stride[i];
    return TAPS_OK;
}

// Whether every row of `heads` heads of `tokens` tokens starts at a multiple of eight elements.
bool by_eights(const taps_heads &t, uint32_t dtype, uint32_t tokens, uint32_t heads) {
    return aligned(t.data, 8 * size_of(dtype)) && (tokens < 2 || t.stride[1] % 8 == 0) &&
           (heads < 2 || t.stride[2] % 8 == 0);
}

// The largest magnitude that is appended: of the codes times powers of two below the
// type's range, as 4 bits (6 x 2^e) or 8 (240 x 2^e) have them.
float most_of(uint32_t dtype, uint32_t bits) {
    if (dtype == TAPS_F16) return bits == 4 ? 49152.f : 61440.f;
    return bits == 4 ? 0x1.8p127f : 0x1.ep127f;
}

}  // namespace

extern "C" {

taps_status taps_mx_append(const taps_append_args *a, uint32_t bits, const void *plan,
                           const void *plan_device, const taps_heads *k, const taps_heads *v,
                           const taps_mx_pages *k_cache, const taps_mx_pages *v_cache,
                           void *stream) {
    if (!a) return fail(TAPS_ERR_ARG, "args is NULL");
    const taps_plan_header *h;
    if (taps_status st = check_plan(plan, plan_device, &h)) return st;
    if (taps_status st = check_format(bits, h->head_dim)) return st;
    if (taps_status st = check_types(a->dtype, a->weight_dtype, h->head_dim, a->rotary_dim, a->eps,
                                     a->table))
        return st;
    if (!aligned(a->k_weight, size_of(a->weight_dtype)))
        return fail(TAPS_ERR_ARG, "k_weight is not aligned to its elements");
    if (!h->appendable)
        return fail(TAPS_ERR_ARG, "a sequence of the plan has more new tokens than keys");
    if (a->rotary_dim && h->max_positions > a->n_positions)
        return fail(TAPS_ERR_ARG, "positions up to %u exceed the table's %u", h->max_positions,
                    a->n_positions);
    if (!h->tokens) return TAPS_OK;
    taps_mx_append_launch p{};
    const taps_heads *const src[2] = {k, v};
    const taps_mx_pages *const dst[2] = {k_cache, v_cache};
    static const char *const names[2][2] = {{"k", "k_cache"}, {"v", "v_cache"}};
    bool vectors = vectors_fit(h->head_dim, a->rotary_dim, a->weight_dtype, a->k_weight, nullptr,
                               a->table);
    for (int side = 0; side < 2; ++side) {
        if (taps_status st = check_heads(src[side], names[side][0], a->dtype)) return st;
        if (taps_status st = check_pages(dst[side], names[side][1], h->n_pages, h->kv_heads,
                                         &p.cache[side]))
            return st;
        p.src[side] = src[side]->data;
        p.src_stride[side][0] = src[side]->stride[1], p.src_stride[side][1] = src[side]->stride[2];
        vectors = vectors && by_eights(*src[side], a->dtype, h->tokens, h->kv_heads);
    }
    p.plan_tokens = (const taps_plan_token *)((const char *)plan_device + h->tokens_at);
    p.weight = a->k_weight, p.float_weight = a->weight_dtype == TAPS_F32;
    p.table = a->table;
    p.tokens = h->tokens, p.heads = h->kv_heads;
    p.dim = h->head_dim, p.rotary = a->rotary_dim;
    p.inverse_dim = 1.0 / h->head_dim;
    p.page_log2 = h->page_log2;
    p.eps = a->eps, p.most = most_of(a->dtype, bits);
    p.interleaved = a->interleaved != 0;
    return launched(taps_launch_mx_append(p, a->dtype, bits, vectors, (hipStream_t)stream),
                    "taps_mx_append");
}

taps_status taps_mx_read(const taps_mx_read_args *a, const taps_mx_pages *k_cache,
                         const taps_mx_pages *v_cache, const taps_heads *k, const taps_heads *v,
                         void *stream) {
    if (!a) return fail(TAPS_ERR_ARG, "args is NULL");
    if (a->dtype > TAPS_F32) return fail(TAPS_ERR_ARG, "dtype %u is none", a->dtype);
    if (taps_status st = check_format(a->bits, a->head_dim)) return st;
    if (a->page_size < TAPS_MIN_PAGE || a->page_size > TAPS_MAX_PAGE ||
        (a->page_size & (a->page_size - 1)))
        return fail(TAPS_ERR_ARG, "page_size %u is not a power of two in %u..%u", a->page_size,
                    TAPS_MIN_PAGE, TAPS_MAX_PAGE);
    if (!a->kv_heads || a->kv_heads > 65535)
        return fail(TAPS_ERR_ARG, "kv_heads %u outside 1..65535", a->kv_heads);
    if (a->tokens >= (1u << 31)) return fail(TAPS_ERR_ARG, "%u tokens are too many", a->tokens);
    if (a->slot_bytes != 4 && a->slot_bytes != 8)
        return fail(TAPS_ERR_ARG, "slot_bytes %u is neither 4 nor 8", a->slot_bytes);
    if (!a->tokens) return TAPS_OK;
    if (!a->slots) return fail(TAPS_ERR_ARG, "slots is NULL");
    if (!aligned(a->slots, a->slot_bytes))
        return fail(TAPS_ERR_ARG, "slots is not aligned to its elements");
    // the kernels read slot 0 for a number that is none
    if (!a->n_pages) return fail(TAPS_ERR_ARG, "the cache has no pages");
    taps_mx_read_launch p{};
    const taps_mx_pages *const src[2] = {k_cache, v_cache};
    const taps_heads *const dst[2] = {k, v};
    static const char *const names[2][2] = {{"k_cache", "k"}, {"v_cache", "v"}};
    bool vectors = true;
    for (int side = 0; side < 2; ++side) {
        if (taps_status st = check_pages(src[side], names[side][0], a->n_pages, a->kv_heads,
                                         &p.cache[side]))
            return st;
        if (taps_status st = check_heads(dst[side], names[side][1], a->dtype)) return st;
        p.dst[side] = dst[side]->data;
        p.dst_stride[side][0] = dst[side]->stride[1], p.dst_stride[side][1] = dst[side]->stride[2];
        vectors = vectors && by_eights(*dst[side], a->dtype, a->tokens, a->kv_heads);
    }
    p.slots = a->slots, p.wide_slots = a->slot_bytes == 8;
    p.page_log2 = (uint32_t)__builtin_ctz(a->page_size);
    p.n_slots = (int64_t)a->n_pages << p.page_log2;
    p.tokens = a->tokens, p.heads = a->kv_heads, p.dim = a->head_dim;
    return launched(taps_launch_mx_read(p, a->dtype, a->bits, vectors, (hipStream_t)stream),
                    "taps_mx_read");
}

taps_status taps_mx_attend(uint32_t dtype, uint32_t bits, const void *plan, const void *plan_device,
                           const taps_heads *q, const taps_mx_pages *k_cache,
                           const taps_mx_pages *v_cache, float scale, const taps_heads *out,
                           float *lse, void *workspace, uint64_t workspace_bytes, void *stream) {
    taps_mx_attend_launch p{};
    const taps_plan_header *h;
    if (taps_status st = check_attend(dtype, plan, plan_device, scale, &h)) return st;
    if (taps_status st = check_format(bits, h->head_dim)) return st;
    if (!h->tokens) return TAPS_OK;
    if (taps_status st = check_rows(q, "q", h->tokens, h->q_heads)) return st;
    taps_mx_place k, v;
    if (taps_status st = check_pages(k_cache, "k_cache", h->n_pages, h->kv_heads, &k)) return st;
    if (taps_status st = check_pages(v_cache, "v_cache", h->n_pages, h->kv_heads, &v)) return st;
    if (taps_status st = check_rows(out, "out", h->tokens, h->q_heads)) return st;
    if (taps_status st = check_results(*h, lse, workspace, workspace_bytes)) return st;
    set_attend(&p, *h, plan_device, *q, scale, *out, lse, workspace);
    p.k_cache = k.codes, p.v_cache = v.codes;
    p.k_page = k.code_stride[0], p.k_head = k.code_stride[1], p.k_slot = k.code_stride[2];
    p.v_page = v.code_stride[0], p.v_head = v.code_stride[1], p.v_slot = v.code_stride[2];
    p.k_scales = k.scales, p.v_scales = v.scales;
    p.ks_page = k.scale_stride[0], p.ks_head = k.scale_stride[1], p.ks_slot = k.scale_stride[2];
    p.vs_page = v.scale_stride[0], p.vs_head = v.scale_stride[1], p.vs_slot = v.scale_stride[2];
    return launched(taps_launch_mx_attend(p, dtype, bits, (hipStream_t)stream), "taps_mx_attend");
}

}  // extern "C"
