// taps_attention_checks.h -- what the C ABIs of libtaps_attention.so share on the
// host: the last error and checks of arguments.
#pragma once
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "taps_attention_internal.h"

namespace taps_checks {

inline thread_local char g_last_error[512] = "";

inline taps_status fail(taps_status st, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_last_error, sizeof g_last_error, fmt, ap);
    va_end(ap);
    return st;
}

inline taps_status launched(hipError_t err, const char *what) {
    if (err == hipSuccess) return TAPS_OK;
    return fail(TAPS_ERR_DEVICE, "%s: %s", what, hipGetErrorString(err));
}

inline uint32_t size_of(uint32_t dtype) { return dtype == TAPS_F32 ? 4 : 2; }

inline bool aligned(const void *p, uint64_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

inline taps_status check_types(uint32_t dtype, uint32_t weight_dtype, uint32_t dim, uint32_t rotary,
                               float eps, const float *table) {
    if (dtype > TAPS_F32) return fail(TAPS_ERR_ARG, "dtype %u is none", dtype);
    if (weight_dtype != dtype && weight_dtype != TAPS_F32)
        return fail(TAPS_ERR_ARG, "weight_dtype %u is neither dtype (%u) nor TAPS_F32", weight_dtype,
                    dtype);
    if (dim < 1 || dim > TAPS_MAX_HEAD_DIM)
        return fail(TAPS_ERR_ARG, "head_dim %u outside 1..%u", dim, TAPS_MAX_HEAD_DIM);
    if (rotary > dim || rotary % 2)
        return fail(TAPS_ERR_ARG, "rotary_dim %u is odd or above head_dim %u", rotary, dim);
    if (rotary && !table) return fail(TAPS_ERR_ARG, "rotary_dim is %u but table is NULL", rotary);
    if (!aligned(table, 4)) return fail(TAPS_ERR_ARG, "table is not aligned to its elements");
    if (!(eps >= 0.f) || std::isinf(eps)) return fail(TAPS_ERR_ARG, "eps is negative or not finite");
    return TAPS_OK;
}

inline taps_status check_heads(const taps_heads *t, const char *what, uint32_t dtype) {
    if (!t || !t->data) return fail(TAPS_ERR_ARG, "%s is NULL", what);
    if (!aligned(t->data, size_of(dtype)))
        return fail(TAPS_ERR_ARG, "%s is not aligned to its elements", what);
    return TAPS_OK;
}

// Whether every row starts at a multiple of four elements.
inline bool by_fours(const taps_heads &t, uint32_t dtype) {
    return aligned(t.data, 4 * size_of(dtype)) && t.stride[0] % 4 == 0 && t.stride[1] % 4 == 0 &&
           t.stride[2] % 4 == 0;
}

inline bool vectors_fit(uint32_t dim, uint32_t rotary, uint32_t weight_dtype, const void *w0,
                        const void *w1, const float *table) {
    const uint32_t w = 4 * size_of(weight_dtype);
    return dim % 8 == 0 && rotary % 8 == 0 && aligned(w0, w) && aligned(w1, w) && aligned(table, 16);
}

inline void set_strides(int64_t (&to)[3], const taps_heads &t) {
    for (int i = 0; i < 3; ++i) to[i] = t.stride[i];
}

inline uint64_t up16(uint64_t v) { return (v + 15) & ~15ull; }

inline uint64_t workspace_of(const taps_plan_header &h) {
    return up16((uint64_t)h.part_rows * h.kv_heads * h.head_dim * 4) +
           up16((uint64_t)h.part_rows * h.kv_heads * 8);
}

inline taps_status check_plan(const void *plan, const void *plan_device, const taps_plan_header **h) {
    if (!plan || !plan_device) return fail(TAPS_ERR_ARG, "plan or plan_device is NULL");
    if (!aligned(plan, 16) || !aligned(plan_device, 16))
        return fail(TAPS_ERR_ARG, "plan or plan_device is not 16-byte aligned");
    *h = (const taps_plan_header *)plan;
    if ((*h)->magic != kPlanMagic) return fail(TAPS_ERR_ARG, "plan was not made by taps_paged_plan");
    return TAPS_OK;
}

// Attention over either cache: types and the plan.
inline taps_status check_attend(uint32_t dtype, const void *plan, const void *plan_device, float scale,
                                const taps_plan_header **h) {
    if (dtype != TAPS_BF16 && dtype != TAPS_F16)
        return fail(TAPS_ERR_ARG, "dtype %u is neither TAPS_BF16 nor TAPS_F16", dtype);
    if (taps_status st = check_plan(plan, plan_device, h)) return st;
    if ((*h)->head_dim % 8 || (*h)->head_dim > TAPS_MAX_ATTEND_DIM)
        return fail(TAPS_ERR_ARG, "head_dim %u is not a multiple of 8 up to %u", (*h)->head_dim,
                    TAPS_MAX_ATTEND_DIM);
    if (!(scale > 0.f) || std::isinf(scale))
        return fail(TAPS_ERR_ARG, "scale is not positive and finite");
    return TAPS_OK;
}

// Rows of 16-bit elements start at multiples of 16 bytes; the lengths are those of the axes
// that stride[1], [2] and [0] step along.
inline taps_status check_rows(const taps_heads *t, const char *what, uint32_t length1,
                              uint32_t length2, uint32_t length0 = 1) {
    if (!t || !t->data) return fail(TAPS_ERR_ARG, "%s is NULL", what);
    // an axis of one is not stepped along
    const uint32_t lengths[3] = {length0, length1, length2};
    bool fits = aligned(t->data, 16);
    for (int k = 0; k < 3; ++k) fits = fits && (lengths[k] < 2 || t->stride[k] % 8 == 0);
    if (!fits) return fail(TAPS_ERR_ARG, "%s: rows do not start at multiples of 16 bytes", what);
    return TAPS_OK;
}

inline taps_status check_results(const taps_plan_header &h, const float *lse, const void *workspace,
                                 uint64_t workspace_bytes) {
    if (!aligned(lse, 4)) return fail(TAPS_ERR_ARG, "lse is not aligned to its elements");
    const uint64_t need = workspace_of(h);
    if (need && !workspace) return fail(TAPS_ERR_ARG, "workspace is NULL");
    if (need > workspace_bytes)
        return fail(TAPS_ERR_CAPACITY, "workspace of %llu bytes, %llu are needed",
                    (unsigned long long)workspace_bytes, (unsigned long long)need);
    if (!aligned(workspace, 16)) return fail(TAPS_ERR_ARG, "workspace is not 16-byte aligned");
    return TAPS_OK;
}

// All of a launch of attention but its cache.
inline void set_attend(taps_attend_launch *p, const taps_plan_header &h, const void *plan_device,
                       const taps_heads &q, float scale, const taps_heads &out, float *lse,
                       void *workspace) {
    const char *dev = (const char *)plan_device;
    p->q = (const char *)q.data, p->out = (char *)out.data, p->lse = lse;
    p->zeros = dev + offsetof(taps_plan_header, zeros);
    p->part_o = (float *)workspace;
    p->part_ml = (float *)((char *)workspace +
                           up16((uint64_t)h.part_rows * h.kv_heads * h.head_dim * 4));
    p->pages = (const int32_t *)(dev + h.pages_at);
    p->items = (const taps_plan_item *)(dev + h.items_at);
    p->joins = (const taps_plan_join *)(dev + h.joins_at);
    p->q_token = 2 * q.stride[1], p->q_head = 2 * q.stride[2];
    p->o_token = 2 * out.stride[1], p->o_head = 2 * out.stride[2];
    p->n_items = h.n_items, p->n_wide = h.n_wide, p->n_few = h.n_few;
    p->n_joins = h.n_joins, p->join_rounds = h.join_rounds;
    p->q_heads = h.q_heads, p->kv_heads = h.kv_heads, p->group = h.q_heads / h.kv_heads;
    p->dim = h.head_dim;
    p->page_log2 = h.page_log2, p->causal = h.causal, p->window = h.window;
    p->scale = scale;
}

}  // namespace taps_checks
