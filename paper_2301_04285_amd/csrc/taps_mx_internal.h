// taps_mx_internal.h -- launch parameters of the cache in microscaling formats.
#pragma once
#include "taps_attention_internal.h"
#include "taps_mx.h"

// Where the codes and scales of one tensor of pages are; strides in bytes.
struct taps_mx_place {
    char *codes, *scales;
    int64_t code_stride[3], scale_stride[3];
};

// Rows: the heads of k and then of v of every token.
struct taps_mx_append_launch {
    const void *src[2];
    int64_t src_stride[2][2];   // token, head; in elements
    taps_mx_place cache[2];
    const void *weight;
    const float *table;
    const taps_plan_token *plan_tokens;
    uint32_t tokens, heads, dim, rotary, page_log2;
    uint32_t across;   // set by the launch
    double inverse_dim;
    float eps, most;   // most: magnitudes above it are taken for it
    uint8_t interleaved, float_weight;
};

struct taps_mx_read_launch {
    void *dst[2];
    int64_t dst_stride[2][2];
    taps_mx_place cache[2];
    const void *slots;
    int64_t n_slots;
    uint32_t tokens, heads, dim, page_log2;
    uint32_t across;   // set by the launch
    uint8_t wide_slots;
};

// Codes take the place of a 16-bit cache's elements.
struct taps_mx_attend_launch : taps_attend_launch {
    const char *k_scales, *v_scales;
    int64_t ks_page, ks_head, ks_slot, vs_page, vs_head, vs_slot;
};

// vectors: rows start at multiples of eight elements, rotary_dim is a multiple of 8.
hipError_t taps_launch_mx_append(taps_mx_append_launch p, uint32_t dtype, uint32_t bits,
                                 bool vectors, hipStream_t stream);
// vectors: rows start at multiples of eight elements.
hipError_t taps_launch_mx_read(taps_mx_read_launch p, uint32_t dtype, uint32_t bits,
                               bool vectors, hipStream_t stream);
hipError_t taps_launch_mx_attend(const taps_mx_attend_launch &p, uint32_t dtype, uint32_t bits,
                                 hipStream_t stream);
