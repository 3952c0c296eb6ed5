// taps_attention_internal.h -- what the host side of libtaps_attention.so and
// its kernels share: the layout of a plan and the launch parameters.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "taps_attention.h"

// ---------------------------------------------------------------------------
// plan of a step (taps_paged_plan): a header and four arrays, the same bytes
// on the host and on the device
// ---------------------------------------------------------------------------

constexpr uint32_t kPlanMagic = 0x54415031;

// Query rows of the kinds of items (taps_attend.hip).  A row is a pair of a
// token and one of the query heads of a key head.
constexpr int kWideRows = 256, kBlockRows = 128, kNarrowRows = 32, kFewRows = 16;
// Only plans for heads of more have wide items.
constexpr uint32_t kWideAbove = 64;
// Keys of a tile: of wide and block items, and of narrow ones.
constexpr int kWideKeys = 64, kNarrowKeys = 32;

struct taps_plan_header {
    uint32_t magic, n_seqs;
    uint64_t bytes;
    uint32_t tokens, q_heads, kv_heads, head_dim;
    uint32_t page_log2, n_pages, causal, window;
    uint32_t n_items, n_joins;   // items: the first n_wide are wide
    uint32_t part_rows;       // rows of partial results over all split pieces
    uint32_t max_positions;   // largest position of a new token, plus one
    uint32_t appendable;      // every sequence has kv_lens >= q_lens
    uint32_t join_rounds;     // workgroups that the rows of a join are spread over, at most
    uint32_t n_wide;
    uint32_t n_few;           // of the items: narrow ones of up to kFewRows rows
    uint32_t zeros[4];        // what attention reads for keys that are not there
    // byte offsets of the arrays
    uint64_t tokens_at, pages_at, items_at, joins_at;
};
static_assert(offsetof(taps_plan_header, zeros) % 16 == 0, "read 16 bytes at a time");

struct taps_plan_token {
    int32_t position;
    int32_t slot;   // page * page_size + slot; -1: not appended
};

// One workgroup of attention per item and key head.  The kinds differ in rows
// and in how a workgroup shares them out (taps_attend.hip).
enum { kWide, kBlock, kNarrow };

struct taps_plan_item {
    int32_t seq, row0;    // rows row0 .. of the sequence
    int32_t lo, hi;       // keys lo .. hi - 1
    int32_t kind;
    int32_t part;         // first row of partial results, or -1: the item is its rows' only one
    // the sequence's, so that nothing waits for a second look-up
    int32_t token0, rows, first_pos, page0;
    int32_t reserved[2];
};

// Rows whose keys were split: `parts` pieces of `rows` rows each.
struct taps_plan_join {
    int32_t seq, row0, rows, part, parts;
    int32_t token0;
    int32_t reserved[2];
};

// Groups of lanes of a workgroup's 8 that share a row's pieces in k_join, which
// takes four of a group's at once.
__host__ __device__ inline int taps_join_across(int parts) {
    return parts <= 4 ? 1 : parts <= 8 ? 2 : parts <= 16 ? 4 : 8;
}

// ---------------------------------------------------------------------------
// launches
// ---------------------------------------------------------------------------

struct taps_rows_launch {
    const void *src[2];    // q, k (append: k, v); backward: the outputs' gradients
    const void *x[2];      // backward: q, k
    void *dst[2];
    int64_t src_stride[2][3], x_stride[2][3], dst_stride[2][3];
    const void *weight[2];
    const float *table;
    const void *positions;               // NULL: first + t
    const taps_plan_token *plan_tokens;  // append
    float *partial;                      // backward: [workgroups][2][head_dim]
    int64_t first;
    uint32_t batch, tokens;   // tokens of one sequence
    uint32_t heads[2];
    uint32_t dim, rotary;
    uint32_t n_positions;
    uint32_t page_log2;
    float eps;
    uint8_t wide_positions, interleaved, float_weights, norm[2];
};

hipError_t taps_launch_norm_rotate(const taps_rows_launch &p, uint32_t dtype, bool vectors,
                                   hipStream_t stream);
hipError_t taps_launch_append(const taps_rows_launch &p, uint32_t dtype, bool vectors,
                              hipStream_t stream);
// Workgroups of the backward kernel, each of which leaves one partial sum:
// enough to fill 256 compute units four times over.
constexpr uint32_t kMostBackwardGroups = 1024;
uint32_t taps_backward_groups(const taps_rows_launch &p, bool vectors);
hipError_t taps_launch_norm_rotate_backward(const taps_rows_launch &p, uint32_t dtype, bool vectors,
                                            void *q_weight_grad, void *k_weight_grad,
                                            hipStream_t stream);

struct taps_attend_launch {
    const char *q, *k_cache, *v_cache;
    const char *zeros;   // 16 bytes
    char *out;
    float *lse;
    float *part_o, *part_ml;   // [part_rows][kv_heads][dim], [part_rows][kv_heads][2]
    const int32_t *pages;
    const taps_plan_item *items;
    const taps_plan_join *joins;
    // strides in bytes
    int64_t q_token, q_head, o_token, o_head;
    int64_t k_page, k_head, k_slot, v_page, v_head, v_slot;
    uint32_t n_items, n_wide, n_few, n_joins, join_rounds, q_heads, kv_heads, group, dim;
    uint32_t page_log2, causal, window;
    float scale;
};

hipError_t taps_launch_attend(const taps_attend_launch &p, uint32_t dtype, hipStream_t stream);
// Adds up the pieces of rows whose keys were split; nothing to do without any.
hipError_t taps_launch_join(const taps_attend_launch &p, uint32_t dtype, hipStream_t stream);
