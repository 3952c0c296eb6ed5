// taps_attention_api.hip -- the C ABI of taps_attention.h: validation, plans
// and launches.  Host code only sizes and checks.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <cstring>
#include <new>
#include <vector>

#include "taps_attention_internal.h"

namespace {

thread_local char g_last_error[512] = "";

taps_status fail(taps_status st, const char *fmt, ...) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(g_last_error, sizeof g_last_error, fmt, ap);
    va_end(ap);
    return st;
}

taps_status launched(hipError_t err, const char *what) {
    if (err == hipSuccess) return TAPS_OK;
    return fail(TAPS_ERR_DEVICE, "%s: %s", what, hipGetErrorString(err));
}

uint32_t size_of(uint32_t dtype) { return dtype == TAPS_F32 ? 4 : 2; }

bool aligned(const void *p, uint64_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// ---------------------------------------------------------------------------
// norm and rotation
// ---------------------------------------------------------------------------

taps_status check_types(uint32_t dtype, uint32_t weight_dtype, uint32_t dim, uint32_t rotary,
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

taps_status check_heads(const taps_heads *t, const char *what, uint32_t dtype) {
    if (!t || !t->data) return fail(TAPS_ERR_ARG, "%s is NULL", what);
    if (!aligned(t->data, size_of(dtype)))
        return fail(TAPS_ERR_ARG, "%s is not aligned to its elements", what);
    return TAPS_OK;
}

// Whether every row starts at a multiple of four elements.
bool by_fours(const taps_heads &t, uint32_t dtype) {
    return aligned(t.data, 4 * size_of(dtype)) && t.stride[0] % 4 == 0 && t.stride[1] % 4 == 0 &&
           t.stride[2] % 4 == 0;
}

bool vectors_fit(uint32_t dim, uint32_t rotary, uint32_t weight_dtype, const void *w0, const void *w1,
                 const float *table) {
    const uint32_t w = 4 * size_of(weight_dtype);
    return dim % 8 == 0 && rotary % 8 == 0 && aligned(w0, w) && aligned(w1, w) && aligned(table, 16);
}

void set_strides(int64_t (&to)[3], const taps_heads &t) {
    for (int i = 0; i < 3; ++i) to[i] = t.stride[i];
}

taps_status check_norm_rotate(const taps_norm_rotate_args *a, taps_rows_launch *p) {
    if (!a) return fail(TAPS_ERR_ARG, "args is NULL");
    if (taps_status st = check_types(a->dtype, a->weight_dtype, a->head_dim, a->rotary_dim, a->eps,
                                     a->table))
        return st;
    if (!a->q_heads) return fail(TAPS_ERR_ARG, "q_heads is 0");
    if ((uint64_t)a->q_heads + a->k_heads > (1u << 20))
        return fail(TAPS_ERR_ARG, "%u + %u heads are too many", a->q_heads, a->k_heads);
    if ((uint64_t)a->batch * a->tokens >= (1ull << 31))
        return fail(TAPS_ERR_ARG, "%u x %u tokens are too many", a->batch, a->tokens);
    if (a->positions) {
        if (a->position_bytes != 4 && a->position_bytes != 8)
            return fail(TAPS_ERR_ARG, "position_bytes %u is neither 4 nor 8", a->position_bytes);
        if (!aligned(a->positions, a->position_bytes))
            return fail(TAPS_ERR_ARG, "positions is not aligned to its elements");
        // the kernels read row 0 for a position that is no row of the table
        if (a->rotary_dim && a->batch && a->tokens && !a->n_positions)
            return fail(TAPS_ERR_ARG, "the table has no rows for positions");
    } else if (a->rotary_dim && a->batch && a->tokens &&
               (a->first_position < 0 || a->first_position > (int64_t)a->n_positions ||
                a->tokens > a->n_positions - (uint64_t)a->first_position)) {
        return fail(TAPS_ERR_ARG, "positions %lld .. + %u exceed the table's %u",
                    (long long)a->first_position, a->tokens, a->n_positions);
    }
    *p = taps_rows_launch{};
    p->weight[0] = a->q_weight, p->weight[1] = a->k_weight;
    p->norm[0] = a->q_weight != nullptr, p->norm[1] = a->k_weight != nullptr;
    p->float_weights = a->weight_dtype == TAPS_F32;
    p->table = a->table;
    p->positions = a->positions;
    p->wide_positions = a->position_bytes == 8;
    p->first = a->first_position;
    p->batch = a->batch, p->tokens = a->tokens;
    p->heads[0] = a->q_heads, p->heads[1] = a->k_heads;
    p->dim = a->head_dim, p->rotary = a->rotary_dim;
    p->n_positions = a->n_positions;
    p->eps = a->eps;
    p->interleaved = a->interleaved != 0;
    if (!a->k_heads) p->norm[1] = 0;
    return TAPS_OK;
}

// ---------------------------------------------------------------------------
// plans
// ---------------------------------------------------------------------------

uint64_t up16(uint64_t v) { return (v + 15) & ~15ull; }

struct Sequence {
    int32_t token0;      // its first token
    int32_t rows;        // query rows: q_len * (q_heads / kv_heads)
    int32_t kv_start, kv_len;
    int32_t first_pos;   // position of its first token
    int32_t page0;       // its pages in the plan's array
};

struct Layout {
    std::vector<Sequence> seqs;
    std::vector<taps_plan_item> items;
    std::vector<taps_plan_join> joins;
    taps_plan_header head{};
};

// Shorter pieces are not made: a split costs a launch and a pass over partial
// results, some 5 us for few rows, in which a narrow item takes about this many
// keys (one token over 1024 keys of 16 heads: 11.3 us whole, 13.7 in four) and a
// block half as many (256 tokens over 1500, 16 heads of 64: 25.5 us whole, 19.5 so).
constexpr int64_t kLeastNarrow = 1024, kLeastPiece = 512;

int64_t least_piece(int32_t kind) { return kind == kNarrow ? kLeastNarrow : kLeastPiece; }

// Query rows that share their keys' loads, before they are split over the keys.
struct Strip {
    int32_t seq, row0, rows, lo, hi, kind;
    // what a key costs: a narrow item waits for its bytes, which come to a
    // compute unit at about half the rate at which the others work keys off
    int64_t cost() const { return cost_of(kind, hi - lo); }
    // pieces of about `piece`: one 3 % above it is not cut again
    int64_t parts(int64_t piece) const {
        const int64_t n = (cost() + piece - 1 - piece / 32) / piece;
        return std::max<int64_t>(1, std::min<int64_t>({n, (hi - lo) / least_piece(kind), 256}));
    }
    static int64_t cost_of(int32_t kind, int64_t keys) { return keys * (kind == kNarrow ? 2 : 1); }
};

// Pieces per compute unit that narrow items are cut into: two fill a unit, and
// their bytes set the time (two tokens over 131001 keys: 187 us, 192 at four).
constexpr int64_t kNarrowPieces = 2;

// The other kinds: the length of a piece, in keys, is the one of those below at
// which the step should end first.  Pieces of like length run in rounds over the
// units, and a last round that few share costs as much as a full one; others,
// dear ones first, fill the gaps.  Nothing ends before its longest piece.  Two
// blocks on a unit take longer than one alone.
//   512 tokens over 32768 keys, 64 wide strips: 249 us as 256 pieces, 297 as 392,
//   331 as 528;
//   4 prompts of 2048, 4 heads, 256 blocks: 49 us whole, 40 as 480 pieces;
//   prompts of 700 and single tokens, 176 blocks: 26 us whole, 34 as 304 pieces.
constexpr double kPieceCost = 256;   // a piece's start and end, in keys
constexpr double kJoinCost = 600;    // the join's launch and pass, in keys
constexpr double kCrowded = 1.6;     // a block's time beside another, by its time alone
constexpr int64_t kMostRounds = 8;   // lengths are tried that come to 1/4, 1/2 .. 8 rounds

int64_t share_of(int64_t total, int64_t times, int64_t among) {
    return (int64_t)std::min((double)total * (double)times / (double)among, 1e18) + 1;
}

int64_t piece_of(const std::vector<Strip> &strips, int32_t kind, int64_t cus, int64_t heads) {
    const int64_t slots = kind == kWide ? cus : 2 * cus;
    int64_t total = 0, all = 0;
    for (const Strip &t : strips)
        if (t.kind == kind) total += t.cost(), ++all;
    int64_t best = 1;
    double least = INFINITY;
    for (int64_t k = 0; all && k <= 4 * kMostRounds; ++k) {   // at 0 nothing is cut
        const int64_t share = k ? share_of(total, 4 * heads, slots * k) : total;
        const int64_t piece = std::max(share, least_piece(kind));
        int64_t n = 0, longest = 1;
        for (const Strip &t : strips)
            if (t.kind == kind) {
                const int64_t parts = t.parts(piece);
                n += parts, longest = std::max(longest, t.cost() / parts);
            }
        const bool crowded = kind == kBlock && n * heads > cus;
        const double mean = (double)total / n, rounds = (double)((n * heads + slots - 1) / slots);
        const double span = std::max<double>(
            longest, std::min(rounds * longest,
                              (double)n * heads / slots * mean + mean * mean / longest));
        const double cost = (crowded ? kCrowded : 1) * span + rounds * kPieceCost +
                            (n > all ? kJoinCost : 0);
        if (cost < least) least = cost, best = piece;
    }
    return best;
}

// The order in which items start: kind by kind.  Workgroups that run at the same
// time should find each other's keys in the cache, and the last ones to start
// should be cheap.  So the items of a sequence follow each other, its dear ones
// first, up to the last sequences, which come to the time of one dear item on
// every slot: of those the dear items come first, whatever their sequence
// (prompts of 2048 of eight sequences, 32 heads: 350 us with all dear items first, 321
// so, 321 by sequences alone; 20 of 100 to 700 tokens: 107, 108 and 119).
// Narrow items share no keys: dear ones first.
void in_order(std::vector<taps_plan_item> *items, int64_t cus, int64_t heads) {
    const auto cost = [](const taps_plan_item &i) { return Strip::cost_of(i.kind, i.hi - i.lo); };
    const auto dear = [&](const taps_plan_item &x, const taps_plan_item &y) {
        return cost(x) >> 8 > cost(y) >> 8;
    };
    std::stable_sort(items->begin(), items->end(),
                     [](const taps_plan_item &x, const taps_plan_item &y) {
                         return std::make_pair(x.kind, x.seq) < std::make_pair(y.kind, y.seq);
                     });
    for (auto at = items->begin(); at != items->end();) {
        const int32_t kind = at->kind;
        const int64_t slots = kind == kWide ? cus : 2 * cus;
        const auto end = std::find_if(at, items->end(),
                                      [&](const taps_plan_item &i) { return i.kind != kind; });
        int64_t sum = 0, most = 0;
        auto rest = end;   // where the last sequences begin
        while (rest != at && (kind == kNarrow || !sum || sum * heads < slots * most)) {
            const int32_t seq = (rest - 1)->seq;
            for (; rest != at && (rest - 1)->seq == seq; --rest)
                sum += cost(*(rest - 1)), most = std::max(most, cost(*(rest - 1)));
        }
        while (at != rest) {
            const int32_t seq = at->seq;
            const auto next = std::find_if(at, rest,
                                           [&](const taps_plan_item &i) { return i.seq != seq; });
            std::stable_sort(at, next, dear);
            at = next;
        }
        std::stable_sort(rest, end, dear);
        at = end;
    }
}

// Whether sequences of more than 128 rows are cut into strips of 256 rows (wide
// items), which read the fewest keys, or of 128.  Wide ones pay
//   - for heads of more than kWideAbove, where two blocks fill a unit (eight prompts of
//     2048, 32 heads of 64: 212 us wide, 177 in blocks; 512 tokens over 32768
//     keys, 32 heads of 64 over 8: 170 and 174; of 96: 209 and 223);
//   - if the keys they see keep the loop busy beside a workgroup's start and end,
//     which nothing covers (32 heads of 128, eight prompts of 1024: 105 and 97, of 1900:
//     301 and 295, of 2047: 322 and 328, of 2500: 455 and 478);
//   - for heads of up to 96, if few of the keys are seen by some rows only, with
//     which wavefronts wait for the strip's last one (32 heads of 96, prompts of 2048:
//     269 to 289 and 264, two of 8000: 820 and 812; 4 chunks of 512 over 4096 keys, 32
//     heads over 8: 101 and 108, one over 32768: 205 and 218);
//   - if there are some rounds of them over the units, pieces counted (4 sequences of
//     2048, 4 heads of 128: 51 and 48).
constexpr int64_t kWideKeysSeen = 960, kWidePiece = 1024, kWideRounds = 4;
constexpr uint32_t kDiagonalUpTo = 96;

bool wide_pays(const taps_paged_batch *b, const std::vector<Sequence> &seqs, int64_t window,
               int64_t cus) {
    int64_t strips = 0, pieces = 0, keys = 0, loaded = 0;
    for (const Sequence &q : seqs) {
        const int64_t n = q.rows / kWideRows, kv = q.kv_len - q.kv_start;
        int64_t seen = b->causal ? kv - (q.kv_len - q.first_pos) / 2 : kv;   // on average
        int64_t most = kv;
        if (window) seen = std::min(seen, window), most = std::min(most, window + kWideRows);
        strips += n, keys += n * seen, loaded += n * most;
        pieces += n * std::max<int64_t>(1, kv / kWidePiece);
    }
    return b->head_dim > kWideAbove && keys >= kWideKeysSeen * strips &&
           (b->head_dim > kDiagonalUpTo || 4 * keys >= 3 * loaded) &&
           pieces * b->kv_heads >= kWideRounds * cus;
}

taps_status lay_out(const taps_paged_batch *b, uint32_t cus, Layout *out) {
    taps_plan_header &h = out->head;
    const uint32_t group = b->q_heads / b->kv_heads;
    const uint32_t log2 = (uint32_t)__builtin_ctz(b->page_size);
    uint64_t tokens = 0, pages = 0;
    int64_t most = 0;
    bool appendable = true;
    std::vector<int32_t> written;
    std::vector<Strip> strips;
    out->seqs.reserve(b->n_seqs);
    for (uint32_t s = 0; s < b->n_seqs; ++s) {
        const int64_t n = b->q_lens[s], kv = b->kv_lens[s], from = b->kv_starts ? b->kv_starts[s] : 0;
        if (n < 0 || kv < 0 || n > (1 << 30) || kv > (1 << 30))
            return fail(TAPS_ERR_ARG, "sequence %u: lengths %lld and %lld outside 0..2^30", s,
                        (long long)n, (long long)kv);
        if (from < 0 || from > kv)
            return fail(TAPS_ERR_ARG, "sequence %u: its keys start at %lld of %lld", s,
                        (long long)from, (long long)kv);
        const int64_t n_pages = (kv + b->page_size - 1) >> log2;
        if (n_pages > b->pages_stride)
            return fail(TAPS_ERR_ARG, "sequence %u: %lld keys need %lld pages of %u", s,
                        (long long)kv, (long long)n_pages, b->pages_stride);
        if (n * group > (1 << 30))
            return fail(TAPS_ERR_ARG, "sequence %u: %lld tokens x %u heads are too many", s,
                        (long long)n, group);
        const int32_t *row = b->pages + (uint64_t)s * b->pages_stride;
        for (int64_t g = from >> log2; g < n_pages; ++g)
            if (from < kv && (row[g] < 0 || (uint32_t)row[g] >= b->n_pages))
                return fail(TAPS_ERR_ARG, "sequence %u: page %d outside 0..%u", s, row[g],
                            b->n_pages);
        const int64_t first = std::max(kv - n, from);   // first appended position
        for (int64_t g = std::max<int64_t>(first, 0) >> log2; g < n_pages; ++g)
            if (n && first < kv) written.push_back(row[g]);
        if (kv < n) appendable = false;
        if (n) most = std::max(most, kv);
        Sequence q{};
        q.token0 = (int32_t)tokens;
        q.rows = (int32_t)(n * group);
        q.kv_start = (int32_t)from, q.kv_len = (int32_t)kv;
        q.first_pos = (int32_t)(kv - n);
        q.page0 = (int32_t)pages;
        out->seqs.push_back(q);
        tokens += (uint64_t)n;
        pages += (uint64_t)n_pages;
        if (tokens >= (1ull << 31) || pages >= (1ull << 31))
            return fail(TAPS_ERR_ARG, "2^31 or more tokens or pages in all");
    }
    std::sort(written.begin(), written.end());
    if (std::adjacent_find(written.begin(), written.end()) != written.end())
        return fail(TAPS_ERR_ARG, "page %d is to be written from two places of the page table",
                    *std::adjacent_find(written.begin(), written.end()));

    const bool wide = wide_pays(b, out->seqs, h.window, cus);
    for (uint32_t s = 0; s < b->n_seqs; ++s) {
        const Sequence &q = out->seqs[s];
        const int32_t kind = q.rows <= kNarrowRows          ? kNarrow
                             : wide && q.rows > kBlockRows ? kWide
                                                           : kBlock;
        const int32_t step = kind == kNarrow ? kNarrowRows : kind == kBlock ? kBlockRows : kWideRows;
        for (int32_t r = 0; r < q.rows; r += step) {
            Strip t{(int32_t)s, r, std::min(step, q.rows - r), q.kv_start, q.kv_len, kind};
            if (b->causal) {
                const int64_t pos_a = q.first_pos + r / (int64_t)group;
                const int64_t pos_b = q.first_pos + (r + t.rows - 1) / (int64_t)group;
                t.hi = (int32_t)std::max<int64_t>(std::min<int64_t>(q.kv_len, pos_b + 1), 0);
                if (h.window)
                    t.lo = (int32_t)std::max<int64_t>(t.lo, pos_a - (int64_t)h.window + 1);
            }
            if (t.hi < t.lo) t.hi = t.lo;
            strips.push_back(t);
        }
    }

    int64_t total = 0;
    for (const Strip &t : strips) total += t.cost();
    const int64_t heads = b->kv_heads;
    const int64_t narrow = share_of(total, heads, cus * kNarrowPieces);
    const int64_t wides = piece_of(strips, kWide, cus, heads);
    const int64_t blocks = piece_of(strips, kBlock, cus, heads);
    uint64_t part_rows = 0;
    for (const Strip &t : strips) {
        int64_t parts = t.parts(t.kind == kNarrow ? narrow : t.kind == kBlock ? blocks : wides);
        // whole tiles, counted from where the strip's first tile starts
        const int64_t start = t.lo & ~15, tiles = (t.hi - start + 127) / 128;
        parts = std::max<int64_t>(1, std::min(parts, tiles));
        if (parts > 1) {
            const uint32_t rows = 8 / taps_join_across((int)parts);
            h.join_rounds = std::max(h.join_rounds, (t.rows + rows - 1) / rows);
            out->joins.push_back({t.seq, t.row0, t.rows, (int32_t)part_rows, (int32_t)parts,
                                  out->seqs[t.seq].token0, {}});
        }
        for (int64_t k = 0; k < parts; ++k) {
            taps_plan_item i{};
            i.seq = t.seq, i.row0 = t.row0, i.kind = t.kind;
            const Sequence &q = out->seqs[t.seq];
            i.token0 = q.token0, i.rows = q.rows, i.first_pos = q.first_pos, i.page0 = q.page0;
            i.lo = (int32_t)std::max<int64_t>(t.lo, start + 128 * (tiles * k / parts));
            i.hi = (int32_t)std::min<int64_t>(t.hi, start + 128 * (tiles * (k + 1) / parts));
            i.part = parts > 1 ? (int32_t)(part_rows + k * t.rows) : -1;
            out->items.push_back(i);
        }
        if (parts > 1) part_rows += (uint64_t)parts * t.rows;
        if (part_rows >= (1ull << 31)) return fail(TAPS_ERR_ARG, "too many rows are split");
    }
    in_order(&out->items, cus, heads);
    for (const taps_plan_item &i : out->items) h.n_wide += i.kind == kWide;
    if (out->items.size() * b->kv_heads >= (1ull << 31) || b->kv_heads > 65535)
        return fail(TAPS_ERR_ARG, "too many workgroups");

    h.magic = kPlanMagic;
    h.n_seqs = b->n_seqs;
    h.tokens = (uint32_t)tokens;
    h.q_heads = b->q_heads, h.kv_heads = b->kv_heads, h.head_dim = b->head_dim;
    h.page_log2 = log2, h.n_pages = b->n_pages, h.causal = b->causal != 0;
    h.n_items = (uint32_t)out->items.size(), h.n_joins = (uint32_t)out->joins.size();
    h.part_rows = (uint32_t)part_rows;
    h.max_positions = (uint32_t)most;
    h.appendable = appendable;
    uint64_t at = up16(sizeof h);
    h.tokens_at = at, at = up16(at + tokens * sizeof(taps_plan_token));
    h.pages_at = at, at = up16(at + pages * 4);
    h.items_at = at, at = up16(at + out->items.size() * sizeof(taps_plan_item));
    h.joins_at = at, at = up16(at + out->joins.size() * sizeof(taps_plan_join));
    h.bytes = at;
    return TAPS_OK;
}

uint64_t workspace_of(const taps_plan_header &h) {
    return up16((uint64_t)h.part_rows * h.kv_heads * h.head_dim * 4) +
           up16((uint64_t)h.part_rows * h.kv_heads * 8);
}

void write_plan(const taps_paged_batch *b, const Layout &l, char *to) {
    const taps_plan_header &h = l.head;
    memcpy(to, &h, sizeof h);
    if (!l.items.empty())
        memcpy(to + h.items_at, l.items.data(), l.items.size() * sizeof l.items[0]);
    if (!l.joins.empty())
        memcpy(to + h.joins_at, l.joins.data(), l.joins.size() * sizeof l.joins[0]);
    auto *token = (taps_plan_token *)(to + h.tokens_at);
    auto *pages = (int32_t *)(to + h.pages_at);
    for (uint32_t s = 0; s < h.n_seqs; ++s) {
        const int32_t *row = b->pages + (uint64_t)s * b->pages_stride;
        const Sequence &q = l.seqs[s];
        const int64_t n_pages = ((int64_t)q.kv_len + b->page_size - 1) >> h.page_log2;
        for (int64_t g = 0; g < n_pages; ++g) *pages++ = row[g];
        for (int64_t p = (int64_t)q.kv_len - b->q_lens[s]; p < q.kv_len; ++p, ++token) {
            token->position = (int32_t)p;
            token->slot = p < q.kv_start || p < 0
                              ? -1
                              : (int32_t)(((int64_t)row[p >> h.page_log2] << h.page_log2) +
                                          (p & (b->page_size - 1)));
        }
    }
}

taps_status check_plan(const void *plan, const void *plan_device, const taps_plan_header **h) {
    if (!plan || !plan_device) return fail(TAPS_ERR_ARG, "plan or plan_device is NULL");
    if (!aligned(plan, 16) || !aligned(plan_device, 16))
        return fail(TAPS_ERR_ARG, "plan or plan_device is not 16-byte aligned");
    *h = (const taps_plan_header *)plan;
    if ((*h)->magic != kPlanMagic) return fail(TAPS_ERR_ARG, "plan was not made by taps_paged_plan");
    return TAPS_OK;
}

}  // namespace

extern "C" {

taps_status taps_norm_rotate(const taps_norm_rotate_args *a, const taps_heads *q, const taps_heads *k,
                             const taps_heads *q_out, const taps_heads *k_out, void *stream) {
    taps_rows_launch p;
    if (taps_status st = check_norm_rotate(a, &p)) return st;
    if (!a->batch || !a->tokens) return TAPS_OK;
    const taps_heads *const src[2] = {q, k}, *const dst[2] = {q_out, k_out};
    static const char *const names[2][2] = {{"q", "q_out"}, {"k", "k_out"}};
    bool vectors = vectors_fit(p.dim, p.rotary, a->weight_dtype, a->q_weight, a->k_weight, a->table);
    for (int side = 0; side < (a->k_heads ? 2 : 1); ++side) {
        if (taps_status st = check_heads(src[side], names[side][0], a->dtype)) return st;
        if (taps_status st = check_heads(dst[side], names[side][1], a->dtype)) return st;
        p.src[side] = src[side]->data, p.dst[side] = dst[side]->data;
        set_strides(p.src_stride[side], *src[side]);
        set_strides(p.dst_stride[side], *dst[side]);
        vectors = vectors && by_fours(*src[side], a->dtype) && by_fours(*dst[side], a->dtype);
    }
    return launched(taps_launch_norm_rotate(p, a->dtype, vectors, (hipStream_t)stream),
                    "taps_norm_rotate");
}

taps_status taps_norm_rotate_backward(const taps_norm_rotate_args *a, const taps_heads *dq_out,
                                      const taps_heads *dk_out, const taps_heads *q,
                                      const taps_heads *k, const taps_heads *dq,
                                      const taps_heads *dk, void *q_weight_grad, void *k_weight_grad,
                                      void *workspace, uint64_t *workspace_bytes, void *stream) {
    taps_rows_launch p;
    if (taps_status st = check_norm_rotate(a, &p)) return st;
    if (!workspace_bytes) return fail(TAPS_ERR_ARG, "workspace_bytes is NULL");
    const bool norms = p.norm[0] || p.norm[1];
    // a partial sum per workgroup; as many workgroups on either path as the other could take
    const uint64_t groups = std::max(taps_backward_groups(p, true), taps_backward_groups(p, false));
    const uint64_t need = norms ? up16(groups * 2 * p.dim * 4) : 16;
    static_assert(TAPS_NORM_ROTATE_WORKSPACE(1) == kMostBackwardGroups * 2 * 4, "as declared");
    if (!workspace) {
        *workspace_bytes = need;
        return TAPS_OK;
    }
    if (*workspace_bytes < need)
        return fail(TAPS_ERR_CAPACITY, "workspace of %llu bytes, %llu are needed",
                    (unsigned long long)*workspace_bytes, (unsigned long long)need);
    if (!aligned(workspace, 16)) return fail(TAPS_ERR_ARG, "workspace is not 16-byte aligned");
    const uint32_t sides = a->k_heads ? 2 : 1;
    if ((q_weight_grad != nullptr) != (a->q_weight != nullptr) ||
        (sides == 2 && (k_weight_grad != nullptr) != (a->k_weight != nullptr)))
        return fail(TAPS_ERR_ARG, "a weight and its gradient go together");
    if (sides == 1) k_weight_grad = nullptr;
    const uint32_t w = size_of(a->weight_dtype);
    if (!aligned(q_weight_grad, w) || !aligned(k_weight_grad, w))
        return fail(TAPS_ERR_ARG, "a weight's gradient is not aligned to its elements");
    const taps_heads *const g[2] = {dq_out, dk_out}, *const x[2] = {q, k}, *const d[2] = {dq, dk};
    static const char *const names[2][3] = {{"dq_out", "q", "dq"}, {"dk_out", "k", "dk"}};
    bool vectors = vectors_fit(p.dim, p.rotary, a->weight_dtype, a->q_weight, a->k_weight, a->table);
    for (uint32_t side = 0; side < sides && a->batch && a->tokens; ++side) {
        if (taps_status st = check_heads(g[side], names[side][0], a->dtype)) return st;
        if (taps_status st = check_heads(x[side], names[side][1], a->dtype)) return st;
        if (taps_status st = check_heads(d[side], names[side][2], a->dtype)) return st;
        p.src[side] = g[side]->data, p.x[side] = x[side]->data, p.dst[side] = d[side]->data;
        set_strides(p.src_stride[side], *g[side]);
        set_strides(p.x_stride[side], *x[side]);
        set_strides(p.dst_stride[side], *d[side]);
        vectors = vectors && by_fours(*g[side], a->dtype) && by_fours(*x[side], a->dtype) &&
                  by_fours(*d[side], a->dtype);
    }
    if (!norms && (!a->batch || !a->tokens)) return TAPS_OK;
    p.partial = norms ? (float *)workspace : nullptr;
    return launched(taps_launch_norm_rotate_backward(p, a->dtype, vectors, q_weight_grad,
                                                     k_weight_grad, (hipStream_t)stream),
                    "taps_norm_rotate_backward");
}

taps_status taps_paged_plan(const taps_paged_batch *b, uint32_t cus, void *plan,
                            uint64_t *plan_bytes, uint64_t *workspace_bytes) {
    if (!b || !plan_bytes || !workspace_bytes)
        return fail(TAPS_ERR_ARG, "batch, plan_bytes or workspace_bytes is NULL");
    if (b->n_seqs && (!b->q_lens || !b->kv_lens || (!b->pages && b->pages_stride)))
        return fail(TAPS_ERR_ARG, "q_lens, kv_lens or pages is NULL");
    if (b->page_size < TAPS_MIN_PAGE || b->page_size > TAPS_MAX_PAGE ||
        (b->page_size & (b->page_size - 1)))
        return fail(TAPS_ERR_ARG, "page_size %u is not a power of two in %u..%u", b->page_size,
                    TAPS_MIN_PAGE, TAPS_MAX_PAGE);
    if ((uint64_t)b->n_pages * b->page_size >= (1ull << 31))
        return fail(TAPS_ERR_ARG, "%u pages of %u slots are 2^31 slots or more", b->n_pages,
                    b->page_size);
    if (!b->kv_heads || !b->q_heads || b->q_heads % b->kv_heads)
        return fail(TAPS_ERR_ARG, "q_heads %u is not a multiple of kv_heads %u", b->q_heads,
                    b->kv_heads);
    if (b->head_dim < 1 || b->head_dim > TAPS_MAX_HEAD_DIM)
        return fail(TAPS_ERR_ARG, "head_dim %u outside 1..%u", b->head_dim, TAPS_MAX_HEAD_DIM);
    if (b->window && !b->causal) return fail(TAPS_ERR_ARG, "a window needs causal");
    try {
        Layout l;
        l.head.window = b->window < (1u << 30) ? b->window : 0;   // beyond every length
        if (taps_status st = lay_out(b, cus ? cus : 256, &l)) return st;
        const uint64_t room = *plan_bytes;
        if (plan && room < l.head.bytes)
            return fail(TAPS_ERR_CAPACITY, "plan of %llu bytes, %llu are needed",
                        (unsigned long long)room, (unsigned long long)l.head.bytes);
        if (plan && !aligned(plan, 16)) return fail(TAPS_ERR_ARG, "plan is not 16-byte aligned");
        *plan_bytes = l.head.bytes;
        *workspace_bytes = workspace_of(l.head);
        if (plan) write_plan(b, l, (char *)plan);
    } catch (const std::bad_alloc &) {
        return fail(TAPS_ERR_CAPACITY, "out of host memory for a plan");
    } catch (...) {
        return fail(TAPS_ERR_ARG, "the plan could not be made");
    }
    return TAPS_OK;
}

taps_status taps_cache_append(const taps_append_args *a, const void *plan, const void *plan_device,
                              const taps_heads *k, const taps_heads *v, const taps_heads *k_cache,
                              const taps_heads *v_cache, void *stream) {
    if (!a) return fail(TAPS_ERR_ARG, "args is NULL");
    const taps_plan_header *h;
    if (taps_status st = check_plan(plan, plan_device, &h)) return st;
    if (taps_status st = check_types(a->dtype, a->weight_dtype, h->head_dim, a->rotary_dim, a->eps,
                                     a->table))
        return st;
    if (!h->appendable)
        return fail(TAPS_ERR_ARG, "a sequence of the plan has more new tokens than keys");
    if (a->rotary_dim && h->max_positions > a->n_positions)
        return fail(TAPS_ERR_ARG, "positions up to %u exceed the table's %u", h->max_positions,
                    a->n_positions);
    if (!h->tokens) return TAPS_OK;
    taps_rows_launch p{};
    const taps_heads *const src[2] = {k, v}, *const dst[2] = {k_cache, v_cache};
    static const char *const names[2][2] = {{"k", "k_cache"}, {"v", "v_cache"}};
    bool vectors =
        vectors_fit(h->head_dim, a->rotary_dim, a->weight_dtype, a->k_weight, nullptr, a->table);
    for (int side = 0; side < 2; ++side) {
        if (taps_status st = check_heads(src[side], names[side][0], a->dtype)) return st;
        if (taps_status st = check_heads(dst[side], names[side][1], a->dtype)) return st;
        p.src[side] = src[side]->data, p.dst[side] = dst[side]->data;
        set_strides(p.src_stride[side], *src[side]);
        p.src_stride[side][0] = 0;
        set_strides(p.dst_stride[side], *dst[side]);
        taps_heads rows = *src[side];
        rows.stride[0] = 0;   // not used
        vectors = vectors && by_fours(rows, a->dtype) && by_fours(*dst[side], a->dtype);
    }
    p.plan_tokens = (const taps_plan_token *)((const char *)plan_device + h->tokens_at);
    p.weight[0] = a->k_weight;
    p.norm[0] = a->k_weight != nullptr;
    p.float_weights = a->weight_dtype == TAPS_F32;
    p.table = a->table;
    p.batch = 1, p.tokens = h->tokens;
    p.heads[0] = p.heads[1] = h->kv_heads;
    p.dim = h->head_dim, p.rotary = a->rotary_dim;
    p.n_positions = a->n_positions;
    p.page_log2 = h->page_log2;
    p.eps = a->eps;
    p.interleaved = a->interleaved != 0;
    return launched(taps_launch_append(p, a->dtype, vectors, (hipStream_t)stream),
                    "taps_cache_append");
}

taps_status taps_attend(uint32_t dtype, const void *plan, const void *plan_device, const taps_heads *q,
                        const taps_heads *k_cache, const taps_heads *v_cache, float scale,
                        const taps_heads *out, float *lse, void *workspace,
                        uint64_t workspace_bytes, void *stream) {
    if (dtype != TAPS_BF16 && dtype != TAPS_F16)
        return fail(TAPS_ERR_ARG, "dtype %u is neither TAPS_BF16 nor TAPS_F16", dtype);
    const taps_plan_header *h;
    if (taps_status st = check_plan(plan, plan_device, &h)) return st;
    if (h->head_dim % 8 || h->head_dim > TAPS_MAX_ATTEND_DIM)
        return fail(TAPS_ERR_ARG, "head_dim %u is not a multiple of 8 up to %u", h->head_dim,
                    TAPS_MAX_ATTEND_DIM);
    if (!(scale > 0.f) || std::isinf(scale))
        return fail(TAPS_ERR_ARG, "scale is not positive and finite");
    if (!h->tokens) return TAPS_OK;
    const taps_heads *const all[4] = {q, k_cache, v_cache, out};
    static const char *const names[4] = {"q", "k_cache", "v_cache", "out"};
    for (int i = 0; i < 4; ++i) {
        const bool cache = i == 1 || i == 2;
        if (!all[i] || !all[i]->data) return fail(TAPS_ERR_ARG, "%s is NULL", names[i]);
        // an axis of one is not stepped along
        const uint32_t lengths[3] = {cache ? h->n_pages : 1, cache ? h->kv_heads : h->tokens,
                                     cache ? 2 : h->q_heads};
        bool fits = aligned(all[i]->data, 16);
        for (int k = 0; k < 3; ++k) fits = fits && (lengths[k] < 2 || all[i]->stride[k] % 8 == 0);
        if (!fits)
            return fail(TAPS_ERR_ARG, "%s: rows do not start at multiples of 16 bytes", names[i]);
        // 16 slots' offsets are held in 32 bits
        if (cache && (all[i]->stride[2] < 0 || all[i]->stride[2] >= (1 << 26)))
            return fail(TAPS_ERR_ARG, "%s: slots are 2^26 elements or more apart", names[i]);
    }
    if (!aligned(lse, 4)) return fail(TAPS_ERR_ARG, "lse is not aligned to its elements");
    const uint64_t need = workspace_of(*h);
    if (need && !workspace) return fail(TAPS_ERR_ARG, "workspace is NULL");
    if (need > workspace_bytes)
        return fail(TAPS_ERR_CAPACITY, "workspace of %llu bytes, %llu are needed",
                    (unsigned long long)workspace_bytes, (unsigned long long)need);
    if (!aligned(workspace, 16)) return fail(TAPS_ERR_ARG, "workspace is not 16-byte aligned");
    taps_attend_launch p{};
    const char *dev = (const char *)plan_device;
    p.q = (const char *)q->data, p.out = (char *)out->data, p.lse = lse;
    p.k_cache = (const char *)k_cache->data, p.v_cache = (const char *)v_cache->data;
    p.zeros = dev + offsetof(taps_plan_header, zeros);
    p.part_o = (float *)workspace;
    p.part_ml = (float *)((char *)workspace +
                          up16((uint64_t)h->part_rows * h->kv_heads * h->head_dim * 4));
    p.pages = (const int32_t *)(dev + h->pages_at);
    p.items = (const taps_plan_item *)(dev + h->items_at);
    p.joins = (const taps_plan_join *)(dev + h->joins_at);
    p.q_token = 2 * q->stride[1], p.q_head = 2 * q->stride[2];
    p.o_token = 2 * out->stride[1], p.o_head = 2 * out->stride[2];
    p.k_page = 2 * k_cache->stride[0], p.k_head = 2 * k_cache->stride[1];
    p.k_slot = 2 * k_cache->stride[2];
    p.v_page = 2 * v_cache->stride[0], p.v_head = 2 * v_cache->stride[1];
    p.v_slot = 2 * v_cache->stride[2];
    p.n_items = h->n_items, p.n_wide = h->n_wide;
    p.n_joins = h->n_joins, p.join_rounds = h->join_rounds;
    p.q_heads = h->q_heads, p.kv_heads = h->kv_heads, p.group = h->q_heads / h->kv_heads;
    p.dim = h->head_dim;
    p.page_log2 = h->page_log2, p.causal = h->causal, p.window = h->window;
    p.scale = scale;
    return launched(taps_launch_attend(p, dtype, (hipStream_t)stream), "taps_attend");
}

const char *taps_attention_last_error(void) { return g_last_error; }

}  // extern "C"
