// taps_attend.hip -- attention of new tokens over a paged cache.
//
//   o = sum_j p_j v_j / sum_j p_j,  p_j = exp(scale (q.k_j) - m)
//
// over the keys j that a token sees, in one pass over the keys with the
// running maximum m and sum l of every query row.  A row is a pair (token,
// query head) of one key head; the rows of a sequence are numbered
// token * group + head, so that all query heads of a key head share its keys.
//
// Both products run on the matrix cores as 32x32x16 tiles with the keys on
// the first axis and the query rows on the second:
//   S^T[key][row] = K Q^T,   O^T[d][row] += V^T P^T.
// In the accumulator's layout a lane then holds 16 of a tile's 32 keys for
// one query row: the softmax needs one exchange between the two halves of a
// wavefront per tile, and P^T, rounded to the cache's type, is the second
// product's operand as it lies in the registers.  V^T comes out of LDS by the
// transposing read (four keys of one column per lane).  The order in which a
// product takes its keys is free, so the second takes them as the first left
// them.
//
// Three kinds of items, each a workgroup's:
//   wide    256 query rows, 32 for each of eight wavefronts, tiles of 64 keys;
//           the halves of the workgroup take products and softmax in turns;
//   block   128 query rows, 32 for each of four wavefronts, tiles of 64 keys;
//   narrow  up to 32 query rows; each of four wavefronts takes every fourth tile
//           of 32 keys, and the four results are joined in LDS.
// Tiles of the first two go straight from memory to LDS while the ones before
// them are in use; those of narrow items wait in registers.
// Where a sequence's keys are split over several items, each leaves its
// unnormalised result, maximum and sum, and k_join adds them up.
#include "taps_attention_internal.h"
#include "taps_lanes.h"

namespace {

constexpr int kThreads = 256, kWaves = 4, kWideThreads = 2 * kWideRows;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kMinusInf = -__builtin_inff();
// The maximum of a row that sees keys whose scores are all -inf; -inf is that of one
// that sees no key.
constexpr float kNoScore = -3.402823466e38f;
// Numerators are held as kLift exp(scale q.k - m), sums of them too; it cancels.
// fp16 has its smallest normal number at 2^-14 and nothing below 2^-25, so there
// the maximum's is placed at 2^10: keys that far below it still count, where many of
// them together outweigh it.  bf16 has the exponents of 32 bits.
// A row's maximum is raised only when a tile's numerators (this lane's 16 or 32)
// add up to more than kMostSum: none exceeds it, inside the type's range, equal
// ones do not reach it, and most tiles neither look for their maximum nor touch
// the accumulators.
template <class T> constexpr float kLift = 1.f;
template <class T> constexpr float kLiftLog2 = 0.f;
template <class T> constexpr float kMostSum = 4096.f;
template <> constexpr float kLift<_Float16> = 1024.f;
template <> constexpr float kLiftLog2<_Float16> = 10.f;
template <> constexpr float kMostSum<_Float16> = 61440.f;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

template <class T> struct Mfma;
template <> struct Mfma<__bf16> {
    typedef __bf16 v8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x16 run(s16x8 a, s16x8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, a),
                                                       __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
};
template <> struct Mfma<_Float16> {
    typedef _Float16 v8 __attribute__((ext_vector_type(8)));
    static __device__ __forceinline__ f32x16 run(s16x8 a, s16x8 b, f32x16 c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a),
                                                      __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
};

template <class T> __device__ __forceinline__ uint32_t pack2(float a, float b) {
    typedef T v2 __attribute__((ext_vector_type(2)));
    v2 v;
    v[0] = (T)a;
    v[1] = (T)b;
    return __builtin_bit_cast(uint32_t, v);
}

// A value of either half of the wavefront: v of lane % 32, v of lane % 32 + 32.
struct Halves {
    float lower, upper;
    __device__ __forceinline__ explicit Halves(float v) {
        const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v),
                                                        __builtin_bit_cast(uint32_t, v), false, false);
        const uint32_t a = r[0], b = r[1];   // scalars: a cast of r[1] itself reads r[0]
        lower = __builtin_bit_cast(float, a);
        upper = __builtin_bit_cast(float, b);
    }
};
__device__ __forceinline__ float half_max(float v) {
    const Halves h(v);
    return fmaxf(h.lower, h.upper);
}
__device__ __forceinline__ float half_sum(float v) {
    const Halves h(v);
    return h.lower + h.upper;
}

// LDS image of a tile: rows of keys without gaps, K's and then V's.  Within a
// row the 16-byte chunks are permuted by a mask of the key's number, so that
// the reads fall on different banks: K is read 16 bytes a lane at the same
// column of consecutive keys (8 or 16 of them at a time must differ), V 8
// bytes a lane, four consecutive keys at four neighbouring chunks.
template <int D> struct Tile {
    static constexpr int kChunks = D / 8, kRow = 2 * D;
    static constexpr int bytes(int keys) { return 2 * keys * kRow; }
    static __device__ __forceinline__ int k_mask(int key) {
        if (D == 128) return key & 15;
        if (D == 64) return ((key >> 1) & 3) | 4 * ((key ^ (key >> 3)) & 1);
        return (((key >> 1) & 1) | ((key >> 1) & 2)) ^ ((key >> 3) & 1);   // the low two bits
    }
    static __device__ __forceinline__ int v_mask(int key) {
        if (D == 128) return 4 * (key & 1) + 5 * (key & 2);
        if (D == 64) return 2 * (key & 1) + 2 * (key & 2);
        return key & 2;
    }
};

constexpr int max_of(int a, int b) { return a > b ? a : b; }
template <int D> constexpr int narrow_bytes() {
    return max_of(kWaves * Tile<D>::bytes(kNarrowKeys), kWaves * kNarrowRows * (D + 4) * 4) +
           kWaves * kNarrowRows * 2 * 4;
}

// The LDS address of a generic pointer to LDS.
__device__ __forceinline__ uint32_t lds_at(const char *p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const char *)p;
}

// 16 bytes a lane from memory to LDS at `lds` + 16 lane, past the registers.
// The compiler does not see the load: wait_loads() before the barrier that
// hands the tile over.
__device__ __forceinline__ void load_to_lds(const char *from, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off"
                 :
                 : "s"(lds), "v"(from)
                 : "m0", "memory");
}
// The same from a uniform address and an offset a lane.
__device__ __forceinline__ void load_to_lds(const char *from, uint32_t offset, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
                 :
                 : "s"(lds), "v"(offset), "s"(from)
                 : "m0", "memory");
}
// (the builtin, unlike an instruction in asm, tells the compiler too that no
// load of its own is under way, or it would wait again inside the loop)
// All but the newest Left loads have ended.
template <int Left> __device__ __forceinline__ void wait_loads() {
    static_assert(Left < 16, "four bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0f70 | Left);   // vmcnt(Left)
    asm volatile("" ::: "memory");
}

// A wavefront's share of a tile: groups of 16 keys, which share a page.  Lane
// by lane it takes the chunks in the order in which they lie in LDS.
template <int D> struct Group {
    static constexpr int kN = D / 32;   // 16 rows of D / 8 chunks / 64 lanes
    int key[kN], k_col[kN], v_col[kN];   // chunk numbers of the row, as permuted
    __device__ __forceinline__ explicit Group(int lane) {
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int at = lane + 64 * i;
            key[i] = at / Tile<D>::kChunks;
            const int c = at % Tile<D>::kChunks;
            k_col[i] = c ^ Tile<D>::k_mask(key[i]);
            v_col[i] = c ^ Tile<D>::v_mask(key[i]);
        }
    }
};

// Where a group of 16 keys lies; `page` is uniform.
struct Place {
    const char *k, *v;
    __device__ __forceinline__ Place(const taps_attend_launch &p, const char *k_head,
                                     const char *v_head, int page, int key) {
        const int64_t slot = key & ((1 << p.page_log2) - 1);
        k = k_head + page * p.k_page + slot * p.k_slot;
        v = v_head + page * p.v_page + slot * p.v_slot;
    }
};

// The page of key `key` of the sequence; no page before that of `lo` or after
// that of hi - 1 is looked up.  Uniform: a scalar load.
__device__ __forceinline__ int page_at(const taps_attend_launch &p, const int32_t *pages, int key,
                                       int lo, int hi) {
    const int at = __builtin_amdgcn_readfirstlane(min(max(key, lo), hi - 1) >> p.page_log2);
    return *(const __attribute__((address_space(4))) int32_t *)(uintptr_t)(pages + at);
}

// Classes of instructions of __builtin_amdgcn_sched_group_barrier.
constexpr int kMfmas = 0x8, kDsReads = 0x100;

// One wavefront's 32 query rows: the rows' operand, running statistics and result.
template <class T, int D> struct Rows {
    static constexpr int kSteps = D / 16, kBlocks = D / 32;
    s16x8 q[kSteps];
    f32x16 o[kBlocks];
    float m, l;        // maximum of the scores, this lane's half of the sum
    int first, last;   // keys of the item this lane's row sees: first .. last

    __device__ __forceinline__ void start(const taps_attend_launch &p, const taps_plan_item &item,
                                          uint32_t head, int row, int lane) {
        const bool real = row < item.rows;
        const int token = row / (int)p.group, sub = row - token * (int)p.group;
        const int pos = item.first_pos + token;
        first = item.lo;
        last = item.hi - 1;
        if (p.causal) {
            last = min(last, pos);
            if (p.window) first = max(first, pos - (int)p.window + 1);
        }
        if (!real) last = -1, first = 0;
        const char *at = p.q + (int64_t)(item.token0 + token) * p.q_token +
                         (int64_t)(head * p.group + sub) * p.q_head;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int d = 16 * k + 8 * (lane >> 5);
            q[k] = s16x8{};
            if (real && d < (int)p.dim) q[k] = *(const s16x8 *)(at + 2 * d);
        }
        m = real ? kMinusInf : 0.f;   // a row that is not there never raises it
        l = 0.f;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) o[b] = f32x16{};
    }

    // Scores of Keys keys, and the numerators they become, as the second
    // product's operands.
    template <int Keys> struct Scores {
        f32x16 s[Keys / 32];
    };
    template <int Keys> struct Numerators {
        u32x4 p[Keys / 16];
    };

    // First product: K is in LDS.
    template <int Keys>
    __device__ __forceinline__ void score(const char *k_lds, Scores<Keys> &x, int lane) const {
        const int half = lane >> 5, k_mask = Tile<D>::k_mask(lane & 31);   // the same for key + 32
#pragma unroll
        for (int n = 0; n < Keys / 32; ++n) x.s[n] = f32x16{};
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const char *at = k_lds + (lane & 31) * Tile<D>::kRow + 16 * ((2 * k + half) ^ k_mask);
#pragma unroll
            for (int n = 0; n < Keys / 32; ++n)
                x.s[n] = Mfma<T>::run(*(const s16x8 *)(at + 32 * n * Tile<D>::kRow), q[k], x.s[n]);
        }
    }

    // Hides the keys this row does not see (t0: the first key's number).
    template <int Keys>
    __device__ __forceinline__ void hide(Scores<Keys> &x, int t0, int lane) const {
        const uint32_t seen = max(last - first + 1, 0), at = t0 + 4 * (lane >> 5) - first;
#pragma unroll
        for (int n = 0; n < Keys / 32; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                x.s[n][i] = at + (32 * n + 8 * (i / 4) + i % 4) < seen ? x.s[n][i] : kMinusInf;
    }

    // Hides keys where a tile needs it and makes the numerators from the maximum
    // as it is; only where their sum shows that it lies too far below a score is
    // it raised and are they made anew.  `c` = scale log2 e.
    template <int Keys>
    __device__ __forceinline__ void soften(Scores<Keys> &x, Numerators<Keys> &y, int t0, bool masked,
                                           float c, int lane) {
        if (masked) hide(x, t0, lane);
        float sum = numerators(x, y, c);
        // the first keys, and scores too far above the maximum
        if (__any(m == kMinusInf || sum > kMostSum<T>)) {
            float most = x.s[0][0];
#pragma unroll
            for (int n = 0; n < Keys / 32; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) most = fmaxf(most, x.s[n][i]);
            const float to = fmaxf(m, half_max(most));
            const float by = to == kMinusInf ? 1.f : __builtin_amdgcn_exp2f((m - to) * c);
            m = to;
            l *= by;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[b][i] *= by;
            sum = numerators(x, y, c);
        }
        l += sum;
    }
    // They are rounded for the product with the values, which takes operands of the
    // cache's type only: an error of up to 2^-8 (bf16) or 2^-11 of each, independent of
    // each other and no larger than the values' own, and in fp16 of 2^-35 of the largest
    // for those below 2^-24 of it.  Their sum is taken before, in 32 bits.
    template <int Keys>
    __device__ __forceinline__ float numerators(const Scores<Keys> &x, Numerators<Keys> &y,
                                                float c) const {
        const float shift = m <= kNoScore ? 0.f : m * c - kLiftLog2<T>;
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int n = 0; n < Keys / 32; ++n)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float e = __builtin_amdgcn_exp2f(x.s[n][2 * i] * c - shift);
                const float f = __builtin_amdgcn_exp2f(x.s[n][2 * i + 1] * c - shift);
                sum[0] += e, sum[1] += f;
                y.p[2 * n + i / 4][i % 4] = pack2<T>(e, f);
            }
        return sum[0] + sum[1];
    }

    // Second product: V is in LDS.
    template <int Keys>
    __device__ __forceinline__ void spend(const char *v_lds, const Numerators<Keys> &y, int lane) {
        constexpr int kRow = Tile<D>::kRow;
        const int half = lane >> 5;
        // lane of a group of 16: key (lane % 16) / 4, columns 4 (lane % 4) ..
        const int v_key = 4 * half + (lane & 15) / 4;
        const int v_chunk = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
        const int v_mask = Tile<D>::v_mask(v_key);   // the same for keys 8 and 16 further
        const char *v0 = v_lds + v_key * kRow + 8 * (lane & 1);
#pragma unroll
        for (int n = 0; n < Keys / 16; ++n)
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) {
                const char *at = v0 + 16 * ((4 * b + v_chunk) ^ v_mask) + 16 * n * kRow;
                const s16x4 u = transposed(at), w = transposed(at + 8 * kRow);
                const s16x8 va = {u[0], u[1], u[2], u[3], w[0], w[1], w[2], w[3]};
                o[b] = Mfma<T>::run(va, __builtin_bit_cast(s16x8, y.p[n]), o[b]);
            }
    }

    // Both: the last tile's numerators by its values, this tile's scores.  The
    // reads of LDS run kAhead operands ahead of the products, which the scheduler
    // would not do by itself (it waited for each pair: 1700 clocks for 32
    // products of 32 clocks, 1300 so).
    template <int Keys>
    __device__ __forceinline__ void products(const char *v_lds, const Numerators<Keys> &y,
                                             const char *k_lds, Scores<Keys> &x, int lane) {
        constexpr int kV = Keys / 16 * kBlocks, kK = Keys / 32 * kSteps, kAhead = 6;
        // before the other wavefront's softmax, which finds issue slots enough between the products
        __builtin_amdgcn_s_setprio(1);
        __builtin_amdgcn_sched_barrier(0);
        spend(v_lds, y, lane);
        score(k_lds, x, lane);
        __builtin_amdgcn_sched_group_barrier(kDsReads, 2 * kAhead, 0);
#pragma unroll
        for (int i = kAhead; i < kV; ++i) {
            __builtin_amdgcn_sched_group_barrier(kMfmas, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kDsReads, 2, 0);
        }
#pragma unroll
        for (int i = 0; i < kK; ++i) {
            __builtin_amdgcn_sched_group_barrier(kMfmas, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kDsReads, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kMfmas, kAhead, 0);
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(0);
    }

    // The sum of its row's numerators, of both lanes; ends the statistics.
    __device__ __forceinline__ float total() {
        const float sum = half_sum(l);
        if (sum == 0.f && m == kMinusInf && first <= last) m = kNoScore;
        return sum;
    }
    // Whether this lane's part of its row's result is not finite.
    __device__ __forceinline__ bool broken() const {
        float sum = 0.f;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) sum += o[b][i] * 0.f;
        return sum != sum;
    }

    static __device__ __forceinline__ s16x4 transposed(const char *at) {
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4 *)at);
    }
};

// Ends a phase of a wide item for all its wavefronts.  Products and
// exponentials do not move from one phase into another.
__device__ __forceinline__ void end_phase() {
    __builtin_amdgcn_sched_barrier(0);
    __syncthreads();
    __builtin_amdgcn_sched_barrier(0);
}

// Where a row's result goes.
template <class T>
__device__ __forceinline__ char *out_row(const taps_attend_launch &p, const taps_plan_item &s,
                                         uint32_t head, int row) {
    const int token = row / (int)p.group, sub = row - token * (int)p.group;
    return p.out + (int64_t)(s.token0 + token) * p.o_token +
           (int64_t)(head * p.group + sub) * p.o_head;
}

// What turns a row's sum of numerators by values into its result.
__device__ __forceinline__ float inverse(float m, float l) {
    return l != 0.f ? 1.f / l : m == kMinusInf ? 0.f : __builtin_nanf("");
}

template <class T>
__device__ __forceinline__ void store_lse(const taps_attend_launch &p, const taps_plan_item &s,
                                          uint32_t head, int row, float m, float l) {
    if (!p.lse) return;
    const int token = row / (int)p.group, sub = row - token * (int)p.group;
    p.lse[(int64_t)(s.token0 + token) * p.q_heads + head * p.group + sub] =
        l != 0.f         ? m * p.scale + __builtin_amdgcn_logf(l / kLift<T>) * kLn2
        : m == kMinusInf ? kMinusInf
                         : __builtin_nanf("");
}

template <class T, int D>
__device__ __forceinline__ void write_rows(const taps_attend_launch &p, const taps_plan_item &item,
                                           uint32_t head, const Rows<T, D> &rows, int row, float l,
                                           int half) {
    constexpr int kBlocks = D / 32;
    if (item.part < 0) {
        const float inv = inverse(rows.m, l);
        char *out = out_row<T>(p, item, head, row);
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = 32 * b + 8 * i + 4 * half;
                const u32x2 v = {pack2<T>(rows.o[b][4 * i] * inv, rows.o[b][4 * i + 1] * inv),
                                 pack2<T>(rows.o[b][4 * i + 2] * inv, rows.o[b][4 * i + 3] * inv)};
                if (d < (int)p.dim) *(u32x2 *)(out + 2 * d) = v;
            }
        if (half == 0) store_lse<T>(p, item, head, row, rows.m, l);
    } else {
        const int64_t at = (int64_t)(item.part + row - item.row0) * p.kv_heads + head;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int d = 32 * b + 8 * i + 4 * half;
                const f32x4 v = {rows.o[b][4 * i], rows.o[b][4 * i + 1], rows.o[b][4 * i + 2],
                                 rows.o[b][4 * i + 3]};
                if (d < (int)p.dim) *(f32x4 *)(p.part_o + at * p.dim + d) = v;
            }
        if (half == 0) p.part_ml[2 * at] = rows.m, p.part_ml[2 * at + 1] = l;
    }
}

// The keys that all 32 rows from `row0` on see, of the item's: a tile outside
// needs a mask.  A wavefront does nothing with the tiles from `end` on but load
// its part of them: a branch within the loop costs the other tiles 64 register
// moves each, a second loop behind it nothing (prompts of 2048: 364 -> 350 us,
// 1024 of 16 heads of 64: 36 -> 33).
struct Seen {
    int from, to;
    int end;   // no row sees a key from here on
    __device__ __forceinline__ Seen(const taps_attend_launch &p, const taps_plan_item &item,
                                    int row0) {
        from = item.lo, to = item.hi - 1, end = row0 < item.rows ? item.hi : item.lo;
        if (!p.causal || item.rows <= (int)p.group) return;   // all rows see the item's keys
        const int a = min(row0, item.rows - 1), b = min(row0 + 31, item.rows - 1);
        end = min(end, item.first_pos + b / (int)p.group + 1);
        to = min(to, item.first_pos + a / (int)p.group);
        if (p.window) from = max(from, item.first_pos + b / (int)p.group - (int)p.window + 1);
    }
    __device__ __forceinline__ bool masks(int t0, int keys) const {
        return t0 < from || t0 + keys - 1 > to;
    }
    // Whether one of the rows does not see a key of the item, which then may be in its
    // tiles for the sake of another row, be it another wavefront's.
    __device__ __forceinline__ bool differ(const taps_plan_item &item) const {
        return from > item.lo || to < item.hi - 1;
    }
};

// The rows of `again` once more, from tiles of 32 keys at t0, t0 + step ..  In the
// matrix products the numerator of a key that a row does not see, 0, meets the key's
// values, which another row of the tile sees; if one is infinite or NaN, so is the
// product, and the row is found by that.  Where all rows see a tile nothing of the kind
// can happen: those are taken as before, only from memory.  In the others the values
// that a row does not see are made zeros, row by row.  m and l do not depend on values.
// (A prompt of 2048, 8 heads of 128 over 4, whose first value is infinite, so that all
// rows are done again: 249 us, 39 without; a row and a key at a time took 9.9 ms.)
// Behind the kernels' other code: between it, it cost a lone token 0.7 us.
template <class T, int D>
__device__ __forceinline__ void redo(const taps_attend_launch &p, const taps_plan_item &item,
                                     uint32_t head, Rows<T, D> &rows, uint32_t again,
                                     const Seen &seen, int t0, int step, int lane) {
    constexpr int kSteps = D / 16, kBlocks = D / 32;
    using R = Rows<T, D>;
    const int half = lane >> 5, lo = item.lo, hi = min(item.hi, seen.end), dim = p.dim;
    const char *k_head = p.k_cache + (int64_t)head * p.k_head;
    const char *v_head = p.v_cache + (int64_t)head * p.v_head;
    const float c = p.scale * kLog2e;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) rows.o[b] = f32x16{};
    for (; lo < hi && t0 < hi; t0 += step) {
        // two groups of 16 keys; of one that lies outside, and of keys outside, the nearest inside
        const char *k_at[2], *v_at[2];
        int key0[2];
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            key0[n] = min(max(t0 + 16 * n, lo & ~15), (hi - 1) & ~15);
            const Place at(p, k_head, v_head, page_at(p, p.pages + item.page0, key0[n], lo, hi),
                           key0[n]);
            k_at[n] = at.k, v_at[n] = at.v;
        }
        const auto in = [&](int key) { return key >= lo && key < hi; };
        const auto slot_of = [&](int key, int n) {
            return (uint32_t)(min(max(key, lo), hi - 1) - key0[n]);
        };
        typename R::template Scores<32> x;
        typename R::template Numerators<32> y;
        x.s[0] = f32x16{};
        {
            const int key = t0 + (lane & 31), n = (lane >> 4) & 1;
            const char *row = (n ? k_at[1] : k_at[0]) +
                              (n ? slot_of(key, 1) : slot_of(key, 0)) * (uint32_t)p.k_slot;
#pragma unroll
            for (int k = 0; k < kSteps; ++k) {
                const int d = 16 * k + 8 * half;
                s16x8 a = *(const s16x8 *)(row + 2 * (d < dim ? d : 0));
                if (!in(key) || d >= dim) a = s16x8{};
                x.s[0] = Mfma<T>::run(a, rows.q[k], x.s[0]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        rows.hide(x, t0, lane);
        rows.numerators(x, y, c);
        const bool masked = seen.masks(t0, 32);
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) {
            const int d = 32 * b + (lane & 31);
            s16x8 v[2];   // column d of the keys of the numerators
            // this path is rare and the kernels' registers are few: no address is kept, no load moved
            uint32_t slot = (uint32_t)p.v_slot;
            asm volatile("" : "+s"(slot));
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int key = t0 + 16 * n + 8 * (e / 4) + 4 * half + e % 4;
                    const short u = *(const short *)(v_at[n] + slot_of(key, n) * slot +
                                                     2 * (d < dim ? d : 0));
                    v[n][e] = in(key) && d < dim ? u : (short)0;
                    if (e % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                }
            if (!masked) {
#pragma unroll
                for (int n = 0; n < 2; ++n)
                    rows.o[b] = Mfma<T>::run(v[n], __builtin_bit_cast(s16x8, y.p[n]), rows.o[b]);
                continue;
            }
            for (uint32_t left = again; left; left &= left - 1) {
                const int r = __builtin_ctz(left);
                const int first = __shfl(rows.first, r, 64), last = __shfl(rows.last, r, 64);
                f32x16 o = {};
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    s16x8 w;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int key = t0 + 16 * n + 8 * (e / 4) + 4 * half + e % 4;
                        w[e] = key >= first && key <= last ? v[n][e] : (short)0;
                    }
                    o = Mfma<T>::run(w, __builtin_bit_cast(s16x8, y.p[n]), o);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    rows.o[b][i] = (lane & 31) == r ? rows.o[b][i] + o[i] : rows.o[b][i];
            }
        }
    }
}

// Hands the results of a wavefront's 32 rows to write(), for some lanes' rows at a
// time; `row` is this lane's, `l` the sum of both its halves, t0 and step the
// wavefront's tiles (32 keys each) in the item.
template <class T, int D, class F>
__device__ __forceinline__ void finish(const taps_attend_launch &p, const taps_plan_item &item,
                                       uint32_t head, Rows<T, D> &rows, const Seen &seen, int row,
                                       float l, int t0, int step, int lane, F &&write) {
    uint32_t again = 0;   // rows to redo: either half of their results is not finite, by values
    if (seen.differ(item)) {
        const uint64_t broken = __ballot(row < item.rows && l == l && rows.broken());
        again = (uint32_t)broken | (uint32_t)(broken >> 32);
    }
    const bool mine = again >> (lane & 31) & 1;
    if (!mine) write();
    if (__builtin_expect(again == 0, 1)) return;
    redo(p, item, head, rows, again, seen, t0, step, lane);
    if (mine) write();
}

// Loads to LDS: a wavefront takes 16 of a tile's 64 keys, of K or of V.  Keys
// outside lo .. hi - 1 and columns beyond the head come from a block of zeros in
// the plan: what memory holds in their place (it may never have been written)
// must not reach a product.
template <int D> struct Loader {
    static constexpr int kN = Group<D>::kN;   // loads of a tile's K or V
    const char *head, *zeros;
    int64_t page_stride, slot_stride;
    int key0, lo, hi, dim, page_log2;
    uint32_t offset[kN];   // of this lane's chunks in a group
    int key_col[kN];       // 16 x chunk number + key
    __device__ __forceinline__ Loader(const taps_attend_launch &p, const taps_plan_item &item,
                                      uint32_t h, bool v, int wave, int lane) {
        head = v ? p.v_cache + (int64_t)h * p.v_head : p.k_cache + (int64_t)h * p.k_head;
        page_stride = v ? p.v_page : p.k_page, slot_stride = v ? p.v_slot : p.k_slot;
        zeros = p.zeros;
        key0 = 16 * (wave & 3), lo = item.lo, hi = item.hi, dim = p.dim, page_log2 = p.page_log2;
        const Group<D> g(lane);
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            const int col = v ? g.v_col[i] : g.k_col[i];
            offset[i] = g.key[i] * (uint32_t)slot_stride + 16 * col;
            key_col[i] = 16 * col + g.key[i];
        }
    }
    // The wavefront's keys of the tile from key t0 on, to `part` (K or V of a tile).
    __device__ __forceinline__ void load(int t0, int page, const char *part) const {
        const int key = t0 + key0;
        const char *at = head + page * page_stride +
                         (int64_t)(key & ((1 << page_log2) - 1)) * slot_stride;
        const uint32_t to = __builtin_amdgcn_readfirstlane(lds_at(part) + key0 * Tile<D>::kRow);
        if (dim == D && key >= lo && key + 16 <= hi) {
#pragma unroll
            for (int i = 0; i < kN; ++i) load_to_lds(at, offset[i], to + 1024 * i);
        } else {
#pragma unroll
            for (int i = 0; i < kN; ++i) {
                const int j = key + (key_col[i] & 15), col = key_col[i] >> 4;
                load_to_lds(j >= lo && j < hi && 8 * col < dim ? at + offset[i] : zeros,
                            to + 1024 * i);
            }
        }
    }
};

// 256 query rows, 32 a wavefront; a unit has one workgroup at a time.  A tile takes
// two phases: products (the numerators of the last tile by its values, the scores
// of this one), and softmax.  While the first four wavefronts, one on each SIMD,
// are in one of them, the others are in the other, so that the matrix cores
// have a wavefront of their own at any time and a tile's loads serve twice the
// rows of a block item.
// 512 tokens over 32768 keys, 32 heads of 128 over 8: 243 us here, 1120 TFLOP/s (279
// in blocks), the matrix cores busy for 58 % of the cycles at 1.9 GHz; the phases that
// wait for each other take the rest.  The products alone, without loads, softmax and
// reads of LDS, reach 1377 at the clocks that they leave, so a fifth is the most
// there is to win.  Eight sequences of 2048 tokens, 32 heads, not causal, take 0.21 us a
// key, 1280 TFLOP/s, and 90 us that do not grow with the keys.  Loading the next item's
// first tiles and queries while the last ends wins none of those back (one workgroup
// a unit that stays: 364 and 360 us).  Causal, a wavefront waits besides for the
// tiles behind its last key that the strip's last one sees: 112 keys on average, a
// tenth of the time for prompts of 2048.
template <class T, int D>
__global__ __launch_bounds__(kWideThreads, 2) void k_attend_wide(taps_attend_launch p) {
    constexpr int kPart = kWideKeys * Tile<D>::kRow;   // a tile's K, or its V
    __shared__ __attribute__((aligned(16))) char lds[6 * kPart];
    const uint32_t head = blockIdx.x % p.kv_heads;
    const taps_plan_item item = p.items[blockIdx.x / p.kv_heads];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool second = wave >= 4;   // the workgroup's second half
    const int32_t *pages = p.pages + item.page0;
    const int start = item.lo & ~15;   // whole groups of 16 share a page
    const float c = p.scale * kLog2e;
    const int row0 = item.row0 + 32 * wave, row = row0 + (lane & 31);
    Rows<T, D> rows;
    rows.start(p, item, head, row, lane);
    const Seen seen(p, item, row0);
    if (item.lo < item.hi) {
        // Both halves use all tiles that they see; the first loads K, the other V.  K of tile i is read in phases
        // 2 i and 2 i + 1, V in the two after them.  Three tiles of each are kept: K of tile i + 2
        // is loaded in phase 2 i + 1, V of tile i + 1 in phase 2 i.
        typename Rows<T, D>::template Scores<kWideKeys> x;
        typename Rows<T, D>::template Numerators<kWideKeys> y;
        const Loader<D> loader(p, item, head, second, wave, lane);
        const char *k_lds = lds, *v_lds = lds + 3 * kPart;
        const int tiles = (item.hi - start + kWideKeys - 1) / kWideKeys;
        const int used = min(max((seen.end - start + kWideKeys - 1) / kWideKeys, 1), tiles);
        const auto tile0 = [&](int i) { return start + i * kWideKeys; };
        const auto page_of = [&](int t0) {
            return page_at(p, pages, t0 + loader.key0, item.lo, item.hi);
        };
        const auto soften = [&](int t0) {
            rows.soften(x, y, t0, seen.masks(t0, kWideKeys), c, lane);
        };
        // buffers: of tiles i - 1, i, i + 1 in the first half's loop, i - 2, i - 1, i in the
        // other's; the oldest is loaded anew
        int b0 = 2, b1 = 0, b2 = 1;
        const auto turn = [&]() {
            const int b = b0;
            b0 = b1, b1 = b2, b2 = b;
        };
        const auto wait = [&](bool newer) {
            if (newer)
                wait_loads<Loader<D>::kN>();
            else
                wait_loads<0>();
        };
        const char *mine = second ? v_lds : k_lds;
        loader.load(tile0(0), page_of(tile0(0)), mine);
        if (tiles > 1) loader.load(tile0(1), page_of(tile0(1)), mine + kPart);
        int page = page_of(tile0(2));
        wait_loads<0>();
        end_phase();
        if (!second) {
            for (int i = 0; i < used; ++i, turn()) {
                if (i)
                    rows.products(v_lds + b0 * kPart, y, k_lds + b1 * kPart, x, lane);
                else
                    rows.score(k_lds, x, lane);
                end_phase();
                if (i + 2 < tiles) loader.load(tile0(i + 2), page, k_lds + b0 * kPart);
                page = page_of(tile0(i + 3));
                soften(tile0(i));
                wait(i + 2 < tiles);
                end_phase();
            }
            rows.spend(v_lds + b0 * kPart, y, lane);   // the last tile's
            for (int i = used; i < tiles; ++i, turn()) {
                end_phase();
                if (i + 2 < tiles) loader.load(tile0(i + 2), page, k_lds + b0 * kPart);
                page = page_of(tile0(i + 3));
                wait(i + 2 < tiles);
                end_phase();
            }
        } else {
            end_phase();
            rows.score(k_lds, x, lane);
            end_phase();
            int i = 1;
            const auto begin = [&]() {
                if (i + 1 < tiles) loader.load(tile0(i + 1), page, v_lds + b0 * kPart);
                page = page_of(tile0(i + 2));
            };
            for (; i < used; ++i, turn()) {
                begin();
                soften(tile0(i - 1));
                end_phase();
                rows.products(v_lds + b1 * kPart, y, k_lds + b2 * kPart, x, lane);
                wait(i + 1 < tiles);
                end_phase();
            }
            begin();
            soften(tile0(used - 1));
            if (used < tiles) end_phase();
            rows.spend(v_lds + b1 * kPart, y, lane);
            for (; i < tiles; ++i, turn()) {
                if (i > used) {
                    begin();
                    end_phase();
                }
                wait(i + 1 < tiles);
                end_phase();
            }
        }
    }
    const float l = rows.total();
    finish(p, item, head, rows, seen, row, l, start, 32, lane, [&]() {
        if (row < item.rows) write_rows(p, item, head, rows, row, l, lane >> 5);
    });
}

// 128 query rows, 32 a wavefront, two workgroups to a unit (three for heads of up to
// 64), which fill each other's gaps.  Tiles of 64 keys in two buffers, one loaded
// while the other is in use.  Eight prompts of 1024, 16 heads of 64: 33 us, of which
// the products alone would take 13 and the bytes 14; short rounds with a start and
// an end each bound it.  (Four wavefronts a SIMD, with 128 registers: 49 for 37.)
template <class T, int D>
__device__ __forceinline__ void attend_block(const taps_attend_launch &p, const taps_plan_item &item,
                                             uint32_t head, char *lds) {
    constexpr int kPart = kWideKeys * Tile<D>::kRow;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t *pages = p.pages + item.page0;
    const int start = item.lo & ~15;
    // no tile of an item without keys: its lo need not be a multiple of 16
    const int hi = item.lo < item.hi ? item.hi : start;
    const float c = p.scale * kLog2e;
    const int row0 = item.row0 + 32 * wave, row = row0 + (lane & 31);
    Rows<T, D> rows;
    rows.start(p, item, head, row, lane);
    const Seen seen(p, item, row0);
    const Loader<D> k(p, item, head, false, wave, lane), v(p, item, head, true, wave, lane);
    const auto page_of = [&](int t0) { return page_at(p, pages, t0 + k.key0, item.lo, item.hi); };
    int page = 0, buffer = 0;
    if (start < hi) {
        page = page_of(start);
        k.load(start, page, lds);
        v.load(start, page, lds + kPart);
        page = page_of(start + kWideKeys);
    }
    int t0 = start;
    // one barrier a tile: the tile's loads have ended in every wavefront, and every
    // wavefront is done with the other buffer
    const auto begin = [&]() {
        const char *next = lds + 2 * (buffer ^ 1) * kPart;
        wait_loads<0>();
        __syncthreads();
        if (t0 + kWideKeys < hi) {
            k.load(t0 + kWideKeys, page, next);
            v.load(t0 + kWideKeys, page, next + kPart);
            page = page_of(t0 + 2 * kWideKeys);
        }
    };
    for (; t0 < min(hi, seen.end); t0 += kWideKeys, buffer ^= 1) {
        const char *tile = lds + 2 * buffer * kPart;
        begin();
        typename Rows<T, D>::template Scores<kWideKeys> x;
        typename Rows<T, D>::template Numerators<kWideKeys> y;
        rows.score(tile, x, lane);
        rows.soften(x, y, t0, seen.masks(t0, kWideKeys), c, lane);
        rows.spend(tile + kPart, y, lane);
    }
    for (; t0 < hi; t0 += kWideKeys, buffer ^= 1) begin();   // the other wavefronts' tiles
    const float l = rows.total();
    finish(p, item, head, rows, seen, row, l, start, 32, lane, [&]() {
        if (row < item.rows) write_rows(p, item, head, rows, row, l, lane >> 5);
    });
}

// Up to 32 query rows: every wavefront has all of them and its own keys, so that
// a unit has eight tiles on their way at any time.  Bytes bound it: 64 tokens over 2 to
// 4000 keys each, 32 heads of 128 over 8, 104 us and 5 for the join, 5.3 TB/s; two
// over 131001, 183 and 5, 5.9 TB/s.
template <class T, int D>
__device__ __forceinline__ void attend_narrow(const taps_attend_launch &p,
                                              const taps_plan_item &item, uint32_t head, char *lds) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t *pages = p.pages + item.page0;
    const char *k_head = p.k_cache + (int64_t)head * p.k_head;
    const char *v_head = p.v_cache + (int64_t)head * p.v_head;
    const int lo = item.lo, hi = item.hi, start = lo & ~15;
    const float c = p.scale * kLog2e;
    constexpr int kBlocks = D / 32;
    const int half = lane >> 5;
    Rows<T, D> rows;
    rows.start(p, item, head, item.row0 + (lane & 31), lane);
    const Seen seen(p, item, item.row0);
    {
        char *tile = lds + wave * Tile<D>::bytes(kNarrowKeys);
        // The next tile, two groups of 16 keys, waits in registers; keys outside lo .. hi - 1 are
        // loaded from an end of that range and become zeros on the way to LDS, as do columns
        // beyond the head.
        const Group<D> g(lane);
        constexpr int kN = Group<D>::kN;
        u32x4 kr[2][kN], vr[2][kN];
        const bool ragged = p.dim < D;
        const auto load = [&](int t0, int page0, int page1) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                // a group wholly outside: the address of the nearest key's group inside
                const int key = min(max(t0 + 16 * h, start), (hi - 1) & ~15);
                const Place at(p, k_head, v_head, h ? page1 : page0, key);
#pragma unroll
                for (int i = 0; i < kN; ++i) {
                    const int row = min(max(key + g.key[i], lo), hi - 1) - key;
                    const int kc = ragged && 8 * g.k_col[i] >= (int)p.dim ? 0 : g.k_col[i];
                    const int vc = ragged && 8 * g.v_col[i] >= (int)p.dim ? 0 : g.v_col[i];
                    kr[h][i] = *(const u32x4 *)(at.k + row * p.k_slot + 16 * kc);
                    vr[h][i] = *(const u32x4 *)(at.v + row * p.v_slot + 16 * vc);
                }
            }
        };
        int t0 = start + kNarrowKeys * wave, page0 = 0, page1 = 0;
        constexpr int kStep = kWaves * kNarrowKeys;
        if (lo < hi && t0 < hi) {
            load(t0, page_at(p, pages, t0, lo, hi), page_at(p, pages, t0 + 16, lo, hi));
            page0 = page_at(p, pages, t0 + kStep, lo, hi);
            page1 = page_at(p, pages, t0 + kStep + 16, lo, hi);
        }
        for (; lo < hi && t0 < hi; t0 += kStep) {
            const bool whole = !ragged && t0 >= lo && t0 + kNarrowKeys <= hi;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < kN; ++i) {
                    const int key = 16 * h + g.key[i];
                    u32x4 k = kr[h][i], v = vr[h][i];
                    if (!whole) {
                        const bool in = t0 + key >= lo && t0 + key < hi;
                        k = in && 8 * g.k_col[i] < (int)p.dim ? k : u32x4{};
                        v = in && 8 * g.v_col[i] < (int)p.dim ? v : u32x4{};
                    }
                    char *to = tile + 16 * h * Tile<D>::kRow + 16 * (lane + 64 * i);
                    *(u32x4 *)to = k;
                    *(u32x4 *)(to + kNarrowKeys * Tile<D>::kRow) = v;
                }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            if (t0 + kStep < hi) {
                load(t0 + kStep, page0, page1);
                page0 = page_at(p, pages, t0 + 2 * kStep, lo, hi);
                page1 = page_at(p, pages, t0 + 2 * kStep + 16, lo, hi);
            }
            const bool masked = seen.masks(t0, kNarrowKeys);
            typename Rows<T, D>::template Scores<kNarrowKeys> x;
            typename Rows<T, D>::template Numerators<kNarrowKeys> y;
            rows.score(tile, x, lane);
            rows.soften(x, y, t0, masked, c, lane);
            rows.spend(tile + kNarrowKeys * Tile<D>::kRow, y, lane);
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
    }
    float *ml = (float *)(lds + narrow_bytes<D>() - 2 * kWaves * kNarrowRows * 4);
    const float l_wave = rows.total();
    __syncthreads();   // the tiles are done with
    if (half == 0) {
        ml[2 * (wave * kNarrowRows + lane)] = rows.m;
        ml[2 * (wave * kNarrowRows + lane) + 1] = l_wave;
    }
    __syncthreads();
    float m = kMinusInf;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, ml[2 * (w * kNarrowRows + (lane & 31))]);
    float *sums = (float *)lds;   // [wave][row][D + 4]
    const auto leave = [&]() {
        const float by = rows.m == kMinusInf ? 0.f : __builtin_amdgcn_exp2f((rows.m - m) * c);
        float *at = sums + (wave * kNarrowRows + (lane & 31)) * (D + 4);
#pragma unroll
        for (int b = 0; b < kBlocks; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 v = {rows.o[b][4 * i] * by, rows.o[b][4 * i + 1] * by,
                                 rows.o[b][4 * i + 2] * by, rows.o[b][4 * i + 3] * by};
                *(f32x4 *)(at + 32 * b + 8 * i + 4 * half) = v;
            }
    };
    finish(p, item, head, rows, seen, item.row0 + (lane & 31), l_wave, start + kNarrowKeys * wave,
           kWaves * kNarrowKeys, lane, leave);
    __syncthreads();
    const int n_rows = min(kNarrowRows, item.rows - item.row0);
    const auto result = [&](int r, int d) {
        f32x4 o = {};
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
            o += *(const f32x4 *)(sums + (w * kNarrowRows + r) * (D + 4) + d);
        return o;
    };
    const auto statistics = [&](int r, float &top, float &l) {
        top = kMinusInf, l = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) top = fmaxf(top, ml[2 * (w * kNarrowRows + r)]);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float mw = ml[2 * (w * kNarrowRows + r)], lw = ml[2 * (w * kNarrowRows + r) + 1];
            l += mw == kMinusInf ? lw : lw * __builtin_amdgcn_exp2f((mw - top) * c);
        }
    };
    for (int k = threadIdx.x; k < n_rows * (D / 4); k += kThreads) {
        const int r = k / (D / 4), d = 4 * (k % (D / 4));
        if (d >= (int)p.dim) continue;
        float top, l;
        statistics(r, top, l);
        const f32x4 o = result(r, d);
        if (item.part < 0) {
            const float inv = inverse(top, l);
            char *out = out_row<T>(p, item, head, item.row0 + r);
            const u32x2 v = {pack2<T>(o[0] * inv, o[1] * inv), pack2<T>(o[2] * inv, o[3] * inv)};
            *(u32x2 *)(out + 2 * d) = v;
            if (d == 0) store_lse<T>(p, item, head, item.row0 + r, top, l);
        } else {
            const int64_t at = (int64_t)(item.part + r) * p.kv_heads + head;
            *(f32x4 *)(p.part_o + at * p.dim + d) = o;
            if (d == 0) p.part_ml[2 * at] = top, p.part_ml[2 * at + 1] = l;
        }
    }
}

// A block or a narrow item; both fit a unit twice.
template <class T, int D>
__global__ __launch_bounds__(kThreads, 2) void k_attend(taps_attend_launch p) {
    __shared__ __attribute__((aligned(16))) char lds[max_of(narrow_bytes<D>(),
                                                            2 * Tile<D>::bytes(kWideKeys))];
    const uint32_t head = blockIdx.x % p.kv_heads;
    const taps_plan_item item = p.items[blockIdx.x / p.kv_heads];
    if (item.kind == kBlock)
        attend_block<T, D>(p, item, head, lds);
    else
        attend_narrow<T, D>(p, item, head, lds);
}

// Adds up the pieces of rows whose keys were split.  A group of 32 lanes, four
// elements a lane, takes every `across`-th piece of a row, four at a time; the
// groups of a row meet in LDS.  With one group a row and one row after the
// other in a workgroup, 2048 rows x 8 heads in 4 pieces took 62 us and 4 rows x
// 8 heads in 32 pieces 28, waiting for one load after the other; so 8.2 and 4.7
// (13 with a group for each of the 4 pieces, for four times the workgroups).
constexpr int kJoinGroups = kThreads / 32;

template <class T>
__global__ __launch_bounds__(kThreads) void k_join(taps_attend_launch p) {
    __shared__ f32x4 sums[kJoinGroups][32];
    __shared__ float ms[kJoinGroups], ls[kJoinGroups];
    const taps_plan_join join = p.joins[blockIdx.x];
    taps_plan_item item{};
    item.token0 = join.token0;
    const uint32_t head = blockIdx.y;
    const float c = p.scale * kLog2e;
    const int group = threadIdx.x >> 5, d = 4 * (threadIdx.x & 31);
    const int across = taps_join_across(join.parts);
    const int r = blockIdx.z * (kJoinGroups / across) + group / across;
    const bool live = d < (int)p.dim;
    float m = kMinusInf, l = 0.f;
    f32x4 o = {};
    if (r < join.rows) {
        constexpr int kAtOnce = 4;
        for (int k0 = group % across; k0 < join.parts; k0 += across * kAtOnce) {
            float mk[kAtOnce], lk[kAtOnce];
            f32x4 ok[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int k = k0 + u * across;
                mk[u] = kMinusInf, lk[u] = 0.f, ok[u] = f32x4{};
                if (k < join.parts) {
                    const int64_t at = (int64_t)(join.part + k * join.rows + r) * p.kv_heads + head;
                    mk[u] = p.part_ml[2 * at];
                    lk[u] = p.part_ml[2 * at + 1];
                    if (live) ok[u] = *(const f32x4 *)(p.part_o + at * p.dim + d);
                }
            }
            float to = m;
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) to = fmaxf(to, mk[u]);
            // a piece without keys has nothing (or NaN) to add at any scale
            const float by = m == kMinusInf ? 1.f : __builtin_amdgcn_exp2f((m - to) * c);
            l *= by, o *= by, m = to;
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const float w = mk[u] == kMinusInf ? 1.f : __builtin_amdgcn_exp2f((mk[u] - m) * c);
                l += lk[u] * w;
                o += ok[u] * w;
            }
        }
    }
    sums[group][threadIdx.x & 31] = o;
    if ((threadIdx.x & 31) == 0) ms[group] = m, ls[group] = l;
    __syncthreads();
    if (r >= join.rows || group % across != 0) return;
    for (int g = group + 1; g < group + across; ++g) m = fmaxf(m, ms[g]);
    l = 0.f, o = f32x4{};
    for (int g = group; g < group + across; ++g) {
        const float w = ms[g] == kMinusInf ? 1.f : __builtin_amdgcn_exp2f((ms[g] - m) * c);
        l += ls[g] * w;
        o += sums[g][threadIdx.x & 31] * w;
    }
    const float inv = inverse(m, l);
    if (live) {
        char *out = out_row<T>(p, item, head, join.row0 + r);
        const u32x2 v = {pack2<T>(o[0] * inv, o[1] * inv), pack2<T>(o[2] * inv, o[3] * inv)};
        *(u32x2 *)(out + 2 * d) = v;
    }
    if (d == 0) store_lse<T>(p, item, head, join.row0 + r, m, l);
}

// Launches of as many of n items as a grid's dimension, fewer than 2^32 threads, holds.
template <class F>
void in_slices(taps_attend_launch p, uint32_t n, int threads, F &&launch_slice) {
    const uint32_t most = max(0xffffffffu / threads / p.kv_heads, 1u);
    for (; n; n -= min(n, most), p.items += most) launch_slice(p, min(n, most) * p.kv_heads);
}

template <class T, int D> void launch_items(taps_attend_launch p, hipStream_t stream) {
    if constexpr (D > kWideAbove)
        in_slices(p, p.n_wide, kWideThreads, [&](const taps_attend_launch &s, uint32_t groups) {
            k_attend_wide<T, D><<<groups, kWideThreads, 0, stream>>>(s);
        });
    p.items += p.n_wide;
    in_slices(p, p.n_items - p.n_wide, kThreads, [&](const taps_attend_launch &s, uint32_t groups) {
        k_attend<T, D><<<groups, kThreads, 0, stream>>>(s);
    });
}

template <class T> hipError_t launch(const taps_attend_launch &p, hipStream_t stream) {
    if (p.dim <= 64)
        launch_items<T, 64>(p, stream);
    else if (p.dim <= 96)
        launch_items<T, 96>(p, stream);
    else
        launch_items<T, 128>(p, stream);
    if (p.n_joins)
        k_join<T><<<dim3(p.n_joins, p.kv_heads, p.join_rounds), kThreads, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t taps_launch_attend(const taps_attend_launch &p, uint32_t dtype, hipStream_t stream) {
    return dtype == TAPS_BF16 ? launch<__bf16>(p, stream) : launch<_Float16>(p, stream);
}
