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
// product's operand as it lies in the registers.  V^T comes out of LDS by the transposing read
// (four keys of one column per lane).  The order in which a product takes its keys is free, so
// the second takes them as the first left them.
//
// Two kinds of items (workgroups of four wavefronts):
//   wide    128 query rows, 32 a wavefront; all share tiles of 64 keys;
//   narrow  up to 32 query rows; every wavefront takes every fourth tile of 32 keys, and the
//           four results are joined in LDS.
// The next tile is on its way while the present one is in use: straight to a
// second buffer in LDS (wide), or in registers (narrow).
// Where a sequence's keys are split over several items, each leaves its
// unnormalised result, maximum and sum, and k_join adds them up.
#include "taps_attention_internal.h"

namespace {

constexpr int kThreads = 256, kWaves = 4;
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kMinusInf = -__builtin_inff();
// A row's maximum is raised only when a tile exceeds it by this much (in
// powers of two): numerators stay below 2^8, far inside every type's range,
// and most tiles leave the accumulators alone.
constexpr float kSlack = 8.f;

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
template <int D> constexpr int shared_bytes() {
    return max_of(2 * Tile<D>::bytes(kWideKeys),
                  max_of(kWaves * Tile<D>::bytes(kNarrowKeys),
                         kWaves * kNarrowRows * (D + 4) * 4) + kWaves * kNarrowRows * 2 * 4);
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
                 : "memory", "m0");
}
// (the builtin, unlike an instruction in asm, tells the compiler too that no
// load of its own is under way, or it would wait again inside the loop)
__device__ __forceinline__ void wait_loads() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0f70);   // vmcnt(0)
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

// One wavefront's 32 query rows: the rows' operand, running statistics and result.
template <class T, int D> struct Rows {
    static constexpr int kSteps = D / 16, kBlocks = D / 32;
    s16x8 q[kSteps];
    f32x16 o[kBlocks];
    float m, l;        // maximum of the scores, this lane's half of the sum
    int first, last;   // keys of the item this lane's row sees: first .. last

    __device__ __forceinline__ void start(const taps_attend_launch &p, const taps_plan_seq &s,
                                          uint32_t head, int row, int lo, int hi, int lane) {
        const bool real = row < s.rows;
        const int token = row / (int)p.group, sub = row - token * (int)p.group;
        const int pos = s.first_pos + token;
        first = lo;
        last = hi - 1;
        if (p.causal) {
            last = min(last, pos);
            if (p.window) first = max(first, pos - (int)p.window + 1);
        }
        if (!real) last = -1, first = 0;
        const char *at = p.q + (int64_t)(s.token0 + token) * p.q_token +
                         (int64_t)(head * p.group + sub) * p.q_head;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int d = 16 * k + 8 * (lane >> 5);
            q[k] = s16x8{};
            if (real && d < (int)p.dim) q[k] = *(const s16x8 *)(at + 2 * d);
        }
        m = kMinusInf;
        l = 0.f;
#pragma unroll
        for (int b = 0; b < kBlocks; ++b) o[b] = f32x16{};
    }

    // Takes Keys keys from LDS; t0 is the first one's number.  `c` = scale log2 e.
    template <int Keys>
    __device__ __forceinline__ void take(const char *lds, int t0, bool masked, float c, int lane) {
        constexpr int kSub = Keys / 32, kRow = Tile<D>::kRow;
        const int half = lane >> 5;
        f32x16 s[kSub];
        const int k_mask = Tile<D>::k_mask(lane & 31);   // the same for key + 32
#pragma unroll
        for (int n = 0; n < kSub; ++n) s[n] = f32x16{};
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const char *at = lds + (lane & 31) * kRow + 16 * ((2 * k + half) ^ k_mask);
#pragma unroll
            for (int n = 0; n < kSub; ++n)
                s[n] = Mfma<T>::run(*(const s16x8 *)(at + 32 * n * kRow), q[k], s[n]);
        }
        if (masked) {
            const uint32_t seen = max(last - first + 1, 0), at = t0 + 4 * half - first;
#pragma unroll
            for (int n = 0; n < kSub; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i)
                    s[n][i] = at + (32 * n + 8 * (i / 4) + i % 4) < seen ? s[n][i] : kMinusInf;
        }
        float most = s[0][0];
#pragma unroll
        for (int n = 0; n < kSub; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) most = fmaxf(most, s[n][i]);
        most = half_max(most);
        if (__any(most * c > m * c + kSlack)) {
            const float to = fmaxf(m, most);
            const float by = to == kMinusInf ? 1.f : __builtin_amdgcn_exp2f((m - to) * c);
            m = to;
            l *= by;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[b][i] *= by;
        }
        const float shift = m == kMinusInf ? 0.f : m * c;
        uint32_t pt[kSub][8];
#pragma unroll
        for (int n = 0; n < kSub; ++n)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float a = __builtin_amdgcn_exp2f(s[n][2 * i] * c - shift);
                const float b = __builtin_amdgcn_exp2f(s[n][2 * i + 1] * c - shift);
                l += a + b;
                pt[n][i] = pack2<T>(a, b);
            }
        // lane of a group of 16: key (lane % 16) / 4, columns 4 (lane % 4) ..
        const int v_key = 4 * half + (lane & 15) / 4;
        const int v_chunk = 2 * ((lane >> 4) & 1) + ((lane >> 1) & 1);
        const int v_mask = Tile<D>::v_mask(v_key);   // the same for keys 8 and 16 further
        const char *v0 = lds + (Keys + v_key) * kRow + 8 * (lane & 1);
#pragma unroll
        for (int n = 0; n < kSub; ++n)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const u32x4 pb = {pt[n][4 * k], pt[n][4 * k + 1], pt[n][4 * k + 2], pt[n][4 * k + 3]};
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    const char *at = v0 + 16 * ((4 * b + v_chunk) ^ v_mask) + (32 * n + 16 * k) * kRow;
                    const s16x4 u = transposed(at), w = transposed(at + 8 * kRow);
                    const s16x8 va = {u[0], u[1], u[2], u[3], w[0], w[1], w[2], w[3]};
                    o[b] = Mfma<T>::run(va, __builtin_bit_cast(s16x8, pb), o[b]);
                }
            }
    }

    static __device__ __forceinline__ s16x4 transposed(const char *at) {
        return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
            (__attribute__((address_space(3))) s16x4 *)at);
    }
};

// Writes one row's result, or a piece of it: `get(i)` = its element i.
template <class T>
__device__ __forceinline__ char *out_row(const taps_attend_launch &p, const taps_plan_seq &s,
                                         uint32_t head, int row) {
    const int token = row / (int)p.group, sub = row - token * (int)p.group;
    return p.out + (int64_t)(s.token0 + token) * p.o_token +
           (int64_t)(head * p.group + sub) * p.o_head;
}

__device__ __forceinline__ void store_lse(const taps_attend_launch &p, const taps_plan_seq &s,
                                          uint32_t head, int row, float m, float l) {
    if (!p.lse) return;
    const int token = row / (int)p.group, sub = row - token * (int)p.group;
    p.lse[(int64_t)(s.token0 + token) * p.q_heads + head * p.group + sub] =
        l == 0.f ? kMinusInf : m * p.scale + __builtin_amdgcn_logf(l) * kLn2;
}

template <class T, int D>
__global__ __launch_bounds__(kThreads, 2) void k_attend(taps_attend_launch p) {
    __shared__ __attribute__((aligned(16))) char lds[shared_bytes<D>()];
    const uint32_t item_at = blockIdx.x / p.kv_heads, head = blockIdx.x % p.kv_heads;
    const taps_plan_item item = p.items[item_at];
    const taps_plan_seq seq = p.seqs[item.seq];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t *pages = p.pages + seq.page0;
    const char *k_head = p.k_cache + (int64_t)head * p.k_head;
    const char *v_head = p.v_cache + (int64_t)head * p.v_head;
    const int lo = item.lo, hi = item.hi, start = lo & ~15;   // whole groups of 16 share a page
    const float c = p.scale * kLog2e;
    Rows<T, D> rows;
    constexpr int kBlocks = D / 32;
    const int half = lane >> 5;

    if (!item.narrow) {
        const int row = item.row0 + 32 * wave + (lane & 31);
        rows.start(p, seq, head, row, lo, hi, lane);
        // keys that every row of the wavefront sees: all_from .. all_to.  (Tiles that no row of one
        // wavefront sees are taken all the same, masked: leaving them out costs the other tiles
        // 64 register moves each.)
        int all_from = lo, all_to = hi - 1;
        if (p.causal) {
            const int row_a = min(item.row0 + 32 * wave, seq.rows - 1);
            const int row_b = min(item.row0 + 32 * wave + 31, seq.rows - 1);
            all_to = min(all_to, seq.first_pos + row_a / (int)p.group);
            if (p.window)
                all_from = max(all_from, seq.first_pos + row_b / (int)p.group - (int)p.window + 1);
        }
        // Each wavefront loads 16 of a tile's 64 keys.  Keys outside lo .. hi - 1 and columns
        // beyond the head come from a block of zeros in the plan: what memory holds in their
        // place (it may never have been written) must not reach a product.
        const Group<D> g(lane);
        const uint32_t mine = __builtin_amdgcn_readfirstlane(lds_at(lds) + 16 * wave * Tile<D>::kRow);
        const bool ragged = p.dim < D;
        const auto load = [&](int t0, int page, int buffer) {
            const int key = t0 + 16 * wave;
            const Place at(p, k_head, v_head, page, key);
            const uint32_t to = mine + buffer * Tile<D>::bytes(kWideKeys);
            const bool whole = !ragged && key >= lo && key + 16 <= hi;
#pragma unroll
            for (int i = 0; i < Group<D>::kN; ++i) {
                const char *k = at.k + g.key[i] * p.k_slot + 16 * g.k_col[i];
                const char *v = at.v + g.key[i] * p.v_slot + 16 * g.v_col[i];
                if (!whole) {
                    const bool in = key + g.key[i] >= lo && key + g.key[i] < hi;
                    k = in && 8 * g.k_col[i] < (int)p.dim ? k : p.zeros;
                    v = in && 8 * g.v_col[i] < (int)p.dim ? v : p.zeros;
                }
                load_to_lds(k, to + 1024 * i);
                load_to_lds(v, to + 1024 * i + kWideKeys * Tile<D>::kRow);
            }
        };
        int page = 0, buffer = 0;
        if (lo < hi) {
            load(start, page_at(p, pages, start + 16 * wave, lo, hi), 0);
            page = page_at(p, pages, start + kWideKeys + 16 * wave, lo, hi);
        }
        for (int t0 = start; lo < hi && t0 < hi; t0 += kWideKeys, buffer ^= 1) {
            // one barrier a tile: the tile's loads have ended in every wavefront, and every
            // wavefront is done with the other buffer
            wait_loads();
            __syncthreads();
            if (t0 + kWideKeys < hi) {
                load(t0 + kWideKeys, page, buffer ^ 1);
                page = page_at(p, pages, t0 + 2 * kWideKeys + 16 * wave, lo, hi);
            }
            const bool masked = t0 < all_from || t0 + kWideKeys - 1 > all_to;
            rows.template take<kWideKeys>(lds + buffer * Tile<D>::bytes(kWideKeys), t0, masked, c,
                                          lane);
        }
        const float l = half_sum(rows.l);
        if (row >= seq.rows) return;
        if (item.part < 0) {
            const float inv = l == 0.f ? 0.f : 1.f / l;
            char *out = out_row<T>(p, seq, head, row);
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int d = 32 * b + 8 * i + 4 * half;
                    const u32x2 v = {
                        pack2<T>(rows.o[b][4 * i] * inv, rows.o[b][4 * i + 1] * inv),
                        pack2<T>(rows.o[b][4 * i + 2] * inv, rows.o[b][4 * i + 3] * inv)};
                    if (d < (int)p.dim) *(u32x2 *)(out + 2 * d) = v;
                }
            if (half == 0) store_lse(p, seq, head, row, rows.m, l);
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
        return;
    }

    // narrow: every wavefront has the same rows and its own keys
    const int row = item.row0 + (lane & 31);
    rows.start(p, seq, head, row, lo, hi, lane);
    {
        const int last_row = min(item.row0 + kNarrowRows, seq.rows) - 1;
        // one token's rows all see the item's keys; several tokens' need masks
        const bool one = item.row0 / (int)p.group == last_row / (int)p.group || !p.causal;
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
            const bool masked = !one || t0 < lo || t0 + kNarrowKeys > hi;
            rows.template take<kNarrowKeys>(tile, t0, masked, c, lane);
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        }
    }
    float *ml = (float *)(lds + shared_bytes<D>() - kWaves * kNarrowRows * 2 * 4);
    const float l_wave = half_sum(rows.l);
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
    {
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
    }
    __syncthreads();
    const int n_rows = min(kNarrowRows, seq.rows - item.row0);
    for (int k = threadIdx.x; k < n_rows * (D / 4); k += kThreads) {
        const int r = k / (D / 4), d = 4 * (k % (D / 4));
        if (d >= (int)p.dim) continue;
        float top = kMinusInf, l = 0.f;
        f32x4 o = {};
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            top = fmaxf(top, ml[2 * (w * kNarrowRows + r)]);
            o += *(const f32x4 *)(sums + (w * kNarrowRows + r) * (D + 4) + d);
        }
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            const float mw = ml[2 * (w * kNarrowRows + r)], lw = ml[2 * (w * kNarrowRows + r) + 1];
            l += mw == kMinusInf ? lw : lw * __builtin_amdgcn_exp2f((mw - top) * c);
        }
        if (item.part < 0) {
            const float inv = l == 0.f ? 0.f : 1.f / l;
            char *out = out_row<T>(p, seq, head, item.row0 + r);
            const u32x2 v = {pack2<T>(o[0] * inv, o[1] * inv), pack2<T>(o[2] * inv, o[3] * inv)};
            *(u32x2 *)(out + 2 * d) = v;
            if (d == 0) store_lse(p, seq, head, item.row0 + r, top, l);
        } else {
            const int64_t at = (int64_t)(item.part + r) * p.kv_heads + head;
            *(f32x4 *)(p.part_o + at * p.dim + d) = o;
            if (d == 0) p.part_ml[2 * at] = top, p.part_ml[2 * at + 1] = l;
        }
    }
}

// Adds up the pieces of rows whose keys were split.  A group of 32 lanes, four
// elements a lane, takes every `across`-th piece of a row, four at a time; the
// groups of a row meet in LDS.  With one group a row and one row after the
// other in a workgroup, 2048 rows x 8 heads in 4 pieces took 62 us and 4 rows x
// 8 heads in 32 pieces 28, waiting for one load after the other.
constexpr int kJoinGroups = kThreads / 32;

template <class T>
__global__ __launch_bounds__(kThreads) void k_join(taps_attend_launch p) {
    __shared__ f32x4 sums[kJoinGroups][32];
    __shared__ float ms[kJoinGroups], ls[kJoinGroups];
    const taps_plan_join join = p.joins[blockIdx.x];
    const taps_plan_seq seq = p.seqs[join.seq];
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
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (live) {
        char *out = out_row<T>(p, seq, head, join.row0 + r);
        const u32x2 v = {pack2<T>(o[0] * inv, o[1] * inv), pack2<T>(o[2] * inv, o[3] * inv)};
        *(u32x2 *)(out + 2 * d) = v;
    }
    if (d == 0) store_lse(p, seq, head, join.row0 + r, m, l);
}

template <class T> hipError_t launch(const taps_attend_launch &p, hipStream_t stream) {
    const uint32_t groups = p.n_items * p.kv_heads;
    if (p.dim <= 64)
        k_attend<T, 64><<<groups, kThreads, 0, stream>>>(p);
    else if (p.dim <= 96)
        k_attend<T, 96><<<groups, kThreads, 0, stream>>>(p);
    else
        k_attend<T, 128><<<groups, kThreads, 0, stream>>>(p);
    if (p.n_joins) k_join<T><<<dim3(p.n_joins, p.kv_heads, p.join_rounds), kThreads, 0, stream>>>(p);
    return hipGetLastError();
}

}  // namespace

hipError_t taps_launch_attend(const taps_attend_launch &p, uint32_t dtype, hipStream_t stream) {
    return dtype == TAPS_BF16 ? launch<__bf16>(p, stream) : launch<_Float16>(p, stream);
}
