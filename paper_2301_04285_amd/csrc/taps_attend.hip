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
#include "taps_attend_device.h"

namespace {

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
    Place() = default;
    __device__ __forceinline__ Place(const taps_attend_launch &p, const char *k_head,
                                     const char *v_head, int page, int key) {
        const int64_t slot = key & ((1 << p.page_log2) - 1);
        k = k_head + page * p.k_page + slot * p.k_slot;
        v = v_head + page * p.v_page + slot * p.v_slot;
    }
};

// What redo reads of a cache in 16 bits.
struct HalfCache {
    typedef const char *Key, *Value;
    const taps_attend_launch &p;
    const uint32_t head;
    __device__ __forceinline__ HalfCache(const taps_attend_launch &launch, uint32_t h)
        : p(launch), head(h) {}
    __device__ __forceinline__ Place at(int page, int key) const {
        return Place(p, p.k_cache + (int64_t)head * p.k_head, p.v_cache + (int64_t)head * p.v_head, page,
                     key);
    }
    __device__ __forceinline__ const char *row(const char *k, uint32_t slot) const {
        return k + slot * (uint32_t)p.k_slot;
    }
    __device__ __forceinline__ s16x8 keys(const char *row, int d) const {
        return *(const s16x8 *)(row + 2 * d);
    }
    __device__ __forceinline__ short value(const char *v, uint32_t slot, uint32_t stride, int d) const {
        return *(const short *)(v + slot * stride + 2 * d);
    }
};

// Loads to LDS: a wavefront takes 16 of a tile's 64 keys, of K or of V.  Keys
// outside lo .. hi - 1 and columns beyond the head come from a block of zeros in
// the plan: what memory holds in their place (it may never have been written)
// must not reach a product.
template <int D> struct Loader {
    static constexpr int kN = Group<D>::kN;   // loads of a tile's K or V
    static constexpr int kAhead = 0;
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
    __device__ __forceinline__ void start(int, int) const {}
    __device__ __forceinline__ void wait(bool newer) const {
        if (newer)
            wait_loads<kN>();
        else
            wait_loads<0>();
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

template <class T, int D>
__global__ __launch_bounds__(kWideThreads, 2) void k_attend_wide(taps_attend_launch p) {
    __shared__ __attribute__((aligned(16))) char lds[6 * kWideKeys * Tile<D>::kRow];
    const uint32_t head = blockIdx.x % p.kv_heads;
    const taps_plan_item item = p.items[blockIdx.x / p.kv_heads];
    attend_wide<T, D, Loader<D>>(p, item, head, HalfCache(p, head), lds);
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
    finish(p, item, HalfCache(p, head), rows, seen, row, l, start, 32, lane, [&]() {
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
    join_waves(p, item, HalfCache(p, head), head, rows, seen, start, lds);
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

template <class T> void launch(const taps_attend_launch &p, hipStream_t stream) {
    if (p.dim <= 64)
        launch_items<T, 64>(p, stream);
    else if (p.dim <= 96)
        launch_items<T, 96>(p, stream);
    else
        launch_items<T, 128>(p, stream);
}

}  // namespace

hipError_t taps_launch_join(const taps_attend_launch &p, uint32_t dtype, hipStream_t stream) {
    if (p.n_joins) {
        const dim3 grid(p.n_joins, p.kv_heads, p.join_rounds);
        if (dtype == TAPS_BF16)
            k_join<__bf16><<<grid, kThreads, 0, stream>>>(p);
        else
            k_join<_Float16><<<grid, kThreads, 0, stream>>>(p);
    }
    return hipGetLastError();
}

hipError_t taps_launch_attend(const taps_attend_launch &p, uint32_t dtype, hipStream_t stream) {
    if (dtype == TAPS_BF16)
        launch<__bf16>(p, stream);
    else
        launch<_Float16>(p, stream);
    return taps_launch_join(p, dtype, stream);
}
