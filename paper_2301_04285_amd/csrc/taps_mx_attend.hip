// taps_mx_attend.hip -- attention of new tokens over a paged cache in microscaling
// formats.
//
// The mathematics, the kinds of items and the layouts of both products are
// those of taps_attend.hip.  Keys and values become 16-bit numbers (exact but at the
// ends of fp16's range) on their way to LDS: a lane fetches a quarter of a key, waits
// for it while the tile before is in use, and converts two elements an instruction.
#include "taps_attend_device.h"
#include "taps_mx_device.h"
#include "taps_mx_internal.h"

namespace {

// A lane's part of 16 keys (or values) that share a page: a quarter of one of them.
template <int D, int Bits> struct Piece {
    static constexpr int kChunks = D / 32;   // of eight elements
    static constexpr int kCodes = kChunks * kWords<Bits>;
    static constexpr int kBytes = kChunks == 3 ? 2 : 1;   // blocks that a quarter touches
    uint32_t code[kCodes], byte[kBytes];

    static __device__ __forceinline__ int key(int lane) { return lane & 15; }
    static __device__ __forceinline__ int chunk(int lane) { return kChunks * (lane >> 4); }
    // Whether a head of up to 32 elements, one block, has this quarter.
    static __device__ __forceinline__ bool exists(int lane, int dim) {
        return kChunks != 2 || dim > 32 || lane < 32;
    }
    __device__ __forceinline__ void fetch(const char *codes, const char *scales, int lane) {
        const uint32_t *from = (const uint32_t *)(codes + chunk(lane) * Bits);
#pragma unroll
        for (int i = 0; i < kCodes; ++i) code[i] = from[i];
        byte[0] = (uint8_t)scales[chunk(lane) / 4];
        if (kBytes > 1) byte[kBytes - 1] = (uint8_t)scales[(chunk(lane) + kChunks - 1) / 4];
    }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < kCodes; ++i) code[i] = 0;
#pragma unroll
        for (int i = 0; i < kBytes; ++i) byte[i] = 127;
    }
    template <class T> __device__ __forceinline__ u32x4 eight(int j, int lane) const {
        const bool first = kBytes == 1 || (chunk(lane) + j) / 4 == chunk(lane) / 4;
        return mx_eight<T, Bits>(code + j * kWords<Bits>, mx_scale(first ? byte[0] : byte[kBytes - 1]));
    }
};

// What redo reads of the cache, and where groups of 16 keys lie.
template <class T, int Bits> struct MxCache {
    struct At {
        const char *k, *v, *ks, *vs;
    };
    struct Row {
        const char *codes, *scales;
    };
    const taps_mx_attend_launch &p;
    const char *k, *v, *ks, *vs;   // of the key head
    __device__ __forceinline__ MxCache(const taps_mx_attend_launch &launch, uint32_t head)
        : p(launch), k(p.k_cache + (int64_t)head * p.k_head), v(p.v_cache + (int64_t)head * p.v_head),
          ks(p.k_scales + (int64_t)head * p.ks_head), vs(p.v_scales + (int64_t)head * p.vs_head) {}
    __device__ __forceinline__ At at(int page, int key) const {
        const int64_t slot = key & ((1 << p.page_log2) - 1);
        return {k + page * p.k_page + slot * p.k_slot, v + page * p.v_page + slot * p.v_slot,
                ks + page * p.ks_page + slot * p.ks_slot, vs + page * p.vs_page + slot * p.vs_slot};
    }
    __device__ __forceinline__ Row row(const At &a, const At &b, bool second, uint32_t slot) const {
        return {(second ? b.k : a.k) + slot * (uint32_t)p.k_slot,
                (second ? b.ks : a.ks) + slot * (uint32_t)p.ks_slot};
    }
    __device__ __forceinline__ s16x8 keys(const Row &row, int d) const {
        uint32_t code[kWords<Bits>];
#pragma unroll
        for (int i = 0; i < kWords<Bits>; ++i) code[i] = ((const uint32_t *)(row.codes + d / 8 * Bits))[i];
        return __builtin_bit_cast(
            s16x8, mx_eight<T, Bits>(code, mx_scale((uint8_t)row.scales[d / 32])));
    }
    __device__ __forceinline__ short value(const At &at, uint32_t slot, uint32_t stride, int d) const {
        const uint8_t byte = at.v[slot * stride + d * Bits / 8];
        const uint32_t code = Bits == 4 && d % 2 ? byte >> 4 : byte;
        const uint8_t scale = at.vs[slot * (uint32_t)p.vs_slot + d / 32];
        return (short)mx_pair<T, Bits, 0>(code, mx_scale(scale));
    }
};

// Fetches a wavefront's 16 keys of K or of V of a tile and puts them into LDS.  Keys outside
// lo .. hi - 1 are fetched from an end of that range and become zeros, as does what is not there
// of a head's second block.
template <class T, int D, int Bits, bool V> struct Stager {
    using P = Piece<D, Bits>;
    const char *codes, *scales;
    int64_t code_page, scale_page;
    uint32_t code_slot, scale_slot;
    int lo, hi, page_log2, lane;
    bool exists;
    P piece;
    __device__ __forceinline__ Stager(const taps_mx_attend_launch &p, const taps_plan_item &item,
                                      uint32_t head, int l) {
        codes = V ? p.v_cache + (int64_t)head * p.v_head : p.k_cache + (int64_t)head * p.k_head;
        scales = V ? p.v_scales + (int64_t)head * p.vs_head : p.k_scales + (int64_t)head * p.ks_head;
        code_page = V ? p.v_page : p.k_page, scale_page = V ? p.vs_page : p.ks_page;
        code_slot = V ? p.v_slot : p.k_slot, scale_slot = V ? p.vs_slot : p.ks_slot;
        lo = item.lo, hi = item.hi, page_log2 = p.page_log2, lane = l;
        exists = P::exists(lane, p.dim);
    }
    // The group of 16 keys from key0 on, a multiple of 16; outside the item: the nearest inside.
    __device__ __forceinline__ void fetch(int key0, int page) {
        key0 = min(max(key0, lo & ~15), (hi - 1) & ~15);
        const int64_t slot = key0 & ((1 << page_log2) - 1);
        const uint32_t row = min(max(key0 + P::key(lane), lo), hi - 1) - key0;
        if (exists)
            piece.fetch(codes + page * code_page + slot * code_slot + row * code_slot,
                        scales + page * scale_page + slot * scale_slot + row * scale_slot, lane);
    }
    // key0: as fetched; `at`: its number in the tile of LDS.
    __device__ __forceinline__ void put(char *tile, int at, int key0) {
        const int key = key0 + P::key(lane);
        if (!exists || key < lo || key >= hi) piece.clear();
        const int n = at + P::key(lane);
        const int mask = V ? Tile<D>::v_mask(n) : Tile<D>::k_mask(n);
#pragma unroll
        for (int j = 0; j < P::kChunks; ++j)
            *(u32x4 *)(tile + n * Tile<D>::kRow + 16 * ((P::chunk(lane) + j) ^ mask)) =
                piece.template eight<T>(j, lane);
    }
};

// 32 query rows for each of Waves wavefronts (block: 4, wide: 8), tiles of 64 keys in two
// buffers: while one is in use the next is on its way through registers into the
// other.  Eight wavefronts share the work of K and V, four do both.
template <class T, int D, int Bits, int Waves>
__device__ __forceinline__ void attend_rows(const taps_mx_attend_launch &p, const taps_plan_item &item,
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
    Stager<T, D, Bits, false> k(p, item, head, lane);
    Stager<T, D, Bits, true> v(p, item, head, lane);
    const bool takes_k = Waves == 4 || wave < 4, takes_v = Waves == 4 || wave >= 4;
    const int mine = 16 * (wave & 3);
    const auto fetch = [&](int t0) {
        if (t0 >= hi) return;
        const int page = page_at(p, pages, t0 + mine, item.lo, item.hi);
        if (takes_k) k.fetch(t0 + mine, page);
        if (takes_v) v.fetch(t0 + mine, page);
    };
    const auto put = [&](int t0, char *tile) {
        if (t0 >= hi) return;
        if (takes_k) k.put(tile, mine, t0 + mine);
        if (takes_v) v.put(tile + kPart, mine, t0 + mine);
    };
    fetch(start);
    put(start, lds);
    __syncthreads();
    int buffer = 0;
    for (int t0 = start; t0 < hi; t0 += kWideKeys, buffer ^= 1) {
        const char *tile = lds + 2 * buffer * kPart;
        fetch(t0 + kWideKeys);
        if (t0 < seen.end) {
            typename Rows<T, D>::template Scores<kWideKeys> x;
            typename Rows<T, D>::template Numerators<kWideKeys> y;
            rows.score(tile, x, lane);
            rows.soften(x, y, t0, seen.masks(t0, kWideKeys), c, lane);
            rows.spend(tile + kPart, y, lane);
        }
        put(t0 + kWideKeys, lds + 2 * (buffer ^ 1) * kPart);
        __syncthreads();
    }
    const float l = rows.total();
    finish(p, item, MxCache<T, Bits>(p, head), rows, seen, row, l, start, 32, lane, [&]() {
        if (row < item.rows) write_rows(p, item, head, rows, row, l, lane >> 5);
    });
}

template <class T, int D, int Bits>
__global__ __launch_bounds__(kWideThreads, 2) void k_mx_attend_wide(taps_mx_attend_launch p) {
    __shared__ __attribute__((aligned(16))) char lds[2 * Tile<D>::bytes(kWideKeys)];
    const uint32_t head = blockIdx.x % p.kv_heads;
    attend_rows<T, D, Bits, 8>(p, p.items[blockIdx.x / p.kv_heads], head, lds);
}

// Up to 32 query rows: every wavefront has all of them and its own keys.
template <class T, int D, int Bits>
__device__ __forceinline__ void attend_narrow(const taps_mx_attend_launch &p,
                                              const taps_plan_item &item, uint32_t head, char *lds) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t *pages = p.pages + item.page0;
    const int lo = item.lo, hi = item.hi, start = lo & ~15;
    const float c = p.scale * kLog2e;
    constexpr int kStep = kWaves * kNarrowKeys;
    Rows<T, D> rows;
    rows.start(p, item, head, item.row0 + (lane & 31), lane);
    const Seen seen(p, item, item.row0);
    char *tile = lds + wave * Tile<D>::bytes(kNarrowKeys);
    Stager<T, D, Bits, false> k[2] = {{p, item, head, lane}, {p, item, head, lane}};
    Stager<T, D, Bits, true> v[2] = {{p, item, head, lane}, {p, item, head, lane}};
    const auto fetch = [&](int t0) {
        if (lo >= hi || t0 >= hi) return;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int page = page_at(p, pages, t0 + 16 * h, lo, hi);
            k[h].fetch(t0 + 16 * h, page);
            v[h].fetch(t0 + 16 * h, page);
        }
    };
    const auto exchange = [&]() {
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };
    int t0 = start + kNarrowKeys * wave;
    fetch(t0);
    for (; lo < hi && t0 < hi; t0 += kStep) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            k[h].put(tile, 16 * h, t0 + 16 * h);
            v[h].put(tile + kNarrowKeys * Tile<D>::kRow, 16 * h, t0 + 16 * h);
        }
        exchange();
        fetch(t0 + kStep);
        typename Rows<T, D>::template Scores<kNarrowKeys> x;
        typename Rows<T, D>::template Numerators<kNarrowKeys> y;
        rows.score(tile, x, lane);
        rows.soften(x, y, t0, seen.masks(t0, kNarrowKeys), c, lane);
        rows.spend(tile + kNarrowKeys * Tile<D>::kRow, y, lane);
        exchange();
    }
    join_waves(p, item, MxCache<T, Bits>(p, head), head, rows, seen, start, lds);
}

// A block or a narrow item; both fit a unit twice.
template <class T, int D, int Bits>
__global__ __launch_bounds__(kThreads, 2) void k_mx_attend(taps_mx_attend_launch p) {
    __shared__ __attribute__((aligned(16))) char lds[max_of(narrow_bytes<D>(),
                                                            2 * Tile<D>::bytes(kWideKeys))];
    const uint32_t head = blockIdx.x % p.kv_heads;
    const taps_plan_item item = p.items[blockIdx.x / p.kv_heads];
    if (item.kind == kBlock)
        attend_rows<T, D, Bits, 4>(p, item, head, lds);
    else
        attend_narrow<T, D, Bits>(p, item, head, lds);
}

template <class T, int D, int Bits> void launch_items(taps_mx_attend_launch p, hipStream_t stream) {
    if constexpr (D > kWideAbove)
        in_slices(p, p.n_wide, kWideThreads, [&](const auto &s, uint32_t groups) {
            k_mx_attend_wide<T, D, Bits><<<groups, kWideThreads, 0, stream>>>(s);
        });
    p.items += p.n_wide;
    in_slices(p, p.n_items - p.n_wide, kThreads, [&](const auto &s, uint32_t groups) {
        k_mx_attend<T, D, Bits><<<groups, kThreads, 0, stream>>>(s);
    });
}

template <class T, int Bits>
hipError_t launch(const taps_mx_attend_launch &p, uint32_t dtype, hipStream_t stream) {
    if (p.dim <= 64)
        launch_items<T, 64, Bits>(p, stream);
    else if (p.dim <= 96)
        launch_items<T, 96, Bits>(p, stream);
    else
        launch_items<T, 128, Bits>(p, stream);
    return taps_launch_join(p, dtype, stream);
}

}  // namespace

hipError_t taps_launch_mx_attend(const taps_mx_attend_launch &p, uint32_t dtype, uint32_t bits,
                                 hipStream_t stream) {
    if (dtype == TAPS_BF16)
        return bits == 4 ? launch<__bf16, 4>(p, dtype, stream) : launch<__bf16, 8>(p, dtype, stream);
    return bits == 4 ? launch<_Float16, 4>(p, dtype, stream) : launch<_Float16, 8>(p, dtype, stream);
}
