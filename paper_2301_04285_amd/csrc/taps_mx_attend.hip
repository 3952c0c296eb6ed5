// taps_mx_attend.hip -- attention of new tokens over a paged cache in microscaling
// formats.
//
// The mathematics, the kinds of items and, but for those of up to 16 rows, the layouts of both
// products are those of taps_attend.hip.  Codes come to registers and become 16-bit numbers there,
// two an instruction with their power of two (exact but at the ends of fp16's range): for items of
// many rows once on the way to LDS, where all rows share them; for those of few rows where the
// products want them.  Products of codes themselves (fp4 by fp8 with scales), which would save the
// conversions of keys, hold their sums to 2^-12 of the largest term and were not taken.
//
// Kernels, by the items of a launch (without the wide ones, which have their own):
//   k_mx_attend_few     all of up to 16 rows;
//   k_mx_attend_alone   others, no more than there are units: eight wavefronts to each;
//   k_mx_attend         others.
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
    // From uniform addresses and this lane's offsets of its quarter's codes and first scale.
    __device__ __forceinline__ void fetch(const char *codes, const char *scales, uint32_t code_at,
                                          uint32_t scale_at, int lane) {
        typedef uint32_t words __attribute__((ext_vector_type(kCodes), aligned(4)));
        const words w = *(const words *)(codes + code_at);
#pragma unroll
        for (int i = 0; i < kCodes; ++i) code[i] = w[i];
        byte[0] = (uint8_t)scales[scale_at];
        if (kBytes > 1) {
            const uint32_t more = (chunk(lane) + kChunks - 1) / 4 - chunk(lane) / 4;
            byte[kBytes - 1] = (uint8_t)scales[scale_at + more];
        }
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
    struct Key {
        const char *codes, *scales;
    };
    typedef Key Value;
    struct At {
        Key k;
        Value v;
    };
    const taps_mx_attend_launch &p;
    const char *k, *v, *ks, *vs;   // of the key head
    __device__ __forceinline__ MxCache(const taps_mx_attend_launch &launch, uint32_t head)
        : p(launch), k(p.k_cache + (int64_t)head * p.k_head), v(p.v_cache + (int64_t)head * p.v_head),
          ks(p.k_scales + (int64_t)head * p.ks_head), vs(p.v_scales + (int64_t)head * p.vs_head) {}
    __device__ __forceinline__ At at(int page, int key) const {
        const int64_t slot = key & ((1 << p.page_log2) - 1);
        return {{k + page * p.k_page + slot * p.k_slot, ks + page * p.ks_page + slot * p.ks_slot},
                {v + page * p.v_page + slot * p.v_slot, vs + page * p.vs_page + slot * p.vs_slot}};
    }
    __device__ __forceinline__ Key row(const Key &a, uint32_t slot) const {
        return {a.codes + slot * (uint32_t)p.k_slot, a.scales + slot * (uint32_t)p.ks_slot};
    }
    __device__ __forceinline__ s16x8 keys(const Key &row, int d) const {
        uint32_t code[kWords<Bits>];
#pragma unroll
        for (int i = 0; i < kWords<Bits>; ++i) code[i] = ((const uint32_t *)(row.codes + d / 8 * Bits))[i];
        return __builtin_bit_cast(
            s16x8, mx_eight<T, Bits>(code, mx_scale((uint8_t)row.scales[d / 32])));
    }
    __device__ __forceinline__ short value(const Value &at, uint32_t slot, uint32_t stride, int d) const {
        const uint8_t byte = at.codes[slot * stride + d * Bits / 8];
        const uint32_t code = Bits == 4 && d % 2 ? byte >> 4 : byte;
        const uint8_t scale = at.scales[slot * (uint32_t)p.vs_slot + d / 32];
        return (short)mx_pair<T, Bits, 0>(code, mx_scale(scale));
    }
};

// 16 keys of K or of V that share a page, on their way to a wavefront.
template <class T, int D, int Bits, bool V> struct Keys {
    using P = Piece<D, Bits>;
    const char *codes, *scales;
    int64_t code_page, scale_page;
    uint32_t code_slot, scale_slot, code_at, scale_at;   // _at: of this lane's quarter
    int lo, hi, page_log2, lane;
    bool exists;
    __device__ __forceinline__ Keys(const taps_mx_attend_launch &p, const taps_plan_item &item,
                                    uint32_t head, int l) {
        codes = V ? p.v_cache + (int64_t)head * p.v_head : p.k_cache + (int64_t)head * p.k_head;
        scales = V ? p.v_scales + (int64_t)head * p.vs_head : p.k_scales + (int64_t)head * p.ks_head;
        code_page = V ? p.v_page : p.k_page, scale_page = V ? p.vs_page : p.ks_page;
        code_slot = V ? p.v_slot : p.k_slot, scale_slot = V ? p.vs_slot : p.ks_slot;
        lo = item.lo, hi = item.hi, page_log2 = p.page_log2, lane = l;
        exists = P::exists(lane, p.dim);
        // a quarter that is not there: the head's first, to be cleared
        code_at = P::key(lane) * code_slot + (exists ? P::chunk(lane) * Bits : 0);
        scale_at = P::key(lane) * scale_slot + (exists ? P::chunk(lane) / 4 : 0);
    }
    // Where the group from key0 on lies, a multiple of 16.  A page has all its slots, so those outside
    // lo .. hi - 1 are fetched too, and cleared.
    struct At {
        const char *codes, *scales;
    };
    __device__ __forceinline__ At at(int key0, int page) const {
        const int64_t slot = key0 & ((1 << page_log2) - 1);
        return {codes + page * code_page + slot * code_slot,
                scales + page * scale_page + slot * scale_slot};
    }
    // The group behind one, on the same page.
    __device__ __forceinline__ At behind(const At &a) const {
        return {a.codes + 16 * code_slot, a.scales + 16 * scale_slot};
    }
    // The nearest group inside the item to the one from key0 on.
    __device__ __forceinline__ At nearest(int key0, int page) const {
        return at(min(max(key0, lo & ~15), (hi - 1) & ~15), page);
    }
    __device__ __forceinline__ void fetch(P &to, const At &a) const {
        to.fetch(a.codes, a.scales, code_at, scale_at, lane);
    }
    // After the wait for it; key0: as fetched.
    __device__ __forceinline__ void blank(P &of, int key0) const {
        const int key = key0 + P::key(lane);
        if (key < lo || key >= hi) of.clear();
    }
    __device__ __forceinline__ void blank_missing(P &of) const {
        if (P::kChunks == 2 && !exists) of.clear();
    }
    // To a tile in LDS, where key0 has the number `at`.
    __device__ __forceinline__ void put(P &from, char *tile, int at, int key0) const {
        if (key0 < lo || key0 + 16 > hi) blank(from, key0);
        blank_missing(from);
        const int n = at + P::key(lane);
        const int mask = V ? Tile<D>::v_mask(n) : Tile<D>::k_mask(n);
#pragma unroll
        for (int j = 0; j < P::kChunks; ++j)
            *(u32x4 *)(tile + n * Tile<D>::kRow + 16 * ((P::chunk(lane) + j) ^ mask)) =
                from.template eight<T>(j, lane);
    }
};

// 128 query rows, 32 for each of four wavefronts, tiles of 64 keys in two buffers: before one is used
// the next, which came to registers meanwhile, goes to the other.  With Split 2 there are four more
// wavefronts, which take every second tile; the results are joined in LDS.
template <class T, int D, int Bits, int Split>
__device__ __forceinline__ void attend_block(const taps_mx_attend_launch &p, const taps_plan_item &item,
                                             uint32_t head, char *lds) {
    constexpr int kPart = kWideKeys * Tile<D>::kRow, kStep = Split * kWideKeys;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int share = Split == 1 ? 0 : wave >> 2, mine = 16 * (wave & 3);   // keys of a tile to load
    const int32_t *pages = p.pages + item.page0;
    const int start = item.lo & ~15;
    // no tile of an item without keys: its lo need not be a multiple of 16
    const int hi = item.lo < item.hi ? item.hi : start;
    const float c = p.scale * kLog2e;
    const int row0 = item.row0 + 32 * (wave & 3), row = row0 + (lane & 31);
    Rows<T, D> rows;
    rows.start(p, item, head, row, lane);
    const Seen seen(p, item, row0);
    const Keys<T, D, Bits, false> k(p, item, head, lane);
    const Keys<T, D, Bits, true> v(p, item, head, lane);
    Piece<D, Bits> k_piece, v_piece;
    const int first = start + kWideKeys * share;
    int page = start < hi ? page_at(p, pages, first + mine, item.lo, item.hi) : 0;
    const auto fetch = [&](int t0) {
        if (t0 >= hi) return;
        k.fetch(k_piece, k.nearest(t0 + mine, page));
        v.fetch(v_piece, v.nearest(t0 + mine, page));
        page = page_at(p, pages, t0 + kStep + mine, item.lo, item.hi);
    };
    const auto put = [&](int t0, char *tile) {
        if (t0 >= hi) return;
        k.put(k_piece, tile, mine, t0 + mine);
        v.put(v_piece, tile + kPart, mine, t0 + mine);
    };
    char *buffers = lds + 4 * kPart * share;
    fetch(first);
    put(first, buffers);
    fetch(first + kStep);
    __syncthreads();
    int buffer = 0;
    // every share takes the same number of steps
    for (int at = start, t0 = first; at < hi; at += kStep, t0 += kStep, buffer ^= 1) {
        const char *tile = buffers + 2 * buffer * kPart;
        put(t0 + kStep, buffers + 2 * (buffer ^ 1) * kPart);
        fetch(t0 + 2 * kStep);
        if (t0 < min(hi, seen.end)) {
            typename Rows<T, D>::template Scores<kWideKeys> x;
            typename Rows<T, D>::template Numerators<kWideKeys> y;
            rows.score(tile, x, lane);
            rows.soften(x, y, t0, seen.masks(t0, kWideKeys), c, lane);
            rows.spend(tile + kPart, y, lane);
        }
        __syncthreads();
    }
    float l = rows.total();
    if constexpr (Split > 1) {
        float *left = (float *)lds + (row - item.row0) * (D + 8);   // results, maximum, sum
        if (share) {
            leave_row(rows, 1.f, left, lane);
            if (lane < 32) left[D] = rows.m, left[D + 1] = l;
        }
        __syncthreads();
        if (share) return;
        const float other = left[D], m = fmaxf(rows.m, other);
        const float by = rows.m == kMinusInf ? 1.f : __builtin_amdgcn_exp2f((rows.m - m) * c);
        const float by_other = other == kMinusInf ? 1.f : __builtin_amdgcn_exp2f((other - m) * c);
        rows.m = m, l = l * by + left[D + 1] * by_other;
#pragma unroll
        for (int b = 0; b < D / 32; ++b)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const f32x4 o = *(const f32x4 *)(left + 32 * b + 8 * i + 4 * (lane >> 5));
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    rows.o[b][4 * i + j] = rows.o[b][4 * i + j] * by + o[j] * by_other;
            }
    }
    finish(p, item, MxCache<T, Bits>(p, head), rows, seen, row, l, start, 32, lane, [&]() {
        if (row < item.rows) write_rows(p, item, head, rows, row, l, lane >> 5);
    });
}

// Loads of a wide item's wavefront: a tile's codes wait in registers until the tile before is on its
// way to LDS, in numbers.  The conversions fall into the phase of the softmax, beside the other half's
// products: 8 prompts of 2048, 32 heads of 128, 325 to 335 us in 4 bits and 335 to 361 in 8 by the card (314 to
// 349 over a 16-bit cache; 405 without the phases), 512 tokens over 32768 keys 241 to 261 (242 to 252).
template <class T, int D, int Bits> struct MxLoader {
    static constexpr int kAhead = 1;
    const Keys<T, D, Bits, false> k;
    const Keys<T, D, Bits, true> v;
    Piece<D, Bits> piece;
    const int key0;
    const bool second;
    __device__ __forceinline__ MxLoader(const taps_mx_attend_launch &p, const taps_plan_item &item,
                                        uint32_t head, bool values, int wave, int lane)
        : k(p, item, head, lane), v(p, item, head, lane), key0(16 * (wave & 3)), second(values) {}
    __device__ __forceinline__ void start(int t0, int page) {
        if (second)
            v.fetch(piece, v.nearest(t0 + key0, page));
        else
            k.fetch(piece, k.nearest(t0 + key0, page));
    }
    __device__ __forceinline__ void load(int t0, int page, const char *part) {
        if (second)
            v.put(piece, const_cast<char *>(part), key0, t0 + key0);
        else
            k.put(piece, const_cast<char *>(part), key0, t0 + key0);
        start(t0 + kWideKeys, page);
    }
    __device__ __forceinline__ void wait(bool) const {}
};

template <class T, int D, int Bits>
__global__ __launch_bounds__(kWideThreads, 2) void k_mx_attend_wide(taps_mx_attend_launch p) {
    __shared__ __attribute__((aligned(16))) char lds[6 * kWideKeys * Tile<D>::kRow];
    const uint32_t head = blockIdx.x % p.kv_heads;
    const taps_plan_item item = p.items[blockIdx.x / p.kv_heads];
    attend_wide<T, D, MxLoader<T, D, Bits>>(p, item, head, MxCache<T, Bits>(p, head), lds);
}

// What a wavefront wrote to LDS is read by its other lanes, and before it is written anew.
__device__ __forceinline__ void exchange() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// 17 to 32 query rows: every wavefront has all of them and its own keys.
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
    const Keys<T, D, Bits, false> k(p, item, head, lane);
    const Keys<T, D, Bits, true> v(p, item, head, lane);
    Piece<D, Bits> k_piece[2], v_piece[2];
    int page[2] = {0, 0};
    const auto look_up = [&](int t0) {
#pragma unroll
        for (int h = 0; h < 2; ++h) page[h] = page_at(p, pages, t0 + 16 * h, lo, hi);
    };
    const auto fetch = [&](int t0) {
        if (lo >= hi || t0 >= hi) return;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            k.fetch(k_piece[h], k.nearest(t0 + 16 * h, page[h]));
            v.fetch(v_piece[h], v.nearest(t0 + 16 * h, page[h]));
        }
        look_up(t0 + kStep);
    };
    int t0 = start + kNarrowKeys * wave;
    if (lo < hi) look_up(t0);
    fetch(t0);
    for (; lo < hi && t0 < hi; t0 += kStep) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            k.put(k_piece[h], tile, 16 * h, t0 + 16 * h);
            v.put(v_piece[h], tile + kNarrowKeys * Tile<D>::kRow, 16 * h, t0 + 16 * h);
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

// Up to 16 query rows: both products as 16x16x32 tiles, in which a lane has eight of a tile's 32
// keys for one row, half of what it has in the others' tiles.  Keys go from the registers that they
// are fetched to into the first product: a lane's quarter of a key is its part of
// the operand, with the queries laid out the same.  Values pass through LDS to be transposed.
// Every wavefront has two tiles on their way, each in registers of its own.
//
// Bytes bound it.  Two tokens over 131001 keys, 8 heads of 128 in 4 bits: 285 MB in 48 us, 5.9 TB/s,
// and 5 for the join.  64 tokens over up to 4000 keys: 160 MB in 31 and 5.  24 times four tokens over
// up to 9999 in 8 bits: 280 MB in 57 and 5 (keys do not come in the order of memory; in that order
// they would have to pass through LDS, which cost a lone token 3 us of 11).  With one tile on its way
// they took 4 to 9 us more, with 32x32x16 tiles, keys through LDS and half of the lanes' scores of rows
// that are not there 11 to 15.
template <class T> struct SmallMfma;
template <> struct SmallMfma<__bf16> {
    static __device__ __forceinline__ f32x4 run(s16x8 a, s16x8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            __builtin_bit_cast(Mfma<__bf16>::v8, a), __builtin_bit_cast(Mfma<__bf16>::v8, b), c, 0, 0, 0);
    }
};
template <> struct SmallMfma<_Float16> {
    static __device__ __forceinline__ f32x4 run(s16x8 a, s16x8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(
            __builtin_bit_cast(Mfma<_Float16>::v8, a), __builtin_bit_cast(Mfma<_Float16>::v8, b), c, 0, 0,
            0);
    }
};

// LDS image of 32 values: rows of 16-byte chunks, permuted by a mask of the key's number.  16 lanes
// write every fourth chunk of four keys (4 bits) or every second one of two (8 bits; heads of up to 64,
// whose rows are half as long: of twice as many keys), 32 read two chunks of eight keys: the mask's lowest
// two bits, or the lowest one, differ among the first, the others among the second.
template <int D, int Bits> struct Values {
    static constexpr int kRow = D <= 64 ? 128 : 256, kBytes = kNarrowKeys * kRow;
    static __device__ __forceinline__ int mask(int key) {
        const int a = D <= 64 ? (key >> 1) & 1 : key & 1, b = D <= 64 ? (key >> 2) & 1 : (key >> 1) & 1;
        const int far = D <= 64 ? 0 : 2 * (key & 4);
        return (Bits == 4 ? 2 * a + 5 * b : 5 * a + 2 * b) + far;
    }
};

struct True {
    static constexpr bool value = true;
};
struct False {
    static constexpr bool value = false;
};

// 16 values as they lie in memory: 16 bytes of codes a lane and load, so that neighbouring lanes share lines.
// They are not kept in the caches: only where sequences share pages does another item read them (64 tokens
// over up to 4000 keys 35.3 us, 39.3 with keys and values kept, 37.0 with neither; two over 131001 54.5, 59.5,
// 52.3.  64 over 4000 keys of which all share none, 3008, 3968: 51, 40.5, 39.1, with values kept 54, 39.9,
// 39.0).  Blocks of 32 bytes
// a lane, in 8 bits, take two loads with half of each line in each, and of heads of 64 leave half of the
// lanes without: a lone token over 1024 keys 8.7 us, 9.8 so; four tokens each over up to 9999 65 to 66, 66.3.
// (Keys, whose layout is the product's, in halves of a line a load: 73, the registers do not suffice.)
template <class T, int D, int Bits> struct Blocks {
    static constexpr int kN = D * Bits / 128;                // pieces of 16 bytes of a row
    static constexpr int kLoads = (16 * kN + 63) / 64;       // of 16 values
    static constexpr int kKeys = 16 / kLoads;                // of a load
    static constexpr int kChunks = 16 / Bits;                // of a piece, of eight elements
    struct Raw {
        uint32_t code[4 * kLoads], byte[kLoads];
    };
    int key, piece;
    bool writes, exists;    // the lane has a piece of a tile, and of the head
    uint32_t code_at, scale_at, code_slot, scale_slot;
    __device__ __forceinline__ Blocks(const taps_mx_attend_launch &p, int lane)
        : code_slot(p.v_slot), scale_slot(p.vs_slot) {
        key = lane / kN, piece = lane % kN;
        const int block = piece * kChunks / 4;
        writes = lane < kKeys * kN, exists = writes && 32 * block < (int)p.dim;
        code_at = exists ? key * code_slot + piece * 16 : 0;
        scale_at = exists ? key * scale_slot + block : 0;
    }
    __device__ __forceinline__ void fetch(Raw &to, const char *codes, const char *scales) const {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const u32x4 w = __builtin_nontemporal_load(
                (const u32x4 *)(codes + kKeys * i * code_slot + code_at));
#pragma unroll
            for (int j = 0; j < 4; ++j) to.code[4 * i + j] = w[j];
            to.byte[i] = (uint8_t)(scales + kKeys * i * scale_slot)[scale_at];
        }
    }
    static __device__ __forceinline__ void clear(Raw &of, int load) {
#pragma unroll
        for (int i = 0; i < 4; ++i) of.code[4 * load + i] = 0;
        of.byte[load] = 127;
    }
    // Where the lane's chunks of eight values go: at ^ 16 j, those of another load kKeys rows further.
    __device__ __forceinline__ uint32_t place() const {
        return key * Values<D, Bits>::kRow + 16 * ((kChunks * piece) ^ Values<D, Bits>::mask(key));
    }
    static __device__ __forceinline__ u32x4 eight(const Raw &of, int load, int j, float scale) {
        return mx_eight<T, Bits>(of.code + 4 * load + j * kWords<Bits>, scale);
    }
};

template <int D, int Waves> constexpr int few_bytes() {
    return max_of(Waves * Values<D, 4>::kBytes, joined_bytes<D, Waves, kFewRows>()) + 8 * Waves * kFewRows;
}

template <class T, int D, int Bits, int Waves>
__device__ __forceinline__ void attend_few(const taps_mx_attend_launch &p, const taps_plan_item &item,
                                           uint32_t head, char *lds) {
    constexpr int kSteps = D / 32, kBlocks = D / 16, kStep = Waves * kNarrowKeys;
    using Part = Piece<D, Bits>;
    using Image = Values<D, Bits>;
    using Lines = Blocks<T, D, Bits>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t *pages = p.pages + item.page0;
    const int lo = item.lo, hi = item.hi, start = lo & ~31;
    const float c = p.scale * kLog2e;
    const int row = item.row0 + (lane & 15), quarter = lane >> 4;
    const bool real = row < item.rows;
    const int token = row / (int)p.group, sub = row - token * (int)p.group;
    // keys of the item that this lane's row sees: first .. last
    int first = lo, last = hi - 1;
    if (p.causal) {
        const int pos = item.first_pos + token;
        last = min(last, pos);
        if (p.window) first = max(first, pos - (int)p.window + 1);
    }
    if (!real) last = -1, first = 0;
    s16x8 q[kSteps];
    {
        const char *at = p.q + (int64_t)(item.token0 + token) * p.q_token +
                         (int64_t)(head * p.group + sub) * p.q_head;
#pragma unroll
        for (int k = 0; k < kSteps; ++k) {
            const int d = 8 * (kSteps * quarter + k);
            q[k] = s16x8{};
            if (real && d < (int)p.dim) q[k] = *(const s16x8 *)(at + 2 * d);
        }
    }
    float m = real ? kMinusInf : 0.f, l = 0.f;   // a row that is not there never raises it
    f32x4 o[kBlocks];
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) o[b] = f32x4{};
    const Seen seen(p, item, item.row0);

    const Keys<T, D, Bits, false> keys(p, item, head, lane);
    const Keys<T, D, Bits, true> values(p, item, head, lane);
    const Lines blocks(p, lane);
    // Two tiles are on their way at any time, each in a set of registers.
    struct Set {
        Part k[2];
        typename Lines::Raw v[2];
        int page[2];
    } set[2];
    const bool one_page = p.page_log2 >= 5;   // tiles start at multiples of 32
    const auto look_up = [&](Set &s, int t) {
        s.page[0] = page_at(p, pages, t, lo, hi);
        if (!one_page) s.page[1] = page_at(p, pages, t + 16, lo, hi);
    };
    const auto fetch = [&](Set &s, int t) {
        auto k0 = keys.at(t, s.page[0]), k1 = keys.behind(k0);
        auto v0 = values.at(t, s.page[0]), v1 = values.behind(v0);
        if (!one_page) {
            k0 = keys.nearest(t, s.page[0]), k1 = keys.nearest(t + 16, s.page[1]);
            v0 = values.nearest(t, s.page[0]), v1 = values.nearest(t + 16, s.page[1]);
        }
        keys.fetch(s.k[0], k0);
        keys.fetch(s.k[1], k1);
        blocks.fetch(s.v[0], v0.codes, v0.scales);
        blocks.fetch(s.v[1], v1.codes, v1.scales);
    };
    char *tile = lds + wave * Image::kBytes;
    // This wavefront's tiles: those that not all rows see all of, the edges, come first, then those
    // between them, plain .. plain_end - 1.
    const int begin = start + kNarrowKeys * wave;
    const auto up = [&](int t) {   // the first tile from t on
        return t <= begin ? begin : begin + (t - begin + kStep - 1) / kStep * kStep;
    };
    const int plain = up(seen.from), plain_end = max(seen.to - kNarrowKeys + 2, plain);
    const auto edge_from = [&](int t) { return t >= plain && t < plain_end ? up(plain_end) : t; };
    // where a lane writes its piece, and reads its columns of the first 16
    uint32_t write_at = blocks.place();
    // lane of a group of 16: key (lane % 16) / 4 of the quarter's four, columns 4 (lane % 4) ..
    const int v_key = 4 * quarter + (lane & 15) / 4;
    uint32_t read_at = v_key * Image::kRow + 8 * (lane & 1) +
                       16 * (((lane >> 1) & 1) ^ Image::mask(v_key));
    // A tile of 32 keys; an edge: some rows do not see some of them.  Again: maxima and sums are
    // known, and an edge's rows are taken one by one, with zeros for the values that a row does not see.
    // next: the tile that the set of registers is for then (hi: none), after_next: the one after it
    const auto step = [&](auto edge, auto again, auto surely, Set &s, int t0, int next, int after_next) {
        constexpr bool kEdge = decltype(edge)::value, kAgain = decltype(again)::value;
        // no address below is kept from tile to tile, registers are few
        asm volatile("" : "+v"(write_at), "+v"(read_at));
        // what was loaded is used here and not, shifted, right behind the load, which would wait for it
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < Part::kBytes; ++i) asm volatile("" : "+v"(s.k[h].byte[i]));
#pragma unroll
            for (int i = 0; i < Lines::kLoads; ++i) asm volatile("" : "+v"(s.v[h].byte[i]));
        }
        f32x4 x[2] = {};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            // those that are not there may be anything: their scores are replaced
            keys.blank_missing(s.k[h]);
#pragma unroll
            for (int k = 0; k < kSteps; ++k)
                x[h] = SmallMfma<T>::run(
                    __builtin_bit_cast(s16x8, s.k[h].template eight<T>(k, lane)), q[k], x[h]);
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int i = 0; i < Lines::kLoads; ++i) {
                const int key = t0 + 16 * h + Lines::kKeys * i + blocks.key;
                if ((kSteps == 2 && !blocks.exists) || (kEdge && (key < lo || key >= hi)))
                    blocks.clear(s.v[h], i);
                const float scale = mx_scale(s.v[h].byte[i]);
#pragma unroll
                for (int j = 0; j < Lines::kChunks; ++j) {
                    const u32x4 v = blocks.eight(s.v[h], i, j, scale);
                    if (Lines::kKeys * Lines::kN == 64 || blocks.writes)
                        *(u32x4 *)(tile + (write_at ^ (16 * j)) +
                                   (16 * h + Lines::kKeys * i) * Image::kRow) = v;
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        exchange();
        if (!kAgain && (decltype(surely)::value || next < hi)) {
            fetch(s, next);
            look_up(s, after_next);
        }
        // x[h][i]: key t0 + 16 h + 4 quarter + i
        if (kEdge) {
            const uint32_t sees = max(last - first + 1, 0), at = t0 + 4 * quarter - first;
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 4; ++i) x[h][i] = at + (16 * h + i) < sees ? x[h][i] : kMinusInf;
        }
        u32x4 y;
        const auto numerators = [&]() {
            const float shift = m <= kNoScore ? 0.f : m * c - kLiftLog2<T>;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = __builtin_amdgcn_exp2f(x[i / 2][2 * (i % 2)] * c - shift);
                const float f = __builtin_amdgcn_exp2f(x[i / 2][2 * (i % 2) + 1] * c - shift);
                sum += e + f;
                y[i] = pack2<T>(e, f);
            }
            return sum;
        };
        float sum = numerators();
        // the first keys, and scores too far above the maximum
        if (!kAgain && __any(m == kMinusInf || sum > kMostSum<T>)) {
            float most = x[0][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) most = fmaxf(most, x[i / 4][i % 4]);
            most = half_max(most);
            most = fmaxf(most, __shfl_xor(most, 16, 64));
            const float to = fmaxf(m, most);
            const float by = to == kMinusInf ? 1.f : __builtin_amdgcn_exp2f((m - to) * c);
            m = to;
            l *= by;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b) o[b] *= by;
            sum = numerators();
        }
        if (!kAgain) l += sum;
        // 16 columns of the values as the second product's operand
        const auto columns = [&](int b) {
            const char *at = tile + (read_at ^ (32 * b));
            const s16x4 u = Rows<T, D>::transposed(at);
            const s16x4 w = Rows<T, D>::transposed(at + 16 * Image::kRow);
            return s16x8{u[0], u[1], u[2], u[3], w[0], w[1], w[2], w[3]};
        };
        if constexpr (!kAgain || !kEdge) {
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
                o[b] = SmallMfma<T>::run(columns(b), __builtin_bit_cast(s16x8, y), o[b]);
        } else {
            const int rows = __builtin_amdgcn_readfirstlane(min(kFewRows, item.rows - item.row0));
            for (int r = 0; r < rows; ++r) {
                const int from = __shfl(first, r, 64), to = __shfl(last, r, 64);
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    s16x8 v = columns(b);
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const int key = t0 + 16 * (e / 4) + 4 * quarter + e % 4;
                        v[e] = key >= from && key <= to ? v[e] : (short)0;
                    }
                    const f32x4 one = SmallMfma<T>::run(v, __builtin_bit_cast(s16x8, y), f32x4{});
                    __builtin_amdgcn_sched_barrier(0);   // whatever rows the lanes have
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[b][i] = (lane & 15) == r ? o[b][i] + one[i] : o[b][i];
                }
            }
        }
        exchange();
    };
    if (lo < hi) {
        const int last_set = plain + kStep < plain_end ? plain + kStep : hi;   // of set 0, after the edges
        int t0 = edge_from(begin);
        const int first_set = t0 < hi ? t0 : last_set;
        look_up(set[1], plain);
        look_up(set[0], first_set);
        if (plain < plain_end) fetch(set[1], plain);   // in the order in which they are waited for
        if (first_set < hi) fetch(set[0], first_set);
        look_up(set[1], plain + 2 * kStep);
        const auto after = [&](int t) {
            const int next = edge_from(t + kStep);
            return next < hi ? next : last_set;
        };
        look_up(set[0], t0 < hi ? after(t0) : plain + 3 * kStep);
        while (t0 < hi) {
            const int next = after(t0);
            step(True{}, False{}, False{}, set[0], t0, next, next == last_set ? plain + 3 * kStep : after(next));
            t0 = edge_from(t0 + kStep);
        }
        for (t0 = plain; t0 + 3 * kStep < plain_end; t0 += 2 * kStep) {
            step(False{}, False{}, True{}, set[1], t0, t0 + 2 * kStep, t0 + 4 * kStep);
            step(False{}, False{}, True{}, set[0], t0 + kStep, t0 + 3 * kStep, t0 + 5 * kStep);
        }
        for (; t0 < plain_end; t0 += 2 * kStep) {   // up to three
            const int next = t0 + 2 * kStep < plain_end ? t0 + 2 * kStep : hi;
            step(False{}, False{}, False{}, set[1], t0, next, hi);
            if (t0 + kStep < plain_end) step(False{}, False{}, False{}, set[0], t0 + kStep, hi, hi);
        }
        // The numerator of a hidden key, 0, times a value that is infinite or NaN is NaN.  Only where
        // rows differ in what they see is there such a thing; all of them are taken again then.
        if (seen.differ(item)) {
            float sum = 0.f;
#pragma unroll
            for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                for (int i = 0; i < 4; ++i) sum += o[b][i] * 0.f;
            if (__builtin_expect(__any(sum != sum), 0)) {
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) o[b] = f32x4{};
                for (t0 = begin; t0 < hi; t0 += kStep) {
                    look_up(set[0], t0);
                    fetch(set[0], t0);
                    step(True{}, True{}, False{}, set[0], t0, hi, hi);
                }
            }
        }
    }
    float total = half_sum(l);
    total += __shfl_xor(total, 16, 64);
    if (total == 0.f && m == kMinusInf && first <= last) m = kNoScore;

    float *ml = (float *)(lds + few_bytes<D, Waves>() - 8 * Waves * kFewRows);
    float *sums = (float *)lds;
    __syncthreads();   // the tiles are done with
    if (quarter == 0) {
        ml[2 * (wave * kFewRows + lane)] = m;
        ml[2 * (wave * kFewRows + lane) + 1] = total;
    }
    __syncthreads();
    float top = kMinusInf;
#pragma unroll
    for (int w = 0; w < Waves; ++w) top = fmaxf(top, ml[2 * (w * kFewRows + (lane & 15))]);
    const float by = m == kMinusInf ? 0.f : __builtin_amdgcn_exp2f((m - top) * c);
    float *mine = sums + (wave * kFewRows + (lane & 15)) * (D + 4);
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) *(f32x4 *)(mine + 16 * b + 4 * quarter) = o[b] * by;
    __syncthreads();
    write_joined<T, D, Waves, kFewRows>(p, item, head, sums, ml);
}

// Four wavefronts an item, three items to a unit; eight where there are no more items than units
// and a lone one's time counts (16 heads of 64, one token over 1024 keys: 9.8 us for 11.3 when it was chosen; 64
// tokens over up to 4000, 784 items: 48 for 39).  The units are those of the whole card, however many a plan
// was cut for: results do not depend on the choice, times of a part of a card would.
constexpr uint32_t kUnits = 256;

template <class T, int D, int Bits, int Waves>
__global__ __launch_bounds__(64 * Waves, Waves == 4 ? 3 : 2) void k_mx_attend_few(taps_mx_attend_launch p) {
    __shared__ __attribute__((aligned(16))) char lds[few_bytes<D, Waves>()];
    const uint32_t head = blockIdx.x % p.kv_heads;
    attend_few<T, D, Bits, Waves>(p, p.items[blockIdx.x / p.kv_heads], head, lds);
}

// Any item but a wide one; two fit a unit, three for heads of up to 64.  8 prompts of 1024, 16 heads of
// 64 in 4 bits: 41 us (34 over a 16-bit cache, whose tiles go past the registers): a third of the
// wavefronts' time are waits, the matrix cores are busy for 24 % of it.  16 times 8 tokens over 8192 keys, 32
// heads of 128 over 8, items of 32 rows: 40 and 5 for the join (102 in all over a 16-bit cache), 143 MB at
// 3.6 TB/s with one tile on its way; keys and values both pass through LDS, in use for 40 % of the time.
template <class T, int D, int Bits>
__global__ __launch_bounds__(kThreads, D <= 64 ? 3 : 2) void k_mx_attend(taps_mx_attend_launch p) {
    __shared__ __attribute__((aligned(16))) char lds[max_of(
        max_of(narrow_bytes<D>(), few_bytes<D, kWaves>()), 2 * Tile<D>::bytes(kWideKeys))];
    const uint32_t head = blockIdx.x % p.kv_heads;
    const taps_plan_item item = p.items[blockIdx.x / p.kv_heads];
    if (item.kind == kBlock)
        attend_block<T, D, Bits, 1>(p, item, head, lds);
    else if (item.rows - item.row0 <= kFewRows)
        attend_few<T, D, Bits, kWaves>(p, item, head, lds);
    else
        attend_narrow<T, D, Bits>(p, item, head, lds);
}

// The same with a unit for each: twice the wavefronts share a block's keys.  Prompts of up to 701 tokens
// and single ones, 212 items of up to 17 tiles one after the other: 24.7 us, 32.8 without.  Loads,
// conversions, products and softmax of a tile follow each other: 46 % of the wavefronts' time are waits, a
// unit's vector instructions issue for 40 % of it, its matrix cores are busy for 19 %.
// Items of 17 to 32 rows are blocks here, of whose eight wavefronts two have rows: 8 tokens over 8192 keys,
// 32 heads of 128 over 8, 27 us in 4 bits and 31 in 8 (21 over a 16-bit cache, in narrow items).
template <class T, int D, int Bits>
__global__ __launch_bounds__(2 * kThreads, 2) void k_mx_attend_alone(taps_mx_attend_launch p) {
    constexpr int kBlockBytes = max_of(4 * Tile<D>::bytes(kWideKeys), kBlockRows * (D + 8) * 4);
    __shared__ __attribute__((aligned(16))) char lds[max_of(few_bytes<D, 2 * kWaves>(), kBlockBytes)];
    const uint32_t head = blockIdx.x % p.kv_heads;
    const taps_plan_item item = p.items[blockIdx.x / p.kv_heads];
    if (item.kind == kNarrow && item.rows - item.row0 <= kFewRows)
        attend_few<T, D, Bits, 2 * kWaves>(p, item, head, lds);
    else
        attend_block<T, D, Bits, 2>(p, item, head, lds);
}

template <class T, int D, int Bits> void launch_items(taps_mx_attend_launch p, hipStream_t stream) {
    if constexpr (D > kWideAbove)
        in_slices(p, p.n_wide, kWideThreads, [&](const auto &s, uint32_t groups) {
            k_mx_attend_wide<T, D, Bits><<<groups, kWideThreads, 0, stream>>>(s);
        });
    p.items += p.n_wide;
    const uint32_t others = p.n_items - p.n_wide;
    const bool few = p.n_few == others;
    in_slices(p, others, 2 * kThreads, [&](const auto &s, uint32_t groups) {
        if (few && groups <= kUnits)
            k_mx_attend_few<T, D, Bits, 8><<<groups, 512, 0, stream>>>(s);
        else if (few)
            k_mx_attend_few<T, D, Bits, 4><<<groups, 256, 0, stream>>>(s);
        else if (groups <= kUnits)
            k_mx_attend_alone<T, D, Bits><<<groups, 2 * kThreads, 0, stream>>>(s);
        else
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
