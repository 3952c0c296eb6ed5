// taps_mx.hip -- the append to a cache in microscaling formats, and reading it back.
//
// A row is one head of one token's keys or values.  For a block of 32 elements with
// the largest magnitude a, with e the smallest integer from -110 on with a <= L 2^e,
//   code_i = nearest(x_i 2^-e),   x'_i = code_i 2^e.
// a 2^-E <= L depends on a's exponent and mantissa alone: integer work on its bits.
// The codes are the conversion instructions', which round to the nearest, the even one
// of two, and take 2^e themselves.
//
// Eight elements a lane: four lanes are a block, and meet for its largest magnitude.
// A rotated element's other half of the pair is in another lane (but for neighbouring
// pairs); lanes hand them over through LDS, inside a wavefront.
//
// Bytes bound both: a row is read and written once.  A group of lanes takes all heads of its token,
// so that a wavefront's groups read and write neighbouring slots of a head at a time, whole lines;
// with a token's heads over the groups a launch touched half lines all over the pages.
//   append   16384 tokens, 32 heads of 128 bf16, keys normed and rotated, to 4 bits: 268 MB in,
//            71 out, 70 us, 4.9 TB/s (about 130 with heads over the groups); to 8 bits 89, from
//            32 bits 124 and 139
//   read     the same back: 71 in, 268 out, 56 us, 6.1 TB/s
//            139 thousand tokens of 8 heads: 151 in, 568 out, 127 us, 5.7 TB/s (240); from 8
//            bits 143; to 32 bits, where a lane's eight elements are two stores with gaps
//            of 16 bytes between the lanes', 559, 2.3 TB/s
// Few tokens only wait for memory: 64 of 8 heads 4.4 and 3.2 us.
#include "taps_lanes.h"
#include "taps_mx_device.h"
#include "taps_mx_internal.h"

namespace {

constexpr int kThreads = 256;
constexpr uint32_t kGridRow = 1u << 22;   // workgroups in a launch's first dimension
__device__ __forceinline__ uint32_t workgroup() { return blockIdx.y * kGridRow + blockIdx.x; }
dim3 grid_of(uint32_t groups) {   // of keys, and of values
    return groups <= kGridRow ? dim3(groups, 1, 2)
                              : dim3(kGridRow, (groups + kGridRow - 1) / kGridRow, 2);
}

// Elements of a lane, and lanes of a row: whole blocks, up to the next power of two.
constexpr int kN = 8;
int lanes_of(uint32_t dim) { return dim <= 32 ? 4 : dim <= 64 ? 8 : 16; }

typedef float f32x4 __attribute__((ext_vector_type(4)));

template <class T> struct Raw {
    typedef T v8 __attribute__((ext_vector_type(8)));
    v8 x = {};
};

// Elements d .. d + 7 of a row of `dim`; zeros beyond it.  Rows are read once and not kept in the L2
// caches, whose lines the codes, written in parts of one, need: 8 prompts of 2048 appended and read
// back 126 us, 137 where they are kept (codes that are read back are, attention will read them: 129
// and 132 for 64 caches).
template <class T, bool Vectors>
__device__ __forceinline__ Raw<T> fetch(const T *row, int d, int dim) {
    Raw<T> r;
    if (Vectors) {
        if (d < dim) r.x = __builtin_nontemporal_load((const typename Raw<T>::v8 *)(row + d));
    } else {
#pragma unroll
        for (int i = 0; i < kN; ++i)
            if (d + i < dim) r.x[i] = row[d + i];
    }
    return r;
}

// cos and +-sin of a lane's elements, so that y = x cos + partner sin, and their partners'
// places in the row.  Elements that are not rotated stay as they are: x 1 + x 0, which is NaN only
// where x, and so its block, is not finite.
template <bool Vectors> struct Turn {
    float c[kN], s[kN];
    int d, half;        // first element; rotary / 2
    __device__ __forceinline__ void start(const taps_mx_append_launch &p, int64_t position, int d0) {
        d = d0, half = p.rotary / 2;
        const bool near = p.interleaved;   // pairs are neighbours
        const float *row = p.table + position * (int64_t)p.rotary;
#pragma unroll
        for (int i = 0; i < kN; ++i) c[i] = 1.f, s[i] = 0.f;
        if (d >= (int)p.rotary) return;
        if (Vectors && !near) {   // four elements lie in one half of the pairs
#pragma unroll
            for (int g = 0; g < kN; g += 4) {
                const bool b = d + g >= half;
                const int angle = b ? d + g - half : d + g;
                const f32x4 u = *(const f32x4 *)(row + angle), v = *(const f32x4 *)(row + half + angle);
#pragma unroll
                for (int i = 0; i < 4; ++i) c[g + i] = u[i], s[g + i] = b ? v[i] : -v[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < kN; ++i)
                if (rotated(i)) {
                    const bool b = near ? (d + i) & 1 : d + i >= half;
                    const int angle = near ? (d + i) / 2 : b ? d + i - half : d + i;
                    c[i] = row[angle];
                    s[i] = b ? row[half + angle] : -row[half + angle];
                }
        }
    }
    __device__ __forceinline__ bool rotated(int i) const { return d + i < 2 * half; }
    // Partners of elements i of this lane, from the row in LDS.
    __device__ __forceinline__ int partner(int i) const {
        return !rotated(i) ? d + i : d + i >= half ? d + i - half : d + i + half;
    }
    __device__ __forceinline__ void partners(const float *row, float (&y)[kN]) const {
        if (Vectors) {
#pragma unroll
            for (int g = 0; g < kN; g += 4) {
                const f32x4 u = *(const f32x4 *)(row + partner(g));
#pragma unroll
                for (int i = 0; i < 4; ++i) y[g + i] = u[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < kN; ++i) y[i] = row[partner(i)];
        }
    }
};

// 1 / sqrt(v) in 64 bits: the instruction's approximation and two steps of Newton's.  With the
// sum in 64 bits too, a key's codes do not hang on the order in which a wavefront adds: an element
// next to the border between two codes would show it.
__device__ __forceinline__ double inverse_root(double v) {
    double y = __builtin_amdgcn_rsq(v);
    if (v == 0.0 || v == __builtin_inf()) return y;
#pragma unroll
    for (int i = 0; i < 2; ++i) y = y + 0.5 * y * __builtin_fma(-v * y, y, 1.0);
    return y;
}

// Sum over groups of Lanes neighbouring lanes, in 64 bits.
template <int Control> __device__ __forceinline__ double of_lane(double v) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const uint32_t low = __builtin_amdgcn_mov_dpp((int)u, Control, 0xf, 0xf, true);
    const uint32_t high = __builtin_amdgcn_mov_dpp((int)(u >> 32), Control, 0xf, 0xf, true);
    return __builtin_bit_cast(double, (uint64_t)high << 32 | low);
}
template <int Lanes> __device__ __forceinline__ double row_sum64(double v) {
    v += of_lane<0xb1>(v);   // 1 0 3 2
    v += of_lane<0x4e>(v);   // 2 3 0 1
    if (Lanes > 4) v += of_lane<0x141>(v);   // 8 lanes mirrored: the other four
    if (Lanes > 8) v += of_lane<0x140>(v);   // 16 lanes mirrored: the other eight
    return v;
}

// Largest of four neighbouring lanes.
__device__ __forceinline__ uint32_t quad_max(uint32_t v) {
    v = max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true));   // 1 0 3 2
    return max(v, (uint32_t)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true));   // 2 3 0 1
}

// The scale byte of a block whose largest magnitude has these bits (finite).
template <int Bits> __device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
    // L = 1.75 x 2^2, 1.8125 x 2^8
    constexpr int kExponent = Bits == 4 ? 2 : 8;
    constexpr uint32_t kMantissa = Bits == 4 ? 0x600000 : 0x680000;
    const int e = (int)(top >> 23) - kExponent + ((top & 0x7fffff) > kMantissa);
    return (uint32_t)max(e, 17);   // 2^-110
}

// Eight elements' codes: x 2^-e, rounded.
template <int Bits>
__device__ __forceinline__ void encode(const float (&x)[kN], float scale, uint32_t (&to)[kWords<Bits>]) {
    if constexpr (Bits == 4) {
        uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, x[0], x[1], scale, 0);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[2], x[3], scale, 1);
        w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[4], x[5], scale, 2);
        to[0] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, x[6], x[7], scale, 3);
    } else {
        typedef short s16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            s16x2 w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(s16x2{}, x[4 * i], x[4 * i + 1], scale,
                                                               false);
            w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, x[4 * i + 2], x[4 * i + 3], scale, true);
            to[i] = __builtin_bit_cast(uint32_t, w);
        }
    }
}

// A workgroup's groups of lanes: `across` of them share a token's heads, the others take
// other tokens; keys and values are other workgroups' (blockIdx.z).
// Rows that a group has on their way at once.
constexpr int kAppendAtOnce = 4, kReadAtOnce = 8;
constexpr uint64_t kFill = 1024;   // workgroups that fill the card

template <class T, int Bits, bool Vectors, int Lanes>
__global__ __launch_bounds__(kThreads) void k_mx_append(taps_mx_append_launch p) {
    __shared__ __attribute__((aligned(16))) float lds[kThreads * kN];
    const uint32_t side = blockIdx.z, across = p.across, group = threadIdx.x / Lanes;
    const uint32_t t = workgroup() * (kThreads / Lanes / across) + group / across;
    if (t >= p.tokens) return;   // whole groups leave; sums and pairs stay inside a group
    const taps_plan_token place = p.plan_tokens[t];
    if (place.slot < 0) return;
    const int64_t page = place.slot >> p.page_log2;
    const int64_t slot = place.slot & ((1 << p.page_log2) - 1);
    const int lane = threadIdx.x % Lanes, d = kN * lane, dim = p.dim;
    const bool held = lane < 4 * (int)((p.dim + 31) / 32);   // codes of whole blocks
    const uint32_t h_first = group % across;
    const T *from = (const T *)p.src[side] + t * p.src_stride[side][0] + h_first * p.src_stride[side][1];
    const taps_mx_place &c = p.cache[side];
    char *codes = c.codes + page * c.code_stride[0] + slot * c.code_stride[2] +
                  h_first * c.code_stride[1] + lane * Bits;
    char *scales = c.scales + page * c.scale_stride[0] + slot * c.scale_stride[2] +
                   h_first * c.scale_stride[1] + lane / 4;
    const int64_t from_step = across * p.src_stride[side][1];
    const int64_t code_step = across * c.code_stride[1], scale_step = across * c.scale_stride[1];
    const bool norms = side == 0 && p.weight, rotates = side == 0 && p.rotary;
    Turn<Vectors> turn;
    if (rotates) turn.start(p, place.position, d);
    float *row = lds + group * Lanes * kN;
    float w[kN];
    if (norms) {
        if (p.float_weight) {
            const Raw<float> r = fetch<float, false>((const float *)p.weight, d, dim);
#pragma unroll
            for (int i = 0; i < kN; ++i) w[i] = r.x[i];
        } else {
            const Raw<T> r = fetch<T, false>((const T *)p.weight, d, dim);
#pragma unroll
            for (int i = 0; i < kN; ++i) w[i] = (float)r.x[i];
        }
    }
    for (uint32_t h0 = h_first; h0 < p.heads; h0 += kAppendAtOnce * across) {
        Raw<T> raw[kAppendAtOnce];
#pragma unroll
        for (int u = 0; u < kAppendAtOnce; ++u) {
            if (h0 + u * across < p.heads) raw[u] = fetch<T, Vectors>(from, d, dim);
            from += from_step;
        }
#pragma unroll
        for (int u = 0; u < kAppendAtOnce; ++u) {
#pragma clang fp contract(off)
            if (h0 + u * across >= p.heads) break;
            float x[kN];
#pragma unroll
            for (int i = 0; i < kN; ++i) x[i] = (float)raw[u].x[i];
            if (norms) {
                double sum = 0.0;
#pragma unroll
                for (int i = 0; i < kN; ++i) sum = __builtin_fma((double)x[i], (double)x[i], sum);
                const float rstd =
                    (float)inverse_root(row_sum64<Lanes>(sum) * p.inverse_dim + (double)p.eps);
#pragma unroll
                for (int i = 0; i < kN; ++i) x[i] = x[i] * rstd * w[i];   // 0 beyond the head: w is
            }
            if (rotates) {
                float y[kN];
                if (p.interleaved) {
#pragma unroll
                    for (int i = 0; i < kN; i += 2) {   // a neighbour's 0 would change the sign of x = -0
                        const bool turned = turn.rotated(i);
                        const float u = x[i], v = x[i + 1];
                        y[i] = turned ? v : u, y[i + 1] = turned ? u : v;
                    }
                } else {
                    *(f32x4 *)(row + d) = f32x4{x[0], x[1], x[2], x[3]};
                    *(f32x4 *)(row + d + 4) = f32x4{x[4], x[5], x[6], x[7]};
                    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                    __builtin_amdgcn_wave_barrier();
                    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                    turn.partners(row, y);
                    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
                    __builtin_amdgcn_wave_barrier();
                    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
                }
#pragma unroll
                for (int i = 0; i < kN; ++i) {
                    const float a = x[i] * turn.c[i], b = y[i] * turn.s[i];
                    x[i] = a + b;
                }
            }
            uint32_t top = 0;
#pragma unroll
            for (int i = 0; i < kN; ++i)
                top = max(top, __builtin_bit_cast(uint32_t, x[i]) & 0x7fffffff);
            top = quad_max(top);
            const uint32_t most = __builtin_bit_cast(uint32_t, p.most);
            uint32_t byte = scale_byte<Bits>(min(top, most)), code[kWords<Bits>];
            if (__builtin_expect(__any(top > most), 0)) {
                const bool finite = top < 0x7f800000;   // NaN's bits are the largest
#pragma unroll
                for (int i = 0; i < kN; ++i) x[i] = finite ? fminf(fmaxf(x[i], -p.most), p.most) : 0.f;
                encode<Bits>(x, mx_scale(byte), code);   // zeros whatever the scale
                byte = finite ? byte : TAPS_MX_NAN;
            } else {
                encode<Bits>(x, mx_scale(byte), code);
            }
            if (held) {
                if constexpr (Bits == 4)
                    *(uint32_t *)codes = code[0];
                else
                    *(u32x2 *)codes = u32x2{code[0], code[1]};
                if (lane % 4 == 0) *scales = (char)byte;
            }
            codes += code_step, scales += scale_step;
        }
    }
}

// Eight codes in the type T.
template <class T, int Bits>
__device__ __forceinline__ typename Raw<T>::v8 decode(const uint32_t *code, float scale) {
    if constexpr (sizeof(T) == 2) {
        return __builtin_bit_cast(typename Raw<T>::v8, mx_eight<T, Bits>(code, scale));
    } else {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        f32x2 y[4];
        if constexpr (Bits == 4) {
            y[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[0], scale, 0);
            y[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[0], scale, 1);
            y[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[0], scale, 2);
            y[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[0], scale, 3);
        } else {
            y[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(code[0], scale, false);
            y[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(code[0], scale, true);
            y[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(code[1], scale, false);
            y[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(code[1], scale, true);
        }
        typename Raw<T>::v8 x;
#pragma unroll
        for (int i = 0; i < kN; ++i) x[i] = y[i / 2][i % 2];
        return x;
    }
}

template <class T, int Bits, bool Vectors, int Lanes>
__global__ __launch_bounds__(kThreads) void k_mx_read(taps_mx_read_launch p) {
    const uint32_t side = blockIdx.z, across = p.across, group = threadIdx.x / Lanes;
    const uint32_t t = workgroup() * (kThreads / Lanes / across) + group / across;
    if (t >= p.tokens) return;
    int64_t at = p.wide_slots ? ((const int64_t *)p.slots)[t] : (int64_t)((const int32_t *)p.slots)[t];
    const bool good = at >= 0 && at < p.n_slots;
    if (!good) at = 0;
    const int64_t page = at >> p.page_log2, slot = at & ((1 << p.page_log2) - 1);
    const int lane = threadIdx.x % Lanes, d = kN * lane;
    if (d >= (int)p.dim) return;
    const uint32_t h_first = group % across;
    const taps_mx_place &c = p.cache[side];
    const char *codes = c.codes + page * c.code_stride[0] + slot * c.code_stride[2] +
                        h_first * c.code_stride[1] + lane * Bits;
    const char *scales = c.scales + page * c.scale_stride[0] + slot * c.scale_stride[2] +
                         h_first * c.scale_stride[1] + lane / 4;
    T *to = (T *)p.dst[side] + t * p.dst_stride[side][0] + h_first * p.dst_stride[side][1] + d;
    const int64_t code_step = across * c.code_stride[1], scale_step = across * c.scale_stride[1];
    const int64_t to_step = across * p.dst_stride[side][1];
    for (uint32_t h0 = h_first; h0 < p.heads; h0 += kReadAtOnce * across) {
        uint32_t code[kReadAtOnce][kWords<Bits>], byte[kReadAtOnce];
#pragma unroll
        for (int u = 0; u < kReadAtOnce; ++u) {
            if (h0 + u * across < p.heads) {
                if constexpr (Bits == 4) {
                    code[u][0] = *(const uint32_t *)codes;
                } else {
                    const u32x2 w = *(const u32x2 *)codes;
                    code[u][0] = w[0], code[u][1] = w[1];
                }
                byte[u] = (uint8_t)*scales;
            }
            codes += code_step, scales += scale_step;
        }
#pragma unroll
        for (int u = 0; u < kReadAtOnce; ++u) {
            if (h0 + u * across >= p.heads) break;
            const typename Raw<T>::v8 x =
                decode<T, Bits>(code[u], mx_scale(good ? byte[u] : TAPS_MX_NAN));
            if (Vectors) {
                __builtin_nontemporal_store(x, (typename Raw<T>::v8 *)to);
            } else {
#pragma unroll
                for (int i = 0; i < kN; ++i) to[i] = x[i];   // head_dim is a multiple of 8
            }
            to += to_step;
        }
    }
}

// Groups of lanes for a token's heads, a power of two: one, so that neighbouring groups read and
// write neighbouring slots, unless the launch would not fill the card then.
uint32_t across_of(uint32_t tokens, uint32_t heads, int lanes) {
    const uint32_t groups = kThreads / lanes;
    uint32_t across = 1;
    while (across < groups && across < heads && 2 * (uint64_t)tokens * across < kFill * groups) across *= 2;
    return across;
}
uint32_t workgroups_of(uint32_t tokens, uint32_t across, int lanes) {
    const uint32_t each = kThreads / lanes / across;
    return (tokens + each - 1) / each;
}

// f with the element type of `dtype`, the number of bits, whether rows are read in vectors and
// the lanes of a row, as types.
template <int N> struct Int {
    static constexpr int value = N;
};
template <class F> void choose(uint32_t dtype, uint32_t bits, bool vectors, int lanes, F &&f) {
    const auto by_lanes = [&](auto type, auto b, auto vec) {
        if (lanes == 4)
            f(type, b, vec, Int<4>{});
        else if (lanes == 8)
            f(type, b, vec, Int<8>{});
        else
            f(type, b, vec, Int<16>{});
    };
    const auto by_vectors = [&](auto type, auto b) {
        if (vectors)
            by_lanes(type, b, Int<1>{});
        else
            by_lanes(type, b, Int<0>{});
    };
    const auto by_bits = [&](auto type) {
        if (bits == 4)
            by_vectors(type, Int<4>{});
        else
            by_vectors(type, Int<8>{});
    };
    if (dtype == TAPS_BF16)
        by_bits((__bf16)0.f);
    else if (dtype == TAPS_F16)
        by_bits((_Float16)0.f);
    else
        by_bits(0.f);
}

}  // namespace

hipError_t taps_launch_mx_append(taps_mx_append_launch p, uint32_t dtype, uint32_t bits,
                                 bool vectors, hipStream_t stream) {
    const int lanes = lanes_of(p.dim);
    p.across = across_of(p.tokens, p.heads, lanes);
    choose(dtype, bits, vectors, lanes, [&](auto type, auto b, auto vec, auto n) {
        k_mx_append<decltype(type), b.value, vec.value != 0, n.value>
            <<<grid_of(workgroups_of(p.tokens, p.across, lanes)), kThreads, 0, stream>>>(p);
    });
    return hipGetLastError();
}

hipError_t taps_launch_mx_read(taps_mx_read_launch p, uint32_t dtype, uint32_t bits,
                               bool vectors, hipStream_t stream) {
    const int lanes = lanes_of(p.dim);
    p.across = across_of(p.tokens, p.heads, lanes);
    choose(dtype, bits, vectors, lanes, [&](auto type, auto b, auto vec, auto n) {
        k_mx_read<decltype(type), b.value, vec.value != 0, n.value>
            <<<grid_of(workgroups_of(p.tokens, p.across, lanes)), kThreads, 0, stream>>>(p);
    });
    return hipGetLastError();
}
