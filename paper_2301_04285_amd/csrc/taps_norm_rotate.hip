// taps_norm_rotate.hip -- norm and rotation of heads, their gradients, and the
// append to a paged cache.
//
// A row is one head of one token.  In 32 bits,
//   y = R n,  n_i = x_i rstd w_i,  rstd = (mean x^2 + eps)^(-1/2),
// R the rotation of the pairs (a, b) by the token's angles.  With g = dL/dy,
// h = R^T g and xh = x rstd,
//   dL/dw_i = sum over rows of h_i xh_i
//   dL/dx   = rstd (h w - xh mean(h w xh)).
// Each row is read once and written once: bytes bound these kernels.  64 heads of
// 128 bf16 elements of 8192 tokens (a large copy does 4.9 TB/s, reads and writes
// together):
//   forwards   268 MB in  48 us  5.6 TB/s
//   backwards  403 MB in 102 us  4.0 TB/s, and 6 us for the weights' gradients
//   append     537 MB in 100 us  5.4 TB/s (16384 tokens of 32 heads, and values)
// Few rows (one token of 32 heads of 64: 3.5 us) only wait for memory.
//
// A row belongs to a group of lanes of one wavefront.  A lane holds the same
// pairs of every row it takes: `a` members in one chunk, `b` members in
// another, so that the rotation needs no other lane, and the table's entries and
// the weights are read once per token and kept.  Elements that are not rotated
// are held in pairs too, but each stays as it is: a product with a sine of 0
// would hand on infinities.  The norm's sum is the only thing that crosses lanes.
#include "taps_attention_internal.h"
#include "taps_lanes.h"

namespace {

constexpr int kThreads = 256;
// Workgroups in the first dimension of a launch, which holds fewer than 2^32
// threads; the second dimension numbers rows of as many.
constexpr uint32_t kGridRow = 1u << 22;
__device__ __forceinline__ uint32_t workgroup() { return blockIdx.y * kGridRow + blockIdx.x; }
dim3 grid_of(uint32_t groups) {
    return groups <= kGridRow ? dim3(groups) : dim3(kGridRow, (groups + kGridRow - 1) / kGridRow);
}
// Rows that a group of lanes has on their way at once.
constexpr int kAtOnce = 4;

template <class T> __device__ __forceinline__ float to_f32(T v) { return (float)v; }
template <class T> __device__ __forceinline__ T from_f32(float v) { return (T)v; }

// The pairs a lane holds.  Vectors: a chunk of four consecutive elements for
// `a` and one for `b` (8 or 16 bytes each), eight elements a lane; needs
// head_dim and rotary_dim to be multiples of 8 and rows that start at
// multiples of four elements.  Otherwise two pairs a lane, one element at a
// time, a wavefront per row: any dimension, stride and alignment.
template <bool Vectors> struct Pairs;

template <> struct Pairs<true> {
    static constexpr int kN = 4;
    // lanes of a row: head_dim / 8, up to the next power of two
    static __host__ __device__ __forceinline__ int lanes(uint32_t dim) {
        return dim <= 8 ? 1 : dim <= 16 ? 2 : dim <= 32 ? 4 : dim <= 64 ? 8 : dim <= 128 ? 16 : 32;
    }
    int a0, b0, angle0;
    bool live, rotated, interleaved;
    __device__ Pairs(const taps_rows_launch &p, int lane) {
        const int rot8 = p.rotary / 8;
        live = lane < (int)p.dim / 8;
        rotated = lane < rot8;
        interleaved = p.interleaved && rotated;
        angle0 = 4 * lane;
        if (interleaved || !rotated) {   // neighbouring chunks
            a0 = 8 * lane;
            b0 = a0 + 4;
        } else {
            a0 = 4 * lane;
            b0 = a0 + p.rotary / 2;
        }
    }
    __device__ __forceinline__ bool turns(int) const { return rotated; }
    template <class T> struct Raw {
        typedef T v4 __attribute__((ext_vector_type(4)));
        v4 u = {}, v = {};
    };
    template <class T> __device__ __forceinline__ Raw<T> fetch(const T *row) const {
        typedef typename Raw<T>::v4 v4;
        Raw<T> r;
        if (live) {
            r.u = *(const v4 *)(row + a0);
            r.v = *(const v4 *)(row + b0);
        }
        return r;
    }
    template <class T>
    __device__ __forceinline__ void unpack(const Raw<T> &r, float (&a)[kN], float (&b)[kN]) const {
        if (interleaved) {
            for (int i = 0; i < 2; ++i) {
                a[i] = to_f32<T>(r.u[2 * i]), b[i] = to_f32<T>(r.u[2 * i + 1]);
                a[2 + i] = to_f32<T>(r.v[2 * i]), b[2 + i] = to_f32<T>(r.v[2 * i + 1]);
            }
        } else {
            for (int i = 0; i < 4; ++i) a[i] = to_f32<T>(r.u[i]), b[i] = to_f32<T>(r.v[i]);
        }
    }
    template <class T>
    __device__ __forceinline__ void store(T *row, const float (&a)[kN], const float (&b)[kN]) const {
        typedef T v4 __attribute__((ext_vector_type(4)));
        if (!live) return;
        v4 u, v;
        if (interleaved) {
            for (int i = 0; i < 2; ++i) {
                u[2 * i] = from_f32<T>(a[i]), u[2 * i + 1] = from_f32<T>(b[i]);
                v[2 * i] = from_f32<T>(a[2 + i]), v[2 * i + 1] = from_f32<T>(b[2 + i]);
            }
        } else {
            for (int i = 0; i < 4; ++i) u[i] = from_f32<T>(a[i]), v[i] = from_f32<T>(b[i]);
        }
        // past the caches: 268 MB in and out 50.1 -> 47.3 us forwards, 112 -> 110
        // backwards, an append of 545 MB 104.3 -> 101.1 (not so by a branch on the
        // size, which the compiler joins into ordinary stores)
        __builtin_nontemporal_store(u, (v4 *)(row + a0));
        __builtin_nontemporal_store(v, (v4 *)(row + b0));
    }
    __device__ __forceinline__ void angles(const taps_rows_launch &p, int64_t pos, float (&c)[kN],
                                           float (&s)[kN]) const {
        typedef float v4 __attribute__((ext_vector_type(4)));
        for (int i = 0; i < 4; ++i) c[i] = 1.f, s[i] = 0.f;
        if (rotated) {
            const float *row = p.table + pos * p.rotary + angle0;
            // rows start at multiples of rotary_dim floats: 32 bytes and more
            const v4 u = *(const v4 *)row, v = *(const v4 *)(row + p.rotary / 2);
            for (int i = 0; i < 4; ++i) c[i] = u[i], s[i] = v[i];
        }
    }
};

template <> struct Pairs<false> {
    static constexpr int kN = 2;   // 64 lanes x 2 pairs: head_dim up to 256
    static __host__ __device__ __forceinline__ int lanes(uint32_t) { return 64; }
    int ia[kN], ib[kN], ang[kN];   // -1: none
    __device__ Pairs(const taps_rows_launch &p, int lane) {
        const int half = p.rotary / 2;
        for (int i = 0; i < kN; ++i) {
            const int k = lane + 64 * i;
            ang[i] = k < half ? k : -1;
            if (k < half) {
                ia[i] = p.interleaved ? 2 * k : k;
                ib[i] = p.interleaved ? 2 * k + 1 : k + half;
            } else {
                ia[i] = 2 * k;   // = rotary + 2 (k - half)
                ib[i] = 2 * k + 1;
            }
            if (ia[i] >= (int)p.dim) ia[i] = -1;
            if (ib[i] >= (int)p.dim) ib[i] = -1;
        }
    }
    __device__ __forceinline__ bool turns(int i) const { return ang[i] >= 0; }
    template <class T> struct Raw {
        T a[kN], b[kN];
    };
    template <class T> __device__ __forceinline__ Raw<T> fetch(const T *row) const {
        Raw<T> r;
        for (int i = 0; i < kN; ++i) {
            r.a[i] = ia[i] >= 0 ? row[ia[i]] : (T)0.f;
            r.b[i] = ib[i] >= 0 ? row[ib[i]] : (T)0.f;
        }
        return r;
    }
    template <class T>
    __device__ __forceinline__ void unpack(const Raw<T> &r, float (&a)[kN], float (&b)[kN]) const {
        for (int i = 0; i < kN; ++i) a[i] = to_f32<T>(r.a[i]), b[i] = to_f32<T>(r.b[i]);
    }
    template <class T>
    __device__ __forceinline__ void store(T *row, const float (&a)[kN], const float (&b)[kN]) const {
        for (int i = 0; i < kN; ++i) {
            if (ia[i] >= 0) row[ia[i]] = from_f32<T>(a[i]);
            if (ib[i] >= 0) row[ib[i]] = from_f32<T>(b[i]);
        }
    }
    __device__ __forceinline__ void angles(const taps_rows_launch &p, int64_t pos, float (&c)[kN],
                                           float (&s)[kN]) const {
        for (int i = 0; i < kN; ++i) {
            const float *row = p.table + pos * p.rotary;
            c[i] = ang[i] >= 0 ? row[ang[i]] : 1.f;
            s[i] = ang[i] >= 0 ? row[p.rotary / 2 + ang[i]] : 0.f;
        }
    }
};

template <class P, class T>
__device__ __forceinline__ void load_weight(const taps_rows_launch &p, const P &pairs, int side,
                                            float (&a)[P::kN], float (&b)[P::kN]) {
    if (!p.norm[side]) {
        for (int i = 0; i < P::kN; ++i) a[i] = b[i] = 1.f;
    } else if (p.float_weights) {
        pairs.unpack(pairs.fetch((const float *)p.weight[side]), a, b);
    } else {
        pairs.unpack(pairs.fetch((const T *)p.weight[side]), a, b);
    }
}

__device__ __forceinline__ int64_t position_of(const taps_rows_launch &p, uint32_t b, uint32_t t) {
    if (!p.positions) return p.first + t;
    const uint64_t at = (uint64_t)b * p.tokens + t;
    return p.wide_positions ? ((const int64_t *)p.positions)[at]
                            : (int64_t)((const int32_t *)p.positions)[at];
}

// Row (b, t, h) of a side's tensor; h counts the heads of both sides.
template <class T>
__device__ __forceinline__ T *row_of(const taps_rows_launch &p, const void *const (&data)[2],
                                     const int64_t (&stride)[2][3], uint32_t b, uint32_t t,
                                     uint32_t h) {
    const int side = h >= p.heads[0];
    const uint32_t hh = side ? h - p.heads[0] : h;
    return (T *)(side ? data[1] : data[0]) + b * (side ? stride[1][0] : stride[0][0]) +
           t * (side ? stride[1][1] : stride[0][1]) + hh * (side ? stride[1][2] : stride[0][2]);
}

// How a workgroup's groups of lanes share tokens and heads: `across` groups
// take a token's heads in turns, the others take other tokens.
struct Split {
    uint32_t across, tokens;   // groups per token, tokens per workgroup
    __host__ __device__ Split(uint32_t heads, int lanes) {
        const uint32_t groups = kThreads / lanes;
        across = groups;
        while (across > 1 && across / 2 >= heads) across /= 2;
        tokens = groups / across;
    }
};

template <class T, bool Vectors, int Lanes>
__global__ __launch_bounds__(kThreads) void k_norm_rotate(taps_rows_launch p) {
    using P = Pairs<Vectors>;
    constexpr int N = P::kN;
    const uint32_t heads = p.heads[0] + p.heads[1];
    const Split split(heads, Lanes);
    const uint32_t group = threadIdx.x / Lanes;
    const uint32_t token = workgroup() * split.tokens + group / split.across;
    if (token >= p.batch * p.tokens) return;   // whole groups leave; sums stay inside a group
    const uint32_t b = token / p.tokens, t = token % p.tokens;
    const P pairs(p, threadIdx.x % Lanes);
    const int64_t pos = position_of(p, b, t);
    const bool good = p.rotary == 0 || (pos >= 0 && pos < (int64_t)p.n_positions);
    float c[N], s[N], wa[2][N], wb[2][N];
    pairs.angles(p, good ? pos : 0, c, s);
    if (!good)
        for (int i = 0; i < N; ++i) c[i] = s[i] = __builtin_nanf("");
    load_weight<P, T>(p, pairs, 0, wa[0], wb[0]);
    load_weight<P, T>(p, pairs, 1, wa[1], wb[1]);
    const float inv_dim = 1.f / (float)p.dim;
    for (uint32_t h0 = group % split.across; h0 < heads; h0 += kAtOnce * split.across) {
        typename P::template Raw<T> raw[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
            if (h0 + u * split.across < heads)
                raw[u] = pairs.fetch(row_of<const T>(p, p.src, p.src_stride, b, t,
                                                     h0 + u * split.across));
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const uint32_t h = h0 + u * split.across;
            if (h >= heads) break;
            const int side = h >= p.heads[0];
            float a[N], bb[N];
            pairs.unpack(raw[u], a, bb);
            float rstd = 1.f;
            if (p.norm[side]) {
                float sum = 0.f;
                for (int i = 0; i < N; ++i) sum += a[i] * a[i] + bb[i] * bb[i];
                rstd = rsqrtf(row_sum<Lanes>(sum) * inv_dim + p.eps);
            }
            for (int i = 0; i < N; ++i) {
                const float na = a[i] * rstd * (side ? wa[1][i] : wa[0][i]);
                const float nb = bb[i] * rstd * (side ? wb[1][i] : wb[0][i]);
                a[i] = pairs.turns(i) ? na * c[i] - nb * s[i] : na;
                bb[i] = pairs.turns(i) ? nb * c[i] + na * s[i] : nb;
            }
            // a position off the table: what is not rotated is NaN too
            if (!good)
                for (int i = 0; i < N; ++i) a[i] = bb[i] = __builtin_nanf("");
            pairs.store(row_of<T>(p, p.dst, p.dst_stride, b, t, h), a, bb);
        }
    }
}

// k rows are normed and rotated, v rows copied; the plan names the slot.
template <class T, bool Vectors, int Lanes>
__global__ __launch_bounds__(kThreads) void k_append(taps_rows_launch p) {
    using P = Pairs<Vectors>;
    constexpr int N = P::kN;
    const uint32_t heads = 2 * p.heads[0];
    const Split split(heads, Lanes);
    const uint32_t group = threadIdx.x / Lanes;
    const uint32_t t = workgroup() * split.tokens + group / split.across;
    if (t >= p.tokens) return;
    const taps_plan_token place = p.plan_tokens[t];
    if (place.slot < 0) return;
    const int64_t page = place.slot >> p.page_log2;
    const int64_t slot = place.slot & ((1 << p.page_log2) - 1);
    const P pairs(p, threadIdx.x % Lanes);
    float c[N], s[N], wa[N], wb[N];
    pairs.angles(p, place.position, c, s);
    load_weight<P, T>(p, pairs, 0, wa, wb);
    const float inv_dim = 1.f / (float)p.dim;
    for (uint32_t h0 = group % split.across; h0 < heads; h0 += kAtOnce * split.across) {
        typename P::template Raw<T> raw[kAtOnce];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
            if (h0 + u * split.across < heads)
                raw[u] = pairs.fetch(row_of<const T>(p, p.src, p.src_stride, 0, t,
                                                     h0 + u * split.across));
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const uint32_t h = h0 + u * split.across;
            if (h >= heads) break;
            const int side = h >= p.heads[0];
            const uint32_t hh = side ? h - p.heads[0] : h;
            float a[N], b[N];
            pairs.unpack(raw[u], a, b);
            if (!side) {
                float rstd = 1.f;
                if (p.norm[0]) {
                    float sum = 0.f;
                    for (int i = 0; i < N; ++i) sum += a[i] * a[i] + b[i] * b[i];
                    rstd = rsqrtf(row_sum<Lanes>(sum) * inv_dim + p.eps);
                }
                for (int i = 0; i < N; ++i) {
                    const float na = a[i] * rstd * wa[i], nb = b[i] * rstd * wb[i];
                    a[i] = pairs.turns(i) ? na * c[i] - nb * s[i] : na;
                    b[i] = pairs.turns(i) ? nb * c[i] + na * s[i] : nb;
                }
            }
            pairs.store((T *)p.dst[side] + page * p.dst_stride[side][0] +
                            hh * p.dst_stride[side][1] + slot * p.dst_stride[side][2], a, b);
        }
    }
}

// Gradients.  Workgroups take tokens in turns and keep the weights' gradients
// of their rows in registers; at the end the groups of lanes add theirs up in
// LDS, in order, and leave one partial sum per workgroup.
template <class T, bool Vectors, int Lanes>
__global__ __launch_bounds__(kThreads) void k_norm_rotate_backward(taps_rows_launch p) {
    using P = Pairs<Vectors>;
    constexpr int N = P::kN;
    const uint32_t heads = p.heads[0] + p.heads[1];
    const Split split(heads, Lanes);
    const uint32_t group = threadIdx.x / Lanes, lane = threadIdx.x % Lanes;
    const P pairs(p, lane);
    float wa[2][N], wb[2][N], ga[2][N] = {}, gb[2][N] = {};
    load_weight<P, T>(p, pairs, 0, wa[0], wb[0]);
    load_weight<P, T>(p, pairs, 1, wa[1], wb[1]);
    const float inv_dim = 1.f / (float)p.dim;
    const uint32_t n_tokens = p.batch * p.tokens;
    for (uint32_t token = blockIdx.x * split.tokens + group / split.across; token < n_tokens;
         token += gridDim.x * split.tokens) {
        const uint32_t b = token / p.tokens, t = token % p.tokens;
        const int64_t pos = position_of(p, b, t);
        const bool good = p.rotary == 0 || (pos >= 0 && pos < (int64_t)p.n_positions);
        float c[N], s[N];
        pairs.angles(p, good ? pos : 0, c, s);
        if (!good)
            for (int i = 0; i < N; ++i) c[i] = s[i] = __builtin_nanf("");
        for (uint32_t h0 = group % split.across; h0 < heads; h0 += kAtOnce * split.across) {
            typename P::template Raw<T> raw_g[kAtOnce], raw_x[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const uint32_t h = h0 + u * split.across;
                if (h < heads) {
                    raw_g[u] = pairs.fetch(row_of<const T>(p, p.src, p.src_stride, b, t, h));
                    raw_x[u] = pairs.fetch(row_of<const T>(p, p.x, p.x_stride, b, t, h));
                }
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const uint32_t h = h0 + u * split.across;
                if (h >= heads) break;
                const int side = h >= p.heads[0];
                float ya[N], yb[N], a[N], bb[N];
                pairs.unpack(raw_g[u], ya, yb);
                pairs.unpack(raw_x[u], a, bb);
                for (int i = 0; i < N; ++i) {   // h = R^T g
                    const float va = ya[i] * c[i] + yb[i] * s[i];
                    const float vb = yb[i] * c[i] - ya[i] * s[i];
                    ya[i] = pairs.turns(i) ? va : ya[i];
                    yb[i] = pairs.turns(i) ? vb : yb[i];
                }
                if (!good)
                    for (int i = 0; i < N; ++i) ya[i] = yb[i] = __builtin_nanf("");
                if (p.norm[side]) {
                    float sum = 0.f, dot = 0.f;
                    for (int i = 0; i < N; ++i) {
                        sum += a[i] * a[i] + bb[i] * bb[i];
                        dot += ya[i] * (side ? wa[1][i] : wa[0][i]) * a[i] +
                               yb[i] * (side ? wb[1][i] : wb[0][i]) * bb[i];
                    }
                    const float rstd = rsqrtf(row_sum<Lanes>(sum) * inv_dim + p.eps);
                    const float mean = row_sum<Lanes>(dot) * rstd * inv_dim;   // mean(h w xh)
                    for (int i = 0; i < N; ++i) {
                        const float xa = a[i] * rstd, xb = bb[i] * rstd;
                        const float da = ya[i] * xa, db = yb[i] * xb;
                        ga[0][i] += side ? 0.f : da, gb[0][i] += side ? 0.f : db;
                        ga[1][i] += side ? da : 0.f, gb[1][i] += side ? db : 0.f;
                        ya[i] = rstd * (ya[i] * (side ? wa[1][i] : wa[0][i]) - xa * mean);
                        yb[i] = rstd * (yb[i] * (side ? wb[1][i] : wb[0][i]) - xb * mean);
                    }
                }
                pairs.store(row_of<T>(p, p.dst, p.dst_stride, b, t, h), ya, yb);
            }
        }
    }
    if (!p.partial) return;
    constexpr int kGroups = kThreads / Lanes;
    __shared__ float sums[kGroups][TAPS_MAX_HEAD_DIM > 8 * Lanes ? 8 * Lanes : TAPS_MAX_HEAD_DIM];
    static_assert(2 * N * Lanes <= (TAPS_MAX_HEAD_DIM > 8 * Lanes ? 8 * Lanes : TAPS_MAX_HEAD_DIM),
                  "a row of sums holds a lane's pairs");
    for (int side = 0; side < 2; ++side) {
        if (!p.norm[side]) continue;
        for (int i = 0; i < N; ++i) {   // lane-major: which element is which only its lane knows
            sums[group][i * Lanes + lane] = ga[side][i];
            sums[group][(N + i) * Lanes + lane] = gb[side][i];
        }
        __syncthreads();
        for (int k = threadIdx.x; k < 2 * N * Lanes; k += kThreads) {
            float v = 0.f;
            for (int g = 0; g < kGroups; ++g) v += sums[g][k];
            sums[0][k] = v;
        }
        __syncthreads();
        if (group == 0) {
            float a[N], b[N];
            for (int i = 0; i < N; ++i) {
                a[i] = sums[0][i * Lanes + lane];
                b[i] = sums[0][(N + i) * Lanes + lane];
            }
            pairs.store(p.partial + ((uint64_t)blockIdx.x * 2 + side) * p.dim, a, b);
        }
        __syncthreads();
    }
}

// The weights' gradients from the workgroups' partial sums: a workgroup per 16
// elements; 64 sums of every 64th row, then those in order.  (16 sums of a
// workgroup of 256 waited for 64 loads one after the other: 21 us for 1024 rows.)
constexpr int kGradThreads = 1024, kGradSums = kGradThreads / 16;

template <class T>
__global__ __launch_bounds__(kGradThreads) void k_weight_grads(const float *partial, uint32_t rows,
                                                               uint32_t dim, bool float_weights,
                                                               void *q_grad, void *k_grad) {
    __shared__ float sums[kGradSums][17];
    const int side = blockIdx.y;
    void *out = side ? k_grad : q_grad;
    if (!out) return;
    const uint32_t i = blockIdx.x * 16 + threadIdx.x % 16, r0 = threadIdx.x / 16;
    float v = 0.f;
    if (i < dim) {
#pragma unroll 8
        for (uint32_t r = r0; r < rows; r += kGradSums)
            v += partial[((uint64_t)r * 2 + side) * dim + i];
    }
    sums[r0][threadIdx.x % 16] = v;
    __syncthreads();
    if (r0 != 0 || i >= dim) return;
    v = 0.f;
#pragma unroll
    for (int r = 0; r < kGradSums; ++r) v += sums[r][threadIdx.x];
    if (float_weights)
        ((float *)out)[i] = v;
    else
        ((T *)out)[i] = from_f32<T>(v);
}

template <class F> void with_type(uint32_t dtype, F &&f) {
    if (dtype == TAPS_BF16)
        f((__bf16)0);
    else if (dtype == TAPS_F16)
        f((_Float16)0);
    else
        f(0.f);
}

template <int L> struct Lanes_ {
    static constexpr int value = L;
};

template <class F> void with_lanes(uint32_t dim, F &&f) {
    switch (Pairs<true>::lanes(dim)) {
    case 1: f(Lanes_<1>()); break;
    case 2: f(Lanes_<2>()); break;
    case 4: f(Lanes_<4>()); break;
    case 8: f(Lanes_<8>()); break;
    case 16: f(Lanes_<16>()); break;
    default: f(Lanes_<32>()); break;
    }
}

uint32_t token_groups(uint64_t tokens, uint32_t heads, int lanes) {
    const Split split(heads, lanes);
    return (uint32_t)((tokens + split.tokens - 1) / split.tokens);
}

int lanes_of(uint32_t dim, bool vectors) {
    return vectors ? Pairs<true>::lanes(dim) : Pairs<false>::lanes(dim);
}

}  // namespace

hipError_t taps_launch_norm_rotate(const taps_rows_launch &p, uint32_t dtype, bool vectors,
                                   hipStream_t stream) {
    const uint32_t groups = token_groups((uint64_t)p.batch * p.tokens, p.heads[0] + p.heads[1],
                                         lanes_of(p.dim, vectors));
    with_type(dtype, [&](auto zero) {
        using T = decltype(zero);
        if (!vectors)
            k_norm_rotate<T, false, 64><<<grid_of(groups), kThreads, 0, stream>>>(p);
        else
            with_lanes(p.dim, [&](auto n) {
                k_norm_rotate<T, true, decltype(n)::value><<<grid_of(groups), kThreads, 0, stream>>>(p);
            });
    });
    return hipGetLastError();
}

hipError_t taps_launch_append(const taps_rows_launch &p, uint32_t dtype, bool vectors,
                              hipStream_t stream) {
    const uint32_t groups = token_groups(p.tokens, 2 * p.heads[0], lanes_of(p.dim, vectors));
    with_type(dtype, [&](auto zero) {
        using T = decltype(zero);
        if (!vectors)
            k_append<T, false, 64><<<grid_of(groups), kThreads, 0, stream>>>(p);
        else
            with_lanes(p.dim, [&](auto n) {
                k_append<T, true, decltype(n)::value><<<grid_of(groups), kThreads, 0, stream>>>(p);
            });
    });
    return hipGetLastError();
}

uint32_t taps_backward_groups(const taps_rows_launch &p, bool vectors) {
    const uint32_t groups = token_groups((uint64_t)p.batch * p.tokens, p.heads[0] + p.heads[1],
                                         lanes_of(p.dim, vectors));
    return groups < 1 ? 1 : groups < kMostBackwardGroups ? groups : kMostBackwardGroups;
}

hipError_t taps_launch_norm_rotate_backward(const taps_rows_launch &p, uint32_t dtype, bool vectors,
                                            void *q_weight_grad, void *k_weight_grad,
                                            hipStream_t stream) {
    const uint32_t groups = taps_backward_groups(p, vectors);
    with_type(dtype, [&](auto zero) {
        using T = decltype(zero);
        if (!vectors)
            k_norm_rotate_backward<T, false, 64><<<groups, kThreads, 0, stream>>>(p);
        else
            with_lanes(p.dim, [&](auto n) {
                k_norm_rotate_backward<T, true, decltype(n)::value>
                    <<<groups, kThreads, 0, stream>>>(p);
            });
        if (p.partial)
            k_weight_grads<T><<<dim3((p.dim + 15) / 16, 2), kGradThreads, 0, stream>>>(
                p.partial, groups, p.dim, p.float_weights, q_weight_grad, k_weight_grad);
    });
    return hipGetLastError();
}
