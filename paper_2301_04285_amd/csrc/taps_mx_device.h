// taps_mx_device.h -- the codes of the microscaling formats on the GPU: the conversions
// of gfx950 take two elements an instruction, with the block's power of two.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace {

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Eight elements' codes are this many 32-bit words.
template <int Bits> constexpr int kWords = Bits / 4;

// The scale byte as the 32-bit number whose exponent the conversions take: 2^(byte - 127), and
// NaN results for 255.
__device__ __forceinline__ float mx_scale(uint32_t byte) {
    return __builtin_bit_cast(float, byte << 23);
}

// Two elements of a word (Pair: which two) in the type T; exact but where T's range ends.
template <class T, int Bits, int Pair>
__device__ __forceinline__ uint32_t mx_pair(uint32_t word, float scale) {
    if constexpr (__is_same(T, __bf16)) {
        if constexpr (Bits == 4)
            return __builtin_bit_cast(uint32_t,
                                      __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale, Pair));
        else
            return __builtin_bit_cast(
                uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(word, scale, (bool)Pair));
    } else {
        if constexpr (Bits == 4)
            return __builtin_bit_cast(uint32_t,
                                      __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale, Pair));
        else
            return __builtin_bit_cast(
                uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(word, scale, (bool)Pair));
    }
}

// Eight elements in a 16-bit type.
template <class T, int Bits>
__device__ __forceinline__ u32x4 mx_eight(const uint32_t *words, float scale) {
    if constexpr (Bits == 4)
        return u32x4{mx_pair<T, 4, 0>(words[0], scale), mx_pair<T, 4, 1>(words[0], scale),
                     mx_pair<T, 4, 2>(words[0], scale), mx_pair<T, 4, 3>(words[0], scale)};
    else
        return u32x4{mx_pair<T, 8, 0>(words[0], scale), mx_pair<T, 8, 1>(words[0], scale),
                     mx_pair<T, 8, 0>(words[1], scale), mx_pair<T, 8, 1>(words[1], scale)};
}

}  // namespace
