// taps_lanes.h -- sums over the lanes of a wavefront.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace {

// Sum over groups of 1, 2, 4 .. 64 neighbouring lanes; every lane of a group gets
// it.  Lanes meet by data-parallel moves: their neighbour, the other pair of four,
// the other four of eight and eight of sixteen (mirrored: those hold one value by
// then), the other 16 and the other 32.
template <int Control> __device__ __forceinline__ float moved(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), Control,
                                                              0xf, 0xf, true));
}
__device__ __forceinline__ float swapped_sum(float v, bool sixteen) {
    const uint32_t u = __builtin_bit_cast(uint32_t, v);
    uint32_t a, b;
    if (sixteen) {
        const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
        a = r[0], b = r[1];
    } else {
        const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
        a = r[0], b = r[1];
    }
    return __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b);
}
template <int Lanes> __device__ __forceinline__ float row_sum(float v) {
    if (Lanes > 1) v += moved<0xb1>(v);    // lanes 1 0 3 2
    if (Lanes > 2) v += moved<0x4e>(v);    // lanes 2 3 0 1
    if (Lanes > 4) v += moved<0x141>(v);   // eight lanes mirrored
    if (Lanes > 8) v += moved<0x140>(v);   // sixteen lanes mirrored
    if (Lanes > 16) v = swapped_sum(v, true);
    if (Lanes > 32) v = swapped_sum(v, false);
    return v;
}

}  // namespace
