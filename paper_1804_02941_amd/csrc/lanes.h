// Sums and maxima over the lanes of a wavefront, and over the wavefronts of a workgroup (norm.hip, adapters.hip).  gfx950 only.
#pragma once

#include "dab_internal.h"

namespace dab {

template <int CONTROL>
__device__ __forceinline__ float dpp(float v) {
    return __uint_as_float(static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(__float_as_uint(v)), CONTROL, 0xf, 0xf, true)));
}

// The sum over groups of 2^LOG neighbouring lanes, in every lane of them, always added in the same order.
template <int LOG>
__device__ __forceinline__ float lanes_sum(float v) {
    if constexpr (LOG >= 1) v += dpp<0xB1>(v);               // lane ^ 1
    if constexpr (LOG >= 2) v += dpp<0x4E>(v);               // lane ^ 2
    if constexpr (LOG >= 3) v += dpp<0x141>(v);              // the other four of eight
    if constexpr (LOG >= 4) v += dpp<0x140>(v);              // the other eight of sixteen
    if constexpr (LOG >= 5) v += __shfl_xor(v, 16);
    if constexpr (LOG >= 6) v += __shfl_xor(v, 32);
    return v;
}

}  // namespace dab
