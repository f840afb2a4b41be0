// Sums across lanes of a wavefront: swaps of halves and of rows of 16 lanes, and DPP inside a row.
#pragma once
#include <hip/hip_runtime.h>

namespace deer {

// sums over the halves: lanes 0 .. 31 get a's, lanes 32 .. 63 b's
__device__ __forceinline__ float sum_halves(float a, float b) {
    const auto s = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    return __builtin_bit_cast(float, (unsigned)s[0]) + __builtin_bit_cast(float, (unsigned)s[1]);
}
// sums over neighbouring rows of 16 lanes: even rows get a's, odd ones b's
__device__ __forceinline__ float sum_rows(float a, float b) {
    const auto s = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, a), __builtin_bit_cast(unsigned, b), false, false);
    return __builtin_bit_cast(float, (unsigned)s[0]) + __builtin_bit_cast(float, (unsigned)s[1]);
}
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
    return v + __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xf, 0xf, true));
}
constexpr int kRor8 = 0x128, kRor4 = 0x124, kMirror = 0x140, kHalfMirror = 0x141, kSwapPairs = 0x4E, kSwapLanes = 0xB1;   // DPP controls

}  // namespace deer
