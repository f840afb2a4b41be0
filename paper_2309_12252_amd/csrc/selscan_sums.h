// Sums across the lanes of a wavefront for the selective scan: of a channel's lanes (64 / Q apart), and of the channels.
#pragma once
#include "lane_sums.h"

namespace deer {

// Four values over the Q lanes of a channel; what a lane gets: value of_lanes<Q>(lane, j) in v[j], j < lanes_keep<Q>
template <int Q> constexpr int lanes_keep = Q == 1 ? 4 : Q == 2 ? 2 : 1;
template <int Q>
__device__ __forceinline__ int of_lanes(int lane, int j) { return Q == 1 ? j : Q == 2 ? (lane >> 5) * 2 + j : (lane >> 5) * 2 + ((lane >> 4) & 1); }
template <int Q>
__device__ __forceinline__ void sum_lanes(float (&v)[4]) {
    if constexpr (Q == 1) return;
    v[0] = sum_halves(v[0], v[2]);
    v[1] = sum_halves(v[1], v[3]);
    if constexpr (Q == 2) return;
    v[0] = sum_rows(v[0], v[1]);
    if constexpr (Q >= 8) v[0] = dpp_add<kRor8>(v[0]);
    if constexpr (Q >= 16) v[0] = dpp_add<kRor4>(v[0]);
}

// lanes whose `bit` (8 or 4) is clear get the sum of a's two lanes, the others of b's: two instructions, the second for half of the banks of four lanes only.
// (a DPP operand must not have been written by the two instructions in front, which nobody looks after inside asm)
__device__ __forceinline__ void pair8(float& a, float b) {
    asm("s_nop 1\n\tv_add_f32_dpp %0, %0, %0 row_ror:8 row_mask:0xf bank_mask:0xf\n\tv_add_f32_dpp %0, %1, %1 row_ror:8 row_mask:0xf bank_mask:0xc" : "+&v"(a) : "v"(b));
}
__device__ __forceinline__ void pair4(float& a, float b) {
    asm("s_nop 1\n\tv_add_f32_dpp %0, %0, %0 row_half_mirror row_mask:0xf bank_mask:0xf\n\tv_add_f32_dpp %0, %1, %1 row_half_mirror row_mask:0xf bank_mask:0xa"
        : "+&v"(a)
        : "v"(b));
}

// Eight values over the 64 / Q channels of a wavefront: the upper bits of a channel's number choose among the values as they are summed, so that 16 instructions
// do for all of them.  What a lane gets: values channels_first<Q>(lane) + j in v[j], j < channels_keep<Q>.
template <int Q> constexpr int channels_keep = Q <= 2 ? 1 : Q == 4 ? 2 : Q == 8 ? 4 : 8;
template <int Q>
__device__ __forceinline__ int channels_first(int lane) {
    return Q == 1 ? lane >> 3 : Q == 2 ? (lane >> 2) & 7 : Q == 4 ? ((lane >> 2) & 3) * 2 : Q == 8 ? (lane & 4) : 0;
}
template <int Q> constexpr int channels_same = Q == 1 ? 7 : 3;   // bits of the lanes that get the same
template <int Q>
__device__ __forceinline__ void sum_channels(float (&v)[8]) {
    if constexpr (Q == 1) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = sum_halves(v[j], v[j + 4]);
        v[0] = sum_rows(v[0], v[2]);
        v[1] = sum_rows(v[1], v[3]);
        pair8(v[0], v[1]);
        v[0] = dpp_add<kHalfMirror>(v[0]);
    } else if constexpr (Q == 2) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[j] = sum_rows(v[j], v[j + 4]);
        pair8(v[0], v[2]);
        pair8(v[1], v[3]);
        pair4(v[0], v[1]);
    } else if constexpr (Q == 4) {
        // (waits: two instructions between a write and a DPP read of it)
        asm("s_nop 1\n\t"
            "v_add_f32_dpp %0, %0, %0 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %1, %1, %1 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %2, %2, %2 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %3, %3, %3 row_ror:8 row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %0, %4, %4 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
            "v_add_f32_dpp %1, %5, %5 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
            "v_add_f32_dpp %2, %6, %6 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
            "v_add_f32_dpp %3, %7, %7 row_ror:8 row_mask:0xf bank_mask:0xc\n\t"
            "v_add_f32_dpp %0, %0, %0 row_half_mirror row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %1, %1, %1 row_half_mirror row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %0, %2, %2 row_half_mirror row_mask:0xf bank_mask:0xa\n\t"
            "v_add_f32_dpp %1, %3, %3 row_half_mirror row_mask:0xf bank_mask:0xa\n\t"
            "s_nop 0\n\t"
            "v_add_f32_dpp %0, %0, %0 quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %1, %1, %1 quad_perm:[2,3,0,1] row_mask:0xf bank_mask:0xf\n\t"
            "s_nop 0\n\t"
            "v_add_f32_dpp %0, %0, %0 quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf\n\t"
            "v_add_f32_dpp %1, %1, %1 quad_perm:[1,0,3,2] row_mask:0xf bank_mask:0xf"
            : "+&v"(v[0]), "+&v"(v[1]), "+&v"(v[2]), "+&v"(v[3])
            : "v"(v[4]), "v"(v[5]), "v"(v[6]), "v"(v[7]));
        return;
    } else if constexpr (Q == 8) {
#pragma unroll
        for (int j = 0; j < 4; ++j) pair4(v[j], v[j + 4]);
    }
#pragma unroll
    for (int j = 0; j < channels_keep<Q>; ++j) v[j] = dpp_add<kSwapLanes>(dpp_add<kSwapPairs>(v[j]));
}

}  // namespace deer
