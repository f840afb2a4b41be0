// What the C entry points of the sequence operators share: checks of the arguments, and how a refusal or a failed launch is told.
#pragma once
#include <cmath>
#include <cstdio>

#include "seq_common.h"

namespace deer {

constexpr size_t kAlign = 256;
inline size_t align_up(size_t v) { return (v + kAlign - 1) / kAlign * kAlign; }

inline deer_status fail(deer_status st, const char* text) {
    set_last_error(text);
    return st;
}
inline deer_status launched(const char* what, hipError_t e) {
    if (e == hipSuccess) return DEER_OK;
    char text[160];
    std::snprintf(text, sizeof(text), "%s: %s", what, hipGetErrorString(e));
    return fail(DEER_ERR_HIP, text);
}

template <typename C> bool is_packed(const C* c) { return (c->packed & 1) != 0; }
template <typename C> bool zero_rest(const C* c) { return (c->packed & (int)DEER_REST_ZERO) != 0; }
inline bool known_type(int dtype) { return dtype == DEER_F32 || dtype == DEER_F64 || dtype == DEER_BF16 || dtype == DEER_F16; }
inline size_t type_bytes(int dtype) { return dtype == DEER_F64 ? 8 : dtype == DEER_F32 ? 4 : 2; }
inline bool misaligned(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes != 0; }

// The mask's counter has 32 bits for blocks of eight rows and for channels; rows and columns are kept where products of them with
// element sizes stay far from 63 bits.
constexpr int64_t kMostRows = (int64_t)1 << 33;
constexpr long double kMostLanes = 4294967295.0L;   // of a launch: its size in work items is a number of 32 bits

inline deer_status check_workspace(const void* ws, size_t have, size_t need) {
    if (need == 0) return DEER_OK;
    if (!ws || misaligned(ws, kAlign) || have < need) {
        char text[160];
        std::snprintf(text, sizeof(text), "workspace NULL, misaligned or smaller than the %zu bytes needed", need);
        return fail(DEER_ERR_WORKSPACE, text);
    }
    return DEER_OK;
}

}  // namespace deer
