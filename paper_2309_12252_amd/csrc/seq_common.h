// Shared declarations of the sequence operators (gated linear recurrences, dropout): element types, the way rows belong to
// sequences, the counter-based generator, and the launch interface between seq_api.hip and the kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/deer.h"

namespace deer {

// How the rows of an array belong to sequences.  Packed: N sequences one behind the other in T rows, sequence s in rows
// bounds[s] .. bounds[s + 1] - 1.  Otherwise N sequences of T rows each, of which the first bounds[n] count (all without bounds).
// Bounds are device data that the host has not seen: whatever they hold is clamped to 0 .. T before it is used as a row.
struct SeqRows {
    const long long* bounds;
    long long T;
    int N;
    int packed;
};

__device__ __forceinline__ long long clamp_row(long long v, long long T) { return v < 0 ? 0 : v > T ? T : v; }

// how many of the packed sequences' N + 1 bounds are at most `row`
__device__ __forceinline__ int bounds_up_to(const SeqRows& s, long long row) {
    int lo = 0, hi = s.N + 1;
    while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        if (clamp_row(s.bounds[mid], s.T) <= row) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

__device__ __forceinline__ long long seq_length(const SeqRows& s, int n) {
    if (s.packed) {
        const long long a = clamp_row(s.bounds[n], s.T), b = clamp_row(s.bounds[n + 1], s.T);
        return b > a ? b - a : 0;
    }
    return s.bounds ? clamp_row(s.bounds[n], s.T) : s.T;
}

// Arrays whose rows that belong to no sequence are zeroed on request, by the call's first kernel over rows (16 rows of a sequence at a time, 256 lanes a
// workgroup).  Packed sequences lie one behind the other, so that these rows are those in front of the first and behind the last.
struct RestArray {
    void* first;
    long long pitch, width;   // bytes from a row to the next, and of a row: multiples of two
};
struct RestRows {
    int count;
    RestArray array[4];
};
template <typename U>
__device__ __forceinline__ void clear_row(char* row, long long width) {
    for (long long i = threadIdx.x; i < width / (long long)sizeof(U); i += 256) reinterpret_cast<U*>(row)[i] = U{};
}
__device__ __forceinline__ void clear_rest(const SeqRows& s, const RestRows& rest, long long block, long long blocks) {
    using U4 = unsigned __attribute__((ext_vector_type(4)));
    if (rest.count == 0 || !s.bounds) return;
    const long long tiles = (s.T + 15) / 16, all = tiles * (s.packed ? 1 : s.N);
    for (long long i = block; i < all; i += blocks) {
        const long long n = i / tiles, from = i % tiles * 16, to = from + 16 < s.T ? from + 16 : s.T;
        const long long lo = s.packed ? clamp_row(s.bounds[0], s.T) : 0, hi = s.packed ? clamp_row(s.bounds[s.N], s.T) : seq_length(s, (int)n);
        if (from >= lo && to <= hi) continue;
        for (long long r = from; r < to; ++r) {
            if (r >= lo && r < hi) continue;
            for (int a = 0; a < rest.count; ++a) {
                const long long pitch = rest.array[a].pitch, width = rest.array[a].width;
                char* row = reinterpret_cast<char*>(rest.array[a].first) + (n * s.T + r) * pitch;
                const unsigned long long low = reinterpret_cast<unsigned long long>(row) | (unsigned long long)width;
                if (low % 16 == 0) clear_row<U4>(row, width);
                else if (low % 4 == 0) clear_row<unsigned>(row, width);
                else clear_row<unsigned short>(row, width);
            }
        }
    }
}

// ---- element types: arithmetic in 32 bits for the 16-bit types and fp32, in 64 for fp64 ----
using BF16 = __bf16;
using F16 = _Float16;
template <typename T> struct Wide { using type = float; };
template <> struct Wide<double> { using type = double; };
template <typename T> using wide_t = typename Wide<T>::type;
template <typename T, int V> struct Vec { using type = T __attribute__((ext_vector_type(V))); };
template <typename T> struct Vec<T, 1> { using type = T; };
template <typename T, int V> using vec_t = typename Vec<T, V>::type;
template <typename T, int V>
__device__ __forceinline__ T vec_at(const vec_t<T, V>& v, int i) {
    if constexpr (V == 1) return v;
    else return v[i];
}
template <typename T, int V>
__device__ __forceinline__ void vec_set(vec_t<T, V>& v, int i, T x) {
    if constexpr (V == 1) v = x;
    else v[i] = x;
}

// Rows of an array by buffer instructions, by a lane's offset in bytes: one register where an address takes two, and a lane without a
// column is out of bounds (reads zero, writes nothing) at kNoColumn and beyond, up to 2^32: offsets are unsigned.  The caller has the rows in bounds.
constexpr unsigned kNoColumn = 0x7FFFFFF0;
constexpr long long kMostStride = 1 << 22;   // elements: 64 rows of 8 bytes each stay below kNoColumn, and it plus them below 2^32
struct RowsAt {
    __amdgpu_buffer_rsrc_t rsrc;
    unsigned pitch;
    template <typename T>
    __device__ __forceinline__ RowsAt(const T* first, long long stride)
        : rsrc(__builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(first), 0, (int)kNoColumn, 0x00020000)), pitch((unsigned)(stride * (long long)sizeof(T))) {}
    template <typename X>
    __device__ __forceinline__ X load(unsigned at) const {
        if constexpr (sizeof(X) == 8) return __builtin_bit_cast(X, __builtin_amdgcn_raw_buffer_load_b64(rsrc, at, 0, 0));
        else if constexpr (sizeof(X) == 4) return __builtin_bit_cast(X, __builtin_amdgcn_raw_buffer_load_b32(rsrc, at, 0, 0));
        else return __builtin_bit_cast(X, (unsigned short)__builtin_amdgcn_raw_buffer_load_b16(rsrc, at, 0, 0));
    }
    template <typename X>
    __device__ __forceinline__ void store(X x, unsigned at) const {
        using U2 = unsigned __attribute__((ext_vector_type(2)));
        if constexpr (sizeof(X) == 8) __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(U2, x), rsrc, at, 0, 0);
        else if constexpr (sizeof(X) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, x), rsrc, at, 0, 0);
        else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, x), rsrc, at, 0, 0);
    }
};

// ---- dropout: Philox4x32-10 (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011) ----
// One block of 128 bits serves eight rows of one channel, 16 bits a row: counter (channel, row / 8, sequence, draw), key = seed.
// Eight rows of a channel rather than eight channels of a row: a lane of the recurrence keeps one channel and runs over
// rows, so it uses a whole block whatever the vector width of its loads.
struct DropParams {
    unsigned seed_lo, seed_hi, draw;
    unsigned cut;        // an element is dropped where its 16 bits are below cut
    double scale;        // 2^16 / (2^16 - cut)
};

// bit i: row 8 * block + i is kept
__device__ __forceinline__ unsigned drop_keep8(const DropParams& d, unsigned channel, unsigned block, unsigned seq) {
    unsigned c0 = channel, c1 = block, c2 = seq, c3 = d.draw, k0 = d.seed_lo, k1 = d.seed_hi;
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const unsigned long long p = (unsigned long long)c0 * 0xD2511F53u, q = (unsigned long long)c2 * 0xCD9E8D57u;
        c0 = (unsigned)(q >> 32) ^ c1 ^ k0;
        c2 = (unsigned)(p >> 32) ^ c3 ^ k1;
        c1 = (unsigned)q;
        c3 = (unsigned)p;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    const unsigned w[4] = {c0, c1, c2, c3};
    unsigned keep = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        keep |= ((w[i] & 0xFFFFu) >= d.cut ? 1u : 0u) << (2 * i);
        keep |= ((w[i] >> 16) >= d.cut ? 1u : 0u) << (2 * i + 1);
    }
    return keep;
}

// ---- launches ----
void set_last_error(const char* text) noexcept;   // what deer_last_error(NULL) returns on this thread

struct DiagrecParams {
    SeqRows rows;
    int D, gate;
    long long stride_gate, stride_in, stride_out;   // elements from a row to the next
    const void *g, *x, *h0;
    void *h, *last;                                 // forward: outputs; gradient: h is an input
    const void *dh, *dlast;                         // gradient
    void *dg, *dx, *dh0;
    DropParams drop;
    bool zero_rest;                                 // rows of no sequence
    // words that tiles publish for each other
    int chunks, groups;                             // tiles and groups of tiles along a sequence
    unsigned long long *agg, *inc;
    unsigned* ticket;
    size_t words;                                   // 8-byte words from agg on, cleared before the launch
};
struct StepRows {
    const int* slots;      // [N] or nullptr (row n has slot n)
    int N, n_slots;
    bool zero_rest;        // rows that are passed over
};
struct DiagstepParams {
    StepRows rows;
    int D, gate;
    long long stride_gate, stride_in, stride_out;
    const void *g, *x;
    void *state, *h;
};
struct DropoutParams {
    int N, D;
    long long T, stride_in, stride_out;
    const void* x;
    void* y;
    DropParams drop;
};

constexpr int kDiagLanes = 512;   // of a workgroup of the recurrence
size_t diagrec_words(int dtype, int N, long long T, int D, bool grad, int* chunks, int* groups, size_t* agg_words);
hipError_t launch_diagrec(int dtype, bool grad, const DiagrecParams& p, hipStream_t stream);
hipError_t launch_diagstep(int dtype, const DiagstepParams& p, hipStream_t stream);
hipError_t launch_dropout(int dtype, const DropoutParams& p, hipStream_t stream);

}  // namespace deer
