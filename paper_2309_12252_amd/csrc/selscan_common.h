// Shared by the kernels of the selective scan: shapes, parameters, how a workgroup finds its rows and channels, what is made of the inputs.
#pragma once
#include "layer_common.h"

namespace deer {

// Four states of a channel lie in one lane, the Q lanes of a channel 64 / Q apart: a wavefront has 64 / Q channels, a workgroup of four 256 / Q, and the rows go
// through LDS kRows at a time.
template <int Q> struct ScanShape {
    static constexpr int kWave = 64 / Q, kChannels = 256 / Q;
    static constexpr int kRows = Q == 1 ? 8 : Q == 2 ? 16 : Q <= 8 ? 32 : 64;
    static constexpr int kItems = kRows * kChannels >= 1024 ? kRows * kChannels / 1024 : 1;   // of four channels of a row, a lane
    static constexpr int kQuads = kRows * Q >= 128 ? kRows * Q / 128 : 1;                     // of four states of B or C of a row, a lane
};
constexpr int kMarkRows = 16;   // rows from one kept state to the next in the gradient, and of its tiles

inline int scan_lanes(int S) { return S <= 4 ? 1 : S <= 8 ? 2 : S <= 16 ? 4 : S <= 32 ? 8 : 16; }

struct SelscanParams {
    SeqRows rows;
    int D, S, G, softplus;
    int per_group, blocks;            // channels of a group; workgroups along the channels of a group
    bool vec, vec_bc;                 // rows of channels (of states) can be read four at a time
    long long stride_x, stride_dt, stride_B, stride_C, stride_z, stride_y;
    const void *x, *dt, *B, *C, *z;
    const float *A, *skip, *bias, *h0;
    void* y;
    float* last;
    // segments of seg_rows rows: of every sequence where they are padded, of all rows where they are packed
    int segs;
    long long seg_rows;
    float *local, *carry, *steps;     // state behind a segment from zero [D][4 Q] (or from a sequence that begins in it), true state in front, sum of dt [D]
    int* resets;                      // whether a sequence begins in the segment (at its first row or later)
    // gradient
    const void* dy;
    const float* dlast;
    void *dx, *ddt, *dB, *dC, *dz;
    float *dA, *dskip, *dbias, *dh0;
    int marks_each;                   // tiles of a segment
    float *marks, *mark_steps;        // states in front of every kMarkRows rows [D][4 Q], sums of dt since the segment's first row [D]
    float *rlocal, *rcarry, *rsteps;  // the same backwards
    int* rresets;
    float *part_bc, *part_A, *part_d; // sums for dB and dC by workgroups, for dA [segment][D][S], for dskip and dbias [segment][2][D]
    bool zero_rest;
};

template <typename T>
__device__ __forceinline__ float as_float(T v) { return (float)v; }

struct ScanPlace {
    long long lo, hi;      // rows, absolute
    long long seg;         // number of the segment
    int i, n;              // number in its sequence; padded: sequence
    int g, block, ch0, channels;
};
template <int Q>
__device__ __forceinline__ ScanPlace scan_place(const SelscanParams& p) {
    ScanPlace s;
    const int across = p.G * p.blocks, cb = blockIdx.x % across;
    s.seg = blockIdx.x / across;
    s.i = (int)(s.seg % p.segs);
    s.n = p.rows.packed ? 0 : (int)(s.seg / p.segs);
    s.g = cb / p.blocks;
    s.block = cb % p.blocks;
    const int in = s.block * ScanShape<Q>::kChannels;
    s.ch0 = s.g * p.per_group + in;
    s.channels = p.per_group - in < ScanShape<Q>::kChannels ? p.per_group - in : ScanShape<Q>::kChannels;
    const long long base = (long long)s.n * p.rows.T;
    long long first = base, behind = base + p.rows.T;
    if (p.rows.packed) {
        first = clamp_row(p.rows.bounds[0], p.rows.T);
        behind = clamp_row(p.rows.bounds[p.rows.N], p.rows.T);
    } else {
        behind = base + seq_length(p.rows, s.n);
    }
    s.lo = base + s.i * p.seg_rows;
    s.hi = s.lo + p.seg_rows;
    if (s.lo < first) s.lo = first;
    if (s.hi > behind) s.hi = behind;
    return s;
}

// The sequence that a row belongs to
struct ScanSeq {
    int n;
    long long start, end;
    __device__ __forceinline__ void load(const SeqRows& s) {
        start = clamp_row(s.bounds[n], s.T);
        end = clamp_row(s.bounds[n + 1], s.T);
    }
    __device__ __forceinline__ void at(const SeqRows& s, const ScanPlace& place, long long row) {
        if (!s.packed) {
            n = place.n;
            start = (long long)n * s.T;
            end = start + seq_length(s, n);
            return;
        }
        n = bounds_up_to(s, row) - 1;
        n = n < 0 ? 0 : n >= s.N ? s.N - 1 : n;
        load(s);
        if (start > row) start = row;   // (bounds that decrease: no meaning, but an end)
        if (end <= row) end = row + 1;
    }
    // on to the sequence that row = end belongs to
    __device__ __forceinline__ void next(const SeqRows& s, long long row) {
        while (s.packed && n + 1 < s.N) {
            ++n;
            load(s);
            if (end > row) break;
        }
        start = row;
        if (end <= row) end = row + 1;
    }
    // back to the sequence of a row in front of start
    __device__ __forceinline__ void back(const SeqRows& s, long long row) {
        while (s.packed && n > 0) {
            --n;
            load(s);
            if (start <= row) break;
        }
        if (start > row) start = row;
        if (end <= row) end = row + 1;
    }
};

// log(1 + exp(v)) = max(v, 0) + 2 atanh(e / (2 + e)), e = exp(-|v|): s = e / (2 + e) is at most 1/3, and 2 atanh(s) / s as a polynomial in s^2, fitted at the Chebyshev
// points of [0, 1/9], is off by 4e-9; so small values keep their digits, which a logarithm of 1 + e would lose.
__device__ __forceinline__ float softplus(float v) {
    const float e = __builtin_amdgcn_exp2f(-1.44269504088896341f * __builtin_fabsf(v));
    const float s = e * __builtin_amdgcn_rcpf(2.0f + e), w = s * s;
    float f = 0.28157779574394226f;
    f = f * w + 0.27965158224105835f;
    f = f * w + 0.4002459645271301f;
    f = f * w + 0.6666632294654846f;
    f = f * w + 2.0f;
    return __builtin_fmaxf(v, 0.0f) + (v != v ? v : s * f);
}
// its derivative, 1 / (1 + exp(-v))
__device__ __forceinline__ float softplus_slope(float v) {
    const float e = __builtin_amdgcn_exp2f(-1.44269504088896341f * __builtin_fabsf(v)), r = __builtin_amdgcn_rcpf(1.0f + e);
    return v >= 0.0f ? r : e * r;
}
__device__ __forceinline__ float fast_silu(float v) { return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896341f * v)); }

// four channels of a row; those behind `count` are zero
template <typename T>
__device__ __forceinline__ void load4(float* to, const void* from, long long at, int count, bool vec) {
    const T* f = reinterpret_cast<const T*>(from) + at;
    if (vec && count >= 4) {
        const vec_t<T, 4> v = *reinterpret_cast<const vec_t<T, 4>*>(f);
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i] = as_float(v[i]);
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) to[i] = i < count ? as_float(f[i]) : 0.0f;
}
template <typename T>
__device__ __forceinline__ void store4(void* to, long long at, const float* from, int count, bool vec) {
    T* t = reinterpret_cast<T*>(to) + at;
    if (vec && count >= 4) {
        vec_t<T, 4> v;
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = (T)from[i];
        *reinterpret_cast<vec_t<T, 4>*>(t) = v;
        return;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < count) t[i] = (T)from[i];
}

// a lane's four states of its channel, in arrays [.. D][S] and, padded, [.. D][4 Q]
struct ScanLane {
    int ch, k0;
    bool on;      // the channel is one
};
__device__ __forceinline__ void load_states(float* h, const float* from, long long row, const ScanLane& l, int D, int S) {
    const float* f = from ? from + (row * D + l.ch) * S + l.k0 : nullptr;
#pragma unroll
    for (int k = 0; k < 4; ++k) h[k] = f && l.on && l.k0 + k < S ? f[k] : 0.0f;
}
__device__ __forceinline__ void store_states(float* to, long long row, const ScanLane& l, int D, int S, const float* h) {
    if (!to || !l.on) return;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (l.k0 + k < S) to[(row * D + l.ch) * S + l.k0 + k] = h[k];
}
using Float4 = float __attribute__((ext_vector_type(4)));
using Float2 = float __attribute__((ext_vector_type(2)));

hipError_t launch_selscan(int dtype, const SelscanParams& p, hipStream_t stream);
hipError_t launch_selscan_marks(int dtype, const SelscanParams& p, hipStream_t stream);
hipError_t launch_selscan_grad(int dtype, const SelscanParams& p, hipStream_t stream);
struct SelstepParams {
    StepRows rows;
    int D, S, G, softplus;
    long long stride_x, stride_dt, stride_B, stride_C, stride_z, stride_y;
    const void *x, *dt, *B, *C, *z;
    const float *A, *skip, *bias;
    float* state;
    void* y;
};
hipError_t launch_selscan_step(int dtype, const SelstepParams& p, hipStream_t stream);

}  // namespace deer
