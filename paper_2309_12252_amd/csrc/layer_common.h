// Shared declarations of the operators of layers with selective states (short convolution, selective scan, group norm): activations, the way a tile of
// rows falls into runs of one sequence each, sums over tiles, and the launch interface between layer_api.hip and the kernels.
#pragma once
#include "seq_common.h"

namespace deer {

// exp and 1 / v of the convolution and the norm: the functions for fp32 and fp64, the hardware's (1 ulp of 2^x and 1 / x) where the results are rounded to 16 bits
template <typename T>
__device__ __forceinline__ wide_t<T> exp_of(wide_t<T> v) {
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_exp2f(v * 1.44269504088896341f);
    else if constexpr (sizeof(T) == 4) return expf(v);
    else return exp(v);
}
template <typename T>
__device__ __forceinline__ wide_t<T> reciprocal(wide_t<T> v) {
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_rcpf(v);
    else return wide_t<T>(1) / v;
}
// v sigmoid(v), and its derivative g (1 + v (1 - g)), g = sigmoid(v)
template <typename T>
__device__ __forceinline__ wide_t<T> silu(wide_t<T> v) {
    using S = wide_t<T>;
    return v * reciprocal<T>(S(1) + exp_of<T>(-v));
}
template <typename T>
__device__ __forceinline__ void silu_both(wide_t<T> v, wide_t<T>& f, wide_t<T>& slope) {
    using S = wide_t<T>;
    const S g = reciprocal<T>(S(1) + exp_of<T>(-v));
    f = v * g;
    slope = g * (S(1) + v * (S(1) - g));
}

// The bounds of packed sequences as a whole wavefront looks at them, for rows that are the same for all its lanes: 64 of them in registers, one a lane, so that a search costs one
// trip to memory and not one for each of its steps.
struct Bounds {
    const SeqRows& s;
    long long v;   // bound base + lane
    int base;
    __device__ __forceinline__ explicit Bounds(const SeqRows& rows) : s(rows), base(0) { load(0); }
    __device__ __forceinline__ void load(int from) {
        base = from;
        const int i = from + (int)(threadIdx.x & 63);
        v = clamp_row(s.bounds[i < s.N ? i : s.N], s.T);
    }
    __device__ __forceinline__ long long at(int i) {   // 0 .. N
        if (i < base || i >= base + 64) load(i);
        const unsigned lo = __builtin_amdgcn_readlane((int)v, i - base), hi = __builtin_amdgcn_readlane((int)(v >> 32), i - base);
        return (long long)((unsigned long long)hi << 32 | lo);
    }
    __device__ __forceinline__ long long last() {
        return s.N < 64 ? at(s.N) : clamp_row(s.bounds[s.N], s.T);
    }
    // how many of the N + 1 bounds are at most `row`
    __device__ __forceinline__ int up_to(long long row) {
        int lo = 0, hi = s.N + 1;
        while (hi - lo > 64) {
            const int step = (hi - lo + 63) / 64, i = lo + (int)(threadIdx.x & 63) * step;
            const int many = __popcll(__ballot(i < hi && clamp_row(s.bounds[i < s.N ? i : s.N], s.T) <= row));
            if (many == 0) return lo;
            const int behind = lo + many * step;
            lo += (many - 1) * step + 1;
            hi = behind < hi ? behind : hi;
        }
        if (base != lo) load(lo);
        return lo + __popcll(__ballot(lo + (int)(threadIdx.x & 63) < hi && v <= row));
    }
};

// Rows lo .. hi - 1 (absolute; of sequence n where sequences are padded), the same for all lanes of a wavefront, as runs of one sequence each: f(sequence, its first row, the row
// behind its last, first and last + 1 row of the run).  Rows of no sequence are in none.
template <typename F>
__device__ __forceinline__ void for_runs(const SeqRows& s, int n, long long lo, long long hi, F f) {
    if (!s.packed) {
        const long long start = (long long)n * s.T, end = start + seq_length(s, n);
        if (lo < start) lo = start;
        if (hi > end) hi = end;
        if (lo < hi) f(n, start, end, lo, hi);
        return;
    }
    Bounds bounds(s);
    const long long first = bounds.at(0), last = bounds.last();
    if (lo < first) lo = first;
    if (hi > last) hi = last;
    if (lo >= hi) return;
    int at = bounds.up_to(lo) - 1;
    if (at < 0) at = 0;
    long long row = lo;
    while (row < hi && at < s.N) {
        const long long end = bounds.at(at + 1);
        if (end > row) {
            const long long start = bounds.at(at), to = end < hi ? end : hi;
            f(at, start < row ? start : row, end, row, to);
            row = to;
        }
        ++at;
    }
}

// first row of sequence n and how many it has
__device__ __forceinline__ long long seq_first(const SeqRows& s, int n) { return s.packed ? clamp_row(s.bounds[n], s.T) : (long long)n * s.T; }

// Sums over tiles, in the order of the tiles and in 64 bits: part [tiles][many + 1][each]; the first many rows of sums into first [each][many], the last into second (either may be
// NULL; without a last row: last false)
struct SumInto {
    void *first, *second;
    int each, many;
    bool last;
};
hipError_t launch_sum_tiles(bool wide, const void* part, long long tiles, const SumInto& into, hipStream_t stream);

// How a launch of 256 lanes goes over rows and channels: `lanes` (a power of two up to 64) side by side along the channels, V each, the others along the rows
struct Lanes {
    int lanes, phases, blocks;   // blocks of channels
};
inline Lanes lanes_for(int D, int V) {
    const int vecs = (D + V - 1) / V;
    int l = 1;
    while (l < vecs && l < 64) l *= 2;
    return Lanes{l, 256 / l, (vecs + l - 1) / l};
}
inline bool rows_fit(const void* p, long long stride, int V, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % (V * bytes) == 0 && stride % V == 0; }

constexpr int kConvRows = 32;        // rows of a lane of the short convolution
struct ConvParams {
    SeqRows rows;
    int D, W, act;
    long long stride_x, stride_y;
    const void *x, *w, *bias, *s0, *dy, *dlast;
    void *y, *last, *dx, *dw, *dbias, *ds0;
    void* part;                      // [tiles][W + 1][D]
    bool zero_rest;
};
struct ConvStepParams {
    StepRows rows;
    int D, W, act;
    long long stride_x, stride_y;
    const void *x, *w, *bias;
    void *state, *y;
};
long long conv_tiles(int D, long long T, int N, bool packed);   // at most, for the sums' workspace
hipError_t launch_shortconv(int dtype, bool grad, const ConvParams& p, hipStream_t stream);
hipError_t launch_shortconv_step(int dtype, const ConvStepParams& p, hipStream_t stream);

struct NormParams {
    SeqRows rows;
    int D, G, act, span;
    double eps;
    long long stride_x, stride_z, stride_y;
    const void *x, *w, *bias, *z, *dy;
    void *y, *stats, *dx, *dw, *dbias, *dz;
    void *part, *sums, *joined;      // workspace: per channel and tile of a sequence; for the weights' gradients; per group and sequence
    bool zero_rest;
};
struct NormLayout {
    long long tiles, part, sums, joined;   // workgroups of the largest launch; elements of the wide type
};
NormLayout norm_layout(int dtype, int D, int G, int span, long long T, int N, bool packed, bool grad);
hipError_t launch_groupnorm(int dtype, bool grad, const NormParams& p, hipStream_t stream);

}  // namespace deer
