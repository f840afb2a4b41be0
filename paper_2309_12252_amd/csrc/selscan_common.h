// Shared by the kernels of the selective scan: shapes, parameters, how a workgroup finds its rows and channels, what is made of the inputs.
#pragma once
#include <type_traits>

#include "layer_common.h"

namespace deer {

// Four states of a channel lie in one lane, the Q lanes of a channel 64 / Q apart: a wavefront has 64 / Q channels, a workgroup of four 256 / Q, and the rows go
// through LDS kRows at a time.  What a state's row costs is instructions, not bytes: product, exponential (two slots), product, sum, and the sum of an output, six of a
// lane's slots, and some four of the row's preparation and of sums over lanes; at 16 states the bytes take a third of that time.  One state a lane more than doubles the sums over
// lanes; a channel with all 16 states a lane, B and C through scalar registers and nothing through LDS, left so few wavefronts that it was slower (outputs of 16,384 rows of
// 4,096 channels 412 us against 304, gradient 1,890 against 1,132 with its 248 accumulation registers).
// Lanes of a channel, as many as its states take.  16,384 rows of 4,096 channels with a gate, us of states behind segments + outputs, and of kept states with fronts + gradient:
//   4 states, bf16: one lane 94 + 136 and 171 + 914, two 133 + 203 and 229 + 737; fp32: one 143 + 277 and 317 + 1,020, two 138 + 210 and 308 + 902 (one lane a channel, the gradient spills)
//   8 states, bf16: two lanes 119 + 180 and 205 + 652, four 184 + 267 and 305 + 1,003; fp32: two 139 + 207 and 314 + 913, four 189 + 285 and 370 + 1,017
template <int Q> struct ScanShape {
    static constexpr int kWave = 64 / Q, kChannels = 256 / Q;
    static constexpr int kRows = Q == 1 ? 8 : Q == 2 ? 16 : Q <= 8 ? 32 : 64;
    static constexpr int kItems = kRows * kChannels >= 1024 ? kRows * kChannels / 1024 : 1;   // of four channels of a row, a lane
    static constexpr int kQuads = kRows * Q >= 256 ? kRows * Q / 256 : 1;                    // of four states of B, and of C, of a row, a lane
};
constexpr int kMarkRows = 16;   // rows from one kept state to the next in the gradient, and of its tiles
constexpr int kSumRows = 1024;  // at most so many rows are summed in 32 bits for dA, dskip and dbias, their sums in 64: equal values over 65,536 rows would be off by 6e-4, over these by 1e-5

inline int scan_lanes(int S) { return S <= 4 ? 1 : S <= 8 ? 2 : S <= 16 ? 4 : S <= 32 ? 8 : 16; }

struct SelscanParams {
    SeqRows rows;
    int D, S, G, softplus;
    int per_group, blocks;            // channels of a group; workgroups along the channels of a group
    bool vec;                         // rows of channels and of states can be read four at a time
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
    float *part_bc, *part_A, *part_d; // sums for dB and dC by workgroups; of every kSumRows rows of a segment for dA [part][D][S], and for dskip and dbias [part][2][D]
    int parts_each;                   // of a segment
    bool zero_rest;
};

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
        Bounds bounds(s);
        n = bounds.up_to(row) - 1;
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

// The scan takes the hardware's 2^x and 1 / x (1 ulp) for fp32 too: an exponential is most of a state's row, and an argument v times log2 e rounds to |v| 2^-24, no more than the product dt A that
// it comes from; gates and slopes keep to it.  (|v| + 6) 2^-24 of a sigmoid, where the functions leave 6.
constexpr float kLog2e = 1.44269504088896341f;

// log(1 + exp(v)) = max(v, 0) + 2 atanh(e / (2 + e)), e = exp(-|v|): s = e / (2 + e) is at most 1/3, and 2 atanh(s) / s as a polynomial in s^2, fitted at the Chebyshev
// points of [0, 1/9], is off by 4e-9; so small values keep their digits, which a logarithm of 1 + e would lose.
__device__ __forceinline__ float softplus(float v) {
    const float e = __builtin_amdgcn_exp2f(-kLog2e * __builtin_fabsf(v));
    const float s = e * __builtin_amdgcn_rcpf(2.0f + e), w = s * s;
    float f = 0.28157779574394226f;
    f = f * w + 0.27965158224105835f;
    f = f * w + 0.4002459645271301f;
    f = f * w + 0.6666632294654846f;
    f = f * w + 2.0f;
    return (v > 0.0f ? v : 0.0f) + s * f;   // (NaN: e is)
}
// its derivative, 1 / (1 + exp(-v))
__device__ __forceinline__ float softplus_slope(float v) {
    const float e = __builtin_amdgcn_exp2f(-kLog2e * __builtin_fabsf(v)), r = __builtin_amdgcn_rcpf(1.0f + e);
    return v >= 0.0f ? r : e * r;
}
__device__ __forceinline__ float fast_silu(float v) { return v * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * v)); }

// v 2^e in two halves, for factors of many rows that 32 bits need not hold by themselves: zero stays zero, and what fits is kept
__device__ __forceinline__ float scaled(float v, float e) {
    const float half = __builtin_amdgcn_exp2f(0.5f * __builtin_fminf(e, 254.0f));
    return half * v * half;
}

// Four elements that lie side by side, of a row of a tile, by buffer instructions: asked for in one piece (VEC) or one by one, as they came; those behind `count`, and all of a
// lane without a row (at kNoColumn), are zero, or not written.  No lane takes another path than the others, so nothing waits for what is on its way.
constexpr long long kScanStride = 1 << 22;   // elements between rows, at most: the 64 of a tile stay below kNoColumn
struct Tile {
    __amdgpu_buffer_rsrc_t rsrc;
    template <typename T>
    __device__ __forceinline__ Tile(const T* first) : rsrc(__builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(first), 0, (int)kNoColumn, 0x00020000)) {}
};
template <typename T, bool VEC>
struct Four {
    using U2 = unsigned __attribute__((ext_vector_type(2)));
    using U4 = unsigned __attribute__((ext_vector_type(4)));
    using Raw = std::conditional_t<sizeof(T) == 4, U4, U2>;
    std::conditional_t<VEC, Raw, T[4]> v;
    __device__ __forceinline__ void load(const Tile& t, unsigned at, int count) {
        if constexpr (VEC) {
            if constexpr (sizeof(T) == 4) v = __builtin_amdgcn_raw_buffer_load_b128(t.rsrc, at, 0, 0);
            else v = __builtin_amdgcn_raw_buffer_load_b64(t.rsrc, at, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned one = i < count ? at + i * (unsigned)sizeof(T) : kNoColumn;
                if constexpr (sizeof(T) == 4) v[i] = __builtin_bit_cast(T, __builtin_amdgcn_raw_buffer_load_b32(t.rsrc, one, 0, 0));
                else v[i] = __builtin_bit_cast(T, (unsigned short)__builtin_amdgcn_raw_buffer_load_b16(t.rsrc, one, 0, 0));
            }
        }
    }
    __device__ __forceinline__ float operator[](int i) const {
        if constexpr (VEC) return (float)__builtin_bit_cast(vec_t<T, 4>, v)[i];
        else return (float)v[i];
    }
    __device__ static __forceinline__ void store(const Tile& t, unsigned at, int count, const float* from) {
        if constexpr (VEC) {
            vec_t<T, 4> w;
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = (T)from[i];
            if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(U4, w), t.rsrc, at, 0, 0);
            else __builtin_amdgcn_raw_buffer_store_b64(__builtin_bit_cast(U2, w), t.rsrc, at, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned one = i < count ? at + i * (unsigned)sizeof(T) : kNoColumn;
                if constexpr (sizeof(T) == 4) __builtin_amdgcn_raw_buffer_store_b32(__builtin_bit_cast(unsigned, from[i]), t.rsrc, one, 0, 0);
                else __builtin_amdgcn_raw_buffer_store_b16(__builtin_bit_cast(unsigned short, (T)from[i]), t.rsrc, one, 0, 0);
            }
        }
    }
};
// A lane's places in a tile: four channels, from c4 on, of rows `step` apart
template <int N>
struct Places {
    unsigned at[N];
    template <typename T>
    __device__ __forceinline__ void set(long long stride, int row0, int step, int c4, T) {
#pragma unroll
        for (int j = 0; j < N; ++j) at[j] = (unsigned)((row0 + j * step) * stride + c4) * (unsigned)sizeof(T);
    }
};

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
// Between wavefronts of a workgroup, about LDS alone: what has been asked for from memory stays on its way, which __syncthreads() would wait for
__device__ __forceinline__ void lds_barrier() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
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
