// Building blocks of the matrix-state recurrence (matrec.hip, matrec_grad.hip): tiles of 64 rows in LDS, operands of the matrix
// instructions, decays of a chunk.
//
// A chunk has 64 rows.  Matrix products are 16 x 16 x 32 tiles; the order of the 32 terms of a contraction is the same for both
// operands and otherwise free.  Everywhere it is
//     element e of lane group g (lanes 16 g .. 16 g + 15) is term 4 g + e for e < 4, 16 + 4 g + e - 4 for e >= 4,
// which is how the accumulators of two neighbouring 16 x 16 tiles hold their rows: a state kept in accumulators is an operand of
// the next product without leaving its registers.  Tiles in LDS keep every 32 columns in that order too, so that a lane's eight
// terms of a row are 16 contiguous bytes (bf16).
#pragma once
#include "seq_common.h"

namespace deer {
namespace {

using F32x4 = float __attribute__((ext_vector_type(4)));
using F32x8 = float __attribute__((ext_vector_type(8)));
using BF16x4 = BF16 __attribute__((ext_vector_type(4)));
using BF16x8 = BF16 __attribute__((ext_vector_type(8)));
using I16x4 = short __attribute__((ext_vector_type(4)));
using I16x8 = short __attribute__((ext_vector_type(8)));

constexpr int kChunk = 64;
constexpr int kWaves = 4;

template <typename T> struct Op;
template <> struct Op<BF16> {
    using Frag = BF16x8;
    static constexpr int PAD = 8;       // elements behind a row of a tile: rows 16 bytes apart in the banks
    static constexpr int PIECES = 2;    // an fp32 number as the sum of two bf16 ones: 2^-17 off at most (half a step of each part)
};
template <> struct Op<float> {
    using Frag = F32x8;
    static constexpr int PAD = 4;
    static constexpr int PIECES = 1;
};
template <typename T> using frag_t = typename Op<T>::Frag;

__device__ __forceinline__ F32x4 mma(BF16x8 a, BF16x8 b, F32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ F32x4 mma(F32x8 a, F32x8 b, F32x4 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

// fp32 values as an operand: rounded once (the first piece), and what that leaves (the second)
template <typename T>
__device__ __forceinline__ void pieces_of(F32x8 x, frag_t<T> (&p)[Op<T>::PIECES]) {
    if constexpr (Op<T>::PIECES == 1) {
        p[0] = x;
    } else {
        p[0] = __builtin_convertvector(x, BF16x8);
        p[1] = __builtin_convertvector(x - __builtin_convertvector(p[0], F32x8), BF16x8);
    }
}
template <typename T>
__device__ __forceinline__ frag_t<T> rounded(F32x8 x) {
    if constexpr (Op<T>::PIECES == 1) return x;
    else return __builtin_convertvector(x, BF16x8);
}
__device__ __forceinline__ F32x8 widened(BF16x8 x) { return __builtin_convertvector(x, F32x8); }
__device__ __forceinline__ F32x8 widened(F32x8 x) { return x; }
__device__ __forceinline__ F32x8 joined(F32x4 a, F32x4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// place of column c of a tile's row: columns 4 a .. 4 a + 3 of a block of 32 stay together
__device__ __forceinline__ int place(int c) {
    const int a = (c >> 2) & 7;
    return (c & ~31) + (a & 3) * 8 + (a >> 2) * 4 + (c & 3);
}

// rows `row` (this lane's), terms of the block of 32 columns s
template <typename T, int LD>
__device__ __forceinline__ frag_t<T> row_frag(const T* tile, int row, int s, int g) {
    return *reinterpret_cast<const frag_t<T>*>(tile + row * LD + 32 * s + 8 * g);
}

// column 16 t + lane % 16, terms of the block of 32 rows s: the transposed operand
template <int LD>
__device__ __forceinline__ BF16x8 col_frag(const BF16* tile, int s, int t, int lane) {
    typedef __attribute__((address_space(3))) I16x4* LdsPtr;
    // a group of 16 lanes hands in four rows of 16 columns, four columns a lane; lane l gets column l of them
    const int g = lane >> 4, l = lane & 15;
    const BF16* at = tile + (32 * s + 4 * g + (l >> 2)) * LD + place(16 * t + 4 * (l & 3));
    const I16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)at);
    const I16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(at + 16 * LD));
    return __builtin_bit_cast(BF16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}
template <int LD>
__device__ __forceinline__ F32x8 col_frag(const float* tile, int s, int t, int lane) {
    const int g = lane >> 4, c = place(16 * t + (lane & 15));
    F32x8 f;
#pragma unroll
    for (int e = 0; e < 8; ++e) f[e] = tile[(32 * s + 4 * g + (e & 3) + (e >= 4 ? 16 : 0)) * LD + c];
    return f;
}

// 64 rows of `cols` columns from memory into a tile of LD - PAD columns; what is not there is zero
template <typename T, int LD>
__device__ __forceinline__ void load_tile(T* tile, const T* from, long long stride, int rows, int cols) {
    using V4 = T __attribute__((ext_vector_type(4)));
    using V8 = T __attribute__((ext_vector_type(8)));
    constexpr int C = LD - Op<T>::PAD;
    const bool wide = cols % 8 == 0 && stride % 8 == 0 && reinterpret_cast<uintptr_t>(from) % 16 == 0;
    if (wide) {
        constexpr int PER = C / 8;
#pragma unroll
        for (int i = 0; i < kChunk * PER / (64 * kWaves); ++i) {
            const int at = i * 64 * kWaves + threadIdx.x, r = at / PER, c = at % PER * 8;
            V8 v = {};
            if (r < rows && c < cols) v = *reinterpret_cast<const V8*>(from + r * stride + c);
            *reinterpret_cast<V4*>(tile + r * LD + place(c)) = __builtin_shufflevector(v, v, 0, 1, 2, 3);
            *reinterpret_cast<V4*>(tile + r * LD + place(c + 4)) = __builtin_shufflevector(v, v, 4, 5, 6, 7);
        }
    } else {
        for (int at = threadIdx.x; at < kChunk * C; at += 64 * kWaves) {
            const int r = at / C, c = at % C;
            tile[r * LD + place(c)] = r < rows && c < cols ? from[r * stride + c] : T(0);
        }
    }
}

// Running sum of a chunk's log gates, inclusive, of which differences are taken: as the sum of two floats (a sum of 64
// gates of down to -1e4, 2^-46 of it off).  A gate below -1e4 stands for it: its factor is zero either way.
struct Cum {
    float hi, lo;
};
__device__ __forceinline__ Cum chunk_cum(const float* gate, long long stride, int rows, int lane) {
    float g = lane < rows ? gate[lane * stride] : 0.0f;
    g = g < -1e4f ? -1e4f : g;
    double c = g;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const double o = __shfl_up(c, d);
        c += lane >= d ? o : 0.0;
    }
    Cum r;
    r.hi = (float)c;
    r.lo = (float)(c - (double)r.hi);
    return r;
}
__device__ __forceinline__ float decay_between(float hi_i, float lo_i, float hi_j, float lo_j) { return expf((hi_i - hi_j) + (lo_i - lo_j)); }

__device__ __forceinline__ float lane_value(float v, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); }

}  // namespace

// ---- how the rows are cut: chunks of 64 rows from every sequence's first, segments of `per` chunks ----
struct MatSegment {
    long long row0;      // first row in the arrays
    long long rows;      // of this segment
    int seq, chunk0;     // sequence; number of its first chunk among all
    int index, count;    // place among the sequence's segments, and how many there are
};
struct MatPlan {
    int* count;          // segments
    MatSegment* segs;    // [max_segs]
    int* seq_seg;        // [N + 1]: a sequence's first segment
    int max_segs, per;
};

struct MatrecParams {
    SeqRows rows;
    MatPlan plan;
    int Hk, Hv, Dk, Dv;
    float scale;
    long long stride_q, stride_k, stride_v, stride_o;   // elements from a row to the next (gradients lie like their arrays)
    const void *q, *k, *v, *dout;
    const float *gate, *s0, *dlast;
    void *o, *dq, *dk, *dv;
    float *last, *dgate, *ds0;
    bool split;                      // several segments a sequence: their states are joined through memory
    float *seg_state, *seg_rstate;   // [max_segs][Hv][Dk][Dv]: sums, then states in front of (behind) each
    float *seg_decay;                // [max_segs][Hv]
    float *chunk_state, *chunk_rstate;   // [chunks][Hv][Dk][Dv], gradient only
};
struct MatstepParams {
    StepRows rows;
    int Hk, Hv, Dk, Dv;
    float scale;
    long long stride_q, stride_k, stride_v, stride_o;
    const void *q, *k, *v;
    const float* gate;
    float* state;
    void* o;
};

hipError_t launch_matrec_plan(const MatrecParams& p, hipStream_t stream);
hipError_t launch_matrec_out(int dtype, const MatrecParams& p, hipStream_t stream);
hipError_t launch_matrec_states(int dtype, const MatrecParams& p, hipStream_t stream);
hipError_t launch_matrec_grad(int dtype, const MatrecParams& p, hipStream_t stream);
hipError_t launch_matstep(int dtype, const MatstepParams& p, hipStream_t stream);

}  // namespace deer
