// Building blocks of the matrix-state recurrence (matrec.hip, matrec_grad.hip): tiles of 64 rows in LDS, operands of the matrix
// instructions, decays of a chunk.
//
// A chunk has 64 rows.  Matrix products are 16 x 16 x 32 tiles: operand A has rows lane % 16, operand B columns lane % 16, and lane group g (lanes 16 g ..
// 16 g + 15) of both has the terms 8 g .. 8 g + 7 of the 32; a result has rows 4 g .. 4 g + 3 of column lane % 16.  A state kept as results is to be
// an operand of the next product without leaving its registers: so the columns of an array are dealt out to tiles of 16 in such an order, column_of(), that
// the results of two neighbouring tiles hold, in lane group g, the columns 8 g .. 8 g + 7 of their 32.
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
constexpr int kRowFloats = 4 * 64 + 4;   // c_i as two floats, scale e^{c_i}, e^{c_64 - c_i}; e^{c_64} and c_64 as two floats

template <typename T> struct Op;
template <> struct Op<BF16> {
    using Frag = BF16x8;
    static constexpr int PIECES = 3;    // an fp32 number as the sum of three bf16 ones: exact to 2^-24 (two: 2.7e-6 measured on states)
};
template <> struct Op<float> {
    using Frag = F32x8;
    static constexpr int PIECES = 1;
};
template <typename T> using frag_t = typename Op<T>::Frag;

__device__ __forceinline__ F32x4 mma(BF16x8 a, BF16x8 b, F32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ F32x4 mma(F32x8 a, F32x8 b, F32x4 c) {
#pragma unroll
    for (int e = 0; e < 8; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
    return c;
}

// fp32 values as an operand: rounded, what that leaves rounded, and so on
template <typename T, int N>
__device__ __forceinline__ void pieces_of(F32x8 x, frag_t<T> (&p)[N]) {
    if constexpr (Op<T>::PIECES == 1) {
        p[0] = x;
    } else {
#pragma unroll
        for (int q = 0; q < N; ++q) {
            p[q] = __builtin_convertvector(x, BF16x8);
            if (q + 1 < N) x -= __builtin_convertvector(p[q], F32x8);
        }
    }
}
__device__ __forceinline__ F32x8 widened(BF16x8 x) { return __builtin_convertvector(x, F32x8); }
__device__ __forceinline__ F32x8 widened(F32x8 x) { return x; }
__device__ __forceinline__ F32x8 joined(F32x4 a, F32x4 b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// column (or row, of a state) that place i of tile n has
__device__ __forceinline__ int column_of(int n, int i) { return 32 * (n >> 1) + 8 * (i >> 2) + 4 * (n & 1) + (i & 3); }

// A tile of 64 rows and C (64 or 128) columns in LDS, in units of eight columns.  bf16: the units' places in a row are turned by the row so that neither
// 16 rows of one unit (row_frag) nor four half units of four rows (col_frag) meet in a bank.  fp32: rows 16 bytes apart in the banks.
template <typename T, int C> struct Tile {
    static_assert(C == 64 || C == 128, "units of a row fill a half or a whole turn of the banks");
    static constexpr int LD = sizeof(T) == 2 ? C : C + 4;
    static constexpr size_t bytes = sizeof(T) * kChunk * LD;
    static __device__ __forceinline__ int turn(int row) { return C == 128 ? ((row & 3) << 2) | ((row >> 2) & 3) : ((row & 2) << 1) | ((row >> 2) & 3); }
    // column c of a row (the next three, or seven, behind it where c is a multiple of four, or eight)
    static __device__ __forceinline__ int at(int row, int c) {
        if constexpr (sizeof(T) == 2) return row * LD + (((c >> 3) ^ turn(row)) << 3) + (c & 7);
        else return row * LD + c;
    }
    // rows `row` (this lane's), terms of the block of 32 columns s
    static __device__ __forceinline__ frag_t<T> row_frag(const T* t, int row, int s, int g) { return *reinterpret_cast<const frag_t<T>*>(t + at(row, 32 * s + 8 * g)); }
    // columns column_of(n, lane % 16), terms of the block of 32 rows s: the transposed operand
    static __device__ __forceinline__ frag_t<T> col_frag(const T* t, int s, int n, int lane) {
        const int g = lane >> 4, l = lane & 15;
        if constexpr (sizeof(T) == 2) {
            typedef __attribute__((address_space(3))) I16x4* LdsPtr;
            // a group of 16 lanes hands in four rows of 16 columns, four columns a lane; lane l gets column l of them
            const int row = 32 * s + 8 * g + (l >> 2), c = 32 * (n >> 1) + 8 * (l & 3) + 4 * (n & 1);
            const I16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(t + at(row, c)));
            const I16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LdsPtr)(t + at(row + 4, c)));
            return __builtin_bit_cast(BF16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            const float* from = t + (32 * s + 8 * g) * LD + column_of(n, l);
            F32x8 f;
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = from[e * LD];
            return f;
        }
    }
};

// The weights of a chunk's pairs in LDS, as N pieces.  Whole rows; or (LOWER, bf16) the ten 16 x 16 tiles on and below the diagonal only, where whole rows would
// leave no room for a second workgroup, the halves of a row turned so that 16 rows of eight terms meet in no bank (outputs of 4 x 4,096 rows and 16 heads of
// 128 x 128: 83 us with whole rows, 88 with tiles).
template <typename T, int N, bool LOWER> struct Pairs {
    using Whole = Tile<T, kChunk>;
    static_assert(!LOWER || sizeof(T) == 2, "halves of a row are 16 bytes");
    static constexpr int PIECE = LOWER ? 10 * 256 : kChunk * Whole::LD;
    static constexpr size_t bytes = sizeof(T) * N * PIECE;
    // four neighbouring weights from column 4 g on of row l of tile (ti, tj)
    static __device__ __forceinline__ int at(int ti, int tj, int l, int g) {
        if constexpr (LOWER) return (ti * (ti + 1) / 2 + tj) * 256 + l * 16 + (((g >> 1) ^ (l >> 3)) << 3) + ((g & 1) << 2);
        else return Whole::at(16 * ti + l, 16 * tj + 4 * g);
    }
    static __device__ __forceinline__ void store(T* p, int ti, int tj, int l, int g, F32x4 x) {
        using V4 = T __attribute__((ext_vector_type(4)));
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const V4 v = __builtin_convertvector(x, V4);
            *reinterpret_cast<V4*>(p + n * PIECE + at(ti, tj, l, g)) = v;
            if (n + 1 < N) x -= __builtin_convertvector(v, F32x4);
        }
    }
    // piece n of rows 16 t + l, terms of the block of 32 columns s (t >= 2 s)
    static __device__ __forceinline__ frag_t<T> row_frag(const T* p, int n, int t, int s, int l, int g) {
        const T* from = p + n * PIECE;
        if constexpr (LOWER) {
            const int tj = 2 * s + (g >> 1);
            const frag_t<T> f = *reinterpret_cast<const frag_t<T>*>(from + at(t, tj < t ? tj : t, l, 2 * (g & 1)));
            return t > 2 * s || g < 2 ? f : frag_t<T>{};
        } else {
            return Whole::row_frag(from, 16 * t + l, s, g);
        }
    }
    // what row_frag reads and nobody writes
    static __device__ __forceinline__ void clear(T* p, int l, int g) {
        using V4 = T __attribute__((ext_vector_type(4)));
        if constexpr (!LOWER) {
#pragma unroll
            for (int n = 0; n < N; ++n) {
                *reinterpret_cast<V4*>(p + n * PIECE + Whole::at(l, 16 + 4 * g)) = V4{};
                *reinterpret_cast<V4*>(p + n * PIECE + Whole::at(32 + l, 48 + 4 * g)) = V4{};
            }
        }
    }
};

// ---- 64 rows of `cols` columns from memory into a tile; what is not there is zero ----
// (2 x 8,192 rows, 16 heads of 128 x 128, forward + backward: bf16 126 + 467 us, element by element with rows an odd number apart 277 + 1,061;
// fp32 389 + 1,224 and 554 + 1,824)
template <typename T>
__device__ __forceinline__ bool wide_rows(const T* base, long long stride, int cols) {   // every row aligned to 16 bytes, a multiple of eight columns
    return cols % 8 == 0 && stride % 8 == 0 && reinterpret_cast<uintptr_t>(base) % 16 == 0 && stride < (1 << 20);
}
// a value that the compiler computes addresses from anew: kept across a loop they would take registers that are better used
__device__ __forceinline__ int again(int v) {
    asm volatile("" : "+v"(v));
    return v;
}
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0F70); }   // all of this wavefront's, also those into LDS

// bf16: straight into LDS, 16 bytes a lane; a wavefront fills 64 units one behind the other, so a lane reads the unit whose turned place it has.
// Bounds of the buffer make the zeros.  `load` returns while rows of wide arrays are on their way: wait_loads() before the barrier.
// BACK: row r of the tile is row rows - 1 - r in memory.
template <typename T, int C, int W, bool BACK>
__device__ __forceinline__ void load_tile(T* tile, const T* from, long long stride, int rows, int cols, bool wide, int lane) {
    constexpr int PER = C / 8;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (sizeof(T) == 2 && wide) {
        typedef __attribute__((address_space(3))) void* LdsPtr;
        constexpr int STEP = 64 / PER, N = kChunk / STEP;   // rows of an instruction; instructions of a tile
        const int pitch = (int)stride * 2;
        const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<T*>(from), 0, rows * pitch, 0x00020000);
        // A wavefront's instructions are W apart, a multiple of 16 rows: the same turn in all of them.
        static_assert(N <= W || W * STEP % 16 == 0, "turn() has a period of 16 rows");
        const int row = wave * STEP + lane / PER, c = ((lane % PER) ^ Tile<T, C>::turn(row)) * 8;
        // (a row in front of the first is far behind the end as an unsigned offset)
        const int off = c < cols ? (BACK ? rows - 1 - row : row) * pitch + c * 2 : 0x60000000;
#pragma unroll
        for (int n = 0; n < (N + W - 1) / W; ++n) {
            if (N % W && wave + n * W >= N) break;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (LdsPtr)(tile + (wave + n * W) * STEP * C), 16, off + (BACK ? -n : n) * W * STEP * pitch, 0, 0, 0);
        }
    } else {
        for (int at = threadIdx.x; at < kChunk * PER; at += 64 * W) {
            using V8 = T __attribute__((ext_vector_type(8)));
            const int row = at / PER, c = at % PER * 8;
            V8 v = {};
            if (row < rows) {
                const T* src = from + (BACK ? rows - 1 - row : row) * stride + c;
                if (wide) {
                    if (c < cols) v = *reinterpret_cast<const V8*>(src);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (c + e < cols) v[e] = src[e];
                }
            }
            *reinterpret_cast<V8*>(tile + Tile<T, C>::at(row, c)) = v;
        }
    }
}

// 64 floats of a chunk's kRowFloats straight into LDS: lane i's is from[place]; zero where place lies behind them
__device__ __forceinline__ void load_floats(float* to, const float* from, int place) {
    typedef __attribute__((address_space(3))) void* LdsPtr;
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(from), 0, kRowFloats * 4, 0x00020000);
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (LdsPtr)to, 4, place * 4, 0, 0, 0);
}

// four values of a row, rounded: one store where the rows allow it
template <typename T>
__device__ __forceinline__ void store_four(T* to, F32x4 x, int count, bool wide) {
    using V4 = T __attribute__((ext_vector_type(4)));
    if (wide) {
        if (count >= 4) *reinterpret_cast<V4*>(to) = __builtin_convertvector(x, V4);
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r)
            if (r < count) to[r] = (T)x[r];
    }
}
template <typename T>
__host__ __device__ __forceinline__ bool four_wide(const T* base, long long stride, int cols) {
    return cols % 4 == 0 && stride % 4 == 0 && reinterpret_cast<uintptr_t>(base) % (4 * sizeof(T)) == 0;
}

// Running sum of a chunk's log gates, inclusive, lane by lane, in units of log 2: as the sum of two floats, of which differences
// are taken (a sum of 64 gates of down to -1e4, 2^-46 of it off).  A gate below -1e4 stands for it: its factor is zero either way.
struct Cum {
    float hi, lo;
};
template <int CTRL, int ROWS>
__device__ __forceinline__ double shifted(double v) {
    const long long b = __double_as_longlong(v);
    const unsigned lo = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)b, CTRL, ROWS, 0xF, true);
    const unsigned hi = (unsigned)__builtin_amdgcn_update_dpp(0, (int)(unsigned)((unsigned long long)b >> 32), CTRL, ROWS, 0xF, true);
    return __longlong_as_double((long long)(((unsigned long long)hi << 32) | lo));
}
__device__ __forceinline__ Cum chunk_cum(float g) {
    double c = (g < -1e4f ? -1e4f : g) * 1.4426950408889634;
    c += shifted<0x111, 0xF>(c);   // one, two, four, eight lanes on within rows of 16
    c += shifted<0x112, 0xF>(c);
    c += shifted<0x114, 0xF>(c);
    c += shifted<0x118, 0xF>(c);
    c += shifted<0x142, 0xA>(c);   // the last lane of a row to the next row, the second's to the upper half
    c += shifted<0x143, 0xC>(c);
    Cum r;
    r.hi = (float)c;
    r.lo = (float)(c - (double)r.hi);
    return r;
}
__device__ __forceinline__ float exp2_of(float x) { return __builtin_amdgcn_exp2f(x); }   // 1 ulp; what is below 2^-126 becomes zero
__device__ __forceinline__ float decay_between(float hi_i, float lo_i, float hi_j, float lo_j) { return exp2_of((hi_i - hi_j) + (lo_i - lo_j)); }

__device__ __forceinline__ float lane_value(float v, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); }

// sum over the 16 lanes of a group, in all of them (DPP rotations of a row of 16 lanes by 8, 4, 2, 1)
template <int CTRL>
__device__ __forceinline__ float rotated(float v) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float group_sum(float v) {
    v += rotated<0x128>(v);
    v += rotated<0x124>(v);
    v += rotated<0x122>(v);
    v += rotated<0x121>(v);
    return v;
}

// sum over the wavefront, in lane 63: the rows' sums, the first, second and third row's handed on
__device__ __forceinline__ float wave_sum(float v) {
    v = group_sum(v);
    v += rotated<0x142>(v);
    v += rotated<0x143>(v);
    return v;
}

// tile n of the ten 16 x 16 tiles on and below the diagonal of a chunk's 64 x 64 pairs
__device__ __forceinline__ void lower_tile(int n, int& ti, int& tj) {
    ti = n < 1 ? 0 : n < 3 ? 1 : n < 6 ? 2 : 3;
    tj = n - ti * (ti + 1) / 2;
}

}  // namespace

// ---- how the rows are cut: chunks of 64 rows from every sequence's first, segments of `per` chunks ----
struct MatSegment {
    long long row0;      // first row in the arrays
    long long rows;      // of this segment
    int seq, chunk0;     // sequence; number of the segment's first chunk among all
    int index, count;    // place among the sequence's segments, and how many there are
};
struct MatPlan {
    // With bounds: filled by the plan's kernel; without, every sequence is cut alike and a segment follows from its number.  Segments of sequences that are cut
    // come first, in their order, then the sequences that are whole: only the former have states in memory.
    int* count;          // segments, chunks, segments of sequences that are cut
    MatSegment* segs;    // [max_segs]
    int *seq_seg, *seq_count;   // [N]: a sequence's first segment, and how many it has
    int max_segs, max_slots, max_chunks, per;
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
    // states in memory between kernels are whole tiles of 64 or 128 rows and columns (the next from Dk and Dv), zero outside the head
    float *seg_state, *seg_rstate;   // [max_slots][Hv][tile]: a segment's own part, then the state in front of it (gradient: behind it)
    float *seg_decay;                // [2][max_slots][Hv]
    float *rows_of;                  // [chunks][Hv][kRowFloats]: a chunk's running gates and the factors that follow from them
    // gradient only
    float *part_q, *part_k;          // [rows][Hv][Dk]: dq and dk by heads of v, where several share one
    float *gate_k;                   // [rows][Hv]: the part of dgate that the run of dk has
    float *read_in, *put_out;        // [chunks][Hv]: sums of q_i . (...) and k_j . (...) over a chunk
    float *size_in, *size_out;       // [chunks][Hv]: sums of the squares of the state in front of a chunk, and of the gradient of the state behind it
    float *front;                    // [max_segs][Hv]: <state, its gradient> in front of a segment
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

// segment number `no`; false behind the last
__device__ __forceinline__ bool segment_of(const MatrecParams& p, int no, MatSegment& s) {
    if (p.rows.bounds) {
        if (no >= *p.plan.count) return false;
        s = p.plan.segs[no];
        return true;
    }
    const int chunks = (int)((p.rows.T + 63) / 64);
    s.count = (chunks + p.plan.per - 1) / p.plan.per;
    if (s.count == 0 || no >= s.count * p.rows.N) return false;
    s.seq = no / s.count;
    s.index = no % s.count;
    s.chunk0 = s.seq * chunks + s.index * p.plan.per;
    const long long first = (long long)s.index * p.plan.per * 64, most = (long long)p.plan.per * 64;
    s.row0 = s.seq * p.rows.T + first;
    s.rows = p.rows.T - first < most ? p.rows.T - first : most;
    return true;
}
// The segment of chunk number `chunk` of all sequences', and which of its chunks that is; false behind the last.  With bounds all lanes of a wavefront
// take part: they look at 64 segments at a time, among those of cut sequences and among whole ones at once, so that up to 4,096 of either are two loads
// one after another.
__device__ __forceinline__ bool segment_of_chunk(const MatrecParams& p, int chunk, MatSegment& s, int& place) {
    if (p.rows.bounds) {
        if (chunk >= p.plan.count[1]) return false;
        // the last one that begins at the chunk or in front of it: in lo .. hi - 1, if there is one
        int lo[2] = {0, p.plan.count[2]}, hi[2] = {p.plan.count[2], p.plan.count[0]};
        do {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int step = (hi[k] - lo[k] + 63) / 64, at = lo[k] + (int)(threadIdx.x & 63) * step;
                const int front = __popcll(__ballot(at < hi[k] && p.plan.segs[at < hi[k] ? at : 0].chunk0 <= chunk));
                lo[k] += front > 0 ? (front - 1) * step : 0;
                hi[k] = front == 0 ? lo[k] : lo[k] + step < hi[k] ? lo[k] + step : hi[k];
            }
        } while (hi[0] - lo[0] > 1 || hi[1] - lo[1] > 1);
        const bool cut = hi[0] > lo[0], whole = hi[1] > lo[1];
        s = p.plan.segs[cut ? lo[0] : lo[1]];
        if (cut && whole) {
            const MatSegment other = p.plan.segs[lo[1]];
            if (other.chunk0 > s.chunk0) s = other;
        }
    } else {
        const int chunks = (int)((p.rows.T + 63) / 64);
        if (chunks == 0 || chunk / chunks >= p.rows.N) return false;
        if (!segment_of(p, chunk / chunks * ((chunks + p.plan.per - 1) / p.plan.per) + chunk % chunks / p.plan.per, s)) return false;
    }
    place = chunk - s.chunk0;
    return true;
}
// first segment of sequence n, and how many it has
__device__ __forceinline__ int first_segment(const MatrecParams& p, int n, int& count) {
    if (p.rows.bounds) {
        count = p.plan.seq_count[n];
        return p.plan.seq_seg[n];
    }
    count = ((int)((p.rows.T + 63) / 64) + p.plan.per - 1) / p.plan.per;
    return n * count;
}

hipError_t launch_matrec_plan(const MatrecParams& p, const RestRows& rest, hipStream_t stream);   // segments, the gates of their chunks, rows of no sequence
hipError_t launch_matrec_out(int dtype, const MatrecParams& p, hipStream_t stream);
hipError_t launch_matrec_join(int dtype, const MatrecParams& p, bool both, hipStream_t stream);   // states in front of the segments (both: behind them too)
hipError_t launch_matrec_grad(int dtype, const MatrecParams& p, hipStream_t stream);
hipError_t launch_matstep(int dtype, const MatstepParams& p, hipStream_t stream);

}  // namespace deer
