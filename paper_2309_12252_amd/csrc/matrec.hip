// Gated linear recurrence with a matrix as state: S_t = e^{g_t} S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t; by chunks of 64 rows on the matrix
// cores.  With c_i the sum of a chunk's log gates up to row i, inclusive, and S the state in front of the chunk,
//   o_i = scale (e^{c_i} S^T q_i + sum_{j <= i} e^{c_i - c_j} (q_i . k_j) v_j)
//   S'  = e^{c_64} S + sum_j e^{c_64 - c_j} k_j v_j^T.
// States are sums over many rows and stay in fp32 accumulators; v_j e^{c_64 - c_j} enters their update as three bf16 pieces, so a state is as exact as
// fp32 sums make it.  The products of the output take S and the 64 x 64 factors as two pieces (2^-16): an output is as exact as its
// own rounding to bf16.  What is NaN or infinite in a row reaches its chunk (products with factors that are zero) and what follows.
#include "matrec_run.h"

namespace deer {
namespace {

__device__ __forceinline__ int segments_of(const MatrecParams& p, long long rows) { return ((int)((rows + kChunk - 1) / kChunk) + p.plan.per - 1) / p.plan.per; }

// One workgroup: sequences' chunks and segments are counted in their order (running sums over the sequences).  5 us for 7 sequences (launch and one
// chain of loads), so it runs only where there are bounds: without, a segment follows from its number.
__global__ __launch_bounds__(1024) void matrec_plan_kernel(const MatrecParams p) {
    const MatPlan& plan = p.plan;
    __shared__ int sums[3][16], all_cut;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (tid == 0) all_cut = 0;
    // bounds that decrease would ask for more chunks than there is room for: then there are no segments at all
    bool bad = false;
    int cut = 0;
    for (int n = tid; n < p.rows.N; n += 1024) {
        if (p.rows.packed) bad = bad || clamp_row(p.rows.bounds[n + 1], p.rows.T) < clamp_row(p.rows.bounds[n], p.rows.T);
        const int segs = segments_of(p, seq_length(p.rows, n));
        cut += segs > 1 ? segs : 0;
    }
    bad = __syncthreads_or(bad) != 0;
    if (cut > 0 && !bad) atomicAdd(&all_cut, cut);
    __syncthreads();
    cut = all_cut;
    int run[3] = {0, 0, 0};   // of the sequences in front: whole ones, chunks, segments of those that are cut
    for (int base = 0; base < p.rows.N; base += 1024) {
        const int n = base + tid;
        const long long len = n < p.rows.N && !bad ? seq_length(p.rows, n) : 0;
        const int chunks = (int)((len + kChunk - 1) / kChunk), segs = segments_of(p, len);
        int mine[3] = {segs == 1 ? 1 : 0, chunks, segs > 1 ? segs : 0}, at[3];   // `at`: exclusive sums over the workgroup behind `run`, which moves on
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            int v = mine[k];
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const int o = __shfl_up(v, d);
                v += lane >= d ? o : 0;
            }
            at[k] = run[k] + v - mine[k];
            if (lane == 63) sums[k][wave] = v;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 3; ++k)
#pragma unroll
            for (int w = 0; w < 16; ++w) {
                const int x = sums[k][w];
                at[k] += w < wave ? x : 0;
                run[k] += x;
            }
        __syncthreads();
        if (n < p.rows.N) {
            const int first_seg = segs > 1 ? at[2] : cut + at[0];
            plan.seq_seg[n] = first_seg;
            plan.seq_count[n] = segs;
            const long long row = p.rows.packed ? clamp_row(p.rows.bounds[n], p.rows.T) : (long long)n * p.rows.T;
            for (int s = 0; s < segs; ++s) {
                const long long first = (long long)s * plan.per * kChunk, most = (long long)plan.per * kChunk;
                MatSegment g;
                g.row0 = row + first;
                g.rows = len - first < most ? len - first : most;
                g.seq = n;
                g.chunk0 = at[1] + s * plan.per;
                g.index = s;
                g.count = segs;
                plan.segs[first_seg + s] = g;
            }
        }
    }
    if (tid == 0) {
        plan.count[0] = run[0] + run[2];
        plan.count[1] = run[1];
        plan.count[2] = run[2];
    }
}

// The gates of every chunk, once for all that use them: their running sum is a chain of dependent steps, and 64 gates of a head lie in as many
// cache lines.  A workgroup has a chunk, a wavefront one head after another.  5 us for 16,384 rows of 16 heads; summed again by every run: outputs
// 91 us against 85, gradient 452 against 431.  On request also zeroes rows of no sequence.
__global__ __launch_bounds__(256) void matrec_rows_kernel(const MatrecParams p, const RestRows rest) {
    clear_rest(p.rows, rest, blockIdx.x, gridDim.x);
    const int lane = threadIdx.x & 63;
    int c;
    MatSegment seg;
    if (!segment_of_chunk(p, blockIdx.x, seg, c)) return;
    const long long left = seg.rows - (long long)c * kChunk;
    const int rows = left < kChunk ? (int)left : kChunk;
    const long long row = seg.row0 + (long long)c * kChunk;
    for (int head = threadIdx.x >> 6; head < p.Hv; head += 4) {
        const Cum cum = chunk_cum(lane < rows ? p.gate[(row + lane) * p.Hv + head] : 0.0f);
        const float end_hi = lane_value(cum.hi, 63), end_lo = lane_value(cum.lo, 63);
        float* to = p.rows_of + ((long long)blockIdx.x * p.Hv + head) * kRowFloats;
        to[lane] = cum.hi;
        to[64 + lane] = cum.lo;
        to[128 + lane] = p.scale * exp2_of(cum.hi + cum.lo);
        to[192 + lane] = decay_between(end_hi, end_lo, cum.hi, cum.lo);
        if (lane < 4) to[256 + lane] = lane == 0 ? exp2_of(end_hi + end_lo) : lane == 1 ? end_hi : lane == 2 ? end_lo : 0.0f;
    }
}

// ---- states ----
// A segment's own part of the state, and its decay, into seg_state (REV: of the gradient of the state in front of it, into seg_rstate: rows backwards,
// (k, v) = (scale q, dout), R <- e^{c_64} R + sum_i e^{c_i} scale q_i dout_i^T).  Wavefront w keeps a quarter of v's columns, transposed: a lane has
// four neighbouring v of one d in 16, so that states go to memory 16 bytes a lane.  A wavefront has 16 columns of v: 48 matrix instructions a chunk (three
// pieces), about as many vector instructions for the pieces, and 32 KiB of rows a chunk for the workgroup: 1 x 32,768 rows, 8 heads of 128 x 64 (100 MB) in
// 24 us, 4.2 TB/s; 39 us for 4 x 4,096 rows and 16 heads of 128 x 128 (134 MB, 3.4 TB/s).  128 registers, so that two workgroups share a CU and one
// computes while the other waits: six wavefronts a SIMD spill (prompts of 8,192 rows 96 -> 107 us).
template <typename T, int DK, int DV>
struct StatesLds {
    static constexpr size_t k = 0, v = Tile<T, DK>::bytes, w = v + Tile<T, DV>::bytes, total = w + 4 * 128;
};
template <typename T, int DK, int DV, bool REV>
__device__ __forceinline__ void states_of(const MatrecParams& p, unsigned char* lds) {
    constexpr int W = DV / 16, NT = DK / 16, P = Op<T>::PIECES;
    using L = StatesLds<T, DK, DV>;
    using TK = Tile<T, DK>;
    using TV = Tile<T, DV>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, l = lane & 15;
    const int seg_no = blockIdx.x / p.Hv, head = blockIdx.x % p.Hv, kh = head / (p.Hv / p.Hk);
    MatSegment seg;
    if (!segment_of(p, seg_no, seg)) return;
    if (seg.index == (REV ? 0 : seg.count - 1)) return;   // nothing comes behind it
    const long long stride_k = REV ? p.stride_q : p.stride_k, stride_v = REV ? p.stride_o : p.stride_v;
    const T* k = reinterpret_cast<const T*>(REV ? p.q : p.k) + (long long)kh * p.Dk + seg.row0 * stride_k;
    const T* v = reinterpret_cast<const T*>(REV ? p.dout : p.v) + (long long)head * p.Dv + seg.row0 * stride_v;
    const float* gates = p.rows_of + ((long long)seg.chunk0 * p.Hv + head) * kRowFloats;
    const bool wide_k = wide_rows(k, stride_k, p.Dk), wide_v = wide_rows(v, stride_v, p.Dv);
    T *tk = reinterpret_cast<T*>(lds + L::k), *tv = reinterpret_cast<T*>(lds + L::v);
    float* weight = reinterpret_cast<float*>(lds + L::w);
    F32x4 S[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) S[t] = F32x4{0, 0, 0, 0};
    const int chunks = (int)((seg.rows + kChunk - 1) / kChunk);
    double total = 0.0;
    auto load = [&](int i) {
        const int c = REV ? chunks - 1 - i : i;
        const long long row = (long long)c * kChunk;
        const int rows = seg.rows - row < kChunk ? (int)(seg.rows - row) : kChunk;
        load_tile<T, DK, W, false>(tk, k + row * stride_k, stride_k, rows, p.Dk, wide_k, lane);
        load_tile<T, DV, W, false>(tv, v + row * stride_v, stride_v, rows, p.Dv, wide_v, lane);
        const float* from = gates + (long long)c * p.Hv * kRowFloats;
        if (wave < 2) load_floats(weight + 64 * wave, from, wave == 0 ? (REV ? 128 : 192) + lane : 256 + lane);
    };
    load(0);
    for (int i = 0; i < chunks; ++i) {
        wait_loads();
        __syncthreads();
        const float whole = weight[64];
        total += (double)weight[65] + (double)weight[66];
#pragma unroll
        for (int t = 0; t < NT; ++t) S[t] *= whole;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const F32x4 w0 = *reinterpret_cast<const F32x4*>(weight + 32 * s + 8 * g), w1 = *reinterpret_cast<const F32x4*>(weight + 32 * s + 8 * g + 4);
            frag_t<T> vp[P];
            pieces_of<T>(widened(TV::col_frag(tv, s, wave, lane)) * joined(w0, w1), vp);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const frag_t<T> kf = TK::col_frag(tk, s, t, lane);
#pragma unroll
                for (int q = P - 1; q >= 0; --q) S[t] = mma(vp[q], kf, S[t]);
            }
        }
        __syncthreads();
        if (i + 1 < chunks) load(i + 1);
    }
    const long long at = (long long)seg_no * p.Hv + head;
    float* to = (REV ? p.seg_rstate : p.seg_state) + at * (DK * DV);   // (outside the head: zero in S too)
#pragma unroll
    for (int t = 0; t < NT; ++t) *reinterpret_cast<F32x4*>(to + column_of(t, l) * DV + column_of(wave, 4 * g)) = S[t];
    if (threadIdx.x == 0) p.seg_decay[(REV ? (long long)p.plan.max_slots * p.Hv : 0) + at] = (float)exp2(total);
}

// blockIdx.y: 0 the states, 1 their gradients
template <typename T, int DK, int DV>
__global__ __launch_bounds__(4 * DV, sizeof(T) == 2 ? 4 : 2) void matrec_states_kernel(const MatrecParams p) {
    extern __shared__ __align__(16) unsigned char lds[];
    if (blockIdx.y == 0) states_of<T, DK, DV, false>(p, lds);
    else states_of<T, DK, DV, true>(p, lds);
}

// The segments' own parts joined along a sequence, in their order: seg_state becomes the state in front of each segment (REV: seg_rstate the gradient
// of the state behind it).  A lane has one cell of a tile and reads eight segments at a time (four cells a
// lane take 180 registers: 28 us against 22 for both directions of 16 heads and 32 segments; 64 KiB a segment and head, read and written once, bound it).  Also what a sequence without rows has in the place
// of a final state (REV: of ds0).
template <int DK, int DV, bool REV>
__device__ __forceinline__ void join_cell(const MatrecParams& p, int n, int head, int cell) {
    const int d = cell / DV, v = cell % DV;
    const bool inside = d < p.Dk && v < p.Dv;
    const long long at = (((long long)n * p.Hv + head) * p.Dk + d) * p.Dv + v;
    const float* ends = REV ? p.dlast : p.s0;
    float* outs = REV ? p.ds0 : p.last;
    int count;
    const int first = first_segment(p, n, count);
    if (count == 1) return;   // (a run takes what is given in front of a sequence from where it is given)
    float s = ends && inside ? ends[at] : 0.0f;
    if (count == 0) {
        if (outs && inside) outs[at] = s;
        return;
    }
    if (!p.split) return;
    float* states = REV ? p.seg_rstate : p.seg_state;
    const float* decay = p.seg_decay + (REV ? (long long)p.plan.max_slots * p.Hv : 0);
    constexpr int K = 8;
    for (int i0 = 0; i0 < count; i0 += K) {
        float own[K], f[K];
#pragma unroll
        for (int i = 0; i < K; ++i) {   // (the last one along the way has none, and none is wanted)
            const bool there = i0 + i < count - 1;
            const long long seg = (first + (REV ? count - 1 - i0 - i : i0 + i)) * (long long)p.Hv + head;
            own[i] = there ? states[seg * (DK * DV) + cell] : 0.0f;
            f[i] = there ? decay[seg] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < K; ++i) {
            if (i0 + i >= count) break;
            const long long seg = (first + (REV ? count - 1 - i0 - i : i0 + i)) * (long long)p.Hv + head;
            if (i0 + i > 0) states[seg * (DK * DV) + cell] = s;
            s = f[i] * s + own[i];
        }
    }
}
// At most as many workgroups as run at a time (two rounds of them): with one for every 256 cells, 32 sequences of 100 rows and 16 heads, of which nothing
// is to be joined, took 32 us, so 18; sequences of many segments the same 14 and 22 us either way.
constexpr int kJoinBlocks = 4096;
template <int DK, int DV>
__global__ __launch_bounds__(256) void matrec_join_kernel(const MatrecParams p) {
    constexpr int PER = DK * DV / 256;
    const long long all = (long long)p.rows.N * p.Hv * PER;
    for (long long id = blockIdx.x; id < all; id += gridDim.x) {
        const long long at = id / PER;
        const int cell = (int)(id % PER) * 256 + threadIdx.x, n = (int)(at / p.Hv), head = (int)(at % p.Hv);
        if (blockIdx.y == 0) join_cell<DK, DV, false>(p, n, head, cell);
        else join_cell<DK, DV, true>(p, n, head, cell);
    }
}

template <typename T, int DK, int DV>
__global__ __launch_bounds__(4 * DV, sizeof(T) == 2 ? (DV == 128 ? 4 : 3) : 2) void matrec_out_kernel(const MatrecParams p) {
    extern __shared__ __align__(16) unsigned char lds[];
    matrec_run<T, DK, DV, DV / 16, RUN_OUT>(p, lds, blockIdx.x);
}

// ---- one token ----
// Memory bound: the state, fp32, is read and written once.  A workgroup has one row and head; a lane V columns of some rows of the state.  64 rows and 16
// heads of 128 x 128 (134 MB): 22 us, 6 TB/s; a column a lane, where the states are not aligned to 16 bytes or Dv is no multiple of four, 28.
template <typename T, int V>
__global__ __launch_bounds__(256) void matstep_kernel(const MatstepParams p) {
    using FV = vec_t<float, V>;
    __shared__ float sums[256 * V];
    const int n = blockIdx.x / p.Hv, head = blockIdx.x % p.Hv, kh = head / (p.Hv / p.Hk);
    int slot = n;
    bool twice = false;
    if (p.rows.slots) {
        slot = p.rows.slots[n];
        for (int m = threadIdx.x; m < n; m += 256) twice = twice || p.rows.slots[m] == slot;
        twice = __syncthreads_or(twice) != 0;
    }
    if (slot < 0 || slot >= p.rows.n_slots || twice) {
        if (p.rows.zero_rest)
            for (int col = threadIdx.x; col < p.Dv; col += 256) reinterpret_cast<T*>(p.o)[n * p.stride_o + (long long)head * p.Dv + col] = (T)0.0f;
        return;
    }
    const int cols = p.Dv / V, per = 256 / cols;               // lanes of a row of the state, rows at a time
    const int c = threadIdx.x % cols, d0 = threadIdx.x / cols;
    const bool on = d0 < per;
    const T* q = reinterpret_cast<const T*>(p.q) + n * p.stride_q + (long long)kh * p.Dk;
    const T* k = reinterpret_cast<const T*>(p.k) + n * p.stride_k + (long long)kh * p.Dk;
    const T* v = reinterpret_cast<const T*>(p.v) + n * p.stride_v + (long long)head * p.Dv + c * V;
    float* state = p.state + ((long long)slot * p.Hv + head) * p.Dk * p.Dv + c * V;
    const float a = expf(p.gate[(long long)n * p.Hv + head]);
    float vv[V], o[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        vv[i] = (float)v[i];
        o[i] = 0.0f;
    }
    if (on) {
#pragma unroll 4
        for (int d = d0; d < p.Dk; d += per) {
            FV s = *reinterpret_cast<const FV*>(state + (long long)d * p.Dv);
            const float kd = (float)k[d], qd = (float)q[d];
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float x = a * vec_at<float, V>(s, i) + kd * vv[i];
                vec_set<float, V>(s, i, x);
                o[i] += qd * x;
            }
            *reinterpret_cast<FV*>(state + (long long)d * p.Dv) = s;
        }
#pragma unroll
        for (int i = 0; i < V; ++i) sums[d0 * p.Dv + c * V + i] = o[i];
    }
    __syncthreads();
    for (int col = threadIdx.x; col < p.Dv; col += 256) {
        float t = 0.0f;
        for (int r = 0; r < per; ++r) t += sums[r * p.Dv + col];
        reinterpret_cast<T*>(p.o)[n * p.stride_o + (long long)head * p.Dv + col] = (T)(p.scale * t);
    }
}

template <typename T, int DK, int DV>
hipError_t join_shape(const MatrecParams& p, bool both, hipStream_t stream) {
    hipError_t e = hipSuccess;
    const unsigned y = both ? 2 : 1;
    if (p.split) e = launch_lds(matrec_states_kernel<T, DK, DV>, dim3((unsigned)((long long)p.plan.max_slots * p.Hv), y), 4 * DV, StatesLds<T, DK, DV>::total, p, stream);
    const bool empty = p.rows.bounds || p.rows.T == 0;   // (there may be sequences without rows)
    if (e != hipSuccess || !(p.split || (empty && (p.last || p.ds0)))) return e;
    const long long blocks = (long long)p.rows.N * p.Hv * (DK * DV / 256);
    hipLaunchKernelGGL((matrec_join_kernel<DK, DV>), dim3((unsigned)(blocks < kJoinBlocks ? blocks : kJoinBlocks), y), dim3(256), 0, stream, p);
    return hipGetLastError();
}
template <typename T, int DK, int DV>
hipError_t out_shape(const MatrecParams& p, hipStream_t stream) {
    const hipError_t e = join_shape<T, DK, DV>(p, false, stream);
    if (e != hipSuccess) return e;
    return launch_lds(matrec_out_kernel<T, DK, DV>, dim3((unsigned)((long long)p.plan.max_segs * p.Hv)), 4 * DV, RunLds<T, DK, DV, DV / 16, RUN_OUT>::total, p, stream);
}

}  // namespace

hipError_t launch_matrec_plan(const MatrecParams& p, const RestRows& rest, hipStream_t stream) {
    hipError_t e = hipSuccess;
    if (p.rows.bounds) {
        hipLaunchKernelGGL(matrec_plan_kernel, dim3(1), dim3(1024), 0, stream, p);
        e = hipGetLastError();
    }
    if (e != hipSuccess || p.plan.max_chunks == 0) return e;
    hipLaunchKernelGGL(matrec_rows_kernel, dim3((unsigned)p.plan.max_chunks), dim3(256), 0, stream, p, rest);
    return hipGetLastError();
}
hipError_t launch_matrec_out(int dtype, const MatrecParams& p, hipStream_t stream) {
    return dtype == DEER_BF16 ? DEER_BY_SHAPE(out_shape, BF16, stream) : DEER_BY_SHAPE(out_shape, float, stream);
}
hipError_t launch_matrec_join(int dtype, const MatrecParams& p, bool both, hipStream_t stream) {
    return dtype == DEER_BF16 ? DEER_BY_SHAPE(join_shape, BF16, both, stream) : DEER_BY_SHAPE(join_shape, float, both, stream);
}

template <typename T>
static hipError_t step_type(const MatstepParams& p, hipStream_t stream) {
    const dim3 grid((unsigned)((long long)p.rows.N * p.Hv));
    if (p.Dv % 4 == 0 && reinterpret_cast<uintptr_t>(p.state) % 16 == 0) hipLaunchKernelGGL((matstep_kernel<T, 4>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((matstep_kernel<T, 1>), grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}
hipError_t launch_matstep(int dtype, const MatstepParams& p, hipStream_t stream) {
    return dtype == DEER_BF16 ? step_type<BF16>(p, stream) : step_type<float>(p, stream);
}

}  // namespace deer
