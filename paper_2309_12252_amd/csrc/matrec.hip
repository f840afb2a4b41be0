// Gated linear recurrence with a matrix as state: S_t = e^{g_t} S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t; by chunks of 64 rows on the matrix
// cores.  With c_i the sum of a chunk's log gates up to row i, inclusive, and S the state in front of the chunk,
//   o_i = scale (e^{c_i} S^T q_i + sum_{j <= i} e^{c_i - c_j} (q_i . k_j) v_j)
//   S'  = e^{c_64} S + sum_j e^{c_64 - c_j} k_j v_j^T.
// States are sums over many rows and stay in fp32 accumulators; v_j e^{c_64 - c_j} enters their update as three bf16 pieces, so a state is as exact as
// fp32 sums make it.  The products of the output take S and the 64 x 64 factors rounded to bf16 once: an output
// is rounded to bf16 itself.  What is NaN or infinite in a row reaches its chunk (products with factors that are zero) and what follows.
#include "matrec_common.h"

namespace deer {
namespace {

// One workgroup: sequences' chunks and segments are counted in their order (running sums over the sequences).
__global__ __launch_bounds__(1024) void matrec_plan_kernel(const MatrecParams p) {
    const MatPlan& plan = p.plan;
    __shared__ int sums[16];
    __shared__ int run_s, run_c;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    if (tid == 0) run_s = run_c = 0;
    __syncthreads();
    auto scan = [&](int mine, int* run) {   // exclusive sum over the workgroup, `run` moved on
        int v = mine;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int o = __shfl_up(v, d);
            v += lane >= d ? o : 0;
        }
        if (lane == 63) sums[wave] = v;
        __syncthreads();
        int before = *run;
        for (int w = 0; w < wave; ++w) before += sums[w];
        const int total = *run + [&] { int t = 0; for (int w = 0; w < 16; ++w) t += sums[w]; return t; }();
        __syncthreads();
        if (tid == 0) *run = total;
        __syncthreads();
        return before + v - mine;
    };
    // bounds that decrease would ask for more chunks than there is room for: then there are no segments at all
    bool bad = false;
    if (p.rows.packed)
        for (int n = tid; n < p.rows.N; n += 1024) bad = bad || clamp_row(p.rows.bounds[n + 1], p.rows.T) < clamp_row(p.rows.bounds[n], p.rows.T);
    bad = __syncthreads_or(bad) != 0;
    for (int base = 0; base < p.rows.N; base += 1024) {
        const int n = base + tid;
        const long long len = n < p.rows.N && !bad ? seq_length(p.rows, n) : 0;
        const int chunks = (int)((len + kChunk - 1) / kChunk), segs = (chunks + plan.per - 1) / plan.per;
        const int s0 = scan(segs, &run_s), c0 = scan(chunks, &run_c);
        if (n < p.rows.N) {
            plan.seq_seg[n] = s0;
            const long long row = p.rows.packed ? clamp_row(p.rows.bounds[n], p.rows.T) : (long long)n * p.rows.T;
            for (int s = 0; s < segs; ++s) {
                const long long first = (long long)s * plan.per * kChunk, most = (long long)plan.per * kChunk;
                MatSegment g;
                g.row0 = row + first;
                g.rows = len - first < most ? len - first : most;
                g.seq = n;
                g.chunk0 = c0 + s * plan.per;
                g.index = s;
                g.count = segs;
                plan.segs[s0 + s] = g;
            }
        }
    }
    __syncthreads();
    if (tid == 0) {
        *plan.count = run_s;
        plan.seq_seg[p.rows.N] = run_s;
    }
}

// ---- states ----
// One segment and head: the state's own part of the segment (STORE = false: into seg_state / seg_rstate, with the segment's decay), or with the state in
// front of the segment known, the state in front of every chunk (REV: the gradient of the state behind it).  REV: rows backwards,
// (k, v) = (scale q, dout), the gradient of the state in front of a chunk is e^{c_64} R + sum_i e^{c_i} scale q_i dout_i^T.
// Wavefront w keeps columns 16 w .. of v, transposed: a lane has four neighbouring v of every 16th d, so that states go to memory 16 bytes a lane.
template <typename T, int DK, int DV, bool REV, bool STORE>
__device__ __forceinline__ void states_of(const MatrecParams& p, int seg_no, int head, T* tk, T* tv, float* weight) {
    constexpr int W = DV / 16, NT = DK / 16, P = Op<T>::PIECES;
    using TK = Tile<T, DK>;
    using TV = Tile<T, DV>;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, l = lane & 15;
    const MatSegment seg = p.plan.segs[seg_no];
    if (!STORE && seg.index == (REV ? 0 : seg.count - 1)) return;   // nothing comes behind it
    const long long cells = (long long)p.Dk * p.Dv;
    const int kh = head / (p.Hv / p.Hk);
    const long long stride_k = REV ? p.stride_q : p.stride_k, stride_v = REV ? p.stride_o : p.stride_v;
    const T* k = reinterpret_cast<const T*>(REV ? p.q : p.k) + (long long)kh * p.Dk + seg.row0 * stride_k;
    const T* v = reinterpret_cast<const T*>(REV ? p.dout : p.v) + (long long)head * p.Dv + seg.row0 * stride_v;
    const float* gate = p.gate + seg.row0 * p.Hv + head;
    float* seg_states = REV ? p.seg_rstate : p.seg_state;
    const int v0 = 16 * wave + 4 * g;
    F32x4 S[NT];
    const bool whole_rows = (p.Dv & 3) == 0;
    auto store = [&](float* to) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
            if (16 * t + l < p.Dk && v0 < p.Dv) store_four<float>(to + (long long)(16 * t + l) * p.Dv + v0, S[t], p.Dv - v0, whole_rows && reinterpret_cast<uintptr_t>(to) % 16 == 0);
    };
    const float* from = nullptr;
    if (STORE) {
        const float* ends = REV ? p.dlast : p.s0;
        const bool at_end = seg.index == (REV ? seg.count - 1 : 0);
        from = at_end ? (ends ? ends + ((long long)seg.seq * p.Hv + head) * cells : nullptr) : seg_states + ((long long)seg_no * p.Hv + head) * cells;
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        S[t] = F32x4{0, 0, 0, 0};
        if (from && 16 * t + l < p.Dk) {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (v0 + r < p.Dv) S[t][r] = from[(long long)(16 * t + l) * p.Dv + v0 + r];
        }
    }
    const int chunks = (int)((seg.rows + kChunk - 1) / kChunk);
    double total = 0.0;
    Stage<T, DK, 64 * W> fk;
    Stage<T, DV, 64 * W> fv;
    float fg = 0.0f;
    auto fetch = [&](int i) {
        const int c = REV ? chunks - 1 - i : i;
        const long long row = (long long)c * kChunk;
        const int rows = seg.rows - row < kChunk ? (int)(seg.rows - row) : kChunk;
        fk.fetch(k + row * stride_k, stride_k, rows, p.Dk);
        fv.fetch(v + row * stride_v, stride_v, rows, p.Dv);
        fg = gate_of(gate + row * p.Hv, p.Hv, rows);
    };
    const int updates = STORE && !REV ? chunks - 1 : chunks;   // (the state behind the last chunk is somebody else's)
    if (updates > 0) fetch(0);
    for (int i = 0; i < chunks; ++i) {
        const int c = REV ? chunks - 1 - i : i;
        if (STORE) {   // whole tiles: what lies outside the head is zero in S too
            float* to = (REV ? p.chunk_rstate : p.chunk_state) + ((long long)(seg.chunk0 + c) * p.Hv + head) * (DK * DV) + l * DV + v0;
#pragma unroll
            for (int t = 0; t < NT; ++t) *reinterpret_cast<F32x4*>(to + 16 * t * DV) = S[t];
        }
        if (i >= updates) break;
        const Cum cum = chunk_cum(fg);
        const float end_hi = lane_value(cum.hi, 63), end_lo = lane_value(cum.lo, 63);
        __syncthreads();
        fk.put(tk);
        fv.put(tv);
        if (wave == 0) weight[lane] = REV ? p.scale * expf(cum.hi + cum.lo) : decay_between(end_hi, end_lo, cum.hi, cum.lo);
        __syncthreads();
        if (i + 1 < updates) fetch(i + 1);
        const float whole = expf(end_hi + end_lo);
#pragma unroll
        for (int t = 0; t < NT; ++t) S[t] *= whole;
        total += (double)end_hi + (double)end_lo;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const F32x4 w0 = *reinterpret_cast<const F32x4*>(weight + 32 * s + 4 * g), w1 = *reinterpret_cast<const F32x4*>(weight + 32 * s + 16 + 4 * g);
            frag_t<T> vp[P];
            pieces_of<T>(widened(TV::col_frag(tv, s, wave, lane)) * joined(w0, w1), vp);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const frag_t<T> kf = TK::col_frag(tk, s, t, lane);
#pragma unroll
                for (int q = P - 1; q >= 0; --q) S[t] = mma(vp[q], kf, S[t]);
            }
        }
    }
    if (STORE) {
        if (REV && seg.index == 0 && p.ds0) store(p.ds0 + ((long long)seg.seq * p.Hv + head) * cells);
    } else {
        store(seg_states + ((long long)seg_no * p.Hv + head) * cells);
        if (threadIdx.x == 0) p.seg_decay[(REV ? (long long)p.plan.max_segs * p.Hv : 0) + (long long)seg_no * p.Hv + head] = (float)exp(total);
    }
}

// blockIdx.y: 0 the states, 1 their gradients
template <typename T, int DK, int DV, bool STORE>
__global__ __launch_bounds__(4 * DV) void matrec_states_kernel(const MatrecParams p) {
    extern __shared__ __align__(16) unsigned char lds[];
    T* tk = reinterpret_cast<T*>(lds);
    T* tv = reinterpret_cast<T*>(lds + Tile<T, DK>::bytes);
    float* weight = reinterpret_cast<float*>(lds + Tile<T, DK>::bytes + Tile<T, DV>::bytes);
    const int seg = blockIdx.x / p.Hv, head = blockIdx.x % p.Hv;
    if (seg >= *p.plan.count) return;
    if (blockIdx.y == 0) states_of<T, DK, DV, false, STORE>(p, seg, head, tk, tv, weight);
    else states_of<T, DK, DV, true, STORE>(p, seg, head, tk, tv, weight);
}

// The segments' own parts joined along a sequence, in their order: seg_state becomes the state in front of each segment (REV: seg_rstate the gradient
// of the state behind it).  A lane has one cell and reads eight segments at a time.  Also what a sequence without rows has in the place of
// a final state (REV: of ds0).
template <bool REV>
__device__ __forceinline__ void join_cell(const MatrecParams& p, int n, int head, int cell) {
    const long long cells = (long long)p.Dk * p.Dv, at = ((long long)n * p.Hv + head) * cells + cell;
    const float* ends = REV ? p.dlast : p.s0;
    float* outs = REV ? p.ds0 : p.last;
    const int first = p.plan.seq_seg[n], count = p.plan.seq_seg[n + 1] - first;
    float s = ends ? ends[at] : 0.0f;
    if (count == 0) {
        if (outs) outs[at] = s;
        return;
    }
    if (!p.split) return;
    float* states = REV ? p.seg_rstate : p.seg_state;
    const float* decay = p.seg_decay + (REV ? (long long)p.plan.max_segs * p.Hv : 0);
    constexpr int K = 8;
    for (int i0 = 0; i0 < count; i0 += K) {
        float own[K], f[K];
#pragma unroll
        for (int i = 0; i < K; ++i) {   // (of the last one along the way nothing is written or used)
            const int j = i0 + i < count - 1 ? i0 + i : 0;
            const long long seg = (first + (REV ? count - 1 - j : j)) * (long long)p.Hv + head;
            own[i] = states[seg * cells + cell];
            f[i] = decay[seg];
        }
#pragma unroll
        for (int i = 0; i < K; ++i) {
            if (i0 + i >= count) break;
            const long long seg = (first + (REV ? count - 1 - i0 - i : i0 + i)) * (long long)p.Hv + head;
            states[seg * cells + cell] = s;
            s = f[i] * s + own[i];
        }
    }
}
__global__ __launch_bounds__(256) void matrec_join_kernel(const MatrecParams p, int blocks_per) {
    const long long id = blockIdx.x / blocks_per;
    const int cell = (int)(blockIdx.x % blocks_per) * 256 + threadIdx.x, n = (int)(id / p.Hv), head = (int)(id % p.Hv);
    if (cell >= p.Dk * p.Dv) return;
    if (blockIdx.y == 0) join_cell<false>(p, n, head, cell);
    else join_cell<true>(p, n, head, cell);
}

// ---- outputs: one segment and head, chunk after chunk, the state in registers ----
// Wavefront w has columns 16 w .. of v: S[d][v] for all d as accumulators, which are an operand of S^T q as they stand; outputs are computed
// transposed, a lane four neighbouring v of a row.  The next chunk's rows are fetched into registers while this one is computed.
template <typename T, int DK, int DV>
struct OutLds {
    static constexpr size_t q = 0, k = Tile<T, DK>::bytes, v = k + Tile<T, DK>::bytes, pairs = v + Tile<T, DV>::bytes, sums = pairs + Tile<T, kChunk>::bytes,
                            total = sums + 4 * 64 * 4;
};
template <typename T, int DK, int DV>
__global__ __launch_bounds__(4 * DV, sizeof(T) == 2 ? (DV == 128 ? 4 : 3) : 1) void matrec_out_kernel(const MatrecParams p) {
    constexpr int W = DV / 16, KS = DK / 32, NT = DK / 16, P = Op<T>::PIECES;
    using L = OutLds<T, DK, DV>;
    using TK = Tile<T, DK>;
    using TV = Tile<T, DV>;
    using TP = Tile<T, kChunk>;
    extern __shared__ __align__(16) unsigned char lds[];
    T *tq = reinterpret_cast<T*>(lds + L::q), *tk = reinterpret_cast<T*>(lds + L::k), *tv = reinterpret_cast<T*>(lds + L::v), *tp = reinterpret_cast<T*>(lds + L::pairs);
    float* cum_hi = reinterpret_cast<float*>(lds + L::sums);
    float *cum_lo = cum_hi + 64, *since = cum_lo + 64, *until = since + 64;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, l = lane & 15;
    const int seg_no = blockIdx.x / p.Hv, head = blockIdx.x % p.Hv;
    if (seg_no >= *p.plan.count) return;
    const MatSegment seg = p.plan.segs[seg_no];
    const long long cells = (long long)p.Dk * p.Dv;
    const int kh = head / (p.Hv / p.Hk);
    const T* q = reinterpret_cast<const T*>(p.q) + (long long)kh * p.Dk + seg.row0 * p.stride_q;
    const T* k = reinterpret_cast<const T*>(p.k) + (long long)kh * p.Dk + seg.row0 * p.stride_k;
    const T* v = reinterpret_cast<const T*>(p.v) + (long long)head * p.Dv + seg.row0 * p.stride_v;
    T* o = reinterpret_cast<T*>(p.o) + (long long)head * p.Dv + seg.row0 * p.stride_o;
    const float* gate = p.gate + seg.row0 * p.Hv + head;
    const bool wide_o = four_wide(o, p.stride_o, p.Dv);
    const int vcol = 16 * wave + l;
    F32x4 S[NT];
    {
        const float* from = p.split && seg.index > 0 ? p.seg_state + ((long long)seg_no * p.Hv + head) * cells
                                                     : (p.s0 ? p.s0 + ((long long)seg.seq * p.Hv + head) * cells : nullptr);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            S[t] = F32x4{0, 0, 0, 0};
            if (from && vcol < p.Dv) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (16 * t + 4 * g + r < p.Dk) S[t][r] = from[(long long)(16 * t + 4 * g + r) * p.Dv + vcol];
            }
        }
    }
    const int chunks = (int)((seg.rows + kChunk - 1) / kChunk);
    const bool ends = seg.index == seg.count - 1;
    Stage<T, DK, 64 * W> fq, fk;
    Stage<T, DV, 64 * W> fv;
    float fg = 0.0f;
    auto fetch = [&](int c) {
        const long long row = (long long)c * kChunk;
        const int rows = seg.rows - row < kChunk ? (int)(seg.rows - row) : kChunk;
        fq.fetch(q + row * p.stride_q, p.stride_q, rows, p.Dk);
        fk.fetch(k + row * p.stride_k, p.stride_k, rows, p.Dk);
        fv.fetch(v + row * p.stride_v, p.stride_v, rows, p.Dv);
        fg = gate_of(gate + row * p.Hv, p.Hv, rows);
    };
    fetch(0);
    if (wave == 0) {   // the two tiles above the diagonal that a product of 32 terms takes in are zero and stay it
        using V4 = T __attribute__((ext_vector_type(4)));
        *reinterpret_cast<V4*>(tp + TP::four(l, 16 + 4 * g)) = V4{};
        *reinterpret_cast<V4*>(tp + TP::four(32 + l, 48 + 4 * g)) = V4{};
    }
    for (int c = 0; c < chunks; ++c) {
        const long long row = (long long)c * kChunk;
        const int rows = seg.rows - row < kChunk ? (int)(seg.rows - row) : kChunk;
        const Cum cum = chunk_cum(fg);
        const float end_hi = lane_value(cum.hi, 63), end_lo = lane_value(cum.lo, 63);
        __syncthreads();
        fq.put(tq);
        fk.put(tk);
        fv.put(tv);
        if (wave == 0) {
            cum_hi[lane] = cum.hi;
            cum_lo[lane] = cum.lo;
            since[lane] = expf(cum.hi + cum.lo);
            until[lane] = decay_between(end_hi, end_lo, cum.hi, cum.lo);
        }
        __syncthreads();
        // the factors e^{c_i - c_j} q_i . k_j, tile by tile, transposed: a lane has one i and four neighbouring j
        for (int n = wave; n < 10; n += W) {
            int ti, tj;
            lower_tile(n, ti, tj);
            const int i = 16 * ti + l, j = 16 * tj + 4 * g;
            F32x4 a = {0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < KS; ++s) a = mma(TK::row_frag(tk, 16 * tj + l, s, g), TK::row_frag(tq, i, s, g), a);
            const float hi_i = cum_hi[i], lo_i = cum_lo[i];
            const F32x4 hj = *reinterpret_cast<const F32x4*>(cum_hi + j), lj = *reinterpret_cast<const F32x4*>(cum_lo + j);
#pragma unroll
            for (int r = 0; r < 4; ++r) a[r] = j + r <= i ? a[r] * decay_between(hi_i, lo_i, hj[r], lj[r]) : 0.0f;
            store_four<T>(tp + TP::four(i, j), a, 4, true);
        }
        if (c + 1 < chunks) fetch(c + 1);
        __syncthreads();
        frag_t<T> vf[2], sf[KS];
#pragma unroll
        for (int s = 0; s < 2; ++s) vf[s] = TV::col_frag(tv, s, wave, lane);
#pragma unroll
        for (int s = 0; s < KS; ++s) sf[s] = rounded<T>(joined(S[2 * s], S[2 * s + 1]));
        F32x4 acc[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[t] = F32x4{0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int t = 0; t < 4; ++t) acc[t] = mma(sf[s], TK::row_frag(tq, 16 * t + l, s, g), acc[t]);
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[t] *= since[16 * t + l];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int t = 2 * s; t < 4; ++t) acc[t] = mma(vf[s], TP::row_frag(tp, 16 * t + l, s, g), acc[t]);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int i = 16 * t + l, v0 = 16 * wave + 4 * g;
            if (i < rows && v0 < p.Dv) store_four<T>(o + (row + i) * p.stride_o + v0, p.scale * acc[t], p.Dv - v0, wide_o);
        }
        if (c == chunks - 1 && !(ends && p.last)) break;   // the next segment's state comes from the join
        const float whole = expf(end_hi + end_lo);
#pragma unroll
        for (int t = 0; t < NT; ++t) S[t] *= whole;
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            const F32x4 w0 = *reinterpret_cast<const F32x4*>(until + 32 * s + 4 * g), w1 = *reinterpret_cast<const F32x4*>(until + 32 * s + 16 + 4 * g);
            frag_t<T> vp[P];
            pieces_of<T>(widened(vf[s]) * joined(w0, w1), vp);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const frag_t<T> kf = TK::col_frag(tk, s, t, lane);
#pragma unroll
                for (int q2 = P - 1; q2 >= 0; --q2) S[t] = mma(kf, vp[q2], S[t]);
            }
        }
    }
    if (ends && p.last && vcol < p.Dv) {
        float* to = p.last + ((long long)seg.seq * p.Hv + head) * cells;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (16 * t + 4 * g + r < p.Dk) to[(long long)(16 * t + 4 * g + r) * p.Dv + vcol] = S[t][r];
    }
}

// ---- one token ----
// Memory bound: the state, fp32, is read and written once.  A workgroup has one row and head; a lane V columns of some rows of the state.
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
    if (slot < 0 || slot >= p.rows.n_slots || twice) return;
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

template <typename K>
hipError_t launch_lds(K kernel, dim3 grid, int threads, size_t lds, const MatrecParams& p, hipStream_t stream) {
    if (grid.x == 0) return hipSuccess;
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, grid, dim3(threads), lds, stream, p);
    return hipGetLastError();
}

// the segments' own parts, and the join; `both`: of the states and of their gradients
template <typename T, int DK, int DV>
hipError_t join_shape(const MatrecParams& p, int both, hipStream_t stream) {
    constexpr size_t lds = Tile<T, DK>::bytes + Tile<T, DV>::bytes + 4 * 64;
    hipError_t e = hipSuccess;
    if (p.split) e = launch_lds(matrec_states_kernel<T, DK, DV, false>, dim3((unsigned)((long long)p.plan.max_segs * p.Hv), 1 + both), 4 * DV, lds, p, stream);
    if (e != hipSuccess || !(p.split || p.rows.bounds || p.rows.T == 0)) return e;
    const int per = (p.Dk * p.Dv + 255) / 256;
    hipLaunchKernelGGL(matrec_join_kernel, dim3((unsigned)((long long)p.rows.N * p.Hv * per), 1 + both), dim3(256), 0, stream, p, per);
    return hipGetLastError();
}
template <typename T, int DK, int DV>
hipError_t out_shape(const MatrecParams& p, hipStream_t stream) {
    const hipError_t e = join_shape<T, DK, DV>(p, 0, stream);
    if (e != hipSuccess) return e;
    return launch_lds(matrec_out_kernel<T, DK, DV>, dim3((unsigned)((long long)p.plan.max_segs * p.Hv)), 4 * DV, OutLds<T, DK, DV>::total, p, stream);
}
template <typename T, int DK, int DV>
hipError_t states_shape(const MatrecParams& p, hipStream_t stream) {
    constexpr size_t lds = Tile<T, DK>::bytes + Tile<T, DV>::bytes + 4 * 64;
    const hipError_t e = join_shape<T, DK, DV>(p, 1, stream);
    if (e != hipSuccess) return e;
    return launch_lds(matrec_states_kernel<T, DK, DV, true>, dim3((unsigned)((long long)p.plan.max_segs * p.Hv), 2), 4 * DV, lds, p, stream);
}
#define DEER_BY_SHAPE(F, T, p, stream)                                                                        \
    ((p).Dk <= 64 ? ((p).Dv <= 64 ? F<T, 64, 64>(p, stream) : F<T, 64, 128>(p, stream)) : ((p).Dv <= 64 ? F<T, 128, 64>(p, stream) : F<T, 128, 128>(p, stream)))

}  // namespace

hipError_t launch_matrec_plan(const MatrecParams& p, hipStream_t stream) {
    hipLaunchKernelGGL(matrec_plan_kernel, dim3(1), dim3(1024), 0, stream, p);
    return hipGetLastError();
}
hipError_t launch_matrec_out(int dtype, const MatrecParams& p, hipStream_t stream) {
    return dtype == DEER_BF16 ? DEER_BY_SHAPE(out_shape, BF16, p, stream) : DEER_BY_SHAPE(out_shape, float, p, stream);
}
hipError_t launch_matrec_states(int dtype, const MatrecParams& p, hipStream_t stream) {
    return dtype == DEER_BF16 ? DEER_BY_SHAPE(states_shape, BF16, p, stream) : DEER_BY_SHAPE(states_shape, float, p, stream);
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
