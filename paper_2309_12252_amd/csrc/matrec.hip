// Gated linear recurrence with a matrix as state: S_t = e^{g_t} S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t; by chunks of 64 rows on the matrix
// cores.  With c_i the sum of a chunk's log gates up to row i, inclusive, and S the state in front of the chunk,
//   o_i = scale (e^{c_i} S^T q_i + sum_{j <= i} e^{c_i - c_j} (q_i . k_j) v_j)
//   S'  = e^{c_64} S + sum_j e^{c_64 - c_j} k_j v_j^T.
// States are sums over many rows and stay in fp32 accumulators; v_j e^{c_64 - c_j} enters their update as two bf16 pieces, so a state is as exact as
// fp32 sums make it (7e-7 measured).  The products of the output take S and the 64 x 64 factors rounded to bf16 once: an output
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
// S[d][v] of a workgroup: wavefront w has columns 16 VT w .. of v and all rows d, as accumulators
template <int KD, int VT>
struct StateTile {
    F32x4 s[4 * KD][VT];
    __device__ __forceinline__ void zero() {
#pragma unroll
        for (int t = 0; t < 4 * KD; ++t)
#pragma unroll
            for (int u = 0; u < VT; ++u) s[t][u] = F32x4{0, 0, 0, 0};
    }
    __device__ __forceinline__ void scale(float f) {
#pragma unroll
        for (int t = 0; t < 4 * KD; ++t)
#pragma unroll
            for (int u = 0; u < VT; ++u) s[t][u] *= f;
    }
    template <typename F>
    __device__ __forceinline__ void each(int wave, int lane, int Dk, int Dv, F f) {
#pragma unroll
        for (int t = 0; t < 4 * KD; ++t)
#pragma unroll
            for (int u = 0; u < VT; ++u)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int d = 16 * t + 4 * (lane >> 4) + r, v = 16 * (VT * wave + u) + (lane & 15);
                    if (d < Dk && v < Dv) s[t][u][r] = f(d * Dv + v, (float)s[t][u][r]);
                }
    }
    __device__ __forceinline__ void load(const float* from, int wave, int lane, int Dk, int Dv) {
        zero();
        if (from) each(wave, lane, Dk, Dv, [&](int at, float) { return from[at]; });
    }
    __device__ __forceinline__ void store(float* to, int wave, int lane, int Dk, int Dv) {
        each(wave, lane, Dk, Dv, [&](int at, float x) {
            to[at] = x;
            return x;
        });
    }
};

// S += K^T (weight V) over the 64 rows of a chunk; `weight` holds the rows' factors in LDS
template <typename T, int KD, int VT, int LDK, int LDV>
__device__ __forceinline__ void update_state(StateTile<KD, VT>& S, const T* tk, const T* tv, const float* weight, int wave, int lane) {
    const int g = lane >> 4;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
        const F32x4 w0 = *reinterpret_cast<const F32x4*>(weight + 32 * s + 4 * g), w1 = *reinterpret_cast<const F32x4*>(weight + 32 * s + 16 + 4 * g);
        frag_t<T> vp[VT][Op<T>::PIECES];
#pragma unroll
        for (int u = 0; u < VT; ++u) pieces_of<T>(widened(col_frag<LDV>(tv, s, VT * wave + u, lane)) * joined(w0, w1), vp[u]);
#pragma unroll
        for (int t = 0; t < 4 * KD; ++t) {
            const frag_t<T> kf = col_frag<LDK>(tk, s, t, lane);
#pragma unroll
            for (int u = 0; u < VT; ++u)
#pragma unroll
                for (int q = Op<T>::PIECES - 1; q >= 0; --q) S.s[t][u] = mma(kf, vp[u][q], S.s[t][u]);
        }
    }
}

// One segment and head: the state's own part of the segment (STORE = false: into seg_state / seg_rstate, with the segment's decay), or with the state in
// front of the segment known, the state in front of every chunk (REV: the gradient of the state behind it).  REV: rows backwards,
// (k, v) = (scale q, dout), the gradient of the state in front of a chunk is e^{c_64} R + sum_i e^{c_i} scale q_i dout_i^T.
template <typename T, int KD, int VT, bool REV, bool STORE>
__device__ __forceinline__ void states_of(const MatrecParams& p, int seg_no, int head, T* tk, T* tv, float* weight) {
    constexpr int LDK = 64 * KD + Op<T>::PAD, LDV = 64 * VT + Op<T>::PAD;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const MatSegment seg = p.plan.segs[seg_no];
    if (!STORE && seg.index == (REV ? 0 : seg.count - 1)) return;   // nothing comes behind it
    const long long cells = (long long)p.Dk * p.Dv;
    const int kh = head / (p.Hv / p.Hk);
    const long long stride_k = REV ? p.stride_q : p.stride_k, stride_v = REV ? p.stride_o : p.stride_v;
    const T* k = reinterpret_cast<const T*>(REV ? p.q : p.k) + (long long)kh * p.Dk;
    const T* v = reinterpret_cast<const T*>(REV ? p.dout : p.v) + (long long)head * p.Dv;
    float* seg_states = REV ? p.seg_rstate : p.seg_state;
    StateTile<KD, VT> S;
    if (STORE) {
        const float* ends = REV ? p.dlast : p.s0;
        const bool at_end = seg.index == (REV ? seg.count - 1 : 0);
        const float* from = at_end ? (ends ? ends + ((long long)seg.seq * p.Hv + head) * cells : nullptr) : seg_states + ((long long)seg_no * p.Hv + head) * cells;
        S.load(from, wave, lane, p.Dk, p.Dv);
    } else {
        S.zero();
    }
    const int chunks = (int)((seg.rows + kChunk - 1) / kChunk);
    double total = 0.0;
    for (int i = 0; i < chunks; ++i) {
        const int c = REV ? chunks - 1 - i : i;
        const long long row = seg.row0 + (long long)c * kChunk;
        const int rows = seg.rows - (long long)c * kChunk < kChunk ? (int)(seg.rows - (long long)c * kChunk) : kChunk;
        if (STORE) {
            float* to = (REV ? p.chunk_rstate : p.chunk_state) + ((long long)(seg.chunk0 + c) * p.Hv + head) * cells;
            S.store(to, wave, lane, p.Dk, p.Dv);
            if (!REV && i == chunks - 1) break;
        }
        const Cum cum = chunk_cum(p.gate + row * p.Hv + head, p.Hv, rows, lane);
        const float end_hi = lane_value(cum.hi, 63), end_lo = lane_value(cum.lo, 63);
        __syncthreads();
        load_tile<T, LDK>(tk, k + row * stride_k, stride_k, rows, p.Dk);
        load_tile<T, LDV>(tv, v + row * stride_v, stride_v, rows, p.Dv);
        if (wave == 0) weight[lane] = REV ? p.scale * expf(cum.hi + cum.lo) : decay_between(end_hi, end_lo, cum.hi, cum.lo);
        __syncthreads();
        S.scale(expf(end_hi + end_lo));
        total += (double)end_hi + (double)end_lo;
        update_state<T, KD, VT, LDK, LDV>(S, tk, tv, weight, wave, lane);
    }
    if (STORE) {
        if (REV && seg.index == 0 && p.ds0) S.store(p.ds0 + ((long long)seg.seq * p.Hv + head) * cells, wave, lane, p.Dk, p.Dv);
    } else {
        S.store(seg_states + ((long long)seg_no * p.Hv + head) * cells, wave, lane, p.Dk, p.Dv);
        if (threadIdx.x == 0) p.seg_decay[(REV ? (long long)p.plan.max_segs * p.Hv : 0) + (long long)seg_no * p.Hv + head] = (float)exp(total);
    }
}

// blockIdx.y: 0 the states, 1 their gradients
template <typename T, int KD, int VT, bool STORE>
__global__ __launch_bounds__(64 * kWaves) void matrec_states_kernel(const MatrecParams p) {
    extern __shared__ __align__(16) unsigned char lds[];
    T* tk = reinterpret_cast<T*>(lds);
    T* tv = tk + kChunk * (64 * KD + Op<T>::PAD);
    float* weight = reinterpret_cast<float*>(tv + kChunk * (64 * VT + Op<T>::PAD));
    const int seg = blockIdx.x / p.Hv, head = blockIdx.x % p.Hv;
    if (seg >= *p.plan.count) return;
    if (blockIdx.y == 0) states_of<T, KD, VT, false, STORE>(p, seg, head, tk, tv, weight);
    else states_of<T, KD, VT, true, STORE>(p, seg, head, tk, tv, weight);
}

// The segments' own parts joined along a sequence, in their order: seg_state becomes the state in front of each segment (REV: seg_rstate the gradient
// of the state behind it).  A lane has one cell.  Also what a sequence without rows has in the place of a final state (REV: of ds0).
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
    for (int i = 0; i < count; ++i) {
        const long long seg = first + (REV ? count - 1 - i : i), cellat = (seg * p.Hv + head) * cells + cell;
        const float own = states[cellat];   // (of the last one along the way: not written, not used)
        states[cellat] = s;
        s = decay[seg * p.Hv + head] * s + own;
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
template <typename T, int KD, int VT>
__global__ __launch_bounds__(64 * kWaves) void matrec_out_kernel(const MatrecParams p) {
    constexpr int LDK = 64 * KD + Op<T>::PAD, LDV = 64 * VT + Op<T>::PAD, LDP = kChunk + Op<T>::PAD, KS = 2 * KD;
    extern __shared__ __align__(16) unsigned char lds[];
    T* tq = reinterpret_cast<T*>(lds);
    T* tk = tq + kChunk * LDK;
    T* tv = tk + kChunk * LDK;
    T* tp = tv + kChunk * LDV;
    float* cum_hi = reinterpret_cast<float*>(tp + kChunk * LDP);
    float *cum_lo = cum_hi + 64, *since = cum_lo + 64, *until = since + 64;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, l = lane & 15;
    const int seg_no = blockIdx.x / p.Hv, head = blockIdx.x % p.Hv;
    if (seg_no >= *p.plan.count) return;
    const MatSegment seg = p.plan.segs[seg_no];
    const long long cells = (long long)p.Dk * p.Dv;
    const int kh = head / (p.Hv / p.Hk);
    const T* q = reinterpret_cast<const T*>(p.q) + (long long)kh * p.Dk;
    const T* k = reinterpret_cast<const T*>(p.k) + (long long)kh * p.Dk;
    const T* v = reinterpret_cast<const T*>(p.v) + (long long)head * p.Dv;
    T* o = reinterpret_cast<T*>(p.o) + (long long)head * p.Dv;
    StateTile<KD, VT> S;
    const float* from = p.split && seg.index > 0 ? p.seg_state + ((long long)seg_no * p.Hv + head) * cells
                                                 : (p.s0 ? p.s0 + ((long long)seg.seq * p.Hv + head) * cells : nullptr);
    S.load(from, wave, lane, p.Dk, p.Dv);
    const int chunks = (int)((seg.rows + kChunk - 1) / kChunk);
    const bool ends = seg.index == seg.count - 1;
    for (int c = 0; c < chunks; ++c) {
        const long long row = seg.row0 + (long long)c * kChunk;
        const int rows = seg.rows - (long long)c * kChunk < kChunk ? (int)(seg.rows - (long long)c * kChunk) : kChunk;
        const Cum cum = chunk_cum(p.gate + row * p.Hv + head, p.Hv, rows, lane);
        const float end_hi = lane_value(cum.hi, 63), end_lo = lane_value(cum.lo, 63);
        __syncthreads();
        load_tile<T, LDK>(tq, q + row * p.stride_q, p.stride_q, rows, p.Dk);
        load_tile<T, LDK>(tk, k + row * p.stride_k, p.stride_k, rows, p.Dk);
        load_tile<T, LDV>(tv, v + row * p.stride_v, p.stride_v, rows, p.Dv);
        if (wave == 0) {
            cum_hi[lane] = cum.hi;
            cum_lo[lane] = cum.lo;
            since[lane] = expf(cum.hi + cum.lo);
            until[lane] = decay_between(end_hi, end_lo, cum.hi, cum.lo);
        }
        __syncthreads();
        // this wavefront's 16 rows i of the factors e^{c_i - c_j} q_i . k_j, as their transpose: a lane has one i and four neighbouring j
        {
            const int i = 16 * wave + l;
            frag_t<T> qf[KS];
#pragma unroll
            for (int s = 0; s < KS; ++s) qf[s] = row_frag<T, LDK>(tq, i, s, g);
            const float hi_i = cum_hi[i], lo_i = cum_lo[i];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if (t > (wave | 1)) break;
                T f[4];
                if (t <= wave) {
                    F32x4 a = {0, 0, 0, 0};
#pragma unroll
                    for (int s = 0; s < KS; ++s) a = mma(row_frag<T, LDK>(tk, 16 * t + l, s, g), qf[s], a);
                    const F32x4 hj = *reinterpret_cast<const F32x4*>(cum_hi + 16 * t + 4 * g), lj = *reinterpret_cast<const F32x4*>(cum_lo + 16 * t + 4 * g);
#pragma unroll
                    for (int r = 0; r < 4; ++r) f[r] = 16 * t + 4 * g + r <= i ? (T)(a[r] * decay_between(hi_i, lo_i, hj[r], lj[r])) : T(0);
                } else {
#pragma unroll
                    for (int r = 0; r < 4; ++r) f[r] = T(0);
                }
                T* to = tp + i * LDP + place(16 * t + 4 * g);
#pragma unroll
                for (int r = 0; r < 4; ++r) to[r] = f[r];
            }
        }
        __syncthreads();
        frag_t<T> vf[2][VT];
#pragma unroll
        for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int u = 0; u < VT; ++u) vf[s][u] = col_frag<LDV>(tv, s, VT * wave + u, lane);
        frag_t<T> sf[KS][VT];
#pragma unroll
        for (int s = 0; s < KS; ++s)
#pragma unroll
            for (int u = 0; u < VT; ++u) sf[s][u] = rounded<T>(joined(S.s[2 * s][u], S.s[2 * s + 1][u]));
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            F32x4 acc[VT];
#pragma unroll
            for (int u = 0; u < VT; ++u) acc[u] = F32x4{0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const frag_t<T> qf = row_frag<T, LDK>(tq, 16 * t + l, s, g);
#pragma unroll
                for (int u = 0; u < VT; ++u) acc[u] = mma(qf, sf[s][u], acc[u]);
            }
            const F32x4 f = *reinterpret_cast<const F32x4*>(since + 16 * t + 4 * g);
#pragma unroll
            for (int u = 0; u < VT; ++u) acc[u] *= f;
#pragma unroll
            for (int s = 0; s <= t / 2; ++s) {
                const frag_t<T> pf = row_frag<T, LDP>(tp, 16 * t + l, s, g);
#pragma unroll
                for (int u = 0; u < VT; ++u) acc[u] = mma(pf, vf[s][u], acc[u]);
            }
#pragma unroll
            for (int u = 0; u < VT; ++u) {
                const int col = 16 * (VT * wave + u) + l;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 16 * t + 4 * g + r;
                    if (i < rows && col < p.Dv) o[(row + i) * p.stride_o + col] = (T)(p.scale * acc[u][r]);
                }
            }
        }
        if (ends && c == chunks - 1 && !p.last) break;
        if (!ends && c == chunks - 1) break;   // the next segment's state comes from the join
        S.scale(expf(end_hi + end_lo));
        update_state<T, KD, VT, LDK, LDV>(S, tk, tv, until, wave, lane);
    }
    if (ends && p.last) S.store(p.last + ((long long)seg.seq * p.Hv + head) * cells, wave, lane, p.Dk, p.Dv);
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

template <typename T, int KD, int VT>
constexpr size_t states_lds() { return sizeof(T) * kChunk * (64 * KD + 64 * VT + 2 * Op<T>::PAD) + 4 * 64; }
template <typename T, int KD, int VT>
constexpr size_t out_lds() { return sizeof(T) * kChunk * (128 * KD + 64 * VT + 64 + 4 * Op<T>::PAD) + 4 * 64 * 4; }

template <typename K>
hipError_t launch_lds(K kernel, dim3 grid, size_t lds, const MatrecParams& p, hipStream_t stream) {
    if (grid.x == 0) return hipSuccess;
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, grid, dim3(64 * kWaves), lds, stream, p);
    return hipGetLastError();
}

template <typename T, int KD, int VT>
hipError_t out_shape(const MatrecParams& p, hipStream_t stream) {
    const unsigned grid = (unsigned)((long long)p.plan.max_segs * p.Hv);
    hipError_t e = hipSuccess;
    if (p.split) e = launch_lds(matrec_states_kernel<T, KD, VT, false>, dim3(grid, 1), states_lds<T, KD, VT>(), p, stream);
    if (e != hipSuccess) return e;
    if (p.split || p.rows.bounds || p.rows.T == 0) {
        const int per = (p.Dk * p.Dv + 255) / 256;
        hipLaunchKernelGGL(matrec_join_kernel, dim3((unsigned)((long long)p.rows.N * p.Hv * per), 1), dim3(256), 0, stream, p, per);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    return launch_lds(matrec_out_kernel<T, KD, VT>, dim3(grid), out_lds<T, KD, VT>(), p, stream);
}
template <typename T, int KD, int VT>
hipError_t states_shape(const MatrecParams& p, hipStream_t stream) {
    const unsigned grid = (unsigned)((long long)p.plan.max_segs * p.Hv);
    hipError_t e = hipSuccess;
    if (p.split) e = launch_lds(matrec_states_kernel<T, KD, VT, false>, dim3(grid, 2), states_lds<T, KD, VT>(), p, stream);
    if (e != hipSuccess) return e;
    if (p.split || p.rows.bounds || p.rows.T == 0) {
        const int per = (p.Dk * p.Dv + 255) / 256;
        hipLaunchKernelGGL(matrec_join_kernel, dim3((unsigned)((long long)p.rows.N * p.Hv * per), 2), dim3(256), 0, stream, p, per);
        if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    return launch_lds(matrec_states_kernel<T, KD, VT, true>, dim3(grid, 2), states_lds<T, KD, VT>(), p, stream);
}
#define DEER_BY_SHAPE(F, T, p, stream) \
    ((p).Dk <= 64 ? ((p).Dv <= 64 ? F<T, 1, 1>(p, stream) : F<T, 1, 2>(p, stream)) : ((p).Dv <= 64 ? F<T, 2, 1>(p, stream) : F<T, 2, 2>(p, stream)))

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
