// Gradient of the matrix-state recurrence, chunk by chunk side by side.  In front of every chunk lies the state S, behind it the gradient R of
// the state there (launch_matrec_states); with A_ij = q_i . k_j, B_ij = dout_i . v_j and E_ij = scale e^{c_i - c_j} for j <= i, else 0,
//   dq_i = sum_j E_ij B_ij k_j + scale e^{c_i} S dout_i        dk_j = sum_i E_ij B_ij q_i + e^{c_64 - c_j} R v_j
//   dv_j = sum_i E_ij A_ij dout_i + e^{c_64 - c_j} R^T k_j
// and the gradient of a log gate, e^{g_t} <S_{t-1}, dS_t>, is the sum over everything that passes row t: pairs i >= t > j inside
// the chunk, what comes from S and is read at i >= t, what j < t adds and R takes on, and what goes through from S to R:
//   dgate_t = sum_{i >= t > j} E_ij A_ij B_ij + sum_{i >= t} q_i . (scale e^{c_i} S dout_i) + sum_{j < t} k_j . (e^{c_64 - c_j} R v_j) + e^{c_64} <S, R>,
// each of them a sum of what belongs to it alone, so that a strong gate's small gradient is no difference of large numbers.  The pairs: running
// sums over j along every row i, of which t takes those of the rows i >= t at j = t - 1.  A and B are exact products of the inputs, S and R enter dgate's products as two bf16 pieces.
// Heads of v that share one of q and k are gone through one after another, their dq and dk added in registers, always in the same order.
#include "matrec_common.h"

namespace deer {
namespace {

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

// eight terms of S (rows of Dv columns in memory, fp32), the block of 32 columns s of row d; zero outside
__device__ __forceinline__ F32x8 state_row(const float* S, int d, int s, int g, int Dk, int Dv) {
    F32x8 x = {0, 0, 0, 0, 0, 0, 0, 0};
    const int c0 = 32 * s + 4 * g;
    if (d >= Dk) return x;
    const float* at = S + (long long)d * Dv + c0;
    if ((Dv & 3) == 0) {   // rows 16 bytes aligned, as the states' array is
        if (c0 < Dv) {
            const F32x4 v = *reinterpret_cast<const F32x4*>(at);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[e] = v[e];
        }
        if (c0 + 16 < Dv) {
            const F32x4 v = *reinterpret_cast<const F32x4*>(at + 16);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[4 + e] = v[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const int c = (e & 3) + (e >= 4 ? 16 : 0);
            if (c0 + c < Dv) x[e] = at[c];
        }
    }
    return x;
}
// column v of S, the block of 32 rows s
__device__ __forceinline__ F32x8 state_col(const float* S, int v, int s, int g, int Dk, int Dv) {
    F32x8 x = {0, 0, 0, 0, 0, 0, 0, 0};
    if (v >= Dv) return x;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const int d = 32 * s + 4 * g + (e & 3) + (e >= 4 ? 16 : 0);
        if (d < Dk) x[e] = S[(long long)d * Dv + v];
    }
    return x;
}

template <typename T, int KD, int VT>
__global__ __launch_bounds__(64 * kWaves) void matrec_grad_kernel(const MatrecParams p) {
    constexpr int LDK = 64 * KD + Op<T>::PAD, LDV = 64 * VT + Op<T>::PAD, LDP = kChunk + Op<T>::PAD, KS = 2 * KD, VS = 2 * VT, P = Op<T>::PIECES;
    extern __shared__ __align__(16) unsigned char lds[];
    T* tq = reinterpret_cast<T*>(lds);
    T* tk = tq + kChunk * LDK;
    T* tv = tk + kChunk * LDK;
    T* td = tv + kChunk * LDV;
    T* tp = td + kChunk * LDV;
    float* cum_hi = reinterpret_cast<float*>(tp + kChunk * LDP);
    float *cum_lo = cum_hi + 64, *since = cum_lo + 64, *until = since + 64;
    float* sum_in = until + 64;          // [4][64]: q_i . (...) by wavefront
    float* sum_out = sum_in + 256;       // [4][64]
    float* sum_pairs = sum_out + 256;    // [4][64]: at j what passes row j + 1
    float* sum_through = sum_pairs + 256;   // [4]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, l = lane & 15;
    const int kh = blockIdx.x % p.Hk, chunk_no = (int)(blockIdx.x / p.Hk), seg_no = chunk_no / p.plan.per, c = chunk_no % p.plan.per;
    if (seg_no >= *p.plan.count) return;
    const MatSegment seg = p.plan.segs[seg_no];
    const long long left = seg.rows - (long long)c * kChunk;
    if (left <= 0) return;
    const int rows = left < kChunk ? (int)left : kChunk, group = p.Hv / p.Hk;
    const long long row = seg.row0 + (long long)c * kChunk, cells = (long long)p.Dk * p.Dv;

    F32x4 dq[4][KD], dk[4][KD];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int u = 0; u < KD; ++u) dq[t][u] = dk[t][u] = F32x4{0, 0, 0, 0};
    load_tile<T, LDK>(tq, reinterpret_cast<const T*>(p.q) + row * p.stride_q + (long long)kh * p.Dk, p.stride_q, rows, p.Dk);
    load_tile<T, LDK>(tk, reinterpret_cast<const T*>(p.k) + row * p.stride_k + (long long)kh * p.Dk, p.stride_k, rows, p.Dk);

    for (int member = 0; member < group; ++member) {
        const int head = kh * group + member;
        const Cum cum = chunk_cum(p.gate + row * p.Hv + head, p.Hv, rows, lane);
        const float end_hi = lane_value(cum.hi, 63), end_lo = lane_value(cum.lo, 63), whole = expf(end_hi + end_lo);
        load_tile<T, LDV>(tv, reinterpret_cast<const T*>(p.v) + row * p.stride_v + (long long)head * p.Dv, p.stride_v, rows, p.Dv);
        load_tile<T, LDV>(td, reinterpret_cast<const T*>(p.dout) + row * p.stride_o + (long long)head * p.Dv, p.stride_o, rows, p.Dv);
        if (wave == 0) {
            cum_hi[lane] = cum.hi;
            cum_lo[lane] = cum.lo;
            since[lane] = p.scale * expf(cum.hi + cum.lo);
            until[lane] = decay_between(end_hi, end_lo, cum.hi, cum.lo);
        }
        __syncthreads();
        const float* S = p.chunk_state + ((long long)(seg.chunk0 + c) * p.Hv + head) * cells;
        const float* R = p.chunk_rstate + ((long long)(seg.chunk0 + c) * p.Hv + head) * cells;

        // ---- the pairs: rows i of this wavefront, as transposes: a lane has one i and four neighbouring j of every tile ----
        F32x4 ea[4];   // E_ij A_ij, for later
        {
            const int i = 16 * wave + l;
            frag_t<T> qf[KS], df[VS];
#pragma unroll
            for (int s = 0; s < KS; ++s) qf[s] = row_frag<T, LDK>(tq, i, s, g);
#pragma unroll
            for (int s = 0; s < VS; ++s) df[s] = row_frag<T, LDV>(td, i, s, g);
            const float hi_i = cum_hi[i], lo_i = cum_lo[i];
            float run = 0.0f;   // sum of the row's pairs in the tiles so far
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                F32x4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
                F32x4 upto = {0, 0, 0, 0};
                if (t <= wave) {
#pragma unroll
                    for (int s = 0; s < KS; ++s) a = mma(row_frag<T, LDK>(tk, 16 * t + l, s, g), qf[s], a);
#pragma unroll
                    for (int s = 0; s < VS; ++s) b = mma(row_frag<T, LDV>(tv, 16 * t + l, s, g), df[s], b);
                    const F32x4 hj = *reinterpret_cast<const F32x4*>(cum_hi + 16 * t + 4 * g), lj = *reinterpret_cast<const F32x4*>(cum_lo + 16 * t + 4 * g);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        const int j = 16 * t + 4 * g + r;
                        const float e = j <= i ? p.scale * decay_between(hi_i, lo_i, hj[r], lj[r]) : 0.0f;
                        upto[r] = (r > 0 ? upto[r > 0 ? r - 1 : 0] : 0.0f) + (j < i ? e * a[r] * b[r] : 0.0f);
                        a[r] = j <= i ? e * a[r] : 0.0f;
                        b[r] = j <= i ? e * b[r] : 0.0f;
                    }
                    // the lane groups in front of this one have the smaller j
                    float front = upto[3];   // this group's and those of the groups in front
                    const float one = __shfl_up(front, 16);
                    front += g >= 1 ? one : 0.0f;
                    const float two = __shfl_up(front, 32);
                    front += g >= 2 ? two : 0.0f;
                    const float before = __shfl_up(front, 16);
                    const float offset = run + (g >= 1 ? before : 0.0f);
                    run += __shfl(front, 48 + l);
#pragma unroll
                    for (int r = 0; r < 4; ++r) upto[r] = 16 * t + 4 * g + r < i ? upto[r] + offset : 0.0f;
                }
                ea[t] = a;
                T* to = tp + i * LDP + place(16 * t + 4 * g);
#pragma unroll
                for (int r = 0; r < 4; ++r) to[r] = (T)b[r];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float s = group_sum(upto[r]);
                    if (l == 0) sum_pairs[64 * wave + 16 * t + 4 * g + r] = s;
                }
            }
        }
        __syncthreads();

        // ---- dq and dk: this wavefront's columns d ----
        {
            float through = 0.0f;
            frag_t<T> sf[VS][KD][P], rf[VS][KD][P];
#pragma unroll
            for (int s = 0; s < VS; ++s)
#pragma unroll
                for (int u = 0; u < KD; ++u) {
                    const int d = 16 * (KD * wave + u) + l;
                    const F32x8 x = state_row(S, d, s, g, p.Dk, p.Dv), y = state_row(R, d, s, g, p.Dk, p.Dv);
#pragma unroll
                    for (int e = 0; e < 8; ++e) through += x[e] * y[e];
                    pieces_of<T>(x, sf[s][u]);
                    pieces_of<T>(y, rf[s][u]);
                }
            through += __shfl_xor(through, 16);
            through += __shfl_xor(through, 32);
            through = group_sum(through);
            if (lane == 0) sum_through[wave] = through;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                F32x4 in[KD], out[KD];
#pragma unroll
                for (int u = 0; u < KD; ++u) in[u] = out[u] = F32x4{0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < VS; ++s) {
                    const frag_t<T> df = row_frag<T, LDV>(td, 16 * t + l, s, g), vf = row_frag<T, LDV>(tv, 16 * t + l, s, g);
#pragma unroll
                    for (int u = 0; u < KD; ++u)
#pragma unroll
                        for (int q = P - 1; q >= 0; --q) {
                            in[u] = mma(df, sf[s][u][q], in[u]);
                            out[u] = mma(vf, rf[s][u][q], out[u]);
                        }
                }
                const F32x4 fi = *reinterpret_cast<const F32x4*>(since + 16 * t + 4 * g), fo = *reinterpret_cast<const F32x4*>(until + 16 * t + 4 * g);
                F32x4 dot_in = {0, 0, 0, 0}, dot_out = {0, 0, 0, 0};
#pragma unroll
                for (int u = 0; u < KD; ++u) {
                    in[u] *= fi;
                    out[u] *= fo;
                    const int col = place(16 * (KD * wave + u) + l);
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        dot_in[r] += (float)tq[(16 * t + 4 * g + r) * LDK + col] * in[u][r];
                        dot_out[r] += (float)tk[(16 * t + 4 * g + r) * LDK + col] * out[u][r];
                    }
                    dq[t][u] += in[u];
                    dk[t][u] += out[u];
                }
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float x = group_sum(dot_in[r]), y = group_sum(dot_out[r]);
                    if (l == 0) {
                        sum_in[64 * wave + 16 * t + 4 * g + r] = x;
                        sum_out[64 * wave + 16 * t + 4 * g + r] = y;
                    }
                }
            }
            // inside the chunk
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                frag_t<T> kf[KD], qf[KD];
#pragma unroll
                for (int u = 0; u < KD; ++u) {
                    kf[u] = col_frag<LDK>(tk, s, KD * wave + u, lane);
                    qf[u] = col_frag<LDK>(tq, s, KD * wave + u, lane);
                }
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    if (s <= t / 2) {   // rows i of tile t take the columns j of the block s
                        const frag_t<T> pf = row_frag<T, LDP>(tp, 16 * t + l, s, g);
#pragma unroll
                        for (int u = 0; u < KD; ++u) dq[t][u] = mma(pf, kf[u], dq[t][u]);
                    }
                    if (s >= t / 2) {   // columns j of tile t take the rows i of the block s
                        const frag_t<T> pf = col_frag<LDP>(tp, s, t, lane);
#pragma unroll
                        for (int u = 0; u < KD; ++u) dk[t][u] = mma(pf, qf[u], dk[t][u]);
                    }
                }
            }
        }
        __syncthreads();

        // ---- dv: this wavefront's columns v; and the gates ----
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            T* to = tp + (16 * wave + l) * LDP + place(16 * t + 4 * g);
#pragma unroll
            for (int r = 0; r < 4; ++r) to[r] = (T)ea[t][r];
        }
        if (wave == 0 && p.dgate) {
            // a lane has row t: sums from t on of what is read there, sums in front of t of what is added there
            float later = 0.0f, earlier = 0.0f, pairs = 0.0f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                later += sum_in[64 * w + lane];
                earlier += sum_out[64 * w + lane];
                pairs += lane > 0 ? sum_pairs[64 * w + lane - 1] : 0.0f;
            }
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const float a = __shfl_down(later, d), b = __shfl_up(earlier, d);
                later += lane + d < 64 ? a : 0.0f;
                earlier += lane >= d ? b : 0.0f;
            }
            earlier = __shfl_up(earlier, 1);
            if (lane == 0) earlier = 0.0f;
            const float through = whole * (sum_through[0] + sum_through[1] + sum_through[2] + sum_through[3]);
            if (lane < rows) p.dgate[(row + lane) * p.Hv + head] = pairs + later + earlier + through;
        }
        F32x4 dv[4][VT];
        {
            frag_t<T> rc[KS][VT];
#pragma unroll
            for (int s = 0; s < KS; ++s)
#pragma unroll
                for (int u = 0; u < VT; ++u) rc[s][u] = rounded<T>(state_col(R, 16 * (VT * wave + u) + l, s, g, p.Dk, p.Dv));
#pragma unroll
            for (int t = 0; t < 4; ++t) {
#pragma unroll
                for (int u = 0; u < VT; ++u) dv[t][u] = F32x4{0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const frag_t<T> kf = row_frag<T, LDK>(tk, 16 * t + l, s, g);
#pragma unroll
                    for (int u = 0; u < VT; ++u) dv[t][u] = mma(kf, rc[s][u], dv[t][u]);
                }
                const F32x4 fo = *reinterpret_cast<const F32x4*>(until + 16 * t + 4 * g);
#pragma unroll
                for (int u = 0; u < VT; ++u) dv[t][u] *= fo;
            }
        }
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 2; ++s) {
            frag_t<T> df[VT];
#pragma unroll
            for (int u = 0; u < VT; ++u) df[u] = col_frag<LDV>(td, s, VT * wave + u, lane);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if (s >= t / 2) {
                    const frag_t<T> pf = col_frag<LDP>(tp, s, t, lane);
#pragma unroll
                    for (int u = 0; u < VT; ++u) dv[t][u] = mma(pf, df[u], dv[t][u]);
                }
            }
        }
        T* dvp = reinterpret_cast<T*>(p.dv) + (long long)head * p.Dv;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int u = 0; u < VT; ++u) {
                const int col = 16 * (VT * wave + u) + l;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int j = 16 * t + 4 * g + r;
                    if (j < rows && col < p.Dv) dvp[(row + j) * p.stride_v + col] = (T)dv[t][u][r];
                }
            }
        __syncthreads();   // the next head's tiles come over these
    }
    T *dqp = reinterpret_cast<T*>(p.dq) + (long long)kh * p.Dk, *dkp = reinterpret_cast<T*>(p.dk) + (long long)kh * p.Dk;
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int u = 0; u < KD; ++u) {
            const int col = 16 * (KD * wave + u) + l;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int i = 16 * t + 4 * g + r;
                if (i < rows && col < p.Dk) {
                    dqp[(row + i) * p.stride_q + col] = (T)dq[t][u][r];
                    dkp[(row + i) * p.stride_k + col] = (T)dk[t][u][r];
                }
            }
        }
}

template <typename T, int KD, int VT>
hipError_t grad_shape(const MatrecParams& p, hipStream_t stream) {
    constexpr size_t lds = sizeof(T) * kChunk * (128 * KD + 128 * VT + 64 + 5 * Op<T>::PAD) + 4 * (4 * 64 + 3 * 256 + 4);
    static_assert(lds <= 160 * 1024, "a workgroup's tiles fit the CU's LDS");
    const dim3 grid((unsigned)((long long)p.plan.max_segs * p.plan.per * p.Hk));
    if (grid.x == 0) return hipSuccess;
    auto kernel = matrec_grad_kernel<T, KD, VT>;
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, grid, dim3(64 * kWaves), lds, stream, p);
    return hipGetLastError();
}
template <typename T>
hipError_t grad_type(const MatrecParams& p, hipStream_t stream) {
    if (p.Dk <= 64) return p.Dv <= 64 ? grad_shape<T, 1, 1>(p, stream) : grad_shape<T, 1, 2>(p, stream);
    return p.Dv <= 64 ? grad_shape<T, 2, 1>(p, stream) : grad_shape<T, 2, 2>(p, stream);
}

}  // namespace

hipError_t launch_matrec_grad(int dtype, const MatrecParams& p, hipStream_t stream) {
    return dtype == DEER_BF16 ? grad_type<BF16>(p, stream) : grad_type<float>(p, stream);
}

}  // namespace deer
