// Gradient of the matrix-state recurrence, chunk by chunk side by side.  In front of every chunk lies the state S, behind it the gradient R of
// the state there (launch_matrec_states); with A_ij = q_i . k_j, B_ij = dout_i . v_j and E_ij = scale e^{c_i - c_j} for j <= i, else 0,
//   dq_i = sum_j E_ij B_ij k_j + scale e^{c_i} S dout_i        dk_j = sum_i E_ij B_ij q_i + e^{c_64 - c_j} R v_j
//   dv_j = sum_i E_ij A_ij dout_i + e^{c_64 - c_j} R^T k_j
// and the gradient of a log gate, e^{g_t} <S_{t-1}, dS_t>, is the sum over everything that passes row t: pairs i >= t > j inside
// the chunk, what comes from S and is read at i >= t, what j < t adds and R takes on, and what goes through from S to R:
//   dgate_t = sum_{i >= t > j} E_ij A_ij B_ij + sum_{i >= t} q_i . (scale e^{c_i} S dout_i) + sum_{j < t} k_j . (e^{c_64 - c_j} R v_j) + e^{c_64} <S, R>,
// each of them a sum of what belongs to it alone, so that a strong gate's small gradient is no difference of large numbers.  The pairs: running
// sums over j along every row i, of which t takes those of the rows i >= t at j = t - 1.  A and B are exact products of the inputs, S and R enter dgate's products as three bf16 pieces.
// Heads of v that share one of q and k are gone through one after another, their dq and dk added in registers, always in the same order.
#include "matrec_common.h"

namespace deer {
namespace {

// Chunk states lie in memory as whole tiles of DK x DV floats, zero outside the head.  Eight terms of row d, the block of 32 columns s:
template <int DV>
__device__ __forceinline__ F32x8 state_row(const float* S, int d, int s, int g) {
    const float* at = S + d * DV + 32 * s + 4 * g;
    return joined(*reinterpret_cast<const F32x4*>(at), *reinterpret_cast<const F32x4*>(at + 16));
}
// column v, the block of 32 rows s
template <int DV>
__device__ __forceinline__ F32x8 state_col(const float* S, int v, int s, int g) {
    F32x8 x;
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = S[(32 * s + 4 * g + (e & 3) + (e >= 4 ? 16 : 0)) * DV + v];
    return x;
}

template <typename T, int DK, int DV>
struct GradLds {
    static constexpr size_t q = 0, k = Tile<T, DK>::bytes, v = k + Tile<T, DK>::bytes, d = v + Tile<T, DV>::bytes, pairs = d + Tile<T, DV>::bytes,
                            sums = pairs + Tile<T, kChunk>::bytes;
    static constexpr int W = (DK > DV ? DK : DV) / 16;
    // cum_hi, cum_lo, since, until; by wavefront: in, out, pairs; totals of four tiles; by wavefront: through
    static constexpr size_t total = sums + 4 * (4 * 64 + (2 * W + 4) * 64 + 4 * 64 + 8);
    static_assert(total <= 160 * 1024, "a workgroup's tiles fit the CU's LDS");
};

// One chunk and head of q and k.  Wavefront w has the columns 16 w .. of d, for dq and dk, and of v, for dv; all of them are computed transposed, a lane
// four neighbouring columns of a row.  States are read from memory straight into operands: every cell once by the wavefront that has
// its row d, R's once more by columns.
template <typename T, int DK, int DV>
__global__ __launch_bounds__(4 * (DK > DV ? DK : DV), sizeof(T) == 2 ? 2 : 1) void matrec_grad_kernel(const MatrecParams p) {
    using L = GradLds<T, DK, DV>;
    using TK = Tile<T, DK>;
    using TV = Tile<T, DV>;
    using TP = Tile<T, kChunk>;
    constexpr int W = L::W, KS = DK / 32, VS = DV / 32, P = Op<T>::PIECES;
    extern __shared__ __align__(16) unsigned char lds[];
    T *tq = reinterpret_cast<T*>(lds + L::q), *tk = reinterpret_cast<T*>(lds + L::k), *tv = reinterpret_cast<T*>(lds + L::v), *td = reinterpret_cast<T*>(lds + L::d),
      *tp = reinterpret_cast<T*>(lds + L::pairs);
    float* cum_hi = reinterpret_cast<float*>(lds + L::sums);
    float *cum_lo = cum_hi + 64, *since = cum_lo + 64, *until = since + 64;
    float* sum_in = until + 64;              // [W][64]: scale e^{c_i} q_i . (S dout_i), the part of a wavefront's columns
    float* sum_out = sum_in + 64 * W;        // [W][64]: e^{c_64 - c_j} k_j . (R v_j)
    float* sum_pairs = sum_out + 64 * W;     // [row tile][64]: at j the pairs (i, j' <= j) of j's tile with i > j, over the rows i of a row tile
    float* row_total = sum_pairs + 256;      // [column tile][64]: the pairs of row i in a tile
    float* sum_through = row_total + 256;    // [W]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4, l = lane & 15;
    const int kh = blockIdx.x % p.Hk, chunk_no = (int)(blockIdx.x / p.Hk), seg_no = chunk_no / p.plan.per, c = chunk_no % p.plan.per;
    if (seg_no >= *p.plan.count) return;
    const MatSegment seg = p.plan.segs[seg_no];
    const long long left = seg.rows - (long long)c * kChunk;
    if (left <= 0) return;
    const int rows = left < kChunk ? (int)left : kChunk, group = p.Hv / p.Hk;
    const long long row = seg.row0 + (long long)c * kChunk;
    const int d0 = 16 * wave + 4 * g;        // a lane's four columns of d, and of v
    const bool has_d = 16 * wave < DK, has_v = 16 * wave < DV;

    Stage<T, DV, 64 * W> fv, fd;
    {
        Stage<T, DK, 64 * W> fq, fk;
        fq.fetch(reinterpret_cast<const T*>(p.q) + row * p.stride_q + (long long)kh * p.Dk, p.stride_q, rows, p.Dk);
        fk.fetch(reinterpret_cast<const T*>(p.k) + row * p.stride_k + (long long)kh * p.Dk, p.stride_k, rows, p.Dk);
        fv.fetch(reinterpret_cast<const T*>(p.v) + row * p.stride_v + (long long)kh * group * p.Dv, p.stride_v, rows, p.Dv);
        fd.fetch(reinterpret_cast<const T*>(p.dout) + row * p.stride_o + (long long)kh * group * p.Dv, p.stride_o, rows, p.Dv);
        fq.put(tq);
        fk.put(tk);
    }
    // pairs above the diagonal that a product of 32 terms takes in are zero
    using V4 = T __attribute__((ext_vector_type(4)));
    if (wave == 0) {
        *reinterpret_cast<V4*>(tp + TP::four(l, 16 + 4 * g)) = V4{};
        *reinterpret_cast<V4*>(tp + TP::four(32 + l, 48 + 4 * g)) = V4{};
    }
    F32x4 dq[4], dk[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) dq[t] = dk[t] = F32x4{0, 0, 0, 0};

    for (int member = 0; member < group; ++member) {
        const int head = kh * group + member;
        const Cum cum = chunk_cum(gate_of(p.gate + row * p.Hv + head, p.Hv, rows));
        const float end_hi = lane_value(cum.hi, 63), end_lo = lane_value(cum.lo, 63), whole = expf(end_hi + end_lo);
        fv.put(tv);
        fd.put(td);
        if (wave == 0) {
            cum_hi[lane] = cum.hi;
            cum_lo[lane] = cum.lo;
            since[lane] = p.scale * expf(cum.hi + cum.lo);
            until[lane] = decay_between(end_hi, end_lo, cum.hi, cum.lo);
        }
        if (threadIdx.x < 256) sum_pairs[threadIdx.x] = row_total[threadIdx.x] = 0.0f;
        __syncthreads();
        const float* S = p.chunk_state + ((long long)(seg.chunk0 + c) * p.Hv + head) * (DK * DV);
        const float* R = p.chunk_rstate + ((long long)(seg.chunk0 + c) * p.Hv + head) * (DK * DV);

        // ---- pairs, tile by tile, as transposes: a lane has one i and four neighbouring j ----
        F32x4 ea[10 / W + 1];   // E_ij A_ij of this wavefront's tiles, for dv
#pragma unroll
        for (int m = 0; m < 10 / W + 1; ++m) {
            const int n = wave + m * W;
            if (n >= 10) break;
            int ti, tj;
            lower_tile(n, ti, tj);
            const int i = 16 * ti + l, j0 = 16 * tj + 4 * g;
            F32x4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < KS; ++s) a = mma(TK::row_frag(tk, 16 * tj + l, s, g), TK::row_frag(tq, i, s, g), a);
#pragma unroll
            for (int s = 0; s < VS; ++s) b = mma(TV::row_frag(tv, 16 * tj + l, s, g), TV::row_frag(td, i, s, g), b);
            const float hi_i = cum_hi[i], lo_i = cum_lo[i];
            const F32x4 hj = *reinterpret_cast<const F32x4*>(cum_hi + j0), lj = *reinterpret_cast<const F32x4*>(cum_lo + j0);
            F32x4 upto;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int j = j0 + r;
                const float e = j <= i ? p.scale * decay_between(hi_i, lo_i, hj[r], lj[r]) : 0.0f;
                upto[r] = (r > 0 ? upto[r > 0 ? r - 1 : 0] : 0.0f) + (j < i ? e * a[r] * b[r] : 0.0f);
                a[r] = j <= i ? e * a[r] : 0.0f;
                b[r] = j <= i ? e * b[r] : 0.0f;
            }
            ea[m] = a;
            store_four<T>(tp + TP::four(i, j0), b, 4, true);
            // the lane groups in front of this one have the smaller j
            float front = upto[3];
            const float one = __shfl_up(front, 16);
            front += g >= 1 ? one : 0.0f;
            const float two = __shfl_up(front, 32);
            front += g >= 2 ? two : 0.0f;
            const float before = __shfl_up(front, 16);
            if (g == 3) row_total[64 * tj + i] = front;
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                float s = j0 + r < i ? upto[r] + (g >= 1 ? before : 0.0f) : 0.0f;
                s = group_sum(s);
                if (l == 0) sum_pairs[64 * ti + j0 + r] = s;
            }
        }
        __syncthreads();

        // ---- dq and dk ----
        if (has_d) {
            F32x4 in[4], out[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) in[t] = out[t] = F32x4{0, 0, 0, 0};
            float through = 0.0f;
#pragma unroll
            for (int s = 0; s < VS; ++s) {
                const F32x8 x = state_row<DV>(S, 16 * wave + l, s, g), y = state_row<DV>(R, 16 * wave + l, s, g);
#pragma unroll
                for (int e = 0; e < 8; ++e) through += x[e] * y[e];
                frag_t<T> xp[P], yp[P];
                pieces_of<T>(x, xp);
                pieces_of<T>(y, yp);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    const frag_t<T> df = TV::row_frag(td, 16 * t + l, s, g), vf = TV::row_frag(tv, 16 * t + l, s, g);
#pragma unroll
                    for (int q = P - 1; q >= 0; --q) {
                        in[t] = mma(xp[q], df, in[t]);
                        out[t] = mma(yp[q], vf, out[t]);
                    }
                }
            }
            through += __shfl_xor(through, 16);
            through += __shfl_xor(through, 32);
            through = group_sum(through);
            if (lane == 0) sum_through[wave] = through;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int i = 16 * t + l;
                in[t] *= since[i];
                out[t] *= until[i];
                const V4 q4 = *reinterpret_cast<const V4*>(tq + TK::four(i, d0)), k4 = *reinterpret_cast<const V4*>(tk + TK::four(i, d0));
                float x = 0.0f, y = 0.0f;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    x += (float)q4[r] * in[t][r];
                    y += (float)k4[r] * out[t][r];
                }
                x += __shfl_xor(x, 16);
                y += __shfl_xor(y, 16);
                x += __shfl_xor(x, 32);
                y += __shfl_xor(y, 32);
                if (g == 0) {
                    sum_in[64 * wave + i] = x;
                    sum_out[64 * wave + i] = y;
                }
                dq[t] += in[t];
                dk[t] += out[t];
            }
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const frag_t<T> kf = TK::col_frag(tk, s, wave, lane), qf = TK::col_frag(tq, s, wave, lane);
#pragma unroll
                for (int t = 0; t < 4; ++t) {
                    if (s <= t / 2) dq[t] = mma(kf, TP::row_frag(tp, 16 * t + l, s, g), dq[t]);   // rows i of tile t take the columns j of block s
                    if (s >= t / 2) dk[t] = mma(qf, TP::col_frag(tp, s, t, lane), dk[t]);         // columns j of tile t the rows i of block s
                }
            }
        } else if (lane == 0) {
            sum_through[wave] = 0.0f;
        }
        if (!has_d) sum_in[64 * wave + lane] = sum_out[64 * wave + lane] = 0.0f;
        __syncthreads();

        // ---- the other pairs, the gates, and dv ----
#pragma unroll
        for (int m = 0; m < 10 / W + 1; ++m) {
            const int n = wave + m * W;
            if (n >= 10) break;
            int ti, tj;
            lower_tile(n, ti, tj);
            store_four<T>(tp + TP::four(16 * ti + l, 16 * tj + 4 * g), ea[m], 4, true);
        }
        if (wave == W - 1 && p.dgate) {
            // a lane has row t: sums from t on of what is read there, sums in front of t of what is added there
            float later = 0.0f, earlier = 0.0f, pairs = 0.0f, through = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                later += sum_in[64 * w + lane];
                earlier += sum_out[64 * w + lane];
                through += sum_through[w];
            }
            float tile[3];   // pairs (i >= t, j) of whole tiles in front of t - 1's
#pragma unroll
            for (int w = 0; w < 4; ++w) pairs += lane > 0 ? sum_pairs[64 * w + lane - 1] : 0.0f;
#pragma unroll
            for (int w = 0; w < 3; ++w) tile[w] = row_total[64 * w + lane];
#pragma unroll
            for (int d = 1; d < 64; d *= 2) {
                const float a = __shfl_down(later, d), b = __shfl_up(earlier, d);
                later += lane + d < 64 ? a : 0.0f;
                earlier += lane >= d ? b : 0.0f;
#pragma unroll
                for (int w = 0; w < 3; ++w) {
                    const float x = __shfl_down(tile[w], d);
                    tile[w] += lane + d < 64 ? x : 0.0f;
                }
            }
            earlier = __shfl_up(earlier, 1);
            if (lane == 0) earlier = 0.0f;
#pragma unroll
            for (int w = 0; w < 3; ++w) pairs += lane > 16 * (w + 1) ? tile[w] : 0.0f;
            if (lane < rows) p.dgate[(row + lane) * p.Hv + head] = pairs + later + earlier + whole * through;
        }
        F32x4 dv[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) dv[t] = F32x4{0, 0, 0, 0};
        if (has_v) {
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const frag_t<T> rc = rounded<T>(state_col<DV>(R, 16 * wave + l, s, g));
#pragma unroll
                for (int t = 0; t < 4; ++t) dv[t] = mma(rc, TK::row_frag(tk, 16 * t + l, s, g), dv[t]);
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) dv[t] *= until[16 * t + l];
        }
        if (member + 1 < group) {   // the next head's rows on their way
            fv.fetch(reinterpret_cast<const T*>(p.v) + row * p.stride_v + (long long)(head + 1) * p.Dv, p.stride_v, rows, p.Dv);
            fd.fetch(reinterpret_cast<const T*>(p.dout) + row * p.stride_o + (long long)(head + 1) * p.Dv, p.stride_o, rows, p.Dv);
        }
        __syncthreads();
        if (has_v) {
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const frag_t<T> df = TV::col_frag(td, s, wave, lane);
#pragma unroll
                for (int t = 0; t < 4; ++t)
                    if (s >= t / 2) dv[t] = mma(df, TP::col_frag(tp, s, t, lane), dv[t]);
            }
            T* to = reinterpret_cast<T*>(p.dv) + (long long)head * p.Dv;
            const bool wide = four_wide(to, p.stride_v, p.Dv);
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int j = 16 * t + l;
                if (j < rows && d0 < p.Dv) store_four<T>(to + (row + j) * p.stride_v + d0, dv[t], p.Dv - d0, wide);
            }
        }
        __syncthreads();   // the next head's tiles come over these
    }
    if (has_d) {
        T *to_q = reinterpret_cast<T*>(p.dq) + (long long)kh * p.Dk, *to_k = reinterpret_cast<T*>(p.dk) + (long long)kh * p.Dk;
        const bool wide_q = four_wide(to_q, p.stride_q, p.Dk), wide_k = four_wide(to_k, p.stride_k, p.Dk);
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int i = 16 * t + l;
            if (i < rows && d0 < p.Dk) {
                store_four<T>(to_q + (row + i) * p.stride_q + d0, dq[t], p.Dk - d0, wide_q);
                store_four<T>(to_k + (row + i) * p.stride_k + d0, dk[t], p.Dk - d0, wide_k);
            }
        }
    }
}

template <typename T, int DK, int DV>
hipError_t grad_shape(const MatrecParams& p, hipStream_t stream) {
    using L = GradLds<T, DK, DV>;
    const dim3 grid((unsigned)((long long)p.plan.max_segs * p.plan.per * p.Hk));
    if (grid.x == 0) return hipSuccess;
    auto kernel = matrec_grad_kernel<T, DK, DV>;
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)L::total);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, grid, dim3(64 * L::W), L::total, stream, p);
    return hipGetLastError();
}
template <typename T>
hipError_t grad_type(const MatrecParams& p, hipStream_t stream) {
    if (p.Dk <= 64) return p.Dv <= 64 ? grad_shape<T, 64, 64>(p, stream) : grad_shape<T, 64, 128>(p, stream);
    return p.Dv <= 64 ? grad_shape<T, 128, 64>(p, stream) : grad_shape<T, 128, 128>(p, stream);
}

}  // namespace

hipError_t launch_matrec_grad(int dtype, const MatrecParams& p, hipStream_t stream) {
    return dtype == DEER_BF16 ? grad_type<BF16>(p, stream) : grad_type<float>(p, stream);
}

}  // namespace deer
