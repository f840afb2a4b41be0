// Gradient of the matrix-state recurrence: with the state S in front of a chunk, the gradient R of the state behind it, A_ij = q_i . k_j, B_ij = dout_i . v_j
// and E_ij = scale e^{c_i - c_j} for j <= i, else 0,
//   dq_i = sum_j E_ij B_ij k_j + scale e^{c_i} S dout_i        dk_j = sum_i E_ij B_ij q_i + e^{c_64 - c_j} R v_j
//   dv_j = sum_i E_ij A_ij dout_i + e^{c_64 - c_j} R^T k_j
// are three runs of the form of matrec_run, one forwards that carries S, two backwards that carry R: no state of a chunk goes through memory.
// The gradient of a log gate, e^{g_t} <S_{t-1}, dS_t>, is the sum over everything that passes row t: pairs i >= t > j inside
// the chunk, what comes from S and is read at i >= t, what j < t adds and R takes on, and what goes through from S to R:
//   dgate_t = sum_{i >= t > j} E_ij A_ij B_ij + sum_{i >= t} u_i + sum_{j < t} w_j + z,
//   u_i = q_i . (scale e^{c_i} S dout_i)     w_j = k_j . (e^{c_64 - c_j} R v_j)     z = e^{c_64} <S, R>.
// The runs have u, w and the pairs: running sums over j along every row i, of which t takes those of the rows i >= t at j = t - 1.  z is not
// computed from S and R, which are never in one place: <S, dS> in front of a chunk is z + sum u, behind it z + sum w, and in front of a
// segment it is taken from both states.  So z comes with the rounding errors of the sums of u and w of a segment's chunks (2^-24 of their terms
// each, 32 chunks at most), which a state that was large in front leaves behind after it is forgotten: the difference is therefore kept within
// e^{c_64} |S| |R| (sums of squares of S and R, which the runs of dq and dk take in front of every chunk), and with it the error; the rest loses nothing to
// cancellation.  M in the sums of u and w is taken as three bf16 pieces, A and B are exact products of the inputs.  Heads of v that share one of q and k: dq and dk as floats by head first, then
// summed in the heads' order.
#include "matrec_run.h"

namespace deer {
namespace {

template <typename T, int DK, int DV>
struct GradShape {
    static constexpr int W = (DK > DV ? DK : DV) / 16;
    static constexpr size_t a = RunLds<T, DV, DK, W, RUN_DQ>::total, b = RunLds<T, DV, DK, W, RUN_DK>::total, c = RunLds<T, DK, DV, W, RUN_DV>::total;
    static constexpr size_t lds = a > b ? (a > c ? a : c) : (b > c ? b : c);
};

// Registers and what bounds it: matrec_run.h.  dq, dk and dv of a segment and head at the same time and on the same XCD (workgroups go to the 8 XCDs in turn): they read the same rows
template <typename T, int DK, int DV>
__global__ __launch_bounds__(4 * (DK > DV ? DK : DV), sizeof(T) == 2 ? (DK == 128 || DV == 128 ? 4 : 3) : 2) void matrec_grad_kernel(const MatrecParams p) {
    extern __shared__ __align__(16) unsigned char lds[];
    constexpr int W = GradShape<T, DK, DV>::W;
    const int run = blockIdx.x / 8 % 3, id = blockIdx.x / 24 * 8 + blockIdx.x % 8;
    if (run == 0) matrec_run<T, DK, DV, W, RUN_DQ>(p, lds, id);
    else if (run == 1) matrec_run<T, DK, DV, W, RUN_DK>(p, lds, id);
    else matrec_run<T, DK, DV, W, RUN_DV>(p, lds, id);
}

// what goes through every chunk, in the place of what is read in it: along a segment from <S, dS> in front of it; a lane has a head of a segment
__global__ __launch_bounds__(256) void matrec_through_kernel(const MatrecParams p) {
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x;
    const int seg_no = (int)(at / p.Hv), head = (int)(at % p.Hv);
    MatSegment seg;
    if (!segment_of(p, seg_no, seg)) return;
    const int chunks = (int)((seg.rows + kChunk - 1) / kChunk);
    float here = p.front[at];
    constexpr int K = 8;
    for (int c0 = 0; c0 < chunks; c0 += K) {
        float u[K], w[K], f[K], most[K];
#pragma unroll
        for (int i = 0; i < K; ++i) {
            const long long c = (long long)(seg.chunk0 + (c0 + i < chunks ? c0 + i : chunks - 1)) * p.Hv + head;
            u[i] = p.read_in[c];
            w[i] = p.put_out[c];
            f[i] = p.rows_of[c * kRowFloats + 256];
            // (squares below the smallest number are lost, 16,384 of them at most; pieces of a state are off by 2^-8, its size by less than 2^-7)
            most[i] = 1.02f * f[i] * __builtin_amdgcn_sqrtf(p.size_in[c] + 1e-33f) * __builtin_amdgcn_sqrtf(p.size_out[c] + 1e-33f);
        }
#pragma unroll
        for (int i = 0; i < K; ++i) {
            if (c0 + i >= chunks) break;
            float z = f[i] < 0x1p-60f ? 0.0f : here - u[i];   // (a factor that leaves nothing of <S, R>)
            if (fabsf(z) > most[i]) z = copysignf(most[i], z);
            p.read_in[(long long)(seg.chunk0 + c0 + i) * p.Hv + head] = z;
            here = z + w[i];
        }
    }
}

// dgate: the parts of the two runs and what goes through; a workgroup has a chunk
__global__ __launch_bounds__(256) void matrec_gates_kernel(const MatrecParams p) {
    int c;
    MatSegment seg;
    if (!segment_of_chunk(p, blockIdx.x, seg, c)) return;
    const long long left = seg.rows - (long long)c * kChunk;
    const int rows = left < kChunk ? (int)left : kChunk;
    const long long first = (seg.row0 + (long long)c * kChunk) * p.Hv, chunk = (long long)blockIdx.x * p.Hv;
    for (int i = threadIdx.x; i < rows * p.Hv; i += 256) p.dgate[first + i] += p.gate_k[first + i] + p.read_in[chunk + i % p.Hv];
}

// dq and dk of shared heads: the heads of v that go with one, in their order; a workgroup has 16 rows of a chunk and up to 64 V columns.
// Memory bound; the columns are spread over workgroups because a short call is one chain of loads after another (gradient of 128 rows, 8 heads of 128
// for 16: 69 us with all columns of 16 rows in a workgroup, one a lane; 35 so).
constexpr int kSharedRows = 16;
template <typename T, int V>
__global__ __launch_bounds__(256) void matrec_shared_kernel(const MatrecParams p) {
    using FV = vec_t<float, V>;
    using TV = vec_t<T, V>;
    constexpr int PARTS = kChunk / kSharedRows;
    int c;
    MatSegment seg;
    if (!segment_of_chunk(p, blockIdx.x / PARTS, seg, c)) return;
    const long long first = (long long)c * kChunk + blockIdx.x % PARTS * kSharedRows, left = seg.rows - first;
    if (left <= 0) return;
    const int rows = left < kSharedRows ? (int)left : kSharedRows, group = p.Hv / p.Hk, cols = p.Hk * p.Dk;
    const bool of_q = blockIdx.y == 0;
    const float* part = of_q ? p.part_q : p.part_k;
    T* to = reinterpret_cast<T*>(of_q ? p.dq : p.dk);
    const long long stride = of_q ? p.stride_q : p.stride_k, row0 = seg.row0 + first;
    for (int col = ((int)blockIdx.z * 64 + threadIdx.x % 64) * V; col < cols; col += (int)gridDim.z * 64 * V) {
        const int kh = col / p.Dk, d = col % p.Dk;
#pragma unroll
        for (int i = 0; i < kSharedRows / 4; ++i) {
            const int r = threadIdx.x / 64 + 4 * i;
            if (r >= rows) break;
            const float* from = part + ((row0 + r) * p.Hv + (long long)kh * group) * p.Dk + d;
            FV s = *reinterpret_cast<const FV*>(from);
            for (int m = 1; m < group; ++m) s += *reinterpret_cast<const FV*>(from + (long long)m * p.Dk);
            T* at = to + (row0 + r) * stride + col;
            if constexpr (V == 1) *at = (T)s;
            else *reinterpret_cast<TV*>(at) = __builtin_convertvector(s, TV);
        }
    }
}
template <typename T>
hipError_t launch_shared(const MatrecParams& p, unsigned chunks, hipStream_t stream) {
    const bool wide = four_wide(reinterpret_cast<const T*>(p.dq), p.stride_q, p.Dk) && four_wide(reinterpret_cast<const T*>(p.dk), p.stride_k, p.Dk);
    const int per = wide ? 256 : 64, parts = (p.Hk * p.Dk + per - 1) / per;
    const dim3 grid(chunks * (kChunk / kSharedRows), 2, parts > 16 ? 16 : parts);
    if (wide) hipLaunchKernelGGL((matrec_shared_kernel<T, 4>), grid, dim3(256), 0, stream, p);
    else hipLaunchKernelGGL((matrec_shared_kernel<T, 1>), grid, dim3(256), 0, stream, p);
    return hipGetLastError();
}

template <typename T, int DK, int DV>
hipError_t grad_shape(const MatrecParams& p, hipStream_t stream) {
    using G = GradShape<T, DK, DV>;
    return launch_lds(matrec_grad_kernel<T, DK, DV>, dim3((unsigned)(((long long)p.plan.max_segs * p.Hv + 7) / 8 * 24)), 64 * G::W, G::lds, p, stream);
}

}  // namespace

hipError_t launch_matrec_grad(int dtype, const MatrecParams& p, hipStream_t stream) {
    hipError_t e = dtype == DEER_BF16 ? DEER_BY_SHAPE(grad_shape, BF16, stream) : DEER_BY_SHAPE(grad_shape, float, stream);
    const unsigned chunks = (unsigned)p.plan.max_chunks;
    if (e != hipSuccess || chunks == 0) return e;
    if (p.Hv != p.Hk) {
        e = dtype == DEER_BF16 ? launch_shared<BF16>(p, chunks, stream) : launch_shared<float>(p, chunks, stream);
        if (e != hipSuccess) return e;
    }
    if (!p.dgate) return hipSuccess;
    hipLaunchKernelGGL(matrec_through_kernel, dim3((unsigned)(((long long)p.plan.max_segs * p.Hv + 255) / 256)), dim3(256), 0, stream, p);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(matrec_gates_kernel, dim3(chunks), dim3(256), 0, stream, p);
    return hipGetLastError();
}

}  // namespace deer
