// Gradient of the selective scan.  With lam_t = dL/dh_t (lam_t = C_t dy_t + a_{t+1} lam_{t+1}, a_t = exp(dt_t A)):
//   dB_t = sum over a group's channels of lam_t dt_t x_t        dC_t = that of dy_t h_t        dx_t = dt_t <lam_t, B_t> + skip dy_t
//   d dt_t = <lam_t, A a_t h_{t-1}> + x_t <lam_t, B_t>          dA = sum over the rows of dt_t lam_t a_t h_{t-1}
// dy here after the gate.  The states are computed again, forwards through 16 rows from a kept state; they stay in registers for the way back.
#include "selscan_common.h"

namespace deer {

hipError_t launch_selscan_empty(const SeqRows& rows, long long cells, const float* from, float* to, hipStream_t stream);

namespace {

constexpr float kLog2e = 1.44269504088896341f;
constexpr int R = kMarkRows;

template <int Q>
__device__ __forceinline__ float over_lanes(float v) {
#pragma unroll
    for (int d = 64 / Q; d < 64; d *= 2) v += __shfl_xor(v, d);
    return v;
}
template <int Q>
__device__ __forceinline__ float over_channels(float v) {
#pragma unroll
    for (int d = 1; d < 64 / Q; d *= 2) v += __shfl_xor(v, d);
    return v;
}

// What comes out at the front of a segment for the rows in front of it: a lam of its first row, from zero behind it (or from a sequence's end inside)
template <typename T, int Q>
__global__ __launch_bounds__(256) void selscan_fronts_kernel(const SelscanParams p) {
    using Sh = ScanShape<Q>;
    constexpr int CW = Sh::kChannels, kAcross = CW / 4, kStep = 256 / kAcross;
    __shared__ Float2 sx[R][CW];   // dt and dy
    __shared__ Float4 cs[R][Q];
    const ScanPlace place = scan_place<Q>(p);
    if (place.lo >= place.hi) return;
    ScanSeq seq;
    seq.at(p.rows, place, place.lo);
    const bool reset = seq.end <= place.hi;
    if (threadIdx.x == 0) p.rresets[place.seg] = reset;
    if (seq.start == place.lo) return;   // nothing of it is in front
    const long long lo = place.lo, hi = reset ? seq.end : place.hi;
    const int lane = threadIdx.x & 63, q = lane / Sh::kWave, c = (threadIdx.x >> 6) * Sh::kWave + lane % Sh::kWave;
    const ScanLane l{place.ch0 + c, 4 * q, c < place.channels};
    float A2[4], r[4], sum_dt = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) A2[k] = l.on && l.k0 + k < p.S ? p.A[(long long)l.ch * p.S + l.k0 + k] * kLog2e : 0.0f;
    load_states(r, reset ? p.dlast : nullptr, seq.n, l, p.D, p.S);
    const int c4 = (threadIdx.x % kAcross) * 4, row0 = threadIdx.x / kAcross, count = place.channels - c4;
    float bias[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) bias[i] = p.bias && i < count ? p.bias[place.ch0 + c4 + i] : 0.0f;
    for (long long t0 = lo + (hi - lo - 1) / R * R; t0 >= lo; t0 -= R) {
        const int rows = hi - t0 < R ? (int)(hi - t0) : R;
        for (int i = row0; i < rows; i += kStep) {
            float dt[4], dy[4], z[4];
            const long long at = place.ch0 + c4;
            load4<T>(dt, p.dt, (t0 + i) * p.stride_dt + at, count, p.vec);
            load4<T>(dy, p.dy, (t0 + i) * p.stride_y + at, count, p.vec);
            if (p.z) load4<T>(z, p.z, (t0 + i) * p.stride_z + at, count, p.vec);
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float raw = dt[v] + bias[v];
                sx[i][c4 + v] = Float2{p.softplus ? softplus(raw) : raw, p.z ? dy[v] * fast_silu(z[v]) : dy[v]};
            }
        }
        for (int e = threadIdx.x; e < rows * Q; e += 256) {
            float v[4];
            load4<T>(v, p.C, (t0 + e / Q) * p.stride_C + (long long)place.g * p.S + 4 * (e % Q), p.S - 4 * (e % Q), p.vec_bc);
            cs[e / Q][e % Q] = Float4{v[0], v[1], v[2], v[3]};
        }
        __syncthreads();
        for (int i = rows - 1; i >= 0; --i) {
            const Float2 s = sx[i][c];
            const Float4 cc = cs[i][q];
            sum_dt += s.x;
#pragma unroll
            for (int k = 0; k < 4; ++k) r[k] = __builtin_amdgcn_exp2f(s.x * A2[k]) * (r[k] + cc[k] * s.y);
        }
        __syncthreads();
    }
    store_states(p.rlocal, place.seg, l, p.D, 4 * Q, r);
    if (q == 0 && l.on) p.rsteps[place.seg * p.D + l.ch] = sum_dt;
}

// a lam of the first row behind every segment, from the last segment on
__global__ __launch_bounds__(256) void selscan_rjoin_kernel(const SelscanParams p, int SP) {
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x, cells = (long long)p.D * SP, seqs = p.rows.packed ? 1 : p.rows.N;
    if (at >= cells * seqs) return;
    const long long n = at / cells, cell = at % cells;
    const int ch = (int)(cell / SP), k = (int)(cell % SP);
    const float A2 = k < p.S ? p.A[(long long)ch * p.S + k] * kLog2e : 0.0f;
    float r = 0.0f;
    for (long long s = (n + 1) * p.segs - 1; s > n * p.segs; --s) {
        const float local = p.rlocal[s * cells + cell], decay = __builtin_amdgcn_exp2f(A2 * p.rsteps[s * p.D + ch]);
        r = p.rresets[s] ? local : local + decay * r;
        p.rcarry[(s - 1) * cells + cell] = r;
    }
}

template <typename T, int Q>
__global__ __launch_bounds__(256) void selscan_grad_kernel(const SelscanParams p, const RestRows rest) {
    using Sh = ScanShape<Q>;
    constexpr int CW = Sh::kChannels, kAcross = CW / 4, kStep = 256 / kAcross, kItems = R * CW >= 1024 ? R * CW / 1024 : 1;
    __shared__ Float4 it[R][CW];         // dt, dt x, dy, y; on the way back <lam, B> and <lam, A a h> in the places of dt x and dy
    __shared__ Float4 bc[R][2][Q];
    __shared__ float red[4][R][2][4 * Q];   // of a wavefront: lam dt x and dy h summed over its channels
    clear_rest(p.rows, rest, blockIdx.x, gridDim.x);
    const ScanPlace place = scan_place<Q>(p);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, q = lane / Sh::kWave, c = wave * Sh::kWave + lane % Sh::kWave;
    const ScanLane l{place.ch0 + c, 4 * q, c < place.channels};
    float A[4], dA[4], r[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        A[k] = l.on && l.k0 + k < p.S ? p.A[(long long)l.ch * p.S + l.k0 + k] : 0.0f;
        dA[k] = 0.0f;
    }
    const int c4 = (threadIdx.x % kAcross) * 4, row0 = threadIdx.x / kAcross, count = place.channels - c4;
    float bias[4], skip[4], dbias[4], dskip[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bias[i] = p.bias && i < count ? p.bias[place.ch0 + c4 + i] : 0.0f;
        skip[i] = p.skip && i < count ? p.skip[place.ch0 + c4 + i] : 0.0f;
        dbias[i] = dskip[i] = 0.0f;
    }
    const long long lo = place.lo, hi = place.hi;
    const long long all_rows = p.rows.T * (p.rows.packed ? 1 : p.rows.N);
    if (lo < hi) {
        ScanSeq seq;   // of the last row of the tile
        seq.at(p.rows, place, hi - 1);
        if (hi == seq.end) load_states(r, p.dlast, seq.n, l, p.D, p.S);
        else load_states(r, p.rcarry, place.seg, l, p.D, 4 * Q);
        for (long long t0 = lo + (hi - lo - 1) / R * R; t0 >= lo; t0 -= R) {
            const int rows = hi - t0 < R ? (int)(hi - t0) : R;
            float x[kItems][4], raw[kItems][4], z[kItems][4], dy[kItems][4];
#pragma unroll
            for (int j = 0; j < kItems; ++j) {
                const int i = row0 + j * kStep;
                if (i >= rows) continue;
                const long long at = place.ch0 + c4;
                load4<T>(x[j], p.x, (t0 + i) * p.stride_x + at, count, p.vec);
                load4<T>(raw[j], p.dt, (t0 + i) * p.stride_dt + at, count, p.vec);
                load4<T>(dy[j], p.dy, (t0 + i) * p.stride_y + at, count, p.vec);
                if (p.z) load4<T>(z[j], p.z, (t0 + i) * p.stride_z + at, count, p.vec);
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    raw[j][v] += bias[v];
                    const float dt = p.softplus ? softplus(raw[j][v]) : raw[j][v];
                    it[i][c4 + v] = Float4{dt, dt * x[j][v], p.z ? dy[j][v] * fast_silu(z[j][v]) : dy[j][v], 0.0f};
                }
            }
            for (int e = threadIdx.x; e < rows * 2 * Q; e += 256) {
                const int qq = e % Q, which = e / Q % 2, i = e / Q / 2;
                float v[4];
                if (which == 0) load4<T>(v, p.B, (t0 + i) * p.stride_B + (long long)place.g * p.S + 4 * qq, p.S - 4 * qq, p.vec_bc);
                else load4<T>(v, p.C, (t0 + i) * p.stride_C + (long long)place.g * p.S + 4 * qq, p.S - 4 * qq, p.vec_bc);
                bc[i][which][qq] = Float4{v[0], v[1], v[2], v[3]};
            }
            __syncthreads();
            // forwards from the state in front of the tile
            ScanSeq first = seq;
            if (first.start > t0) first.back(p.rows, t0);
            float before[4], a[R][4], h[R][4];
            {
                const long long mark = place.seg * p.marks_each + (t0 - lo) / R;
                load_states(before, p.marks, mark, l, p.D, 4 * Q);
                if (p.segs > 1 && first.start < lo) {
                    float carry[4];
                    load_states(carry, p.carry, place.seg, l, p.D, 4 * Q);
                    const float steps = l.on ? p.mark_steps[mark * p.D + l.ch] : 0.0f;
#pragma unroll
                    for (int k = 0; k < 4; ++k) before[k] += __builtin_amdgcn_exp2f(steps * A[k] * kLog2e) * carry[k];
                }
            }
            ScanSeq now = first;
#pragma unroll
            for (int i = 0; i < R; ++i) {
                if (i >= rows) continue;
                float in[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) in[k] = i ? h[i ? i - 1 : 0][k] : before[k];
                if (t0 + i == now.end) {
                    now.next(p.rows, t0 + i);
                    load_states(in, p.h0, now.n, l, p.D, p.S);
                }
                const Float4 s = it[i][c];
                const Float4 b = bc[i][0][q], cc = bc[i][1][q];
                float y = 0.0f;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    a[i][k] = __builtin_amdgcn_exp2f(s.x * (A[k] * kLog2e));
                    h[i][k] = a[i][k] * in[k] + s.y * b[k];
                    y += cc[k] * h[i][k];
                }
                if (p.z) {
                    y = over_lanes<Q>(y);
                    if (q == 0) it[i][c].w = y;
                }
            }
            // and back
#pragma unroll
            for (int i = R - 1; i >= 0; --i) {
                if (i >= rows) continue;
                if (t0 + i < now.start) {
                    now.back(p.rows, t0 + i);
                    load_states(r, p.dlast, now.n, l, p.D, p.S);
                }
                float in[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) in[k] = i ? h[i ? i - 1 : 0][k] : before[k];
                const bool begins = t0 + i == now.start;
                if (begins) load_states(in, p.h0, now.n, l, p.D, p.S);
                const Float4 s = it[i][c];
                const Float4 b = bc[i][0][q], cc = bc[i][1][q];
                float read = 0.0f, ddt = 0.0f;
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const float lam = r[k] + cc[k] * s.z;
                    const float dB = over_channels<Q>(lam * s.y), dC = over_channels<Q>(s.z * h[i][k]);
                    if (lane % Sh::kWave == 0) {
                        red[wave][i][0][4 * q + k] = dB;
                        red[wave][i][1][4 * q + k] = dC;
                    }
                    read += lam * b[k];
                    r[k] = a[i][k] * lam;
                    const float g = r[k] * in[k];
                    dA[k] += s.x * g;
                    ddt += A[k] * g;
                }
                read = over_lanes<Q>(read);
                ddt = over_lanes<Q>(ddt);
                if (q == 0) {
                    it[i][c].y = read;
                    it[i][c].z = ddt;
                }
                if (begins) store_states(p.dh0, now.n, l, p.D, p.S, r);
            }
            seq = first;
            if (t0 > lo && seq.start == t0) {   // the rows in front are another sequence's
                seq.back(p.rows, t0 - 1);
                load_states(r, p.dlast, seq.n, l, p.D, p.S);
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < kItems; ++j) {
                const int i = row0 + j * kStep;
                if (i >= rows || count <= 0) continue;
                float dx[4], ddt[4], dz[4];
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const Float4 s = it[i][c4 + v];
                    float gate = 1.0f, slope = 0.0f;
                    if (p.z) silu_both<BF16>(z[j][v], gate, slope);
                    const float out = dy[j][v] * gate;
                    dx[v] = s.x * s.y + skip[v] * out;
                    ddt[v] = (s.z + x[j][v] * s.y) * (p.softplus ? softplus_slope(raw[j][v]) : 1.0f);
                    dz[v] = dy[j][v] * (s.w + skip[v] * x[j][v]) * slope;
                    dskip[v] += out * x[j][v];
                    dbias[v] += ddt[v];
                }
                const long long at = place.ch0 + c4;
                store4<T>(p.dx, (t0 + i) * p.stride_x + at, dx, count, p.vec);
                store4<T>(p.ddt, (t0 + i) * p.stride_dt + at, ddt, count, p.vec);
                if (p.z) store4<T>(p.dz, (t0 + i) * p.stride_z + at, dz, count, p.vec);
            }
            for (int e = threadIdx.x; e < rows * 8 * Q; e += 256) {
                const int i = e / (8 * Q), k = e % (8 * Q);
                const float* f = &red[0][i][0][0] + k;
                constexpr int step = R * 8 * Q;
                p.part_bc[(((long long)place.block * all_rows + t0 + i) * p.G + place.g) * 8 * Q + k] = (f[0] + f[step]) + (f[2 * step] + f[3 * step]);
            }
        }
    }
    // sums over the segment's rows
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (l.on && l.k0 + k < p.S) p.part_A[(place.seg * p.D + l.ch) * p.S + l.k0 + k] = dA[k];
    float* sums = reinterpret_cast<float*>(&it[0][0]);
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        __syncthreads();
#pragma unroll
        for (int v = 0; v < 4; ++v) sums[row0 * CW + c4 + v] = w ? dbias[v] : dskip[v];
        __syncthreads();
        for (int i = threadIdx.x; i < place.channels; i += 256) {
            float sum = 0.0f;
            for (int f = 0; f < kStep; ++f) sum += sums[f * CW + i];
            p.part_d[(place.seg * 2 + w) * p.D + place.ch0 + i] = sum;
        }
    }
}

// dB and dC of rows that belong to a sequence: the workgroups' sums, in order
template <typename T>
__global__ __launch_bounds__(256) void selscan_bc_kernel(const SelscanParams p, int SP) {
    const long long all_rows = p.rows.T * (p.rows.packed ? 1 : p.rows.N), each = (long long)p.G * 2 * p.S;
    const long long step = all_rows * p.G * 2 * SP;
    for (long long e = (long long)blockIdx.x * 256 + threadIdx.x; e < all_rows * each; e += (long long)gridDim.x * 256) {
        const long long row = e / each;
        const int in = (int)(e % each), g = in / (2 * p.S), which = in / p.S % 2, k = in % p.S;
        if (p.rows.bounds) {
            if (p.rows.packed ? row < clamp_row(p.rows.bounds[0], p.rows.T) || row >= clamp_row(p.rows.bounds[p.rows.N], p.rows.T)
                              : row % p.rows.T >= clamp_row(p.rows.bounds[row / p.rows.T], p.rows.T))
                continue;
        }
        const float* f = p.part_bc + ((row * p.G + g) * 2 + which) * SP + k;
        float sum = 0.0f;
        for (int b = 0; b < p.blocks; ++b) sum += f[b * step];
        if (which == 0) reinterpret_cast<T*>(p.dB)[row * p.stride_B + g * p.S + k] = (T)sum;
        else reinterpret_cast<T*>(p.dC)[row * p.stride_C + g * p.S + k] = (T)sum;
    }
}

template <typename T, int Q>
hipError_t launch_lanes(const SelscanParams& p, hipStream_t stream) {
    const long long seqs = p.rows.packed ? 1 : p.rows.N, segs = seqs * p.segs, cells = (long long)p.D * 4 * Q, rows = p.rows.T * seqs;
    const dim3 grid((unsigned)(segs * p.G * p.blocks)), block(256);
    const long long e = sizeof(T);
    RestRows rest{};
    if (p.zero_rest) {
        auto add = [&](void* first, long long stride, long long width) { rest.array[rest.count++] = RestArray{first, stride * e, width * e}; };
        add(p.dx, p.stride_x, p.D);
        add(p.ddt, p.stride_dt, p.D);
        add(p.dB, p.stride_B, (long long)p.G * p.S);
        add(p.dC, p.stride_C, (long long)p.G * p.S);
        if (p.z) add(p.dz, p.stride_z, p.D);
    }
    if (p.segs > 1) {
        hipLaunchKernelGGL((selscan_fronts_kernel<T, Q>), grid, block, 0, stream, p);
        hipLaunchKernelGGL(selscan_rjoin_kernel, dim3((unsigned)((cells * seqs + 255) / 256)), block, 0, stream, p, 4 * Q);
    }
    if (p.rows.T) {
        hipLaunchKernelGGL((selscan_grad_kernel<T, Q>), grid, block, 0, stream, p, rest);
        const long long want = rows * p.G * 2 * p.S / 1024;
        hipLaunchKernelGGL((selscan_bc_kernel<T>), dim3((unsigned)(want < 1 ? 1 : want > 8192 ? 8192 : want)), block, 0, stream, p, 4 * Q);
    }
    hipError_t err = hipGetLastError();
    if (err == hipSuccess && p.dh0 && (p.rows.bounds || !p.rows.T)) err = launch_selscan_empty(p.rows, (long long)p.D * p.S, p.dlast, p.dh0, stream);
    if (err != hipSuccess) return err;
    SumInto into{};
    into.each = p.D * p.S;
    into.to[0] = p.dA;
    into.stride[0] = 1;
    err = launch_sum_tiles(false, p.part_A, p.rows.T ? segs : 0, p.D * p.S, into, stream);
    if (err != hipSuccess || (!p.dskip && !p.dbias)) return err;
    into.each = p.D;
    into.to[0] = p.dskip;
    into.to[1] = p.dbias;
    into.stride[1] = 1;
    return launch_sum_tiles(false, p.part_d, p.rows.T ? segs : 0, 2 * p.D, into, stream);
}
template <typename T>
hipError_t launch_type(const SelscanParams& p, hipStream_t stream) {
    switch (scan_lanes(p.S)) {
        case 1: return launch_lanes<T, 1>(p, stream);
        case 2: return launch_lanes<T, 2>(p, stream);
        case 4: return launch_lanes<T, 4>(p, stream);
        case 8: return launch_lanes<T, 8>(p, stream);
        default: return launch_lanes<T, 16>(p, stream);
    }
}

}  // namespace

hipError_t launch_selscan_grad(int dtype, const SelscanParams& p, hipStream_t stream) {
    switch (dtype) {
        case DEER_F32: return launch_type<float>(p, stream);
        case DEER_BF16: return launch_type<BF16>(p, stream);
        default: return launch_type<F16>(p, stream);
    }
}

}  // namespace deer
