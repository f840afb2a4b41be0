// Gradient of the selective scan.  With lam_t = dL/dh_t (lam_t = C_t dy_t + a_{t+1} lam_{t+1}, a_t = exp(dt_t A)):
//   dB_t = sum over a group's channels of lam_t dt_t x_t        dC_t = that of dy_t h_t        dx_t = dt_t <lam_t, B_t> + skip dy_t
//   d dt_t = <lam_t, A a_t h_{t-1}> + x_t <lam_t, B_t>          dA = sum over the rows of dt_t lam_t a_t h_{t-1}
// dy here after the gate.  The states are computed again, forwards through 16 rows from a kept state; they stay in registers for the way back.
#include <type_traits>

#include "selscan_common.h"
#include "selscan_sums.h"

namespace deer {

hipError_t launch_selscan_empty(const SeqRows& rows, long long cells, const float* from, float* to, hipStream_t stream);

namespace {

constexpr int R = kMarkRows;

// What the rows in front of a segment get from it, row by row, where the product of its factors has overflowed: rows of no weight do not make it infinite
template <typename T>
__device__ float front_by_rows(const SelscanParams& p, long long n, int seg, int ch, int k, float A2) {
    const long long base = n * p.rows.T, first = p.rows.packed ? clamp_row(p.rows.bounds[0], p.rows.T) : base;
    const long long behind = p.rows.packed ? clamp_row(p.rows.bounds[p.rows.N], p.rows.T) : base + seq_length(p.rows, (int)n);
    long long lo = base + seg * p.seg_rows, hi = lo + p.seg_rows, end = behind, at = n;
    lo = lo < first ? first : lo;
    hi = hi > behind ? behind : hi;
    if (lo >= hi || k >= p.S) return 0.0f;
    if (p.rows.packed) {
        at = bounds_up_to(p.rows, lo) - 1;
        at = at < 0 ? 0 : at >= p.rows.N ? p.rows.N - 1 : at;
        end = clamp_row(p.rows.bounds[at + 1], p.rows.T);
    }
    float r = end <= hi && p.dlast ? p.dlast[(at * p.D + ch) * p.S + k] : 0.0f;
    for (long long t = (end < hi ? end : hi) - 1; t >= lo && r == r; --t) {
        const float raw = (float)reinterpret_cast<const T*>(p.dt)[t * p.stride_dt + ch] + (p.bias ? p.bias[ch] : 0.0f), dt = p.softplus ? softplus(raw) : raw;
        float dy = (float)reinterpret_cast<const T*>(p.dy)[t * p.stride_y + ch];
        if (p.z) dy *= fast_silu((float)reinterpret_cast<const T*>(p.z)[t * p.stride_z + ch]);
        const float c = (float)reinterpret_cast<const T*>(p.C)[t * p.stride_C + (long long)(ch / p.per_group) * p.S + k];
        r = __builtin_amdgcn_exp2f(dt * A2) * (r + c * dy);
    }
    return r;
}

// a lam of the first row behind every segment, from the last segment on
template <typename T>
__global__ __launch_bounds__(256) void selscan_rjoin_kernel(const SelscanParams p, int SP) {
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x, cells = (long long)p.D * SP, seqs = p.rows.packed ? 1 : p.rows.N;
    if (at >= cells * seqs) return;
    const long long n = at / cells, cell = at % cells;
    const int ch = (int)(cell / SP), k = (int)(cell % SP);
    const float A2 = k < p.S ? p.A[(long long)ch * p.S + k] * kLog2e : 0.0f;
    float r = 0.0f;
    const long long first = n * p.segs;
    for (int s0 = p.segs - 1; s0 > 0; s0 -= 8) {
        float local[8], steps[8];
        int reset[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const long long s = first + (s0 - i > 0 ? s0 - i : 1);
            local[i] = p.rlocal[s * cells + cell];
            steps[i] = p.rsteps[s * p.D + ch];
            reset[i] = p.rresets[s];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (s0 - i <= 0) break;
            if (local[i] == __builtin_inff()) local[i] = front_by_rows<T>(p, n, s0 - i, ch, k, A2);
            r = reset[i] ? local[i] : local[i] + scaled(r, A2 * steps[i]);
            p.rcarry[(first + s0 - i - 1) * cells + cell] = r;
        }
    }
}

// Some 28 vector instructions for every state of a row, a quarter of them for the sums of dB and dC over channels (16 of 8 values a row and wavefront, by DPP) and their products: 16,384
// rows of 4,096 channels and 16 states in bf16 1,132 us, where the bytes take 240.  Two wavefronts a SIMD by registers; the factors are computed twice rather than kept.  Keeping them
// with a state kept every 8 rows is 11 % fewer instructions and 1,119 us, for twice the workspace; three wavefronts a SIMD (spills) 1,334; LDS read two rows ahead 1,135 to 1,314.
template <typename T, int Q, bool VEC>
__global__ __launch_bounds__(256, 2) void selscan_grad_kernel(const SelscanParams p, const RestRows rest) {
    using Sh = ScanShape<Q>;
    constexpr int CW = Sh::kChannels, kAcross = CW / 4, kStep = 256 / kAcross, kItems = R * CW >= 1024 ? R * CW / 1024 : 1;
    __shared__ Float4 it[R][CW];         // dt, dt x, dy, y; on the way back <lam, B> and <lam, A a h> in the places of dt x and dy
    __shared__ Float4 bc[R][2][Q];
    __shared__ float red[4][R][Q][8];    // of a wavefront: lam dt x and dy h of four states, summed over its channels
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
    // sums over kSumRows rows, once the first of them is done
    auto hand_over = [&](int part) {
        const long long at = place.seg * p.parts_each + part;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (l.on && l.k0 + k < p.S) p.part_A[(at * p.D + l.ch) * p.S + l.k0 + k] = dA[k];
            dA[k] = 0.0f;
        }
        float* sums = reinterpret_cast<float*>(&it[0][0]);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
            lds_barrier();
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                sums[row0 * CW + c4 + v] = w ? dbias[v] : dskip[v];
                (w ? dbias[v] : dskip[v]) = 0.0f;
            }
            lds_barrier();
            for (int i = threadIdx.x; i < place.channels; i += 256) {
                float sum = 0.0f;
                for (int f = 0; f < kStep; ++f) sum += sums[f * CW + i];
                p.part_d[(at * 2 + w) * p.D + place.ch0 + i] = sum;
            }
        }
        lds_barrier();
    };
    // (parts without rows)
    for (int part = lo < hi ? (int)((hi - lo + kSumRows - 1) / kSumRows) : 0; part < p.parts_each; ++part) {
        const long long at = place.seg * p.parts_each + part;
        for (int i = threadIdx.x; i < place.channels * p.S; i += 256) p.part_A[(at * p.D + place.ch0) * p.S + i] = 0.0f;
        for (int i = threadIdx.x; i < place.channels; i += 256) p.part_d[at * 2 * p.D + place.ch0 + i] = p.part_d[(at * 2 + 1) * p.D + place.ch0 + i] = 0.0f;
    }
    const long long all_rows = p.rows.T * (p.rows.packed ? 1 : p.rows.N);
    if (lo < hi) {
        ScanSeq seq;   // of the last row of the tile
        seq.at(p.rows, place, hi - 1);
        if (hi == seq.end) load_states(r, p.dlast, seq.n, l, p.D, p.S);
        else load_states(r, p.rcarry, place.seg, l, p.D, 4 * Q);
        // what a tile reads is asked for while the tile behind it is worked on
        Places<kItems> px, pd, py, pz;
        px.set(p.stride_x, row0, kStep, c4, T{});
        pd.set(p.stride_dt, row0, kStep, c4, T{});
        py.set(p.stride_y, row0, kStep, c4, T{});
        pz.set(p.stride_z, row0, kStep, c4, T{});
        auto tile_at = [&](const void* first, long long stride, long long t0, long long more) { return Tile(reinterpret_cast<const T*>(first) + t0 * stride + more); };
        Four<T, VEC> nx[kItems], nd[kItems], ny[kItems], nz[kItems], nb[2];
        float mark[4], steps = 0.0f;
        const int quad_row = threadIdx.x / Q, quad = 4 * (threadIdx.x % Q);
        auto ask = [&](long long t0) {
            const int rows = hi - t0 < R ? (int)(hi - t0) : R;
            const Tile x = tile_at(p.x, p.stride_x, t0, place.ch0), d = tile_at(p.dt, p.stride_dt, t0, place.ch0), y = tile_at(p.dy, p.stride_y, t0, place.ch0);
#pragma unroll
            for (int j = 0; j < kItems; ++j) {
                const bool on = count > 0 && row0 + j * kStep < rows;
                nx[j].load(x, on ? px.at[j] : kNoColumn, count);
                nd[j].load(d, on ? pd.at[j] : kNoColumn, count);
                ny[j].load(y, on ? py.at[j] : kNoColumn, count);
            }
            if (p.z) {
                const Tile z = tile_at(p.z, p.stride_z, t0, place.ch0);
#pragma unroll
                for (int j = 0; j < kItems; ++j) nz[j].load(z, count > 0 && row0 + j * kStep < rows ? pz.at[j] : kNoColumn, count);
            }
#pragma unroll
            for (int w = 0; w < 2; ++w) {
                const long long stride = w ? p.stride_C : p.stride_B;
                nb[w].load(tile_at(w ? p.C : p.B, stride, t0, (long long)place.g * p.S),
                           quad_row < rows && quad < p.S ? (unsigned)(quad_row * stride + quad) * (unsigned)sizeof(T) : kNoColumn, p.S - quad);
            }
            const long long at = place.seg * p.marks_each + (t0 - lo) / R;
            const __amdgpu_buffer_rsrc_t m = __builtin_amdgcn_make_buffer_rsrc(p.marks + at * p.D * 4 * Q, 0, (int)kNoColumn, 0x00020000);
            const Float4 four = __builtin_bit_cast(Float4, __builtin_amdgcn_raw_buffer_load_b128(m, l.on ? (unsigned)(l.ch * 4 * Q + l.k0) * 4u : kNoColumn, 0, 0));
#pragma unroll
            for (int k = 0; k < 4; ++k) mark[k] = four[k];
            if (p.segs > 1) steps = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(Tile(p.mark_steps + at * p.D).rsrc, l.on ? l.ch * 4u : kNoColumn, 0, 0));
        };
        float carry[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (p.segs > 1) {
            ScanSeq first = seq;
            if (first.start > lo) first.at(p.rows, place, lo);
            if (first.start < lo) load_states(carry, p.carry, place.seg, l, p.D, 4 * Q);
        }
        const long long t_last = lo + (hi - lo - 1) / R * R;
        ask(t_last);
        for (long long t0 = t_last; t0 >= lo; t0 -= R) {
            const int rows = hi - t0 < R ? (int)(hi - t0) : R;
            Four<T, VEC> x[kItems], z[kItems], dy[kItems], dt_in[kItems];
#pragma unroll
            for (int j = 0; j < kItems; ++j) {
                const int i = row0 + j * kStep;
                x[j] = nx[j];
                dt_in[j] = nd[j];
                dy[j] = ny[j];
                z[j] = nz[j];
                Float4 all[4];
#pragma unroll
                for (int v = 0; v < 4; ++v) {
                    const float raw = dt_in[j][v] + bias[v], dt = p.softplus ? softplus(raw) : raw;
                    all[v] = Float4{dt, dt * x[j][v], dy[j][v], 0.0f};
                }
                if (p.z)
#pragma unroll
                    for (int v = 0; v < 4; ++v) all[v].z *= fast_silu(z[j][v]);
                if (kStep * kItems <= R || i < R)
#pragma unroll
                    for (int v = 0; v < 4; ++v) it[i][c4 + v] = all[v];
            }
            if (R * Q >= 256 || threadIdx.x < R * Q) {
                bc[quad_row][0][threadIdx.x % Q] = Float4{nb[0][0], nb[0][1], nb[0][2], nb[0][3]};
                bc[quad_row][1][threadIdx.x % Q] = Float4{nb[1][0], nb[1][1], nb[1][2], nb[1][3]};
            }
            ScanSeq first = seq;
            if (first.start > t0) first.back(p.rows, t0);
            float before[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) before[k] = mark[k];
            if (p.segs > 1 && first.start < lo) {
#pragma unroll
                for (int k = 0; k < 4; ++k) before[k] += scaled(carry[k], steps * A[k] * kLog2e);
            }
            lds_barrier();
            if (t0 > lo) ask(t0 - R);
            // forwards from the state in front of the tile (that of a sequence that begins with it is its initial one), and back.  WHOLE: 16 rows of one sequence
            auto there_and_back = [&](auto whole) {
                constexpr bool WHOLE = decltype(whole)::value;
                float h[R][4];
                ScanSeq now = first;
#pragma unroll
                for (int i0 = 0; i0 < R; i0 += 4) {
                    if (!WHOLE && i0 >= rows) continue;
                    float y[4];
#pragma unroll
                    for (int u = 0; u < 4; ++u) {
                        const int i = i0 + u;
                        y[u] = 0.0f;
                        if (!WHOLE && i >= rows) continue;
                        float in[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) in[k] = i ? h[i ? i - 1 : 0][k] : before[k];
                        if (!WHOLE && t0 + i == now.end) {
                            now.next(p.rows, t0 + i);
                            load_states(in, p.h0, now.n, l, p.D, p.S);
                        }
                        const Float4 s = it[i][c];
                        const Float4 b = bc[i][0][q];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            h[i][k] = __builtin_amdgcn_exp2f(s.x * (A[k] * kLog2e)) * in[k] + s.y * b[k];
                        }
                        if (p.z) {
                            const Float4 cc = bc[i][1][q];
#pragma unroll
                            for (int k = 0; k < 4; ++k) y[u] += cc[k] * h[i][k];
                        }
                    }
                    __builtin_amdgcn_sched_barrier(0);
                    if (p.z) {
                        sum_lanes<Q>(y);
#pragma unroll
                        for (int j = 0; j < lanes_keep<Q>; ++j) it[i0 + of_lanes<Q>(lane, j)][c].w = y[j];
                    }
                }
#pragma unroll
                for (int i0 = R - 2; i0 >= 0; i0 -= 2) {
                    if (!WHOLE && i0 >= rows) continue;
                    float two[4];   // <lam, B> and <lam, A a h> of both rows
#pragma unroll
                    for (int u = 1; u >= 0; --u) {
                        const int i = i0 + u;
                        two[2 * u] = two[2 * u + 1] = 0.0f;
                        if (!WHOLE && i >= rows) continue;
                        float in[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) in[k] = i ? h[i ? i - 1 : 0][k] : before[k];
                        bool begins = false;
                        if (!WHOLE) {
                            if (t0 + i < now.start) {
                                now.back(p.rows, t0 + i);
                                load_states(r, p.dlast, now.n, l, p.D, p.S);
                            }
                            begins = t0 + i == now.start;
                            if (begins) load_states(in, p.h0, now.n, l, p.D, p.S);
                        }
                        const Float4 s = it[i][c];
                        const Float4 b = bc[i][0][q], cc = bc[i][1][q];
                        float over[8];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const float lam = r[k] + cc[k] * s.z;
                            over[k] = lam * s.y;
                            over[4 + k] = s.z * h[i][k];
                            two[2 * u] += lam * b[k];
                            r[k] = __builtin_amdgcn_exp2f(s.x * (A[k] * kLog2e)) * lam;
                            const float g = r[k] * in[k];
                            dA[k] += s.x * g;
                            two[2 * u + 1] += A[k] * g;
                        }
                        sum_channels<Q>(over);
                        if ((lane & channels_same<Q>) == 0) {
#pragma unroll
                            for (int j = 0; j < channels_keep<Q>; ++j) red[wave][i][q][channels_first<Q>(lane) + j] = over[j];
                        }
                        if (!WHOLE && begins) store_states(p.dh0, now.n, l, p.D, p.S, r);
                    }
                    sum_lanes<Q>(two);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int j = 0; j < lanes_keep<Q>; ++j) {
                        const int e = of_lanes<Q>(lane, j);
                        reinterpret_cast<float*>(&it[i0 + (e >> 1)][c])[1 + (e & 1)] = two[j];
                    }
                }
                if (WHOLE && first.start == t0) store_states(p.dh0, first.n, l, p.D, p.S, r);
            };
            if (rows == R && first.start <= t0 && first.end >= t0 + R) there_and_back(std::true_type{});
            else there_and_back(std::false_type{});
            seq = first;
            if (t0 > lo && seq.start == t0) {   // the rows in front are another sequence's
                seq.back(p.rows, t0 - 1);
                load_states(r, p.dlast, seq.n, l, p.D, p.S);
            }
            lds_barrier();
            {
                const Tile dxs = tile_at(p.dx, p.stride_x, t0, place.ch0), dds = tile_at(p.ddt, p.stride_dt, t0, place.ch0), dzs = tile_at(p.z ? p.dz : p.dx, p.stride_z, t0, place.ch0);
#pragma unroll
                for (int j = 0; j < kItems; ++j) {
                    const int i = row0 + j * kStep;
                    const bool on = count > 0 && i < rows;
                    float dx[4], ddt[4], dz[4];
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        const Float4 s = it[i < R ? i : 0][c4 + v];
                        float gate = 1.0f, slope = 0.0f;
                        if (p.z) silu_both<BF16>(z[j][v], gate, slope);   // (the hardware's functions, as fast_silu)
                        const float out = dy[j][v] * gate;
                        dx[v] = s.x * s.y + skip[v] * out;
                        ddt[v] = (s.z + x[j][v] * s.y) * (p.softplus ? softplus_slope(dt_in[j][v] + bias[v]) : 1.0f);
                        dz[v] = dy[j][v] * (s.w + skip[v] * x[j][v]) * slope;
                        dskip[v] += out * x[j][v];
                        dbias[v] += on ? ddt[v] : 0.0f;
                    }
                    Four<T, VEC>::store(dxs, on ? px.at[j] : kNoColumn, count, dx);
                    Four<T, VEC>::store(dds, on ? pd.at[j] : kNoColumn, count, ddt);
                    if (p.z) Four<T, VEC>::store(dzs, on ? pz.at[j] : kNoColumn, count, dz);
                }
            }
            for (int e = threadIdx.x; e < rows * 8 * Q; e += 256) {
                const int i = e / (8 * Q), k = e % (8 * Q);
                const float* f = &red[0][i][0][0] + k;
                constexpr int step = R * 8 * Q;
                p.part_bc[(((long long)place.block * all_rows + t0 + i) * p.G + place.g) * 8 * Q + k] = (f[0] + f[step]) + (f[2 * step] + f[3 * step]);
            }
            if ((t0 - lo) % kSumRows == 0) hand_over((int)((t0 - lo) / kSumRows));
        }
    }
}

// dB and dC of rows that belong to a sequence: the workgroups' sums, in order.  64 x 16,384 x 32 of them 29 us (4.6 TB/s; with one read on its way 104)
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
        const float* f = p.part_bc + (row * p.G + g) * 2 * SP + (k / 4) * 8 + which * 4 + k % 4;
        float sum = 0.0f;
#pragma unroll 8
        for (int b = 0; b < p.blocks; ++b) sum += f[b * step];
        if (which == 0) reinterpret_cast<T*>(p.dB)[row * p.stride_B + g * p.S + k] = (T)sum;
        else reinterpret_cast<T*>(p.dC)[row * p.stride_C + g * p.S + k] = (T)sum;
    }
}

template <typename T, int Q, bool VEC>
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
    if (p.segs > 1) hipLaunchKernelGGL((selscan_rjoin_kernel<T>), dim3((unsigned)((cells * seqs + 255) / 256)), block, 0, stream, p, 4 * Q);
    if (p.rows.T) {
        hipLaunchKernelGGL((selscan_grad_kernel<T, Q, VEC>), grid, block, 0, stream, p, rest);
        const long long want = rows * p.G * 2 * p.S / 256;
        hipLaunchKernelGGL((selscan_bc_kernel<T>), dim3((unsigned)(want < 1 ? 1 : want > 16384 ? 16384 : want)), block, 0, stream, p, 4 * Q);
    }
    hipError_t err = hipGetLastError();
    if (err == hipSuccess && p.dh0 && (p.rows.bounds || !p.rows.T)) err = launch_selscan_empty(p.rows, (long long)p.D * p.S, p.dlast, p.dh0, stream);
    if (err != hipSuccess) return err;
    const long long parts = p.rows.T ? segs * p.parts_each : 0;
    err = launch_sum_tiles(false, p.part_A, parts, SumInto{p.dA, nullptr, p.D * p.S, 1, false}, stream);
    if (err != hipSuccess || (!p.dskip && !p.dbias)) return err;
    return launch_sum_tiles(false, p.part_d, parts, SumInto{p.dskip, p.dbias, p.D, 1, true}, stream);
}
template <typename T>
hipError_t launch_type(const SelscanParams& p, hipStream_t stream) {
    switch (scan_lanes(p.S)) {
        case 1: return p.vec ? launch_lanes<T, 1, true>(p, stream) : launch_lanes<T, 1, false>(p, stream);
        case 2: return p.vec ? launch_lanes<T, 2, true>(p, stream) : launch_lanes<T, 2, false>(p, stream);
        case 4: return p.vec ? launch_lanes<T, 4, true>(p, stream) : launch_lanes<T, 4, false>(p, stream);
        case 8: return p.vec ? launch_lanes<T, 8, true>(p, stream) : launch_lanes<T, 8, false>(p, stream);
        default: return p.vec ? launch_lanes<T, 16, true>(p, stream) : launch_lanes<T, 16, false>(p, stream);
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
