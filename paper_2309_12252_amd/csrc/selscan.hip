// Selective scan: h_t = exp(dt_t A) h_{t-1} + dt_t x_t B_t, y_t = <C_t, h_t> + skip x_t, gated.  Outputs, states between segments, single tokens.
#include <type_traits>

#include "selscan_common.h"
#include "selscan_sums.h"

namespace deer {
namespace {

// y and the final states; the states behind segments; these and the states in front of every kMarkRows rows; these and what comes out at the front of a segment on the way back
enum { kOutputs, kEnds, kMarks, kFronts };

// Bound by the rate of vector instructions once there are eight workgroups a CU: 16,384 rows of 4,096 channels and 16 states in bf16 304 us for outputs (the bytes 104), 212 for the states
// behind segments, 221 with states kept (268 MB); 345 with what comes out at the front too (439 in two kernels; with five wavefronts a SIMD, which spill, 375).  Four wavefronts a SIMD for that one: 309 us for
// 326 without a bound in bf16; in fp32, where 7 to 12 registers spill, 425 for 416, and 320 for 264 with 8 states.  With one workgroup a CU (670 us) half of the time is waiting for LDS; reading it two rows ahead brings that to 480, and costs 340 us with
// eight.  Loads by buffer instructions whose offsets lie out of bounds where there is nothing, so that no lane takes another path and what is ahead stays on its way over the
// barriers.
template <typename T, int Q, int WHAT, bool VEC>
__global__ __launch_bounds__(256, WHAT == kFronts ? 4 : 1) void selscan_kernel(const SelscanParams p, const RestRows rest) {
    using Sh = ScanShape<Q>;
    constexpr int R = Sh::kRows, CW = Sh::kChannels, kAcross = CW / 4, kStep = 256 / kAcross;
    __shared__ Float2 sx[R][CW];       // dt and dt x; y in the place of the latter
    __shared__ Float4 bc[R][2][Q];
    constexpr bool MARKS = WHAT == kMarks || WHAT == kFronts, FRONTS = WHAT == kFronts;
    __shared__ float sdy[FRONTS ? R : 1][FRONTS ? CW : 1];
    if (WHAT == kOutputs) clear_rest(p.rows, rest, blockIdx.x, gridDim.x);
    const ScanPlace place = scan_place<Q>(p);
    long long lo = place.lo;
    const long long hi = place.hi;
    if (lo >= hi) return;
    const int lane = threadIdx.x & 63, q = lane / Sh::kWave, c = (threadIdx.x >> 6) * Sh::kWave + lane % Sh::kWave;
    const ScanLane l{place.ch0 + c, 4 * q, c < place.channels};
    float A2[4], h[4], sum_dt = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) A2[k] = l.on && l.k0 + k < p.S ? p.A[(long long)l.ch * p.S + l.k0 + k] * kLog2e : 0.0f;
    ScanSeq seq;
    if (WHAT == kEnds) {   // only what comes behind the last beginning of a sequence counts
        seq.at(p.rows, place, hi - 1);
        const bool reset = seq.start >= lo;
        if (threadIdx.x == 0) p.resets[place.seg] = reset;
        if (reset) lo = seq.start;
        if (reset) load_states(h, p.h0, seq.n, l, p.D, p.S);
        else
#pragma unroll
            for (int k = 0; k < 4; ++k) h[k] = 0.0f;
    } else {
        seq.at(p.rows, place, lo);
        if (seq.start == lo) load_states(h, p.h0, seq.n, l, p.D, p.S);
        else if (WHAT == kOutputs) load_states(h, p.carry, place.seg, l, p.D, 4 * Q);
        else
#pragma unroll
            for (int k = 0; k < 4; ++k) h[k] = 0.0f;
    }
    bool reset = seq.start == lo;
    // What the rows in front of the segment get from it, a lam of its first row, from zero behind it (or from the end of the sequence that reaches into it): with the product of the
    // factors from its first row on it is a sum along the rows, sum_t (a_lo .. a_t) C_t dy_t, and needs no second pass from the last row.
    bool front = FRONTS && seq.start < lo;
    float through[4], out[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        through[k] = 1.0f;
        out[k] = 0.0f;
    }
    auto front_ends = [&](bool with_sequence) {
        if (!FRONTS || !front) return;
        front = false;
        if (with_sequence) {
            float d[4];
            load_states(d, p.dlast, seq.n, l, p.D, p.S);
#pragma unroll
            for (int k = 0; k < 4; ++k) out[k] += through[k] * d[k];
        }
        // (a product that 32 bits do not hold, and that stays so: the join goes over these rows one by one)
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (!(through[k] <= __FLT_MAX__)) out[k] = __builtin_inff();
        if (threadIdx.x == 0) p.rresets[place.seg] = with_sequence;
        store_states(p.rlocal, place.seg, l, p.D, 4 * Q, out);
        if (q == 0 && l.on) p.rsteps[place.seg * p.D + l.ch] = sum_dt;
    };
    if (FRONTS && !front && threadIdx.x == 0) p.rresets[place.seg] = seq.end <= hi;   // (the segment in front ends with its sequence: nothing is asked of this one)
    // a lane's items: four channels of rows kStep apart
    const int c4 = (threadIdx.x % kAcross) * 4, row0 = threadIdx.x / kAcross, count = place.channels - c4;
    float bias[4], skip[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        bias[i] = p.bias && i < count ? p.bias[place.ch0 + c4 + i] : 0.0f;
        skip[i] = WHAT == kOutputs && p.skip && i < count ? p.skip[place.ch0 + c4 + i] : 0.0f;
    }
    const bool has = c4 < place.channels;
    Places<Sh::kItems> px, pd, pz, py;
    px.set(p.stride_x, row0, kStep, c4, T{});
    pd.set(p.stride_dt, row0, kStep, c4, T{});
    if (WHAT == kOutputs || FRONTS) {
        pz.set(p.stride_z, row0, kStep, c4, T{});
        py.set(p.stride_y, row0, kStep, c4, T{});
    }
    // the same for B and C: four states of a row
    constexpr int kBoth = WHAT == kOutputs || FRONTS ? 2 : 1;
    auto tile_at = [&](const void* first, long long stride, long long r, long long more) { return Tile(reinterpret_cast<const T*>(first) + r * stride + more); };
    // what a tile reads is asked for while the one in front of it is worked on
    Four<T, VEC> nx[Sh::kItems], nd[Sh::kItems], nz[Sh::kItems], ny[Sh::kItems], nb[kBoth][Sh::kQuads];
    auto ask = [&](long long r) {
        const int rows = hi - r < R ? (int)(hi - r) : R;
        const Tile x = tile_at(p.x, p.stride_x, r, place.ch0), d = tile_at(p.dt, p.stride_dt, r, place.ch0);
#pragma unroll
        for (int j = 0; j < Sh::kItems; ++j) {
            const bool on = has && row0 + j * kStep < rows;
            nx[j].load(x, on ? px.at[j] : kNoColumn, count);
            nd[j].load(d, on ? pd.at[j] : kNoColumn, count);
        }
        if (FRONTS) {
            const Tile y = tile_at(p.dy, p.stride_y, r, place.ch0);
#pragma unroll
            for (int j = 0; j < Sh::kItems; ++j) ny[j].load(y, has && row0 + j * kStep < rows ? py.at[j] : kNoColumn, count);
        }
        if ((WHAT == kOutputs || FRONTS) && p.z) {
            const Tile z = tile_at(p.z, p.stride_z, r, place.ch0);
#pragma unroll
            for (int j = 0; j < Sh::kItems; ++j) nz[j].load(z, has && row0 + j * kStep < rows ? pz.at[j] : kNoColumn, count);
        }
#pragma unroll
        for (int w = 0; w < kBoth; ++w) {
            const Tile s = w ? tile_at(p.C, p.stride_C, r, (long long)place.g * p.S) : tile_at(p.B, p.stride_B, r, (long long)place.g * p.S);
            const long long stride = w ? p.stride_C : p.stride_B;
#pragma unroll
            for (int j = 0; j < Sh::kQuads; ++j) {
                const int e = threadIdx.x + j * 256, qq = e % Q, i = e / Q;
                nb[w][j].load(s, i < rows && 4 * qq < p.S ? (unsigned)(i * stride + 4 * qq) * (unsigned)sizeof(T) : kNoColumn, p.S - 4 * qq);
            }
        }
    };
    ask(lo);
    for (long long r = lo; r < hi; r += R) {
        const int rows = hi - r < R ? (int)(hi - r) : R;
        Four<T, VEC> x[Sh::kItems], z[Sh::kItems];
#pragma unroll
        for (int j = 0; j < Sh::kItems; ++j) {
            const int i = row0 + j * kStep;
            x[j] = nx[j];
            if (WHAT == kOutputs) z[j] = nz[j];
            Float2 both[4];
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const float raw = nd[j][v] + bias[v], step = p.softplus ? softplus(raw) : raw;
                both[v] = Float2{step, step * x[j][v]};
            }
            if (kStep * Sh::kItems <= R || i < R) {
#pragma unroll
                for (int v = 0; v < 4; ++v) sx[i][c4 + v] = both[v];
                if constexpr (FRONTS) {
#pragma unroll
                    for (int v = 0; v < 4; ++v) sdy[i][c4 + v] = p.z ? ny[j][v] * fast_silu(nz[j][v]) : ny[j][v];
                }
            }
        }
#pragma unroll
        for (int w = 0; w < kBoth; ++w)
#pragma unroll
            for (int j = 0; j < Sh::kQuads; ++j) {
                const int e = threadIdx.x + j * 256;
                if (R * Q >= 256 || e < R * Q) bc[e / Q][w][e % Q] = Float4{nb[w][j][0], nb[w][j][1], nb[w][j][2], nb[w][j][3]};
            }
        lds_barrier();
        if (r + R < hi) ask(r + R);
        // four rows at a time.  WHOLE: all rows of the tile are there, and of one sequence
        auto go = [&](auto whole, auto fronts) {
            constexpr bool WHOLE = decltype(whole)::value, TO_FRONT = decltype(fronts)::value;
#pragma unroll 2
            for (int i0 = 0; i0 < R; i0 += 4) {
                if (!WHOLE && i0 >= rows) break;
                if (MARKS && (r + i0 - lo) % kMarkRows == 0) {
                    if (!WHOLE && r + i0 == seq.end) {
                        front_ends(true);
                        seq.next(p.rows, r + i0);
                        load_states(h, p.h0, seq.n, l, p.D, p.S);
                        reset = true;
                    }
                    const long long mark = place.seg * p.marks_each + (r + i0 - lo) / kMarkRows;
                    store_states(p.marks, mark, l, p.D, 4 * Q, h);
                    if (q == 0 && l.on) p.mark_steps[mark * p.D + l.ch] = sum_dt;
                }
                float y[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int i = i0 + u;
                    y[u] = 0.0f;
                    if (!WHOLE && i >= rows) continue;
                    if (!WHOLE && r + i == seq.end) {
                        if (WHAT == kOutputs) store_states(p.last, seq.n, l, p.D, p.S, h);
                        front_ends(true);
                        seq.next(p.rows, r + i);
                        load_states(h, p.h0, seq.n, l, p.D, p.S);
                        reset = true;
                    }
                    const Float2 s = sx[i][c];
                    const Float4 b = bc[i][0][q];
                    if (WHAT != kOutputs) sum_dt += s.x;
                    float a[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        a[k] = __builtin_amdgcn_exp2f(s.x * A2[k]);
                        h[k] = a[k] * h[k] + s.y * b[k];
                    }
                    if constexpr (TO_FRONT) {
                        if (WHOLE || front) {
                            const float dy = sdy[i][c];
                            const Float4 cc = bc[i][1][q];
#pragma unroll
                            for (int k = 0; k < 4; ++k) {
                                through[k] *= a[k];
                                out[k] += through[k] * (cc[k] * dy);
                            }
                        }
                    }
                    if (WHAT != kOutputs) continue;
                    const Float4 cc = bc[i][1][q];
#pragma unroll
                    for (int k = 0; k < 4; ++k) y[u] += cc[k] * h[k];
                }
                if (WHAT != kOutputs) continue;
                sum_lanes<Q>(y);
#pragma unroll
                for (int j = 0; j < lanes_keep<Q>; ++j) sx[i0 + of_lanes<Q>(lane, j)][c].y = y[j];
            }
        };
        using Fronts = std::bool_constant<FRONTS>;
        if (!(rows == R && seq.end >= r + R)) go(std::false_type{}, Fronts{});
        else if (FRONTS && front) go(std::true_type{}, Fronts{});
        else go(std::true_type{}, std::false_type{});
        lds_barrier();
        if (WHAT == kOutputs) {
            const Tile ys = tile_at(p.y, p.stride_y, r, place.ch0);
#pragma unroll
            for (int j = 0; j < Sh::kItems; ++j) {
                const int i = row0 + j * kStep;
                float y[4];
#pragma unroll
                for (int v = 0; v < 4; ++v) y[v] = sx[i < R ? i : 0][c4 + v].y + skip[v] * x[j][v];
                if (p.z)
#pragma unroll
                    for (int v = 0; v < 4; ++v) y[v] *= fast_silu(z[j][v]);
                Four<T, VEC>::store(ys, has && i < rows ? py.at[j] : kNoColumn, count, y);
            }
        }
        // the tile behind a whole one may begin with another sequence
        if (r + R < hi && r + R == seq.end) {
            if (WHAT == kOutputs) store_states(p.last, seq.n, l, p.D, p.S, h);
            front_ends(true);
            seq.next(p.rows, r + R);
            load_states(h, p.h0, seq.n, l, p.D, p.S);
            reset = true;
        }
    }
    if (WHAT == kOutputs) {
        if (hi == seq.end) store_states(p.last, seq.n, l, p.D, p.S, h);
        return;
    }
    if (p.segs == 1) return;
    front_ends(hi == seq.end);
    if (MARKS && threadIdx.x == 0) p.resets[place.seg] = reset;
    store_states(p.local, place.seg, l, p.D, 4 * Q, h);
    if (q == 0 && l.on) p.steps[place.seg * p.D + l.ch] = sum_dt;
}

// The states in front of the segments, one after the other
__global__ __launch_bounds__(256) void selscan_join_kernel(const SelscanParams p, int SP) {
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x, cells = (long long)p.D * SP, seqs = p.rows.packed ? 1 : p.rows.N;
    if (at >= cells * seqs) return;
    const long long n = at / cells, cell = at % cells;
    const int ch = (int)(cell / SP), k = (int)(cell % SP);
    const float A2 = k < p.S ? p.A[(long long)ch * p.S + k] * kLog2e : 0.0f;
    float h = 0.0f;
    const long long first = n * p.segs;
    for (int s0 = 0; s0 < p.segs - 1; s0 += 8) {   // (eight at a time: what is asked for does not wait for what is written)
        float local[8], steps[8];
        int reset[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const long long s = first + (s0 + i < p.segs - 1 ? s0 + i : p.segs - 2);
            local[i] = p.local[s * cells + cell];
            steps[i] = p.steps[s * p.D + ch];
            reset[i] = p.resets[s];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            if (s0 + i >= p.segs - 1) break;
            h = reset[i] ? local[i] : local[i] + scaled(h, A2 * steps[i]);
            p.carry[(first + s0 + i + 1) * cells + cell] = h;
        }
    }
}

__global__ __launch_bounds__(256) void selscan_empty_kernel(const SeqRows rows, long long cells, const float* from, float* to) {
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < rows.N * cells; i += (long long)gridDim.x * 256)
        if (seq_length(rows, (int)(i / cells)) == 0) to[i] = from ? from[i] : 0.0f;
}

// One token for every row.  A lane has four states of a channel, the lanes of a channel lie side by side: states are read and written as they lie (VEC: in one piece).  Memory bound and
// latency: 64 rows of 4,096 channels and 16 states, 36 MB, 12 us (21 with single loads; the bytes 7), 16 with the call from Python.
template <typename T, int Q, bool VEC>
__global__ __launch_bounds__(256) void selscan_step_kernel(const SelstepParams p) {
    constexpr int CW = 256 / Q;
    const int per = (p.D + CW - 1) / CW, n = blockIdx.x / per, ch = (blockIdx.x % per) * CW + (int)threadIdx.x / Q, q = threadIdx.x % Q;
    int slot = n;
    bool twice = false;
    if (p.rows.slots) {
        slot = p.rows.slots[n];
        for (int m = threadIdx.x; m < n; m += 256) twice = twice || p.rows.slots[m] == slot;
    }
    const bool in = ch < p.D && slot >= 0 && slot < p.rows.n_slots, lane = in && 4 * q < p.S;
    const ScanLane l{ch, 4 * q, in};
    Float4 h = {}, a = {}, b = {}, c = {};
    float x = 0.0f, dt = 0.0f, z = 0.0f, skip = 0.0f;
    float* const state = p.state + ((long long)slot * p.D + ch) * p.S + 4 * q;
    if (lane) {
        const long long group = (long long)(ch / (p.D / p.G)) * p.S + 4 * q;
        const T* bs = reinterpret_cast<const T*>(p.B) + (long long)n * p.stride_B + group;
        const T* cs = reinterpret_cast<const T*>(p.C) + (long long)n * p.stride_C + group;
        const float* as = p.A + (long long)ch * p.S + 4 * q;
        if constexpr (VEC) {
            h = *reinterpret_cast<const Float4*>(state);
            a = *reinterpret_cast<const Float4*>(as);
            const vec_t<T, 4> b4 = *reinterpret_cast<const vec_t<T, 4>*>(bs), c4 = *reinterpret_cast<const vec_t<T, 4>*>(cs);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                b[k] = (float)b4[k];
                c[k] = (float)c4[k];
            }
        } else {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (4 * q + k < p.S) {
                    h[k] = state[k];
                    a[k] = as[k];
                    b[k] = (float)bs[k];
                    c[k] = (float)cs[k];
                }
        }
    }
    if (in) {
        x = (float)reinterpret_cast<const T*>(p.x)[(long long)n * p.stride_x + ch];
        dt = (float)reinterpret_cast<const T*>(p.dt)[(long long)n * p.stride_dt + ch] + (p.bias ? p.bias[ch] : 0.0f);
        if (p.z) z = (float)reinterpret_cast<const T*>(p.z)[(long long)n * p.stride_z + ch];
        if (p.skip) skip = p.skip[ch];
    }
    twice = p.rows.slots ? __syncthreads_or(twice) != 0 : false;
    T* y = reinterpret_cast<T*>(p.y) + (long long)n * p.stride_y + ch;
    if (ch < p.D && (!in || twice)) {
        if (p.rows.zero_rest && q == 0) *y = (T)0.0f;
        return;
    }
    if (p.softplus) dt = softplus(dt);
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        h[k] = __builtin_amdgcn_exp2f(dt * a[k] * kLog2e) * h[k] + dt * x * b[k];
        sum += c[k] * h[k];
    }
#pragma unroll
    for (int d = 1; d < Q; d *= 2) sum += __shfl_xor(sum, d);
    if (lane) {
        if constexpr (VEC) *reinterpret_cast<Float4*>(state) = h;
        else
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (4 * q + k < p.S) state[k] = h[k];
    }
    if (!in || q != 0) return;
    sum += skip * x;
    *y = (T)(p.z ? sum * fast_silu(z) : sum);
}

template <typename T, int Q, bool VEC>
hipError_t launch_lanes(const SelscanParams& p, bool marks, hipStream_t stream) {
    const long long seqs = p.rows.packed ? 1 : p.rows.N, segs = seqs * p.segs, cells = (long long)p.D * 4 * Q;
    const dim3 grid((unsigned)(segs * p.G * p.blocks)), block(256);
    RestRows rest{};
    if (p.zero_rest) rest.array[rest.count++] = RestArray{p.y, p.stride_y * (long long)sizeof(T), p.D * (long long)sizeof(T)};
    if (marks) {
        if (p.segs > 1) hipLaunchKernelGGL((selscan_kernel<T, Q, kFronts, VEC>), grid, block, 0, stream, p, rest);
        else if (p.rows.T) hipLaunchKernelGGL((selscan_kernel<T, Q, kMarks, VEC>), grid, block, 0, stream, p, rest);
    } else if (p.segs > 1) {
        hipLaunchKernelGGL((selscan_kernel<T, Q, kEnds, VEC>), grid, block, 0, stream, p, rest);
    }
    if (p.segs > 1) hipLaunchKernelGGL(selscan_join_kernel, dim3((unsigned)((cells * seqs + 255) / 256)), block, 0, stream, p, 4 * Q);
    if (marks) return hipGetLastError();
    if (p.rows.T) hipLaunchKernelGGL((selscan_kernel<T, Q, kOutputs, VEC>), grid, block, 0, stream, p, rest);
    if (p.last && (p.rows.bounds || !p.rows.T)) {
        const long long all = (long long)p.rows.N * p.D * p.S / 1024;
        hipLaunchKernelGGL(selscan_empty_kernel, dim3((unsigned)(all < 1 ? 1 : all > 1024 ? 1024 : all)), block, 0, stream, p.rows, (long long)p.D * p.S, p.h0, p.last);
    }
    return hipGetLastError();
}
template <typename T>
hipError_t launch_type(const SelscanParams& p, bool marks, hipStream_t stream) {
    switch (scan_lanes(p.S)) {
        case 1: return p.vec ? launch_lanes<T, 1, true>(p, marks, stream) : launch_lanes<T, 1, false>(p, marks, stream);
        case 2: return p.vec ? launch_lanes<T, 2, true>(p, marks, stream) : launch_lanes<T, 2, false>(p, marks, stream);
        case 4: return p.vec ? launch_lanes<T, 4, true>(p, marks, stream) : launch_lanes<T, 4, false>(p, marks, stream);
        case 8: return p.vec ? launch_lanes<T, 8, true>(p, marks, stream) : launch_lanes<T, 8, false>(p, marks, stream);
        default: return p.vec ? launch_lanes<T, 16, true>(p, marks, stream) : launch_lanes<T, 16, false>(p, marks, stream);
    }
}
hipError_t launch_any(int dtype, const SelscanParams& p, bool marks, hipStream_t stream) {
    switch (dtype) {
        case DEER_F32: return launch_type<float>(p, marks, stream);
        case DEER_BF16: return launch_type<BF16>(p, marks, stream);
        default: return launch_type<F16>(p, marks, stream);
    }
}
template <typename T, int Q>
hipError_t launch_step_lanes(const SelstepParams& p, hipStream_t stream) {
    constexpr int CW = 256 / Q;
    const dim3 grid((unsigned)((long long)((p.D + CW - 1) / CW) * p.rows.N)), block(256);
    const bool vec = p.S % 4 == 0 && rows_fit(p.state, 0, 4, 4) && rows_fit(p.A, 0, 4, 4) && rows_fit(p.B, p.stride_B, 4, sizeof(T)) && rows_fit(p.C, p.stride_C, 4, sizeof(T));
    if (vec) hipLaunchKernelGGL((selscan_step_kernel<T, Q, true>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((selscan_step_kernel<T, Q, false>), grid, block, 0, stream, p);
    return hipGetLastError();
}
template <typename T>
hipError_t launch_step_type(const SelstepParams& p, hipStream_t stream) {
    switch (scan_lanes(p.S)) {
        case 1: return launch_step_lanes<T, 1>(p, stream);
        case 2: return launch_step_lanes<T, 2>(p, stream);
        case 4: return launch_step_lanes<T, 4>(p, stream);
        case 8: return launch_step_lanes<T, 8>(p, stream);
        default: return launch_step_lanes<T, 16>(p, stream);
    }
}

}  // namespace

hipError_t launch_selscan(int dtype, const SelscanParams& p, hipStream_t stream) { return launch_any(dtype, p, false, stream); }
hipError_t launch_selscan_marks(int dtype, const SelscanParams& p, hipStream_t stream) { return launch_any(dtype, p, true, stream); }
hipError_t launch_selscan_empty(const SeqRows& rows, long long cells, const float* from, float* to, hipStream_t stream) {
    const long long all = rows.N * cells / 1024;
    hipLaunchKernelGGL(selscan_empty_kernel, dim3((unsigned)(all < 1 ? 1 : all > 1024 ? 1024 : all)), dim3(256), 0, stream, rows, cells, from, to);
    return hipGetLastError();
}
hipError_t launch_selscan_step(int dtype, const SelstepParams& p, hipStream_t stream) {
    switch (dtype) {
        case DEER_F32: return launch_step_type<float>(p, stream);
        case DEER_BF16: return launch_step_type<BF16>(p, stream);
        default: return launch_step_type<F16>(p, stream);
    }
}

}  // namespace deer
