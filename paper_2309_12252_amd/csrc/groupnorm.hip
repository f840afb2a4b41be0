// Group norm with an activation and a gate, channels last: forward and gradient, statistics over rows or over sequences.
#include "lane_sums.h"
#include "layer_common.h"

namespace deer {
namespace {

template <typename T, int V>
__device__ __forceinline__ void load_wide(wide_t<T>* to, const void* from, long long at) {
    const vec_t<T, V> v = *reinterpret_cast<const vec_t<T, V>*>(reinterpret_cast<const T*>(from) + at);
#pragma unroll
    for (int i = 0; i < V; ++i) to[i] = (wide_t<T>)vec_at<T, V>(v, i);
}
template <typename T, int V>
__device__ __forceinline__ void store_narrow(void* to, long long at, const wide_t<T>* from) {
    vec_t<T, V> v;
#pragma unroll
    for (int i = 0; i < V; ++i) vec_set<T, V>(v, i, (T)from[i]);
    *reinterpret_cast<vec_t<T, V>*>(reinterpret_cast<T*>(to) + at) = v;
}

// One element: y of x, or du = dL/du and what else its gradient needs
template <typename T>
struct Through {
    using S = wide_t<T>;
    S u, dv, dz;
    __device__ __forceinline__ S operator()(const NormParams& p, S x, S z, S dy, S mean, S rstd, S w, S b) {
        u = (x - mean) * rstd;
        const S pre = u * w + b;
        S f = pre, slope = S(1), gate = S(1), gslope = S(0);
        if (p.act == DEER_ACT_SILU) silu_both<T>(pre, f, slope);
        if (p.z) silu_both<T>(z, gate, gslope);
        dv = dy * gate * slope;
        dz = dy * f * gslope;
        return dv * w;
    }
};

// ---- every row by itself ----
// How a workgroup goes over rows and groups: L lanes (a power of two) have a group of a row, M vectors of V channels each; groups side by side, then rows
struct RowShape {
    int L, groups, rows, blocks;   // lanes of a group; groups and rows side by side in a workgroup; workgroups along the groups
};
inline RowShape row_shape(int D, int G, int V, int M) {
    const int vecs = D / G / V;
    RowShape s{1, 1, 1, 1};
    while (s.L * M < vecs && s.L < 256) s.L *= 2;
    const int units = 256 / s.L;
    while (s.groups < units && s.groups < G) s.groups *= 2;
    s.rows = units / s.groups;
    s.blocks = (G + s.groups - 1) / s.groups;
    return s;
}

// sum over the L lanes of a group, the same for all of them
template <typename S>
__device__ __forceinline__ S group_sum(S v, int L, S* shared) {
    for (int d = 1; d < L && d < 64; d *= 2) v += __shfl_xor(v, d);
    if (L <= 64) return v;
    const int wave = threadIdx.x >> 6, first = wave / (L / 64) * (L / 64);
    __syncthreads();
    shared[wave] = v;
    __syncthreads();
    v = S(0);
    for (int i = 0; i < L / 64; ++i) v += shared[first + i];
    return v;
}

// whether row (of sequence n where they are padded) belongs to a sequence
__device__ __forceinline__ bool row_counts(const SeqRows& s, long long row) {
    if (!s.bounds) return true;
    if (s.packed) return row >= clamp_row(s.bounds[0], s.T) && row < clamp_row(s.bounds[s.N], s.T);
    const long long n = row <= 0xFFFFFFFFll && s.T <= 0xFFFFFFFFll ? (unsigned)row / (unsigned)s.T : row / s.T;   // (64 bits take many times as long)
    return row - n * s.T < clamp_row(s.bounds[n], s.T);
}

// Wider groups.  M vectors a lane are kept, so that a row is read once; with FEW false groups may have more than 256 M vectors, and are gone over again.  A row at a time, bound by the way to memory and back: 16,384 rows
// of 4,096 channels in one group, with a gate, in bf16 442 us and the gradient 565 (403 MB and 671 MB: 0.9 and 1.2 TB/s), in fp32 233 and 342
template <typename T, int V, int M, bool GRAD, bool FEW>
__global__ __launch_bounds__(256) void rownorm_kernel(const NormParams p, const RowShape s, const RestRows rest, long long rows_each) {
    using S = wide_t<T>;
    __shared__ S shared[4];
    clear_rest(p.rows, rest, blockIdx.x, gridDim.x);
    const int unit = threadIdx.x / s.L, l = threadIdx.x % s.L, n = p.D / p.G, vecs = n / V;
    const int block = blockIdx.x % s.blocks, g = block * s.groups + unit % s.groups, ch0 = g * n;
    const long long rows = p.rows.T * (p.rows.packed ? 1 : p.rows.N), lo = (long long)(blockIdx.x / s.blocks) * rows_each, hi = lo + rows_each < rows ? lo + rows_each : rows;
    const bool has = g < p.G;
    const S count = S(n);
    const int turns = FEW ? 1 : (vecs + s.L * M - 1) / (s.L * M);
    S* part = reinterpret_cast<S*>(p.part) + (long long)(blockIdx.x / s.blocks * s.rows + unit / s.groups) * 2 * p.D;
    S dw[M][V], db[M][V];
#pragma unroll
    for (int m = 0; m < M; ++m)
#pragma unroll
        for (int v = 0; v < V; ++v) dw[m][v] = db[m][v] = S(0);
    auto at = [&](int turn, int m) { return (turn * M + m) * s.L + l; };   // a lane's vectors
    if (GRAD && !FEW && has)
        for (int i = l * V; i < n; i += s.L * V)
#pragma unroll
            for (int v = 0; v < V; ++v) part[ch0 + i + v] = part[p.D + ch0 + i + v] = S(0);
    auto read = [&](const void* from, long long first, int turn, S(*to)[V]) {
#pragma unroll
        for (int m = 0; m < M; ++m) {
            if (at(turn, m) < vecs) load_wide<T, V>(to[m], from, first + ch0 + at(turn, m) * V);
            else
#pragma unroll
                for (int v = 0; v < V; ++v) to[m][v] = S(0);
        }
    };
    // (rounds of the same number for all lanes of the workgroup, for the sums over more than one wavefront)
    for (long long round = lo; round < hi; round += s.rows) {
        const long long row = round + unit / s.groups;
        const bool on = has && row < hi && row_counts(p.rows, row);
        S x[M][V], mean = S(0), rstd = S(0), sum = S(0), dy[M][V], z[M][V];
        const S* stats = reinterpret_cast<const S*>(p.stats) + (row * p.G + g) * 2;
        if (!GRAD) {
            for (int t = 0; t < turns; ++t) {
                if (on) read(p.x, row * p.stride_x, t, x);
#pragma unroll
                for (int m = 0; m < M; ++m)
#pragma unroll
                    for (int v = 0; v < V; ++v) sum += on ? x[m][v] : S(0);
            }
            mean = group_sum(sum, s.L, shared) / count;
            sum = S(0);
            for (int t = 0; t < turns; ++t) {
                if (!FEW && on) read(p.x, row * p.stride_x, t, x);
#pragma unroll
                for (int m = 0; m < M; ++m)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const S off = x[m][v] - mean;
                        sum += on && at(t, m) < vecs ? off * off : S(0);
                    }
            }
            rstd = S(1) / sqrt(group_sum(sum, s.L, shared) / count + (S)p.eps);
            if (on && l == 0) {
                const_cast<S*>(stats)[0] = mean;
                const_cast<S*>(stats)[1] = rstd;
            }
        } else if (on) {
            mean = stats[0];
            rstd = stats[1];
        }
        S s1 = S(0), s2 = S(0);
        // gradient: dy through gate and activation, and its sums
        auto through = [&](int t, int m, int v, S& unit_x, S& dv, S& dz) {
            const int c = ch0 + at(t, m) * V + v;
            const S w = p.w ? reinterpret_cast<const S*>(p.w)[c] : S(1), b = p.bias ? reinterpret_cast<const S*>(p.bias)[c] : S(0);
            Through<T> th;
            const S du = th(p, x[m][v], p.z ? z[m][v] : S(0), dy[m][v], mean, rstd, w, b);
            unit_x = th.u;
            dv = th.dv;
            dz = th.dz;
            return du;
        };
        if (GRAD)
            for (int t = 0; t < turns; ++t) {
                if (!on) break;
                read(p.x, row * p.stride_x, t, x);
                read(p.dy, row * p.stride_y, t, dy);
                if (p.z) read(p.z, row * p.stride_z, t, z);
#pragma unroll
                for (int m = 0; m < M; ++m) {
                    if (at(t, m) >= vecs) continue;
                    S dz[V];
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        S ux, dv;
                        const S du = through(t, m, v, ux, dv, dz[v]);
                        s1 += du;
                        s2 += du * ux;
                        if (FEW) {
                            dw[m][v] += dv * ux;
                            db[m][v] += dv;
                            x[m][v] = ux;
                            dy[m][v] = du;
                        }
                    }
                    if (FEW && p.z) store_narrow<T, V>(p.dz, row * p.stride_z + ch0 + at(t, m) * V, dz);
                }
            }
        if (GRAD) {
            s1 = group_sum(s1, s.L, shared) / count;
            s2 = group_sum(s2, s.L, shared) / count;
        }
        if (!on) continue;
        for (int t = 0; t < turns; ++t) {
            if (!FEW) {
                read(p.x, row * p.stride_x, t, x);
                if (GRAD) read(p.dy, row * p.stride_y, t, dy);
            }
            if (p.z && (!GRAD || !FEW)) read(p.z, row * p.stride_z, t, z);
#pragma unroll
            for (int m = 0; m < M; ++m) {
                if (at(t, m) >= vecs) continue;
                S out[V], dz[V];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const int c = ch0 + at(t, m) * V + v;
                    if (!GRAD) {
                        const S w = p.w ? reinterpret_cast<const S*>(p.w)[c] : S(1), b = p.bias ? reinterpret_cast<const S*>(p.bias)[c] : S(0);
                        const S pre = (x[m][v] - mean) * rstd * w + b;
                        out[v] = p.act == DEER_ACT_SILU ? silu<T>(pre) : pre;
                        if (p.z) out[v] *= silu<T>(z[m][v]);
                    } else {
                        S ux = x[m][v], du = dy[m][v], dv;
                        if (!FEW) {
                            du = through(t, m, v, ux, dv, dz[v]);
                            // (a lane's own element of the workgroup's sums: read and written by no other)
                            S* own = part + c;
                            own[0] += dv * ux;
                            own[p.D] += dv;
                        }
                        out[v] = rstd * ((du - s1) - ux * s2);
                    }
                }
                store_narrow<T, V>(GRAD ? p.dx : p.y, row * (GRAD ? p.stride_x : p.stride_y) + ch0 + at(t, m) * V, out);
                if (GRAD && !FEW && p.z) store_narrow<T, V>(p.dz, row * p.stride_z + ch0 + at(t, m) * V, dz);
            }
        }
    }
    if (GRAD && FEW && has) {
#pragma unroll
        for (int m = 0; m < M; ++m)
            if (at(0, m) < vecs)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    part[ch0 + at(0, m) * V + v] = dw[m][v];
                    part[p.D + ch0 + at(0, m) * V + v] = db[m][v];
                }
    }
}


// sums over the L lanes of a group, of B values side by side, the same for all lanes
template <typename S, int B>
__device__ __forceinline__ void lanes_sum(S (&v)[B], int L) {
    if constexpr (sizeof(S) == 8) {
        for (int d = 1; d < L; d *= 2)
#pragma unroll
            for (int b = 0; b < B; ++b) v[b] += __shfl_xor(v[b], d);
    } else {
        if (L > 1)
#pragma unroll
            for (int b = 0; b < B; ++b) v[b] = dpp_add<kSwapLanes>(v[b]);
        if (L > 2)
#pragma unroll
            for (int b = 0; b < B; ++b) v[b] = dpp_add<kSwapPairs>(v[b]);
        if (L > 4)
#pragma unroll
            for (int b = 0; b < B; ++b) v[b] = dpp_add<kHalfMirror>(v[b]);
        if (L > 8)
#pragma unroll
            for (int b = 0; b < B; ++b) v[b] = dpp_add<kMirror>(v[b]);
        if (L > 16)
#pragma unroll
            for (int b = 0; b < B; ++b) v[b] = sum_rows(v[b], v[b]);
        if (L > 32)
#pragma unroll
            for (int b = 0; b < B; ++b) v[b] = sum_halves(v[b], v[b]);
    }
}

// Groups of at most 64 vectors, a vector a lane, B rows at a time so that their loads and sums overlap.  Memory bound: 16,384 rows of 16 x 128 channels in bf16 with a gate, 201 MB in 52 us
// (3.9 TB/s), the gradient's 335 MB in 81; a row at a time, sums through LDS, 155 and 176.  16 bytes a lane: with 8 the gradient takes 110.
template <typename T, int V, int B, bool GRAD>
__global__ __launch_bounds__(256) void rownorm_few_kernel(const NormParams p, const RowShape s, const RestRows rest, long long rows_each) {
    using S = wide_t<T>;
    const int unit = threadIdx.x / s.L, l = threadIdx.x % s.L, n = p.D / p.G, lane_row = unit / s.groups;
    const int g = blockIdx.x % s.blocks * s.groups + unit % s.groups;
    const bool has = g < p.G && l * V < n;
    const int ch = has ? g * n + l * V : 0;
    const long long block = blockIdx.x / s.blocks, rows = p.rows.T * (p.rows.packed ? 1 : p.rows.N), lo = block * rows_each, hi = lo + rows_each < rows ? lo + rows_each : rows;
    const long long from = p.rows.packed ? clamp_row(p.rows.bounds[0], p.rows.T) : 0, to = p.rows.packed ? clamp_row(p.rows.bounds[p.rows.N], p.rows.T) : rows;
    const bool lengths = !p.rows.packed && p.rows.bounds;
    const S share = S(1) / S(n);
    S w[V], bias[V], dw[V], db[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        w[v] = p.w && has ? reinterpret_cast<const S*>(p.w)[ch + v] : S(1);
        bias[v] = p.bias && has ? reinterpret_cast<const S*>(p.bias)[ch + v] : S(0);
        dw[v] = db[v] = S(0);
    }
    for (long long round = lo + lane_row; round < hi; round += s.rows * B) {
        bool on[B];
        S x[B][V], y[B][V], z[B][V], mean[B], rstd[B], one[B], two[B];
        long long row[B];
#pragma unroll
        for (int b = 0; b < B; ++b) {
            row[b] = round + b * s.rows < hi ? round + b * s.rows : round;   // (a row again where there are no more: not written)
            on[b] = has && round + b * s.rows < hi && (lengths ? row_counts(p.rows, row[b]) : row[b] >= from && row[b] < to);
            load_wide<T, V>(x[b], p.x, row[b] * p.stride_x + ch);
            if (p.z) load_wide<T, V>(z[b], p.z, row[b] * p.stride_z + ch);
            if (GRAD) {
                load_wide<T, V>(y[b], p.dy, row[b] * p.stride_y + ch);
                const S* stats = reinterpret_cast<const S*>(p.stats) + (row[b] * p.G + (has ? g : 0)) * 2;
                mean[b] = stats[0];
                rstd[b] = stats[1];
            }
        }
#pragma unroll
        for (int b = 0; b < B; ++b) {
            one[b] = two[b] = S(0);
            if (!GRAD)
#pragma unroll
                for (int v = 0; v < V; ++v) one[b] += has ? x[b][v] : S(0);
        }
        if (!GRAD) {
            lanes_sum(one, s.L);
#pragma unroll
            for (int b = 0; b < B; ++b) {
                mean[b] = one[b] / S(n);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const S off = x[b][v] - mean[b];
                    two[b] += has ? off * off : S(0);
                }
            }
            lanes_sum(two, s.L);
#pragma unroll
            for (int b = 0; b < B; ++b) {
                rstd[b] = S(1) / sqrt(two[b] * share + (S)p.eps);
                S* stats = reinterpret_cast<S*>(p.stats) + (row[b] * p.G + g) * 2;
                if (on[b] && l == 0) {
                    stats[0] = mean[b];
                    stats[1] = rstd[b];
                }
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const S pre = (x[b][v] - mean[b]) * rstd[b] * w[v] + bias[v];
                    y[b][v] = p.act == DEER_ACT_SILU ? silu<T>(pre) : pre;
                }
                if (p.z)
#pragma unroll
                    for (int v = 0; v < V; ++v) y[b][v] *= silu<T>(z[b][v]);
                if (on[b]) store_narrow<T, V>(p.y, row[b] * p.stride_y + ch, y[b]);
            }
            continue;
        }
        // x becomes u = (x - mean) rstd, y dL/du
#pragma unroll
        for (int b = 0; b < B; ++b) {
            S dz[V];
#pragma unroll
            for (int v = 0; v < V; ++v) {
                Through<T> th;
                const S du = th(p, x[b][v], p.z ? z[b][v] : S(0), y[b][v], mean[b], rstd[b], w[v], bias[v]);
                x[b][v] = th.u;
                y[b][v] = du;
                dz[v] = th.dz;
                one[b] += has ? du : S(0);
                two[b] += has ? du * th.u : S(0);
                dw[v] += on[b] ? th.dv * th.u : S(0);
                db[v] += on[b] ? th.dv : S(0);
            }
            if (p.z && on[b]) store_narrow<T, V>(p.dz, row[b] * p.stride_z + ch, dz);
        }
        lanes_sum(one, s.L);
        lanes_sum(two, s.L);
#pragma unroll
        for (int b = 0; b < B; ++b) {
            const S s1 = n > 1 ? one[b] * share : one[b], s2 = two[b] * share;
#pragma unroll
            for (int v = 0; v < V; ++v) y[b][v] = rstd[b] * ((y[b][v] - s1) - x[b][v] * s2);
            if (on[b]) store_narrow<T, V>(p.dx, row[b] * p.stride_x + ch, y[b]);
        }
    }
    clear_rest(p.rows, rest, blockIdx.x, gridDim.x);
    if (!GRAD || !has) return;
    S* part = reinterpret_cast<S*>(p.part) + (block * s.rows + lane_row) * 2 * p.D + ch;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        part[v] = dw[v];
        part[p.D + v] = db[v];
    }
}

// ---- statistics over sequences ----
// Pieces of sequences in tiles have places of their own: tile + sequence where rows are packed (one of the two grows from a piece to the next)
__device__ __forceinline__ long long piece_at(const SeqRows& s, long long tile, int seq) { return s.packed ? tile + seq : tile; }

struct SpanPlace {
    int n, ch, phase;
    long long tile, lo, hi;
    bool on;
};
template <int V>
__device__ __forceinline__ SpanPlace span_place(const NormParams& p, const Lanes& l, int rows) {
    const long long tiles = (p.rows.T + rows - 1) / rows;
    SpanPlace at;
    at.tile = blockIdx.x / l.blocks;
    at.n = p.rows.packed ? 0 : (int)(at.tile / tiles);
    at.ch = ((int)(blockIdx.x % l.blocks) * l.lanes + (int)(threadIdx.x & (l.lanes - 1))) * V;
    at.phase = threadIdx.x / l.lanes;
    at.on = at.ch < p.D;
    const long long in = (p.rows.packed ? at.tile : at.tile % tiles) * rows, base = (long long)at.n * p.rows.T;
    at.lo = base + in;
    at.hi = base + (in + rows < p.rows.T ? in + rows : p.rows.T);
    return at;
}

// sums of two values a channel over the phases; those of phase 0 get them: over the phases of a wavefront, then over the wavefronts
template <typename S, int V>
__device__ __forceinline__ void phase_sums(S (*two)[V], const Lanes& l, S* shared) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int d = l.lanes; d < 64; d *= 2)
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int v = 0; v < V; ++v) two[k][v] += __shfl_xor(two[k][v], d);
    __syncthreads();
    if (wave > 0 && lane < l.lanes)
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int v = 0; v < V; ++v) shared[((wave * 2 + k) * 64 + lane) * V + v] = two[k][v];
    __syncthreads();
    if ((int)threadIdx.x < l.lanes)
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int f = 1; f < 4; ++f) two[k][v] += shared[((f * 2 + k) * 64 + lane) * V + v];
}
constexpr int kPhaseRoom = 4 * 2 * 64;

// Of a lane's rows of a piece: mean = hi + lo, and the sum of squares about it
template <typename S, int V>
struct Moments {
    S hi[V], lo[V], squares[V];
    int rows;
};
// sum over the phases of a wavefront, `lanes` apart, the same for all of them
template <typename S>
__device__ __forceinline__ S wave_phases(S v, int lanes) {
    if constexpr (sizeof(S) == 8) {
        for (int d = lanes; d < 64; d *= 2) v += __shfl_xor(v, d);
    } else {
        if (lanes <= 1) v = dpp_add<kSwapLanes>(v);
        if (lanes <= 2) v = dpp_add<kSwapPairs>(v);
        if (lanes <= 4) v = dpp_add<kRor4>(v);
        if (lanes <= 8) v = dpp_add<kRor8>(v);
        if (lanes <= 16) v = sum_rows(v, v);
        if (lanes <= 32) v = sum_halves(v, v);
    }
    return v;
}
__device__ __forceinline__ float inverse(float v) { return __builtin_amdgcn_rcpf(v); }   // (of a number of rows: off by 1 ulp, which a mean's distance from its offset takes)
__device__ __forceinline__ double inverse(double v) { return 1.0 / v; }

// The phases' moments joined; those of phase 0 get them.  Within a wavefront in two passes as over single values, first the mean and then the squares about it, in differences from its first phase's mean;
// then the wavefronts' one after another: nothing is the small difference of large sums.  hi + lo: differences between means far from zero keep their digits.
template <typename S, int V>
__device__ __forceinline__ void phase_moments(Moments<S, V>& m, const Lanes& l, S* shared, int* rows) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (l.lanes < 64) {
        S first[V], off[V], sum[V];
        const S all = wave_phases((S)m.rows, l.lanes);   // (at most 2,048: exact)
#pragma unroll
        for (int v = 0; v < V; ++v) {
            first[v] = __shfl(m.hi[v], lane & (l.lanes - 1));
            off[v] = m.rows ? (m.hi[v] - first[v]) + m.lo[v] : S(0);
            sum[v] = wave_phases((S)m.rows * off[v], l.lanes);
        }
        const S share = all > S(0) ? inverse(all) : S(0);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            sum[v] *= share;
            off[v] -= sum[v];
            m.squares[v] = wave_phases(m.squares[v] + (S)m.rows * off[v] * off[v], l.lanes);
            m.hi[v] = first[v] + sum[v];
            m.lo[v] = (first[v] - m.hi[v]) + sum[v];
        }
        m.rows = (int)all;
    }
    __syncthreads();
    if (wave > 0 && lane < l.lanes) {
#pragma unroll
        for (int v = 0; v < V; ++v) {
            shared[((wave * 3 + 0) * 64 + lane) * V + v] = m.hi[v];
            shared[((wave * 3 + 1) * 64 + lane) * V + v] = m.lo[v];
            shared[((wave * 3 + 2) * 64 + lane) * V + v] = m.squares[v];
        }
        if (lane == 0) rows[wave] = m.rows;
    }
    __syncthreads();
    if ((int)threadIdx.x >= l.lanes) return;
    for (int f = 1; f < 4; ++f) {
        if (rows[f] == 0) break;   // (nor do those behind it have any)
        const int all = m.rows + rows[f];
        const S share = (S)rows[f] * inverse((S)all);
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const S hi = shared[((f * 3 + 0) * 64 + lane) * V + v], lo = shared[((f * 3 + 1) * 64 + lane) * V + v];
            const S apart = (hi - m.hi[v]) + (lo - m.lo[v]), by = m.lo[v] + share * apart, mean = m.hi[v] + by;
            m.squares[v] += shared[((f * 3 + 2) * 64 + lane) * V + v] + (S)m.rows * share * apart * apart;
            m.lo[v] = (m.hi[v] - mean) + by;
            m.hi[v] = mean;
        }
        m.rows = all;
    }
}
constexpr int kMomentRoom = 4 * 3 * 64;

// Mean and sum of squares about it, of every channel in every piece.  A lane sums the differences from the mean of its first eight rows: whatever value lies far off is one of the summed, and the squares about the
// lane's own mean are at least a quarter of those about that offset (32 rows at most), so that no more than two bits cancel.  (Differences from a piece's first row lose a factor of the piece's rows, up to 8,192, where that row lies far
// off: rstd was off by 7e-5 behind a first row 100 deviations away.)  32,768 rows of 2,560 channels in bf16, 168 MB, 44 us (3.8 TB/s; 75
// without rows on their way); 32 x 17,984 rows of 16 in fp32 11.8 (10.0 with differences from first rows, 13.7 with sums by shuffles).
template <typename T, int V>
__global__ __launch_bounds__(256) void moments_kernel(const NormParams p, const Lanes l, int rows, const RestRows rest) {
    using S = wide_t<T>;
    __shared__ S shared[kMomentRoom * V];
    __shared__ int counts[4];
    const SpanPlace at = span_place<V>(p, l, rows);
    for_runs(p.rows, at.n, at.lo, at.hi, [&](int seq, long long, long long, long long r0, long long r1) {
        const int many = (int)(r1 - r0) - at.phase;
        Moments<S, V> m{};
        m.rows = many > 0 ? (int)((unsigned)(many + l.phases - 1) / (unsigned)l.phases) : 0;
        if (at.on && m.rows) {
            // eight rows at a time, the next eight on their way
            using TV = vec_t<T, V>;
            constexpr int B = 8;
            const long long step = l.phases * p.stride_x;
            const T* from = reinterpret_cast<const T*>(p.x) + (r0 + at.phase) * p.stride_x + at.ch;
            TV now[B], next[B];
            auto ask = [&](long long r) {   // (rows behind the last: the first of the piece)
                if (r + (B - 1) * l.phases < r1) {
#pragma unroll
                    for (int i = 0; i < B; ++i) next[i] = *reinterpret_cast<const TV*>(from + i * step);
                } else {
                    const T* first_row = reinterpret_cast<const T*>(p.x) + r0 * p.stride_x + at.ch;
#pragma unroll
                    for (int i = 0; i < B; ++i) next[i] = *reinterpret_cast<const TV*>(r + i * l.phases < r1 ? from + i * step : first_row);
                }
                from += B * step;
            };
            ask(r0 + at.phase);
            S first[V] = {}, two[2][V] = {};
            const S part = inverse((S)(m.rows < B ? m.rows : B));
#pragma unroll
            for (int i = 0; i < B; ++i)
                if (i < m.rows)
#pragma unroll
                    for (int v = 0; v < V; ++v) first[v] += part * (S)vec_at<T, V>(next[i], v);
            for (int left = m.rows; left > 0; left -= B) {
#pragma unroll
                for (int i = 0; i < B; ++i) now[i] = next[i];
                if (left > B) ask(r0 + at.phase + (long long)(m.rows - left + B) * l.phases);
                auto add = [&](int i) {
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        const S off = (S)vec_at<T, V>(now[i], v) - first[v];
                        two[0][v] += off;
                        two[1][v] += off * off;
                    }
                };
                if (left >= B) {
#pragma unroll
                    for (int i = 0; i < B; ++i) add(i);
                } else {
#pragma unroll
                    for (int i = 0; i < B; ++i)
                        if (i < left) add(i);
                }
            }
            const S share = inverse((S)m.rows);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const S mean = two[0][v] * share, squares = two[1][v] - two[0][v] * mean;
                m.hi[v] = first[v] + mean;
                m.lo[v] = (first[v] - m.hi[v]) + mean;
                m.squares[v] = squares > S(0) || !(squares <= S(0)) ? squares : S(0);   // (NaN stays)
            }
        }
        phase_moments<S, V>(m, l, shared, counts);
        if (!at.on || (int)threadIdx.x >= l.lanes) return;
        S* to = reinterpret_cast<S*>(p.part) + piece_at(p.rows, at.tile, seq) * 2 * p.D + at.ch;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            to[v] = m.hi[v] + m.lo[v];
            to[p.D + v] = m.squares[v];
        }
    });
    clear_rest(p.rows, rest, blockIdx.x, gridDim.x);
}

constexpr int kJoinLanes = 1024;
__device__ __forceinline__ double block_sum(double v, double* shared) {
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
#pragma unroll
    for (int i = 0; i < kJoinLanes / 64; ++i) v += shared[i];
    return v;
}

// Over a sequence's pieces and a group's channels, in 64 bits: mean and rstd (grad false), or the sums of dL/du and of dL/du u, u = (x - mean) rstd, over the number of
// values (grad true).  Nine sequences of 32,768 rows in all, 32 groups of 80 channels: 10 us, mostly the way of two rounds of loads (16 with lanes in rows of 128 a tile)
template <typename S>
__global__ __launch_bounds__(kJoinLanes) void join_kernel(const NormParams p, int rows, bool grad) {
    __shared__ double shared[kJoinLanes / 64];
    const int seq = blockIdx.x / p.G, g = blockIdx.x % p.G, n = p.D / p.G, ch0 = g * n;
    const long long len = seq_length(p.rows, seq), tiles = (p.rows.T + rows - 1) / rows;
    S* to = reinterpret_cast<S*>(grad ? p.joined : p.stats) + (long long)blockIdx.x * 2;
    if (len == 0) {
        if (threadIdx.x < 2) to[threadIdx.x] = S(0);
        return;
    }
    const long long start = p.rows.packed ? seq_first(p.rows, seq) : 0, first = start / rows, last = (start + len - 1) / rows;
    const S* part = reinterpret_cast<const S*>(p.part) + (p.rows.packed ? (long long)seq : (long long)seq * tiles) * 2 * p.D + ch0;
    const S* w = grad ? reinterpret_cast<const S*>(p.w) : nullptr;
    auto count = [&](long long tile) {
        const long long lo = tile * rows > start ? tile * rows : start, hi = (tile + 1) * rows < start + len ? (tile + 1) * rows : start + len;
        return (double)(hi - lo);
    };
    // a lane takes every 1,024th of the pieces' channels, eight of them on their way; those stay for the second time
    constexpr int B = 8;
    struct Place {
        long long tile;
        int c;
    };
    const Place begin{first + threadIdx.x / n, (int)threadIdx.x % n};
    const int far = kJoinLanes / n, more = kJoinLanes % n;
    auto go_on = [&](Place& at) {
        at.c += more;
        at.tile += far;
        if (at.c >= n) {
            at.c -= n;
            ++at.tile;
        }
    };
    S one[B], two[B], scale[B];
    auto ask = [&](Place at) {
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const bool on = at.tile <= last;
            const S* from = part + (on ? at.tile : first) * 2 * p.D + at.c;
            one[i] = from[0];
            two[i] = from[p.D];
            scale[i] = w ? w[ch0 + at.c] : S(1);
            go_on(at);
        }
    };
    double a = 0, b = 0;
    const bool whole = (last - first + 1) * n <= (long long)B * kJoinLanes;
    for (Place at = begin; at.tile <= last;) {
        ask(at);
#pragma unroll
        for (int i = 0; i < B; ++i) {
            if (at.tile <= last) {
                a += (grad ? (double)scale[i] : count(at.tile)) * (double)one[i];
                if (grad) b += (double)scale[i] * (double)two[i];
            }
            go_on(at);
        }
    }
    const double all = (double)len * n;
    a = block_sum(a, shared) / all;
    if (!grad)
        for (Place at = begin; at.tile <= last;) {
            if (!whole) ask(at);
#pragma unroll
            for (int i = 0; i < B; ++i) {
                if (at.tile <= last) {
                    const double off = (double)one[i] - a;
                    b += (double)two[i] + count(at.tile) * off * off;
                }
                go_on(at);
            }
        }
    b = block_sum(b, shared) / all;
    if (threadIdx.x == 0) {
        to[0] = (S)a;
        to[1] = grad ? (S)b : (S)(1.0 / sqrt(b + p.eps));
    }
}

// Memory bound: y of 32,768 rows of 2,560 channels in bf16 73 us for 335 MB (4.6 TB/s), the gradient's two passes 102 for 335 MB and 111 for 503 MB; fp64, 4 x 4,096 rows of 1,024 with a gate, 67, 96 and 142.  Statistics over a
// sequence read x twice: it is read again while the last-level cache has some of it.
// STEP 0: y; 1: the sums of dL/dv and dL/dv u of every channel in every piece, v = w u + bias, and in every tile; 2: dx and dz
template <typename T, int V, int STEP>
__global__ __launch_bounds__(256) void span_kernel(const NormParams p, const Lanes l, int rows, const RestRows rest) {
    using S = wide_t<T>;
    __shared__ S shared[STEP == 1 ? kPhaseRoom * V : 1];
    const SpanPlace at = span_place<V>(p, l, rows);
    S w[V], b[V], total[2][V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        w[v] = p.w && at.on ? reinterpret_cast<const S*>(p.w)[at.ch + v] : S(1);
        b[v] = p.bias && at.on ? reinterpret_cast<const S*>(p.bias)[at.ch + v] : S(0);
        total[0][v] = total[1][v] = S(0);
    }
    const int g = (at.on ? at.ch : 0) / (p.D / p.G);
    for_runs(p.rows, at.n, at.lo, at.hi, [&](int seq, long long, long long, long long r0, long long r1) {
        const S* stats = reinterpret_cast<const S*>(p.stats) + ((long long)seq * p.G + g) * 2;
        const S mean = stats[0], rstd = stats[1];
        S s1 = S(0), s2 = S(0), two[2][V];
        if (STEP == 2) {
            s1 = reinterpret_cast<const S*>(p.joined)[((long long)seq * p.G + g) * 2];
            s2 = reinterpret_cast<const S*>(p.joined)[((long long)seq * p.G + g) * 2 + 1];
        }
#pragma unroll
        for (int v = 0; v < V; ++v) two[0][v] = two[1][v] = S(0);
        if (at.on)
#pragma unroll 4
            for (long long r = r0 + at.phase; r < r1; r += l.phases) {
                S x[V], z[V], dy[V], out[V], dz[V];
                load_wide<T, V>(x, p.x, r * p.stride_x + at.ch);
                if (p.z) load_wide<T, V>(z, p.z, r * p.stride_z + at.ch);
                if (STEP != 0) load_wide<T, V>(dy, p.dy, r * p.stride_y + at.ch);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    if (STEP == 0) {
                        const S pre = (x[v] - mean) * rstd * w[v] + b[v];
                        out[v] = p.act == DEER_ACT_SILU ? silu<T>(pre) : pre;
                        if (p.z) out[v] *= silu<T>(z[v]);
                    } else {
                        Through<T> th;
                        const S du = th(p, x[v], p.z ? z[v] : S(0), dy[v], mean, rstd, w[v], b[v]);
                        if (STEP == 1) {
                            two[0][v] += th.dv;
                            two[1][v] += th.dv * th.u;
                        }
                        out[v] = rstd * ((du - s1) - th.u * s2);
                        dz[v] = th.dz;
                    }
                }
                if (STEP == 0) store_narrow<T, V>(p.y, r * p.stride_y + at.ch, out);
                if (STEP == 2) {
                    store_narrow<T, V>(p.dx, r * p.stride_x + at.ch, out);
                    if (p.z) store_narrow<T, V>(p.dz, r * p.stride_z + at.ch, dz);
                }
            }
        if (STEP != 1) return;
        phase_sums<S, V>(two, l, shared);
        if (!at.on || (int)threadIdx.x >= l.lanes) return;
        S* to = reinterpret_cast<S*>(p.part) + piece_at(p.rows, at.tile, seq) * 2 * p.D + at.ch;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            to[v] = two[0][v];
            to[p.D + v] = two[1][v];
            total[0][v] += two[0][v];
            total[1][v] += two[1][v];
        }
    });
    if (STEP == 1) clear_rest(p.rows, rest, blockIdx.x, gridDim.x);
    if (STEP != 1 || !at.on || (int)threadIdx.x >= l.lanes) return;
    S* to = reinterpret_cast<S*>(p.sums) + at.tile * 2 * p.D + at.ch;
#pragma unroll
    for (int v = 0; v < V; ++v) {
        to[v] = total[1][v];
        to[p.D + v] = total[0][v];
    }
}

// Rows of a tile: 32 a phase; where that makes few workgroups, fewer, down to 8.  32 x 17,984 rows of 16 channels in fp32: y with 32 (281 workgroups) 29 us, with 8 17; the gradient's two passes
// 66 and 46
int span_rows(int D, int V, long long rows) {
    const Lanes l = lanes_for(D, V);
    int each = 32;
    while (each > 8 && rows / (each * l.phases) * l.blocks < 1024) each /= 2;
    return each * l.phases;
}
// Channels of a lane: 16 bytes; over sequences of 16 bits 8 bytes (moments of 32,768 rows of 2,560 in bf16 45 us, with 16 bytes 53)
template <typename T> constexpr int vector(int span) { return sizeof(T) == 8 ? 2 : sizeof(T) == 4 || span == DEER_SPAN_SEQUENCE ? 4 : 8; }

RestRows rest_of(const NormParams& p, bool grad, long long bytes) {
    RestRows rest{};
    if (!p.zero_rest) return rest;
    auto add = [&](void* first, long long stride, long long width) { rest.array[rest.count++] = RestArray{first, stride * bytes, width * bytes}; };
    if (grad) {
        add(p.dx, p.stride_x, p.D);
        if (p.z) add(p.dz, p.stride_z, p.D);
        return rest;
    }
    add(p.y, p.stride_y, p.D);
    if (p.span == DEER_SPAN_ROW) {
        const long long wide = bytes == 8 ? 16 : 8;   // mean and rstd
        rest.array[rest.count++] = RestArray{p.stats, wide * p.G, wide * p.G};
    }
    return rest;
}

template <typename T, int V>
hipError_t launch_sequences(bool grad, const NormParams& p, hipStream_t stream) {
    using S = wide_t<T>;
    const Lanes l = lanes_for(p.D, V);
    const int rows = span_rows(p.D, V, p.rows.T * (p.rows.packed ? 1 : p.rows.N));
    const long long tiles = (p.rows.T + rows - 1) / rows * (p.rows.packed ? 1 : p.rows.N);
    const dim3 grid((unsigned)(tiles * l.blocks)), block(256);
    const RestRows rest = rest_of(p, grad, sizeof(T));
    if (tiles) {
        if (grad) hipLaunchKernelGGL((span_kernel<T, V, 1>), grid, block, 0, stream, p, l, rows, rest);
        else hipLaunchKernelGGL((moments_kernel<T, V>), grid, block, 0, stream, p, l, rows, rest);
    }
    hipLaunchKernelGGL((join_kernel<S>), dim3((unsigned)((long long)p.rows.N * p.G)), dim3(kJoinLanes), 0, stream, p, rows, grad);
    if (tiles) {
        if (grad) hipLaunchKernelGGL((span_kernel<T, V, 2>), grid, block, 0, stream, p, l, rows, rest);
        else hipLaunchKernelGGL((span_kernel<T, V, 0>), grid, block, 0, stream, p, l, rows, rest);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !grad || (!p.dw && !p.dbias)) return e;
    return launch_sum_tiles(sizeof(S) == 8, p.sums, tiles, SumInto{p.dw, p.dbias, p.D, 1, true}, stream);
}

// rows of a workgroup, and how many workgroups along the rows: about 1,024 in all; 512 in the gradient, where each has sums of its own.  16,384 rows of 16 x 128 channels in bf16, as so many:
// forward 512 57 us, 1,024 52, 2,048 53, 4,096 59; gradient with the sums over workgroups 256 126, 512 86, 1,024 94, 2,048 112.  No lane sums more than kSumRounds rows for dw and dbias in 32 bits: equal
// rows would be off by 1.5e-4 over 16,384 of them, over these by 1e-5
constexpr long long kSumRounds = 1024;
struct RowCut {
    long long each, blocks;
};
RowCut row_cut(const RowShape& s, long long rows, bool grad) {
    const int all = grad ? 512 : 1024;
    long long rounds = (rows + s.rows - 1) / s.rows, want = all / s.blocks < 1 ? 1 : all / s.blocks;
    long long per = (rounds + want - 1) / want;
    if (grad && per > kSumRounds) per = kSumRounds;
    RowCut c;
    c.each = (per < 1 ? 1 : per) * s.rows;
    c.blocks = (rows + c.each - 1) / c.each;
    return c;
}
// A vector a lane where a wavefront has the group.  16,384 rows, forward and gradient: 16 x 128 channels in bf16 50 and 81 us, with four a lane 217 and 240, in fp32 87 and 135, with four 122 and 172; 512 channels of one group in
// bf16 20 and 26, with four 47 and 78
int vectors_each(int vecs) { return vecs <= 64 ? 1 : 4; }

template <typename T, int V, int M, bool GRAD, bool FEW>
hipError_t launch_rows_as(const NormParams& p, hipStream_t stream) {
    using S = wide_t<T>;
    const RowShape s = row_shape(p.D, p.G, V, M);
    const RowCut c = row_cut(s, p.rows.T * (p.rows.packed ? 1 : p.rows.N), GRAD);
    const dim3 grid((unsigned)(c.blocks * s.blocks)), block(256);
    const RestRows rest = rest_of(p, GRAD, sizeof(T));
    if constexpr (M == 1) {
        if (c.blocks) hipLaunchKernelGGL((rownorm_few_kernel<T, V, GRAD ? 2 : 4, GRAD>), grid, block, 0, stream, p, s, rest, c.each);
    } else if (c.blocks) {
        hipLaunchKernelGGL((rownorm_kernel<T, V, M, GRAD, FEW>), grid, block, 0, stream, p, s, rest, c.each);
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !GRAD || (!p.dw && !p.dbias)) return e;
    return launch_sum_tiles(sizeof(S) == 8, p.part, c.blocks * s.rows, SumInto{p.dw, p.dbias, p.D, 1, true}, stream);
}
template <typename T, int V, bool GRAD>
hipError_t launch_rows(const NormParams& p, hipStream_t stream) {
    const int vecs = p.D / p.G / V;
    if (vecs > 1024) return launch_rows_as<T, V, 4, GRAD, false>(p, stream);
    return vectors_each(vecs) == 1 ? launch_rows_as<T, V, 1, GRAD, true>(p, stream) : launch_rows_as<T, V, 4, GRAD, true>(p, stream);
}

template <typename T>
hipError_t launch_type(bool grad, const NormParams& p, hipStream_t stream) {
    constexpr int VR = vector<T>(DEER_SPAN_ROW), VS = vector<T>(DEER_SPAN_SEQUENCE);
    const int V = p.span == DEER_SPAN_ROW ? VR : VS;
    const size_t e = sizeof(T);
    bool vec = p.D / p.G % V == 0 && rows_fit(p.x, p.stride_x, V, e) && (!p.z || rows_fit(p.z, p.stride_z, V, e));
    if (grad) vec = vec && rows_fit(p.dy, p.stride_y, V, e) && rows_fit(p.dx, p.stride_x, V, e) && (!p.z || rows_fit(p.dz, p.stride_z, V, e));
    else vec = vec && rows_fit(p.y, p.stride_y, V, e);
    if (p.span == DEER_SPAN_SEQUENCE) return vec ? launch_sequences<T, VS>(grad, p, stream) : launch_sequences<T, 1>(grad, p, stream);
    if (vec) return grad ? launch_rows<T, VR, true>(p, stream) : launch_rows<T, VR, false>(p, stream);
    return grad ? launch_rows<T, 1, true>(p, stream) : launch_rows<T, 1, false>(p, stream);
}

}  // namespace

// (which vectors a call can use follows from its pointers: room for either)
NormLayout norm_layout(int dtype, int D, int G, int span, long long T, int N, bool packed, bool grad) {
    const int wide = dtype == DEER_F32 ? vector<float>(span) : dtype == DEER_F64 ? vector<double>(span) : vector<BF16>(span);
    NormLayout l{};
    for (const int V : {1, wide}) {
        long long part = 0, sums = 0;
        if (span == DEER_SPAN_SEQUENCE) {
            const int rows = span_rows(D, V, T * (packed ? 1 : N));
            const long long tiles = (T + rows - 1) / rows * (packed ? 1 : N);
            part = (tiles + (packed ? N : 0)) * 2 * D;
            if (grad) sums = tiles * 2 * D;
            if (tiles * lanes_for(D, V).blocks > l.tiles) l.tiles = tiles * lanes_for(D, V).blocks;
        } else if (D / G % V == 0) {
            const int vecs = D / G / V;
            const RowShape s = row_shape(D, G, V, vecs > 1024 ? 4 : vectors_each(vecs));
            const RowCut c = row_cut(s, T * (packed ? 1 : N), grad);
            if (grad) part = c.blocks * s.rows * 2 * D;
            if (c.blocks * s.blocks > l.tiles) l.tiles = c.blocks * s.blocks;
        }
        if (part > l.part) l.part = part;
        if (sums > l.sums) l.sums = sums;
    }
    if (span == DEER_SPAN_SEQUENCE && grad) l.joined = (long long)N * G * 2;
    return l;
}

hipError_t launch_groupnorm(int dtype, bool grad, const NormParams& p, hipStream_t stream) {
    switch (dtype) {
        case DEER_F32: return launch_type<float>(grad, p, stream);
        case DEER_F64: return launch_type<double>(grad, p, stream);
        case DEER_BF16: return launch_type<BF16>(grad, p, stream);
        default: return launch_type<F16>(grad, p, stream);
    }
}

}  // namespace deer
