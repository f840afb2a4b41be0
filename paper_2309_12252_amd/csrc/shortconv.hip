// Short causal convolution of every channel, with an activation: forward, gradient, single tokens.
#include <type_traits>

#include "layer_common.h"

namespace deer {
namespace {

template <typename T, int V>
__device__ __forceinline__ void load_wide(wide_t<T>* to, const T* from) {
    const vec_t<T, V> v = *reinterpret_cast<const vec_t<T, V>*>(from);
#pragma unroll
    for (int i = 0; i < V; ++i) to[i] = (wide_t<T>)vec_at<T, V>(v, i);
}
template <typename T, int V>
__device__ __forceinline__ void store_narrow(T* to, const wide_t<T>* from) {
    vec_t<T, V> v;
#pragma unroll
    for (int i = 0; i < V; ++i) vec_set<T, V>(v, i, (T)from[i]);
    *reinterpret_cast<vec_t<T, V>*>(to) = v;
}

// Row `row` of the sequence that begins at `start`: of x, or of the initial rows in front of it
template <typename T, int V>
__device__ __forceinline__ void row_or_initial(wide_t<T>* to, const ConvParams& p, int seq, long long start, long long row, int ch) {
    using S = wide_t<T>;
    if (row >= start) {
        load_wide<T, V>(to, reinterpret_cast<const T*>(p.x) + row * p.stride_x + ch);
        return;
    }
    const S* s0 = reinterpret_cast<const S*>(p.s0);
    const long long at = ((long long)seq * (p.W - 1) + (row - start + p.W - 1)) * p.D + ch;
#pragma unroll
    for (int v = 0; v < V; ++v) to[v] = s0 ? s0[at + v] : S(0);
}

struct ConvPlace {
    int n, ch;
    long long lo, hi;             // rows of the lane
    long long tile_lo, tile_hi;   // and of the workgroup
    bool on;
};
// which rows and channels a lane has: tiles of kConvRows rows a phase, sequences apart where they are padded
template <int V>
__device__ __forceinline__ ConvPlace conv_place(const ConvParams& p, const Lanes& l, long long block) {
    const long long per = (long long)kConvRows * l.phases, tiles = (p.rows.T + per - 1) / per, tile = block / l.blocks;
    ConvPlace at;
    at.n = p.rows.packed ? 0 : (int)(tile / tiles);
    at.ch = ((int)(block % l.blocks) * l.lanes + (int)(threadIdx.x & (l.lanes - 1))) * V;
    at.on = at.ch < p.D;
    const long long in = (p.rows.packed ? tile : tile % tiles) * per + (threadIdx.x / l.lanes) * kConvRows, base = (long long)at.n * p.rows.T;
    at.lo = base + in;
    at.hi = base + (in + kConvRows < p.rows.T ? in + kConvRows : p.rows.T);
    at.tile_lo = base + (p.rows.packed ? tile : tile % tiles) * per;
    at.tile_hi = at.tile_lo + per < base + p.rows.T ? at.tile_lo + per : base + p.rows.T;
    return at;
}

// The rows of the state behind every sequence
template <typename T>
__device__ __forceinline__ void conv_last(const ConvParams& p, long long block, long long blocks) {
    using S = wide_t<T>;
    const long long all = (long long)p.rows.N * (p.W - 1) * p.D;
    for (long long i = block * 256 + threadIdx.x; i < all; i += blocks * 256) {
        const int ch = (int)(i % p.D), k = (int)(i / p.D % (p.W - 1)), n = (int)(i / p.D / (p.W - 1));
        const long long start = seq_first(p.rows, n), row = start + seq_length(p.rows, n) - (p.W - 1) + k;
        row_or_initial<T, 1>(reinterpret_cast<S*>(p.last) + i, p, n, start, row, ch);
    }
}

// Memory bound: 32,768 packed rows of 2,560 channels in bf16, 335 MB, 74 us (4.5 TB/s; a large copy 5.2).  Eight rows at a time: a row is read once (and the W - 1 rows in front of a
// lane's 32 once more).  M weights.
template <typename T, int V, int M>
__global__ __launch_bounds__(256) void shortconv_kernel(const ConvParams p, const Lanes l, const RestRows rest, long long tile_blocks) {
    using S = wide_t<T>;
    if ((long long)blockIdx.x >= tile_blocks) {
        const long long block = blockIdx.x - tile_blocks, blocks = gridDim.x - tile_blocks;
        clear_rest(p.rows, rest, block, blocks);
        if (p.last && p.W > 1) conv_last<T>(p, block, blocks);
        return;
    }
    const ConvPlace at = conv_place<V>(p, l, blockIdx.x);
    S w[M][V], bias[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        bias[v] = p.bias && at.on ? reinterpret_cast<const S*>(p.bias)[at.ch + v] : S(0);
#pragma unroll
        for (int k = 0; k < M; ++k) w[k][v] = at.on ? reinterpret_cast<const S*>(p.w)[(long long)(at.ch + v) * M + k] : S(0);
    }
    for_runs(p.rows, at.n, at.tile_lo, at.tile_hi, [&](int seq, long long start, long long, long long r0, long long r1) {
        if (r0 < at.lo) r0 = at.lo;
        if (r1 > at.hi) r1 = at.hi;
        if (!at.on || r0 >= r1) return;
        S x[M - 1 + 8][V];
#pragma unroll
        for (int k = 0; k < M - 1; ++k) row_or_initial<T, V>(x[k], p, seq, start, r0 - (M - 1) + k, at.ch);
        const T* xs = reinterpret_cast<const T*>(p.x) + r0 * p.stride_x + at.ch;
        T* ys = reinterpret_cast<T*>(p.y) + r0 * p.stride_y + at.ch;
        for (long long r = r0; r < r1; r += 8, xs += 8 * p.stride_x, ys += 8 * p.stride_y) {
            const int rows = r1 - r < 8 ? (int)(r1 - r) : 8;
            if (rows == 8)
#pragma unroll
                for (int i = 0; i < 8; ++i) load_wide<T, V>(x[M - 1 + i], xs + i * p.stride_x);
            else
#pragma unroll
                for (int i = 0; i < 8; ++i) load_wide<T, V>(x[M - 1 + i], xs + (i < rows ? i : rows - 1) * p.stride_x);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (i >= rows) break;
                S y[V];
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    S sum = bias[v];
#pragma unroll
                    for (int k = 0; k < M; ++k) sum = w[k][v] * x[i + k][v] + sum;
                    y[v] = p.act == DEER_ACT_SILU ? silu<T>(sum) : sum;
                }
                store_narrow<T, V>(ys + i * p.stride_y, y);
            }
#pragma unroll
            for (int k = 0; k < M - 1; ++k)
#pragma unroll
                for (int v = 0; v < V; ++v) x[k][v] = x[8 + k][v];
        }
    });
}

// Gradient: dv_t = dy_t act'(v_t) with v computed again, dx_t = sum_j w_j dv_{t + W - 1 - j}, dw_j = sum_t dv_t x_{t - W + 1 + j}.  A lane goes on for W - 1 rows behind
// its own, whose dv its last rows need.  503 MB (the same rows, dy and dx) in 150 us, 3.4 TB/s: vector instructions take some 60 % of the time (36 an element), and with
// three wavefronts a SIMD the loads ahead do not cover all of the way to memory.  Two channels a lane are no faster, four wavefronts a SIMD spill (422).  B: 16 bits four rows at a time 158, one 182; fp32
// two rows 235, four 224; fp64, 16,384 rows of 1,280 channels, 114 (outputs 64).  Rows times strides in 64 bits for every load took a third of the time; widths that the compiler does not know, with a test for every weight: 539 us for 217 with 8 weights.
template <typename T, int V, int M>
__global__ __launch_bounds__(256) void shortconv_grad_kernel(const ConvParams p, const Lanes l, const RestRows rest, long long tile_blocks) {
    using S = wide_t<T>;
    constexpr int B = sizeof(T) == 2 ? 2 : 4;
    __shared__ S sums[256 * V];
    if ((long long)blockIdx.x >= tile_blocks) {
        const long long block = blockIdx.x - tile_blocks, blocks = gridDim.x - tile_blocks, per = (long long)(p.W - 1) * p.D, all = p.rows.N * per;
        clear_rest(p.rows, rest, block, blocks);
        if (p.ds0)
            for (long long i = block * 256 + threadIdx.x; i < all; i += blocks * 256)
                if (seq_length(p.rows, (int)(i / per)) == 0) reinterpret_cast<S*>(p.ds0)[i] = p.dlast ? reinterpret_cast<const S*>(p.dlast)[i] : S(0);
        return;
    }
    const ConvPlace at = conv_place<V>(p, l, blockIdx.x);
    constexpr int behind = M - 1;
    S w[M][V], bias[V], dw[M][V], dbias[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        bias[v] = p.bias && at.on ? reinterpret_cast<const S*>(p.bias)[at.ch + v] : S(0);
        dbias[v] = S(0);
#pragma unroll
        for (int k = 0; k < M; ++k) {
            w[k][v] = at.on ? reinterpret_cast<const S*>(p.w)[(long long)(at.ch + v) * M + k] : S(0);
            dw[k][v] = S(0);
        }
    }
    {
        for_runs(p.rows, at.n, at.tile_lo, at.tile_hi, [&](int seq, long long start, long long end, long long r0, long long r1) {
            if (r0 < at.lo) r0 = at.lo;
            if (r1 > at.hi) r1 = at.hi;
            if (!at.on || r0 >= r1) return;
            S x[M - 1 + B][V], d[M - 1 + B][V];
            const long long stop = r1 + behind < end ? r1 + behind : end;   // rows whose dv is needed
#pragma unroll
            for (int k = 0; k < M - 1; ++k) {
                row_or_initial<T, V>(x[k], p, seq, start, r0 - (M - 1) + k, at.ch);
#pragma unroll
                for (int v = 0; v < V; ++v) d[k][v] = S(0);
            }
            // B rows at a time, the next B on their way
            using TV = vec_t<T, V>;
            TV nx[B], ny[B];
            const T* xs = reinterpret_cast<const T*>(p.x) + r0 * p.stride_x + at.ch;
            const T* ds = reinterpret_cast<const T*>(p.dy) + r0 * p.stride_y + at.ch;
            T* outs = reinterpret_cast<T*>(p.dx) + (r0 - behind) * p.stride_x + at.ch;   // (of the row that a row completes)
            auto ask = [&](long long r) {
                const int rows = stop - r < B ? (int)(stop - r) : B;
                if (rows == B) {
#pragma unroll
                    for (int i = 0; i < B; ++i) {
                        nx[i] = *reinterpret_cast<const TV*>(xs + i * p.stride_x);
                        ny[i] = *reinterpret_cast<const TV*>(ds + i * p.stride_y);
                    }
                } else if (rows > 0) {
#pragma unroll
                    for (int i = 0; i < B; ++i) {
                        nx[i] = *reinterpret_cast<const TV*>(xs + (i < rows ? i : rows - 1) * p.stride_x);
                        ny[i] = *reinterpret_cast<const TV*>(ds + (i < rows ? i : rows - 1) * p.stride_y);
                    }
                }
                xs += B * p.stride_x;
                ds += B * p.stride_y;
            };
            ask(r0);
            for (long long r = r0; r < r1 + behind; r += B, outs += B * p.stride_x) {
                S dy[B][V];
#pragma unroll
                for (int i = 0; i < B; ++i)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        x[M - 1 + i][v] = (S)vec_at<T, V>(nx[i], v);
                        dy[i][v] = (S)vec_at<T, V>(ny[i], v);
                    }
                if (r + B < r1 + behind) ask(r + B);
                // INSIDE: all B rows are the lane's own, and so are the rows whose dx they complete, none of which the final states see
                auto go = [&](auto inside) {
                    constexpr bool INSIDE = decltype(inside)::value;
#pragma unroll
                    for (int i = 0; i < B; ++i) {
                        const long long row = r + i, out = row - behind;
                        S dx[V];
#pragma unroll
                        for (int v = 0; v < V; ++v) {
                            S slope = S(1);
                            if (p.act == DEER_ACT_SILU) {
                                S sum = bias[v], f;
#pragma unroll
                                for (int k = 0; k < M; ++k) sum = w[k][v] * x[i + k][v] + sum;
                                silu_both<T>(sum, f, slope);
                            }
                            const S dv = INSIDE || row < stop ? dy[i][v] * slope : S(0);
                            d[M - 1 + i][v] = dv;
                            if (INSIDE || row < r1) {
                                dbias[v] += dv;
#pragma unroll
                                for (int k = 0; k < M; ++k) dw[k][v] = dv * x[i + k][v] + dw[k][v];
                            }
                            // weight m goes with the row m in front of this one
                            S sum = S(0);
#pragma unroll
                            for (int m = 0; m < M; ++m) sum = w[m][v] * d[M - 1 + i - m][v] + sum;
                            dx[v] = sum;
                        }
                        if (INSIDE) {
                            store_narrow<T, V>(outs + i * p.stride_x, dx);
                            continue;
                        }
                        if (out >= r1 || (out < r0 && r0 != start)) continue;
                        if (out >= end - behind && p.dlast) {
                            const S* from = reinterpret_cast<const S*>(p.dlast) + ((long long)seq * behind + out - (end - behind)) * p.D + at.ch;
#pragma unroll
                            for (int v = 0; v < V; ++v) dx[v] += from[v];
                        }
                        if (out >= r0) store_narrow<T, V>(outs + i * p.stride_x, dx);
                        else if (p.ds0) {
                            S* to = reinterpret_cast<S*>(p.ds0) + ((long long)seq * behind + out - start + behind) * p.D + at.ch;
#pragma unroll
                            for (int v = 0; v < V; ++v) to[v] = dx[v];
                        }
                    }
                };
                if (r >= r0 + behind && r + B <= r1) go(std::true_type{});
                else go(std::false_type{});
#pragma unroll
                for (int k = 0; k < M - 1; ++k)
#pragma unroll
                    for (int v = 0; v < V; ++v) {
                        x[k][v] = x[B + k][v];
                        d[k][v] = d[B + k][v];
                    }
            }
        });
    }
    // the phases' sums, one weight at a time
    S* part = reinterpret_cast<S*>(p.part) + (long long)(blockIdx.x / l.blocks) * (M + 1) * p.D;
    const int wide = l.lanes * V, first = (int)(blockIdx.x % l.blocks) * wide;
#pragma unroll
    for (int k = 0; k <= M; ++k) {
        __syncthreads();
#pragma unroll
        for (int v = 0; v < V; ++v) sums[threadIdx.x * V + v] = k == M ? dbias[v] : dw[k < M ? k : 0][v];
        __syncthreads();
        for (int c = threadIdx.x; c < wide; c += 256) {
            S sum = S(0);
            for (int f = 0; f < l.phases; ++f) sum += sums[f * wide + c];
            if (first + c < p.D) part[(long long)k * p.D + first + c] = sum;
        }
    }
}

// One token for every row: latency bound, one launch, a lane a channel (32 rows of 2,048 channels 3.6 us, 11 with the call from Python); slots as in the recurrences' steps
template <typename T>
__global__ __launch_bounds__(256) void shortconv_step_kernel(const ConvStepParams p) {
    using S = wide_t<T>;
    const int per = (p.D + 255) / 256, n = blockIdx.x / per, ch = (blockIdx.x % per) * 256 + threadIdx.x;
    int slot = n;
    bool twice = false;
    if (p.rows.slots) {
        slot = p.rows.slots[n];
        for (int m = threadIdx.x; m < n; m += 256) twice = twice || p.rows.slots[m] == slot;
    }
    const bool in = ch < p.D && slot >= 0 && slot < p.rows.n_slots;
    S* state = reinterpret_cast<S*>(p.state) + (long long)slot * (p.W - 1) * p.D + ch;
    S x[8], w[8], sum = S(0);
    if (in) {
        sum = p.bias ? reinterpret_cast<const S*>(p.bias)[ch] : S(0);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            if (k >= p.W) break;
            x[k] = k == p.W - 1 ? (S)reinterpret_cast<const T*>(p.x)[(long long)n * p.stride_x + ch] : state[(long long)k * p.D];
            w[k] = reinterpret_cast<const S*>(p.w)[(long long)ch * p.W + k];
        }
    }
    twice = p.rows.slots ? __syncthreads_or(twice) != 0 : false;
    if (!in || twice) {
        if (p.rows.zero_rest && ch < p.D) reinterpret_cast<T*>(p.y)[(long long)n * p.stride_y + ch] = (T)0;
        return;
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        if (k >= p.W) break;
        sum = w[k] * x[k] + sum;
        if (k > 0) state[(long long)(k - 1) * p.D] = x[k];
    }
    reinterpret_cast<T*>(p.y)[(long long)n * p.stride_y + ch] = (T)(p.act == DEER_ACT_SILU ? silu<T>(sum) : sum);
}

template <typename T, int V, int M>
hipError_t launch_taps(bool grad, const ConvParams& p, hipStream_t stream) {
    const Lanes l = lanes_for(p.D, V);
    const long long per = (long long)kConvRows * l.phases, tiles = (p.rows.T + per - 1) / per * (p.rows.packed ? 1 : p.rows.N), blocks = tiles * l.blocks;
    RestRows rest{};
    if (p.zero_rest)
        rest.array[rest.count++] = grad ? RestArray{p.dx, p.stride_x * (long long)sizeof(T), p.D * (long long)sizeof(T)}
                                        : RestArray{p.y, p.stride_y * (long long)sizeof(T), p.D * (long long)sizeof(T)};
    // what is not a tile's: rows of no sequence, and the states' rows, 1,024 elements a workgroup
    const long long rest_tiles = rest.count ? (p.rows.T + 15) / 16 * (p.rows.packed ? 1 : p.rows.N) : 0, cells = (long long)p.rows.N * (p.W - 1) * p.D / 1024;
    long long extra = rest_tiles > cells ? rest_tiles : cells;
    extra = extra < 1 ? 1 : extra > 512 ? 512 : extra;
    const dim3 grid((unsigned)(blocks + extra)), block(256);
    if (!grad) {
        hipLaunchKernelGGL((shortconv_kernel<T, V, M>), grid, block, 0, stream, p, l, rest, blocks);
        return hipGetLastError();
    }
    hipLaunchKernelGGL((shortconv_grad_kernel<T, V, M>), grid, block, 0, stream, p, l, rest, blocks);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    return launch_sum_tiles(sizeof(wide_t<T>) == 8, p.part, tiles, SumInto{p.dw, p.dbias, p.D, p.W, true}, stream);
}

template <typename T, int V>
hipError_t launch_width(bool grad, const ConvParams& p, hipStream_t stream) {
    // half as many channels a lane for registers' sake: gradient of 32,768 rows of 2,560 channels with 8 weights, fp32 289 us for 368, fp64 511 for 586; bf16 227 for 217, so not there
    constexpr int H = sizeof(T) > 2 && V > 1 ? V / 2 : V;
    switch (p.W) {
        case 1: return launch_taps<T, V, 1>(grad, p, stream);
        case 2: return launch_taps<T, V, 2>(grad, p, stream);
        case 3: return launch_taps<T, V, 3>(grad, p, stream);
        case 4: return launch_taps<T, V, 4>(grad, p, stream);
        case 5: return launch_taps<T, H, 5>(grad, p, stream);
        case 6: return launch_taps<T, H, 6>(grad, p, stream);
        case 7: return launch_taps<T, H, 7>(grad, p, stream);
        default: return launch_taps<T, H, 8>(grad, p, stream);
    }
}
template <typename T>
hipError_t launch_type(bool grad, const ConvParams& p, hipStream_t stream) {
    constexpr int V = sizeof(T) == 2 ? 4 : sizeof(T) == 4 ? 4 : 2;
    const bool vec = p.D % V == 0 && rows_fit(p.x, p.stride_x, V, sizeof(T)) &&
                     (grad ? rows_fit(p.dy, p.stride_y, V, sizeof(T)) && rows_fit(p.dx, p.stride_x, V, sizeof(T)) : rows_fit(p.y, p.stride_y, V, sizeof(T)));
    return vec ? launch_width<T, V>(grad, p, stream) : launch_width<T, 1>(grad, p, stream);
}

template <typename T>
hipError_t launch_step_type(const ConvStepParams& p, hipStream_t stream) {
    hipLaunchKernelGGL((shortconv_step_kernel<T>), dim3((unsigned)((long long)((p.D + 255) / 256) * p.rows.N)), dim3(256), 0, stream, p);
    return hipGetLastError();
}

// 16 columns and 64 shares of the tiles a workgroup: few columns of many tiles are all latency (32 columns of 1,124 tiles 4 us, 18 with 16 shares)
constexpr int kSumLanes = 1024, kShares = kSumLanes / 16;
template <typename S>
__global__ __launch_bounds__(kSumLanes) void sum_tiles_kernel(const S* part, long long tiles, int cols, const SumInto into) {
    __shared__ double sums[kShares][17];
    const int c = blockIdx.x * 16 + (threadIdx.x & 15), f = threadIdx.x >> 4;
    double sum = 0;
    if (c < cols)
#pragma unroll 4
        for (long long t = f; t < tiles; t += kShares) sum += (double)part[t * cols + c];
    sums[f][threadIdx.x & 15] = sum;
    __syncthreads();
    if (f != 0 || c >= cols) return;
    sum = 0;
#pragma unroll 8
    for (int i = 0; i < kShares; ++i) sum += sums[i][threadIdx.x];
    const int row = c / into.each, at = c % into.each;
    S* to = reinterpret_cast<S*>(row < into.many ? into.first : into.second);
    if (to) to[row < into.many ? (long long)at * into.many + row : at] = (S)sum;
}

}  // namespace

hipError_t launch_sum_tiles(bool wide, const void* part, long long tiles, const SumInto& into, hipStream_t stream) {
    const int cols = into.each * (into.many + (into.last ? 1 : 0));
    const dim3 grid((cols + 15) / 16), block(kSumLanes);
    if (wide) hipLaunchKernelGGL((sum_tiles_kernel<double>), grid, block, 0, stream, reinterpret_cast<const double*>(part), tiles, cols, into);
    else hipLaunchKernelGGL((sum_tiles_kernel<float>), grid, block, 0, stream, reinterpret_cast<const float*>(part), tiles, cols, into);
    return hipGetLastError();
}

// (with one element a lane there are the fewest lanes along the rows: the most tiles)
long long conv_tiles(int D, long long T, int N, bool packed) {
    const long long per = (long long)kConvRows * lanes_for(D, 1).phases;
    return (T + per - 1) / per * (packed ? 1 : N);
}

hipError_t launch_shortconv(int dtype, bool grad, const ConvParams& p, hipStream_t stream) {
    switch (dtype) {
        case DEER_F32: return launch_type<float>(grad, p, stream);
        case DEER_F64: return launch_type<double>(grad, p, stream);
        case DEER_BF16: return launch_type<BF16>(grad, p, stream);
        default: return launch_type<F16>(grad, p, stream);
    }
}

hipError_t launch_shortconv_step(int dtype, const ConvStepParams& p, hipStream_t stream) {
    switch (dtype) {
        case DEER_F32: return launch_step_type<float>(p, stream);
        case DEER_F64: return launch_step_type<double>(p, stream);
        case DEER_BF16: return launch_step_type<BF16>(p, stream);
        default: return launch_step_type<F16>(p, stream);
    }
}

}  // namespace deer
