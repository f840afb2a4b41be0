// Dropout of trajectories: y = x / (1 - p) or 0, from a counter-based generator; the mask is never stored.
#include "seq_common.h"

namespace deer {
namespace {

// A lane has eight rows of V channels: one block of random bits a channel.  Memory bound: x read once, y written once; the generator
// takes about 20 vector cycles an element, which hides behind the memory: 268 MB of bf16, other arrays in every call, in 47 us (5.7 TB/s; a large copy 5.2); the same
// arrays again, which the last-level cache has in part, in 41.
template <typename T, int V>
__global__ __launch_bounds__(256) void dropout_kernel(const DropoutParams p) {
    using S = wide_t<T>;
    using TV = vec_t<T, V>;
    const long long blocks = (p.T + 7) >> 3;
    const int cols = p.D / V;
    const long long at = (long long)blockIdx.x * 256 + threadIdx.x, all = blocks * cols * p.N;
    if (at >= all) return;
    const int ch = (int)(at % cols) * V;
    const long long rest = at / cols, block = rest % blocks;
    const int n = (int)(rest / blocks);
    const long long row0 = block * 8, base = (long long)n * p.T + row0;
    const int rows = p.T - row0 < 8 ? (int)(p.T - row0) : 8;
    TV x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = *reinterpret_cast<const TV*>(reinterpret_cast<const T*>(p.x) + (base + (j < rows ? j : rows - 1)) * p.stride_in + ch);
    unsigned keep[V];
#pragma unroll
    for (int v = 0; v < V; ++v) keep[v] = drop_keep8(p.drop, (unsigned)(ch + v), (unsigned)block, (unsigned)n);
    const S scale = (S)p.drop.scale;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        if (j >= rows) break;
        TV y;
#pragma unroll
        for (int v = 0; v < V; ++v) vec_set<T, V>(y, v, (keep[v] >> j) & 1u ? (T)((S)vec_at<T, V>(x[j], v) * scale) : (T)0);
        *reinterpret_cast<TV*>(reinterpret_cast<T*>(p.y) + (base + j) * p.stride_out + ch) = y;
    }
}

template <typename T, int V>
hipError_t launch_vec(const DropoutParams& p, hipStream_t stream) {
    const long long all = ((p.T + 7) >> 3) * (p.D / V) * p.N;
    if (all == 0) return hipSuccess;
    hipLaunchKernelGGL((dropout_kernel<T, V>), dim3((unsigned)((all + 255) / 256)), dim3(256), 0, stream, p);
    return hipGetLastError();
}

template <typename T>
hipError_t launch_type(const DropoutParams& p, hipStream_t stream) {
    auto fits = [&](int v) {
        const uintptr_t bytes = v * sizeof(T);
        return p.D % v == 0 && p.stride_in % v == 0 && p.stride_out % v == 0 && reinterpret_cast<uintptr_t>(p.x) % bytes == 0 &&
               reinterpret_cast<uintptr_t>(p.y) % bytes == 0;
    };
    // 8 bytes a lane at least (rows of pairs in 16 bits are no faster than single elements): the same 64 Mi elements again in bf16 41 us, one a lane 64; fp32 94, 107
    constexpr int V = sizeof(T) == 2 ? 4 : 2;
    return fits(V) ? launch_vec<T, V>(p, stream) : launch_vec<T, 1>(p, stream);
}

}  // namespace

hipError_t launch_dropout(int dtype, const DropoutParams& p, hipStream_t stream) {
    switch (dtype) {
        case DEER_F32: return launch_type<float>(p, stream);
        case DEER_F64: return launch_type<double>(p, stream);
        case DEER_BF16: return launch_type<BF16>(p, stream);
        default: return launch_type<F16>(p, stream);
    }
}

}  // namespace deer
