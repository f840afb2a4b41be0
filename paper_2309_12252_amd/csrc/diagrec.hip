// Gated linear recurrences with one state a channel: h_t = a_t h_{t-1} + u_t, forward and backward in one pass over the data,
// and the step of one token.
//
//   factor   a = g           u = x                        LOG      a = exp(g)      u = x
//   sigmoid  a = 1/(1+e^-g)  u = (1 - a) x                (x may be multiplied by the dropout mask first)
// Backward: with mu_{T+1} = dL/dh_T of the final state, lambda_t = dh_t + mu_{t+1} and mu_t = a_t lambda_t,
//   dL/da_t = lambda_t h_{t-1}   dL/du_t = lambda_t   dL/dh_0 = mu_1,
// again a recurrence of the same form, mu_t = a_t mu_{t+1} + a_t dh_t, along the reversed rows.
#include <type_traits>

#include "seq_common.h"

namespace deer {
namespace {

constexpr int kGroup = 16;                        // tiles of a group: the carry is passed on from group to group
constexpr unsigned long long kUnset = ~0ull;      // a word that has not been published (two NaNs that are never published)
constexpr long long kPolls = 1ll << 22;           // polls before a tile gives up on its predecessors (seconds; its rows become NaN)

// Tile of W wavefronts, R rows each; a lane has V channels.  As many rows as the registers of two workgroups a CU hold without scratch: long tiles mean
// few published words and few waits.  Measured on 32,768 packed rows of 2,560 channels in bf16, sigmoid gates and dropout, forward: R = 8 180 us, 16
// 160, 32 144 (backward, where a row has four arrays: R = 8 245 us, 16 208); W = 4 148 us, 16 160 (log gates without dropout 227 and 257 against 216);
// groups of 8 tiles instead of 16 the same within 2 %.
template <typename T, bool REV> struct Shape {
    static constexpr int W = kDiagLanes / 64;
    static constexpr int V = sizeof(T) == 8 ? 1 : 2;
    static constexpr int R = sizeof(T) == 2 ? (REV ? 16 : 32) : REV ? 8 : 16;
};

template <typename T> __device__ __forceinline__ T fast_exp(T v) { return exp(v); }
template <> __device__ __forceinline__ float fast_exp<float>(float v) { return __expf(v); }

// a and the weight of x.  The 16-bit types take the hardware's exp and reciprocal (2^-21 off, far below their rounding).
template <typename T, int KIND>
__device__ __forceinline__ void gate_factors(wide_t<T> g, wide_t<T>& a, wide_t<T>& w) {
    using S = wide_t<T>;
    if constexpr (KIND == DEER_GATE_FACTOR) {
        a = g;
        w = S(1);
    } else if constexpr (KIND == DEER_GATE_LOG) {
        a = sizeof(T) == 2 ? fast_exp(g) : exp(g);
        w = S(1);
    } else if constexpr (sizeof(T) == 2) {   // both a and 1 - a without cancellation; 2^126 stands for what is more (a NaN stays one)
        float t = g * -1.442695041f;
        t = t > 126.0f ? 126.0f : t;
        const float e = __builtin_amdgcn_exp2f(t);
        a = __builtin_amdgcn_rcpf(1.0f + e);
        w = e * a;
    } else {
        const S m = g < S(0) ? g : -g;
        const S e = exp(m), r = S(1) / (S(1) + e), er = e * r;
        a = g < S(0) ? er : r;
        w = g < S(0) ? r : er;
    }
}

// Published words: (a, h) of a tile as one word of two floats, or two words of a double each.  A word is valid as soon as it
// is not kUnset, so no flag and no fence goes with it; NaNs are published as the one quiet NaN.
__device__ __forceinline__ unsigned long long word_of(float a, float h) {
    const unsigned ua = a != a ? 0x7FC00000u : __float_as_uint(a), uh = h != h ? 0x7FC00000u : __float_as_uint(h);
    return ((unsigned long long)uh << 32) | ua;
}
__device__ __forceinline__ unsigned long long word_of(double v) {
    return v != v ? 0x7FF8000000000000ull : (unsigned long long)__double_as_longlong(v);
}
__device__ __forceinline__ void put_word(unsigned long long* p, unsigned long long v) {
    __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ __forceinline__ unsigned long long get_word(const unsigned long long* p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// `count` of K items of E words each, `step` words apart, and what `front` points to, once all of them are there; kUnset in their place after kPolls polls
template <int K, int E>
__device__ __forceinline__ void wait_words(const unsigned long long* p, long long step, int count, unsigned long long (&w)[K * E], const unsigned long long* front,
                                           unsigned long long& f) {
    for (long long poll = 0; poll < kPolls; ++poll) {
        f = front ? get_word(front) : 0;
        bool all = true;
#pragma unroll
        for (int k = 0; k < K * E; ++k) w[k] = k / E < count ? get_word(p + k / E * step + k % E) : 0;
#pragma unroll
        for (int k = 0; k < K * E; ++k) all = all && w[k] != kUnset;
        if (__all(all && f != kUnset)) return;
        __builtin_amdgcn_s_sleep(2);
    }
}

// V values of a row as the bits that they were read as: arrays of 16-bit values would be kept a register each
template <int BYTES> struct Bits;
template <> struct Bits<2> { using type = unsigned short; };
template <> struct Bits<4> { using type = unsigned; };
template <> struct Bits<8> { using type = unsigned long long; };
template <typename T, int V> using bits_t = typename Bits<sizeof(T) * V>::type;
template <typename T, int V>
__device__ __forceinline__ wide_t<T> value_of(bits_t<T, V> b, int v) {
    if constexpr (sizeof(T) == 2 && V == 2) {
        const unsigned short h = (unsigned short)(v == 0 ? b : b >> 16);
        return (wide_t<T>)__builtin_bit_cast(T, h);
    } else if constexpr (sizeof(T) == 4 && V == 2) {
        return __builtin_bit_cast(T, (unsigned)(v == 0 ? b : b >> 32));
    } else {
        return (wide_t<T>)__builtin_bit_cast(T, b);
    }
}
template <typename T, int V>
__device__ __forceinline__ void set_value(bits_t<T, V>& b, int v, T x) {
    if constexpr (sizeof(T) == 4 && V == 2) {
        const unsigned long long u = __builtin_bit_cast(unsigned, x);
        b = v == 0 ? (b & ~0xFFFFFFFFull) | u : (b & 0xFFFFFFFFull) | u << 32;
    } else {
        b = __builtin_bit_cast(bits_t<T, V>, x);
    }
}
template <typename T, int V, bool DROP>
__device__ __forceinline__ wide_t<T> input_of(bits_t<T, V> b, int v, unsigned kept, wide_t<T> scale) {
    const wide_t<T> x = value_of<T, V>(b, v);
    if constexpr (DROP) return kept ? x * scale : wide_t<T>(0);
    else return x;
}
// the compiler is not to keep what it derived from x: what is needed again is computed again
template <typename X>
__device__ __forceinline__ void forget(X& x) {
    asm volatile("" : "+v"(x));
}

// The state behind `front` (nullptr: a first tile that sets it) and `count` tiles' maps.  What is in front comes with the first of the maps: they are there
// before it, so that one trip to memory is left when it arrives (3 x 5,003 rows of 50 channels in fp64, where the maps came four at a time and
// after it: 16.4 + 24.4 us, so 13.9 + 17.8; four or six at a time 15.5 + 21).
__device__ __forceinline__ float fold_tiles(const unsigned long long* agg, long long step, int count, const unsigned long long* front, float) {
    constexpr int K = 8;
    float h = 0.0f;
    for (int at = 0; at == 0 || at < count; at += K) {
        unsigned long long w[K], f;
        wait_words<K, 1>(agg + (long long)at * step, step, count - at, w, at == 0 ? front : nullptr, f);
        if (at == 0 && front) h = __uint_as_float((unsigned)(f >> 32));
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (at + k < count) {
                const float a = __uint_as_float((unsigned)w[k]), u = __uint_as_float((unsigned)(w[k] >> 32));
                h = (!front && at + k == 0) ? u : a * h + u;
            }
    }
    return h;
}
__device__ __forceinline__ double fold_tiles(const unsigned long long* agg, long long step, int count, const unsigned long long* front, double) {
    constexpr int K = 8;
    double h = 0.0;
    for (int at = 0; at == 0 || at < count; at += K) {
        unsigned long long w[2 * K], f;
        wait_words<K, 2>(agg + (long long)at * step, step, count - at, w, at == 0 ? front : nullptr, f);
        if (at == 0 && front) h = __longlong_as_double((long long)f);
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (at + k < count) {
                const double a = __longlong_as_double((long long)w[2 * k]), u = __longlong_as_double((long long)w[2 * k + 1]);
                h = (!front && at + k == 0) ? u : a * h + u;
            }
    }
    return h;
}

// Memory bound: every input is read once and every output written once (805 MB of bf16 in 156 us with log gates, 5.2 TB/s, the rate of a large copy;
// with sigmoid gates and dropout the generator and the exponentials decide: 142 us forward, 208 us backward for 32,768 packed rows of 2,560
// channels in bf16, where the bytes take 97 and 195).  Few rows are latency bound: chains along the rows
// and the wait for the carry (3 x 5,003 rows of 50 channels in fp64: 14 us, backward 18).  A lane keeps V channels and R rows of the inputs in
// registers (raw: 16 rows of two bf16 arrays are 32 registers), so the rows are gone over twice without a second read: once
// for the tile's own map (product of the factors, state from zero), once more from the carry.  The carry of a tile is the fold, in a fixed
// order, of its predecessors' maps since the last group of kGroup tiles and that group's carry, so two runs give the
// same bits.  Tiles are dealt out by a ticket in the order of the rows: a tile waits for tiles that are running or done only.
template <typename T, int KIND, int V, int R, int W, bool REV, bool DROP>
__global__ __launch_bounds__(64 * W, 4) void diagrec_kernel(const DiagrecParams p) {
    using S = wide_t<T>;
    using TV = vec_t<T, V>;
    constexpr int C = 64 * V;     // channels of a tile
    constexpr int L = R * W;      // rows of a tile
    constexpr int WORDS = sizeof(S) == 8 ? 2 : 1;
    static_assert(R + 1 <= 64 && R % 8 == 0, "a lane looks up one row's sequence; the mask's blocks are eight rows");
    __shared__ S sh_a[W][C], sh_h[W][C], sh_carry[C];
    __shared__ int sh_reset[W], sh_begin;
    __shared__ unsigned sh_ticket;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (threadIdx.x == 0) sh_ticket = atomicAdd(p.ticket, 1u);
    __syncthreads();
    const unsigned ticket = __builtin_amdgcn_readfirstlane(sh_ticket);
    const unsigned dgroups = (p.D + C - 1) / C, seqs = p.rows.packed ? 1u : (unsigned)p.rows.N, per = dgroups * seqs;
    const int c = (int)(ticket / per);                 // tile along the scan
    const unsigned rest = ticket - (unsigned)c * per;
    const int n = (int)(rest / dgroups);
    const int ch = (int)(rest % dgroups) * C + lane * V;
    const bool on = ch < p.D;
    const int chl = on ? ch : 0;                       // (lanes without a channel look at the first one's states, and write nothing)
    const unsigned col = on ? (unsigned)ch * (unsigned)sizeof(T) : kNoColumn;
    const long long tile_row = (long long)(REV ? p.chunks - 1 - c : c) * L;
    const long long row0 = tile_row + (REV ? W - 1 - wave : wave) * R;

    // lane j: the sequence of row row0 + j, and whether a sequence begins there (or the last one ends)
    int seq;
    bool live, edge;
    {
        const long long r = row0 + (lane <= R ? lane : R);
        if (p.rows.packed) {
            const int u = bounds_up_to(p.rows, r);
            seq = u - 1;
            live = u >= 1 && u <= p.rows.N && r < p.rows.T;
            edge = u >= 1 && clamp_row(p.rows.bounds[u - 1], p.rows.T) == r;
        } else {
            const long long len = seq_length(p.rows, n);
            seq = n;
            live = r < len;
            edge = r == 0 || r == len;
        }
    }
    const unsigned long long live_bits = __ballot(live && lane < R), edge_bits = __ballot(edge && lane <= R);
    const unsigned long long begins = live_bits & edge_bits, finishes = live_bits & (edge_bits >> 1);
    const unsigned long long starts = REV ? finishes : begins, ends = REV ? begins : finishes;   // in the order of the scan

    const T* g = reinterpret_cast<const T*>(p.g);
    const T* x = reinterpret_cast<const T*>(p.x);
    const S* init = reinterpret_cast<const S*>(REV ? p.dlast : p.h0);
    S* fin = reinterpret_cast<S*>(REV ? p.dh0 : p.last);
    const long long base = p.rows.packed ? 0 : (long long)n * p.rows.T;

    // ---- the rows' inputs, all reads at a time ----
    constexpr bool NEED_X = !REV || KIND == DEER_GATE_SIGMOID;
    // an exponential that has as many bits as its gate takes the gate's place once it is known
    constexpr bool IN_PLACE = KIND == DEER_GATE_LOG && sizeof(T) >= 4;
    constexpr int SECOND = IN_PLACE ? (int)DEER_GATE_FACTOR : KIND;
    using B = bits_t<T, V>;
    B rg[R], rx[NEED_X ? R : 1], rh[REV ? R : 1], rd[REV ? R : 1];
    unsigned keep[DROP ? V : 1] = {};
    if (live_bits) {
        const int first = __builtin_ctzll(live_bits), last = 63 - __builtin_clzll(live_bits);
        const long long r0 = base + row0;
        const int ahead = row0 > 0 ? 1 : 0;              // (the row in front of the first is h0's)
        const RowsAt ag(g + r0 * p.stride_gate, p.stride_gate), ax(x + r0 * p.stride_in, p.stride_in);
        const RowsAt ad(reinterpret_cast<const T*>(p.dh) + r0 * p.stride_out, p.stride_out);
        const RowsAt ah(reinterpret_cast<const T*>(p.h) + (r0 - ahead) * p.stride_out, p.stride_out);
        // a row that is none reads the nearest one that is
        unsigned at_g = col + first * ag.pitch, at_x = col + first * ax.pitch, at_d = col + first * ad.pitch, at_h = col + (first + ahead > 0 ? first + ahead - 1 : 0) * ad.pitch;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            rg[j] = ag.template load<B>(at_g);
            if constexpr (NEED_X) rx[j] = ax.template load<B>(at_x);
            if constexpr (REV) {
                rd[j] = ad.template load<B>(at_d);
                rh[j] = ah.template load<B>(at_h);
            }
            if (j >= first && j < last) {
                at_g += ag.pitch;
                at_x += ax.pitch;
                at_d += ad.pitch;
                if (j + ahead > 0) at_h += ad.pitch;
            }
        }
        if constexpr (DROP) {
#pragma unroll
            for (int v = 0; v < V; ++v) {
                keep[v] = 0;
#pragma unroll
                for (int b = 0; b < R / 8; ++b)
                    keep[v] |= drop_keep8(p.drop, (unsigned)(chl + v), (unsigned)((row0 >> 3) + b), (unsigned)n) << (8 * b);
            }
        }
    }
    const S scale = DROP ? (S)p.drop.scale : S(1);
    // ---- this wavefront's map ----
    S A[V], H[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        A[v] = S(1);
        H[v] = S(0);
    }
    // PLAIN: all rows are live and none begins or ends a sequence, the ordinary case inside a long one (without it: 1 x 65,536 x 2,048 in bf16 175 us, 159 with)
    const bool plain = live_bits == (1ull << R) - 1 && !starts && !ends;
    auto first_pass = [&](auto all) __attribute__((always_inline)) {
        constexpr bool PLAIN = decltype(all)::value;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int j = REV ? R - 1 - i : i;
            if (!PLAIN && ((starts >> j) & 1)) {
                const long long s = __builtin_amdgcn_readlane(seq, j);
#pragma unroll
                for (int v = 0; v < V; ++v) H[v] = init ? init[s * p.D + chl + v] : S(0);
            }
            if (PLAIN || ((live_bits >> j) & 1)) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    S a, w;
                    gate_factors<T, KIND>(value_of<T, V>(rg[j], v), a, w);
                    if constexpr (IN_PLACE) set_value<T, V>(rg[j], v, a);
                    if constexpr (REV) H[v] = a * (value_of<T, V>(rd[j], v) + H[v]);
                    else H[v] = a * H[v] + w * input_of<T, V, DROP>(rx[j], v, (keep[DROP ? v : 0] >> j) & 1u, scale);
                    A[v] *= a;
                }
            }
        }
    };
    if (plain) first_pass(std::true_type{});
    else first_pass(std::false_type{});
#pragma unroll
    for (int v = 0; v < V; ++v) {
        sh_a[wave][lane * V + v] = A[v];
        sh_h[wave][lane * V + v] = H[v];
    }
    if (lane == 0) sh_reset[wave] = starts != 0;
    if (wave == 0) {
        constexpr int j0 = REV ? R - 1 : 0;   // the tile's first row along the scan
        int begin_c = -1;
        if (((live_bits >> j0) & 1) && !((starts >> j0) & 1)) {
            long long begin;
            if (!p.rows.packed) begin = REV ? seq_length(p.rows, n) - 1 : 0;
            else {
                const int s = __builtin_amdgcn_readlane(seq, j0);
                begin = REV ? clamp_row(p.rows.bounds[s + 1], p.rows.T) - 1 : clamp_row(p.rows.bounds[s], p.rows.T);
            }
            begin_c = (int)(REV ? p.chunks - 1 - begin / L : begin / L);
            if (begin_c < 0) begin_c = 0;     // (bounds that decrease)
        }
        if (lane == 0) sh_begin = begin_c;
    }
    __syncthreads();

    // ---- the first V wavefronts publish the tile's map and find its carry, a channel a lane ----
    if (wave < V) {
        const int tc = 64 * wave + lane, tch = (int)(rest % dgroups) * C + tc;
        const bool has = tch < p.D;
        S ta = sh_a[0][tc], th = sh_h[0][tc];
        bool reset = sh_reset[0] != 0;
        for (int w = 1; w < W; ++w) {
            const bool r = sh_reset[w] != 0;
            reset = reset || r;
            const S a = sh_a[w][tc], h = sh_h[w][tc];
            th = r ? h : a * th + h;
            ta *= a;
        }
        const long long D = p.D;
        unsigned long long* agg = p.agg + ((long long)n * p.chunks * D + tch) * WORDS;
        unsigned long long* inc = p.inc + (long long)n * p.groups * D + tch;
        if (has) {
            if constexpr (WORDS == 1) {
                put_word(agg + (long long)c * D, word_of(ta, th));
            } else {
                put_word(agg + (long long)c * D * 2, word_of(ta));
                put_word(agg + (long long)c * D * 2 + 1, word_of(th));
            }
        }
        S carry = S(0);
        const int begin_c = sh_begin;       // the tile in which the sequence of the tile's first row began; -1: this one needs no carry
        if (begin_c >= 0 && has) {
            const int c_group = c / kGroup * kGroup;
            const bool from_group = begin_c < c_group;
            const int from = from_group ? c_group : (begin_c < c ? begin_c : c);
            carry = fold_tiles(agg + (long long)from * D * WORDS, D * WORDS, c - from, from_group ? inc + (long long)(c / kGroup - 1) * D : nullptr, S(0));
        }
        if (has && c % kGroup == kGroup - 1) {
            const S out = reset ? th : ta * carry + th;
            if constexpr (WORDS == 1) put_word(inc + (long long)(c / kGroup) * D, word_of(0.0f, out));
            else put_word(inc + (long long)(c / kGroup) * D, word_of(out));
        }
        sh_carry[tc] = carry;
    }
    __syncthreads();

    // ---- the rows once more, from the carry ----
    const RowsAt oh(reinterpret_cast<const T*>(p.h) + (base + row0) * p.stride_out, p.stride_out);
    const RowsAt odg(reinterpret_cast<const T*>(p.dg) + (base + row0) * p.stride_gate, p.stride_gate);
    const RowsAt odx(reinterpret_cast<const T*>(p.dx) + (base + row0) * p.stride_in, p.stride_in);
    if (live_bits) {
#pragma unroll
        for (int j = 0; j < R; ++j) {
            forget(rg[j]);
            if constexpr (NEED_X) forget(rx[j]);
            if constexpr (REV) forget(rd[j]);
        }
    }
    auto second_pass = [&](auto all) __attribute__((always_inline)) {
        constexpr bool PLAIN = decltype(all)::value;
        S h[V];
#pragma unroll
        for (int v = 0; v < V; ++v) h[v] = sh_carry[lane * V + v];
        for (int w = 0; w < wave; ++w) {
            const bool r = sh_reset[w] != 0;
#pragma unroll
            for (int v = 0; v < V; ++v) h[v] = r ? sh_h[w][lane * V + v] : sh_a[w][lane * V + v] * h[v] + sh_h[w][lane * V + v];
        }
        const unsigned pitch_1 = REV ? odg.pitch : oh.pitch, pitch_2 = odx.pitch;
        unsigned next_1 = col + (REV ? (R - 1) * pitch_1 : 0), next_2 = col + (R - 1) * pitch_2;
#pragma unroll
        for (int i = 0; i < R; ++i) {
            const int j = REV ? R - 1 - i : i;
            const unsigned at_1 = next_1, at_2 = next_2;
            next_1 = REV ? next_1 - pitch_1 : next_1 + pitch_1;
            next_2 -= pitch_2;
            if (!PLAIN && !((live_bits >> j) & 1)) continue;
            if (!PLAIN && ((starts >> j) & 1)) {
                const long long s = __builtin_amdgcn_readlane(seq, j);
#pragma unroll
                for (int v = 0; v < V; ++v) h[v] = init ? init[s * p.D + chl + v] : S(0);
            }
            TV o1, o2;
            S before[V];
            if constexpr (REV) {
                if (!PLAIN && ((ends >> j) & 1)) {   // the row in front of the sequence's first is the initial state
                    const long long s = __builtin_amdgcn_readlane(seq, j);
#pragma unroll
                    for (int v = 0; v < V; ++v) before[v] = p.h0 ? reinterpret_cast<const S*>(p.h0)[s * p.D + chl + v] : S(0);
                } else {
#pragma unroll
                    for (int v = 0; v < V; ++v) before[v] = value_of<T, V>(rh[j], v);
                }
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                S a, w;
                gate_factors<T, SECOND>(value_of<T, V>(rg[j], v), a, w);
                if constexpr (REV) {
                    const S lam = value_of<T, V>(rd[j], v) + h[v];
                    h[v] = a * lam;
                    S dg, du = lam;
                    if constexpr (KIND == DEER_GATE_FACTOR) dg = lam * before[v];
                    else if constexpr (KIND == DEER_GATE_LOG) dg = h[v] * before[v];
                    else {
                        dg = h[v] * w * (before[v] - input_of<T, V, DROP>(rx[j], v, (keep[DROP ? v : 0] >> j) & 1u, scale));
                        du = w * lam;
                    }
                    if constexpr (DROP) du = (keep[v] >> j) & 1u ? du * scale : S(0);
                    vec_set<T, V>(o1, v, (T)dg);
                    vec_set<T, V>(o2, v, (T)du);
                } else {
                    h[v] = a * h[v] + w * input_of<T, V, DROP>(rx[j], v, (keep[DROP ? v : 0] >> j) & 1u, scale);
                    vec_set<T, V>(o1, v, (T)h[v]);
                }
            }
            if constexpr (REV) {
                odg.store(o1, at_1);
                odx.store(o2, at_2);
            } else {
                oh.store(o1, at_1);
            }
            if (!PLAIN && on) {
                if (((ends >> j) & 1) && fin) {
                    const long long s = __builtin_amdgcn_readlane(seq, j);
#pragma unroll
                    for (int v = 0; v < V; ++v) fin[s * p.D + ch + v] = h[v];
                }
            }
        }
    };
    if (plain) second_pass(std::true_type{});
    else second_pass(std::false_type{});
}

// Clears the published words, the ticket and, on request, rows of no sequence, and gives sequences without rows their final state (in the gradient: the
// gradient of their initial state).  A kernel and no memset: the call may be captured into a graph.
template <typename S>
__global__ __launch_bounds__(256) void diagrec_prepare_kernel(const DiagrecParams p, bool grad, const RestRows rest) {
    clear_rest(p.rows, rest, blockIdx.x, gridDim.x);
    const size_t at = (size_t)blockIdx.x * blockDim.x + threadIdx.x, all = (size_t)gridDim.x * blockDim.x;
    for (size_t i = at; i < p.words; i += all) p.agg[i] = kUnset;
    if (at == 0) *p.ticket = 0;
    const S* from = reinterpret_cast<const S*>(grad ? p.dlast : p.h0);
    S* to = reinterpret_cast<S*>(grad ? p.dh0 : p.last);
    if (!to) return;
    for (long long i = at; i < (long long)p.rows.N * p.D; i += all) {
        if (seq_length(p.rows, (int)(i / p.D)) == 0) to[i] = from ? from[i] : S(0);
    }
}

template <typename T, int KIND, bool REV, bool DROP>
hipError_t launch_one(const DiagrecParams& p, int V, hipStream_t stream) {
    using Sh = Shape<T, REV>;
    const long long seqs = p.rows.packed ? 1 : p.rows.N, groups = (p.D + 64 * V - 1) / (64 * V);
    const dim3 grid((unsigned)(seqs * groups * p.chunks)), block(64 * Sh::W);
    if (grid.x == 0) return hipSuccess;
    if (V == 1) hipLaunchKernelGGL((diagrec_kernel<T, KIND, 1, Sh::R, Sh::W, REV, DROP>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((diagrec_kernel<T, KIND, Sh::V, Sh::R, Sh::W, REV, DROP>), grid, block, 0, stream, p);
    return hipGetLastError();
}

template <typename T, bool REV>
hipError_t launch_type(const DiagrecParams& p, hipStream_t stream) {
    using S = wide_t<T>;
    const long long cells = (long long)p.rows.N * p.D;
    const size_t work = p.words > (size_t)cells ? p.words : (size_t)cells;
    RestRows rest{};
    if (p.zero_rest) {
        auto add = [&](void* first, long long stride) { rest.array[rest.count++] = RestArray{first, stride * (long long)sizeof(T), p.D * (long long)sizeof(T)}; };
        if (REV) {
            add(p.dg, p.stride_gate);
            add(p.dx, p.stride_in);
        } else {
            add(p.h, p.stride_out);
        }
    }
    const long long tiles = rest.count ? (p.rows.T + 15) / 16 * (p.rows.packed ? 1 : p.rows.N) : 0;
    const long long want = (long long)(work / 1024) > tiles ? (long long)(work / 1024) : tiles;
    const unsigned blocks = (unsigned)(want < 1 ? 1 : want > 2048 ? 2048 : want);
    hipLaunchKernelGGL((diagrec_prepare_kernel<S>), dim3(blocks), dim3(256), 0, stream, p, REV, rest);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    // Vectors of V channels where every row of every array begins at a multiple of them: 4 x 16,384 x 1,024 in bf16 98 + 141 us (forward + backward), a
    // channel a lane 129 + 211; fp32 169 + 260 and 196 + 346.  Up to 64 channels a channel a lane fills the wavefronts: 64 x 4,096 x 64 in bf16 36 + 46 us
    // against 39 + 49 with half of the lanes idle, fp32 48 + 79 against 60 + 103.
    constexpr int VV = Shape<T, REV>::V;
    auto fits = [](const void* q, long long stride) {
        return reinterpret_cast<uintptr_t>(q) % (VV * sizeof(T)) == 0 && stride % VV == 0;
    };
    bool vec = p.D % VV == 0 && p.D > 64 && fits(p.g, p.stride_gate) && fits(p.x, p.stride_in) && fits(p.h, p.stride_out);
    if (REV) vec = vec && fits(p.dh, p.stride_out) && fits(p.dg, p.stride_gate) && fits(p.dx, p.stride_in);
    const int V = vec ? VV : 1;
    const bool drop = p.drop.cut != 0;
    switch (p.gate) {
        case DEER_GATE_FACTOR: return drop ? launch_one<T, DEER_GATE_FACTOR, REV, true>(p, V, stream) : launch_one<T, DEER_GATE_FACTOR, REV, false>(p, V, stream);
        case DEER_GATE_LOG: return drop ? launch_one<T, DEER_GATE_LOG, REV, true>(p, V, stream) : launch_one<T, DEER_GATE_LOG, REV, false>(p, V, stream);
        default: return drop ? launch_one<T, DEER_GATE_SIGMOID, REV, true>(p, V, stream) : launch_one<T, DEER_GATE_SIGMOID, REV, false>(p, V, stream);
    }
}

// One token for every row: state <- a state + u in place.  A row whose slot is out of range, or has come in an earlier row, is
// passed over.  Latency bound (32 rows of 2,048 channels: 3 us, 11 with the call from Python): one launch, every lane one channel, the slots in front looked at while the operands are on their way.
template <typename T, int KIND>
__global__ __launch_bounds__(256) void diagstep_kernel(const DiagstepParams p) {
    using S = wide_t<T>;
    const int per = (p.D + 255) / 256, n = blockIdx.x / per, ch = (blockIdx.x % per) * 256 + threadIdx.x;
    int slot = n;
    bool twice = false;
    if (p.rows.slots) {
        slot = p.rows.slots[n];
        for (int m = threadIdx.x; m < n; m += 256) twice = twice || p.rows.slots[m] == slot;
    }
    const bool in = ch < p.D && slot >= 0 && slot < p.rows.n_slots;
    S g = S(0), x = S(0), h = S(0);
    S* state = reinterpret_cast<S*>(p.state) + (long long)slot * p.D + ch;
    if (in) {
        g = (S)reinterpret_cast<const T*>(p.g)[(long long)n * p.stride_gate + ch];
        x = (S)reinterpret_cast<const T*>(p.x)[(long long)n * p.stride_in + ch];
        h = *state;
    }
    twice = p.rows.slots ? __syncthreads_or(twice) != 0 : false;
    if (!in || twice) {
        if (p.rows.zero_rest && ch < p.D) reinterpret_cast<T*>(p.h)[(long long)n * p.stride_out + ch] = (T)0;
        return;
    }
    S a, w;
    gate_factors<T, KIND>(g, a, w);
    h = a * h + w * x;
    *state = h;
    reinterpret_cast<T*>(p.h)[(long long)n * p.stride_out + ch] = (T)h;
}

template <typename T>
hipError_t launch_step_type(const DiagstepParams& p, hipStream_t stream) {
    const dim3 grid((unsigned)((long long)((p.D + 255) / 256) * p.rows.N)), block(256);
    if (p.gate == DEER_GATE_FACTOR) hipLaunchKernelGGL((diagstep_kernel<T, DEER_GATE_FACTOR>), grid, block, 0, stream, p);
    else if (p.gate == DEER_GATE_LOG) hipLaunchKernelGGL((diagstep_kernel<T, DEER_GATE_LOG>), grid, block, 0, stream, p);
    else hipLaunchKernelGGL((diagstep_kernel<T, DEER_GATE_SIGMOID>), grid, block, 0, stream, p);
    return hipGetLastError();
}

template <typename T, bool REV> constexpr int tile_rows() { return Shape<T, REV>::R * Shape<T, REV>::W; }

}  // namespace

size_t diagrec_words(int dtype, int N, long long T, int D, bool grad, int* chunks, int* groups, size_t* agg_words) {
    const int L = dtype == DEER_F64   ? (grad ? tile_rows<double, true>() : tile_rows<double, false>())
                  : dtype == DEER_F32 ? (grad ? tile_rows<float, true>() : tile_rows<float, false>())
                                      : (grad ? tile_rows<BF16, true>() : tile_rows<BF16, false>());
    const long long c = (T + L - 1) / L, g = (c + kGroup - 1) / kGroup;
    *chunks = (int)c;
    *groups = (int)g;
    *agg_words = (size_t)N * c * D * (dtype == DEER_F64 ? 2 : 1);
    return *agg_words + (size_t)N * g * D;
}

hipError_t launch_diagrec(int dtype, bool grad, const DiagrecParams& p, hipStream_t stream) {
    switch (dtype) {
        case DEER_F32: return grad ? launch_type<float, true>(p, stream) : launch_type<float, false>(p, stream);
        case DEER_F64: return grad ? launch_type<double, true>(p, stream) : launch_type<double, false>(p, stream);
        case DEER_BF16: return grad ? launch_type<BF16, true>(p, stream) : launch_type<BF16, false>(p, stream);
        default: return grad ? launch_type<F16, true>(p, stream) : launch_type<F16, false>(p, stream);
    }
}

hipError_t launch_diagstep(int dtype, const DiagstepParams& p, hipStream_t stream) {
    switch (dtype) {
        case DEER_F32: return launch_step_type<float>(p, stream);
        case DEER_F64: return launch_step_type<double>(p, stream);
        case DEER_BF16: return launch_step_type<BF16>(p, stream);
        default: return launch_step_type<F16>(p, stream);
    }
}

}  // namespace deer
