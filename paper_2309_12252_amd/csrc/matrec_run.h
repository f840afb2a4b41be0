// The run over a segment's chunks that all products with a state share (matrec.hip: outputs; matrec_grad.hip: dq, dk, dv).  For rows a, b of D1 columns,
// c of D2 columns and a state M [D1][D2] that it carries along,
//   out_i = f_i M^T a_i + sum_{j <= i} scale e^{c_i - c_j} (a_i . b_j) c_j,     M <- e^{c_64} M + sum_j w_j b_j c_j^T.
//   Out  a, b, c = q, k, v         M = S     f_i = scale e^{c_i}      w_j = e^{c_64 - c_j}
//   Dq   a, b, c = dout, v, k      M = S^T   the same
//   Dk   a, b, c = v, dout, q      M = R^T   rows and chunks backwards: c_i stands for -c_i, f_i = e^{c_64 - c_i}, w_j = scale e^{c_j}
//   Dv   a, b, c = k, q, dout      M = R     backwards, the same
// (S the state in front of a chunk, R the gradient of the state behind it.)  Wavefront w has 16 of c's columns: M's, as
// results, which are operands of M^T a as they stand, and the outputs', transposed, a lane four neighbouring columns of a row.
// What bounds it: 80 to 120 matrix instructions of 16 cycles and some 900 other vector instructions a wavefront and chunk of 128 columns, which a SIMD does one
// after another, and 64 KiB of rows a chunk.  Two workgroups fill a CU and go on while the other one waits for its rows, which go straight to LDS: no
// registers for them, so that 128 are enough (one workgroup a CU with its next rows in registers: gradient of 4 x 4,096 rows, 16 heads of
// 128 x 128, 431 us; so 309 to 345).  Vector instructions take 60 % of a SIMD's cycles there and matrix instructions 25 %, and they do not overlap.  Outputs: 49 us for prompts of 8,192 rows
// and 16 heads of 128 x 128, 54 for 1 x 32,768 rows and 8 heads of 128 x 64, 83 for 4 x 4,096 rows and 16 heads of 128 x 128.  fp32: the
// products are four-term instructions of 32 cycles and bound it.
#pragma once
#include "matrec_common.h"

namespace deer {
namespace {

enum MatRun { RUN_OUT, RUN_DQ, RUN_DK, RUN_DV };

template <typename T, int D1, int D2, int W, int MODE>
struct RunLds {
    static constexpr bool FOUR = MODE == RUN_DQ;        // q, for the gates
    static constexpr bool SUMS = MODE == RUN_DQ || MODE == RUN_DK;
    // Pieces in bf16.  READ: of the state in M^T a; all where the gates' sums take it as it is.  TAKE: of what rows add to the state; two where it is only read as
    // two.  PAIRS: of the pairs' weights.  So results are as exact as their own rounding makes them: all together 1.66e-3 off, with one piece each 2.35e-3 (prompts
    // of 8,192 rows 92 us instead of 96, training step of 4 x 4,096 rows 4 % less).
    static constexpr int P = Op<T>::PIECES, READ = SUMS || P == 1 ? P : 2, TAKE = MODE == RUN_DV && P > 1 ? 2 : P, PAIRS = P > 1 ? 2 : 1;
    using Weights = Pairs<T, PAIRS, FOUR && P != 1>;
    static constexpr size_t a = 0, b = Tile<T, D1>::bytes, c = b + Tile<T, D1>::bytes, q = c + Tile<T, D2>::bytes, pairs = q + (FOUR ? Tile<T, D2>::bytes : 0),
                            rows = pairs + Weights::bytes,               // cum_hi, cum_lo, f, w, and the chunk's factor
                            dots = rows + 4 * 5 * 64,                    // [W][64]
                            by_col = dots + (SUMS ? 4 * 64 * W : 0),   // [row tile][64]
                            by_row = by_col + (FOUR ? 4 * 256 : 0),      // [column tile][64]
                            size = by_row + (FOUR ? 4 * 256 : 0),        // [W][16]: squares of the state's columns
                            total = size + (SUMS ? 4 * 16 * W : 0);
    static_assert(total <= 160 * 1024 / (sizeof(T) == 2 ? 2 : 1), "a workgroup's tiles fit the CU's LDS, in bf16 two workgroups'");
};

// a state of Dk x Dv in the caller's layout, or a whole tile DK x DV: element (k row, v column), and four neighbouring columns
struct StateAt {
    const float* at;
    int Dk, Dv, ld;
    bool fours;      // every row aligned to 16 bytes
    __device__ __forceinline__ StateAt(const float* from, int dk, int dv, int pitch)
        : at(from), Dk(dk), Dv(dv), ld(pitch), fours(dv % 4 == 0 && pitch % 4 == 0 && reinterpret_cast<uintptr_t>(from) % 16 == 0) {}
    __device__ __forceinline__ float operator()(int d, int v) const { return at && d < Dk && v < Dv ? at[d * ld + v] : 0.0f; }
    __device__ __forceinline__ F32x4 four(int d, int v) const {
        F32x4 x = {0, 0, 0, 0};
        if (!at || d >= Dk) return x;
        if (fours) {
            if (v < Dv) x = *reinterpret_cast<const F32x4*>(at + d * ld + v);
        } else {
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (v + r < Dv) x[r] = at[d * ld + v + r];
        }
        return x;
    }
};

template <typename T, int DK, int DV, int W, int MODE>
__device__ __forceinline__ void matrec_run(const MatrecParams& p, unsigned char* lds, int id) {
    constexpr bool BACK = MODE == RUN_DK || MODE == RUN_DV, KEYS = MODE == RUN_DQ || MODE == RUN_DK;   // KEYS: D1 is the values', D2 the keys'
    constexpr int D1 = KEYS ? DV : DK, D2 = KEYS ? DK : DV, KS = D1 / 32, NT = D1 / 16, P = Op<T>::PIECES;
    static_assert(16 * W >= D2, "a wavefront has 16 of c's columns");
    using L = RunLds<T, D1, D2, W, MODE>;
    using T1 = Tile<T, D1>;
    using T2 = Tile<T, D2>;
    using TP = typename L::Weights;
    using V4 = T __attribute__((ext_vector_type(4)));
    const int lane0 = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int lane = lane0, g = lane >> 4, l = lane & 15;
    const int seg_no = id / p.Hv, head = id % p.Hv, kh = head / (p.Hv / p.Hk);
    MatSegment seg;
    if (!segment_of(p, seg_no, seg)) return;
    const int d1 = KEYS ? p.Dv : p.Dk, d2 = KEYS ? p.Dk : p.Dv;
    const bool strip = 16 * wave < D2;                                           // (this wavefront has columns)
    const int col0 = column_of(wave, 4 * g);                                     // a lane's first of four

    // ---- arrays of rows ----
    const T* q = reinterpret_cast<const T*>(p.q) + (long long)kh * p.Dk + seg.row0 * p.stride_q;
    const T* k = reinterpret_cast<const T*>(p.k) + (long long)kh * p.Dk + seg.row0 * p.stride_k;
    const T* v = reinterpret_cast<const T*>(p.v) + (long long)head * p.Dv + seg.row0 * p.stride_v;
    const T* d = MODE == RUN_OUT ? nullptr : reinterpret_cast<const T*>(p.dout) + (long long)head * p.Dv + seg.row0 * p.stride_o;
    const T *ra = MODE == RUN_OUT ? q : MODE == RUN_DQ ? d : MODE == RUN_DK ? v : k, *rb = MODE == RUN_OUT ? k : MODE == RUN_DQ ? v : MODE == RUN_DK ? d : q,
            *rc = MODE == RUN_OUT ? v : MODE == RUN_DQ ? k : MODE == RUN_DK ? q : d;
    const long long sa = MODE == RUN_OUT ? p.stride_q : MODE == RUN_DQ ? p.stride_o : MODE == RUN_DK ? p.stride_v : p.stride_k,
                    sb = MODE == RUN_OUT ? p.stride_k : MODE == RUN_DQ ? p.stride_v : MODE == RUN_DK ? p.stride_o : p.stride_q,
                    sc = MODE == RUN_OUT ? p.stride_v : MODE == RUN_DQ ? p.stride_k : MODE == RUN_DK ? p.stride_q : p.stride_o;
    // outputs: rows of T, or of floats where heads that share one are added later
    const bool parts = KEYS && p.Hv != p.Hk;
    T* out = MODE == RUN_OUT ? reinterpret_cast<T*>(p.o) + (long long)head * p.Dv : MODE == RUN_DV ? reinterpret_cast<T*>(p.dv) + (long long)head * p.Dv
             : reinterpret_cast<T*>(MODE == RUN_DQ ? p.dq : p.dk) + (long long)kh * p.Dk;
    const long long so = MODE == RUN_OUT ? p.stride_o : MODE == RUN_DV ? p.stride_v : MODE == RUN_DQ ? p.stride_q : p.stride_k;
    out += seg.row0 * so;
    float* out_part = parts ? (MODE == RUN_DQ ? p.part_q : p.part_k) + (seg.row0 * p.Hv + head) * p.Dk : nullptr;
    const bool wide_out = parts ? p.Dk % 4 == 0 : four_wide(out, so, d2);
    const float* gates = p.rows_of + ((long long)seg.chunk0 * p.Hv + head) * kRowFloats;

    // ---- the state ----
    const int chunks = (int)((seg.rows + kChunk - 1) / kChunk);
    const bool first = seg.index == 0, last = seg.index == seg.count - 1;
    const long long cells = (long long)p.Dk * p.Dv, of_seq = ((long long)seg.seq * p.Hv + head) * cells, of_seg = ((long long)seg_no * p.Hv + head) * (DK * DV);
    F32x4 M[NT];
    {
        const bool given = BACK ? last : first;
        const StateAt st = given ? StateAt{BACK ? (p.dlast ? p.dlast + of_seq : nullptr) : (p.s0 ? p.s0 + of_seq : nullptr), p.Dk, p.Dv, p.Dv}
                                 : StateAt{(BACK ? p.seg_rstate : p.seg_state) + of_seg, DK, DV, DV};
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int x = column_of(t, 4 * g), y = column_of(wave, l);   // (and the three rows behind x)
            if constexpr (KEYS) M[t] = st.four(y, x);
            else M[t] = F32x4{st(x, y), st(x + 1, y), st(x + 2, y), st(x + 3, y)};
        }
    }
    // the state behind the run's last chunk is wanted: the final one, or what the gates and ds0 need
    const bool to_the_end = MODE == RUN_OUT ? last && p.last : MODE == RUN_DK;

    // ---- a chunk's rows into LDS ----
    const bool wide_a = wide_rows(ra, sa, d1), wide_b = wide_rows(rb, sb, d1), wide_c = wide_rows(rc, sc, d2), wide_q = wide_rows(q, p.stride_q, p.Dk), wide_k = wide_rows(k, p.stride_k, p.Dk);
    auto rows_of = [&](int c, long long& row) {
        row = (long long)(BACK ? chunks - 1 - c : c) * kChunk;
        return seg.rows - row < kChunk ? (int)(seg.rows - row) : kChunk;
    };
    T *ta = reinterpret_cast<T*>(lds + L::a), *tb = reinterpret_cast<T*>(lds + L::b), *tc = reinterpret_cast<T*>(lds + L::c), *tq = reinterpret_cast<T*>(lds + L::q),
      *tp = reinterpret_cast<T*>(lds + L::pairs);
    float *cum_hi = reinterpret_cast<float*>(lds + L::rows), *cum_lo = cum_hi + 64, *f_out = cum_hi + 128, *w_in = cum_hi + 192;
    float *dots = reinterpret_cast<float*>(lds + L::dots), *by_col = reinterpret_cast<float*>(lds + L::by_col), *by_row = reinterpret_cast<float*>(lds + L::by_row),
          *size = reinterpret_cast<float*>(lds + L::size);
    auto load = [&](int c) {
        long long row;
        const int rows = rows_of(c, row), i = again(lane0);
        load_tile<T, D1, W, BACK>(ta, ra + row * sa, sa, rows, d1, wide_a, i);
        load_tile<T, D1, W, BACK>(tb, rb + row * sb, sb, rows, d1, wide_b, i);
        load_tile<T, D2, W, BACK>(tc, rc + row * sc, sc, rows, d2, wide_c, i);
        if constexpr (L::FOUR) load_tile<T, D2, W, BACK>(tq, q + row * p.stride_q, p.stride_q, rows, d2, wide_q, i);
        // cum_hi, cum_lo, f, w, whole; backwards: rows turned round, f and w the other way round
        const float* from = gates + (long long)(BACK ? chunks - 1 - c : c) * p.Hv * kRowFloats;
        for (int n = wave; n < 5; n += W) load_floats(cum_hi + 64 * n, from, 64 * (!BACK || n < 2 || n > 3 ? n : 5 - n) + (BACK && n < 4 && i < rows ? rows - 1 - i : i));
    };
    // what is never written but taken in: pairs above the diagonal, sums of tiles there
    if (wave == 0) TP::clear(tp, l, g);
    if constexpr (L::FOUR) {
        if (threadIdx.x < 256) by_col[threadIdx.x] = by_row[threadIdx.x] = 0.0f;
    }
    load(0);
    wait_loads();
    __syncthreads();

    for (int c = 0; c < chunks; ++c) {
        lane = again(lane0);
        g = lane >> 4;
        l = lane & 15;
        const float whole = w_in[64];
        long long row;
        const int rows = rows_of(c, row);
        const bool more = c + 1 < chunks;

        // Dk: this lane's columns of k, for the gates, on their way while the pairs are computed
        V4 kr[MODE == RUN_DK ? 4 : 1];
        if constexpr (MODE == RUN_DK) {
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const int i = 16 * t + l;
                const T* from = k + (row + rows - 1 - i) * p.stride_k + col0;
                V4 x = {};
                if (strip && i < rows) {
                    if (wide_k) {
                        if (col0 < p.Dk) x = *reinterpret_cast<const V4*>(from);
                    } else {
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (col0 + r < p.Dk) x[r] = from[r];
                    }
                }
                kr[t] = x;
            }
        }

        // ---- pairs, tile by tile, transposed: a lane has one i and four neighbouring j ----
        auto pair_tile = [&](int n) {
            int ti, tj;
            lower_tile(n, ti, tj);
            const int i = 16 * ti + l, j0 = 16 * tj + 4 * g;
            F32x4 x = {0, 0, 0, 0};
#pragma unroll
            for (int s = 0; s < KS; ++s) x = mma(T1::row_frag(tb, 16 * tj + l, s, g), T1::row_frag(ta, i, s, g), x);
            const float hi_i = cum_hi[i], lo_i = cum_lo[i];
            const F32x4 hj = *reinterpret_cast<const F32x4*>(cum_hi + j0), lj = *reinterpret_cast<const F32x4*>(cum_lo + j0);
#pragma unroll
            for (int r = 0; r < 4; ++r) x[r] = j0 + r <= i ? p.scale * x[r] * (BACK ? decay_between(hj[r], lj[r], hi_i, lo_i) : decay_between(hi_i, lo_i, hj[r], lj[r])) : 0.0f;
            TP::store(tp, ti, tj, l, g, x);
            if constexpr (MODE == RUN_DQ) {
                // the gates' pairs: (dout_i . v_j) (q_i . k_j), summed over j along every row i, over the rows by groups of 16
                F32x4 y = {0, 0, 0, 0};
#pragma unroll
                for (int s = 0; s < D2 / 32; ++s) y = mma(T2::row_frag(tc, 16 * tj + l, s, g), T2::row_frag(tq, i, s, g), y);
                F32x4 upto;
#pragma unroll
                for (int r = 0; r < 4; ++r) upto[r] = (r > 0 ? upto[r > 0 ? r - 1 : 0] : 0.0f) + (j0 + r < i ? x[r] * y[r] : 0.0f);
                // the lane groups in front of this one have the smaller j
                float front = upto[3];
                const float one = __shfl_up(front, 16);
                front += g >= 1 ? one : 0.0f;
                const float two = __shfl_up(front, 32);
                front += g >= 2 ? two : 0.0f;
                const float before = __shfl_up(front, 16);
                if (g == 3) by_row[64 * tj + i] = front;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float s = group_sum(j0 + r < i ? upto[r] + (g >= 1 ? before : 0.0f) : 0.0f);
                    if (l == 0) by_col[64 * ti + j0 + r] = s;
                }
            }
        };
        // Products go in front of the other workgroup's wavefronts, which load or store, the state's in front of all: outputs of 4 x 4,096 rows
        // and 16 heads of 128 x 128 99 -> 83 us, gradient 350 -> 321.
        __builtin_amdgcn_s_setprio(1);
        pair_tile(wave);
        if (W < 8) pair_tile(wave + W);
        if (wave < 10 % W) pair_tile(wave + 10 / W * W);

        __builtin_amdgcn_s_setprio(2);
        // ---- the state: what it gives to the outputs, then the chunk's rows into it ----
        F32x4 acc[4];
        frag_t<T> cf[2];
#pragma unroll
        for (int t = 0; t < 4; ++t) acc[t] = F32x4{0, 0, 0, 0};
        if (strip) {
        // L::SUMS: how large the state is, for the bound of what goes through the chunk, from its first pieces: products of its columns with each other, of
        // which the diagonal is taken (four matrix instructions, which have time; fp32: sums of squares)
        F32x4 square = {0, 0, 0, 0};
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            frag_t<T> m[L::READ];
            pieces_of<T>(joined(M[2 * s], M[2 * s + 1]), m);
            if constexpr (L::SUMS) {
                if constexpr (P > 1) square = mma(m[0], m[0], square);
                else square += M[2 * s] * M[2 * s] + M[2 * s + 1] * M[2 * s + 1];
            }
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const frag_t<T> af = T1::row_frag(ta, 16 * t + l, s, g);
#pragma unroll
                for (int n = L::READ - 1; n >= 0; --n) acc[t] = mma(m[n], af, acc[t]);
            }
        }
        if constexpr (L::SUMS) {
            float x = (l & 2) != 0 ? ((l & 1) != 0 ? square[3] : square[2]) : (l & 1) != 0 ? square[1] : square[0];
            if constexpr (P == 1) {
                x = (square[0] + square[1]) + (square[2] + square[3]);
                x += __shfl_xor(x, 16);
                x += __shfl_xor(x, 32);
            }
            if (g == l >> 2) size[16 * wave + l] = x;
        }
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int i = 16 * t + l;
            const float f = f_out[i];
            acc[t] *= f;
            if constexpr (L::SUMS) {   // q_i (Dk: k_i) with what came in
                float x = 0.0f;
                V4 with;
                if constexpr (MODE == RUN_DQ) with = *reinterpret_cast<const V4*>(tq + T2::at(i, col0));
                else with = kr[t];
#pragma unroll
                for (int r = 0; r < 4; ++r) x += (float)with[r] * acc[t][r];
                x += __shfl_xor(x, 16);
                x += __shfl_xor(x, 32);
                if (g == 0) dots[64 * wave + i] = x;
            }
        }
#pragma unroll
        for (int s = 0; s < 2; ++s) cf[s] = T2::col_frag(tc, s, wave, lane);
        if (more || to_the_end) {
#pragma unroll
            for (int t = 0; t < NT; ++t) M[t] *= whole;
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const F32x4 w0 = *reinterpret_cast<const F32x4*>(w_in + 32 * s + 8 * g), w1 = *reinterpret_cast<const F32x4*>(w_in + 32 * s + 8 * g + 4);
                frag_t<T> cp[L::TAKE];
                pieces_of<T>(widened(cf[s]) * joined(w0, w1), cp);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const frag_t<T> bf = T1::col_frag(tb, s, t, lane);
#pragma unroll
                    for (int n = L::TAKE - 1; n >= 0; --n) M[t] = mma(bf, cp[n], M[t]);
                }
            }
        }
        } else if (L::SUMS) {
            dots[64 * wave + lane] = 0.0f;
            if (g == 0) size[16 * wave + l] = 0.0f;
        }
        __syncthreads();

        __builtin_amdgcn_s_setprio(0);
        // ---- the pairs' part ----
        if (strip) {
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
                for (int t = 2 * s; t < 4; ++t) {
#pragma unroll
                    for (int n = L::PAIRS - 1; n >= 0; --n) acc[t] = mma(cf[s], TP::row_frag(tp, n, t, s, l, g), acc[t]);
                }
        }
        const long long chunk = (long long)(seg.chunk0 + (BACK ? chunks - 1 - c : c)) * p.Hv + head;
        if (L::SUMS && p.dgate && wave == 0) {
            const float squares = wave_sum(size[lane] + (W > 4 ? size[W > 4 ? 64 + lane : 0] : 0.0f));
            if (lane == 63) (MODE == RUN_DQ ? p.size_in : p.size_out)[chunk] = squares;
        }
        if (L::SUMS && p.dgate && wave == W - 1) {
            // A lane has row i.  Dq: sums from i on of what is read there, and the pairs that pass i.  Dk (backwards): sums behind i of
            // what is put out there, i.e. of the rows in front.
            float x = 0.0f;
#pragma unroll
            for (int w = 0; w < W; ++w) x += dots[64 * w + lane];
            float pairs = 0.0f, tile[3] = {0.0f, 0.0f, 0.0f};
            if constexpr (MODE == RUN_DQ) {
#pragma unroll
                for (int w = 0; w < 4; ++w) pairs += lane > 0 ? by_col[64 * w + lane - 1] : 0.0f;
#pragma unroll
                for (int w = 0; w < 3; ++w) tile[w] = by_row[64 * w + lane];
            }
#pragma unroll
            for (int n = 1; n < 64; n *= 2) {
                const float a = __shfl_down(x, n);
                x += lane + n < 64 ? a : 0.0f;
                if constexpr (MODE == RUN_DQ) {
#pragma unroll
                    for (int w = 0; w < 3; ++w) {
                        const float a2 = __shfl_down(tile[w], n);
                        tile[w] += lane + n < 64 ? a2 : 0.0f;
                    }
                }
            }
            if (lane == 0) (MODE == RUN_DQ ? p.read_in : p.put_out)[chunk] = x;
            if constexpr (MODE == RUN_DQ) {
#pragma unroll
                for (int w = 0; w < 3; ++w) pairs += lane > 16 * (w + 1) ? tile[w] : 0.0f;
                if (lane < rows) p.dgate[(seg.row0 + row + lane) * p.Hv + head] = pairs + x;
            } else {
                const float next = __shfl_down(x, 1);
                if (lane < rows) p.gate_k[(seg.row0 + row + rows - 1 - lane) * p.Hv + head] = lane < 63 ? next : 0.0f;
            }
        }
        if (strip && col0 < d2) {
            const int i0 = again(lane0) & 15;
            const long long first_row = row + (BACK ? rows - 1 - i0 : i0);
            const int back = BACK ? -16 : 16;
            T* to = out + first_row * so + col0;
            float* to_part = parts ? out_part + first_row * p.Hv * p.Dk + col0 : nullptr;
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                if (16 * t + i0 < rows) {
                    if (parts) store_four<float>(to_part + (long long)t * back * p.Hv * p.Dk, acc[t], d2 - col0, wide_out);
                    else store_four<T>(to + (long long)t * back * so, acc[t], d2 - col0, wide_out);
                }
            }
        }
        if (more) load(c + 1);   // over the tiles; the pairs and the sums lie beside them
        wait_loads();
        __syncthreads();
    }

    // ---- the state at the run's end ----
    if (MODE == RUN_OUT && to_the_end) {
        float* to = p.last + of_seq;
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int x = column_of(t, 4 * g + r), y = column_of(wave, l);
                if (x < p.Dk && y < p.Dv) to[(long long)x * p.Dv + y] = M[t][r];
            }
    }
    if constexpr (MODE == RUN_DK) {
        // the gradient of the state in front of the segment: ds0 of its sequence, and its product with that state for the gates
        const StateAt st = first ? StateAt{p.s0 ? p.s0 + of_seq : nullptr, p.Dk, p.Dv, p.Dv} : StateAt{p.seg_state + of_seg, DK, DV, DV};
        const bool wide_ds0 = p.Dv % 4 == 0 && reinterpret_cast<uintptr_t>(p.ds0) % 16 == 0;
        float x = 0.0f;
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int vv = column_of(t, 4 * g), dd = column_of(wave, l);
            const F32x4 y = st.four(dd, vv);
#pragma unroll
            for (int r = 0; r < 4; ++r) x += y[r] * M[t][r];
            if (first && p.ds0 && dd < p.Dk && vv < p.Dv) store_four<float>(p.ds0 + of_seq + (long long)dd * p.Dv + vv, M[t], p.Dv - vv, wide_ds0);
        }
        x = group_sum(x);
        x += __shfl_xor(x, 16);
        x += __shfl_xor(x, 32);
        __syncthreads();
        float* sums = reinterpret_cast<float*>(lds);
        if (lane == 0) sums[wave] = x;
        __syncthreads();
        if (threadIdx.x == 0 && p.dgate) {
            float total = 0.0f;
            for (int w = 0; w < W; ++w) total += sums[w];
            p.front[(long long)seg_no * p.Hv + head] = total;
        }
    }
}

template <typename K>
hipError_t launch_lds(K kernel, dim3 grid, int threads, size_t lds, const MatrecParams& p, hipStream_t stream) {
    if (grid.x == 0) return hipSuccess;
    hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, grid, dim3(threads), lds, stream, p);
    return hipGetLastError();
}

#define DEER_BY_SHAPE(F, T, ...)                                                                                                      \
    (p.Dk <= 64 ? (p.Dv <= 64 ? F<T, 64, 64>(p, __VA_ARGS__) : F<T, 64, 128>(p, __VA_ARGS__)) : (p.Dv <= 64 ? F<T, 128, 64>(p, __VA_ARGS__) : F<T, 128, 128>(p, __VA_ARGS__)))

}  // namespace
}  // namespace deer
