// C entry points of the sequence operators (include/deer.h): checks of the arguments, the workspace's layout, launches.  Nothing
// here allocates or synchronises.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdio>

#include "matrec_common.h"
#include "seq_check.h"

using namespace deer;

namespace {

const char* bad_drop(double p) {
    if (!(p >= 0.0 && p < 1.0)) return "dropout: the share that is dropped must lie in [0, 1)";
    if (std::lround(p * 65536.0) > 65535) return "dropout: the share that is dropped must be at most 1 - 2^-16";
    return nullptr;
}
DropParams drop_params(double p, uint64_t seed, uint32_t draw) {
    DropParams d;
    d.seed_lo = (unsigned)seed;
    d.seed_hi = (unsigned)(seed >> 32);
    d.draw = draw;
    d.cut = (unsigned)std::lround(p * 65536.0);
    d.scale = 65536.0 / (65536.0 - d.cut);
    return d;
}

const char* bad_config(const deer_diagrec_config* c, bool step) {
    if (!c) return "config is NULL";
    if (!known_type(c->dtype)) return "unknown dtype";
    if (c->gate != DEER_GATE_FACTOR && c->gate != DEER_GATE_LOG && c->gate != DEER_GATE_SIGMOID) return "unknown gate";
    if (c->N < 1 || c->D < 1) return "N and D must be positive";
    if (c->stride_gate < 0 || c->stride_in < 0 || c->stride_out < 0) return "strides must not be negative";
    if ((c->stride_gate && c->stride_gate < c->D) || (c->stride_in && c->stride_in < c->D) || (c->stride_out && c->stride_out < c->D))
        return "a stride is smaller than a row";
    if (step) return nullptr;
    if (c->T < 0 || (c->packed & ~(int)DEER_REST_ZERO & ~1)) return "T must not be negative, packed 0 or 1 (and DEER_REST_ZERO)";
    return bad_drop(c->drop);
}
struct DiagLayout {
    int chunks, groups;
    size_t agg_words, words, total;
};
DiagLayout diag_layout(const deer_diagrec_config* c, bool grad) {
    DiagLayout l;
    l.words = diagrec_words(c->dtype, is_packed(c) ? 1 : c->N, c->T, c->D, grad, &l.chunks, &l.groups, &l.agg_words);
    l.total = kAlign + align_up(l.words * 8);
    return l;
}

bool too_large(const deer_diagrec_config* c, bool grad) {
    if (c->T > kMostRows || c->D > kMostStride || c->stride_gate > kMostStride || c->stride_in > kMostStride || c->stride_out > kMostStride) return true;
    if ((long double)c->N * c->D > 1e15L) return true;
    const long double seqs = is_packed(c) ? 1 : c->N, cols = (c->D + 63) / 64;   // (a channel a lane: most workgroups)
    return cols * seqs * diag_layout(c, grad).chunks * kDiagLanes > kMostLanes;
}

DiagrecParams diag_params(const deer_diagrec_config* c, const DiagLayout& l, const int64_t* bounds, void* ws) {
    DiagrecParams p{};
    p.rows = SeqRows{reinterpret_cast<const long long*>(bounds), c->T, c->N, is_packed(c)};
    p.D = c->D;
    p.gate = c->gate;
    p.stride_gate = c->stride_gate ? c->stride_gate : c->D;
    p.stride_in = c->stride_in ? c->stride_in : c->D;
    p.stride_out = c->stride_out ? c->stride_out : c->D;
    p.drop = drop_params(c->drop, c->seed, c->draw);
    p.zero_rest = zero_rest(c);
    p.chunks = l.chunks;
    p.groups = l.groups;
    p.ticket = reinterpret_cast<unsigned*>(ws);
    p.agg = reinterpret_cast<unsigned long long*>(reinterpret_cast<char*>(ws) + kAlign);
    p.inc = p.agg + l.agg_words;
    p.words = l.words;
    return p;
}

// ---- matrix states ----
const char* bad_config(const deer_matrec_config* c, bool step) {
    if (!c) return "config is NULL";
    if (!known_type(c->dtype)) return "unknown dtype";
    if (c->N < 1 || c->Hk < 1 || c->Hv < 1 || c->Dk < 1 || c->Dv < 1) return "N, Hk, Hv, Dk and Dv must be positive";
    if (c->Hv % c->Hk) return "Hv must be a multiple of Hk";
    if (c->reserved != 0) return "reserved must be 0";
    if (!std::isfinite((float)c->scale)) return "scale must be finite in 32 bits";
    if (c->stride_q < 0 || c->stride_k < 0 || c->stride_v < 0 || c->stride_o < 0) return "strides must not be negative";
    const int64_t keys = (int64_t)c->Hk * c->Dk, values = (int64_t)c->Hv * c->Dv;
    if ((c->stride_q && c->stride_q < keys) || (c->stride_k && c->stride_k < keys) || (c->stride_v && c->stride_v < values) || (c->stride_o && c->stride_o < values))
        return "a stride is smaller than a row";
    if (!step && (c->T < 0 || (c->packed & ~(int)DEER_REST_ZERO & ~1))) return "T must not be negative, packed 0 or 1 (and DEER_REST_ZERO)";
    return nullptr;
}

// How the rows are cut into segments, each a workgroup a head.  A sequence is cut only where whole sequences do not make enough workgroups
// for 256 CUs, and then into as many as do.  Measured, 128 x 128 in bf16, forward + backward:
//   whole from 256 N Hv on: 192 (3 x 64 heads of 4,096 rows) 413 + 1,115 us whole, 362 + 1,067 cut; 256 425 us whole, 422 cut (forward); 320 472 and 622
//   512 workgroups at a time: 4 x 4,096 rows and 16 heads with 256 of them 164 + 429 us, 384 144 + 418, 512 128 + 391, 768 153 + 407, 1,024 150 + 437
//   up to 4 chunks whole: 64 heads of 256 rows 34 + 57 us whole, 39 + 84 cut; 4 heads of them 28 + 42 and 22 + 33; with no other least length: 4 heads
//   of 2,048 rows 32 + 50 us, with segments of 4 chunks at least 44 + 63
// What the sequences' lengths are is not known here; nearly all rows may be one sequence's.  Forward, 16 heads, into arrays that are handed in:
//   packed, a segment has at most two 512ths of all rows: one sequence of 32,768 rows and 63 of one, 128 x 128, 367 us (cut by the number of sequences
//   alone 3,080); one of 16,384 and 127 of 128 376 us (1,633); 64 of 1,024 342 us (349); 48 of 2,048 533 us (534)
//   a padded batch with lengths, at most 32 chunks: 16 to 4,096 rows, 128 x 128, all of them 417 us (whole 443), one long 261 us (364); 16 to 32,768, 64 x 64, one
//   long 170 us (1,600)
struct MatLayout {
    long long chunks, max_segs, max_slots;   // at most
    int per;
    bool split;
    size_t off_segs, off_seq, off_state, off_rstate, off_decay, off_part_q, off_part_k, off_gate, off_read, off_put, off_size_in, off_size_out, off_rows, off_front, total;
};
MatLayout mat_layout(const deer_matrec_config* c, bool grad, bool bounds) {
    MatLayout l{};
    const long long longest = (c->T + kChunk - 1) / kChunk;
    l.chunks = is_packed(c) ? longest + c->N : longest * c->N;
    long long per = longest < 1 ? 1 : longest;
    if (longest > 4 && (is_packed(c) || (long long)c->N * c->Hv < 256)) {
        // 512 workgroups run at a time; every sequence's last segment is a short one, half of the others' length on average
        const long long all = 512 / c->Hv, least = all / 2 > 1 ? all / 2 : 1;
        long long segs = all - (is_packed(c) ? c->N / 2 : 0);
        if (segs < least) segs = least;
        per = ((is_packed(c) ? longest : l.chunks) + segs - 1) / segs;
        if (per > longest) per = longest;
    }
    if (bounds && !is_packed(c) && per > 32) per = 32;
    if (grad && per > 32) per = 32;   // what goes through the chunks of a segment (matrec_grad.hip) takes the rounding errors of all of them
    l.per = (int)per;
    l.split = per < longest;
    l.max_segs = is_packed(c) ? l.chunks / per + c->N : (longest + per - 1) / per * c->N;
    // A packed sequence that is cut has r > 64 per rows, and fewer than r / (64 per) + 1 segments: in all fewer than twice as many as all rows make
    l.max_slots = is_packed(c) && 2 * c->T / (kChunk * per) < l.max_segs ? 2 * c->T / (kChunk * per) : l.max_segs;
    const size_t states = (size_t)c->Hv * (c->Dk <= 64 ? 64 : 128) * (c->Dv <= 64 ? 64 : 128) * 4;
    size_t at = kAlign;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += align_up(bytes);
        return here;
    };
    l.off_segs = take((size_t)l.max_segs * sizeof(MatSegment));
    l.off_seq = take((size_t)c->N * 8);
    l.off_rows = take((size_t)l.chunks * c->Hv * kRowFloats * 4);
    if (l.split) {
        l.off_state = take((size_t)l.max_slots * states);
        if (grad) l.off_rstate = take((size_t)l.max_slots * states);
        l.off_decay = take((size_t)l.max_slots * c->Hv * 8);
    }
    if (grad) {
        const size_t rows = (size_t)c->T * (is_packed(c) ? 1 : c->N), by_head = (size_t)c->Hv * 4;
        if (c->Hv != c->Hk) {
            l.off_part_q = take(rows * by_head * c->Dk);
            l.off_part_k = take(rows * by_head * c->Dk);
        }
        l.off_gate = take(rows * by_head);
        l.off_read = take((size_t)l.chunks * by_head);
        l.off_put = take((size_t)l.chunks * by_head);
        l.off_size_in = take((size_t)l.chunks * by_head);
        l.off_size_out = take((size_t)l.chunks * by_head);
        l.off_front = take((size_t)l.max_segs * by_head);
    }
    l.total = at;
    return l;
}
const char* unsupported(const deer_matrec_config* c, bool step) {
    if (c->dtype != DEER_F32 && c->dtype != DEER_BF16) return "matrix states: fp32 and bf16 only";
    if (c->Dk > 128 || c->Dv > 128) return "matrix states: Dk and Dv up to 128";
    if (step) return (long double)c->N * c->Hv * 256 > kMostLanes ? "more rows than a launch holds" : nullptr;
    if (c->T > kMostRows || (long double)c->N * c->Hv * 64 > 2147483647.0L || ((long double)(c->T + 63) / 64 + 4) * (is_packed(c) ? 1 : c->N) * c->Hv > 2147483647.0L)
        return "more rows than a launch holds";
    // Launches of both directions, so that no forward runs whose gradient is refused: a workgroup of up to 512 lanes a segment and head (gradient: three); four
    // of 256 a chunk
    for (const bool grad : {false, true}) {
        const MatLayout l = mat_layout(c, grad, true);   // (no fewer segments than without bounds)
        if (((long double)l.max_segs * c->Hv + 8) * (grad ? 3 : 1) * 512 > kMostLanes || (long double)l.chunks * 4 * 256 > kMostLanes) return "more rows than a launch holds";
    }
    return nullptr;
}
// the row outputs of a direction, to be zeroed where no sequence is
RestRows mat_rest(const deer_matrec_config* c, const MatrecParams& p, bool grad) {
    RestRows rest{};
    if (!zero_rest(c)) return rest;
    const long long e = (long long)type_bytes(c->dtype), keys = (long long)c->Hk * c->Dk * e, values = (long long)c->Hv * c->Dv * e;
    auto add = [&](void* first, long long pitch, long long width) {
        if (first) rest.array[rest.count++] = RestArray{first, pitch, width};
    };
    if (grad) {
        add(p.dq, p.stride_q * e, keys);
        add(p.dk, p.stride_k * e, keys);
        add(p.dv, p.stride_v * e, values);
        add(p.dgate, 4ll * c->Hv, 4ll * c->Hv);
    } else {
        add(p.o, p.stride_o * e, values);
    }
    return rest;
}
MatrecParams mat_params(const deer_matrec_config* c, const MatLayout& l, bool grad, const int64_t* bounds, void* workspace) {
    char* ws = reinterpret_cast<char*>(workspace);
    MatrecParams p{};
    p.rows = SeqRows{reinterpret_cast<const long long*>(bounds), c->T, c->N, is_packed(c)};
    p.plan.count = reinterpret_cast<int*>(ws);
    p.plan.segs = reinterpret_cast<MatSegment*>(ws + l.off_segs);
    p.plan.seq_seg = reinterpret_cast<int*>(ws + l.off_seq);
    p.plan.seq_count = p.plan.seq_seg + c->N;
    p.plan.max_segs = (int)l.max_segs;
    p.plan.max_slots = (int)l.max_slots;
    p.plan.max_chunks = (int)l.chunks;
    p.plan.per = l.per;
    p.Hk = c->Hk;
    p.Hv = c->Hv;
    p.Dk = c->Dk;
    p.Dv = c->Dv;
    p.scale = (float)c->scale;
    p.stride_q = c->stride_q ? c->stride_q : (long long)c->Hk * c->Dk;
    p.stride_k = c->stride_k ? c->stride_k : (long long)c->Hk * c->Dk;
    p.stride_v = c->stride_v ? c->stride_v : (long long)c->Hv * c->Dv;
    p.stride_o = c->stride_o ? c->stride_o : (long long)c->Hv * c->Dv;
    p.split = l.split;
    p.rows_of = reinterpret_cast<float*>(ws + l.off_rows);
    if (l.split) {
        p.seg_state = reinterpret_cast<float*>(ws + l.off_state);
        if (grad) p.seg_rstate = reinterpret_cast<float*>(ws + l.off_rstate);
        p.seg_decay = reinterpret_cast<float*>(ws + l.off_decay);
    }
    if (grad) {
        if (c->Hv != c->Hk) {
            p.part_q = reinterpret_cast<float*>(ws + l.off_part_q);
            p.part_k = reinterpret_cast<float*>(ws + l.off_part_k);
        }
        p.gate_k = reinterpret_cast<float*>(ws + l.off_gate);
        p.read_in = reinterpret_cast<float*>(ws + l.off_read);
        p.put_out = reinterpret_cast<float*>(ws + l.off_put);
        p.size_in = reinterpret_cast<float*>(ws + l.off_size_in);
        p.size_out = reinterpret_cast<float*>(ws + l.off_size_out);
        p.front = reinterpret_cast<float*>(ws + l.off_front);
    }
    return p;
}

}  // namespace

extern "C" {

deer_status deer_diagrec_workspace_bytes(const deer_diagrec_config* c, int32_t grad, size_t* bytes) {
    if (!bytes) return fail(DEER_ERR_INVALID_ARG, "bytes is NULL");
    if (const char* why = bad_config(c, false)) return fail(DEER_ERR_INVALID_ARG, why);
    if (too_large(c, grad != 0)) return fail(DEER_ERR_UNSUPPORTED, "more rows or tiles than a launch holds, or rows more than 2^22 elements apart");
    *bytes = diag_layout(c, grad != 0).total;
    return DEER_OK;
}

deer_status deer_diagrec_solve(const deer_diagrec_config* c, const void* d_gate, const void* d_in, const void* d_h0, const int64_t* d_bounds,
                               void* d_h, void* d_last, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    if (const char* why = bad_config(c, false)) return fail(DEER_ERR_INVALID_ARG, why);
    if (too_large(c, false)) return fail(DEER_ERR_UNSUPPORTED, "more rows or tiles than a launch holds, or rows more than 2^22 elements apart");
    if ((c->T > 0 && (!d_gate || !d_in || !d_h)) || (is_packed(c) && !d_bounds)) return fail(DEER_ERR_INVALID_ARG, "a required pointer is NULL");
    const size_t e = type_bytes(c->dtype), w = c->dtype == DEER_F64 ? 8 : 4;
    if (misaligned(d_gate, e) || misaligned(d_in, e) || misaligned(d_h, e) || misaligned(d_h0, w) || misaligned(d_last, w) || misaligned(d_bounds, 8))
        return fail(DEER_ERR_INVALID_ARG, "a pointer is not aligned to its element");
    const DiagLayout l = diag_layout(c, false);
    if (deer_status st = check_workspace(d_workspace, workspace_bytes, l.total)) return st;
    DiagrecParams p = diag_params(c, l, d_bounds, d_workspace);
    p.g = d_gate;
    p.x = d_in;
    p.h0 = d_h0;
    p.h = d_h;
    p.last = d_last;
    return launched("deer_diagrec_solve", launch_diagrec(c->dtype, false, p, reinterpret_cast<hipStream_t>(hip_stream)));
}

deer_status deer_diagrec_grad(const deer_diagrec_config* c, const void* d_gate, const void* d_in, const void* d_h0, const int64_t* d_bounds,
                              const void* d_h, const void* d_dh, const void* d_dlast, void* d_dgate, void* d_din, void* d_dh0,
                              void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    if (const char* why = bad_config(c, false)) return fail(DEER_ERR_INVALID_ARG, why);
    if (too_large(c, true)) return fail(DEER_ERR_UNSUPPORTED, "more rows or tiles than a launch holds, or rows more than 2^22 elements apart");
    if ((c->T > 0 && (!d_gate || !d_in || !d_h || !d_dh || !d_dgate || !d_din)) || (is_packed(c) && !d_bounds))
        return fail(DEER_ERR_INVALID_ARG, "a required pointer is NULL");
    const size_t e = type_bytes(c->dtype), w = c->dtype == DEER_F64 ? 8 : 4;
    if (misaligned(d_gate, e) || misaligned(d_in, e) || misaligned(d_h, e) || misaligned(d_dh, e) || misaligned(d_dgate, e) || misaligned(d_din, e) ||
        misaligned(d_h0, w) || misaligned(d_dlast, w) || misaligned(d_dh0, w) || misaligned(d_bounds, 8))
        return fail(DEER_ERR_INVALID_ARG, "a pointer is not aligned to its element");
    const DiagLayout l = diag_layout(c, true);
    if (deer_status st = check_workspace(d_workspace, workspace_bytes, l.total)) return st;
    DiagrecParams p = diag_params(c, l, d_bounds, d_workspace);
    p.g = d_gate;
    p.x = d_in;
    p.h0 = d_h0;
    p.h = const_cast<void*>(d_h);   // (read only in this direction)
    p.dh = d_dh;
    p.dlast = d_dlast;
    p.dg = d_dgate;
    p.dx = d_din;
    p.dh0 = d_dh0;
    return launched("deer_diagrec_grad", launch_diagrec(c->dtype, true, p, reinterpret_cast<hipStream_t>(hip_stream)));
}

deer_status deer_diagrec_step(const deer_diagrec_config* c, const void* d_gate, const void* d_in, const int32_t* d_slots, int32_t n_slots,
                              void* d_state, void* d_h, void* hip_stream) {
    if (const char* why = bad_config(c, true)) return fail(DEER_ERR_INVALID_ARG, why);
    if (n_slots < 1) return fail(DEER_ERR_INVALID_ARG, "n_slots must be positive");
    if (!d_gate || !d_in || !d_state || !d_h) return fail(DEER_ERR_INVALID_ARG, "a required pointer is NULL");
    const size_t e = type_bytes(c->dtype), w = c->dtype == DEER_F64 ? 8 : 4;
    if (misaligned(d_gate, e) || misaligned(d_in, e) || misaligned(d_h, e) || misaligned(d_state, w) || misaligned(d_slots, 4))
        return fail(DEER_ERR_INVALID_ARG, "a pointer is not aligned to its element");
    if (c->D > (1 << 30) || (long double)c->N * ((c->D + 255) / 256) * 256 > kMostLanes) return fail(DEER_ERR_UNSUPPORTED, "more rows or channels than a launch holds");
    DiagstepParams p{};
    p.rows = StepRows{d_slots, c->N, n_slots, zero_rest(c)};
    p.D = c->D;
    p.gate = c->gate;
    p.stride_gate = c->stride_gate ? c->stride_gate : c->D;
    p.stride_in = c->stride_in ? c->stride_in : c->D;
    p.stride_out = c->stride_out ? c->stride_out : c->D;
    p.g = d_gate;
    p.x = d_in;
    p.state = d_state;
    p.h = d_h;
    return launched("deer_diagrec_step", launch_diagstep(c->dtype, p, reinterpret_cast<hipStream_t>(hip_stream)));
}

deer_status deer_dropout(int32_t dtype, int32_t N, int64_t T, int32_t D, const void* d_x, int64_t stride_in, void* d_y, int64_t stride_out,
                         double p, uint64_t seed, uint32_t draw, void* hip_stream) {
    if (!known_type(dtype)) return fail(DEER_ERR_INVALID_ARG, "unknown dtype");
    if (N < 1 || D < 1 || T < 0) return fail(DEER_ERR_INVALID_ARG, "N and D must be positive, T not negative");
    if (stride_in < 0 || stride_out < 0 || (stride_in && stride_in < D) || (stride_out && stride_out < D))
        return fail(DEER_ERR_INVALID_ARG, "a stride is negative or smaller than a row");
    if (const char* why = bad_drop(p)) return fail(DEER_ERR_INVALID_ARG, why);
    if (T > 0 && (!d_x || !d_y)) return fail(DEER_ERR_INVALID_ARG, "a required pointer is NULL");
    if (misaligned(d_x, type_bytes(dtype)) || misaligned(d_y, type_bytes(dtype))) return fail(DEER_ERR_INVALID_ARG, "a pointer is not aligned to its element");
    if (T > kMostRows || (long double)N * ((T + 7) / 8) * D > kMostLanes - 256) return fail(DEER_ERR_UNSUPPORTED, "more elements than a launch holds");
    DropoutParams q{};
    q.N = N;
    q.D = D;
    q.T = T;
    q.stride_in = stride_in ? stride_in : D;
    q.stride_out = stride_out ? stride_out : D;
    q.x = d_x;
    q.y = d_y;
    q.drop = drop_params(p, seed, draw);
    return launched("deer_dropout", launch_dropout(dtype, q, reinterpret_cast<hipStream_t>(hip_stream)));
}

deer_status deer_matrec_workspace_bytes(const deer_matrec_config* c, int32_t grad, size_t* bytes) {
    if (!bytes) return fail(DEER_ERR_INVALID_ARG, "bytes is NULL");
    if (const char* why = bad_config(c, false)) return fail(DEER_ERR_INVALID_ARG, why);
    if (const char* why = unsupported(c, false)) return fail(DEER_ERR_UNSUPPORTED, why);
    const size_t with = mat_layout(c, grad != 0, true).total, without = mat_layout(c, grad != 0, false).total;
    *bytes = with > without ? with : without;
    return DEER_OK;
}

deer_status deer_matrec_solve(const deer_matrec_config* c, const void* d_q, const void* d_k, const void* d_v, const float* d_gate, const float* d_s0,
                              const int64_t* d_bounds, void* d_o, float* d_last, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    if (const char* why = bad_config(c, false)) return fail(DEER_ERR_INVALID_ARG, why);
    if (const char* why = unsupported(c, false)) return fail(DEER_ERR_UNSUPPORTED, why);
    if ((c->T > 0 && (!d_q || !d_k || !d_v || !d_gate || !d_o)) || (is_packed(c) && !d_bounds)) return fail(DEER_ERR_INVALID_ARG, "a required pointer is NULL");
    const size_t e = type_bytes(c->dtype);
    if (misaligned(d_q, e) || misaligned(d_k, e) || misaligned(d_v, e) || misaligned(d_o, e) || misaligned(d_gate, 4) || misaligned(d_s0, 4) ||
        misaligned(d_last, 4) || misaligned(d_bounds, 8))
        return fail(DEER_ERR_INVALID_ARG, "a pointer is not aligned to its element");
    const MatLayout l = mat_layout(c, false, d_bounds != nullptr);
    if (deer_status st = check_workspace(d_workspace, workspace_bytes, l.total)) return st;
    MatrecParams p = mat_params(c, l, false, d_bounds, d_workspace);
    p.q = d_q;
    p.k = d_k;
    p.v = d_v;
    p.gate = d_gate;
    p.s0 = d_s0;
    p.o = d_o;
    p.last = d_last;
    hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
    hipError_t err = launch_matrec_plan(p, mat_rest(c, p, false), stream);
    if (err == hipSuccess) err = launch_matrec_out(c->dtype, p, stream);
    return launched("deer_matrec_solve", err);
}

deer_status deer_matrec_grad(const deer_matrec_config* c, const void* d_q, const void* d_k, const void* d_v, const float* d_gate, const float* d_s0,
                             const int64_t* d_bounds, const void* d_do, const float* d_dlast, void* d_dq, void* d_dk, void* d_dv, float* d_dgate,
                             float* d_ds0, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    if (const char* why = bad_config(c, false)) return fail(DEER_ERR_INVALID_ARG, why);
    if (const char* why = unsupported(c, false)) return fail(DEER_ERR_UNSUPPORTED, why);
    if ((c->T > 0 && (!d_q || !d_k || !d_v || !d_gate || !d_do || !d_dq || !d_dk || !d_dv)) || (is_packed(c) && !d_bounds))
        return fail(DEER_ERR_INVALID_ARG, "a required pointer is NULL");
    const size_t e = type_bytes(c->dtype);
    if (misaligned(d_q, e) || misaligned(d_k, e) || misaligned(d_v, e) || misaligned(d_do, e) || misaligned(d_dq, e) || misaligned(d_dk, e) ||
        misaligned(d_dv, e) || misaligned(d_gate, 4) || misaligned(d_s0, 4) || misaligned(d_dlast, 4) || misaligned(d_dgate, 4) || misaligned(d_ds0, 4) ||
        misaligned(d_bounds, 8))
        return fail(DEER_ERR_INVALID_ARG, "a pointer is not aligned to its element");
    const MatLayout l = mat_layout(c, true, d_bounds != nullptr);
    if (deer_status st = check_workspace(d_workspace, workspace_bytes, l.total)) return st;
    MatrecParams p = mat_params(c, l, true, d_bounds, d_workspace);
    p.q = d_q;
    p.k = d_k;
    p.v = d_v;
    p.gate = d_gate;
    p.s0 = d_s0;
    p.dout = d_do;
    p.dlast = d_dlast;
    p.dq = d_dq;
    p.dk = d_dk;
    p.dv = d_dv;
    p.dgate = d_dgate;
    p.ds0 = d_ds0;
    hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
    hipError_t err = launch_matrec_plan(p, mat_rest(c, p, true), stream);
    if (err == hipSuccess) err = launch_matrec_join(c->dtype, p, true, stream);
    if (err == hipSuccess) err = launch_matrec_grad(c->dtype, p, stream);
    return launched("deer_matrec_grad", err);
}

deer_status deer_matrec_step(const deer_matrec_config* c, const void* d_q, const void* d_k, const void* d_v, const float* d_gate, const int32_t* d_slots,
                             int32_t n_slots, float* d_state, void* d_o, void* hip_stream) {
    if (const char* why = bad_config(c, true)) return fail(DEER_ERR_INVALID_ARG, why);
    if (const char* why = unsupported(c, true)) return fail(DEER_ERR_UNSUPPORTED, why);
    if (n_slots < 1) return fail(DEER_ERR_INVALID_ARG, "n_slots must be positive");
    if (!d_q || !d_k || !d_v || !d_gate || !d_state || !d_o) return fail(DEER_ERR_INVALID_ARG, "a required pointer is NULL");
    const size_t e = type_bytes(c->dtype);
    if (misaligned(d_q, e) || misaligned(d_k, e) || misaligned(d_v, e) || misaligned(d_o, e) || misaligned(d_gate, 4) || misaligned(d_state, 4) || misaligned(d_slots, 4))
        return fail(DEER_ERR_INVALID_ARG, "a pointer is not aligned to its element");
    MatstepParams p{};
    p.rows = StepRows{d_slots, c->N, n_slots, zero_rest(c)};
    p.Hk = c->Hk;
    p.Hv = c->Hv;
    p.Dk = c->Dk;
    p.Dv = c->Dv;
    p.scale = (float)c->scale;
    p.stride_q = c->stride_q ? c->stride_q : (long long)c->Hk * c->Dk;
    p.stride_k = c->stride_k ? c->stride_k : (long long)c->Hk * c->Dk;
    p.stride_v = c->stride_v ? c->stride_v : (long long)c->Hv * c->Dv;
    p.stride_o = c->stride_o ? c->stride_o : (long long)c->Hv * c->Dv;
    p.q = d_q;
    p.k = d_k;
    p.v = d_v;
    p.gate = d_gate;
    p.state = d_state;
    p.o = d_o;
    return launched("deer_matrec_step", launch_matstep(c->dtype, p, reinterpret_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
