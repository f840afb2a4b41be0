// C entry points of the short convolution, the selective scan and the group norm (include/deer.h): checks of the arguments, the workspaces' layout,
// launches.  Nothing here allocates or synchronises.
#include <hip/hip_runtime.h>

#include "layer_common.h"
#include "selscan_common.h"
#include "seq_check.h"

using namespace deer;

namespace {

struct Room {   // of a workspace, part by part
    size_t at = 0;
    size_t take(size_t bytes) {
        const size_t here = at;
        at += align_up(bytes);
        return here;
    }
};

template <typename C>
const char* bad_rows(const C* c, bool step) {
    if (!c) return "config is NULL";
    if (!known_type(c->dtype)) return "unknown dtype";
    if (c->N < 1 || c->D < 1) return "N and D must be positive";
    if (!step && (c->T < 0 || (c->packed & ~(int)DEER_REST_ZERO & ~1))) return "T must not be negative, packed 0 or 1 (and DEER_REST_ZERO)";
    return nullptr;
}
bool bad_stride(int64_t stride, int64_t row) { return stride < 0 || (stride && stride < row); }
template <typename C>
SeqRows rows_of(const C* c, const int64_t* bounds) { return SeqRows{reinterpret_cast<const long long*>(bounds), c->T, c->N, is_packed(c)}; }
template <typename C>
long double row_count(const C* c) { return (long double)c->T * (is_packed(c) ? 1 : c->N); }
size_t wide_bytes(int dtype) { return dtype == DEER_F64 ? 8 : 4; }
constexpr const char* kStride = "a stride is negative or smaller than a row";
constexpr const char* kLarge = "more rows or channels than a launch holds";
constexpr const char* kMissing = "a required pointer is NULL";
constexpr const char* kAligned = "a pointer is not aligned to its element";
template <typename... P>
bool any_misaligned(size_t bytes, P... p) { return (misaligned(p, bytes) || ...); }

// ---- short convolution ----
const char* bad_config(const deer_shortconv_config* c, bool step) {
    if (const char* why = bad_rows(c, step)) return why;
    if (c->act != DEER_ACT_NONE && c->act != DEER_ACT_SILU) return "unknown activation: DEER_ACT_NONE or DEER_ACT_SILU";
    if (c->W < 1 || c->W > 8) return "W must lie in 1 .. 8";
    if (bad_stride(c->stride_x, c->D) || bad_stride(c->stride_y, c->D)) return kStride;
    return nullptr;
}
const char* too_large(const deer_shortconv_config* c) {
    // (the last: the sums over tiles, 64 lanes a column)
    if (c->T > kMostRows || c->D > (1 << 27) || row_count(c) * c->D > 1e17L || (long double)c->D * (c->W + 1) * 64 > kMostLanes - 1024) return kLarge;
    const Lanes l = lanes_for(c->D, 1);   // (a channel a lane: most workgroups)
    return ((long double)conv_tiles(c->D, c->T, c->N, is_packed(c)) * l.blocks + 512) * 256 > kMostLanes ? kLarge : nullptr;
}
ConvParams conv_params(const deer_shortconv_config* c, const int64_t* bounds) {
    ConvParams p{};
    p.rows = rows_of(c, bounds);
    p.D = c->D;
    p.W = c->W;
    p.act = c->act;
    p.stride_x = c->stride_x ? c->stride_x : c->D;
    p.stride_y = c->stride_y ? c->stride_y : c->D;
    p.zero_rest = zero_rest(c);
    return p;
}
size_t conv_workspace(const deer_shortconv_config* c) {
    return kAlign + align_up((size_t)conv_tiles(c->D, c->T, c->N, is_packed(c)) * (c->W + 1) * c->D * wide_bytes(c->dtype));
}

// ---- selective scan ----
const char* bad_config(const deer_selscan_config* c, bool step) {
    if (const char* why = bad_rows(c, step)) return why;
    if (c->dt_act != DEER_ACT_NONE && c->dt_act != DEER_ACT_SOFTPLUS) return "unknown activation of dt: DEER_ACT_NONE or DEER_ACT_SOFTPLUS";
    if (c->S < 1 || c->G < 1 || c->D % c->G) return "S and G must be positive, G a divisor of D";
    if (c->reserved != 0) return "reserved must be 0";
    const int64_t states = (int64_t)c->G * c->S;
    if (bad_stride(c->stride_x, c->D) || bad_stride(c->stride_dt, c->D) || bad_stride(c->stride_B, states) || bad_stride(c->stride_C, states) ||
        bad_stride(c->stride_z, c->D) || bad_stride(c->stride_y, c->D))
        return kStride;
    return nullptr;
}
struct ScanLayout {
    int lanes, blocks, segs, marks_each, parts_each;   // lanes of a channel, workgroups along a group's channels
    long long seg_rows, all_segs;
    size_t local, carry, steps, resets, rlocal, rcarry, rsteps, rresets, marks, mark_steps, part_bc, part_A, part_d, total;
};
// How the rows are cut into segments, each a workgroup for 256 / Q channels.  A cut costs a second look at the rows (the gradient's first look takes more), so sequences are whole where they make
// 512 workgroups.  Measured on 4 x 4,096 rows of 4,096 channels with 16 states in bf16 (whole: 256 workgroups), as so many workgroups in all:
//   outputs 256 669 us, 512 411, 1,024 321, 2,048 310; states behind segments 512 285, 1,024 235, 2,048 215
//   gradient with its kept states 256 496 + 1,680 us; with fronts too 512 452 + 1,144, 1,024 362 + 1,172, 2,048 350 + 1,152; solve and gradient 2,863, 2,215, 1,963, 1,877
// 8 x 2,048 rows of them, solve and gradient: whole (512 workgroups) 1,774 us, cut (2,048) 1,893.
// Packed rows, and padded ones with lengths, may be nearly all one sequence's: always cut.  8,192 rows in all: 256 332 + 225 us, 512 195 + 136, 1,024 158 + 115, 2,048 149 + 108; gradient 372 + 857, 218 + 539, 165 +
// 524, 160 + 514.
ScanLayout scan_layout(const deer_selscan_config* c, bool grad, bool bounds) {
    ScanLayout l{};
    l.lanes = scan_lanes(c->S);
    const int width = 256 / l.lanes, per_group = c->D / c->G;
    l.blocks = (per_group + width - 1) / width;
    const long long seqs = is_packed(c) ? 1 : c->N, across = (long long)c->G * l.blocks * seqs;
    long long want = !is_packed(c) && !bounds && across >= 512 ? 1 : (2048 + across - 1) / across;   // of 64 rows at least
    const long long most = (c->T + 63) / 64;
    want = want > most ? most : want;
    want = want < 1 ? 1 : want;
    l.seg_rows = ((c->T + want - 1) / want + 63) / 64 * 64;
    if (l.seg_rows < 64) l.seg_rows = 64;
    l.segs = (int)((c->T + l.seg_rows - 1) / l.seg_rows);
    if (l.segs < 1) l.segs = 1;
    l.all_segs = seqs * l.segs;
    l.marks_each = (int)(l.seg_rows / kMarkRows);
    l.parts_each = (int)((l.seg_rows + kSumRows - 1) / kSumRows);
    const size_t cells = (size_t)c->D * 4 * l.lanes * 4, channels = (size_t)c->D * 4;
    Room r;
    if (l.segs > 1) {
        l.local = r.take(l.all_segs * cells);
        l.carry = r.take(l.all_segs * cells);
        l.steps = r.take(l.all_segs * channels);
        l.resets = r.take(l.all_segs * 4);
        if (grad) {
            l.rlocal = r.take(l.all_segs * cells);
            l.rcarry = r.take(l.all_segs * cells);
            l.rsteps = r.take(l.all_segs * channels);
            l.rresets = r.take(l.all_segs * 4);
        }
    }
    if (grad) {
        l.marks = r.take((size_t)l.all_segs * l.marks_each * cells);
        l.mark_steps = r.take((size_t)l.all_segs * l.marks_each * channels);
        l.part_bc = r.take((size_t)l.blocks * c->T * seqs * c->G * 8 * l.lanes * 4);
        l.part_A = r.take((size_t)l.all_segs * l.parts_each * c->D * c->S * 4);
        l.part_d = r.take((size_t)l.all_segs * l.parts_each * 2 * channels);
    }
    l.total = r.at + kAlign;
    return l;
}
const char* unsupported(const deer_selscan_config* c, bool step) {
    if (c->dtype == DEER_F64) return "selective scan: fp32, bf16 and fp16 only";
    if (c->S > 64) return "selective scan: up to 64 states";
    if (c->D > (1 << 24)) return kLarge;
    if (step) return (long double)c->N * ((long long)c->D * scan_lanes(c->S) + 256) > kMostLanes ? kLarge : nullptr;
    for (const int64_t stride : {c->stride_x, c->stride_dt, c->stride_B, c->stride_C, c->stride_z, c->stride_y, (int64_t)c->D, (int64_t)c->G * c->S})
        if (stride > kScanStride) return "selective scan: rows at most 2^22 elements apart";
    const long double seqs = is_packed(c) ? 1 : c->N;
    if (c->T > kMostRows || row_count(c) * c->D > 1e15L || seqs * c->D * 64 > kMostLanes || (long double)c->D * c->S * 64 > kMostLanes - 1024) return kLarge;
    const ScanLayout l = scan_layout(c, true, true);   // (no fewer segments than without bounds)
    return (long double)l.all_segs * c->G * l.blocks * 256 > kMostLanes || l.all_segs > 0x7FFFFFFF / 4 ? kLarge : nullptr;
}
SelscanParams scan_params(const deer_selscan_config* c, const ScanLayout& l, const int64_t* bounds, void* workspace, bool grad) {
    char* ws = reinterpret_cast<char*>(workspace);
    auto floats = [&](size_t at) { return reinterpret_cast<float*>(ws + at); };
    SelscanParams p{};
    p.rows = rows_of(c, bounds);
    p.D = c->D;
    p.S = c->S;
    p.G = c->G;
    p.softplus = c->dt_act == DEER_ACT_SOFTPLUS;
    p.per_group = c->D / c->G;
    p.blocks = l.blocks;
    const int64_t states = (int64_t)c->G * c->S;
    p.stride_x = c->stride_x ? c->stride_x : c->D;
    p.stride_dt = c->stride_dt ? c->stride_dt : c->D;
    p.stride_B = c->stride_B ? c->stride_B : states;
    p.stride_C = c->stride_C ? c->stride_C : states;
    p.stride_z = c->stride_z ? c->stride_z : c->D;
    p.stride_y = c->stride_y ? c->stride_y : c->D;
    p.segs = l.segs;
    p.seg_rows = l.seg_rows;
    p.marks_each = l.marks_each;
    p.parts_each = l.parts_each;
    p.zero_rest = zero_rest(c);
    if (l.segs > 1) {
        p.local = floats(l.local);
        p.carry = floats(l.carry);
        p.steps = floats(l.steps);
        p.resets = reinterpret_cast<int*>(ws + l.resets);
        if (grad) {
            p.rlocal = floats(l.rlocal);
            p.rcarry = floats(l.rcarry);
            p.rsteps = floats(l.rsteps);
            p.rresets = reinterpret_cast<int*>(ws + l.rresets);
        }
    }
    if (grad) {
        p.marks = floats(l.marks);
        p.mark_steps = floats(l.mark_steps);
        p.part_bc = floats(l.part_bc);
        p.part_A = floats(l.part_A);
        p.part_d = floats(l.part_d);
    }
    return p;
}
bool scan_vec(const SelscanParams& p, size_t e, bool grad) {
    bool vec = p.per_group % 4 == 0 && p.S % 4 == 0 && rows_fit(p.x, p.stride_x, 4, e) && rows_fit(p.dt, p.stride_dt, 4, e) && rows_fit(p.B, p.stride_B, 4, e) &&
               rows_fit(p.C, p.stride_C, 4, e) && (!p.z || rows_fit(p.z, p.stride_z, 4, e));
    if (grad) return vec && rows_fit(p.dy, p.stride_y, 4, e) && rows_fit(p.dx, p.stride_x, 4, e) && rows_fit(p.ddt, p.stride_dt, 4, e) && (!p.z || rows_fit(p.dz, p.stride_z, 4, e));
    return vec && rows_fit(p.y, p.stride_y, 4, e);
}

// ---- group norm ----
const char* bad_config(const deer_groupnorm_config* c) {
    if (const char* why = bad_rows(c, false)) return why;
    if (c->act != DEER_ACT_NONE && c->act != DEER_ACT_SILU) return "unknown activation: DEER_ACT_NONE or DEER_ACT_SILU";
    if (c->span != DEER_SPAN_ROW && c->span != DEER_SPAN_SEQUENCE) return "unknown span";
    if (c->G < 1 || c->D % c->G) return "G must be a divisor of D";
    if (c->reserved != 0) return "reserved must be 0";
    if (!(c->eps >= 0.0) || !std::isfinite((float)c->eps)) return "eps must not be negative, and finite in 32 bits";
    if (bad_stride(c->stride_x, c->D) || bad_stride(c->stride_z, c->D) || bad_stride(c->stride_y, c->D)) return kStride;
    return nullptr;
}
struct NormRoom {
    size_t part, sums, joined, total;
};
NormRoom norm_room(const deer_groupnorm_config* c, const NormLayout& l) {
    const size_t w = wide_bytes(c->dtype);
    Room r;
    NormRoom n{};
    n.part = r.take((size_t)l.part * w);
    n.sums = r.take((size_t)l.sums * w);
    n.joined = r.take((size_t)l.joined * w);
    n.total = r.at ? r.at + kAlign : 0;   // (norms of rows need none)
    return n;
}
NormLayout norm_layout_of(const deer_groupnorm_config* c, bool grad) { return norm_layout(c->dtype, c->D, c->G, c->span, c->T, c->N, is_packed(c), grad); }
const char* too_large(const deer_groupnorm_config* c) {
    if (c->T > kMostRows || c->D > (1 << 27) || row_count(c) * c->D > 1e17L || (c->span == DEER_SPAN_SEQUENCE && (long double)c->N * c->G * 1024 > kMostLanes) || (long double)c->D * 2 * 64 > kMostLanes - 1024) return kLarge;
    for (const bool grad : {false, true})
        if ((long double)norm_layout_of(c, grad).tiles * 256 > kMostLanes) return kLarge;
    return nullptr;
}
NormParams norm_params(const deer_groupnorm_config* c, const NormRoom& room, const int64_t* bounds, void* workspace) {
    char* ws = reinterpret_cast<char*>(workspace);
    NormParams p{};
    p.rows = rows_of(c, bounds);
    p.D = c->D;
    p.G = c->G;
    p.act = c->act;
    p.span = c->span;
    p.eps = c->eps;
    p.stride_x = c->stride_x ? c->stride_x : c->D;
    p.stride_z = c->stride_z ? c->stride_z : c->D;
    p.stride_y = c->stride_y ? c->stride_y : c->D;
    p.part = ws + room.part;
    p.sums = ws + room.sums;
    p.joined = ws + room.joined;
    p.zero_rest = zero_rest(c);
    return p;
}

}  // namespace

extern "C" {

deer_status deer_shortconv_workspace_bytes(const deer_shortconv_config* c, size_t* bytes) {
    if (!bytes) return fail(DEER_ERR_INVALID_ARG, "bytes is NULL");
    if (const char* why = bad_config(c, false)) return fail(DEER_ERR_INVALID_ARG, why);
    if (const char* why = too_large(c)) return fail(DEER_ERR_UNSUPPORTED, why);
    *bytes = conv_workspace(c);
    return DEER_OK;
}

deer_status deer_shortconv_solve(const deer_shortconv_config* c, const void* d_x, const void* d_w, const void* d_bias, const void* d_s0, const int64_t* d_bounds,
                                 void* d_y, void* d_last, void* hip_stream) {
    if (const char* why = bad_config(c, false)) return fail(DEER_ERR_INVALID_ARG, why);
    if (const char* why = too_large(c)) return fail(DEER_ERR_UNSUPPORTED, why);
    if (!d_w || (c->T > 0 && (!d_x || !d_y)) || (is_packed(c) && !d_bounds)) return fail(DEER_ERR_INVALID_ARG, kMissing);
    if (any_misaligned(type_bytes(c->dtype), d_x, d_y) || any_misaligned(wide_bytes(c->dtype), d_w, d_bias, d_s0, d_last) || misaligned(d_bounds, 8))
        return fail(DEER_ERR_INVALID_ARG, kAligned);
    ConvParams p = conv_params(c, d_bounds);
    p.x = d_x;
    p.w = d_w;
    p.bias = d_bias;
    p.s0 = d_s0;
    p.y = d_y;
    p.last = d_last;
    return launched("deer_shortconv_solve", launch_shortconv(c->dtype, false, p, reinterpret_cast<hipStream_t>(hip_stream)));
}

deer_status deer_shortconv_grad(const deer_shortconv_config* c, const void* d_x, const void* d_w, const void* d_bias, const void* d_s0, const int64_t* d_bounds,
                                const void* d_dy, const void* d_dlast, void* d_dx, void* d_dw, void* d_dbias, void* d_ds0, void* d_workspace,
                                size_t workspace_bytes, void* hip_stream) {
    if (const char* why = bad_config(c, false)) return fail(DEER_ERR_INVALID_ARG, why);
    if (const char* why = too_large(c)) return fail(DEER_ERR_UNSUPPORTED, why);
    if (!d_w || !d_dw || (c->T > 0 && (!d_x || !d_dy || !d_dx)) || (is_packed(c) && !d_bounds)) return fail(DEER_ERR_INVALID_ARG, kMissing);
    if (any_misaligned(type_bytes(c->dtype), d_x, d_dy, d_dx) || any_misaligned(wide_bytes(c->dtype), d_w, d_bias, d_s0, d_dlast, d_dw, d_dbias, d_ds0) ||
        misaligned(d_bounds, 8))
        return fail(DEER_ERR_INVALID_ARG, kAligned);
    if (deer_status st = check_workspace(d_workspace, workspace_bytes, conv_workspace(c))) return st;
    ConvParams p = conv_params(c, d_bounds);
    p.x = d_x;
    p.w = d_w;
    p.bias = d_bias;
    p.s0 = d_s0;
    p.dy = d_dy;
    p.dlast = d_dlast;
    p.dx = d_dx;
    p.dw = d_dw;
    p.dbias = d_dbias;
    p.ds0 = d_ds0;
    p.part = d_workspace;
    return launched("deer_shortconv_grad", launch_shortconv(c->dtype, true, p, reinterpret_cast<hipStream_t>(hip_stream)));
}

deer_status deer_shortconv_step(const deer_shortconv_config* c, const void* d_x, const void* d_w, const void* d_bias, const int32_t* d_slots, int32_t n_slots,
                                void* d_state, void* d_y, void* hip_stream) {
    if (const char* why = bad_config(c, true)) return fail(DEER_ERR_INVALID_ARG, why);
    if (n_slots < 1) return fail(DEER_ERR_INVALID_ARG, "n_slots must be positive");
    if (!d_x || !d_w || !d_y || (c->W > 1 && !d_state)) return fail(DEER_ERR_INVALID_ARG, kMissing);
    if (any_misaligned(type_bytes(c->dtype), d_x, d_y) || any_misaligned(wide_bytes(c->dtype), d_w, d_bias, d_state) || misaligned(d_slots, 4))
        return fail(DEER_ERR_INVALID_ARG, kAligned);
    if (c->D > (1 << 27) || (long double)c->N * ((c->D + 255) / 256) * 256 > kMostLanes) return fail(DEER_ERR_UNSUPPORTED, kLarge);
    ConvStepParams p{};
    p.rows = StepRows{d_slots, c->N, n_slots, zero_rest(c)};
    p.D = c->D;
    p.W = c->W;
    p.act = c->act;
    p.stride_x = c->stride_x ? c->stride_x : c->D;
    p.stride_y = c->stride_y ? c->stride_y : c->D;
    p.x = d_x;
    p.w = d_w;
    p.bias = d_bias;
    p.state = d_state;
    p.y = d_y;
    return launched("deer_shortconv_step", launch_shortconv_step(c->dtype, p, reinterpret_cast<hipStream_t>(hip_stream)));
}

deer_status deer_selscan_workspace_bytes(const deer_selscan_config* c, int32_t grad, size_t* bytes) {
    if (!bytes) return fail(DEER_ERR_INVALID_ARG, "bytes is NULL");
    if (const char* why = bad_config(c, false)) return fail(DEER_ERR_INVALID_ARG, why);
    if (const char* why = unsupported(c, false)) return fail(DEER_ERR_UNSUPPORTED, why);
    const size_t with = scan_layout(c, grad != 0, true).total, without = scan_layout(c, grad != 0, false).total;
    *bytes = with > without ? with : without;
    return DEER_OK;
}

deer_status deer_selscan_solve(const deer_selscan_config* c, const void* d_x, const void* d_dt, const float* d_A, const void* d_B, const void* d_C,
                               const float* d_skip, const void* d_z, const float* d_dt_bias, const float* d_h0, const int64_t* d_bounds, void* d_y,
                               float* d_last, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    if (const char* why = bad_config(c, false)) return fail(DEER_ERR_INVALID_ARG, why);
    if (const char* why = unsupported(c, false)) return fail(DEER_ERR_UNSUPPORTED, why);
    if (!d_A || (c->T > 0 && (!d_x || !d_dt || !d_B || !d_C || !d_y)) || (is_packed(c) && !d_bounds)) return fail(DEER_ERR_INVALID_ARG, kMissing);
    const size_t e = type_bytes(c->dtype);
    if (any_misaligned(e, d_x, d_dt, d_B, d_C, d_z, d_y) || any_misaligned(4, d_A, d_skip, d_dt_bias, d_h0, d_last) || misaligned(d_bounds, 8))
        return fail(DEER_ERR_INVALID_ARG, kAligned);
    const ScanLayout l = scan_layout(c, false, d_bounds != nullptr);
    if (deer_status st = check_workspace(d_workspace, workspace_bytes, l.total)) return st;
    SelscanParams p = scan_params(c, l, d_bounds, d_workspace, false);
    p.x = d_x;
    p.dt = d_dt;
    p.A = d_A;
    p.B = d_B;
    p.C = d_C;
    p.skip = d_skip;
    p.z = d_z;
    p.bias = d_dt_bias;
    p.h0 = d_h0;
    p.y = d_y;
    p.last = d_last;
    p.vec = scan_vec(p, e, false);
    return launched("deer_selscan_solve", launch_selscan(c->dtype, p, reinterpret_cast<hipStream_t>(hip_stream)));
}

deer_status deer_selscan_grad(const deer_selscan_config* c, const void* d_x, const void* d_dt, const float* d_A, const void* d_B, const void* d_C,
                              const float* d_skip, const void* d_z, const float* d_dt_bias, const float* d_h0, const int64_t* d_bounds, const void* d_dy,
                              const float* d_dlast, void* d_dx, void* d_ddt, float* d_dA, void* d_dB, void* d_dC, float* d_dskip, void* d_dz, float* d_dbias,
                              float* d_dh0, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    if (const char* why = bad_config(c, false)) return fail(DEER_ERR_INVALID_ARG, why);
    if (const char* why = unsupported(c, false)) return fail(DEER_ERR_UNSUPPORTED, why);
    if (!d_A || !d_dA || (c->T > 0 && (!d_x || !d_dt || !d_B || !d_C || !d_dy || !d_dx || !d_ddt || !d_dB || !d_dC || (d_z && !d_dz))) || (is_packed(c) && !d_bounds))
        return fail(DEER_ERR_INVALID_ARG, kMissing);
    const size_t e = type_bytes(c->dtype);
    if (any_misaligned(e, d_x, d_dt, d_B, d_C, d_z, d_dy, d_dx, d_ddt, d_dB, d_dC, d_dz) ||
        any_misaligned(4, d_A, d_skip, d_dt_bias, d_h0, d_dlast, d_dA, d_dskip, d_dbias, d_dh0) || misaligned(d_bounds, 8))
        return fail(DEER_ERR_INVALID_ARG, kAligned);
    const ScanLayout l = scan_layout(c, true, d_bounds != nullptr);
    if (deer_status st = check_workspace(d_workspace, workspace_bytes, l.total)) return st;
    SelscanParams p = scan_params(c, l, d_bounds, d_workspace, true);
    p.x = d_x;
    p.dt = d_dt;
    p.A = d_A;
    p.B = d_B;
    p.C = d_C;
    p.skip = d_skip;
    p.z = d_z;
    p.bias = d_dt_bias;
    p.h0 = d_h0;
    p.dy = d_dy;
    p.dlast = d_dlast;
    p.dx = d_dx;
    p.ddt = d_ddt;
    p.dA = d_dA;
    p.dB = d_dB;
    p.dC = d_dC;
    p.dskip = d_dskip;
    p.dz = d_dz;
    p.dbias = d_dbias;
    p.dh0 = d_dh0;
    p.vec = scan_vec(p, e, true);
    hipStream_t stream = reinterpret_cast<hipStream_t>(hip_stream);
    hipError_t err = launch_selscan_marks(c->dtype, p, stream);
    if (err == hipSuccess) err = launch_selscan_grad(c->dtype, p, stream);
    return launched("deer_selscan_grad", err);
}

deer_status deer_selscan_step(const deer_selscan_config* c, const void* d_x, const void* d_dt, const float* d_A, const void* d_B, const void* d_C,
                              const float* d_skip, const void* d_z, const float* d_dt_bias, const int32_t* d_slots, int32_t n_slots, float* d_state,
                              void* d_y, void* hip_stream) {
    if (const char* why = bad_config(c, true)) return fail(DEER_ERR_INVALID_ARG, why);
    if (const char* why = unsupported(c, true)) return fail(DEER_ERR_UNSUPPORTED, why);
    if (n_slots < 1) return fail(DEER_ERR_INVALID_ARG, "n_slots must be positive");
    if (!d_x || !d_dt || !d_A || !d_B || !d_C || !d_state || !d_y) return fail(DEER_ERR_INVALID_ARG, kMissing);
    if (any_misaligned(type_bytes(c->dtype), d_x, d_dt, d_B, d_C, d_z, d_y) || any_misaligned(4, d_A, d_skip, d_dt_bias, d_state, d_slots))
        return fail(DEER_ERR_INVALID_ARG, kAligned);
    SelstepParams p{};
    p.rows = StepRows{d_slots, c->N, n_slots, zero_rest(c)};
    p.D = c->D;
    p.S = c->S;
    p.G = c->G;
    p.softplus = c->dt_act == DEER_ACT_SOFTPLUS;
    const int64_t states = (int64_t)c->G * c->S;
    p.stride_x = c->stride_x ? c->stride_x : c->D;
    p.stride_dt = c->stride_dt ? c->stride_dt : c->D;
    p.stride_B = c->stride_B ? c->stride_B : states;
    p.stride_C = c->stride_C ? c->stride_C : states;
    p.stride_z = c->stride_z ? c->stride_z : c->D;
    p.stride_y = c->stride_y ? c->stride_y : c->D;
    p.x = d_x;
    p.dt = d_dt;
    p.B = d_B;
    p.C = d_C;
    p.z = d_z;
    p.A = d_A;
    p.skip = d_skip;
    p.bias = d_dt_bias;
    p.state = d_state;
    p.y = d_y;
    return launched("deer_selscan_step", launch_selscan_step(c->dtype, p, reinterpret_cast<hipStream_t>(hip_stream)));
}

deer_status deer_groupnorm_workspace_bytes(const deer_groupnorm_config* c, int32_t grad, size_t* bytes) {
    if (!bytes) return fail(DEER_ERR_INVALID_ARG, "bytes is NULL");
    if (const char* why = bad_config(c)) return fail(DEER_ERR_INVALID_ARG, why);
    if (const char* why = too_large(c)) return fail(DEER_ERR_UNSUPPORTED, why);
    *bytes = norm_room(c, norm_layout_of(c, grad != 0)).total;
    return DEER_OK;
}

deer_status deer_groupnorm_solve(const deer_groupnorm_config* c, const void* d_x, const void* d_w, const void* d_bias, const void* d_z, const int64_t* d_bounds,
                                 void* d_y, void* d_stats, void* d_workspace, size_t workspace_bytes, void* hip_stream) {
    if (const char* why = bad_config(c)) return fail(DEER_ERR_INVALID_ARG, why);
    if (const char* why = too_large(c)) return fail(DEER_ERR_UNSUPPORTED, why);
    const bool stats = c->T > 0 || c->span == DEER_SPAN_SEQUENCE;
    if ((stats && !d_stats) || (c->T > 0 && (!d_x || !d_y)) || (is_packed(c) && !d_bounds)) return fail(DEER_ERR_INVALID_ARG, kMissing);
    if (any_misaligned(type_bytes(c->dtype), d_x, d_z, d_y) || any_misaligned(wide_bytes(c->dtype), d_w, d_bias, d_stats) || misaligned(d_bounds, 8))
        return fail(DEER_ERR_INVALID_ARG, kAligned);
    const NormRoom room = norm_room(c, norm_layout_of(c, false));
    if (deer_status st = check_workspace(d_workspace, workspace_bytes, room.total)) return st;
    NormParams p = norm_params(c, room, d_bounds, d_workspace);
    p.x = d_x;
    p.w = d_w;
    p.bias = d_bias;
    p.z = d_z;
    p.y = d_y;
    p.stats = d_stats;
    return launched("deer_groupnorm_solve", launch_groupnorm(c->dtype, false, p, reinterpret_cast<hipStream_t>(hip_stream)));
}

deer_status deer_groupnorm_grad(const deer_groupnorm_config* c, const void* d_x, const void* d_w, const void* d_bias, const void* d_z, const int64_t* d_bounds,
                                const void* d_stats, const void* d_dy, void* d_dx, void* d_dw, void* d_dbias, void* d_dz, void* d_workspace,
                                size_t workspace_bytes, void* hip_stream) {
    if (const char* why = bad_config(c)) return fail(DEER_ERR_INVALID_ARG, why);
    if (const char* why = too_large(c)) return fail(DEER_ERR_UNSUPPORTED, why);
    if ((c->T > 0 && (!d_x || !d_stats || !d_dy || !d_dx || (d_z && !d_dz))) || (is_packed(c) && !d_bounds)) return fail(DEER_ERR_INVALID_ARG, kMissing);
    if (any_misaligned(type_bytes(c->dtype), d_x, d_z, d_dy, d_dx, d_dz) || any_misaligned(wide_bytes(c->dtype), d_w, d_bias, d_stats, d_dw, d_dbias) ||
        misaligned(d_bounds, 8))
        return fail(DEER_ERR_INVALID_ARG, kAligned);
    const NormRoom room = norm_room(c, norm_layout_of(c, true));
    if (deer_status st = check_workspace(d_workspace, workspace_bytes, room.total)) return st;
    NormParams p = norm_params(c, room, d_bounds, d_workspace);
    p.x = d_x;
    p.w = d_w;
    p.bias = d_bias;
    p.z = d_z;
    p.stats = const_cast<void*>(d_stats);   // (read only in this direction)
    p.dy = d_dy;
    p.dx = d_dx;
    p.dw = d_dw;
    p.dbias = d_dbias;
    p.dz = d_dz;
    return launched("deer_groupnorm_grad", launch_groupnorm(c->dtype, true, p, reinterpret_cast<hipStream_t>(hip_stream)));
}

}  // extern "C"
