/*
 * deer.h -- C ABI of the DEER hot path for one AMD MI355X (gfx950).
 *
 * DEER (arxiv 2309.12252) evaluates a non-linear recurrence y_i = f(y_{i-1}, x_i)
 * (Sec. 3.4) or an ODE dy/dt = f(y) on a time grid (Sec. 3.3) by the fixed-point
 * iteration  y <- L_G^{-1}[ f(y_shifted) + G y_shifted ],  G = -df/dy  (Sec. 3.1
 * eq. 3 and 5), where L_G^{-1} solves a linear recurrence with an associative scan
 * over affine pairs (Sec. 3.3 eq. 9-10, Sec. 3.4 eq. 11).  Gradients take one
 * application of the transposed, reversed operator followed by the vector-Jacobian
 * product of f (Sec. 3.1.1 eq. 7).
 *
 * Conventions for every entry point
 *   - Pointers named d_* are DEVICE pointers owned by the caller; all other
 *     pointers are HOST pointers owned by the caller.  The library allocates no
 *     device memory: the caller hands in a workspace of deer_workspace_bytes().
 *     (deer_create() allocates a few hundred bytes of pinned HOST memory and the
 *     HIP events of the context; deer_destroy() frees them.)
 *   - Arrays are dense, row-major, in the dtype of the configuration (fp32 or
 *     fp64).  d_* arrays must be 16-byte aligned.
 *   - Work is enqueued on the HIP stream given to deer_create().  deer_eval()
 *     synchronises that stream (it reads the convergence error back) and returns
 *     with its outputs complete; deer_grad() and deer_linrec_solve() synchronise
 *     before returning as well.
 *   - Every call returns a deer_status; nothing throws or aborts across the ABI.
 *     After a non-OK status deer_last_error() describes what went wrong.
 *   - Calls on one context must not overlap in time.
 *
 * The model
 *   GRU cell (the paper names the cell but prints no equations; this is the
 *   reading used, gates r, z and candidate c, reset applied after the hidden
 *   projection):
 *       r = sigmoid(W_r x + b_r + U_r h)     z = sigmoid(W_z x + b_z + U_z h)
 *       q = U_c h + b_hc                     c = tanh(W_c x + b_c + r * q)
 *       f(h, x) = (1 - z) * c + z * h
 *     theta (flat): W[3n,d] (rows r|z|c), U[3n,n] (rows r|z|c), b[3n] (r|z|c), b_hc[n].
 *   LSTM cell (Sec. 3.4 names it as an instance of the recurrence; cell = DEER_CELL_LSTM, n = number of units u,
 *   1..16, d = 1..8).  The state is y = (h | c) with 2u entries, so y0 is [B,2u] and y, the guess and dL/dy are
 *   [B,T,2u]; gates in the order input, forget, candidate, output:
 *       i = sigmoid(W_i x + U_i h + b_i)   f = sigmoid(W_f x + U_f h + b_f)
 *       g = tanh(W_g x + U_g h + b_g)      o = sigmoid(W_o x + U_o h + b_o)
 *       c' = f * c + i * g                 h' = o * tanh(c')
 *     theta (flat): W[4u,d], U[4u,u], b[4u].  In fp32 with more than 4 units an iteration is a step by chunks (see
 *     deer_eval; with 5 to 8 units from some 8,000 positions or 1,500 steps on); otherwise a Jacobian kernel followed by the scan over the 2u x 2u
 *     Jacobians (embedded in the next state size with a scan kernel).
 *   LEM cell (the cell of the paper's last experiment, which trains it with DEER; the paper prints no equations, the
 *   ones of the publication it cites are used; cell = DEER_CELL_LEM, n = number of units u, 1..16, d = 1..8, t1 = the
 *   cell's step dt > 0).  The state is (y | z) with 2u entries, laid out like the LSTM's; two learned time scales:
 *       s1 = dt * sigmoid(W_1 x + U_1 y + b_1)   s2 = dt * sigmoid(W_2 x + U_2 y + b_2)
 *       z' = (1 - s1) * z + s1 * tanh(W_z x + U_z y + b_z)
 *       y' = (1 - s2) * y + s2 * tanh(W_y x + U_y z' + b_y)
 *     theta (flat): W[4u,d], U[4u,u], b[4u], row blocks in the order 1 | 2 | z | y.  Kernels as for the LSTM (with 8 units
 *     a small problem has its gradient alone by chunks).
 *   Multi-head GRU with strides (Sec. 4.4, App. B.4; heads > 1 or stride_levels > 1): the state is H heads of n
 *   channels, every head a GRU cell of its own on its own d input channels, and head h looks back
 *   s_h = 2^(h mod K) steps instead of one (the K stride levels are dealt out to the heads in turn):
 *       y[b,i,h,:] = f_h(y[b,i-s_h,h,:], x[b,i,h,:]),  with y0[b,h,:] in place of y[b,i-s_h,h,:] while i < s_h.
 *     Arrays: x [B,T,H,d], y0 [B,H,n], y / guess / dL/dy [B,T,H,n], dL/dx [B,T,H,d], dL/dy0 [B,H,n];
 *     theta and dL/dtheta [H][theta of one cell]; deer_theta_count() returns the total.  n = 2, 4 or 8, d <= 8,
 *     H <= 64, K <= 8.  A head that takes all input channels is obtained by projecting the inputs beforehand
 *     (a plain matrix product outside this library).
 *   MLP vector field (autonomous), L hidden layers of width w with activation s = tanh or softplus
 *   (s(a) = log(1 + exp(a)); App. B.2 uses six linear layers with softplus on all but the last):
 *       f(y) = W_out s(W_L s(... s(W_1 y + b_1) ...) + b_L) + b_out
 *     theta (flat): W_1[w,n], b_1[w], then W_l[w,w], b_l[w] for l = 2..L, then W_out[n,w], b_out[n].
 *   Two tanh layers of width 16, 32 or 64 (a multiple of n) have kernels of their own (fp32 with n = 8: on
 *   the matrix cores); every other depth, width and the softplus activation run general kernels.
 */
#ifndef DEER_H
#define DEER_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    DEER_OK = 0,
    DEER_ERR_INVALID_ARG = 1,  /* NULL where a pointer is required, non-positive size, bad enum          */
    DEER_ERR_UNSUPPORTED = 2,  /* a shape or mode this build has no kernel for                           */
    DEER_ERR_WORKSPACE = 3,    /* workspace NULL, misaligned or smaller than deer_workspace_bytes()      */
    DEER_ERR_HIP = 4,          /* a HIP runtime call failed, or a kernel reported an internal time-out   */
    DEER_ERR_NONFINITE = 5     /* the iteration produced a NaN/Inf; outputs hold the last iterate        */
} deer_status;

typedef enum { DEER_CELL_GRU = 0, DEER_CELL_MLP_ODE = 1, DEER_CELL_LSTM = 2, DEER_CELL_LEM = 3 } deer_cell;
typedef enum { DEER_F32 = 0, DEER_F64 = 1, DEER_BF16 = 2, DEER_F16 = 3 } deer_dtype; /* 16 bits: sequence operators only */
/* factor a_t of a gated recurrence, from its gate g: a = g; a = exp(g); a = 1 / (1 + exp(-g)), the input weighted with 1 - a */
typedef enum { DEER_GATE_FACTOR = 0, DEER_GATE_LOG = 1, DEER_GATE_SIGMOID = 2 } deer_gate;
/* how rows lie (member `packed`), and what becomes of rows in the outputs that belong to no sequence: left as they are, or zeroed */
typedef enum { DEER_ROWS_PADDED = 0, DEER_ROWS_PACKED = 1, DEER_REST_ZERO = 256 } deer_rows;
typedef enum { DEER_ACT_TANH = 0, DEER_ACT_SOFTPLUS = 1 } deer_activation;

typedef struct {
    int32_t cell;               /* deer_cell                                                             */
    int32_t dtype;              /* deer_dtype                                                            */
    int32_t B;                  /* batch: independent sequences                                          */
    int32_t T;                  /* GRU: number of steps; MLP_ODE: number of grid points (>= 2)           */
    int32_t n;                  /* state size.  GRU: 1..64, above 32 in fp32 only (1, 2, 4, 8, 16, 32, 64 have  */
                                /* kernels of their own; any other size runs embedded in the next of     */
                                /* those, with identical results);                                       */
                                /* MLP_ODE: 2, 4 or 8; multi-head GRU: 2, 4 or 8 per head; LSTM and LEM: */
                                /* the number of units u, 1..16 (the state has 2u entries)               */
    int32_t d;                  /* GRU input size (1..32); LSTM and LEM: 1..8; ignored for MLP_ODE       */
    int32_t mlp_width;          /* MLP_ODE hidden width w: a multiple of 4, 4..64; ignored for GRU       */
    int32_t mlp_hidden_layers;  /* MLP_ODE: hidden layers L, 1..5 (L + 1 linear layers)                  */
    double t0, t1;              /* MLP_ODE: uniform grid t_j = t0 + j (t1 - t0)/(T - 1); LEM: t1 = step dt */
    int32_t mlp_activation;     /* MLP_ODE: deer_activation of the hidden layers (0 = tanh)              */
    int32_t heads;              /* GRU: number of heads H (0 or 1: the plain cell); see "multi-head GRU"  */
    int32_t stride_levels;      /* GRU: stride levels K (0 or 1: every head has stride 1)                */
    int32_t reserved;           /* must be 0                                                             */
} deer_config;

typedef struct deer_ctx deer_ctx; /* opaque, host memory owned by the library */

/* Accumulated per-kernel device time, filled while profiling is on (see deer_set_profiling). */
typedef struct {
    double funceval_ms;   int64_t funceval_launches;   /* f, Jacobian and right-hand side            */
    double discretise_ms; int64_t discretise_launches; /* ODE only: exp(-G dt), phi1; in deer_grad also   */
                                                       /* the residual and the dual discretisation       */
    double scan_ms;       int64_t scan_launches;       /* inverse linear operator (+ fused max|dy|)  */
    double vjp_ms;        int64_t vjp_launches;        /* VJP of f + parameter-gradient reduction    */
    double fused_ms;      int64_t fused_launches;      /* GRU: cell + scan + max|dy| in one launch;   */
                                                       /* in deer_grad: cell inside the reverse scan  */
    double newton_ms;     int64_t newton_launches;     /* GRU, small problems: a whole solve in one   */
    int64_t newton_iterations;                         /* Newton iterations inside those launches     */
} deer_profile;

/* Number of parameters in the flat theta of this configuration (layouts above); 0 if invalid. */
size_t deer_theta_count(const deer_config* cfg);

/* Bytes of device workspace deer_create() needs for cfg: a second trajectory buffer, the words the scan's
 * tiles publish for each other, counters, partial sums of dL/dtheta -- and, only where a kernel pair exchanges
 * them through memory (MLP_ODE; GRU in fp64 with n >= 16, with d beyond what the in-scan cell or the chunks take, or with the
 * DEER_FUSED / DEER_GRAD_FUSED knobs at 0; LSTM and LEM where they do not step by chunks), the Jacobian stream [B,T,n,n] and the right-hand side, the O(n^2 T)
 * memory of Sec. 3.5.  Where the cell is evaluated inside the scans the workspace is O(n T).  Where steps run by chunks
 * (see deer_eval) every chunk has a map of N^2 + N scalars (N = state size, for LSTM and LEM 2u rounded up to 16 or 32): one for every 4 to 64
 * positions, so short sequences in large numbers take up to (N + 1) / 4 trajectories of it, long ones a fraction of one.  Large multi-head
 * layers of three stride levels and more have copies of x and of a trajectory by heads there, 16 GiB at most.
 * The environment variables listed under "Environment" below are read here and in deer_create(); both calls must
 * see the same values. */
deer_status deer_workspace_bytes(const deer_config* cfg, size_t* bytes);

/* Create a context.  d_workspace (device, 256-byte aligned, >= deer_workspace_bytes) stays owned by
 * the caller and must outlive the context; the library may overwrite all of it in any call.
 * hip_stream is a hipStream_t (NULL = the default stream).  On failure *out is NULL. */
deer_status deer_create(const deer_config* cfg, void* d_workspace, size_t workspace_bytes,
                        void* hip_stream, deer_ctx** out);

/* Forward evaluation by DEER (Sec. 3.1 eq. 3 with eq. 5; iteration control as in App. B.1).
 *   d_theta   in  parameters, deer_theta_count() entries
 *   d_x       in  GRU: inputs [B,T,d]; MLP_ODE: ignored (may be NULL)
 *   d_y0      in  initial state [B,n]
 *   d_y_guess in  initial guess [B,T,n], or NULL for all zeros (the paper's benchmarks start from
 *                 zeros; a previous solution can be passed as a warm start, Sec. 3.1)
 *   tol       in  stop when err = max|y_next - y| <= tol (paper: 1e-4 fp32, 1e-7 fp64)
 *   max_iter  in  at most this many iterations (>= 0)
 *   d_y       out GRU: y[b,i-1,:] = y_i for i = 1..T.  MLP_ODE: y[b,j,:] = y(t_j), y[b,0,:] = y0;
 *                 the first grid point is pinned to y0 in every iterate, so err runs over j >= 1
 *   iters     out number of iterations (linear solves) performed, including the one whose err met tol
 *   final_err out err of the last iteration (1e10 if max_iter == 0)
 *   converged out 1 if final_err <= tol else 0.  Not converging is not an error: DEER_OK is returned
 *                 with iters == max_iter (Newton's method may diverge far from the solution, Sec. 3.5).
 * The convergence test is global over batch, time and state.  DEER_ERR_NONFINITE if err is NaN/Inf.
 * d_y doubles as one of the two iterate buffers: it is overwritten during the call; d_y_guess may be
 * the same buffer as d_y.  How the iterations are put on the device does not change the result and is
 * chosen from the shapes: for the GRU with n <= 8 the cell is evaluated inside the scan kernel (the
 * Jacobians never reach memory), and when all tiles of the problem fit on the device at once the
 * whole solve is one kernel launch; for n = 16, 32 in fp32 the cell is evaluated inside the matrix-core
 * scan.  In fp32 large problems of the GRU with n = 5..8 (plain and multi-head with n = 8) and n = 9..32, the GRU with n = 33..64 at every
 * size (each with d up to 8 or 16), LSTM and LEM step by chunks instead: chunks of 4 to 64 positions are reduced to one affine map each, the
 * maps are folded into carries and the chunks walked side by side, two launches an iteration.  Otherwise an iteration is a
 * Jacobian kernel followed by a scan kernel (see "Environment").
 * A solve whose Jacobians expand can overflow single precision before its iterates do: the product of the Jacobians over one tile of a scan or
 * one chunk (up to 64 positions; 1,024 in the n <= 8 scan) has to be representable.
 * The Jacobians of the last iteration are not kept for deer_grad(): Sec. 3.1.1 offers that as a way to trade memory
 * for speed, this library always recomputes them at the trajectory it is given (exact for any trajectory, and the
 * O(n^2 T) buffer is not needed), so there is no save-the-Jacobian option in deer_config. */
deer_status deer_eval(deer_ctx* ctx, const void* d_theta, const void* d_x, const void* d_y0,
                      const void* d_y_guess, double tol, int32_t max_iter, void* d_y,
                      int32_t* iters, double* final_err, int32_t* converged);

/* Backward derivative (Sec. 3.1.1 eq. 7): the cotangent g = dL/dy is pushed through the transposed,
 * time-reversed linear operator (one reverse scan), then through the vector-Jacobian product of f.
 * The Jacobians are recomputed at the trajectory d_y that is passed in, so the trajectory may
 * come from deer_eval() or from a sequential evaluation (Sec. 3.1.1, last paragraph).
 *   GRU:     lam_T = g_T, lam_i = g_i + J_{i+1}^T lam_{i+1};  dL/dtheta = sum_i (df/dtheta)_i^T lam_i, same for x.
 *   MLP_ODE: on the discretised operator of Sec. 3.3 eq. 8-9 with G frozen at the trajectory:
 *            lam_{T-1} = g_{T-1}, lam_j = g_j + Gbar_j^T lam_{j+1};  dL/dy0 = lam_0;
 *            dL/dtheta = sum_j (df/dtheta)(y_j)^T w_j,  w_j = (P_j^T lam_{j+1} + P_{j-1}^T lam_j) / 2,
 *            P_j = dt phi1(-Gc_j dt) (terms outside the grid dropped).  This is the derivative eq. 7 defines;
 *            it differs from the derivative of the discrete solution by O(dt^2).  d_x, d_y0 and d_dLdx are
 *            ignored (the field is autonomous and y[:,0,:] is the initial state).
 *   d_y        in  trajectory [B,T,n]          d_dLdy   in  g = dL/dy [B,T,n]
 *   d_dLdx     out [B,T,d], or NULL to skip    d_dLdtheta out [theta_count] (overwritten, not accumulated)
 *   d_dLdy0    out [B,n], or NULL to skip
 * The parameter gradient is summed in a fixed order: two calls with the same inputs return the same bits.
 * For the GRU the transposed Jacobians are computed inside the reverse scan wherever deer_eval() evaluates the
 * cell inside the forward scan (n <= 8 with d <= 8; fp32 n = 16, 32 with d <= 16), and in fp32 with n = 16, 32, 64
 * the vector-Jacobian product runs on the matrix cores (so does the MLP field's for fp32, n = 8 and width 16,
 * 32 or 64).  By chunks the vector-Jacobian product is part of the reverse walk (n = 8, 16, multi-head, LSTM, LEM); see "Environment" for the knobs that select the separate kernels instead. */
deer_status deer_grad(deer_ctx* ctx, const void* d_theta, const void* d_x, const void* d_y0,
                      const void* d_y, const void* d_dLdy, void* d_dLdx, void* d_dLdtheta,
                      void* d_dLdy0);

/* The inverse linear operator alone (Sec. 3.3 eq. 9-10, Sec. 3.4 eq. 11):
 * y_i = A_i y_{i-1} + b_i for i = 1..T from y_0, for B independent sequences, by the blocked
 * associative scan.  Shapes come from the context (B, T, n, dtype).
 * (plain GRU-shaped contexts with n = 1, 2, 4, 8, 16, 32 or, in fp32, 64 only).
 *   d_A [B,T,n,n]   d_b [B,T,n]   d_y0 [B,n] (NULL = zeros)   d_y out [B,T,n]
 *   reverse != 0 applies the dual (transposed, time-reversed) operator of Sec. 3.1.1 eq. 7 instead:
 *   y_T = b_T, y_i = b_i + A_{i+1}^T y_{i+1}; d_y0 is ignored.  A is read as stored and transposed
 *   on the fly. */
deer_status deer_linrec_solve(deer_ctx* ctx, const void* d_A, const void* d_b, const void* d_y0,
                              void* d_y, int32_t reverse);

/* deer_linrec_solve() for callers that cannot allocate device memory or hand in a workspace: code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc.  The same scan kernels run, but the words their
 * tiles publish for each other, the tile dispenser and the status word live in a static device array inside the
 * library (64 MiB; every GPU the library runs on holds its own copy until the process ends) instead of a workspace,
 * and no context is needed.  The call allocates nothing (no hipMalloc/hipFree, no pinned host memory, no events),
 * enqueues three kernels on hip_stream (a fill that clears the part of the array it uses, the scan, a one-word
 * copy) and returns without synchronising: outputs are complete when the stream reaches that point.
 *   dtype, B, T, n   as in deer_config (n = 1, 2, 4, 8, 16, 32 or, in fp32, 64)
 *   d_A [B,T,n,n]  d_b [B,T,n]  d_y0 [B,n] or NULL (zeros)  d_y out [B,T,n]  reverse: as in deer_linrec_solve()
 *   hip_stream     hipStream_t (NULL = the default stream)
 *   d_status       out, DEVICE int32, or NULL: 0, or non-zero if a tile waited too long for its predecessors
 *                  (then d_y is not valid); the host-side return value cannot report that without a synchronisation
 * Limit: the published words of all tiles must fit the array; a shape beyond it is rejected with
 * DEER_ERR_WORKSPACE before anything is enqueued (n = 32: about 480,000 positions in all; n = 8: several 10^7).
 * All calls on one GPU share that GPU's array: calls that overlap in time on one GPU (two streams, two threads) race.
 * Returns DEER_OK once everything is enqueued; errors are reported through deer_last_error(NULL). */
deer_status deer_linrec_solve_static(int32_t dtype, int32_t B, int32_t T, int32_t n, const void* d_A, const void* d_b,
                                     const void* d_y0, void* d_y, int32_t reverse, void* hip_stream,
                                     int32_t* d_status);

/* ---------------------------------------------------------------------------------------------------------------------
 * Sequence operators: recurrences that are linear from the start (deer_eval() makes linear ones of a non-linear one), with gates,
 * for every length from one token on, and dropout.
 *
 * Conventions, beyond those at the top of this file
 *   - No context.  Every call enqueues its kernels on hip_stream (a stream of the current device; NULL = the default stream) and
 *     returns without synchronising; nothing is allocated, so a call may be captured into a HIP graph (each captured call with a workspace
 *     of its own, or never replayed at the same time).  Errors are reported through deer_last_error(NULL).
 *   - Types: DEER_F32, DEER_F64 (deer_diagrec_*, deer_dropout), DEER_BF16, DEER_F16 (deer_diagrec_*, deer_dropout).  deer_matrec_*: DEER_F32 and DEER_BF16.  Sums and states are held in
 *     32 bits (fp64: 64); h0, last, dlast, dh0, states and their gradients are arrays of that wider type, dense.
 *   - Rows.  packed = 0: N sequences of T rows, row t of sequence n is row n T + t of every array; d_bounds (device, int64 [N], or NULL) holds how
 *     many rows of each count.  packed = 1: the sequences lie one behind the other in T rows; d_bounds (device, int64 [N + 1], not NULL) holds
 *     where they begin, its last entry where the last one ends.  Sequences may be empty: their final state is the initial
 *     one.  Rows that belong to no sequence have no influence; in the outputs they are not written, or zeroed where
 *     DEER_REST_ZERO is added to packed.  Bounds outside 0 .. T are clamped;
 *     packed bounds that decrease give results without meaning, within the arrays.
 *   - stride_*: elements from one row to the next (0: dense), so that slices of a wider array can be handed in; the
 *     last dimension is dense (deer_diagrec_solve(), deer_diagrec_grad(): rows and strides of at most 2^22).  A call whose largest launch
 *     would have 2^32 work items or more is refused (DEER_ERR_UNSUPPORTED).
 *   - Pointers are aligned to the element; where all rows are aligned to more, wider loads are used.  Outputs must not overlap
 *     inputs, except where an operator says so.
 *   - What is NaN or infinite in a sequence stays in that sequence. */
typedef struct {
    int32_t dtype;       /* deer_dtype                                                                     */
    int32_t gate;        /* deer_gate                                                                      */
    int32_t N;           /* sequences (deer_diagrec_step: rows), >= 1                                      */
    int32_t D;           /* channels, >= 1                                                                 */
    int64_t T;           /* rows of a sequence, packed: of all of them; >= 0                               */
    int32_t packed;      /* 0 or 1, and DEER_REST_ZERO                                                     */
    uint32_t draw;       /* dropout: number of the draw under this seed                                    */
    int64_t stride_gate; /* rows of d_gate and d_dgate                                                     */
    int64_t stride_in;   /* rows of d_in and d_din                                                         */
    int64_t stride_out;  /* rows of d_h and d_dh                                                           */
    double drop;         /* share of the inputs that is dropped, 0 <= drop < 1 (see deer_dropout)          */
    uint64_t seed;       /* dropout: seed                                                                  */
} deer_diagrec_config;

/* Bytes of device workspace (256-byte aligned) that deer_diagrec_solve() (grad = 0) or deer_diagrec_grad() (grad = 1) needs: some
 * 8 bytes a channel for every 64 to 256 rows (fp64: 16). */
deer_status deer_diagrec_workspace_bytes(const deer_diagrec_config* cfg, int32_t grad, size_t* bytes);

/* Gated linear recurrence, a state for every channel: h_t = a_t h_{t-1} + u_t, u_t = x_t (DEER_GATE_SIGMOID: (1 - a_t) x_t), x after dropout.
 *   d_gate, d_in  in  [rows, D]      d_h0  in  [N, D] or NULL (zeros)
 *   d_h           out [rows, D] (may be d_in, with the same stride)      d_last  out [N, D] state behind every sequence's last row, or NULL
 * One pass over the data; two calls with the same inputs return the same bits.  The product of the factors over 256 rows has to be
 * representable (gates that make the state grow can overflow it). */
deer_status deer_diagrec_solve(const deer_diagrec_config* cfg, const void* d_gate, const void* d_in, const void* d_h0,
                               const int64_t* d_bounds, void* d_h, void* d_last, void* d_workspace, size_t workspace_bytes,
                               void* hip_stream);

/* Its gradient, at the trajectory d_h that is handed in (deer_diagrec_solve()'s): in 16 bits dL/dgate has the state of the row in front as it was rounded there.
 *   d_dh     in  dL/dh [rows, D]            d_dlast  in  dL/dlast [N, D] or NULL (zeros)
 *   d_dgate  out dL/dgate [rows, D]         d_din    out dL/din [rows, D]          d_dh0  out [N, D] or NULL */
deer_status deer_diagrec_grad(const deer_diagrec_config* cfg, const void* d_gate, const void* d_in, const void* d_h0,
                              const int64_t* d_bounds, const void* d_h, const void* d_dh, const void* d_dlast, void* d_dgate,
                              void* d_din, void* d_dh0, void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* One token for each of N rows (T and drop are not looked at, of packed DEER_REST_ZERO only): the states lie in n_slots slots [n_slots, D] and are updated
 * in place; row n has slot d_slots[n] (device, int32 [N]; NULL: slot n).  A row whose slot is out of range, as in a
 * padded batch, or is the slot of a row in front of it is passed over: the state stays as it is, and so does its row of d_h, or is zeroed with DEER_REST_ZERO.
 * Repeated slots are found by comparing with all rows in front, which is for batches of up to some thousand rows (4,096 of 64 channels 10 us, 16,384 70 us; with
 * d_slots NULL 5 and 11). */
deer_status deer_diagrec_step(const deer_diagrec_config* cfg, const void* d_gate, const void* d_in, const int32_t* d_slots,
                              int32_t n_slots, void* d_state, void* d_h, void* hip_stream);

/* Dropout: y = x / (1 - p) where an element is kept, 0 where it is dropped.  Which ones are kept follows from (seed, draw) and the element's
 * sequence, row and channel alone, so the backward pass is the same call on the gradient and no mask is stored; deer_diagrec_*
 * with drop = p draws the same mask (packed rows count as one sequence, in either call).  p is rounded to 2^-16 (and the scale taken from the rounded value).
 *   d_x in, d_y out [N, T, D], rows stride_in and stride_out apart (0: dense); d_y may be d_x with the same stride. */
deer_status deer_dropout(int32_t dtype, int32_t N, int64_t T, int32_t D, const void* d_x, int64_t stride_in, void* d_y,
                         int64_t stride_out, double p, uint64_t seed, uint32_t draw, void* hip_stream);

/* Gated linear recurrence with a matrix as the state of every head: S_t = exp(g_t) S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t, S [Dk, Dv]. */
typedef struct {
    int32_t dtype;     /* DEER_F32 or DEER_BF16: q, k, v, o and their gradients                            */
    int32_t N;         /* sequences (deer_matrec_step: rows), >= 1                                         */
    int64_t T;         /* rows of a sequence, packed: of all of them; >= 0                                 */
    int32_t packed;    /* 0 or 1, and DEER_REST_ZERO                                                       */
    int32_t Hk, Hv;    /* heads of q and k, heads of v: a multiple; head h goes with h / (Hv / Hk)         */
    int32_t Dk, Dv;    /* 1 .. 128                                                                         */
    int32_t reserved;  /* must be 0                                                                        */
    double scale;      /* of the outputs; a finite number of 32 bits                                       */
    int64_t stride_q, stride_k, stride_v, stride_o;   /* rows (0: Hk Dk, Hk Dk, Hv Dv, Hv Dv); gradients lie like their arrays, dL/do like o */
} deer_matrec_config;

/* Bytes of device workspace (256-byte aligned) that deer_matrec_solve() (grad = 0) or deer_matrec_grad() (grad = 1) needs: the
 * states between the segments that long sequences are cut into, and for the gradient dq and dk by heads of v in float32 where several share one. */
deer_status deer_matrec_workspace_bytes(const deer_matrec_config* cfg, int32_t grad, size_t* bytes);

/* d_q, d_k in [rows, Hk, Dk]   d_v in [rows, Hv, Dv]   d_gate in [rows, Hv] float32, the logarithms of the factors (dense)   d_s0 in [N, Hv, Dk, Dv]
 * float32 or NULL (zeros)   d_o out [rows, Hv, Dv]   d_last out [N, Hv, Dk, Dv] float32 or NULL.  By chunks of 64 rows on the matrix cores; states
 * in fp32 (bf16: sums of products in fp32, whose weights enter as three bf16 pieces; an output reads states and weights of pairs as two: it is off by its own rounding
 * and 2^-16 of its terms), two calls with the same inputs return the same bits.
 * What is not finite in a row reaches the outputs of its chunk, also in front of it, and all that come later. */
deer_status deer_matrec_solve(const deer_matrec_config* cfg, const void* d_q, const void* d_k, const void* d_v, const float* d_gate,
                              const float* d_s0, const int64_t* d_bounds, void* d_o, float* d_last, void* d_workspace,
                              size_t workspace_bytes, void* hip_stream);

/* Its gradient.  d_do in dL/do   d_dlast in [N, Hv, Dk, Dv] or NULL (zeros)   d_dq, d_dk, d_dv out   d_dgate out [rows, Hv] float32 or NULL   d_ds0 out
 * [N, Hv, Dk, Dv] float32 or NULL.  The states are computed again; gradients of shared heads are summed in a fixed order.  bf16: weights of pairs, and the state
 * in dv, enter as two pieces, as in the outputs. */
deer_status deer_matrec_grad(const deer_matrec_config* cfg, const void* d_q, const void* d_k, const void* d_v, const float* d_gate,
                             const float* d_s0, const int64_t* d_bounds, const void* d_do, const float* d_dlast, void* d_dq, void* d_dk,
                             void* d_dv, float* d_dgate, float* d_ds0, void* d_workspace, size_t workspace_bytes, void* hip_stream);

/* One token for each of N rows (T is not looked at, of packed DEER_REST_ZERO only): states in n_slots slots [n_slots, Hv, Dk, Dv], float32, updated in place; slots as in
 * deer_diagrec_step(). */
deer_status deer_matrec_step(const deer_matrec_config* cfg, const void* d_q, const void* d_k, const void* d_v, const float* d_gate,
                             const int32_t* d_slots, int32_t n_slots, float* d_state, void* d_o, void* hip_stream);

/* Switch per-kernel timing with HIP events on the context's stream on or off (off by default;
 * turning it on resets the accumulated numbers), and read the numbers accumulated so far. */
deer_status deer_set_profiling(deer_ctx* ctx, int32_t on);
deer_status deer_get_profile(deer_ctx* ctx, deer_profile* out);

/* Text of the last error on this context (never NULL; valid until the next call on ctx).
 * With ctx == NULL: the last error of a failed deer_create()/deer_workspace_bytes() on this thread. */
const char* deer_last_error(const deer_ctx* ctx);

/* Free the context (host memory and HIP events only; the workspace stays with the caller). */
void deer_destroy(deer_ctx* ctx);

/* Environment.  Every variable the library reads; all are meant for tests and measurements, none changes a
 * result beyond rounding.  Read by deer_workspace_bytes() and deer_create() (the plan and the workspace size
 * depend on them), except DEER_VJP_MFMA and DEER_MLP_MFMA, which deer_grad() / deer_eval() read at each call.
 *   DEER_FUSED=0        GRU, LSTM, LEM: run the cell kernel and the plain scan as two launches per iteration (needs the
 *                       Jacobian stream in the workspace) instead of the scan with the cell inside
 *   DEER_GRAD_FUSED=0   GRU deer_grad(): Jacobian kernel + plain reverse scan instead of the reverse scan with the
 *                       cell inside (needs the Jacobian stream in the workspace); LSTM, LEM and the GRU with n = 5..8 then
 *                       do not step by chunks in deer_eval() either
 *   DEER_ONE_LAUNCH=0   GRU, n <= 8: one launch per iteration even when the whole solve fits one launch
 *   DEER_FUSED_L, DEER_FUSED_W, DEER_SCAN_L
 *                       tile shapes of the n <= 8 kernels: positions per lane group (1, 2, 4, 8, 10, 12, 16; 24 for
 *                       the plain n = 4 scan) and wavefronts per tile (4 or 8); ignored when no such variant exists.  DEER_FUSED_L also keeps the GRU with n = 5..8
 *                       and the multi-head GRU off the chunks
 *   DEER_CHUNK_L, DEER_CHUNK_UNIT
 *                       GRU with n = 5..8, 16, 32, 64, multi-head GRU with n = 8, LSTM and LEM in fp32: positions per chunk of the step by chunks (a multiple of
 *                       four, at least four), which is then taken at every size (by default where it is faster), and
 *                       chunks per workgroup of its first launch (4, 8 or 16)
 *   DEER_BATCH          Newton iterations enqueued per host round trip on a fresh context (1..8, default 4)
 *   DEER_VJP_MFMA=0     vector-ALU kernels for the vector-Jacobian products instead of the matrix-core ones; no effect where
 *                       the product is part of the reverse walk by chunks (DEER_FUSED=0 or DEER_FUSED_L leave that route)
 *   DEER_MLP_MFMA=0     MLP fields outside the two-layer tanh shapes (fp32, n = 8, width 32 or 64): vector-ALU field
 *                       kernel instead of the matrix-core one
 * Test hooks (exercise paths that ordinary runs reach rarely; never set them in production):
 *   DEER_EPOCH0         first launch epoch of the context (default 1), to reach the wrap-around of the 30-bit
 *                       epoch that tags published words
 *   DEER_TEST_SPIN_LIMIT, DEER_TEST_EXTRA_WORKGROUPS
 *                       polls before a wait in the one-launch solve gives up, and a number (1..4) of workgroups
 *                       that solve also waits for although they do not exist: together they force the give-up path,
 *                       after which deer_eval() solves launch by launch */

#ifdef __cplusplus
}
#endif
#endif /* DEER_H */
