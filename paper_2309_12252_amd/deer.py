"""Thin ctypes binding of the C-ABI HIP library (include/deer.h).

Argument marshalling only: every step of the path runs in the library's kernels.
PyTorch supplies device memory and the stream.  Loading fails loudly when the
library has not been built (``python -m paper_2309_12252_amd.build``); there is no
CPU fallback.
"""
import ctypes
import functools
import operator
import os

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdeer_hip.so")

DEER_OK, DEER_ERR_INVALID_ARG, DEER_ERR_UNSUPPORTED, DEER_ERR_WORKSPACE, DEER_ERR_HIP, DEER_ERR_NONFINITE = range(6)
DEER_CELL_GRU, DEER_CELL_MLP_ODE, DEER_CELL_LSTM, DEER_CELL_LEM = 0, 1, 2, 3
DEER_F32, DEER_F64, DEER_BF16, DEER_F16 = 0, 1, 2, 3
DEER_GATE_FACTOR, DEER_GATE_LOG, DEER_GATE_SIGMOID = 0, 1, 2
DEER_ROWS_PADDED, DEER_ROWS_PACKED, DEER_REST_ZERO = 0, 1, 256

EXPORTS = ["deer_theta_count", "deer_workspace_bytes", "deer_create", "deer_eval", "deer_grad",
           "deer_linrec_solve", "deer_linrec_solve_static", "deer_set_profiling", "deer_get_profile", "deer_last_error", "deer_destroy",
           "deer_diagrec_workspace_bytes", "deer_diagrec_solve", "deer_diagrec_grad", "deer_diagrec_step", "deer_dropout",
           "deer_matrec_workspace_bytes", "deer_matrec_solve", "deer_matrec_grad", "deer_matrec_step"]


class DeerConfig(ctypes.Structure):
    _fields_ = [("cell", ctypes.c_int32), ("dtype", ctypes.c_int32), ("B", ctypes.c_int32), ("T", ctypes.c_int32),
                ("n", ctypes.c_int32), ("d", ctypes.c_int32), ("mlp_width", ctypes.c_int32),
                ("mlp_hidden_layers", ctypes.c_int32), ("t0", ctypes.c_double), ("t1", ctypes.c_double),
                ("mlp_activation", ctypes.c_int32), ("heads", ctypes.c_int32), ("stride_levels", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class DeerProfile(ctypes.Structure):
    _fields_ = [("funceval_ms", ctypes.c_double), ("funceval_launches", ctypes.c_int64),
                ("discretise_ms", ctypes.c_double), ("discretise_launches", ctypes.c_int64),
                ("scan_ms", ctypes.c_double), ("scan_launches", ctypes.c_int64),
                ("vjp_ms", ctypes.c_double), ("vjp_launches", ctypes.c_int64),
                ("fused_ms", ctypes.c_double), ("fused_launches", ctypes.c_int64),
                ("newton_ms", ctypes.c_double), ("newton_launches", ctypes.c_int64),
                ("newton_iterations", ctypes.c_int64)]


class DiagrecConfig(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("gate", ctypes.c_int32), ("N", ctypes.c_int32), ("D", ctypes.c_int32),
                ("T", ctypes.c_int64), ("packed", ctypes.c_int32), ("draw", ctypes.c_uint32),
                ("stride_gate", ctypes.c_int64), ("stride_in", ctypes.c_int64), ("stride_out", ctypes.c_int64),
                ("drop", ctypes.c_double), ("seed", ctypes.c_uint64)]


class MatrecConfig(ctypes.Structure):
    _fields_ = [("dtype", ctypes.c_int32), ("N", ctypes.c_int32), ("T", ctypes.c_int64), ("packed", ctypes.c_int32),
                ("Hk", ctypes.c_int32), ("Hv", ctypes.c_int32), ("Dk", ctypes.c_int32), ("Dv", ctypes.c_int32),
                ("reserved", ctypes.c_int32), ("scale", ctypes.c_double), ("stride_q", ctypes.c_int64),
                ("stride_k", ctypes.c_int64), ("stride_v", ctypes.c_int64), ("stride_o", ctypes.c_int64)]


class DeerError(RuntimeError):
    def __init__(self, status, message):
        super().__init__("deer status %d: %s" % (status, message))
        self.status = status


_lib = None


def load_library():
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError("%s is missing: build it with `python -m paper_2309_12252_amd.build` "
                           "(there is no fallback path)" % LIB_PATH)
    lib = ctypes.CDLL(LIB_PATH)
    vp, i32, dbl = ctypes.c_void_p, ctypes.c_int32, ctypes.c_double
    cfgp = ctypes.POINTER(DeerConfig)
    lib.deer_theta_count.restype = ctypes.c_size_t
    lib.deer_theta_count.argtypes = [cfgp]
    lib.deer_workspace_bytes.restype = ctypes.c_int
    lib.deer_workspace_bytes.argtypes = [cfgp, ctypes.POINTER(ctypes.c_size_t)]
    lib.deer_create.restype = ctypes.c_int
    lib.deer_create.argtypes = [cfgp, vp, ctypes.c_size_t, vp, ctypes.POINTER(vp)]
    lib.deer_eval.restype = ctypes.c_int
    lib.deer_eval.argtypes = [vp, vp, vp, vp, vp, dbl, i32, vp, ctypes.POINTER(i32), ctypes.POINTER(dbl),
                              ctypes.POINTER(i32)]
    lib.deer_grad.restype = ctypes.c_int
    lib.deer_grad.argtypes = [vp] * 9
    lib.deer_linrec_solve.restype = ctypes.c_int
    lib.deer_linrec_solve.argtypes = [vp, vp, vp, vp, vp, i32]
    lib.deer_linrec_solve_static.restype = ctypes.c_int
    lib.deer_linrec_solve_static.argtypes = [i32, i32, i32, i32, vp, vp, vp, vp, i32, vp, vp]
    lib.deer_set_profiling.restype = ctypes.c_int
    lib.deer_set_profiling.argtypes = [vp, i32]
    lib.deer_get_profile.restype = ctypes.c_int
    lib.deer_get_profile.argtypes = [vp, ctypes.POINTER(DeerProfile)]
    lib.deer_last_error.restype = ctypes.c_char_p
    lib.deer_last_error.argtypes = [vp]
    lib.deer_destroy.restype = None
    lib.deer_destroy.argtypes = [vp]
    size, i64, u32, u64 = ctypes.c_size_t, ctypes.c_int64, ctypes.c_uint32, ctypes.c_uint64
    dcp, mcp = ctypes.POINTER(DiagrecConfig), ctypes.POINTER(MatrecConfig)
    for name, args in (("deer_diagrec_workspace_bytes", [dcp, i32, ctypes.POINTER(size)]),
                       ("deer_diagrec_solve", [dcp] + [vp] * 7 + [size, vp]),
                       ("deer_diagrec_grad", [dcp] + [vp] * 11 + [size, vp]),
                       ("deer_diagrec_step", [dcp] + [vp] * 3 + [i32] + [vp] * 3),
                       ("deer_matrec_workspace_bytes", [mcp, i32, ctypes.POINTER(size)]),
                       ("deer_matrec_solve", [mcp] + [vp] * 9 + [size, vp]),
                       ("deer_matrec_grad", [mcp] + [vp] * 14 + [size, vp]),
                       ("deer_matrec_step", [mcp] + [vp] * 5 + [i32] + [vp] * 3),
                       ("deer_dropout", [i32, i32, i64, i32, vp, i64, vp, i64, dbl, u64, u32, vp])):
        getattr(lib, name).restype = ctypes.c_int
        getattr(lib, name).argtypes = args
    _lib = lib
    return lib


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else None


DEER_ACT_TANH, DEER_ACT_SOFTPLUS = 0, 1


def make_config(cell, dtype, B, T, n, d=0, mlp_width=0, mlp_hidden_layers=0, t0=0.0, t1=0.0, mlp_activation=0,
                heads=0, stride_levels=0):
    return DeerConfig(int(cell), int(dtype), int(B), int(T), int(n), int(d), int(mlp_width),
                      int(mlp_hidden_layers), float(t0), float(t1), int(mlp_activation), int(heads), int(stride_levels), 0)


def theta_count(cfg):
    return int(load_library().deer_theta_count(ctypes.byref(cfg)))


def workspace_bytes(cfg):
    lib = load_library()
    out = ctypes.c_size_t(0)
    st = lib.deer_workspace_bytes(ctypes.byref(cfg), ctypes.byref(out))
    if st != DEER_OK:
        raise DeerError(st, lib.deer_last_error(None).decode())
    return int(out.value)


class DeerContext:
    """One deer_ctx plus the torch tensor that backs its workspace."""

    def __init__(self, cfg, device="cuda:0", stream=None):
        self.lib = load_library()
        self.cfg = cfg
        self.device = torch.device(device)
        self.torch_dtype = torch.float32 if cfg.dtype == DEER_F32 else torch.float64
        nbytes = workspace_bytes(cfg)
        self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
        base = self.workspace.data_ptr()
        self._ws_ptr = (base + 255) // 256 * 256
        self.stream = stream if stream is not None else torch.cuda.current_stream(self.device)
        handle = ctypes.c_void_p(None)
        st = self.lib.deer_create(ctypes.byref(cfg), ctypes.c_void_p(self._ws_ptr), nbytes,
                                  ctypes.c_void_p(self.stream.cuda_stream), ctypes.byref(handle))
        if st != DEER_OK:
            raise DeerError(st, self.lib.deer_last_error(None).decode())
        self.handle = handle

    def _check(self, st, allow=()):
        if st != DEER_OK and st not in allow:
            raise DeerError(st, self.lib.deer_last_error(self.handle).decode())
        return st

    def _tensor(self, t, shape=None):
        if t is None:
            return None
        assert t.is_cuda and t.dtype == self.torch_dtype and t.is_contiguous(), "need a contiguous device tensor"
        if shape is not None:
            assert tuple(t.shape) == tuple(shape), (tuple(t.shape), tuple(shape))
        return t

    def _shapes(self):
        """(trajectory, inputs, initial state) shapes: with heads, arrays carry a head axis in front of the channels"""
        c = self.cfg
        if c.cell == DEER_CELL_GRU and (c.heads > 1 or c.stride_levels > 1):
            H = max(1, c.heads)
            return (c.B, c.T, H, c.n), (c.B, c.T, H, c.d), (c.B, H, c.n)
        if c.cell in (DEER_CELL_LSTM, DEER_CELL_LEM):   # n units, state (h | c) or (y | z)
            return (c.B, c.T, 2 * c.n), (c.B, c.T, c.d), (c.B, 2 * c.n)
        return (c.B, c.T, c.n), (c.B, c.T, c.d), (c.B, c.n)

    def eval(self, theta, x, y0, y_guess=None, tol=1e-4, max_iter=100, out=None, allow_nonfinite=False):
        """deer_eval.  Returns (y, iters, final_err, converged, status)."""
        c = self.cfg
        ys, xs, y0s = self._shapes()
        y = out if out is not None else torch.empty(ys, dtype=self.torch_dtype, device=self.device)
        assert theta.numel() == theta_count(c)
        self._tensor(theta)
        if c.cell != DEER_CELL_MLP_ODE:
            self._tensor(x, xs)
        self._tensor(y0, y0s)
        self._tensor(y_guess, ys)
        self._tensor(y, ys)
        iters, conv, err = ctypes.c_int32(0), ctypes.c_int32(0), ctypes.c_double(0.0)
        st = self.lib.deer_eval(self.handle, _ptr(theta), _ptr(x), _ptr(y0), _ptr(y_guess), float(tol),
                                int(max_iter), _ptr(y), ctypes.byref(iters), ctypes.byref(err), ctypes.byref(conv))
        self._check(st, allow=(DEER_ERR_NONFINITE,) if allow_nonfinite else ())
        return y, int(iters.value), float(err.value), bool(conv.value), st

    def grad(self, theta, x, y0, y, dLdy, want_dx=True, want_dy0=True):
        """deer_grad.  Returns (dL/dtheta, dL/dx or None, dL/dy0 or None)."""
        c = self.cfg
        ode = c.cell == DEER_CELL_MLP_ODE   # autonomous field: no inputs, hence no dL/dx; x and y0 may be None
        for t in (theta, x, y0, y, dLdy):
            self._tensor(t)
        ys, xs, y0s = self._shapes()
        dtheta = torch.empty(theta_count(c), dtype=self.torch_dtype, device=self.device)
        dx = torch.empty(xs, dtype=self.torch_dtype, device=self.device) if (want_dx and not ode) else None
        dy0 = torch.empty(y0s, dtype=self.torch_dtype, device=self.device) if want_dy0 else None
        st = self.lib.deer_grad(self.handle, _ptr(theta), _ptr(x), _ptr(y0), _ptr(y), _ptr(dLdy), _ptr(dx),
                                _ptr(dtheta), _ptr(dy0))
        self._check(st)
        return dtheta, dx, dy0

    def linrec_solve(self, A, b, y0=None, reverse=False, out=None):
        c = self.cfg
        self._tensor(A, (c.B, c.T, c.n, c.n))
        self._tensor(b, (c.B, c.T, c.n))
        self._tensor(y0, (c.B, c.n))
        y = out if out is not None else torch.empty((c.B, c.T, c.n), dtype=self.torch_dtype, device=self.device)
        st = self.lib.deer_linrec_solve(self.handle, _ptr(A), _ptr(b), _ptr(y0), _ptr(y), 1 if reverse else 0)
        self._check(st)
        return y

    def set_profiling(self, on):
        self._check(self.lib.deer_set_profiling(self.handle, 1 if on else 0))

    def profile(self):
        p = DeerProfile()
        self._check(self.lib.deer_get_profile(self.handle, ctypes.byref(p)))
        return {k: getattr(p, k) for k, _ in DeerProfile._fields_}

    def close(self):
        if getattr(self, "handle", None):
            self.lib.deer_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def linrec_solve_static(A, b, y0=None, reverse=False, out=None, status=None, stream=None):
    """deer_linrec_solve_static: the scan alone without a context or workspace (nothing is allocated by the
    library).  A [B,T,n,n], b [B,T,n], y0 [B,n] or None; `out` and the int32 device tensor `status` are the
    caller's.  Asynchronous on `stream` (default: torch's current stream).  Returns out."""
    lib = load_library()
    assert A.is_cuda and A.is_contiguous() and b.is_contiguous() and A.dtype == b.dtype
    B, T, n, _ = A.shape
    assert tuple(b.shape) == (B, T, n) and (y0 is None or tuple(y0.shape) == (B, n))
    dtype = DEER_F32 if A.dtype == torch.float32 else DEER_F64
    y = out if out is not None else torch.empty((B, T, n), dtype=A.dtype, device=A.device)
    stream = stream if stream is not None else torch.cuda.current_stream(A.device)
    st = lib.deer_linrec_solve_static(dtype, B, T, n, _ptr(A), _ptr(b), _ptr(y0), _ptr(y), 1 if reverse else 0,
                                      ctypes.c_void_p(stream.cuda_stream), _ptr(status))
    if st != DEER_OK:
        raise DeerError(st, lib.deer_last_error(None).decode())
    return y


# ---------------------------------------------------------------------------------------------------------------------
# Sequence operators.  Every call is asynchronous on `stream` (default: torch's current stream of the tensors' device); outputs
# and workspaces come from torch's allocator on that stream, a workspace for every call, so calls on several
# streams, in several threads and captured into several graphs do not meet in one.  Rows that belong to no sequence (behind `lengths`,
# outside `offsets`) or that a step passes over are zero in arrays that the call makes and left as they are in arrays that are handed in.
# No call records anything for torch.autograd: results of inputs that require gradients do not, and the gradient is the call of that name.
# ---------------------------------------------------------------------------------------------------------------------
_DTYPES = {torch.float32: DEER_F32, torch.float64: DEER_F64, torch.bfloat16: DEER_BF16, torch.float16: DEER_F16}


def _refuse(text):
    raise DeerError(DEER_ERR_INVALID_ARG, text)


def _raise(lib, st):
    raise DeerError(st, lib.deer_last_error(None).decode())


def _on_stream(f):
    """Runs f with the device of its first argument current, and with its keyword `stream` as that device's current stream.  Where that is
    another stream than the caller's, tensors that go in and come out are marked as used on both, so that neither's allocations take
    their memory early; waiting for what the other stream has to do is left to the caller."""
    name = f.__code__.co_varnames[0]

    @functools.wraps(f)
    def call(*args, stream=None, **kw):
        first = args[0] if args else kw.get(name)
        if not isinstance(first, torch.Tensor) or not first.is_cuda:
            _refuse("need device tensors")
        if stream is not None:
            if stream.device != first.device:
                _refuse("the stream belongs to another device than the tensors")
            here = torch.cuda.current_stream(first.device)
            with torch.cuda.stream(stream):
                result = f(*args, **kw)
            if stream != here:
                for t in args + tuple(kw.values()):
                    if isinstance(t, torch.Tensor) and t.is_cuda:
                        t.record_stream(stream)
                for t in result if isinstance(result, tuple) else (result,):
                    t.record_stream(here)
            return result
        if first.device.index == torch.cuda.current_device():
            return f(*args, **kw)
        with torch.cuda.device(first.device):
            return f(*args, **kw)
    return call


_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)   # (a step's call is as long as its kernel; this saves a tenth of it)


def _stream_of(device):
    return _raw_stream(device.index) if _raw_stream is not None else torch.cuda.current_stream(device).cuda_stream


def _int32(*sizes):
    for n in sizes:
        if n > 0x7FFFFFFF:
            _refuse("sequences, channels and slots are counted in 32 bits")


def _draw_of(seed, draw):
    """number of the draw and seed as the library takes them, in 32 and 64 bits"""
    seed, draw = operator.index(seed), operator.index(draw)
    if not 0 <= draw < 1 << 32:
        _refuse("draw: must lie in 0 .. 2^32 - 1")
    if not -(1 << 63) <= seed < 1 << 64:
        _refuse("seed: must be a number of 64 bits")
    return draw, seed & 0xFFFFFFFFFFFFFFFF


def _row_stride(t, what, lead):
    """Elements from a row of t to the next: `lead` leading dimensions that lie like rows one behind another, the dimensions behind them dense."""
    shape = t.shape
    inner = 1
    for n in shape[lead:]:
        inner *= n
    if t.is_contiguous():
        return inner
    strides, dense = t.stride(), 1
    for k in range(len(shape) - 1, lead - 1, -1):
        if shape[k] > 1 and strides[k] != dense:
            _refuse(what + ": the dimensions behind the rows must be dense")
        dense *= shape[k]
    if lead == 2 and shape[0] > 1 and shape[1] > 1 and strides[0] != shape[1] * strides[1]:
        _refuse(what + ": sequences must lie one behind another")
    first = strides[1] if lead == 2 and shape[1] > 1 else strides[0]
    if t.numel() == 0 or (shape[0] if lead == 1 else shape[0] * shape[1]) <= 1:
        return inner
    if first < inner:
        _refuse(what + ": rows must not overlap")
    return first


def _check_like(t, what, shape, dtype, device):
    if not isinstance(t, torch.Tensor) or t.device != device:
        _refuse(what + ": need a tensor on the same device")
    if t.dtype is not dtype:
        _refuse("%s: need %s, got %s" % (what, dtype, t.dtype))
    if t.shape != shape:
        _refuse("%s: need shape %s, got %s" % (what, tuple(shape), tuple(t.shape)))


def _dense(t, what, shape, dtype, device):
    """pointer of a contiguous tensor, or of none"""
    if t is None:
        return 0
    _check_like(t, what, shape, dtype, device)
    if not t.is_contiguous():
        _refuse(what + ": must be contiguous")
    return t.data_ptr()


def _rows_of(x, inner, offsets, lengths):
    """(N, T, packed, pointer of the bounds, leading dimensions) of x [N, T, ...] with optional `lengths` int64 [N], or of packed
    rows [rows, ...] with `offsets` int64 [N + 1]"""
    shape = x.shape
    if offsets is not None:
        if lengths is not None:
            _refuse("offsets (packed rows) and lengths (a padded batch) exclude each other")
        if len(shape) != 1 + inner:
            _refuse("packed rows have no dimension for the sequences")
        if not isinstance(offsets, torch.Tensor) or offsets.dim() != 1 or offsets.shape[0] < 2:
            _refuse("offsets: need [N + 1], N >= 1")
        return offsets.shape[0] - 1, shape[0], 1, _dense(offsets, "offsets", offsets.shape, torch.int64, x.device), 1
    if len(shape) != 2 + inner:
        _refuse("need [N, T, ...], or [rows, ...] with offsets")
    return shape[0], shape[1], 0, _dense(lengths, "lengths", shape[:1], torch.int64, x.device), 2


def _rows_like(t, stride):
    """an array of t's shape whose rows lie `stride` elements apart, as slices of a wider one do"""
    strides = [1] * t.dim()
    for k in range(t.dim() - 2, -1, -1):
        strides[k] = stride if k == t.dim() - 2 else strides[k + 1] * t.shape[k + 1]
    return torch.empty_strided(t.shape, strides, dtype=t.dtype, device=t.device)


def _zero_rest(bounds, *made):
    """Flag for the kernels to zero rows of no sequence, where every output of rows is the call's own; where some are the caller's, the call's own are
    zeroed here.  made: arrays that the call has made, None for the caller's"""
    if not bounds:
        return 0
    own = [t for t in made if t is not None]
    if len(own) == len(made):
        return DEER_REST_ZERO
    for t in own:
        t.zero_()
    return 0


@functools.lru_cache(maxsize=512)
def _diag_workspace(grad, dtype, N, D, T, packed):
    lib, size = load_library(), ctypes.c_size_t(0)
    cfg = DiagrecConfig(dtype, DEER_GATE_FACTOR, N, D, T, packed, 0, 0, 0, 0, 0.0, 0)   # (of every gate)
    st = lib.deer_diagrec_workspace_bytes(ctypes.byref(cfg), grad, ctypes.byref(size))
    if st != DEER_OK:
        _raise(lib, st)
    return size.value


def _diag_inputs(gate, x, kind, offsets, lengths):
    """(dtype, kind, N, D, T, packed, bounds, leading dimensions) of a diagonal recurrence's arrays"""
    if not isinstance(x, torch.Tensor):
        _refuse("need device tensors")
    dtype = _DTYPES.get(x.dtype)
    if dtype is None:
        _refuse("need float32, float64, bfloat16 or float16")
    _check_like(x, "x", gate.shape, gate.dtype, gate.device)
    N, T, packed, bounds, lead = _rows_of(x, 1, offsets, lengths)
    _int32(N, x.shape[-1])
    return dtype, int(kind), N, x.shape[-1], T, packed, bounds, lead


@_on_stream
def diagrec_solve(gate, x, h0=None, *, kind=DEER_GATE_FACTOR, offsets=None, lengths=None, drop=0.0, seed=0, draw=0, out=None):
    """deer_diagrec_solve: h_t = a_t h_{t-1} + u_t for every channel (a, u from gate and x: see deer_gate).  gate, x [N, T, D] with
    optional int64 `lengths` [N], or packed [rows, D] with int64 `offsets` [N + 1]; rows may be slices of wider ones.  h0 [N, D] in
    float32 (float64 with float64).  Rows of no sequence are zero in the result, left as they are in `out`.  Returns (h, state behind the last rows);
    torch.autograd does not see the call, diagrec_grad is its gradient."""
    lib = load_library()
    dtype, kind, N, D, T, packed, bounds, lead = _diag_inputs(gate, x, kind, offsets, lengths)
    dev, w = x.device, torch.float64 if dtype == DEER_F64 else torch.float32
    if out is None:
        h = torch.empty_like(x, memory_format=torch.contiguous_format)
    else:
        h = out
        _check_like(h, "out", x.shape, x.dtype, dev)
    rest = _zero_rest(bounds, h if out is None else None)
    draw, seed = _draw_of(seed, draw)
    cfg = DiagrecConfig(dtype, kind, N, D, T, packed | rest, draw, _row_stride(gate, "gate", lead), _row_stride(x, "x", lead),
                        _row_stride(h, "out", lead), drop, seed)
    last = torch.empty((N, D), dtype=w, device=dev)
    h0p = _dense(h0, "h0", last.shape, w, dev)
    size = _diag_workspace(0, dtype, N, D, T, packed)
    ws = x.new_empty(size, dtype=torch.uint8)   # (torch's blocks are aligned to 512 bytes)
    st = lib.deer_diagrec_solve(ctypes.byref(cfg), gate.data_ptr(), x.data_ptr(), h0p, bounds, h.data_ptr(), last.data_ptr(), ws.data_ptr(), size,
                                _stream_of(dev))
    if st != DEER_OK:
        _raise(lib, st)
    return h, last


@_on_stream
def diagrec_grad(gate, x, h, dh, h0=None, dlast=None, *, kind=DEER_GATE_FACTOR, offsets=None, lengths=None, drop=0.0, seed=0, draw=0,
                 dgate=None, dx=None):
    """deer_diagrec_grad at the trajectory h: (dL/dgate, dL/dx, dL/dh0) from dh = dL/dh and dlast = dL/d(final state).  dgate and dx, where
    given, have the row strides of gate and x, and their rows of no sequence are left as they are; otherwise these are zero."""
    lib = load_library()
    dtype, kind, N, D, T, packed, bounds, lead = _diag_inputs(gate, x, kind, offsets, lengths)
    dev, w = x.device, torch.float64 if dtype == DEER_F64 else torch.float32
    _check_like(h, "h", x.shape, x.dtype, dev)
    _check_like(dh, "dh", x.shape, x.dtype, dev)
    stride_h = _row_stride(h, "h", lead)
    if _row_stride(dh, "dh", lead) != stride_h:
        h, dh, stride_h = h.contiguous(), dh.contiguous(), D
    stride_g, stride_x = _row_stride(gate, "gate", lead), _row_stride(x, "x", lead)
    given = (dgate is not None, dx is not None)
    if dgate is None:
        dgate = torch.empty_like(gate, memory_format=torch.contiguous_format) if stride_g == D else _rows_like(gate, stride_g)
    else:
        _check_like(dgate, "dgate", x.shape, x.dtype, dev)
        if _row_stride(dgate, "dgate", lead) != stride_g:
            _refuse("dgate: rows must lie like those of gate")
    if dx is None:
        dx = torch.empty_like(x, memory_format=torch.contiguous_format) if stride_x == D else _rows_like(x, stride_x)
    else:
        _check_like(dx, "dx", x.shape, x.dtype, dev)
        if _row_stride(dx, "dx", lead) != stride_x:
            _refuse("dx: rows must lie like those of x")
    draw, seed = _draw_of(seed, draw)
    rest = _zero_rest(bounds, *(None if g else t for g, t in zip(given, (dgate, dx))))
    cfg = DiagrecConfig(dtype, kind, N, D, T, packed | rest, draw, stride_g, stride_x, stride_h, drop, seed)
    dh0 = torch.empty((N, D), dtype=w, device=dev)
    h0p, dlp = _dense(h0, "h0", dh0.shape, w, dev), _dense(dlast, "dlast", dh0.shape, w, dev)
    size = _diag_workspace(1, dtype, N, D, T, packed)
    ws = x.new_empty(size, dtype=torch.uint8)
    st = lib.deer_diagrec_grad(ctypes.byref(cfg), gate.data_ptr(), x.data_ptr(), h0p, bounds, h.data_ptr(), dh.data_ptr(), dlp, dgate.data_ptr(),
                               dx.data_ptr(), dh0.data_ptr(), ws.data_ptr(), size, _stream_of(dev))
    if st != DEER_OK:
        _raise(lib, st)
    return dgate, dx, dh0


@_on_stream
def diagrec_step(gate, x, state, *, kind=DEER_GATE_FACTOR, slots=None, out=None):
    """deer_diagrec_step: one token for each of N rows, gate and x [N, D]; `state` [slots, D] (float32; float64 with float64) is updated
    in place, row n at slots[n] (int32 [N]; None: n).  Rows whose slot is out of range or has come before are passed over: zero in
    the result, left as they are in `out`.  Returns h [N, D]."""
    lib = load_library()
    dtype = _DTYPES.get(x.dtype) if isinstance(x, torch.Tensor) else None
    if dtype is None or x.dim() != 2:
        _refuse("need x [N, D] in float32, float64, bfloat16 or float16")
    dev, shape = x.device, x.shape
    _check_like(gate, "gate", shape, x.dtype, dev)
    if out is None:
        h = torch.empty_like(x, memory_format=torch.contiguous_format)
    else:
        h = out
        _check_like(h, "out", shape, x.dtype, dev)
    if not isinstance(state, torch.Tensor) or state.dim() != 2 or state.shape[1] != shape[1]:
        _refuse("state: need [slots, D]")
    sp = _dense(state, "state", state.shape, torch.float64 if dtype == DEER_F64 else torch.float32, dev)
    tp = _dense(slots, "slots", shape[:1], torch.int32, dev)
    _int32(shape[0], shape[1], state.shape[0])
    cfg = DiagrecConfig(dtype, int(kind), shape[0], shape[1], 1, DEER_REST_ZERO if out is None else 0, 0, _row_stride(gate, "gate", 1), _row_stride(x, "x", 1),
                        _row_stride(h, "out", 1), 0.0, 0)
    st = lib.deer_diagrec_step(ctypes.byref(cfg), gate.data_ptr(), x.data_ptr(), tp, state.shape[0], sp, h.data_ptr(), _stream_of(dev))
    if st != DEER_OK:
        _raise(lib, st)
    return h


@functools.lru_cache(maxsize=512)
def _mat_workspace(grad, dtype, N, T, packed, Hk, Hv, Dk, Dv):
    lib, size = load_library(), ctypes.c_size_t(0)
    cfg = MatrecConfig(dtype, N, T, packed, Hk, Hv, Dk, Dv, 0, 1.0, 0, 0, 0, 0)
    st = lib.deer_matrec_workspace_bytes(ctypes.byref(cfg), grad, ctypes.byref(size))
    if st != DEER_OK:
        _raise(lib, st)
    return size.value


def _mat_config(q, k, v, gate, o, offsets, lengths, scale, lead=None):
    """configuration, pointers of the bounds and of the gates, leading dimensions; lead: given for a step, whose rows are not sequences"""
    for t in (k, v, gate):
        if not isinstance(t, torch.Tensor):
            _refuse("need device tensors")
    dtype = _DTYPES.get(q.dtype)
    if dtype is None:
        _refuse("need float32 or bfloat16")
    if lead is None:
        N, T, packed, bounds, lead = _rows_of(q, 2, offsets, lengths)
    else:
        if q.dim() != 3:
            _refuse("need q [N, Hk, Dk]")
        N, T, packed, bounds = q.shape[0], 1, 0, 0
    dev, rows = q.device, q.shape[:lead]
    Hk, Dk = q.shape[lead:]
    _check_like(k, "k", q.shape, q.dtype, dev)
    if v.dim() != q.dim():
        _refuse("v: need as many dimensions as q")
    Hv, Dv = v.shape[lead:]
    _int32(N, Hk, Hv, Dk, Dv)
    _check_like(v, "v", rows + v.shape[lead:], q.dtype, dev)
    if Hk < 1 or Hv % Hk:
        _refuse("the heads of v must be a multiple of those of q and k")
    gp = _dense(gate, "gate", rows + v.shape[lead:lead + 1], torch.float32, dev)
    if o is not None:
        _check_like(o, "out", v.shape, v.dtype, dev)
    cfg = MatrecConfig(dtype, N, T, packed, Hk, Hv, Dk, Dv, 0, Dk ** -0.5 if scale is None else scale, _row_stride(q, "q", lead),
                       _row_stride(k, "k", lead), _row_stride(v, "v", lead), _row_stride(o, "out", lead) if o is not None else Hv * Dv)
    return cfg, bounds, gp, lead


@_on_stream
def matrec_solve(q, k, v, gate, s0=None, *, offsets=None, lengths=None, scale=None, out=None):
    """deer_matrec_solve: S_t = exp(gate_t) S_{t-1} + k_t v_t^T, o_t = scale S_t^T q_t for every head of v.  q, k [N, T, Hk, Dk], v [N, T, Hv, Dv] in
    float32 or bfloat16, gate [N, T, Hv] float32, with optional int64 `lengths` [N]; or packed [rows, ...] with int64 `offsets` [N + 1].  s0 [N, Hv, Dk, Dv]
    float32.  scale: Dk^-1/2 by default.  Rows of no sequence are zero in the result, left as they are in `out`.  Returns (o, states behind the last rows);
    torch.autograd does not see the call, matrec_grad is its gradient."""
    lib = load_library()
    o = out if out is not None else torch.empty_like(v, memory_format=torch.contiguous_format) if isinstance(v, torch.Tensor) else None
    cfg, bounds, gp, _ = _mat_config(q, k, v, gate, o, offsets, lengths, scale)
    dev, shape = q.device, (cfg.N, cfg.Hv, cfg.Dk, cfg.Dv)
    s0p = _dense(s0, "s0", shape, torch.float32, dev)
    size = _mat_workspace(0, cfg.dtype, cfg.N, cfg.T, cfg.packed, cfg.Hk, cfg.Hv, cfg.Dk, cfg.Dv)
    ws = q.new_empty(size, dtype=torch.uint8)
    last = torch.empty(shape, dtype=torch.float32, device=dev)
    cfg.packed |= _zero_rest(bounds, o if out is None else None)
    st = lib.deer_matrec_solve(ctypes.byref(cfg), q.data_ptr(), k.data_ptr(), v.data_ptr(), gp, s0p, bounds, o.data_ptr(), last.data_ptr(),
                               ws.data_ptr(), size, _stream_of(dev))
    if st != DEER_OK:
        _raise(lib, st)
    return o, last


@_on_stream
def matrec_grad(q, k, v, gate, do, s0=None, dlast=None, *, offsets=None, lengths=None, scale=None, dq=None, dk=None, dv=None, dgate=None):
    """deer_matrec_grad: (dq, dk, dv, dgate, ds0) from do = dL/do and dlast = dL/d(final states).  dq, dk and dv, where given, have the row
    strides of q, k and v, dgate is dense; their rows of no sequence are left as they are, and are zero in arrays that are not given."""
    lib = load_library()
    cfg, bounds, gp, lead = _mat_config(q, k, v, gate, do, offsets, lengths, scale)
    dev = q.device
    outs, made = [], []
    for t, given, name, stride in ((q, dq, "dq", cfg.stride_q), (k, dk, "dk", cfg.stride_k), (v, dv, "dv", cfg.stride_v)):
        d = given
        if d is None:
            d = torch.empty(t.shape, dtype=t.dtype, device=dev) if t.is_contiguous() else _rows_like(t.flatten(-2), stride).unflatten(-1, t.shape[-2:])
        else:
            _check_like(d, name, t.shape, t.dtype, dev)
            if _row_stride(d, name, lead) != stride:
                _refuse(name + ": rows must lie like those of what it is the gradient of")
        outs.append(d)
        made.append(d if given is None else None)
    shape = (cfg.N, cfg.Hv, cfg.Dk, cfg.Dv)
    s0p, dlp = _dense(s0, "s0", shape, torch.float32, dev), _dense(dlast, "dlast", shape, torch.float32, dev)
    size = _mat_workspace(1, cfg.dtype, cfg.N, cfg.T, cfg.packed, cfg.Hk, cfg.Hv, cfg.Dk, cfg.Dv)
    ws = q.new_empty(size, dtype=torch.uint8)
    if dgate is None:
        dgate = torch.empty(gate.shape, dtype=torch.float32, device=dev)
        made.append(dgate)
    else:
        _dense(dgate, "dgate", gate.shape, torch.float32, dev)
        made.append(None)
    cfg.packed |= _zero_rest(bounds, *made)
    ds0 = torch.empty(shape, dtype=torch.float32, device=dev)
    st = lib.deer_matrec_grad(ctypes.byref(cfg), q.data_ptr(), k.data_ptr(), v.data_ptr(), gp, s0p, bounds, do.data_ptr(), dlp, outs[0].data_ptr(),
                              outs[1].data_ptr(), outs[2].data_ptr(), dgate.data_ptr(), ds0.data_ptr(), ws.data_ptr(), size, _stream_of(dev))
    if st != DEER_OK:
        _raise(lib, st)
    return outs[0], outs[1], outs[2], dgate, ds0


@_on_stream
def matrec_step(q, k, v, gate, state, *, slots=None, scale=None, out=None):
    """deer_matrec_step: one token for each of N rows, q, k [N, Hk, Dk], v [N, Hv, Dv], gate [N, Hv]; `state` [slots, Hv, Dk, Dv] float32 is updated
    in place, row n at slots[n] (int32 [N]; None: n).  Rows whose slot is out of range or has come before are passed over: zero in
    the result, left as they are in `out`.  Returns o."""
    lib = load_library()
    o = out if out is not None else torch.empty_like(v, memory_format=torch.contiguous_format) if isinstance(v, torch.Tensor) else None
    cfg, _, gp, _ = _mat_config(q, k, v, gate, o, None, None, scale, lead=1)
    dev = q.device
    if not isinstance(state, torch.Tensor) or state.dim() != 4:
        _refuse("state: need [slots, Hv, Dk, Dv]")
    sp = _dense(state, "state", (state.shape[0], cfg.Hv, cfg.Dk, cfg.Dv), torch.float32, dev)
    tp = _dense(slots, "slots", q.shape[:1], torch.int32, dev)
    _int32(state.shape[0])
    cfg.packed = DEER_REST_ZERO if out is None else 0
    st = lib.deer_matrec_step(ctypes.byref(cfg), q.data_ptr(), k.data_ptr(), v.data_ptr(), gp, tp, state.shape[0], sp, o.data_ptr(), _stream_of(dev))
    if st != DEER_OK:
        _raise(lib, st)
    return o


@_on_stream
def dropout(x, p, seed, draw=0, *, out=None):
    """deer_dropout: x [N, T, D] or packed [rows, D] with a share p dropped and the rest divided by 1 - p; the backward pass is the same
    call on the gradient (torch.autograd does not see it).  `out` may be x."""
    lib = load_library()
    dtype, lead, dev = _DTYPES.get(x.dtype), x.dim() - 1, x.device
    if dtype is None or lead not in (1, 2):
        _refuse("need x [N, T, D] or [rows, D] in float32, float64, bfloat16 or float16")
    if out is None:
        y = torch.empty_like(x, memory_format=torch.contiguous_format)
    else:
        y = out
        _check_like(y, "out", x.shape, x.dtype, dev)
    draw, seed = _draw_of(seed, draw)
    N, T, D = x.shape if lead == 2 else (1,) + tuple(x.shape)
    _int32(N, D)
    st = lib.deer_dropout(dtype, N, T, D, x.data_ptr(), _row_stride(x, "x", lead), y.data_ptr(), _row_stride(y, "out", lead), p,
                          seed, draw, _stream_of(dev))
    if st != DEER_OK:
        _raise(lib, st)
    return y


def context_for(workload, dtype=DEER_F32, device="cuda:0"):
    """Context for an ``inputs.Workload``."""
    cfg = make_config(workload.cell, dtype, workload.B, workload.T, workload.n, workload.d, workload.mlp_width,
                      workload.mlp_hidden_layers, workload.t0, workload.t1, workload.mlp_activation,
                      workload.heads, workload.stride_levels)
    return DeerContext(cfg, device=device)
