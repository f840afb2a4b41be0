"""Operators of layers with selective states that are timed: the short causal convolution in front of the states, the selective scan
itself, and the group norm behind heads and channels.

A case is a dict: `op` (conv, scan, norm), `run` (forward, train = forward and then the gradient, step = one token for every sequence), the data
type and the sizes.  `lengths`: the sequences' lengths, packed one behind the other (in its absence N sequences of T rows).
With `own` false the same is computed by elementary torch operations.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f64": torch.float64, "bf16": torch.bfloat16, "f16": torch.float16}


def _case(name, op, run, dtype, **sizes):
    c = {"op": op, "run": run, "dtype": dtype, "N": 1, "T": 1, "lengths": "", "D": 0, "W": 0, "S": 0, "G": 1, "gated": False, "silu": False, "rows": True}
    c.update(sizes)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # decoding: one token for each of 32 sequences, their last inputs in a pool of slots; all latency
        _case("conv_step_bf16", "conv", "step", "bf16", N=32, D=2048, W=4, silu=True),
        # training on packed documents of different lengths; one of them is empty, one a single token
        _case("conv_train_packed_bf16", "conv", "train", "bf16", lengths="4096,1,7001,0,513,2047,11111,3999,4000", D=2560, W=4, silu=True),
        # single precision at odd sizes, forward only
        _case("conv_ragged_f32", "conv", "forward", "f32", N=3, T=5003, D=1030, W=3),
        # decoding with selective states: 64 sequences
        _case("scan_step_bf16", "scan", "step", "bf16", N=64, D=4096, S=16, gated=True),
        # a packed batch of prompts
        _case("scan_prompts_bf16", "scan", "forward", "bf16", lengths="1021,2048,1,3500,129,64,1429", D=4096, S=16, gated=True),
        # one very long prompt: the length has to be split
        _case("scan_long_f16", "scan", "forward", "f16", N=1, T=32768, D=2048, S=16, gated=True),
        # a training step on ordinary sequences
        _case("scan_train_bf16", "scan", "train", "bf16", N=4, T=4096, D=4096, S=16, gated=True),
        # training in single precision at odd sizes, two groups of channels, more states than usual
        _case("scan_train_ragged_f32", "scan", "train", "f32", N=3, T=777, D=330, S=24, G=2),
        # decoding: the norm of the heads' outputs, with its gate, of 32 tokens
        _case("norm_token_bf16", "norm", "forward", "bf16", N=32, T=1, D=2048, G=16, gated=True),
        # the same in a training step on ordinary sequences, 16 heads of 128 channels
        _case("norm_heads_train_bf16", "norm", "train", "bf16", N=4, T=4096, D=2048, G=16, gated=True),
        # statistics over whole trajectories at the length of the EigenWorms recordings, channels last
        _case("norm_trajectories_train_f32", "norm", "train", "f32", N=32, T=17984, D=16, G=4, silu=True, rows=False),
        # the same over packed documents with many channels, forward only
        _case("norm_documents_bf16", "norm", "forward", "bf16", lengths="4096,1,7001,0,513,2047,11111,3999,4000", D=2560, G=32, silu=True, rows=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _lengths(rng, total):
    """`total` rows cut at random places into a few sequences"""
    cuts = sorted(rng.randint(0, total) for _ in range(rng.randint(1, 9)))
    return ",".join(str(b - a) for a, b in zip([0] + cuts, cuts + [total]))


def _shape(rng, rows, packed):
    if packed:
        return {"lengths": _lengths(rng, rows)}
    N = _log(rng, 1, min(64, rows))
    return {"N": N, "T": max(1, rows // N)}


def draw(rng):
    op = rng.choice(["conv", "scan", "scan", "norm"])
    run = rng.choice(["forward", "train", "train", "step"])
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"] + (["f64"] if op != "scan" else []))
    packed = rng.random() < 0.5
    if op == "conv":
        D, W, silu = _log(rng, 1, 4096), rng.randint(2, 8), rng.random() < 0.7
        if run == "step":
            return _case("", op, run, dtype, N=_log(rng, 1, 256), D=D, W=W, silu=silu)
        rows = _log(rng, 16, max(16, min(65536, 60000000 // D)))
        return _case("", op, run, dtype, D=D, W=W, silu=silu, **_shape(rng, rows, packed))
    if op == "scan":
        S = rng.choice([16, 16, rng.randint(1, 64)])
        G = rng.choice([1, 1, 2, 4])
        D, gated = G * _log(rng, 1, 4096 // G), rng.random() < 0.6
        if run == "step":
            return _case("", op, run, dtype, N=_log(rng, 1, 128), D=D, S=S, G=G, gated=gated)
        rows = _log(rng, 16, max(16, min(32768, 300000000 // (D * S))))
        return _case("", op, run, dtype, D=D, S=S, G=G, gated=gated, **_shape(rng, rows, packed))
    G = _log(rng, 1, 64)
    D, over_rows = G * _log(rng, 8, 4096 // G), rng.random() < 0.5   # (two or three values are all but fixed by their norm: no gradient)
    rows = _log(rng, 16, max(16, min(65536, 60000000 // D)))
    return _case("", op, "forward" if run == "step" else run, dtype, D=D, G=G, gated=rng.random() < 0.5, silu=rng.random() < 0.5, rows=over_rows,
                 **_shape(rng, rows, packed))


def _sizes(c):
    """(lengths of the sequences, rows in all)"""
    lens = [int(x) for x in c["lengths"].split(",")] if c["lengths"] else [c["T"]] * c["N"]
    return lens, sum(lens)


def prepare(case, seed):
    c = dict(case)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    dtype = TYPES[c["dtype"]]
    wide = torch.float64 if c["dtype"] == "f64" else torch.float32
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV, dtype=wide)   # noqa: E731
    uniform = lambda *s: torch.rand(*s, generator=gen, device=DEV, dtype=wide)   # noqa: E731
    lens, rows = _sizes(c)
    N, D, step, packed = len(lens), c["D"], c["run"] == "step", bool(c["lengths"])
    lead = (rows,) if packed else (N,) if step else (N, c["T"])
    s = {"case": c, "wide": wide, "lens": lens, "offsets": None, "z": None}
    if packed:
        edges = np.concatenate([[0], np.cumsum(lens)])
        s["offsets"] = torch.from_numpy(edges.astype(np.int64)).to(DEV)
    if step:   # the states live in a pool with some slots more, in an order of their own
        s["slots"] = torch.randperm(N + 5, generator=gen, device=DEV)[:N].to(torch.int32)
    s["x"] = rand(*lead, D).to(dtype)
    if c["gated"]:
        s["z"] = rand(*lead, D).to(dtype)
    if c["run"] == "train":
        s["dy"] = rand(*lead, D).to(dtype)
    if c["op"] == "conv":
        s["w"], s["bias"] = rand(D, c["W"]) / c["W"] ** 0.5, 0.1 * rand(D)
        states = (c["W"] - 1, D)
    elif c["op"] == "scan":
        # memories from a few steps to a thousand, as such layers begin with: steps of 0.001 to 0.1, spread by the inputs; rates from 1 to S
        first = torch.exp(math.log(0.001) + uniform(D) * math.log(100.0))
        s["dt_bias"] = first + torch.log(-torch.expm1(-first))
        s["dt"] = (0.5 * rand(*lead, D)).to(dtype)
        s["A"] = -torch.arange(1, c["S"] + 1, device=DEV, dtype=wide) * torch.exp(0.1 * rand(D, c["S"]))
        s["B"], s["C"] = rand(*lead, c["G"], c["S"]).to(dtype), rand(*lead, c["G"], c["S"]).to(dtype)
        s["skip"] = 1.0 + 0.1 * rand(D)
        states = (D, c["S"])
    else:
        s["w"], s["bias"] = 1.0 + 0.1 * rand(D), 0.1 * rand(D)
        s["x"] = (s["x"].to(wide) + rand(D)).to(dtype)
        return s
    if step:
        s["state"] = rand(N + 5, *states)
    else:
        s["s0"] = rand(N, *states)
        if c["run"] == "train":
            s["dlast"] = rand(N, *states)
    return s


def run(state):
    op, direction = state["case"]["op"], state["case"]["run"]
    if own:
        return _own(state, op, direction)
    if op == "norm":
        return _plain_norm(state)
    if direction == "step":
        return _plain_conv_step(state) if op == "conv" else _plain_scan_step(state)
    return _plain_conv(state) if op == "conv" else _plain_scan(state)


# ---------------------------------------------------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------------------------------------------------
def _own(s, op, direction):
    from paper_2309_12252_amd import deer
    c = s["case"]
    act = deer.DEER_ACT_SILU if c["silu"] else deer.DEER_ACT_NONE
    if op == "conv":
        if direction == "step":
            return {"y": deer.shortconv_step(s["x"], s["w"], s["state"], s["bias"], act=act, slots=s["slots"]), "state": s["state"]}
        y, last = deer.shortconv_solve(s["x"], s["w"], s["bias"], s["s0"], act=act, offsets=s["offsets"])
        if direction == "forward":
            return {"y": y, "last": last}
        dx, dw, dbias, ds0 = deer.shortconv_grad(s["x"], s["w"], s["dy"], s["bias"], s["s0"], s["dlast"], act=act, offsets=s["offsets"])
        return {"y": y, "last": last, "dx": dx, "dw": dw, "dbias": dbias, "ds0": ds0}
    if op == "scan":
        about = {"skip": s["skip"], "z": s["z"], "dt_bias": s["dt_bias"]}
        if direction == "step":
            return {"y": deer.selscan_step(s["x"], s["dt"], s["A"], s["B"], s["C"], s["state"], slots=s["slots"], **about), "state": s["state"]}
        y, last = deer.selscan_solve(s["x"], s["dt"], s["A"], s["B"], s["C"], h0=s["s0"], offsets=s["offsets"], **about)
        if direction == "forward":
            return {"y": y, "last": last}
        dx, ddt, dA, dB, dC, dskip, dz, dbias, dh0 = deer.selscan_grad(s["x"], s["dt"], s["A"], s["B"], s["C"], s["dy"], h0=s["s0"], dlast=s["dlast"],
                                                                       offsets=s["offsets"], **about)
        return {"y": y, "last": last, "dx": dx, "ddt": ddt, "dA": dA, "dB": dB, "dC": dC, "dskip": dskip, "dz": dz, "dbias": dbias, "dh0": dh0}
    more = {"z": s["z"], "act": act, "span": deer.DEER_SPAN_ROW if c["rows"] else deer.DEER_SPAN_SEQUENCE, "offsets": s["offsets"]}
    y, stats = deer.groupnorm_solve(s["x"], c["G"], s["w"], s["bias"], **more)
    if direction == "forward":
        return {"y": y, "stats": stats}
    dx, dw, dbias, dz = deer.groupnorm_grad(s["x"], c["G"], stats, s["dy"], s["w"], s["bias"], **more)
    return {"y": y, "stats": stats, "dx": dx, "dw": dw, "dbias": dbias, "dz": dz}


# ---------------------------------------------------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------------------------------------------------
def _padded(s, T, t, fill=0.0):
    """[rows, ...] of packed sequences as [N, T, ...] in 32 or 64 bits"""
    t = t.to(s["wide"])
    if s["offsets"] is None:
        return t
    out = torch.full((len(s["lens"]), T) + t.shape[1:], fill, dtype=t.dtype, device=t.device)
    at, inside = _places(s, T)
    out[inside] = t[at[inside]]
    return out


def _places(s, T):
    """row of every place of the padded batch, and whether there is one"""
    first = s["offsets"][:-1, None] + torch.arange(T, device=DEV)[None, :]
    return first, first < s["offsets"][1:, None]


def _packed(s, T, t, dtype):
    return (t if s["offsets"] is None else t[_places(s, T)[1]]).to(dtype)


def _total(t, dims):
    """sums over many rows in 64 bits"""
    return t.sum(dims, dtype=torch.float64).to(t.dtype)


def _silu(v):
    """v sigmoid(v) and its derivative"""
    g = torch.sigmoid(v)
    return v * g, g * (1.0 + v * (1.0 - g))


def _softplus(v):
    return torch.clamp(v, min=0.0) + torch.log1p(torch.exp(-torch.abs(v)))


def _plain_conv(s):
    """y_t = act(bias + sum_j w_j x_{t - W + 1 + j}), in front of a sequence its initial rows"""
    c, T, W, dtype = s["case"], max(s["lens"]), s["case"]["W"], s["x"].dtype
    N, D = len(s["lens"]), c["D"]
    ends = torch.tensor(s["lens"], device=DEV)[:, None] + torch.arange(W - 1, device=DEV)[None, :]   # the last W - 1 rows of a sequence with its initial ones
    ends = ends[..., None].expand(N, W - 1, D)
    rows = torch.cat([s["s0"], _padded(s, T, s["x"])], 1)
    v = (rows.unfold(1, W, 1) * s["w"]).sum(-1) + s["bias"]
    act, slope = _silu(v) if c["silu"] else (v, torch.ones((), device=DEV, dtype=s["wide"]))
    got = {"y": _packed(s, T, act, dtype), "last": rows.gather(1, ends)}
    if c["run"] == "forward":
        return got
    dv = _padded(s, T, s["dy"]) * slope
    zero = dv.new_zeros(N, W - 1, D)
    drows = (torch.cat([zero, dv, zero], 1).unfold(1, W, 1) * s["w"].flip(1)).sum(-1)
    drows = drows.scatter_add(1, ends, s["dlast"])
    dw = _total(rows.unfold(1, W, 1) * dv[..., None], (0, 1))
    got.update(dx=_packed(s, T, drows[:, W - 1:], dtype), dw=dw, dbias=_total(dv, (0, 1)), ds0=drows[:, :W - 1].clone())
    return got


def _plain_conv_step(s):
    at, x, state = s["slots"].long(), s["x"], s["state"]
    rows = torch.cat([state[at], x.to(s["wide"])[:, None]], 1)
    v = (rows * s["w"].t()).sum(1) + s["bias"]
    state[at] = rows[:, 1:]
    return {"y": (_silu(v)[0] if s["case"]["silu"] else v).to(x.dtype), "state": state}


def _scan(a, u):
    """h_t = a_t h_{t-1} + u_t along dim 1 from zero by doubling, and the products of a up to t"""
    a, h, d, T = a.clone(), u, 1, a.shape[1]
    while d < T:
        h[:, d:] = h[:, d:] + a[:, d:] * h[:, :-d]
        a[:, d:] = a[:, d:] * a[:, :-d]
        d *= 2
    return h, a


def _plain_scan(s):
    """h_t = exp(dt_t A) h_{t-1} + dt_t x_t B_t for every channel and state, y_t = <C_t, h_t> + skip x_t, gated"""
    c, T, dtype, h0 = s["case"], max(s["lens"]), s["x"].dtype, s["s0"]
    N, D, G = len(s["lens"]), c["D"], c["G"]
    per = D // G
    channels = lambda t: t.repeat_interleave(per, 2)   # noqa: E731    [N, T, G, S] -> [N, T, D, S]
    groups = lambda t: t.reshape(t.shape[0], t.shape[1], G, per, t.shape[3]).sum(3)   # noqa: E731
    x, raw = _padded(s, T, s["x"]), s["dt"].to(s["wide"]) + s["dt_bias"]
    dt = _padded(s, T, _softplus(raw))   # rows behind a sequence's end keep its state: a step of zero
    B, C = channels(_padded(s, T, s["B"])), channels(_padded(s, T, s["C"]))
    a = torch.exp(dt[..., None] * s["A"])
    h, prod = _scan(a, (dt * x)[..., None] * B)
    h = h.addcmul_(prod, h0[:, None])
    del prod
    plain = (h * C).sum(-1) + s["skip"] * x
    gate, slope = _silu(_padded(s, T, s["z"])) if c["gated"] else (torch.ones((), device=DEV), None)
    got = {"y": _packed(s, T, plain * gate, dtype), "last": h[:, -1].clone()}
    if c["run"] == "forward":
        return got
    dy = _padded(s, T, s["dy"])
    if c["gated"]:
        got["dz"] = _packed(s, T, dy * plain * slope, dtype)
    dy = dy * gate
    got["dC"] = _packed(s, T, groups(dy[..., None] * h), dtype)
    # mu_t = a_t (C_t dy_t + mu_{t+1}) from mu_{T+1} = dlast, along the reversed rows
    read = dy[..., None] * C
    mu, prod = _scan(a.flip(1), (a * read).flip(1))
    mu = mu.addcmul_(prod, s["dlast"][:, None]).flip(1)
    del prod, C
    got["dh0"] = mu[:, 0].clone()
    lam = read + torch.cat([mu[:, 1:], s["dlast"][:, None]], 1)
    del read, mu
    g = lam * torch.cat([h0[:, None], h[:, :-1]], 1) * a   # dL/d(dt A)
    del a, h
    got["dB"] = _packed(s, T, groups(lam * (dt * x)[..., None]), dtype)
    read = (lam * B).sum(-1)
    ddt = ((g * s["A"]).sum(-1) + read * x) * _padded(s, T, torch.sigmoid(raw))
    got.update(dx=_packed(s, T, read * dt + s["skip"] * dy, dtype), ddt=_packed(s, T, ddt, dtype), dA=_total(g * dt[..., None], (0, 1)),
               dskip=_total(dy * x, (0, 1)), dbias=_total(ddt, (0, 1)))
    return got


def _plain_scan_step(s):
    c, at, state, wide = s["case"], s["slots"].long(), s["state"], s["wide"]
    x, per = s["x"].to(wide), c["D"] // c["G"]
    B, C = (s[n].to(wide).repeat_interleave(per, 1) for n in "BC")
    dt = _softplus(s["dt"].to(wide) + s["dt_bias"])
    h = torch.exp(dt[..., None] * s["A"]) * state[at] + (dt * x)[..., None] * B
    state[at] = h
    y = (h * C).sum(-1) + s["skip"] * x
    return {"y": (y * _silu(s["z"].to(wide))[0] if c["gated"] else y).to(s["x"].dtype), "state": state}


EPS = 1e-5


def _plain_norm(s):
    """y = act((x - mean) rstd w + bias) silu(z); mean and variance of a group's channels, over one row or all of a sequence's"""
    c, T, dtype, wide = s["case"], max(s["lens"]), s["x"].dtype, s["wide"]
    N, D, G = len(s["lens"]), c["D"], c["G"]
    grouped = lambda t: t.reshape(t.shape[0], t.shape[1], G, D // G)   # noqa: E731
    x, w = grouped(_padded(s, T, s["x"])), s["w"].reshape(G, D // G)
    count = torch.full((), D // G, device=DEV, dtype=torch.float64) if c["rows"] else torch.tensor(s["lens"], device=DEV).double()[:, None, None, None] * (D // G)
    dims = (3,) if c["rows"] else (1, 3)
    inside = torch.ones((), device=DEV, dtype=wide) if s["offsets"] is None else _places(s, T)[1][..., None, None].to(wide)

    def mean(t):   # over what a norm spans; zero where that is nothing
        return (t.sum(dims, keepdim=True, dtype=torch.float64) / count.clamp(min=1)).to(wide)

    mu = mean(x)
    off = (x - mu) * inside
    rstd = 1.0 / torch.sqrt(mean(off * off) + EPS) * (count > 0)
    rstd = rstd.to(wide)
    unit = off * rstd
    v = unit * w + s["bias"].reshape(G, D // G)
    act, slope = _silu(v) if c["silu"] else (v, torch.ones((), device=DEV, dtype=wide))
    flat = lambda t: t.reshape(N, T, D)   # noqa: E731
    gate, gslope = _silu(grouped(_padded(s, T, s["z"]))) if c["gated"] else (torch.ones((), device=DEV, dtype=wide), None)
    stats = torch.stack([mu, rstd], -1)
    stats = _packed(s, T, stats.reshape(N, T, G, 2), wide) if c["rows"] else stats.reshape(N, G, 2)
    got = {"y": _packed(s, T, flat(act * gate), dtype), "stats": stats}
    if c["run"] == "forward":
        return got
    dy = grouped(_padded(s, T, s["dy"]))
    if c["gated"]:
        got["dz"] = _packed(s, T, flat(dy * act * gslope), dtype)
    dv = dy * gate * slope
    du = dv * w
    dx = rstd * (du - mean(du) - unit * mean(du * unit))
    got.update(dx=_packed(s, T, flat(dx), dtype), dw=_total(dv * unit, (0, 1)).reshape(D), dbias=_total(dv, (0, 1)).reshape(D))
    return got


# ---------------------------------------------------------------------------------------------------------------------
def work(case):
    c = case
    lens, rows = _sizes(c)
    N, D = len(lens), c["D"]
    e, w = TYPES[c["dtype"]].itemsize, 8 if c["dtype"] == "f64" else 4
    rows = N if c["run"] == "step" else rows
    n, train = rows * D, c["run"] == "train"
    if c["op"] == "conv":   # x and y (and dy, dx), weights and bias (and their gradients), two sets of states (four)
        k = 2 if train else 1
        return {"bytes": k * (2 * e * n + w * D * (c["W"] + 1) + 2 * w * N * D * (c["W"] - 1)), "flops": (6 if train else 2) * n * c["W"] + 6 * n}
    arrays = 3 if c["gated"] else 2   # of rows and channels: x, y, and z where there is one
    if c["op"] == "scan":   # dt as well; B and C; A, skip and the bias of dt; two sets of states
        arrays = 2 * (arrays + 1) if train else arrays + 1   # with dy and the gradients of all but y
        k = 2 if train else 1
        return {"bytes": e * n * arrays + k * (2 * e * rows * c["G"] * c["S"] + w * D * (c["S"] + 2) + 2 * w * N * D * c["S"]),
                "flops": (24 if train else 7) * n * c["S"] + 20 * n}
    stats = 2 * w * c["G"] * (rows if c["rows"] else N)
    if train:   # x, y, dy, dx, and z and dz
        return {"bytes": e * n * (6 if c["gated"] else 4) + 4 * w * D + stats, "flops": 40 * n}
    return {"bytes": e * n * arrays + 2 * w * D + stats, "flops": 12 * n}


# ---------------------------------------------------------------------------------------------------------------------
# 64 bits: states row by row, the other operators sequence by sequence
# ---------------------------------------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    d = {k: t.double() for k, t in s.items() if torch.is_tensor(t) and t.is_floating_point()}
    if s["case"]["op"] == "norm":
        return _exact_norm(s, d)
    if s["case"]["run"] == "step":
        return _exact_conv_step(s, d) if s["case"]["op"] == "conv" else _exact_scan_step(s, d)
    return _exact_conv(s, d) if s["case"]["op"] == "conv" else _exact_scan(s, d)


def _by_sequence(s, t):
    """[N, T, ...] or packed rows as a list of sequences"""
    return list(t) if s["offsets"] is None else list(t.split(s["lens"]))


def _joined(s, ts):
    return torch.stack(ts) if s["offsets"] is None else torch.cat(ts)


def _exact_silu(v):
    return v / (1 + torch.exp(-v))


def _exact_conv(s, d):
    c, W = s["case"], s["case"]["W"]
    w, bias = d["w"].requires_grad_(), d["bias"].requires_grad_()
    xs, s0 = [x.detach().requires_grad_() for x in _by_sequence(s, d["x"])], [t.detach().requires_grad_() for t in d["s0"]]
    ys, lasts = [], []
    for x, front in zip(xs, s0):
        rows = torch.cat([front, x])
        L = x.shape[0]
        y = bias.expand(L, -1)
        for j in range(W):
            y = y + w[:, j] * rows[j:j + L]
        ys.append(_exact_silu(y) if c["silu"] else y)
        lasts.append(rows[L:])
    out = {"y": _joined(s, ys).detach(), "last": torch.stack(lasts).detach()}
    if c["run"] == "forward":
        return out
    got = torch.autograd.grad([_joined(s, ys), torch.stack(lasts)], [w, bias] + xs + s0, [d["dy"], d["dlast"]])
    n = len(xs)
    out.update(dw=got[0], dbias=got[1], dx=_joined(s, list(got[2:2 + n])), ds0=torch.stack(got[2 + n:]))
    return out


def _exact_conv_step(s, d):
    c, state, ys = s["case"], d["state"].clone(), []
    for n, slot in enumerate(s["slots"].tolist()):
        window = torch.cat([state[slot], d["x"][n:n + 1]])
        v = d["bias"] + torch.einsum("wd,dw->d", window, d["w"])
        ys.append(_exact_silu(v) if c["silu"] else v)
        state[slot] = window[1:]
    return {"y": torch.stack(ys), "state": state}


def _exact_norm(s, d):
    c, D, G = s["case"], s["case"]["D"], s["case"]["G"]
    w, bias = d["w"].requires_grad_(), d["bias"].requires_grad_()
    xs = [x.detach().requires_grad_() for x in _by_sequence(s, d["x"])]
    zs = [z.detach().requires_grad_() for z in _by_sequence(s, d["z"])] if c["gated"] else []
    ys, stats = [], []
    for i, x in enumerate(xs):
        L = x.shape[0]
        if L == 0:
            ys.append(x * 1.0)
            stats.append(x.new_zeros((0, G, 2) if c["rows"] else (G, 2)))
            continue
        g = x.reshape(L, G, D // G)
        dims = (2,) if c["rows"] else (0, 2)
        var, mu = torch.var_mean(g, dims, correction=0, keepdim=True)
        rstd = (var + EPS) ** -0.5
        v = ((g - mu) * rstd).reshape(L, D) * w + bias
        v = _exact_silu(v) if c["silu"] else v
        ys.append(v * _exact_silu(zs[i]) if c["gated"] else v)
        both = torch.stack([mu, rstd], -1)
        stats.append(both.reshape(L, G, 2) if c["rows"] else both.reshape(G, 2))
    out = {"y": _joined(s, ys).detach(), "stats": (_joined(s, stats) if c["rows"] else torch.stack(stats)).detach()}
    if c["run"] == "forward":
        return out
    got = torch.autograd.grad(_joined(s, ys), [w, bias] + xs + zs, d["dy"])
    n = len(xs)
    out.update(dw=got[0], dbias=got[1], dx=_joined(s, list(got[2:2 + n])))
    if c["gated"]:
        out["dz"] = _joined(s, list(got[2 + n:]))
    return out


def _exact_scan(s, d):
    c = s["case"]
    lens, N, D, G, S = s["lens"], len(s["lens"]), c["D"], c["G"], c["S"]
    T = max(lens)
    train = c["run"] == "train"

    def side_by_side(t):   # [T, N, ...]: row t of every sequence, zeros where it has ended
        out = t.new_zeros((T, N) + t.shape[1 if s["offsets"] is not None else 2:])
        for n, x in enumerate(_by_sequence(s, t)):
            out[:x.shape[0], n] = x
        return out

    apart = lambda t: _joined(s, [t[:L, n] for n, L in enumerate(lens)])   # noqa: E731
    L = np.array(lens)
    alive = [torch.from_numpy(np.flatnonzero(L > t)).to(DEV) if (L <= t).any() else slice(None) for t in range(T)]
    x, raw = side_by_side(d["x"]), side_by_side(d["dt"] + d["dt_bias"])
    dt = torch.where(raw > 0, raw + torch.log1p(torch.exp(-raw.abs())), torch.log1p(torch.exp(-raw.abs())))
    B, C = side_by_side(d["B"]), side_by_side(d["C"])   # [T, N, G, S]
    A = d["A"].reshape(G, D // G, S)
    split = lambda t: t.reshape(t.shape[:-1] + (G, D // G))   # noqa: E731
    whole = lambda t: t.reshape(t.shape[:-2] + (D,))   # noqa: E731
    block, kept = 64, []
    h, y = d["s0"].reshape(N, G, D // G, S).clone(), torch.zeros_like(x)

    def step(h, t):
        on = alive[t]
        b = split(dt[t][on])[..., None]
        h[on] = torch.exp(b * A) * h[on] + b * split(x[t][on])[..., None] * B[t][on][..., None, :]

    for t in range(T):
        if t % block == 0 and train:
            kept.append(h.clone())
        step(h, t)
        y[t] = whole(torch.matmul(h, C[t][..., None])[..., 0])
    y = y + d["skip"] * x
    z = side_by_side(d["z"]) if c["gated"] else None
    gate = 1.0 if z is None else _exact_silu(z)
    out = {"y": apart(y * gate), "last": h.reshape(N, D, S)}
    if not train:
        return out
    dy = side_by_side(d["dy"])
    if z is not None:
        e = torch.exp(-z)
        out["dz"] = apart(dy * y * (1 + e + z * e) / (1 + e) ** 2)
    dy = dy * gate
    lam = d["dlast"].reshape(N, G, D // G, S).clone()
    dx, ddt, dB, dC, dA = d["skip"] * dy, torch.zeros_like(x), torch.zeros_like(B), torch.zeros_like(C), torch.zeros_like(A)
    for b in range(len(kept) - 1, -1, -1):
        states, rows = [kept[b]], range(b * block, min(T, (b + 1) * block))
        for t in rows:
            states.append(states[-1].clone())
            step(states[-1], t)
        for t in reversed(rows):
            on = alive[t]
            now, before, u = states[t - b * block + 1][on], states[t - b * block][on], split(dy[t][on])
            delta, xt = split(dt[t][on]), split(x[t][on])
            dC[t][on] = torch.matmul(u[..., None, :], now)[..., 0, :]
            l = lam[on] + u[..., None] * C[t][on][..., None, :]
            dB[t][on] = torch.matmul((delta * xt)[..., None, :], l)[..., 0, :]
            read = torch.matmul(l, B[t][on][..., None])[..., 0]
            dx[t][on] += whole(delta * read)
            l = l * torch.exp(delta[..., None] * A)
            ddt[t][on] = whole((l * before * A).sum(-1) + xt * read)
            dA += (l * before * delta[..., None]).sum(0)
            lam[on] = l
    ddt = ddt / (1 + torch.exp(-raw))
    out.update(dx=apart(dx), ddt=apart(ddt), dB=apart(dB), dC=apart(dC), dA=dA.reshape(D, S), dskip=(dy * x).sum((0, 1)), dbias=ddt.sum((0, 1)),
               dh0=lam.reshape(N, D, S))
    return out


def _exact_scan_step(s, d):
    c, state, ys = s["case"], d["state"].clone(), []
    per = c["D"] // c["G"]
    group = torch.arange(c["D"], device=DEV) // per
    for n, slot in enumerate(s["slots"].tolist()):
        delta = torch.log(1 + torch.exp(d["dt"][n] + d["dt_bias"]))
        state[slot] = torch.exp(delta[:, None] * d["A"]) * state[slot] + (delta * d["x"][n])[:, None] * d["B"][n][group]
        y = torch.einsum("ds,ds->d", state[slot], d["C"][n][group]) + d["skip"] * d["x"][n]
        ys.append(y * _exact_silu(d["z"][n]) if c["gated"] else y)
    return {"y": torch.stack(ys), "state": state}
