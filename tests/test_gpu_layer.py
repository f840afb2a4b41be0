"""The operators of a layer with selective states as they are used: one behind the other, for prompts and then token by token, on streams, captured, many short
sequences, rows beyond 2^31 elements, workspaces and outputs with anything in them."""
import numpy as np
import pytest
import torch

import layer_oracle as lo
from paper_2309_12252_amd import deer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
SILU, NONE = deer.DEER_ACT_SILU, deer.DEER_ACT_NONE


def layer_weights(D, S, G, W, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)   # noqa: E731
    w = {"cw": r(D, W) / W ** 0.5, "cb": 0.1 * r(D), "A": -torch.exp(r(D, S)), "skip": r(D), "db": r(D) - 2, "nw": 1 + 0.1 * r(D), "nb": 0.1 * r(D)}
    return {k: t.float().to(DEV) for k, t in w.items()}


def layer_inputs(lead, D, S, G, dtype, seed):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen, dtype=torch.float64)   # noqa: E731
    return {k: t.to(lo.TYPES[dtype]).to(DEV) for k, t in {"x": r(*lead, D), "dt": r(*lead, D), "B": r(*lead, G, S), "C": r(*lead, G, S), "z": r(*lead, D), "dy": r(*lead, D)}.items()}


def forward(i, w, groups, conv0=None, h0=None, **more):
    u, conv = deer.shortconv_solve(i["x"], w["cw"], w["cb"], conv0, **more)
    v, h = deer.selscan_solve(u, i["dt"], w["A"], i["B"], i["C"], w["skip"], None, w["db"], h0, **more)
    y, stats = deer.groupnorm_solve(v, groups, w["nw"], w["nb"], i["z"], **more)
    return {"u": u, "v": v, "y": y, "stats": stats, "conv": conv, "h": h}


def backward(i, w, f, groups, **more):
    dv, dnw, dnb, dz = deer.groupnorm_grad(f["v"], groups, f["stats"], i["dy"], w["nw"], w["nb"], i["z"], **more)
    du, ddt, dA, dB, dC, dskip, _, ddb, _ = deer.selscan_grad(f["u"], i["dt"], w["A"], i["B"], i["C"], dv, w["skip"], None, w["db"], **more)
    dx, dcw, dcb, _ = deer.shortconv_grad(i["x"], w["cw"], du, w["cb"], **more)
    return {"x": dx, "dt": ddt, "B": dB, "C": dC, "z": dz, "cw": dcw, "cb": dcb, "A": dA, "skip": dskip, "db": ddb, "nw": dnw, "nb": dnb}


def plain(i, w, groups, lens):
    """the layer by elementary operations in float64 with gradients: i of [N, T, ...] on the host"""
    p = {k: t.detach().cpu().double().requires_grad_() for k, t in dict(i, **w).items()}
    x, D = p["x"], i["x"].shape[-1]
    N, T = x.shape[:2]
    W, G = w["cw"].shape[1], i["B"].shape[2]
    rows = torch.cat([torch.zeros(N, W - 1, D, dtype=torch.float64), x], 1)
    u = torch.nn.functional.silu(sum(p["cw"][:, j] * rows[:, j:j + T] for j in range(W)) + p["cb"])
    dt = torch.nn.functional.softplus(p["dt"] + p["db"])
    B, C = (p[n].repeat_interleave(D // G, 2) for n in "BC")
    h, vs = torch.zeros(N, D, w["A"].shape[1], dtype=torch.float64), []
    for t in range(T):
        h = torch.exp(dt[:, t, :, None] * p["A"]) * h + (dt[:, t] * u[:, t])[..., None] * B[:, t]
        vs.append((C[:, t] * h).sum(-1) + p["skip"] * u[:, t])
    v = torch.stack(vs, 1).reshape(N, T, groups, -1)
    n = ((v - v.mean(-1, keepdim=True)) / torch.sqrt(v.var(-1, correction=0, keepdim=True) + 1e-5)).reshape(N, T, D) * p["nw"] + p["nb"]
    y = n * torch.nn.functional.silu(p["z"])
    inside = torch.arange(T)[None] < torch.tensor(lens)[:, None]
    grads = torch.autograd.grad((y * p["dy"] * inside[..., None]).sum(), [p[k] for k in p if k != "dy"], allow_unused=True)
    return y.detach(), dict(zip([k for k in p if k != "dy"], grads)), inside


@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("D,S,G,groups", [(24, 16, 1, 3), (32, 5, 2, 4)])
def test_together(D, S, G, groups, packed):
    """float32: every result of the chain within what some hundred roundings of a row's path leave, all together; values below a row's norm by eight channels' norms"""
    T, W, lens = 70, 4, [70, 33, 0, 1]
    w = layer_weights(D, S, G, W, "f32", 1)
    i = layer_inputs((4, T), D, S, G, "f32", 2)
    want, grads, inside = plain(i, w, groups, lens)
    more = {"lengths": torch.tensor(lens, device=DEV)}
    if packed:
        i = {k: t[inside.to(DEV)] for k, t in i.items()}
        more = {"offsets": torch.tensor(np.concatenate([[0], np.cumsum(lens)]), device=DEV)}
    f = forward(i, w, groups, **more)
    got = backward(i, w, f, groups, **more)
    rel = lambda a, b: float((a - b).norm() / b.norm())   # noqa: E731
    most = 4 * (T + 128) * 2.0 ** -24
    flat = (lambda t: t.cpu().double()) if packed else (lambda t: t.cpu().double()[inside])
    assert rel(flat(f["y"]), want[inside]) <= most
    for k, g in grads.items():
        a, b = got[k], g
        a, b = (flat(a), b[inside]) if k in ("x", "dt", "B", "C", "z") else (a.cpu().double(), b)
        print(k, rel(a, b), most, flush=True)
        assert rel(a, b) <= 4 * most, k   # (the norm's gradient amplifies by rstd, of order one here)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_prompt_and_then_tokens(dtype):
    """a layer over a prompt and then token by token from pools of states: as over the whole.  Half a step of the type in u and v each, which pass on through the rest"""
    N, T, more, D, S, groups, W = 3, 21, 6, 40, 16, 5, 4
    w = layer_weights(D, S, 1, W, dtype, 3)
    i = layer_inputs((N, T + more), D, S, 1, dtype, 4)
    whole = forward(i, w, groups)
    first = forward({k: t[:, :T].contiguous() for k, t in i.items()}, w, groups)
    slots = torch.tensor([3, 0, 4], dtype=torch.int32, device=DEV)
    conv, h = torch.zeros(5, W - 1, D, device=DEV), torch.zeros(5, D, S, device=DEV)
    conv[slots.long()], h[slots.long()] = first["conv"], first["h"]
    for t in range(T, T + more):
        now = {k: v[:, t].contiguous() for k, v in i.items()}
        u = deer.shortconv_step(now["x"], w["cw"], conv, w["cb"], slots=slots)
        v = deer.selscan_step(u, now["dt"], w["A"], now["B"], now["C"], h, w["skip"], None, w["db"], slots=slots)
        y, _ = deer.groupnorm_solve(v[:, None], groups, w["nw"], w["nb"], now["z"][:, None])
        assert torch.equal(u, whole["u"][:, t])   # (the same products in the same order)
        a, b = v.double(), whole["v"][:, t].double()
        assert float((a - b).norm() / b.norm()) <= 2 * lo.HALF[dtype] + 64 * 2.0 ** -24, t
        a, b = y[:, 0].double(), whole["y"][:, t].double()
        assert float((a - b).norm() / b.norm()) <= 8 * lo.HALF[dtype] + 256 * 2.0 ** -24, t
    assert torch.equal(conv[slots.long()], whole["conv"])


def everything(i, w, groups, **more):
    f = forward(i, w, groups, **more)
    seq = dict(more, span=deer.DEER_SPAN_SEQUENCE)
    y2, stats2 = deer.groupnorm_solve(f["v"], groups, w["nw"], w["nb"], i["z"], act=SILU, **seq)
    g2 = deer.groupnorm_grad(f["v"], groups, stats2, i["dy"], w["nw"], w["nb"], i["z"], act=SILU, **seq)
    return list(f.values()) + list(backward(i, w, f, groups, **more).values()) + [y2, stats2] + list(g2)


def test_the_same_bits_twice_and_on_another_stream():
    w, i = layer_weights(72, 16, 1, 4, "bf16", 5), layer_inputs((500,), 72, 16, 1, "bf16", 6)
    more = {"offsets": torch.tensor([3, 100, 100, 333, 490], device=DEV)}
    one, two = everything(i, w, 9, **more), everything(i, w, 9, **more)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    three = everything(i, w, 9, stream=side, **more)
    torch.cuda.current_stream().wait_stream(side)
    for a, b, c in zip(one, two, three):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_workspaces_and_outputs_hold_anything(monkeypatch):
    """what is allocated without a value holds NaN, workspaces all bits"""
    w, i = layer_weights(72, 16, 1, 4, "f32", 5), layer_inputs((700,), 72, 16, 1, "f32", 6)
    more = {"offsets": torch.tensor([3, 100, 100, 600, 690], device=DEV)}
    want = everything(i, w, 9, **more)

    def fill(make):
        def made(*args, **kw):
            t = make(*args, **kw)
            return t.fill_(float("nan")) if t.is_floating_point() else t
        return made
    for name in ("empty", "empty_like", "empty_strided"):
        monkeypatch.setattr(torch, name, fill(getattr(torch, name)))
    plain_new = torch.Tensor.new_empty
    monkeypatch.setattr(torch.Tensor, "new_empty", lambda self, *a, **kw: plain_new(self, *a, **kw).fill_(255))
    for a, b in zip(want, everything(i, w, 9, **more)):
        assert torch.equal(a, b) and bool(torch.isfinite(b).all())


def test_captured_with_other_lengths_in_every_replay():
    """two graphs, each call with workspaces of its own; bounds and inputs change between replays, eager work lies between them"""
    groups, graphs = 4, []
    w = layer_weights(64, 16, 1, 4, "bf16", 7)
    for k in range(2):
        i = layer_inputs((300,), 64, 16, 1, "bf16", 8 + k)
        offsets = torch.tensor([0, 100, 200, 300], device=DEV)
        everything(i, w, groups, offsets=offsets)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = everything(i, w, groups, offsets=offsets)
        graphs.append((graph, i, offsets, out))
    for turn, bounds in enumerate(([0, 100, 200, 300], [5, 5, 250, 251], [0, 0, 0, 300], [17, 18, 50, 60])):
        for k, (graph, i, offsets, out) in enumerate(graphs):
            offsets.copy_(torch.tensor(bounds))
            for n, t in layer_inputs((300,), 64, 16, 1, "bf16", 100 * turn + k).items():
                i[n].copy_(t)
            graph.replay()
            want = everything(i, w, groups, offsets=offsets)
            torch.cuda.synchronize()
            for a, b in zip(out, want):
                assert torch.equal(a, b), (turn, k)


def test_captured_tokens():
    D, S, W, N = 64, 16, 4, 5
    w, i = layer_weights(D, S, 1, W, "bf16", 9), layer_inputs((N,), D, S, 1, "bf16", 10)
    slots = torch.tensor([4, 0, 2, 1, 3], dtype=torch.int32, device=DEV)
    conv, h = torch.zeros(6, W - 1, D, device=DEV), torch.zeros(6, D, S, device=DEV)

    def token(conv, h):
        u = deer.shortconv_step(i["x"], w["cw"], conv, w["cb"], slots=slots)
        v = deer.selscan_step(u, i["dt"], w["A"], i["B"], i["C"], h, w["skip"], i["z"], w["db"], slots=slots)
        return deer.groupnorm_solve(v[:, None], 8, w["nw"], w["nb"])[0]
    token(conv, h)
    torch.cuda.synchronize()
    conv.zero_(), h.zero_()
    conv2, h2 = conv.clone(), h.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = token(conv, h)
    conv.zero_(), h.zero_()
    for turn in range(5):
        for n, t in layer_inputs((N,), D, S, 1, "bf16", 20 + turn).items():
            i[n].copy_(t)
        slots.copy_(torch.tensor([[4, 0, 2, 1, 3], [1, -1, 3, 3, 9], [0, 1, 2, 3, 4], [5, 4, 3, 2, 1], [4, 4, 4, 4, 4]][turn]))
        graph.replay()
        want = token(conv2, h2)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(conv, conv2) and torch.equal(h, h2), turn


@pytest.mark.parametrize("N,longest", [(700, 3), (65, 9), (64, 9), (63, 9), (5000, 2)])
def test_many_short_sequences(N, longest):
    """as a padded batch of the same rows: the same products and sums in the same order, but for sums over all rows"""
    rng = np.random.default_rng(N)
    lens = rng.integers(0, longest + 1, N)
    D, S, groups, W = 8, 5, 2, 3
    w, i = layer_weights(D, S, 1, W, "f32", 11), layer_inputs((N, longest), D, S, 1, "f32", 12)
    inside = torch.arange(longest, device=DEV)[None] < torch.from_numpy(lens).to(DEV)[:, None]
    flat = {k: t[inside] for k, t in i.items()}
    a = forward(flat, w, groups, offsets=torch.tensor(np.concatenate([[0], np.cumsum(lens)]), device=DEV))
    b = forward(i, w, groups, lengths=torch.from_numpy(lens).to(DEV))
    for k in ("u", "conv"):
        assert torch.equal(a[k], b[k][inside] if k == "u" else b[k]), k
    close = lambda x, y: float((x.double() - y.double()).norm()) <= 64 * 2.0 ** -24 * float(y.double().norm())   # noqa: E731
    assert close(a["v"], b["v"][inside]) and close(a["h"], b["h"]) and close(a["y"], b["y"][inside])
    ga = backward(flat, w, a, groups, offsets=torch.tensor(np.concatenate([[0], np.cumsum(lens)]), device=DEV))
    gb = backward(i, w, b, groups, lengths=torch.from_numpy(lens).to(DEV))
    for k in ga:
        x, y = ga[k], gb[k][inside] if k in ("x", "dt", "B", "C", "z") else gb[k]
        assert float((x.double() - y.double()).norm()) <= 1024 * 2.0 ** -24 * float(y.double().norm()) + 1e-6, k
    seq = deer.DEER_SPAN_SEQUENCE
    ya, sa = deer.groupnorm_solve(flat["x"], groups, span=seq, offsets=torch.tensor(np.concatenate([[0], np.cumsum(lens)]), device=DEV))
    yb, sb = deer.groupnorm_solve(i["x"], groups, span=seq, lengths=torch.from_numpy(lens).to(DEV))
    assert close(ya, yb[inside]) and close(sa, sb)


def test_bounds_are_clamped():
    w, i = layer_weights(16, 4, 1, 4, "f32", 13), layer_inputs((50,), 16, 4, 1, "f32", 14)
    for bad, good in (([-5, 10, 1000], [0, 10, 50]), ([60, 70, 80], [50, 50, 50]), ([-9, -3, 20], [0, 0, 20])):
        a, b = everything(i, w, 4, offsets=torch.tensor(bad, device=DEV)), everything(i, w, 4, offsets=torch.tensor(good, device=DEV))
        for x, y in zip(a, b):
            assert torch.equal(x, y)


def test_rows_beyond_32_bits():
    """more than 2^32 bytes and 2^31 elements in an array: the last rows as from the states in front of them"""
    T, D, S, tail = 1050000, 2100, 2, 3000
    x = torch.empty(1, T, D, dtype=torch.bfloat16, device=DEV)
    x[:, :].fill_(0.25)
    gen = torch.Generator(device=DEV).manual_seed(1)
    x[:, -2 * tail:] = torch.randn(1, 2 * tail, D, generator=gen, device=DEV).bfloat16()
    wc = torch.randn(D, 4, generator=gen, device=DEV)
    last = x[:, -tail:].contiguous()
    y, state = deer.shortconv_solve(x, wc)
    front = x[:, -tail - 3:-tail].float().contiguous()
    y2, state2 = deer.shortconv_solve(last, wc, s0=front)
    assert torch.equal(y[:, -tail:], y2) and torch.equal(state, state2)
    del y
    dx = deer.shortconv_grad(x, wc, x)[0]
    assert torch.equal(dx[:, -tail:], deer.shortconv_grad(last, wc, last, s0=front)[0])
    del dx
    for span in (deer.DEER_SPAN_ROW,):
        y, stats = deer.groupnorm_solve(x, 7, span=span)
        y2, stats2 = deer.groupnorm_solve(last, 7, span=span)
        assert torch.equal(y[:, -tail:], y2) and torch.equal(stats[:, -tail:], stats2)
        del y
    A = -torch.rand(D, S, generator=gen, device=DEV) - 8.0   # (steps of 0.8 and more: what is 30 rows back is below 2^-200)
    B = torch.randn(1, T, 1, S, generator=gen, device=DEV).bfloat16()
    y, h = deer.selscan_solve(x, x, A, B, B, dt_bias=torch.full((D,), 4.0, device=DEV))
    y2, h2 = deer.selscan_solve(last, last, A, B[:, -tail:].contiguous(), B[:, -tail:].contiguous(), dt_bias=torch.full((D,), 4.0, device=DEV))
    assert torch.equal(y[:, -tail + 100:], y2[:, 100:]) and torch.equal(h, h2)


def test_refusals_of_the_binding():
    w, i = layer_weights(16, 4, 2, 4, "bf16", 1), layer_inputs((2, 9), 16, 4, 2, "bf16", 2)
    x, z, dt, B, C = i["x"], i["z"], i["dt"], i["B"], i["C"]
    state, pool = torch.zeros(2, 16, 4, device=DEV), torch.zeros(2, 3, 16, device=DEV)
    _, stats = deer.groupnorm_solve(x, 4)
    lengths = torch.tensor([3, 9], device=DEV)
    for call in (
            lambda: deer.shortconv_solve(x, w["cw"].bfloat16()), lambda: deer.shortconv_solve(x, w["cw"][:8]), lambda: deer.shortconv_solve(x, w["cw"], w["cb"][:8]),
            lambda: deer.shortconv_solve(x, w["cw"], s0=pool[:, :2]), lambda: deer.shortconv_solve(x, w["cw"], lengths=lengths.int()),
            lambda: deer.shortconv_solve(x, w["cw"], lengths=lengths, offsets=lengths), lambda: deer.shortconv_solve(x[0], w["cw"]),
            lambda: deer.shortconv_solve(x.long(), w["cw"]), lambda: deer.shortconv_solve(x, w["cw"].cpu()), lambda: deer.shortconv_solve(x, w["cw"], act=1),
            lambda: deer.shortconv_solve(x[..., ::2], w["cw"][::2].contiguous()), lambda: deer.shortconv_solve(x[:, :1].expand(2, 9, 16), w["cw"]),
            lambda: deer.shortconv_step(x, w["cw"], pool), lambda: deer.shortconv_step(x[0], w["cw"], pool[:, :2]), lambda: deer.shortconv_step(x[0], w["cw"], pool, slots=lengths),
            lambda: deer.shortconv_grad(x, w["cw"], x[:, :5]), lambda: deer.shortconv_grad(x, w["cw"], x, dx=torch.zeros(2, 9, 32, dtype=x.dtype, device=DEV)[..., :16]),
            lambda: deer.selscan_solve(x.double(), dt, w["A"], B, C), lambda: deer.selscan_solve(x, dt.float(), w["A"], B, C), lambda: deer.selscan_solve(x, dt, w["A"][:8], B, C),
            lambda: deer.selscan_solve(x, dt, w["A"], B, C[..., :3]), lambda: deer.selscan_solve(x, dt, w["A"], B[..., 0, :], C[..., 0, :]),
            lambda: deer.selscan_solve(x, dt, w["A"], B, C, w["skip"][:8]), lambda: deer.selscan_solve(x, dt, w["A"], B, C, z=z[:, :4]),
            lambda: deer.selscan_solve(x, dt, w["A"], B.expand(2, 9, 2, 4)[:, :, :1].expand(2, 9, 3, 4).contiguous(), C, h0=state),
            lambda: deer.selscan_solve(x, dt, w["A"], B, C, h0=state[:1]), lambda: deer.selscan_grad(x, dt, w["A"], B, C, x, dz=x.clone()),
            lambda: deer.selscan_grad(x, dt, w["A"], B, C, x.float()), lambda: deer.selscan_step(x[0], dt[0], w["A"], B[0], C[0], state.double()),
            lambda: deer.selscan_step(x, dt, w["A"], B, C, state), lambda: deer.groupnorm_solve(x, 3), lambda: deer.groupnorm_solve(x, 4, span=2),
            lambda: deer.groupnorm_solve(x, 4, eps=-1.0), lambda: deer.groupnorm_solve(x, 4, w["nw"].double()), lambda: deer.groupnorm_solve(x, 4, z=z[:1]),
            lambda: deer.groupnorm_grad(x, 4, stats[..., :1], x), lambda: deer.groupnorm_grad(x, 4, None, x), lambda: deer.groupnorm_grad(x, 4, stats, x, dz=x.clone()),
            lambda: deer.groupnorm_grad(x, 4, stats, x, span=deer.DEER_SPAN_SEQUENCE)):
        with pytest.raises(deer.DeerError) as e:
            call()
        assert e.value.status == deer.DEER_ERR_INVALID_ARG
    with pytest.raises(deer.DeerError) as e:
        deer.selscan_solve(x, dt, torch.zeros(16, 65, device=DEV), torch.zeros(2, 9, 1, 65, dtype=x.dtype, device=DEV), torch.zeros(2, 9, 1, 65, dtype=x.dtype, device=DEV))
    assert e.value.status == deer.DEER_ERR_UNSUPPORTED
