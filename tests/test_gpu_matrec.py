"""Gated linear recurrences with a matrix as state, against row-by-row 64-bit forms."""
import numpy as np
import pytest
import torch

import seq_oracle as so
from paper_2309_12252_amd import deer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
NAMES = ("o", "last", "dq", "dk", "dv", "dgate", "ds0")


def host(t):
    return t.detach().cpu().double().numpy()


def make(dtype, lead, N, Hk, Hv, Dk, Dv, seed, strong=False):
    rng = np.random.default_rng(seed)
    t = so.TYPES[dtype]
    dev = lambda a, ty=t: torch.from_numpy(np.ascontiguousarray(a)).to(ty).to(DEV)   # noqa: E731
    k = rng.standard_normal(lead + (Hk, Dk))
    g = -np.exp(1.5 * rng.standard_normal(lead + (Hv,)) + (1.0 if strong else -3.0))
    return {"q": dev(rng.standard_normal(lead + (Hk, Dk))), "k": dev(k / np.linalg.norm(k, axis=-1, keepdims=True)), "v": dev(rng.standard_normal(lead + (Hv, Dv))),
            "g": dev(g, torch.float32), "s0": dev(rng.standard_normal((N, Hv, Dk, Dv)), torch.float32), "do": dev(rng.standard_normal(lead + (Hv, Dv))),
            "dlast": dev(rng.standard_normal((N, Hv, Dk, Dv)), torch.float32)}


def both(d, **more):
    o, last = deer.matrec_solve(d["q"], d["k"], d["v"], d["g"], d["s0"], **more)
    return dict(zip(NAMES, (o, last) + deer.matrec_grad(d["q"], d["k"], d["v"], d["g"], d["do"], d["s0"], d["dlast"], **more)))


def compare(d, got, seqs, dtype, scale):
    flat = {n: host(t).reshape((-1,) + t.shape[-2:] if n != "g" else (-1, t.shape[-1])) for n, t in d.items() if n not in ("s0", "dlast")}
    s0, dlast = host(d["s0"]), host(d["dlast"])
    want, absolute, passing = so.matrix(flat["q"], flat["k"], flat["v"], flat["g"], s0, seqs, scale, flat["do"], dlast)
    alive = np.zeros(flat["g"].shape[0], dtype=bool)
    for r0, n in seqs:
        alive[r0:r0 + n] = True
    at = torch.from_numpy(alive).to(DEV)
    g2 = {}
    for n, t in got.items():
        if n in ("last", "ds0"):
            g2[n] = t
            continue
        g2[n] = t.reshape((alive.size,) + want[n].shape[1:])[at]
        want[n], absolute[n] = want[n][alive], absolute[n][alive]
    so.check_matrix(g2, want, absolute, passing[alive], dtype, max(n for _, n in seqs))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,T,Hk,Hv,Dk,Dv", [(1, 1, 1, 1, 1, 1), (2, 3, 1, 2, 16, 8), (1, 63, 2, 2, 64, 64), (1, 64, 1, 1, 128, 128), (2, 65, 1, 3, 33, 70), (1, 200, 2, 4, 128, 64),
                                             (1, 300, 1, 1, 64, 128), (3, 130, 1, 2, 5, 100), (1, 700, 1, 1, 40, 72), (1, 129, 2, 2, 127, 31)])
def test_batch(dtype, N, T, Hk, Hv, Dk, Dv):
    d = make(dtype, (N, T), N, Hk, Hv, Dk, Dv, T + Dk)
    compare(d, both(d), so.sequences(T, N), dtype, Dk ** -0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_strong_gates(dtype):
    # factors from one down to far below the smallest number, and gates of -inf: what is forgotten is gone, its gradient too
    d = make(dtype, (1, 400), 1, 2, 2, 48, 32, 5, strong=True)
    d["g"][0, ::13] = -float("inf")
    d["g"][0, 5::17] = 0.0
    d["g"][0, 7::29] = -3.0e38
    got = both(d, scale=0.7)
    assert bool((got["dgate"][torch.isinf(d["g"])] == 0).all())
    compare(d, got, so.sequences(400, 1), dtype, 0.7)


PACKED = {"mixed": [0, 130, 131, 131, 500, 501, 900, 900], "tokens": list(range(0, 41)), "behind": [3, 3, 20, 150, 260], "one": [0, 1100], "empty": [0, 0, 0]}


@pytest.mark.parametrize("dtype,Hk,Hv,Dk,Dv", [("bf16", 2, 4, 64, 40), ("f32", 1, 1, 24, 65)])
@pytest.mark.parametrize("name", list(PACKED))
def test_packed(name, dtype, Hk, Hv, Dk, Dv):
    off = PACKED[name]
    N, rows = len(off) - 1, off[-1] + 9
    d = make(dtype, (rows,), N, Hk, Hv, Dk, Dv, 7)
    for n in ("q", "k", "v", "do", "g"):   # rows of no sequence are not looked at
        d[n][off[-1]:] = float("nan")
        d[n][:off[0]] = float("nan")
    offsets = torch.tensor(off, dtype=torch.int64, device=DEV)
    mark = lambda t: torch.full_like(t, 7.0)   # noqa: E731
    o, last = deer.matrec_solve(d["q"], d["k"], d["v"], d["g"], d["s0"], offsets=offsets, out=mark(d["v"]))
    back = deer.matrec_grad(d["q"], d["k"], d["v"], d["g"], d["do"], d["s0"], d["dlast"], offsets=offsets, dq=mark(d["q"]), dk=mark(d["k"]), dv=mark(d["v"]))
    for t in (o,) + back[:3]:
        assert bool((t[off[-1]:] == 7).all()) and bool((t[:off[0]] == 7).all())
    for n in ("q", "k", "v", "do", "g"):
        d[n].nan_to_num_(0.0)
    compare(d, dict(zip(NAMES, (o, last) + back)), so.sequences(rows, N, offsets=off), dtype, Dk ** -0.5)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_padded_batch(dtype):
    N, T, lens = 5, 200, [200, 0, 1, 64, 129]
    d = make(dtype, (N, T), N, 1, 2, 32, 48, 3)
    for n, L in enumerate(lens):
        for x in ("q", "k", "v", "do", "g"):
            d[x][n, L:] = float("nan")
    lengths = torch.tensor(lens, dtype=torch.int64, device=DEV)
    mark = lambda t: torch.full_like(t, 3.0)   # noqa: E731
    o, last = deer.matrec_solve(d["q"], d["k"], d["v"], d["g"], d["s0"], lengths=lengths, out=mark(d["v"]))
    back = deer.matrec_grad(d["q"], d["k"], d["v"], d["g"], d["do"], d["s0"], d["dlast"], lengths=lengths, dq=mark(d["q"]), dk=mark(d["k"]), dv=mark(d["v"]))
    for n, L in enumerate(lens):
        for t in (o,) + back[:3]:
            assert bool((t[n, L:] == 3).all())
    for x in ("q", "k", "v", "do", "g"):
        d[x].nan_to_num_(0.0)
    compare(d, dict(zip(NAMES, (o, last) + back)), so.sequences(T, N, lengths=lens), dtype, 32 ** -0.5)


@pytest.mark.parametrize("dtype,Hk,Hv,Dk,Dv", [("bf16", 2, 4, 64, 32), ("bf16", 1, 2, 20, 36), ("f32", 1, 3, 17, 9)])
def test_slices_of_a_projection(dtype, Hk, Hv, Dk, Dv):
    N, T = 2, 150
    d = make(dtype, (N, T), N, Hk, Hv, Dk, Dv, 5)
    a, b = Hk * Dk, Hv * Dv
    qkv = torch.cat([d["q"].flatten(2), d["k"].flatten(2), d["v"].flatten(2)], -1).contiguous()
    parts = lambda t: (t[..., :a].unflatten(-1, (Hk, Dk)), t[..., a:2 * a].unflatten(-1, (Hk, Dk)), t[..., 2 * a:].unflatten(-1, (Hv, Dv)))   # noqa: E731
    q, k, v = parts(qkv)
    wide = torch.zeros(N, T, b + 3, dtype=v.dtype, device=DEV)
    o, last = deer.matrec_solve(q, k, v, d["g"], d["s0"], out=wide[..., :b].unflatten(-1, (Hv, Dv)))
    assert bool((wide[..., b:] == 0).all())
    grad = torch.empty_like(qkv)
    dq, dk, dv = parts(grad)
    back = deer.matrec_grad(q, k, v, d["g"], d["do"], d["s0"], d["dlast"], dq=dq, dk=dk, dv=dv)
    compare(d, dict(zip(NAMES, (o, last) + back)), so.sequences(T, N), dtype, Dk ** -0.5)
    for x, y in zip(deer.matrec_grad(q, k, v, d["g"], d["do"], d["s0"], d["dlast"]), back):
        assert torch.equal(x, y)


def test_without_states_and_empty_arrays():
    d = make("bf16", (2, 70), 2, 1, 2, 16, 24, 4)
    o, last = deer.matrec_solve(d["q"], d["k"], d["v"], d["g"])
    back = deer.matrec_grad(d["q"], d["k"], d["v"], d["g"], d["do"])
    d["s0"].zero_()
    d["dlast"].zero_()
    compare(d, dict(zip(NAMES, (o, last) + back)), so.sequences(70, 2), "bf16", 0.25)
    e = {n: t[:, :0].contiguous() if n not in ("s0", "dlast") else t for n, t in d.items()}
    s0 = torch.randn_like(d["s0"])
    o, last = deer.matrec_solve(e["q"], e["k"], e["v"], e["g"], s0)
    assert o.shape == (2, 0, 2, 24) and torch.equal(last, s0)
    assert torch.equal(deer.matrec_grad(e["q"], e["k"], e["v"], e["g"], e["do"], s0, s0)[4], s0)


def test_not_finite_stays_in_its_sequence_and_head():
    off = [0, 300, 600, 900]
    d = make("bf16", (900,), 3, 2, 2, 32, 32, 2)
    offsets = torch.tensor(off, device=DEV)
    clean, clast = deer.matrec_solve(d["q"], d["k"], d["v"], d["g"], d["s0"], offsets=offsets)
    v = d["v"].clone()
    v[450, 1, 3] = float("nan")
    o, last = deer.matrec_solve(d["q"], d["k"], v, d["g"], d["s0"], offsets=offsets)
    assert bool(torch.isnan(o[450:600, 1, 3]).all())
    ok = torch.ones_like(o, dtype=torch.bool)
    ok[428:600, 1] = False   # from the first row of its chunk (300 + 128) on
    assert torch.equal(o[ok], clean[ok])
    assert torch.equal(last[[0, 2]], clast[[0, 2]]) and torch.equal(last[1, 0], clast[1, 0])


def test_the_same_bits_again_and_other_streams():
    ds = [make("bf16", (1, 3000), 1, 2, 4, 64, 64, s) for s in (1, 2)]
    want = [both(d) for d in ds]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(3):
        for s, d in zip(streams, ds):
            got.append(both(d, stream=s))
    torch.cuda.synchronize()
    for i, r in enumerate(got):
        for n in NAMES:
            assert torch.equal(r[n], want[i % 2][n]), n


def test_captured():
    d = make("bf16", (900,), 3, 1, 2, 64, 64, 2)
    offsets = torch.tensor([0, 300, 310, 900], device=DEV)
    state = torch.randn(4, 2, 64, 64, device=DEV)
    first = state.clone()

    def step():
        r = both(d, offsets=offsets)
        state.copy_(first)
        return tuple(r[n] for n in NAMES) + (deer.matrec_step(d["q"][:4], d["k"][:4], d["v"][:4], d["g"][:4], state), state.clone())

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graphs, outs = [], []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step())
        graphs.append(graph)
    for _ in range(4):
        d["v"].copy_(torch.randn(d["v"].shape, device=DEV))
        for graph, out in zip(graphs, outs):
            for t in out:
                t.fill_(5)
            graph.replay()
        torch.cuda.synchronize()
        want = step()
        for out in outs:
            for a, b in zip(out, want):
                assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,Hk,Hv,Dk,Dv", [(1, 1, 1, 1, 1), (3, 2, 4, 64, 64), (2, 1, 3, 33, 70), (5, 2, 2, 128, 128), (2, 1, 1, 128, 3)])
def test_step(dtype, N, Hk, Hv, Dk, Dv):
    d = make(dtype, (N,), N, Hk, Hv, Dk, Dv, 9)
    state = torch.randn(N + 3, Hv, Dk, Dv, device=DEV)
    slots = torch.randperm(N + 3)[:N].to(torch.int32)
    before = state.clone()
    o = deer.matrec_step(d["q"], d["k"], d["v"], d["g"], state, slots=slots.to(DEV))
    want, absolute, _ = so.matrix(host(d["q"]), host(d["k"]), host(d["v"]), host(d["g"]), host(before)[slots.numpy()], [(n, 1) for n in range(N)], Dk ** -0.5)
    # fp32 throughout: factor, two products, a sum; then the sum over Dk columns
    so.check("state", state[slots.long().to(DEV)], want["last"], 6 * 2.0 ** -24 * absolute["last"], "f32")
    so.check("o", o, want["o"], (Dk + 8) * 2.0 ** -24 * absolute["o"], dtype)
    rest = [s for s in range(N + 3) if s not in slots.tolist()]
    assert torch.equal(state[rest], before[rest])


def test_step_passes_over_bad_and_repeated_slots():
    d = make("f32", (6,), 6, 1, 2, 32, 32, 1)
    state = torch.randn(4, 2, 32, 32, device=DEV)
    before, out = state.clone(), torch.full_like(d["v"], 9.0)
    slots = torch.tensor([2, -1, 4, 2, 0, 2000000000], dtype=torch.int32, device=DEV)
    deer.matrec_step(d["q"], d["k"], d["v"], d["g"], state, slots=slots, out=out)
    for n in (1, 2, 3, 5):
        assert bool((out[n] == 9).all())
    assert not bool((out[[0, 4]] == 9).any())
    assert torch.equal(state[[1, 3]], before[[1, 3]]) and not torch.equal(state[0], before[0]) and not torch.equal(state[2], before[2])
    alone = before.clone()
    deer.matrec_step(d["q"][:1], d["k"][:1], d["v"][:1], d["g"][:1], alone, slots=slots[:1])
    assert torch.equal(alone[2], state[2])


def test_steps_continue_a_prompt():
    N, T, more = 2, 150, 4
    d = make("f32", (N, T + more), N, 1, 2, 32, 16, 11)
    o, last = deer.matrec_solve(d["q"], d["k"], d["v"], d["g"], d["s0"])
    cut = lambda t: t[:, :T].contiguous()   # noqa: E731
    _, state = deer.matrec_solve(cut(d["q"]), cut(d["k"]), cut(d["v"]), cut(d["g"]), d["s0"])
    for t in range(T, T + more):
        one = deer.matrec_step(*(d[n][:, t].contiguous() for n in ("q", "k", "v", "g")), state)
        # both within 4 (T + 128) roundings of the exact ones, whose absolute sums stay below 20 times the largest value here
        assert float((one - o[:, t]).abs().max()) <= 2 * 4 * (T + 128) * 2.0 ** -24 * 20 * float(o.abs().max())
    assert float((state - last).abs().max()) <= 2 * 4 * (T + 128) * 2.0 ** -24 * 20 * float(last.abs().max())


def test_layer_of_both_recurrences():
    # as they are used together: dropout, a diagonal recurrence along the channels, then heads with matrix states on packed rows; gradients back
    # through all of them by the chain rule, against autograd over the plain forms in 64 bits
    off, D, H, Dk, Dv = [0, 90, 91, 230], 48, 2, 8, 8
    rows, N = off[-1], 3
    gen = torch.Generator(device=DEV)
    gen.manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=gen, device=DEV)   # noqa: E731
    gate, x, g, do = r(rows, D), r(rows, D), -torch.exp(r(rows, H) - 2), r(rows, H, Dv)
    offsets = torch.tensor(off, device=DEV)
    a = {"kind": deer.DEER_GATE_SIGMOID, "offsets": offsets, "drop": 0.2, "seed": 17, "draw": 5}
    h, _ = deer.diagrec_solve(gate, x, **a)
    q, k, v = (h[:, i * 16:(i + 1) * 16].unflatten(-1, (H, 8)) for i in range(3))
    o, _ = deer.matrec_solve(q, k, v, g, offsets=offsets)
    dh = torch.empty_like(h)
    parts = [dh[:, i * 16:(i + 1) * 16].unflatten(-1, (H, 8)) for i in range(3)]
    _, _, _, dg, _ = deer.matrec_grad(q, k, v, g, do, offsets=offsets, dq=parts[0], dk=parts[1], dv=parts[2])
    dgate, dx, _ = deer.diagrec_grad(gate, x, h, dh, **a)
    leaf = lambda t: t.cpu().double().requires_grad_()   # noqa: E731
    G, X, L = leaf(gate), leaf(x), leaf(g)
    keep = torch.from_numpy(so.philox_keep(1, rows, D, 0.2, 17, 5)[0])
    hs, os_ = [], []
    for s in range(N):
        state, S = torch.zeros(D, dtype=torch.float64), torch.zeros(H, Dk, Dv, dtype=torch.float64)
        for t in range(off[s], off[s + 1]):
            f = torch.sigmoid(G[t])
            state = f * state + (1 - f) * X[t] * keep[t]
            hs.append(state)
            qq, kk, vv = state.view(3, H, 8)
            S = torch.exp(L[t])[:, None, None] * S + kk[:, :, None] * vv[:, None, :]
            os_.append((qq[:, :, None] * S).sum(1) * 8 ** -0.5)
    O = torch.stack(os_)
    (O * do.cpu().double()).sum().backward()
    # fp32 throughout: some 4 (T + 128) roundings of sums, whose absolute values stay within 50 of the largest result
    for name, got, want in (("h", h, torch.stack(hs)), ("o", o, O), ("dgate", dgate, G.grad), ("dx", dx, X.grad), ("dg", dg, L.grad)):
        want = want.detach().numpy()
        err = np.abs(host(got) - want).max() / np.abs(want).max()
        print(name, err)
        assert err <= 4 * (139 + 128) * 2.0 ** -24 * 50, (name, err)


def test_gradient_by_differences():
    # fp32 forward passes: the difference quotient along a direction, halved steps
    N, T = 2, 70
    d = make("f32", (N, T), N, 1, 2, 8, 8, 15)
    grads = dict(zip(("q", "k", "v", "g", "s0"), deer.matrec_grad(d["q"], d["k"], d["v"], d["g"], d["do"], d["s0"], d["dlast"])))

    def loss(e):
        o, last = deer.matrec_solve(e["q"], e["k"], e["v"], e["g"], e["s0"])
        return float((o.double() * d["do"]).sum() + (last.double() * d["dlast"]).sum())

    for n in grads:
        direction = torch.randn(d[n].shape, generator=torch.Generator().manual_seed(3)).to(DEV)
        step = 1e-2
        up, down = loss(dict(d, **{n: d[n] + step * direction})), loss(dict(d, **{n: d[n] - step * direction}))
        want = float((grads[n].double() * direction).sum())
        size = float((grads[n].double() * direction).abs().sum())
        # the third derivative along the direction stays below 100 times the first's absolute sum (v, s0, q: linear, no truncation); rounding: the
        # losses' own, some sqrt(outputs) 2^-24 of their absolute sum, over the step
        rounding = 2.0 ** -24 * (float(d["do"].abs().sum()) + float(d["dlast"].abs().sum())) * 20 / step
        assert abs((up - down) / (2 * step) - want) <= step * step / 6 * 100 * size + rounding, (n, (up - down) / (2 * step), want)


def test_refusals():
    q = torch.zeros(2, 8, 2, 4, device=DEV)
    g = torch.zeros(2, 8, 2, device=DEV)
    bad = [
        (1, lambda: deer.matrec_solve(q, q, q, g.half())),
        (1, lambda: deer.matrec_solve(q, q[:, :4], q, g)),
        (1, lambda: deer.matrec_solve(q, q, q[:, :, :1], g[:, :, :1].contiguous())),
        (1, lambda: deer.matrec_solve(q, q, q, g, torch.zeros(2, 2, 4, 5, device=DEV))),
        (1, lambda: deer.matrec_solve(q, q, q.bfloat16(), g)),
        (1, lambda: deer.matrec_solve(q, q, q, g, scale=float("nan"))),
        (1, lambda: deer.matrec_solve(q, q, q, g.transpose(0, 1).contiguous().transpose(0, 1))),
        (1, lambda: deer.matrec_solve(q.transpose(2, 3).contiguous().transpose(2, 3), q, q, g)),
        (2, lambda: deer.matrec_solve(q.half(), q.half(), q.half(), g)),
        (2, lambda: deer.matrec_solve(q.double(), q.double(), q.double(), g)),
        (2, lambda: deer.matrec_solve(*[torch.zeros(1, 4, 1, 129, device=DEV)] * 3, torch.zeros(1, 4, 1, device=DEV))),
        (1, lambda: deer.matrec_grad(q, q, q, g, q, dq=q.half())),
        (1, lambda: deer.matrec_step(q[0], q[0], q[0], g[0], torch.zeros(8, 2, 4, 4, device=DEV), slots=torch.zeros(8, device=DEV))),
        (1, lambda: deer.matrec_step(q[0], q[0], q[0], g[0], torch.zeros(8, 2, 4, 4, device=DEV).bfloat16())),
    ]
    for status, call in bad:
        with pytest.raises(deer.DeerError) as e:
            call()
        assert e.value.status == status


def test_rows_beyond_32_bits():
    T, far = 1100, 1 << 22                                 # 1,100 rows 2^22 elements apart: offsets up to 4.6e9 elements
    d = make("bf16", (T,), 2, 1, 2, 32, 64, 6)
    offsets = torch.tensor([0, 300, T], device=DEV)
    want = both(d, offsets=offsets)
    wide = torch.empty(T, far, dtype=torch.bfloat16, device=DEV)
    e, at = dict(d), 0
    for n in ("q", "k", "v", "do"):
        H, D = d[n].shape[1:]
        e[n] = wide[:, at:at + H * D].unflatten(-1, (H, D))
        e[n].copy_(d[n])
        at += H * D
    grads = {}
    for n, like in (("dq", "q"), ("dk", "k"), ("dv", "v")):
        H, D = d[like].shape[1:]
        grads[n] = wide[:, at:at + H * D].unflatten(-1, (H, D))
        at += H * D
    got = deer.matrec_solve(e["q"], e["k"], e["v"], e["g"], e["s0"], offsets=offsets)
    got += deer.matrec_grad(e["q"], e["k"], e["v"], e["g"], e["do"], e["s0"], e["dlast"], offsets=offsets, **grads)
    for n, a in zip(NAMES, got):
        assert torch.equal(a, want[n]), n


def test_many_sequences_of_a_row_or_none():
    """more cells of states than a launch has work items"""
    N, H, K, V = 16400, 64, 4, 4
    rng = torch.Generator(device="cuda").manual_seed(3)
    lengths = torch.randint(0, 2, (N,), device=DEV, generator=rng)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device=DEV), lengths.cumsum(0)])
    T = int(offsets[-1])
    q, k = torch.randn(T, H, K, device=DEV, generator=rng), torch.randn(T, H, K, device=DEV, generator=rng)
    v, g = torch.randn(T, H, V, device=DEV, generator=rng), -torch.rand(T, H, device=DEV, generator=rng)
    s0 = torch.randn(N, H, K, V, device=DEV, generator=rng)
    o, last = deer.matrec_solve(q, k, v, g, s0, offsets=offsets, scale=1.0)
    want, some = s0.double(), lengths == 1
    want[some] = want[some] * g.double().exp()[..., None, None] + k.double()[..., :, None] * v.double()[..., None, :]
    size = s0.abs().max().double() + k.abs().max() * v.abs().max()
    # two products and a sum, and a factor of 2 units in the last place: five roundings
    assert float((last - want).abs().max()) <= 5 * 2.0 ** -24 * float(size)
    assert torch.equal(last[~some], s0[~some])
    wo = (want[some] * q.double()[..., :, None]).sum(-2)
    assert float((o - wo).abs().max()) <= (5 + 1 + K) * 2.0 ** -24 * K * float(size * q.abs().max())
