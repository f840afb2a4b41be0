"""Gated linear recurrences with a state for every channel, and dropout, against row-by-row 64-bit forms."""
import numpy as np
import pytest
import torch

import seq_oracle as so
from paper_2309_12252_amd import deer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = {"factor": deer.DEER_GATE_FACTOR, "log": deer.DEER_GATE_LOG, "sigmoid": deer.DEER_GATE_SIGMOID}


def host(t):
    return t.detach().cpu().double().numpy()


def make(kind, dtype, lead, N, D, seed):
    rng = np.random.default_rng(seed)
    g = rng.standard_normal(lead + (D,))
    if kind == "sigmoid":
        g = 1.0 + 2.0 * g
    else:
        g = -np.exp(1.2 * g - 2.0)
        if kind == "factor":
            g = np.exp(g) * rng.choice([1.0, 1.0, -1.0], size=g.shape)
    t, w = so.TYPES[dtype], torch.float64 if dtype == "f64" else torch.float32
    dev = lambda a, ty: torch.from_numpy(a).to(ty).to(DEV)   # noqa: E731
    return (dev(g, t), dev(rng.standard_normal(lead + (D,)), t), dev(rng.standard_normal((N, D)), w), dev(rng.standard_normal(lead + (D,)), t),
            dev(rng.standard_normal((N, D)), w))


def compare(kind, dtype, gate, x, h0, dh, dlast, seqs, got, keep=None):
    """got: h, last, dgate, dx, dh0 of the library"""
    D, k, c_u = x.shape[-1], KINDS[kind], so.ROUNDINGS[dtype] * so.UNIT[dtype]
    flat = lambda t: host(t).reshape(-1, D)   # noqa: E731
    h, last, dgate, dx, dh0 = got
    g, xs = flat(gate), flat(x)
    xd = xs if keep is None else xs * keep.reshape(-1, D)
    zero = np.zeros((len(seqs), D))
    H0, DL = (zero if h0 is None else host(h0)), (zero if dlast is None else host(dlast))
    alive = np.zeros(g.shape[0], dtype=bool)
    for r0, length in seqs:
        alive[r0:r0 + length] = True
    wide = "f64" if dtype == "f64" else "f32"
    wh, wl, E, El = so.diag_forward(k, g, xd, H0, seqs, c_u)
    so.check("h", h.reshape(-1, D)[torch.from_numpy(alive).to(h.device)], wh[alive], E[alive], dtype)
    so.check("last", last, wl, El, wide)
    if dgate is None:
        return
    wg, wx, w0, Eg, Ex, E0 = so.diag_backward(k, g, xd, flat(h), flat(dh), H0, DL, seqs, c_u)
    if keep is not None:
        wx, Ex = wx * keep.reshape(-1, D), Ex * keep.reshape(-1, D) + c_u * np.abs(wx * keep.reshape(-1, D))
    at = torch.from_numpy(alive).to(h.device)
    so.check("dgate", dgate.reshape(-1, D)[at], wg[alive], Eg[alive], dtype)
    so.check("dx", dx.reshape(-1, D)[at], wx[alive], Ex[alive], dtype)
    so.check("dh0", dh0, w0, E0, wide)


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16", "f16"])
@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("N,T,D", [(1, 1, 1), (2, 2, 3), (3, 15, 64), (1, 17, 130), (2, 127, 66), (1, 128, 256), (1, 129, 65), (2, 385, 132), (1, 4200, 70)])
def test_batch(kind, dtype, N, T, D):
    gate, x, h0, dh, dlast = make(kind, dtype, (N, T), N, D, N * 1000 + T + D)
    h, last = deer.diagrec_solve(gate, x, h0, kind=KINDS[kind])
    back = deer.diagrec_grad(gate, x, h, dh, h0, dlast, kind=KINDS[kind])
    compare(kind, dtype, gate, x, h0, dh, dlast, so.sequences(T, N), (h, last) + back)


PACKED = {"mixed": [0, 130, 131, 131, 500, 501, 4100, 4100], "tokens": list(range(0, 41)), "behind": [3, 3, 20, 150, 260], "one": [0, 2049], "empty": [0, 0, 0]}


@pytest.mark.parametrize("dtype,kind,D", [("bf16", "sigmoid", 132), ("f32", "log", 67), ("f64", "factor", 5), ("f16", "log", 96)])
@pytest.mark.parametrize("name", list(PACKED))
def test_packed(name, dtype, kind, D):
    off = PACKED[name]
    N, rows = len(off) - 1, off[-1] + 9      # nine rows behind the last sequence
    gate, x, h0, dh, dlast = make(kind, dtype, (rows,), N, D, 7)
    offsets = torch.tensor(off, dtype=torch.int64, device=DEV)
    mark = torch.full_like(x, 7.0)
    h, last = deer.diagrec_solve(gate, x, h0, kind=KINDS[kind], offsets=offsets, out=mark.clone())
    dgate, dx, dh0 = deer.diagrec_grad(gate, x, h, dh, h0, dlast, kind=KINDS[kind], offsets=offsets, dgate=mark.clone(), dx=mark.clone())
    for t in (h, dgate, dx):   # rows of no sequence are left as they were
        assert bool((t[off[-1]:] == 7).all()) and bool((t[:off[0]] == 7).all())
    compare(kind, dtype, gate, x, h0, dh, dlast, so.sequences(rows, N, offsets=off), (h, last, dgate, dx, dh0))


@pytest.mark.parametrize("dtype,kind", [("bf16", "log"), ("f32", "sigmoid")])
def test_padded_batch(dtype, kind):
    N, T, D, lens = 5, 300, 70, [300, 0, 1, 129, 256]
    gate, x, h0, dh, dlast = make(kind, dtype, (N, T), N, D, 3)
    for n, L in enumerate(lens):   # what lies behind a sequence's end is never looked at
        gate[n, L:], x[n, L:], dh[n, L:] = float("nan"), float("inf"), float("nan")
    lengths = torch.tensor(lens, dtype=torch.int64, device=DEV)
    h, last = deer.diagrec_solve(gate, x, h0, kind=KINDS[kind], lengths=lengths, out=torch.full_like(x, 3.0))
    dgate, dx, dh0 = deer.diagrec_grad(gate, x, h, dh, h0, dlast, kind=KINDS[kind], lengths=lengths, dgate=torch.full_like(x, 3.0), dx=torch.full_like(x, 3.0))
    for n, L in enumerate(lens):
        for t in (h, dgate, dx):
            assert bool((t[n, L:] == 3).all())
    for t in (gate, x, dh):
        t.nan_to_num_(0.0, 0.0, 0.0)
    compare(kind, dtype, gate, x, h0, dh, dlast, so.sequences(T, N, lengths=lens), (h, last, dgate, dx, dh0))


@pytest.mark.parametrize("dtype,kind,D", [("bf16", "sigmoid", 128), ("f32", "factor", 33), ("bf16", "log", 65)])
def test_slices_of_a_projection(dtype, kind, D):
    # gate and x are halves of one array, h and dh have rows of their own length
    N, T = 2, 200
    gate, x, h0, dh, dlast = make(kind, dtype, (N, T), N, D, 5)
    both = torch.cat([gate, x], -1).contiguous()
    gs, xs = both[..., :D], both[..., D:]
    wide = torch.zeros(N, T, D + 5, dtype=x.dtype, device=DEV)
    h, last = deer.diagrec_solve(gs, xs, h0, kind=KINDS[kind], out=wide[..., :D])
    assert h.data_ptr() == wide.data_ptr() and bool((wide[..., D:] == 0).all())
    dboth = torch.empty_like(both)
    back = deer.diagrec_grad(gs, xs, h, dh, h0, dlast, kind=KINDS[kind], dgate=dboth[..., :D], dx=dboth[..., D:])
    compare(kind, dtype, gate, x, h0, dh, dlast, so.sequences(T, N), (h, last) + back)
    plain = deer.diagrec_grad(gs, xs, h, dh, h0, dlast, kind=KINDS[kind])
    for p, q in zip(plain, back):
        assert torch.equal(p, q)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("dtype,packed", [("bf16", True), ("f32", False), ("f64", True)])
def test_dropout_inside(kind, dtype, packed):
    T, D, p, seed = 333, 66, 0.3, (5 << 32) + 77
    N = 1 if packed else 2
    gate, x, h0, dh, dlast = make(kind, dtype, (T,) if packed else (N, T), 3 if packed else N, D, 9)
    off = [0, 100, 101, T]
    more = {"kind": KINDS[kind], "drop": p, "seed": seed, "draw": 12}
    if packed:
        more["offsets"] = torch.tensor(off, dtype=torch.int64, device=DEV)
    h, last = deer.diagrec_solve(gate, x, h0, **more)
    back = deer.diagrec_grad(gate, x, h, dh, h0, dlast, **more)
    keep = so.philox_keep(N, T, D, p, seed, 12)
    seqs = so.sequences(T, 3, offsets=off) if packed else so.sequences(T, N)
    compare(kind, dtype, gate, x, h0, dh, dlast, seqs, (h, last) + back, keep=keep)
    # the same mask as the operator alone
    alone = host(deer.dropout(torch.ones_like(x), p, seed, 12)).reshape(keep.shape)
    assert np.array_equal(alone != 0, keep != 0)


@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16", "f16"])
@pytest.mark.parametrize("N,T,D", [(1, 1, 1), (2, 7, 3), (1, 8, 4), (3, 9, 16), (2, 1001, 18), (1, 70, 1030)])
def test_dropout(dtype, N, T, D):
    rng = np.random.default_rng(1)
    x = torch.from_numpy(rng.standard_normal((N, T, D))).to(so.TYPES[dtype]).to(DEV)
    y = deer.dropout(x, 0.25, 123456789, 3)
    keep = so.philox_keep(N, T, D, 0.25, 123456789, 3)
    want = host(x) * keep
    # one product in the wide type and one rounding
    so.check("y", y, want, so.UNIT[dtype] * np.abs(want), dtype)
    assert np.array_equal(host(y) == 0, (keep == 0) | (host(x) == 0))
    assert torch.equal(deer.dropout(x, 0.0, 5), x)
    z = x.clone()
    assert deer.dropout(z, 0.25, 123456789, 3, out=z) is z and torch.equal(z, y)
    if N == 1:
        assert torch.equal(deer.dropout(x[0], 0.25, 123456789, 3), y[0])
    if N * T * D > 2000:   # a share of 1/4 within five deviations, and other masks for other draws
        n, k = keep.size, int((keep == 0).sum())
        assert abs(k - n / 4) < 5 * (n * 3 / 16) ** 0.5
        assert not torch.equal(deer.dropout(x, 0.25, 123456789, 4), y) and not torch.equal(deer.dropout(x, 0.25, 123456790, 3), y)


def test_dropout_drops_what_is_not_finite_and_keeps_infinities():
    x = torch.full((1, 64, 8), float("inf"), device=DEV)
    y = deer.dropout(x, 0.5, 9)
    keep = torch.from_numpy(so.philox_keep(1, 64, 8, 0.5, 9, 0) != 0).to(DEV)
    assert bool((y[keep] == float("inf")).all()) and bool((y[~keep] == 0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_states_and_empty_arrays(dtype):
    gate, x, _, dh, _ = make("log", dtype, (2, 40), 2, 10, 4)
    h, last = deer.diagrec_solve(gate, x, kind=1)
    compare("log", dtype, gate, x, None, dh, None, so.sequences(40, 2), (h, last) + deer.diagrec_grad(gate, x, h, dh, kind=1))
    none = torch.empty(2, 0, 10, dtype=x.dtype, device=DEV)
    h0 = torch.randn(2, 10, device=DEV)
    h, last = deer.diagrec_solve(none, none, h0)
    assert h.shape == (2, 0, 10) and torch.equal(last, h0)
    assert torch.equal(deer.diagrec_grad(none, none, none, none, h0, h0)[2], h0)
    assert deer.dropout(none, 0.5, 1).shape == none.shape


def test_hard_gates():
    # a log gate of -inf and a sigmoid gate of -inf forget all, +inf of the sigmoid keeps all and takes nothing
    N, T, D = 1, 300, 64
    for kind, lo, hi in (("log", -float("inf"), 0.0), ("sigmoid", -float("inf"), float("inf"))):
        gate, x, h0, dh, dlast = make(kind, "f32", (N, T), N, D, 8)
        gate[0, ::7] = lo
        gate[0, 3::11] = hi
        h, last = deer.diagrec_solve(gate, x, h0, kind=KINDS[kind])
        back = deer.diagrec_grad(gate, x, h, dh, h0, dlast, kind=KINDS[kind])
        compare(kind, "f32", gate, x, h0, dh, dlast, so.sequences(T, N), (h, last) + back)


def test_not_finite_stays_in_its_sequence_and_channel():
    off = [0, 700, 1400, 5000]
    gate, x, h0, dh, dlast = make("log", "f32", (5000,), 3, 70, 2)
    clean, clast = deer.diagrec_solve(gate, x, h0, kind=1, offsets=torch.tensor(off, device=DEV))
    x2 = x.clone()
    x2[900, 5], x2[800, 6] = float("nan"), float("inf")
    # a NaN with all bits set, which the tiles' words use as a mark
    x2[910, 7] = torch.tensor(-1, dtype=torch.int32).view(torch.float32).item()
    x2.view(torch.int32)[910, 7] = -1
    h, last = deer.diagrec_solve(gate, x2, h0, kind=1, offsets=torch.tensor(off, device=DEV))
    assert bool(torch.isnan(h[900:1400, 5]).all()) and bool(torch.isnan(h[910:1400, 7]).all()) and not bool(torch.isfinite(h[800:1400, 6]).any())
    ok = torch.ones_like(h, dtype=torch.bool)
    ok[900:1400, 5] = ok[910:1400, 7] = ok[800:1400, 6] = False
    assert torch.equal(h[ok], clean[ok])
    assert torch.equal(last[[0, 2]], clast[[0, 2]])


def test_in_place_and_the_same_bits_again():
    gate, x, h0, dh, dlast = make("sigmoid", "bf16", (1, 9000), 1, 256, 6)
    h, last = deer.diagrec_solve(gate, x, h0, kind=2)
    first = deer.diagrec_grad(gate, x, h, dh, h0, dlast, kind=2)
    for _ in range(3):
        y = x.clone()
        h2, last2 = deer.diagrec_solve(gate, y, h0, kind=2, out=y)
        assert h2 is y and torch.equal(h2, h) and torch.equal(last2, last)
        for p, q in zip(first, deer.diagrec_grad(gate, x, h, dh, h0, dlast, kind=2)):
            assert torch.equal(p, q)


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16", "f16"])
@pytest.mark.parametrize("N,D", [(1, 1), (3, 65), (40, 300)])
def test_step(kind, dtype, N, D):
    gate, x, _, _, _ = make(kind, dtype, (N,), N, D, 21)
    state = torch.randn(N + 3, D, dtype=torch.float64 if dtype == "f64" else torch.float32, device=DEV)
    slots = torch.randperm(N + 3)[:N].to(torch.int32)
    before = state.clone()
    h = deer.diagrec_step(gate, x, state, kind=KINDS[kind], slots=slots.to(DEV))
    c_u = so.ROUNDINGS[dtype] * so.UNIT[dtype]
    want, last, E, El = so.diag_forward(KINDS[kind], host(gate), host(x), host(before)[slots.numpy()], [(n, 1) for n in range(N)], c_u)
    so.check("h", h, want, E, dtype)
    so.check("state", state[slots.long().to(DEV)], last, El, "f64" if dtype == "f64" else "f32")
    rest = [s for s in range(N + 3) if s not in slots.tolist()]
    assert torch.equal(state[rest], before[rest])


def test_step_passes_over_bad_and_repeated_slots():
    gate, x, _, _, _ = make("log", "f32", (6,), 6, 300, 1)
    state = torch.randn(4, 300, device=DEV)
    before, out = state.clone(), torch.full_like(x, 9.0)
    slots = torch.tensor([2, -1, 4, 2, 0, 2000000000], dtype=torch.int32, device=DEV)
    deer.diagrec_step(gate, x, state, kind=1, slots=slots, out=out)
    for n in (1, 2, 3, 5):
        assert bool((out[n] == 9).all())
    for n, s in ((0, 2), (4, 0)):
        want = torch.exp(gate[n].double()) * before[s].double() + x[n].double()
        assert float((state[s].double() - want).abs().max()) <= 8 * 2.0 ** -24 * float(want.abs().max() + before.abs().max())
        assert torch.equal(out[n], state[s])
    assert torch.equal(state[[1, 3]], before[[1, 3]])


def test_steps_continue_a_prompt():
    # a prompt, then tokens one by one: the same as the whole sequence at once
    N, T, D, more = 3, 200, 96, 5
    gate, x, h0, _, _ = make("sigmoid", "f32", (N, T + more), N, D, 11)
    whole, last = deer.diagrec_solve(gate, x, h0, kind=2)
    _, state = deer.diagrec_solve(gate[:, :T].contiguous(), x[:, :T].contiguous(), h0, kind=2)
    for t in range(T, T + more):
        h = deer.diagrec_step(gate[:, t].contiguous(), x[:, t].contiguous(), state, kind=2)
        assert float((h - whole[:, t]).abs().max()) <= 2 * 12 * 2.0 ** -24 * 20 * float(whole.abs().max())
    # (both sides within the bound of the oracle: sums of a geometric series of ratio below 0.95, i.e. 20 terms)


def test_another_stream_and_two_at_once():
    args = [make("log", "bf16", (1, 20000), 1, 512, s) for s in (1, 2)]
    want = [deer.diagrec_solve(a[0], a[1], a[2], kind=1) for a in args]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for _ in range(4):
        for s, a in zip(streams, args):
            got.append(deer.diagrec_solve(a[0], a[1], a[2], kind=1, stream=s))
    torch.cuda.synchronize()
    for i, (h, last) in enumerate(got):
        assert torch.equal(h, want[i % 2][0]) and torch.equal(last, want[i % 2][1])


def test_captured():
    gate, x, h0, dh, dlast = make("sigmoid", "bf16", (1, 5000), 1, 256, 13)

    def step():
        h, last = deer.diagrec_solve(gate, x, h0, kind=2, drop=0.2, seed=4)
        return (h, last) + deer.diagrec_grad(gate, x, h, dh, h0, dlast, kind=2, drop=0.2, seed=4) + (deer.dropout(h, 0.1, 6),)

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
    for k in range(4):
        x.copy_(torch.randn(x.shape, device=DEV))
        for graph, out in zip(graphs, outs):
            for t in out:
                t.fill_(5)
            graph.replay()
        torch.cuda.synchronize()
        want = step()
        for out in outs:
            for a, b in zip(out, want):
                assert torch.equal(a, b)


def test_gradient_by_differences():
    # d(loss)/d(parameter) of the library's own forward pass in 64 bits
    N, T, D, p = 2, 9, 3, 0.25
    for kind in KINDS:
        gate, x, h0, dh, dlast = make(kind, "f64", (N, T), N, D, 15)
        more = {"kind": KINDS[kind], "drop": p, "seed": 3}

        def loss():
            h, last = deer.diagrec_solve(gate, x, h0, **more)
            return float((h * dh).sum() + (last * dlast).sum())

        h, _ = deer.diagrec_solve(gate, x, h0, **more)
        for t, d in zip((gate, x, h0), deer.diagrec_grad(gate, x, h, dh, h0, dlast, **more)):
            flat, step = t.view(-1), 1e-5
            for i in range(0, flat.numel(), 5):
                keep = float(flat[i])
                flat[i] = keep + step
                up = loss()
                flat[i] = keep - step
                down = loss()
                flat[i] = keep
                # truncation step^2 / 6 times the third derivative (below 100 here), rounding 2^-53 |loss| / step
                assert abs((up - down) / (2 * step) - float(d.reshape(-1)[i])) < 1e-10 / 6 * 100 + 2.0 ** -53 * 100 / step


def test_refusals():
    x = torch.zeros(2, 8, 4, device=DEV)
    bad = [
        lambda: deer.diagrec_solve(x, x.half()),
        lambda: deer.diagrec_solve(x, x[:, :4]),
        lambda: deer.diagrec_solve(x, x, torch.zeros(2, 5, device=DEV)),
        lambda: deer.diagrec_solve(x, x, torch.zeros(2, 4, device=DEV).double()),
        lambda: deer.diagrec_solve(x, x, kind=3),
        lambda: deer.diagrec_solve(x, x, drop=1.0),
        lambda: deer.diagrec_solve(x, x, drop=float("nan")),
        lambda: deer.diagrec_solve(x, x, lengths=torch.tensor([1, 2], dtype=torch.int32, device=DEV)),
        lambda: deer.diagrec_solve(x[0], x[0], offsets=torch.tensor([0], device=DEV)),
        lambda: deer.diagrec_solve(x, x, offsets=torch.tensor([0, 8], device=DEV)),
        lambda: deer.diagrec_solve(x.transpose(1, 2), x.transpose(1, 2)),
        lambda: deer.diagrec_solve(x.transpose(0, 1), x.transpose(0, 1)),
        lambda: deer.diagrec_solve(x[:, :1].expand(2, 8, 4), x),
        lambda: deer.diagrec_solve(x.int(), x.int()),
        lambda: deer.diagrec_step(x[0], x[0], x[0].half()),
        lambda: deer.diagrec_step(x[0], x[0], x[0], slots=torch.zeros(8, dtype=torch.int64, device=DEV)),
        lambda: deer.dropout(x, -0.1, 1),
        lambda: deer.dropout(x, 0.9999999, 1),
        lambda: deer.diagrec_grad(x, x, x, x, dgate=x.half()),
    ]
    for call in bad:
        with pytest.raises(deer.DeerError) as e:
            call()
        assert e.value.status == deer.DEER_ERR_INVALID_ARG


def test_inputs_given_up_while_another_stream_reads_them():
    gate, x, h0 = make("sigmoid", "bf16", (1, 4000), 1, 512, 21)[:3]
    want = deer.diagrec_solve(gate=gate, x=x, h0=h0, kind=2)[0]
    side = torch.cuda.Stream()
    mine = x.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    got = deer.diagrec_solve(gate, mine, h0, kind=2, stream=side)[0]
    del mine
    other = [torch.full_like(x, 7.0) for _ in range(4)]   # would take the memory of `mine` on this stream, with nothing to wait for
    torch.cuda.synchronize()
    assert torch.equal(got, want) and len(other) == 4


def test_rows_beyond_32_bits():
    T, far = 1100, 1 << 22                                 # 1,100 rows 2^22 elements apart: offsets up to 4.6e9 elements
    gate, x, h0, dh, dlast = make("sigmoid", "bf16", (T,), 2, 128, 22)
    offsets = torch.tensor([0, 700, T], device=DEV)
    h, last = deer.diagrec_solve(gate, x, h0, kind=2, offsets=offsets)
    want = (h, last) + deer.diagrec_grad(gate, x, h, dh, h0, dlast, kind=2, offsets=offsets) + (deer.dropout(x, 0.3, 5),)
    wide = torch.empty(T, far, dtype=torch.bfloat16, device=DEV)
    g, u, d, y, dg, du, z = (wide[:, 128 * i:128 * i + 128] for i in range(7))
    for a, b in ((g, gate), (u, x), (d, dh)):
        a.copy_(b)
    got = deer.diagrec_solve(g, u, h0, kind=2, offsets=offsets, out=y)
    got += deer.diagrec_grad(g, u, y, d, h0, dlast, kind=2, offsets=offsets, dgate=dg, dx=du) + (deer.dropout(u, 0.3, 5, out=z),)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
