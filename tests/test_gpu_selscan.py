"""Selective scan against a row-by-row 64-bit form: batches, packed rows, padded batches, groups, slices, single tokens."""
import numpy as np
import pytest
import torch

import layer_oracle as lo
from paper_2309_12252_amd import deer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def host(t):
    return None if t is None else t.detach().cpu().double().numpy()


def make(dtype, lead, N, D, S, G, gated, seed, softplus=True):
    rng = np.random.default_rng(seed)
    t = lo.TYPES[dtype]
    dev = lambda a, ty=torch.float32: torch.from_numpy(np.asarray(a)).to(ty).to(DEV)   # noqa: E731
    r = rng.standard_normal
    c = {"x": dev(r(lead + (D,)), t), "dt": dev(r(lead + (D,)) if softplus else np.exp(r(lead + (D,)) - 2), t), "A": dev(-np.exp(r((D, S)))),
         "B": dev(r(lead + (G, S)), t), "C": dev(r(lead + (G, S)), t), "skip": dev(r(D)), "z": dev(r(lead + (D,)), t) if gated else None,
         "dt_bias": dev(r(D) - 2 if softplus else 0.01 * np.exp(r(D))), "h0": dev(r((N, D, S))), "dy": dev(r(lead + (D,)), t), "dlast": dev(r((N, D, S)))}
    c["softplus"] = softplus
    return c


NAMES = ("dx", "ddt", "dA", "dB", "dC", "dskip", "dz", "dbias", "dh0")


def run(c, **more):
    about = {"skip": c["skip"], "z": c["z"], "dt_bias": c["dt_bias"], "h0": c["h0"], "softplus": c["softplus"]}
    y, last = deer.selscan_solve(c["x"], c["dt"], c["A"], c["B"], c["C"], **about, **more)
    got = {"y": y, "last": last}
    got.update(zip(NAMES, deer.selscan_grad(c["x"], c["dt"], c["A"], c["B"], c["C"], c["dy"], dlast=c["dlast"], **about, **more)))
    if c["z"] is None:
        assert got.pop("dz") is None
    return got


def compare(c, got, dtype, seqs):
    D, (G, S) = c["x"].shape[-1], c["B"].shape[-2:]
    flat = lambda t, *inner: None if t is None else host(t).reshape((-1,) + inner)   # noqa: E731
    zero = lambda t, like: np.zeros(like) if t is None else host(t)   # noqa: E731
    N = len(seqs)
    want = lo.scan(flat(c["x"], D), flat(c["dt"], D), host(c["A"]), flat(c["B"], G, S), flat(c["C"], G, S), zero(c["skip"], D), flat(c["z"], D), zero(c["dt_bias"], D),
                   zero(c["h0"], (N, D, S)), seqs, c["softplus"], flat(c["dy"], D), zero(c["dlast"], (N, D, S)))
    alive = np.zeros(flat(c["x"], D).shape[0], dtype=bool)
    for r0, L in seqs:
        alive[r0:r0 + L] = True
    at = torch.from_numpy(alive).to(DEV)
    for name, t in got.items():
        w, E = want[name]
        if name in ("y", "dx", "ddt", "dz", "dB", "dC"):
            inner = t.shape[-2:] if name in ("dB", "dC") else t.shape[-1:]
            t, w, E, kind = t.reshape((-1,) + tuple(inner))[at], w[alive], E[alive], dtype
        else:
            kind = "f32"
        lo.check(name, t, w, E, kind)
        # all together: random roundings, half a step of the type over sqrt 3 each, and what 32 bits leave of some hundred rows
        if w.size >= 500 and np.linalg.norm(w) > 0:
            rel = np.linalg.norm(host(t).reshape(w.shape) - w) / np.linalg.norm(w)
            most = (lo.HALF[kind] if kind != "f32" else 0.0) + 64 * 2.0 ** -24
            assert rel <= most, (name, rel, most)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("N,T,D,S,G,gated", [
    (1, 1, 1, 1, 1, True), (2, 2, 3, 4, 1, False), (3, 15, 64, 16, 1, True), (1, 17, 130, 16, 2, True), (2, 33, 66, 7, 3, False), (1, 128, 260, 16, 1, True),
    (1, 129, 68, 8, 1, True), (2, 70, 300, 3, 1, True), (1, 200, 40, 32, 2, False), (2, 100, 36, 64, 3, True), (1, 65, 20, 33, 1, True), (1, 700, 24, 16, 1, True)])
def test_batch(dtype, N, T, D, S, G, gated):
    c = make(dtype, (N, T), N, D, S, G, gated, N * 1000 + T + D + S)
    compare(c, run(c), dtype, lo.sequences(T, N))


PACKED = {"mixed": [0, 130, 131, 131, 400, 401, 700, 700], "tokens": list(range(0, 41)), "behind": [3, 3, 20, 150, 260], "one": [0, 449], "empty": [0, 0, 0],
          "edges": [0, 16, 32, 64, 65, 128, 192]}


@pytest.mark.parametrize("dtype,D,S,G,gated", [("bf16", 68, 16, 1, True), ("f32", 30, 5, 2, False), ("f16", 16, 40, 1, True), ("f32", 70, 3, 1, True)])
@pytest.mark.parametrize("name", list(PACKED))
def test_packed(name, dtype, D, S, G, gated):
    off = PACKED[name]
    N, rows = len(off) - 1, off[-1] + 9
    c = make(dtype, (rows,), N, D, S, G, gated, 7)
    by_row = [k for k in ("x", "dt", "B", "C", "z", "dy") if c[k] is not None]
    for k in by_row:   # what belongs to no sequence is never looked at
        c[k][:off[0]] = float("nan")
        c[k][off[-1]:] = float("inf")
    offsets = torch.tensor(off, dtype=torch.int64, device=DEV)
    got = run(c, offsets=offsets)
    about = {"skip": c["skip"], "z": c["z"], "dt_bias": c["dt_bias"], "h0": c["h0"], "offsets": offsets}
    into = {"d" + k: torch.full_like(c[k], 7.0) for k in ("x", "dt", "B", "C", "z") if c[k] is not None}
    y, _ = deer.selscan_solve(c["x"], c["dt"], c["A"], c["B"], c["C"], out=torch.full_like(c["x"], 7.0), **about)
    deer.selscan_grad(c["x"], c["dt"], c["A"], c["B"], c["C"], c["dy"], dlast=c["dlast"], **about, **into)
    for name, t in dict(into, y=y).items():
        plain = got[name]
        assert bool((t[off[-1]:] == 7).all()) and bool((t[:off[0]] == 7).all()), name
        assert bool((plain[off[-1]:] == 0).all()) and bool((plain[:off[0]] == 0).all()), name
        assert torch.equal(t[off[0]:off[-1]], plain[off[0]:off[-1]]), name
    for k in by_row:
        c[k].nan_to_num_(0.0, 0.0, 0.0)
    compare(c, got, dtype, lo.sequences(rows, N, offsets=off))


@pytest.mark.parametrize("dtype,S,G", [("bf16", 16, 1), ("f32", 10, 2)])
def test_padded_batch(dtype, S, G):
    N, T, D, lens = 6, 300, 36, [300, 0, 1, 129, 256, 64]
    c = make(dtype, (N, T), N, D, S, G, True, 3)
    for n, L in enumerate(lens):
        for k in ("x", "dt", "B", "C", "z", "dy"):
            c[k][n, L:] = float("nan")
    got = run(c, lengths=torch.tensor(lens, dtype=torch.int64, device=DEV))
    for n, L in enumerate(lens):
        for k in ("y", "dx", "ddt", "dB", "dC", "dz"):
            assert bool((got[k][n, L:] == 0).all()), k
    for k in ("x", "dt", "B", "C", "z", "dy"):
        c[k].nan_to_num_(0.0, 0.0, 0.0)
    compare(c, got, dtype, lo.sequences(T, N, lengths=lens))


@pytest.mark.parametrize("dtype,D,S", [("bf16", 128, 16), ("f32", 33, 4), ("f16", 66, 9)])
def test_slices_of_projections(dtype, D, S):
    """x and z halves of one array, dt, B and C parts of another; no skip, no bias, no states"""
    N, T = 2, 150
    c = make(dtype, (N, T), N, D, S, 1, True, 5)
    one = torch.cat([c["x"], c["z"]], -1).contiguous()
    two = torch.cat([c["dt"], c["B"].flatten(-2), c["C"].flatten(-2)], -1).contiguous()
    x, z, dt = one[..., :D], one[..., D:], two[..., :D]
    B, C = two[..., D:D + S].unflatten(-1, (1, S)), two[..., D + S:].unflatten(-1, (1, S))
    y, last = deer.selscan_solve(x, dt, c["A"], B, C, z=z)
    got = dict({"y": y, "last": last}, **dict(zip(NAMES, deer.selscan_grad(x, dt, c["A"], B, C, c["dy"], z=z))))
    for k, of in (("dx", x), ("dz", z), ("ddt", dt), ("dB", B), ("dC", C)):
        assert got[k].stride()[:2] == of.stride()[:2] and got[k].shape == of.shape
    c.update(skip=None, dt_bias=None, h0=None, dlast=None)
    compare(c, got, dtype, lo.sequences(T, N))
    # into parts of wider arrays
    done, dtwo = torch.zeros_like(one), torch.zeros_like(two)
    deer.selscan_grad(x, dt, c["A"], B, C, c["dy"], z=z, dx=done[..., :D], dz=done[..., D:], ddt=dtwo[..., :D], dB=dtwo[..., D:D + S].unflatten(-1, (1, S)),
                      dC=dtwo[..., D + S:].unflatten(-1, (1, S)))
    assert torch.equal(done, torch.cat([got["dx"], got["dz"]], -1))
    assert torch.equal(dtwo, torch.cat([got["ddt"], got["dB"].flatten(-2), got["dC"].flatten(-2)], -1))


@pytest.mark.parametrize("dtype,S", [("f32", 16), ("bf16", 5)])
def test_steps_as_they_are(dtype, S):
    """without softplus: dt is the step"""
    c = make(dtype, (2, 90), 2, 20, S, 1, True, 21, softplus=False)
    compare(c, run(c), dtype, lo.sequences(90, 2))


def test_steps_far_out():
    """steps whose softplus is all but zero, or all but the number itself, and rates that forget all at once"""
    c = make("f32", (1, 200), 1, 24, 16, 1, True, 4)
    c["dt"][0, ::5] = -40.0
    c["dt"][0, 3::7] = 30.0
    c["A"][:, 0] = -1e4
    c["A"][:, 1] = 0.0
    got = run(c)
    for t in got.values():
        assert bool(torch.isfinite(t).all())
    compare(c, got, "f32", lo.sequences(200, 1))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("D,S,G", [(70, 16, 1), (12, 1, 1), (40, 8, 4), (9, 30, 3), (20, 64, 2), (130, 6, 1)])
def test_tokens_go_on_where_a_prompt_ends(dtype, D, S, G):
    N, T, more = 3, 20, 5
    c = make(dtype, (N, T + more), N, D, S, G, True, 11)
    about = {"skip": c["skip"], "dt_bias": c["dt_bias"]}
    first = {k: c[k][:, :T].contiguous() for k in ("x", "dt", "B", "C", "z")}
    y, state = deer.selscan_solve(first["x"], first["dt"], c["A"], first["B"], first["C"], z=first["z"], h0=c["h0"], **about)
    pool = torch.full((N + 4, D, S), 9.0, device=DEV)
    slots = torch.tensor([5, 0, 3], dtype=torch.int32, device=DEV)
    pool[slots.long()] = state
    ys = [y]
    for t in range(T, T + more):
        now = {k: c[k][:, t].contiguous() for k in ("x", "dt", "B", "C", "z")}
        ys.append(deer.selscan_step(now["x"], now["dt"], c["A"], now["B"], now["C"], pool, z=now["z"], slots=slots, **about)[:, None])
    compare(c, {"y": torch.cat(ys, 1), "last": pool[slots.long()]}, dtype, lo.sequences(T + more, N))
    assert bool((pool[[i for i in range(N + 4) if i not in (5, 0, 3)]] == 9).all())


def test_step_passes_over_bad_and_repeated_slots():
    N, D, S = 6, 300, 16
    c = make("bf16", (N,), N, D, S, 1, True, 2)
    pool = torch.randn(4, D, S, device=DEV)
    before = pool.clone()
    slots = torch.tensor([2, -1, 4, 0, 2, 1], dtype=torch.int32, device=DEV)
    args = (c["x"], c["dt"], c["A"], c["B"], c["C"])
    y = deer.selscan_step(*args, pool, z=c["z"], slots=slots)
    kept = deer.selscan_step(*args, before.clone(), z=c["z"], slots=slots, out=torch.full_like(y, 3.0))
    for n, slot in enumerate([2, None, None, 0, None, 1]):
        if slot is None:
            assert bool((y[n] == 0).all()) and bool((kept[n] == 3).all())
            continue
        one = {k: c[k][n:n + 1] for k in ("x", "dt", "B", "C", "z")}
        alone = before[slot:slot + 1].clone()
        assert torch.equal(deer.selscan_step(one["x"], one["dt"], c["A"], one["B"], one["C"], alone, z=one["z"])[0], y[n]) and torch.equal(kept[n], y[n])
        assert torch.equal(pool[slot], alone[0])
    assert torch.equal(pool[3], before[3])


def test_not_finite_stays_in_its_sequence_and_channel():
    off = torch.tensor([0, 150, 300, 500], device=DEV)
    c = make("f32", (500,), 3, 40, 16, 1, True, 1)
    clean = run(c, offsets=off)
    c["x"][200, 7] = float("nan")
    got = run(c, offsets=off)
    for name in ("y", "dx", "ddt", "dz"):
        same = got[name] == clean[name]
        same[150:300, 7] = True
        assert bool(same.all()), name
    assert bool(torch.isnan(got["y"][200:300, 7]).all())
    for name in ("dB", "dC"):   # sums over the channels
        assert torch.equal(got[name][:150], clean[name][:150]) and torch.equal(got[name][300:], clean[name][300:])
    for name in ("last", "dh0"):
        same = (got[name] == clean[name]).flatten(2).all(-1)
        same[1, 7] = True
        assert bool(same.all()), name


def test_gradient_against_differences():
    """central differences of L = <y, dy> + <last, dlast> in the arguments, in directions: h^2 and 2^-24 / h of sizes of a few hundred"""
    c = make("f32", (2, 60), 2, 12, 16, 2, True, 13)
    got = run(c)
    rng = np.random.default_rng(3)

    def loss(c):
        about = {"skip": c["skip"], "z": c["z"], "dt_bias": c["dt_bias"], "h0": c["h0"]}
        y, last = deer.selscan_solve(c["x"], c["dt"], c["A"], c["B"], c["C"], **about)
        return float((y.double() * c["dy"].double()).sum() + (last.double() * c["dlast"].double()).sum())

    for k, name in (("x", "dx"), ("dt", "ddt"), ("A", "dA"), ("B", "dB"), ("C", "dC"), ("skip", "dskip"), ("z", "dz"), ("dt_bias", "dbias"), ("h0", "dh0")):
        v = torch.from_numpy(rng.standard_normal(tuple(c[k].shape))).float().to(DEV)
        h = 2.0 ** -8
        up, down = dict(c), dict(c)
        up[k], down[k] = c[k] + h * v, c[k] - h * v
        want, have = (loss(up) - loss(down)) / (2 * h), float((got[name].double() * v.double()).sum())
        size = float((got[name].double() * v.double()).abs().sum())
        assert abs(want - have) <= 2e-3 * size + 1e-2, (name, want, have, size)


def test_empty_arrays():
    c = make("f32", (2, 0), 2, 10, 16, 1, False, 4)
    got = run(c)
    assert got["y"].shape == (2, 0, 10) and torch.equal(got["last"], c["h0"]) and torch.equal(got["dh0"], c["dlast"])
    assert bool((got["dA"] == 0).all()) and bool((got["dskip"] == 0).all())


@pytest.mark.parametrize("N,D,S", [(64, 128, 64), (256, 512, 4)])
def test_many_whole_sequences(N, D, S):
    """as many workgroups as there need be without a cut: the same call with lengths is cut"""
    T = 130
    c = make("f32", (N, T), N, D, S, 1, True, 17)
    whole, cut = run(c), run(c, lengths=torch.full((N,), T, dtype=torch.int64, device=DEV))
    compare(c, whole, "f32", lo.sequences(T, N))
    compare(c, cut, "f32", lo.sequences(T, N))
