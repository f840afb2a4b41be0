"""Group norm with an activation and a gate against a 64-bit form: statistics over rows and over sequences."""
import numpy as np
import pytest
import torch

import layer_oracle as lo
from paper_2309_12252_amd import deer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-5


def host(t):
    return None if t is None else t.detach().cpu().double().numpy()


def make(dtype, lead, D, gated, seed):
    rng = np.random.default_rng(seed)
    t, w = lo.TYPES[dtype], torch.float64 if dtype == "f64" else torch.float32
    dev = lambda a, ty: torch.from_numpy(a).to(ty).to(DEV)   # noqa: E731
    r = rng.standard_normal
    return {"x": dev(r(lead + (D,)) + 2 * r(D), t), "w": dev(1 + 0.5 * r(D), w), "bias": dev(r(D), w), "z": dev(r(lead + (D,)), t) if gated else None,
            "dy": dev(r(lead + (D,)), t)}


def run(c, G, by_row, silu, **more):
    about = {"z": c["z"], "span": deer.DEER_SPAN_ROW if by_row else deer.DEER_SPAN_SEQUENCE, "act": deer.DEER_ACT_SILU if silu else deer.DEER_ACT_NONE}
    y, stats = deer.groupnorm_solve(c["x"], G, c["w"], c["bias"], eps=EPS, **about, **more)
    dx, dw, dbias, dz = deer.groupnorm_grad(c["x"], G, stats, c["dy"], c["w"], c["bias"], **about, **more)
    got = {"y": y, "stats": stats, "dx": dx, "dw": dw, "dbias": dbias}
    if c["z"] is None:
        assert dz is None
    else:
        got["dz"] = dz
    return got


def compare(c, got, G, by_row, silu, dtype, seqs, w=None, bias=None):
    D = c["x"].shape[-1]
    flat = lambda t: None if t is None else host(t).reshape(-1, D)   # noqa: E731
    want = lo.norm(flat(c["x"]), G, host(c["w"]) if w is None else w, host(c["bias"]) if bias is None else bias, flat(c["z"]), seqs, by_row, EPS, silu, lo.U[dtype], flat(c["dy"]))
    alive = np.zeros(flat(c["x"]).shape[0], dtype=bool)
    for r0, L in seqs:
        alive[r0:r0 + L] = True
    at = torch.from_numpy(alive).to(DEV)
    wide = "f64" if dtype == "f64" else "f32"
    for name, t in got.items():
        w, E = want[name]
        if name in ("y", "dx", "dz"):
            lo.check(name, t.reshape(-1, D)[at], w[alive], E[alive], dtype)
        elif name == "stats" and by_row:
            lo.check(name, t.reshape(-1, G, 2)[at], w[alive], E[alive], wide)
        else:
            lo.check(name, t, w, E, wide)


@pytest.mark.parametrize("by_row", [True, False])
@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16", "f16"])
@pytest.mark.parametrize("N,T,D,G,gated,silu", [
    (1, 1, 8, 1, True, False), (2, 3, 24, 3, False, True), (2, 65, 64, 4, True, True), (1, 130, 130, 10, False, False), (3, 33, 256, 2, True, False),
    (1, 200, 36, 4, True, True), (1, 9, 1024, 1, True, False), (2, 5, 600, 1, False, True), (1, 300, 16, 16, True, False), (1, 7, 2600, 2, True, True)])
def test_batch(dtype, by_row, N, T, D, G, gated, silu):
    c = make(dtype, (N, T), D, gated, N + T + D + G)
    compare(c, run(c, G, by_row, silu), G, by_row, silu, dtype, lo.sequences(T, N))


@pytest.mark.parametrize("dtype,D", [("f32", 4100), ("bf16", 8200), ("f32", 1027), ("bf16", 16000), ("f64", 2100)])
def test_wide_groups(dtype, D):
    """more channels than a workgroup keeps"""
    c = make(dtype, (1, 5), D, True, D)
    compare(c, run(c, 1, True, True), 1, True, True, dtype, lo.sequences(5, 1))


PACKED = {"mixed": [0, 130, 131, 131, 500, 501, 900, 900], "tokens": list(range(0, 41)), "behind": [3, 3, 20, 150, 260], "empty": [0, 0, 0], "edges": [0, 128, 256, 640]}


@pytest.mark.parametrize("by_row", [True, False])
@pytest.mark.parametrize("dtype,D,G,gated,silu", [("bf16", 128, 4, True, False), ("f32", 66, 6, False, True), ("f64", 20, 2, True, True)])
@pytest.mark.parametrize("name", list(PACKED))
def test_packed(name, dtype, D, G, gated, silu, by_row):
    off = PACKED[name]
    N, rows = len(off) - 1, off[-1] + 9
    c = make(dtype, (rows,), D, gated, 7)
    by = [k for k in ("x", "z", "dy") if c[k] is not None]
    for k in by:
        c[k][:off[0]] = float("nan")
        c[k][off[-1]:] = float("inf")
    offsets = torch.tensor(off, dtype=torch.int64, device=DEV)
    got = run(c, G, by_row, silu, offsets=offsets)
    for k in ("y", "dx", "dz"):
        if k in got:
            assert bool((got[k][off[-1]:] == 0).all()) and bool((got[k][:off[0]] == 0).all()), k
    if by_row:
        assert bool((got["stats"][off[-1]:] == 0).all()) and bool((got["stats"][:off[0]] == 0).all())
    about = {"z": c["z"], "span": deer.DEER_SPAN_ROW if by_row else deer.DEER_SPAN_SEQUENCE, "act": deer.DEER_ACT_SILU if silu else deer.DEER_ACT_NONE, "offsets": offsets}
    y, stats = deer.groupnorm_solve(c["x"], G, c["w"], c["bias"], eps=EPS, out=torch.full_like(c["x"], 7.0), **about)
    assert bool((y[off[-1]:] == 7).all()) and bool((y[:off[0]] == 7).all()) and torch.equal(y[off[0]:off[-1]], got["y"][off[0]:off[-1]])
    assert torch.equal(stats, got["stats"])
    dx = deer.groupnorm_grad(c["x"], G, stats, c["dy"], c["w"], c["bias"], dx=torch.full_like(c["x"], 7.0), **about)[0]
    assert bool((dx[off[-1]:] == 7).all()) and torch.equal(dx[off[0]:off[-1]], got["dx"][off[0]:off[-1]])
    for k in by:
        c[k].nan_to_num_(0.0, 0.0, 0.0)
    compare(c, got, G, by_row, silu, dtype, lo.sequences(rows, N, offsets=off))


@pytest.mark.parametrize("by_row", [True, False])
def test_padded_batch(by_row):
    N, T, D, G, lens = 5, 300, 48, 3, [300, 0, 1, 129, 256]
    c = make("bf16", (N, T), D, True, 3)
    for n, L in enumerate(lens):
        for k in ("x", "z", "dy"):
            c[k][n, L:] = float("nan")
    got = run(c, G, by_row, True, lengths=torch.tensor(lens, dtype=torch.int64, device=DEV))
    for n, L in enumerate(lens):
        for k in ("y", "dx", "dz"):
            assert bool((got[k][n, L:] == 0).all()), k
    for k in ("x", "z", "dy"):
        c[k].nan_to_num_(0.0, 0.0, 0.0)
    compare(c, got, G, by_row, True, "bf16", lo.sequences(T, N, lengths=lens))


@pytest.mark.parametrize("by_row", [True, False])
@pytest.mark.parametrize("dtype,D", [("bf16", 64), ("f32", 30)])
def test_slices_without_weights(dtype, D, by_row):
    N, T, G = 2, 90, 2
    c = make(dtype, (N, T), D, True, 5)
    one = torch.cat([c["x"], c["z"]], -1).contiguous()
    x, z = one[..., :D], one[..., D:]
    about = {"z": z, "span": deer.DEER_SPAN_ROW if by_row else deer.DEER_SPAN_SEQUENCE}
    y, stats = deer.groupnorm_solve(x, G, **about)
    dx, dw, dbias, dz = deer.groupnorm_grad(x, G, stats, c["dy"], **about)
    assert dx.stride() == x.stride() and dz.stride() == z.stride()
    got = {"y": y, "stats": stats, "dx": dx, "dw": dw, "dbias": dbias, "dz": dz}
    compare(c, got, G, by_row, False, dtype, lo.sequences(T, N), w=np.ones(D), bias=np.zeros(D))
    done = torch.zeros_like(one)
    deer.groupnorm_grad(x, G, stats, c["dy"], dx=done[..., :D], dz=done[..., D:], **about)
    assert torch.equal(done, torch.cat([dx, dz], -1))


@pytest.mark.parametrize("by_row", [True, False])
def test_constant_and_far_values(by_row):
    """no variance: rstd is eps^-1/2 and nothing is left; a mean far from zero costs its own digits only"""
    x = torch.full((2, 40, 32), 3.0, device=DEV)
    span = deer.DEER_SPAN_ROW if by_row else deer.DEER_SPAN_SEQUENCE
    y, stats = deer.groupnorm_solve(x, 4, span=span)
    assert bool((y == 0).all()) and bool((stats[..., 0] == 3).all()) and bool(((stats[..., 1] - EPS ** -0.5).abs() <= 4 * 2.0 ** -24 * EPS ** -0.5).all())
    assert bool((deer.groupnorm_grad(x, 4, stats, torch.zeros_like(x), span=span)[0] == 0).all())
    far = torch.from_numpy(1000.0 + np.random.default_rng(1).standard_normal((2, 300, 32))).float().to(DEV)
    c = {"x": far, "w": torch.ones(32, device=DEV), "bias": torch.zeros(32, device=DEV), "z": None, "dy": torch.randn(2, 300, 32, device=DEV)}
    compare(c, run(c, 4, by_row, False), 4, by_row, False, "f32", lo.sequences(300, 2))


def test_one_channel_a_group_has_no_gradient():
    c = make("f32", (2, 9), 12, False, 8)
    got = run(c, 12, True, False)
    assert bool((got["dx"] == 0).all()) and torch.equal(got["y"], c["bias"].expand_as(got["y"]))


def test_not_finite_stays_in_its_sequence_and_group():
    off = torch.tensor([0, 150, 300, 500], device=DEV)
    for by_row in (True, False):
        c = make("f32", (500,), 40, True, 1)
        clean = run(c, 4, by_row, True, offsets=off)
        c["x"][200, 7] = float("nan")
        got = run(c, 4, by_row, True, offsets=off)
        for name in ("y", "dx", "dz"):
            same = got[name] == clean[name]
            same[200 if by_row else slice(150, 300), :10] = True
            assert bool(same.all()), name


def test_empty_arrays():
    for by_row in (True, False):
        c = make("f32", (2, 0), 12, True, 4)
        got = run(c, 3, by_row, True)
        assert got["y"].shape == (2, 0, 12) and bool((got["dw"] == 0).all()) and bool((got["dbias"] == 0).all())
        assert got["stats"].shape == ((2, 0, 3, 2) if by_row else (2, 3, 2)) and bool((got["stats"] == 0).all())


def test_rows_of_many_sequences():
    """2^16 and some sequences of one row, 64 groups each, are what as many rows of one sequence are"""
    N, D, G = 70001, 256, 64
    c = make("f32", (N, 1), D, True, 9)
    one = {k: t.reshape(1, N, D) if t.dim() == 3 else t for k, t in c.items()}
    got, want = run(c, G, True, True), run(one, G, True, True)
    for name, t in got.items():
        assert torch.equal(t.reshape(want[name].shape), want[name]), name
