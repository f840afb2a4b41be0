"""Statistics over sequences that begin far from what follows: a start token, a transient in front of a recording.

Bound of the sum of squares' rounding, u the unit roundoff, M the squares about the mean.  A lane sums at most 32 rows' differences from the mean of its first eight: that lies at most (M / 8 - M / 32)^1/2
off, so that the squares s about it are at most 4 M.  34 u s for them, 2 x 32 u (3 M s)^1/2 for the square of the sum that is taken off, 9 u M for its own: 375 u M.  Lanes and wavefronts are joined by differences of
their means, sums of 64 and of 4: 225 u M with room.  600 u of the variance are 300 u of rstd, and 20 for its own roundings and those of the pieces' means.  Where rows lie 100 or 1,000 away from noise, differences
from a piece's first row would leave up to 10,000 u."""
import numpy as np
import pytest
import torch

import layer_oracle as lo
from paper_2309_12252_amd import deer
from test_gpu_groupnorm import DEV, EPS, compare, make, run

pytestmark = pytest.mark.gpu


def check_rstd(x, stats, G, seqs, dtype):
    x = x.detach().cpu().double().numpy().astype(np.longdouble).reshape(-1, x.shape[-1])
    stats = stats.cpu().double().numpy()
    for n, (r0, L) in enumerate(seqs):
        if L == 0:
            continue
        v = x[r0:r0 + L].reshape(L, G, -1)
        want = (v.var((0, 2)) + EPS) ** -0.5
        off = np.abs(stats[n, :, 1] / want - 1).max()
        print("sequence %d: rstd off by %.1f u of 320" % (n, off / lo.U[dtype]), flush=True)
        assert off <= 320 * lo.U[dtype], (n, float(off))


@pytest.mark.parametrize("far", [100.0, 1000.0])
@pytest.mark.parametrize("dtype", ["f32", "f64", "bf16"])
@pytest.mark.parametrize("N,T,D,G", [(8, 2048, 4, 4), (4, 2000, 16, 16), (2, 4100, 6, 2), (3, 700, 130, 10), (5, 9, 8, 2)])
def test_batch(dtype, far, N, T, D, G):
    c = make(dtype, (N, T), D, False, N + T + D)
    c["x"][:, 0] += far
    got = run(c, G, False, False)
    check_rstd(c["x"], got["stats"], G, lo.sequences(T, N), dtype)
    compare(c, got, G, False, False, dtype, lo.sequences(T, N))


@pytest.mark.parametrize("dtype", ["f32", "f64"])
def test_packed(dtype):
    off = [5, 5, 3000, 3001, 3007, 9000, 9000, 11048]
    c = make(dtype, (off[-1] + 9,), 4, False, 3)
    for a in off[:-1]:
        c["x"][a] += 300.0
    got = run(c, 2, False, False, offsets=torch.tensor(off, dtype=torch.int64, device=DEV))
    check_rstd(c["x"], got["stats"], 2, lo.sequences(off[-1] + 9, len(off) - 1, offsets=off), dtype)


def test_long_pieces():
    """8,192 rows of a piece: 32 for each of 256 lanes"""
    N, T = 1040, 8192
    x = torch.randn(N, T, 2, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    x[:, 0] += 1000.0
    _, stats = deer.groupnorm_solve(x, 1, span=deer.DEER_SPAN_SEQUENCE, eps=EPS)
    want = (x.double().var((1, 2), correction=0) + EPS) ** -0.5
    assert float((stats[:, 0, 1].double() / want - 1).abs().max()) <= 320 * lo.U["f32"]


def test_sums_over_many_rows():
    """2^23 equal rows, one channel a group (dbias is all that there is): a lane sums at most 1,024 of them in 32 bits, u each, 64 bits take the rest; 16 for what else is rounded"""
    rows, D = 1 << 23, 256
    x = torch.zeros(1, rows, D, device=DEV)
    dy = torch.full_like(x, 0.7)
    _, _, dbias, _ = deer.groupnorm_grad(x, D, torch.zeros(1, rows, D, 2, device=DEV), dy)
    off = float((dbias.double() / (rows * float(dy[0, 0, 0])) - 1).abs().max())
    print("dbias off by %.1f u" % (off / lo.U["f32"]), flush=True)
    assert off <= (1024 + 16) * lo.U["f32"]


def test_large_constants():
    """no sum of eight values overflows"""
    x = torch.full((2, 40, 8), 2.0 ** 127, device=DEV)
    y, stats = deer.groupnorm_solve(x, 2, span=deer.DEER_SPAN_SEQUENCE)
    assert bool((y == 0).all()) and bool((stats[..., 0] == 2.0 ** 127).all())
