"""Selective scan with factors above one, whose products over a segment's rows 32 bits do not hold: where states and gradients are finite, so are the results, cut or not."""
import pytest
import torch

import layer_oracle as lo
from paper_2309_12252_amd import deer
from test_gpu_selscan import DEV, compare, make, run

pytestmark = pytest.mark.gpu


def ordinary(dtype, lead, N, D, S, gated, seed):
    """steps of one, rates of -1/2"""
    c = make(dtype, lead, N, D, S, 1, gated, seed, softplus=False)
    c["dt"].fill_(1.0), c["dt_bias"].zero_(), c["A"].fill_(-0.5)
    return c


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_growth_without_anything_in_it(dtype, gated):
    """e^2 a row over 140 rows: states begin with the last 10 rows, gradients end with the first 10"""
    T = 140
    c = ordinary(dtype, (1, T), 1, 3, 2, gated, 1)
    c["A"][0] = 2.0
    c["x"][:, :T - 10, 0], c["h0"][:, 0] = 0.0, 0.0
    c["dy"][:, 10:, 0], c["dlast"][:, 0] = 0.0, 0.0
    got = run(c)
    for name, t in got.items():
        assert bool(torch.isfinite(t).all()), name
    compare(c, got, dtype, lo.sequences(T, 1))


@pytest.mark.parametrize("dtype", ["f32", "f16"])
@pytest.mark.parametrize("off", [[0, 108], [20, 130], [5, 5, 20, 128, 131]])
def test_growth_from_small_states(dtype, off):
    """e^1.5 a row over some 110 rows, 10^-36 at the beginning and behind the end"""
    N, rows = len(off) - 1, off[-1] + 3
    c = ordinary(dtype, (rows,), N, 2, 2, False, 2)
    c["A"][0] = 1.5
    long = [n for n in range(N) if off[n + 1] - off[n] > 50]
    for n in long:
        c["h0"][n, 0] *= 1e-36
        c["dlast"][n, 0] *= 1e-36
        c["x"][off[n]:off[n + 1], 0] = 0.0
        c["dy"][off[n]:off[n + 1], 0] = 0.0
    got = run(c, offsets=torch.tensor(off, dtype=torch.int64, device=DEV))
    if dtype == "f16":   # (ends at 65,504, and e^1.5 a row over 15 rows of ordinary values are 6e9: what is held in 32 bits)
        got = {k: got[k] for k in ("last", "dh0", "dA", "dskip", "dbias")}
    for name, t in got.items():
        assert bool(torch.isfinite(t).all()), name
    compare(c, got, dtype, lo.sequences(rows, N, offsets=off))


def test_not_a_number_in_a_front():
    """stays in its sequence where the join looks at rows"""
    off = torch.tensor([0, 200, 400], device=DEV)
    c = ordinary("f32", (400,), 2, 3, 2, True, 3)
    clean = run(c, offsets=off)
    c["dt"][100, 1] = float("nan")
    got = run(c, offsets=off)
    for name in ("y", "dx", "ddt", "dz"):
        same = got[name] == clean[name]
        same[:200, 1] = True
        assert bool(same.all()), name
    assert bool(torch.isnan(got["dx"][:101, 1]).all()) and bool(torch.isnan(got["y"][100:200, 1]).all())
