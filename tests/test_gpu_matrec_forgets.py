"""Gradient of the gates behind a stretch of large values that is forgotten again: what goes through a chunk is a difference of sums that may be as
large as what the state held before, and is known to no more than those sums' rounding, unless the factors say that less is left."""
import numpy as np
import pytest
import torch

import seq_oracle as so
import test_gpu_matrec as tm
from paper_2309_12252_amd import deer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
C = 64   # rows of a chunk


def sizes(q, k, v, g, s0, do, dlast, scale):
    """norms, by chunk and head, of the state in front of a chunk and of the gradient of the state behind it, in 64 bits"""
    T = g.shape[0]
    S, R, front, behind = s0.copy(), dlast.copy(), [], []
    norm = lambda x: np.sqrt((x * x).sum((-1, -2)))   # noqa: E731
    for t in range(T):
        if t % C == 0:
            front.append(norm(S))
        S = np.exp(g[t])[:, None, None] * S + k[t][:, :, None] * v[t][:, None, :]
    for t in range(T - 1, -1, -1):
        if t % C == C - 1 or t == T - 1:
            behind.append(norm(R))
        R = np.exp(g[t])[:, None, None] * (R + scale * q[t][:, :, None] * do[t][:, None, :])
    return np.stack(front), np.stack(behind[::-1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("large,gate", [(1e4, -0.5), (1e6, -0.5), (1e6, -0.1), (1e3, -0.02)])
def test_large_values_that_are_forgotten(dtype, large, gate):
    T, H, D = 2048, 256, 8          # 32 chunks in one segment: 256 heads of whole sequences
    d = tm.make(dtype, (T,), 1, H, H, D, D, 3)
    d = {n: t[None].contiguous() if n not in ("s0", "dlast") else t for n, t in d.items()}
    d["v"][0, 59:63] *= large   # at the end of a chunk: read by the next one, and forgotten there
    d["g"].uniform_(1.2 * gate, 0.8 * gate, generator=torch.Generator(device=DEV).manual_seed(1))
    scale = D ** -0.5
    dgate = deer.matrec_grad(d["q"], d["k"], d["v"], d["g"], d["do"], d["s0"], d["dlast"])[3][0]
    q, k, v, do = (tm.host(d[n])[0] for n in ("q", "k", "v", "do"))
    g, s0, dlast = tm.host(d["g"])[0], tm.host(d["s0"]), tm.host(d["dlast"])
    want, absolute, _ = so.matrix(q, k, v, g, s0, [(0, T)], scale, do, dlast)
    front, behind = sizes(q, k, v, g, s0[0], do, dlast[0], scale)
    # What goes through chunk c, taken from in front: <S, dS> less what is read in the chunk; then what it puts out is added.  Each is off by at most as many
    # roundings of its terms as the oracle counts (64 rows and two sums of 128 columns); and the result, kept within 1.02 of it, by no more than its bound and 1.02 of it (2.03: the rounding of the bound itself)
    u = (C + 128 + 128) * 2.0 ** -24
    read, put = ((np.abs(a) * absolute[n]).sum(-1) for a, n in ((q, "dq"), (k, "dk")))
    off, passing = u * (np.abs(s0[0]) * absolute["ds0"][0]).sum((-1, -2)), np.zeros_like(g)
    for c in range(T // C):
        rows = slice(c * C, (c + 1) * C)
        most = np.exp(g[rows].sum(0)) * front[c] * behind[c]
        off = np.minimum(off + u * read[rows].sum(0), 2.03 * most)
        passing[rows] = off
        off = off + u * put[rows].sum(0)
    rest = 4 * (T + 128) * 2.0 ** -24 + (2.0 ** -16 if dtype == "bf16" else 0.0)
    so.check("dgate", dgate, want["dgate"], rest * absolute["dgate"] + passing, "f32")
    # behind the stretch, where it is forgotten, as exact as anywhere: half of a 2^-24 a row and column, in the mean
    if gate <= -0.5:
        far = slice(4 * C, T)
        err = np.linalg.norm(tm.host(dgate)[far] - want["dgate"][far]) / np.linalg.norm(want["dgate"][far])
        print("far behind: %.2g" % err)
        assert err <= (4 * (T + 128)) ** 0.5 * 2.0 ** -24 + (2.0 ** -16 if dtype == "bf16" else 0.0)
