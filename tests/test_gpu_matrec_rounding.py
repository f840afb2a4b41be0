"""Outputs and gradients of the matrix-state recurrence in bf16: what one rounding of the exact values leaves, whoever asks for the final states."""
import ctypes

import pytest
import torch

import seq_oracle as so
import test_gpu_matrec as tm
from paper_2309_12252_amd import deer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("T,Hk,Hv,Dk,Dv", [(1, 1, 1, 128, 128), (64, 1, 2, 64, 64), (200, 2, 4, 128, 128), (500, 1, 2, 128, 64), (300, 1, 1, 33, 70), (700, 2, 2, 64, 128)])
def test_outputs_are_rounded_once(T, Hk, Hv, Dk, Dv):
    d = tm.make("bf16", (1, T), 1, Hk, Hv, Dk, Dv, T)
    o, _ = deer.matrec_solve(d["q"], d["k"], d["v"], d["g"], d["s0"])
    want, absolute, _ = so.matrix(*(tm.host(d[n])[0] for n in ("q", "k", "v", "g")), tm.host(d["s0"]), [(0, T)], Dk ** -0.5)
    # every term has one factor in two pieces, off by at most half a step of the second: 2^-16; and sums as in fp32
    so.check("o", o, want["o"], (4 * (T + 128) * 2.0 ** -24 + 2.0 ** -16) * absolute["o"], "bf16")


@pytest.mark.parametrize("N,T,Hk,Hv,Dk,Dv", [(1, 1, 1, 1, 128, 128), (1, 64, 1, 2, 64, 64), (1, 200, 2, 4, 128, 128), (1, 500, 1, 2, 128, 64), (2, 300, 1, 1, 33, 70),
                                             (1, 700, 2, 2, 64, 128), (1, 1100, 64, 64, 16, 8)])
def test_gradients_are_rounded_once(N, T, Hk, Hv, Dk, Dv):
    d = tm.make("bf16", (N, T), N, Hk, Hv, Dk, Dv, T + 1)
    got = deer.matrec_grad(d["q"], d["k"], d["v"], d["g"], d["do"], d["s0"], d["dlast"])
    rows = lambda n: tm.host(d[n]).reshape((N * T,) + d[n].shape[2:])   # noqa: E731
    want, absolute, _ = so.matrix(rows("q"), rows("k"), rows("v"), rows("g"), tm.host(d["s0"]), so.sequences(T, N), Dk ** -0.5, rows("do"), tm.host(d["dlast"]))
    # as the outputs; the state in dv takes rows in as two pieces as well
    for n, t, unit in (("dq", got[0], 2.0 ** -16), ("dk", got[1], 2.0 ** -16), ("dv", got[2], 2.0 ** -15)):
        so.check(n, t, want[n], (4 * (T + 128) * 2.0 ** -24 + unit) * absolute[n], "bf16")


@pytest.mark.parametrize("T", [100, 1000])
def test_outputs_do_not_depend_on_the_final_states_being_wanted(T):
    H, D = 2, 64
    d = tm.make("bf16", (1, T), 1, H, H, D, D, 2)
    o, _ = deer.matrec_solve(d["q"], d["k"], d["v"], d["g"], d["s0"])
    lib, size = deer.load_library(), ctypes.c_size_t(0)
    cfg = deer.MatrecConfig(deer.DEER_BF16, 1, T, 0, H, H, D, D, 0, D ** -0.5, 0, 0, 0, 0)
    assert lib.deer_matrec_workspace_bytes(ctypes.byref(cfg), 0, ctypes.byref(size)) == deer.DEER_OK
    ws, got = torch.empty(size.value, dtype=torch.uint8, device=DEV), torch.empty_like(o)
    assert lib.deer_matrec_solve(ctypes.byref(cfg), d["q"].data_ptr(), d["k"].data_ptr(), d["v"].data_ptr(), d["g"].data_ptr(), d["s0"].data_ptr(), None,
                                 got.data_ptr(), None, ws.data_ptr(), size, torch.cuda.current_stream().cuda_stream) == deer.DEER_OK
    assert torch.equal(got, o)
