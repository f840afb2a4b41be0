"""Host-side checks of the C entry points of the short convolution, the selective scan and the group norm: argument validation without a GPU, no compute calls."""
import ctypes

import pytest
import torch

from paper_2309_12252_amd import deer

WORD = ctypes.c_void_p(256)   # (looked at for NULL and alignment only)
ODD = ctypes.c_void_p(257)
ROOM = 1 << 50


def conv(**kw):
    c = dict(dtype=deer.DEER_F32, act=deer.DEER_ACT_SILU, N=2, D=8, T=100, packed=0, W=4, stride_x=0, stride_y=0)
    c.update(kw)
    return deer.ShortconvConfig(*[c[name] for name, _ in deer.ShortconvConfig._fields_])


def scan(**kw):
    c = dict(dtype=deer.DEER_BF16, dt_act=deer.DEER_ACT_SOFTPLUS, N=2, D=8, T=100, packed=0, S=16, G=2, reserved=0, stride_x=0, stride_dt=0, stride_B=0, stride_C=0,
             stride_z=0, stride_y=0)
    c.update(kw)
    return deer.SelscanConfig(*[c[name] for name, _ in deer.SelscanConfig._fields_])


def norm(**kw):
    c = dict(dtype=deer.DEER_F32, act=deer.DEER_ACT_NONE, span=deer.DEER_SPAN_ROW, N=2, D=8, G=2, T=100, packed=0, reserved=0, eps=1e-5, stride_x=0, stride_z=0, stride_y=0)
    c.update(kw)
    return deer.GroupnormConfig(*[c[name] for name, _ in deer.GroupnormConfig._fields_])


def conv_calls(cfg, ws=WORD, room=ROOM, x=WORD, w=WORD, y=WORD, bounds=None, dw=WORD):
    lib, ref = deer.load_library(), ctypes.byref(cfg)
    return (lib.deer_shortconv_solve(ref, x, w, None, None, bounds, y, None, None),
            lib.deer_shortconv_grad(ref, x, w, None, None, bounds, y, None, y, dw, None, None, ws, room, None))


def scan_calls(cfg, ws=WORD, room=ROOM, x=WORD, A=WORD, B=WORD, z=None, dz=None, bounds=None):
    lib, ref = deer.load_library(), ctypes.byref(cfg)
    return (lib.deer_selscan_solve(ref, x, WORD, A, B, WORD, None, z, None, None, bounds, WORD, None, ws, room, None),
            lib.deer_selscan_grad(ref, x, WORD, A, B, WORD, None, z, None, None, bounds, WORD, None, WORD, WORD, WORD, WORD, WORD, None, dz, None, None, ws, room, None))


def norm_calls(cfg, ws=WORD, room=ROOM, x=WORD, stats=WORD, z=None, dz=None, bounds=None):
    lib, ref = deer.load_library(), ctypes.byref(cfg)
    return (lib.deer_groupnorm_solve(ref, x, None, None, z, bounds, WORD, stats, ws, room, None),
            lib.deer_groupnorm_grad(ref, x, None, None, z, bounds, stats, WORD, WORD, None, None, dz, ws, room, None))


@pytest.mark.parametrize("change,status", [
    (dict(dtype=4), 1), (dict(act=0), 1), (dict(act=4), 1), (dict(N=0), 1), (dict(D=0), 1), (dict(T=-1), 1), (dict(packed=2), 1), (dict(W=0), 1), (dict(W=9), 1),
    (dict(stride_x=7), 1), (dict(stride_y=-8), 1), (dict(T=(1 << 33) + 1), 2), (dict(N=2000000000, T=1 << 20), 2), (dict(D=(1 << 27) + 1), 2)])
def test_shortconv_refuses(change, status):
    lib, cfg, size = deer.load_library(), conv(**change), ctypes.c_size_t(0)
    assert lib.deer_shortconv_workspace_bytes(ctypes.byref(cfg), ctypes.byref(size)) == status
    assert conv_calls(cfg) == (status, status) and lib.deer_last_error(None)


def test_shortconv_pointers_and_workspace():
    lib, cfg, size = deer.load_library(), conv(), ctypes.c_size_t(0)
    assert lib.deer_shortconv_workspace_bytes(None, ctypes.byref(size)) == 1 and lib.deer_shortconv_workspace_bytes(ctypes.byref(cfg), None) == 1
    assert lib.deer_shortconv_workspace_bytes(ctypes.byref(cfg), ctypes.byref(size)) == 0 and size.value > 0
    for bad in (dict(x=None), dict(w=None), dict(y=None), dict(x=ODD), dict(w=ODD), dict(bounds=ctypes.c_void_p(260))):
        assert conv_calls(cfg, **bad) == (1, 1), bad
    assert conv_calls(cfg, dw=None)[1] == 1 and conv_calls(conv(packed=1)) == (1, 1)
    for bad in (dict(ws=None), dict(ws=ctypes.c_void_p(320)), dict(room=size.value - 1)):
        assert conv_calls(cfg, **bad)[1] == deer.DEER_ERR_WORKSPACE
    step = lambda c=cfg, x=WORD, n=4, s=WORD, slots=None: lib.deer_shortconv_step(ctypes.byref(c), x, WORD, None, slots, n, s, WORD, None)   # noqa: E731
    for bad in (dict(x=None), dict(n=0), dict(s=None), dict(s=ODD), dict(slots=ODD), dict(c=conv(W=9))):
        assert step(**bad) == 1, bad
    assert step(c=conv(N=1 << 24, D=1)) == 2


@pytest.mark.parametrize("change,status", [
    (dict(dtype=4), 1), (dict(dtype=deer.DEER_F64), 2), (dict(dt_act=deer.DEER_ACT_SILU), 1), (dict(dt_act=0), 1), (dict(N=0), 1), (dict(D=0), 1), (dict(T=-1), 1),
    (dict(packed=2), 1), (dict(S=0), 1), (dict(S=65), 2), (dict(G=0), 1), (dict(G=3), 1), (dict(reserved=1), 1), (dict(stride_x=7), 1), (dict(stride_B=31), 1),
    (dict(stride_z=-1), 1), (dict(T=(1 << 33) + 1), 2), (dict(N=1 << 30, T=1 << 20), 2)])
def test_selscan_refuses(change, status):
    lib, cfg, size = deer.load_library(), scan(**change), ctypes.c_size_t(0)
    for grad in (0, 1):
        assert lib.deer_selscan_workspace_bytes(ctypes.byref(cfg), grad, ctypes.byref(size)) == status
    assert scan_calls(cfg) == (status, status) and lib.deer_last_error(None)


def test_selscan_pointers_and_workspace():
    lib, cfg, size = deer.load_library(), scan(), ctypes.c_size_t(0)
    assert lib.deer_selscan_workspace_bytes(None, 0, ctypes.byref(size)) == 1 and lib.deer_selscan_workspace_bytes(ctypes.byref(cfg), 0, None) == 1
    need = []
    for grad in (0, 1):
        assert lib.deer_selscan_workspace_bytes(ctypes.byref(cfg), grad, ctypes.byref(size)) == 0 and size.value > 0
        need.append(size.value)
    for bad in (dict(x=None), dict(A=None), dict(B=None), dict(x=ODD), dict(A=ctypes.c_void_p(258)), dict(z=ODD, dz=WORD), dict(bounds=ctypes.c_void_p(260))):
        assert scan_calls(cfg, **bad) == (1, 1), bad
    assert scan_calls(cfg, z=WORD)[1] == 1   # no place for dz
    assert scan_calls(scan(packed=1)) == (1, 1)
    for bad in (dict(ws=None), dict(ws=ctypes.c_void_p(320)), dict(room=need[0] - 1)):
        assert scan_calls(cfg, **bad) == (deer.DEER_ERR_WORKSPACE,) * 2
    assert scan_calls(cfg, room=need[1] - 1)[1] == deer.DEER_ERR_WORKSPACE
    step = lambda c=cfg, x=WORD, n=4, s=WORD, slots=None: lib.deer_selscan_step(ctypes.byref(c), x, WORD, WORD, WORD, WORD, None, None, None, slots, n, s, WORD, None)   # noqa: E731
    for bad in (dict(x=None), dict(n=0), dict(s=None), dict(s=ODD), dict(slots=ODD), dict(c=scan(G=3))):
        assert step(**bad) == 1, bad
    assert step(c=scan(S=65)) == 2 and step(c=scan(N=1 << 26, D=64)) == 2


@pytest.mark.parametrize("change,status", [
    (dict(dtype=4), 1), (dict(act=1), 1), (dict(span=2), 1), (dict(N=0), 1), (dict(D=0), 1), (dict(T=-1), 1), (dict(packed=2), 1), (dict(G=0), 1), (dict(G=3), 1),
    (dict(reserved=1), 1), (dict(eps=-1e-5), 1), (dict(eps=float("nan")), 1), (dict(eps=1e39), 1), (dict(stride_x=7), 1), (dict(stride_z=-1), 1),
    (dict(T=(1 << 33) + 1), 2), (dict(N=1 << 30, G=8, D=8, span=1), 2), (dict(D=1 << 28), 2)])
def test_groupnorm_refuses(change, status):
    lib, cfg, size = deer.load_library(), norm(**change), ctypes.c_size_t(0)
    for grad in (0, 1):
        assert lib.deer_groupnorm_workspace_bytes(ctypes.byref(cfg), grad, ctypes.byref(size)) == status
    assert norm_calls(cfg) == (status, status) and lib.deer_last_error(None)


def test_groupnorm_pointers_and_workspace():
    lib, size = deer.load_library(), ctypes.c_size_t(0)
    for span in (deer.DEER_SPAN_ROW, deer.DEER_SPAN_SEQUENCE):
        cfg = norm(span=span)
        for bad in (dict(x=None), dict(stats=None), dict(x=ODD), dict(stats=ctypes.c_void_p(258)), dict(z=ODD, dz=WORD), dict(bounds=ctypes.c_void_p(260))):
            assert norm_calls(cfg, **bad) == (1, 1), bad
        assert norm_calls(cfg, z=WORD)[1] == 1 and norm_calls(norm(span=span, packed=1)) == (1, 1)
        none = 1 if span == deer.DEER_SPAN_ROW else 0   # (forward over rows: no workspace)
        assert norm_calls(cfg, ws=None)[none:] == (deer.DEER_ERR_WORKSPACE,) * (2 - none) and norm_calls(cfg, ws=ctypes.c_void_p(320))[1] == deer.DEER_ERR_WORKSPACE
        for grad in (0, 1):
            assert lib.deer_groupnorm_workspace_bytes(ctypes.byref(cfg), grad, ctypes.byref(size)) == 0 and (size.value > 0) == (grad >= none)
            if size.value:
                assert norm_calls(cfg, room=size.value - 1)[grad] == deer.DEER_ERR_WORKSPACE
    assert lib.deer_groupnorm_workspace_bytes(None, 0, ctypes.byref(size)) == 1 and lib.deer_groupnorm_workspace_bytes(ctypes.byref(norm()), 0, None) == 1


def test_rows_of_no_sequence_are_zeroed_on_request():
    lib, size, plain = deer.load_library(), ctypes.c_size_t(0), ctypes.c_size_t(0)
    for make, ask in ((conv, lambda c, s: lib.deer_shortconv_workspace_bytes(c, s)), (scan, lambda c, s: lib.deer_selscan_workspace_bytes(c, 1, s)),
                      (norm, lambda c, s: lib.deer_groupnorm_workspace_bytes(c, 1, s))):
        for packed in (deer.DEER_ROWS_PADDED, deer.DEER_ROWS_PACKED):
            assert ask(ctypes.byref(make(packed=packed)), ctypes.byref(plain)) == 0
            assert ask(ctypes.byref(make(packed=packed | deer.DEER_REST_ZERO)), ctypes.byref(size)) == 0 and size.value == plain.value
        for bad in (2, deer.DEER_REST_ZERO | 2, 512, -1):
            assert ask(ctypes.byref(make(packed=bad)), ctypes.byref(size)) == 1


def test_workspaces_are_of_the_arrays_order():
    """states of every 16th row and 8 floats of sums a row for each of a quarter of the states and 256 of its channels; what the others need is small"""
    lib, size = deer.load_library(), ctypes.c_size_t(0)
    rows, D, S = 16384, 4096, 16
    assert lib.deer_selscan_workspace_bytes(ctypes.byref(scan(N=4, T=4096, D=D, S=S, G=1)), 1, ctypes.byref(size)) == 0
    assert size.value < rows / 16 * D * (S + 1) * 4 * 1.3 + rows * D * 2 * 1.1
    assert lib.deer_selscan_workspace_bytes(ctypes.byref(scan(N=1, T=1 << 20, D=2048, S=S, G=1)), 0, ctypes.byref(size)) == 0
    assert size.value < (1 << 20) * 2048 * 2 / 64
    assert lib.deer_groupnorm_workspace_bytes(ctypes.byref(norm(N=4, T=4096, D=D, G=32, span=1)), 1, ctypes.byref(size)) == 0 and size.value < rows * D * 4 / 8
    assert lib.deer_shortconv_workspace_bytes(ctypes.byref(conv(N=4, T=4096, D=D)), ctypes.byref(size)) == 0 and size.value < rows * D * 4 / 4


def test_binding_needs_device_tensors():
    x, w = torch.zeros(2, 8, 4), torch.zeros(4, 3)
    for call in (lambda: deer.shortconv_solve(x, w), lambda: deer.shortconv_step(x[0], w, x), lambda: deer.selscan_solve(x, x, w, x, x), lambda: deer.groupnorm_solve(x, 2),
                 lambda: deer.groupnorm_solve(None, 2), lambda: deer.selscan_grad(x, x, w, x, x, x)):
        with pytest.raises(deer.DeerError) as e:
            call()
        assert e.value.status == deer.DEER_ERR_INVALID_ARG


@pytest.mark.parametrize("call", [
    lambda x, w: deer.shortconv_solve.__wrapped__(x, w), lambda x, w: deer.shortconv_grad.__wrapped__(x, w, x),
    lambda x, w: deer.shortconv_step.__wrapped__(x[0], w, torch.zeros(8, 0, 4))])
def test_no_weights_are_refused_by_the_binding(call):
    """in front of an array of -1 rows for the states"""
    with pytest.raises(deer.DeerError) as e:
        call(torch.zeros(2, 8, 4), torch.zeros(4, 0))
    assert e.value.status == deer.DEER_ERR_INVALID_ARG


def test_more_work_items_than_a_launch_holds():
    """2^32 - 1 of them, in any of a call's launches: sums over tiles have 64 a column"""
    lib, size = deer.load_library(), ctypes.c_size_t(0)
    ask = lambda c: lib.deer_shortconv_workspace_bytes(ctypes.byref(c), ctypes.byref(size))   # noqa: E731
    assert ask(conv(N=1, T=1, D=(1 << 26) // 5 - 100)) == 0 and ask(conv(N=1, T=1, D=(1 << 26) // 5 + 1)) == 2
    for grad in (0, 1):
        ask = lambda c: lib.deer_selscan_workspace_bytes(ctypes.byref(c), grad, ctypes.byref(size))   # noqa: E731, B023
        assert ask(scan(N=1, T=1, D=1 << 20, G=1, S=63)) == 0 and ask(scan(N=1, T=1, D=1 << 20, G=1, S=64)) == 2
        assert ask(scan(D=1 << 22, G=1, S=4)) == 0 and ask(scan(D=(1 << 22) + 1, G=1, S=1)) == 2
        assert ask(scan(stride_x=1 << 22)) == 0 and ask(scan(stride_z=(1 << 22) + 1)) == 2 and ask(scan(stride_B=(1 << 22) + 1)) == 2
        assert ask(scan(N=1 << 20, D=64, G=1, T=1)) == 2   # 2^32 states between segments
        ask = lambda c: lib.deer_groupnorm_workspace_bytes(ctypes.byref(c), grad, ctypes.byref(size))   # noqa: E731, B023
        assert ask(norm(N=1, T=1, D=1 << 24)) == 0 and ask(norm(N=1, T=1, D=1 << 25)) == 2
        assert ask(norm(N=1 << 20, T=1, D=8, G=4, span=1)) == 2   # 1,024 lanes for each of 2^22 groups of sequences


def test_groups_of_rows_are_not_counted_like_those_of_sequences():
    """2^17 sequences of 64 groups: no launch of 1,024 lanes for each where statistics are over rows"""
    lib, size = deer.load_library(), ctypes.c_size_t(0)
    for grad in (0, 1):
        ask = lambda c: lib.deer_groupnorm_workspace_bytes(ctypes.byref(c), grad, ctypes.byref(size))   # noqa: E731, B023
        assert ask(norm(N=1 << 17, T=1, D=512, G=64, span=0)) == 0 and ask(norm(N=1 << 17, T=1, D=512, G=64, span=1)) == 2
