"""Host-side checks of the sequence operators' C entry points: argument validation without a GPU, no compute calls."""
import ctypes

import pytest

from paper_2309_12252_amd import deer

WORD = ctypes.c_void_p(256)   # (looked at for NULL and alignment only)


def diag(**kw):
    c = dict(dtype=deer.DEER_F32, gate=0, N=2, D=8, T=100, packed=0, draw=0, stride_gate=0, stride_in=0, stride_out=0, drop=0.0, seed=0)
    c.update(kw)
    return deer.DiagrecConfig(*[c[name] for name, _ in deer.DiagrecConfig._fields_])


@pytest.mark.parametrize("change,status", [
    (dict(dtype=4), 1), (dict(dtype=-1), 1), (dict(gate=3), 1), (dict(N=0), 1), (dict(D=0), 1), (dict(T=-1), 1), (dict(packed=2), 1),
    (dict(stride_in=7), 1), (dict(stride_out=-8), 1), (dict(drop=-0.5), 1), (dict(drop=1.0), 1), (dict(drop=float("nan")), 1),
    (dict(T=(1 << 33) + 1), 2), (dict(N=2000000000, T=1 << 20), 2), (dict(stride_in=(1 << 22) + 1), 2)])
def test_diagrec_refuses(change, status):
    lib, cfg, size = deer.load_library(), diag(**change), ctypes.c_size_t(0)
    assert lib.deer_diagrec_workspace_bytes(ctypes.byref(cfg), 0, ctypes.byref(size)) == status
    assert lib.deer_diagrec_solve(ctypes.byref(cfg), WORD, WORD, None, None, WORD, None, WORD, 1 << 40, None) == status
    assert lib.deer_diagrec_grad(ctypes.byref(cfg), WORD, WORD, None, None, WORD, WORD, None, WORD, WORD, None, WORD, 1 << 40, None) == status
    assert lib.deer_last_error(None)


def test_diagrec_pointers_and_workspace():
    lib, cfg, size = deer.load_library(), diag(), ctypes.c_size_t(0)
    ref = ctypes.byref(cfg)
    assert lib.deer_diagrec_workspace_bytes(None, 0, ctypes.byref(size)) == deer.DEER_ERR_INVALID_ARG
    assert lib.deer_diagrec_workspace_bytes(ref, 0, None) == deer.DEER_ERR_INVALID_ARG
    assert lib.deer_diagrec_workspace_bytes(ref, 0, ctypes.byref(size)) == deer.DEER_OK and size.value > 0
    solve = lambda c, g=WORD, x=WORD, b=None, h=WORD, ws=WORD, n=1 << 40: lib.deer_diagrec_solve(c, g, x, None, b, h, None, ws, n, None)   # noqa: E731
    for bad in (dict(g=None), dict(x=None), dict(h=None), dict(g=ctypes.c_void_p(258)), dict(b=ctypes.c_void_p(260))):
        assert solve(ref, **bad) == deer.DEER_ERR_INVALID_ARG
    assert solve(ref, ws=None) == deer.DEER_ERR_WORKSPACE
    assert solve(ref, ws=ctypes.c_void_p(512 + 64)) == deer.DEER_ERR_WORKSPACE
    assert solve(ref, n=size.value - 1) == deer.DEER_ERR_WORKSPACE
    packed = diag(packed=1)
    assert solve(ctypes.byref(packed)) == deer.DEER_ERR_INVALID_ARG   # no bounds
    # the words of the tiles: 8 bytes a channel and tile, little beside the arrays themselves
    big = diag(dtype=deer.DEER_BF16, N=1, T=1 << 20, D=2048)
    assert lib.deer_diagrec_workspace_bytes(ctypes.byref(big), 0, ctypes.byref(size)) == deer.DEER_OK
    assert size.value < (1 << 20) * 2048 * 2 / 16


def test_step_and_dropout_refuse():
    lib, cfg = deer.load_library(), diag()
    step = lambda c, g=WORD, slots=None, n=4, s=WORD, h=WORD: lib.deer_diagrec_step(ctypes.byref(c), g, WORD, slots, n, s, h, None)   # noqa: E731
    for bad in (dict(g=None), dict(n=0), dict(s=None), dict(h=None), dict(slots=ctypes.c_void_p(258)), dict(s=ctypes.c_void_p(258))):
        assert step(cfg, **bad) == deer.DEER_ERR_INVALID_ARG
    assert step(diag(N=0)) == deer.DEER_ERR_INVALID_ARG
    drop = lambda dtype=0, N=1, T=8, D=4, x=WORD, si=0, y=WORD, so=0, p=0.5: lib.deer_dropout(dtype, N, T, D, x, si, y, so, p, 1, 0, None)   # noqa: E731
    for bad in (dict(dtype=7), dict(N=0), dict(T=-1), dict(D=0), dict(x=None), dict(y=None), dict(si=3), dict(so=-4), dict(p=1.0), dict(p=-0.1),
                dict(p=0.999999), dict(p=float("nan")), dict(x=ctypes.c_void_p(257))):
        assert drop(**bad) == deer.DEER_ERR_INVALID_ARG
    assert drop(T=1 << 40) == deer.DEER_ERR_UNSUPPORTED


def test_binding_needs_device_tensors():
    import torch
    x = torch.zeros(2, 8, 4)
    for call in (lambda: deer.diagrec_solve(x, x), lambda: deer.diagrec_step(x[0], x[0], x[0]), lambda: deer.dropout(x, 0.5, 1),
                 lambda: deer.diagrec_solve(None, x)):
        with pytest.raises(deer.DeerError) as e:
            call()
        assert e.value.status == deer.DEER_ERR_INVALID_ARG


def mat(**kw):
    c = dict(dtype=deer.DEER_BF16, N=2, T=100, packed=0, Hk=2, Hv=4, Dk=64, Dv=64, reserved=0, scale=1.0, stride_q=0, stride_k=0, stride_v=0, stride_o=0)
    c.update(kw)
    return deer.MatrecConfig(*[c[name] for name, _ in deer.MatrecConfig._fields_])


@pytest.mark.parametrize("change,status", [
    (dict(dtype=4), 1), (dict(dtype=deer.DEER_F64), 2), (dict(dtype=deer.DEER_F16), 2), (dict(N=0), 1), (dict(Hk=0), 1), (dict(Hv=3), 1), (dict(Dk=0), 1),
    (dict(Dk=129), 2), (dict(Dv=129), 2), (dict(T=-1), 1), (dict(packed=2), 1), (dict(reserved=1), 1), (dict(scale=float("inf")), 1), (dict(stride_q=127), 1),
    (dict(stride_o=-256), 1), (dict(T=(1 << 33) + 1), 2), (dict(N=1 << 30, T=1 << 20), 2)])
def test_matrec_refuses(change, status):
    lib, cfg, size = deer.load_library(), mat(**change), ctypes.c_size_t(0)
    ref = ctypes.byref(cfg)
    assert lib.deer_matrec_workspace_bytes(ref, 1, ctypes.byref(size)) == status
    assert lib.deer_matrec_solve(ref, WORD, WORD, WORD, WORD, None, None, WORD, None, WORD, 1 << 50, None) == status
    assert lib.deer_matrec_grad(ref, WORD, WORD, WORD, WORD, None, None, WORD, None, WORD, WORD, WORD, None, None, WORD, 1 << 50, None) == status


def test_matrec_pointers_and_workspace():
    lib, cfg, size = deer.load_library(), mat(), ctypes.c_size_t(0)
    ref = ctypes.byref(cfg)
    for grad in (0, 1):
        assert lib.deer_matrec_workspace_bytes(ref, grad, ctypes.byref(size)) == deer.DEER_OK and size.value > 0
    need = size.value
    solve = lambda c, q=WORD, o=WORD, g=WORD, b=None, ws=WORD, n=1 << 40: lib.deer_matrec_solve(c, q, WORD, WORD, g, None, b, o, None, ws, n, None)   # noqa: E731
    for bad in (dict(q=None), dict(o=None), dict(g=None), dict(q=ctypes.c_void_p(257)), dict(g=ctypes.c_void_p(258)), dict(b=ctypes.c_void_p(260))):
        assert solve(ref, **bad) == deer.DEER_ERR_INVALID_ARG
    assert solve(ref, ws=None) == deer.DEER_ERR_WORKSPACE and solve(ref, ws=ctypes.c_void_p(320)) == deer.DEER_ERR_WORKSPACE
    grad = lib.deer_matrec_grad(ref, WORD, WORD, WORD, WORD, None, None, WORD, None, WORD, WORD, WORD, None, None, WORD, need - 1, None)
    assert grad == deer.DEER_ERR_WORKSPACE
    packed = mat(packed=1)
    assert solve(ctypes.byref(packed)) == deer.DEER_ERR_INVALID_ARG
    step = lambda c, q=WORD, n=4, s=WORD: lib.deer_matrec_step(ctypes.byref(c), q, WORD, WORD, WORD, None, n, s, WORD, None)   # noqa: E731
    for c, bad in ((cfg, dict(q=None)), (cfg, dict(n=0)), (cfg, dict(s=None)), (cfg, dict(s=ctypes.c_void_p(258))), (mat(Hv=3), {})):
        assert step(c, **bad) == deer.DEER_ERR_INVALID_ARG
    assert step(mat(Dk=200)) == deer.DEER_ERR_UNSUPPORTED


def test_more_work_items_than_a_launch_holds():
    """2^32 - 1 of them: a workgroup has 512 (recurrences) or 256 (single tokens)"""
    lib, size = deer.load_library(), ctypes.c_size_t(0)
    for grad in (0, 1):
        assert lib.deer_diagrec_workspace_bytes(ctypes.byref(diag(N=(1 << 23) - 1, T=1, D=1)), grad, ctypes.byref(size)) == deer.DEER_OK
        assert lib.deer_diagrec_workspace_bytes(ctypes.byref(diag(N=1 << 23, T=1, D=1)), grad, ctypes.byref(size)) == deer.DEER_ERR_UNSUPPORTED
        assert lib.deer_diagrec_workspace_bytes(ctypes.byref(diag(N=1 << 17, T=1 << 12, D=1024)), grad, ctypes.byref(size)) == deer.DEER_ERR_UNSUPPORTED
    step = lambda **kw: lib.deer_diagrec_step(ctypes.byref(diag(**kw)), WORD, WORD, None, 4, WORD, WORD, None)   # noqa: E731
    assert step(D=0x7FFFFFFF) == deer.DEER_ERR_UNSUPPORTED and step(N=1 << 24, D=1) == deer.DEER_ERR_UNSUPPORTED
    assert lib.deer_dropout(0, 1 << 20, 1 << 16, 1, WORD, 0, WORD, 0, 0.5, 1, 0, None) == deer.DEER_ERR_UNSUPPORTED
    assert lib.deer_matrec_workspace_bytes(ctypes.byref(mat(N=1 << 18, T=1)), 0, ctypes.byref(size)) == deer.DEER_OK
    assert lib.deer_matrec_workspace_bytes(ctypes.byref(mat(N=1 << 20, T=1)), 0, ctypes.byref(size)) == deer.DEER_ERR_UNSUPPORTED
    assert lib.deer_matrec_step(ctypes.byref(mat(N=1 << 22)), WORD, WORD, WORD, WORD, None, 4, WORD, WORD, None) == deer.DEER_ERR_UNSUPPORTED


def test_binding_takes_keywords_and_counts_in_32_bits():
    import torch
    x = torch.zeros(2, 8, 4)
    for call in (lambda: deer.diagrec_solve(gate=x, x=x), lambda: deer.diagrec_solve(x=x), lambda: deer.dropout(x=x, p=0.5, seed=1)):
        with pytest.raises(deer.DeerError) as e:
            call()
        assert e.value.status == deer.DEER_ERR_INVALID_ARG
    deer._int32(0x7FFFFFFF)
    with pytest.raises(deer.DeerError):
        deer._int32(1, 0x80000000)


def test_rows_of_no_sequence_are_zeroed_on_request():
    lib, size, plain = deer.load_library(), ctypes.c_size_t(0), ctypes.c_size_t(0)
    for make, ask in ((diag, lib.deer_diagrec_workspace_bytes), (mat, lib.deer_matrec_workspace_bytes)):
        for grad in (0, 1):
            for packed in (deer.DEER_ROWS_PADDED, deer.DEER_ROWS_PACKED):
                assert ask(ctypes.byref(make(packed=packed)), grad, ctypes.byref(plain)) == deer.DEER_OK
                assert ask(ctypes.byref(make(packed=packed | deer.DEER_REST_ZERO)), grad, ctypes.byref(size)) == deer.DEER_OK
                assert size.value == plain.value
            for bad in (2, deer.DEER_REST_ZERO | 2, 512, -1):
                assert ask(ctypes.byref(make(packed=bad)), grad, ctypes.byref(size)) == deer.DEER_ERR_INVALID_ARG
    packed = diag(packed=deer.DEER_ROWS_PACKED | deer.DEER_REST_ZERO)   # (still needs bounds)
    assert lib.deer_diagrec_solve(ctypes.byref(packed), WORD, WORD, None, None, WORD, None, WORD, 1 << 40, None) == deer.DEER_ERR_INVALID_ARG


def test_launches_of_both_directions_are_looked_at():
    """a workgroup a chunk that there can be: T / 64 + N of them for packed rows, however these are cut"""
    lib, size = deer.load_library(), ctypes.c_size_t(0)
    for grad in (0, 1):
        ask = lambda **kw: lib.deer_matrec_workspace_bytes(ctypes.byref(mat(packed=1, **kw)), grad, ctypes.byref(size))   # noqa: E731
        for N, T, H in ((4096, 1 << 18, 16), (1024, 1 << 20, 16), (1 << 16, 1 << 22, 4)):
            assert ask(N=N, T=T, Hk=H, Hv=H) == deer.DEER_OK
        # 2^32 / 1,024 lanes: up to 4,194,303 chunks
        assert ask(N=1, T=4194302 * 64, Hk=1, Hv=1) == deer.DEER_OK and ask(N=1, T=4194303 * 64, Hk=1, Hv=1) == deer.DEER_ERR_UNSUPPORTED


def test_one_long_sequence_among_many_is_cut():
    """seen by the room for the states of its segments: 64 x 64 floats a segment and head"""
    lib, size = deer.load_library(), ctypes.c_size_t(0)

    def room(**kw):
        assert lib.deer_matrec_workspace_bytes(ctypes.byref(mat(Hk=16, Hv=16, **kw)), 0, ctypes.byref(size)) == deer.DEER_OK
        chunks = kw["T"] // 64 + kw["N"] if kw.get("packed") else kw["T"] // 64 * kw["N"]
        return (size.value - chunks * 16 * 260 * 4) / (16 * 64 * 64 * 4)   # (260 floats a chunk and head for the gates)

    # 512 chunks on 256 CUs and 16 heads: at least 16 segments where one sequence may have them all
    for N in (1, 8, 64, 1024):
        assert room(packed=1, N=N, T=32768) >= 16
    assert room(N=16, T=32768) >= 16 * 16   # a padded batch, for all may be long


# Matrix states: calls whose sequences are cut into segments of several chunks.  segs: for how many states there is room
LONG = {
    "six": dict(H=64, Hk=64, Dk=8, Dv=8, lens=[3001], packed=0, segs=8),                     # 47 chunks on 512 workgroups: 8 segments of 6, the last of 5
    "twelve": dict(H=128, Hk=64, Dk=5, Dv=9, lens=[3001], packed=0, segs=4),                 # 12 chunks, the last 11
    "cap": dict(H=256, Hk=256, Dk=4, Dv=4, lens=[3001], packed=0, segs=2),                   # forward whole (room as with lengths), gradient 32 and 15 chunks
    "packed": dict(H=64, Hk=32, Dk=8, Dv=4, lens=[1500, 3, 0, 2000, 64, 700], packed=1, segs=9),    # 67 + 6 chunks, by 14: fewer than 4,267 / 32 / 14 segments of cut ones
    "padded": dict(H=128, Hk=128, Dk=4, Dv=4, lens=[2200, 100], packed=0, segs=4),           # 35 chunks: 32 and 3, in either direction
    "wide": dict(H=64, Hk=64, Dk=128, Dv=72, lens=[1100], packed=0, segs=6),                 # 18 chunks by 3
}


def test_shapes_with_segments_of_several_chunks():
    lib, size = deer.load_library(), ctypes.c_size_t(0)
    for name, c in LONG.items():
        N, T = len(c["lens"]), sum(c["lens"]) if c["packed"] else max(c["lens"])
        chunks = (T + 63) // 64 + N if c["packed"] else (T + 63) // 64 * N
        cfg = mat(N=N, T=T, packed=c["packed"], Hk=c["Hk"], Hv=c["H"], Dk=c["Dk"], Dv=c["Dv"])
        tile = c["H"] * (64 if c["Dk"] <= 64 else 128) * (64 if c["Dv"] <= 64 else 128) * 4
        assert lib.deer_matrec_workspace_bytes(ctypes.byref(cfg), 0, ctypes.byref(size)) == deer.DEER_OK
        segs = (size.value - chunks * c["H"] * 260 * 4) / tile   # what is left beside the states is less than one of them
        assert c["segs"] <= segs < c["segs"] + 1, (name, segs)


def test_draws_and_seeds_are_not_cut_short():
    assert deer._draw_of(-1, 0) == (0, 2 ** 64 - 1) and deer._draw_of(2 ** 64 - 1, 2 ** 32 - 1) == (2 ** 32 - 1, 2 ** 64 - 1)
    for seed, draw in ((0, 2 ** 32), (0, -1), (2 ** 64, 0), (-2 ** 63 - 1, 0)):
        with pytest.raises(deer.DeerError) as e:
            deer._draw_of(seed, draw)
        assert e.value.status == deer.DEER_ERR_INVALID_ARG


@pytest.mark.parametrize("scale", [1e39, -1e300, float("nan")])
def test_scale_is_a_number_of_32_bits(scale):
    lib, cfg, size = deer.load_library(), mat(scale=scale), ctypes.c_size_t(0)
    ref = ctypes.byref(cfg)
    assert lib.deer_matrec_workspace_bytes(ref, 0, ctypes.byref(size)) == deer.DEER_ERR_INVALID_ARG
    assert lib.deer_matrec_solve(ref, WORD, WORD, WORD, WORD, None, None, WORD, None, WORD, 1 << 40, None) == deer.DEER_ERR_INVALID_ARG
    assert lib.deer_matrec_step(ref, WORD, WORD, WORD, WORD, None, 4, WORD, WORD, None) == deer.DEER_ERR_INVALID_ARG


def test_workspace_does_not_grow_with_sequences_that_are_not_cut():
    """a packed batch of many short sequences: states for what may be cut only, beside 260 floats a chunk and head for the gates"""
    lib, size = deer.load_library(), ctypes.c_size_t(0)
    for N, T, H in ((4096, 1 << 18, 16), (16400, 8200, 64), (100000, 200000, 8)):
        for grad in (0, 1):
            cfg = mat(packed=1, N=N, T=T, Hk=H, Hv=H, Dk=128, Dv=128)
            assert lib.deer_matrec_workspace_bytes(ctypes.byref(cfg), grad, ctypes.byref(size)) == deer.DEER_OK
            chunks, tile = T // 64 + N, H * 128 * 128 * 4
            # two 512ths of the rows a segment (gradient: 32 chunks at most), a state for each of twice as many as that makes; and small numbers by segment, chunk and row
            per = min(max(2 * (T // 64) * H // 512, 1), 32 if grad else 1 << 30)
            assert size.value <= chunks * H * 1200 + 4 * T * H + (1 + grad) * (2 * (T // 64) // per + 1) * tile + 100 * (chunks // per + N) * (1 + H // 8)
            assert size.value < 0.1 * (1 + grad) * N * tile


def test_draws_and_seeds_of_numpy():
    import numpy as np
    for kind in (np.int64, np.uint64, np.int32, np.uint32):
        assert deer._draw_of(kind(7), kind(9)) == (9, 7)
    assert deer._draw_of(np.int64(-1), np.uint32(2 ** 32 - 1)) == (2 ** 32 - 1, 2 ** 64 - 1)
    with pytest.raises(TypeError):
        deer._draw_of(0.5, 0)
