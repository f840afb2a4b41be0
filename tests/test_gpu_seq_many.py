"""Matrix states: packed batches of many sequences, and sequences whose segments have several chunks."""
import pytest
import torch

import seq_oracle as so
import test_gpu_matrec as tm
from paper_2309_12252_amd import deer
from test_seq_abi import LONG

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def arrays(seed, dtype, lead, H, Dk, Dv):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    r = lambda *s: torch.randn(lead + s, generator=gen, device=DEV)   # noqa: E731
    return [t.to(dtype) for t in (r(H, Dk), r(H, Dk) / Dk ** 0.5, r(H, Dv), r(H, Dv))] + [-r(H).abs() * 0.1]


@pytest.mark.parametrize("N,L,H,grad", [(4096, 64, 4, True), (4096, 64, 16, False), (1024, 1024, 16, False), (3000, 100, 2, True)])
def test_many_equal_sequences(N, L, H, grad):
    """the same bits as an unpacked batch of them, whose sequences are whole as well; more of them than a chunk's look-up sees at once"""
    q, k, v, do, g = arrays(N, torch.bfloat16, (N * L,), H, 8, 4)
    offsets = torch.arange(N + 1, device=DEV) * L
    apart = lambda t: t.view((N, L) + t.shape[1:])   # noqa: E731
    o, last = deer.matrec_solve(q, k, v, g, offsets=offsets)
    want, wlast = deer.matrec_solve(*(apart(t) for t in (q, k, v, g)))
    assert torch.equal(apart(o), want) and torch.equal(last, wlast)
    if grad:
        got = deer.matrec_grad(q, k, v, g, do, offsets=offsets)
        want = deer.matrec_grad(*(apart(t) for t in (q, k, v, g, do)))
        for a, b in zip(got, want):
            assert torch.equal(a.view(b.shape), b)


def test_many_sequences_of_any_length():
    """5,000 sequences of 0 to 300 rows, every one as it is alone"""
    gen = torch.Generator().manual_seed(5)
    lens = torch.randint(0, 301, (5000,), generator=gen) * (torch.rand(5000, generator=gen) > 0.2)
    lens[17] = 5000
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64), lens.cumsum(0)])
    q, k, v, do, g = arrays(1, torch.float32, (int(offsets[-1]),), 2, 4, 4)
    more = {"offsets": offsets.to(DEV)}
    o, last = deer.matrec_solve(q, k, v, g, **more)
    grads = deer.matrec_grad(q, k, v, g, do, **more)
    for n in [0, 1, 16, 17, 18, 63, 64, 65, 2047, 2048, 4095, 4096, 4998, 4999]:
        a, b = int(offsets[n]), int(offsets[n + 1])
        if a == b:
            assert bool((last[n] == 0).all())
            continue
        alone = [t[None, a:b].contiguous() for t in (q, k, v, g, do)]
        wo, wlast = deer.matrec_solve(*alone[:4])
        wants = deer.matrec_grad(*alone)
        # The sequence is cut elsewhere: every result is a sum of at most 4 (5,000 + 128) rounded terms in either, as in the oracle's bound;
        # the absolute sums behind them stay below 100 of the largest result
        for x, y in zip((o[a:b], last[n]) + tuple(t[a:b] for t in grads[:4]), (wo[0], wlast[0]) + tuple(t[0] for t in wants[:4])):
            assert float((x - y).abs().max()) <= 2 * 4 * (b - a + 128) * 2.0 ** -24 * 100 * float(y.abs().max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(LONG))
def test_segments_of_several_chunks(name, dtype):
    """cut sequences whose segments have more than one chunk: their own parts, the states that are joined, the runs from these"""
    c = LONG[name]
    H, lens, packed = c["H"], c["lens"], c["packed"]
    N, T = len(lens), sum(lens) if packed else max(lens)
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    d = tm.make(dtype, (T,) if packed else (N, T), N, c["Hk"], H, c["Dk"], c["Dv"], len(name))
    more = {"offsets": torch.tensor(off, device=DEV)} if packed else {"lengths": torch.tensor(lens, device=DEV)} if min(lens) < T else {}
    tm.compare(d, tm.both(d, **more), so.sequences(T, N, offsets=off if packed else None, lengths=lens), dtype, c["Dk"] ** -0.5)


@pytest.mark.parametrize("dtype,D", [(torch.float64, 65), (torch.bfloat16, 65), (torch.float32, 130)])
def test_lanes_without_a_channel_at_the_largest_stride(dtype, D):
    """their offsets pass 2^31 on the way along the rows"""
    T, far = 40, 1 << 22
    wide = torch.full((T, far), 5.0, dtype=dtype, device=DEV)
    gate, x, dh = (torch.randn(T, D, device=DEV).to(dtype) for _ in range(3))
    g, u, d, h, dg, du = (wide[:, 200 * i:200 * i + D] for i in range(6))
    for a, b in ((g, gate), (u, x), (d, dh)):
        a.copy_(b)
    offsets = torch.tensor([0, 7, T], device=DEV)
    more = {"kind": deer.DEER_GATE_SIGMOID, "offsets": offsets}
    want = deer.diagrec_solve(gate, x, **more)
    want += deer.diagrec_grad(gate, x, want[0], dh, **more)
    got = deer.diagrec_solve(g, u, out=h, **more)
    got += deer.diagrec_grad(g, u, h, d, dgate=dg, dx=du, **more)
    for a, b in zip(got, want):
        assert torch.equal(a, b)
    for i in range(6):   # nothing beside the rows
        assert bool((wide[:, 200 * i + D:200 * i + 200] == 5).all())
    assert bool((wide[:, 1200:1 << 20] == 5).all())
