"""Plain 64-bit forms of the sequence operators, row by row on the host, with running bounds of the rounding errors that 32-bit
(or 64-bit) arithmetic may make, for the tests' tolerances.

The bounds: a state h_t = a_t h_{t-1} + u_t computed in any association of its products and sums is off by at most E_t,
E_t = |a_t| E_{t-1} + c u (|a_t| M_{t-1} + |u_t|), where M is the same recurrence over absolute values, u the unit roundoff and c counts the
roundings that one row adds to every term that passes it: the factor itself (its exp or sigmoid), its product into the running
product of the factors, the product with the state and the sum, of the term's input likewise.
"""
import numpy as np
import torch

TYPES = {"f32": torch.float32, "f64": torch.float64, "bf16": torch.bfloat16, "f16": torch.float16}
# half a step of the output type, relative; smallest step, absolute (16-bit floats and below have numbers without leading one)
HALF = {"f32": 2.0 ** -24, "f64": 2.0 ** -53, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TINY = {"f32": 2.0 ** -126, "f64": 1e-300, "bf16": 2.0 ** -126, "f16": 2.0 ** -24}
UNIT = {"f32": 2.0 ** -24, "f64": 2.0 ** -53, "bf16": 2.0 ** -24, "f16": 2.0 ** -24}
# roundings a row adds: 2 sums and products and 1 product of factors, 2 more for the carry's, and the factor: exp within 1 ulp = 2 u (sigmoid: exp, sum,
# reciprocal, product = 5 u).  With 16-bit inputs the hardware's exp and reciprocal: 2 ulp of 2^x, and the product
# with log2 e in front of it rounds an argument of up to |g| = 12 to 2^-24 * 12 * 1.44 relative to one: 24 in all.
ROUNDINGS = {"f32": 12, "f64": 12, "bf16": 32, "f16": 32}


def sequences(T, N, offsets=None, lengths=None):
    """(first row, length) of every sequence in the flat rows"""
    if offsets is not None:
        return [(offsets[n], offsets[n + 1] - offsets[n]) for n in range(len(offsets) - 1)]
    return [(n * T, T if lengths is None else lengths[n]) for n in range(N)]


def factors(kind, g):
    with np.errstate(over="ignore"):
        if kind == 2:
            a = np.where(g >= 0, 1 / (1 + np.exp(-np.abs(g))), np.exp(-np.abs(g)) / (1 + np.exp(-np.abs(g))))
            return a, np.where(g >= 0, np.exp(-np.abs(g)) / (1 + np.exp(-np.abs(g))), 1 / (1 + np.exp(-np.abs(g))))
        return (np.exp(g) if kind == 1 else g), np.ones_like(g)


def philox_keep(N, T, D, p, seed, draw):
    """[N, T, D]: 2^16 / (2^16 - cut) where an element is kept, else 0"""
    cut = int(round(p * 65536))
    c = [np.empty((N, (T + 7) // 8, D), dtype=np.uint64) for _ in range(4)]
    c[0][:], c[1][:] = np.arange(D, dtype=np.uint64), np.arange(c[0].shape[1], dtype=np.uint64)[:, None]
    c[2][:], c[3][:] = np.arange(N, dtype=np.uint64)[:, None, None], np.uint64(draw)
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    low = np.uint64(0xFFFFFFFF)
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> np.uint64(32)) ^ c[1] ^ np.uint64(k0), p1 & low, (p0 >> np.uint64(32)) ^ c[3] ^ np.uint64(k1), p0 & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    bits = np.stack([w >> np.uint64(s) & np.uint64(0xFFFF) for w in c for s in (0, 16)], axis=2)   # N, block, row of the block, D
    keep = bits.reshape(N, -1, D)[:, :T] >= cut
    return np.where(keep, 65536.0 / (65536 - cut), 0.0)


def diag_forward(kind, g, x, h0, seqs, c_u):
    """flat rows -> h, last, bounds of both"""
    a, w = factors(kind, g)
    u = w * x
    h, E = np.zeros_like(x), np.zeros_like(x)
    last, Elast = np.array(h0), np.zeros_like(h0)
    for s, (r0, length) in enumerate(seqs):
        now, M, e = h0[s].copy(), np.abs(h0[s]), np.zeros_like(h0[s])
        for r in range(r0, r0 + length):
            e = np.abs(a[r]) * e + c_u * (np.abs(a[r]) * M + np.abs(u[r]))
            now = a[r] * now + u[r]
            M = np.abs(a[r]) * M + np.abs(u[r])
            h[r], E[r] = now, e
        last[s], Elast[s] = now, e
    return h, last, E, Elast


def diag_backward(kind, g, x, h, dh, h0, dlast, seqs, c_u):
    """at the trajectory h: dgate, dx, dh0 and their bounds"""
    a, w = factors(kind, g)
    dg, dx, Eg, Ex = (np.zeros_like(x) for _ in range(4))
    dh0, E0 = np.array(dlast), np.zeros_like(dlast)
    for s, (r0, length) in enumerate(seqs):
        mu, M, e = dlast[s].copy(), np.abs(dlast[s]), np.zeros_like(dlast[s])
        for r in range(r0 + length - 1, r0 - 1, -1):
            before = h[r - 1] if r > r0 else h0[s]
            lam, el, al = dh[r] + mu, e + c_u * (np.abs(dh[r]) + M), np.abs(dh[r]) + M
            if kind == 2:
                size = np.abs(before) + np.abs(x[r])
                dg[r], Eg[r] = lam * a[r] * w[r] * (before - x[r]), a[r] * w[r] * size * (el + c_u * al)
                dx[r], Ex[r] = lam * w[r], w[r] * (el + c_u * al)
            else:
                f = a[r] if kind == 1 else np.ones_like(a[r])
                dg[r], Eg[r] = lam * before * f, np.abs(f * before) * (el + c_u * al)
                dx[r], Ex[r] = lam, el
            mu, e, M = a[r] * lam, np.abs(a[r]) * el + c_u * np.abs(a[r]) * al, np.abs(a[r]) * al
        dh0[s], E0[s] = mu, e
    return dg, dx, dh0, Eg, Ex, E0


def check(name, got, want, bound, dtype):
    """|got - want| <= bound + half a step of the type (of the true value, and of the bound's worth), element by element"""
    got = got.detach().cpu().double().numpy().reshape(want.shape)
    tol = bound + HALF[dtype] * (np.abs(want) + bound) * (1 + 2.0 ** -7) + TINY[dtype]
    off = np.abs(got - want)
    bad = ~(off <= tol)
    worst = float((off / tol).max()) if off.size else 0.0
    print("%s: largest error over its bound %.3f" % (name, worst), flush=True)
    assert not bad.any(), "%s: %d of %d outside, worst %.3g at %s (want %.6g got %.6g)" % (
        name, bad.sum(), bad.size, worst, np.unravel_index((off / tol).argmax(), off.shape), want.flat[(off / tol).argmax()], got.flat[(off / tol).argmax()])


# ---- matrix states ----
# For every output its value and the same formula over absolute values ("abs"), which the errors are measured by: a rounding of a factor or of
# a partial sum moves an output by at most half a step of it times abs.  In bf16 an output has one rounded factor in every term (the 64 x 64 factors,
# or the state): 2^-8; states and gates only factors of two pieces: 2^-16.  In fp32 sums of T rows and 128 columns: 4 (T + 128) roundings.
def matrix(q, k, v, g, s0, seqs, scale, do=None, dlast=None):
    """flat rows: q, k [rows, Hk, Dk], v [rows, Hv, Dv], g [rows, Hv] -> dict of (value, abs)"""
    rows, Hv, Dv = v.shape
    kv = np.arange(Hv) * q.shape[1] // Hv
    Q, K = q[:, kv], k[:, kv]
    out = {n: np.zeros(sh) for n, sh in (("o", v.shape), ("last", s0.shape), ("dq", Q.shape), ("dk", Q.shape), ("dv", v.shape), ("dgate", g.shape), ("ds0", s0.shape))}
    absolute = {n: x.copy() for n, x in out.items()}
    with np.errstate(over="ignore", under="ignore"):
        for sign, res in ((False, out), (True, absolute)):
            f = np.abs if sign else (lambda x: x)
            for s, (r0, n) in enumerate(seqs):
                S, states = f(s0[s]).copy(), []
                for r in range(r0, r0 + n):
                    states.append(S)
                    S = np.exp(g[r])[:, None, None] * S + f(K[r])[:, :, None] * f(v[r])[:, None, :]
                    res["o"][r] = scale * np.einsum("hd,hdv->hv", f(Q[r]), S)
                res["last"][s] = S
                if do is None:
                    continue
                states.append(S)
                R = f(dlast[s]).copy()
                for i in range(n - 1, -1, -1):
                    r = r0 + i
                    R = R + scale * f(Q[r])[:, :, None] * f(do[r])[:, None, :]
                    res["dq"][r] = scale * np.einsum("hdv,hv->hd", states[i + 1], f(do[r]))
                    res["dk"][r] = np.einsum("hdv,hv->hd", R, f(v[r]))
                    res["dv"][r] = np.einsum("hdv,hd->hv", R, f(K[r]))
                    R = np.exp(g[r])[:, None, None] * R
                    res["dgate"][r] = np.einsum("hdv,hdv->h", states[i], R)
                res["ds0"][s] = R
    # What goes through a chunk is <S, dS> in front of a segment less and plus sums over its chunks of q_i . dq_i (from the state) and k_j . dk_j:
    # at most all of the sequence's, each a sum of 64 rows of 128 columns of products with sums of 128 columns and the gates' factors
    passing = np.zeros(g.shape)
    if do is not None:
        terms = (np.abs(Q) * absolute["dq"] + np.abs(K) * absolute["dk"]).sum(-1)
        for r0, n in seqs:
            passing[r0:r0 + n] = (64 + 128 + 128) * 2.0 ** -24 * terms[r0:r0 + n].sum(0)
    shared = lambda x: np.stack([x[:, kv == h].sum(1) for h in range(q.shape[1])], 1)   # noqa: E731
    for res in (out, absolute):
        res["dq"], res["dk"] = shared(res["dq"]), shared(res["dk"])
    return out, absolute, passing


def check_matrix(got, want, absolute, passing, dtype, T):
    sums = 4 * (T + 128) * 2.0 ** -24
    for name, t in got.items():
        w, a = want[name], absolute[name]
        if name in ("last", "ds0", "dgate"):
            bound, kind = (sums + (2.0 ** -16 if dtype == "bf16" else 0.0)) * a, "f32"
            if name == "dgate":
                bound = bound + passing
        else:
            bound, kind = (sums + (2.0 ** -8 + 2.0 ** -14 if dtype == "bf16" else 0.0)) * a, dtype
        check(name, t, w, bound, kind)
        # all together: one output of many is off by a random walk of its roundings (each half a step / sqrt 3 at most): in bf16 two of
        # 2^-8 / sqrt 3, for what is fp32 with pieces one of 2^-16 / sqrt 3; fp32: sqrt(4 (T + 128)) of 2^-24 / sqrt 3, rounded up
        if w.size >= 500 and np.linalg.norm(w) > 0:
            rel = np.linalg.norm(t.detach().cpu().double().numpy().reshape(w.shape) - w) / np.linalg.norm(w)
            most = (4 * (T + 128)) ** 0.5 * 2.0 ** -24 + (2.0 ** -16 if dtype == "bf16" else 0.0) if kind == "f32" else 2.0 ** -8
            print("%s: all together %.2g of at most %.2g" % (name, rel, most), flush=True)
            assert rel <= most, (name, rel, most)
