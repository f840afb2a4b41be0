"""Plain 64-bit forms of the short convolution, the selective scan and the group norm, row by row on the host, with bounds of the rounding errors that 32-bit (or
64-bit) arithmetic may make, for the tests' tolerances.  Rows are flat; `seqs` are (first row, length) of the sequences.

u is the unit roundoff of the arithmetic.  A sum of n products in any order is off by at most (n + 1) u times the sum of their sizes.  exp is off by 2 u and by
what its argument is off by: the product with log2 e in front of the hardware's 2^x rounds v to |v| u.  1 / x: 2 u.  So sigmoid(v) = 1 / (1 + exp(-v)) is off by (|v| + 6) u
of itself, v sigmoid(v) by (|v| + 7) u of itself, and the derivative g (1 + v (1 - g)) by (|v| + 8)(1 + |v|) u (g and 1 - g at most 1, three more roundings)."""
import numpy as np

from seq_oracle import HALF, TINY, TYPES, check, sequences   # noqa: F401

U = {"f32": 2.0 ** -24, "f64": 2.0 ** -53, "bf16": 2.0 ** -24, "f16": 2.0 ** -24}


def sigmoid(v):
    with np.errstate(over="ignore"):
        return np.where(v >= 0, 1 / (1 + np.exp(-np.abs(v))), np.exp(-np.abs(v)) / (1 + np.exp(-np.abs(v))))


def act_of(silu, v, E, u):
    """value and derivative of the activation at v, which is off by E, and their bounds (the second derivative is at most 1/2)"""
    if not silu:
        return v, np.ones_like(v), E, np.zeros_like(v)
    g = sigmoid(v)
    slope = g * (1 + v * (1 - g))
    return v * g, slope, 1.1 * E + (np.abs(v) + 7) * u * np.abs(v * g), 0.5 * E + (np.abs(v) + 8) * (1 + np.abs(v)) * u


# ---- short convolution ----
def conv(x, w, bias, s0, seqs, silu, u, dy=None, dlast=None):
    """dict of (value, bound): y, last, and dx, dw, dbias, ds0"""
    rows, D = x.shape
    W = w.shape[1]
    out = {n: [np.zeros(sh), np.zeros(sh)] for n, sh in (("y", x.shape), ("last", s0.shape), ("dx", x.shape), ("dw", w.shape), ("dbias", bias.shape), ("ds0", s0.shape))}
    sizes = np.zeros(w.shape), np.zeros(bias.shape)
    for n, (r0, L) in enumerate(seqs):
        full = np.concatenate([s0[n], x[r0:r0 + L]])
        out["last"][0][n] = full[L:]
        win = np.stack([full[j:j + L] for j in range(W)], -1)   # [L, D, W]
        v, size = bias + (win * w).sum(-1), np.abs(bias) + np.abs(win * w).sum(-1)
        y, slope, Ey, Es = act_of(silu, v, (W + 2) * u * size, u)
        out["y"][0][r0:r0 + L], out["y"][1][r0:r0 + L] = y, Ey
        if dy is None:
            continue
        d, Ed = dy[r0:r0 + L] * slope, np.abs(dy[r0:r0 + L]) * (Es + 2 * u * np.abs(slope))
        dfull, Efull = np.zeros_like(full), np.zeros_like(full)
        for j in range(W):
            dfull[j:j + L] += w[:, j] * d
            Efull[j:j + L] += np.abs(w[:, j]) * (Ed + (W + 3) * u * np.abs(d))
            out["dw"][0][:, j] += (d * win[..., j]).sum(0)
            out["dw"][1][:, j] += (Ed * np.abs(win[..., j])).sum(0)
            sizes[0][:, j] += np.abs(d * win[..., j]).sum(0)
        out["dbias"][0] += d.sum(0)
        out["dbias"][1] += Ed.sum(0)
        sizes[1][:] += np.abs(d).sum(0)
        dfull[L:] += dlast[n]
        Efull[L:] += 2 * u * np.abs(dlast[n])
        out["ds0"][0][n], out["ds0"][1][n] = dfull[:W - 1], Efull[:W - 1]
        out["dx"][0][r0:r0 + L], out["dx"][1][r0:r0 + L] = dfull[W - 1:], Efull[W - 1:]
    # sums over the rows: 40 in a row by a lane and a workgroup's phases, then in 64 bits
    for k, name in enumerate(("dw", "dbias")):
        out[name][1] = out[name][1] + 300 * u * sizes[k]
    return out


# ---- selective scan ----
def scan(x, dt, A, B, C, skip, z, bias, h0, seqs, softplus, dy=None, dlast=None):
    """x, dt, z [rows, D], B, C [rows, G, S] -> dict of (value, bound).  The 32 bits of the kernels: u = 2^-24."""
    u = 2.0 ** -24
    rows, D = x.shape
    G, S = B.shape[1:]
    group = np.arange(D) // (D // G)
    raw = dt + bias
    with np.errstate(over="ignore"):
        d = np.where(raw > 0, raw, 0) + np.log1p(np.exp(-np.abs(raw))) if softplus else raw
    # softplus: raw is off by |raw| u, which moves it by at most as much of itself, exp(-|raw|) by (|raw| + 2) u, and ten roundings; no softplus: one rounding
    ed = (2 * np.abs(raw) + 14) * u if softplus else np.full_like(raw, u) * np.abs(raw) / np.maximum(np.abs(d), 1e-300)
    Bc, Cc = B[:, group], C[:, group]   # [rows, D, S]
    names = {"y": x.shape, "last": h0.shape, "dx": x.shape, "ddt": x.shape, "dA": A.shape, "dB": B.shape, "dC": C.shape, "dskip": (D,), "dz": x.shape, "dbias": (D,),
             "dh0": h0.shape}
    out = {n: [np.zeros(sh), np.zeros(sh)] for n, sh in names.items()}
    gate, gslope, Eg, Egs = act_of(z is not None, z, np.zeros_like(z), u) if z is not None else (np.ones_like(x), np.zeros_like(x), np.zeros_like(x), np.zeros_like(x))
    sizes = {n: np.zeros(names[n]) for n in ("dA", "dskip", "dbias")}
    up = lambda t, ax: t.reshape(t.shape[:ax] + (G, D // G) + t.shape[ax + 1:]).sum(ax + 1)   # noqa: E731
    for n, (r0, L) in enumerate(seqs):
        if L == 0:
            out["last"][0][n] = h0[n]
            if dy is not None:
                out["dh0"][0][n] = dlast[n]
            continue
        sl = slice(r0, r0 + L)
        arg = d[sl, :, None] * A
        with np.errstate(over="ignore"):
            a = np.exp(arg)
        # the argument: dt, its product, A times log2 e and the product with it; sums of dt over a segment of at most L rows
        ea = np.abs(arg) * (ed[sl, :, None] + (4 + L) * u) + 3 * u
        inp = (d[sl] * x[sl])[..., None] * Bc[sl]
        h, E, M = np.zeros((L, D, S)), np.zeros((L, D, S)), np.zeros((L, D, S))
        now, e, m = h0[n], np.zeros((D, S)), np.abs(h0[n])
        for t in range(L):
            e = a[t] * e + (ea[t] + 3 * u) * a[t] * m + (ed[r0 + t, :, None] + 5 * u) * np.abs(inp[t])
            now, m = a[t] * now + inp[t], a[t] * m + np.abs(inp[t])
            h[t], E[t], M[t] = now, e, m
        out["last"][0][n], out["last"][1][n] = now, e
        pre = (Cc[sl] * h).sum(-1) + skip * x[sl]
        size = (np.abs(Cc[sl]) * M).sum(-1) + np.abs(skip * x[sl])
        Epre = (np.abs(Cc[sl]) * E).sum(-1) + (S + 3) * u * size
        out["y"][0][sl], out["y"][1][sl] = pre * gate[sl], Epre * np.abs(gate[sl]) + size * (Eg[sl] + 2 * u * np.abs(gate[sl]))
        if dy is None:
            continue
        out["dz"][0][sl], out["dz"][1][sl] = dy[sl] * pre * gslope[sl], np.abs(dy[sl]) * (Epre * np.abs(gslope[sl]) + size * (Egs[sl] + 3 * u * np.abs(gslope[sl])))
        o, Eo = dy[sl] * gate[sl], np.abs(dy[sl]) * (Eg[sl] + u * np.abs(gate[sl]))
        r, er, mr = dlast[n], np.zeros((D, S)), np.abs(dlast[n])
        lam, El, Ml = np.zeros_like(h), np.zeros_like(h), np.zeros_like(h)
        for t in range(L - 1, -1, -1):
            term, Et = o[t][:, None] * Cc[r0 + t], Eo[t][:, None] * np.abs(Cc[r0 + t])
            lam[t], Ml[t] = r + term, mr + np.abs(term)
            El[t] = er + Et + 3 * u * Ml[t]
            r, er, mr = a[t] * lam[t], a[t] * El[t] + (ea[t] + 2 * u) * a[t] * Ml[t], a[t] * Ml[t]
        out["dh0"][0][n], out["dh0"][1][n] = r, er
        hp, Ep, Mp = np.concatenate([h0[n][None], h[:-1]]), np.concatenate([np.zeros((1, D, S)), E[:-1]]), np.concatenate([np.abs(h0[n])[None], M[:-1]])
        g = lam * a * hp
        Gm = Ml * a * Mp
        EG = El * a * Mp + Ml * a * Ep + (ea + 3 * u) * Gm
        out["dA"][0] += (d[sl][..., None] * g).sum(0)
        dd = np.abs(d[sl])[..., None]
        out["dA"][1] += (dd * (EG + ed[sl][..., None] * Gm)).sum(0)
        sizes["dA"] += (dd * Gm).sum(0)
        read, Mread = (lam * Bc[sl]).sum(-1), (Ml * np.abs(Bc[sl])).sum(-1)
        Eread = (El * np.abs(Bc[sl])).sum(-1) + (S + 2) * u * Mread
        w, Mw = (A * g).sum(-1), (np.abs(A) * Gm).sum(-1)
        Ew = (np.abs(A) * EG).sum(-1) + (S + 2) * u * Mw
        dd = dd[..., 0]
        out["dx"][0][sl] = d[sl] * read + skip * o
        out["dx"][1][sl] = dd * (Eread + (ed[sl] + 2 * u) * Mread) + np.abs(skip) * (Eo + 2 * u * np.abs(o))
        slope = sigmoid(raw[sl]) if softplus else np.ones_like(w)
        es = (2 * np.abs(raw[sl]) + 8) * u if softplus else 0.0
        ddt, Mdt = (w + x[sl] * read) * slope, (Mw + np.abs(x[sl]) * Mread) * slope
        Edt = (Ew + np.abs(x[sl]) * Eread) * slope + (es + 4 * u) * Mdt
        out["ddt"][0][sl], out["ddt"][1][sl] = ddt, Edt
        out["dbias"][0] += ddt.sum(0)
        out["dbias"][1] += Edt.sum(0)
        sizes["dbias"] += Mdt.sum(0)
        out["dskip"][0] += (o * x[sl]).sum(0)
        out["dskip"][1] += (Eo * np.abs(x[sl])).sum(0)
        sizes["dskip"] += np.abs(o * x[sl]).sum(0)
        dx = (d[sl] * x[sl])[..., None]
        out["dB"][0][sl] = up(lam * dx, 1)
        out["dB"][1][sl] = up(El * np.abs(dx) + (ed[sl][..., None] + (D // G + 3) * u) * Ml * np.abs(dx), 1)
        out["dC"][0][sl] = up(o[..., None] * h, 1)
        out["dC"][1][sl] = up(Eo[..., None] * M + np.abs(o)[..., None] * (E + (D // G + 2) * u * M), 1)
    for n, t in sizes.items():   # sums over at most as many rows as there are
        out[n][1] = out[n][1] + (rows + 4) * u * t
    return out


# ---- group norm ----
def norm(x, G, w, bias, z, seqs, by_row, eps, silu, u, dy=None):
    """x, z [rows, D] -> dict of (value, bound): y, stats, and dx, dw, dbias, dz"""
    rows, D = x.shape
    per = D // G
    shape = (rows, G, 2) if by_row else (len(seqs), G, 2)
    out = {n: [np.zeros(sh), np.zeros(sh)] for n, sh in (("y", x.shape), ("stats", shape), ("dx", x.shape), ("dw", (D,)), ("dbias", (D,)), ("dz", x.shape))}
    sizes = np.zeros(D), np.zeros(D)
    spans = [(n, r0 + r, 1) for n, (r0, L) in enumerate(seqs) for r in range(L)] if by_row else [(n, r0, L) for n, (r0, L) in enumerate(seqs) if L]
    for n, r0, L in spans:
        sl = slice(r0, r0 + L)
        v = x[sl].reshape(L, G, per)
        count = L * per
        mean = v.mean((0, 2), keepdims=True)
        var = ((v - mean) ** 2).mean((0, 2), keepdims=True)
        rstd = (var + eps) ** -0.5
        # Sums of at most k values in 32 bits (a row's channels; 64 rows of a piece, joined in 64 bits).  The mean is off by k u of the mean size of what is summed; over pieces these are
        # differences from a row: at most |x - mean| + |first - mean|, and then the mean itself rounded.  The variance: of differences that are off by Em each, and
        # over pieces 66 times the squares' rounding, which the difference with the piece's mean leaves.
        k = per + 2 if by_row else 66
        size = np.abs(v).mean((0, 2), keepdims=True) if by_row else np.abs(v - mean).mean((0, 2), keepdims=True) + np.abs(v - mean).max((0, 2), keepdims=True)
        Em = k * u * size + 2 * u * np.abs(mean)
        Evar = 2 * Em ** 2 + (k + 4) * u * var * (1 if by_row else 66) + 4 * u * np.abs(mean) * var ** 0.5
        er = 0.5 * Evar / (var + eps) + 4 * u
        out["stats"][0][r0 if by_row else n] = np.stack([mean, rstd], -1)[0, :, 0]
        out["stats"][1][r0 if by_row else n] = np.stack([Em, er * rstd], -1)[0, :, 0]
        unit = (v - mean) * rstd
        Eu = (Em + u * np.abs(v - mean)) * rstd + (er + 2 * u) * np.abs(unit)
        unit, Eu, Er = unit.reshape(L, D), Eu.reshape(L, D), np.repeat(er.reshape(G), per)
        R = np.repeat(rstd.reshape(G), per)
        pre = unit * w + bias
        f, slope, Ef, Es = act_of(silu, pre, Eu * np.abs(w) + 3 * u * (np.abs(unit * w) + np.abs(bias)), u)
        zero = np.zeros_like(f)
        gate, gslope, Eg, Egs = act_of(True, z[sl], zero, u) if z is not None else (zero + 1, zero, zero, zero)
        out["y"][0][sl], out["y"][1][sl] = f * gate, Ef * np.abs(gate) + np.abs(f) * (Eg + 2 * u * np.abs(gate))
        if dy is None:
            continue
        o = np.abs(dy[sl])
        out["dz"][0][sl], out["dz"][1][sl] = dy[sl] * f * gslope, o * (Ef * np.abs(gslope) + np.abs(f) * (Egs + 3 * u * np.abs(gslope)))
        dv = dy[sl] * gate * slope
        Edv = o * (Eg * np.abs(slope) + np.abs(gate) * Es) + 3 * u * np.abs(dv)
        du, Edu = dv * w, Edv * np.abs(w) + u * np.abs(dv * w)
        each = lambda t: np.repeat(t.reshape(L, G, per).mean((0, 2)), per)   # noqa: E731
        s1, s2 = each(du), each(du * unit)
        Esum = (k + 3) * u if by_row else 70 * u
        E1, E2 = each(Edu + Esum * np.abs(du)), each(Edu * np.abs(unit) + np.abs(du) * Eu + Esum * np.abs(du * unit))
        inner = du - s1 - unit * s2
        out["dx"][0][sl] = R * inner
        out["dx"][1][sl] = R * (Edu + E1 + np.abs(unit) * E2 + Eu * np.abs(s2) + 5 * u * (np.abs(du) + np.abs(s1) + np.abs(unit * s2)) + Er * np.abs(inner))
        out["dw"][0] += (dv * unit).sum(0)
        out["dw"][1] += (Edv * np.abs(unit) + np.abs(dv) * Eu).sum(0)
        out["dbias"][0] += dv.sum(0)
        out["dbias"][1] += Edv.sum(0)
        sizes[0][:] += np.abs(dv * unit).sum(0)
        sizes[1][:] += np.abs(dv).sum(0)
    for i, name in enumerate(("dw", "dbias")):   # sums over the rows, at most so many
        out[name][1] = out[name][1] + (rows + 4) * u * sizes[i]
    return out
