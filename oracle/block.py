"""CPU oracle of the row operators, fp64 numpy: 8-bit checkpoints, and the residual block around a layer (norm behind it, gate,
residual scale, residual sum, norm in front of the next layer) with its gradients, from the formulas of the header.

Every function of the block also returns, under ``abs``, the formula evaluated on the magnitudes of its terms: an fp32 evaluation
with k roundings on the way to an entry is off by at most about k * 2^-24 times that."""
from __future__ import annotations

import numpy as np

GROUP = 32


def act8_pack(X):
    """(q int8 [n, D], scale bytes in their layout) of an fp32 matrix.  The scale of a group is the least power of two 2^s, s >= -126,
    with max|x| < 127.5 * 2^s, at most 2^121; q = x / 2^s to the nearest integer, ties to even; byte s + 127, 255 for groups that are
    not finite."""
    X = np.asarray(X, dtype=np.float64)
    n, D = X.shape
    G = -(-D // GROUP)
    q = np.zeros((n, D), np.int8)
    byte = np.zeros((-(-n // 8) * 8, G), np.uint8)
    for g in range(G):
        v = X[:, g * GROUP:(g + 1) * GROUP]
        top = np.abs(v).max(axis=1)
        fine = np.isfinite(top)
        s = np.full(n, -126)
        for _ in range(248):
            s = np.where(fine & (top >= np.ldexp(127.5, s)) & (s < 121), s + 1, s)
        with np.errstate(invalid="ignore"):
            c = np.clip(np.rint(np.where(fine[:, None], v, 0.0) / np.ldexp(1.0, s)[:, None]), -127, 127)
        q[:, g * GROUP:(g + 1) * GROUP] = c
        byte[:n, g] = np.where(fine, s + 127, 255)
    return q, byte.reshape(-1, 8, G).transpose(0, 2, 1).reshape(-1).copy()


def act8_values(q, scale):
    n, D = q.shape
    G = -(-D // GROUP)
    b = scale.reshape(-1, G, 8).transpose(0, 2, 1).reshape(-1, G)[:n].astype(int)
    f = np.where(b == 255, np.nan, np.ldexp(1.0, b - 127))
    return q.astype(np.float64) * np.repeat(f, GROUP, axis=1)[:, :D]


def row_stats(x, layer, eps):
    """(m, r), each [n, 1]"""
    m = x.mean(axis=1, keepdims=True) if layer else np.zeros((x.shape[0], 1))
    return m, 1 / np.sqrt(((x - m) ** 2).mean(axis=1, keepdims=True) + eps)


def _sigmoid(g):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-g))


def _or(v, D, value):
    return np.full(D, float(value)) if v is None else np.asarray(v, dtype=np.float64)


def _mean(x):
    return x.mean(axis=1, keepdims=True)


def block_fwd(X, Y=None, G=None, layer=False, eps=1e-5, w_after=None, b_after=None, scale=None, w_before=None, b_before=None):
    X = np.asarray(X, dtype=np.float64)
    D = X.shape[1]
    wa, ba, sc, wb, bb = (_or(v, D, o) for v, o in ((w_after, 1), (b_after, 0), (scale, 1), (w_before, 1), (b_before, 0)))
    out, mag = {}, {}
    x, dx = X, np.zeros_like(X)
    if Y is not None:
        y = np.asarray(Y, dtype=np.float64)
        m, r = row_stats(y, layer, eps)
        yh = (y - m) * r
        g = 1.0 if G is None else _sigmoid(np.asarray(G, dtype=np.float64))
        x = X + sc * g * (yh * wa + ba)
        # magnitudes: the mean of a row is off by what its entries weigh, |m| r + 1 in units of the deviation
        dx = np.abs(X) + np.abs(sc * g) * (np.abs(wa) * (np.abs(yh) + np.abs(m) * r + 1) + np.abs(ba))
        out.update(X_out=x, m_after=m, r_after=r)
        mag.update(X_out=dx)
    m, r = row_stats(x, layer, eps)
    xh = (x - m) * r
    out.update(N=xh * wb + bb, m_before=m, r_before=r)
    err = np.maximum(dx, np.abs(x))
    mag["N"] = np.abs(wb) * (r * (err + _mean(err)) + np.abs(xh) * (1 + r * np.sqrt(_mean(err ** 2))) + np.abs(m) * r + 1) + np.abs(bb)
    # the statistics: a mean is off by the entries' magnitudes, a deviation by its own relative error and the mean of their errors
    mag["m_before"], mag["r_before"] = _mean(err), r * (1 + r * np.sqrt(_mean(err ** 2)))
    if Y is not None:
        mag["m_after"] = _mean(np.abs(y))
        mag["r_after"] = out["r_after"] * (1 + out["r_after"] * np.sqrt(_mean(y ** 2)))
    return dict(out, abs=mag)


def block_bwd(dX_out=None, dN=None, X_out=None, stats_before=None, Y=None, stats_after=None, G=None, layer=False, w_after=None,
              b_after=None, scale=None, w_before=None):
    """Statistics are pairs (m, r) of [n, 1].  X_out, Y, G: the values the gradient is taken at."""
    some = dX_out if dX_out is not None else dN
    n, D = some.shape
    f = lambda a: None if a is None else np.asarray(a, dtype=np.float64)          # noqa: E731
    dX_out, dN, X_out, Y, G = (f(a) for a in (dX_out, dN, X_out, Y, G))
    wa, ba, sc, wb = (_or(v, D, o) for v, o in ((w_after, 1), (b_after, 0), (scale, 1), (w_before, 1)))
    out, mag = {}, {}

    def through(g, ag, xh, ah, r):
        """gradient of a norm's input from that of its result, and its magnitude"""
        v = r * (g - (_mean(g) if layer else 0.0) - xh * _mean(g * xh))
        return v, r * (ag + (_mean(ag) if layer else 0.0) + ah * _mean(ag * ah))

    d = np.zeros((n, D)) if dX_out is None else dX_out.copy()
    ad = np.abs(d)
    if dN is not None:
        m, r = stats_before
        xh, ah = (X_out - m) * r, (np.abs(X_out) + np.abs(m)) * r
        b, ab = through(dN * wb, np.abs(dN * wb), xh, ah, r)
        d, ad = d + b, ad + ab
        out.update(dw_before=(dN * xh).sum(0), db_before=dN.sum(0))
        mag.update(dw_before=(np.abs(dN) * ah).sum(0), db_before=np.abs(dN).sum(0))
    out["dX"], mag["dX"] = d, ad
    if Y is not None:
        m, r = stats_after
        yh, ah = (Y - m) * r, (np.abs(Y) + np.abs(m)) * r
        u, au = yh * wa + ba, ah * np.abs(wa) + np.abs(ba)
        sig = np.ones((n, 1)) if G is None else _sigmoid(G)
        du, adu = d * sc * sig, ad * np.abs(sc) * sig
        if G is not None:
            shut = _sigmoid(-G)                       # 1 - sig
            dG, adG = d * sc * u * sig * shut, ad * np.abs(sc) * au * sig * shut
            if G.shape[1] == 1 and D > 1:
                dG, adG = dG.sum(1, keepdims=True), adG.sum(1, keepdims=True)
            out["dG"], mag["dG"] = dG, adG
        out.update(dw_after=(du * yh).sum(0), db_after=du.sum(0), dscale=(d * sig * u).sum(0))
        mag.update(dw_after=(adu * ah).sum(0), db_after=adu.sum(0), dscale=(ad * sig * au).sum(0))
        out["dY"], mag["dY"] = through(du * wa, adu * np.abs(wa), yh, ah, r)
    return dict(out, abs=mag)
