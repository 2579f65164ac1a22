"""The sequence layers in plain 64-bit loops, from their formulas, with a bound on what fp32 arithmetic may be off.

Every function returns {name: (value, bound)}: `bound` is an absolute error bound, element by element, for an implementation
that computes in fp32 with elementary functions good to a few units in the last place, before the one rounding to the
storage type.  It is carried through the recurrences as a majorant (absolute values, each step's own rounding added), so
it holds for any order in which the steps are combined.
"""
import numpy as np

U = 2.0 ** -24                      # half a unit in the last place of fp32, relative


def sigmoid(t):
    t = np.asarray(t, np.float64)
    e = np.exp(-np.abs(t))
    return np.where(t >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


def softplus(t):
    t = np.asarray(t, np.float64)
    return np.maximum(t, 0.0) + np.log1p(np.exp(-np.abs(t)))


def recur(x, r, i, lam, spans, h0=None, scale=8.0, dh=None, dhT=None):
    """spans: [(first row, one behind the last row)] of the sequences; rows of none come back as 0.  With dh, the gradients."""
    x, r, i, lam = (np.asarray(t, np.float64) for t in (x, r, i, lam))
    T, C = x.shape
    S = len(spans)
    sr, si = sigmoid(r), sigmoid(i)
    decay = scale * softplus(lam)
    l = -decay * sr
    a = np.exp(l)
    b2 = -np.expm1(2 * l)
    b = np.sqrt(b2)
    # a: the exponent is a product of four factors with 8 roundings, then exp with 4; u: b (12), sigmoid (6), products (2)
    ea, eu = (4 + 8 * np.abs(l)) * U, 24 * U
    # fp32 values below 2^-126 may be taken for 0: then sigmoid(r) is off by that, 1 - a^2 by 2 decay 2^-126 and, where it is
    # that small itself, by 2^-126; b is off by no more than the root of either
    tiny = np.sqrt(2 * decay * 2.0 ** -126) + 2.0 ** -63
    u = b * si * x
    h, herr, hmaj = np.zeros((T, C)), np.zeros((T, C)), np.zeros((T, C))
    before, berr, bmaj = np.zeros((T, C)), np.zeros((T, C)), np.zeros((T, C))
    hT, hTerr = np.zeros((S, C)), np.zeros((S, C))
    for s, (lo, hi) in enumerate(spans):
        st = np.zeros(C) if h0 is None else np.asarray(h0[s], np.float64).copy()
        er, mj = np.zeros(C), np.abs(st)
        for t in range(lo, hi):
            before[t], berr[t], bmaj[t] = st, er, mj
            er = a[t] * er + (ea[t] + 2 * U) * a[t] * mj + eu * np.abs(u[t]) + tiny * np.abs(x[t])
            st, mj = a[t] * st + u[t], a[t] * mj + np.abs(u[t])
            er = er + 2 * U * mj
            h[t], herr[t], hmaj[t] = st, er, mj
        hT[s], hTerr[s] = st, er
    out = {"h": (h, herr), "hT": (hT, hTerr)}
    if dh is None:
        return out
    dh = np.asarray(dh, np.float64)
    g, gerr, gmaj = np.zeros((T, C)), np.zeros((T, C)), np.zeros((T, C))
    dh0, dh0err = np.zeros((S, C)), np.zeros((S, C))
    inside = np.zeros((T, 1))
    for s, (lo, hi) in enumerate(spans):
        inside[lo:hi] = 1
        e = np.zeros(C) if dhT is None else np.asarray(dhT[s], np.float64).copy()
        er, mj = np.zeros(C), np.abs(e)
        for t in range(hi - 1, lo - 1, -1):
            g[t], gmaj[t] = dh[t] + e, np.abs(dh[t]) + mj
            gerr[t] = er + 2 * U * gmaj[t]
            er = a[t] * gerr[t] + (ea[t] + 2 * U) * a[t] * gmaj[t]
            e, mj = a[t] * g[t], a[t] * gmaj[t]
        dh0[s], dh0err[s] = e, er
    with np.errstate(divide="ignore", invalid="ignore"):
        slope = np.where(b > 0, l * a * a / np.where(b > 0, b, 1.0), 0.0)         # l * a^2 / b, 0 where b is
    q = l * a * g * before - slope * g * si * x
    qerr = np.abs(l) * a * (gerr * bmaj + gmaj * berr) + np.abs(slope * si * x) * gerr \
        + (32 + 8 * np.abs(l)) * U * (np.abs(l) * a * gmaj * bmaj + np.abs(slope * si * x) * gmaj) + tiny * np.abs(x) * gmaj
    q, qerr = q * inside, qerr * inside
    dx = b * si * g * inside
    dxerr = (b * si * gerr + 32 * U * b * si * gmaj + tiny * gmaj) * inside
    di = b * x * g * si * (1 - si) * inside
    # 1 - sigmoid loses its leading digits where the gate is open: an absolute error of a few U
    dierr = (np.abs(b * x * si * (1 - si)) * gerr + np.abs(b * x * si) * gmaj * (32 * (1 - si) + 4) * U + tiny * np.abs(x) * gmaj) * inside
    dr = q * (1 - sr)
    drerr = qerr * (1 - sr) + np.abs(q) * 8 * U
    ratio = np.where(lam < -30, 1.0, sigmoid(lam) / softplus(np.maximum(lam, -30)))
    dlam = q.sum(0) * ratio
    dlamerr = (qerr.sum(0) + (T + 16) * U * np.abs(q).sum(0)) * ratio
    out.update(dx=(dx, dxerr), dr=(dr, drerr), di=(di, dierr), dlam=(dlam, dlamerr), dh0=(dh0, dh0err))
    return out


def _act(v, act):
    """act, its slope, and a bound on the slope's slope."""
    from math import pi
    if act == "none":
        return v, np.ones_like(v), 0.0
    if act == "silu":
        s = sigmoid(v)
        return v * s, s * (1 + v * (1 - s)), 0.5
    import torch
    cdf = 0.5 * torch.erfc(torch.from_numpy(-v / np.sqrt(2.0))).numpy()
    pdf = np.exp(-0.5 * v * v) / np.sqrt(2 * pi)
    return v * cdf, cdf + v * pdf, 0.8


def group_norm(x, gamma, beta, groups, eps, act="none", mask=None, dy=None):
    """x [N][P][C].  With dy, the gradients.  Values under the mask are not looked at."""
    x = np.asarray(x, np.float64)
    N, P, C = x.shape
    D = C // groups
    keep = np.ones((N, P, 1, 1)) if mask is None else (np.asarray(mask).reshape(N, P, 1, 1) == 0).astype(np.float64)
    xg = np.where(keep > 0, x.reshape(N, P, groups, D), 0.0)
    gam = np.ones(C) if gamma is None else np.asarray(gamma, np.float64)
    bet = np.zeros(C) if beta is None else np.asarray(beta, np.float64)
    gam, bet = gam.reshape(groups, D), bet.reshape(groups, D)
    count = keep.sum(1, keepdims=True) * D
    M = np.maximum(count, 1)
    total = lambda t: t.sum((1, 3), keepdims=True)
    # sums of M values in at least 32 partial sums that are joined by at most 64 more additions
    es = (M / 32 + 72) * U
    mean = total(xg) / M
    merr = es * total(np.abs(xg)) / M
    d = (xg - mean) * keep
    var = total(d * d) / M
    verr = es * var + 2 * merr * total(np.abs(d)) / M + merr ** 2 + 4 * U * var
    rstd = np.where(count > 0, 1 / np.sqrt(np.where(count > 0, var, 0) + eps) if eps > 0 else 1 / np.sqrt(np.where(var > 0, var, 1)), 0.0)
    rrel = 0.5 * verr / np.maximum(var + eps, 1e-300) + 6 * U
    xh = d * rstd
    xerr = (merr + U * (np.abs(xg) + np.abs(mean))) * rstd + np.abs(xh) * rrel
    v = xh * gam + bet
    verr2 = xerr * np.abs(gam) + 4 * U * (np.abs(xh * gam) + np.abs(bet))
    y, slope, bend = _act(v, act)
    yerr = verr2 * 1.2 + 8 * U * np.abs(v) + 1e-30
    flat = lambda t: (t * keep).reshape(N, P, C)
    stats = np.concatenate((mean.reshape(N, groups, 1), rstd.reshape(N, groups, 1)), 2)
    serr = np.concatenate(((merr + U * np.abs(mean)).reshape(N, groups, 1), (rstd * rrel).reshape(N, groups, 1)), 2)
    out = {"y": (flat(y), flat(yerr)), "stats": (stats, serr)}
    if dy is None:
        return out
    dyg = np.where(keep > 0, np.asarray(dy, np.float64).reshape(N, P, groups, D), 0.0)
    dv = dyg * slope
    dverr = np.abs(dyg) * (bend * verr2 + 16 * U * (1 + np.abs(v))) * keep
    big = (N * P / 32 + 72) * U
    both = lambda t: t.sum((0, 1)).reshape(C)
    dbeta, dberr = both(dv), both(dverr) + big * both(np.abs(dv))
    dgamma, dgerr = both(dv * xh), both(dverr * np.abs(xh) + np.abs(dv) * xerr) + big * both(np.abs(dv * xh))
    w, werr = dv * gam, dverr * np.abs(gam) + 2 * U * np.abs(dv * gam)
    s1, s2 = total(w) / M, total(w * xh) / M
    s1err = total(werr) / M + es * total(np.abs(w)) / M
    s2err = total(werr * np.abs(xh) + np.abs(w) * xerr) / M + es * total(np.abs(w * xh)) / M
    dx = rstd * (w - s1 - xh * s2)
    size = np.abs(w) + np.abs(s1) + np.abs(xh * s2)
    dxerr = rstd * (werr + s1err + np.abs(xh) * s2err + xerr * np.abs(s2) + (rrel + 8 * U) * size)
    out.update(dx=(flat(dx), flat(dxerr)), dgamma=(dgamma, dgerr), dbeta=(dbeta, dberr))
    return out
