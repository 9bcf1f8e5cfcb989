"""Linear attention with decay and group norm in float64 NumPy, token by token and
group by group, with their gradients from the formulas (test infrastructure)."""
import math

import numpy as np


def spans(T, B, cu):
    """(batch row, start, end) of every sequence."""
    if cu is None:
        return [(b, 0, T) for b in range(B)]
    return [(0, int(cu[i]), int(cu[i + 1])) for i in range(len(cu) - 1)]


def linattn(q, k, v, a, scale, s0=None, cu=None, do=None, dsf=None):
    """o, final states; with do (and dsf) also dq, dk, dv, da, ds0."""
    B, T, Hk, Dk = q.shape
    H, Dv = v.shape[2:]
    G = H // Hk
    tok = a if a.ndim == 3 else np.broadcast_to(a, (B, T, H))
    seqs = spans(T, B, cu)
    o = np.zeros((B, T, H, Dv))
    sf = np.zeros((len(seqs), H, Dk, Dv))
    dq, dk, dv = np.zeros((B, T, H, Dk)), np.zeros((B, T, H, Dk)), np.zeros((B, T, H, Dv))
    da, ds0 = np.zeros((B, T, H)), np.zeros_like(sf)
    qh, kh = np.repeat(q, G, 2), np.repeat(k, G, 2)
    for n, (b, t0, t1) in enumerate(seqs):
        S = np.zeros((H, Dk, Dv)) if s0 is None else s0[n].copy()
        before = []
        for t in range(t0, t1):
            before.append(S)
            S = np.exp(tok[b, t])[:, None, None] * S + kh[b, t][:, :, None] * v[b, t][:, None, :]
            o[b, t] = scale * np.einsum("hi,hij->hj", qh[b, t], S)
            if do is not None:
                dq[b, t] = scale * np.einsum("hij,hj->hi", S, do[b, t])
        sf[n] = S
        if do is None:
            continue
        M = np.zeros((H, Dk, Dv)) if dsf is None else dsf[n].copy()
        for t in range(t1 - 1, t0 - 1, -1):
            M = M + scale * qh[b, t][:, :, None] * do[b, t][:, None, :]
            dk[b, t] = np.einsum("hij,hj->hi", M, v[b, t])
            dv[b, t] = np.einsum("hij,hi->hj", M, kh[b, t])
            e = np.exp(tok[b, t])
            da[b, t] = e * (before[t - t0] * M).sum((1, 2))
            M = e[:, None, None] * M
        ds0[n] = M
    if do is None:
        return o, sf
    share = lambda g: g.reshape(B, T, Hk, G, Dk).sum(3)  # noqa: E731
    return o, sf, share(dq), share(dk), dv, (da if a.ndim == 3 else da.sum((0, 1))), ds0


def _erf(z):
    return np.vectorize(math.erf)(z)


def group_norm(x, G, w=None, b=None, eps=1e-5, act="none", dy=None):
    """y (and dx, dw, db with dy); x (B, L, C)."""
    B, L, C = x.shape
    w = np.ones(C) if w is None else w
    b = np.zeros(C) if b is None else b
    v = x.reshape(B, L, G, C // G)
    mean = v.mean((1, 3), keepdims=True)
    r = 1 / np.sqrt(((v - mean) ** 2).mean((1, 3), keepdims=True) + eps)
    xh = ((v - mean) * r).reshape(B, L, C)
    z = xh * w + b
    if act == "silu":
        g = 1 / (1 + np.exp(-z))
        y, slope = z * g, g * (1 + z * (1 - g))
    elif act == "gelu":
        cdf = 0.5 * (1 + _erf(z / math.sqrt(2)))
        y, slope = z * cdf, cdf + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    else:
        y, slope = z, np.ones_like(z)
    if dy is None:
        return y
    dz = dy * slope
    d = (dz * w).reshape(v.shape)
    xg = xh.reshape(v.shape)
    dx = r * (d - d.mean((1, 3), keepdims=True) - xg * (d * xg).mean((1, 3), keepdims=True))
    return y, dx.reshape(x.shape), (dz * xh).sum((0, 1)), dz.sum((0, 1))
