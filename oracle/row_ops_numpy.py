"""fp64 numpy oracle for the operators on rows of the model width: RMSNorm with the residual's addition and a tangent, its
backward, rows in 8 bits, and their products.

TEST INFRASTRUCTURE ONLY.  Shares no code with the CUDA path and must never be imported by the product package.

Every function returns its results together with their `size`: for each element the sum of the magnitudes of the terms that
its formula adds up.  The rounding errors of an fp32 evaluation are bounded by a number of roundings times that.

    h = x + res     r = sqrt(mean(h^2) + eps)     u = h / r     y = g u     (paper Sec. 4 "semi-Lipschitz control")
    th = tx + tres                                ty = g J th   with J v = (v - u (u . v) / D) / r
"""
import numpy as np


def _dot(a, b):
    return (a * b).sum(axis=-1, keepdims=True)


def rmsnorm_jvp_fwd(x, res, tx, tres, g, eps):
    """{"y", "h", "ty", "th": (value, size)} for (..., D) arrays; res, tx, tres, g may be None (ty, th then are too)."""
    D = x.shape[-1]
    h = x if res is None else x + res
    t = tx if tres is None else tx + tres
    g = np.ones(D) if g is None else g
    r = np.sqrt(_dot(h, h) / D + eps)
    u = h / r
    out = {"y": (g * u, np.abs(g * u)), "h": (h, np.abs(h)), "ty": (None, None), "th": (None, None)}
    if t is not None:
        out["th"] = (t, np.abs(t))
        out["ty"] = (g * (t - u * _dot(u, t) / D) / r, np.abs(g) * (np.abs(t) + np.abs(u) * _dot(np.abs(u), np.abs(t)) / D) / r)
    return out


def rmsnorm_jvp_bwd(h, dy, th, dty, dh, dth, g, eps):
    """{"dx", "dtx", "dg": (value, size)}.  dx and dtx as sums over the terms of the derivative; dg over all rows."""
    D = h.shape[-1]
    g = np.ones(D) if g is None else g
    r = np.sqrt(_dot(h, h) / D + eps)
    u, a = h / r, g * dy
    zero = np.zeros_like(h)

    def J(v):
        return (v - u * _dot(u, v) / D) / r, (np.abs(v) + np.abs(u) * _dot(np.abs(u), np.abs(v)) / D) / r

    dx, dx_size = J(a)
    dg, dg_size = dy * u, np.abs(dy * u)
    out = {"dtx": (None, None)}
    if th is not None:
        b = g * dty
        dtx, dtx_size = J(b)
        s, bx, bt = _dot(h, th), _dot(b, h), _dot(b, th)
        s_a, bx_a, bt_a = _dot(np.abs(h), np.abs(th)), _dot(np.abs(b), np.abs(h)), _dot(np.abs(b), np.abs(th))
        dx = dx - (bt * h + s * b + bx * th) / (D * r ** 3) + 3 * bx * s * h / (D * D * r ** 5)
        dx_size = (dx_size + (bt_a * np.abs(h) + s_a * np.abs(b) + bx_a * np.abs(th)) / (D * r ** 3)
                   + 3 * bx_a * s_a * np.abs(h) / (D * D * r ** 5))
        jt, jt_size = J(th)
        dg, dg_size = dg + dty * jt, dg_size + np.abs(dty) * jt_size
        dth = zero if dth is None else dth
        out["dtx"] = (dtx + dth, dtx_size + np.abs(dth))
    dh = zero if dh is None else dh
    out["dx"] = (dx + dh, dx_size + np.abs(dh))
    out["dg"] = (dg.reshape(-1, D).sum(axis=0), dg_size.reshape(-1, D).sum(axis=0))
    return out


def rows_to_8_bits(v):
    """The scales max|v| / 127 of rows (..., D), and v in steps of them (not rounded; zeros for a row of zeros)."""
    s = np.abs(v).max(axis=-1) / 127
    return s, np.divide(v, s[..., None], out=np.zeros_like(v), where=s[..., None] > 0)


def linear_s8(q, s, w, ws, bias):
    """(value, size) of s[m] ws[n] sum_k q[m, k] w[n, k] + bias[n]; the sum in 64-bit integers."""
    y = (q.astype(np.int64) @ w.astype(np.int64).T).astype(np.float64) * s[..., None] * ws
    b = np.zeros(len(ws)) if bias is None else bias
    return y + b, np.abs(y) + np.abs(b)
