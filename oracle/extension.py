"""Float64 oracle of the parametric extension's operators: layer norm, the
gated feed-forward block and the AdamW step, written from their formulas."""
import math

import numpy as np

BLOCK = 256  # elements that share a scale of 8-bit states


def _phi(x):
    """The normal distribution function; by erfc, which keeps the lower tail."""
    return 0.5 * np.vectorize(math.erfc, otypes=[np.float64])(-np.asarray(x) / math.sqrt(2.0))


def layer_norm(X, gamma=None, beta=None, eps=1e-5):
    """(Y, mean, rstd)."""
    X = np.asarray(X, dtype=np.float64)
    mean = X.mean(axis=1)
    rstd = 1.0 / np.sqrt(((X - mean[:, None]) ** 2).mean(axis=1) + eps)
    Y = (X - mean[:, None]) * rstd[:, None]
    if gamma is not None:
        Y = Y * gamma
    if beta is not None:
        Y = Y + beta
    return Y, mean, rstd


def layer_norm_backward(dY, X, gamma=None, eps=1e-5, add=None):
    """(dX, dgamma, dbeta)."""
    h, _, rstd = layer_norm(X, eps=eps)
    dY = np.asarray(dY, dtype=np.float64)
    g = dY if gamma is None else dY * gamma
    dX = rstd[:, None] * (g - g.mean(axis=1, keepdims=True)
                          - h * (g * h).mean(axis=1, keepdims=True))
    if add is not None:
        dX = dX + add
    return dX, (dY * h).sum(axis=0), dY.sum(axis=0)


def activation(g, act):
    """act(g) and its derivative."""
    if act == "silu":
        z = 1.0 / (1.0 + np.exp(-g))
        return g * z, z + g * z * (1.0 - z)
    z = _phi(g)
    return g * z, z + g * np.exp(-g * g / 2.0) / math.sqrt(2.0 * math.pi)


def gated(X, Wg, Wu, Wd, bg=0.0, bu=0.0, bd=0.0, R=0.0, act="silu"):
    """(Y, G, U, H)."""
    X, Wg, Wu, Wd = (np.asarray(a, dtype=np.float64) for a in (X, Wg, Wu, Wd))
    G, U = X @ Wg.T + bg, X @ Wu.T + bu
    H = activation(G, act)[0] * U
    return H @ Wd.T + bd + R, G, U, H


def gated_backward(dY, X, Wg, Wu, Wd, bg=0.0, bu=0.0, act="silu"):
    """The gradients by name."""
    dY, X, Wg, Wu, Wd = (np.asarray(a, dtype=np.float64) for a in (dY, X, Wg, Wu, Wd))
    _, G, U, H = gated(X, Wg, Wu, Wd, bg, bu, act=act)
    value, slope = activation(G, act)
    dH = dY @ Wd
    dG, dU = dH * U * slope, dH * value
    return {"dX": dG @ Wg + dU @ Wu, "dWg": dG.T @ X, "dWu": dU.T @ X, "dWd": dY.T @ H,
            "dbg": dG.sum(axis=0), "dbu": dU.sum(axis=0), "dbd": dY.sum(axis=0)}


def adamw(p, g, m, v, step, lr, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0,
          grad_scale=1.0):
    """(p, m, v) after one step."""
    p, g, m, v = (np.asarray(a, dtype=np.float64) for a in (p, g, m, v))
    g = g * grad_scale
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    mhat, vhat = m / (1.0 - beta1 ** step), v / (1.0 - beta2 ** step)
    return p - lr * weight_decay * p - lr * mhat / (np.sqrt(vhat) + eps), m, v


def e4m3_values():
    """The finite non-negative values of the 8-bit float type (4 exponent bits,
    3 mantissa bits, bias 7, largest 448), in order of their codes 0 .. 126."""
    out = []
    for code in range(127):
        e, f = code >> 3, code & 7
        out.append((f / 8.0) * 2.0 ** -6 if e == 0 else (1.0 + f / 8.0) * 2.0 ** (e - 7))
    return np.array(out)


def to_e4m3(x, root=False):
    """(values, scale per block) of x rounded to nearest, ties to the even code;
    the scale is the block's largest magnitude / 448.  root: positive values do
    not round to zero."""
    x = np.asarray(x, dtype=np.float64)
    table = e4m3_values()
    mid = (table[1:] + table[:-1]) / 2.0
    values, scales = np.zeros_like(x), []
    for a in range(0, len(x), BLOCK):
        b = x[a:a + BLOCK]
        fine = np.isfinite(b)
        top = np.abs(b[fine]).max(initial=0.0)
        scales.append(top / 448.0)
        if top == 0.0:
            continue
        y = np.where(fine, np.abs(b) * (448.0 / top), 0.0)
        code = np.searchsorted(mid, y, side="left")
        tie = (code < len(mid)) & (y == mid[np.minimum(code, len(mid) - 1)]) & (code % 2 == 1)
        code = code + tie
        if root:
            code = np.where(b > 0, np.maximum(code, 1), code)
        values[a:a + BLOCK] = np.where(fine, np.sign(b) * table[code], np.nan)
    return values, np.array(scales)
