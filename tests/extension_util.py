"""What the extension operators' tests compare with: every result of the gated
block in float64, and the size of the terms that each of its elements sums.

An error is measured over a row, a column or an element's neighbourhood against
the 2-norm of those sizes, so that a single wrong row or column shows however
large the matrix: sums of many independent terms that cancel keep an error of
their terms' size, whatever is left of them.
"""
import math

import numpy as np
import torch

from oracle import extension as ox

GRADS = ("dX", "dWg", "dWu", "dWd", "dbg", "dbu", "dbd")


def _activation(g, act):
    """ox.activation for float64 tensors."""
    if act == "silu":
        z = torch.sigmoid(g)
        return g * z, z + g * z * (1.0 - z)
    z = 0.5 * torch.special.erfc(-g / math.sqrt(2.0))
    return g * z, z + g * torch.exp(-g * g / 2.0) / math.sqrt(2.0 * math.pi)


def gated_results(a, act, residual):
    """{name: (values, sizes)} of Y and the gradients for the float64 arrays in `a`:
    the oracle's formulas, evaluated on the GPU where they would take long here."""
    x, wg, wu, wd, dy = (a[k] for k in ("X", "Wg", "Wu", "Wd", "dY"))
    bg, bu, bd = (a[k] for k in ("bg", "bu", "bd"))
    r = a["R"] if residual else 0.0
    activation = ox.activation
    if x.shape[0] * wg.shape[0] * (2 * x.shape[1] + wd.shape[0]) > 2e9:
        x, wg, wu, wd, dy, bg, bu, bd, r = (
            torch.from_numpy(v).cuda() if isinstance(v, np.ndarray) else v
            for v in (x, wg, wu, wd, dy, bg, bu, bd, r))
        activation = _activation
    with np.errstate(over="ignore"):
        G, U = x @ wg.T + bg, x @ wu.T + bu
        value, slope = activation(G, act)
    H = value * U
    dH = dy @ wd
    dG, dU = dH * U * slope, dH * value
    values = {"Y": H @ wd.T + bd + r, "dX": dG @ wg + dU @ wu, "dWg": dG.T @ x, "dWu": dU.T @ x,
              "dWd": dy.T @ H, "dbg": dG.sum(0), "dbu": dU.sum(0), "dbd": dy.sum(0)}
    # each inner value by what errors of the sums in it leave: those of G, U and dH, times its
    # derivative by them (the activation's second one is at most about a half)
    dy2, x2 = dy ** 2, x ** 2
    g2, u2 = x2 @ (wg ** 2).T + bg ** 2 + G ** 2, x2 @ (wu ** 2).T + bu ** 2 + U ** 2
    dh2 = dy2 @ wd ** 2 + dH ** 2
    H2 = (slope * U) ** 2 * g2 + value ** 2 * u2
    dg2 = dh2 * ((slope * U) ** 2 + slope ** 2 * u2 + 0.25 * U ** 2 * g2)
    du2 = dh2 * (value ** 2 + slope ** 2 * g2)
    sizes = {"Y": H2 @ (wd ** 2).T + bd ** 2 + r ** 2, "dX": dg2 @ wg ** 2 + du2 @ wu ** 2,
             "dWg": dg2.T @ x2, "dWu": du2.T @ x2, "dWd": dy2.T @ H2, "dbg": dg2.sum(0),
             "dbu": du2.sum(0), "dbd": dy2.sum(0)}

    def host(v):
        return v.cpu().numpy() if isinstance(v, torch.Tensor) else v

    return {k: (host(values[k]), np.sqrt(host(sizes[k]))) for k in values}


def worst_lines(got, want, size):
    """The largest relative errors over single rows, over single columns, and
    over the last row, column and 32 x 32 corner together with the whole."""
    got, want, size = (np.atleast_2d(np.asarray(x, dtype=np.float64)) for x in (got, want, size))
    assert got.shape == want.shape and np.isfinite(got).all()
    off, ref = np.square(got - want), np.maximum(np.square(want), np.square(size))

    def ratio(o, r):
        return np.sqrt(np.where(o == 0.0, 0.0, o / np.where(r > 0.0, r, np.finfo(float).tiny))).max()

    out = {"row": ratio(off.sum(1), ref.sum(1)), "column": ratio(off.sum(0), ref.sum(0)),
           "all": ratio(off.sum(), ref.sum())}
    for name, at in (("last row", np.s_[-1:, :]), ("last column", np.s_[:, -1:]),
                     ("corner", np.s_[-32:, -32:]), ("last element", np.s_[-1:, -1:])):
        out[name] = ratio(off[at].sum(), ref[at].sum())
    return out


class Framed:
    """A matrix or vector inside a larger allocation of NaNs: rows `pad` elements further
    apart, `offset` elements in.  `intact` says whether all around it still has its bits."""

    def __init__(self, shape, dtype, pad=0, offset=0):
        self.cols = shape[-1]
        rows = shape[0] if len(shape) == 2 else 1
        self.ld = self.cols + pad
        self.room = torch.full((offset + rows * self.ld + 64,), float("nan"), dtype=dtype, device="cuda")
        self.body = self.room[offset:offset + rows * self.ld].view(rows, self.ld)
        self.t = self.body[:, :self.cols] if len(shape) == 2 else self.body[0, :self.cols]
        self.before = self._around()

    def _around(self):
        bits = self.room.view(torch.int32 if self.room.dtype == torch.float32 else torch.int16).clone()
        at = self.body.storage_offset() - self.room.storage_offset()
        rows = self.body.shape[0]
        bits[at:at + rows * self.ld].view(rows, self.ld)[:, :self.cols] = 0
        return bits

    def intact(self):
        return torch.equal(self._around(), self.before)
