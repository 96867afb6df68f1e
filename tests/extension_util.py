"""What the extension operators' tests compare with: every result of the gated
block in float64, and the size of the terms that each of its elements sums.

An error is measured over a row, a column or an element's neighbourhood against
the 2-norm of those sizes, so that a single wrong row or column shows however
large the matrix: sums of many independent terms that cancel keep an error of
their terms' size, whatever is left of them.
"""
import numpy as np

from oracle import extension as ox

GRADS = ("dX", "dWg", "dWu", "dWd", "dbg", "dbu", "dbd")


def gated_results(a, act, residual):
    """{name: (values, sizes)} of Y and the gradients for the arrays in `a`."""
    r = a["R"] if residual else 0.0
    with np.errstate(over="ignore"):
        Y, G, U, H = ox.gated(a["X"], a["Wg"], a["Wu"], a["Wd"], a["bg"], a["bu"], a["bd"], r, act)
        grads = ox.gated_backward(a["dY"], a["X"], a["Wg"], a["Wu"], a["Wd"], a["bg"], a["bu"], act)
        value, slope = ox.activation(G, act)
    sq = {k: np.square(a[k]) for k in ("X", "Wg", "Wu", "Wd", "dY")}
    dh = np.sqrt(sq["dY"] @ sq["Wd"])
    dg, du = (dh * np.abs(U * slope)) ** 2, (dh * np.abs(value)) ** 2
    H2 = H ** 2
    sizes = {"Y": H2 @ sq["Wd"].T + np.square(a["bd"]) + np.square(r),
             "dX": dg @ sq["Wg"] + du @ sq["Wu"], "dWg": dg.T @ sq["X"], "dWu": du.T @ sq["X"],
             "dWd": sq["dY"].T @ H2, "dbg": dg.sum(0), "dbu": du.sum(0), "dbd": sq["dY"].sum(0)}
    return {k: (v, np.sqrt(sizes[k])) for k, v in dict(grads, Y=Y).items()}


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
