"""The extension's operators where values are of very unlike size: what one row,
feature or step is like leaves the others' digits alone.

Tolerances as in the operators' other tests: two bfloat16 roundings, 2^-7, and
8e-6 in float32, here for every row and column by itself, against the size of the
terms that it sums.
"""
import numpy as np
import pytest
import torch

from extension_util import GRADS, gated_results, worst_lines
from gpu_util import case, device, to_np
from oracle import extension as ox
from paper_2609_38198_amd import _lib as fd
from test_gpu_extension_ops import BF16, F32, GATED_TOL, gated_inputs

pytestmark = pytest.mark.gpu

WEIGHTS = ("X", "Wg", "Wu", "Wd", "bg", "bu", "bd")


def set_rows(t, a, name, rows, f):
    """Row `rows` of input `name` is f of itself, on the device and in float64."""
    x = t[name].clone()
    x[rows] = f(x[rows])
    t[name].copy_(x)
    a[name] = to_np(t[name])


# narrow, tiled with H in two planes, tiled with one
RANGE_SHAPES = [(70, 48, 160, 40), (70, 96, 160, 80), (1500, 96, 512, 260)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale", [1e6, 1e10, 1e12])
@pytest.mark.parametrize("n, d, f, o", RANGE_SHAPES)
def test_a_large_row_leaves_its_neighbours_gradients(n, d, f, o, scale, dtype):
    # a padding row: large values, no gradient; it adds zero to every sum
    for save in (True, False):
        t, a = gated_inputs(n, d, f, o, dtype, True, 3 * n + d)
        set_rows(t, a, "X", 9, lambda x: x * scale)
        set_rows(t, a, "dY", 9, lambda x: x * 0.0)
        case(f"gated beside a row of {scale:g} {(n, d, f, o)} {dtype} saved {save}")
        w = [t[k] for k in WEIGHTS]
        _, saved = fd.fd_gated_forward(*w, save=save)
        g = fd.fd_gated_backward(t["dY"], *w, saved=saved)
        want = gated_results(a, "silu", False)
        for name in GRADS:
            off = worst_lines(to_np(getattr(g, name)), *want[name])
            assert max(off["row"], off["column"]) <= GATED_TOL[dtype], (name, off)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_a_large_row_leaves_its_own_small_features(dtype):
    # features 3 and 40 see nothing of X but their biases: in the large row too their G and U
    # are of size one, and with them that row's share of dWg, dWu and dWd
    n, d, f, o = 70, 96, 160, 80
    t, a = gated_inputs(n, d, f, o, dtype, True, 21)
    for name in ("Wg", "Wu"):
        set_rows(t, a, name, [3, 40], lambda x: x * 0.0)
    set_rows(t, a, "X", 9, lambda x: x * 1e11)
    case(f"gated small features of a large row {dtype}")
    w = [t[k] for k in WEIGHTS]
    _, saved = fd.fd_gated_forward(*w, save=True)
    g = fd.fd_gated_backward(t["dY"], *w, saved=saved)
    want = gated_results(a, "silu", False)
    for name in ("dWg", "dWu", "dWd", "dbg", "dbu"):
        at = np.s_[..., [3, 40]] if name == "dWd" else np.s_[[3, 40]]
        off = worst_lines(to_np(getattr(g, name))[at], want[name][0][at], want[name][1][at])
        assert max(off["row"], off["column"]) <= GATED_TOL[dtype], (name, off)
