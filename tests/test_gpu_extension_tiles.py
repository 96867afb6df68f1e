"""The gated block in every tile, split and way that its plans take, at odd sizes: each
row and column by itself against float64, outputs in padded rows whose padding stays.

A CPU test (test_host_gated_plans.py) asks the plans which kernels these sizes take, and fails
where sizes drawn over the operators' range take others.

Tolerances: two bfloat16 roundings, 2^-7 (single elements of long sums are off by
2^-9 / sqrt 3 of their terms' size, one standard deviation, and 2^-9 of themselves), and 8e-6 in
float32.
"""
import numpy as np
import pytest
import torch

from extension_util import GRADS, Framed, gated_results, worst_lines
from gpu_util import case, to_np
from oracle import extension as ox
from paper_2609_38198_amd import _lib as fd
from test_gpu_extension_ops import BF16, F32, GATED_TOL, gated_inputs

pytestmark = pytest.mark.gpu

# N, D, F, O: the cheapest odd sizes that take each kernel, then wider ones whose tiles are many
TILE_SHAPES = [(1, 17, 17, 491), (1, 463, 17, 45), (1, 851, 17, 39), (519, 5, 19, 5),
               (1, 93, 6285, 1773), (249, 5, 2151, 63), (3, 415, 7939, 1533), (79, 859, 225, 1993),
               (11133, 65, 69, 25), (22559, 11, 17, 323), (99, 81, 6467, 109), (25453, 5, 77, 79),
               (25093, 377, 33, 71), (8847, 1455, 35, 9), (25307, 57, 67, 931), (9101, 11, 3329, 67),
               (59605, 5, 37, 5), (64425, 5, 237, 5),
               (3001, 201, 2501, 199), (5003, 509, 1365, 509), (1349, 21, 6169, 1473),
               (8195, 131, 4101, 129), (16403, 521, 2099, 601), (16385, 1031, 2049, 1029),
               # widths of whole 16 bytes, which need no packing
               (771, 96, 264, 72), (4104, 520, 1048, 264)]
WEIGHTS = ("X", "Wg", "Wu", "Wd", "bg", "bu", "bd")


def check_every_line(n, d, f, o, dtype, act, bias, fine=False):
    t, a = gated_inputs(n, d, f, o, dtype, bias, 7 * n + d + f)
    w = [t[k] for k in WEIGHTS]
    want = gated_results(a, act, True)
    tol = GATED_TOL[dtype]
    shapes = {"dX": (n, d), "dWg": (f, d), "dWu": (f, d), "dWd": (o, f), "dbg": (f,), "dbu": (f,),
              "dbd": (o,)}
    # aligned rows further apart, and rows and starts that are not aligned
    for save, pad, offset in ((True, 8, 0), (False, 3, 1)):
        Y = Framed((n, o), dtype, pad, offset)
        _, saved = fd.fd_gated_forward(*w, R=t["R"], act=act, save=save, Y=Y.t, fine=fine)
        g = {k: None if k.startswith("db") and not bias else
             Framed(shapes[k], dtype, 0 if k.startswith("db") else pad, offset) for k in GRADS}
        fd.fd_gated_backward(t["dY"], *w, act=act, saved=saved, fine=fine,
                             grads=fd.GatedGrads(*[None if g[k] is None else g[k].t for k in GRADS]))
        for name, x in dict(g, Y=Y).items():
            if x is None:
                continue
            assert x.intact(), f"{name}: written outside, saved {save}"
            off = worst_lines(to_np(x.t), *want[name])
            assert max(off.values()) <= tol, (name, save, off)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n, d, f, o", TILE_SHAPES)
def test_every_line_of_every_tile(n, d, f, o, dtype):
    act = "gelu" if (n + f) % 4 == 0 else "silu"
    bias = (d + f) % 3 != 0
    case(f"gated, every line {n} x {d} -> {f} -> {o} {dtype} {act} bias {bias}")
    check_every_line(n, d, f, o, dtype, act, bias)


def test_every_line_with_two_planes_above_the_line():
    for n, d, f, o in ((3001, 201, 2501, 199), (25307, 57, 67, 931), (771, 520, 264, 272)):
        case(f"gated, every line, fine {n} x {d} -> {f} -> {o}")
        check_every_line(n, d, f, o, BF16, "silu", True, fine=True)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_float64_on_the_gpu_is_the_oracle(act):
    # the sizes above 2e9 multiplications are compared with these
    t, a = gated_inputs(1400, 400, 1100, 520, F32, True, 5)
    case(f"float64 on the GPU {act}")
    want = gated_results(a, act, True)
    ref = ox.gated_backward(a["dY"], *[a[k] for k in WEIGHTS[:6]], act)
    ref["Y"] = ox.gated(*[a[k] for k in WEIGHTS], a["R"], act)[0]
    for name, x in ref.items():
        assert np.linalg.norm(want[name][0] - x) <= 1e-12 * np.linalg.norm(x), name
