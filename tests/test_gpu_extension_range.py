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


# Phi's tail: the activation alone, act(g) = act(X[n, 0]) in every row, by each way through the
# block: few rows, the narrow kernel, the tiles.  float32: some eight roundings of 2^-24 (the
# polynomial's last steps, the exponential, the reciprocal, products), 16 x 2^-24 =
# 9.5e-7 with room; SiLU's exponential has |g| 2^-24 more.  bfloat16: the inner and the last rounding.
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("n, d", [(30, 1), (4000, 1), (4000, 65)])
def test_activation_in_its_tails(n, d, act, dtype):
    dev = device()
    X = torch.zeros(n, d, dtype=dtype, device=dev)
    X[:, 0] = torch.linspace(-12.0, 8.0, n, device=dev).to(dtype)
    Wg, Wu = torch.zeros(1, d, dtype=dtype, device=dev), torch.zeros(1, d, dtype=dtype, device=dev)
    Wg[0, 0] = 1.0
    one = torch.ones(1, 1, dtype=dtype, device=dev)
    case(f"{act} of {n} values, {d} features, {dtype}")
    Y, saved = fd.fd_gated_forward(X, Wg, Wu, one, bu=one[0], act=act, save=n > 30)
    g = to_np(X)[:, 0]
    # the negative branch by erfc, which the oracle's 1 + erf has lost at -6
    import math
    phi = np.array([0.5 * math.erfc(-x / math.sqrt(2.0)) for x in g])
    z = phi if act == "gelu" else 1.0 / (1.0 + np.exp(-g))
    tol = 2.0 ** -8 if dtype == BF16 else 2.0 ** -24 * (16.0 + (np.abs(g) if act == "silu" else 0.0))
    off = np.abs(to_np(Y)[:, 0] - g * z)
    assert (off <= tol * np.abs(g * z)).all(), np.max(off / np.maximum(np.abs(g * z), 1e-300))
    # dX = act'(g) where U does not depend on X; measured against its two terms
    b = fd.fd_gated_backward(torch.ones_like(Y), X, Wg, Wu, one, bu=one[0], act=act, saved=saved)
    rest = g * np.exp(-g * g / 2) / math.sqrt(2 * math.pi) if act == "gelu" else g * z * (1 - z)
    off = np.abs(to_np(b.dX)[:, 0] - (z + rest))
    assert (off <= tol * (np.abs(z) + np.abs(rest))).all(), np.max(off / (np.abs(z) + np.abs(rest)))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n, d, f, o", [(50, 40, 96, 24), (300, 130, 200, 70)])
def test_gelu_gates_that_sit_negative(n, d, f, o, dtype):
    # gates around -6 to -3: every H is a tail's
    t, a = gated_inputs(n, d, f, o, dtype, True, 5 * n)
    set_rows(t, a, "bg", slice(None), lambda x: torch.linspace(-6.0, -3.0, f).to(x))
    set_rows(t, a, "Wg", slice(None), lambda x: x * 0.25)
    a["bd"], a["R"] = np.zeros(o), np.zeros((n, o))
    case(f"gated, negative gates {(n, d, f, o)} {dtype}")
    w = [t[k] for k in WEIGHTS[:6]] + [None]
    want = gated_results(a, "gelu", False)
    Y, saved = fd.fd_gated_forward(*w, act="gelu", save=True)
    g = fd.fd_gated_backward(t["dY"], *w, act="gelu", saved=saved)
    for name in ("Y", "dX", "dWg", "dWu", "dWd", "dbg", "dbu"):
        off = worst_lines(to_np(Y if name == "Y" else getattr(g, name)), *want[name])
        assert max(off["row"], off["column"]) <= GATED_TOL[dtype], (name, off)


def test_host_workspaces_are_refused():
    t, _ = gated_inputs(40, 24, 48, 16, F32, False, 1)
    w = [t[k] for k in WEIGHTS[:4]]
    room = torch.empty(1 << 24, dtype=torch.uint8)
    case("host workspaces")
    Y, saved = fd.fd_gated_forward(*w, save=True)
    _, stats = fd.fd_layer_norm(t["X"])
    for call in (lambda: fd.fd_gated_forward(*w, ws=room),
                 lambda: fd.fd_gated_backward(t["dY"], *w, ws=room),
                 lambda: fd.fd_gated_backward(t["dY"], *w, saved=saved.cpu()),
                 lambda: fd.fd_layer_norm_backward(t["X"], t["X"], None, stats, ws=room),
                 lambda: fd.fd_kernel_matmul(t["X"], None, 1.0, t["X"], ws=room)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_packs_of_more_threads_than_a_launch_holds():
    # 480 million rows of 65 bfloat16 features (62 GB) are packed by 4.32e9 threads; rows all over
    # it, against the same rows by themselves
    n, d, f = 480_000_000, 65, 16
    dev = device()
    need = 2 * n * (d + 72 + 64 + 2) + (1 << 32)
    if torch.cuda.mem_get_info()[0] < need:
        pytest.skip("needs 200 GB of GPU memory")
    case(f"gated {n} x {d} -> {f} -> 1")
    gen = torch.Generator(device=dev).manual_seed(3)

    def normal(*shape):
        return torch.randn(*shape, device=dev, generator=gen).to(BF16)

    X = torch.zeros(n, d, dtype=BF16, device=dev)
    at = torch.cat([torch.arange(40, device=dev), torch.arange(1, 200, device=dev) * (n // 200) + 17,
                    n - 1 - torch.arange(40, device=dev)])
    X[at] = normal(len(at), d)
    w = [normal(f, d) * 0.1, normal(f, d) * 0.1, normal(1, f), normal(f), normal(f)]
    Y, _ = fd.fd_gated_forward(X, *w)
    few, _ = fd.fd_gated_forward(X[at].contiguous(), *w)
    # H in one plane and in two: two bfloat16 roundings apart at most, of the sum's terms
    got, want = to_np(Y[at]), to_np(few)
    del X, Y
    torch.cuda.empty_cache()
    assert np.linalg.norm(got - want) <= 2.0 ** -7 * np.linalg.norm(want)
    assert np.abs(got - want).max() <= 2.0 ** -6 * np.abs(want).max()
