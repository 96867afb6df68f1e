"""How the extension's operators are called: types, strides and places of the arguments."""
import numpy as np
import pytest
import torch

from gpu_util import case, device, to_np
from oracle import extension as ox
from paper_2609_38198_amd import _lib as fd
from test_gpu_extension_ops import BF16, F32, GATED_TOL, NORM_TOL, err, gated_inputs, make

pytestmark = pytest.mark.gpu

WEIGHTS = ("X", "Wg", "Wu", "Wd", "bg", "bu", "bd")


@pytest.mark.parametrize("how", ["wdtype", "array"])
@pytest.mark.parametrize("dtype, wtype", [(BF16, F32), (F32, BF16), (BF16, BF16)])
def test_shift_without_scale_has_a_gradient_of_its_type(dtype, wtype, how):
    # a shift of another type than X: what the forward pass takes, the backward pass gives
    rng = np.random.default_rng(3)
    X, x = make(rng, (70, 52), dtype)
    beta, be = make(rng, (52,), wtype)
    dY, dy = make(rng, (70, 52), dtype)
    case(f"layer norm, shift {wtype} beside {dtype}, by {how}")
    Y, stats = fd.fd_layer_norm(X, None, beta)
    assert err(Y, ox.layer_norm(x, None, be)[0]) <= NORM_TOL[dtype]
    kw = {"wdtype": wtype} if how == "wdtype" else {"dbeta": torch.empty_like(beta)}
    g = fd.fd_layer_norm_backward(dY, X, None, stats, **kw)
    assert g.dbeta.dtype == wtype
    assert err(g.dbeta, dy.sum(0), np.linalg.norm(dy)) <= NORM_TOL[wtype]


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_one_row_has_no_leading_dimension(dtype):
    # one inner feature and one point: rows of larger matrices, whose strides differ
    rng = np.random.default_rng(4)
    dev = device()

    def part(cols, stride):
        room = torch.from_numpy(rng.normal(size=(3, stride))).to(dtype).to(dev)
        return room[1:2, :cols]

    d, o = 24, 5
    Wg, Wu, dY = part(d, 40), part(d, 56), part(o, 9)
    Wd = torch.from_numpy(rng.normal(size=(o, 1))).to(dtype).to(dev)
    X, R = part(d, 33), part(o, 12)
    case(f"gated, single rows of other strides {dtype}")
    Y, saved = fd.fd_gated_forward(X, Wg, Wu, Wd, R=R, save=True)
    c = [x.contiguous() for x in (X, Wg, Wu, Wd)]
    Y0, saved0 = fd.fd_gated_forward(*c, R=R.contiguous(), save=True)
    assert torch.equal(Y, Y0)
    out = fd.GatedGrads(part(d, 31), part(d, 48), part(d, 40), torch.empty_like(Wd), None, None, None)
    g = fd.fd_gated_backward(dY, X, Wg, Wu, Wd, saved=saved, grads=out)
    g0 = fd.fd_gated_backward(dY.contiguous(), *c, saved=saved0)
    for name in ("dX", "dWg", "dWu", "dWd"):
        assert torch.equal(getattr(g, name), getattr(g0, name)), name
    assert to_np(g.dWg).any()


# What is off is the rounding of the float64 values itself, and 2^-15 of the kept G and U: the
# bound of small problems, at sizes that would round H, dG and dU to one bfloat16 without it.
@pytest.mark.parametrize("n, d, f, o, act", [(5003, 509, 365, 260, "silu"), (1200, 96, 640, 520, "gelu"),
                                             (70000, 40, 128, 48, "silu")])
def test_gated_fine_is_rounded_once_at_any_size(n, d, f, o, act):
    t, a = gated_inputs(n, d, f, o, BF16, True, n + o)
    case(f"gated, fine {(n, d, f, o)} {act}")
    w = [t[k] for k in WEIGHTS]
    inner = [a[k] for k in WEIGHTS[:6]]
    want = dict(ox.gated_backward(a["dY"], *inner, act), Y=ox.gated(*inner, a["bd"], act=act)[0])

    def ratio(got, name):
        once = torch.from_numpy(want[name]).to(BF16).double().numpy()
        return np.linalg.norm(to_np(got) - want[name]) / np.linalg.norm(once - want[name])

    for save in (False, True):
        Y, saved = fd.fd_gated_forward(*w, act=act, save=save, fine=True)
        g = fd.fd_gated_backward(t["dY"], *w, act=act, saved=saved, fine=True)
        off = {k: ratio(Y if k == "Y" else getattr(g, k), k) for k in ("Y", "dX", "dWg", "dWu", "dWd")}
        assert max(off.values()) <= 1.1, off
    # float32 takes the flag and does as before
    x = [None if v is None else v.float() for v in w]
    assert torch.equal(fd.fd_gated_forward(*x, act=act)[0], fd.fd_gated_forward(*x, act=act, fine=True)[0])
