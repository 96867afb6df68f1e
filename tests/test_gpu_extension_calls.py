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
