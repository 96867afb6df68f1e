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
