"""The example network: gradients of all its parameters against float64
autograd, training, and the graph capture of a pass."""
import os
import sys

import numpy as np
import pytest
import torch

from gpu_util import case, device

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def reference_grads(net, X, dY, act):
    """Gradients in float64 by torch's autograd, on the CPU."""
    p = [w.detach().cpu().double().requires_grad_(True) for w in net.weights]
    f = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[act]

    def block(x, i):
        wg, wu, wd, bg, bu, bd = p[6 * i:6 * i + 6]
        return (f(x @ wg.T + bg) * (x @ wu.T + bu)) @ wd.T + bd

    h = block(X.cpu().double(), 0)
    for i in range(1, net.layers):
        at = 6 * net.layers + 2 * (i - 1)
        z = torch.nn.functional.layer_norm(h, h.shape[1:], p[at], p[at + 1], 1e-5)
        y = block(z, i)
        h = h + y if i + 1 < net.layers else y
    h.backward(dY.cpu().double())
    return h.detach(), [w.grad for w in p]


# float32: every layer's own error (8e-6 at most, tests of the operators) adds up over
# five layers and their norms; bfloat16: 2^-7 a block, and the roundings of the
# activations and gradients between them, 2^-8 each
@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("dtype, tol", [(torch.float32, 5e-5), (torch.bfloat16, 5e-2)])
def test_network_gradients(dtype, tol, act):
    from extension_net import ExtensionNet

    case(f"extension network gradients {dtype} {act}")
    net = ExtensionNet(4, 5, width=48, hidden=100, depth=3, dtype=dtype, act=act)
    gen = torch.Generator(device="cuda").manual_seed(2)
    X = torch.randn(333, 4, device=device(), generator=gen).to(dtype)
    dY = torch.randn(333, 5, device=device(), generator=gen).to(dtype)
    Y, tape = net.forward(X, save=True)
    net.backward(dY, tape)
    want, grads = reference_grads(net, X, dY, act)
    assert (Y.cpu().double() - want).norm() <= tol * want.norm()
    for got, ref in zip(net.grads, grads):
        assert (got.cpu().double() - ref).norm() <= tol * ref.norm()


@pytest.mark.parametrize("dtype, bits", [(torch.float32, 32), (torch.bfloat16, 8)])
def test_network_learns(dtype, bits):
    from extension_net import ExtensionNet, torus

    case(f"extension network training {dtype} {bits}-bit states")
    X = torus(4096, 3)
    target = torch.stack([X[:, 0] * X[:, 2], X[:, 1]], 1)
    net = ExtensionNet(4, 2, width=32, hidden=64, depth=1, dtype=dtype, bits=bits)
    errs = [float(net.train_step(X.to(dtype), target, 3e-3)) for _ in range(150)]
    assert np.isfinite(errs).all() and errs[-1] <= 0.05 * errs[0]


def test_forward_in_a_graph():
    from extension_net import ExtensionNet

    case("extension network forward pass in a graph")
    net = ExtensionNet(30, 8, width=64, hidden=128, depth=2, dtype=torch.bfloat16)
    X = torch.randn(500, 30, device=device()).to(torch.bfloat16)
    net.forward(X)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        Y, _ = net.forward(X)
    for i in range(4):
        X.copy_(torch.randn(500, 30, device=device()))
        want, _ = net.forward(X)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, want), i
