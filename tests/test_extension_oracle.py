"""The extension operators' oracle against differences and known values, and
the entry points' refusals (no GPU needed)."""
import ctypes

import numpy as np
import pytest

from oracle import extension as ox
from paper_2609_38198_amd import _lib as fd


def difference(f, x, h=1e-6):
    out = np.zeros_like(x)
    for i in np.ndindex(*x.shape):
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        out[i] = (f(a) - f(b)) / (2 * h)
    return out


def test_layer_norm_gradients_are_the_differences():
    rng = np.random.default_rng(0)
    x, dy, add = (rng.normal(size=(4, 6)) for _ in range(3))
    ga, be = rng.normal(size=6), rng.normal(size=6)
    dx, dga, dbe = ox.layer_norm_backward(dy, x, ga, add=add)
    loss = lambda x, ga, be: (ox.layer_norm(x, ga, be)[0] * dy).sum()
    assert np.allclose(dx, difference(lambda z: loss(z, ga, be), x) + add, atol=1e-8)
    assert np.allclose(dga, difference(lambda z: loss(x, z, be), ga), atol=1e-8)
    assert np.allclose(dbe, difference(lambda z: loss(x, ga, z), be), atol=1e-8)


@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_gradients_are_the_differences(act):
    rng = np.random.default_rng(1)
    a = [rng.normal(size=s) for s in ((3, 4), (5, 4), (5, 4), (2, 5), (5,), (5,), (2,))]
    dy = rng.normal(size=(3, 2))
    got = ox.gated_backward(dy, *a[:6], act=act)
    for i, name in enumerate(("dX", "dWg", "dWu", "dWd", "dbg", "dbu", "dbd")):
        f = lambda z: (ox.gated(*a[:i], z, *a[i + 1:], act=act)[0] * dy).sum()
        assert np.allclose(got[name], difference(f, a[i]), atol=1e-7), name


def test_e4m3():
    table = ox.e4m3_values()
    assert table[0] == 0 and table[1] == 2.0 ** -9 and table[-1] == 448 and (np.diff(table) > 0).all()
    v, s = ox.to_e4m3(np.concatenate([table, -table]))
    assert (v == np.concatenate([table, -table])).all() and s[0] == 1.0
    v, _ = ox.to_e4m3(np.array([448.0, 2.0 ** -11, -5.0, 17.0]), root=True)
    assert v.tolist() == [448.0, 2.0 ** -9, -5.0, 16.0]


def test_adamw_first_step_moves_by_the_rate():
    p, m, v = ox.adamw(np.zeros(3), np.array([1.0, -2.0, 1e-3]), np.zeros(3), np.zeros(3), 1, 0.1)
    assert np.allclose(p, [-0.1, 0.1, -0.1], rtol=1e-4)


def test_refusals_of_layer_norm():
    lib = fd.load()
    p = ctypes.c_void_p(256)

    def norm(X=p, xt=0, N=4, D=8, ldx=8, wt=0, eps=1e-5, Y=p, ldy=8, stats=None):
        return lib.fd_layer_norm(X, xt, N, D, ldx, None, None, wt, eps, Y, ldy, stats, None)

    for bad in (dict(X=None), dict(Y=None), dict(xt=2), dict(wt=-1), dict(N=-1), dict(D=0),
                dict(ldx=7), dict(ldy=7), dict(eps=-1.0), dict(eps=float("nan")),
                dict(D=(1 << 20) + 1, ldx=1 << 21, ldy=1 << 21), dict(N=(1 << 30) + 1),
                dict(X=ctypes.c_void_p(258)), dict(stats=ctypes.c_void_p(260)), dict(ldy=9)):
        assert norm(**bad) == 1, bad
        assert lib.fd_last_error()
    assert norm(N=0, X=None, Y=None) == 0
    assert fd.load().fd_layer_norm_workspace_size(10, 0) == 0
    assert fd.load().fd_layer_norm_workspace_size(10, 8) > 0

    def back(dY=p, lddy=8, add=None, ldadd=0, dX=ctypes.c_void_p(512), lddx=8, stats=p, ws=p,
             nws=1 << 20):
        return lib.fd_layer_norm_backward(dY, lddy, p, 0, 4, 8, 8, None, 0, stats, add, ldadd, dX,
                                          lddx, None, None, ws, nws, None)

    for bad in (dict(dY=None), dict(dX=None), dict(stats=None), dict(lddy=7), dict(lddx=7),
                dict(add=p, ldadd=7), dict(dX=p, lddx=9)):
        assert back(**bad) == 1, bad
    for bad in (dict(ws=None), dict(nws=8), dict(ws=ctypes.c_void_p(128))):
        assert back(**bad) == 3, bad


def block(**kw):
    b = fd.GatedBlock(N=4, D=8, F=16, O=8, type=0, act=0, X=256, Wg=256, Wu=256, Wd=256, ldx=8,
                      ldwi=8, ldwd=16)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def test_refusals_of_the_gated_block():
    lib = fd.load()
    p = ctypes.c_void_p(256)

    def fwd(b, Y=p, ldy=8, R=None, ldr=0, saved=None, nsaved=0, ws=p, nws=1 << 24):
        return lib.fd_gated_forward(b, R, ldr, Y, ldy, saved, nsaved, ws, nws, None)

    for bad in (dict(N=-1), dict(D=0), dict(F=0), dict(O=0), dict(type=2), dict(act=2),
                dict(X=None), dict(Wg=None), dict(Wu=None), dict(Wd=None), dict(ldx=7),
                dict(ldwi=7), dict(ldwd=15), dict(X=258), dict(bd=257)):
        assert fwd(block(**bad)) == 1, bad
        assert lib.fd_last_error()
    assert fwd(block(F=(1 << 20) + 1, ldwd=1 << 21)) == 2
    for bad in (dict(Y=None), dict(ldy=7), dict(R=p, ldr=7), dict(R=p, ldr=9)):
        assert fwd(block(), **bad) == 1, bad
    for bad in (dict(ws=None), dict(nws=64), dict(ws=ctypes.c_void_p(264)),
                dict(saved=p, nsaved=16), dict(saved=ctypes.c_void_p(264), nsaved=1 << 20)):
        assert fwd(block(), **bad) == 3, bad
    assert fwd(block(N=0, X=None), Y=None) == 0
    g = fd.GatedGradsC(dX=512, dWg=512, dWu=512, dWd=512, lddx=8, lddwi=8, lddwd=16)

    def bwd(b=None, g=g, dY=p, lddy=8, ws=p, nws=1 << 24, saved=None, nsaved=0):
        return lib.fd_gated_backward(b or block(), dY, lddy, saved, nsaved, g, ws, nws, None)

    assert bwd(g=None) == 1 and bwd(dY=None) == 1 and bwd(lddy=7) == 1
    for bad in (dict(lddx=7), dict(lddwi=7), dict(lddwd=15), dict(dX=514)):
        h = fd.GatedGradsC.from_buffer_copy(g)
        for k, v in bad.items():
            setattr(h, k, v)
        assert bwd(g=h) == 1, bad
    assert bwd(nws=64) == 3 and bwd(ws=None) == 3 and bwd(saved=p, nsaved=8) == 3
    assert lib.fd_gated_saved_size(block()) > 0 and lib.fd_gated_saved_size(block(D=0)) == 0
    sizes = [lib.fd_gated_workspace_size(block(), i) for i in (0, 1, 2)]
    assert 0 < sizes[0] < sizes[1] < sizes[2]
    assert lib.fd_gated_workspace_size(block(), 3) == 0


def test_refusals_of_adamw():
    lib = fd.load()
    good = dict(p=256, g=256, m=256, v=256, m_scale=None, v_scale=None, copy=None, n=4, gt=0,
                decay=1.0)
    opts = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, grad_scale=1.0,
                step=1, state_bits=32)

    def step(t=None, o=None, count=1):
        t = fd.AdamwTensor(**dict(good, **(t or {})))
        return lib.fd_adamw_step(t, count, fd.AdamwOpts(**dict(opts, **(o or {}))), None)

    for bad in (dict(p=None), dict(g=None), dict(m=None), dict(v=None), dict(n=-1), dict(gt=3),
                dict(decay=float("nan")), dict(p=258), dict(m=257), dict(copy=257)):
        assert step(bad) == 1, bad
    for bad in (dict(step=0), dict(beta1=1.0), dict(beta2=-0.1), dict(eps=-1.0),
                dict(lr=float("inf")), dict(grad_scale=float("nan"))):
        assert step(None, bad) == 1, bad
    assert step(None, dict(state_bits=16)) == 2
    assert step(None, dict(state_bits=8)) == 1  # no scales
    assert lib.fd_adamw_step(None, 1, None, None) == 1
    assert lib.fd_adamw_step(None, 0, None, None) == 0
    assert step(dict(n=0, p=None)) == 0
    o = fd.AdamwOpts()
    lib.fd_adamw_default_opts(o)
    assert (o.lr, o.beta1, o.beta2, o.step, o.state_bits) == (1e-3, 0.9, 0.999, 1, 32)


def test_struct_layouts(tmp_path):
    import os
    import shutil
    import subprocess

    cc = shutil.which("gcc") or shutil.which("cc")
    if cc is None:
        pytest.skip("no C compiler")
    structs = {"fd_gated_block": fd.GatedBlock, "fd_gated_grads": fd.GatedGradsC,
               "fd_adamw_tensor": fd.AdamwTensor, "fd_adamw_opts": fd.AdamwOpts}
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "flashdiff.h"',
             "int main(void) {"]
    for name, cls in structs.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f}));' for f, _ in cls._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0;", "}"]))
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run([cc, "-std=c11", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)],
                   check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True,
                                          check=True).stdout.split()]
    want = []
    for cls in structs.values():
        want.append(ctypes.sizeof(cls))
        want += [getattr(cls, f).offset for f, _ in cls._fields_]
    assert got == want


def test_binding_refuses_what_is_not_on_the_gpu():
    import torch

    x = torch.zeros(4, 8)
    with pytest.raises(ValueError):
        fd.fd_layer_norm(x)
    with pytest.raises(TypeError):
        fd.fd_layer_norm(x.to(torch.float16))
    with pytest.raises(ValueError):
        fd.fd_gated_forward(x, x, x, x)
    with pytest.raises(ValueError):
        fd.fd_gated_forward(x, x, x, x, act="relu")
    with pytest.raises(ValueError):
        fd.fd_adamw_plan([x], [x], fd.fd_adamw_state([x]))


def test_sizes_of_no_rows():
    lib = fd.load()
    assert lib.fd_gated_saved_size(block(N=0)) == 0
    assert all(lib.fd_gated_workspace_size(block(N=0), i) > 0 for i in (0, 1, 2))
    assert lib.fd_layer_norm_workspace_size(0, 8) > 0
