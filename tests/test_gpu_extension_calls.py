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


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n, d", [(1, 5), (33, 7), (300, 96), (70, 301), (9, 2049), (5, 8200), (3, 20001)])
def test_layer_norm_in_place(n, d, dtype):
    # Y in X's place; dX in add's and in dY's: the same bits as apart
    rng = np.random.default_rng(n + d)
    pad = 3 if d % 2 else 8
    X, _ = make(rng, (n, d), dtype, 2.0, pad=pad)
    gamma, _ = make(rng, (d,), F32, 0.2, 1.0)
    beta, _ = make(rng, (d,), F32)
    dY, _ = make(rng, (n, d), dtype, pad=pad)
    add, _ = make(rng, (n, d), dtype, pad=pad)
    case(f"layer norm in place {n} x {d} {dtype}")
    Y, stats = fd.fd_layer_norm(X, gamma, beta)
    g = fd.fd_layer_norm_backward(dY, X, gamma, stats, add=add)
    for name in ("add", "dY"):
        t = {"add": add.clone(), "dY": dY.clone()}
        h = fd.fd_layer_norm_backward(t["dY"], X, gamma, stats, add=t["add"], dX=t[name])
        assert h.dX.data_ptr() == t[name].data_ptr()
        for k in ("dX", "dgamma", "dbeta"):
            assert torch.equal(getattr(h, k), getattr(g, k)), (name, k)
    Z, stats2 = fd.fd_layer_norm(X, gamma, beta, Y=X)
    assert Z.data_ptr() == X.data_ptr() and torch.equal(X, Y) and torch.equal(stats, stats2)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n, d, f, o", [(3, 40, 96, 40), (200, 40, 600, 30), (5000, 24, 64, 24),
                                        (300, 90, 200, 70), (60, 96, 3000, 72), (2000, 200, 400, 200)])
def test_gated_into_the_residual(n, d, f, o, dtype):
    # few rows, the narrow kernel whole and in parts, the tiles whole and in parts
    t, _ = gated_inputs(n, d, f, o, dtype, True, n + d, pad=3)
    w = [t[k] for k in WEIGHTS]
    case(f"gated into the residual {(n, d, f, o)} {dtype}")
    for save in (False, True):
        Y, _ = fd.fd_gated_forward(*w, R=t["R"], save=save)
        R = t["R"].clone()
        Z, _ = fd.fd_gated_forward(*w, R=R, Y=R, save=save)
        assert Z.data_ptr() == R.data_ptr() and torch.equal(Y, R)


@pytest.mark.parametrize("dtype, bits", [(F32, 32), (BF16, 32), (BF16, 8)])
def test_training_pass_in_a_graph(dtype, bits):
    # layer norm and block forward and backward and the step, captured; replays with eager
    # work between them, each against the eager result.  (A captured step keeps its number.)
    dev = device()
    gen = torch.Generator(device=dev).manual_seed(4)
    n, d, f = 700, 72, 200

    def normal(*shape, scale=1.0, dtype=dtype):
        return (torch.randn(*shape, device=dev, generator=gen) * scale).to(dtype)

    params = [normal(f, d, scale=0.1, dtype=F32), normal(f, d, scale=0.1, dtype=F32),
              normal(d, f, scale=0.1, dtype=F32), torch.ones(d, device=dev), torch.zeros(d, device=dev)]
    weights = [p.to(dtype) for p in params]
    grads = [torch.zeros_like(w) for w in weights]
    state = fd.fd_adamw_state(params, bits)
    plan = fd.fd_adamw_plan(params, grads, state, copies=weights if dtype == BF16 else None)
    if dtype == F32:
        weights = params
    X, dY = normal(n, d), normal(n, d, scale=1e-2)

    def step():
        Z, stats = fd.fd_layer_norm(X, weights[3], weights[4])
        Y, saved = fd.fd_gated_forward(Z, *weights[:3], R=X, save=True)
        g = fd.GatedGrads(torch.empty_like(Z), *grads[:3], None, None, None)
        fd.fd_gated_backward(dY, Z, *weights[:3], saved=saved, grads=g)
        dX = fd.fd_layer_norm_backward(g.dX, X, weights[3], stats, add=dY, dgamma=grads[3],
                                       dbeta=grads[4]).dX
        fd.fd_adamw_step(plan, 7, lr=1e-2, rounding="unbiased")
        return Y, dX

    held = params + ([] if dtype == F32 else weights) + state.m + state.v
    held += [] if bits == 32 else state.m_scale + state.v_scale
    case(f"training pass in a graph {dtype} {bits}-bit states")
    step()
    torch.cuda.synchronize()
    start = [x.clone() for x in held]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        Y, dX = step()
    for i in range(4):
        X.copy_(normal(n, d))
        dY.copy_(normal(n, d, scale=1e-2))
        for x, s in zip(held, start):
            x.copy_(s)
        Y0, dX0 = step()
        want = [x.clone() for x in held]
        for x, s in zip(held, start):
            x.copy_(s)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(Y, Y0) and torch.equal(dX, dX0), i
        for a, b in zip(held, want):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i


def test_two_threads_on_streams_of_their_own():
    import threading

    case("two threads")
    jobs = []
    for k, (n, d, f, o, dtype) in enumerate(((600, 90, 200, 70, BF16), (40, 48, 300, 64, F32))):
        t, _ = gated_inputs(n, d, f, o, dtype, True, 50 + k)
        w = [t[x] for x in WEIGHTS]
        Y, saved = fd.fd_gated_forward(*w, save=True)
        g = fd.fd_gated_backward(t["dY"], *w, saved=saved)
        _, stats = fd.fd_layer_norm(t["X"])
        dX = fd.fd_layer_norm_backward(t["X"], t["X"], None, stats).dX
        jobs.append((t, w, Y, g, stats, dX))
    torch.cuda.synchronize()
    wrong = []

    def work(job, bad):
        t, w, Y, g, stats, dX = job
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(30):
                    Y1, saved = fd.fd_gated_forward(*w, save=True)
                    g1 = fd.fd_gated_backward(t["dY"], *w, saved=saved)
                    _, st = fd.fd_layer_norm(t["X"])
                    dX1 = fd.fd_layer_norm_backward(t["X"], t["X"], None, st).dX
                    try:  # the message is the thread's own
                        fd._check(fd.load().fd_adamw_step(None, bad, None, None))
                    except fd.FdError as e:
                        assert "tensor list" in e.msg
                    torch.cuda.current_stream().synchronize()
                    same = torch.equal(Y1, Y) and torch.equal(st, stats) and torch.equal(dX1, dX)
                    for name in ("dX", "dWg", "dWu", "dWd", "dbg", "dbu", "dbd"):
                        same = same and torch.equal(getattr(g1, name), getattr(g, name))
                    if not same:
                        wrong.append(job[1][0].shape)
        except Exception as e:  # a thread's failure is the test's
            wrong.append(repr(e))

    threads = [threading.Thread(target=work, args=(job, 1)) for job in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
