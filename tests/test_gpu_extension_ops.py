"""Layer norm, the gated block and AdamW against the float64 oracle.

Tolerances (2-norm of the difference over 2-norm of the result, or over the
norm of the terms that cancel in it where that is more):

* bfloat16: a rounding is at most 2^-9 of a value.  Layer norm rounds its
  result once: 2^-8 leaves a factor of two.  The block rounds H (or dG, dU) and the
  result; a product of independent errors keeps their relative size: 2^-7.
* float32: a sum of K products carries about sqrt(K) 2^-24; K up to 3,000
  here gives 3.3e-6; twice that for the intermediate's own error: 8e-6.  Layer
  norm's longest sums (4,099 rows) stay below 64 2^-24 = 4e-6.
"""
import numpy as np
import pytest
import torch

from gpu_util import case, device, to_np
from oracle import extension as ox
from paper_2609_38198_amd import _lib as fd

pytestmark = pytest.mark.gpu

NORM_TOL = {torch.float32: 4e-6, torch.bfloat16: 2.0 ** -8}
GATED_TOL = {torch.float32: 8e-6, torch.bfloat16: 2.0 ** -7}
F32, BF16 = torch.float32, torch.bfloat16


def err(got, want, scale=0.0):
    """Relative 2-norm error; `scale`: the norm of what cancels in `want`."""
    got, want = to_np(got), np.asarray(want)
    assert got.shape == want.shape
    assert np.isfinite(got).all()
    d, n = np.linalg.norm(got - want), max(np.linalg.norm(want), scale)
    return 0.0 if d == 0.0 else d / n


def make(rng, shape, dtype, scale=1.0, mean=0.0, pad=0, offset=0):
    """A matrix (rows `pad` elements further apart, `offset` elements into its
    allocation) of seeded values, on the device, and its float64 values."""
    x = torch.from_numpy(rng.normal(size=shape) * scale + mean).to(dtype)
    if len(shape) == 1:
        room = torch.full((shape[0] + offset,), float("nan"), dtype=dtype, device=device())
        t = room[offset:]
    else:
        rows, cols = shape
        room = torch.full((rows * (cols + pad) + offset,), float("nan"), dtype=dtype,
                          device=device())
        t = room[offset:].view(rows, cols + pad)[:, :cols]
    t.copy_(x)
    return t, x.double().numpy()


# ---------------------------------------------------------------- layer norm

NORM_SHAPES = [(1, 1), (1, 8), (3, 2), (5, 3), (17, 30), (64, 64), (33, 127), (7, 129), (9, 301),
               (4099, 64), (257, 509), (130, 513), (65, 1000), (40, 1025), (21, 2047), (12, 2049),
               (5, 4100), (3, 8200), (2, 16384), (2, 16385), (3, 20001),
               # many rows of less than a chunk, rows of one group of lanes less or more than whole
               (3001, 3), (5000, 7), (300, 20000), (999, 61), (70, 259), (11, 5001)]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n, d", NORM_SHAPES)
def test_layer_norm_and_gradients(n, d, dtype):
    rng = np.random.default_rng(n * 100003 + d)
    wdtype = BF16 if (n + d) % 3 == 0 else F32
    pad, off = ((3, 1) if d % 2 else (8, 0))
    X, x = make(rng, (n, d), dtype, 2.0, 0.7, pad, off)
    gamma, ga = make(rng, (d,), wdtype, 0.2, 1.0, offset=off)
    beta, be = make(rng, (d,), wdtype, 0.1)
    dY, dy = make(rng, (n, d), dtype, 0.3, pad=pad)
    add, ad = make(rng, (n, d), dtype, 0.3)
    case(f"layer norm {n} x {d} {dtype} weights {wdtype}")
    Y, stats = fd.fd_layer_norm(X, gamma, beta, 1e-5)
    want, mean, rstd = ox.layer_norm(x, ga, be)
    tol = NORM_TOL[dtype]
    assert err(Y, want) <= tol
    assert err(stats[:, 0], mean, np.linalg.norm(x) / np.sqrt(d)) <= 4e-6
    # (x - mean) cancels where features are few: its error is of x's size
    assert err(stats[:, 1], rstd) <= 4e-6 * (1 if d > 3 else 100)
    g = fd.fd_layer_norm_backward(dY, X, gamma, stats, add=add)
    dx, dga, dbe = ox.layer_norm_backward(dy, x, ga, add=ad)
    size = np.linalg.norm(rstd[:, None] * dy * ga)
    wtol = max(NORM_TOL[wdtype], 4e-6)
    assert err(g.dX, dx, size) <= tol
    h = ox.layer_norm(x)[0]
    assert err(g.dgamma, dga, np.linalg.norm(dy * h)) <= wtol
    assert err(g.dbeta, dbe, np.linalg.norm(dy)) <= wtol
    # no weights, no branch; dX in dY's place
    Y, stats = fd.fd_layer_norm(X, None, None, 1e-5)
    want = ox.layer_norm(x)[0]
    assert err(Y, want, np.sqrt(n * d) if d == 1 else 0.0) <= tol
    g = fd.fd_layer_norm_backward(dY, X, None, stats, weight_grads=False, dX=dY)
    assert g.dX.data_ptr() == dY.data_ptr() and g.dgamma is None
    assert err(dY, ox.layer_norm_backward(dy, x)[0], np.linalg.norm(rstd[:, None] * dy)) <= tol


def test_layer_norm_far_from_zero_and_constant_rows():
    # the variance comes from centred values: rows at 1,000 +- 0.01 keep the
    # digits that float32 inputs have (2^-24 1000 / 0.01 = 6e-3 of a deviation in the input itself)
    rng = np.random.default_rng(5)
    x = torch.from_numpy(1000.0 + 0.01 * rng.normal(size=(33, 200))).float()
    case("layer norm far from zero")
    Y, _ = fd.fd_layer_norm(x.to(device()), eps=0.0)
    want, mean, _ = ox.layer_norm(x.double().numpy(), eps=0.0)
    # the mean's own rounding, 2^-24 1000, is 6e-3 of a deviation at most
    assert err(Y, want) <= 6e-3
    case("layer norm of constant rows")
    Y, stats = fd.fd_layer_norm(torch.full((4, 64), 3.0, device=device()))
    assert (to_np(Y) == 0.0).all() and np.allclose(to_np(stats[:, 1]), 1e-5 ** -0.5)


def test_layer_norm_nan_stays_in_its_row():
    rng = np.random.default_rng(6)
    X, x = make(rng, (50, 96), F32)
    X[7, 3] = float("nan")
    X[20, 0] = float("inf")
    case("layer norm with a NaN and an infinity")
    Y, stats = fd.fd_layer_norm(X)
    bad = np.isnan(to_np(Y)).any(axis=1)
    assert bad.nonzero()[0].tolist() == [7, 20]
    keep = ~bad
    assert np.linalg.norm(to_np(Y)[keep] - ox.layer_norm(x)[0][keep]) <= 4e-6 * np.sqrt(50 * 96)


def test_layer_norm_no_rows():
    case("layer norm of no rows")
    X = torch.empty((0, 40), dtype=BF16, device=device())
    gamma = torch.ones(40, dtype=BF16, device=device())
    Y, stats = fd.fd_layer_norm(X, gamma)
    g = fd.fd_layer_norm_backward(X, X, gamma, stats)
    assert Y.shape == (0, 40) and not to_np(g.dgamma).any() and not to_np(g.dbeta).any()


# ---------------------------------------------------------------- gated block

# N, D, F, O: single rows, odd widths, sizes around the tiles' edges, widths of
# 16-byte multiples that need no packing, few tiles with long contractions
GATED_SHAPES = [(1, 1, 1, 1), (1, 4, 16, 4), (1, 1024, 512, 256), (2, 30, 97, 64), (5, 64, 256, 3),
                (16, 257, 300, 129), (17, 64, 64, 64), (31, 33, 65, 31), (64, 512, 1024, 512),
                (127, 130, 191, 66), (129, 128, 128, 128), (200, 8, 24, 16), (257, 509, 333, 509),
                (1000, 30, 512, 64), (2049, 96, 160, 72), (3000, 16, 40, 8),
                # many rows, wide inner, wide outer sides, few tiles and long sums over D and O (the
                # tiles that these do not take: test_gpu_extension_tiles.py)
                (70, 2000, 90, 1500), (336, 1696, 372, 700),
                (33000, 7, 70, 33), (501, 33, 31, 64), (4100, 24, 2100, 16), (4104, 4100, 40, 4098), (700, 40, 4099, 2050)]


def gated_inputs(n, d, f, o, dtype, bias, seed, pad=0):
    rng = np.random.default_rng(seed)
    t, a = {}, {}
    for name, shape, scale in (("X", (n, d), 1.0), ("Wg", (f, d), d ** -0.5),
                               ("Wu", (f, d), d ** -0.5), ("Wd", (o, f), f ** -0.5),
                               ("dY", (n, o), 1.0), ("R", (n, o), 1.0)):
        t[name], a[name] = make(rng, shape, dtype, scale, pad=pad)
    for name, size in (("bg", f), ("bu", f), ("bd", o)):
        t[name], a[name] = make(rng, (size,), dtype, 0.5) if bias else (None, 0.0)
    return t, a


def check_gated(t, a, dtype, act, bias, save=True, residual=True):
    tol = GATED_TOL[dtype]
    w = [t[k] for k in ("X", "Wg", "Wu", "Wd", "bg", "bu", "bd")]
    Y, saved = fd.fd_gated_forward(*w, R=t["R"] if residual else None, act=act, save=save)
    want, G, U, H = ox.gated(a["X"], a["Wg"], a["Wu"], a["Wd"], a["bg"], a["bu"], a["bd"],
                             a["R"] if residual else 0.0, act)
    # sums of few terms may cancel: measured against the size of H Wd^T's terms
    terms = np.sqrt(((H ** 2) @ (a["Wd"] ** 2).T).sum())
    assert err(Y, want, terms) <= tol
    g = fd.fd_gated_backward(t["dY"], *w, act=act, saved=saved)
    want = ox.gated_backward(a["dY"], a["X"], a["Wg"], a["Wu"], a["Wd"], a["bg"], a["bu"], act)
    value, slope = ox.activation(G, act)
    dH = a["dY"] @ a["Wd"]
    size = np.sqrt(((a["dY"] ** 2) @ (a["Wd"] ** 2)))  # of dH's terms
    dG, dU = size * np.abs(U * slope), size * np.abs(value)
    scales = {"dX": np.sqrt(((dG ** 2) @ a["Wg"] ** 2 + (dU ** 2) @ a["Wu"] ** 2).sum()),
              "dWg": np.sqrt(((dG ** 2).T @ a["X"] ** 2).sum()),
              "dWu": np.sqrt(((dU ** 2).T @ a["X"] ** 2).sum()),
              "dWd": np.sqrt(((a["dY"] ** 2).T @ H ** 2).sum()),
              "dbg": np.linalg.norm(dG), "dbu": np.linalg.norm(dU),
              "dbd": np.linalg.norm(a["dY"])}
    for name, x in want.items():
        got = getattr(g, name)
        if name.startswith("db") and not bias:
            assert got is None
            continue
        assert err(got, x, scales[name]) <= tol, name
    return Y, g


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("n, d, f, o", GATED_SHAPES)
def test_gated_block_and_gradients(n, d, f, o, dtype):
    act = "gelu" if (n + d) % 2 else "silu"
    bias = f % 3 != 0
    t, a = gated_inputs(n, d, f, o, dtype, bias, n * 7 + d * 3 + f)
    case(f"gated {n} x {d} -> {f} -> {o} {dtype} {act} bias {bias}")
    check_gated(t, a, dtype, act, bias)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("n, d, f, o", [(1, 3, 5, 2), (1, 1024, 700, 300), (2, 63, 64, 65),
                                        (16, 500, 1030, 17), (17, 129, 48, 16), (33, 260, 515, 70),
                                        (64, 96, 2050, 33), (65, 96, 205, 33)])
def test_gated_few_rows_forward(n, d, f, o, pad, dtype):
    act = "gelu" if n % 2 else "silu"
    t, a = gated_inputs(n, d, f, o, dtype, d % 2 == 1, 31 * n + d, pad=pad)
    case(f"gated few rows {n} x {d} -> {f} -> {o} {dtype} pad {pad}")
    Y, _ = fd.fd_gated_forward(*[t[k] for k in ("X", "Wg", "Wu", "Wd", "bg", "bu", "bd")],
                               R=t["R"], act=act)
    want, _, _, H = ox.gated(a["X"], a["Wg"], a["Wu"], a["Wd"], a["bg"], a["bu"], a["bd"], a["R"],
                             act)
    assert err(Y, want, np.sqrt(((H ** 2) @ (a["Wd"] ** 2).T).sum())) <= GATED_TOL[dtype]


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gated_strides_recomputation_and_repeatability(dtype):
    # rows 3 elements further apart: nothing is 16-byte aligned
    t, a = gated_inputs(150, 64, 192, 40, dtype, True, 11, pad=3)
    case(f"gated padded rows {dtype}")
    Y1, g1 = check_gated(t, a, dtype, "silu", True, save=False, residual=False)
    Y2, g2 = check_gated(t, a, dtype, "silu", True, save=True, residual=False)
    assert torch.equal(Y1, Y2)
    for name in ("dX", "dWg", "dWu", "dWd", "dbg", "dbu", "dbd"):
        assert torch.equal(getattr(g1, name), getattr(g2, name)), name


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gated_single_gradients(dtype):
    # each gradient alone, the others NULL: the same bits, and nothing else is needed
    t, a = gated_inputs(300, 72, 130, 90, dtype, True, 17)
    w = [t[k] for k in ("X", "Wg", "Wu", "Wd", "bg", "bu", "bd")]
    case(f"gated single gradients {dtype}")
    full = fd.fd_gated_backward(t["dY"], *w)
    lib = fd.load()
    b = fd._gated_block(*w, "silu")
    ws = torch.empty(lib.fd_gated_workspace_size(b, 2), dtype=torch.uint8, device=device())
    stream = torch.cuda.current_stream().cuda_stream
    for name in ("dX", "dWg", "dWu", "dWd", "dbg", "dbu", "dbd"):
        want = getattr(full, name)
        got = torch.full_like(want, float("nan"))
        g = fd.GatedGradsC(lddx=72, lddwi=72, lddwd=130)
        setattr(g, name, got.data_ptr())
        assert lib.fd_gated_backward(b, t["dY"].data_ptr(), 90, None, 0, g, ws.data_ptr(),
                                     ws.numel(), stream) == 0
        assert torch.equal(got, want), name


# Small problems round to bfloat16 nowhere but at the end: what is off is the rounding of the
# float64 values itself, and 2^-15 of the kept G and U (1.1 leaves room for an eighth of the
# rounding, by derivatives of up to two or three); H, dG and dU once rounded would give 1.4.
@pytest.mark.parametrize("n, d, f, o", [(1, 600, 900, 700), (30, 96, 128, 80), (24, 128, 333, 96),
                                        (100, 30, 97, 64), (150, 64, 640, 40), (70, 200, 72, 90),
                                        (257, 129, 250, 101), (64, 700, 64, 500)])
def test_gated_small_bfloat16_is_rounded_once(n, d, f, o):
    t, a = gated_inputs(n, d, f, o, BF16, True, n + d + f)
    case(f"gated rounded once {(n, d, f, o)}")
    w = [t[k] for k in ("X", "Wg", "Wu", "Wd", "bg", "bu", "bd")]
    inner = [a[k] for k in ("X", "Wg", "Wu", "Wd", "bg", "bu")]

    def rounded_once(got, want):
        once = torch.from_numpy(want).to(BF16).double().numpy()
        assert np.linalg.norm(to_np(got) - want) <= 1.1 * np.linalg.norm(once - want)

    want = ox.gated(*inner, a["bd"])[0]
    grads = ox.gated_backward(a["dY"], *inner, "silu")
    for save in (False, True):
        Y, saved = fd.fd_gated_forward(*w, save=save)
        rounded_once(Y, want)
        g = fd.fd_gated_backward(t["dY"], *w, saved=saved)
        for name in ("dX", "dWg", "dWu", "dWd"):
            rounded_once(getattr(g, name), grads[name])


def test_gated_gradients_against_differences():
    # float64 differences of the oracle's own forward: the formulas themselves
    t, a = gated_inputs(6, 5, 9, 4, F32, True, 12)
    case("gated gradients against differences")
    w = [t[k] for k in ("X", "Wg", "Wu", "Wd", "bg", "bu", "bd")]
    for act in ("silu", "gelu"):
        g = fd.fd_gated_backward(t["dY"], *w, act=act)
        for name, grad in (("X", g.dX), ("Wg", g.dWg), ("Wu", g.dWu), ("Wd", g.dWd),
                           ("bg", g.dbg), ("bu", g.dbu), ("bd", g.dbd)):
            got, x = to_np(grad), a[name]
            num = np.zeros_like(x)
            for i in np.ndindex(*x.shape):
                side = []
                for h in (1e-5, -1e-5):
                    b = {k: np.array(v, copy=True) for k, v in a.items()}
                    b[name][i] += h
                    y = ox.gated(b["X"], b["Wg"], b["Wu"], b["Wd"], b["bg"], b["bu"], b["bd"],
                                 act=act)[0]
                    side.append((y * a["dY"]).sum())
                num[i] = (side[0] - side[1]) / 2e-5
            # differences are good to 1e-9 here; the kernel to float32
            assert np.linalg.norm(got - num) <= 8e-6 * max(1.0, np.linalg.norm(num)), (act, name)


def test_gated_nan_stays_in_its_row():
    for dtype in (F32, BF16):
        t, a = gated_inputs(140, 48, 80, 24, dtype, False, 13)
        t["X"][9, 5] = float("nan")
        case(f"gated with a NaN row {dtype}")
        Y, _ = fd.fd_gated_forward(t["X"], t["Wg"], t["Wu"], t["Wd"])
        bad = np.isnan(to_np(Y)).any(axis=1)
        assert bad.nonzero()[0].tolist() == [9]


def test_gated_large_values_stay_finite():
    # pre-activations far out on both sides: exp overflows inside, the results do not
    case("gated far out")
    X = torch.tensor([[1.0], [-1.0]], device=device())
    W = torch.tensor([[200.0], [2000.0], [1e18]], device=device())
    one = torch.ones((1, 3), device=device())
    for act in ("silu", "gelu"):
        Y, _ = fd.fd_gated_forward(X, W, torch.ones_like(W), one, act=act)
        want = 200.0 + 2000.0 + 1e18
        assert abs(to_np(Y)[0, 0] / want - 1) <= 1e-6 and abs(to_np(Y)[1, 0]) <= 1e-30


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_gated_no_rows(dtype):
    t, a = gated_inputs(4, 10, 20, 6, dtype, True, 14)
    case("gated of no rows")
    w = [t[k] for k in ("Wg", "Wu", "Wd", "bg", "bu", "bd")]
    X, dY = t["X"][:0], t["dY"][:0]
    Y, saved = fd.fd_gated_forward(X, *w, save=True)
    g = fd.fd_gated_backward(dY, X, *w, saved=saved)
    assert Y.shape == (0, 6) and g.dX.shape == (0, 10)
    for x in (g.dWg, g.dWu, g.dWd, g.dbg, g.dbu, g.dbd):
        assert not to_np(x).any()


def test_gated_on_another_stream():
    t, a = gated_inputs(300, 64, 128, 64, BF16, True, 15)
    w = [t[k] for k in ("X", "Wg", "Wu", "Wd", "bg", "bu", "bd")]
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    case("gated on a side stream")
    with torch.cuda.stream(s):
        Y, _ = fd.fd_gated_forward(*w)
    s.synchronize()
    Y0, _ = fd.fd_gated_forward(*w)
    assert torch.equal(Y, Y0)


# ---------------------------------------------------------------- AdamW


def adamw_tensors(sizes, gdtype, bits, copy, seed):
    rng = np.random.default_rng(seed)
    dev = device()
    ps, gs, copies = [], [], [] if copy else None
    for n in sizes:
        ps.append(torch.from_numpy(rng.normal(size=n) * 0.05).float().to(dev))
        gs.append(torch.from_numpy(rng.normal(size=n) * 1e-3 * np.exp(rng.normal(size=n)))
                  .to(gdtype).to(dev))
        if copy:
            copies.append(torch.zeros(n, dtype=BF16, device=dev))
    return ps, gs, fd.fd_adamw_state(ps, bits), copies


@pytest.mark.parametrize("gdtype", [F32, BF16])
def test_adamw_float32_states(gdtype):
    # float32 elementwise: a handful of roundings each, 16 x 2^-24
    sizes = [1, 0, 3, 255, 256, 257, 4096, 4097, 10007] + [5] * 60
    ps, gs, st, copies = adamw_tensors(sizes, gdtype, 32, True, 1)
    decay = [float(i % 2) for i in range(len(sizes))]
    plan = fd.fd_adamw_plan(ps, gs, st, copies, decay)
    ref = [(to_np(p), np.zeros(p.numel()), np.zeros(p.numel())) for p in ps]
    case(f"adamw float32 states, gradients {gdtype}")
    for step in range(1, 5):
        fd.fd_adamw_step(plan, step, lr=1e-2, weight_decay=0.1, grad_scale=0.5)
        ref = [ox.adamw(p, to_np(g), m, v, step, 1e-2, weight_decay=0.1 * w, grad_scale=0.5)
               for (p, m, v), g, w in zip(ref, gs, decay)]
    for i, (p, m, v) in enumerate(ref):
        if len(p) == 0:
            continue
        assert np.abs(to_np(ps[i]) - p).max() <= 4 * 16 * 2.0 ** -24 * (np.abs(p).max() + 1e-2)
        assert err(st.m[i], m) <= 1e-6 and err(st.v[i], v) <= 1e-6
        assert torch.equal(copies[i], ps[i].to(BF16))


@pytest.mark.parametrize("gdtype", [F32, BF16])
def test_adamw_8bit_states(gdtype):
    # a moment is off by half a step of the 8-bit type (2^-4) at most, or by half its
    # smallest value (2^-10) of the block's largest / 448
    sizes = [1, 255, 256, 257, 4096, 4097, 10007, 0, 3]
    ps, gs, st, copies = adamw_tensors(sizes, gdtype, 8, False, 2)
    plan = fd.fd_adamw_plan(ps, gs, st, copies)
    table = ox.e4m3_values()
    case(f"adamw 8-bit states, gradients {gdtype}")
    for step in range(1, 4):
        before = [[to_np(x) for x in (p, m.float(), ms, r.float(), rs)] for p, m, ms, r, rs in
                  zip(ps, st.m, st.m_scale, st.v, st.v_scale)]
        fd.fd_adamw_step(plan, step, lr=1e-2, weight_decay=0.1)
        for i, (p, m, ms, r, rs) in enumerate(before):
            if len(p) == 0:
                continue
            at = np.arange(len(p)) // 256
            p1, m1, v1 = ox.adamw(p, to_np(gs[i]), m * ms[at], (r * rs[at]) ** 2, step, 1e-2,
                                  weight_decay=0.1)
            assert np.abs(to_np(ps[i]) - p1).max() <= 16 * 2.0 ** -24 * (np.abs(p1).max() + 1e-2)
            for q, scale, x, root in ((st.m[i], st.m_scale[i], m1, False),
                                      (st.v[i], st.v_scale[i], np.sqrt(v1), True)):
                want, wscale = ox.to_e4m3(x, root)
                assert np.allclose(to_np(scale), wscale, rtol=1e-6, atol=0)
                got, s = to_np(q.float()), to_np(scale)[at]
                least = np.where(root & (x > 0), 2.0 ** -9, 2.0 ** -10)
                assert (np.abs(got * s - x) <= 1.0001 * np.maximum(np.abs(x) * 2.0 ** -4, least * s)).all()
                # the code itself, except within float32's roundings (three of the
                # moment, two of the inverse scale, one of their product) of the
                # line between two, where bfloat16 gradients often are exactly
                y, line = np.abs(x) / wscale[at], (table[1:] + table[:-1]) / 2
                off = np.abs(y[:, None] - line[None, :]).min(axis=1)
                assert (got == want)[off > 8 * 2.0 ** -24 * y].all()
                if root:
                    assert ((got > 0) == (x > 0)).all()


def test_adamw_8bit_not_finite_stays_alone():
    ps, gs, st, _ = adamw_tensors([600], F32, 8, False, 3)
    gs[0][300] = float("inf")
    gs[0][5] = float("nan")
    case("adamw 8-bit with a NaN and an infinite gradient")
    fd.fd_adamw_step(fd.fd_adamw_plan(ps, gs, st), 1)
    for t in (ps[0], st.m[0].float(), st.v[0].float()):
        bad = ~np.isfinite(to_np(t))
        assert bad.nonzero()[0].tolist() == [5, 300]
    assert np.isfinite(to_np(st.m_scale[0])).all()


def test_adamw_zero_gradients_and_nothing_to_do():
    case("adamw of zero gradients")
    for bits in (32, 8):
        ps, gs, st, _ = adamw_tensors([500, 40], F32, bits, False, 4)
        for g in gs:
            g.zero_()
        before = [to_np(p) for p in ps]
        fd.fd_adamw_step(fd.fd_adamw_plan(ps, gs, st), 1, lr=0.1, weight_decay=0.0)
        for p, b in zip(ps, before):
            assert (to_np(p) == b).all()
    fd.fd_adamw_step(fd.fd_adamw_plan([], [], fd.fd_adamw_state([])), 1)
