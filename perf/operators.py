"""Operators of a parametric extension: what a program asks of the library
when it trains a network x -> psi(x) on diffusion coordinates, and when it
evaluates that network at new points.

A case is a dict of plain values.  ``op`` names the operator:

* ``norm``   layer norm of ``n`` rows of ``d`` features; with ``train`` its
  backward pass too, the residual branch's gradient added in;
* ``gated``  the gated feed-forward block act(x Wg + bg) * (x Wu + bu) -> Wd + bd
  of ``n`` rows, ``d`` -> ``f`` -> ``o`` features; with ``train`` its backward
  pass too (gradients of the input, the weights and the biases);
* ``adamw``  one AdamW step over the tensors whose sizes ``sizes`` lists, the
  first ``decayed`` of them with weight decay, states in ``bits`` bits,
  gradients in ``dtype``; with ``copy`` also a bfloat16 copy of the parameters.

``own`` chooses between the library's entry points and the plain form, which
computes in float32 whatever the type and rounds once at the end.
"""
import math

import torch

own = False

EPS = 1e-5                                     # of the layer norm
LR, B1, B2, ADAM_EPS, DECAY = 1e-4, 0.9, 0.999, 1e-8, 0.05
BLOCK = 256                                    # elements that share a scale of 8-bit states
FP8_TOP = 448.0                                # largest value of the 8-bit float type
FP8_LEAST = 2.0 ** -9                          # its smallest positive value
MOST_FLOPS = 5.0e12                            # of a drawn case: the largest listed one's
MOST_ELEMENTS = 1 << 27

BASE = {"op": "norm", "dtype": "bf16", "train": True, "n": 1, "d": 64, "f": 0, "o": 0,
        "act": "silu", "bias": True, "residual": False, "sizes": "", "decayed": 0, "bits": 32,
        "copy": False}


def _case(name=None, **kw):
    c = dict(BASE, **kw)
    if name is not None:
        c["name"] = name
    return c


def _network(width, hidden, blocks, d, k):
    """Sizes of an encoder's tensors: matrices first, then norms and biases."""
    dims = [(d, width)] + [(width, width)] * blocks + [(width, k)]
    mats = [s for a, b in dims for s in (hidden * a, hidden * a, b * hidden)]
    vecs = [s for a, b in dims for s in (hidden, hidden, b)] + [width] * (2 * blocks)
    return {"sizes": ",".join(map(str, mats + vecs)), "decayed": len(mats)}


def listed():
    return [
        # normalising one small batch of new points: latency
        _case("norm_small", op="norm", train=False, n=64, d=512),
        # a ragged width and row count of a float32 training batch
        _case("norm_train_ragged", op="norm", dtype="f32", n=30011, d=301),
        # a wide network's largest batch
        _case("norm_train_large", op="norm", n=65536, d=2048),
        # one new point through a wide block: latency and the weights' bytes
        _case("gated_point", op="gated", train=False, n=1, d=1024, f=4096, o=1024, residual=True),
        # the first layer at the points of a Nystrom extension, in place of it:
        # molecule-like features to 64 coordinates
        _case("gated_extend", op="gated", dtype="f32", train=False, n=30011, d=30, f=512, o=64),
        # a 2-torus batch: every point, a small float32 block
        _case("gated_train_small", op="gated", dtype="f32", n=2048, d=64, f=256, o=64,
              act="gelu"),
        # odd sizes throughout
        _case("gated_train_ragged", op="gated", n=5003, d=509, f=1365, o=509, act="gelu",
              residual=True),
        # a float32 batch of a wide network
        _case("gated_train_f32", op="gated", dtype="f32", n=8192, d=1024, f=4096, o=1024),
        # the largest: a wide network's batch in bfloat16, without biases
        _case("gated_train_large", op="gated", n=16384, d=2048, f=8192, o=2048, bias=False,
              residual=True),
        # the small encoder's tensors: many, short
        _case("adamw_small", op="adamw", dtype="f32", **_network(64, 256, 4, 30, 64)),
        # an ordinary encoder, bfloat16 gradients and copies, states in 32 bits
        _case("adamw_ordinary", op="adamw", copy=True, **_network(509, 1365, 6, 30, 64)),
        # a wide encoder, states in 8 bits
        _case("adamw_large_8bit", op="adamw", bits=8, copy=True, **_network(2048, 8192, 2, 64, 64)),
    ]


def _size(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """A width: any number, or often a multiple of 32."""
    s = _size(rng, lo, hi)
    return s if rng.random() < 0.5 or s < 32 else s // 32 * 32


def draw(rng):
    op = rng.choice(["norm", "gated", "gated", "adamw"])
    dtype = rng.choice(["bf16", "f32"])
    while True:
        if op == "norm":
            c = _case(op=op, dtype=dtype, train=rng.random() < 0.6, n=_size(rng, 1, 200000),
                      d=_width(rng, 8, 8192))
            if c["n"] * c["d"] <= MOST_ELEMENTS:
                return c
        elif op == "gated":
            d = _width(rng, 4, 2048)
            o = d if rng.random() < 0.5 else _width(rng, 4, 2048)
            c = _case(op=op, dtype=dtype, train=rng.random() < 0.6, n=_size(rng, 1, 65536), d=d,
                      f=_width(rng, 16, 8192), o=o, act=rng.choice(["silu", "gelu"]),
                      bias=rng.random() < 0.5, residual=d == o and rng.random() < 0.5)
            # a float32 product counts four times
            if work(c)["flops"] * (4 if dtype == "f32" else 1) <= MOST_FLOPS and c["n"] * c["f"] <= MOST_ELEMENTS:
                return c
        else:
            count = _size(rng, 1, 96)
            top = _size(rng, 256, 1 << 25)
            sizes = sorted((_size(rng, max(1, top // 4096), top) for _ in range(count)), reverse=True)
            c = _case(op=op, dtype=dtype, sizes=",".join(map(str, sizes)),
                      decayed=rng.randint(0, count), bits=rng.choice([32, 8]),
                      copy=rng.random() < 0.5)
            if sum(sizes) <= MOST_ELEMENTS:
                return c


def work(case):
    c = dict(BASE, **case)
    e = 4 if c["dtype"] == "f32" else 2
    n, d, f, o = c["n"], c["d"], c["f"], c["o"]
    if c["op"] == "norm":
        fwd = {"bytes": e * (2 * n * d + 2 * d) + 8 * n, "flops": 8.0 * n * d}
        if not c["train"]:
            return fwd
        # dY and the branch's gradient in, dX out; X and the weights are in already
        return {"bytes": fwd["bytes"] + e * (3 * n * d + 2 * d), "flops": fwd["flops"] + 14.0 * n * d}
    if c["op"] == "gated":
        weights = 2 * d * f + f * o + ((2 * f + o) if c["bias"] else 0)
        rows = d + o + (o if c["residual"] else 0)
        fwd = {"bytes": e * (weights + n * rows), "flops": 4.0 * n * d * f + 2.0 * n * f * o}
        if not c["train"]:
            return fwd
        return {"bytes": fwd["bytes"] + e * (weights + n * (o + d)), "flops": 3 * fwd["flops"]}
    total = sum(_sizes(c))
    state = 16 if c["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": total * (8 + e + state + (2 if c["copy"] else 0)), "flops": 16.0 * total}


# ------------------------------------------------------------------ inputs


def _sizes(c):
    return [int(s) for s in c["sizes"].split(",")]


def _starts(c):
    """Where each tensor starts in the flat buffers: on a block's boundary."""
    at, starts = 0, []
    for s in _sizes(c):
        starts.append(at)
        at += -(-s // BLOCK) * BLOCK
    return starts, at


def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _make(c, seed):
    """The inputs, from the seed alone."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    t = _dtype(c)

    def normal(*shape, scale=1.0, mean=0.0):
        x = torch.randn(*shape, device="cuda", generator=gen)
        return x.mul_(scale).add_(mean).to(t)

    n, d, f, o = c["n"], c["d"], c["f"], c["o"]
    if c["op"] == "norm":
        # a residual stream: features of unlike size around means of their own
        size = torch.exp(0.5 * torch.randn(d, device="cuda", generator=gen))
        mean = 0.5 * torch.randn(d, device="cuda", generator=gen)
        x = torch.randn(n, d, device="cuda", generator=gen).mul_(size).add_(mean).to(t)
        return {"x": x, "gamma": normal(d, scale=0.2, mean=1.0), "beta": normal(d, scale=0.1),
                "dy": normal(n, d, scale=1e-2), "add": normal(n, d, scale=1e-2)}
    if c["op"] == "gated":
        s = {"x": normal(n, d), "wg": normal(f, d, scale=d ** -0.5),
             "wu": normal(f, d, scale=d ** -0.5), "wd": normal(o, f, scale=f ** -0.5),
             "bg": None, "bu": None, "bd": None, "r": None,
             "dy": normal(n, o, scale=1e-2) if c["train"] else None}
        if c["bias"]:
            s.update(bg=normal(f, scale=0.1), bu=normal(f, scale=0.1), bd=normal(o, scale=0.1))
        if c["residual"]:
            s["r"] = normal(n, o)
        return s
    starts, total = _starts(c)
    inside = torch.zeros(total, device="cuda")
    for a, size in zip(starts, _sizes(c)):
        inside[a:a + size] = 1.0
    # gradients of widely different sizes, and moments that follow them
    size = 1e-3 * torch.exp(1.5 * torch.randn(total, device="cuda", generator=gen)) * inside
    s = {"p": 0.02 * torch.randn(total, device="cuda", generator=gen) * inside,
         "g": (size * torch.randn(total, device="cuda", generator=gen)).to(t),
         "copy": torch.zeros(total, device="cuda", dtype=torch.bfloat16) if c["copy"] else None,
         "step": 1000}
    m = 0.3 * size * torch.randn(total, device="cuda", generator=gen)
    root = size * torch.exp(0.2 * torch.randn(total, device="cuda", generator=gen))
    if c["bits"] == 32:
        s.update(m=m, v=root * root)
    else:
        (s["m"], s["ms"]), (s["r"], s["rs"]) = _to_8bit(m, False), _to_8bit(root, True)
    # where weight decay ends
    s["split"] = starts[c["decayed"]] if c["decayed"] < len(starts) else total
    return s


def prepare(case, seed):
    c = dict(BASE, **case)
    s = dict(_make(c, seed), c=c)
    if own and c["op"] == "adamw":
        from paper_2609_38198_amd import _lib as fd

        def views(x, per=1):
            return [x[a // per:a // per - (-size // per)] for a, size in zip(_starts(c)[0], _sizes(c))]

        state = (fd.AdamwState(m=views(s["m"]), v=views(s["v"])) if c["bits"] == 32 else
                 fd.AdamwState(m=views(s["m"]), v=views(s["r"]), m_scale=views(s["ms"], BLOCK),
                               v_scale=views(s["rs"], BLOCK)))
        s["plan"] = fd.fd_adamw_plan(views(s["p"]), views(s["g"]), state,
                                     copies=views(s["copy"]) if c["copy"] else None,
                                     decay=[float(i < c["decayed"]) for i in range(len(_sizes(c)))])
    return s


# ------------------------------------------------------------------ one pass


def run(s):
    c = s["c"]
    if c["op"] == "norm":
        return _run_norm(s, c) if own else _plain_norm(s, c)
    if c["op"] == "gated":
        return _run_gated(s, c) if own else _plain_gated(s, c)
    s["step"] += 1
    if own:
        from paper_2609_38198_amd import _lib as fd
        fd.fd_adamw_step(s["plan"], s["step"], lr=LR, beta1=B1, beta2=B2, eps=ADAM_EPS,
                         weight_decay=DECAY)
    else:
        _plain_adamw(s, c)
    return _adamw_outputs(s, c)


def _adamw_outputs(s, c):
    out = {"p": s["p"], "m": s["m"], "copy": s["copy"]}
    out.update({"v": s["v"]} if c["bits"] == 32 else {"r": s["r"], "ms": s["ms"], "rs": s["rs"]})
    return out


def _run_norm(s, c):
    from paper_2609_38198_amd import _lib as fd

    y, stats = fd.fd_layer_norm(s["x"], s["gamma"], s["beta"], EPS)
    if not c["train"]:
        return {"y": y}
    g = fd.fd_layer_norm_backward(s["dy"], s["x"], s["gamma"], stats, add=s["add"])
    return {"y": y, "dx": g.dX, "dgamma": g.dgamma, "dbeta": g.dbeta}


def _run_gated(s, c):
    from paper_2609_38198_amd import _lib as fd

    y, saved = fd.fd_gated_forward(s["x"], s["wg"], s["wu"], s["wd"], s["bg"], s["bu"], s["bd"],
                                   R=s["r"], act=c["act"], save=c["train"])
    if not c["train"]:
        return {"y": y}
    g = fd.fd_gated_backward(s["dy"], s["x"], s["wg"], s["wu"], s["wd"], s["bg"], s["bu"], s["bd"],
                             act=c["act"], saved=saved)
    return {"y": y, "dx": g.dX, "dwg": g.dWg, "dwu": g.dWu, "dwd": g.dWd, "dbg": g.dbg,
            "dbu": g.dbu, "dbd": g.dbd}


def _plain_norm(s, c):
    t = s["x"].dtype
    x, gamma = s["x"].float(), s["gamma"].float()
    xc = x - x.sum(1, keepdim=True) / c["d"]
    rstd = 1.0 / torch.sqrt((xc * xc).sum(1, keepdim=True) / c["d"] + EPS)
    h = xc * rstd
    y = (h * gamma + s["beta"].float()).to(t)
    if not c["train"]:
        return {"y": y}
    dy = s["dy"].float()
    g = dy * gamma
    dx = rstd * (g - g.sum(1, keepdim=True) / c["d"] - h * ((g * h).sum(1, keepdim=True) / c["d"]))
    return {"y": y, "dx": (dx + s["add"].float()).to(t), "dgamma": (dy * h).sum(0).to(t),
            "dbeta": dy.sum(0).to(t)}


def _act(g, act):
    """The activation and its derivative."""
    if act == "silu":
        z = 1.0 / (1.0 + torch.exp(-g))
        return g * z, z * (1.0 + g * (1.0 - z))
    z = 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))
    return g * z, z + g * torch.exp(-0.5 * g * g) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_gated(s, c):
    t = s["x"].dtype
    x, wg, wu, wd = (s[k].float() for k in ("x", "wg", "wu", "wd"))
    g, u = x @ wg.T, x @ wu.T
    if c["bias"]:
        g, u = g + s["bg"].float(), u + s["bu"].float()
    a, slope = _act(g, c["act"])
    h = a * u
    y = h @ wd.T
    if c["bias"]:
        y = y + s["bd"].float()
    if c["residual"]:
        y = y + s["r"].float()
    if not c["train"]:
        return {"y": y.to(t)}
    dy = s["dy"].float()
    dh = dy @ wd
    dg, du = dh * u * slope, dh * a
    out = {"y": y, "dx": dg @ wg + du @ wu, "dwg": dg.T @ x, "dwu": du.T @ x, "dwd": dy.T @ h,
           "dbg": dg.sum(0) if c["bias"] else None, "dbu": du.sum(0) if c["bias"] else None,
           "dbd": dy.sum(0) if c["bias"] else None}
    return {k: None if v is None else v.to(t) for k, v in out.items()}


def _to_8bit(x, root):
    """x as 8-bit floats and one scale per block; a positive root stays positive."""
    b = x.view(-1, BLOCK)
    top = b.abs().amax(1, keepdim=True)
    y = b * torch.where(top > 0, FP8_TOP / top, 0.0)
    if root:
        y = torch.where(b > 0, y.clamp_min(FP8_LEAST), y)
    return y.to(torch.float8_e4m3fn).view(-1), (top / FP8_TOP).view(-1)


def _from_8bit(q, scale):
    return (q.float().view(-1, BLOCK) * scale.view(-1, 1)).view(-1)


def _plain_adamw(s, c):
    g = s["g"].float()
    if c["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        m, r = _from_8bit(s["m"], s["ms"]), _from_8bit(s["r"], s["rs"])
        v = r * r
    m = B1 * m + (1.0 - B1) * g
    v = B2 * v + (1.0 - B2) * (g * g)
    r = torch.sqrt(v)
    rate = LR / (1.0 - B1 ** s["step"])
    keep = 1.0 / math.sqrt(1.0 - B2 ** s["step"])
    p = s["p"]
    p[:s["split"]] *= 1.0 - LR * DECAY
    p -= rate * m / (r * keep + ADAM_EPS)
    if c["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
    else:
        for to, of in ((("m", "ms"), _to_8bit(m, False)), (("r", "rs"), _to_8bit(r, True))):
            s[to[0]].copy_(of[0])
            s[to[1]].copy_(of[1])
    if c["copy"]:
        s["copy"].copy_(p)


# ------------------------------------------------------------------ in 64 bits


def exact(case, seed):
    c = dict(BASE, **case)
    s = {k: v.double() if isinstance(v, torch.Tensor) and v.dtype != torch.float8_e4m3fn else v
         for k, v in _make(c, seed).items()}
    if c["op"] == "norm":
        return _exact_norm(s, c)
    if c["op"] == "gated":
        return _exact_gated(s, c)
    step = s["step"] + 1
    if c["bits"] == 32:
        m0, v0 = s["m"], s["v"]
    else:
        def wide(q, scale):
            return q.to(torch.float64) * scale.repeat_interleave(BLOCK)
        m0, v0 = wide(s["m"], s["ms"]), wide(s["r"], s["rs"]).square()
    m = torch.lerp(s["g"], m0, B1)
    v = torch.lerp(s["g"].square(), v0, B2)
    wd = torch.zeros_like(m)
    wd[:s["split"]] = DECAY
    mhat, vhat = m / (1.0 - B1 ** step), v / (1.0 - B2 ** step)
    p = s["p"] - LR * (mhat / (vhat.sqrt() + ADAM_EPS) + wd * s["p"])
    out = {"p": p, "copy": p if c["copy"] else None}
    if c["bits"] == 32:
        return dict(out, m=m, v=v)

    def top(x):
        return x.view(-1, BLOCK).abs().max(dim=1).values / FP8_TOP
    # which of two neighbouring 8-bit values a state takes is left open
    return dict(out, m=None, r=None, ms=top(m), rs=top(v.sqrt()))


def _exact_norm(s, c):
    x = s["x"]
    var, mu = torch.var_mean(x, dim=1, correction=0, keepdim=True)
    std = (var + EPS).sqrt()
    h = (x - mu) / std
    out = {"y": h * s["gamma"] + s["beta"]}
    if c["train"]:
        g = s["dy"] * s["gamma"]
        out.update(dx=(g - g.mean(1, keepdim=True) - h * (g * h).mean(1, keepdim=True)) / std + s["add"],
                   dgamma=(s["dy"] * h).sum(0), dbeta=s["dy"].sum(0))
    return out


def _exact_gated(s, c):
    x, wg, wu, wd = s["x"], s["wg"], s["wu"], s["wd"]
    g, u = x.mm(wg.T), x.mm(wu.T)
    if c["bias"]:
        g += s["bg"]
        u += s["bu"]
    if c["act"] == "silu":
        cdf = torch.sigmoid(g)
        slope = cdf + g * cdf * (1 - cdf)
    else:
        cdf = torch.special.ndtr(g)
        slope = cdf + g * torch.exp(-g.square() / 2) / math.sqrt(2 * math.pi)
    h = g * cdf * u
    y = h.mm(wd.T)
    for extra in ("bd", "r"):
        if s[extra] is not None:
            y = y + s[extra]
    if not c["train"]:
        return {"y": y}
    dy = s["dy"]
    dwd = dy.T.mm(h)
    dh = dy.mm(wd)
    dg = dh * u * slope
    du = dh * g * cdf
    b = c["bias"]
    return {"y": y, "dx": dg.mm(wg).addmm_(du, wu), "dwg": dg.T.mm(x), "dwu": du.T.mm(x),
            "dwd": dwd, "dbg": dg.sum(0) if b else None, "dbu": du.sum(0) if b else None,
            "dbd": dy.sum(0) if b else None}
