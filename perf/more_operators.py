"""Timed cases of the rest of an update step: products with what follows them in their epilogue, the residual stream with the norms
around a block, and the orthogonalised update of a weight matrix.

Every case is one operator.  `direction`: the forward call alone (scoring, decode) or the forward call and the backward call that a
training step makes (`step`); the orthogonalised update has no gradient.  Sizes are those of the repository's shapes (hidden 256, 512,
1024, 2560 and 4096, their query widths and intermediate sizes) and odd ones around them.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
NEWTON = (3.4445, -4.7750, 2.0315)      # a, b, c of X <- a X + b (X X^T) X + c (X X^T)^2 X
STEPS = 5


def listed():
    return [
        # the O projection of one trajectory's next token, added to the residual stream
        dict(name="linear-1-residual", kind="linear", rows=1, inner=4096, outer=2560, gated=False, bias=False, activation="none", residual="fp32",
             dtype="bf16", direction="forward"),
        # gate, up and their product for a small decode batch
        dict(name="linear-37-gated", kind="linear", rows=37, inner=2560, outer=9728, gated=True, bias=False, activation="silu", residual="none",
             dtype="bf16", direction="forward"),
        # a small fp32 layer of odd widths with bias: latency
        dict(name="linear-fp32-odd-step", kind="linear", rows=61, inner=257, outer=517, gated=False, bias=True, activation="gelu", residual="none",
             dtype="fp32", direction="step"),
        # an update over 4096 packed tokens: the down projection and the residual stream
        dict(name="linear-4b-residual-step", kind="linear", rows=4096, inner=9728, outer=2560, gated=False, bias=False, activation="none",
             residual="fp32", dtype="bf16", direction="step"),
        # an update over 2744 packed tokens: gate, up and their product
        dict(name="linear-4b-gated-step", kind="linear", rows=2744, inner=2560, outer=9728, gated=True, bias=False, activation="silu",
             residual="none", dtype="bf16", direction="step"),
        # a decode batch: attention's output joins the stream, the norm before the next projection follows
        dict(name="residual-norm-128", kind="residual", rows=128, width=2560, centered=False, bias=False, post=False, gate="none", stream="fp32",
             dtype="bf16", residual_scale=1.0, block_scale=1.0, direction="forward"),
        # the same in an update over 7777 packed tokens
        dict(name="residual-norm-4b-step", kind="residual", rows=7777, width=2560, centered=False, bias=False, post=False, gate="none",
             stream="fp32", dtype="bf16", residual_scale=1.0, block_scale=1.0, direction="step"),
        # a block with norms before and after it and a learned gate per channel
        dict(name="residual-norm-post-gate-step", kind="residual", rows=4001, width=1024, centered=False, bias=False, post=True, gate="channel",
             stream="bf16", dtype="bf16", residual_scale=1.0, block_scale=0.25, direction="step"),
        # layer norms with bias of an odd width, gated element by element, fp32
        dict(name="residual-norm-fp32-odd-step", kind="residual", rows=333, width=1023, centered=True, bias=True, post=True, gate="full",
             stream="fp32", dtype="fp32", residual_scale=0.7, block_scale=1.0, direction="step"),
        # the update of a small fp32 model's up projections: latency
        dict(name="orthogonal-fp32-small", kind="orthogonal", count=3, rows=512, columns=256, dtype="fp32"),
        # all query projections of a model at once
        dict(name="orthogonal-0.6b-stack", kind="orthogonal", count=28, rows=2048, columns=1024, dtype="bf16"),
        # one down projection
        dict(name="orthogonal-4b", kind="orthogonal", count=1, rows=2560, columns=9728, dtype="bf16"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["linear", "linear", "residual", "orthogonal"])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    direction = rng.choice(["forward", "step", "step"])
    if kind == "linear":
        inner, outer = (rng.choice([256, 512, 1024, 2560, 4096, 9728, 8 * log(4, 1200), log(30, 9000)]) for _ in range(2))
        gated = rng.random() < 0.4
        flops = (6e11 if dtype == "bf16" else 1e11) / (6 if direction == "step" else 2) / (2 if gated else 1)
        return dict(kind=kind, rows=log(1, max(1, min(8000, int(flops / (inner * outer))))), inner=inner, outer=outer, gated=gated,
                    bias=rng.random() < 0.4, activation=rng.choice(["silu", "gelu", "gelu_tanh", "relu"] + ([] if gated else ["none"] * 4)),
                    residual=rng.choice(["none", "fp32", "same"]), dtype=dtype, direction=direction)
    if kind == "residual":
        width = rng.choice([256, 512, 1024, 2560, 4096, log(50, 8000), log(50, 8000)])
        return dict(kind=kind, rows=log(1, max(1, 16_000_000 // width)), width=width, centered=rng.random() < 0.3, bias=rng.random() < 0.3,
                    post=rng.random() < 0.5, gate=rng.choice(["none", "channel", "full", "row"]), stream=rng.choice(["fp32", dtype]), dtype=dtype,
                    residual_scale=rng.choice([1.0, 1.0, 0.8]), block_scale=rng.choice([1.0, 0.25]), direction=direction)
    short = rng.choice([64, 256, 512, 1024, log(8, 2000)])
    long = max(short, rng.choice([short, 256, 2048, 4096, log(16, 8000)]))
    if dtype == "fp32":
        short, long = min(short, 1024), min(long, 4096)
    most = int((1.5e12 if dtype == "bf16" else 0.2e12) / (5 * (4 * short * short * long + 2 * short ** 3)))
    rows, columns = rng.choice([(short, long), (long, short)])
    return dict(kind=kind, count=log(1, max(1, min(40, most))), rows=rows, columns=columns, dtype=dtype)


# ---- inputs ------------------------------------------------------------------------------------------------------
def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, dtype=dt):
        return (torch.randn(*shape, generator=g, device=dev) * std).to(dtype)

    s = dict(case)
    if case["kind"] == "linear":
        rows, k, n = case["rows"], case["inner"], case["outer"]
        wide = torch.float32 if case["residual"] == "fp32" else dt
        s["x"] = normal(rows, k)                                    # normed rows
        s["weight"] = normal(n, k, std=k ** -0.5)
        s["up"] = normal(n, k, std=k ** -0.5) if case["gated"] else None
        s["b"] = normal(n, std=0.1) if case["bias"] else None
        s["up_b"] = normal(n, std=0.1) if case["bias"] and case["gated"] else None
        s["r"] = normal(rows, n, std=3.0, dtype=wide) if case["residual"] != "none" else None
        s["dy"] = normal(rows, n, std=0.01, dtype=wide)
    elif case["kind"] == "residual":
        rows, w = case["rows"], case["width"]
        stream = DTYPES[case["stream"]]
        size = torch.rand(rows, 1, generator=g, device=dev) * 3 + 0.2      # rows of different size, off centre
        s["h"] = ((torch.randn(rows, w, generator=g, device=dev) + 0.1) * size).to(stream)
        s["y"] = normal(rows, w)
        s["weight"] = (1 + 0.1 * torch.randn(w, generator=g, device=dev)).to(dt)
        s["b"] = normal(w, std=0.1) if case["bias"] else None
        s["post_weight"] = (1 + 0.1 * torch.randn(w, generator=g, device=dev)).to(dt) if case["post"] else None
        s["post_b"] = normal(w, std=0.1) if case["bias"] and case["post"] else None
        shape = {"none": None, "channel": (w,), "full": (rows, w), "row": (rows, 1)}[case["gate"]]
        s["g"] = None if shape is None else (0.5 + 0.3 * torch.randn(*shape, generator=g, device=dev)).to(dt)
        s["dh"], s["da"] = normal(rows, w, std=0.01, dtype=stream), normal(rows, w, std=0.01)
        s["eps"] = 1e-6
    else:
        b, m, n = case["count"], case["rows"], case["columns"]
        # averaged gradients: a few dozen strong directions over a floor of noise
        r = min(32, m, n)
        strong = torch.randn(b, m, r, generator=g, device=dev) @ (torch.randn(b, r, n, generator=g, device=dev)
                                                                  / torch.arange(1, r + 1, device=dev)[:, None])
        s["x"] = ((strong + 0.2 * torch.randn(b, m, n, generator=g, device=dev)) * 1e-4).to(dt)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------
def run(state):
    s = state
    step = s.get("direction") == "step"
    if own:
        from paper_2509_06980_amd import policy_ops as ops
        if s["kind"] == "linear":
            y, kept = ops.linear_forward(s["x"], s["weight"], s["b"], up=s["up"], up_bias=s["up_b"], activation=s["activation"], residual=s["r"],
                                         keep=step)
            if not step:
                return {"y": y}
            dx, dw, db, dup, dup_b = ops.linear_backward(s["dy"], s["x"], s["weight"], kept, up=s["up"], activation=s["activation"],
                                                         biased=s["b"] is not None, up_biased=s["up_b"] is not None)
            return {"y": y, "dx": dx, "dweight": dw, "dbias": db, "dup": dup, "dup_bias": dup_b}
        if s["kind"] == "residual":
            h, a, stats = ops.residual_norm_forward(s["h"], s["y"], s["weight"], s["b"], post_weight=s["post_weight"], post_bias=s["post_b"],
                                                    gate=s["g"], residual_scale=s["residual_scale"], block_scale=s["block_scale"], eps=s["eps"],
                                                    centered=s["centered"])
            if not step:
                return {"h": h, "a": a}
            dh, dy, dw, db, dpw, dpb, dg = ops.residual_norm_backward(
                s["dh"], s["da"], h, s["y"], stats, s["weight"], post_weight=s["post_weight"], post_bias=s["post_b"], gate=s["g"],
                residual_scale=s["residual_scale"], block_scale=s["block_scale"], centered=s["centered"], biased=s["b"] is not None)
            return {"h": h, "a": a, "dh": dh, "dy": dy, "dweight": dw, "dbias": db, "dpost_weight": dpw, "dpost_bias": dpb, "dgate": dg}
        return {"x": ops.orthogonalize(s["x"], steps=STEPS, coefficients=NEWTON)}
    return {"linear": _linear, "residual": _residual, "orthogonal": _orthogonal}[s["kind"]](s, step)


def _activation(z, name):
    """A value and its derivative."""
    if name == "relu":
        return z.clamp(min=0), (z > 0).float()
    if name == "silu":
        p = 1 / (1 + (-z).exp())
        return z * p, p * (1 + z * (1 - p))
    if name == "gelu":
        p = 0.5 * (1 + (z * 0.5 ** 0.5).erf())
        return z * p, p + z * (-0.5 * z * z).exp() * (2 * math.pi) ** -0.5
    if name == "gelu_tanh":
        c = (2 / math.pi) ** 0.5
        t = (c * (z + 0.044715 * z * z * z)).tanh()
        return 0.5 * z * (1 + t), 0.5 * (1 + t) + 0.5 * z * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    return z, torch.ones_like(z)


def _linear(s, step):
    dt, dy = s["x"].dtype, s["dy"].float()
    x, w, up = s["x"].float(), s["weight"].float(), s["up"].float() if s["gated"] else None
    z = x @ w.t()
    if s["b"] is not None:
        z = z + s["b"].float()
    act, slope = _activation(z, s["activation"])
    u = None
    if s["gated"]:
        u = x @ up.t()
        if s["up_b"] is not None:
            u = u + s["up_b"].float()
    y = act * u if s["gated"] else act
    if s["r"] is not None:
        y = y + s["r"].float()
    out = {"y": y.to(s["dy"].dtype)}
    if not step:
        return out
    dz = dy * slope * u if s["gated"] else dy * slope
    dx = dz @ w
    out |= {"dweight": (dz.t() @ x).to(dt), "dbias": dz.sum(0).to(dt) if s["b"] is not None else None, "dup": None, "dup_bias": None}
    if s["gated"]:
        du = dy * act
        dx = dx + du @ up
        out["dup"] = (du.t() @ x).to(dt)
        out["dup_bias"] = du.sum(0).to(dt) if s["up_b"] is not None else None
    return out | {"dx": dx.to(dt)}


def _normed(x, eps, centered):
    if centered:
        x = x - x.mean(-1, keepdim=True)
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    return x * r, r


def _norm_gradient(dn, n, r, centered):
    d = dn - n * (dn * n).mean(-1, keepdim=True)
    return (d - dn.mean(-1, keepdim=True) if centered else d) * r


def _residual(s, step):
    dt, c = s["y"].dtype, s["centered"]
    y, w = s["y"].float(), s["weight"].float()
    gate = s["g"].float() if s["g"] is not None else torch.ones(1, device=y.device)
    u = y
    if s["post"]:
        pw = s["post_weight"].float()
        pn, pr = _normed(y, s["eps"], c)
        u = pn * pw if s["post_b"] is None else pn * pw + s["post_b"].float()
    h = s["h"].float() * s["residual_scale"] + s["block_scale"] * gate * u
    n, r = _normed(h, s["eps"], c)
    a = n * w if s["b"] is None else n * w + s["b"].float()
    out = {"h": h.to(s["h"].dtype), "a": a.to(dt)}
    if not step:
        return out
    da = s["da"].float()
    dh = s["dh"].float() + _norm_gradient(da * w, n, r, c)
    du = dh * gate * s["block_scale"]
    out |= {"dh": (dh * s["residual_scale"]).to(s["h"].dtype), "dweight": (da * n).sum(0).to(dt), "dbias": da.sum(0).to(dt) if s["b"] is not None else None,
            "dpost_weight": None, "dpost_bias": None, "dgate": None}
    if s["g"] is not None:
        dg = dh * u * s["block_scale"]
        out["dgate"] = (dg.sum(0) if s["gate"] == "channel" else dg.sum(-1, keepdim=True) if s["gate"] == "row" else dg).to(dt)
    if s["post"]:
        out["dpost_weight"] = (du * pn).sum(0).to(dt)
        out["dpost_bias"] = du.sum(0).to(dt) if s["post_b"] is not None else None
        du = _norm_gradient(du * pw, pn, pr, c)
    return out | {"dy": du.to(dt)}


def _orthogonal(s, step):
    x = s["x"].float()
    tall = x.shape[-2] > x.shape[-1]
    if tall:
        x = x.transpose(-1, -2).contiguous()
    x = x / (x.square().sum((-1, -2), dtype=torch.float64).sqrt().float()[:, None, None] + 1e-7)
    a, b, c = NEWTON
    for _ in range(STEPS):
        g = x @ x.transpose(-1, -2).contiguous()
        x = a * x + (b * g + c * (g @ g)) @ x
    return {"x": (x.transpose(-1, -2) if tall else x).to(s["x"].dtype).contiguous()}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    """Inputs once, outputs once.  The backward pass of a product has two products for each of the forward pass; an activation's values
    before it count as written and read once.  X X^T and its square are symmetric: half of their elements."""
    el, step = (2 if case["dtype"] == "bf16" else 4), case.get("direction") == "step"
    if case["kind"] == "linear":
        rows, k, n, mats = case["rows"], case["inner"], case["outer"], 2 if case["gated"] else 1
        wide = 4 if case["residual"] == "fp32" else el
        forward = (rows * k + mats * n * k) * el + rows * n * wide * (2 if case["residual"] != "none" else 1)
        kept = rows * n * mats * el * 2 if case["activation"] != "none" else 0
        backward = rows * n * wide + (rows * k + mats * n * k) * el + kept
        return {"bytes": forward + (backward if step else 0), "flops": 2 * rows * k * n * mats * (3 if step else 1)}
    if case["kind"] == "residual":
        n, wide = case["rows"] * case["width"], 4 if case["stream"] == "fp32" else 2
        gate = {"none": 0, "channel": case["width"], "row": case["rows"], "full": n}[case["gate"]] * el
        one = n * (2 * wide + 2 * el) + gate
        return {"bytes": one + (n * (2 * wide + 2 * el) + gate if step else 0), "flops": n * (30 if step else 10)}
    m, n = sorted((case["rows"], case["columns"]))
    return {"bytes": 2 * case["count"] * m * n * el, "flops": case["count"] * STEPS * (m * m * n + m ** 3 + 2 * m * m * n)}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    step = case.get("direction") == "step"
    F = torch.nn.functional
    if case["kind"] == "linear":
        leaf = {n: s[n].double().requires_grad_(step) for n in ("x", "weight", "b", "up", "up_b") if s[n] is not None}
        act = {"none": lambda v: v, "relu": F.relu, "silu": F.silu, "gelu": F.gelu, "gelu_tanh": lambda v: F.gelu(v, approximate="tanh")}[case["activation"]]
        y = act(F.linear(leaf["x"], leaf["weight"], leaf.get("b")))
        if case["gated"]:
            y = y * F.linear(leaf["x"], leaf["up"], leaf.get("up_b"))
        if s["r"] is not None:
            y = y + s["r"].double()
        if not step:
            return {"y": y}
        got = dict(zip(leaf, torch.autograd.grad(y, list(leaf.values()), s["dy"].double())))
        return {"y": y.detach(), "dx": got["x"], "dweight": got["weight"], "dbias": got.get("b"), "dup": got.get("up"), "dup_bias": got.get("up_b")}
    if case["kind"] == "residual":
        leaf = {n: s[n].double().requires_grad_(step) for n in ("h", "y", "weight", "b", "post_weight", "post_b", "g") if s[n] is not None}

        def norm(v, weight, bias):
            if case["centered"]:
                return F.layer_norm(v, (case["width"],), weight, bias, s["eps"])
            v = v / (v.pow(2).sum(-1, keepdim=True) / case["width"] + s["eps"]).sqrt() * weight
            return v if bias is None else v + bias

        block = norm(leaf["y"], leaf["post_weight"], leaf.get("post_b")) if case["post"] else leaf["y"]
        h = leaf["h"] * case["residual_scale"] + block * case["block_scale"] * leaf.get("g", 1.0)
        a = norm(h, leaf["weight"], leaf.get("b"))
        if not step:
            return {"h": h, "a": a}
        got = dict(zip(leaf, torch.autograd.grad([h, a], list(leaf.values()), [s["dh"].double(), s["da"].double()])))
        return {"h": h.detach(), "a": a.detach(), "dh": got["h"], "dy": got["y"], "dweight": got["weight"], "dbias": got.get("b"),
                "dpost_weight": got.get("post_weight"), "dpost_bias": got.get("post_b"), "dgate": got.get("g")}
    a, b, c = NEWTON
    out = []
    for x in s["x"].double():
        x = x / (x.norm() + 1e-7)
        left = x.shape[0] <= x.shape[1]      # the smaller of X X^T and X^T X
        for _ in range(STEPS):
            if left:
                g = torch.mm(x, x.t())
                x = a * x + b * torch.mm(g, x) + c * torch.mm(g, torch.mm(g, x))
            else:
                g = torch.mm(x.t(), x)
                x = a * x + b * torch.mm(x, g) + c * torch.mm(torch.mm(x, g), g)
        out.append(x)
    return {"x": torch.stack(out)}
