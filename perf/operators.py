"""Timed cases of the policy-update operators: norms, rotary positions, attention over packed trajectories and
log-probs of tokens, each with the backward pass that the update needs.

The policy update follows the rollout: the trajectories that the engine generated are run through the decoder again,
the log-probs of the sampled tokens enter the objective, and its gradient goes back through the same operators.  Every
case is one operator; `direction` says whether a pass is the forward call alone (scoring, decode) or the forward call
and the backward call that a training step makes (`step`).

Sizes are those of the repository's shapes (hidden 256, 1024, 2560 and 4096, 4 to 32 heads over 2 to 8 KV heads, head
sizes 64 and 128, vocabularies of 4096 and 151936) and odd ones around them.
"""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def listed():
    return [
        # layer norm of a short trajectory in fp32, odd width: latency
        dict(name="norm-layer-fp32-odd-step", kind="norm", rows=61, heads=1, width=1023, total=1, centered=True, dtype="fp32", direction="step"),
        # the norm before a projection in an update over 16 trajectories of about 500 tokens
        dict(name="norm-4b-step", kind="norm", rows=7777, heads=1, width=2560, total=1, centered=False, dtype="bf16", direction="step"),
        # QK-norm of the query heads where they lie in the fused QKV projection
        dict(name="norm-heads-step", kind="norm", rows=4001, heads=32, width=128, total=48, centered=False, dtype="bf16", direction="step"),
        # a decode batch of 128 trajectories at contexts of some thousand tokens, table stretched for long contexts
        dict(name="rotary-decode-128", kind="rotary", tokens=128, q_heads=32, kv_heads=8, head_dim=128, rot_dim=128, interleaved=False,
             positions=16384, stretch=4.0, dtype="bf16", direction="forward"),
        # an update over 12000 packed tokens, heads read from the fused projection
        dict(name="rotary-4b-step", kind="rotary", tokens=12007, q_heads=32, kv_heads=8, head_dim=128, rot_dim=128, interleaved=False,
             positions=4096, stretch=1.0, dtype="bf16", direction="step"),
        # fp32, neighbouring pairs, half of the head turned, long positions
        dict(name="rotary-part-fp32-step", kind="rotary", tokens=3001, q_heads=16, kv_heads=8, head_dim=64, rot_dim=32, interleaved=True,
             positions=100000, stretch=8.0, dtype="fp32", direction="step"),
        # the fp32 shape's update: 4 trajectories of about 100 tokens
        dict(name="attention-tiny-fp32-step", kind="attention", sequences=4, longest=104, shortest=57, suffix=1.0, q_heads=4, kv_heads=2,
             head_dim=64, dtype="fp32", direction="step"),
        # ragged trajectories of several turns, 4B head layout
        dict(name="attention-ragged-step", kind="attention", sequences=16, longest=1511, shortest=97, suffix=1.0, q_heads=32, kv_heads=8,
             head_dim=128, dtype="bf16", direction="step"),
        # one long trajectory, 0.6B head layout
        dict(name="attention-long-step", kind="attention", sequences=1, longest=8192, shortest=8192, suffix=1.0, q_heads=16, kv_heads=8,
             head_dim=128, dtype="bf16", direction="step"),
        # the fp32 shape's loss
        dict(name="logprob-tiny-fp32-step", kind="logprob", rows=288, sampled=0.67, hidden=256, vocab=4096, temperature=1.0, dtype="fp32",
             direction="step"),
        # a reference policy scores finished trajectories: no gradient, half the tokens are observations
        dict(name="logprob-0.6b-score", kind="logprob", rows=8191, sampled=0.5, hidden=1024, vocab=151936, temperature=1.0, dtype="bf16",
             direction="forward"),
        # the loss of an update and its gradient, a third of the tokens masked out
        dict(name="logprob-4b-step", kind="logprob", rows=4096, sampled=0.67, hidden=2560, vocab=151936, temperature=1.0, dtype="bf16",
             direction="step"),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["norm", "rotary", "attention", "attention", "logprob", "logprob"])
    dtype = "fp32" if rng.random() < 0.25 else "bf16"
    direction = rng.choice(["forward", "step", "step"])
    if kind == "norm":
        width = rng.choice([64, 128, 256, 1024, 2560, 4096, log(50, 8000), log(50, 8000)])
        heads = rng.choice([1, 1, 8, 32]) if width <= 256 else 1
        return dict(kind=kind, rows=log(1, max(1, 20_000_000 // (width * heads))), heads=heads, width=width, total=heads + rng.choice([0, 0, 1, 16]),
                    centered=rng.random() < 0.4, dtype=dtype, direction=direction)
    if kind == "rotary":
        head_dim = rng.choice([64, 128, 128, 96])
        kv_heads = rng.choice([1, 2, 8])
        q_heads = kv_heads * rng.choice([1, 2, 4])
        return dict(kind=kind, tokens=log(1, 400_000 // (q_heads + kv_heads)), q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                    rot_dim=head_dim if rng.random() < 0.6 else 2 * rng.randint(1, head_dim // 2), interleaved=rng.random() < 0.4,
                    positions=log(100, 130_000), stretch=rng.choice([1.0, 4.0, 8.0]), dtype=dtype, direction=direction)
    if kind == "attention":
        kv_heads = rng.choice([1, 2, 8])
        q_heads = kv_heads * rng.choice([1, 2, 4, 8] if kv_heads < 8 else [1, 2, 4])
        sequences = log(1, 32)
        longest = log(8, min(6000, int(math.sqrt(1.5e9 / (sequences * q_heads)))))
        if dtype == "fp32":
            longest = min(longest, 2000)
        return dict(kind=kind, sequences=sequences, longest=longest, shortest=rng.choice([longest, 1, max(1, longest // 8)]),
                    suffix=1.0 if rng.random() < 0.7 else round(rng.uniform(0.02, 0.9), 3), q_heads=q_heads, kv_heads=kv_heads,
                    head_dim=rng.choice([64, 128, 128, 80]), dtype=dtype, direction=direction)
    hidden = rng.choice([256, 1024, 2560, 4096, 8 * log(16, 400)])
    vocab = rng.choice([4096, 8192, 151936, log(1000, 150_000)])
    rows = log(1, min(8000, int((0.8e12 if dtype == "bf16" else 0.15e12) / (hidden * vocab))))
    return dict(kind=kind, rows=rows, sampled=round(rng.uniform(0.3, 1.0), 2), hidden=hidden, vocab=vocab,
                temperature=rng.choice([1.0, 1.0, 0.7, 1.3]), dtype=dtype, direction=direction)


# ---- inputs ------------------------------------------------------------------------------------------------------
def _lengths(case):
    """Lengths of the case's trajectories, the same for every seed: the longest, the shortest, the rest between them on a
    logarithmic scale, in mixed order.  `suffix`: share of a trajectory whose tokens are queries (at least one)."""
    n, hi, lo = case["sequences"], case["longest"], case["shortest"]
    r = random.Random(1000003 * n + hi)
    keys = [hi] if n == 1 else [hi, lo] + [int(round(math.exp(r.uniform(math.log(lo), math.log(hi))))) for _ in range(n - 2)]
    r.shuffle(keys)
    return [max(1, int(round(k * case["suffix"]))) for k in keys], keys


def _kept(case):
    """Tokens of a log-prob case that were sampled, the same number for every seed."""
    return max(1, int(round(case["rows"] * case["sampled"])))


def _table(case, device):
    """cos and sin of every position's angles: rates theta^(-2i / rot_dim), the slow ones divided by `stretch` (a band in
    between gradually), computed in 64 bits and kept in 32."""
    half = case["rot_dim"] // 2
    i = torch.arange(half, dtype=torch.float64, device=device)
    rate = 1e6 ** (-2.0 * i / case["rot_dim"])
    turns = rate * 4096 / (2 * math.pi)
    slow = ((32.0 - turns) / 31.0).clamp(0.0, 1.0)
    rate = rate * (1.0 - slow) + rate / case["stretch"] * slow
    angle = torch.arange(case["positions"], dtype=torch.float64, device=device)[:, None] * rate
    return torch.stack([angle.cos(), angle.sin()], -1).float().contiguous()


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device=dev) * std).to(dt)

    s = dict(case)
    if case["kind"] == "norm":
        rows, heads, width = case["rows"], case["heads"], case["width"]
        # activations of a residual stream: rows of different size, off centre
        size = torch.rand(rows, 1, 1, generator=g, device=dev) * 3 + 0.2
        full = ((torch.randn(rows, case["total"], width, generator=g, device=dev) + 0.1) * size).to(dt)
        s["x"] = full[:, :heads]
        s["weight"] = (1 + 0.1 * torch.randn(width, generator=g, device=dev)).to(dt)
        s["bias"] = normal(width, std=0.1) if case["centered"] else None
        s["dy"] = normal(rows, heads, width, std=0.01)
        s["eps"] = 1e-6
    elif case["kind"] == "rotary":
        t, nq, nk, d = case["tokens"], case["q_heads"], case["kv_heads"], case["head_dim"]
        qkv = normal(t, nq + 2 * nk, d)
        s["q"], s["k"] = qkv[:, :nq], qkv[:, nq:nq + nk]
        s["dq"], s["dk"] = normal(t, nq, d, std=0.01), normal(t, nk, d, std=0.01)
        s["positions"] = torch.randint(0, case["positions"], (t,), generator=g, device=dev, dtype=torch.int32)
        s["table"] = _table(case, dev)
    elif case["kind"] == "attention":
        lq, lk = _lengths(case)
        nq, nk, d = case["q_heads"], case["kv_heads"], case["head_dim"]
        s["q"] = normal(sum(lq), nq, d, std=1.5)          # after QK-norm and its gains
        kv = normal(sum(lk), 2 * nk, d)
        s["k"], s["v"] = kv[:, :nk], kv[:, nk:]
        s["do"] = normal(sum(lq), nq, d, std=0.01)
        s["cu_q"], s["cu_k"] = (torch.tensor([sum(l[:i]) for i in range(len(l) + 1)], dtype=torch.int32, device=dev) for l in (lq, lk))
        s["max_q"], s["max_k"] = max(lq), max(lk)
        s["scale"] = d ** -0.5
    else:
        rows, h, v = case["rows"], case["hidden"], case["vocab"]
        std = 2.0 / math.sqrt(h)
        s["weight"] = normal(v, h, std=std)
        target = torch.randint(0, v, (rows,), generator=g, device=dev, dtype=torch.int32)
        # normed rows that lean towards the token that was sampled: log-probs from about -12 to about -0.1
        lean = torch.rand(rows, 1, generator=g, device=dev) * 14 / (std * std * h)
        s["hidden_rows"] = (torch.randn(rows, h, generator=g, device=dev) + lean * s["weight"][target.long()].float()).to(dt)
        masked = torch.randperm(rows, generator=g, device=dev)[: rows - _kept(case)]
        target[masked] = -1                                # observation tokens take no part
        s["targets"] = target
        s["dlogp"] = torch.randn(rows, generator=g, device=dev) * 1e-3
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------
def run(state):
    s = state
    step = s["direction"] == "step"
    if own:
        from paper_2509_06980_amd import policy_ops as ops
        if s["kind"] == "norm":
            y, mean, rstd = ops.norm_forward(s["x"], s["weight"], s["bias"], eps=s["eps"], centered=s["centered"])
            if not step:
                return {"y": y}
            dx, dweight, dbias = ops.norm_backward(s["dy"], s["x"], s["weight"], mean, rstd, centered=s["centered"])
            return {"y": y, "dx": dx, "dweight": dweight, **({"dbias": dbias} if s["centered"] else {})}
        if s["kind"] == "rotary":
            q, k = ops.rotary(s["q"], s["k"], s["positions"], s["table"], interleaved=s["interleaved"])
            if not step:
                return {"q": q, "k": k}
            dq, dk = ops.rotary(s["dq"], s["dk"], s["positions"], s["table"], interleaved=s["interleaved"], inverse=True)
            return {"q": q, "k": k, "dq": dq, "dk": dk}
        if s["kind"] == "attention":
            o, lse = ops.attention_forward(s["q"], s["k"], s["v"], s["cu_q"], s["cu_k"], scale=s["scale"], causal=True)
            if not step:
                return {"o": o, "lse": lse}
            dq, dk, dv = ops.attention_backward(s["do"], s["q"], s["k"], s["v"], o, lse, s["cu_q"], s["cu_k"], scale=s["scale"], causal=True)
            return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv}
        logp, lse = ops.token_logprobs_forward(s["hidden_rows"], s["weight"], s["targets"], temperature=s["temperature"])
        if not step:
            return {"logp": logp, "lse": lse}
        dhidden, dweight = ops.token_logprobs_backward(s["dlogp"], s["hidden_rows"], s["weight"], s["targets"], lse, temperature=s["temperature"])
        return {"logp": logp, "lse": lse, "dhidden": dhidden, "dweight": dweight}
    return {"norm": _norm, "rotary": _rotary, "attention": _attention, "logprob": _logprob}[s["kind"]](s, step)


def _norm(s, step):
    dt = s["x"].dtype
    x, w = s["x"].float(), s["weight"].float()
    if s["centered"]:
        x = x - x.mean(-1, keepdim=True)
    rstd = (x.square().mean(-1, keepdim=True) + s["eps"]).rsqrt()
    n = x * rstd
    y = (n * w + s["bias"].float() if s["centered"] else n * w).to(dt)
    if not step:
        return {"y": y}
    dy = s["dy"].float()
    dn = dy * w
    dx = dn - n * (dn * n).mean(-1, keepdim=True)
    if s["centered"]:
        dx = dx - dn.mean(-1, keepdim=True)
    out = {"y": y, "dx": (dx * rstd).to(dt), "dweight": (dy * n).sum((0, 1)).to(dt)}
    if s["centered"]:
        out["dbias"] = dy.sum((0, 1)).to(dt)
    return out


def _rotary(s, step):
    r, cs = s["rot_dim"], s["table"][s["positions"].long()]

    def turn(x, sign):
        t = x.float()
        c, n = cs[:, None, :, 0], cs[:, None, :, 1] * sign
        if s["interleaved"]:
            a, b = t[..., 0:r:2], t[..., 1:r:2]
            turned = torch.stack([a * c - b * n, b * c + a * n], -1).flatten(-2)
        else:
            a, b = t[..., :r // 2], t[..., r // 2:r]
            turned = torch.cat([a * c - b * n, b * c + a * n], -1)
        return torch.cat([turned, t[..., r:]], -1).to(x.dtype)

    out = {"q": turn(s["q"], 1.0), "k": turn(s["k"], 1.0)}
    if step:
        out |= {"dq": turn(s["dq"], -1.0), "dk": turn(s["dk"], -1.0)}
    return out


def _attention(s, step):
    dt, dev, group = s["q"].dtype, s["q"].device, s["q_heads"] // s["kv_heads"]

    def places(cu, total, longest):
        """Of every token: its sequence and position; of every (sequence, position): its token (any where there is none)."""
        t = torch.arange(total, device=dev)
        seq = torch.searchsorted(cu[1:].long(), t, right=True)
        return seq, t - cu.long()[seq], (cu[:-1, None].long() + torch.arange(longest, device=dev)).clamp(max=total - 1)

    seq_q, pos_q, at_q = places(s["cu_q"], s["q"].shape[0], s["max_q"])
    seq_k, pos_k, at_k = places(s["cu_k"], s["k"].shape[0], s["max_k"])
    lq, lk = (s["cu_q"].diff()[:, None, None], s["cu_k"].diff()[:, None, None])
    i, j = torch.arange(s["max_q"], device=dev)[None, :, None], torch.arange(s["max_k"], device=dev)[None, None, :]
    seen = ((i < lq) & (j < lk) & (j <= i + lk - lq))[:, None]
    heads = torch.arange(s["q_heads"], device=dev) // group
    q = s["q"].float()[at_q].transpose(1, 2)
    k = s["k"].float()[at_k][:, :, heads].transpose(1, 2)
    v = s["v"].float()[at_k][:, :, heads].transpose(1, 2)
    z = (q @ k.transpose(-1, -2) * s["scale"]).masked_fill(~seen, -math.inf)
    top = z.amax(-1, keepdim=True)
    e = (z - top.masked_fill(top == -math.inf, 0.0)).exp()
    del z
    total = e.sum(-1, keepdim=True)
    p = e / total.masked_fill(total == 0, 1.0)
    del e
    lse = (top + total.log())[..., 0]
    o = p @ v
    out = {"o": o[seq_q, :, pos_q].to(dt), "lse": lse[seq_q, :, pos_q].t().contiguous()}
    if not step:
        return out
    do = s["do"].float()[at_q].transpose(1, 2)
    dv = p.transpose(-1, -2) @ do
    dz = p * (do @ v.transpose(-1, -2) - (do * o).sum(-1, keepdim=True)) * s["scale"]
    del p
    dq = dz @ k
    dk = dz.transpose(-1, -2) @ q
    del dz

    def grouped(x):
        return x.unflatten(1, (s["kv_heads"], group)).sum(2)[seq_k, :, pos_k].to(dt)

    return out | {"dq": dq[seq_q, :, pos_q].to(dt), "dk": grouped(dk), "dv": grouped(dv)}


def _logprob(s, step):
    dt, kept = s["hidden_rows"].dtype, s["targets"] >= 0
    x, w, y = s["hidden_rows"][kept].float(), s["weight"].float(), s["targets"][kept].long()[:, None]
    z = x @ w.t() / s["temperature"]
    top = z.amax(-1, keepdim=True)
    lse = top + (z - top).exp().sum(-1, keepdim=True).log()
    rows = s["targets"].shape[0]
    out = {"logp": torch.zeros(rows, device=x.device), "lse": torch.zeros(rows, device=x.device)}
    out["logp"][kept] = (z.gather(1, y) - lse)[:, 0]
    out["lse"][kept] = lse[:, 0]
    if not step:
        return out
    g = s["dlogp"][kept][:, None] / s["temperature"]
    dz = (z - lse).exp() * -g
    del z
    dz.scatter_add_(1, y, g)
    dhidden = torch.zeros(rows, x.shape[1], dtype=dt, device=x.device)
    dhidden[kept] = (dz @ w).to(dt)
    return out | {"dhidden": dhidden, "dweight": (dz.t() @ x).to(dt)}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------
def work(case):
    """Inputs once, outputs once.  The backward passes of attention and of the log-probs get no probabilities from the
    forward pass (one number a row is kept), so their scores count a second time."""
    el, step = (2 if case["dtype"] == "bf16" else 4), case["direction"] == "step"
    if case["kind"] == "norm":
        n = case["rows"] * case["heads"] * case["width"]
        return {"bytes": n * el * (4 if step else 2) + case["width"] * el * (2 if step else 1) * (2 if case["centered"] else 1),
                "flops": n * (14 if step else 4)}
    if case["kind"] == "rotary":
        n = case["tokens"] * (case["q_heads"] + case["kv_heads"]) * case["head_dim"]
        rows = min(case["tokens"], case["positions"]) * case["rot_dim"] * 4 + case["tokens"] * 4
        return {"bytes": n * el * (4 if step else 2) + rows, "flops": n * (6 if step else 3)}
    if case["kind"] == "attention":
        lq, lk = _lengths(case)
        pairs = sum(a * b - a * (a - 1) // 2 for a, b in zip(lq, lk))
        q, k = sum(lq) * case["q_heads"] * case["head_dim"] * el, sum(lk) * case["kv_heads"] * case["head_dim"] * el
        return {"bytes": (2 * q + 2 * k) * (2 if step else 1) + sum(lq) * case["q_heads"] * 4,
                "flops": pairs * case["q_heads"] * case["head_dim"] * (14 if step else 4)}
    rows, h, v = _kept(case), case["hidden"], case["vocab"]
    return {"bytes": (rows * h + v * h) * el * (2 if step else 1) + case["rows"] * (16 if step else 12), "flops": 2 * rows * h * v * (4 if step else 1)}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    step = case["direction"] == "step"
    if case["kind"] == "norm":
        x = s["x"].double().requires_grad_()
        w = s["weight"].double().requires_grad_()
        b = s["bias"].double().requires_grad_() if case["centered"] else None
        if case["centered"]:
            y = torch.nn.functional.layer_norm(x, (case["width"],), w, b, s["eps"])
        else:
            y = x / (x.pow(2).sum(-1, keepdim=True) / case["width"] + s["eps"]).sqrt() * w
        if not step:
            return {"y": y.detach()}
        grads = torch.autograd.grad(y, [x, w] + ([b] if case["centered"] else []), s["dy"].double())
        return {"y": y.detach(), **dict(zip(("dx", "dweight", "dbias"), grads))}
    if case["kind"] == "rotary":
        r = case["rot_dim"]
        angle = s["table"].double()[s["positions"].long()]
        turned = torch.complex(angle[..., 0], angle[..., 1])[:, None]

        def turn(x, by):
            x = x.double()
            pairs = x[..., :r].unflatten(-1, (r // 2, 2)) if case["interleaved"] else x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * by)
            z = z if case["interleaved"] else z.transpose(-1, -2)
            return torch.cat([z.flatten(-2), x[..., r:]], -1)

        out = {"q": turn(s["q"], turned), "k": turn(s["k"], turned)}
        return out | {"dq": turn(s["dq"], turned.conj()), "dk": turn(s["dk"], turned.conj())} if step else out
    if case["kind"] == "attention":
        group = case["q_heads"] // case["kv_heads"]
        leaf = {n: s[n].double() for n in ("q", "k", "v", "do")}
        o, lse = torch.zeros_like(leaf["q"]), torch.zeros(case["q_heads"], leaf["q"].shape[0], dtype=torch.float64, device="cuda")
        dq, dk, dv = (torch.zeros_like(leaf[n]) for n in ("q", "k", "v"))
        q0 = k0 = 0
        for a, b in zip(*_lengths(case)):
            hidden = torch.ones(a, b, dtype=torch.bool, device="cuda").triu(b - a + 1)
            for h in range(case["q_heads"]):
                part = [leaf["q"][q0:q0 + a, h], leaf["k"][k0:k0 + b, h // group], leaf["v"][k0:k0 + b, h // group]]
                part = [t.clone().requires_grad_(step) for t in part]
                with torch.set_grad_enabled(step):
                    z = (part[0] @ part[1].t() * s["scale"]).masked_fill(hidden, -math.inf)
                    r = torch.softmax(z, -1) @ part[2]
                lse[h, q0:q0 + a] = torch.logsumexp(z.detach(), -1)
                o[q0:q0 + a, h] = r.detach()
                if step:
                    d = torch.autograd.grad(r, part, leaf["do"][q0:q0 + a, h])
                    dq[q0:q0 + a, h] = d[0]
                    dk[k0:k0 + b, h // group] += d[1]
                    dv[k0:k0 + b, h // group] += d[2]
            q0, k0 = q0 + a, k0 + b
        return {"o": o, "lse": lse, "dq": dq, "dk": dk, "dv": dv} if step else {"o": o, "lse": lse}
    rows = s["targets"].shape[0]
    kept = (s["targets"] >= 0).nonzero()[:, 0]
    w = s["weight"].double()
    out = {n: torch.zeros(rows, dtype=torch.float64, device="cuda") for n in ("logp", "lse")}
    dhidden, dweight = torch.zeros(rows, case["hidden"], dtype=torch.float64, device="cuda"), torch.zeros_like(w) if step else None
    for at in kept.split(1024):
        x, y = s["hidden_rows"][at].double(), s["targets"][at].long()
        lp = torch.log_softmax(x @ w.t() / case["temperature"], -1)
        out["logp"][at] = lp.gather(1, y[:, None])[:, 0]
        out["lse"][at] = (x * w[y]).sum(-1) / case["temperature"] - out["logp"][at]
        if step:
            dz = -lp.exp_()
            dz[torch.arange(len(at), device="cuda"), y] += 1.0
            dz *= s["dlogp"][at].double()[:, None] / case["temperature"]
            dhidden[at] = dz @ w
            dweight += dz.t() @ x
    return out | {"dhidden": dhidden, "dweight": dweight} if step else out
