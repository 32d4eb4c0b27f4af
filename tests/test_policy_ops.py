"""The policy update's operators on the GPU against their formulas in float64, at sizes where tiles, strides and masks can go wrong.

Bounds, per element, are first-order error bounds of the arithmetic that the header states, with u = 2^-8 for a rounding to bf16 (8 significant bits) and
e = 2^-24 for one in fp32 (a sum of n terms is allowed n + 16 of them, more than any order of adding needs):
rounded once:        u |y| + e-term of the sums that lead to y;
rounded operand:     the same rounding on every term of the product it enters, sum of u |a| |b|;
below 2^-126:        relative errors mean nothing there, TINY covers the terms of a sum that fall below it.
"""
import math

import pytest
import torch

from paper_2509_06980_amd import policy_ops as ops
from paper_2509_06980_amd.binding import RolloutError, debug_token_logprob_loads

pytestmark = pytest.mark.gpu
BF, FP = torch.bfloat16, torch.float32
E32 = 2.0 ** -24
TINY = 1e-35


def unit(dt):
    return 2.0 ** -8 if dt == BF else 0.0


def gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def randn(g, *shape, dt=FP, std=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dt)


def within(name, got, want, bound):
    got = got.double()
    assert got.shape == want.shape, name
    assert torch.equal(got.isnan(), want.isnan()), f"{name}: numbers and no numbers"
    inf = want.isinf()
    assert torch.equal(got[inf], want[inf]), f"{name}: infinities"
    ok = want.isfinite()
    bad = (got[ok] - want[ok]).abs() - bound.expand_as(want)[ok] - TINY
    assert bad.numel() == 0 or bad.max() <= 0, f"{name}: {bad.max().item():.3g} beyond its bound"


# ---- norms ---------------------------------------------------------------------------------------------------------
def norm_reference(x, w, b, eps, centered, dy, dt):
    x, w, dy = x.double(), w.double(), dy.double()
    width = x.shape[-1]
    mu = x.mean(-1, keepdim=True) if centered else torch.zeros_like(x[..., :1])
    d = x - mu
    r = (d.square().mean(-1, keepdim=True) + eps).rsqrt()
    n = d * r
    y = n * w + (b.double() if b is not None else 0)
    dn = dy * w
    m1, m2 = (dn * n).mean(-1, keepdim=True), (dn.mean(-1, keepdim=True) if centered else 0)
    dx = r * (dn - n * m1 - m2)
    e = E32 * (width + 16)
    u = unit(dt)
    big = d.abs() + (x.abs().mean(-1, keepdim=True) if centered else 0)      # what the rounding of the mean moves
    ey = e * (big * r * w.abs() + y.abs()) + 2 * E32 * (b.double().abs() if b is not None else 0)
    a1 = (dn * n).abs().mean(-1, keepdim=True) + (dn.abs() * big * r).mean(-1, keepdim=True)
    edx = 4 * e * r * (dn.abs() + big * r * (a1 + m1.abs()) + dn.abs().mean(-1, keepdim=True))
    rows = x.numel() // width
    er = E32 * (rows + 2 * width + 32)
    dw, db = (dy * n).flatten(0, -2).sum(0), dy.flatten(0, -2).sum(0)
    edw = er * (dy.abs() * (n.abs() + big * r)).flatten(0, -2).sum(0)
    edb = er * dy.abs().flatten(0, -2).sum(0)
    return dict(y=(y, ey + u * y.abs()), dx=(dx, edx + u * dx.abs()), dw=(dw, edw + u * dw.abs()), db=(db, edb + u * db.abs()))


@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("centered", [False, True])
@pytest.mark.parametrize("rows,width", [(1, 1), (3, 5), (1, 2560), (61, 1023), (5, 64), (700, 128), (33, 513), (130, 4096), (3, 4104), (7, 8192),
                                        (2, 16384), (3, 16392), (2, 20001), (2100, 256), (9, 2049)])
def test_norm(rows, width, centered, dt):
    g = gen(rows * 7 + width)
    x = randn(g, rows, width, dt=dt) * 2 + 0.25
    w, b, dy = (1 + randn(g, width, std=0.2)).to(dt), randn(g, width, dt=dt), randn(g, rows, width, dt=dt)
    bias = b if centered else None
    y, mean, rstd = ops.norm_forward(x, w, bias, eps=1e-6, centered=centered)
    dx, dw, db = ops.norm_backward(dy, x, w, mean, rstd, centered=centered)
    ref = norm_reference(x, w, bias, 1e-6, centered, dy, dt)
    within("y", y, *ref["y"])
    if width > 1 or not centered:      # a layer norm of one element: 0 / sqrt(eps), its gradient all cancellation
        within("dx", dx, *ref["dx"])
        within("dw", dw, *ref["dw"])
    if centered:
        within("db", db, *ref["db"])
    else:
        assert mean is None and db is None


@pytest.mark.parametrize("centered", [False, True])
@pytest.mark.parametrize("rows,width", [(1, 3080), (600, 3400), (1030, 4088)])
def test_norm_of_wide_bf16_rows(rows, width, centered):
    g = gen(rows + width)
    x, w, dy = randn(g, rows, width, dt=BF) * 2 + 0.25, (1 + randn(g, width, std=0.2)).to(BF), randn(g, rows, width, dt=BF)
    bias = randn(g, width, dt=BF) if centered else None
    y, mean, rstd = ops.norm_forward(x, w, bias, eps=1e-6, centered=centered)
    dx, dw, db = ops.norm_backward(dy, x, w, mean, rstd, centered=centered)
    ref = norm_reference(x, w, bias, 1e-6, centered, dy, BF)
    for name, got in (("y", y), ("dx", dx), ("dw", dw)) + ((("db", db),) if centered else ()):
        within(name, got, *ref[name])


@pytest.mark.parametrize("dt", [BF, FP])
def test_norm_of_heads_in_a_fused_projection(dt):
    g = gen(5)
    qkv, w = randn(g, 77, 12, 128, dt=dt), (1 + randn(g, 128, std=0.1)).to(dt)
    x, dy = qkv[:, 2:10], randn(g, 77, 20, 128, dt=dt)[:, 3:11]
    y, mean, rstd = ops.norm_forward(x, w)
    dx, dw, _ = ops.norm_backward(dy, x, w, mean, rstd)
    assert not x.is_contiguous() and rstd.shape == (77, 8)
    ref = norm_reference(x, w, None, 1e-6, False, dy, dt)
    for name, got in (("y", y), ("dx", dx), ("dw", dw)):
        within(name, got, *ref[name])
    # the same from other places: unaligned, transposed, contiguous gradients
    off = randn(g, 77 * 12 * 128 + 1, dt=dt)[1:].view(77, 12, 128)
    off.copy_(qkv)
    assert torch.equal(ops.norm_forward(off[:, 2:10].contiguous(), w)[0], y)
    within("y unaligned", ops.norm_forward(off[:, 2:10], w)[0], *ref["y"])
    within("y transposed", ops.norm_forward(x.transpose(0, 1), w)[0].transpose(0, 1), *ref["y"])
    within("dx mixed", ops.norm_backward(dy.contiguous(), x, w, mean, rstd)[0], *ref["dx"])
    within("dx mixed", ops.norm_backward(dy, x.contiguous(), w, mean, rstd)[0], *ref["dx"])
    zero = torch.zeros(1, 1, 128, dtype=dt, device="cuda")
    assert not ops.norm_backward(zero.expand(77, 8, 128), x, w, mean, rstd)[0].any()


def test_norm_without_rows_and_of_odd_values():
    w = torch.ones(64, device="cuda")
    x = torch.zeros(0, 64, device="cuda")
    y, mean, rstd = ops.norm_forward(x, w)
    dx, dw, db = ops.norm_backward(x, x, w, mean, rstd, biased=True)
    assert y.shape == dx.shape == (0, 64) and not dw.any() and not db.any()
    x = torch.zeros(4, 64, device="cuda")
    x[1], x[2, 3], x[3] = 1e-30, math.nan, 1e18
    y = ops.norm_forward(x, w, eps=1e-6)[0]
    assert not y[0].any() and y[1].abs().max() < 1e-26 and y[2].isnan().all() and torch.allclose(y[3], torch.ones_like(y[3]))


# ---- rotary positions ----------------------------------------------------------------------------------------------
def rotary_reference(x, cs, interleaved, sign):
    r = 2 * cs.shape[1]
    x, c, s = x.double(), cs[:, None, :, 0].double(), cs[:, None, :, 1].double() * sign
    i = torch.arange(r // 2, device="cuda")
    first, second = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
    y, big = x.clone(), torch.zeros_like(x)
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., second] * c + x[..., first] * s
    big[..., first] = big[..., second] = (x[..., first] * c).abs() + (x[..., second] * s).abs() + (x[..., second] * c).abs() + (x[..., first] * s).abs()
    return y, big


@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,nq,nk,d,rot", [(1, 1, 0, 2, 2), (1, 32, 8, 128, 128), (129, 4, 2, 64, 64), (37, 3, 1, 96, 32), (50, 16, 8, 80, 6),
                                                (3, 40, 1, 128, 64), (7, 5, 5, 66, 66), (2, 300, 2, 512, 512), (5, 2, 1, 33, 16)])
def test_rotary(tokens, nq, nk, d, rot, interleaved, dt):
    g = gen(tokens + d)
    x = randn(g, tokens, nq + 2 * nk, d, dt=dt)
    q, k = x[:, :nq], x[:, nq:nq + nk] if nk else None
    table = ops.rotary_table(1000, rot, theta=1e6, stretch=4.0, trained_positions=100, gain=1.1)
    pos = torch.randint(0, 1000, (tokens,), generator=g, device="cuda", dtype=torch.int32)
    cs = table[pos.long()]
    for inverse in (False, True):
        got = ops.rotary(q, k, pos, table, interleaved=interleaved, inverse=inverse)
        for a, b in ((got[0], q), (got[1], k)):
            if b is None:
                assert a is None
                continue
            want, big = rotary_reference(b, cs, interleaved, -1 if inverse else 1)
            assert a.is_contiguous()
            within("turned", a, want, 3 * E32 * big + unit(dt) * want.abs())
            assert torch.equal(a[..., rot:], b[..., rot:])
    # in place, into the projection it came from
    want = ops.rotary(q, k, pos, table, interleaved=interleaved)
    ops.rotary(q, k, pos, table, interleaved=interleaved, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and (k is None or torch.equal(k, want[1]))


def test_rotary_positions_outside_the_table_and_no_tokens():
    table = ops.rotary_table(10, 8)
    x = torch.ones(4, 2, 16, device="cuda")
    y, _ = ops.rotary(x, None, torch.tensor([9, 10, -1, 0], dtype=torch.int32, device="cuda"), table)
    assert y[[1, 2], :, :8].isnan().all() and not y[:, :, 8:].isnan().any() and not y[[0, 3]].isnan().any()
    y, _ = ops.rotary(x[:0], None, torch.empty(0, dtype=torch.int32, device="cuda"), table)
    assert y.shape == (0, 2, 16)


def test_rotary_table_rules():
    plain, half = ops.rotary_table(64, 32, theta=1e4), ops.rotary_table(64, 32, theta=1e4, stretch=2.0)
    assert torch.allclose(half[::2], plain[:32], atol=1e-6)          # all angles divided
    mixed = ops.rotary_table(64, 32, theta=1e4, stretch=2.0, trained_positions=512)
    assert torch.equal(mixed[:, 0], plain[:, 0]) and torch.equal(mixed[:, -1], half[:, -1])
    i = torch.arange(16, dtype=torch.float64)
    want = torch.arange(64, dtype=torch.float64)[:, None] * 1e4 ** (-i / 16)
    assert torch.equal(plain.cpu(), torch.stack([want.cos(), want.sin()], -1).float()) or torch.allclose(plain.cpu().double(), torch.stack([want.cos(), want.sin()], -1), atol=2e-7)


def test_rotary_outputs_are_known_to_autograd():
    g = gen(14)
    table, pos = ops.rotary_table(50, 64), torch.arange(9, device="cuda", dtype=torch.int32)
    x, k = randn(g, 9, 4, 64), randn(g, 9, 2, 64)
    y, z = x.clone(), k.clone()
    a = torch.ones_like(x).requires_grad_()
    product = (a * y).sum()      # keeps y for its gradient
    before = y._version, z._version
    ops.rotary(y, z, pos, table, q_out=y, k_out=z)
    assert y._version > before[0] and z._version > before[1]
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        product.backward()
    # an output that a gradient is wanted of, and one whose elements share memory
    for bad in (dict(q_out=x.clone().requires_grad_()), dict(k_out=k.clone().requires_grad_()), dict(q_out=(x.clone().requires_grad_() * 1)),
                dict(q_out=x[:, :1].expand(9, 4, 64)), dict(k_out=k[:1].expand(9, 2, 64))):
        with pytest.raises(RolloutError):
            ops.rotary(x, k, pos, table, **bad)
    leaf = x.clone().requires_grad_()
    with torch.no_grad():
        ops.rotary(x, None, pos, table, q_out=leaf)
    assert torch.equal(leaf, y)


# ---- attention -----------------------------------------------------------------------------------------------------
def attention_reference(q, k, v, do, lq, lk, causal, scale, dt, mfma):
    """(results, bounds) in float64; `mfma`: probabilities and score gradients are rounded to bf16 on their way."""
    q, k, v, do = (t.double() for t in (q, k, v, do))
    group = q.shape[1] // k.shape[1]
    d = q.shape[2]
    u, uo = (unit(dt) if mfma else 0.0), unit(dt)
    names = ("o", "lse", "dq", "dk", "dv")
    out = dict(zip(names, (torch.zeros_like(q), torch.full((q.shape[1], q.shape[0]), -math.inf, dtype=torch.float64, device="cuda"), torch.zeros_like(q),
                           torch.zeros_like(k), torch.zeros_like(v))))
    err = {n: torch.zeros_like(t) for n, t in out.items()}
    q0 = k0 = 0
    for a, b in zip(lq, lk):
        seen = torch.ones(a, b, dtype=torch.bool, device="cuda")
        if causal:
            seen = seen.tril(b - a)
        for h in range(q.shape[1]):
            qs, gs, ks, vs = q[q0:q0 + a, h], do[q0:q0 + a, h], k[k0:k0 + b, h // group], v[k0:k0 + b, h // group]
            if a == 0 or b == 0:
                continue
            z = (qs @ ks.t() * scale).masked_fill(~seen, -math.inf)
            lse = torch.logsumexp(z, -1, keepdim=True)
            some = lse > -math.inf
            p = torch.where(some, (z - lse.where(some, torch.zeros_like(lse))).exp(), 0.0)
            ez = E32 * (d + 16) * (qs.abs() @ ks.abs().t()) * abs(scale) + 8 * E32 * (1 + z.where(seen, 0.0).abs())
            ez = ez.where(seen, 0.0)
            ep = p * (2 * ez + 2 * (p * ez).sum(-1, keepdim=True) + E32 * (b + 16))      # a probability's error in 32 bits
            o = p @ vs
            eo = (ep + u * p) @ vs.abs() + E32 * (b + 16) * (p @ vs.abs())
            dp = gs @ vs.t()
            delta = (gs * o).sum(-1, keepdim=True)
            edp = E32 * (d + 16) * (gs.abs() @ vs.abs().t() + (gs.abs() * o.abs()).sum(-1, keepdim=True)) + (gs.abs() * (eo + uo * o.abs())).sum(-1, keepdim=True)
            dz = p * (dp - delta)
            edz = ep * (dp - delta).abs() + p * edp + u * dz.abs() * 1.01 + u * p * edp
            s = slice(q0, q0 + a), slice(k0, k0 + b)
            out["o"][s[0], h], err["o"][s[0], h] = o, eo
            out["lse"][h, s[0]], err["lse"][h, s[0]] = lse[:, 0], 2 * ez.amax(-1) + E32 * (b + 16) + 2 * E32 * lse[:, 0].where(some[:, 0], 0.0).abs()
            n = E32 * (group * a + b + 32)
            sc = abs(scale)
            out["dq"][s[0], h] = dz @ ks * scale
            err["dq"][s[0], h] = (edz + n * dz.abs()) @ ks.abs() * sc
            out["dk"][s[1], h // group] += dz.t() @ qs * scale
            err["dk"][s[1], h // group] += (edz + n * dz.abs()).t() @ qs.abs() * sc
            out["dv"][s[1], h // group] += p.t() @ gs
            err["dv"][s[1], h // group] += (ep + (u + n) * p).t() @ gs.abs()
        q0, k0 = q0 + a, k0 + b
    for n in ("o", "dq", "dk", "dv"):
        err[n] += uo * (out[n].abs() + err[n])
    return out, err


def offsets(lens):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")


CASES = [
    # lengths of queries, of keys (None: the same), heads, KV heads, head size
    ([1], None, 1, 1, 64), ([5], None, 4, 2, 64), ([64], None, 2, 1, 128), ([65, 1, 31], None, 4, 4, 128), ([129], None, 8, 1, 128),
    ([200, 0, 333], None, 6, 2, 128), ([16, 17, 15, 127, 128], None, 2, 2, 64), ([257], None, 3, 1, 80), ([40, 3], None, 2, 1, 7),
    ([1, 1, 1], [300, 1, 64], 8, 2, 128), ([7, 130], [500, 131], 4, 2, 128), ([3, 20], [0, 5], 2, 1, 64), ([90, 40], [30, 40], 4, 2, 128),
    ([0, 0], [5, 6], 2, 2, 64), ([33], [700], 16, 2, 96), ([520], None, 2, 2, 128),
]


@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_attention(case, causal, dt):
    lq, lk, nq, nk, d = CASES[case]
    lk = lk or lq
    g = gen(case)
    q, kv, do = randn(g, sum(lq), nq, d, dt=dt, std=1.5), randn(g, sum(lk), 2 * nk + 1, d, dt=dt), randn(g, sum(lq), nq, d, dt=dt)
    k, v = kv[:, :nk], kv[:, nk:2 * nk]
    cq, ck = offsets(lq), offsets(lk)
    scale = None if case % 2 else 0.2
    o, lse = ops.attention_forward(q, k, v, cq, ck, causal=causal, scale=scale)
    dq, dk, dv = ops.attention_backward(do, q, k, v, o, lse, cq, ck, causal=causal, scale=scale)
    want, err = attention_reference(q, k, v, do, lq, lk, causal, d ** -0.5 if scale is None else scale, dt, True)
    for name, got in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        within(name, got, want[name], err[name])


@pytest.mark.parametrize("dt,lq,lk,nq,nk,d", [
    (BF, [4111], None, 16, 16, 128), (BF, [4111], None, 16, 16, 64), (BF, [3000, 1301], [3501, 1000], 16, 16, 128),
    (FP, [40, 3, 77] * 12, None, 16, 16, 64), (FP, [33, 90] * 14, [50, 64] * 14, 16, 16, 128), (BF, [40] * 30, None, 16, 16, 33)])
def test_attention_where_whole_tiles_fill_the_chip(dt, lq, lk, nq, nk, d):
    # many keys of few sequences (dk and dv by 128 keys), and rows enough that no tile is split over waves
    lk = lk or lq
    g = gen(sum(lq))
    q, k, v, do = randn(g, sum(lq), nq, d, dt=dt), randn(g, sum(lk), nk, d, dt=dt), randn(g, sum(lk), nk, d, dt=dt), randn(g, sum(lq), nq, d, dt=dt)
    cq, ck = offsets(lq), offsets(lk)
    o, lse = ops.attention_forward(q, k, v, cq, ck)
    dq, dk, dv = ops.attention_backward(do, q, k, v, o, lse, cq, ck)
    want, err = attention_reference(q, k, v, do, lq, lk, True, d ** -0.5, dt, True)
    for name, got in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        within(name, got, want[name], err[name])


@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("n", [2, 63, 64, 65, 130])
def test_attention_of_many_sequences(dt, n):
    lq = [(7 * i * i + 3 * i) % 41 * (i % 5 != 2) + 150 * (i % 29 == 11) for i in range(n)]
    lk = [a + 37 * (i % 3 == 1) - (a > 20 and i % 7 == 3) * 15 for i, a in enumerate(lq)]
    nq, nk, d = 2, 1, 64
    g = gen(n)
    q, do = randn(g, sum(lq), nq, d, dt=dt), randn(g, sum(lq), nq, d, dt=dt)
    k, v = randn(g, sum(lk), nk, d, dt=dt), randn(g, sum(lk), nk, d, dt=dt)
    cq, ck = offsets(lq), offsets(lk)
    o, lse = ops.attention_forward(q, k, v, cq, ck)
    dq, dk, dv = ops.attention_backward(do, q, k, v, o, lse, cq, ck)
    want, err = attention_reference(q, k, v, do, lq, lk, True, d ** -0.5, dt, True)
    for name, got in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        within(name, got, want[name], err[name])


@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lq,lk,nq,nk,d", [([1100], None, 8, 1, 128), ([700, 0, 90, 333], None, 16, 2, 64), ([400, 260], [20, 900], 12, 1, 40),
                                           ([513], None, 16, 1, 7)])
def test_attention_of_few_kv_heads(dt, causal, lq, lk, nq, nk, d):
    lk = lk or lq
    g = gen(sum(lq) + d)
    q, do = randn(g, sum(lq), nq, d, dt=dt), randn(g, sum(lq), nq, d, dt=dt)
    k, v = randn(g, sum(lk), nk, d, dt=dt), randn(g, sum(lk), nk, d, dt=dt)
    cq, ck = offsets(lq), offsets(lk)
    o, lse = ops.attention_forward(q, k, v, cq, ck, causal=causal)
    dq, dk, dv = ops.attention_backward(do, q, k, v, o, lse, cq, ck, causal=causal)
    want, err = attention_reference(q, k, v, do, lq, lk, causal, d ** -0.5, dt, True)
    for name, got in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        within(name, got, want[name], err[name])


@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("causal,d", [(True, 128), (False, 64)])
def test_attention_with_a_negative_scale(dt, causal, d):
    lens, nq, nk = [150, 3, 260], 4, 2
    g = gen(17)
    q, do = randn(g, sum(lens), nq, d, dt=dt), randn(g, sum(lens), nq, d, dt=dt)
    k, v = randn(g, sum(lens), nk, d, dt=dt), randn(g, sum(lens), nk, d, dt=dt)
    cu = offsets(lens)
    o, lse = ops.attention_forward(q, k, v, cu, cu, causal=causal, scale=-0.3)
    dq, dk, dv = ops.attention_backward(do, q, k, v, o, lse, cu, cu, causal=causal, scale=-0.3)
    want, err = attention_reference(q, k, v, do, lens, lens, causal, -0.3, dt, True)
    for name, got in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
        within(name, got, want[name], err[name])


@pytest.mark.parametrize("dt", [BF, FP])
def test_attention_of_views_and_large_scores(dt):
    g = gen(3)
    lens = [70, 5, 200]
    n = sum(lens)
    fused = randn(g, n, 4 + 2 + 2, 128, dt=dt)
    heads_first = randn(g, 4, n, 128, dt=dt)
    heads_first.copy_(fused[:, :4].transpose(0, 1))
    k, v, do = fused[:, 4:6], fused[:, 6:], randn(g, n, 4, 128, dt=dt)
    odd = torch.empty(n * 8 * 128 + 3, dtype=dt, device="cuda")[3:].view(n, 8, 128)
    odd.copy_(fused)
    cu = offsets(lens)
    want, err = attention_reference(fused[:, :4], k, v, do, lens, lens, True, 2.0, dt, True)      # scores of some hundreds
    for q, kk, vv in ((fused[:, :4], k, v), (heads_first.transpose(0, 1), k, v), (odd[:, :4], odd[:, 4:6], odd[:, 6:])):
        o, lse = ops.attention_forward(q, kk, vv, cu, cu, scale=2.0)
        dq, dk, dv = ops.attention_backward(do, q, kk, vv, o, lse, cu, cu, scale=2.0)
        for name, got in (("o", o), ("lse", lse), ("dq", dq), ("dk", dk), ("dv", dv)):
            within(name, got, want[name], err[name])
    # one value for all heads: a broadcast view
    o, _ = ops.attention_forward(fused[:, :4], k, v[:, :1].expand(n, 2, 128), cu, cu)
    p, _ = ops.attention_forward(fused[:, :4], k, v[:, :1].expand(n, 2, 128).contiguous(), cu, cu)
    assert torch.equal(o, p)


@pytest.mark.parametrize("dt", [BF, FP])
def test_attention_keeps_sequences_apart(dt):
    # what is no number in one sequence, and in the keys that a tile reads beyond the end of another, stays there
    g = gen(9)
    lens = [50, 33, 130]
    n = sum(lens)
    q, k, v, do = (randn(g, n, 2, 128, dt=dt) for _ in range(4))
    cu = offsets(lens)
    clean = ops.attention_forward(q, k, v, cu, cu)
    grads = ops.attention_backward(do, q, k, v, *clean, cu, cu)
    for t, bad in ((q, math.nan), (k, math.inf), (v, math.nan), (do, -math.inf)):
        t[50:83] = bad
    o, lse = ops.attention_forward(q, k, v, cu, cu)
    dirty = ops.attention_backward(do, q, k, v, o, lse, cu, cu)
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[50:83] = False
    assert torch.equal(o[keep], clean[0][keep]) and torch.equal(lse[:, keep], clean[1][:, keep]) and o[~keep].isnan().all()
    for a, b in zip(dirty, grads):
        assert torch.equal(a[keep], b[keep])


def test_attention_tokens_of_no_sequence_are_left_out():
    g = gen(11)
    q, k, v, do = (randn(g, 100, 2, 64, dt=BF) for _ in range(4))
    cu = torch.tensor([10, 40, 90], dtype=torch.int32, device="cuda")
    o, lse = ops.attention_forward(q, k, v, cu, cu)
    got = ops.attention_backward(do, q, k, v, o, lse, cu, cu)
    cut = [t[10:90].contiguous() for t in (q, k, v, do)]
    c2 = cu - 10
    o2, lse2 = ops.attention_forward(*cut[:3], c2, c2)
    want = ops.attention_backward(cut[3], *cut[:3], o2, lse2, c2, c2)
    assert torch.equal(o[10:90], o2) and torch.equal(lse[:, 10:90], lse2)
    for a, b in zip(got, want):
        assert torch.equal(a[10:90], b)


def _dirty():
    """Memory that the allocator gives out next holds NaN."""
    hold = [torch.full((n,), math.nan, device="cuda") for n in [1 << k for k in range(7, 25)] * 3]
    del hold


@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lq,lk,lead,tail,nq,nk,d", [
    # lengths; tokens of no sequence before the first and behind the last one, of the queries and of the keys
    ([30, 50], None, (10, 10), (10, 10), 2, 2, 64), ([30, 50], [45, 60], (0, 7), (300, 0), 4, 2, 40), ([1, 70], None, (1, 1), (0, 129), 2, 1, 33),
    ([1100], None, (3, 3), (200, 200), 8, 1, 128), ([0, 0], [0, 0], (2, 0), (3, 90), 4, 2, 128), ([40], [0], (0, 0), (0, 5), 2, 2, 64),
    ([0], [40], (700, 0), (0, 1), 2, 2, 64), ([4100], None, (0, 0), (150, 150), 16, 16, 64), ([40, 3, 77] * 12, None, (5, 70), (70, 5), 16, 16, 64)])
def test_attention_of_tokens_outside_all_sequences_is_nothing(lq, lk, lead, tail, nq, nk, d, causal, dt):
    lk = lk or lq
    g = gen(sum(lq) + d)
    tq, tk = lead[0] + sum(lq) + tail[0], lead[1] + sum(lk) + tail[1]
    iq, ik = slice(lead[0], lead[0] + sum(lq)), slice(lead[1], lead[1] + sum(lk))
    q, k, v, do = (randn(g, n, h, d, dt=dt) for n, h in ((tq, nq), (tk, nk), (tk, nk), (tq, nq)))
    want, err = attention_reference(q[iq], k[ik], v[ik], do[iq], lq, lk, causal, d ** -0.5, dt, True)
    for t, inside in ((q, iq), (k, ik), (v, ik), (do, iq)):      # nothing outside is looked at
        t[:inside.start], t[inside.stop:] = math.nan, math.nan
    cq, ck = offsets(lq) + lead[0], offsets(lk) + lead[1]
    _dirty()
    o, lse = ops.attention_forward(q, k, v, cq, ck, causal=causal)
    dq, dk, dv = ops.attention_backward(do, q, k, v, o, lse, cq, ck, causal=causal)
    for name, got, inside, none in (("o", o, iq, 0.0), ("lse", lse.t(), iq, -math.inf), ("dq", dq, iq, 0.0), ("dk", dk, ik, 0.0), ("dv", dv, ik, 0.0)):
        to = (lambda x: x.t()) if name == "lse" else (lambda x: x)
        assert (got[:inside.start] == none).all() and (got[inside.stop:] == none).all(), name
        within(name, to(got[inside]), want[name], err[name])


@pytest.mark.parametrize("dt", [BF, FP])
def test_gradients_of_a_padded_batch_reach_the_projections_whole(dt):
    g = gen(12)
    x, w = randn(g, 120, 96, dt=dt), (randn(g, 6 * 64, 96, dt=dt, std=0.1)).requires_grad_()
    cu = torch.tensor([0, 30, 83], dtype=torch.int32, device="cuda")
    grads = []
    for n in (120, 83):      # with padding behind the sequences, and without
        q, k, v = (x @ w.t())[:n].view(n, 6, 64).split([4, 1, 1], 1)
        _dirty()
        o = ops.attention(q, k, v, cu, cu)
        w.grad = None
        o[:83].float().square().sum().backward()
        grads.append(w.grad)
    assert torch.equal(*grads) and grads[0].any()


# ---- log-probs -----------------------------------------------------------------------------------------------------
def logprob_reference(h, w, y, g, temperature, dt):
    kept = y >= 0
    x, w64 = h.double()[kept], w.double()
    n = h.shape[1]
    z = x @ w64.t() / temperature
    lse = torch.logsumexp(z, -1)
    lp = z.gather(1, y[kept].long()[:, None])[:, 0] - lse
    ez = E32 * (n + 16) * (x.abs() @ w64.abs().t()) / temperature + 4 * E32 * z.abs()
    e_lse = ez.amax(-1) + E32 * (w.shape[0] + 64) + 4 * E32 * lse.abs()
    rows = torch.zeros(h.shape[0], dtype=torch.float64, device="cuda")
    full = lambda t: rows.masked_scatter(kept, t)  # noqa: E731
    out = dict(logp=(full(lp), full(e_lse + ez.amax(-1))), lse=(full(lse), full(e_lse)))
    if g is None:
        return out
    gk = g.double()[kept][:, None] / temperature
    p = (z - lse[:, None]).exp()
    dz = -gk * p
    dz.scatter_add_(1, y[kept].long()[:, None], gk)
    u = unit(dt)
    edz = gk.abs() * p * (2 * ez + 2 * e_lse[:, None] + 8 * E32) + (u + 4 * E32) * dz.abs()
    dh, dw = torch.zeros_like(h, dtype=torch.float64), dz.t() @ x
    edh = torch.zeros_like(dh)
    dh[kept] = dz @ w64
    edh[kept] = (edz * (1 + u) + E32 * (w.shape[0] + 64) * dz.abs()) @ w64.abs()
    edw = (edz * (1 + u) + E32 * (h.shape[0] + 64) * dz.abs()).t() @ x.abs()
    out["dh"] = (dh, edh + u * (dh.abs() + edh))
    out["dw"] = (dw, edw + u * (dw.abs() + edw))
    return out


@pytest.mark.parametrize("dt", [BF, FP])
@pytest.mark.parametrize("rows,hidden,vocab,sampled", [
    (1, 8, 2, 1.0), (1, 256, 4096, 1.0), (3, 64, 1, 1.0), (72, 256, 4096, 0.6), (130, 512, 1000, 0.5), (300, 136, 5001, 0.9), (257, 1024, 8192, 1.0),
    (64, 2560, 3001, 0.3), (520, 640, 2048, 1.0), (33, 100, 777, 0.7), (20, 7, 50, 0.5), (1100, 64, 600, 0.97)])
def test_token_logprobs(rows, hidden, vocab, sampled, dt):
    g = gen(rows + hidden + vocab)
    w = randn(g, vocab, hidden, dt=dt, std=2 / math.sqrt(hidden))
    y = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    h = (torch.randn(rows, hidden, generator=g, device="cuda") + 1.5 * w[y.long()].float()).to(dt)
    y[torch.rand(rows, generator=g, device="cuda") >= sampled] = -1
    dlogp = randn(g, rows)
    dlogp[::5] = 0.0
    temperature = 1.0 if rows % 2 else 0.7
    logp, lse = ops.token_logprobs_forward(h, w, y, temperature)
    dh, dw = ops.token_logprobs_backward(dlogp, h, w, y, lse, temperature)
    ref = logprob_reference(h, w, y, dlogp, temperature, dt)
    for name, got in (("logp", logp), ("lse", lse), ("dh", dh), ("dw", dw)):
        within(name, got, *ref[name])
    assert not dh[(y < 0) | (dlogp == 0)].any()


@pytest.mark.parametrize("dt,rows,hidden,vocab", [(BF, 300, 64, 160_000), (BF, 90, 8, 150_001), (FP, 300, 64, 20_001), (FP, 700, 8, 40_003),
                                                  (FP, 40, 4, 70_000)])
def test_token_logprobs_of_many_tiles_a_workgroup(dt, rows, hidden, vocab):
    _check_token_logprobs(dt, rows, hidden, vocab)


# many slices of the vocabulary in the gradient of the hidden rows, whole tiles and those of few rows; tiles of 128 in every product
@pytest.mark.parametrize("rows,hidden,vocab", [(700, 72, 140_000), (90, 776, 135_000), (260, 264, 30_011)])
def test_token_logprobs_of_large_vocabularies(rows, hidden, vocab):
    _check_token_logprobs(BF, rows, hidden, vocab)


# The columns of dz go on to a multiple of 256: a tile can begin behind the vocabulary, at 60032 of 60000 and at 20096 of 20001 in tiles of
# 128 columns, at 20032 of 20001 in tiles of 64.
@pytest.mark.parametrize("dt,rows,hidden,vocab", [(BF, 260, 512, 20_001), (FP, 60, 512, 20_001), (FP, 300, 4096, 60_000)])
def test_token_logprobs_where_a_tile_begins_behind_the_vocabulary(dt, rows, hidden, vocab):
    assert debug_token_logprob_loads(rows, rows - len(range(0, rows, 7)), hidden, vocab, dt == BF, True) == (0, 0, 0)
    _check_token_logprobs(dt, rows, hidden, vocab)


def _check_token_logprobs(dt, rows, hidden, vocab):
    g = gen(rows + vocab)
    w, h = randn(g, vocab, hidden, dt=dt, std=2 / math.sqrt(hidden)), randn(g, rows, hidden, dt=dt)
    y = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    y[::7] = -1
    y[1], y[2] = 0, vocab - 1
    dlogp = randn(g, rows)
    logp, lse = ops.token_logprobs_forward(h, w, y, 0.7)
    dh, dw = ops.token_logprobs_backward(dlogp, h, w, y, lse, 0.7)
    ref = logprob_reference(h, w, y, dlogp, 0.7, dt)
    for name, got in (("logp", logp), ("lse", lse), ("dh", dh), ("dw", dw)):
        within(name, got, *ref[name])


@pytest.mark.parametrize("rows,hidden,vocab", [(1, 64, 1000), (17, 1024, 4096), (63, 100, 30_000), (64, 768, 140_000)])
def test_token_logprobs_of_few_rows_are_rounded_once(rows, hidden, vocab):
    # up to 64 rows: the gradient of the logits keeps 16 bits on its way, so the bound of 32 bits holds but for u^2 of it, and one rounding
    g = gen(rows + hidden)
    w = randn(g, vocab, hidden, dt=BF, std=2 / math.sqrt(hidden))
    y = torch.randint(0, vocab, (rows,), generator=g, device="cuda", dtype=torch.int32)
    y[5::6] = -1
    h = (torch.randn(rows, hidden, generator=g, device="cuda") + w[y.long()].float()).to(BF)
    dlogp, u = randn(g, rows), unit(BF)
    logp, lse = ops.token_logprobs_forward(h, w, y, 1.3)
    got = dict(zip(("dh", "dw"), ops.token_logprobs_backward(dlogp, h, w, y, lse, 1.3)))
    ref = logprob_reference(h, w, y, dlogp, 1.3, FP)
    gk = torch.where(y >= 0, dlogp.double(), 0.0)[:, None] / 1.3
    dz = gk.abs() * (h.double() @ w.double().t() / 1.3 - lse.double()[:, None]).exp()
    dz.scatter_add_(1, y.clamp(min=0).long()[:, None], gk.abs())
    left = {"dh": dz @ w.double().abs(), "dw": dz.t() @ h.double().abs()}
    for name in ("dh", "dw"):
        want, err = ref[name]
        err = err + u * u * left[name]
        within(name, got[name], want, err + u * (want.abs() + err))


@pytest.mark.parametrize("dt", [BF, FP])
def test_token_logprobs_over_several_pieces_of_the_vocabulary(dt):
    # pieces hold at least 1024 tokens: rows enough that the budget of a piece stays at that, few of them with a target
    g = gen(2)
    rows, hidden, vocab = (70_000 if dt == FP else 140_000), 64, 5000
    w, h = randn(g, vocab, hidden, dt=dt, std=0.25), randn(g, rows, hidden, dt=dt)
    y = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    at = torch.randperm(rows, generator=g, device="cuda")[:400]
    y[at] = torch.randint(0, vocab, (400,), generator=g, device="cuda", dtype=torch.int32)
    dlogp = randn(g, rows)
    logp, lse = ops.token_logprobs_forward(h, w, y)
    dh, dw = ops.token_logprobs_backward(dlogp, h, w, y, lse)
    ref = logprob_reference(h, w, y, dlogp, 1.0, dt)
    for name, got in (("logp", logp), ("lse", lse), ("dh", dh), ("dw", dw)):
        within(name, got, *ref[name])


@pytest.mark.parametrize("dt", [BF, FP])
def test_token_logprobs_of_strided_rows_and_odd_targets(dt):
    g = gen(4)
    w, wide = randn(g, 700, 72, dt=dt, std=0.2), randn(g, 40, 3, 72, dt=dt)
    y = torch.randint(0, 700, (40,), generator=g, device="cuda", dtype=torch.int32)
    h, dlogp = wide[:, 1], randn(g, 40)
    logp, lse = ops.token_logprobs_forward(h, w, y)
    got = ops.token_logprobs_backward(dlogp, h, w, y, lse)
    assert torch.equal(logp, ops.token_logprobs_forward(h.contiguous(), w, y)[0])
    ref = logprob_reference(h, w, y, dlogp, 1.0, dt)
    for name, t in (("logp", logp), ("dh", got[0]), ("dw", got[1])):
        within(name, t, *ref[name])
    none = torch.full_like(y, -1)
    logp, lse = ops.token_logprobs_forward(h, w, none)
    dh, dw = ops.token_logprobs_backward(dlogp, h, w, none, lse)
    assert not logp.any() and not dh.any() and not dw.any()
    odd = y.clone()
    odd[7], odd[8] = 700, 2**31 - 1
    logp, lse = ops.token_logprobs_forward(h, w, odd)
    dh, _ = ops.token_logprobs_backward(dlogp, h, w, odd, lse)
    assert logp[7:9].isnan().all() and dh[7:9].isnan().all() and logp.isnan().sum() == 2 and dh.isnan().any(1).sum() == 2
    dh, dw = ops.token_logprobs_backward(dlogp[:0], h[:0], w, y[:0], lse[:0])
    assert dh.shape == (0, 72) and not dw.any() and ops.token_logprobs_forward(h[:0], w, y[:0])[0].shape == (0,)
    # a logit far above the others, rows of zeros
    h = torch.zeros(3, 72, dtype=dt, device="cuda")
    h[0] = w[5] * 400
    logp, _ = ops.token_logprobs_forward(h, w, torch.tensor([5, 6, 7], dtype=torch.int32, device="cuda"))
    assert logp[0].abs() < 1e-6 and torch.allclose(logp[1:], torch.full((2,), -math.log(700), device="cuda"), atol=1e-6)


# ---- gradients against differences, repetition, streams, graphs ------------------------------------------------------
def test_gradients_against_differences_of_the_formulas():
    # d/dt f(x + t v) at 0 by central differences in float64 against the kernels' gradients in fp32
    g = gen(21)
    lens = [5, 9]
    cu = offsets(lens)
    n, nq, nk, d, vocab = sum(lens), 4, 2, 16, 50
    table = ops.rotary_table(20, d)
    pos = torch.arange(n, device="cuda", dtype=torch.int32)
    y = torch.randint(0, vocab, (n,), generator=g, device="cuda", dtype=torch.int32)
    y[3] = -1
    c = torch.randn(n, generator=g, device="cuda")
    x = [randn(g, n, nq, d), randn(g, n, nk, d), randn(g, n, nk, d), randn(g, d), randn(g, d), randn(g, vocab, nq * d, std=0.2)]

    def through_the_kernels(q, k, v, wn, b, w):
        q, k = ops.rotate(ops.norm(q, wn, b, centered=True), k, pos, table)
        o = ops.attention(q, k, v, cu, cu)
        return (ops.token_logprobs(o.flatten(1), w, y, 0.8) * c).sum()

    def in_64_bits(q, k, v, wn, b, w):
        mu = q.mean(-1, keepdim=True)
        q = (q - mu) / ((q - mu).square().mean(-1, keepdim=True) + 1e-6).sqrt() * wn + b
        q, k = (rotary_reference(t, table[pos.long()], False, 1)[0] for t in (q, k))
        want, _ = attention_reference(q, k, v, torch.zeros_like(q), lens, lens, True, d ** -0.5, FP, False)
        return (logprob_reference(want["o"].flatten(1), w, y, None, 0.8, FP)["logp"][0] * c.double()).sum()

    leaves = [t.clone().requires_grad_() for t in x]
    value = through_the_kernels(*leaves)
    value.backward()
    x64 = [t.double() for t in x]
    assert abs(value.item() - in_64_bits(*x64).item()) < 1e-4
    for i in range(len(x)):
        v = torch.randn(x[i].shape, generator=g, device="cuda", dtype=torch.float64)
        h = 1e-5
        plus, minus = ([t + (s * h * v if j == i else 0) for j, t in enumerate(x64)] for s in (1, -1))
        slope = ((in_64_bits(*plus) - in_64_bits(*minus)) / (2 * h)).item()
        got = (leaves[i].grad.double() * v).sum().item()
        # differences: h^2 times third derivatives and 1e-16 / h; gradients: fp32 over sums of some hundred terms
        size = (leaves[i].grad.double() * v).abs().sum().item()
        assert abs(got - slope) < 2e-5 * size + 1e-6, (i, got, slope)


def _everything(dt, seed):
    g = gen(seed)
    n = 300
    lens = [120, 1, 179]
    cu = offsets(lens)
    q, k, v, do = randn(g, n, 8, 128, dt=dt), randn(g, n, 2, 128, dt=dt), randn(g, n, 2, 128, dt=dt), randn(g, n, 8, 128, dt=dt)
    wn, b = randn(g, 128, dt=dt), randn(g, 128, dt=dt)
    table = ops.rotary_table(400, 128)
    pos = torch.arange(n, device="cuda", dtype=torch.int32)
    h, w = randn(g, n, 256, dt=dt), randn(g, 3000, 256, dt=dt, std=0.1)
    y = torch.randint(-200, 3000, (n,), generator=g, device="cuda", dtype=torch.int32)
    dlogp = randn(g, n)

    def run():
        o, lse = ops.attention_forward(q, k, v, cu, cu)
        out = [o, lse, *ops.attention_backward(do, q, k, v, o, lse, cu, cu), *ops.rotary(q, k, pos, table)]
        yn, mean, rstd = ops.norm_forward(q, wn, b, centered=True)
        out += [yn, *ops.norm_backward(do, q, wn, mean, rstd, centered=True)]
        logp, l = ops.token_logprobs_forward(h, w, y)
        return out + [logp, l, *ops.token_logprobs_backward(dlogp, h, w, y, l)]
    return run


@pytest.mark.parametrize("dt", [BF, FP])
def test_the_same_bits_again_on_another_stream_and_in_a_graph(dt):
    run = _everything(dt, 31)
    first = [t.clone() for t in run()]
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, run()))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        second = run()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(first, second))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = run()
    for _ in range(3):
        for t in captured:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, captured))
        assert all(torch.equal(a, b) for a, b in zip(first, run()))


# ---- more than a launch takes ---------------------------------------------------------------------------------------
# (fewer than 2^32 threads along a grid's first dimension; a launch of more runs some of them and reports no error)
def test_norm_of_more_rows_than_a_launch_takes():
    rows, width = (1 << 26) + 5, 33      # four rows a workgroup of 256
    x = torch.empty(rows, width, dtype=BF, device="cuda").normal_(generator=gen(41))
    w, b = randn(gen(42), width, dt=BF), randn(gen(43), width, dt=BF)
    y, mean, rstd = ops.norm_forward(x, w, b, centered=True)
    for at in (0, (1 << 25) - 3, (1 << 26) - 3, rows - 8):
        part = ops.norm_forward(x[at:at + 8], w, b, centered=True)
        assert all(torch.equal(a[at:at + 8], c) for a, c in zip((y, mean, rstd), part)), at


def test_rotary_of_more_tokens_than_a_launch_takes():
    tokens, d = (1 << 24) + 5, 257       # a workgroup of 256 a token
    x = torch.empty(tokens, 1, d, dtype=BF, device="cuda").normal_(generator=gen(44))
    table = ops.rotary_table(1000, 2)
    pos = torch.arange(tokens, device="cuda", dtype=torch.int32) % 1000
    places = [slice(at, at + 8) for at in (0, (1 << 23) - 3, (1 << 24) - 3, tokens - 8)]
    want = [ops.rotary(x[p].clone(), None, pos[p], table)[0] for p in places]
    ops.rotary(x, None, pos, table, q_out=x)
    for p, c in zip(places, want):
        assert torch.equal(x[p], c), p


def test_attention_of_more_sequences_than_one_grid_takes():
    n, nq, nk, d = 1 << 19, 32, 16, 8      # one token each: o = v, lse = scale q.k
    g = gen(45)
    q, k, v, do = randn(g, n, nq, d, dt=BF), randn(g, n, nk, d, dt=BF), randn(g, n, nk, d, dt=BF), randn(g, n, nq, d, dt=BF)
    cu = torch.arange(n + 1, device="cuda", dtype=torch.int32)
    o, lse = ops.attention_forward(q, k, v, cu, cu, scale=0.5)
    assert torch.equal(o.view(n, nk, 2, d), v[:, :, None].expand(n, nk, 2, d))
    assert torch.allclose(lse.t().view(n, nk, 2), 0.5 * (q.view(n, nk, 2, d).float() * k[:, :, None].float()).sum(-1), atol=1e-4, rtol=1e-5)
    dq, dk, dv = ops.attention_backward(do, q, k, v, o, lse, cu, cu, scale=0.5)
    # zero but for what 32 bits leave of dp - delta: 40 roundings of 8 products of values up to 6, times scale, key or queries
    assert dq.abs().max() < 0.01 and dk.abs().max() < 0.01
    assert torch.allclose(dv.float(), do.view(n, nk, 2, d).float().sum(2), atol=1e-3, rtol=2.0 ** -7)


# ---- refusals ------------------------------------------------------------------------------------------------------
def test_refusals():
    x, w = torch.ones(4, 2, 8, device="cuda"), torch.ones(8, device="cuda")
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    cu, table, pos = i32(0, 4), ops.rotary_table(5, 8), i32(0, 1, 2, 3)
    _, mean, rstd = ops.norm_forward(x, w, centered=True)
    h, wt, y = torch.ones(4, 8, device="cuda"), torch.ones(9, 8, device="cuda"), i32(0, 1, 2, 3)
    o, lse = ops.attention_forward(x, x, x, cu, cu)
    calls = [
        lambda: ops.norm_forward(x.half(), w.half()), lambda: ops.norm_forward(x.cpu(), w.cpu()), lambda: ops.norm_forward(x, w.to(BF)),
        lambda: ops.norm_forward(x, w[:4]), lambda: ops.norm_forward(x, w, eps=-1.0), lambda: ops.norm_forward(x, w, w[:3]),
        lambda: ops.norm_backward(x[:2], x, w, mean, rstd), lambda: ops.norm_backward(x, x, w, mean, rstd[:2]),
        lambda: ops.norm_backward(x, x, w, mean.double(), rstd, centered=True),
        lambda: ops.rotary(x, None, pos.long(), table), lambda: ops.rotary(x, None, pos[:3], table), lambda: ops.rotary(x, x[:2], pos, table),
        lambda: ops.rotary(x[..., :6], None, pos, table), lambda: ops.rotary(x, None, pos, table, q_out=x[:, :1]), lambda: ops.rotary_table(4, 3),
        lambda: ops.attention_forward(x, x[:, :1].expand(4, 3, 8), x[:, :1].expand(4, 3, 8), cu, cu), lambda: ops.attention_forward(x, x, x, cu, i32(0, 2, 4)),
        lambda: ops.attention_forward(x, x, x, cu.long(), cu), lambda: ops.attention_forward(x, x, x, cu, cu, scale=math.inf),
        lambda: ops.attention_forward(x, x, x, i32(0), i32(0)), lambda: ops.attention_forward(*(3 * [torch.ones(4, 2, 136, device="cuda")]), cu, cu),
        lambda: ops.attention_backward(x[:2], x, x, x, o, lse, cu, cu), lambda: ops.attention_backward(x, x, x, x, o, lse.t(), cu, cu),
        lambda: ops.token_logprobs_forward(h, wt, y, 0.0), lambda: ops.token_logprobs_forward(h, wt, y, math.nan), lambda: ops.token_logprobs_forward(h, wt[:, :4], y),
        lambda: ops.token_logprobs_forward(h, wt, y.long()), lambda: ops.token_logprobs_forward(h, wt.t().contiguous().t(), y),
        lambda: ops.token_logprobs_backward(h[:, 0].double(), h, wt, y, h[:, 0].contiguous()),
    ]
    for i, call in enumerate(calls):
        with pytest.raises(RolloutError):
            call()
            pytest.fail(f"call {i} was not refused")
