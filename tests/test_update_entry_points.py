"""CPU-side checks of the C entry points of linear layers, residual stream and orthogonalised updates: what they refuse before anything touches a GPU, workspace
sizes, and what the loads of their products reach."""
import ctypes as C
import math
import os
import random

import pytest

import paper_2509_06980_amd as rl

P = 0x1000          # stands for a device address: none of these calls gets as far as using it
F32, BF16 = 0, 1


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(rl.LIB_PATH):
        from paper_2509_06980_amd import build
        build.build()
    return rl.load_library()


def linear_forward(lib, x=P, rows=4, inner=8, w=P, up=0, outer=8, bias=0, up_bias=0, act=0, r=0, r_dtype=F32, dtype=F32, y=P, kept=0, ws=P, nbytes=1 << 40, stride=8):
    return lib.rl_linear_forward(x, stride, rows, inner, w, stride, up, stride, outer, bias, up_bias, act, r, 8, r_dtype, dtype, y, kept, ws, nbytes, None)


def linear_backward(lib, dy=P, dy_dtype=F32, x=P, rows=4, inner=8, w=P, up=0, outer=8, act=0, kept=0, dtype=F32, dx=P, dw=P, dup=0, db=0, dub=0, ws=P, nbytes=1 << 40):
    return lib.rl_linear_backward(dy, 8, dy_dtype, x, 8, rows, inner, w, 8, up, 8, outer, act, kept, dtype, dx, dw, dup, db, dub, ws, nbytes, None)


def residual_forward(lib, h=P, y=P, rows=4, width=8, w=P, b=0, pw=0, pb=0, gate=0, eps=1e-6, stream=F32, dtype=F32, out=P, a=P, stats=P):
    return lib.rl_residual_norm_forward(h, 8, y, 8, rows, width, w, b, pw, pb, gate, 0, 1, 1.0, 1.0, eps, 0, stream, dtype, out, a, stats, None)


def residual_backward(lib, dout=P, da=P, out=P, y=P, stats=P, rows=4, width=8, w=P, pw=0, pb=0, gate=0, stream=F32, dtype=F32, dh=P, dy=P, dw=P, db=0, dpw=0, dpb=0, dg=0,
                      columns=1, gate_rows=0, ws=P, nbytes=1 << 40):
    return lib.rl_residual_norm_backward(dout, 8, da, 8, out, 8, y, 8, stats, rows, width, w, pw, pb, gate, 0, columns, 1.0, 1.0, 0, stream, dtype, dh, dy, dw, db, dpw, dpb,
                                         dg, gate_rows, ws, nbytes, None)


def orthogonalize(lib, x=P, count=2, rows=8, columns=8, steps=1, c=(1.0, 2.0, 3.0), eps=1e-7, dtype=F32, out=P, ws=P, nbytes=1 << 40):
    table = (C.c_float * len(c))(*c) if c else None
    return lib.rl_orthogonalize(x, rows * columns, columns, count, rows, columns, steps, table, eps, dtype, out, ws, nbytes, None)


REFUSED = [
    (linear_forward, [dict(x=0), dict(w=0), dict(y=0), dict(up_bias=P), dict(rows=-1), dict(inner=0), dict(outer=0), dict(inner=1 << 20), dict(outer=1 << 20), dict(rows=(1 << 26) + 1),
                      dict(inner=1 << 16, outer=1 << 15), dict(act=-1), dict(act=5), dict(dtype=2), dict(dtype=-1), dict(r=P, r_dtype=BF16), dict(ws=P + 128), dict(ws=0, rows=200, stride=9),
                      dict(rows=200, nbytes=100, stride=9), dict(rows=200, inner=7, nbytes=100)]),
    (linear_backward, [dict(dy=0), dict(x=0), dict(w=0), dict(act=2), dict(up=P), dict(dup=P), dict(dub=P), dict(dy_dtype=BF16), dict(dtype=3), dict(rows=-1), dict(inner=0),
                       dict(ws=0), dict(ws=P + 8), dict(nbytes=1)]),
    (residual_forward, [dict(h=0), dict(y=0), dict(out=0), dict(a=0), dict(stats=0), dict(stats=P + 8), dict(rows=-1), dict(width=0), dict(width=(1 << 24) + 1), dict(rows=(1 << 24) + 1),
                        dict(eps=-1.0), dict(eps=math.nan), dict(dtype=2), dict(stream=BF16), dict(w=0, b=P), dict(pb=P)]),
    (residual_backward, [dict(dout=0, da=0), dict(out=0), dict(y=0), dict(stats=0), dict(w=0), dict(dw=0), dict(dh=0), dict(dy=0), dict(db=P, da=0), dict(pw=P), dict(pb=P), dict(dpb=P),
                         dict(dg=P), dict(gate=P, columns=0), dict(ws=0), dict(ws=P + 4), dict(nbytes=4 * 8 * 4 * 5 - 1), dict(dtype=2), dict(stream=BF16), dict(rows=-1)]),
    (orthogonalize, [dict(x=0), dict(out=0), dict(ws=0), dict(ws=P + 64), dict(nbytes=100), dict(count=-1), dict(count=65536), dict(rows=0), dict(columns=0), dict(rows=1 << 20),
                     dict(rows=1 << 15, columns=1 << 15), dict(steps=0), dict(steps=65), dict(c=()), dict(c=(1.0, math.inf, 0.0)), dict(c=(math.nan, 0.0, 0.0)), dict(eps=-1.0),
                     dict(eps=math.nan), dict(dtype=2)]),
]


@pytest.mark.parametrize("call,changes", REFUSED, ids=[c.__name__ for c, _ in REFUSED])
def test_bad_arguments_are_refused_with_a_message(lib, call, changes):
    for change in changes:
        assert call(lib, **change) == -1, (call.__name__, change)
        assert lib.rl_last_error(), change


def test_calls_without_rows_succeed_without_a_gpu(lib):
    assert linear_forward(lib, rows=0, x=0, y=0, ws=0, nbytes=0) == 0
    assert residual_forward(lib, rows=0, h=0, y=0, out=0) == 0
    assert orthogonalize(lib, count=0, x=0, out=0, ws=0, nbytes=0) == 0


def test_workspaces(lib):
    size = lib.rl_linear_workspace
    for bad in ((0, 8, 8, 0, 0, 0, 0), (4, 0, 8, 0, 0, 0, 0), (4, 8, 0, 0, 0, 1, 0), (4, 8, 8, 0, 2, 1, 0), (4, 1 << 16, 1 << 15, 0, 1, 0, 0)):
        assert size(*bad) == 0
    assert size(1, 4096, 2560, 0, BF16, 0, 1) == 0                         # nothing to copy, no slices
    assert size(4096, 2560, 9728, 0, BF16, 0, 0) >= 2 * (4096 + 9728) * 2560
    assert size(4096, 2560, 9728, 1, BF16, 1, 1) >= 2 * 2 * 4096 * 9728      # dz and du
    for gated in (0, 1):
        for dtype in (F32, BF16):
            for backward in (0, 1):
                for rows, inner, outer in ((1, 1, 1), (17, 100, 300), (4000, 2560, 9728)):
                    assert size(rows, inner, outer, gated, dtype, backward, 1) <= size(rows, inner, outer, gated, dtype, backward, 0)
    assert lib.rl_residual_norm_workspace(10, 100) == 10 * 100 * 4 * 5 and lib.rl_residual_norm_workspace(10, 0) == lib.rl_residual_norm_workspace(-1, 8) == 0
    assert lib.rl_residual_norm_workspace(1 << 20, 100) == lib.rl_residual_norm_workspace(1 << 24, 100) > 0      # shares, not rows
    # in bf16 X twice, what its rounding leaves, A and B
    n = lib.rl_orthogonalize_workspace(28, 2048, 1024, BF16)
    assert n >= 28 * (3 * 2048 * 1024 * 2 + 2 * 1024 * 1024 * 2) and lib.rl_orthogonalize_workspace(0, 8, 8, F32) == lib.rl_orthogonalize_workspace(1, 0, 8, F32) == 0


def test_operators_refuse_tensors_that_are_not_on_a_gpu(lib):
    import torch

    from paper_2509_06980_amd import policy_ops as ops
    x, w, v = torch.ones(4, 8), torch.ones(6, 8), torch.ones(8)
    for call in (lambda: ops.linear_forward(x, w), lambda: ops.linear_backward(torch.ones(4, 6), x, w), lambda: ops.residual_norm_forward(x, x, v),
                 lambda: ops.residual_norm_backward(x, x, x, x, torch.ones(4, 4), v), lambda: ops.orthogonalize(x), lambda: ops.orthogonalize(x, coefficients=(1.0, 2.0)),
                 lambda: ops.orthogonalize(x, coefficients=[(1.0, 2.0, 3.0)] * 4)):
        with pytest.raises(rl.RolloutError) as e:
            call()
        assert e.value.code == -1


def test_loads_of_the_products_stay_inside_their_operands(lib):
    rng = random.Random(11)

    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    cases = [(1, 1, 1, 0, 0, 0), (4096, 9728, 2560, 0, 0, 0), (2744, 2560, 9728, 0, 0, 0), (37, 2560, 9728, 0, 0, 0), (61, 257, 517, 0, 0, 0), (300_000, 9728, 2560, 0, 0, 0),
             (3_000_000, 1024, 4096, 8, 0, 0)]
    for _ in range(400):
        cases.append((log(1, 9000), rng.choice([8 * log(1, 1300), log(1, 9000)]), rng.choice([8 * log(1, 1300), log(1, 9000)]), rng.choice([0, 0, 8, 3, 128]),
                      rng.choice([0, 0, 8, 5, 64]), rng.choice([0, 0, 8, 1])))
    for rows, inner, outer, dx, dw, dy in cases:
        for gated in (False, True):
            for bf16 in (False, True):
                for backward in (False, True):
                    beyond, offsets, products = rl.debug_linear_loads(rows, inner, outer, inner + dx, inner + dw, outer + dy, gated, bf16, backward)
                    assert beyond <= 0 and offsets <= 0, (rows, inner, outer, dx, dw, dy, gated, bf16, backward)
                    assert products == (2 if backward else 1 if rows > 16 else 0)
    for _ in range(200):
        count, rows, columns = log(1, 40), log(1, 6000), log(1, 9000)
        for bf16 in (False, True):
            beyond, offsets, products = rl.debug_orthogonalize_loads(count, rows, columns, bf16)
            assert beyond <= 0 and offsets <= 0 and products == 3, (count, rows, columns, bf16)
    with pytest.raises(rl.RolloutError):
        rl.debug_linear_loads(0, 8, 8, 8, 8, 8, False, False, False)
    with pytest.raises(rl.RolloutError):
        rl.debug_orthogonalize_loads(0, 8, 8, False)


def test_states_of_muon_stay_in_32_bits_when_they_are_loaded():
    torch = pytest.importorskip("torch")
    from paper_2509_06980_amd.policy_update import Muon
    def stepped():
        p, q = (torch.ones(5, dtype=torch.bfloat16, requires_grad=True) for _ in range(2))
        return [p, q], Muon([dict(params=[p]), dict(params=[q])])
    params, muon = stepped()
    for k in range(3):
        for p in params[:1]:                      # the other one has no gradient and no state
            p.grad = torch.linspace(0.1, 0.7 + k, 5).bfloat16()
        muon.step()
    saved = muon.state_dict()
    again, other = stepped()
    other.load_state_dict(saved)
    state, loaded = muon.state[params[0]], other.state[again[0]]
    assert loaded["step"] == 3 and not other.state.get(again[1])
    for name in ("first", "second"):
        assert loaded[name].dtype == torch.float32 and torch.equal(loaded[name], state[name]) and loaded[name].data_ptr() != state[name].data_ptr()


@pytest.mark.parametrize("changes", [dict(coefficients=()), dict(coefficients=None), dict(coefficients={"a": 1.0}), dict(coefficients=(1.0, "b", 2.0)),
                                     dict(coefficients=[(1.0, 2.0, 3.0), (1.0,)], steps=2), dict(steps=0), dict(steps=10 ** 12), dict(steps=2.5)])
def test_steps_and_coefficients_that_are_none_are_refused(lib, changes):
    torch = pytest.importorskip("torch")
    from paper_2509_06980_amd import policy_ops as ops
    with pytest.raises(rl.RolloutError, match="coefficients") as e:
        ops.orthogonalize(torch.ones(4, 8), **changes)
    assert e.value.code == -1
