"""Orthogonalised updates in bf16 whose X is far from 1: |G| far below eps, coefficients that shrink or enlarge, steps that enlarge the smallest singular values;
against the same steps in float64."""
import pytest
import torch

from balls import E32
from paper_2509_06980_amd import policy_ops as ops
from test_update_operators import BF, gen, matrices, newton

pytestmark = pytest.mark.gpu
F16 = 2.0 ** -11      # half a step of fp16
# Steps in which B is nothing beside a: X as fp16 holds it in the last one, the remainders of those before (2^-22 each, at most five here), sums and scales in 32 bits
PLAIN = F16 + 5 * 2.0 ** -22 + 64 * E32


def off(got, want):
    return ((got.double() - want).norm() / want.norm()).item()


def last_rounding(want):
    """What rounding the exact result to bf16 leaves, relative; that of a result a little off is as large, but for 1 / sqrt(elements) < 0.2 % of chance."""
    return 1.01 * off(want.to(BF), want)


def sized(x, *sizes):
    return torch.stack([m / m.norm() * s for m, s in zip(x, sizes)]).to(BF)


@pytest.mark.parametrize("kind", ["noise", "strong"])
@pytest.mark.parametrize("rows,columns", [(256, 1024), (1000, 264), (640, 2304)])
@pytest.mark.parametrize("size,eps", [(7e-13, 1e-7), (7e-14, 1e-7), (7e-15, 1e-7), (1e-30, 1e-7), (7e-7, 1.0), (1e-20, 1e10)])
def test_updates_far_below_eps(rows, columns, size, eps, kind):
    # each by its own size: beside one of them, one whose eps does not count and one of zeros
    x = sized(matrices(gen(rows), 3, rows, columns, torch.float64, kind), size, 1000 * eps, 1)
    x[2] = 0
    got = ops.orthogonalize(x, eps=eps)
    want = newton(x[0], True, None, eps=eps, roundings=False)      # |X|^2 (|b| + |c|) stays below 1e-5 up to the last step: B's roundings, 2^-10 of it, are nothing
    assert off(got[0], want) < last_rounding(want) + PLAIN
    want = newton(x[1], True, None, eps=eps, roundings=False)
    assert off(got[1], want) < last_rounding(want) + 2 * off(newton(x[1], True, gen(2), eps=eps), want)      # twice the model's roundings
    assert not got[2].any()


@pytest.mark.parametrize("eps", [0.3, 3.0, 100.0])
def test_updates_about_as_large_as_eps(eps):
    for kind in ("noise", "strong"):
        x = sized(matrices(gen(7), 1, 300, 700, torch.float64, kind), 1.0)[0]
        want = newton(x, True, None, eps=eps, roundings=False)
        model = off(newton(x, True, gen(3), eps=eps), want)
        assert off(ops.orthogonalize(x, eps=eps), want) < last_rounding(want) + 2 * model + 1e-6, (kind, eps)


@pytest.mark.parametrize("coefficients", [[(0.01, 0.0, 0.0)] * 5, [(0.001, 0.0, 0.0)] * 3, [(1e-3, -5e-4, 0.0)] * 3, [(-1e-2, 0.0, 5e-3)] * 4, [(0.01, 0.0, 0.0)] * 64, [(500.0, 0.0, 0.0)] * 4,
                                          [(2.0, 0.0, 0.0)] * 64, [(1e-8, 0.0, 0.0), (1e8, 0.0, 0.0)], [(3.0, 0.0, 0.0)]])
def test_steps_that_shrink_or_enlarge(coefficients):
    for kind in ("noise", "strong"):
        x = sized(matrices(gen(8), 1, 256, 1024, torch.float64, kind), 1.0)[0]
        want = x.double() / x.double().norm()
        c32 = torch.tensor(coefficients, dtype=torch.float32).double().tolist()
        for a, b, c in c32:
            gram = want @ want.t()
            want = a * want + (b * gram + c * gram @ gram) @ want
        if want.abs().max() < 1e-36:      # bf16 holds nothing that small in full
            continue
        # a step's B is rounded twice, 2^-11 of it each time, and |b| + |c| is at most half of |a|, so B at most what is left of a: 2^-10 in the first step, after which X is a
        # hundredth and B nothing.  64 roundings of 2^-22 in chains of 64 steps
        assert off(ops.orthogonalize(x, steps=len(c32), coefficients=coefficients, eps=0.0), want) < last_rounding(want) + PLAIN + 2 * F16 + 64 * 2.0 ** -22, kind


@pytest.mark.parametrize("steps", [5, 8, 10, 12, 16])
@pytest.mark.parametrize("power", [12, 16, 20, 24])
def test_singular_values_that_many_steps_enlarge(steps, power):
    for tall in (False, True):
        x = sized(matrices(gen(9), 1, 256, 1024, torch.float64, "noise"), 1.0)[0]
        x[32:] *= 2.0 ** -power
        x = x.t().contiguous() if tall else x
        got = ops.orthogonalize(x, steps=steps, eps=0.0)
        want = newton(x, False, None, steps=steps, eps=0.0, roundings=False)
        # fp16's share as stated, 0.003 together with the last rounding; where 2^15 is passed, from nine steps on, that of the fp32 products' model
        bound = 0.003 if steps <= 8 else last_rounding(want) + 2 * off(newton(x, False, gen(4), steps=steps, eps=0.0), want) + 1e-6
        assert off(got, want) < bound, (tall, off(got, want), bound)


@pytest.mark.parametrize("coefficients,steps", [((1.5, -0.5, 0.0), 20), ((15 / 8, -10 / 8, 3 / 8), 12)])
def test_steps_that_converge(coefficients, steps):
    for kind in ("noise", "strong"):
        x = matrices(gen(10), 1, 300, 900, BF, kind)[0]
        want = newton(x, True, None, steps, coefficients, roundings=False)
        model = off(newton(x, True, gen(5), steps, coefficients), want)
        assert off(ops.orthogonalize(x, steps=steps, coefficients=coefficients), want) < last_rounding(want) + 2 * model + 1e-6


def test_an_update_of_coefficients_that_change_sign():
    # q(s) = 1 - 4 s^2: X's parts near s = 1/2 vanish; fp32 products
    x = sized(matrices(gen(11), 1, 256, 600, torch.float64, "strong"), 1.0)[0]
    want = newton(x, False, None, 3, (1.0, -4.0, 0.0), roundings=False)
    assert off(ops.orthogonalize(x, steps=3, coefficients=(1.0, -4.0, 0.0)), want) < last_rounding(want) + 2 * off(newton(x, False, gen(6), 3, (1.0, -4.0, 0.0)), want) + 1e-6
