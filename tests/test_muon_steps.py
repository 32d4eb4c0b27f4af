"""Muon's steps in 16 bits."""
import pytest
import torch

from paper_2509_06980_amd import policy_update as pu

BF = torch.bfloat16


def within_half_a_step(p, exact):
    """One rounding to bf16 of what 32 bits hold (a dozen roundings of 2^-24 of the step and of the weight before it)."""
    return ((p.double() - exact).abs() <= 2.0 ** -8 * exact.abs() * (1 + 2.0 ** -8) + 16 * 2.0 ** -24).all()


def test_adam_steps_of_muon_are_rounded_once():
    g = torch.Generator().manual_seed(1)
    for decay in (0.0, 0.1, 0.5):
        p = torch.randn(4000, generator=g).to(BF).requires_grad_()
        muon = pu.Muon([dict(params=[p])], adam_lr=0.02, weight_decay=decay)
        first = second = 0.0
        for step in range(1, 4):
            before = p.detach().double()
            p.grad = torch.randn(p.shape, generator=g).to(BF)
            d = p.grad.double()
            muon.step()
            first, second = 0.9 * first + 0.1 * d, 0.95 * second + 0.05 * d * d
            exact = before * (1 - 0.02 * decay) - 0.02 * (first / (1 - 0.9 ** step)) / ((second / (1 - 0.95 ** step)).sqrt() + 1e-8)
            assert within_half_a_step(p.detach(), exact), (decay, step)


def test_parameters_of_64_bits_stay_that_precise():
    p = torch.linspace(0.1, 1.0, 50, dtype=torch.float64).requires_grad_()
    muon, before = pu.Muon([dict(params=[p])], adam_lr=2.0 ** -10, weight_decay=0.5), p.detach().clone()
    p.grad = torch.zeros_like(p)
    muon.step()
    assert torch.equal(p.detach(), before * (1 - 2.0 ** -11))      # the step is 0


@pytest.mark.gpu
def test_orthogonal_steps_of_muon_are_rounded_once():
    from paper_2509_06980_amd import policy_ops as ops
    g = torch.Generator("cuda").manual_seed(2)
    for decay in (0.0, 0.1, 0.5):
        p = torch.randn(96, 40, generator=g, device="cuda").to(BF).requires_grad_()
        muon, m = pu.Muon([dict(params=[p], orthogonal=True)], lr=0.1, weight_decay=decay), torch.zeros(96, 40, device="cuda")
        for step in range(3):
            before = p.detach().double()
            p.grad = torch.randn(p.shape, generator=g, device="cuda").to(BF)
            m = 0.95 * m + p.grad.float()
            o = ops.orthogonalize((p.grad.float() + 0.95 * m).to(BF)).double()
            muon.step()
            assert within_half_a_step(p.detach(), before * (1 - 0.1 * decay) - 0.1 * (96 / 40) ** 0.5 * o), (decay, step)


def test_groups_that_are_added_later_are_checked_too():
    q = torch.ones(4, 4, requires_grad=True)
    muon = pu.Muon([dict(params=[torch.ones(3, 4, requires_grad=True)], orthogonal=True)])
    for shape in ((3,), (2, 3, 4), ()):
        with pytest.raises(ValueError, match="matrices"):
            muon.add_param_group(dict(params=iter([q, torch.ones(shape, requires_grad=True)]), orthogonal=True))
        assert len(muon.param_groups) == 1
    muon.add_param_group(dict(params=[q], orthogonal=True))      # nothing of a refused group stays
    muon.add_param_group(dict(params=[torch.ones(3, requires_grad=True)]))
    assert [len(g["params"]) for g in muon.param_groups] == [1, 1, 1]
