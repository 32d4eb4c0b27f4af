"""The policy update with linear layers, residual stream and orthogonalised steps by their own operators: against the engine, against a plain float64
decoder, and a step against its formula."""
import numpy as np
import pytest
import torch

from synthetic import make_weight_blob
from test_policy_update import CASES, SMALL, in_64_bits, rollout

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", CASES)
def test_fused_logprobs_are_the_engines(name):
    from paper_2509_06980_amd import policy_update as pu
    shape, tol = CASES[name]
    blob = make_weight_blob(shape, seed=5, weight_std=0.04, gain_std=0.1)
    engine, ids = rollout(shape, blob)
    tokens, mask, _, lens = pu.read_trajectories(engine, ids)
    want = engine.recompute_logprobs(ids, 1.0)
    engine.close()
    plain, fused = (pu.PolicyModel(blob, fused=f).logprobs(tokens, mask, lens).detach().cpu().numpy() for f in (False, True))
    assert np.array_equal(fused == 0, want == 0)
    assert np.abs(fused - want).max() < 2 * tol and np.abs(fused - plain).max() < 2 * tol


@pytest.mark.parametrize("name", ["tiny", "tied"])
def test_fused_gradient_is_that_of_the_plain_decoder(name):
    from paper_2509_06980_amd import policy_update as pu
    shape, _ = CASES[name]
    shape = shape.replace(vocab=min(shape.vocab, 512))
    blob = make_weight_blob(shape, seed=6, weight_std=0.05, gain_std=0.1)
    engine, ids = rollout(shape, blob)
    tokens, mask, old, lens = pu.read_trajectories(engine, ids)
    engine.close()
    old = old + np.random.default_rng(2).normal(0, 0.15, old.shape).astype(np.float32) * (mask == 0)
    adv = pu.group_advantages(np.random.default_rng(1).random(len(ids)), 4)
    model = pu.PolicyModel(blob, fused=True)
    value = pu.grpo_objective(model.logprobs(tokens, mask, lens), old, mask, lens, adv, 0.2, 0.1, old - 0.05)
    value.backward()
    lp, w = in_64_bits(model, tokens, mask, lens)
    want = pu.grpo_objective(lp, old, mask, lens, adv, 0.2, 0.1, old - 0.05)
    want.backward()
    assert abs(value.item() - want.item()) < 1e-5
    for n, p in model.params.items():
        if w[n].grad is None:
            assert p.grad is None
            continue
        off = (p.grad.double().cpu() - w[n].grad).norm() / w[n].grad.norm()
        # fp32 through two layers: some hundred roundings of 2^-24 on every way from a log-prob to a weight, with cancellation between tokens
        assert off < 1e-4, (n, off.item())


def test_a_step_of_muon_is_its_formula():
    from paper_2509_06980_amd import policy_update as pu
    from test_update_operators import newton
    g = torch.Generator("cuda").manual_seed(3)
    shapes = [(40, 24), (24, 40), (40, 24), (7,), (5, 6)]
    params = [torch.randn(s, generator=g, device="cuda").requires_grad_() for s in shapes]
    unused = torch.ones(3, 3, device="cuda", requires_grad=True)
    muon = pu.Muon([dict(params=params[:3] + [unused], orthogonal=True), dict(params=params[3:])], lr=0.1, weight_decay=0.5, adam_lr=0.01)
    want = [p.detach().double().clone() for p in params]
    m = [torch.zeros_like(w) for w in want]
    first, second = [torch.zeros_like(w) for w in want], [torch.zeros_like(w) for w in want]
    for step in range(1, 4):
        for i, p in enumerate(params):
            p.grad = torch.randn(p.shape, generator=g, device="cuda")
            d = p.grad.double()
            if i < 3:
                m[i] = 0.95 * m[i] + d
                o = newton(d + 0.95 * m[i], False, None, roundings=False)
                want[i] = want[i] * (1 - 0.1 * 0.5) - 0.1 * max(1.0, p.shape[0] / p.shape[1]) ** 0.5 * o
            else:
                first[i], second[i] = 0.9 * first[i] + 0.1 * d, 0.95 * second[i] + 0.05 * d * d
                want[i] = want[i] * (1 - 0.01 * 0.5) - 0.01 * (first[i] / (1 - 0.9 ** step)) / ((second[i] / (1 - 0.95 ** step)).sqrt() + 1e-8)
        muon.step()
    for p, w in zip(params, want):
        # steps in 32 bits: some thousand roundings of 2^-24 in a step's products
        assert (p.double() - w).abs().max() < 1e-4
    assert torch.equal(unused, torch.ones_like(unused))
    with pytest.raises(ValueError):
        pu.Muon([dict(params=[torch.ones(3, device="cuda")], orthogonal=True)])


def test_updates_run_together(capsys):
    from paper_2509_06980_amd import policy_update as pu
    blob = make_weight_blob(SMALL, seed=7, weight_std=0.05)
    engine, ids = rollout(SMALL, blob)
    rewards = np.random.default_rng(4).random(len(ids))
    model = pu.PolicyModel(blob, fused=True)
    before = {n: p.detach().clone() for n, p in model.params.items()}
    optimizer = pu.Muon(model.parameter_groups(), lr=0.01)
    assert abs(pu.update(model, optimizer, engine, ids, rewards, 4)) < 1e-5      # ratios of 1, advantages that add up to nothing in a group
    engine.close()
    for n, p in model.params.items():
        assert p.isfinite().all() and (p.grad is None or not torch.equal(p, before[n])), n
    pu.main(["--fused", "--muon", "--updates", "2"])
    assert capsys.readouterr().out.count("mean reward") == 2
