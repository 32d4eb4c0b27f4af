"""What the policy update refuses before anything reaches a GPU: an index out of range on a GPU ends the process."""
import numpy as np
import pytest
import torch

from paper_2509_06980_amd import policy_update as pu
from synthetic import SHAPES, make_weight_blob

SHAPE = SHAPES["tiny"].replace(hidden=64, n_q_heads=4, n_kv_heads=2, head_dim=16, intermediate=96, vocab=128)


@pytest.fixture(scope="module")
def model():
    return pu.PolicyModel(make_weight_blob(SHAPE, seed=1), device="cpu")


@pytest.mark.parametrize("tokens", [[3, 128, 5], [3, 5, -1], [2 ** 31, 1, 1], [-2 ** 31, 1, 1], [1 << 40, 1, 1]])
def test_tokens_outside_the_vocabulary_are_refused(model, tokens):
    for form in (np.asarray(tokens), torch.tensor(tokens), tokens):
        with pytest.raises(ValueError, match="vocabulary"):
            model.logprobs(form, [1, 0, 0], [3])
    with pytest.raises(ValueError, match="vocabulary"):
        model.hidden(torch.tensor(tokens), [3])


def test_rows_without_their_trajectories_are_refused(model):
    for lens in ([2], [4], [3, 0], [], [4, -1]):
        with pytest.raises(ValueError, match="lengths"):
            model.hidden(torch.tensor([1, 2, 3]), lens)
        with pytest.raises(ValueError, match="lengths"):
            model.logprobs([1, 2, 3], [1, 0, 0], lens)


def test_objective_of_arrays_that_do_not_fit_is_refused():
    lp, mask, adv = torch.zeros(5), [1, 0, 0, 1, 0], [1.0, -1.0]
    good = dict(logprobs=lp, old_logprobs=lp, obs_mask=mask, lens=[3, 2], advantages=adv, clip_eps=0.2, beta=0.1, ref_logprobs=lp)
    assert torch.isfinite(pu.grpo_objective(**good))
    for bad in (dict(lens=[3, 3]), dict(lens=[3, 1]), dict(lens=[3]), dict(lens=[6, -1]), dict(lens=[]), dict(advantages=[1.0]), dict(advantages=[1.0, 2.0, 3.0]),
                dict(old_logprobs=lp[:4]), dict(obs_mask=mask[:4]), dict(obs_mask=mask + [0]), dict(ref_logprobs=torch.zeros(6)), dict(logprobs=lp[:4])):
        with pytest.raises(ValueError):
            pu.grpo_objective(**{**good, **bad})


def test_a_trajectory_without_tokens_adds_nothing():
    # as in rl_grpo_objective: it counts as a trajectory, with 0; also as the last one, where its place is behind all tokens
    g = torch.Generator().manual_seed(3)
    lp, old = -torch.rand(5, generator=g), -torch.rand(5, generator=g)
    mask = [1, 0, 0, 1, 0]
    two = pu.grpo_objective(lp, old, mask, [3, 2], [1.0, -0.5], 0.2)
    for lens, adv in (([3, 2, 0], [1.0, -0.5, 2.0]), ([0, 3, 2], [2.0, 1.0, -0.5]), ([3, 0, 2], [1.0, 2.0, -0.5])):
        assert torch.allclose(pu.grpo_objective(lp, old, mask, lens, adv, 0.2), two * 2 / 3)
