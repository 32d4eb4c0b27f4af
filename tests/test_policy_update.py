"""The policy update on the GPU: log-probs and objective against the rollout engine's own, gradients against a plain float64 decoder."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

import paper_2509_06980_amd as rl
from synthetic import SHAPES, make_weight_blob

pytestmark = pytest.mark.gpu

SMALL = SHAPES["tiny"].replace(hidden=64, n_q_heads=4, n_kv_heads=2, head_dim=16, intermediate=96, vocab=128)
# bounds of one data path against the exact log-probs at temperature 1 (test_gpu_parity.py); two of them may be twice as far apart
CASES = {"tiny": (SHAPES["tiny"], 1e-4), "tied": (SMALL.replace(tie_embeddings=1, qk_norm=0), 1e-4), "small-d128": (SHAPES["small-d128"], 3e-2)}


def rollout(shape, blob, groups=2, group=4, turns=((7, 9), (5, 3), (6, 0))):
    engine = rl.RolloutEngine(blob, max_context=128, max_trajectories=groups * group, kv_pool_pages=groups * group * 8)
    rng = np.random.default_rng(3)
    ids = np.arange(groups * group)
    engine.append_observation(ids[::group], rng.integers(0, shape.vocab, groups * 21), [21] * groups)
    for i in ids[::group]:
        engine.fork(int(i), np.arange(i + 1, i + group))
    for n, (gen, obs) in enumerate(turns):
        engine.decode_steps(ids, gen, 1.0, 77 + n)
        if obs:
            lens = [obs + int(i) % 3 for i in ids]
            engine.append_observation(ids, rng.integers(0, shape.vocab, sum(lens)), lens)
    return engine, ids


def in_64_bits(model, tokens, mask, lens):
    """Log-probs by a decoder written out with torch's elementary operations in float64, one trajectory at a time, and its parameters."""
    c = model.config
    w = {n: p.detach().double().cpu().requires_grad_() for n, p in model.params.items()}
    norm = lambda x, g: x / (x.square().mean(-1, keepdim=True) + c.rms_eps).sqrt() * g  # noqa: E731
    out, at = [], 0
    for n in lens:
        x = torch.as_tensor(tokens[at:at + n]).long()
        angle = torch.arange(n, dtype=torch.float64)[:, None] * c.rope_theta ** (-torch.arange(0, c.head_dim, 2, dtype=torch.float64) / c.head_dim)
        cos, sin = angle.cos()[:, None], angle.sin()[:, None]

        def turn(t):
            a, b = t.chunk(2, -1)
            return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)

        h = w["embed"][x]
        for i in range(c.n_layers):
            p = lambda name: w[f"l{i}.{name}"]  # noqa: E731
            a = norm(h, p("g_in"))
            q, k, v = ((a @ p(m).t()).view(n, -1, c.head_dim) for m in ("w_q", "w_k", "w_v"))
            if c.qk_norm:
                q, k = norm(q, p("g_q")), norm(k, p("g_k"))
            q, k = turn(q), turn(k)
            k, v = (t.repeat_interleave(c.n_q_heads // c.n_kv_heads, 1) for t in (k, v))
            z = torch.einsum("ihd,jhd->hij", q, k) / c.head_dim ** 0.5
            z = z.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -torch.inf)
            h = h + torch.einsum("hij,jhd->ihd", z.softmax(-1), v).flatten(1) @ p("w_o").t()
            b = norm(h, p("g_post"))
            h = h + (F.silu(b @ p("w_gate").t()) * (b @ p("w_up").t())) @ p("w_down").t()
        z = norm(h, w["g_final"]) @ w["embed" if c.tie_embeddings else "lm_head"].t()
        lp = torch.log_softmax(z[:-1], -1).gather(1, x[1:, None])[:, 0]
        out.append(torch.cat([lp.new_zeros(1), torch.where(torch.as_tensor(mask[at + 1:at + n]) == 0, lp, 0.0)]))
        at += n
    return torch.cat(out), w


@pytest.mark.parametrize("name", CASES)
def test_logprobs_and_objective_are_the_engines(name):
    from paper_2509_06980_amd import policy_update as pu
    shape, tol = CASES[name]
    blob = make_weight_blob(shape, seed=5, weight_std=0.04, gain_std=0.1)
    engine, ids = rollout(shape, blob)
    model = pu.PolicyModel(blob)
    tokens, mask, old, lens = pu.read_trajectories(engine, ids)
    for temperature in (1.0, 0.7):
        want = engine.recompute_logprobs(ids, temperature)
        got = model.logprobs(tokens, mask, lens, temperature).detach().cpu().numpy()
        assert np.array_equal(got == 0, want == 0)
        assert np.abs(got - want).max() < 2 * tol / min(1.0, temperature)
    rewards = np.random.default_rng(1).random(len(ids))
    ref = old - 0.1
    want = engine.grpo_objective(ids, 4, rewards, 1.0, 0.2, 0.05, ref_logprobs=ref)
    adv = pu.group_advantages(rewards, 4)
    lp = model.logprobs(tokens, mask, lens)
    got = pu.grpo_objective(lp, old, mask, lens, adv, 0.2, 0.05, ref)
    assert np.allclose(adv.numpy(), want["advantages"], atol=1e-5)      # the engine's rewards are float32
    assert abs(got.item() - want["objective"]) < 2 * tol
    assert np.array_equal(model.to_blob(), np.asarray(blob))
    engine.close()


@pytest.mark.parametrize("name", ["tiny", "tied"])
def test_gradient_is_that_of_the_plain_decoder(name):
    from paper_2509_06980_amd import policy_update as pu
    shape, _ = CASES[name]
    shape = shape.replace(vocab=min(shape.vocab, 512))
    blob = make_weight_blob(shape, seed=6, weight_std=0.05, gain_std=0.1)
    engine, ids = rollout(shape, blob)
    tokens, mask, old, lens = pu.read_trajectories(engine, ids)
    engine.close()
    old = old + np.random.default_rng(2).normal(0, 0.15, old.shape).astype(np.float32) * (mask == 0)      # some ratios clipped
    adv = pu.group_advantages(np.random.default_rng(1).random(len(ids)), 4)
    model = pu.PolicyModel(blob)
    value = pu.grpo_objective(model.logprobs(tokens, mask, lens), old, mask, lens, adv, 0.2, 0.1, old - 0.05)
    value.backward()
    lp, w = in_64_bits(model, tokens, mask, lens)
    want = pu.grpo_objective(lp, old, mask, lens, adv, 0.2, 0.1, old - 0.05)
    want.backward()
    assert abs(value.item() - want.item()) < 1e-5
    for n, p in model.params.items():
        if w[n].grad is None:      # QK-norm gains of a model without QK-norm
            assert p.grad is None
            continue
        off = (p.grad.double().cpu() - w[n].grad).norm() / w[n].grad.norm()
        # fp32 through two layers: some hundred roundings of 2^-24 on every way from a log-prob to a weight, with cancellation between tokens
        assert off < 1e-4, (n, off.item())


def test_updates_raise_the_objective_and_go_back_into_the_engine():
    from paper_2509_06980_amd import policy_update as pu
    shape = SMALL
    blob = make_weight_blob(shape, seed=7, weight_std=0.05)
    engine, ids = rollout(shape, blob)
    rewards = np.random.default_rng(4).random(len(ids))
    model = pu.PolicyModel(blob)
    optimizer = torch.optim.SGD(model.parameters(), lr=0.05)
    values = [pu.update(model, optimizer, engine, ids, rewards, 4) for _ in range(4)]
    assert abs(values[0]) < 1e-5                       # ratios of 1, advantages that add up to nothing in a group
    assert values[1] > values[0] and values[3] > values[1]
    # the updated weights in an engine of their own: the same objective of the same trajectories
    tokens, mask, old, lens = pu.read_trajectories(engine, ids)
    engine.close()
    again = rl.RolloutEngine(model.to_blob(), max_context=128, max_trajectories=len(ids), kv_pool_pages=64)
    at = 0
    for i, n in zip(ids, lens):                        # the same tokens, sampled ones forced
        for t in range(n):
            if mask[at + t]:
                again.append_observation([i], [tokens[at + t]], [1])
            else:
                again.decode_step_forced([i], 1.0, [tokens[at + t]])
        at += n
    got = again.grpo_objective(ids, 4, rewards, 1.0, 0.2, 0.0, old_logprobs=old)["objective"]
    with torch.no_grad():
        want = pu.grpo_objective(model.logprobs(tokens, mask, lens), old, mask, lens, pu.group_advantages(rewards, 4), 0.2).item()
    assert abs(got - want) < 1e-4 and want > values[0]
    again.close()


def test_refuses_what_is_no_blob_or_no_batch():
    from paper_2509_06980_amd import policy_update as pu
    blob = np.asarray(make_weight_blob(SMALL, seed=1))
    for bad in (blob[:40], blob[:-4], np.concatenate([[0], blob[1:]]).astype(np.uint8)):
        with pytest.raises(ValueError):
            pu.PolicyModel(bad)
    model = pu.PolicyModel(blob)
    for tokens, mask, lens in (([1, 2], [0, 0], [1]), ([1, 2], [0], [2]), ([1, 2], [0, 0], [2, 0])):
        with pytest.raises(ValueError):
            model.logprobs(tokens, mask, lens)


def test_trajectories_may_be_anywhere():
    from paper_2509_06980_amd import policy_update as pu
    blob = make_weight_blob(SMALL, seed=9, weight_std=0.05)
    engine, ids = rollout(SMALL, blob)
    model = pu.PolicyModel(blob)
    tokens, mask, old, lens = pu.read_trajectories(engine, ids)
    engine.close()
    adv = pu.group_advantages(np.random.default_rng(1).random(len(ids)), 4)
    lp = model.logprobs(tokens, mask, lens)
    ref = old - 0.1
    want = pu.grpo_objective(lp, old, mask, lens, adv, 0.2, 0.05, ref)
    there = lambda x: torch.as_tensor(x, device="cuda")  # noqa: E731
    for to in (there, torch.as_tensor, list):
        assert torch.equal(model.logprobs(to(tokens), to(mask), to(lens)), lp)
        assert torch.equal(pu.grpo_objective(lp, to(old), to(mask), to(lens), to(adv), 0.2, 0.05, to(ref)), want)
    # a reference policy's own log-probs, as they come
    assert torch.equal(pu.grpo_objective(lp, there(old), mask, lens, adv, 0.2, 0.05, lp.detach()), pu.grpo_objective(lp, old, mask, lens, adv, 0.2))
