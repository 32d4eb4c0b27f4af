"""The policy update behind a rollout (Section 2.3.2 of the paper: rollout, reward, update; loss mask on tool results).

The trajectories that the rollout engine generated are run through the same decoder again, packed one after the other, with the
operators of `policy_ops`: norms, rotary positions, attention over packed trajectories and the log-probs of the sampled
tokens, each with its backward pass; the projections between them are plain matrix products.  The objective is the masked GRPO
objective that the engine evaluates forward (rl_grpo_objective); here it has a gradient, and `to_blob` gives the updated
weights back in the form that the engine loads.

    python -m paper_2509_06980_amd.policy_update        # rollouts of a small model, reward, updates, rollouts of the updated model
"""
import struct
from types import SimpleNamespace

import numpy as np
import torch
import torch.nn.functional as F

from . import policy_ops as ops

_HEADER = 64
_FIELDS = ("n_layers", "hidden", "n_q_heads", "n_kv_heads", "head_dim", "intermediate", "vocab", "rms_eps", "rope_theta", "qk_norm",
           "tie_embeddings", "weight_dtype")


def _tensors(c):
    """[(name, shape)] in the order of the weight blob (include/rl_rollout.h, rl_model_load)."""
    qw, kw = c.n_q_heads * c.head_dim, c.n_kv_heads * c.head_dim
    names = [("embed", (c.vocab, c.hidden))]
    for i in range(c.n_layers):
        names += [(f"l{i}.{n}", s) for n, s in (
            ("g_in", (c.hidden,)), ("w_q", (qw, c.hidden)), ("w_k", (kw, c.hidden)), ("w_v", (kw, c.hidden)), ("g_q", (c.head_dim,)),
            ("g_k", (c.head_dim,)), ("w_o", (c.hidden, qw)), ("g_post", (c.hidden,)), ("w_gate", (c.intermediate, c.hidden)),
            ("w_up", (c.intermediate, c.hidden)), ("w_down", (c.hidden, c.intermediate)))]
    names.append(("g_final", (c.hidden,)))
    return names if c.tie_embeddings else names + [("lm_head", (c.vocab, c.hidden))]


def _lengths(lens, total, least):
    """lens as a list of numbers, `least` or more each, that add up to `total`."""
    lens = [int(n) for n in _tensor(lens).tolist()]
    if not lens or min(lens) < least or sum(lens) != total:
        raise ValueError("lens are the lengths of " + ("non-empty " if least else "") + "packed trajectories, together all of their tokens")
    return lens


def _tensor(x, device=None):
    """x as a tensor on `device` (None: where it is)."""
    return torch.as_tensor(x if isinstance(x, torch.Tensor) else np.asarray(x), device=device)


class PolicyModel:
    """The engine's decoder as torch parameters, from and to its weight blob."""

    def __init__(self, blob, device="cuda"):
        raw = np.ascontiguousarray(np.asarray(blob, np.uint8))
        if raw.size < _HEADER or bytes(raw[:4]) != b"RLW1":
            raise ValueError("no weight blob")
        version, *fields = struct.unpack("<I7i2f3i", bytes(raw[4:56]))
        if version != 1:
            raise ValueError("weight blob of another version")
        self.config = c = SimpleNamespace(**dict(zip(_FIELDS, fields)))
        self.dtype = torch.bfloat16 if c.weight_dtype == 1 else torch.float32
        self.header = raw[:_HEADER].copy()
        table = _tensors(c)
        el = 2 if c.weight_dtype == 1 else 4
        if raw.size != _HEADER + el * sum(int(np.prod(s)) for _, s in table):
            raise ValueError("weight blob of another size")
        self.params, at = {}, _HEADER
        for name, shape in table:
            n = int(np.prod(shape)) * el
            t = torch.from_numpy(raw[at:at + n].copy()).view(self.dtype).reshape(shape).to(device)
            self.params[name] = t.requires_grad_()
            at += n
        self.device = torch.device(device)
        self._table = None

    def parameters(self):
        return list(self.params.values())

    def to_blob(self):
        """The weights as rl_model_load takes them."""
        parts = [self.header] + [p.detach().reshape(-1).view(torch.uint8).cpu().numpy() for p in self.params.values()]
        return np.concatenate(parts)

    def _in_vocabulary(self, tokens):
        """Refuses other tokens: looked up on a GPU, one would end the process.  Waits for tokens that are on one."""
        if tokens.numel():
            low, high = torch.aminmax(tokens)
            if low < 0 or high >= self.config.vocab:
                raise ValueError(f"tokens outside the vocabulary of {self.config.vocab}")

    def hidden(self, tokens, lens):
        """Rows behind the final norm [tokens, hidden] of packed trajectories; residual stream and norms in 32 bits."""
        lens = _lengths(lens, tokens.shape[0], 1)
        self._in_vocabulary(tokens)
        return self._rows(tokens, lens)

    def _rows(self, tokens, lens):
        c, p = self.config, self.params
        total, longest = sum(lens), max(lens)
        offsets = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        cu = torch.from_numpy(offsets).to(self.device)
        positions = (torch.arange(total, device=self.device, dtype=torch.int32)
                     - torch.repeat_interleave(cu[:-1], cu.diff().long(), output_size=total))
        if self._table is None or self._table.shape[0] < longest:
            self._table = ops.rotary_table(longest, c.head_dim, theta=c.rope_theta, device=self.device)

        def norm(x, gain):
            return ops.norm(x, p[gain].float(), eps=c.rms_eps).to(self.dtype)

        def heads(x, gain, n):
            x = x.view(total, n, c.head_dim)
            return ops.norm(x, p[gain], eps=c.rms_eps) if c.qk_norm else x

        h = F.embedding(tokens, p["embed"]).float()
        for i in range(c.n_layers):
            w = lambda name: f"l{i}.{name}"  # noqa: B023,E731
            a = norm(h, w("g_in"))
            q, k = heads(F.linear(a, p[w("w_q")]), w("g_q"), c.n_q_heads), heads(F.linear(a, p[w("w_k")]), w("g_k"), c.n_kv_heads)
            v = F.linear(a, p[w("w_v")]).view(total, c.n_kv_heads, c.head_dim)
            q, k = ops.rotate(q, k, positions, self._table)
            h = h + F.linear(ops.attention(q, k, v, cu, cu).flatten(1), p[w("w_o")]).float()
            b = norm(h, w("g_post"))
            h = h + F.linear(F.silu(F.linear(b, p[w("w_gate")])) * F.linear(b, p[w("w_up")]), p[w("w_down")]).float()
        return norm(h, "g_final")

    def logprobs(self, tokens, obs_mask, lens, temperature=1.0):
        """Differentiable rl_recompute_logprobs: one float32 a token of the packed trajectories, the log-prob of a sampled token
        given all before it, 0 for appended tokens and first ones.  tokens, obs_mask: integers on any device; lens: per trajectory."""
        tokens = _tensor(tokens)
        sampled = _tensor(obs_mask, self.device) == 0
        if tokens.dim() != 1 or sampled.shape != tokens.shape:
            raise ValueError("one token id and one mask a token")
        lens = _lengths(lens, tokens.shape[0], 1)
        self._in_vocabulary(tokens)
        tokens = tokens.to(self.device).long()
        first = torch.zeros_like(sampled)
        first[torch.as_tensor(np.concatenate([[0], np.cumsum(lens)[:-1]]), device=self.device)] = True
        target = torch.where(sampled & ~first, tokens, -1).int()      # of the row before
        head = self.params["embed" if self.config.tie_embeddings else "lm_head"]
        temperature = 1.0 if temperature == 0 else float(temperature)
        lp = ops.token_logprobs(self._rows(tokens, lens), head, torch.cat([target[1:], target.new_full((1,), -1)]), temperature)
        return torch.cat([lp.new_zeros(1), lp[:-1]])


def group_advantages(rewards, group_size, eps_std=1e-6, std_ddof=0):
    """(r - mean) / (std + eps_std) within groups of consecutive rewards."""
    r = torch.as_tensor(rewards, dtype=torch.float64).reshape(-1, group_size)
    return ((r - r.mean(1, keepdim=True)) / (r.std(1, keepdim=True, correction=std_ddof) + eps_std)).reshape(-1)


def grpo_objective(logprobs, old_logprobs, obs_mask, lens, advantages, clip_eps, beta=0.0, ref_logprobs=None):
    """The masked GRPO objective of rl_grpo_objective, differentiable by `logprobs` (all arrays packed, one value a token, on any device): mean
    over trajectories of the mean over their sampled tokens (0 of one that has none) of min(rho A, clip(rho) A) - beta k3."""
    dev, total = logprobs.device, logprobs.shape[0]
    counts = _lengths(lens, total, 0)
    lens = torch.as_tensor(counts, device=dev)
    used = _tensor(obs_mask, dev) == 0
    old = _tensor(old_logprobs, dev).double()
    a = _tensor(advantages, dev).double()
    ref = None if ref_logprobs is None else _tensor(ref_logprobs, dev).double()
    if any(x is not None and x.shape != logprobs.shape for x in (used, old, ref)) or a.shape != lens.shape:
        raise ValueError("one mask and log-prob a token, one advantage a trajectory")
    which = torch.repeat_interleave(torch.arange(len(lens), device=dev), lens, output_size=total)
    used[(torch.cumsum(lens, 0) - lens)[lens > 0]] = False      # a first token has no log-prob
    lp, old, a = logprobs[used].double(), old[used], a[which[used]]
    rho = (lp - old).exp()
    term = torch.minimum(rho * a, rho.clamp(1 - clip_eps, 1 + clip_eps) * a)
    if ref is not None:
        d = ref[used] - lp
        term = term - beta * (d.exp() - d - 1)
    count = torch.zeros(len(lens), dtype=torch.float64, device=dev).index_add_(0, which[used], torch.ones_like(term))
    return (term / count[which[used]]).sum() / len(lens)


def read_trajectories(engine, traj_ids):
    """(tokens, observation mask, recorded log-probs, lengths) of an engine's trajectories, packed in call order."""
    parts = [engine.traj_read(int(i))[:3] for i in traj_ids]
    return (*(np.concatenate(x) for x in zip(*parts)), [len(p[0]) for p in parts])


def update(model, optimizer, engine, traj_ids, rewards, group_size, temperature=1.0, clip_eps=0.2, beta=0.0, ref_logprobs=None):
    """One step of `optimizer` up the objective of the engine's trajectories -> the objective before the step."""
    tokens, mask, old, lens = read_trajectories(engine, traj_ids)
    optimizer.zero_grad(set_to_none=True)
    lp = model.logprobs(tokens, mask, lens, temperature)
    value = grpo_objective(lp, old, mask, lens, group_advantages(rewards, group_size), clip_eps, beta, ref_logprobs)
    (-value).backward()
    optimizer.step()
    return value.item()


def main():
    import sys
    from pathlib import Path
    sys.path.insert(0, str(Path(__file__).resolve().parent.parent))
    from synthetic import SHAPES, make_weight_blob

    from . import RolloutEngine
    shape = SHAPES["small-d128"]
    model = PolicyModel(make_weight_blob(shape, seed=1, weight_std=0.03))
    optimizer = torch.optim.Adam(model.parameters(), lr=5e-3)
    prompts, group, n_new = 8, 32, 24
    rng = np.random.default_rng(0)
    for step in range(10):
        engine = RolloutEngine(model.to_blob(), max_context=128, max_trajectories=prompts * group, kv_pool_pages=prompts * group * 8)
        ids = np.arange(prompts * group)
        engine.append_observation(ids[::group], rng.integers(0, shape.vocab, prompts * 16), [16] * prompts)
        for i in ids[::group]:
            engine.fork(i, np.arange(i + 1, i + group))
        engine.decode_steps(ids, n_new // 2, 1.0, step)
        engine.append_observation(ids, rng.integers(0, shape.vocab, len(ids) * 8), [8] * len(ids))      # what a tool returned
        engine.decode_steps(ids, n_new // 2, 1.0, step)
        tokens, mask, _, lens = read_trajectories(engine, ids)
        # a reward that can be checked by eye: sampled tokens from the lower half of the vocabulary
        low = ((tokens < shape.vocab // 2) & (mask == 0)).reshape(len(ids), -1).sum(1) / n_new
        value = update(model, optimizer, engine, ids, low, group)
        engine.close()
        print(f"step {step}: mean reward {low.mean():.3f}, objective {value:+.4f}")


if __name__ == "__main__":
    main()
