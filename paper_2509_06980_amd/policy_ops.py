"""The policy update's operators on torch tensors: norms, rotary positions, attention over packed trajectories, log-probs of tokens,
linear layers with what follows them and the residual stream with its norms, forward and backward (the calls of include/rl_rollout.h
under the same names), and as functions of torch.autograd; orthogonalised updates.

Tensors live on one GPU; work is enqueued on torch's current stream and nothing waits for it.  Arguments are checked in
compiled code; what is refused raises RolloutError.
"""
import math

import torch

from .binding import RolloutError, load_library

load_library()

try:
    from . import _policy_torch as _native
except ImportError as e:
    raise RuntimeError("the operators are not built: `python paper_2509_06980_amd/build.py` (needs hipcc and g++)") from e

_raw_stream = torch._C._cuda_getCurrentRawStream


def _refuse(message):
    raise RolloutError(-1, message)


def _stream(x):
    """torch's current stream on x's GPU."""
    index = x.get_device()
    if index < 0:
        _refuse("tensors have to be on the GPU")
    return _raw_stream(index)


# ---- norms ---------------------------------------------------------------------------------------------------------
def norm_forward(x, weight, bias=None, eps=1e-6, centered=False):
    """RMS norm (layer norm where `centered`) over the last dimension -> (y, mean, rstd); y is contiguous, mean (None in the RMS
    form) and rstd have x's shape without its last dimension."""
    return _native.norm_forward(x, weight, bias, eps, centered, _stream(x))


def norm_backward(dy, x, weight, mean, rstd, centered=False, biased=None):
    """Gradients of norm_forward -> (dx, dweight, dbias); dbias is None unless `biased` (None: where `centered`)."""
    return _native.norm_backward(dy, x, weight, mean, rstd, centered, centered if biased is None else biased, _stream(x))


# ---- rotary positions ----------------------------------------------------------------------------------------------
def rotary_table(n_positions, rot_dim, theta=10000.0, stretch=1.0, trained_positions=None, fast_turns=32.0, slow_turns=1.0,
                 gain=1.0, device="cuda"):
    """cos and sin of every position's angles, [n_positions, rot_dim / 2, 2] in float32, computed in float64.

    Pair i turns by theta^(-2 i / rot_dim) a position.  For contexts `stretch` times longer than trained on: without
    `trained_positions` all angles are divided by `stretch`; with it, pairs that make `fast_turns` turns or more over the trained
    positions keep their rate, those with `slow_turns` or fewer are divided, the ones between go over linearly.  `gain` multiplies
    cos and sin (temperature of the attention logits at long contexts)."""
    if n_positions < 1 or rot_dim < 2 or rot_dim % 2 or theta <= 0 or stretch <= 0:
        _refuse("n_positions >= 1, an even rot_dim >= 2, theta and stretch > 0")
    if trained_positions is not None and not fast_turns > slow_turns:
        _refuse("fast_turns has to be above slow_turns")
    rate = theta ** (-torch.arange(0, rot_dim, 2, dtype=torch.float64) / rot_dim)
    if trained_positions is None:
        rate = rate / stretch
    else:
        turns = rate * trained_positions / (2 * math.pi)
        slow = ((fast_turns - turns) / (fast_turns - slow_turns)).clamp(0.0, 1.0)
        rate = rate * (1 - slow) + rate / stretch * slow
    angle = torch.arange(n_positions, dtype=torch.float64, device=device)[:, None] * rate.to(device)
    return (torch.stack([angle.cos(), angle.sin()], -1) * gain).float().contiguous()


def rotary(q, k, positions, table, interleaved=False, inverse=False, q_out=None, k_out=None):
    """Turn the heads of q [tokens, heads, head_dim] and k (or None) by their positions -> (q, k); `inverse`: the backward pass.
    Results are new contiguous tensors unless q_out / k_out say where (they may be q and k themselves, but lie over no other part of them);
    autograd sees these as changed in place, and one that requires a gradient is refused."""
    return _native.rotary(q, k, positions, table, interleaved, inverse, q_out, k_out, _stream(q))


# ---- attention over packed trajectories ------------------------------------------------------------------------------
def attention_forward(q, k, v, cu_q, cu_k, causal=True, scale=None):
    """Attention of packed sequences -> (o [tokens, heads, head_dim], lse [heads, tokens]); see rl_attention_forward.  Tokens of
    no sequence (padding before cu[0] and from cu[-1] on) get o = 0 and lse = -infinity.  scale None: head_dim^-1/2."""
    return _native.attention_forward(q, k, v, cu_q, cu_k, causal, scale, _stream(q))


def attention_backward(do, q, k, v, o, lse, cu_q, cu_k, causal=True, scale=None):
    """Gradients of attention_forward -> (dq, dk, dv), contiguous; those of tokens of no sequence are 0."""
    return _native.attention_backward(do, q, k, v, o, lse, cu_q, cu_k, causal, scale, _stream(q))


# ---- log-probs of tokens ---------------------------------------------------------------------------------------------
def token_logprobs_forward(hidden, weight, targets, temperature=1.0):
    """Log-probs of `targets` under softmax(hidden weight^T / temperature), without keeping the logits -> (logp, lse), float32.
    Rows with a negative target take no part (0)."""
    return _native.token_logprobs_forward(hidden, weight, targets, temperature, _stream(hidden))


def token_logprobs_backward(dlogp, hidden, weight, targets, lse, temperature=1.0):
    """Gradients of token_logprobs_forward's logp -> (dhidden, dweight)."""
    return _native.token_logprobs_backward(dlogp, hidden, weight, targets, lse, temperature, _stream(hidden))


# ---- linear layers ---------------------------------------------------------------------------------------------------
def linear_forward(x, weight, bias=None, up=None, up_bias=None, activation="none", residual=None, keep=False):
    """act(x weight^T + bias) [* (x up^T + up_bias)] [+ residual] -> (y, kept); see rl_linear_forward.  x: [.., inner], weights: [outer, inner];
    activation: none, relu, silu, gelu or gelu_tanh.  The residual has y's shape and x's type or float32; y has its type.  kept: what the
    backward call needs, where `keep` (None where it needs nothing)."""
    return _native.linear_forward(x, weight, bias, up, up_bias, activation, residual, keep, _stream(x))


def linear_backward(dy, x, weight, kept=None, up=None, activation="none", biased=False, up_biased=False, wanted=(True, True, True)):
    """Gradients of linear_forward -> (dx, dweight, dbias, dup, dup_bias), each None where there is none or, of dx, dweight and dup, it is not
    `wanted`.  dy is of y's type; it is the residual's gradient too."""
    dx, dw, dup, db, dub = _native.linear_backward(dy, x, weight, kept, up, activation, biased, up_biased, *wanted, _stream(x))
    return dx, dw, db, dup, dub


# ---- the residual stream around a block --------------------------------------------------------------------------------
def residual_norm_forward(h, y, weight, bias=None, post_weight=None, post_bias=None, gate=None, residual_scale=1.0, block_scale=1.0, eps=1e-6,
                          centered=False):
    """A block's result y joins the stream h, the next block's norm follows -> (h_new, a, stats); see rl_residual_norm_forward.

    h_new = residual_scale h + block_scale gate u, with u = y, or norm(y) post_weight + post_bias; a = norm(h_new) weight + bias (None without
    weight).  Norms over the last dimension, RMS (layer norm where `centered`).  h is float32 or of y's type.  gate: [width], y's shape, or
    y's shape with one column."""
    return _native.residual_norm_forward(h, y, weight, bias, post_weight, post_bias, gate, residual_scale, block_scale, eps, centered, _stream(y))


def residual_norm_backward(dh_new, da, h_new, y, stats, weight, post_weight=None, post_bias=None, gate=None, residual_scale=1.0, block_scale=1.0,
                           centered=False, biased=False):
    """Gradients of residual_norm_forward from those of h_new and of a (one of the two may be None) -> (dh, dy, dweight, dbias, dpost_weight,
    dpost_bias, dgate), None where there is none."""
    return _native.residual_norm_backward(dh_new, da, h_new, y, stats, weight, post_weight, post_bias, gate, residual_scale, block_scale, centered,
                                          biased, _stream(y))


# ---- orthogonalised updates --------------------------------------------------------------------------------------------
def orthogonalize(x, steps=5, coefficients=(3.4445, -4.7750, 2.0315), eps=1e-7):
    """Every matrix of x [.., rows, columns] with its singular values driven towards 1 -> a new tensor: x / (|x| + eps), then `steps` times
    X <- a X + b (X X^T) X + c (X X^T)^2 X; see rl_orthogonalize.  coefficients: (a, b, c), or one such triple a step.
    No gradient passes through it."""
    table = []
    try:
        if steps in range(1, 65):
            triples = [coefficients] * steps if not hasattr(coefficients[0], "__len__") else coefficients
            table = [(float(a), float(b), float(c)) for a, b, c in triples]
    except (TypeError, ValueError, LookupError):
        pass
    if not table or len(table) != steps:
        _refuse("1 to 64 steps; coefficients are three numbers, or three numbers for each step")
    table = [v for triple in table for v in triple]
    return _native.orthogonalize(x, table, eps, _stream(x))


# ---- torch.autograd --------------------------------------------------------------------------------------------------
class _Norm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, centered):
        y, mean, rstd = norm_forward(x, weight, bias, eps, centered)
        ctx.save_for_backward(x, weight, mean, rstd)
        ctx.centered, ctx.biased = centered, bias is not None
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, mean, rstd = ctx.saved_tensors
        return (*norm_backward(dy, x, weight, mean, rstd, ctx.centered, ctx.biased), None, None)


class _Rotary(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, positions, table, interleaved):
        ctx.save_for_backward(positions, table)
        ctx.interleaved = interleaved
        return rotary(q, k, positions, table, interleaved)

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dq, dk):
        positions, table = ctx.saved_tensors
        return (*rotary(dq, dk, positions, table, ctx.interleaved, inverse=True), None, None, None)


class _Attention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, cu_q, cu_k, causal, scale):
        o, lse = attention_forward(q, k, v, cu_q, cu_k, causal, scale)
        ctx.save_for_backward(q, k, v, o, lse, cu_q, cu_k)
        ctx.causal, ctx.scale = causal, scale
        return o

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, do):
        q, k, v, o, lse, cu_q, cu_k = ctx.saved_tensors
        return (*attention_backward(do, q, k, v, o, lse, cu_q, cu_k, ctx.causal, ctx.scale), None, None, None, None)


class _TokenLogprobs(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, weight, targets, temperature):
        logp, lse = token_logprobs_forward(hidden, weight, targets, temperature)
        ctx.save_for_backward(hidden, weight, targets, lse)
        ctx.temperature = temperature
        return logp

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dlogp):
        hidden, weight, targets, lse = ctx.saved_tensors
        return (*token_logprobs_backward(dlogp.contiguous(), hidden, weight, targets, lse, ctx.temperature), None, None)


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, up, up_bias, activation, residual, keep):
        y, kept = linear_forward(x, weight, bias, up, up_bias, activation, residual, keep)
        ctx.save_for_backward(x, weight, up, kept)
        ctx.activation = activation
        return y

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dy):
        x, weight, up, kept = ctx.saved_tensors
        need = ctx.needs_input_grad
        grads = (None,) * 5
        if any(need[:5]):
            dx, dw, db, dup, dub = linear_backward(dy, x, weight, kept, up, ctx.activation, need[2], need[4], (need[0], need[1], need[3]))
            grads = dx, dw, db, dup, dub
        return (*grads, None, dy if need[6] else None, None)


class _ResidualNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, h, y, weight, bias, post_weight, post_bias, gate, residual_scale, block_scale, eps, centered):
        h_new, a, stats = residual_norm_forward(h, y, weight, bias, post_weight, post_bias, gate, residual_scale, block_scale, eps, centered)
        ctx.save_for_backward(h_new, y, stats, weight, post_weight, post_bias, gate)
        ctx.rest = residual_scale, block_scale, centered, bias is not None
        ctx.set_materialize_grads(False)
        return h_new, a

    @staticmethod
    @torch.autograd.function.once_differentiable
    def backward(ctx, dh_new, da):
        h_new, y, stats, weight, post_weight, post_bias, gate = ctx.saved_tensors
        if dh_new is None and da is None:
            return (None,) * 11
        return (*residual_norm_backward(dh_new, da, h_new, y, stats, weight, post_weight, post_bias, gate, *ctx.rest), None, None, None, None)


def norm(x, weight, bias=None, eps=1e-6, centered=False):
    """Differentiable norm_forward -> y."""
    return _Norm.apply(x, weight, bias, eps, centered)


def rotate(q, k, positions, table, interleaved=False):
    """Differentiable rotary -> (q, k)."""
    return _Rotary.apply(q, k, positions, table, interleaved)


def attention(q, k, v, cu_q, cu_k, causal=True, scale=None):
    """Differentiable attention_forward -> o."""
    return _Attention.apply(q, k, v, cu_q, cu_k, causal, scale)


def token_logprobs(hidden, weight, targets, temperature=1.0):
    """Differentiable token_logprobs_forward -> logp.  Its backward pass forms both gradients, also where only one is asked for."""
    return _TokenLogprobs.apply(hidden, weight, targets, temperature)


def linear(x, weight, bias=None, up=None, up_bias=None, activation="none", residual=None):
    """Differentiable linear_forward -> y."""
    keep = torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in (x, weight, bias, up, up_bias))
    return _Linear.apply(x, weight, bias, up, up_bias, activation, residual, keep)


def residual_norm(h, y, weight, bias=None, post_weight=None, post_bias=None, gate=None, residual_scale=1.0, block_scale=1.0, eps=1e-6, centered=False):
    """Differentiable residual_norm_forward -> (h_new, a)."""
    return _ResidualNorm.apply(h, y, weight, bias, post_weight, post_bias, gate, residual_scale, block_scale, eps, centered)
