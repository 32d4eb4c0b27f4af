"""The policy update's operators on torch tensors: norms, rotary positions, attention over packed trajectories and log-probs
of tokens, forward and backward (the calls of include/rl_rollout.h under the same names), and as functions of torch.autograd.

Tensors live on one GPU; work is enqueued on torch's current stream and nothing waits for it.  Arguments are checked here
and in the library; what is refused raises RolloutError.
"""
import math

import torch

from .binding import RolloutError, load_library

_DTYPES = {torch.float32: 0, torch.bfloat16: 1}


def _refuse(message):
    raise RolloutError(-1, message)


def _call(name, device, *args):
    """name(*args, stream) on `device`'s current stream."""
    lib = load_library()
    index = device.index
    if index is not None and index != torch.cuda.current_device():
        with torch.cuda.device(index):
            rc = getattr(lib, name)(*args, torch.cuda.current_stream().cuda_stream)
    else:
        rc = getattr(lib, name)(*args, torch._C._cuda_getCurrentRawStream(torch.cuda.current_device()))
    if rc != 0:
        raise RolloutError(rc, lib.rl_last_error().decode())


def _same(first, **others):
    """All tensors on the GPU of `first`, and of its type."""
    if first.dtype not in _DTYPES:
        _refuse(f"float32 or bfloat16 tensors, got {first.dtype}")
    if first.device.type != "cuda":
        _refuse("tensors have to be on the GPU")
    for name, t in others.items():
        if t is not None and (t.dtype != first.dtype or t.device != first.device):
            _refuse(f"{name} is {t.dtype} on {t.device}, the others are {first.dtype} on {first.device}")
    return _DTYPES[first.dtype]


def _of_type(dtype, device, **others):
    for name, t in others.items():
        if t.dtype != dtype or t.device != device or not t.is_contiguous():
            _refuse(f"{name} has to be a contiguous {dtype} tensor on {device}")


def _ptr(t):
    return 0 if t is None else t.data_ptr()


def _workspace(nbytes, device):
    return torch.empty(max(nbytes, 1), dtype=torch.uint8, device=device)


# ---- norms ---------------------------------------------------------------------------------------------------------
def _rows(x):
    """(tensor, outer, inner, outer stride, inner stride) of x's rows; a copy only where two strides cannot say where they are."""
    if x.dim() and (x.stride(-1) == 1 or x.shape[-1] == 1):
        if x.is_contiguous():
            w = x.shape[-1]
            return x, (x.numel() // w if w else 0), 1, w, 0
        if x.dim() == 2:
            return x, x.shape[0], 1, x.stride(0), 0
        if x.dim() == 3:
            return x, x.shape[0], x.shape[1], x.stride(0), x.stride(1)
    return _rows(x.contiguous())


def norm_forward(x, weight, bias=None, eps=1e-6, centered=False):
    """RMS norm (layer norm where `centered`) over the last dimension -> (y, mean, rstd); y is contiguous, mean (None in the RMS
    form) and rstd have x's shape without its last dimension."""
    dt = _same(x, weight=weight, bias=bias)
    if x.dim() < 1 or weight.shape != x.shape[-1:] or (bias is not None and bias.shape != weight.shape):
        _refuse("weight and bias have to have the length of a row")
    if not weight.is_contiguous() or (bias is not None and not bias.is_contiguous()):
        _refuse("weight and bias have to be contiguous")
    x, outer, inner, so, si = _rows(x)
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    rstd = torch.empty(x.shape[:-1], dtype=torch.float32, device=x.device)
    mean = torch.empty_like(rstd) if centered else None
    _call("rl_norm_forward", x.device, x.data_ptr(), outer, inner, x.shape[-1], so, si, weight.data_ptr(), _ptr(bias), eps,
          int(centered), dt, y.data_ptr(), _ptr(mean), rstd.data_ptr())
    return y, mean, rstd


def norm_backward(dy, x, weight, mean, rstd, centered=False, biased=None):
    """Gradients of norm_forward -> (dx, dweight, dbias); dbias is None unless `biased` (None: where `centered`)."""
    biased = centered if biased is None else biased
    dt = _same(x, dy=dy, weight=weight)
    if dy.shape != x.shape or x.dim() < 1 or weight.shape != x.shape[-1:] or not weight.is_contiguous():
        _refuse("dy has x's shape, weight the length of a row")
    _of_type(torch.float32, x.device, rstd=rstd, **({"mean": mean} if centered else {}))
    if rstd.shape != x.shape[:-1] or (centered and mean.shape != rstd.shape):
        _refuse("mean and rstd are one number a row")
    x, outer, inner, so, si = _rows(x)
    dy, d_outer, d_inner, do, di = _rows(dy)
    if d_inner != inner:      # one of the two is strided: the other's rows in the same two steps
        n = max(inner, d_inner)
        w = x.shape[-1]
        outer, (so, si), (do, di) = outer * inner // n, (so, si) if inner == n else (n * w, w), (do, di) if d_inner == n else (n * w, w)
        inner = n
    width = x.shape[-1]
    dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    dweight = torch.empty_like(weight)
    dbias = torch.empty_like(weight) if biased else None
    nbytes = load_library().rl_norm_workspace(outer * inner, width, int(biased))
    ws = _workspace(nbytes, x.device)
    _call("rl_norm_backward", x.device, dy.data_ptr(), do, di, x.data_ptr(), outer, inner, width, so, si, weight.data_ptr(),
          _ptr(mean) if centered else 0, rstd.data_ptr(), int(centered), dt, dx.data_ptr(), dweight.data_ptr(), _ptr(dbias),
          ws.data_ptr(), nbytes)
    return dx, dweight, dbias


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
    Results are new contiguous tensors unless q_out / k_out say where (they may be q and k themselves)."""
    dt = _same(q, k=k, q_out=q_out, k_out=k_out)
    if q.dim() != 3 or (k is not None and (k.dim() != 3 or k.shape[0] != q.shape[0] or k.shape[2] != q.shape[2])):
        _refuse("q and k are [tokens, heads, head_dim]")
    _of_type(torch.int32, q.device, positions=positions)
    _of_type(torch.float32, q.device, table=table)
    tokens, heads, d = q.shape
    if positions.shape != (tokens,) or table.dim() != 3 or table.shape[2] != 2 or 2 * table.shape[1] > d:
        _refuse("one position a token, and a table [positions, rot_dim / 2, 2] with rot_dim at most head_dim")

    def both(x, out):
        if x.stride(-1) != 1 and d > 1:
            x = x.contiguous()
        if out is None:
            out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        elif out.shape != x.shape or (out.stride(-1) != 1 and d > 1):
            _refuse("an output has its input's shape and contiguous heads")
        return x, out, (x.data_ptr(), out.data_ptr(), x.shape[1], x.stride(0), x.stride(1), out.stride(0), out.stride(1))

    q, q_out, q_args = both(q, q_out)
    k_args = (0, 0, 0, 0, 0, 0, 0)
    if k is not None:
        k, k_out, k_args = both(k, k_out)
    _call("rl_rotary", q.device, *q_args, *k_args, tokens, d, 2 * table.shape[1], int(interleaved), int(inverse),
          positions.data_ptr(), table.data_ptr(), table.shape[0], dt)
    return q_out, k_out


# ---- attention over packed trajectories ------------------------------------------------------------------------------
def _packed(q, k, v, cu_q, cu_k, scale):
    dt = _same(q, k=k, v=v)
    if q.dim() != 3 or k.dim() != 3 or v.shape != k.shape or k.shape[2] != q.shape[2]:
        _refuse("q is [tokens, heads, head_dim], k and v [tokens, KV heads, head_dim]")
    _of_type(torch.int32, q.device, cu_q=cu_q, cu_k=cu_k)
    if cu_q.dim() != 1 or cu_q.shape != cu_k.shape or cu_q.shape[0] < 1:
        _refuse("cu_q and cu_k are offsets of the same sequences")
    q, k, v = (t if t.stride(-1) == 1 or t.shape[-1] == 1 else t.contiguous() for t in (q, k, v))
    strides = [(t.data_ptr(), t.stride(0), t.stride(1)) for t in (q, k, v)]
    shape = (cu_q.data_ptr(), cu_k.data_ptr(), cu_q.shape[0] - 1, q.shape[0], k.shape[0], q.shape[1], k.shape[1], q.shape[2],
             q.shape[2] ** -0.5 if scale is None else scale)
    return dt, (q, k, v), strides, shape


def attention_forward(q, k, v, cu_q, cu_k, causal=True, scale=None):
    """Attention of packed sequences -> (o [tokens, heads, head_dim], lse [heads, tokens]); see rl_attention_forward.  Tokens of
    no sequence keep what the new tensors happen to hold.  scale None: head_dim^-1/2."""
    dt, kept, strides, shape = _packed(q, k, v, cu_q, cu_k, scale)
    o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    lse = torch.empty((q.shape[1], q.shape[0]), dtype=torch.float32, device=q.device)
    _call("rl_attention_forward", q.device, *strides[0], *strides[1], *strides[2], *shape, int(causal), dt, o.data_ptr(),
          lse.data_ptr())
    return o, lse


def attention_backward(do, q, k, v, o, lse, cu_q, cu_k, causal=True, scale=None):
    """Gradients of attention_forward -> (dq, dk, dv), contiguous."""
    dt, kept, strides, shape = _packed(q, k, v, cu_q, cu_k, scale)
    _same(q, do=do, o=o)
    if do.shape != q.shape or o.shape != q.shape or lse.shape != (q.shape[1], q.shape[0]):
        _refuse("do and o have q's shape, lse is [heads, tokens]")
    do, o = do.contiguous(), o.contiguous()
    _of_type(torch.float32, q.device, lse=lse)
    dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
    nbytes = load_library().rl_attention_workspace(q.shape[0], q.shape[1])
    ws = _workspace(nbytes, q.device)
    _call("rl_attention_backward", q.device, do.data_ptr(), *strides[0], *strides[1], *strides[2], o.data_ptr(), lse.data_ptr(),
          *shape, int(causal), dt, dq.data_ptr(), dk.data_ptr(), dv.data_ptr(), ws.data_ptr(), nbytes)
    return dq, dk, dv


# ---- log-probs of tokens ---------------------------------------------------------------------------------------------
def _head(hidden, weight, targets):
    dt = _same(hidden, weight=weight)
    if hidden.dim() != 2 or weight.dim() != 2 or weight.shape[1] != hidden.shape[1] or targets.shape != hidden.shape[:1]:
        _refuse("hidden is [rows, hidden], weight [vocab, hidden], targets [rows]")
    if not weight.is_contiguous():
        _refuse("weight has to be contiguous")
    _of_type(torch.int32, hidden.device, targets=targets)
    return dt, hidden if hidden.stride(1) == 1 or hidden.shape[1] == 1 else hidden.contiguous()


def token_logprobs_forward(hidden, weight, targets, temperature=1.0):
    """Log-probs of `targets` under softmax(hidden weight^T / temperature), without keeping the logits -> (logp, lse), float32.
    Rows with a negative target take no part (0)."""
    dt, hidden = _head(hidden, weight, targets)
    rows, width = hidden.shape
    logp = torch.empty(rows, dtype=torch.float32, device=hidden.device)
    lse = torch.empty_like(logp)
    nbytes = load_library().rl_token_logprobs_workspace(rows, width, weight.shape[0], dt, 0)
    ws = _workspace(nbytes, hidden.device)
    _call("rl_token_logprobs_forward", hidden.device, hidden.data_ptr(), hidden.stride(0), rows, width, weight.data_ptr(),
          weight.shape[0], targets.data_ptr(), temperature, dt, logp.data_ptr(), lse.data_ptr(), ws.data_ptr(), nbytes)
    return logp, lse


def token_logprobs_backward(dlogp, hidden, weight, targets, lse, temperature=1.0):
    """Gradients of token_logprobs_forward's logp -> (dhidden, dweight)."""
    dt, hidden = _head(hidden, weight, targets)
    _of_type(torch.float32, hidden.device, dlogp=dlogp, lse=lse)
    if dlogp.shape != targets.shape or lse.shape != targets.shape:
        _refuse("dlogp and lse are one number a row")
    rows, width = hidden.shape
    dhidden = torch.empty((rows, width), dtype=hidden.dtype, device=hidden.device)
    dweight = torch.empty_like(weight)
    nbytes = load_library().rl_token_logprobs_workspace(rows, width, weight.shape[0], dt, 1)
    ws = _workspace(nbytes, hidden.device)
    _call("rl_token_logprobs_backward", hidden.device, dlogp.data_ptr(), hidden.data_ptr(), hidden.stride(0), rows, width,
          weight.data_ptr(), weight.shape[0], targets.data_ptr(), lse.data_ptr(), temperature, dt, dhidden.data_ptr(),
          dweight.data_ptr(), ws.data_ptr(), nbytes)
    return dhidden, dweight


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
    """Differentiable token_logprobs_forward -> logp."""
    return _TokenLogprobs.apply(hidden, weight, targets, temperature)
