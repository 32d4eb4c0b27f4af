"""CPU-side checks of the policy update's C entry points: what they refuse before anything touches a GPU, and workspace sizes."""
import math
import os
import random

import numpy as np
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


def norm_forward(lib, x=P, outer=4, inner=1, width=8, weight=P, bias=0, eps=1e-6, centered=0, dtype=F32, y=P, mean=0, rstd=P):
    return lib.rl_norm_forward(x, outer, inner, width, width, 0, weight, bias, eps, centered, dtype, y, mean, rstd, None)


def norm_backward(lib, dy=P, x=P, outer=4, inner=1, width=8, weight=P, mean=0, rstd=P, centered=0, dtype=F32, dx=P, dw=P, db=0, ws=P, nbytes=1 << 20):
    return lib.rl_norm_backward(dy, width, 0, x, outer, inner, width, width, 0, weight, mean, rstd, centered, dtype, dx, dw, db, ws, nbytes, None)


def rotary(lib, q=P, out=P, heads=2, k=P, k_out=P, k_heads=1, tokens=3, d=8, rot=8, positions=P, table=P, n=5, dtype=F32):
    return lib.rl_rotary(q, out, heads, 16, 8, 16, 8, k, k_out, k_heads, 8, 8, 8, 8, tokens, d, rot, 0, 0, positions, table, n, dtype, None)


def attention_forward(lib, q=P, k=P, v=P, cu_q=P, cu_k=P, n=1, tq=4, tk=4, nq=2, nk=1, d=8, scale=1.0, dtype=F32, o=P, lse=P):
    return lib.rl_attention_forward(q, 16, 8, k, 8, 8, v, 8, 8, cu_q, cu_k, n, tq, tk, nq, nk, d, scale, 1, dtype, o, lse, None)


def attention_backward(lib, do=P, q=P, k=P, v=P, o=P, lse=P, n=1, tq=4, tk=4, nq=2, nk=1, d=8, scale=1.0, dtype=F32, dq=P, dk=P, dv=P, ws=P, nbytes=1 << 20):
    return lib.rl_attention_backward(do, q, 16, 8, k, 8, 8, v, 8, 8, o, lse, P, P, n, tq, tk, nq, nk, d, scale, 1, dtype, dq, dk, dv, ws, nbytes, None)


def logprobs_forward(lib, h=P, rows=4, hidden=8, w=P, vocab=9, y=P, t=1.0, dtype=F32, lp=P, lse=P, ws=P, nbytes=1 << 40):
    return lib.rl_token_logprobs_forward(h, hidden, rows, hidden, w, vocab, y, t, dtype, lp, lse, ws, nbytes, None)


def logprobs_backward(lib, g=P, h=P, rows=4, hidden=8, w=P, vocab=9, y=P, lse=P, t=1.0, dtype=F32, dh=P, dw=P, ws=P, nbytes=1 << 40):
    return lib.rl_token_logprobs_backward(g, h, hidden, rows, hidden, w, vocab, y, lse, t, dtype, dh, dw, ws, nbytes, None)


REFUSED = [
    (norm_forward, [dict(x=0), dict(weight=0), dict(y=0), dict(rstd=0), dict(centered=1), dict(outer=-1), dict(inner=0), dict(width=0), dict(eps=-1.0),
                    dict(eps=math.nan), dict(dtype=2), dict(dtype=-1), dict(outer=1 << 31), dict(outer=1 << 30, inner=2)]),
    (norm_backward, [dict(dy=0), dict(x=0), dict(weight=0), dict(rstd=0), dict(dx=0), dict(dw=0), dict(ws=0), dict(ws=P + 2), dict(nbytes=4 * 8 * 4 - 1),
                     dict(db=P, nbytes=4 * 8 * 4), dict(centered=1), dict(dtype=7), dict(width=-3)]),
    (rotary, [dict(q=0), dict(out=0), dict(k=0), dict(k_out=0), dict(positions=0), dict(table=0), dict(table=P + 4), dict(d=0), dict(d=513), dict(rot=7),
              dict(rot=10), dict(rot=-2), dict(tokens=-1), dict(heads=0), dict(k_heads=-1), dict(n=0), dict(dtype=3)]),
    (attention_forward, [dict(q=0), dict(k=0), dict(v=0), dict(cu_q=0), dict(cu_k=0), dict(o=0), dict(lse=0), dict(n=-1), dict(n=0), dict(tq=-1), dict(tk=-1),
                         dict(nq=0), dict(nk=0), dict(nq=3, nk=2), dict(d=0), dict(d=129), dict(scale=math.nan), dict(scale=math.inf), dict(dtype=2)]),
    (attention_backward, [dict(do=0), dict(q=0), dict(k=0), dict(v=0), dict(o=0), dict(lse=0), dict(dq=0), dict(dk=0), dict(dv=0), dict(ws=0), dict(ws=P + 1),
                          dict(nbytes=4 * 2 * 2 * 4 - 1), dict(nq=3, nk=2), dict(scale=-math.inf)]),
    (logprobs_forward, [dict(h=0), dict(w=0), dict(y=0), dict(lp=0), dict(lse=0), dict(ws=0), dict(ws=P + 128), dict(nbytes=100), dict(rows=-1), dict(hidden=0),
                        dict(vocab=0), dict(vocab=1 << 23), dict(hidden=65537), dict(t=0.0), dict(t=-1.0), dict(t=math.nan), dict(t=math.inf), dict(t=1e-45), dict(dtype=2)]),
    (logprobs_backward, [dict(g=0), dict(h=0), dict(w=0), dict(y=0), dict(lse=0), dict(dh=0), dict(dw=0), dict(ws=0), dict(nbytes=100), dict(rows=0, dw=0),
                         dict(t=0.0), dict(dtype=5)]),
]


@pytest.mark.parametrize("call,changes", REFUSED, ids=[c.__name__ for c, _ in REFUSED])
def test_bad_arguments_are_refused_with_a_message(lib, call, changes):
    for change in changes:
        assert call(lib, **change) == -1, (call.__name__, change)
        assert lib.rl_last_error(), change


def test_calls_without_rows_succeed_without_a_gpu(lib):
    assert norm_forward(lib, outer=0, x=0, y=0) == 0
    assert rotary(lib, tokens=0, q=0, out=0) == 0
    assert attention_forward(lib, tq=0, q=0, o=0, lse=0) == 0
    assert attention_backward(lib, tq=0, tk=0, nbytes=0) == 0
    assert logprobs_forward(lib, rows=0, h=0) == 0


def test_workspaces_grow_with_the_problem_and_are_nothing_for_what_is_refused(lib):
    assert lib.rl_norm_workspace(10, 100, 0) == 4000 and lib.rl_norm_workspace(10, 100, 1) == 8000
    assert lib.rl_norm_workspace(10**9, 64, 0) == 512 * 64 * 4
    assert lib.rl_norm_workspace(-1, 64, 0) == lib.rl_norm_workspace(5, 0, 0) == 0
    assert lib.rl_attention_workspace(1000, 32) == 1000 * 32 * 8 and lib.rl_attention_workspace(-1, 2) == 0
    size = lib.rl_token_logprobs_workspace
    for bad in ((0, 8, 9, 0, 0), (4, 0, 9, 0, 0), (4, 8, 0, 0, 1), (4, 8, 9, 2, 1), (4, 8, 1 << 23, 0, 0)):
        assert size(*bad) == 0
    # a piece of the vocabulary, never all logits: 1 GB of gradients of logits, and what the rows need
    rows, hidden, vocab = 16384, 2560, 151936
    got = size(rows, hidden, vocab, BF16, 1)
    assert 1 << 30 <= got < (1 << 30) + (600 << 20) + 2 * rows * hidden * 8 < rows * vocab * 2
    for dtype in (F32, BF16):
        assert size(rows, hidden, vocab, dtype, 0) < rows * vocab * 2 / 8


def test_operators_refuse_tensors_that_are_not_on_a_gpu(lib):
    import torch

    from paper_2509_06980_amd import policy_ops as ops
    x, w, i = torch.ones(4, 2, 8), torch.ones(8), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: ops.norm_forward(x, w), lambda: ops.norm_backward(x, x, w, None, torch.ones(4, 2)), lambda: ops.rotary(x, None, i, torch.ones(5, 4, 2)),
                 lambda: ops.attention_forward(x, x, x, i[:2], i[:2]), lambda: ops.token_logprobs_forward(x[:, 0], torch.ones(9, 8), i)):
        with pytest.raises(rl.RolloutError) as e:
            call()
        assert e.value.code == -1
    table = ops.rotary_table(6, 8, theta=100.0, device="cpu")
    assert table.shape == (6, 4, 2) and np.allclose(table[5, 1], [math.cos(5 * 100 ** -0.25), math.sin(5 * 100 ** -0.25)])


def test_the_larger_workspace_of_attention(lib):
    least = lib.rl_attention_workspace(2000, 8)
    assert lib.rl_attention_fast_workspace(1, 2000, 2000, 8, 1, 128, 1) >= least + 2 * 2 * 2000 * 128 * 4      # two parts at least
    assert least <= lib.rl_attention_fast_workspace(1, 2000, 2000, 8, 8, 128, 1) < least + 2000 * 8 * 128 * 8 * 32
    assert lib.rl_attention_fast_workspace(64, 100_000, 100_000, 32, 8, 128, 1) == lib.rl_attention_workspace(100_000, 32)      # 25.6 MB, a multiple of 256
    assert lib.rl_attention_fast_workspace(1, 2000, 2000, 8, 3, 128, 1) == 0 and lib.rl_attention_fast_workspace(1, 10, 10, 8, 1, 129, 0) == 0
    assert lib.rl_attention_fast_workspace(0, 0, 0, 8, 1, 64, 0) == 0


def test_sizes_that_no_launch_takes_are_refused(lib):
    for call, changes in ((norm_forward, dict(width=(1 << 27) - 31)), (norm_backward, dict(width=(1 << 27) - 31, nbytes=1 << 50)), (attention_forward, dict(n=(1 << 24) - 4, tq=1 << 10)),
                          (attention_forward, dict(n=1 << 24)), (attention_backward, dict(n=1 << 23, tk=1 << 30, nbytes=1 << 50)),
                          (logprobs_forward, dict(rows=(1 << 24) - 255, nbytes=1 << 60)), (logprobs_backward, dict(rows=1 << 24, nbytes=1 << 60))):
        assert call(lib, **changes) == -1 and b"workspace" not in lib.rl_last_error(), (call.__name__, changes)
    # the largest that are taken
    assert lib.rl_token_logprobs_workspace((1 << 24) - 256, 8, 9, F32, 1) > 0 and lib.rl_token_logprobs_workspace((1 << 24) - 255, 8, 9, F32, 1) == 0
    assert lib.rl_attention_fast_workspace((1 << 24) - 17, 1 << 10, 1 << 10, 2, 1, 8, F32) > 0 and lib.rl_attention_fast_workspace((1 << 24) - 16, 1 << 10, 1 << 10, 2, 1, 8, F32) == 0
    assert lib.rl_norm_workspace(1, (1 << 27) - 32, 0) > 0 and lib.rl_norm_workspace(1, (1 << 27) - 31, 0) == lib.rl_norm_workspace(1 << 31, 8, 0) == 0
    assert norm_forward(lib, width=(1 << 27) - 32, outer=0) == 0


def test_loads_of_the_token_logprob_products_stay_inside_their_operands():
    # also where the last tile of dz begins behind the vocabulary (its columns go on to a multiple of 256: 60032 of 60000 in tiles of 64),
    # with few rows kept or none, in several pieces of the vocabulary and slices of it
    rng = random.Random(11)
    cases = [(300, 201, 4096, 60000), (300, 64, 20001 // 8 * 8, 20001), (700, 700, 8, 40003), (1100, 500, 64, 600), (4096, 2744, 2560, 151936), (8191, 4096, 1024, 151936),
             (30, 20, 4096, 151936), (64, 64, 768, 140_000), (1, 1, 8, 1), (1, 0, 8, 257), (16384, 9000, 2560, 151936), (2000, 1999, 65536, 3000)]
    for _ in range(200):
        rows = int(math.exp(rng.uniform(0, math.log(9000))))
        hidden, vocab = 8 * int(math.exp(rng.uniform(0, math.log(600)))), int(math.exp(rng.uniform(0, math.log(160_000))))
        cases.append((rows, rng.choice([0, 1, rows, rng.randint(0, rows)]), hidden, rng.choice([vocab, vocab // 256 * 256 + 1, vocab // 64 * 64 + 32])))
    taken = 0
    for rows, kept, hidden, vocab in cases:
        for bf16 in (False, True):
            for backward in (False, True):
                try:
                    beyond = rl.debug_token_logprob_loads(rows, kept, hidden, vocab, bf16, backward)
                except rl.RolloutError as e:
                    assert "other kernels" in str(e)
                    continue
                taken += 1
                assert beyond == (0, 0, 0), (rows, kept, hidden, vocab, bf16, backward, beyond)
    assert taken > 3.5 * len(cases)


def test_loads_of_sizes_that_the_products_do_not_take_are_refused(lib):
    for bad in ((0, 0, 8, 9, 1, 1), (4, 5, 8, 9, 1, 1), (4, -1, 8, 9, 1, 1), (4, 4, 6, 9, 1, 0), (4, 4, 8, 0, 0, 0), (1 << 23, 1, 4096, 9, 1, 1)):
        with pytest.raises(rl.RolloutError):
            rl.debug_token_logprob_loads(*bad)
