"""Every kernel that calls of linear layers and orthogonalised updates can come to: the list of calls below reaches all that a million drawn calls do, by the calls' own planning;
on the GPU each call of the list against 64 bits."""
import os
import shutil
import subprocess

import pytest
import torch

import paper_2509_06980_amd as rl
from test_kernel_resources import _kernels
from test_product_tiles import CSRC, HIPCC

BF, FP = torch.bfloat16, torch.float32
FAR = 1 << 20      # elements from one row of x to the next: dW takes its rows in segments of 2 GiB
ACTIVATIONS = ["none", "relu", "silu", "gelu", "gelu_tanh"]
# rows, inner, outer, stride of x (0: inner), gated, bias, activation, residual (0: of the call's type), type, wanted (0: the forward call alone; else 1 dx + 2 dweight + 4 dup)
LINEAR = [
    (1, 40, 40, 0, False, True, "none", None, BF, 3), (1, 40, 242, 0, False, False, "gelu", 0, FP, 1), (1, 47, 38, 0, False, True, "none", FP, FP, 3),
    (1, 48, 35, 0, False, False, "none", None, FP, 0), (1, 1409, 5472, 0, False, False, "silu", 0, BF, 3), (1, 4320, 1014, 0, True, True, "none", None, BF, 3),
    (1, 9168, 136, 0, True, True, "relu", None, FP, 7), (1, 11944, 835, 0, False, False, "none", None, BF, 3), (17, 34, 40, 0, False, True, "gelu", 0, BF, 0),
    (17, 567, 41, 0, True, False, "none", 0, BF, 0), (17, 848, 48, 0, False, False, "none", None, BF, 0), (18, 664, 40, 0, False, True, "none", 0, BF, 0),
    (18, 688, 40, 0, False, True, "relu", FP, BF, 0), (18, 1488, 6560, 0, False, False, "none", None, BF, 0), (18, 1778, 4912, 0, False, True, "silu", None, BF, 0),
    (19, 256, 33, 0, False, False, "gelu_tanh", 0, FP, 0), (20, 46, 36, 0, False, False, "none", None, BF, 0), (23, 41, 40, 0, False, False, "none", None, FP, 0),
    (65, 1152, 6444, 0, False, True, "none", None, FP, 0), (73, 1049, 9840, 0, False, False, "none", None, FP, 0), (76, 560, 13576, 0, False, True, "silu", None, FP, 0),
    (129, 3763, 8485, 0, False, False, "gelu", 0, BF, 0), (134, 8358, 2240, 0, True, False, "none", 0, BF, 5), (137, 17344, 3208, 0, False, False, "none", None, BF, 0),
    (197, 36, 17912, 0, True, True, "none", 0, BF, 0), (248, 12951, 65, 0, True, False, "relu", FP, FP, 6), (249, 48, 36, 0, True, True, "none", FP, FP, 3),
    (517, 2072, 2975, FAR, False, False, "none", None, FP, 3), (575, 12312, 69, FAR, False, True, "none", FP, FP, 3),
    (627, 72, 17533, FAR, False, True, "gelu", FP, FP, 3), (632, 40, 40, FAR, False, False, "none", FP, FP, 3), (641, 40, 40, 0, True, False, "none", FP, BF, 7),
    (1028, 160, 16440, FAR, True, False, "none", FP, BF, 6), (1054, 48, 37, FAR, False, True, "none", None, BF, 3),
    (1061, 6512, 104, FAR, True, False, "gelu_tanh", None, BF, 7), (1132, 264, 10972, FAR, False, False, "relu", 0, BF, 3),
    (1772, 40, 2389, FAR, True, False, "relu", FP, BF, 7), (2055, 4496, 35, 0, False, True, "none", FP, BF, 3), (3776, 12048, 160, FAR, False, True, "none", 0, BF, 2),
    (10921, 2652, 145, 0, False, True, "none", 0, BF, 0), (10969, 4668, 130, 0, False, False, "none", None, BF, 0), (11576, 144, 4696, 0, False, True, "gelu", 0, BF, 3),
    (13230, 2336, 65, 0, True, True, "gelu_tanh", FP, BF, 0), (16487, 2864, 136, 0, False, False, "silu", 0, BF, 0),
    (16664, 40, 333, 0, False, False, "none", None, FP, 0), (16664, 2535, 165, 0, False, False, "none", FP, BF, 0),
    (22067, 288, 40, 0, True, False, "silu", None, BF, 5), (24582, 240, 279, 0, False, False, "none", FP, BF, 0), (25332, 304, 297, 0, False, True, "gelu", FP, BF, 0),
    (25495, 77, 260, 0, False, True, "none", FP, FP, 1), (26082, 66, 133, 0, True, False, "none", 0, FP, 7), (33904, 41, 46, 0, False, True, "none", 0, BF, 0),
    (34178, 48, 130, 0, False, True, "none", 0, BF, 0), (34493, 40, 35, 0, False, False, "gelu", FP, BF, 1), (35244, 36, 152, 0, False, False, "none", None, BF, 0),
    (35776, 40, 41, 0, False, False, "none", None, BF, 0), (38771, 40, 138, 0, False, True, "gelu_tanh", FP, BF, 0), (51191, 104, 33, 0, True, False, "none", FP, FP, 7),
    (52416, 40, 72, 0, False, False, "gelu_tanh", None, FP, 0), (52787, 264, 144, 0, False, False, "none", None, BF, 0),
    (53627, 45, 88, 0, False, True, "none", None, FP, 0),
]
# count, rows, columns, type
ORTHOGONAL = [
    (1, 20, 20, FP), (1, 21, 20, FP), (1, 244, 246, BF), (1, 257, 1915, BF), (1, 261, 243, FP), (1, 737, 749, BF), (1, 803, 738, BF), (1, 1154, 1027, BF), (1, 1310, 1354, BF),
    (1, 1794, 256, BF), (2, 4958, 257, FP), (3, 260, 7241, BF), (4, 2908, 258, BF), (11, 257, 833, FP), (22, 2216, 20, BF), (26, 399, 487, BF), (26, 807, 197, BF),
    (27, 775, 262, BF), (28, 585, 597, FP), (31, 681, 581, FP), (33, 391, 387, BF), (35, 20, 1371, FP), (38, 322, 347, FP),
]
SWEEP = 1_000_000


def calls_of(case):
    """The forward calls, with and without what is kept for the backward call, and the backward call."""
    rows, inner, outer, stride, gated, bias, activation, residual, dt, wanted = case
    last = f"{[None, 0, FP].index(residual)} {int(dt == BF)}"
    rest = f"linear {rows} {inner} {outer} {stride} {int(gated)} {int(bias)} {ACTIVATIONS.index(activation)}"
    yield f"{rest} 0 {last} 0"
    if gated or activation != "none":
        yield f"{rest} 1 {last} 0"
    if wanted:
        yield f"{rest} 0 {last} {wanted}"


@pytest.mark.skipif(not shutil.which(HIPCC), reason="no compiler")
def test_every_kernel_that_a_call_can_come_to_is_in_the_list(tmp_path):
    program, source = tmp_path / "forms", os.path.join(os.path.dirname(os.path.abspath(__file__)), "product_forms.hip")
    subprocess.run([HIPCC, "--offload-host-only", "-O1", "-std=c++17", "-w", "-Wl,--unresolved-symbols=ignore-all", f"-I{CSRC}", "-o", program, source], check=True, capture_output=True, timeout=300)
    calls = [f"sweep {SWEEP}"] + [c for case in LINEAR for c in calls_of(case)] + [f"orthogonalize {n} {r} {c} {int(dt == BF)}" for n, r, c, dt in ORTHOGONAL]
    out = subprocess.run([program], input="\n".join(calls) + "\n", capture_output=True, text=True, timeout=120, check=True).stdout
    assert "refused" not in out
    found = [line.split(" ", 1) for line in out.splitlines()]
    reachable, listed = {name for n, name in found if n == "0"}, {name for n, name in found if n != "0"}
    assert len(reachable) > 100 and not reachable - listed, sorted(reachable - listed)
    # and no kernel is built that none comes to
    if not os.path.exists(rl.LIB_PATH):
        from paper_2509_06980_amd import build
        build.build()
    built = [k for k in _kernels(rl.LIB_PATH)["product", ()] if "product_kernel" in k[".name"]]
    assert len(built) == len({name.split("[")[1] for name in reachable if not name.startswith("few rows")})


@pytest.mark.gpu
@pytest.mark.parametrize("case", LINEAR, ids=lambda c: "-".join(str(v).removeprefix("torch.") for v in c))
def test_linear_by_every_kernel(case):
    from test_update_operators import gen, linear_case, linear_check
    rows, inner, outer, stride, gated, bias, activation, residual, dt, wanted = case
    made, dy = linear_case(gen(rows + 3 * inner), rows, inner, outer, dt, gated, bias, dt if residual == 0 else residual)
    if stride:
        x = torch.empty(rows, stride, dtype=dt, device="cuda")[:, :inner]
        made["x"] = x.copy_(made["x"])
    linear_check(made, dy, activation, tuple(bool(wanted & bit) for bit in (1, 2, 4)))


@pytest.mark.gpu
@pytest.mark.parametrize("count,rows,columns,dt", ORTHOGONAL)
def test_orthogonalize_by_every_kernel(count, rows, columns, dt):
    from paper_2509_06980_amd import policy_ops as ops
    from test_update_operators import gen, matrices, orthogonal_check
    x = matrices(gen(rows + columns), count, rows, columns, dt, "strong")
    orthogonal_check(x, ops.orthogonalize(x), dt == BF and min(rows, columns) >= 256)
