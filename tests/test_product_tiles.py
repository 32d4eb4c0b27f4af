"""Tiles of the products of linear layers and orthogonalised updates, by their host arithmetic, compiled alone: what a tile's loads may reach wherever it lies, products by
plans that no kernel is built for, and whether the check of a call's loads finds mistakes."""
import os
import shutil
import subprocess

import pytest

HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_06980_amd", "csrc")
PROGRAM = r"""
#include <cstdio>
#include "kernels_orthogonal.hip"
int rl_fail(int code, const char*) { return code; }
int main() {
  using namespace product;
  // rows of 40 of 48 elements
  for (int n : {1, 7, 64, 100, 300})
    for (int rows : {64, 128, 256})
      for (int at = 0; at <= 4 * rows; at += rows)
        for (bool strided : {false, true}) {
          const int width = strided ? n : 40, count = strided ? 40 : n;      // strided: 40 rows of n elements
          const int64_t ld = strided ? n + 8 : 48, all = ((int64_t)(count - 1) * ld + width) * 2;
          const Reach r = reach_of<bf16_t>(strided, ld, count, width, at, rows);
          if (r.begin < 0 || r.bytes == 0 || r.begin * 2 + (int64_t)r.bytes > all) printf("reach %d %d %d %d: %ld %u of %ld\n", n, rows, at, strided, (long)r.begin, r.bytes, (long)all);
        }
  // every plan, built or not
  int products = 0;
  for (int mb = 1; mb <= 5; mb++)
    for (int nb = 1; nb <= 5; nb++)
      for (int size : {1, 100, 129, 192, 300, 1000}) {
        Probe found{};
        probe = &found;
        const _Float16* at = (const _Float16*)(1ll << 44);
        const int ld = (size + 7) / 8 * 8;
        Product<_Float16> p{};
        p.a = p.b = Operand<_Float16>{at, ld, 0, 0, size, size, ld, ld, (int64_t)size * ld};
        p.k = p.last_k = ld, p.rows = p.cols = size, p.segments = p.batches = 1;
        launch<_Float16, false, false>(p, Plan{mb, nb, 1}, Gram<_Float16>{}, nullptr);
        launch<_Float16, false, false>(p, Plan{mb, nb, 1}, Step<_Float16>{}, nullptr);
        p.a.width = p.b.width = p.a.last_width = p.b.last_width = size, p.k = p.last_k = size;
        launch<_Float16, true, true>(p, Plan{mb, nb, 1}, Gram<_Float16>{}, nullptr);
        p.a.width = p.a.last_width = ld;
        launch<_Float16, false, true>(p, Plan{mb, nb, 1}, Step<_Float16>{}, nullptr);
        probe = nullptr;
        products += found.products;
        if (found.buffers > 0 || found.offsets > 0) printf("plan %d %d of %d: %ld %ld\n", mb, nb, size, (long)found.buffers, (long)found.offsets);
      }
  printf("products %d\n", products);
}
"""

# the operands of a gated layer, 300 x 72 -> 200, and of its dx, with one mistake each: bytes that the check finds too many
MISTAKES = r"""
#include <cstdio>
#include "kernels_linear.hip"
int rl_fail(int code, const char*) { return code; }
int main() {
  using namespace product;
  const bf16_t* const w = (const bf16_t*)(2ll << 42);
  const bf16_t* const u = (const bf16_t*)(1ll << 42);
  for (int rows : {300, 7}) {
    auto forward = [&](const char* name, auto change) {
      Probe found{};
      probe = &found;
      Product<bf16_t> p{};
      p.a = {(const bf16_t*)(3ll << 42), 80, 0, 0, rows, rows, 72, 72, (rows - 1) * 80 + 72};
      p.b = {w, 80, 0, 0, 200, 200, 72, 72, 199 * 80 + 72};
      p.b2 = u - w, p.u = u, p.u_elements = 199 * 80 + 72;
      p.k = p.last_k = 72, p.rows = rows, p.cols = 200, p.segments = p.batches = 1;
      change(p);
      if (rows > kFewRows) launch<bf16_t, false, false>(p, Plan{4, 4, 1}, Finish<bf16_t, true, false>{}, nullptr);
      else launch_few_rows<bf16_t>(p, Finish<bf16_t, true, false>{}, nullptr);
      probe = nullptr;
      printf("%s %ld\n", name, (long)found.buffers);
    };
    forward("none", [](auto&) {});
    forward("w for u", [](auto& p) { p.b2 = 0; });
    forward("behind u", [](auto& p) { p.b2 += 3; });
    forward("before u", [](auto& p) { p.b2 -= 5; });
    forward("less of u", [](auto& p) { p.u_elements -= 2; });
    forward("less of w", [](auto& p) { p.b.elements -= 2; });
    forward("less of x", [](auto& p) { p.a.elements -= 4; });
  }
  auto dx = [&](const char* name, auto change) {
    Probe found{};
    probe = &found;
    Product<bf16_t> p{};
    p.a = {(const bf16_t*)(3ll << 42), 200, 0, 300 * 200, 300, 300, 200, 200, 2 * 300 * 200};
    p.b = {w, 72, 0, u - w, 200, 200, 72, 72, 200 * 72};
    p.u = u, p.u_elements = 200 * 72;
    p.k = p.last_k = 200, p.rows = 300, p.cols = 72, p.segments = 2, p.batches = 1;
    change(p);
    launch<bf16_t, false, true>(p, Plan{4, 4, 1}, Finish<bf16_t, false, true>{}, nullptr);
    probe = nullptr;
    printf("%s %ld\n", name, (long)found.buffers);
  };
  dx("none", [](auto&) {});
  dx("w for u", [](auto& p) { p.b.segment = 0; });
  dx("behind u", [](auto& p) { p.b.segment += 7; });
  dx("less of u", [](auto& p) { p.u_elements -= 1; });
  dx("behind dz", [](auto& p) { p.a.segment += 4; });
}
"""


def _output(tmp_path, text):
    source, program = tmp_path / "tiles.hip", tmp_path / "tiles"
    source.write_text(text)
    subprocess.run([HIPCC, "--offload-host-only", "-O1", "-std=c++17", "-w", "-Wl,--unresolved-symbols=ignore-all", f"-I{CSRC}", "-o", program, source], check=True, capture_output=True, timeout=300)
    return subprocess.run([program], capture_output=True, text=True, timeout=60, check=True).stdout


@pytest.mark.skipif(not shutil.which(HIPCC), reason="no compiler")
def test_no_tile_reaches_behind_its_operand(tmp_path):
    out = _output(tmp_path, PROGRAM)
    assert out == f"products {25 * 6 * 4}\n", out[:2000]


@pytest.mark.skipif(not shutil.which(HIPCC), reason="no compiler")
def test_the_check_of_the_loads_finds_mistakes(tmp_path):
    forward = ["none 0", f"w for u {(1 << 42) + 2 * (200 - 1) * 80 + 2 * 72 - 2 * (199 * 80 + 72)}", "behind u 6", "before u 10", "less of u 4", "less of w 4", "less of x 8"]
    dx = ["none 0", f"w for u {1 << 42}", "behind u 14", "less of u 2", "behind dz 8"]
    assert _output(tmp_path, MISTAKES).splitlines() == 2 * forward + dx
