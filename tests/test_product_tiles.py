"""Tiles of the products of linear layers and orthogonalised updates, by their host arithmetic, compiled alone: what a tile's loads may reach wherever it lies, and products by
plans that no kernel is built for."""
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


@pytest.mark.skipif(not shutil.which(HIPCC), reason="no compiler")
def test_no_tile_reaches_behind_its_operand(tmp_path):
    source, program = tmp_path / "tiles.hip", tmp_path / "tiles"
    source.write_text(PROGRAM)
    subprocess.run([HIPCC, "--offload-host-only", "-O1", "-std=c++17", "-w", "-Wl,--unresolved-symbols=ignore-all", f"-I{CSRC}", "-o", program, source], check=True, capture_output=True, timeout=300)
    out = subprocess.run([program], capture_output=True, text=True, timeout=60).stdout
    assert out == f"products {25 * 6 * 4}\n", out[:2000]
