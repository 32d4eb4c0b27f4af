// The kernels that calls launch for their products, by the calls' own planning, without a GPU.  Reads calls from the standard input, one a line:
//   linear ROWS INNER OUTER X_STRIDE GATED BIAS ACTIVATION KEPT RESIDUAL(0 none, 1 of dtype, 2 float32) DTYPE WANTED(0: the forward call; else 1 dx + 2 dweight + 4 dup)
//   orthogonalize COUNT ROWS COLUMNS DTYPE
// and writes their kernels, one a line, behind the number of the call; "sweep N" stands for N calls drawn over the sizes that are allowed and fit a GPU.
#include <cstdio>
#include <cstring>
#include <iostream>
#include <random>
#include <set>
#include <sstream>
#include <string>

#include "kernels_linear.hip"
#include "kernels_orthogonal.hip"

int rl_fail(int, const char* message) {
  printf("refused: %s\n", message);
  return -1;
}

struct Call {
  bool linear;
  int v[11];
};
std::set<std::string> kernels_of(const Call& c) {
  product::Probe found{};
  product::probe = &found;
  auto place = [&](int i, bool wanted = true) { return wanted ? (char*)(1ll << 44) + ((int64_t)i << 42) : nullptr; };
  const int* v = c.v;
  if (c.linear) {
    const int rows = v[0], inner = v[1], outer = v[2], gated = v[4], act = v[6], dtype = v[9], wanted = v[10];
    const int64_t stride = v[3] ? v[3] : inner, bytes = rl_linear_workspace(rows, inner, outer, gated, dtype, wanted != 0, 0);
    if (wanted)
      rl_linear_backward(place(1), outer, dtype, place(2), stride, rows, inner, place(3), inner, place(4, gated), inner, outer, act, (float*)place(5), dtype, place(6, wanted & 1),
                         place(7, wanted & 2), place(8, wanted & 4), nullptr, nullptr, place(9), bytes, nullptr);
    else
      rl_linear_forward(place(1), stride, rows, inner, place(2), inner, place(3, gated), inner, outer, place(4, v[5]), nullptr, act, place(5, v[8]), outer, v[8] == 2 ? 0 : dtype, dtype,
                        place(6), (float*)place(7, v[7]), place(8), bytes, nullptr);
  } else {
    const float twice[6] = {3.4445f, -4.7750f, 2.0315f, 3.4445f, -4.7750f, 2.0315f};
    rl_orthogonalize(place(1), (int64_t)v[1] * v[2], v[2], v[0], v[1], v[2], 2, twice, 1e-7f, v[3], place(2), place(3), rl_orthogonalize_workspace(v[0], v[1], v[2], v[3]), nullptr);
  }
  product::probe = nullptr;
  if (found.buffers > 0 || found.offsets > 0) printf("refused: loads reach %ld bytes too far\n", (long)std::max(found.buffers, found.offsets));
  std::set<std::string> names;
  for (int i = 0; i < found.n_forms; i++) {
    const char* name = found.forms[i].kernel;
    names.insert(std::string(strstr(name, "few_rows") ? "few rows " : found.forms[i].segments > 1 ? "segments " : "") + strstr(name, "[T"));
  }
  return names;
}
Call drawn(std::mt19937_64& r) {
  auto log = [&](double lo, double hi) { return (int)std::lround(lo * std::exp(std::log(hi / lo) * (double)(r() >> 11) * 0x1p-53)); };
  for (;;) {
    Call c{};
    c.linear = r() % 3 > 0;
    int* v = c.v;
    if (c.linear) {
      v[0] = log(1, 60000), v[1] = log(1, 20000), v[2] = log(1, 20000);
      for (int i : {1, 2})
        if (r() % 2) v[i] = (v[i] + 7) / 8 * 8;
      v[4] = r() % 3 == 0, v[5] = r() % 2, v[6] = r() % 2 ? 0 : 1 + (int)(r() % 4), v[8] = (int)(r() % 3), v[9] = (int)(r() % 2);
      v[10] = r() % 2 ? 0 : v[4] ? 1 + (int)(r() % 7) : 1 + (int)(r() % 3);
      v[7] = !v[10] && (v[6] || v[4]) && r() % 2;
      if (r() % 20 == 0) v[0] = log(300, 5000), v[1] = (v[1] + 7) / 8 * 8, v[3] = 1 << 20;
      if ((double)v[0] * v[1] * v[2] < 3e11) return c;
    } else {
      v[0] = log(1, 40), v[1] = log(1, 9000), v[2] = log(1, 9000), v[3] = (int)(r() % 2);
      const double s = std::min(v[1], v[2]), l = std::max(v[1], v[2]);
      if (v[0] * (2 * s * s * l + s * s * s) < 5e12) return c;
    }
  }
}
int main() {
  std::string line;
  std::mt19937_64 r(1);
  for (int n = 0; std::getline(std::cin, line); n++) {
    std::istringstream words(line);
    std::string what;
    words >> what;
    std::set<std::string> names;
    if (what == "sweep") {
      int64_t calls = 0;
      words >> calls;
      while (calls-- > 0)
        for (const std::string& name : kernels_of(drawn(r))) names.insert(name);
    } else {
      Call c{what == "linear", {}};
      for (int& x : c.v) words >> x;
      names = kernels_of(c);
    }
    for (const std::string& name : names) printf("%d %s\n", n, name.c_str());
  }
}
