// Orthogonalised updates: Newton-Schulz products on whole stacks of matrices.
#include <cmath>

#include "product.h"

namespace {
using namespace product;

// =============================================================================================
// X = G / (|G| + eps), then in every step  A = X X^T, B = b A + c A^2, X <- a X + B X  (matrices with more rows than columns: A = X^T X, X <- a X +
// X B, so that A has the smaller of the two sizes and nothing is transposed).  Singular values s become p(s) = a s + b s^3 + c s^5, again and
// again; the singular vectors stay.
// A and B are symmetric: tiles on and under the diagonal are computed, the others are stored from them.
// Bound by the matrix units: 2560 x 9728 in five steps 1.38 ms (0.75 PFLOP/s of the products as computed, half of the symmetric ones), 28 x 2048 x 1024
// 1.84 ms; small stacks by the ten products' and joins' length one after another (3 x 512 x 256 169 us).
// fp32: everything in 32 bits.  bf16: the operands of the products are rounded to fp16 (11 bits instead of the 8 of bf16, at the same rate), X and A times powers of two
// that keep their elements in the middle of that range (Schedule).  What the rounding of X leaves is kept beside it in fp16 where more than one step follows, since a X
// carries the small singular values, which the steps enlarge (400 times in five of them) with whatever roundings are in them; the first X is exact as it is.  B's diagonal, near
// b + c towards the end, is kept in 32 bits.  Relative error of the result against 64 bits, of which its last rounding alone is 0.0017: 0.0017 to 0.0021 in five steps, to 0.0025 where
// a few elements or rows hold nearly all of |G|, to 0.003 in eight (fp16 alone: 0.02 for a matrix of 32 strong directions over a floor of noise; operands in bf16: 0.2).  Steps
// whose roundings would show more (schedule_of) and matrices with a side below 256 take the fp32 products, which cost nothing there: fp16's error is largest in small ones.
// =============================================================================================
const int kMostSteps = 64;
const int kNormShares = 1024;
const int kHalfFrom = 256;
// X goes past the caches where it would not stay in the last one of 256 MB with what else a step reads.  Past them | through them: 10 x 2048 x 1024 (42 MB) 759 | 737 us,
// 2560 x 9728 (50 MB) 1407 | 1377, 4096 x 8192 (67 MB) 2990 | 2969; 24 x 2048 x 1024 (101 MB) 1621 | 1644, 28 of them (117 MB) 1844 | 1866, 3 x 2560 x 9728 (149 MB) 4290 | 4429;
// 18 x 2048 x 1024 (75 MB), 2 x 4096 x 8192 (134 MB), 40 x 2048 x 1024 (168 MB) the same within 0.4 %; 20 x 2048 x 1024 (84 MB), at the border, 1325 | 1369.
const int64_t kStream = 80 << 20;
const float kLow = 2048.f;      // the low half of an element is kept times this
// fp16: X_t is kept times 2^(kTop - e_t), where none of its singular values is above 2^e_t: elements stay below 2^kTop (four times that fits) and as far above
// fp16's smallest as they can, however small |G| is beside eps and whatever the steps do to X.  A is that of X_t 2^-e_t, its size goes into the next two
// coefficients, and all three are kept times 2^-g_t.
const int kTop = 14;
struct Schedule {
  int steps;
  // singular values of X_t are at most 2^bound[t]; and at most 2^growth[t] times those of X_0, which may be any below 1 where eps outweighs |G|
  int16_t bound[kMostSteps + 1], growth[kMostSteps + 1], g[kMostSteps];
  float a[kMostSteps], b[kMostSteps], c[kMostSteps];      // times 2^-g
};

// Elements of a matrix in pieces of V, by all threads of a grid's first dimension: f(piece's row, its first column)
template <int V, typename F>
__device__ __forceinline__ void for_pieces(int rows, int width, F f) {
  const unsigned per = (unsigned)(width + V - 1) / V, n = (unsigned)rows * per;      // at most 2^30
  for (unsigned i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
    const unsigned r = i / per;
    f((int)r, (int)(i - r * per) * V);
  }
}
__device__ __forceinline__ double block_sum(double s, double* join) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if ((threadIdx.x & 63) == 0) join[threadIdx.x >> 6] = s;
  __syncthreads();
  return (join[0] + join[1]) + (join[2] + join[3]);
}
// Sums of squares of a matrix in shares: part[matrix][share], in 64 bits: no size of the elements overflows
template <typename T>
__global__ __launch_bounds__(256) void squares_kernel(const T* __restrict__ x, int64_t matrix, int64_t stride, int rows, int columns, int vec,
                                                      double* __restrict__ part) {
  __shared__ double join[4];
  const T* p = x + blockIdx.y * matrix;
  double s = 0.0;
  for_pieces<8>(rows, columns, [&](int r, int c) {
    float v[8];
    load_row<T, 8>(p + r * stride + c, vec, columns - c, v);
#pragma unroll
    for (int e = 0; e < 8; e++) s = fma((double)v[e], (double)v[e], s);
  });
  s = block_sum(s, join);
  if (threadIdx.x == 0) part[blockIdx.y * gridDim.x + blockIdx.x] = s;
}
// The products' first operand, rows of ld with zeros behind the last column: X in 32 bits; or in fp16 G times the power of two that brings |G| to 2^(kTop - 1) or above,
// exact for bf16 but for elements below 2^-30 |G|.  With it what a matrix's steps take, scales[matrix][step]: b and c for A as it is kept, and what takes a step's
// sums to the next X as it is kept, or the last one's to X: in two factors, where X is only just in a float's range and one of them would not be.
template <typename T, typename X>
__global__ __launch_bounds__(256) void normalise_kernel(const T* __restrict__ x, int64_t matrix, int64_t stride, int rows, int columns, int ld, int vec,
                                                        const double* __restrict__ part, int shares, double eps, Schedule schedule, X* __restrict__ to,
                                                        float4* __restrict__ scales) {
  constexpr bool HALF = sizeof(X) == 2;
  __shared__ double join[4];
  double s = 0.0;
  for (int i = threadIdx.x; i < shares; i += 256) s += part[blockIdx.y * shares + i];
  const double size = sqrt(block_sum(s, join)), norm = size + eps, inverse = 1.0 / norm;
  int power = 0;
  if constexpr (HALF) {
    const bool some = size > 0.0 && size < 1e300;
    if (some) power = kTop - 1 - ilogb(size);
    const int t = threadIdx.x;
    if (blockIdx.x == 0 && t < schedule.steps) {
      const int first = some ? ilogb(size * inverse) + 1 : 0;      // no singular value of X_0 is above 2^first
      auto e = [&](int t) { return min((int)schedule.bound[t], first + schedule.growth[t]); };
      const double unit = t > 0 ? ldexp(1.0, e(t)) : some ? ldexp(inverse, kTop - power) : 0.0, square = unit * unit;
      const int to_next = schedule.g[t] - kTop + (t + 1 == schedule.steps ? 0 : kTop - e(t + 1)), down = to_next + ilogb(unit) < -60 ? 64 : 0;
      const float nan = size < 1e300 && norm > 0.0 ? 0.f : __builtin_nanf("");      // X_0 is no number: neither is all that follows
      scales[blockIdx.y * kMostSteps + t] = make_float4((float)(schedule.b[t] * square) + nan, (float)(schedule.c[t] * square * square) + nan, (float)ldexp(unit, to_next + down) + nan, (float)ldexp(1.0, -down));
    }
  }
  const T* p = x + blockIdx.y * matrix;
  X* const out = to + (int64_t)blockIdx.y * rows * ld;
  constexpr int V = kPiece<X>;
  for_pieces<V>(rows, ld, [&](int r, int c) {
    float v[V];
    load_row<T, V>(p + r * stride + c, vec, columns - c, v);
#pragma unroll
    for (int e = 0; e < V; e++) v[e] = HALF ? ldexpf(v[e], power) : (float)((double)v[e] * inverse);
    store_row<X, V>(out + (int64_t)r * ld + c, true, V, v);
  });
}

// A = the sums (fp16: of X as it is kept, times 2^-2 kTop); rows of ld, zeros behind the last column
template <typename T>
struct Gram {
  static constexpr bool GATED = false, SYMMETRIC = true;
  static constexpr int V = kPiece<T>, SLICED = 4;
  T* out;
  int64_t matrix;
  int ld, n;
  struct Extra {};
  static constexpr bool UNROLL = false;
  __device__ __forceinline__ void fetch(int, int, int, Extra&) const {}
  __device__ __forceinline__ void across(int batch, int row, int col, float (&v)[V]) const {
#pragma unroll
    for (int e = 0; e < V; e++)
      if (col + e >= n) v[e] = 0.f;
    store_row<T, V>(out + batch * matrix + (int64_t)row * ld + col, true, V, v);
  }
  __device__ __forceinline__ void operator()(int batch, int row, int col, float (&v)[V], float (&)[V], const Extra&) const {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int e = 0; e < V; e++) v[e] *= 1.f / (1 << (2 * kTop));
    }
    across(batch, row, col, v);
  }
};
// B = b A + c A^2; fp16: its diagonal apart
template <typename T>
struct Polynomial {
  static constexpr bool GATED = false, SYMMETRIC = true;
  static constexpr int V = kPiece<T>, SLICED = sizeof(T) == 2 ? 0 : 4;
  const T* a;
  T* out;
  float* diagonal;
  int64_t matrix;
  int ld, n;
  float b, c;
  const float4* scales;      // fp16: of a step, in place of b and c
  struct Extra { float a[V]; };
  static constexpr bool UNROLL = false;
  __device__ __forceinline__ void fetch(int batch, int row, int col, Extra& x) const { load_row<T, V>(a + batch * matrix + (int64_t)row * ld + col, true, V, x.a); }
  __device__ __forceinline__ void across(int batch, int row, int col, float (&v)[V]) const {
#pragma unroll
    for (int e = 0; e < V; e++)
      if (col + e >= n) v[e] = 0.f;
    store_row<T, V>(out + batch * matrix + (int64_t)row * ld + col, true, V, v);
  }
  __device__ __forceinline__ void operator()(int batch, int row, int col, float (&v)[V], float (&)[V], const Extra& x) const {
    float first = b, second = c;
    if constexpr (sizeof(T) == 2) first = scales[batch * kMostSteps].x, second = scales[batch * kMostSteps].y;
#pragma unroll
    for (int e = 0; e < V; e++) v[e] = first * x.a[e] + second * v[e];
    asm volatile("" : "+v"(row), "+v"(col));      // or parts of their difference are kept in scalar registers, of which there are too few, through the products
    if (sizeof(T) == 2 && (unsigned)(row - col) < V) {
      float one = 0.f;
#pragma unroll
      for (int e = 0; e < V; e++) {
        one = col + e == row ? v[e] : one;
        v[e] = col + e == row ? 0.f : v[e];
      }
      diagonal[batch * padded(n) + row] = one;
    }
    across(batch, row, col, v);
  }
};
// X <- a X + B X; the last step's goes out in the caller's type
template <typename T>
struct Step {
  static constexpr bool GATED = false, SYMMETRIC = false;
  static constexpr int V = kPiece<T>, SLICED = 4;
  const T* x;              // the products' operand; fp16: X as it is kept, rounded,
  const _Float16* low;     // and what the rounding left, unless null
  T* next;
  _Float16* next_low;
  void* out;               // the last step's results, else null
  const float* diagonal;
  const float4* scales;    // fp16: of a step
  int64_t matrix;
  int rows, cols, ld, by_column, bf16_out, vec, stream;
  float a;
  struct Extra { u32x4 x, low; };      // as they lie in memory
  static constexpr bool UNROLL = true;
  __device__ __forceinline__ void fetch(int batch, int row, int col, Extra& e) const {
    const int64_t at = batch * matrix + (int64_t)row * ld + col;
    e.x = *(const u32x4*)(x + at);
    if (sizeof(T) == 2) {
      e.low = u32x4{0, 0, 0, 0};
      if (low) e.low = *(const u32x4*)(low + at);
    }
  }
  __device__ __forceinline__ void operator()(int batch, int row, int col, float (&v)[V], float (&)[V], const Extra& given) const {
    const int64_t at = batch * matrix + (int64_t)row * ld + col;
    const int left = cols - col;
    struct alignas(16) Pieces { T x[V]; };
    const Pieces hp = __builtin_bit_cast(Pieces, given.x);
    float h[V];
#pragma unroll
    for (int e = 0; e < V; e++) h[e] = wide(hp.x[e]);
    if constexpr (sizeof(T) == 2) {
      const Pieces lp = __builtin_bit_cast(Pieces, given.low);
      float d[V], l[V];
#pragma unroll
      for (int e = 0; e < V; e++) d[e] = 0.f, l[e] = wide(lp.x[e]);
      if (by_column) {
        load_row<float, V>(diagonal + (int64_t)batch * padded(cols) + col, true, V, d);
      } else {
        const float one = diagonal[(int64_t)batch * padded(rows) + row];
#pragma unroll
        for (int e = 0; e < V; e++) d[e] = one;
      }
      const float4 f = scales[batch * kMostSteps];
#pragma unroll
      for (int e = 0; e < V; e++) v[e] = fmaf(a, fmaf(l[e], 1.f / kLow, h[e]), fmaf(d[e], h[e], v[e])) * f.w * f.z;
    } else {
#pragma unroll
      for (int e = 0; e < V; e++) v[e] = fmaf(a, h[e], v[e]);
    }
    if (out) {
      const int64_t to = ((int64_t)batch * rows + row) * cols + col;
      if (bf16_out) return store_row<bf16_t, V>((bf16_t*)out + to, vec, left, v);
      return store_row<float, V>((float*)out + to, vec, left, v);
    }
#pragma unroll
    for (int e = 0; e < V; e++)
      if (e >= left) v[e] = 0.f;
    if (stream) store_row<T, V, true>(next + at, true, V, v);
    else store_row<T, V>(next + at, true, V, v);
    if constexpr (sizeof(T) == 2) {
      if (next_low) {
#pragma unroll
        for (int e = 0; e < V; e++) v[e] = (v[e] - (float)(_Float16)v[e]) * kLow;
        if (stream) store_row<_Float16, V, true>(next_low + at, true, V, v);
        else store_row<_Float16, V>(next_low + at, true, V, v);
      }
    }
  }
};

struct Stack {
  int count, rows, columns;
  int small() const { return std::min(rows, columns); }
};
template <typename T>
struct Layout {      // of the workspace
  int ld, ld_small;
  Plan gram, square, step;
  int64_t matrix, small, shares, scales, x, next, low, a, b, diagonal, part, bytes;
  explicit Layout(const Stack& n) {
    constexpr int V = kPiece<T>;
    const int s = n.small(), l = std::max(n.rows, n.columns);
    ld = (int)up(n.columns, V), ld_small = (int)up(s, V);
    gram = plan_of<T>({s, s, n.count, chunks<T>(l, 64), true, false, true, (float)sizeof(T), Gram<T>::SLICED});
    square = plan_of<T>({s, s, n.count, chunks<T>(s, 64), true, false, true, 2.f * sizeof(T), Polynomial<T>::SLICED});
    step = plan_of<T>({n.rows, n.columns, n.count, chunks<T>(s, 64), false, false, n.rows <= n.columns, 8.f, Step<T>::SLICED});
    matrix = (int64_t)n.rows * ld, small = (int64_t)s * ld_small;
    int64_t at = 0;
    auto take = [&](int64_t b) {
      const int64_t p = at;
      at += up(b, 256);
      return p;
    };
    const bool half = sizeof(T) == 2;
    shares = take((int64_t)n.count * kNormShares * sizeof(double));
    scales = half ? take((int64_t)n.count * kMostSteps * sizeof(float4)) : 0;
    x = take(n.count * matrix * sizeof(T));
    next = take(n.count * matrix * sizeof(T));
    low = half ? take(n.count * matrix * sizeof(T)) : 0;
    a = take(n.count * small * sizeof(T));
    b = take(n.count * small * sizeof(T));
    diagonal = half ? take((int64_t)n.count * padded(s) * sizeof(float)) : 0;
    part = take(std::max({part_bytes(step, n.rows, n.columns, n.count, false), part_bytes(gram, s, s, n.count, false), part_bytes(square, s, s, n.count, false)}));
    bytes = at;
  }
};

// The schedule of fp16 products; false where their roundings would show.  In 64 bits, of q(s) = a + b s^2 + c s^4, what a step multiplies a singular value s
// by, over 0 <= s <= m, the largest that can be.
//   Gain: by how much the steps enlarge the smallest singular values beside the largest.  Up to 2^15 the results are 0.0017 to 0.003 off, whatever the singular
//   values are (simulated on matrices whose rows or singular values fall by up to 10^8; eight steps of (3.4445, -4.775, 2.0315)).
//   Gap: by how much |X_t| may fall below its bound, for any |X_0|: up to 2^10 elements are 2^14 times fp16's smallest in matrices of 2^30 elements.
//   A q that changes its sign may bring |X_t| to nothing.
bool schedule_of(int steps, const float* coefficients, Schedule& to) {
  const int points = 64;
  double most = 1.0, gain = 1.0, gap = 1.0, growth = 0.0;
  to.steps = steps;
  to.bound[0] = to.growth[0] = 0;
  for (int t = 0; t < steps; t++) {
    const double a = coefficients[3 * t], b = coefficients[3 * t + 1], c = coefficients[3 * t + 2], m2 = most * most;
    auto factor = [&](double s2) { return a + s2 * (b + c * s2); };
    // where q and s q are largest: at the ends, or where 2 b + 4 c s^2 or a + 3 b s^2 + 5 c s^4 is 0
    double at[points + 4];      // s^2
    int n = 0;
    auto inside = [&](double s2) {
      if (s2 > 0.0 && s2 < m2) at[n++] = s2;
    };
    for (int i = 0; i <= points; i++) at[n++] = m2 * i * i / (points * points);
    if (c != 0.0) {
      inside(-b / (2.0 * c));
      const double root = 9.0 * b * b - 20.0 * a * c;
      if (root >= 0.0)
        for (double sign : {-1.0, 1.0}) inside((-3.0 * b + sign * std::sqrt(root)) / (10.0 * c));
    } else if (b != 0.0) {
      inside(-a / (3.0 * b));
    }
    std::sort(at, at + n);
    double largest = 0.0, next = 0.0;
    for (int i = 0; i < n; i++) largest = std::max(largest, std::fabs(factor(at[i]))), next = std::max(next, std::sqrt(at[i]) * std::fabs(factor(at[i])));
    if (!(next > 1e-30 && next < 1e36 && largest < 1e36)) return false;
    next *= 1.01;      // roundings
    double least = largest, fall = 1.0;
    for (int i = 0; i < n; i++) {
      const double q = factor(at[i]);
      if (q == 0.0 || (q > 0.0) != (a > 0.0)) return false;
      least = std::min(least, std::fabs(q));
      fall = std::max(fall, (at[i] > 0.0 ? std::min(largest, next / std::sqrt(at[i])) : largest) / least);
    }
    gain *= largest * most / next, gap *= fall;
    growth += std::log2(largest * 1.01);
    const int g = (int)std::ceil(std::log2(largest));
    to.g[t] = (int16_t)g;
    to.a[t] = (float)std::ldexp(a, -g), to.b[t] = (float)std::ldexp(b, -g), to.c[t] = (float)std::ldexp(c, -g);
    to.bound[t + 1] = (int16_t)std::ceil(std::log2(next)), to.growth[t + 1] = (int16_t)std::ceil(growth);
    most = next;
  }
  return gain <= 32768.0 && gap <= 1024.0;
}

template <typename T, typename G>
int orthogonalize(const G* x, int64_t x_matrix, int64_t x_stride, const Stack& n, int steps, const float* coefficients, const Schedule& schedule, float eps,
                  void* out, char* ws, hipStream_t s) {
  constexpr bool HALF = sizeof(T) == 2;
  const Layout<T> w(n);
  const int small = n.small(), rows = n.rows, columns = n.columns;
  const bool tall = rows > columns;
  double* const shares = (double*)(ws + w.shares);
  float4* const scales = (float4*)(ws + w.scales);
  const int64_t pieces = (int64_t)rows * (w.ld / kPiece<T>);
  const int n_shares = (int)std::min<int64_t>((pieces + 1023) / 1024, std::max(std::min(2048 / n.count, kNormShares), 1));
  T *now = (T*)(ws + w.x), *next = (T*)(ws + w.next);
  _Float16* const low = (_Float16*)(ws + w.low);
  if (!probe) {
    const bool whole = aligned16(x) && columns % 8 == 0 && x_stride % 8 == 0 && x_matrix % 8 == 0;
    squares_kernel<G><<<dim3(n_shares, n.count), 256, 0, s>>>(x, x_matrix, x_stride, rows, columns, whole, shares);
    normalise_kernel<G, T><<<dim3((unsigned)std::min<int64_t>((pieces + 511) / 512, std::max(2048 / n.count, 1)), n.count), 256, 0, s>>>(
        x, x_matrix, x_stride, rows, columns, w.ld, whole, shares, n_shares, (double)eps, schedule, now, scales);
  }
  T *const a = (T*)(ws + w.a), *const b = (T*)(ws + w.b);
  float* const diagonal = (float*)(ws + w.diagonal);
  for (int t = 0; t < steps; t++) {
    const float* c = coefficients + 3 * t;
    const bool last = t == steps - 1;
    Product<T> p{};
    p.segments = 1, p.batches = n.count, p.part = (float*)(ws + w.part);
    {
      const Operand<T> o{now, w.ld, w.matrix, 0, rows, rows, w.ld, w.ld, n.count * w.matrix};
      p.a = p.b = o;
      p.k = p.last_k = tall ? rows : w.ld, p.rows = p.cols = small;
      const Gram<T> e{a, w.small, w.ld_small, small};
      if (tall) launch<T, true, true>(p, w.gram, e, s);
      else launch<T, false, false>(p, w.gram, e, s);
    }
    const Operand<T> square{a, w.ld_small, w.small, 0, small, small, w.ld_small, w.ld_small, n.count * w.small};
    p.a = p.b = square, p.k = p.last_k = w.ld_small;
    launch<T, false, false>(p, w.square, Polynomial<T>{a, b, diagonal, w.small, w.ld_small, small, c[1], c[2], scales + t}, s);
    {
      const Operand<T> o{now, w.ld, w.matrix, 0, rows, rows, w.ld, w.ld, n.count * w.matrix};
      Operand<T> poly = square;
      poly.p = b;
      p.rows = rows, p.cols = columns;
      Step<T> e{now, HALF && t > 0 && !last ? low : nullptr, next, HALF && t + 2 < steps ? low : nullptr, last ? out : nullptr, diagonal,
                scales + t, w.matrix, rows, columns, w.ld, tall, std::is_same<G, bf16_t>::value, 0, n.count * w.matrix * (int64_t)sizeof(T) > kStream, HALF ? schedule.a[t] : c[0]};
      e.vec = columns % kPiece<T> == 0 && columns % (16 / sizeof(G)) == 0 && aligned16(out);
      p.k = p.last_k = w.ld_small;
      if (tall) {
        p.a = o, p.b = poly;
        launch<T, false, false>(p, w.step, e, s);
      } else {
        p.a = poly, p.b = o;
        launch<T, false, true>(p, w.step, e, s);
      }
    }
    std::swap(now, next);
  }
  return probe ? RL_OK : launched();
}

bool takes_half(const Stack& n, int dtype, int steps, const float* coefficients, Schedule& schedule) {
  return dtype == RL_DTYPE_BF16 && n.small() >= kHalfFrom && schedule_of(steps, coefficients, schedule);
}
const char* stack_argument(int32_t count, int32_t rows, int32_t columns, int32_t dtype) {
  if (dtype != RL_DTYPE_F32 && dtype != RL_DTYPE_BF16) return "dtype is RL_DTYPE_F32 or RL_DTYPE_BF16";
  if (count < 0 || count > 65535 || rows < 1 || columns < 1 || rows > (1 << 20) - 8 || columns > (1 << 20) - 8) return "count, rows or columns out of range";
  const int64_t l = std::max(rows, columns), s = std::min(rows, columns);
  if ((l + 8) * (s + 8) > (1ll << 30) - (1 << 20)) return "matrices of more than 2^30 - 2^20 elements";
  return nullptr;
}
}  // namespace

extern "C" int64_t rl_orthogonalize_workspace(int32_t count, int32_t rows, int32_t columns, int32_t dtype) {
  if (stack_argument(count, rows, columns, dtype) || count == 0) return 0;
  const Stack n{count, rows, columns};
  const int64_t full = Layout<float>(n).bytes;
  return dtype == RL_DTYPE_BF16 && n.small() >= kHalfFrom ? std::max(full, Layout<_Float16>(n).bytes) : full;
}

extern "C" int rl_orthogonalize(const void* d_x, int64_t matrix_stride, int64_t row_stride, int32_t count, int32_t rows, int32_t columns, int32_t steps,
                                const float* coefficients, float eps, int32_t dtype, void* d_out, void* d_workspace, int64_t workspace_bytes, void* stream) {
  if (const char* m = stack_argument(count, rows, columns, dtype)) return rl_fail(RL_E_ARG, m);
  if (steps < 1 || steps > kMostSteps || !coefficients) return rl_fail(RL_E_ARG, "1 to 64 steps with three coefficients each");
  for (int i = 0; i < 3 * steps; i++)
    if (!std::isfinite(coefficients[i])) return rl_fail(RL_E_ARG, "a coefficient is infinite or no number");
  if (!(eps >= 0.f)) return rl_fail(RL_E_ARG, "eps is negative or no number");
  if (count == 0) return RL_OK;
  if (!d_x || !d_out || !d_workspace) return rl_fail(RL_E_ARG, "null pointer");
  if (workspace_bytes < rl_orthogonalize_workspace(count, rows, columns, dtype)) return rl_fail(RL_E_ARG, "workspace smaller than rl_orthogonalize_workspace says");
  if ((uintptr_t)d_workspace & 255) return rl_fail(RL_E_ARG, "workspace not aligned to 256 bytes");
  const Stack n{count, rows, columns};
  hipStream_t s = (hipStream_t)stream;
  char* ws = (char*)d_workspace;
  Schedule schedule{};
  if (dtype == RL_DTYPE_F32) return orthogonalize<float>((const float*)d_x, matrix_stride, row_stride, n, steps, coefficients, schedule, eps, d_out, ws, s);
  if (takes_half(n, dtype, steps, coefficients, schedule))
    return orthogonalize<_Float16>((const bf16_t*)d_x, matrix_stride, row_stride, n, steps, coefficients, schedule, eps, d_out, ws, s);
  return orthogonalize<float>((const bf16_t*)d_x, matrix_stride, row_stride, n, steps, coefficients, schedule, eps, d_out, ws, s);
}

extern "C" int rl_debug_orthogonalize_loads(int32_t count, int32_t rows, int32_t columns, int32_t dtype, int64_t* out) {
  if (!out || count < 1) return rl_fail(RL_E_ARG, "null pointer or no matrices");
  Probe found{};
  probe = &found;
  const float c[3] = {3.4445f, -4.7750f, 2.0315f};
  char* const at = (char*)(1ll << 44);      // nothing is there: only distances count
  const int rc = rl_orthogonalize(at, (int64_t)rows * columns, columns, count, rows, columns, 1, c, 1e-7f, dtype, at + (1ll << 42), at + (2ll << 42),
                                  rl_orthogonalize_workspace(count, rows, columns, dtype), nullptr);
  probe = nullptr;
  if (rc != RL_OK) return rc;
  out[0] = found.buffers, out[1] = found.offsets, out[2] = found.products;
  return RL_OK;
}
