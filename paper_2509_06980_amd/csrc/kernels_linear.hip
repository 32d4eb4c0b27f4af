// Linear layers of the policy update, forward and backward: a product with bias, activation, a second matrix that gates it and a residual in its
// epilogue.
#include "product.h"

namespace {
using namespace product;

// =============================================================================================
// z = x W^T + b, u = x U^T + ub (gated);  y = act(z) [u] [+ r].
// Backward: dz = dy act'(z) [u], du = dy act(z);  dx = dz W [+ du U], dW = dz^T x, db = sum over rows of dz, dr = dy.
// z and u are kept in 32 bits for the backward call: rounded to bf16 they alone would make the gradients of a gated layer 0.0029 off (relative; the
// roundings of dz and of the gradient itself 0.0024).  dz and du are rounded to the weights' type once, as the operands that they become.
// Many rows are bound by the matrix units: 4096 rows, 9728 -> 2560 with a residual, forward and backward 616 us (0.99 PFLOP/s): 239 forward, 12 for dz, 231
// for dx, 214 for dW.  2744 rows, 2560 -> 9728 twice, gated by silu: 892 us (0.92 PFLOP/s): 384, 70, 271 and 13 to join slices, 249 (profiled, which takes
// 5 to 10 % longer).
// Few by the weights' bytes.
// =============================================================================================
struct Activated {      // act(z) and act'(z)
  float value, slope;
};
__device__ __forceinline__ float sigmoid(float z) { return 1.f / (1.f + __expf(-z)); }
template <bool SLOPE>
__device__ __forceinline__ Activated activate(float z, int act) {
  switch (act) {
    case RL_ACT_RELU: return {z > 0.f || z != z ? z : 0.f, z > 0.f ? 1.f : 0.f};
    case RL_ACT_SILU: {
      const float p = sigmoid(z), v = p == 0.f ? 0.f : z * p;      // z = -infinity: 0
      return {v, SLOPE ? p + v * (1.f - p) : 0.f};
    }
    case RL_ACT_GELU: {
      const float p = 0.5f * erfcf(-0.70710678118654752f * z), v = p == 0.f ? 0.f : z * p;
      const float e = SLOPE ? __expf(-0.5f * z * z) * 0.39894228040143268f : 0.f;
      return {v, SLOPE ? p + (e == 0.f ? 0.f : z * e) : 0.f};
    }
    case RL_ACT_GELU_TANH: {
      const float c = 0.79788456080286536f, k = 0.044715f, q = 1.f / (1.f + __expf(-2.f * c * (z + k * z * z * z)));      // (1 + tanh) / 2
      const float v = q == 0.f ? 0.f : z * q, s = 2.f * q * (1.f - q);
      return {v, SLOPE ? q + (s == 0.f ? 0.f : z * s * c * (1.f + 3.f * k * z * z)) : 0.f};
    }
    default: return {z, 1.f};
  }
}
template <bool SLOPE, int N>
__device__ __forceinline__ void activate_all(const float (&z)[N], int act, float (&value)[N], float (&slope)[N]) {
  auto all = [&](auto a) {
#pragma unroll
    for (int e = 0; e < N; e++) {
      const Activated s = activate<SLOPE>(z[e], decltype(a)::value);
      value[e] = s.value;
      if (SLOPE) slope[e] = s.slope;
    }
  };
  switch (act) {      // once for all N
    case RL_ACT_RELU: all(std::integral_constant<int, RL_ACT_RELU>()); break;
    case RL_ACT_SILU: all(std::integral_constant<int, RL_ACT_SILU>()); break;
    case RL_ACT_GELU: all(std::integral_constant<int, RL_ACT_GELU>()); break;
    case RL_ACT_GELU_TANH: all(std::integral_constant<int, RL_ACT_GELU_TANH>()); break;
    default: all(std::integral_constant<int, RL_ACT_NONE>());
  }
}

// What follows a product's sums; PLAIN: they are rounded and stored, nothing else.  Results go past the caches, which keeps the operands there: 4096 rows x 2560 -> 9728 196 us,
// 210 through them, 8192 rows 337 and 365, 512 rows 37 and 40, up to 128 rows the same.  The next operator pays for it where it would have found them in the caches: gate, up, down and
// the norm behind them of 2744 rows 495 and 487 us, of 64 rows 57.8 and 56.3, of 4096 rows the same, of 8192 rows 1308 and 1341.
// SHORT: no activation and nothing kept.
template <typename T, bool GATED_, bool PLAIN, bool SHORT = PLAIN>
struct Finish {
  static constexpr bool GATED = GATED_, SYMMETRIC = false, UNROLL = SHORT;
  static constexpr int SLICED = 16;
  static constexpr int V = kPiece<T>;
  void* y;
  int64_t y_batch;               // elements from one batch's results to the next's
  int cols, vec;                 // vec: results and what joins them lie in whole 16 bytes
  int act, wide;                 // wide: residual and results in 32 bits
  const T *bias, *up_bias;
  const void* residual;
  int64_t residual_stride;
  float* kept;

  struct None {};
  struct Joins { float r[V]; };
  using Extra = std::conditional_t<PLAIN, None, Joins>;
  __device__ __forceinline__ void fetch(int, int row, int col, Extra& x) const {
    if constexpr (!PLAIN) {
      if (!residual) return;
      const int64_t at = (int64_t)row * residual_stride + col;
      if (wide) load_row<float, V>((const float*)residual + at, vec, cols - col, x.r);
      else load_row<T, V>((const T*)residual + at, vec, cols - col, x.r);
    }
  }
  __device__ __forceinline__ void operator()(int batch, int row, int col, float (&v)[V], float (&u)[V], const Extra& joins) const {
    const int left = cols - col;
    if constexpr (!PLAIN) {
      float x[V];
      if (bias) {
        load_row<T, V>(bias + col, vec, left, x);
#pragma unroll
        for (int e = 0; e < V; e++) v[e] += x[e];
      }
      if constexpr (GATED) {
        if (up_bias) {
          load_row<T, V>(up_bias + col, vec, left, x);
#pragma unroll
          for (int e = 0; e < V; e++) u[e] += x[e];
        }
      }
      if constexpr (!SHORT) {
        if (kept) {
          float* const k = kept + (int64_t)row * cols * (GATED ? 2 : 1) + col;
          store_row<float, V, true>(k, vec, left, v);
          if constexpr (GATED) store_row<float, V, true>(k + cols, vec, left, u);
        }
        activate_all<false, V>(v, act, v, x);
      }
      if constexpr (GATED) {
#pragma unroll
        for (int e = 0; e < V; e++) v[e] *= u[e];
      }
      if (residual) {
#pragma unroll
        for (int e = 0; e < V; e++) v[e] += joins.r[e];
      }
      if (wide) return store_row<float, V, true>((float*)y + (int64_t)row * cols + col, vec, left, v);
    }
    store_row<T, V, true>((T*)y + batch * y_batch + (int64_t)row * cols + col, vec, left, v);
  }
};

// ---- few rows ---------------------------------------------------------------------------------------------------------------------
// Up to 16 rows: bound by the weights' bytes.  A workgroup takes 16 rows of W (and of U) and all rows of x; its waves share k, operands go from memory straight
// into registers (weights as the row operand of 16x16x32 instructions, fp32 16x16x4; a lane's 16 bytes are 8 or 4 k of one row), and the waves'
// sums are added in LDS in a fixed order.  x comes from the caches.  What a block of 16 rows has too many reads the last row again and is not stored.
// One row x 4096 x 2560 with a residual: 6.9 us (3.0 TB/s, of it 2 us to begin and end), by the tiles of many rows 14.  From 17 rows on those tiles are faster (37 rows x 2560 x 9728, gated: 29 us with
// the slices' sums; this way, three blocks of rows a workgroup, 50).
const int kFewRows = 16, kFewWaves = 8;
// Where a lane's reads of an operand begin, in elements: row `row`, or the last one in place of those behind it
__host__ __device__ __forceinline__ int64_t few_rows_begin(int row, int rows, int64_t ld) { return (int64_t)(row < rows ? row : rows - 1) * ld; }
template <typename T, typename EPI>
__global__ __launch_bounds__(64 * kFewWaves) void few_rows_kernel(const T* __restrict__ x, int64_t x_ld, const T* __restrict__ w, int64_t w_ld, int64_t second,
                                                                  int rows, int k, int outer, EPI epi) {
  constexpr int E = 16 / sizeof(T), KS = 4 * E, M = EPI::GATED ? 2 : 1, U = 8, V = kPiece<T>;
  __shared__ float sums[M][kFewWaves][16][17];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n0 = blockIdx.x * 16, r = lane & 15, kl = lane / 16 * E;
  const T* const wp = w + few_rows_begin(n0 + r, outer, w_ld) + kl;
  const T* const xp = x + few_rows_begin(r, rows, x_ld) + kl;
  f32x4 acc[M];
#pragma unroll
  for (int m = 0; m < M; m++) acc[m] = f32x4{0.f, 0.f, 0.f, 0.f};
  const int steps = (k + KS - 1) / KS, begin = slice_begin(wave, kFewWaves, steps), end = slice_begin(wave + 1, kFewWaves, steps);
  for (int s = begin; s < end; s += U) {
    u32x4 a[U][M], b[U];
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int at = (s + u) * KS;
      b[u] = u32x4{0, 0, 0, 0};
#pragma unroll
      for (int m = 0; m < M; m++) a[u][m] = u32x4{0, 0, 0, 0};
      if (s + u < end && at + kl < k) {
#pragma unroll
        for (int m = 0; m < M; m++) a[u][m] = *(const u32x4*)(wp + (m ? second : 0) + at);
        b[u] = *(const u32x4*)(xp + at);
      }
    }
#pragma unroll
    for (int u = 0; u < U; u++)
#pragma unroll
      for (int m = 0; m < M; m++) {
        if constexpr (sizeof(T) == 2) {
          acc[m] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[u][m]), __builtin_bit_cast(bf16x8, b[u]), acc[m], 0, 0, 0);
        } else {
          const f32x4 p = __builtin_bit_cast(f32x4, a[u][m]), q = __builtin_bit_cast(f32x4, b[u]);
#pragma unroll
          for (int e = 0; e < 4; e++) acc[m] = __builtin_amdgcn_mfma_f32_16x16x4f32(p[e], q[e], acc[m], 0, 0, 0);
        }
      }
  }
#pragma unroll
  for (int m = 0; m < M; m++)
#pragma unroll
    for (int e = 0; e < 4; e++) sums[m][wave][r][lane / 16 * 4 + e] = acc[m][e];
  __syncthreads();
  constexpr int PIECES = 16 / V;
  const int i = threadIdx.x, row = i / PIECES, c = i % PIECES * V;
  if (row >= rows || n0 + c >= outer) return;
  float v[V], u[V];
#pragma unroll
  for (int e = 0; e < V; e++) {
    v[e] = u[e] = 0.f;
#pragma unroll
    for (int q = 0; q < kFewWaves; q++) {
      v[e] += sums[0][q][row][c + e];
      if constexpr (M == 2) u[e] += sums[1][q][row][c + e];
    }
  }
  typename EPI::Extra extra;
  epi.fetch(0, row, n0 + c, extra);
  epi(0, row, n0 + c, v, u, extra);
}
template <typename T, typename EPI>
void launch_few_rows(const Product<T>& p, const EPI& epi, hipStream_t s) {
  const int groups = (p.cols + 15) / 16;
  if (probe) {      // a row's pieces begin before k, which is whole pieces
    probe->form(__PRETTY_FUNCTION__, 1);
    auto look = [&](int64_t from, int last, int rows, int64_t ld, int64_t elements) {
      probe->buffers = std::max({probe->buffers, -from * (int64_t)sizeof(T), (from + few_rows_begin(last, rows, ld) + p.k - elements) * (int64_t)sizeof(T)});
    };
    look(0, 15, p.rows, p.a.ld, p.a.elements);
    look(0, groups * 16 - 1, p.cols, p.b.ld, p.b.elements);
    if (EPI::GATED) look(p.b.p + p.b2 - p.u, groups * 16 - 1, p.cols, p.b.ld, p.u_elements);
    return;
  }
  few_rows_kernel<T, EPI><<<groups, 64 * kFewWaves, 0, s>>>(p.a.p, p.a.ld, p.b.p, p.b.ld, p.b2, p.rows, p.k, p.cols, epi);
}

// ---- rows of an operand in whole 16 bytes: [rows][ld], zeros behind `width` -----------------------------------------------------------
// up to three at once
template <typename T>
struct Copies {
  struct One {
    const T* x;
    int64_t stride, rows;
    int width, ld;
    T* to;
  } one[3];
  int n = 0;
  int64_t most = 0;      // elements of the largest
};
template <typename T>
__global__ __launch_bounds__(256) void copy_rows_kernel(Copies<T> copies) {
  const typename Copies<T>::One& c = copies.one[blockIdx.y];
  const int64_t n = c.rows * c.ld;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t r = i / c.ld;
    const int j = (int)(i - r * c.ld);
    c.to[i] = j < c.width ? c.x[r * c.stride + j] : T(0);
  }
}

// ---- dz and du, and their sums over rows --------------------------------------------------------------------------------------
// A thread takes 8 columns of every fourth row of a workgroup's share of rows.  Bound by memory: 2744 x 9728 of a gated layer reads dy, z and u and writes dz and
// du, 374 MB, in 71 us (5.3 TB/s, z and u partly still in the last cache).
const int kGradColumns = 512, kGradShares = 256;
template <typename T>
struct Gradient {
  const void* dy;
  int64_t dy_stride;
  int wide, act, rows, cols, mats, ldz, vec, per_share;
  const float* kept;              // null: no activation
  T* dz;                          // [mats][rows][ldz]; null: sums alone
  float* part;                    // [shares][mats][cols]; null: no sums
};
template <typename T, bool GATED>
__global__ __launch_bounds__(256) void gradient_kernel(Gradient<T> g) {
  constexpr int V = 8, M = GATED ? 2 : 1;
  __shared__ float join[3][64 * 8 + 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = (blockIdx.x * 64 + lane) * V, left = g.cols - c;
  const int first = blockIdx.y * g.per_share, end = min(g.rows, first + g.per_share);
  float sum[M][V];
#pragma unroll
  for (int m = 0; m < M; m++)
#pragma unroll
    for (int e = 0; e < V; e++) sum[m][e] = 0.f;
  if (left > 0) {
    for (int r = first + wave; r < end; r += 4) {
      float d[V], z[V], u[V], value[V], slope[V];
      const bool vec = g.vec && left >= V;
      if (g.wide) load_row<float, V>((const float*)g.dy + r * g.dy_stride + c, vec, left, d);
      else load_row<T, V>((const T*)g.dy + r * g.dy_stride + c, vec, left, d);
      if (g.kept) {
        const float* k = g.kept + (int64_t)r * g.cols * M + c;
        load_row<float, V>(k, vec, left, z);
        if constexpr (GATED) load_row<float, V>(k + g.cols, vec, left, u);
        activate_all<true, V>(z, g.act, value, slope);
#pragma unroll
        for (int e = 0; e < V; e++) {
          if constexpr (GATED) {
            u[e] = d[e] * slope[e] * u[e];
            z[e] = d[e] * value[e];
          } else {
            u[e] = d[e] * slope[e];
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < V; e++) u[e] = d[e];
      }
#pragma unroll
      for (int e = 0; e < V; e++) {
        sum[0][e] += u[e];
        if constexpr (GATED) sum[1][e] += z[e];
      }
      if (g.dz) {      // rows of whole pieces: zeros behind the last column
#pragma unroll
        for (int e = 0; e < V; e++)
          if (e >= left) u[e] = z[e] = 0.f;
        T* to = g.dz + (int64_t)r * g.ldz + c;
        store_row<T, V>(to, true, V, u);
        if constexpr (GATED) store_row<T, V>(to + (int64_t)g.rows * g.ldz, true, V, z);
      }
    }
  }
  if (!g.part) return;
#pragma unroll
  for (int m = 0; m < M; m++) {
    if (wave > 0) {
#pragma unroll
      for (int e = 0; e < V; e++) join[wave - 1][e * 64 + lane] = sum[m][e];
    }
    __syncthreads();
    if (wave == 0) {
      float* to = g.part + ((int64_t)blockIdx.y * M + m) * g.cols + c;
#pragma unroll
      for (int e = 0; e < V; e++)
        if (e < left) to[e] = ((sum[m][e] + join[0][e * 64 + lane]) + join[1][e * 64 + lane]) + join[2][e * 64 + lane];
    }
    __syncthreads();
  }
}
template <typename T>
__global__ __launch_bounds__(256) void share_sum_kernel(const float* __restrict__ part, int shares, int mats, int cols, T* __restrict__ a, T* __restrict__ b) {
  const int c = blockIdx.x * 256 + threadIdx.x, m = blockIdx.y;
  T* const to = m ? b : a;
  if (c >= cols || !to) return;
  float s = 0.f;
#pragma unroll 8
  for (int i = 0; i < shares; i++) s += part[((int64_t)i * mats + m) * cols + c];
  to[c] = narrow<T>(s);
}
template <typename T>
__global__ __launch_bounds__(256) void fill_kernel(T* to, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) to[i] = T(0);
}
unsigned blocks_for(int64_t n) { return (unsigned)std::min<int64_t>((n + 255) / 256, 8192); }

// ---- host ---------------------------------------------------------------------------------------------------------------------------
constexpr int64_t kAlign = 256;
struct Room {      // pieces of a workspace
  char* base;
  int64_t used = 0;
  void* take(int64_t bytes) {
    void* p = base + used;
    used += up(bytes, kAlign);
    return p;
  }
};
struct Shape {
  int rows, inner, outer, mats;
};
template <typename T>
struct In {      // an operand as the products take it
  const T* p;
  int64_t ld;
  int width;
  int64_t elements;
};
// Whole 16 bytes a row, offsets within a tile in 31 bits
template <typename T>
bool direct(const void* p, int64_t stride, int width) {
  constexpr int V = 16 / sizeof(T);
  return aligned16(p) && stride % V == 0 && width % V == 0 && stride >= width && stride <= (1 << 20);
}
template <typename T>
int64_t copy_bytes(int64_t rows, int width) { return up(rows * up(width, 16 / sizeof(T)) * (int64_t)sizeof(T), kAlign); }
template <typename T>
In<T> copied(const void* p, int64_t stride, int64_t rows, int width, Room& room, Copies<T>& copies) {
  const int ld = (int)up(width, 16 / sizeof(T));
  T* to = (T*)room.take(rows * ld * (int64_t)sizeof(T));
  copies.one[copies.n++] = {(const T*)p, stride, rows, width, ld, to};
  copies.most = std::max(copies.most, rows * ld);
  return {to, ld, ld, rows * ld};
}
template <typename T>
In<T> taken(const void* p, int64_t stride, int64_t rows, int width, Room& room, Copies<T>& copies) {
  if (direct<T>(p, stride, width)) return {(const T*)p, stride, width, (rows - 1) * stride + width};
  return copied<T>(p, stride, rows, width, room, copies);
}
template <typename T>
void make(const Copies<T>& copies, hipStream_t s) {
  if (copies.n > 0 && !probe) copy_rows_kernel<T><<<dim3((unsigned)std::min<int64_t>((copies.most + 255) / 256, 8192), copies.n), 256, 0, s>>>(copies);
}
// Rows of a k-strided operand that one descriptor takes: whole chunks in less than 2 GiB
template <typename T>
int64_t segment_rows(int64_t ld) { return std::max<int64_t>((1ll << 31) / (ld * (int64_t)sizeof(T)) / 64 * 64, 64); }

template <typename T>
Plan forward_plan(const Shape& n) {      // results, and as a guess a residual or what is kept of each matrix
  return plan_of<T>({n.rows, n.outer, 1, chunks<T>(n.inner, 64), false, n.mats == 2, false, n.mats == 2 ? 10.f : 8.f});
}
template <typename T>
Plan dx_plan(const Shape& n) { return plan_of<T>({n.rows, n.inner, 1, (int64_t)chunks<T>(n.outer, 64) * n.mats, false, false, true, (float)sizeof(T)}); }
template <typename T>
Plan dw_plan(const Shape& n, int batches) { return plan_of<T>({n.outer, n.inner, batches, chunks<T>(n.rows, 64), false, false, true, (float)sizeof(T)}); }

template <typename T>
int64_t forward_room(const Shape& n, bool x_direct, bool w_direct) {
  return (x_direct ? 0 : copy_bytes<T>(n.rows, n.inner)) + (w_direct ? 0 : n.mats * copy_bytes<T>(n.outer, n.inner)) +
         (n.rows <= kFewRows ? 0 : up(part_bytes(forward_plan<T>(n), n.rows, n.outer, 1, n.mats == 2), kAlign));
}
// Shares of rows: enough workgroups for the card, four rows each (of a wave one) at least
int shares_of(const Shape& n) {
  const int strips = (n.outer + kGradColumns - 1) / kGradColumns;
  return std::min({(n.rows + 3) / 4, std::max(2048 / strips, 1), kGradShares});
}
template <typename T>
int64_t backward_room(const Shape& n, bool x_direct, bool w_direct) {
  const int64_t dz = n.mats * up((int64_t)n.rows * up(n.outer, 8) * (int64_t)sizeof(T), kAlign);
  const int64_t sums = up((int64_t)kGradShares * n.mats * n.outer * (int64_t)sizeof(float), kAlign);
  int64_t part = part_bytes(dx_plan<T>(n), n.rows, n.inner, 1, false);
  for (int batches = 1; batches <= n.mats; batches++)      // one of a gated layer's weights may be wanted alone
    part = std::max(part, part_bytes(dw_plan<T>(n, batches), n.outer, n.inner, batches, false));
  return (x_direct ? 0 : copy_bytes<T>(n.rows, n.inner)) + (w_direct ? 0 : n.mats * copy_bytes<T>(n.outer, n.inner)) + dz + sums + up(part, kAlign);
}

struct Forward {
  const void* x;
  int64_t x_stride;
  const void* w;
  int64_t w_stride;
  const void* up;
  int64_t up_stride;
  const void *bias, *up_bias, *residual;
  int64_t residual_stride;
  int act, wide;
  void* y;
  float* kept;
};
template <typename T>
bool weights_direct(const void* w, int64_t w_stride, const void* up, int64_t up_stride, const Shape& n) {
  return direct<T>(w, w_stride, n.inner) && (n.mats == 1 || (direct<T>(up, up_stride, n.inner) && up_stride == w_stride)) &&
         (int64_t)n.outer * w_stride * (int64_t)sizeof(T) < (1ll << 32) - (1 << 20);
}
// both matrices alike: both as they lie or both copied
template <typename T>
void take_weights(const void* w, int64_t w_stride, const void* up_, int64_t up_stride, const Shape& n, Room& room, Copies<T>& copies, In<T>& a, In<T>& b) {
  b = {};
  if (weights_direct<T>(w, w_stride, up_, up_stride, n)) {
    const int64_t elements = (n.outer - 1) * w_stride + n.inner;
    a = {(const T*)w, w_stride, n.inner, elements};
    if (n.mats == 2) b = {(const T*)up_, up_stride, n.inner, elements};
    return;
  }
  a = copied<T>(w, w_stride, n.outer, n.inner, room, copies);
  if (n.mats == 2) b = copied<T>(up_, up_stride, n.outer, n.inner, room, copies);
}

template <typename T>
int forward(const Shape& n, const Forward& f, void* ws, hipStream_t s) {
  Room room{(char*)ws};
  Copies<T> copies;
  const In<T> x = taken<T>(f.x, f.x_stride, n.rows, n.inner, room, copies);
  In<T> w, u;
  take_weights<T>(f.w, f.w_stride, f.up, f.up_stride, n, room, copies, w, u);
  make(copies, s);
  Product<T> p{};
  p.k = p.last_k = w.width, p.segments = 1, p.batches = 1;
  p.a = {x.p, x.ld, 0, 0, n.rows, n.rows, w.width, w.width, x.elements};
  p.b = {w.p, w.ld, 0, 0, n.outer, n.outer, w.width, w.width, w.elements};
  p.rows = n.rows, p.cols = n.outer;
  const Plan plan = forward_plan<T>(n);
  if (n.rows > kFewRows) p.part = (float*)room.take(part_bytes(plan, n.rows, n.outer, 1, n.mats == 2));
  auto finish = [&](auto e) {
    e.y = f.y, e.cols = n.outer, e.act = f.act, e.wide = f.wide, e.bias = (const T*)f.bias, e.up_bias = (const T*)f.up_bias;
    e.residual = f.residual, e.residual_stride = f.residual_stride, e.kept = f.kept;
    e.vec = n.outer % 8 == 0 && f.residual_stride % 8 == 0 && aligned16(f.y) && aligned16(f.bias) && aligned16(f.up_bias) && aligned16(f.residual) &&
            aligned16(f.kept);
    return e;
  };
  auto product = [&](const auto& e) {
    if (n.rows <= kFewRows) launch_few_rows<T>(p, e, s);
    else launch<T, false, false>(p, plan, e, s);
  };
  if (n.mats == 2) {
    p.b2 = u.p - w.p, p.u = u.p, p.u_elements = u.elements;
    product(finish(Finish<T, true, false>{}));
  } else if (f.act == RL_ACT_NONE && !f.bias && !f.residual && !f.kept) {
    product(finish(Finish<T, false, true>{}));
  } else if (f.act == RL_ACT_NONE && !f.kept) {
    product(finish(Finish<T, false, false, true>{}));
  } else {
    product(finish(Finish<T, false, false>{}));
  }
  return probe ? RL_OK : launched();
}

struct Backward {
  const void* dy;
  int64_t dy_stride;
  int wide;
  const void* x;
  int64_t x_stride;
  const void* w;
  int64_t w_stride;
  const void* up;
  int64_t up_stride;
  int act;
  const float* kept;
  void *dx, *dw, *dup, *db, *dub;
};
template <typename T>
int backward(const Shape& n, const Backward& f, void* ws, hipStream_t s) {
  Room room{(char*)ws};
  constexpr int V = 16 / sizeof(T);
  // gradients of the products' sums
  const bool same = f.act == RL_ACT_NONE && n.mats == 1 && (!f.wide || sizeof(T) == 4) && direct<T>(f.dy, f.dy_stride, n.outer);
  In<T> dz{(const T*)f.dy, f.dy_stride, n.outer, (n.rows - 1) * f.dy_stride + n.outer};
  const int ldz = (int)up(n.outer, 8), shares = shares_of(n);
  T* own = nullptr;
  if (!same) {
    own = (T*)room.take(n.mats * up((int64_t)n.rows * ldz * (int64_t)sizeof(T), kAlign));
    dz = {own, ldz, (int)up(n.outer, V), (int64_t)n.mats * n.rows * ldz};
  }
  float* const sums = (float*)room.take((int64_t)kGradShares * n.mats * n.outer * (int64_t)sizeof(float));
  const bool biased = f.db || f.dub;
  if ((!same || biased) && !probe) {
    Gradient<T> g{f.dy, f.dy_stride, f.wide, f.act, n.rows, n.outer, n.mats, ldz, 0, 0, f.act == RL_ACT_NONE && n.mats == 1 ? nullptr : f.kept, own,
                  biased ? sums : nullptr};
    g.vec = n.outer % 8 == 0 && f.dy_stride % 8 == 0 && aligned16(f.dy) && aligned16(f.kept);
    g.per_share = (n.rows + shares - 1) / shares;
    const dim3 grid((n.outer + kGradColumns - 1) / kGradColumns, shares);
    if (n.mats == 2) gradient_kernel<T, true><<<grid, 256, 0, s>>>(g);
    else gradient_kernel<T, false><<<grid, 256, 0, s>>>(g);
    if (biased)
      share_sum_kernel<T><<<dim3((n.outer + 255) / 256, n.mats), 256, 0, s>>>(sums, shares, n.mats, n.outer, (T*)f.db, (T*)f.dub);
  }
  const int64_t dz_matrix = (int64_t)n.rows * ldz;      // from dz to du
  Finish<T, false, true> e{};
  e.cols = n.inner;
  Copies<T> copies;
  In<T> w, u, x;
  if (f.dx) take_weights<T>(f.w, f.w_stride, f.up, f.up_stride, n, room, copies, w, u);
  if (f.dw || f.dup) x = taken<T>(f.x, f.x_stride, n.rows, n.inner, room, copies);
  make(copies, s);
  if (f.dx) {
    Room r = room;      // both products' sums of slices lie in one place
    Product<T> p{};
    p.a = {dz.p, dz.ld, 0, dz_matrix, n.rows, n.rows, dz.width, dz.width, dz.elements};
    p.b = {w.p, w.ld, 0, n.mats == 2 ? u.p - w.p : 0, n.outer, n.outer, w.width, w.width, w.elements};
    p.u = u.p, p.u_elements = u.elements;
    p.k = p.last_k = dz.width, p.segments = n.mats, p.batches = 1;
    p.rows = n.rows, p.cols = n.inner;
    const Plan plan = dx_plan<T>(n);
    p.part = (float*)r.take(part_bytes(plan, n.rows, n.inner, 1, false));
    e.y = f.dx, e.y_batch = 0, e.vec = n.inner % 8 == 0 && aligned16(f.dx);
    launch<T, false, true>(p, plan, e, s);
  }
  if (f.dw || f.dup) {
    Room r = room;
    const int64_t most = segment_rows<T>(std::max(dz.ld, x.ld)), segments = (n.rows + most - 1) / most, last = n.rows - (segments - 1) * most;
    const int each = (int)std::min<int64_t>(most, n.rows);
    const bool first = f.dw, both = f.dw && f.dup;
    Product<T> p{};
    p.a = {dz.p + (first ? 0 : dz_matrix), dz.ld, dz_matrix, most * dz.ld, each, (int)last, dz.width, dz.width, dz.elements - (first ? 0 : dz_matrix)};
    p.b = {x.p, x.ld, 0, most * x.ld, each, (int)last, x.width, x.width, x.elements};
    p.k = each, p.last_k = (int)last, p.segments = (int)segments, p.batches = both ? 2 : 1;
    p.rows = n.outer, p.cols = n.inner;
    const Plan plan = dw_plan<T>(n, p.batches);
    p.part = (float*)r.take(part_bytes(plan, n.outer, n.inner, p.batches, false));
    e.y = first ? f.dw : f.dup, e.y_batch = both ? (T*)f.dup - (T*)f.dw : 0;
    e.vec = n.inner % 8 == 0 && aligned16(f.dw) && aligned16(f.dup);
    launch<T, true, true>(p, plan, e, s);
  }
  return probe ? RL_OK : launched();
}

const int64_t kMostWeights = (1ll << 30) - (1 << 20);
const char* linear_argument(int32_t rows, int32_t inner, int32_t outer, int32_t dtype) {
  if (dtype != RL_DTYPE_F32 && dtype != RL_DTYPE_BF16) return "dtype is RL_DTYPE_F32 or RL_DTYPE_BF16";
  if (rows < 0 || inner < 1 || outer < 1 || rows > (1 << 26) || inner > (1 << 20) - 8 || outer > (1 << 20) - 8) return "rows, inner or outer out of range";
  if ((int64_t)up(inner, 8) * outer > kMostWeights) return "weights of more than 2^30 - 2^20 elements";
  return nullptr;
}
}  // namespace

extern "C" int64_t rl_linear_workspace(int32_t rows, int32_t inner, int32_t outer, int32_t gated, int32_t dtype, int32_t backward, int32_t aligned) {
  if (linear_argument(rows, inner, outer, dtype) || rows == 0) return 0;
  const Shape n{rows, inner, outer, gated ? 2 : 1};
  const bool direct = aligned && inner % (dtype == RL_DTYPE_F32 ? 4 : 8) == 0;
  if (dtype == RL_DTYPE_F32) return backward ? backward_room<float>(n, direct, direct) : forward_room<float>(n, direct, direct);
  return backward ? backward_room<bf16_t>(n, direct, direct) : forward_room<bf16_t>(n, direct, direct);
}

extern "C" int rl_linear_forward(const void* d_x, int64_t x_stride, int32_t rows, int32_t inner, const void* d_weight, int64_t weight_stride,
                                 const void* d_up, int64_t up_stride, int32_t outer, const void* d_bias, const void* d_up_bias, int32_t activation,
                                 const void* d_residual, int64_t residual_stride, int32_t residual_dtype, int32_t dtype, void* d_y, float* d_kept,
                                 void* d_workspace, int64_t workspace_bytes, void* stream) {
  if (const char* m = linear_argument(rows, inner, outer, dtype)) return rl_fail(RL_E_ARG, m);
  if (activation < RL_ACT_NONE || activation > RL_ACT_GELU_TANH) return rl_fail(RL_E_ARG, "no such activation");
  if (d_residual && residual_dtype != dtype && residual_dtype != RL_DTYPE_F32) return rl_fail(RL_E_ARG, "the residual is of the call's type or float32");
  if (rows == 0) return RL_OK;
  if (!d_x || !d_weight || !d_y || (d_up_bias && !d_up)) return rl_fail(RL_E_ARG, "null pointer");
  const Shape n{rows, inner, outer, d_up ? 2 : 1};
  const Forward f{d_x, x_stride, d_weight, weight_stride, d_up, up_stride, d_bias, d_up_bias, d_residual, residual_stride, activation,
                  d_residual && residual_dtype == RL_DTYPE_F32 && dtype != RL_DTYPE_F32, d_y, d_kept};
  auto need = [&](auto t) {
    using T = decltype(t);
    return forward_room<T>(n, direct<T>(d_x, x_stride, inner), weights_direct<T>(d_weight, weight_stride, d_up, up_stride, n));
  };
  const int64_t bytes = dtype == RL_DTYPE_F32 ? need(float()) : need(bf16_t());
  if (bytes > 0 && (workspace_bytes < bytes || !d_workspace)) return rl_fail(RL_E_ARG, "workspace smaller than rl_linear_workspace says");
  if ((uintptr_t)d_workspace & (kAlign - 1)) return rl_fail(RL_E_ARG, "workspace not aligned to 256 bytes");
  return dtype == RL_DTYPE_F32 ? forward<float>(n, f, d_workspace, (hipStream_t)stream) : forward<bf16_t>(n, f, d_workspace, (hipStream_t)stream);
}

extern "C" int rl_linear_backward(const void* d_dy, int64_t dy_stride, int32_t dy_dtype, const void* d_x, int64_t x_stride, int32_t rows, int32_t inner,
                                  const void* d_weight, int64_t weight_stride, const void* d_up, int64_t up_stride, int32_t outer, int32_t activation,
                                  const float* d_kept, int32_t dtype, void* d_dx, void* d_dweight, void* d_dup, void* d_dbias, void* d_dup_bias,
                                  void* d_workspace, int64_t workspace_bytes, void* stream) {
  if (const char* m = linear_argument(rows, inner, outer, dtype)) return rl_fail(RL_E_ARG, m);
  if (activation < RL_ACT_NONE || activation > RL_ACT_GELU_TANH) return rl_fail(RL_E_ARG, "no such activation");
  if (dy_dtype != dtype && dy_dtype != RL_DTYPE_F32) return rl_fail(RL_E_ARG, "dy is of the call's type or float32");
  if ((d_dup || d_dup_bias) && !d_up) return rl_fail(RL_E_ARG, "gradients of a second matrix that there is none of");
  hipStream_t s = (hipStream_t)stream;
  if (rows == 0) {      // sums of nothing
    auto clear = [&](void* p, int64_t elements) {
      if (!p) return;
      if (dtype == RL_DTYPE_F32) fill_kernel<float><<<blocks_for(elements), 256, 0, s>>>((float*)p, elements);
      else fill_kernel<bf16_t><<<blocks_for(elements), 256, 0, s>>>((bf16_t*)p, elements);
    };
    for (void* p : {d_dweight, d_dup}) clear(p, (int64_t)inner * outer);
    for (void* p : {d_dbias, d_dup_bias}) clear(p, outer);
    return launched();
  }
  const bool kept = activation != RL_ACT_NONE || d_up;
  if (!d_dy || (d_dx && !d_weight) || ((d_dweight || d_dup) && !d_x) || (kept && !d_kept)) return rl_fail(RL_E_ARG, "null pointer");
  const Shape n{rows, inner, outer, d_up ? 2 : 1};
  const Backward f{d_dy, dy_stride, dy_dtype == RL_DTYPE_F32 && dtype != RL_DTYPE_F32, d_x, x_stride, d_weight, weight_stride, d_up, up_stride,
                   activation, d_kept, d_dx, d_dweight, d_dup, d_dbias, d_dup_bias};
  auto need = [&](auto t) {
    using T = decltype(t);
    return backward_room<T>(n, direct<T>(d_x, x_stride, inner), weights_direct<T>(d_weight, weight_stride, d_up, up_stride, n));
  };
  const int64_t bytes = dtype == RL_DTYPE_F32 ? need(float()) : need(bf16_t());
  if (workspace_bytes < bytes || !d_workspace) return rl_fail(RL_E_ARG, "workspace smaller than rl_linear_workspace says");
  if ((uintptr_t)d_workspace & (kAlign - 1)) return rl_fail(RL_E_ARG, "workspace not aligned to 256 bytes");
  return dtype == RL_DTYPE_F32 ? backward<float>(n, f, d_workspace, s) : backward<bf16_t>(n, f, d_workspace, s);
}

extern "C" int rl_debug_linear_loads(int32_t rows, int32_t inner, int32_t outer, int64_t x_stride, int64_t weight_stride, int64_t dy_stride, int32_t gated,
                                     int32_t dtype, int32_t backward, int64_t* out) {
  if (!out || rows < 1) return rl_fail(RL_E_ARG, "null pointer or no rows");
  Probe found{};
  probe = &found;
  // addresses that nothing is at: only distances count
  char* const at = (char*)(1ll << 44);
  auto place = [&](int i) { return at + ((int64_t)i << 42); };
  const int64_t bytes = rl_linear_workspace(rows, inner, outer, gated, dtype, backward, 0);
  const int rc = backward ? rl_linear_backward(place(1), dy_stride, dtype, place(2), x_stride, rows, inner, place(3), weight_stride, gated ? place(4) : nullptr,
                                               weight_stride, outer, gated ? RL_ACT_SILU : RL_ACT_NONE, (const float*)place(5), dtype, place(6), place(7),
                                               gated ? place(8) : nullptr, nullptr, nullptr, place(9), bytes, nullptr)
                          : rl_linear_forward(place(1), x_stride, rows, inner, place(2), weight_stride, gated ? place(3) : nullptr, weight_stride, outer, nullptr,
                                              nullptr, RL_ACT_NONE, nullptr, 0, dtype, dtype, place(4), nullptr, place(5), bytes, nullptr);
  probe = nullptr;
  if (rc != RL_OK) return rc;
  out[0] = found.buffers, out[1] = found.offsets, out[2] = found.products;
  return RL_OK;
}
