// Log-probs of target tokens from hidden rows and the lm-head's weights, with their gradient, without keeping the logits.
#include <algorithm>
#include <type_traits>

#include "token_logprob.h"

namespace {

// =============================================================================================
// z = h W^T / T, lse = log sum_v e^(z_v), logp = z_y - lse.  Backward: dz_v = g / T ([v = y] - e^(z_v - lse)), dh = dz W, dW = dz^T h.
// Forward: the product's epilogue leaves (max, sum of e^(z - max)) of every row and strip of the vocabulary, a second kernel joins
// the strips.  Backward: a piece of the vocabulary at a time, its logits are formed again and only dz is stored, in the type of the
// weights, since it is an operand of the two products behind it (relative error of the gradients: sqrt 2 times that of their last rounding); dh is added up over the pieces in 32 bits and rounded once.
// Rows without target (observation tokens) or, backward, with g = 0 take no part: the others are gathered first.
// =============================================================================================

// Kept rows in order: a scan of the targets by 1024 threads.  place[t]: where row t went, -1: nowhere, -2: its target lies behind the
// vocabulary, which shows as NaN.  Forward (g null): logp and lse of the others are written here.
struct RowScan {
  const int32_t* targets;
  int rows, vocab;
  const float *g, *lse_in;
  float inv_t;
  int32_t *count, *list, *place, *target;
  float *lse_kept, *g_kept, *logp, *lse;
  SliceRule rule;
  int twins;
};
// Returns how many rows are kept; found: the row that went to place `wanted`, for one thread at most.
__device__ __forceinline__ int scan_rows(const RowScan& s, bool write, int wanted, int* found) {
  __shared__ int waves[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int done = 0;
  for (int t0 = 0; t0 < s.rows; t0 += 1024) {
    const int t = t0 + threadIdx.x, y = t < s.rows ? s.targets[t] : -1;
    const float gt = s.g && t < s.rows ? s.g[t] : 1.f;
    const bool keep = y >= 0 && y < s.vocab && gt != 0.f;
    const uint64_t mask = __ballot(keep);
    if (lane == 0) waves[wave] = __popcll(mask);
    __syncthreads();
    int before = done, all = 0;
#pragma unroll
    for (int i = 0; i < 16; i++) {
      if (i < wave) before += waves[i];
      all += waves[i];
    }
    done += all;
    const int at = before + __popcll(mask & ((1ull << lane) - 1));
    if (keep && at == wanted) *found = t;
    if (keep && write) {
      s.list[at] = t;
      for (int k = 0; k < (s.twins ? 2 : 1); k++) {
        const int i = at + k * s.twins;
        s.target[i] = y;
        if (s.g) {
          s.lse_kept[i] = s.lse_in[t];
          s.g_kept[i] = gt * s.inv_t;
        }
      }
    }
    if (t < s.rows && write) {
      const float none = y >= s.vocab ? __builtin_nanf("") : 0.f;
      if (s.g) {
        s.place[t] = keep ? at : y >= s.vocab ? -2 : -1;
      } else if (!keep) {
        s.logp[t] = none;
        s.lse[t] = none;
      }
    }
    __syncthreads();
  }
  if (!write) return done;
  for (int i = done + threadIdx.x; i < (int)((done + kRowPad - 1) / kRowPad * kRowPad); i += 1024) {
    if (s.twins && i >= s.twins && i < s.twins + done) continue;
    s.target[i] = -1;
    if (s.g) s.lse_kept[i] = 0.f, s.g_kept[i] = 0.f;
  }
  if (threadIdx.x == 0) {
    const int all = s.twins && done ? 2 * s.twins : done;
    s.count[0] = all;
    if (s.g) {
      const int n = choose_slices(s.rule, all);
      s.count[1] = n;
      s.count[2] = slice_width(s.rule, n);
    }
  }
  return done;
}
__global__ __launch_bounds__(1024) void keep_rows_kernel(RowScan s) { scan_rows(s, true, -1, nullptr); }

// A kept row (null: zeros), zeros behind column `hidden`
template <typename T, int VEC>
__device__ __forceinline__ void copy_row(const T* src, int hidden, int ld, T* out) {
  for (int c = threadIdx.x * VEC; c < ld; c += blockDim.x * VEC) {
    float v[VEC];
    if (src && c < hidden) {
      ldv<VEC>(src + c, v);
    } else {
#pragma unroll
      for (int e = 0; e < VEC; e++) v[e] = 0.f;
    }
    stv<VEC>(out + c, v);
  }
}
// Kept rows of h one after the other, zeros behind the last one up to the padding.
template <typename T, int VEC>
__global__ __launch_bounds__(256) void gather_rows_kernel(const T* __restrict__ h, int64_t stride, int hidden, int ld,
                                                          const int32_t* __restrict__ list, const int32_t* __restrict__ count,
                                                          T* __restrict__ out) {
  const int r = blockIdx.x, n = *count;
  if (r >= (n + kRowPad - 1) / kRowPad * kRowPad) return;
  copy_row<T, VEC>(r < n ? h + list[r] * stride : nullptr, hidden, ld, out + (size_t)r * ld);
}
// Both in one launch: every workgroup scans all rows for its own.
template <typename T, int VEC>
__global__ __launch_bounds__(1024) void keep_and_gather_kernel(RowScan s, const T* __restrict__ h, int64_t stride, int hidden, int ld, T* __restrict__ out) {
  __shared__ int mine;
  const int r = blockIdx.x, at = s.twins && r >= s.twins ? r - s.twins : r, n = scan_rows(s, r == 0, at, &mine);
  if (r >= (n + kRowPad - 1) / kRowPad * kRowPad) return;
  copy_row<T, VEC>(at < n ? h + mine * stride : nullptr, hidden, ld, out + (size_t)r * ld);
}

// ---- products in 32 bits for every type and size ----------------------------------------------
// C[i, j] = sum_k A[i, k] B[j, k], tiles of 128 x 128, four waves of 64 x 64 on 32x32x2 matrix instructions, 16 k at a time through
// LDS as [k][row].  An operand is K-major (element (i, k) at i * ld + k) or not (at k * ld + i).
template <typename T>
struct Operand {
  const T* p;
  int64_t ld;
  int n, vec;      // rows; 16-byte accesses allowed
};
template <typename T, bool KMAJOR>
__device__ __forceinline__ void fetch8(const Operand<T>& o, int i0, int k0, int k1, float (&v)[8]) {
  const int tid = threadIdx.x;
  const int i = KMAJOR ? i0 + tid / 2 : i0 + tid % 16 * 8, k = KMAJOR ? k0 + tid % 2 * 8 : k0 + tid / 16;
  const bool line = KMAJOR ? i < o.n : k < k1;
  const T* p = KMAJOR ? o.p + (int64_t)i * o.ld + k : o.p + (int64_t)k * o.ld + i;
  const int left = !line ? 0 : KMAJOR ? k1 - k : o.n - i;
  if (left >= 8 && o.vec) {
    if constexpr (sizeof(T) == 2) {
      ldv<8>(p, v);
    } else {
      float a[4], b[4];
      ldv<4>(p, a);
      ldv<4>(p + 4, b);
#pragma unroll
      for (int e = 0; e < 4; e++) v[e] = a[e], v[4 + e] = b[e];
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; e++) v[e] = e < left ? ldf(p + e) : 0.f;
  }
}
constexpr int kPitch = 128 + 4;
template <bool KMAJOR>
__device__ __forceinline__ void put8(float (*to)[kPitch], const float (&v)[8]) {
  const int tid = threadIdx.x;
  if constexpr (KMAJOR) {
#pragma unroll
    for (int e = 0; e < 8; e++) to[tid % 2 * 8 + e][tid / 2] = v[e];
  } else {
    *(float4*)&to[tid / 16][tid % 16 * 8] = make_float4(v[0], v[1], v[2], v[3]);
    *(float4*)&to[tid / 16][tid % 16 * 8 + 4] = make_float4(v[4], v[5], v[6], v[7]);
  }
}
template <typename T, bool AK, bool BK, typename TB>
__device__ __forceinline__ void product128(const Operand<T>& A, const Operand<TB>& B, int i0, int j0, int k0, int k1, f32x16 (&acc)[2][2]) {
  __shared__ float as[16][kPitch], bs[16][kPitch];
  const int lane = threadIdx.x & 63, wm = (threadIdx.x >> 7) * 64, wn = ((threadIdx.x >> 6) & 1) * 64;
#pragma unroll
  for (int a = 0; a < 2; a++)
#pragma unroll
    for (int b = 0; b < 2; b++)
#pragma unroll
      for (int e = 0; e < 16; e++) acc[a][b][e] = 0.f;
  float va[8], vb[8];
  if (k0 < k1) {
    fetch8<T, AK>(A, i0, k0, k1, va);
    fetch8<TB, BK>(B, j0, k0, k1, vb);
  }
  for (int k = k0; k < k1; k += 16) {
    __syncthreads();
    put8<AK>(as, va);
    put8<BK>(bs, vb);
    __syncthreads();
    if (k + 16 < k1) {
      fetch8<T, AK>(A, i0, k + 16, k1, va);
      fetch8<TB, BK>(B, j0, k + 16, k1, vb);
    }
#pragma unroll
    for (int s = 0; s < 16; s += 2) {
      float x[2], y[2];
#pragma unroll
      for (int a = 0; a < 2; a++) {
        x[a] = as[s + (lane >> 5)][wm + 32 * a + (lane & 31)];
        y[a] = bs[s + (lane >> 5)][wn + 32 * a + (lane & 31)];
      }
#pragma unroll
      for (int a = 0; a < 2; a++)
#pragma unroll
        for (int b = 0; b < 2; b++) acc[a][b] = __builtin_amdgcn_mfma_f32_32x32x2f32(x[a], y[b], acc[a][b], 0, 0, 0);
    }
  }
}
// element e of a 32 x 32 result: column lane % 32, row
__device__ __forceinline__ int row32(int lane, int e) { return 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3); }

// logits of 128 tokens of the vocabulary (rows of the result) and 128 hidden rows (its columns: a lane holds one row's)
template <typename T>
__global__ __launch_bounds__(256) void logits_strip_kernel(const T* __restrict__ h, int ld, const T* __restrict__ w, int64_t ldw, int vocab,
                                                           int hidden, int vec, KeptRows kept, float inv_t, float2* __restrict__ part,
                                                           int padded, float* __restrict__ zt) {
  const int n = *kept.count, j0 = blockIdx.x * 128, i0 = blockIdx.y * 128;
  if (j0 >= n) return;
  f32x16 acc[2][2];
  product128<T, true, true>(Operand<T>{w, ldw, vocab, vec}, Operand<T>{h, ld, n, 1}, i0, j0, 0, hidden, acc);
  __shared__ float2 half[2][128];
  const int lane = threadIdx.x & 63, wm = threadIdx.x >> 7, wn = (threadIdx.x >> 6) & 1;
#pragma unroll
  for (int b = 0; b < 2; b++) {
    const int col = wn * 64 + b * 32 + (lane & 31), j = j0 + col, y = j < n ? kept.target[j] : -1;
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int a = 0; a < 2; a++)
#pragma unroll
      for (int e = 0; e < 16; e++) {
        const int v = i0 + wm * 64 + a * 32 + row32(lane, e);
        acc[a][b][e] = v < vocab ? acc[a][b][e] * inv_t : -INFINITY;
        if (v == y) zt[j] = acc[a][b][e];
        top = fmaxf(top, acc[a][b][e]);
      }
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float ref = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int a = 0; a < 2; a++)
#pragma unroll
      for (int e = 0; e < 16; e++) sum += expf(acc[a][b][e] - ref);
    sum += __shfl_xor(sum, 32, 64);
    if (lane < 32) half[wm][col] = make_float2(top, sum);
  }
  __syncthreads();
  if (threadIdx.x < 128 && j0 + (int)threadIdx.x < n) {
    const float2 a = half[0][threadIdx.x], b = half[1][threadIdx.x];
    const float top = fmaxf(a.x, b.x), ref = top == -INFINITY ? 0.f : top;
    part[(size_t)blockIdx.y * padded + j0 + threadIdx.x] = make_float2(top, a.y * expf(a.x - ref) + b.y * expf(b.x - ref));
  }
}

// 16 kept rows: their strips joined by 64 threads each, in a fixed order (4096 rows x 594 strips: 10 us, 64 rows by 16 threads each 23)
__global__ __launch_bounds__(1024) void join_strips_kernel(const float2* __restrict__ part, int strips, int padded, const float* __restrict__ zt,
                                                           const int32_t* __restrict__ list, const int32_t* __restrict__ count,
                                                           float* __restrict__ logp, float* __restrict__ lse) {
  __shared__ float2 share[16][16];
  const int n = *count, r = blockIdx.x * 16 + (threadIdx.x & 15), k = threadIdx.x >> 4;
  if (blockIdx.x * 16 >= n) return;
  float top = -INFINITY, sum = 0.f;
  auto join = [&](float2 p) {
    const float t = fmaxf(top, p.x), ref = t == -INFINITY ? 0.f : t;
    sum = sum * expf(top - ref) + p.y * expf(p.x - ref);
    top = t;
  };
  if (r < n) {
#pragma unroll 4
    for (int i = k; i < strips; i += 64) join(part[(size_t)i * padded + r]);
  }
#pragma unroll
  for (int o = 16; o < 64; o *= 2) {
    const float2 other = make_float2(__shfl_xor(top, o, 64), __shfl_xor(sum, o, 64));
    join(other);
  }
  if ((threadIdx.x & 63) < 16) share[threadIdx.x >> 6][threadIdx.x & 15] = make_float2(top, sum);
  __syncthreads();
  if (k == 0 && r < n) {
#pragma unroll
    for (int i = 1; i < 16; i++) join(share[i][threadIdx.x]);
    const float l = top + logf(sum);
    logp[list[r]] = zt[r] - l;
    lse[list[r]] = l;
  }
}

// dz of 128 tokens of a piece and 128 hidden rows; zeros where there is no token or no row
template <typename T>
__global__ __launch_bounds__(256) void logits_gradient_kernel(const T* __restrict__ h, int ld, const T* __restrict__ w, int64_t ldw, int vocab,
                                                              int hidden, int vec, KeptRows kept, float inv_t, VocabPiece piece,
                                                              T* __restrict__ dz) {
  const int n = *kept.count, j0 = blockIdx.x * 128, i0 = piece.v0 + blockIdx.y * 128;
  if (j0 >= (n + kRowPad - 1) / kRowPad * kRowPad) return;
  f32x16 acc[2][2];
  product128<T, true, true>(Operand<T>{w, ldw, vocab, vec}, Operand<T>{h, ld, n, 1}, i0, j0, 0, hidden, acc);
  const int lane = threadIdx.x & 63, wm = threadIdx.x >> 7, wn = (threadIdx.x >> 6) & 1;
#pragma unroll
  for (int b = 0; b < 2; b++) {
    const int j = j0 + wn * 64 + b * 32 + (lane & 31), y = kept.target[j];
    const float l = kept.lse[j], g = kept.g[j];
#pragma unroll
    for (int a = 0; a < 2; a++)
#pragma unroll
      for (int e = 0; e < 16; e++) {
        const int v = i0 + wm * 64 + a * 32 + row32(lane, e);
        const float d = j < n && v < vocab ? g * ((v == y ? 1.f : 0.f) - expf(acc[a][b][e] * inv_t - l)) : 0.f;
        st1(dz + (size_t)j * piece.ld + (v - piece.v0), kept.twins && j >= kept.twins ? rounding_left(d) : d);
      }
  }
}

// slice z of dh (+)= dz W over its share of the piece
template <typename T>
__global__ __launch_bounds__(256) void hidden_gradient_kernel(const T* __restrict__ dz, VocabPiece piece, const T* __restrict__ w, int64_t ldw,
                                                              int hidden, int vec, const int32_t* __restrict__ count, float* __restrict__ dh, size_t slice_stride, int first) {
  const int n = *count, i0 = blockIdx.x * 128, j0 = blockIdx.y * 128;
  if (i0 >= n || (int)blockIdx.z >= count[1]) return;
  const int k0 = blockIdx.z * count[2], k1 = min(k0 + count[2], piece.width);
  f32x16 acc[2][2];
  product128<T, true, false>(Operand<T>{dz, piece.ld, n, 1}, Operand<T>{w + (int64_t)piece.v0 * ldw, ldw, hidden, vec}, i0, j0, k0, k1, acc);
  const int lane = threadIdx.x & 63, wm = threadIdx.x >> 7, wn = (threadIdx.x >> 6) & 1;
  float* out = dh + blockIdx.z * slice_stride;
#pragma unroll
  for (int a = 0; a < 2; a++)
#pragma unroll
    for (int b = 0; b < 2; b++) {
      const int j = j0 + wn * 64 + b * 32 + (lane & 31);
#pragma unroll
      for (int e = 0; e < 16; e++) {
        const int i = i0 + wm * 64 + a * 32 + row32(lane, e);
        if (i < n && j < hidden) {
          float* p = out + (size_t)i * hidden + j;
          *p = first ? acc[a][b][e] : *p + acc[a][b][e];
        }
      }
    }
}

// dW of a piece = dz^T h
template <typename T>
__global__ __launch_bounds__(256) void weight_gradient_kernel(const T* __restrict__ dz, VocabPiece piece, const T* __restrict__ h, int ld,
                                                              int hidden, const int32_t* __restrict__ count, T* __restrict__ dw) {
  const int n = *count, i0 = blockIdx.y * 128, j0 = blockIdx.x * 128;
  f32x16 acc[2][2];
  product128<T, false, false>(Operand<T>{dz, piece.ld, piece.width, 1}, Operand<T>{h, ld, hidden, 1}, i0, j0, 0, n, acc);
  const int lane = threadIdx.x & 63, wm = threadIdx.x >> 7, wn = (threadIdx.x >> 6) & 1;
#pragma unroll
  for (int a = 0; a < 2; a++)
#pragma unroll
    for (int b = 0; b < 2; b++) {
      const int j = j0 + wn * 64 + b * 32 + (lane & 31);
#pragma unroll
      for (int e = 0; e < 16; e++) {
        const int i = i0 + wm * 64 + a * 32 + row32(lane, e);
        if (i < piece.width && j < hidden) st1(dw + (size_t)(piece.v0 + i) * hidden + j, acc[a][b][e]);
      }
    }
}

// Rows of dh: the slices' sum, zeros where a row takes no part.  SPLIT: waves that share a row's slices, for few rows, which have many
// (64 rows of 1024 in 64 slices twice: 66 us by one).
template <typename T, int VEC, int SPLIT>
__global__ __launch_bounds__(256) void hidden_gradient_rows_kernel(const float* __restrict__ slices, const int32_t* __restrict__ count, size_t slice_stride,
                                                                   int hidden, const int32_t* __restrict__ place, int twins, T* __restrict__ dh) {
  constexpr int THREADS = 256 / SPLIT, N = SPLIT > 1 ? 8 : 2;      // threads of a piece of a row
  __shared__ float part[SPLIT > 1 ? SPLIT : 1][SPLIT > 1 ? THREADS * VEC : 1];
  const int t = blockIdx.x, at = place[t], n = count[1], all = at < 0 ? 0 : twins ? 2 * n : n, share = threadIdx.x / THREADS, lane = threadIdx.x % THREADS;
  for (int c0 = blockIdx.y * THREADS * VEC; c0 < hidden; c0 += gridDim.y * THREADS * VEC) {
    const int c = c0 + lane * VEC;
    float v[VEC];
#pragma unroll
    for (int e = 0; e < VEC; e++) v[e] = at == -2 ? __builtin_nanf("") : 0.f;
    if (c < hidden) {
      const float* p = slices + (size_t)max(at, 0) * hidden + c;
      for (int s0 = share; s0 < all; s0 += N * SPLIT) {      // N at once
        float x[N][VEC];
#pragma unroll
        for (int i = 0; i < N; i++) {
          const int s = min(s0 + i * SPLIT, all - 1);
          ldv<VEC>(p + (s < n ? s * slice_stride : (s - n) * slice_stride + (size_t)twins * hidden), x[i]);
        }
#pragma unroll
        for (int i = 0; i < N; i++)
#pragma unroll
          for (int e = 0; e < VEC; e++) v[e] += s0 + i * SPLIT < all ? x[i][e] : 0.f;
      }
    }
    if constexpr (SPLIT > 1) {
#pragma unroll
      for (int e = 0; e < VEC; e++) part[share][e * THREADS + lane] = v[e];
      __syncthreads();
      if (share == 0) {
#pragma unroll
        for (int e = 0; e < VEC; e++) {
#pragma unroll
          for (int w = 1; w < SPLIT; w++) v[e] += part[w][e * THREADS + lane];
        }
      }
      __syncthreads();
    }
    if (share == 0 && c < hidden) stv<VEC>(dh + (size_t)t * hidden + c, v);
  }
}

// no rows at all: the weights' gradient is zero
__global__ __launch_bounds__(256) void zeros_kernel(uint16_t* __restrict__ p, int64_t n) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) p[i] = 0;
}

// ---- where everything lies in the workspace ----------------------------------------------------
// A piece's dz takes up to 1 GB: enough tokens of the vocabulary for full launches at any number of rows that fits a card, and
// little beside 288 GB.
const int64_t kPieceBytes = 1ll << 30;
struct Workspace {
  int64_t padded;            // rows, padded
  int ld;                    // of the gathered rows
  int strips;                // forward
  int width, ldz;            // backward: vocabulary of a piece, row length of dz
  SliceRule slices;          // backward: of the product dz W
  int64_t count, list, place, target, lse, g, zt, rows, part, dz, dh, bytes;
};
Workspace plan(int64_t rows, int hidden, int vocab, int dtype, bool backward) {
  const int el = dtype == RL_DTYPE_BF16 ? 2 : 4;
  Workspace w{};
  w.padded = up(rows, kRowPad);
  w.ld = (int)(up(hidden, 128) + (up(hidden, 128) % 256 == 0 ? 128 : 0));
  auto take = [&](int64_t n) {
    const int64_t at = w.bytes;
    w.bytes = up(at + n, 256);
    return at;
  };
  w.count = take(12);
  w.list = take(w.padded * 4);
  w.target = take(w.padded * 4);
  w.rows = take(w.padded * w.ld * el);
  if (!backward) {
    w.strips = (vocab + 63) / 64;      // as many as any tile leaves
    w.zt = take(w.padded * 4);
    w.part = take(w.padded * w.strips * 8);
    return w;
  }
  w.place = take(w.padded * 4);
  w.lse = take(w.padded * 4);
  w.g = take(w.padded * 4);
  const int64_t fit = std::max<int64_t>(std::min<int64_t>(kPieceBytes / (w.padded * el), ((1ll << 31) - (1 << 20)) / (hidden * el)) / 256 * 256, 1024);
  const int64_t pieces = (vocab + fit - 1) / fit;
  w.width = (int)up((vocab + pieces - 1) / pieces, 256);
  // slices of the vocabulary in dz W: up to 64, 512 MB of sums
  if (el == 2) token_logprob_slice_tile<bf16_t>((int)rows, hidden, w.width, w.slices);
  else token_logprob_slice_tile<float>((int)rows, hidden, w.width, w.slices);
  w.slices.width = w.width;
  w.slices.most = (int)std::max<int64_t>(std::min({(int64_t)64, kPieceBytes / 2 / (w.padded * hidden * 4), (int64_t)w.width / 256}), 1);
  w.slices.slice_us = (float)(hidden * 8 / 4.8e6);
  w.ldz = w.width + 128;
  w.dz = take(w.padded * w.ldz * el);
  w.dh = take(w.padded * hidden * 4 * w.slices.most);
  return w;
}

const char* logprob_argument(int64_t rows, int32_t hidden, int32_t vocab, float temperature, int32_t dtype) {
  if (dtype != RL_DTYPE_F32 && dtype != RL_DTYPE_BF16) return "dtype is RL_DTYPE_F32 or RL_DTYPE_BF16";
  if (rows < 0 || up(rows, kRowPad) > most_workgroups(256) || hidden < 1 || hidden > 65536 || vocab < 1 || vocab > (1 << 22)) return "rows, hidden or vocab out of range";
  if (!(temperature > 0.f) || temperature - temperature != 0.f || !(1.f / temperature <= 3.4e38f))
    return "temperature is a positive finite number with a finite reciprocal";
  return nullptr;
}

// Kept rows and their data, up to 512 rows in one launch (256 x 4096 in fp32, both directions: 30 rows 53 us, in two launches 57; 288 rows 62
// and 65; 1024 rows 102 and 101).
template <typename T, int VEC>
void keep(const RowScan& scan, const void* h, int64_t stride, int hidden, const Workspace& w, char* ws, hipStream_t s) {
  T* rows = (T*)(ws + w.rows);
  if (scan.rows <= 512) {
    keep_and_gather_kernel<T, VEC><<<(unsigned)w.padded, 1024, 0, s>>>(scan, (const T*)h, stride, hidden, w.ld, rows);
  } else {
    keep_rows_kernel<<<1, 1024, 0, s>>>(scan);
    gather_rows_kernel<T, VEC><<<(unsigned)w.padded, 256, 0, s>>>((const T*)h, stride, hidden, w.ld, scan.list, scan.count, rows);
  }
}
template <typename T>
void keep(const RowScan& scan, const void* h, int64_t stride, int hidden, const Workspace& w, char* ws, hipStream_t s) {
  constexpr int VEC = 16 / sizeof(T);
  if (hidden % VEC == 0 && stride % VEC == 0 && aligned16(h)) keep<T, VEC>(scan, h, stride, hidden, w, ws, s);
  else keep<T, 1>(scan, h, stride, hidden, w, ws, s);
}

template <typename T>
int forward(const void* h, int64_t stride, int rows, int hidden, const void* weight, int vocab, const int32_t* targets, float inv_t,
            float* logp, float* lse, char* ws, hipStream_t s) {
  const Workspace w = plan(rows, hidden, vocab, sizeof(T) == 2 ? RL_DTYPE_BF16 : RL_DTYPE_F32, false);
  const KeptRows kept{(int32_t*)(ws + w.count), (int32_t*)(ws + w.target), nullptr, nullptr, 0};
  keep<T>(RowScan{targets, rows, vocab, nullptr, nullptr, inv_t, (int32_t*)(ws + w.count), (int32_t*)(ws + w.list), nullptr,
                  (int32_t*)(ws + w.target), nullptr, nullptr, logp, lse, SliceRule{}, 0},
          h, stride, hidden, w, ws, s);
  int strips = (vocab + 127) / 128;
  const bool mfma = token_logprob_takes_mfma<T>(w.padded, w.ld, hidden, 0, weight, nullptr);
  if (mfma)
    strips = launch_logits_strips_mfma<T>(s, (const T*)(ws + w.rows), w.ld, rows, w.padded, (const T*)weight, vocab, hidden, kept, inv_t,
                                          (float2*)(ws + w.part), (float*)(ws + w.zt));
  const int vec = hidden % (16 / sizeof(T)) == 0 && aligned16(weight);
  if (!mfma)
    logits_strip_kernel<T><<<dim3((rows + 127) / 128, strips), 256, 0, s>>>((const T*)(ws + w.rows), w.ld, (const T*)weight, hidden, vocab, hidden,
                                                                           vec, kept, inv_t, (float2*)(ws + w.part), (int)w.padded,
                                                                           (float*)(ws + w.zt));
  join_strips_kernel<<<(rows + 15) / 16, 1024, 0, s>>>((const float2*)(ws + w.part), strips, (int)w.padded, (const float*)(ws + w.zt),
                                                       (const int32_t*)(ws + w.list), kept.count, logp, lse);
  return launched();
}

template <typename T>
int backward(const float* g, const void* h, int64_t stride, int rows, int hidden, const void* weight, int vocab, const int32_t* targets,
             const float* lse, float inv_t, void* dh, void* dw, char* ws, hipStream_t s) {
  const Workspace w = plan(rows, hidden, vocab, sizeof(T) == 2 ? RL_DTYPE_BF16 : RL_DTYPE_F32, true);
  const int twins = twins_of(rows, sizeof(T) == 2);
  const KeptRows kept{(int32_t*)(ws + w.count), (int32_t*)(ws + w.target), (float*)(ws + w.lse), (float*)(ws + w.g), twins};
  keep<T>(RowScan{targets, rows, vocab, g, lse, inv_t, (int32_t*)(ws + w.count), (int32_t*)(ws + w.list), (int32_t*)(ws + w.place),
                  (int32_t*)(ws + w.target), (float*)(ws + w.lse), (float*)(ws + w.g), nullptr, nullptr, w.slices, twins},
          h, stride, hidden, w, ws, s);
  const int vec = hidden % (16 / sizeof(T)) == 0 && aligned16(weight);
  const T *hr = (const T*)(ws + w.rows), *wt = (const T*)weight;
  T* dz = (T*)(ws + w.dz);
  const bool mfma = token_logprob_takes_mfma<T>(w.padded, w.ld, hidden, w.ldz, weight, dw);
  const unsigned rt = (rows + 127) / 128, ht = (hidden + 127) / 128;
  for (int v0 = 0; v0 < vocab; v0 += w.width) {
    const VocabPiece piece{v0, std::min(w.width, vocab - v0), w.ldz};
    const unsigned vt = (piece.width + 127) / 128;
    if (mfma) {
      launch_logits_gradient_mfma<T>(s, hr, w.ld, rows, w.padded, wt, vocab, hidden, kept, inv_t, piece, dz);
      launch_hidden_gradient_mfma<T>(s, dz, piece, rows, w.padded, wt, vocab, hidden, kept, w.slices.most, (float*)(ws + w.dh),
                                     (size_t)w.padded * hidden, v0 == 0);
      launch_weight_gradient_mfma<T>(s, dz, piece, hr, w.ld, w.padded, hidden, kept, (T*)dw);
      continue;
    }
    logits_gradient_kernel<T><<<dim3((unsigned)(w.padded / 128), vt), 256, 0, s>>>(hr, w.ld, wt, hidden, vocab, hidden, vec, kept, inv_t, piece, dz);
    hidden_gradient_kernel<T><<<dim3(rt, ht, w.slices.most), 256, 0, s>>>(dz, piece, wt, hidden, hidden, vec, kept.count,
                                                                         (float*)(ws + w.dh), (size_t)w.padded * hidden, v0 == 0);
    weight_gradient_kernel<T><<<dim3(ht, vt), 256, 0, s>>>(dz, piece, hr, w.ld, hidden, kept.count, (T*)dw);
  }
  const float* slices = (const float*)(ws + w.dh);
  const int32_t* place = (const int32_t*)(ws + w.place);
  constexpr int VEC = 16 / sizeof(T);
  auto rows_of_dh = [&](auto vec_of, auto split) {
    constexpr int W = decltype(vec_of)::value, S = decltype(split)::value;
    hidden_gradient_rows_kernel<T, W, S><<<dim3(rows, S > 1 ? (hidden + 64 * W - 1) / (64 * W) : 1), 256, 0, s>>>(
        slices, kept.count, (size_t)w.padded * hidden, hidden, place, twins, (T*)dh);
  };
  const std::integral_constant<int, 1> one;
  const std::integral_constant<int, 4> four;
  const std::integral_constant<int, VEC> whole;
  const bool wide = hidden % VEC == 0 && aligned16(dh);
  if (rows <= 512) wide ? rows_of_dh(whole, four) : rows_of_dh(one, four);
  else wide ? rows_of_dh(whole, one) : rows_of_dh(one, one);
  return launched();
}

}  // namespace

extern "C" int64_t rl_token_logprobs_workspace(int32_t rows, int32_t hidden, int32_t vocab, int32_t dtype, int32_t backward) {
  if (rows < 1 || logprob_argument(rows, hidden, vocab, 1.f, dtype)) return 0;
  return plan(rows, hidden, vocab, dtype, backward != 0).bytes;
}

extern "C" int rl_token_logprobs_forward(const void* d_hidden, int64_t row_stride, int32_t rows, int32_t hidden, const void* d_weight,
                                         int32_t vocab, const int32_t* d_targets, float temperature, int32_t dtype, float* d_logp,
                                         float* d_lse, void* d_workspace, int64_t workspace_bytes, void* stream) {
  if (const char* m = logprob_argument(rows, hidden, vocab, temperature, dtype)) return rl_fail(RL_E_ARG, m);
  if (rows == 0) return RL_OK;
  if (!d_hidden || !d_weight || !d_targets || !d_logp || !d_lse || !d_workspace) return rl_fail(RL_E_ARG, "null pointer");
  if (workspace_bytes < rl_token_logprobs_workspace(rows, hidden, vocab, dtype, 0))
    return rl_fail(RL_E_ARG, "workspace smaller than rl_token_logprobs_workspace says");
  if ((uintptr_t)d_workspace & 255) return rl_fail(RL_E_ARG, "workspace not aligned to 256 bytes");
  const float inv_t = 1.f / temperature;
#define RL_GO(T) forward<T>(d_hidden, row_stride, rows, hidden, d_weight, vocab, d_targets, inv_t, d_logp, d_lse, (char*)d_workspace, (hipStream_t)stream)
  return dtype == RL_DTYPE_F32 ? RL_GO(float) : RL_GO(bf16_t);
#undef RL_GO
}

extern "C" int rl_token_logprobs_backward(const float* d_dlogp, const void* d_hidden, int64_t row_stride, int32_t rows, int32_t hidden,
                                          const void* d_weight, int32_t vocab, const int32_t* d_targets, const float* d_lse,
                                          float temperature, int32_t dtype, void* d_dhidden, void* d_dweight, void* d_workspace,
                                          int64_t workspace_bytes, void* stream) {
  if (const char* m = logprob_argument(rows, hidden, vocab, temperature, dtype)) return rl_fail(RL_E_ARG, m);
  if (rows == 0) {
    if (!d_dweight) return rl_fail(RL_E_ARG, "null pointer");
    const int64_t n = (int64_t)vocab * hidden * (dtype == RL_DTYPE_BF16 ? 1 : 2);
    zeros_kernel<<<1024, 256, 0, (hipStream_t)stream>>>((uint16_t*)d_dweight, n);
    return launched();
  }
  if (!d_dlogp || !d_hidden || !d_weight || !d_targets || !d_lse || !d_dhidden || !d_dweight || !d_workspace)
    return rl_fail(RL_E_ARG, "null pointer");
  if (workspace_bytes < rl_token_logprobs_workspace(rows, hidden, vocab, dtype, 1))
    return rl_fail(RL_E_ARG, "workspace smaller than rl_token_logprobs_workspace says");
  if ((uintptr_t)d_workspace & 255) return rl_fail(RL_E_ARG, "workspace not aligned to 256 bytes");
  const float inv_t = 1.f / temperature;
#define RL_GO(T) \
  backward<T>(d_dlogp, d_hidden, row_stride, rows, hidden, d_weight, vocab, d_targets, d_lse, inv_t, d_dhidden, d_dweight, \
              (char*)d_workspace, (hipStream_t)stream)
  return dtype == RL_DTYPE_F32 ? RL_GO(float) : RL_GO(bf16_t);
#undef RL_GO
}

extern "C" int rl_debug_token_logprob_loads(int32_t rows, int32_t kept, int32_t hidden, int32_t vocab, int32_t dtype, int32_t backward,
                                            int64_t* out) {
  if (!out || rows < 1 || kept < 0 || kept > rows) return rl_fail(RL_E_ARG, "bad argument");
  if (const char* m = logprob_argument(rows, hidden, vocab, 1.f, dtype)) return rl_fail(RL_E_ARG, m);
  const Workspace w = plan(rows, hidden, vocab, dtype, backward != 0);
  const bool bf16 = dtype == RL_DTYPE_BF16;
  const int twins = backward ? twins_of(rows, bf16) : 0, all = twins && kept ? 2 * twins : kept;
  if (!(bf16 ? token_logprob_takes_mfma<bf16_t>(w.padded, w.ld, hidden, w.ldz, nullptr, nullptr)
             : token_logprob_takes_mfma<float>(w.padded, w.ld, hidden, w.ldz, nullptr, nullptr)))
    return rl_fail(RL_E_ARG, "a size that other kernels take");
  const int slices = backward ? choose_slices(w.slices, all) : 1;
  const LogprobSizes n{rows, all, hidden, vocab, backward, w.padded, w.ld, w.strips, w.width, w.ldz, w.slices.most, slices, backward ? slice_width(w.slices, slices) : 0};
  const LoadOverreach most = bf16 ? token_logprob_overreach<bf16_t>(n) : token_logprob_overreach<float>(n);
  out[0] = most.buffers, out[1] = most.offsets, out[2] = most.stores;
  return RL_OK;
}
