// Norms and rotary positions of packed rows, forward and backward (the policy update's form of them; a decode step has its own
// inside its products and attention).
#include <algorithm>

#include "policy_common.h"

namespace {

// =============================================================================================
// RMS and layer norm.  n = (x - mu) r, y = n w (+ b), r = 1 / sqrt(mean((x - mu)^2) + eps), mu = 0 in the RMS form.
// Backward: dn = dy w, dx = r (dn - n mean(dn n) [- mean(dn)]), dw = sum over rows of dy n, db = sum of dy.
// Bound by memory: x in, y out; backward dy and x in, dx out.  A row is held in registers by L threads, NV pieces of VEC elements
// each, so it is read once: a part of a wave for rows of up to 32 pieces, a wave up to 384 (512 of fewer elements), a workgroup above; NV = 0 takes rows
// too long for that in several passes.  Everything is computed in 32 bits and rounded once.  Measured, 7777 rows of 2560 in bf16: forward 16.4 us
// (4.85 TB/s, the rate of a copy), backward 27.5 (4.3 TB/s), its sums over rows 4.4.
// Row r is at (r / inner) * so + (r % inner) * si: heads of a fused projection need no copy.
// =============================================================================================
struct Rows {
  int n;                          // below 2^31
  int64_t so, si;
  unsigned inner, magic, shift;
  // r / inner = (r * magic >> 32) >> shift for r < 2^31: magic = ceil(2^(32 + shift) / inner), 2^shift < inner <= 2^(shift + 1)
  Rows(int64_t rows, int64_t outer_stride, int64_t inner_stride, int inner_rows)
      : n((int)rows), so(outer_stride), si(inner_stride), inner((unsigned)inner_rows), magic(0), shift(0) {
    if (inner < 2) return;
    while ((2ull << shift) < inner) shift++;
    magic = (unsigned)(((1ull << (32 + shift)) + inner - 1) / inner);
  }
  __device__ __forceinline__ int64_t at(int r) const {
    if (inner == 1) return r * so;
    const int o = (int)(__umulhi((unsigned)r, magic) >> shift);
    return o * so + (int64_t)(r - o * (int)inner) * si;
  }
};

// Pieces of a thread that lie inside every row that row_plan gives the plan (L, NV): those of the next smaller plan.
constexpr int full_pieces(int L, int NV) { return L < 64 ? 0 : NV == 8 ? 6 : L == 256 && NV == 6 ? 4 : NV - 1; }

template <int L>
__device__ __forceinline__ float group_sum(float v, float* lds) {
#pragma unroll
  for (int o = (L < 64 ? L : 64) / 2; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  if constexpr (L == 256) {
    __syncthreads();      // the last sum has been read
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    v = (lds[0] + lds[1]) + (lds[2] + lds[3]);
  }
  return v;
}

template <typename T, int VEC, int L, int NV>
__global__ __launch_bounds__(256) void norm_forward_kernel(const T* __restrict__ x, Rows rows, int first, int width, const T* __restrict__ w,
                                                           const T* __restrict__ b, float eps, int centered, T* __restrict__ y,
                                                           float* __restrict__ mean_out, float* __restrict__ rstd_out) {
  __shared__ float lds[4];
  const int lane = threadIdx.x % L;
  const int row = first + (int)blockIdx.x * (256 / L) + (L >= 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / L) : threadIdx.x / L);
  const bool live = row < rows.n;      // groups without a row run along: their lanes take part in no other group's sums
  const T* xr = x + (live ? rows.at(row) : 0);
  T* yr = y + (int64_t)(live ? row : 0) * width;
  const float inv = 1.f / (float)width;
  float mu = 0.f, rstd;
  if constexpr (NV > 0) {
    float v[NV][VEC];
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int c = (i * L + lane) * VEC;
      if (live && c < width) {
        ldv<VEC>(xr + c, v[i]);
      } else {
#pragma unroll
        for (int e = 0; e < VEC; e++) v[i][e] = 0.f;
      }
    }
    if (centered) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < NV; i++)
#pragma unroll
        for (int e = 0; e < VEC; e++) s += v[i][e];
      mu = group_sum<L>(s, lds) * inv;
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const bool in = (i * L + lane) * VEC < width;
#pragma unroll
      for (int e = 0; e < VEC; e++) {
        v[i][e] -= mu;
        s += in ? v[i][e] * v[i][e] : 0.f;
      }
    }
    rstd = 1.f / sqrtf(group_sum<L>(s, lds) * inv + eps);
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int c = (i * L + lane) * VEC;
      if (live && c < width) {
        float g[VEC], o[VEC];
        ldv<VEC>(w + c, g);
        if (b) ldv<VEC>(b + c, o);
#pragma unroll
        for (int e = 0; e < VEC; e++) o[e] = v[i][e] * rstd * g[e] + (b ? o[e] : 0.f);
        stv<VEC>(yr + c, o);
      }
    }
  } else {
    static_assert(NV > 0 || L == 256, "long rows take a workgroup");
    float v[VEC], s = 0.f;
    if (centered) {
      for (int c = lane * VEC; c < width; c += L * VEC) {
        ldv<VEC>(xr + c, v);
#pragma unroll
        for (int e = 0; e < VEC; e++) s += v[e];
      }
      mu = group_sum<L>(s, lds) * inv;
      s = 0.f;
    }
    for (int c = lane * VEC; c < width; c += L * VEC) {
      ldv<VEC>(xr + c, v);
#pragma unroll
      for (int e = 0; e < VEC; e++) s += (v[e] - mu) * (v[e] - mu);
    }
    rstd = 1.f / sqrtf(group_sum<L>(s, lds) * inv + eps);
    for (int c = lane * VEC; c < width; c += L * VEC) {
      float g[VEC], o[VEC];
      ldv<VEC>(xr + c, v);
      ldv<VEC>(w + c, g);
      if (b) ldv<VEC>(b + c, o);
#pragma unroll
      for (int e = 0; e < VEC; e++) o[e] = (v[e] - mu) * rstd * g[e] + (b ? o[e] : 0.f);
      stv<VEC>(yr + c, o);
    }
  }
  if (live && lane == 0) {
    if (mean_out) mean_out[row] = mu;
    rstd_out[row] = rstd;
  }
}

// VEC elements as they lie in memory, in as few registers
template <typename T, int VEC>
struct Raw {
  using type = u32x4;
};
template <typename T>
struct Raw<T, 1> {
  using type = T;
};
template <typename T, int VEC>
__device__ __forceinline__ void widen(const typename Raw<T, VEC>::type& r, float (&v)[VEC]) {
  if constexpr (VEC == 1) v[0] = ldf(&r);
  else ldv<VEC>((const T*)&r, v);
}

// Workgroup p walks over the rows p G + i G gridDim, G = THREADS / L of them at a time, and leaves its share of dw (and db, behind all
// of dw) in part[p][width]; norm_reduce_kernel adds the shares in a fixed order.  One workgroup a CU of as many waves as the
// registers allow: as much on its way as memory needs, and few shares.
template <typename T, int VEC, int L, int NV, bool BIASED, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_backward_kernel(const T* __restrict__ dy, Rows drows, const T* __restrict__ x, Rows rows,
                                                                int width, const T* __restrict__ w, const float* __restrict__ mean,
                                                                const float* __restrict__ rstd, int centered, T* __restrict__ dx,
                                                                float* __restrict__ part) {
  __shared__ float lds[4];
  const int lane = threadIdx.x % L, group = L >= 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / L) : threadIdx.x / L;
  const float inv = 1.f / (float)width;
  float* pw = part + (size_t)blockIdx.x * width;
  float* pb = pw + (size_t)gridDim.x * width;
  constexpr int G = THREADS / L, W = L < 64 ? 64 / L : 1;      // groups; of a wave
  using R = typename Raw<T, VEC>::type;
  if constexpr (NV > 0) {
    __shared__ float sum[G == 1 ? 1 : L * NV * VEC];
    float aw[NV][VEC], ab[BIASED ? NV : 1][VEC];
    R xr[NV], dr[NV];
    float mu = 0.f, r = 0.f;
    auto inside = [&](int i) { return i < full_pieces(L, NV) || (i * L + lane) * VEC < width; };
#pragma unroll
    for (int i = 0; i < NV; i++) {
#pragma unroll
      for (int e = 0; e < VEC; e++) aw[i][e] = 0.f;
      if constexpr (BIASED) {
#pragma unroll
        for (int e = 0; e < VEC; e++) ab[i][e] = 0.f;
      }
    }
    auto fetch = [&](int row) {      // rows behind the last: zeros, which add nothing
      const bool live = row < rows.n;
      mu = live && centered ? mean[row] : 0.f;
      r = live ? rstd[row] : 0.f;
      const T* xp = x + (live ? rows.at(row) : 0);
      const T* dp = dy + (live ? drows.at(row) : 0);
#pragma unroll
      for (int i = 0; i < NV; i++) {
        const int c = (i * L + lane) * VEC;
        xr[i] = R{}, dr[i] = R{};
        if (live && inside(i)) {
          xr[i] = *(const R*)(xp + c);
          dr[i] = *(const R*)(dp + c);
        }
      }
    };
    const int step = (int)gridDim.x * G;      // r0 + step stays below 2^31 + 2^18
    for (unsigned r0 = blockIdx.x * G; r0 < (unsigned)rows.n; r0 += step) {
      const int row = min((int)min(r0 + group, 0x7fffffffu), rows.n);
      // the row stays as it lies in memory and is widened twice
      fetch(row);
      const T* wp = w;
      asm volatile("" : "+s"(wp));      // read anew for every row: kept in 32 bits, the weights would take the registers
      auto widened = [&](int i, float (&gw)[VEC], float (&n)[VEC], float (&d)[VEC]) {
        R g{};
        if (inside(i)) g = *(const R*)(wp + (i * L + lane) * VEC);
        widen<T, VEC>(g, gw);
        widen<T, VEC>(xr[i], n);
        widen<T, VEC>(dr[i], d);
#pragma unroll
        for (int e = 0; e < VEC; e++) n[e] = inside(i) ? (n[e] - mu) * r : 0.f;
      };
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int i = 0; i < NV; i++) {
        float gw[VEC], n[VEC], d[VEC];
        widened(i, gw, n, d);
#pragma unroll
        for (int e = 0; e < VEC; e++) {
          aw[i][e] += d[e] * n[e];
          asm volatile("" : "+v"(aw[i][e]));      // added here: put off to the row's end, every factor stays in a register
          if constexpr (BIASED) {
            ab[i][e] += d[e];
            asm volatile("" : "+v"(ab[i][e]));
          }
          s1 += d[e] * gw[e] * n[e];
          s2 += d[e] * gw[e];
        }
        __builtin_amdgcn_sched_barrier(0);      // one piece in 32 bits at a time
      }
      s1 = group_sum<L>(s1, lds) * inv;
      s2 = centered ? group_sum<L>(s2, lds) * inv : 0.f;
      const bool live = row < rows.n;
      T* out = dx + (int64_t)(live ? row : 0) * width;
#pragma unroll
      for (int i = 0; i < NV; i++) {
        if constexpr (VEC > 1) asm volatile("" : "+v"(xr[i]), "+v"(dr[i]));      // or the compiler keeps both forms
        if (live && inside(i)) {
          float gw[VEC], n[VEC], d[VEC];
          widened(i, gw, n, d);
#pragma unroll
          for (int e = 0; e < VEC; e++) d[e] = (d[e] * gw[e] - n[e] * s1 - s2) * r;
          stv<VEC>(out + (i * L + lane) * VEC, d);
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    // the groups' shares: of a wave by shuffles, then one wave after the other
    auto joined = [&](auto& a, float* to) {
      if constexpr (L < 64) {
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
          for (int e = 0; e < VEC; e++)
#pragma unroll
            for (int o = L; o < 64; o *= 2) a[i][e] += __shfl_xor(a[i][e], o, 64);
      }
      if constexpr (G == 1) {
#pragma unroll
        for (int i = 0; i < NV; i++) {
          const int c = (i * L + lane) * VEC;
#pragma unroll
          for (int e = 0; e < VEC; e++)
            if (c + e < width) to[c + e] = a[i][e];
        }
        return;
      }
      for (int k = 0; k < G; k += W) {
        if (group == k) {
#pragma unroll
          for (int i = 0; i < NV; i++)
#pragma unroll
            for (int e = 0; e < VEC; e++) {
              float* s = sum + (i * VEC + e) * L + lane;
              *s = k == 0 ? a[i][e] : *s + a[i][e];
            }
        }
        __syncthreads();
      }
      for (int c = threadIdx.x; c < width; c += THREADS) {
        const int piece = c / VEC;
        to[c] = sum[(piece / L * VEC + c % VEC) * L + piece % L];
      }
      __syncthreads();
    };
    joined(aw, pw);
    if constexpr (BIASED) joined(ab, pb);
  } else {
    for (int c = lane * VEC; c < width; c += L * VEC)
#pragma unroll
      for (int e = 0; e < VEC; e++) {
        pw[c + e] = 0.f;
        if (BIASED) pb[c + e] = 0.f;
      }
    for (unsigned row = blockIdx.x; row < (unsigned)rows.n; row += gridDim.x) {
      const float mu = centered ? mean[row] : 0.f, r = rstd[row];
      const T* xr = x + rows.at(row);
      const T* dr = dy + drows.at(row);
      float n[VEC], d[VEC], g[VEC], s1 = 0.f, s2 = 0.f;
      for (int c = lane * VEC; c < width; c += L * VEC) {
        ldv<VEC>(xr + c, n);
        ldv<VEC>(dr + c, d);
        ldv<VEC>(w + c, g);
#pragma unroll
        for (int e = 0; e < VEC; e++) {
          n[e] = (n[e] - mu) * r;
          pw[c + e] += d[e] * n[e];
          if (BIASED) pb[c + e] += d[e];
          s1 += d[e] * g[e] * n[e];
          s2 += d[e] * g[e];
        }
      }
      s1 = group_sum<L>(s1, lds) * inv;
      s2 = centered ? group_sum<L>(s2, lds) * inv : 0.f;
      for (int c = lane * VEC; c < width; c += L * VEC) {
        ldv<VEC>(xr + c, n);
        ldv<VEC>(dr + c, d);
        ldv<VEC>(w + c, g);
#pragma unroll
        for (int e = 0; e < VEC; e++) d[e] = (d[e] * g[e] - (n[e] - mu) * r * s1 - s2) * r;
        stv<VEC>(dx + (int64_t)row * width + c, d);
      }
    }
  }
}

// out[c] = sum over n shares of part[p][c]: 32 threads a column, each every 32nd share.
template <typename T>
__global__ __launch_bounds__(1024) void norm_reduce_kernel(const float* __restrict__ part, int n, int width, T* __restrict__ dw,
                                                           T* __restrict__ db) {
  __shared__ float sum[32][33];
  const int x = threadIdx.x & 31, k = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
  const float* p = part + (size_t)blockIdx.y * n * width;
  float s = 0.f;
  if (c < width) {
#pragma unroll 8
    for (int i = k; i < n; i += 32) s += p[(size_t)i * width + c];
  }
  sum[k][x] = s;
  __syncthreads();
  s = sum[x][k];      // column k, shares x
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
  if (x == 0 && blockIdx.x * 32 + k < width) st1((blockIdx.y ? db : dw) + blockIdx.x * 32 + k, s);
}

// Threads that hold a row, and pieces of a row a thread holds (0: the row is read again instead).  Measured, bf16, both directions:
// 7777 x 32 rows of 128 on 16 lanes each 60 us, on a wave each 160; 7777 rows of 2560 on a wave 47 us, on a workgroup 65; 7777 rows of 4096
// on a wave (8 pieces of 8, four waves a CU) 85 us, on a workgroup 69; in fp32 rows of 2048 (8 pieces of 4) 58 and 60.
struct RowPlan { int L, NV; };
RowPlan row_plan(int width, int vec) {
  const int n = (width + vec - 1) / vec;
  for (int l = 8; l <= 64; l *= 2)
    if (n <= l) return {l, 1};
  for (int v : {2, 3, 4, 5, 6, 8})
    if (n <= 64 * v && (v < 8 || vec < 8)) return {64, v};
  for (int v : {2, 3, 4, 6, 8})
    if (n <= 256 * v) return {256, v};
  return {256, 0};
}
template <int VEC, typename F>
void with_row_plan(const RowPlan& p, F f) {
  auto is = [&](auto l, auto v) {
    constexpr int L = decltype(l)::value, NV = decltype(v)::value;
    if constexpr ((VEC < 8 || L != 64 || NV != 8) && (VEC == 8 || L != 256 || NV != 2)) {      // plans of this VEC
      if (p.L == L && p.NV == NV) f(l, v);
    }
  };
#define RL_I(x) std::integral_constant<int, x>()
  is(RL_I(8), RL_I(1)); is(RL_I(16), RL_I(1)); is(RL_I(32), RL_I(1)); is(RL_I(64), RL_I(1)); is(RL_I(64), RL_I(2));
  is(RL_I(64), RL_I(3)); is(RL_I(64), RL_I(4)); is(RL_I(64), RL_I(5)); is(RL_I(64), RL_I(6)); is(RL_I(64), RL_I(8));
  is(RL_I(256), RL_I(2)); is(RL_I(256), RL_I(3)); is(RL_I(256), RL_I(4)); is(RL_I(256), RL_I(6)); is(RL_I(256), RL_I(8)); is(RL_I(256), RL_I(0));
#undef RL_I
}
// Workgroups of the backward pass: one a CU; of four waves (rows that take a workgroup), two.
const int kShares = 512;
constexpr int norm_threads(int L, int NV, int vec, bool biased) {
  const int regs = NV * (vec * (biased ? 2 : 1) + (vec == 8 ? 20 : 14)) + 45;      // what the compiler takes, about
  return L == 256 || regs > 256 ? 256 : regs > 128 ? 512 : 1024;
}
int norm_shares(int rows, const RowPlan& p, int vec, bool biased) {
  const int threads = norm_threads(p.L, p.NV, vec, biased), group = threads / p.L, most = threads == 256 ? 512 : 256;
  const int n = (rows - 1) / group + 1;
  return n < most ? n : most;
}
template <typename T, int VEC>
int norm_forward(const void* x, const Rows& rows, int width, const void* w, const void* b, float eps, int centered, void* y, float* mean,
                 float* rstd, hipStream_t s) {
  const RowPlan p = row_plan(width, VEC);
  with_row_plan<VEC>(p, [&](auto l, auto v) {
    constexpr int L = decltype(l)::value, NV = decltype(v)::value;
    constexpr int64_t most = most_workgroups(256);
    for (int64_t first = 0; first < rows.n; first += most * (256 / L))
      norm_forward_kernel<T, VEC, L, NV><<<(unsigned)std::min(most, (rows.n - first - 1) / (256 / L) + 1), 256, 0, s>>>(
          (const T*)x, rows, (int)first, width, (const T*)w, (const T*)b, eps, centered, (T*)y, mean, rstd);
  });
  return launched();
}
template <typename T, int VEC>
int norm_backward(const void* dy, const Rows& drows, const void* x, const Rows& rows, int width, const void* w, const float* mean,
                  const float* rstd, int centered, void* dx, void* dw, void* db, float* part, hipStream_t s) {
  const RowPlan p = row_plan(width, VEC);
  const int n = norm_shares(rows.n, p, VEC, db != nullptr);
  with_row_plan<VEC>(p, [&](auto l, auto v) {
    constexpr int L = decltype(l)::value, NV = decltype(v)::value;
    auto go = [&](auto biased) {
      constexpr int THREADS = norm_threads(L, NV, VEC, decltype(biased)::value);
      norm_backward_kernel<T, VEC, L, NV, decltype(biased)::value, THREADS><<<n, THREADS, 0, s>>>(
          (const T*)dy, drows, (const T*)x, rows, width, (const T*)w, mean, rstd, centered, (T*)dx, part);
    };
    if (db) go(std::true_type());
    else go(std::false_type());
  });
  norm_reduce_kernel<T><<<dim3((width + 31) / 32, db ? 2 : 1), 1024, 0, s>>>(part, n, width, (T*)dw, (T*)db);
  return launched();
}

const int64_t kMostWidth = 32 * most_workgroups(1024);      // what the sums over rows launch for
const char* norm_argument(const void* x, int64_t outer, int32_t inner, int32_t width, int32_t dtype) {
  if (outer < 0 || inner < 1 || width < 1 || outer > 0x7fffffff / inner || width > kMostWidth)
    return "outer, inner or width out of range (rows: below 2^31, width: below 2^27 - 32)";
  if (dtype != RL_DTYPE_F32 && dtype != RL_DTYPE_BF16) return "dtype is RL_DTYPE_F32 or RL_DTYPE_BF16";
  if (outer > 0 && !x) return "null pointer";
  return nullptr;
}

}  // namespace

extern "C" int rl_norm_forward(const void* d_x, int64_t outer, int32_t inner, int32_t width, int64_t outer_stride, int64_t inner_stride,
                               const void* d_weight, const void* d_bias, float eps, int32_t centered, int32_t dtype, void* d_y,
                               float* d_mean, float* d_rstd, void* stream) {
  if (const char* m = norm_argument(d_x, outer, inner, width, dtype)) return rl_fail(RL_E_ARG, m);
  if (!(eps >= 0.f)) return rl_fail(RL_E_ARG, "eps is negative or no number");
  if (outer == 0) return RL_OK;
  if (!d_weight || !d_y || !d_rstd || (centered && !d_mean)) return rl_fail(RL_E_ARG, "null pointer");
  const Rows rows(outer * inner, outer_stride, inner_stride, inner);
  auto vec = [&](int n) {
    return width % n == 0 && outer_stride % n == 0 && (inner == 1 || inner_stride % n == 0) && aligned16(d_x) && aligned16(d_weight) &&
           aligned16(d_bias) && aligned16(d_y);
  };
  hipStream_t s = (hipStream_t)stream;
#define RL_GO(T, V) norm_forward<T, V>(d_x, rows, width, d_weight, d_bias, eps, centered, d_y, centered ? d_mean : nullptr, d_rstd, s)
  if (dtype == RL_DTYPE_F32) return vec(4) ? RL_GO(float, 4) : RL_GO(float, 1);
  return vec(8) ? RL_GO(bf16_t, 8) : RL_GO(bf16_t, 1);
#undef RL_GO
}

extern "C" int64_t rl_norm_workspace(int64_t rows, int32_t width, int32_t biased) {
  if (rows < 0 || rows > 0x7fffffff || width < 1 || width > kMostWidth) return 0;
  const int64_t n = rows < kShares ? rows : kShares;      // as many shares as any plan makes
  return n * width * (biased ? 2 : 1) * (int64_t)sizeof(float);
}

extern "C" int rl_norm_backward(const void* d_dy, int64_t dy_outer_stride, int64_t dy_inner_stride, const void* d_x, int64_t outer,
                                int32_t inner, int32_t width, int64_t outer_stride, int64_t inner_stride, const void* d_weight,
                                const float* d_mean, const float* d_rstd, int32_t centered, int32_t dtype, void* d_dx, void* d_dweight,
                                void* d_dbias, void* d_workspace, int64_t workspace_bytes, void* stream) {
  if (const char* m = norm_argument(d_x, outer, inner, width, dtype)) return rl_fail(RL_E_ARG, m);
  if (!d_weight || !d_dweight) return rl_fail(RL_E_ARG, "null pointer");
  if (outer > 0 && (!d_dy || !d_rstd || !d_dx || !d_workspace || (centered && !d_mean))) return rl_fail(RL_E_ARG, "null pointer");
  if (workspace_bytes < rl_norm_workspace(outer * inner, width, d_dbias != nullptr)) return rl_fail(RL_E_ARG, "workspace smaller than rl_norm_workspace says");
  if ((uintptr_t)d_workspace & 3) return rl_fail(RL_E_ARG, "workspace not aligned to 4 bytes");
  const Rows rows(outer * inner, outer_stride, inner_stride, inner), drows(outer * inner, dy_outer_stride, dy_inner_stride, inner);
  auto vec = [&](int n) {
    return width % n == 0 && outer_stride % n == 0 && dy_outer_stride % n == 0 &&
           (inner == 1 || (inner_stride % n == 0 && dy_inner_stride % n == 0)) && aligned16(d_x) && aligned16(d_dy) && aligned16(d_weight) &&
           aligned16(d_dx);
  };
  hipStream_t s = (hipStream_t)stream;
#define RL_GO(T, V) \
  norm_backward<T, V>(d_dy, drows, d_x, rows, width, d_weight, d_mean, d_rstd, centered, d_dx, d_dweight, d_dbias, (float*)d_workspace, s)
  if (outer == 0) {      // no rows: sums of nothing
    if (dtype == RL_DTYPE_F32)
      norm_reduce_kernel<float><<<dim3((width + 31) / 32, d_dbias ? 2 : 1), 1024, 0, s>>>(nullptr, 0, width, (float*)d_dweight, (float*)d_dbias);
    else
      norm_reduce_kernel<bf16_t><<<dim3((width + 31) / 32, d_dbias ? 2 : 1), 1024, 0, s>>>(nullptr, 0, width, (bf16_t*)d_dweight, (bf16_t*)d_dbias);
    return launched();
  }
  if (dtype == RL_DTYPE_F32) return vec(4) ? RL_GO(float, 4) : RL_GO(float, 1);
  return vec(8) ? RL_GO(bf16_t, 8) : RL_GO(bf16_t, 1);
#undef RL_GO
}

// =============================================================================================
// Rotary positions.  Pair i of a head's first rot_dim elements, (a, b) = elements (i, i + rot_dim / 2) or (2 i, 2 i + 1), becomes
// (a c - b s, b c + a s) with (c, s) = table[position][i]; the others are copied.  The map is linear and the backward pass is its
// transpose, the same with -s (`sign`).  Bound by memory: q and k in and out.  A workgroup is one token: a thread keeps the cos and
// sin of its VEC pairs and walks over the heads, so the table, twice the bytes of a head, is read once a token.  Measured: 12007 tokens of 32 + 8
// heads of 128 in bf16, both directions 95 us (5.2 TB/s, q and k in part from the cache); 128 tokens, one direction 5.7 us (one launch).
// =============================================================================================
namespace {

struct RotaryTensor {
  const void* in;
  void* out;
  int heads;
  int64_t it, ih, ot, oh;      // strides of token and head, in elements
};

template <typename T, int VEC, bool INTERLEAVED>
__global__ void rotary_kernel(RotaryTensor q, RotaryTensor k, const int32_t* __restrict__ positions, const float* __restrict__ table,
                              int n_positions, int rot_dim, int head_dim, float sign) {
  // chunks of a head: VEC pairs each (neighbouring pairs: VEC / 2, or one), then VEC elements behind rot_dim each
  constexpr int P = INTERLEAVED && VEC > 1 ? VEC / 2 : VEC;
  constexpr int E = INTERLEAVED ? (VEC > 1 ? VEC : 2) : VEC;      // elements of the first access
  const int half = rot_dim >> 1, turned = half / P, c = threadIdx.x;
  const int64_t t = blockIdx.x;
  float cs[P], sn[P];
  if (c < turned) {
    const int pos = positions[t];
    if ((unsigned)pos < (unsigned)n_positions) {
      const float2* row = (const float2*)table + (size_t)pos * half + c * P;
#pragma unroll
      for (int i = 0; i < P; i++) {
        const float2 f = row[i];
        cs[i] = f.x;
        sn[i] = f.y * sign;
      }
    } else {      // no such position
#pragma unroll
      for (int i = 0; i < P; i++) cs[i] = sn[i] = __builtin_nanf("");
    }
  }
  for (int h = threadIdx.y; h < q.heads + k.heads; h += blockDim.y) {
    const bool first = h < q.heads;
    const RotaryTensor& x = first ? q : k;
    const int hh = first ? h : h - q.heads;
    const T* in = (const T*)x.in + t * x.it + hh * x.ih;
    T* out = (T*)x.out + t * x.ot + hh * x.oh;
    if (c >= turned) {
      const int at = rot_dim + (c - turned) * VEC;
      float v[VEC];
      ldv<VEC>(in + at, v);
      stv<VEC>(out + at, v);
    } else if constexpr (INTERLEAVED) {
      float v[E];
      if constexpr (VEC > 1) {
        ldv<VEC>(in + c * VEC, v);
      } else {
        v[0] = ldf(in + 2 * c);
        v[1] = ldf(in + 2 * c + 1);
      }
#pragma unroll
      for (int i = 0; i < P; i++) {
        const float a = v[2 * i], b = v[2 * i + 1];
        v[2 * i] = a * cs[i] - b * sn[i];
        v[2 * i + 1] = b * cs[i] + a * sn[i];
      }
      if constexpr (VEC > 1) {
        stv<VEC>(out + c * VEC, v);
      } else {
        st1(out + 2 * c, v[0]);
        st1(out + 2 * c + 1, v[1]);
      }
    } else {
      float a[VEC], b[VEC];
      ldv<VEC>(in + c * VEC, a);
      ldv<VEC>(in + half + c * VEC, b);
#pragma unroll
      for (int i = 0; i < VEC; i++) {
        const float u = a[i];
        a[i] = u * cs[i] - b[i] * sn[i];
        b[i] = b[i] * cs[i] + u * sn[i];
      }
      stv<VEC>(out + c * VEC, a);
      stv<VEC>(out + half + c * VEC, b);
    }
  }
}

template <typename T, int VEC, bool INTERLEAVED>
int rotary(const RotaryTensor& q, const RotaryTensor& k, int64_t tokens, const int32_t* positions, const float* table, int n_positions,
           int rot_dim, int head_dim, float sign, hipStream_t s) {
  constexpr int P = INTERLEAVED && VEC > 1 ? VEC / 2 : VEC;
  const int nc = rot_dim / 2 / P + (head_dim - rot_dim) / VEC, heads = q.heads + k.heads;
  const int hl = 256 / nc < 1 ? 1 : 256 / nc < heads ? 256 / nc : heads;
  const int64_t most = most_workgroups(nc * hl);
  auto from = [](const RotaryTensor& x, int64_t t) {      // tokens from t on; a null tensor has no heads
    RotaryTensor y = x;
    y.in = (const T*)x.in + t * x.it;
    y.out = (T*)x.out + t * x.ot;
    return y;
  };
  for (int64_t t = 0; t < tokens; t += most)
    rotary_kernel<T, VEC, INTERLEAVED><<<(unsigned)std::min(most, tokens - t), dim3(nc, hl), 0, s>>>(from(q, t), from(k, t), positions + t, table,
                                                                                                   n_positions, rot_dim, head_dim, sign);
  return launched();
}

}  // namespace

extern "C" int rl_rotary(const void* d_q, void* d_q_out, int32_t n_q_heads, int64_t q_token_stride, int64_t q_head_stride,
                         int64_t q_out_token_stride, int64_t q_out_head_stride, const void* d_k, void* d_k_out, int32_t n_k_heads,
                         int64_t k_token_stride, int64_t k_head_stride, int64_t k_out_token_stride, int64_t k_out_head_stride,
                         int64_t tokens, int32_t head_dim, int32_t rot_dim, int32_t interleaved, int32_t inverse,
                         const int32_t* d_positions, const float* d_table, int32_t n_positions, int32_t dtype, void* stream) {
  if (dtype != RL_DTYPE_F32 && dtype != RL_DTYPE_BF16) return rl_fail(RL_E_ARG, "dtype is RL_DTYPE_F32 or RL_DTYPE_BF16");
  if (head_dim < 1 || head_dim > 512 || rot_dim < 0 || (rot_dim & 1) || rot_dim > head_dim)
    return rl_fail(RL_E_ARG, "head_dim is 1 to 512, rot_dim even and at most head_dim");
  if (tokens < 0 || tokens > 0x7fffffff || n_q_heads < 1 || n_k_heads < 0 || n_q_heads > 65536 || n_k_heads > 65536 || n_positions < 1)
    return rl_fail(RL_E_ARG, "tokens, heads or positions out of range");
  if (tokens == 0) return RL_OK;
  if (!d_q || !d_q_out || !d_positions || !d_table || (n_k_heads > 0 && (!d_k || !d_k_out))) return rl_fail(RL_E_ARG, "null pointer");
  if ((uintptr_t)d_table & 7) return rl_fail(RL_E_ARG, "table not aligned to 8 bytes");
  const RotaryTensor q{d_q, d_q_out, n_q_heads, q_token_stride, q_head_stride, q_out_token_stride, q_out_head_stride};
  const RotaryTensor k{d_k, d_k_out, n_k_heads, k_token_stride, k_head_stride, k_out_token_stride, k_out_head_stride};
  auto vec = [&](int n) {
    auto one = [&](const RotaryTensor& x) {
      return aligned16(x.in) && aligned16(x.out) && x.it % n == 0 && x.ih % n == 0 && x.ot % n == 0 && x.oh % n == 0;
    };
    return head_dim % n == 0 && rot_dim % (interleaved ? n : 2 * n) == 0 && one(q) && (n_k_heads == 0 || one(k));
  };
  hipStream_t s = (hipStream_t)stream;
  const float sign = inverse ? -1.f : 1.f;
#define RL_GO(T, V) \
  (interleaved ? rotary<T, V, true>(q, k, tokens, d_positions, d_table, n_positions, rot_dim, head_dim, sign, s) \
               : rotary<T, V, false>(q, k, tokens, d_positions, d_table, n_positions, rot_dim, head_dim, sign, s))
  if (dtype == RL_DTYPE_F32) return vec(4) ? RL_GO(float, 4) : RL_GO(float, 1);
  return vec(8) ? RL_GO(bf16_t, 8) : RL_GO(bf16_t, 1);
#undef RL_GO
}
