// The residual stream around a block: the block's result, normed and gated where wanted, joins the stream, and the norm before the next block
// follows; forward and backward.
#include <algorithm>
#include <type_traits>

#include "policy_common.h"

namespace {

// =============================================================================================
// u = y, or norm(y) pw (+ pb);  h' = rs h + bs g u;  a = norm(h') w (+ b), with g nothing, one value a column, a row or an element, and the norm of
// kernels_rows.hip (RMS, or layer norm where `centered`).
// Backward, from dh' and da:  dH = dh' + r (da w - n mean(da w n) [- mean(da w)]),  dh = rs dH,  dU = bs g dH,  dg = bs u dH (summed over what shares a
// gate),  dy = dU or the post norm's gradient of it; sums over rows for the weights, the biases and a gate a column.
// Bound by memory: h and y in, h' and a out; backward dh', da, h' and y in, dh and dy out.  A row is held in registers by L threads, NV pieces of VEC
// elements each, so everything is read once; NV = 0 takes rows too long for that in several passes.  The stream may be in 32 bits beside a block
// in bf16 (S, T).  Everything is computed in 32 bits and rounded once; a is the norm of h' before its rounding.
// 7777 x 2560, stream in 32 bits, block in bf16: forward 239 MB in 56 us (4.3 TB/s), backward 319 MB in 57 us (5.6 TB/s, h' partly still in the last cache)
// and 4.7 us for the sums of the shares; 128 rows forward 6.2 us, of which a launch alone is most.
// =============================================================================================
struct Shape {
  int rows, width;
  int64_t h, y, gate, dh, da;      // strides of rows
  int gate_column;                 // 1: a gate for each column of a row
  int centered;
  float rs, bs, eps;
};
template <typename S, typename T>
struct ForwardCall {
  Shape n;
  const S* h;
  const T *y, *weight, *bias, *post_weight, *post_bias, *gate;
  S* out;
  T* a;                            // null: no norm
  float4* stats;                   // mean and rstd of the row, of the block's row
};
template <typename S, typename T>
struct BackwardCall {
  Shape n;
  const S *dout, *out;             // dout null: 0
  const T *da, *y, *weight, *post_weight, *post_bias, *gate;      // da null: no norm
  const float4* stats;
  S* dh;
  T *dy, *dgate;                   // dgate: of a row or an element
  int gate_sums, biased, post_biased;      // sums over rows that are wanted beside those of the weights
  float* part;                     // [sum][share][width]
};
enum { SUM_WEIGHT, SUM_BIAS, SUM_POST_WEIGHT, SUM_POST_BIAS, SUM_GATE, SUMS };

// Sums of two numbers over the L threads of a row; every thread of the workgroup calls it equally often.
template <int L>
struct Joined {
  float2* lds;      // two halves, used in turn: whoever writes one again has passed the barrier behind the reads of it
  int turn = 0;
  __device__ __forceinline__ float2 operator()(float a, float b) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      a += __shfl_xor(a, o, 64);
      b += __shfl_xor(b, o, 64);
    }
    if constexpr (L > 64) {
      constexpr int W = L / 64;
      float2* const at = lds + turn * W;
      if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = make_float2(a, b);
      __syncthreads();
      a = b = 0.f;
#pragma unroll
      for (int w = 0; w < W; w++) a += at[w].x, b += at[w].y;
      turn ^= 1;
    }
    return make_float2(a, b);
  }
};

template <int N, typename X>
__device__ __forceinline__ void row_of(const X* p, int c, float (&v)[N]) { ldv<N>(p + c, v); }
// Gates of N elements from column c on
template <int N, typename T>
__device__ __forceinline__ void gates(const T* g, const Shape& n, int row, int c, float (&v)[N]) {
  const T* p = g + row * n.gate;
  if (n.gate_column) {
    ldv<N>(p + c, v);
  } else {
    const float x = ldf(p);
#pragma unroll
    for (int e = 0; e < N; e++) v[e] = x;
  }
}

template <typename S, typename T, int VEC, int L, int NV>
__global__ __launch_bounds__(L > 256 ? L : 256) void residual_norm_forward_kernel(ForwardCall<S, T> f) {
  constexpr int THREADS = L > 256 ? L : 256, PIECES = NV > 0 ? NV : 1;
  __shared__ float2 lds[2 * (L > 64 ? L / 64 : 1)];
  Joined<L> joined{lds};
  const Shape& n = f.n;
  const int lane = threadIdx.x % L, row = (int)blockIdx.x * (THREADS / L) + (L == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / L) : 0);
  if (row >= n.rows) return;      // of a wave of its own, or of the whole workgroup
  const float inv = 1.f / (float)n.width;
  const S* hr = f.h + row * n.h;
  const T* yr = f.y + row * n.y;
  S* const out = f.out + (int64_t)row * n.width;
  float mu = 0.f, rstd = 0.f, pmu = 0.f, prstd = 0.f;
  // one piece of the stream, from a piece of the block's result
  auto stream = [&](int c, const float (&y)[VEC], const float (&h)[VEC], float (&to)[VEC]) {
    float u[VEC], x[VEC];
#pragma unroll
    for (int e = 0; e < VEC; e++) u[e] = y[e];
    if (f.post_weight) {
      row_of<VEC>(f.post_weight, c, x);
#pragma unroll
      for (int e = 0; e < VEC; e++) u[e] = (u[e] - pmu) * prstd * x[e];
      if (f.post_bias) {
        row_of<VEC>(f.post_bias, c, x);
#pragma unroll
        for (int e = 0; e < VEC; e++) u[e] += x[e];
      }
    }
    if (f.gate) {
      gates<VEC>(f.gate, n, row, c, x);
#pragma unroll
      for (int e = 0; e < VEC; e++) u[e] *= x[e];
    }
#pragma unroll
    for (int e = 0; e < VEC; e++) to[e] = n.rs * h[e] + n.bs * u[e];
  };
  auto normed = [&](int c, const float (&h)[VEC]) {
    float w[VEC], b[VEC];
    row_of<VEC>(f.weight, c, w);
    if (f.bias) row_of<VEC>(f.bias, c, b);
#pragma unroll
    for (int e = 0; e < VEC; e++) w[e] = (h[e] - mu) * rstd * w[e] + (f.bias ? b[e] : 0.f);
    stv<VEC>(f.a + (int64_t)row * n.width + c, w);
  };
  if constexpr (NV > 0) {
    float y[PIECES][VEC], h[PIECES][VEC];
    auto inside = [&](int i) { return (i * L + lane) * VEC < n.width; };
#pragma unroll
    for (int i = 0; i < NV; i++) {
      const int c = (i * L + lane) * VEC;
#pragma unroll
      for (int e = 0; e < VEC; e++) y[i][e] = h[i][e] = 0.f;
      if (inside(i)) {
        row_of<VEC>(yr, c, y[i]);
        row_of<VEC>(hr, c, h[i]);
      }
    }
    auto moments = [&](float (&v)[PIECES][VEC], float& m, float& r) {
      m = 0.f;
      if (n.centered) {
        float s = 0.f;
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
          for (int e = 0; e < VEC; e++) s += v[i][e];
        m = joined(s, 0.f).x * inv;
      }
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < NV; i++)
#pragma unroll
        for (int e = 0; e < VEC; e++) s += inside(i) ? (v[i][e] - m) * (v[i][e] - m) : 0.f;
      r = 1.f / sqrtf(joined(s, 0.f).x * inv + n.eps);
    };
    if (f.post_weight) moments(y, pmu, prstd);
#pragma unroll
    for (int i = 0; i < NV; i++)
      if (inside(i)) {
        const int c = (i * L + lane) * VEC;
        stream(c, y[i], h[i], h[i]);
        stv<VEC>(out + c, h[i]);
      }
    if (f.a) {
      moments(h, mu, rstd);
#pragma unroll
      for (int i = 0; i < NV; i++)
        if (inside(i)) normed((i * L + lane) * VEC, h[i]);
    }
  } else {
    float y[VEC], h[VEC];
    auto moments = [&](auto get, float& m, float& r) {
      m = 0.f;
      float v[VEC];
      if (n.centered) {
        float s = 0.f;
        for (int c = lane * VEC; c < n.width; c += L * VEC) {
          get(c, v);
#pragma unroll
          for (int e = 0; e < VEC; e++) s += v[e];
        }
        m = joined(s, 0.f).x * inv;
      }
      float s = 0.f;
      for (int c = lane * VEC; c < n.width; c += L * VEC) {
        get(c, v);
#pragma unroll
        for (int e = 0; e < VEC; e++) s += (v[e] - m) * (v[e] - m);
      }
      r = 1.f / sqrtf(joined(s, 0.f).x * inv + n.eps);
    };
    auto of_block = [&](int c, float (&v)[VEC]) { row_of<VEC>(yr, c, v); };
    auto of_stream = [&](int c, float (&v)[VEC]) {      // formed anew: what was stored is rounded
      row_of<VEC>(yr, c, y);
      row_of<VEC>(hr, c, h);
      stream(c, y, h, v);
    };
    if (f.post_weight) moments(of_block, pmu, prstd);
    if (f.a) moments(of_stream, mu, rstd);
    for (int c = lane * VEC; c < n.width; c += L * VEC) {
      float v[VEC];
      of_stream(c, v);
      stv<VEC>(out + c, v);
      if (f.a) normed(c, v);
    }
  }
  if (lane == 0) f.stats[row] = make_float4(mu, rstd, pmu, prstd);
}

// Workgroup p walks over the rows p G + i G gridDim, G = THREADS / L at a time, and leaves its share of the sums over rows; reduce_kernel adds the
// shares in a fixed order.  PLAIN: no norm behind the block, no gate, no bias: one sum.
template <typename S, typename T, int VEC, int L, int NV, bool PLAIN>
__global__ __launch_bounds__(L > 256 ? L : 256) void residual_norm_backward_kernel(BackwardCall<S, T> f) {
  constexpr int THREADS = L > 256 ? L : 256, G = THREADS / L, PIECES = NV > 0 ? NV : 1, KINDS = PLAIN ? 1 : SUMS;
  __shared__ float2 lds[2 * (L > 64 ? L / 64 : 1)];
  __shared__ float shared_sum[G > 1 ? PIECES * VEC * L : 1];
  Joined<L> joined{lds};
  const Shape& n = f.n;
  const int lane = threadIdx.x % L, group = L == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / L) : 0;
  const float inv = 1.f / (float)n.width;
  const bool post = !PLAIN && f.post_weight, gated = !PLAIN && f.gate;
  auto wanted = [&](int kind) {
    if (kind == SUM_WEIGHT) return f.da != nullptr;
    return !PLAIN && (kind == SUM_BIAS ? f.biased : kind == SUM_POST_WEIGHT ? post : kind == SUM_POST_BIAS ? f.post_biased : f.gate_sums) != 0;
  };
  auto share = [&](int kind) { return f.part + ((int64_t)kind * gridDim.x + blockIdx.x) * n.width; };
  float sum[KINDS][PIECES][VEC];
#pragma unroll
  for (int k = 0; k < KINDS; k++)
#pragma unroll
    for (int i = 0; i < PIECES; i++)
#pragma unroll
      for (int e = 0; e < VEC; e++) sum[k][i][e] = 0.f;
  if constexpr (NV == 0) {
    for (int k = 0; k < KINDS; k++)
      if (wanted(k)) {
        float* to = share(k);
        for (int c = lane; c < n.width; c += L) to[c] = 0.f;
      }
    __syncthreads();
  }
  const int step = (int)gridDim.x * G;
  for (int r0 = blockIdx.x * G; r0 < n.rows; r0 += step) {
    const int row = r0 + group;
    if (L == 64 && row >= n.rows) break;      // a wave's own rows
    const float4 st = f.stats[row];
    const float mu = st.x, r = st.y, pmu = st.z, pr = st.w;
    // of a piece: dn = da w and n; sums of the first norm's gradient
    auto read = [&](int c, float (&dn)[VEC], float (&nn)[VEC], float (&da)[VEC]) {
      float w[VEC];
      row_of<VEC>(f.da + row * n.da, c, da);
      row_of<VEC>(f.out + (int64_t)row * n.h, c, nn);
      row_of<VEC>(f.weight, c, w);
#pragma unroll
      for (int e = 0; e < VEC; e++) {
        nn[e] = (nn[e] - mu) * r;
        dn[e] = da[e] * w[e];
      }
    };
    // of a piece, from dH: dh, dU and what the post norm and the gate take
    float gate_dot = 0.f;
    auto pass = [&](int c, const float (&dH)[VEC], float (&y)[VEC], float (&dU)[VEC], auto add) {
      float x[VEC], u[VEC];
#pragma unroll
      for (int e = 0; e < VEC; e++) dU[e] = n.bs * dH[e];
      if constexpr (!PLAIN) {
        if (post || gated) row_of<VEC>(f.y + row * n.y, c, y);
        if (post) {
#pragma unroll
          for (int e = 0; e < VEC; e++) y[e] = (y[e] - pmu) * pr;
        }
        if (gated) {
#pragma unroll
          for (int e = 0; e < VEC; e++) u[e] = y[e];
          if (post) {
            row_of<VEC>(f.post_weight, c, x);
#pragma unroll
            for (int e = 0; e < VEC; e++) u[e] *= x[e];
            if (f.post_bias) {
              row_of<VEC>(f.post_bias, c, x);
#pragma unroll
              for (int e = 0; e < VEC; e++) u[e] += x[e];
            }
          }
          gates<VEC>(f.gate, n, row, c, x);
#pragma unroll
          for (int e = 0; e < VEC; e++) {
            u[e] *= dU[e];
            dU[e] *= x[e];
          }
          if (f.gate_sums) {
            add(SUM_GATE, u);
          } else if (f.dgate) {
            if (n.gate_column) {
              stv<VEC>(f.dgate + (int64_t)row * n.width + c, u);
            } else {
#pragma unroll
              for (int e = 0; e < VEC; e++) gate_dot += u[e];
            }
          }
        }
        if (post) {
          if (f.post_biased) add(SUM_POST_BIAS, dU);
          row_of<VEC>(f.post_weight, c, x);
#pragma unroll
          for (int e = 0; e < VEC; e++) u[e] = dU[e] * y[e];
          add(SUM_POST_WEIGHT, u);
#pragma unroll
          for (int e = 0; e < VEC; e++) dU[e] *= x[e];
        }
      }
    };
    if constexpr (NV > 0) {
      float dn[PIECES][VEC], nn[PIECES][VEC], dH[PIECES][VEC];
      auto inside = [&](int i) { return (i * L + lane) * VEC < n.width; };
      float s1 = 0.f, s2 = 0.f;
#pragma unroll
      for (int i = 0; i < NV; i++) {
        const int c = (i * L + lane) * VEC;
#pragma unroll
        for (int e = 0; e < VEC; e++) dn[i][e] = nn[i][e] = dH[i][e] = 0.f;
        if (inside(i)) {
          if (f.dout) row_of<VEC>(f.dout + row * n.dh, c, dH[i]);
          if (f.da) {
            float da[VEC];
            read(c, dn[i], nn[i], da);
#pragma unroll
            for (int e = 0; e < VEC; e++) {
              sum[SUM_WEIGHT][i][e] += da[e] * nn[i][e];
              if constexpr (!PLAIN) sum[SUM_BIAS][i][e] += da[e];
              s1 += dn[i][e] * nn[i][e];
              s2 += dn[i][e];
            }
          }
        }
      }
      if (f.da) {
        const float2 s = joined(s1, s2);
        s1 = s.x * inv, s2 = n.centered ? s.y * inv : 0.f;
#pragma unroll
        for (int i = 0; i < NV; i++)
#pragma unroll
          for (int e = 0; e < VEC; e++) dH[i][e] += r * (dn[i][e] - nn[i][e] * s1 - s2);
      }
      float t1 = 0.f, t2 = 0.f;
#pragma unroll
      for (int i = 0; i < NV; i++)
        if (inside(i)) {
          const int c = (i * L + lane) * VEC;
          float out[VEC];
#pragma unroll
          for (int e = 0; e < VEC; e++) out[e] = n.rs * dH[i][e];
          stv<VEC>(f.dh + (int64_t)row * n.width + c, out);
          pass(c, dH[i], nn[i], dn[i], [&](int kind, const float (&v)[VEC]) {
            if constexpr (!PLAIN) {
#pragma unroll
              for (int e = 0; e < VEC; e++) sum[kind][i][e] += v[e];
            }
          });
          if (post) {
#pragma unroll
            for (int e = 0; e < VEC; e++) {
              t1 += dn[i][e] * nn[i][e];
              t2 += dn[i][e];
            }
          }
        }
      if (post) {
        const float2 s = joined(t1, t2);
        t1 = s.x * inv, t2 = n.centered ? s.y * inv : 0.f;
      }
#pragma unroll
      for (int i = 0; i < NV; i++)
        if (inside(i)) {
          if (post) {
#pragma unroll
            for (int e = 0; e < VEC; e++) dn[i][e] = pr * (dn[i][e] - nn[i][e] * t1 - t2);
          }
          stv<VEC>(f.dy + (int64_t)row * n.width + (i * L + lane) * VEC, dn[i]);
        }
    } else {
      float dn[VEC], nn[VEC], dH[VEC], da[VEC], s1 = 0.f, s2 = 0.f;
      auto to_share = [&](int kind, int c, const float (&v)[VEC]) {
        float* to = share(kind) + c;
#pragma unroll
        for (int e = 0; e < VEC; e++) to[e] += v[e];
      };
      if (f.da) {
        for (int c = lane * VEC; c < n.width; c += L * VEC) {
          read(c, dn, nn, da);
          if (wanted(SUM_BIAS)) to_share(SUM_BIAS, c, da);
#pragma unroll
          for (int e = 0; e < VEC; e++) {
            da[e] *= nn[e];
            s1 += dn[e] * nn[e];
            s2 += dn[e];
          }
          to_share(SUM_WEIGHT, c, da);
        }
        const float2 s = joined(s1, s2);
        s1 = s.x * inv, s2 = n.centered ? s.y * inv : 0.f;
      }
      auto of_stream = [&](int c) {
#pragma unroll
        for (int e = 0; e < VEC; e++) dH[e] = 0.f;
        if (f.dout) row_of<VEC>(f.dout + row * n.dh, c, dH);
        if (f.da) {
          read(c, dn, nn, da);
#pragma unroll
          for (int e = 0; e < VEC; e++) dH[e] += r * (dn[e] - nn[e] * s1 - s2);
        }
      };
      float t1 = 0.f, t2 = 0.f;
      for (int c = lane * VEC; c < n.width; c += L * VEC) {
        of_stream(c);
        float out[VEC];
#pragma unroll
        for (int e = 0; e < VEC; e++) out[e] = n.rs * dH[e];
        pass(c, dH, nn, dn, [&](int kind, const float (&v)[VEC]) { to_share(kind, c, v); });
        stv<VEC>(f.dh + (int64_t)row * n.width + c, out);
        if (post) {
#pragma unroll
          for (int e = 0; e < VEC; e++) {
            t1 += dn[e] * nn[e];
            t2 += dn[e];
          }
        } else {
          stv<VEC>(f.dy + (int64_t)row * n.width + c, dn);
        }
      }
      if (post) {
        const float2 s = joined(t1, t2);
        t1 = s.x * inv, t2 = n.centered ? s.y * inv : 0.f;
        const float dot = gate_dot;
        for (int c = lane * VEC; c < n.width; c += L * VEC) {
          of_stream(c);
          pass(c, dH, nn, dn, [](int, const float (&)[VEC]) {});
#pragma unroll
          for (int e = 0; e < VEC; e++) dn[e] = pr * (dn[e] - nn[e] * t1 - t2);
          stv<VEC>(f.dy + (int64_t)row * n.width + c, dn);
        }
        gate_dot = dot;
      }
    }
    if constexpr (!PLAIN) {
      if (f.gate && f.dgate && !n.gate_column) {      // one gate a row
        const float dot = joined(gate_dot, 0.f).x;
        if (lane == 0) st1(f.dgate + row, dot);
      }
    }
  }
  if constexpr (NV > 0) {
#pragma unroll
    for (int k = 0; k < KINDS; k++) {
      if (!wanted(k)) continue;
      float* to = share(k);
      if constexpr (G == 1) {
#pragma unroll
        for (int i = 0; i < NV; i++) {
          const int c = (i * L + lane) * VEC;
          if (c < n.width) stv<VEC>(to + c, sum[k][i]);
        }
      } else {      // one wave after the other
        for (int g = 0; g < G; g++) {
          if (group == g) {
#pragma unroll
            for (int i = 0; i < NV; i++)
#pragma unroll
              for (int e = 0; e < VEC; e++) {
                float* s = shared_sum + (i * VEC + e) * L + lane;
                *s = g == 0 ? sum[k][i][e] : *s + sum[k][i][e];
              }
          }
          __syncthreads();
        }
        for (int c = threadIdx.x; c < n.width; c += THREADS) {
          const int piece = c / VEC;
          to[c] = shared_sum[(piece / L * VEC + c % VEC) * L + piece % L];
        }
        __syncthreads();
      }
    }
  }
}

// to[kind][c] = sum over n shares of part[kind][share][c]: 32 threads a column, each every 32nd share.
template <typename T>
struct Results { T* to[SUMS]; };
template <typename T>
__global__ __launch_bounds__(1024) void reduce_kernel(const float* __restrict__ part, int n, int width, Results<T> results) {
  __shared__ float sum[32][33];
  T* const to = results.to[blockIdx.y];
  if (!to) return;
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
  if (x == 0 && blockIdx.x * 32 + k < width) st1(to + blockIdx.x * 32 + k, s);
}

// Threads that hold a row, and pieces of it a thread holds (0: the row is read again instead): one wave as long as its registers hold the row, for its sums need no
// barrier.  The backward pass keeps up to four sums a column beside it and goes to more threads earlier.
struct RowPlan { int L, NV; };
RowPlan forward_plan(int width, int vec) {
  const int n = (width + vec - 1) / vec;
  for (int v : {1, 2, 3, 4, 5, 6})
    if (n <= 64 * v) return {64, v};
  for (int v : {2, 4})
    if (n <= 256 * v) return {256, v};
  for (int v : {2, 4})
    if (n <= 1024 * v) return {1024, v};
  return {256, 0};
}
RowPlan backward_plan(int width, int vec) {
  const int n = (width + vec - 1) / vec;
  for (int v : {1, 2})
    if (n <= 64 * v) return {64, v};
  for (int v : {1, 2, 4})
    if (n <= 256 * v) return {256, v};
  for (int v : {2, 4})      // of more elements, the sums do not fit the registers of 1024 threads
    if (n <= 1024 * v && v * vec <= 8) return {1024, v};
  return {256, 0};
}
#define RL_I(x) std::integral_constant<int, x>()
template <typename F>
void with_forward(const RowPlan& p, F f) {
  auto is = [&](auto l, auto v) {
    if (p.L == decltype(l)::value && p.NV == decltype(v)::value) f(l, v);
  };
  is(RL_I(64), RL_I(1)); is(RL_I(64), RL_I(2)); is(RL_I(64), RL_I(3)); is(RL_I(64), RL_I(4)); is(RL_I(64), RL_I(5)); is(RL_I(64), RL_I(6));
  is(RL_I(256), RL_I(2)); is(RL_I(256), RL_I(4)); is(RL_I(1024), RL_I(2)); is(RL_I(1024), RL_I(4)); is(RL_I(256), RL_I(0));
}
template <int VEC, typename F>
void with_backward(const RowPlan& p, F f) {
  auto is = [&](auto l, auto v) {
    if constexpr (decltype(l)::value < 1024 || decltype(v)::value * VEC <= 8) {
      if (p.L == decltype(l)::value && p.NV == decltype(v)::value) f(l, v);
    }
  };
  is(RL_I(64), RL_I(1)); is(RL_I(64), RL_I(2)); is(RL_I(256), RL_I(1)); is(RL_I(256), RL_I(2)); is(RL_I(256), RL_I(4)); is(RL_I(1024), RL_I(2));
  is(RL_I(1024), RL_I(4)); is(RL_I(256), RL_I(0));
}
#undef RL_I
// Workgroups of the backward pass, each with a share of the sums: three a CU.  4001 x 1024 with a norm behind the block and a gate takes 18 us; 25 with 256
// of them, 22 with 1024, whose shares take longer to add.
const int kShares = 768;
int shares_of(int rows, const RowPlan& p) {
  const int group = p.L == 64 ? 4 : 1, n = (rows - 1) / group + 1;
  return std::min(n, p.L == 1024 ? 256 : kShares);
}

template <typename S, typename T, int VEC>
int forward(const ForwardCall<S, T>& f, hipStream_t s) {
  with_forward(forward_plan(f.n.width, VEC), [&](auto l, auto v) {
    constexpr int L = decltype(l)::value, NV = decltype(v)::value, G = L == 64 ? 4 : 1, THREADS = L > 256 ? L : 256;
    constexpr int64_t most = most_workgroups(THREADS) * G;      // rows of one launch
    for (int64_t first = 0; first < f.n.rows; first += most) {
      ForwardCall<S, T> part = f;
      part.n.rows = (int)std::min<int64_t>(most, f.n.rows - first);
      part.h += first * f.n.h, part.y += first * f.n.y, part.out += first * f.n.width, part.stats += first;
      if (f.a) part.a += first * f.n.width;
      if (f.gate) part.gate += first * f.n.gate;
      residual_norm_forward_kernel<S, T, VEC, L, NV><<<(part.n.rows - 1) / G + 1, THREADS, 0, s>>>(part);
    }
  });
  return launched();
}
template <typename S, typename T, int VEC>
int backward(const BackwardCall<S, T>& f, const Results<T>& results, hipStream_t s) {
  const RowPlan p = backward_plan(f.n.width, VEC);
  const int shares = shares_of(f.n.rows, p);
  const bool plain = !f.post_weight && !f.gate && !f.biased;
  with_backward<VEC>(p, [&](auto l, auto v) {
    constexpr int L = decltype(l)::value, NV = decltype(v)::value;
    if (plain) residual_norm_backward_kernel<S, T, VEC, L, NV, true><<<shares, L > 256 ? L : 256, 0, s>>>(f);
    else residual_norm_backward_kernel<S, T, VEC, L, NV, false><<<shares, L > 256 ? L : 256, 0, s>>>(f);
  });
  bool any = false;
  for (T* to : results.to) any |= to != nullptr;
  if (any) reduce_kernel<T><<<dim3((f.n.width + 31) / 32, SUMS), 1024, 0, s>>>(f.part, shares, f.n.width, results);
  return launched();
}

const int64_t kMostWidth = 1 << 24;
const char* argument(int32_t rows, int32_t width, int32_t stream_dtype, int32_t dtype) {
  if ((dtype != RL_DTYPE_F32 && dtype != RL_DTYPE_BF16) || (stream_dtype != dtype && stream_dtype != RL_DTYPE_F32))
    return "dtype is RL_DTYPE_F32 or RL_DTYPE_BF16, the stream's type that or float32";
  if (rows < 0 || width < 1 || width > kMostWidth || rows > (1 << 24)) return "rows or width out of range";
  return nullptr;
}
// Strides in multiples of 16 bytes, 16-byte aligned pointers: pieces of `vec` elements
bool pieces(int vec, int width, std::initializer_list<const void*> pointers, std::initializer_list<int64_t> strides) {
  bool ok = width % vec == 0;
  for (const void* p : pointers) ok = ok && aligned16(p);
  for (int64_t x : strides) ok = ok && x % vec == 0;
  return ok;
}
}  // namespace

extern "C" int rl_residual_norm_forward(const void* d_h, int64_t h_stride, const void* d_y, int64_t y_stride, int32_t rows, int32_t width,
                                        const void* d_weight, const void* d_bias, const void* d_post_weight, const void* d_post_bias, const void* d_gate,
                                        int64_t gate_row_stride, int32_t gate_columns, float residual_scale, float block_scale, float eps,
                                        int32_t centered, int32_t stream_dtype, int32_t dtype, void* d_out, void* d_a, float* d_stats, void* stream) {
  if (const char* m = argument(rows, width, stream_dtype, dtype)) return rl_fail(RL_E_ARG, m);
  if (!(eps >= 0.f)) return rl_fail(RL_E_ARG, "eps is negative or no number");
  if ((d_bias && !d_weight) || (d_post_bias && !d_post_weight)) return rl_fail(RL_E_ARG, "a bias without its weight");
  if (rows == 0) return RL_OK;
  if (!d_h || !d_y || !d_out || !d_stats || (d_weight && !d_a)) return rl_fail(RL_E_ARG, "null pointer");
  if ((uintptr_t)d_stats & 15) return rl_fail(RL_E_ARG, "stats not aligned to 16 bytes");
  const Shape n{rows, width, h_stride, y_stride, gate_row_stride, 0, 0, gate_columns != 0, centered != 0, residual_scale, block_scale, eps};
  const auto ok = [&](int vec) {
    return pieces(vec, width, {d_h, d_y, d_weight, d_bias, d_post_weight, d_post_bias, d_gate, d_out, d_a}, {h_stride, y_stride, gate_columns ? gate_row_stride : 0});
  };
  hipStream_t s = (hipStream_t)stream;
  auto go = [&](auto stream_type, auto type, auto vec) {
    using S = decltype(stream_type);
    using T = decltype(type);
    const ForwardCall<S, T> f{n, (const S*)d_h, (const T*)d_y, (const T*)d_weight, (const T*)d_bias, (const T*)d_post_weight, (const T*)d_post_bias,
                              (const T*)d_gate, (S*)d_out, d_weight ? (T*)d_a : nullptr, (float4*)d_stats};
    return ok(decltype(vec)::value) ? forward<S, T, decltype(vec)::value>(f, s) : forward<S, T, 1>(f, s);
  };
  if (dtype == RL_DTYPE_F32) return go(float(), float(), std::integral_constant<int, 4>());
  if (stream_dtype == RL_DTYPE_F32) return go(float(), bf16_t(), std::integral_constant<int, 8>());
  return go(bf16_t(), bf16_t(), std::integral_constant<int, 8>());
}

extern "C" int64_t rl_residual_norm_workspace(int32_t rows, int32_t width) {
  if (rows < 0 || rows > (1 << 24) || width < 1 || width > kMostWidth) return 0;
  return (int64_t)std::min(rows, kShares) * width * SUMS * (int64_t)sizeof(float);      // as many shares as any plan makes
}

extern "C" int rl_residual_norm_backward(const void* d_dout, int64_t dout_stride, const void* d_da, int64_t da_stride, const void* d_out,
                                         int64_t out_stride, const void* d_y, int64_t y_stride, const float* d_stats, int32_t rows, int32_t width,
                                         const void* d_weight, const void* d_post_weight, const void* d_post_bias, const void* d_gate,
                                         int64_t gate_row_stride, int32_t gate_columns, float residual_scale, float block_scale, int32_t centered,
                                         int32_t stream_dtype, int32_t dtype, void* d_dh, void* d_dy, void* d_dweight, void* d_dbias,
                                         void* d_dpost_weight, void* d_dpost_bias, void* d_dgate, int32_t gate_rows, void* d_workspace,
                                         int64_t workspace_bytes, void* stream) {
  if (const char* m = argument(rows, width, stream_dtype, dtype)) return rl_fail(RL_E_ARG, m);
  hipStream_t s = (hipStream_t)stream;
  if (rows == 0) {      // sums of nothing; a gate of no rows or elements has none
    auto none = [&](auto type) {
      using T = decltype(type);
      const Results<T> results{{(T*)d_dweight, (T*)d_dbias, (T*)d_dpost_weight, (T*)d_dpost_bias, gate_rows ? nullptr : (T*)d_dgate}};
      reduce_kernel<T><<<dim3((width + 31) / 32, SUMS), 1024, 0, s>>>(nullptr, 0, width, results);
      return launched();
    };
    return dtype == RL_DTYPE_F32 ? none(float()) : none(bf16_t());
  }
  if ((d_da && !d_weight) || (d_da && !d_dweight) || (d_dbias && !d_da) || (d_post_bias && !d_post_weight) || (d_post_weight && !d_dpost_weight) ||
      (d_dpost_bias && !d_post_weight) || (d_dgate && !d_gate) || (!gate_rows && d_gate && !gate_columns))
    return rl_fail(RL_E_ARG, "null pointer, or a result without what it is the gradient of");
  if (!d_y || !d_stats || !d_dh || !d_dy || (d_da && !d_out) || (!d_dout && !d_da)) return rl_fail(RL_E_ARG, "null pointer");
  if ((uintptr_t)d_stats & 15) return rl_fail(RL_E_ARG, "stats not aligned to 16 bytes");
  const int64_t bytes = rl_residual_norm_workspace(rows, width);
  if (workspace_bytes < bytes || !d_workspace) return rl_fail(RL_E_ARG, "workspace smaller than rl_residual_norm_workspace says");
  if ((uintptr_t)d_workspace & 15) return rl_fail(RL_E_ARG, "workspace not aligned to 16 bytes");
  const Shape n{rows, width, out_stride, y_stride, gate_row_stride, dout_stride, da_stride, gate_columns != 0, centered != 0, residual_scale, block_scale, 0.f};
  const bool sums = d_gate && d_dgate && !gate_rows;      // a gate a column: summed over rows
  const auto ok = [&](int vec) {
    return pieces(vec, width, {d_dout, d_da, d_out, d_y, d_weight, d_post_weight, d_post_bias, d_gate, d_dh, d_dy, d_dgate},
                  {d_dout ? dout_stride : 0, d_da ? da_stride : 0, out_stride, y_stride, gate_columns ? gate_row_stride : 0});
  };
  auto go = [&](auto stream_type, auto type, auto vec) {
    using S = decltype(stream_type);
    using T = decltype(type);
    const BackwardCall<S, T> f{n, (const S*)d_dout, (const S*)d_out, (const T*)d_da, (const T*)d_y, (const T*)d_weight, (const T*)d_post_weight,
                               (const T*)d_post_bias, (const T*)d_gate, (const float4*)d_stats, (S*)d_dh, (T*)d_dy, sums ? nullptr : (T*)d_dgate, sums,
                               d_dbias != nullptr, d_dpost_bias != nullptr, (float*)d_workspace};
    const Results<T> results{{d_da ? (T*)d_dweight : nullptr, (T*)d_dbias, d_post_weight ? (T*)d_dpost_weight : nullptr, (T*)d_dpost_bias,
                              sums ? (T*)d_dgate : nullptr}};
    return ok(decltype(vec)::value) ? backward<S, T, decltype(vec)::value>(f, results, s) : backward<S, T, 1>(f, results, s);
  };
  if (dtype == RL_DTYPE_F32) return go(float(), float(), std::integral_constant<int, 4>());
  if (stream_dtype == RL_DTYPE_F32) return go(float(), bf16_t(), std::integral_constant<int, 8>());
  return go(bf16_t(), bf16_t(), std::integral_constant<int, 8>());
}
