// Attention over packed sequences, forward and backward: entry points, and the kernels for every type and layout.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "packed_attention.h"

namespace {

// =============================================================================================
// z = scale q.k over the keys that a query sees, lse = log sum e^z, o = sum e^(z - lse) v.  Backward, with p = e^(z - lse) formed
// again: dv = p^T do, delta = rowsum(do o), dz = p (do v^T - delta), dq = scale dz k, dk = scale dz^T q.
// These kernels take both types, any head size up to 128 and any strides.  They compute in 32 bits throughout, products on
// 16x16x4 matrix instructions: lane l holds row (column) l % 16 at k = l / 16 of an operand, the result has column l % 16 and rows
// 4 (l / 16) + r.  A wave has 16 rows of its side and walks over the other side, 32 rows at a time, in LDS.  SPLIT = 1: the four waves have
// different rows and share what is in LDS; SPLIT = 4: they have the same 16 rows, each takes every fourth 32 of the other side, and
// their sums are joined at the end.  The first reads a quarter of the bytes, the second has four times the workgroups and a quarter
// of the steps: it is taken where the first would not fill the chip (4 sequences of 96 rows, 4 heads over 2, forward and backward: 56 us against 41).  Bound by the
// fp32 matrix rate (8 sequences of 1024, 8 heads of 128, causal: 1.54 ms), the small ones by one tile's chain of loads and products.
// A query head reads KV head h / (nq / nkv); the gradient of a KV head is added up over its query heads in the workgroup that owns
// its rows, in a fixed order.
// =============================================================================================
constexpr int BN = 32;      // rows of the other side that a wave takes at a time
constexpr int PAD = 12;      // of a row in LDS: 16 rows at one column, 4 k apart, lie in 64 different banks
typedef float f32;

__device__ __forceinline__ f32x4 mfma4(f32 a, f32 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// rows [r0, r0 + n) of a tensor into LDS, rows from `len` on and columns from d on as zeros; vec: four elements at a time
template <typename T, int D, int S>
__device__ __forceinline__ void stage(const T* base, int64_t stride, int r0, int n, int len, int d, bool vec, f32 (*to)[S]) {
  if (vec) {
#pragma unroll 4
    for (int i = threadIdx.x; i < n * (D / 4); i += 256) {
      const int r = i / (D / 4), c = i % (D / 4) * 4;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r0 + r < len && c < d) ld4(base + (int64_t)(r0 + r) * stride + c, v.x, v.y, v.z, v.w);
      *(float4*)&to[r][c] = v;
    }
  } else {
    for (int i = threadIdx.x; i < n * D; i += 256) {
      const int r = i / D, c = i - r * D;
      to[r][c] = r0 + r < len && c < d ? ldf(base + (int64_t)(r0 + r) * stride + c) : 0.f;
    }
  }
}
// row operand of 16 rows x D in registers: lane's row (clamped into [0, len)), element 4 s + lane / 16
template <typename T, int D>
__device__ __forceinline__ void operand(const T* base, int64_t stride, int row, int len, int d, int lane, f32 (&a)[D / 4]) {
#pragma unroll
  for (int s = 0; s < D / 4; s++) {
    const int c = 4 * s + (lane >> 4);
    a[s] = row < len && c < d ? ldf(base + (int64_t)row * stride + c) : 0.f;
  }
}

// The waves' shares of a sum [16 rows][D], in the layout of a result, added up in their order; f(row, column, sum) for every element.
template <int D, typename F>
__device__ __forceinline__ void join_waves(const f32x4 (&acc)[D / 16], f32* lds, F f) {
  constexpr int S = D + 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < D / 16; j++)
#pragma unroll
    for (int r = 0; r < 4; r++) lds[(wave * 16 + 4 * (lane >> 4) + r) * S + 16 * j + (lane & 15)] = acc[j][r];
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * D; i += 256) {
    const int row = i / D, c = i - row * D;
    f(row, c, (lds[row * S + c] + lds[(16 + row) * S + c]) + (lds[(32 + row) * S + c] + lds[(48 + row) * S + c]));
  }
}

template <typename T, int D, int SPLIT>
__global__ __launch_bounds__(256) void attention_rows_forward(PackedShape p, int vec, const T* __restrict__ q, const T* __restrict__ k,
                                                              const T* __restrict__ v, T* __restrict__ o, float* __restrict__ lse) {
  constexpr int BM = 64 / SPLIT, BT = BN * SPLIT;
  extern __shared__ f32 dynamic[];
  f32(*ks)[D + PAD] = (f32(*)[D + PAD])dynamic;
  f32(*vs)[D + PAD] = (f32(*)[D + PAD])(dynamic + BT * (D + PAD));
  f32(*ps)[16][BN + 4] = (f32(*)[16][BN + 4])(dynamic + BT * 2 * (D + PAD));
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = blockIdx.y, l16 = lane & 15, l4 = lane >> 4;
  const int mine = SPLIT == 1 ? wave * 16 : 0, part = SPLIT == 1 ? 0 : wave * BN;      // wave's rows, and its share of what is in LDS
  const OutsideRows outside(p.cu_q, p.n_seq, p.total_q);
  const PackedTile t = packed_tile(p.cu_q, p.n_seq, p.total_q, BM, blockIdx.x);
  outside.clear<T>(p.nq * p.d, o, nullptr, lse, p.nq);
  if (t.row0 >= t.len) return;
  const int k0 = packed_bound(p.cu_k, t.seq, p.total_k), lk = max(packed_bound(p.cu_k, t.seq + 1, p.total_k) - k0, 0);
  const int hk = h / (p.nq / p.nkv), shift = lk - t.len;
  const T* kb = k + (int64_t)k0 * p.kt + (int64_t)hk * p.kh;
  const T* vb = v + (int64_t)k0 * p.vt + (int64_t)hk * p.vh;
  f32 a[D / 4], m[4], sum[4];
  operand<T, D>(q + (int64_t)t.first * p.qt + (int64_t)h * p.qh, p.qt, t.row0 + mine + l16, t.len, p.d, lane, a);
  f32x4 acc[D / 16];
#pragma unroll
  for (int j = 0; j < D / 16; j++) acc[j] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int r = 0; r < 4; r++) m[r] = -INFINITY, sum[r] = 0.f;
  const int last = p.causal ? min(lk, max(t.row0 + BM + shift, 0)) : lk;
  for (int j0 = 0; j0 < last; j0 += BT) {
    __syncthreads();
    stage<T, D>(kb, p.kt, j0, BT, lk, p.d, vec, ks);
    stage<T, D>(vb, p.vt, j0, BT, lk, p.d, vec, vs);
    __syncthreads();
    f32x4 z[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int s = 0; s < D / 4; s++)
#pragma unroll
      for (int b = 0; b < 2; b++) z[b] = mfma4(a[s], ks[part + b * 16 + l16][4 * s + l4], z[b]);
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const int i = t.row0 + mine + 4 * l4 + r;
      const int end = p.causal ? min(lk, i + shift + 1) : lk;      // keys [0, end) are seen
      f32 top = m[r];
#pragma unroll
      for (int b = 0; b < 2; b++) {
        z[b][r] = j0 + part + b * 16 + l16 < end ? z[b][r] * p.scale : -INFINITY;
        top = fmaxf(top, z[b][r]);
      }
#pragma unroll
      for (int x = 8; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
      const f32 ref = top == -INFINITY ? 0.f : top, old = expf(m[r] - ref);      // nothing seen so far: e^-inf = 0, not NaN
      m[r] = top;
      f32 s = 0.f;
#pragma unroll
      for (int b = 0; b < 2; b++) {
        const f32 e = expf(z[b][r] - ref);
        ps[wave][4 * l4 + r][b * 16 + l16] = e;
        s += e;
      }
      sum[r] = sum[r] * old + s;
#pragma unroll
      for (int j = 0; j < D / 16; j++) acc[j][r] *= old;
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < BN / 4; s++)
#pragma unroll
      for (int j = 0; j < D / 16; j++) acc[j] = mfma4(ps[wave][l16][4 * s + l4], vs[part + 4 * s + l4][16 * j + l16], acc[j]);
  }
  __shared__ f32 tops[4][16], sums[4][16];
#pragma unroll
  for (int r = 0; r < 4; r++) {
    f32 s = sum[r];
#pragma unroll
    for (int x = 8; x > 0; x >>= 1) s += __shfl_xor(s, x, 64);
    sum[r] = s;
    if (SPLIT > 1 && l16 == 0) tops[wave][4 * l4 + r] = m[r], sums[wave][4 * l4 + r] = s;
  }
  if constexpr (SPLIT > 1) {      // one reference for the four shares
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const int row = 4 * l4 + r;
      f32 top = tops[0][row], s = 0.f;
#pragma unroll
      for (int w = 1; w < 4; w++) top = fmaxf(top, tops[w][row]);
      const f32 ref = top == -INFINITY ? 0.f : top, old = expf(m[r] - ref);
#pragma unroll
      for (int w = 0; w < 4; w++) s += sums[w][row] * expf(tops[w][row] - ref);
#pragma unroll
      for (int j = 0; j < D / 16; j++) acc[j][r] *= old;
      m[r] = top, sum[r] = s;
    }
  }
  f32 inv[4];
#pragma unroll
  for (int r = 0; r < 4; r++) {
    const int i = t.row0 + mine + 4 * l4 + r;
    inv[r] = sum[r] > 0.f ? 1.f / sum[r] : sum[r] == 0.f ? 0.f : sum[r];      // no key: zeros; no number stays so
    if (i < t.len && l16 == 0 && (SPLIT == 1 || wave == 0)) lse[(size_t)h * p.total_q + t.first + i] = m[r] + logf(sum[r]);
#pragma unroll
    for (int j = 0; j < D / 16; j++) acc[j][r] *= inv[r];
  }
  T* out = o + (int64_t)(t.first + t.row0) * p.ot + (int64_t)h * p.oh;
  if constexpr (SPLIT > 1) {
    join_waves<D>(acc, dynamic, [&](int row, int c, f32 x) {
      if (t.row0 + row < t.len && c < p.d) st1(out + row * p.ot + c, x);
    });
  } else {
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const int row = mine + 4 * l4 + r;
      if (t.row0 + row >= t.len) continue;
#pragma unroll
      for (int j = 0; j < D / 16; j++)
        if (16 * j + l16 < p.d) st1(out + row * p.ot + 16 * j + l16, acc[j][r]);
    }
  }
}

// dq of 64 / SPLIT query rows, and delta, which the other kernel reads
template <typename T, int D, int SPLIT>
__global__ __launch_bounds__(256) void attention_rows_dq(PackedShape p, int vec, const T* __restrict__ dout, const T* __restrict__ q,
                                                         const T* __restrict__ k, const T* __restrict__ v, const T* __restrict__ o,
                                                         const float* __restrict__ lse, T* __restrict__ dq, float* __restrict__ delta) {
  constexpr int BM = 64 / SPLIT, BT = BN * SPLIT;
  extern __shared__ f32 dynamic[];
  f32(*ks)[D + PAD] = (f32(*)[D + PAD])dynamic;
  f32(*vs)[D + PAD] = (f32(*)[D + PAD])(dynamic + BT * (D + PAD));
  f32(*ds)[16][BN + 4] = (f32(*)[16][BN + 4])(dynamic + BT * 2 * (D + PAD));
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = blockIdx.y, l16 = lane & 15, l4 = lane >> 4;
  const int own = SPLIT == 1 ? wave * 16 : 0, part = SPLIT == 1 ? 0 : wave * BN;
  const OutsideRows outside(p.cu_q, p.n_seq, p.total_q);
  const PackedTile t = packed_tile(p.cu_q, p.n_seq, p.total_q, BM, blockIdx.x);
  outside.clear<T>(p.nq * p.d, dq, nullptr, nullptr, 0);
  if (t.row0 >= t.len) return;
  const int k0 = packed_bound(p.cu_k, t.seq, p.total_k), lk = max(packed_bound(p.cu_k, t.seq + 1, p.total_k) - k0, 0);
  const int hk = h / (p.nq / p.nkv), shift = lk - t.len;
  const T* kb = k + (int64_t)k0 * p.kt + (int64_t)hk * p.kh;
  const T* vb = v + (int64_t)k0 * p.vt + (int64_t)hk * p.vh;
  const int mine = t.row0 + own + l16;
  const int64_t ds_ = (int64_t)p.nq * p.d;      // token stride of dO and dq
  f32 a[D / 4], g[D / 4], dl = 0.f;
  operand<T, D>(q + (int64_t)t.first * p.qt + (int64_t)h * p.qh, p.qt, mine, t.len, p.d, lane, a);
  operand<T, D>(dout + (int64_t)t.first * ds_ + (int64_t)h * p.d, ds_, mine, t.len, p.d, lane, g);
  {
    f32 y[D / 4];
    operand<T, D>(o + (int64_t)t.first * p.ot + (int64_t)h * p.oh, p.ot, mine, t.len, p.d, lane, y);
#pragma unroll
    for (int s = 0; s < D / 4; s++) dl += g[s] * y[s];
    dl += __shfl_xor(dl, 16, 64);
    dl += __shfl_xor(dl, 32, 64);
    if (lane < 16 && mine < t.len && (SPLIT == 1 || wave == 0)) delta[(size_t)h * p.total_q + t.first + mine] = dl;
  }
  f32 l[4], dr[4];
#pragma unroll
  for (int r = 0; r < 4; r++) {
    const int i = t.row0 + own + 4 * l4 + r;
    l[r] = i < t.len ? lse[(size_t)h * p.total_q + t.first + i] : 0.f;
    dr[r] = __shfl(dl, 4 * l4 + r, 64);
  }
  f32x4 acc[D / 16];
#pragma unroll
  for (int j = 0; j < D / 16; j++) acc[j] = {0.f, 0.f, 0.f, 0.f};
  const int last = p.causal ? min(lk, max(t.row0 + BM + shift, 0)) : lk;
  for (int j0 = 0; j0 < last; j0 += BT) {
    __syncthreads();
    stage<T, D>(kb, p.kt, j0, BT, lk, p.d, vec, ks);
    stage<T, D>(vb, p.vt, j0, BT, lk, p.d, vec, vs);
    __syncthreads();
    f32x4 z[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}}, dp[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int s = 0; s < D / 4; s++)
#pragma unroll
      for (int b = 0; b < 2; b++) {
        z[b] = mfma4(a[s], ks[part + b * 16 + l16][4 * s + l4], z[b]);
        dp[b] = mfma4(g[s], vs[part + b * 16 + l16][4 * s + l4], dp[b]);
      }
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const int i = t.row0 + own + 4 * l4 + r, end = p.causal ? min(lk, i + shift + 1) : lk;
#pragma unroll
      for (int b = 0; b < 2; b++)
        ds[wave][4 * l4 + r][b * 16 + l16] = j0 + part + b * 16 + l16 < end ? expf(z[b][r] * p.scale - l[r]) * (dp[b][r] - dr[r]) * p.scale : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < BN / 4; s++)
#pragma unroll
      for (int j = 0; j < D / 16; j++) acc[j] = mfma4(ds[wave][l16][4 * s + l4], ks[part + 4 * s + l4][16 * j + l16], acc[j]);
  }
  T* out = dq + (int64_t)(t.first + t.row0) * ds_ + (int64_t)h * p.d;
  if constexpr (SPLIT > 1) {
    join_waves<D>(acc, dynamic, [&](int row, int c, f32 x) {
      if (t.row0 + row < t.len && c < p.d) st1(out + row * ds_ + c, x);
    });
  } else {
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const int row = own + 4 * l4 + r;
      if (t.row0 + row >= t.len) continue;
#pragma unroll
      for (int j = 0; j < D / 16; j++)
        if (16 * j + l16 < p.d) st1(out + row * ds_ + 16 * j + l16, acc[j][r]);
    }
  }
}

// dk and dv of 64 / SPLIT key rows of one KV head, over its query heads and the query tiles that see them
template <typename T, int D, int SPLIT>
__global__ __launch_bounds__(256) void attention_rows_dkv(PackedShape p, int vec, const T* __restrict__ dout, const T* __restrict__ q,
                                                          const T* __restrict__ k, const T* __restrict__ v, const float* __restrict__ lse,
                                                          const float* __restrict__ delta, T* __restrict__ dk, T* __restrict__ dv, KeyParts parts) {
  constexpr int BM = 64 / SPLIT, BT = BN * SPLIT;
  extern __shared__ f32 dynamic[];
  f32(*qs)[D + PAD] = (f32(*)[D + PAD])dynamic;
  f32(*gs)[D + PAD] = (f32(*)[D + PAD])(dynamic + BT * (D + PAD));
  f32(*pt)[16][BN + 4] = (f32(*)[16][BN + 4])(dynamic + 2 * BT * (D + PAD));
  f32(*dt)[16][BN + 4] = pt + 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hk = blockIdx.y, l16 = lane & 15, l4 = lane >> 4;
  const int own = SPLIT == 1 ? wave * 16 : 0, part = SPLIT == 1 ? 0 : wave * BN;
  const OutsideRows outside(p.cu_k, p.n_seq, p.total_k);
  const PackedTile t = packed_tile(p.cu_k, p.n_seq, p.total_k, BM, blockIdx.x);
  outside.clear<T>(p.nkv * p.d, dk, dv, nullptr, 0);
  if (t.row0 >= t.len) return;
  const int q0 = packed_bound(p.cu_q, t.seq, p.total_q), lq = max(packed_bound(p.cu_q, t.seq + 1, p.total_q) - q0, 0);
  const int group = p.nq / p.nkv, shift = t.len - lq, mine = t.row0 + own + l16;
  const int64_t ds_ = (int64_t)p.nq * p.d, dks = (int64_t)p.nkv * p.d;
  f32 a[D / 4], b[D / 4];
  operand<T, D>(k + (int64_t)t.first * p.kt + (int64_t)hk * p.kh, p.kt, mine, t.len, p.d, lane, a);
  operand<T, D>(v + (int64_t)t.first * p.vt + (int64_t)hk * p.vh, p.vt, mine, t.len, p.d, lane, b);
  f32x4 ak[D / 16], av[D / 16];
#pragma unroll
  for (int j = 0; j < D / 16; j++) ak[j] = av[j] = {0.f, 0.f, 0.f, 0.f};
  const int first = p.causal ? max(t.row0 - shift, 0) / BN * BN : 0;
  const int per_head = max((lq - first + BT - 1) / BT, 0);
  for (int pair = blockIdx.z; pair < per_head * group; pair += parts.n) {      // (query head, query tile)
    const int h = hk * group + pair / per_head, i0 = first + pair % per_head * BT;
    const T* qb = q + (int64_t)q0 * p.qt + (int64_t)h * p.qh;
    const T* gb = dout + (int64_t)q0 * ds_ + (int64_t)h * p.d;
    __syncthreads();
    stage<T, D>(qb, p.qt, i0, BT, lq, p.d, vec, qs);
    stage<T, D>(gb, ds_, i0, BT, lq, p.d, vec, gs);
    __syncthreads();
    f32x4 z[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}}, dp[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int s = 0; s < D / 4; s++)
#pragma unroll
      for (int c = 0; c < 2; c++) {
        z[c] = mfma4(a[s], qs[part + c * 16 + l16][4 * s + l4], z[c]);
        dp[c] = mfma4(b[s], gs[part + c * 16 + l16][4 * s + l4], dp[c]);
      }
#pragma unroll
    for (int c = 0; c < 2; c++) {
      const int i = i0 + part + c * 16 + l16;
      const bool in = i < lq;
      const f32 l = in ? lse[(size_t)h * p.total_q + q0 + i] : 0.f, dl = in ? delta[(size_t)h * p.total_q + q0 + i] : 0.f;
      const int end = !in ? 0 : p.causal ? min(t.len, i + shift + 1) : t.len;      // this query sees the keys [0, end)
#pragma unroll
      for (int r = 0; r < 4; r++) {
        const f32 e = t.row0 + own + 4 * l4 + r < end ? expf(z[c][r] * p.scale - l) : 0.f;
        pt[wave][4 * l4 + r][c * 16 + l16] = e;
        dt[wave][4 * l4 + r][c * 16 + l16] = e != 0.f ? e * (dp[c][r] - dl) * p.scale : 0.f;
      }
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < BN / 4; s++) {
      const f32 x = pt[wave][l16][4 * s + l4], y = dt[wave][l16][4 * s + l4];
#pragma unroll
      for (int j = 0; j < D / 16; j++) {
        av[j] = mfma4(x, gs[part + 4 * s + l4][16 * j + l16], av[j]);
        ak[j] = mfma4(y, qs[part + 4 * s + l4][16 * j + l16], ak[j]);
      }
    }
  }
  const int64_t at = (int64_t)(t.first + t.row0) * dks + (int64_t)hk * p.d;
  if constexpr (SPLIT > 1) {
    auto to = [&](T* out) {
      return [&, out](int row, int c, f32 x) {
        if (t.row0 + row < t.len && c < p.d) st1(out + at + row * dks + c, x);
      };
    };
    join_waves<D>(ak, dynamic, to(dk));
    join_waves<D>(av, dynamic, to(dv));
  } else {
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const int row = own + 4 * l4 + r;
      if (t.row0 + row >= t.len) continue;
#pragma unroll
      for (int j = 0; j < D / 16; j++)
        if (16 * j + l16 < p.d) {
          const int64_t i = at + row * dks + 16 * j + l16;
          if (parts.n > 1) {
            parts.of(p, blockIdx.z, 0)[i] = ak[j][r];
            parts.of(p, blockIdx.z, 1)[i] = av[j][r];
          } else {
            st1(dk + i, ak[j][r]);
            st1(dv + i, av[j][r]);
          }
        }
    }
  }
}

// Four elements at a time: aligned rows of whole fours.
template <typename T>
bool fours(const void* x, int64_t ts, int64_t hs, int d) {
  return ((uintptr_t)x & (4 * sizeof(T) - 1)) == 0 && ts % 4 == 0 && hs % 4 == 0 && d % 4 == 0;
}
// dk and dv of 8 keys of one KV head from the sums of their parts, in their order
template <typename T>
__global__ __launch_bounds__(256) void attention_join_parts(PackedShape p, KeyParts parts, T* __restrict__ dk, T* __restrict__ dv) {
  const PackedTile t = packed_tile(p.cu_k, p.n_seq, p.total_k, 64, blockIdx.x);
  const int row0 = t.row0 + blockIdx.z * 8, rows = min(t.len - row0, 8);
  const int64_t step = (int64_t)p.total_k * p.nkv * p.d;
  for (int i = threadIdx.x; i < rows * p.d; i += 256) {
    const int64_t at = ((int64_t)(t.first + row0 + i / p.d) * p.nkv + blockIdx.y) * p.d + i % p.d;
    const float* x = parts.sums + at;
    f32 a = 0.f, b = 0.f;
#pragma unroll 4
    for (int n = 0; n < parts.n; n++) a += x[2 * n * step], b += x[(2 * n + 1) * step];
    st1(dk + at, a);
    st1(dv + at, b);
  }
}

template <auto kernel, typename... A>
void launch_rows(int tiles, int heads, int depth, int lds, hipStream_t s, A... args) {
  static std::atomic<uint64_t> done;      // more than 64 KB of LDS need an opt-in, once per kernel and device
  int dev = 0;
  (void)hipGetDevice(&dev);
  const uint64_t bit = 1ull << (dev & 63);
  if (lds > 65536 && !(done.load(std::memory_order_acquire) & bit)) {
    (void)hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    done.fetch_or(bit, std::memory_order_release);
  }
  kernel<<<dim3(tiles, heads, depth), 256, lds, s>>>(args...);
}
// 16 rows split over four waves in place of 64 rows, 16 a wave, where tiles of 64 would leave half the CUs idle.  Measured, forward and
// backward of one sequence in 64 and 128 dimensions: 1024 tokens, 4 heads (68 tiles) 148 and 347 us, unsplit 324 and 629; 8 heads (136) 373
// and 668, unsplit 370 and 678; 16 heads (272) 617 and 1049, unsplit 497 and 858.
bool split_rows(int total, int n_seq, int heads) { return (int64_t)packed_tiles(total, n_seq, 64) * heads < 128; }
template <int D>
constexpr int rows_lds(int split) {      // what the largest of the kernels needs: two tiles, two sets of scores
  return (BN * split * 2 * (D + PAD) + 2 * 4 * 16 * (BN + 4)) * 4;
}

template <typename T, int D>
void forward(hipStream_t s, const PackedShape& p, const void* q, const void* k, const void* v, void* o, float* lse) {
  const int vec = fours<T>(k, p.kt, p.kh, p.d) && fours<T>(v, p.vt, p.vh, p.d);
  if (split_rows(p.total_q, p.n_seq, p.nq))
    launch_rows<attention_rows_forward<T, D, 4>>(packed_tiles(p.total_q, p.n_seq, 16), p.nq, 1, rows_lds<D>(4), s, p, vec, (const T*)q, (const T*)k,
                (const T*)v, (T*)o, lse);
  else
    launch_rows<attention_rows_forward<T, D, 1>>(packed_tiles(p.total_q, p.n_seq, 64), p.nq, 1, rows_lds<D>(1), s, p, vec, (const T*)q, (const T*)k,
                (const T*)v, (T*)o, lse);
}
template <typename T, int D>
void backward(hipStream_t s, const PackedShape& p, const void* dout, const void* q, const void* k, const void* v, const void* o,
              const float* lse, void* dq, void* dk, void* dv, float* delta, const KeyParts& parts) {
  const int by_key = fours<T>(k, p.kt, p.kh, p.d) && fours<T>(v, p.vt, p.vh, p.d);
  const int by_query = fours<T>(q, p.qt, p.qh, p.d) && fours<T>(dout, p.ot, p.oh, p.d);
  if (p.total_q > 0) {
    auto go = [&](auto split) {
      constexpr int S = decltype(split)::value;
      launch_rows<attention_rows_dq<T, D, S>>(packed_tiles(p.total_q, p.n_seq, 64 / S), p.nq, 1, rows_lds<D>(S), s, p, by_key, (const T*)dout,
                  (const T*)q, (const T*)k, (const T*)v, (const T*)o, lse, (T*)dq, delta);
    };
    if (split_rows(p.total_q, p.n_seq, p.nq)) go(std::integral_constant<int, 4>());
    else go(std::integral_constant<int, 1>());
  }
  if (p.total_k > 0) {
    auto go = [&](auto split) {
      constexpr int S = decltype(split)::value;
      launch_rows<attention_rows_dkv<T, D, S>>(packed_tiles(p.total_k, p.n_seq, 64 / S), p.nkv, parts.n, rows_lds<D>(S), s, p, by_query, (const T*)dout,
                  (const T*)q, (const T*)k, (const T*)v, lse, delta, (T*)dk, (T*)dv, parts);
    };
    if (parts.n == 1 && split_rows(p.total_k, p.n_seq, p.nkv)) go(std::integral_constant<int, 4>());
    else go(std::integral_constant<int, 1>());
  }
}

int64_t parts_bytes(const PackedShape& p) { return (int64_t)p.total_k * p.nkv * p.d * 2 * (int64_t)sizeof(float); }
// bf16: a workgroup a CU, fp32: two, and where rows could be split over waves instead, four parts or none.  Measured, both directions, with
// parts and without: bf16, one sequence of 2000, 8 heads over 1 of 128, 129 and 301 us, of 6000 583 and 882, 8 sequences of 256, 8 heads
// over 1 of 64, 33 and 40; fp32, one of 2000, 1118 and 2520, of 1500, 32 over 8, 2047 and 2521; 4 heads of 64, 1024 tokens, two parts 179, split 152.
int parts_of(const PackedShape& p, int32_t dtype) {
  if (dtype == RL_DTYPE_BF16) return key_parts(p, 256);
  const int n = key_parts(p, 512);
  return n < 4 && split_rows(p.total_k, p.n_seq, p.nkv) ? 1 : n;
}

const char* attention_argument(const PackedShape& p, int32_t dtype) {
  if (dtype != RL_DTYPE_F32 && dtype != RL_DTYPE_BF16) return "dtype is RL_DTYPE_F32 or RL_DTYPE_BF16";
  if (p.n_seq < 0 || p.n_seq > (1 << 24) || p.total_q < 0 || p.total_k < 0) return "sequences or tokens out of range";
  if (p.total_q > (1 << 30) || p.total_k > (1 << 30)) return "more than 2^30 tokens";
  if (packed_tiles(std::max(p.total_q, p.total_k), p.n_seq, 64) > most_workgroups(256)) return "more sequences and tokens than a launch takes";
  if (p.nq < 1 || p.nkv < 1 || p.nq % p.nkv || p.nq > 4096) return "n_q_heads is a multiple of n_kv_heads, at most 4096";
  if (p.d < 1 || p.d > 128) return "head_dim is 1 to 128";
  if (!(p.scale == p.scale) || p.scale - p.scale != 0.f) return "scale is no finite number";
  if (p.n_seq == 0 && (p.total_q > 0 || p.total_k > 0)) return "tokens without a sequence";
  if (p.n_seq > 0 && (!p.cu_q || !p.cu_k)) return "null pointer";
  return nullptr;
}

}  // namespace

extern "C" int rl_attention_forward(const void* d_q, int64_t q_token_stride, int64_t q_head_stride, const void* d_k, int64_t k_token_stride,
                                    int64_t k_head_stride, const void* d_v, int64_t v_token_stride, int64_t v_head_stride,
                                    const int32_t* d_cu_q, const int32_t* d_cu_k, int32_t n_seq, int32_t total_q, int32_t total_k,
                                    int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, float scale, int32_t causal, int32_t dtype,
                                    void* d_o, float* d_lse, void* stream) {
  const PackedShape p{d_cu_q, d_cu_k, n_seq, total_q, total_k, n_q_heads, n_kv_heads, head_dim, q_token_stride, q_head_stride,
                      k_token_stride, k_head_stride, v_token_stride, v_head_stride, (int64_t)n_q_heads * head_dim, head_dim, scale, causal};
  if (const char* m = attention_argument(p, dtype)) return rl_fail(RL_E_ARG, m);
  if (total_q == 0) return RL_OK;
  if (!d_q || !d_o || !d_lse || (total_k > 0 && (!d_k || !d_v))) return rl_fail(RL_E_ARG, "null pointer");
  hipStream_t s = (hipStream_t)stream;
  if (dtype == RL_DTYPE_F32) {
    if (head_dim <= 64) forward<float, 64>(s, p, d_q, d_k, d_v, d_o, d_lse);
    else forward<float, 128>(s, p, d_q, d_k, d_v, d_o, d_lse);
  } else if (attention_takes_mfma(p, d_q, d_k, d_v, d_o, nullptr)) {
    launch_attention_mfma_forward(s, p, (const bf16_t*)d_q, (const bf16_t*)d_k, (const bf16_t*)d_v, (bf16_t*)d_o, d_lse);
  } else {
    if (head_dim <= 64) forward<bf16_t, 64>(s, p, d_q, d_k, d_v, d_o, d_lse);
    else forward<bf16_t, 128>(s, p, d_q, d_k, d_v, d_o, d_lse);
  }
  return launched();
}

extern "C" int64_t rl_attention_workspace(int32_t total_q, int32_t n_q_heads) {
  return total_q < 0 || n_q_heads < 1 ? 0 : (int64_t)total_q * n_q_heads * 2 * (int64_t)sizeof(float);
}

extern "C" int64_t rl_attention_fast_workspace(int32_t n_seq, int32_t total_q, int32_t total_k, int32_t n_q_heads, int32_t n_kv_heads,
                                               int32_t head_dim, int32_t dtype) {
  const int32_t none = 0;      // offsets are not looked at
  const PackedShape p{&none, &none, n_seq, total_q, total_k, n_q_heads, n_kv_heads, head_dim, 0, 0, 0, 0, 0, 0, 0, 0, 1.f, 0};
  if (attention_argument(p, dtype)) return 0;
  const int parts = parts_of(p, dtype);
  return up(rl_attention_workspace(total_q, n_q_heads), 256) + (parts > 1 ? parts * parts_bytes(p) : 0);
}

extern "C" int rl_attention_backward(const void* d_do, const void* d_q, int64_t q_token_stride, int64_t q_head_stride, const void* d_k,
                                     int64_t k_token_stride, int64_t k_head_stride, const void* d_v, int64_t v_token_stride,
                                     int64_t v_head_stride, const void* d_o, const float* d_lse, const int32_t* d_cu_q,
                                     const int32_t* d_cu_k, int32_t n_seq, int32_t total_q, int32_t total_k, int32_t n_q_heads,
                                     int32_t n_kv_heads, int32_t head_dim, float scale, int32_t causal, int32_t dtype, void* d_dq,
                                     void* d_dk, void* d_dv, void* d_workspace, int64_t workspace_bytes, void* stream) {
  const PackedShape p{d_cu_q, d_cu_k, n_seq, total_q, total_k, n_q_heads, n_kv_heads, head_dim, q_token_stride, q_head_stride,
                      k_token_stride, k_head_stride, v_token_stride, v_head_stride, (int64_t)n_q_heads * head_dim, head_dim, scale, causal};
  if (const char* m = attention_argument(p, dtype)) return rl_fail(RL_E_ARG, m);
  if (total_q == 0 && total_k == 0) return RL_OK;
  if (total_q > 0 && (!d_do || !d_q || !d_o || !d_lse || !d_dq || !d_workspace)) return rl_fail(RL_E_ARG, "null pointer");
  if (total_k > 0 && (!d_k || !d_v || !d_dk || !d_dv)) return rl_fail(RL_E_ARG, "null pointer");
  if (workspace_bytes < rl_attention_workspace(total_q, n_q_heads))
    return rl_fail(RL_E_ARG, "workspace smaller than rl_attention_workspace says");
  if ((uintptr_t)d_workspace & 3) return rl_fail(RL_E_ARG, "workspace not aligned to 4 bytes");
  hipStream_t s = (hipStream_t)stream;
  float* delta = (float*)d_workspace;
  // parts where the workspace has room for them
  const int64_t base = up(rl_attention_workspace(total_q, n_q_heads), 256);
  const int most = parts_of(p, dtype);
  const bool room = most > 1 && aligned16(d_workspace) && workspace_bytes >= base + most * parts_bytes(p);
  const KeyParts parts{room ? most : 1, room ? (float*)((char*)d_workspace + base) : nullptr};
#define RL_GO(T, D) backward<T, D>(s, p, d_do, d_q, d_k, d_v, d_o, d_lse, d_dq, d_dk, d_dv, delta, parts)
  if (dtype == RL_DTYPE_F32) {
    if (head_dim <= 64) RL_GO(float, 64);
    else RL_GO(float, 128);
  } else if (attention_takes_mfma(p, d_q, d_k, d_v, d_o, d_do) && aligned16(d_dq) && aligned16(d_dk) && aligned16(d_dv)) {
    launch_attention_mfma_backward(s, p, (const bf16_t*)d_do, (const bf16_t*)d_q, (const bf16_t*)d_k, (const bf16_t*)d_v, (const bf16_t*)d_o,
                                   d_lse, (bf16_t*)d_dq, (bf16_t*)d_dk, (bf16_t*)d_dv, delta, parts);
  } else {
    if (head_dim <= 64) RL_GO(bf16_t, 64);
    else RL_GO(bf16_t, 128);
  }
#undef RL_GO
  if (parts.n > 1) {
    const dim3 grid(packed_tiles(total_k, n_seq, 64), n_kv_heads, 8);
    if (dtype == RL_DTYPE_F32) attention_join_parts<float><<<grid, 256, 0, s>>>(p, parts, (float*)d_dk, (float*)d_dv);
    else attention_join_parts<bf16_t><<<grid, 256, 0, s>>>(p, parts, (bf16_t*)d_dk, (bf16_t*)d_dv);
  }
  return launched();
}
