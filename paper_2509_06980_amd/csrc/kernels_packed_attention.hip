// Attention over packed sequences, forward and backward: entry points, and the kernels for every type and layout.
#include "packed_attention.h"

namespace {

// =============================================================================================
// z = scale q.k over the keys that a query sees, lse = log sum e^z, o = sum e^(z - lse) v.  Backward, with p = e^(z - lse) formed
// again: dv = p^T do, delta = rowsum(do o), dz = p (do v^T - delta), dq = scale dz k, dk = scale dz^T q.
// These kernels take both types, any head size up to 128 and any strides.  They compute in 32 bits throughout, products on
// 16x16x4 matrix instructions: lane l holds row (column) l % 16 at k = l / 16 of an operand, the result has column l % 16 and rows
// 4 (l / 16) + r.  Tiles of 64 rows, a wave 16 of them, walk over tiles of 32 rows of the other side in LDS.
// A query head reads KV head h / (nq / nkv); the gradient of a KV head is added up over its query heads in the workgroup that owns
// its rows, in a fixed order.
// =============================================================================================
constexpr int BM = 64, BN = 32;
typedef float f32;

__device__ __forceinline__ f32x4 mfma4(f32 a, f32 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

// rows [r0, r0 + n) of a tensor into LDS, rows from `len` on and columns from d on as zeros
template <typename T, int D, int S>
__device__ __forceinline__ void stage(const T* base, int64_t stride, int r0, int n, int len, int d, f32 (*to)[S]) {
  for (int i = threadIdx.x; i < n * D; i += 256) {
    const int r = i / D, c = i - r * D;
    to[r][c] = r0 + r < len && c < d ? ldf(base + (int64_t)(r0 + r) * stride + c) : 0.f;
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

template <typename T, int D>
__global__ __launch_bounds__(256) void attention_rows_forward(PackedShape p, const T* __restrict__ q, const T* __restrict__ k,
                                                              const T* __restrict__ v, T* __restrict__ o, float* __restrict__ lse) {
  __shared__ f32 ks[BN][D + 4], vs[BN][D + 16], ps[4][16][BN + 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = blockIdx.y, l16 = lane & 15, l4 = lane >> 4;
  const PackedTile t = packed_tile(p.cu_q, p.n_seq, p.total_q, BM, blockIdx.x);
  if (t.row0 >= t.len) return;
  const int k0 = packed_bound(p.cu_k, t.seq, p.total_k), lk = max(packed_bound(p.cu_k, t.seq + 1, p.total_k) - k0, 0);
  const int hk = h / (p.nq / p.nkv), shift = lk - t.len;
  const T* kb = k + (int64_t)k0 * p.kt + (int64_t)hk * p.kh;
  const T* vb = v + (int64_t)k0 * p.vt + (int64_t)hk * p.vh;
  f32 a[D / 4], m[4], sum[4];
  operand<T, D>(q + (int64_t)t.first * p.qt + (int64_t)h * p.qh, p.qt, t.row0 + wave * 16 + l16, t.len, p.d, lane, a);
  f32x4 acc[D / 16];
#pragma unroll
  for (int j = 0; j < D / 16; j++) acc[j] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int r = 0; r < 4; r++) m[r] = -INFINITY, sum[r] = 0.f;
  const int last = p.causal ? min(lk, max(t.row0 + BM + shift, 0)) : lk;
  for (int j0 = 0; j0 < last; j0 += BN) {
    __syncthreads();
    stage<T, D>(kb, p.kt, j0, BN, lk, p.d, ks);
    stage<T, D>(vb, p.vt, j0, BN, lk, p.d, vs);
    __syncthreads();
    f32x4 z[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int s = 0; s < D / 4; s++)
#pragma unroll
      for (int b = 0; b < 2; b++) z[b] = mfma4(a[s], ks[b * 16 + l16][4 * s + l4], z[b]);
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const int i = t.row0 + wave * 16 + 4 * l4 + r;
      const int end = p.causal ? min(lk, i + shift + 1) : lk;      // keys [0, end) are seen
      f32 top = m[r];
#pragma unroll
      for (int b = 0; b < 2; b++) {
        z[b][r] = j0 + b * 16 + l16 < end ? z[b][r] * p.scale : -INFINITY;
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
      for (int j = 0; j < D / 16; j++) acc[j] = mfma4(ps[wave][l16][4 * s + l4], vs[4 * s + l4][16 * j + l16], acc[j]);
  }
#pragma unroll
  for (int r = 0; r < 4; r++) {
    f32 s = sum[r];
#pragma unroll
    for (int x = 8; x > 0; x >>= 1) s += __shfl_xor(s, x, 64);
    const int i = t.row0 + wave * 16 + 4 * l4 + r;
    if (i >= t.len) continue;
    const f32 inv = s > 0.f ? 1.f / s : s == 0.f ? 0.f : s;      // no key: zeros; no number stays so
    T* out = o + (int64_t)(t.first + i) * p.ot + (int64_t)h * p.oh;
#pragma unroll
    for (int j = 0; j < D / 16; j++)
      if (16 * j + l16 < p.d) st1(out + 16 * j + l16, acc[j][r] * inv);
    if (l16 == 0) lse[(size_t)h * p.total_q + t.first + i] = m[r] + logf(s);
  }
}

// dq of 64 query rows, and delta, which the other kernel reads
template <typename T, int D>
__global__ __launch_bounds__(256) void attention_rows_dq(PackedShape p, const T* __restrict__ dout, const T* __restrict__ q,
                                                         const T* __restrict__ k, const T* __restrict__ v, const T* __restrict__ o,
                                                         const float* __restrict__ lse, T* __restrict__ dq, float* __restrict__ delta) {
  __shared__ f32 ks[BN][D + 16], vs[BN][D + 4], ds[4][16][BN + 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = blockIdx.y, l16 = lane & 15, l4 = lane >> 4;
  const PackedTile t = packed_tile(p.cu_q, p.n_seq, p.total_q, BM, blockIdx.x);
  if (t.row0 >= t.len) return;
  const int k0 = packed_bound(p.cu_k, t.seq, p.total_k), lk = max(packed_bound(p.cu_k, t.seq + 1, p.total_k) - k0, 0);
  const int hk = h / (p.nq / p.nkv), shift = lk - t.len;
  const T* kb = k + (int64_t)k0 * p.kt + (int64_t)hk * p.kh;
  const T* vb = v + (int64_t)k0 * p.vt + (int64_t)hk * p.vh;
  const int mine = t.row0 + wave * 16 + l16;
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
    if (lane < 16 && mine < t.len) delta[(size_t)h * p.total_q + t.first + mine] = dl;
  }
  f32 l[4], dr[4];
#pragma unroll
  for (int r = 0; r < 4; r++) {
    const int i = t.row0 + wave * 16 + 4 * l4 + r;
    l[r] = i < t.len ? lse[(size_t)h * p.total_q + t.first + i] : 0.f;
    dr[r] = __shfl(dl, 4 * l4 + r, 64);
  }
  f32x4 acc[D / 16];
#pragma unroll
  for (int j = 0; j < D / 16; j++) acc[j] = {0.f, 0.f, 0.f, 0.f};
  const int last = p.causal ? min(lk, max(t.row0 + BM + shift, 0)) : lk;
  for (int j0 = 0; j0 < last; j0 += BN) {
    __syncthreads();
    stage<T, D>(kb, p.kt, j0, BN, lk, p.d, ks);
    stage<T, D>(vb, p.vt, j0, BN, lk, p.d, vs);
    __syncthreads();
    f32x4 z[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}}, dp[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int s = 0; s < D / 4; s++)
#pragma unroll
      for (int b = 0; b < 2; b++) {
        z[b] = mfma4(a[s], ks[b * 16 + l16][4 * s + l4], z[b]);
        dp[b] = mfma4(g[s], vs[b * 16 + l16][4 * s + l4], dp[b]);
      }
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const int i = t.row0 + wave * 16 + 4 * l4 + r, end = p.causal ? min(lk, i + shift + 1) : lk;
#pragma unroll
      for (int b = 0; b < 2; b++)
        ds[wave][4 * l4 + r][b * 16 + l16] = j0 + b * 16 + l16 < end ? expf(z[b][r] * p.scale - l[r]) * (dp[b][r] - dr[r]) * p.scale : 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < BN / 4; s++)
#pragma unroll
      for (int j = 0; j < D / 16; j++) acc[j] = mfma4(ds[wave][l16][4 * s + l4], ks[4 * s + l4][16 * j + l16], acc[j]);
  }
#pragma unroll
  for (int r = 0; r < 4; r++) {
    const int i = t.row0 + wave * 16 + 4 * l4 + r;
    if (i >= t.len) continue;
    T* out = dq + (int64_t)(t.first + i) * ds_ + (int64_t)h * p.d;
#pragma unroll
    for (int j = 0; j < D / 16; j++)
      if (16 * j + l16 < p.d) st1(out + 16 * j + l16, acc[j][r]);
  }
}

// dk and dv of 64 key rows of one KV head, over its query heads and the query tiles that see them
template <typename T, int D>
__global__ __launch_bounds__(256) void attention_rows_dkv(PackedShape p, const T* __restrict__ dout, const T* __restrict__ q,
                                                          const T* __restrict__ k, const T* __restrict__ v, const float* __restrict__ lse,
                                                          const float* __restrict__ delta, T* __restrict__ dk, T* __restrict__ dv) {
  __shared__ f32 qs[BN][D + 16], gs[BN][D + 16], pt[4][16][BN + 4], dt[4][16][BN + 4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hk = blockIdx.y, l16 = lane & 15, l4 = lane >> 4;
  const PackedTile t = packed_tile(p.cu_k, p.n_seq, p.total_k, BM, blockIdx.x);
  if (t.row0 >= t.len) return;
  const int q0 = packed_bound(p.cu_q, t.seq, p.total_q), lq = max(packed_bound(p.cu_q, t.seq + 1, p.total_q) - q0, 0);
  const int group = p.nq / p.nkv, shift = t.len - lq, mine = t.row0 + wave * 16 + l16;
  const int64_t ds_ = (int64_t)p.nq * p.d, dks = (int64_t)p.nkv * p.d;
  f32 a[D / 4], b[D / 4];
  operand<T, D>(k + (int64_t)t.first * p.kt + (int64_t)hk * p.kh, p.kt, mine, t.len, p.d, lane, a);
  operand<T, D>(v + (int64_t)t.first * p.vt + (int64_t)hk * p.vh, p.vt, mine, t.len, p.d, lane, b);
  f32x4 ak[D / 16], av[D / 16];
#pragma unroll
  for (int j = 0; j < D / 16; j++) ak[j] = av[j] = {0.f, 0.f, 0.f, 0.f};
  const int first = p.causal ? max(t.row0 - shift, 0) / BN * BN : 0;
  for (int h = hk * group; h < (hk + 1) * group; h++) {
    const T* qb = q + (int64_t)q0 * p.qt + (int64_t)h * p.qh;
    const T* gb = dout + (int64_t)q0 * ds_ + (int64_t)h * p.d;
    for (int i0 = first; i0 < lq; i0 += BN) {
      __syncthreads();
      stage<T, D>(qb, p.qt, i0, BN, lq, p.d, qs);
      stage<T, D>(gb, ds_, i0, BN, lq, p.d, gs);
      __syncthreads();
      f32x4 z[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}}, dp[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
      for (int s = 0; s < D / 4; s++)
#pragma unroll
        for (int c = 0; c < 2; c++) {
          z[c] = mfma4(a[s], qs[c * 16 + l16][4 * s + l4], z[c]);
          dp[c] = mfma4(b[s], gs[c * 16 + l16][4 * s + l4], dp[c]);
        }
#pragma unroll
      for (int c = 0; c < 2; c++) {
        const int i = i0 + c * 16 + l16;
        const bool in = i < lq;
        const f32 l = in ? lse[(size_t)h * p.total_q + q0 + i] : 0.f, dl = in ? delta[(size_t)h * p.total_q + q0 + i] : 0.f;
        const int end = !in ? 0 : p.causal ? min(t.len, i + shift + 1) : t.len;      // this query sees the keys [0, end)
#pragma unroll
        for (int r = 0; r < 4; r++) {
          const f32 e = t.row0 + wave * 16 + 4 * l4 + r < end ? expf(z[c][r] * p.scale - l) : 0.f;
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
          av[j] = mfma4(x, gs[4 * s + l4][16 * j + l16], av[j]);
          ak[j] = mfma4(y, qs[4 * s + l4][16 * j + l16], ak[j]);
        }
      }
    }
  }
#pragma unroll
  for (int r = 0; r < 4; r++) {
    const int i = t.row0 + wave * 16 + 4 * l4 + r;
    if (i >= t.len) continue;
    const int64_t at = (int64_t)(t.first + i) * dks + (int64_t)hk * p.d;
#pragma unroll
    for (int j = 0; j < D / 16; j++)
      if (16 * j + l16 < p.d) {
        st1(dk + at + 16 * j + l16, ak[j][r]);
        st1(dv + at + 16 * j + l16, av[j][r]);
      }
  }
}

template <typename T, int D>
void forward(hipStream_t s, const PackedShape& p, const void* q, const void* k, const void* v, void* o, float* lse) {
  attention_rows_forward<T, D><<<dim3(packed_tiles(p.total_q, p.n_seq, BM), p.nq), 256, 0, s>>>(p, (const T*)q, (const T*)k, (const T*)v,
                                                                                                (T*)o, lse);
}
template <typename T, int D>
void backward(hipStream_t s, const PackedShape& p, const void* dout, const void* q, const void* k, const void* v, const void* o,
              const float* lse, void* dq, void* dk, void* dv, float* delta) {
  if (p.total_q > 0)
    attention_rows_dq<T, D><<<dim3(packed_tiles(p.total_q, p.n_seq, BM), p.nq), 256, 0, s>>>(
        p, (const T*)dout, (const T*)q, (const T*)k, (const T*)v, (const T*)o, lse, (T*)dq, delta);
  if (p.total_k > 0)
    attention_rows_dkv<T, D><<<dim3(packed_tiles(p.total_k, p.n_seq, BM), p.nkv), 256, 0, s>>>(
        p, (const T*)dout, (const T*)q, (const T*)k, (const T*)v, lse, delta, (T*)dk, (T*)dv);
}

const char* attention_argument(const PackedShape& p, int32_t dtype) {
  if (dtype != RL_DTYPE_F32 && dtype != RL_DTYPE_BF16) return "dtype is RL_DTYPE_F32 or RL_DTYPE_BF16";
  if (p.n_seq < 0 || p.n_seq > (1 << 24) || p.total_q < 0 || p.total_k < 0) return "sequences or tokens out of range";
  if (p.total_q > (1 << 30) || p.total_k > (1 << 30)) return "more than 2^30 tokens";
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
#define RL_GO(T, D) backward<T, D>(s, p, d_do, d_q, d_k, d_v, d_o, d_lse, d_dq, d_dk, d_dv, delta)
  if (dtype == RL_DTYPE_F32) {
    if (head_dim <= 64) RL_GO(float, 64);
    else RL_GO(float, 128);
  } else if (attention_takes_mfma(p, d_q, d_k, d_v, d_o, d_do) && aligned16(d_dq) && aligned16(d_dk) && aligned16(d_dv)) {
    launch_attention_mfma_backward(s, p, (const bf16_t*)d_do, (const bf16_t*)d_q, (const bf16_t*)d_k, (const bf16_t*)d_v, (const bf16_t*)d_o,
                                   d_lse, (bf16_t*)d_dq, (bf16_t*)d_dk, (bf16_t*)d_dv, delta);
  } else {
    if (head_dim <= 64) RL_GO(bf16_t, 64);
    else RL_GO(bf16_t, 128);
  }
#undef RL_GO
  return launched();
}
