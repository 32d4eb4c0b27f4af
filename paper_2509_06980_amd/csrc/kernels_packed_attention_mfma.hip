// Attention over packed sequences in bf16 on matrix instructions, forward and backward.
#include <atomic>
#include <type_traits>
#include <utility>

#include "lds_load.h"
#include "packed_attention.h"

namespace {

// =============================================================================================
// Three kernels of one shape: a wave owns 32 rows of one side (queries: forward and dq, four waves a workgroup; keys: dk and dv, eight) as
// columns of its 32x32x16 products, their operands in registers.  The other side streams through LDS, straight from memory, and
// serves as row operand:
//   forward   z^T = K Q^T,  o^T += V^T p^T
//   dq        z^T = K Q^T,  dp^T = V dO^T,  dq^T += K^T dz^T
//   dk, dv    z = Q K^T,  dp = dO V^T,  dv^T += dO^T p,  dk^T += Q^T dz
// So a lane holds scores of one of its own rows (columns) in registers, and they are the column operand of the next product as they
// are: the result of a product has rows 8 (e / 4) + 4 (lane / 32) + e % 4 in register e, so registers 8 s .. 8 s + 7 are the 16 k of
// step s in an order that the row operand, read from LDS by its transposing read, follows.  No score crosses lanes.
// The backward pass forms the scores twice, in both kernels (14 instead of 10 products' flops), rather than add dq up by atomics in an
// order that changes, or write the gradients of the scores out.  Probabilities and gradients of the scores are rounded to bf16, as the
// operands that they become; all sums, and the softmax's statistics, are kept in 32 bits.
// Bound by the matrix units (busy 53 to 70 % of the cycles for one sequence of 8192, 25 to 31 % for 16 ragged ones) with the exponentials beside
// them and by the LDS (1 KB per product instruction); the long case also by the clock that its data leaves: 1.6 to 1.8 GHz against 2.1 to
// 2.2 in the ragged case, in the same number of cycles on two GPUs whose clocks differ by 4 %, and zeros for data take 20 % less time.
// Measured, one sequence of 8192, 16 heads over 8 of 128, causal: forward 0.28 ms (0.98 PFLOP/s of the pairs that are seen), dq 0.36
// (1.16), dk and dv 0.57 (0.97); 16 sequences of 97 to 1511, 32 heads over 8: 100, 129 and 175 us.
// LDS: rows of D elements, 16-byte piece p of row r at p ^ f(r).  f moves 16 rows of one piece (read as they lie) to different
// banks, and the 4 rows x 32 columns of a transposing read as well.
// The two waves of a SIMD ought to be in different parts of a step, one at the products alone while the other has exponentials to
// form.  Issue priority (s_setprio) for the part with the arithmetic keeps them so; measured for one sequence of 8192, 16 heads of
// 128, with it and without: forward 278 and 297 us, dq 359 and 386, dk and dv 557 and 583.  Where it begins and ends is worth as much: dq
// with its end half a pass later 389.
// =============================================================================================
constexpr int BM = 128, BN = 64;      // rows owned, rows of a stage
constexpr int kFar = 0x7fff0000;      // a lane's offset behind every buffer's end: zeros
constexpr float kLog2e = 1.44269504088896341f;

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) float lds_float;
typedef __attribute__((address_space(3))) f32x4 lds_f32x4;

__device__ __forceinline__ f32x16 mfma(const u32x4& row, const u32x4& col, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, row), __builtin_bit_cast(bf16x8, col), c, 0, 0, 0);
}
// The same into the accumulation registers: left to itself the compiler moves sums that live through a loop between the two halves
// of the register file.  s_nop: it does not know how far back the operands were written.
__device__ __forceinline__ void accumulate(f32x16& c, const u32x4& row, const u32x4& col) {
  asm volatile("s_nop 1\n\tv_mfma_f32_32x32x16_bf16 %0, %1, %2, %0" : "+a"(c) : "v"(row), "v"(col));
}
__device__ __forceinline__ f32x16 zero16() {
  f32x16 z;
#pragma unroll
  for (int e = 0; e < 16; e++) z[e] = 0.f;
  return z;
}

// f(0), f(1), ... f(N - 1) with the numbers as types
template <int... I, typename F>
__device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F f) {
  (f(std::integral_constant<int, I>()), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F f) {
  each_of(std::make_integer_sequence<int, N>(), f);
}

// Tiles of 64 rows of a tensor on their way into LDS.  The descriptor ends with the sequence's last row: rows behind it are zeros.
template <int D>
struct Stream {
  static constexpr int N = D / 32;                 // 1 KB loads of a wave per tile
  u32x4 rsrc;
  int off[N];
  unsigned step;
  __device__ __forceinline__ void init(const bf16_t* p, int64_t stride, int len, int d, int wave, int lane) {
    rsrc = buffer_rsrc(p, (unsigned)(((int64_t)(len - 1) * stride + d) * 2));
    step = (unsigned)stride * (BN * 2);
    constexpr int PIECES = D / 8, ROWS = 64 / PIECES;      // of a row; of a load
#pragma unroll
    for (int j = 0; j < N; j++) {
      const int r = (j * 4 + wave) * ROWS + lane / PIECES, p8 = (lane % PIECES) ^ swizzle(r);
      off[j] = p8 * 8 < d ? (int)(r * stride * 2) + p8 * 16 : kFar;
    }
    settle(rsrc);
  }
  static __device__ __forceinline__ int swizzle(int r) {
    return D == 128 ? ((r & 3) << 2) | (r >> 2 & 3) : ((r >> 1 & 1) << 2) | (r >> 2 & 3);
  }
  __device__ __forceinline__ void load(int tile, unsigned lds, int wave) const {
#pragma unroll
    for (int j = 0; j < N; j++) load_to_lds(lds + (unsigned)(j * 4 + wave) * 1024u, off[j], rsrc, min((unsigned)tile * step, rsrc[2]));
  }
};

// Reads from tiles.  A lane's addresses differ in bits 5 to 7 alone, by exclusive or with a constant; tiles begin at multiples of 256
// bytes, so moving to another one leaves those bits: one addition a tile, one exclusive or a read, the rest is in the instruction.
template <int D>
struct Reads {
  lds_char *row, *tr;
  __device__ __forceinline__ Reads(lds_char* base, int lane) {
    const int i = lane & 15, h = lane >> 5, w = lane >> 4 & 1;
    const int f = D == 128 ? (i >> 2) << 2 : (i >> 3 & 1) << 2;
    row = base + (lane & 31) * (D * 2) + ((h ^ Stream<D>::swizzle(lane & 31)) << 4);
    tr = base + (4 * h + (i >> 2)) * (D * 2) + ((f | ((2 * w + (i >> 1 & 1)) ^ h)) << 4) + ((i & 1) << 3);
  }
  __device__ __forceinline__ void move(int bytes) {
    row += bytes;
    tr += bytes;
    asm volatile("" : "+v"(row), "+v"(tr));      // or the compiler keeps every read's address in a register of its own
  }
  static __device__ __forceinline__ lds_char* turned(lds_char* p, unsigned bits) {
    return (lds_char*)((unsigned)(uintptr_t)p ^ bits);
  }
  // 32 rows from row 32 x of the tile `at` bytes on, k = columns 16 s .. + 15
  __device__ __forceinline__ u32x4 rows(int at, int x, int s) const {
    return *(lds_u32x4*)(turned(row, s << 5) + (at + x * 32 * (D * 2)));
  }
  // rows = columns 32 b .. + 31, k = rows 32 x + 16 s .. + 15 in the order of a result's registers
  __device__ __forceinline__ u32x4 columns(int at, int x, int s, int b) const {
    const int off = at + (32 * x + 16 * s) * (D * 2);
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(turned(tr, b << 6) + off));
    const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(turned(tr, b << 6 | 32) + (off + 8 * (D * 2))));
    return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
};

// column operand of a wave's 32 rows: row lane % 32, columns 16 s + 8 (lane / 32) .. + 7
template <int D>
__device__ __forceinline__ void own_rows(const bf16_t* p, int64_t stride, int row, int len, int d, int lane, u32x4 (&q)[D / 16]) {
#pragma unroll
  for (int s = 0; s < D / 16; s++) {
    const int c = 16 * s + 8 * (lane >> 5);
    const bool in = row < len && c < d;
    q[s] = *(const u32x4*)(in ? p + (int64_t)row * stride + c : p);      // len >= 1: no branch around a load
    if (!in) q[s] = u32x4{0, 0, 0, 0};
  }
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
  const bf16x2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}
// registers 8 s .. 8 s + 7 of a result as the column operand of step s
__device__ __forceinline__ u32x4 as_operand(const f32x16& v, int s) {
  return u32x4{pack2(v[8 * s], v[8 * s + 1]), pack2(v[8 * s + 2], v[8 * s + 3]), pack2(v[8 * s + 4], v[8 * s + 5]), pack2(v[8 * s + 6], v[8 * s + 7])};
}
// row (of the streamed side) of register e
__device__ __forceinline__ int row_of(int e, int lane) { return 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3); }
// a wave's result^T [D x 32 rows] to memory, times f; lane's row at p
template <int D>
__device__ __forceinline__ void store_rows(const f32x16 (&acc)[D / 32], float f, bf16_t* p, int d, int lane) {
#pragma unroll
  for (int b = 0; b < D / 32; b++)
#pragma unroll
    for (int q = 0; q < 4; q++) {
      const int c = 32 * b + 8 * q + 4 * (lane >> 5);
      if (c < d) *(uint2*)(p + c) = make_uint2(pack2(acc[b][4 * q] * f, acc[b][4 * q + 1] * f), pack2(acc[b][4 * q + 2] * f, acc[b][4 * q + 3] * f));
    }
}

// What a workgroup of the query side works on.
struct QuerySide {
  PackedTile t;
  int h, hk, k0, lk, shift, last;      // last: keys [0, last) are seen by some row of the tile
};
__device__ __forceinline__ bool query_side(const PackedShape& p, QuerySide& w) {
  // KV heads fastest, so workgroups on one XCD share keys; row tiles from the last to the first: causal ones begin with the longest
  const int id = blockIdx.x, n = packed_tiles(p.total_q, p.n_seq, BM);
  w.hk = id % p.nkv;
  w.h = w.hk * (p.nq / p.nkv) + id / p.nkv % (p.nq / p.nkv);
  w.t = packed_tile(p.cu_q, p.n_seq, p.total_q, BM, n - 1 - id / p.nq);
  if (w.t.row0 >= w.t.len) return false;
  w.k0 = packed_bound(p.cu_k, w.t.seq, p.total_k);
  w.lk = max(packed_bound(p.cu_k, w.t.seq + 1, p.total_k) - w.k0, 0);
  w.shift = w.lk - w.t.len;
  w.last = p.causal ? min(w.lk, max(min(w.t.row0 + BM, w.t.len) + w.shift, 0)) : w.lk;
  return true;
}

template <int D>
__global__ __launch_bounds__(256, 2) void attention_forward_kernel(PackedShape p, const bf16_t* __restrict__ q, const bf16_t* __restrict__ k,
                                                                   const bf16_t* __restrict__ v, bf16_t* __restrict__ o,
                                                                   float* __restrict__ lse) {
  constexpr int TILE = BN * D * 2;      // LDS: two tiles of keys, three of values
  extern __shared__ u32x4 smem[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const OutsideRows outside(p.cu_q, p.n_seq, p.total_q);
  QuerySide w;
  const bool some_rows = query_side(p, w);
  outside.clear<bf16_t>(p.nq * p.d, o, nullptr, lse, p.nq);
  if (!some_rows) return;
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
  Reads<D> lds((lds_char*)(__attribute__((address_space(3))) void*)smem, lane);      // of the keys, of the values in work
  lds.tr += 2 * TILE;
  const int mine = w.t.row0 + wave * 32 + (lane & 31);      // lane's query
  u32x4 qr[D / 16];
  own_rows<D>(q + (int64_t)w.t.first * p.qt + (int64_t)w.h * p.qh, p.qt, mine, w.t.len, p.d, lane, qr);
  const unsigned flip = p.scale < 0.f ? 0x80008000u : 0u;      // c > 0 below: the largest product is the largest score
#pragma unroll
  for (int s = 0; s < D / 16; s++)
#pragma unroll
    for (int i = 0; i < 4; i++) qr[s][i] ^= flip;
  f32x16 acc[D / 32];
#pragma unroll
  for (int b = 0; b < D / 32; b++) acc[b] = zero16();
  float ref = -INFINITY, sum = 0.f;      // ref: log2 units; sum of this half's terms
  const float c = fabsf(p.scale) * kLog2e;
  const int seen = p.causal ? min(w.lk, mine + w.shift + 1) : w.lk;             // lane's query sees the keys [0, seen)
  const int row_a = w.t.row0 + wave * 32, row_b = min(row_a + 32, w.t.len);     // wave's queries
  const int all = row_a >= w.t.len ? 0 : p.causal ? min(w.lk, row_a + w.shift + 1) : w.lk;      // keys that all of them see
  const int some = row_a >= w.t.len ? 0 : p.causal ? min(w.lk, row_b + w.shift) : w.lk;         // ... that one sees
  const int tiles = (w.last + BN - 1) / BN, steps = (max(some, 0) + 31) / 32;
  // top: the largest of the lane's 16 products; moves the reference of the exponents only where a term would exceed 2^8:
  // rounding is relative, and sums stay far from overflow
  auto refer = [&](float top) {
    top *= c;
    if (__any(top > ref + 8.f)) {
      top = fmaxf(top, __shfl_xor(top, 32, 64));
      const float now = fmaxf(ref, top), f = now == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ref - now);
      ref = now;
      sum *= f;
#pragma unroll
      for (int b = 0; b < D / 32; b++)
#pragma unroll
        for (int e = 0; e < 16; e++) acc[b][e] *= f;
    }
  };
  auto mask = [&](f32x16& z, int j) {      // keys from j on
    if (j + 32 > all) {
#pragma unroll
      for (int e = 0; e < 16; e++)
        if (j + row_of(e, lane) >= seen) z[e] = -INFINITY;
    }
  };
  // A step of 32 keys, in slots as in the backward pass: first the scores of the next step beside the exponentials of this one, then
  // this one's values beside the largest of the next scores.
  constexpr int S = D / 16, AHEAD = D == 128 ? 5 : 4, EXPS = 3 * S / 2;
  u32x4 a[8];
  auto step = [&](auto half, auto more, int n, f32x16& z, f32x16& next, auto middle) {
    constexpr int H = decltype(half)::value;
    constexpr bool MORE = decltype(more)::value;
    const float r = ref == -INFINITY ? 0.f : ref;      // nothing seen yet: e^-inf = 0
    float top = -INFINITY;
    u32x4 pr[2];
    if constexpr (MORE) next = zero16();
    each<2 * S>([&](auto slot) {
      constexpr int m = decltype(slot)::value, later = m + AHEAD;
      if constexpr (m == S / 2) __builtin_amdgcn_s_setprio(1);
      if constexpr (m == EXPS) __builtin_amdgcn_s_setprio(0);
      if constexpr (m == S && H == 0) middle();      // the next tile has landed
      if constexpr (later == 2 * S && H == 0 && MORE) {      // every read of this tile's keys is under way
        lds.row += (n >> 1 & 1) ? -TILE : TILE;
        asm volatile("" : "+v"(lds.row));
      }
      if constexpr (later < S) {
        if constexpr (MORE) a[later & 7] = lds.rows(0, 1 - H, later);
      } else if constexpr (later < 2 * S) {
        a[later & 7] = lds.columns(0, H, (later - S) / (D / 32), (later - S) % (D / 32));
      } else if constexpr (MORE) {
        a[later & 7] = lds.rows(0, H, later - 2 * S);
      }
      if constexpr (m < S) {
        if constexpr (MORE) next = mfma(a[m & 7], qr[m], next);
      } else {
        acc[(m - S) % (D / 32)] = mfma(a[m & 7], pr[(m - S) / (D / 32)], acc[(m - S) % (D / 32)]);
      }
      if constexpr (m < EXPS) {
#pragma unroll
        for (int e = m * 16 / EXPS; e < (m + 1) * 16 / EXPS; e++) {
          z[e] = __builtin_amdgcn_exp2f(fmaf(z[e], c, -r));
          sum += z[e];
        }
        asm volatile("" : "+v"(sum));      // here, not all at the end
        if constexpr (m == S - 1) pr[0] = as_operand(z, 0);      // probabilities rounded to bf16; their sum is not
        if constexpr (m == EXPS - 1) pr[1] = as_operand(z, 1);
      } else if constexpr (MORE) {
        if constexpr (m == EXPS) mask(next, 32 * n + 32);
#pragma unroll
        for (int e = (m - EXPS) * 32 / S; e < (m - EXPS + 1) * 32 / S; e++) top = fmaxf(top, next[e]);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (MORE) refer(top);
  };
  Stream<D> ks, vs;
  if (tiles > 0) {
    ks.init(k + (int64_t)w.k0 * p.kt + (int64_t)w.hk * p.kh, p.kt, w.lk, p.d, wave, lane);
    vs.init(v + (int64_t)w.k0 * p.vt + (int64_t)w.hk * p.vh, p.vt, w.lk, p.d, wave, lane);
    ks.load(0, lds0, wave);
    vs.load(0, lds0 + 2 * TILE, wave);
    if (tiles > 1) {
      ks.load(1, lds0 + TILE, wave);
      vs.load(1, lds0 + 3 * TILE, wave);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
  }
  f32x16 z[2];
  if (steps > 0) {
    z[0] = zero16();
#pragma unroll
    for (int s = 0; s < S; s++) z[0] = mfma(lds.rows(0, 0, s), qr[s], z[0]);
    mask(z[0], 0);
    float top = -INFINITY;
#pragma unroll
    for (int e = 0; e < 16; e++) top = fmaxf(top, z[0][e]);
    refer(top);
    each<AHEAD>([&](auto m) { a[decltype(m)::value] = lds.rows(0, 1, decltype(m)::value); });
  }
  const std::integral_constant<int, 0> first;
  const std::integral_constant<int, 1> second;
  for (int t = 0; t < tiles; t++) {
    const int n = 2 * t;
    // Tile t + 1 has landed, for every wave; every wave is done with the keys of tile t and with the values of tile t - 1.
    auto middle = [&]() {
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      if (t + 2 < tiles) {
        ks.load(t + 2, lds0 + (unsigned)(t & 1) * TILE, wave);
        vs.load(t + 2, lds0 + 2 * TILE + (unsigned)((t + 2) % 3) * TILE, wave);
      }
    };
    if (n < steps) step(first, std::true_type(), n, z[0], z[1], middle);
    else middle();
    if (n + 1 < steps) step(second, std::true_type(), n + 1, z[1], z[0], []() {});
    lds.tr += t % 3 == 2 ? -2 * TILE : TILE;
    asm volatile("" : "+v"(lds.tr));
  }
  sum += __shfl_xor(sum, 32, 64);
  if (mine < w.t.len) {
    const float inv = sum > 0.f ? 1.f / sum : sum == 0.f ? 0.f : sum;      // no key: zeros; no number stays so
    store_rows<D>(acc, inv, o + (int64_t)(w.t.first + mine) * p.ot + (int64_t)w.h * p.oh, p.d, lane);
    if (lane < 32) lse[(size_t)w.h * p.total_q + w.t.first + mine] = sum == 0.f ? -INFINITY : (ref + __builtin_amdgcn_logf(sum)) * (1.f / kLog2e);
  }
}

// dq, and what the other kernel reads of a query: - lse / scale, with which its sums of q.k begin (where it sees no key an infinity that
// makes the probabilities 0), and - delta, delta = rowsum(dO o) = sum of p dp
template <int D>
__global__ __launch_bounds__(256, 2) void attention_dq_kernel(PackedShape p, const bf16_t* __restrict__ dout, const bf16_t* __restrict__ q,
                                                              const bf16_t* __restrict__ k, const bf16_t* __restrict__ v,
                                                              const bf16_t* __restrict__ o, const float* __restrict__ lse,
                                                              bf16_t* __restrict__ dq, float* __restrict__ stats) {
  constexpr int TILE = BN * D * 2, STAGE = 2 * TILE;
  extern __shared__ u32x4 smem[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const OutsideRows outside(p.cu_q, p.n_seq, p.total_q);
  QuerySide w;
  const bool some_rows = query_side(p, w);
  outside.clear<bf16_t>(p.nq * p.d, dq, nullptr, nullptr, 0);
  if (!some_rows) return;
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
  Reads<D> lds((lds_char*)(__attribute__((address_space(3))) void*)smem, lane);      // of the stage in work
  const int mine = w.t.row0 + wave * 32 + (lane & 31);
  const int tiles = __builtin_amdgcn_readfirstlane((w.last + BN - 1) / BN);
  const bool few = tiles > 0 && tiles <= 2;
  Stream<D> ks, vs;
  ks.init(k + (int64_t)w.k0 * p.kt + (int64_t)w.hk * p.kh, p.kt, max(w.lk, 1), p.d, wave, lane);
  vs.init(v + (int64_t)w.k0 * p.vt + (int64_t)w.hk * p.vh, p.vt, max(w.lk, 1), p.d, wave, lane);
  if (tiles > 0) {
    ks.load(0, lds0, wave);
    vs.load(0, lds0 + TILE, wave);
  }
  if (few && tiles > 1) {
    ks.load(1, lds0 + STAGE, wave);
    vs.load(1, lds0 + STAGE + TILE, wave);
  }
  // all that the rows need is requested before the first of it is waited for
  const size_t stat = (size_t)w.h * p.total_q + w.t.first + min(mine, w.t.len - 1);
  float dl = 0.f, l = lse[stat] * kLog2e;
  u32x4 qr[D / 16], gr[D / 16], orow[D / 16];
  own_rows<D>(dout + (int64_t)w.t.first * p.ot + (int64_t)w.h * p.oh, p.ot, mine, w.t.len, p.d, lane, gr);
  own_rows<D>(o + (int64_t)w.t.first * p.ot + (int64_t)w.h * p.oh, p.ot, mine, w.t.len, p.d, lane, orow);
  own_rows<D>(q + (int64_t)w.t.first * p.qt + (int64_t)w.h * p.qh, p.qt, mine, w.t.len, p.d, lane, qr);
#pragma unroll
  for (int s = 0; s < D / 16; s++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
      dl = fmaf(bf2f((bf16_t)(gr[s][i] & 0xffffu)), bf2f((bf16_t)(orow[s][i] & 0xffffu)), dl);
      dl = fmaf(bf2f((bf16_t)(gr[s][i] >> 16)), bf2f((bf16_t)(orow[s][i] >> 16)), dl);
    }
  dl += __shfl_xor(dl, 32, 64);
  if (l == -INFINITY) l = INFINITY;
  const float c = p.scale * kLog2e;
  const int seen = p.causal ? min(w.lk, mine + w.shift + 1) : w.lk;
  const int row_a = w.t.row0 + wave * 32, row_b = min(row_a + 32, w.t.len);
  const int all = row_a >= w.t.len ? 0 : p.causal ? min(w.lk, row_a + w.shift + 1) : w.lk;
  const int some = row_a >= w.t.len ? 0 : p.causal ? min(w.lk, row_b + w.shift) : w.lk;
  // Queries of few keys: o is large there, its rounding to bf16 moves delta by as much as the gradients of the scores are rounded below.
  // Up to 128 keys fit both stages, so delta is taken as sum of p dp without reading any twice: relative error of these queries' dq 0.0024,
  // from the rounded o 0.0026, of the last rounding alone 0.0017.  Of more keys o is smaller, about by the root of their number, and its
  // rounding counts for less: 0.0025 at 128 to 512 keys, 0.0024 beyond.
  if (few) {
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    dl = 0.f;
    for (int j = 0; j < some; j += 32) {
      const int at = j / BN * STAGE, x = j / 32 & 1;
      f32x16 z = zero16(), dp = zero16();
#pragma unroll
      for (int s = 0; s < D / 16; s++) {
        z = mfma(lds.rows(at, x, s), qr[s], z);
        dp = mfma(lds.rows(at + TILE, x, s), gr[s], dp);
      }
#pragma unroll
      for (int e = 0; e < 16; e++)
        if (j + row_of(e, lane) < seen) dl = fmaf(__builtin_amdgcn_exp2f(fmaf(z[e], c, -l)), dp[e], dl);
    }
    dl += __shfl_xor(dl, 32, 64);
  }
  f32x16 acc[D / 32];
#pragma unroll
  for (int b = 0; b < D / 32; b++) acc[b] = zero16();
  // 32 keys, in slots of one row operand, read three slots ahead, its product, and a share of the arithmetic on the scores
  constexpr int S = D / 16, SLOTS = 3 * S, AHEAD = 3, PER = 16 / S;
  auto tile = [&](int j0, int x, bool masked) {
    u32x4 a[4], dz[2];
    f32x16 z, dp;
    auto read = [&](auto slot) {
      constexpr int n = decltype(slot)::value, m = n % S;
      if constexpr (n < S) return lds.rows(0, x, n);
      else if constexpr (n < 2 * S) return lds.rows(TILE, x, m);
      else return lds.columns(0, x, m / (D / 32), m % (D / 32));
    };
    each<AHEAD>([&](auto n) { a[decltype(n)::value] = read(n); });
#pragma unroll
    for (int e = 0; e < 16; e++) z[e] = 0.f, dp[e] = -dl;
    each<SLOTS>([&](auto slot) {
      constexpr int n = decltype(slot)::value, m = n % S, later = n + AHEAD;
      if constexpr (n == S / 2) __builtin_amdgcn_s_setprio(1);
      if constexpr (n == 2 * S) __builtin_amdgcn_s_setprio(0);
      if constexpr (later < SLOTS) a[later & 3] = read(std::integral_constant<int, later>());
      const u32x4 row = a[n & 3];
      if constexpr (n < S) {                   // scores
        z = mfma(row, qr[n], z);
      } else if constexpr (n < 2 * S) {        // gradients of the probabilities, less delta; probabilities
        dp = mfma(row, gr[m], dp);
#pragma unroll
        for (int e = m * PER; e < (m + 1) * PER; e++) z[e] = __builtin_amdgcn_exp2f(fmaf(z[e], c, -l));
        if constexpr (m == S - 1) {
          if (masked) {
#pragma unroll
            for (int e = 0; e < 16; e++)
              if (j0 + 32 * x + row_of(e, lane) >= seen) z[e] = 0.f;
          }
#pragma unroll
          for (int e = 0; e < 16; e++) dp[e] *= z[e];
          dz[0] = as_operand(dp, 0);
          dz[1] = as_operand(dp, 1);
        }
      } else {
        acc[m % (D / 32)] = mfma(row, dz[m / (D / 32)], acc[m % (D / 32)]);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  for (int t = 0; t < tiles; t++) {
    const int at = (t & 1) * STAGE;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    if (!few && t + 1 < tiles) {
      ks.load(t + 1, lds0 + (unsigned)(STAGE - at), wave);
      vs.load(t + 1, lds0 + (unsigned)(STAGE - at + TILE), wave);
    }
    const int j0 = t * BN;
    if (j0 < some) {
      tile(j0, 0, j0 + 32 > all);
      tile(j0, 1, j0 + BN > all);
    }
    lds.move(t & 1 ? -STAGE : STAGE);
  }
  if (mine < w.t.len && lane < 32) {
    stats[stat] = l / -(p.scale * kLog2e);
    stats[stat + (size_t)p.nq * p.total_q] = -dl;
  }
  if (mine < w.t.len) store_rows<D>(acc, p.scale, dq + (int64_t)(w.t.first + mine) * p.ot + (int64_t)w.h * p.oh, p.d, lane);
}

// dk and dv of 32 BLOCKS keys of one KV head.  Eight waves: BLOCKS blocks of 32 keys x 8 / BLOCKS streams, which take the (query head of
// the group, 32 queries) that see the keys in turn, through a ring of LDS stages of their own; the streams' sums are added up in LDS at the end, in their order.  A wave has its keys as
// operand and both sums in registers (128 of them, the accumulation half of the file), the values lie in LDS: with them two waves a
// SIMD would not fit.  A step is laid out by hand in slots of one row operand, read three slots ahead, its product, and a share of
// the arithmetic on the scores of the products before.
template <int D, int BLOCKS, int R>
__global__ __launch_bounds__(512, 2) void attention_dkv_kernel(PackedShape p, const bf16_t* __restrict__ dout, const bf16_t* __restrict__ q,
                                                               const bf16_t* __restrict__ k, const bf16_t* __restrict__ v,
                                                               const float* __restrict__ query_stats, bf16_t* __restrict__ dk,
                                                               bf16_t* __restrict__ dv, KeyParts parts) {
  constexpr int STREAMS = 8 / BLOCKS, KEYS = 32 * BLOCKS;
  constexpr int TILE = 32 * D * 2, STAGE = 2 * TILE + 512;      // of a stream: queries, dO, then - lse / scale and - delta of the queries
  constexpr int S = D / 16, SLOTS = 4 * S, AHEAD = 3, VA = 2, PER = 16 / S;
  extern __shared__ u32x4 smem[];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, block = wave % BLOCKS, stream = wave / BLOCKS;
  const OutsideRows outside(p.cu_k, p.n_seq, p.total_k);
  const int hk = blockIdx.x % p.nkv, group = p.nq / p.nkv;
  // The tiles that most queries see first: a workgroup that begins last should not be the longest.  Measured, 16 sequences of 97 to 1511:
  // 171 us, in the order of the sequences 184; one sequence is in order as it is (562 us, counted through 569).
  const int tile = blockIdx.x / p.nkv;
  const PackedTile t = p.n_seq > 1 && p.n_seq <= 64 ? packed_tile_by_rest(p.cu_k, p.n_seq, p.total_k, KEYS, tile)
                                                    : packed_tile(p.cu_k, p.n_seq, p.total_k, KEYS, tile);
  outside.clear<bf16_t>(p.nkv * p.d, dk, dv, nullptr, 0);
  if (t.row0 >= t.len) return;
  const int q0 = packed_bound(p.cu_q, t.seq, p.total_q), lq = max(packed_bound(p.cu_q, t.seq + 1, p.total_q) - q0, 0);
  const int shift = t.len - lq;
  lds_char* const lds_base = (lds_char*)(__attribute__((address_space(3))) void*)smem;
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
  const int own = stream * R * STAGE;      // of the stream's stages
  lds_char *const base = lds_base + own, *const value_base = lds_base + STREAMS * R * STAGE + block * TILE;
  f32x16 ak[D / 32], av[D / 32];
#pragma unroll
  for (int b = 0; b < D / 32; b++) ak[b] = av[b] = zero16();
  {
    Stream<D> vs;      // the values: 64 rows by four waves
    vs.init(v + (int64_t)t.first * p.vt + (int64_t)hk * p.vh, p.vt, t.len, p.d, wave & 3, lane);
    if (2 * (wave >> 2) < BLOCKS) vs.load(t.row0 / 64 + (wave >> 2), lds0 + STREAMS * R * STAGE + (unsigned)(wave >> 2) * (2 * TILE), wave & 3);
  }
  const int first = p.causal ? max(t.row0 - shift, 0) / 32 : 0, per_head = max((lq + 31) / 32 - first, 0);
  const int step_by = STREAMS * parts.n, begin_at = blockIdx.y * STREAMS;      // this workgroup's share of the (query head, query tile) pairs
  const int rounds = max((per_head * group - begin_at + step_by - 1) / step_by, 0);
  const int mine = t.row0 + 32 * block + (lane & 31);                                   // lane's key
  const int all = p.causal ? max(t.row0 + 32 * block + 31 - shift, 0) : 0;              // queries from here on see all keys of the wave
  u32x4 kr[S];
  const float c2 = p.scale * kLog2e;
  // The waves of a stream share its loads: the first half takes the queries, the second dO; 1 KB a load, ROWS rows.  A scalar offset
  // never leaves its buffer; a stream without work reads nothing but zeros, which add nothing (queries behind the end are zeros too).
  constexpr int ROWS = 512 / D, LOADS = 2 * (32 / ROWS) / BLOCKS;
  const bool second = block >= BLOCKS / 2;
  const int j0 = block % (BLOCKS / 2) * LOADS;
  const bf16_t* const from = second ? dout : q;
  const int64_t ts = second ? p.ot : p.qt, hs = second ? p.oh : p.qh;
  const float* const stats_from = query_stats + (second ? (size_t)p.nq * p.total_q : 0);
  const unsigned full = (unsigned)(((int64_t)(lq - 1) * ts + p.d) * 2);
  int item = begin_at + stream, h = hk * group;      // next tile of the current head
  auto load = [&](int at) {
    while (h < (hk + 1) * group && item >= per_head) {
      item -= per_head;
      h++;
    }
    const bool some = h < (hk + 1) * group;
    const unsigned bytes = some ? full : 0u, sbytes = some ? (unsigned)lq * 4u : 0u;
    const int hd = some ? h : 0;
    u32x4 rsrc = buffer_rsrc(from + (int64_t)q0 * ts + (int64_t)hd * hs, bytes);
    const u32x4 srsrc = buffer_rsrc(stats_from + (size_t)hd * p.total_q + q0, sbytes);
    settle(rsrc);
    const int i = first + item;
    int ln = lane;
    asm volatile("" : "+v"(ln));      // the offsets are formed anew: registers
    const int r = ln / (D / 8), row_off = r * (int)ts * 2;
#pragma unroll
    for (int j = 0; j < LOADS; j++) {
      const int p8 = (ln % (D / 8)) ^ Stream<D>::swizzle((j0 + j) * ROWS + r);
      load_to_lds(lds0 + (unsigned)(own + at + (second ? TILE : 0) + (j0 + j) * 1024), p8 * 8 < p.d ? row_off + p8 * 16 : kFar, rsrc,
                  min((unsigned)(i * 32 + (j0 + j) * ROWS) * (unsigned)ts * 2u, bytes));
    }
    load_dword_to_lds(lds0 + (unsigned)(own + at + 2 * TILE + (second ? 256 : 0)), ln < 32 ? ln * 4 : kFar, srsrc, min((unsigned)i * 128u, sbytes));
  };
  // One round of 32 queries.  MID: the first operands of the next round are read at the end of this one, its rows have landed by then;
  // the barrier stands in the middle of the round for the first four waves and at its beginning for the others.  That keeps the two
  // waves of a SIMD half a round apart: one has its products while the other waits for scores.
  constexpr bool MID = R == 3;
  u32x4 a[4];
  Reads<D> lds(base, lane);      // of the round in work
  const Reads<D> values(value_base, lane);
  auto read = [&](auto slot) {      // row operand of a slot
    constexpr int n = decltype(slot)::value, m = n % S;
    if constexpr (n < S) return lds.rows(0, 0, n);
    else if constexpr (n < 2 * S) return lds.rows(TILE, 0, m);
    else return lds.columns(n < 3 * S ? TILE : 0, 0, m / (D / 32), m % (D / 32));
  };
  auto begin = [&]() {
    each<AHEAD>([&](auto n) { a[decltype(n)::value] = read(n); });
  };
  auto step = [&](int i0, int at, int after, auto middle) {
    lds_char* value_row = values.row;
    asm volatile("" : "+v"(value_row));
    u32x4 vr[VA + 1], pr[2], dz[2];
    f32x16 z, dp;
    const lds_float* stats = (const lds_float*)(lds_base + own + at + 2 * TILE) + 4 * (lane >> 5);
#pragma unroll
    for (int g = 0; g < 4; g++) {
      const f32x4 l = *(const lds_f32x4*)(stats + 8 * g);
#pragma unroll
      for (int r = 0; r < 4; r++) z[4 * g + r] = l[r];
    }
    each<SLOTS>([&](auto slot) {
      constexpr int n = decltype(slot)::value, m = n % S, later = n + AHEAD;
      if constexpr (n == 0) __builtin_amdgcn_s_setprio(1);
      if constexpr (n == 2 * S) __builtin_amdgcn_s_setprio(0);
      if constexpr (MID && (n == 0 || n == 2 * S)) {
        if ((wave >> 2) == (n == 0)) middle();
      }
      if constexpr (later < SLOTS) a[later & 3] = read(std::integral_constant<int, later>());
      else if constexpr (MID) {
        if constexpr (later == SLOTS) lds.move(after - at);      // every read of this round is under way
        a[later & 3] = read(std::integral_constant<int, later - SLOTS>());
      }
      if constexpr (n + VA >= S && n + VA < 2 * S) vr[(n + VA) % (VA + 1)] = *(lds_u32x4*)Reads<D>::turned(value_row, (n + VA - S) << 5);
      const u32x4 x = a[n & 3];
      if constexpr (n < S) {                   // scores
        z = mfma(x, kr[n], z);
        if constexpr (n == S - 2) {
#pragma unroll
          for (int g = 0; g < 4; g++) {
            const f32x4 dl = *(const lds_f32x4*)(stats + 64 + 8 * g);
#pragma unroll
            for (int r = 0; r < 4; r++) dp[4 * g + r] = dl[r];
          }
        }
      } else if constexpr (n < 2 * S) {        // gradients of the probabilities, less delta; probabilities
        dp = mfma(x, vr[n % (VA + 1)], dp);
#pragma unroll
        for (int e = m * PER; e < (m + 1) * PER; e++) z[e] = __builtin_amdgcn_exp2f(z[e] * c2);
        if constexpr (m == S - 1) {
          if (i0 < all) {      // the diagonal runs through the tile: queries from `seen` on see the lane's key
            const int seen = t.row0 + 32 * block + (lane & 31) - shift;
#pragma unroll
            for (int e = 0; e < 16; e++)
              if (i0 + row_of(e, lane) < seen) z[e] = 0.f;
          }
          pr[0] = as_operand(z, 0);
          pr[1] = as_operand(z, 1);
        }
      } else if constexpr (n < 3 * S) {        // dv; gradients of the scores
        accumulate(av[m % (D / 32)], x, pr[m / (D / 32)]);
#pragma unroll
        for (int e = m * PER; e < (m + 1) * PER; e++) dp[e] *= z[e];
        if constexpr (m == S - 1) {
          dz[0] = as_operand(dp, 0);
          dz[1] = as_operand(dp, 1);
        }
      } else {                                 // dk
        accumulate(ak[m % (D / 32)], x, dz[m / (D / 32)]);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  // Loads go R - 1 rounds ahead, whether there is work or not.  Tiles of the rounds in work are counted apart from those loaded: the
  // same walk over (head, tile).
  int done = begin_at + stream;
  int at = 0, next = (R - 1) * STAGE;
  auto landed = [&]() {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
  };
  auto load_next = [&]() {
    load(next);
    item += step_by;
    next = next + STAGE == R * STAGE ? 0 : next + STAGE;
  };
#pragma unroll
  for (int r = 0; r < R - 1; r++) {
    load(r * STAGE);
    item += step_by;
  }
  own_rows<D>(k + (int64_t)t.first * p.kt + (int64_t)hk * p.kh, p.kt, mine, t.len, p.d, lane, kr);
  if constexpr (MID) {
    landed();
    begin();
  }
  for (int r = 0; r < rounds; r++) {
    while (done >= per_head) done -= per_head;
    const int i0 = (first + done) * 32, after = at + STAGE == R * STAGE ? 0 : at + STAGE;
    if constexpr (MID) {
      // the next round's rows have landed for every wave, and every wave is done with the round before
      step(i0, at, after, [&]() {
        landed();
        load_next();
      });
    } else {
      landed();      // this round's rows, and every wave is done with the round before
      load_next();
      begin();
      step(i0, at, after, []() {});
      lds.move(after - at);
    }
    at = after;
    done += step_by;
  }
  asm volatile("s_waitcnt vmcnt(0)\n\ts_nop 15\n\ts_nop 15" ::: "memory");      // results of the assembly's last products
  // the streams' sums: [stream][key][D + 4] in LDS; several threads add up and store a key
  constexpr int PITCH = D + 4;
  lds_float* const sums = (lds_float*)lds_base;
  auto join = [&](const f32x16 (&acc)[D / 32], float f, bf16_t* out, int which) {
    __syncthreads();
#pragma unroll
    for (int b = 0; b < D / 32; b++)
#pragma unroll
      for (int g = 0; g < 4; g++)
        *(lds_f32x4*)(sums + (stream * KEYS + 32 * block + (lane & 31)) * PITCH + 32 * b + 8 * g + 4 * (lane >> 5)) =
            f32x4{acc[b][4 * g], acc[b][4 * g + 1], acc[b][4 * g + 2], acc[b][4 * g + 3]};
    __syncthreads();
    constexpr int SHARE = 512 / KEYS;      // threads of a key
    const int key = threadIdx.x / SHARE;
    if (t.row0 + key < t.len) {
      const int64_t row_at = (int64_t)(t.first + t.row0 + key) * p.nkv * p.d + (int64_t)hk * p.d;
      bf16_t* row = out + row_at;
      float* const sum_row = parts.n > 1 ? parts.of(p, blockIdx.y, which) + row_at : nullptr;
#pragma unroll
      for (int j = 0; j < D / 8 / SHARE; j++) {
        const int col = (threadIdx.x % SHARE) * 8 + 8 * SHARE * j;
        float y[8];
#pragma unroll
        for (int w = 0; w < STREAMS; w++) {
          const lds_float* part = sums + (w * KEYS + key) * PITCH + col;
          const f32x4 lo = *(const lds_f32x4*)part, hi = *(const lds_f32x4*)(part + 4);
#pragma unroll
          for (int e = 0; e < 4; e++) {
            y[e] = w ? y[e] + lo[e] : lo[e];
            y[4 + e] = w ? y[4 + e] + hi[e] : hi[e];
          }
        }
        if (col < p.d && sum_row) {
          *(float4*)(sum_row + col) = make_float4(y[0] * f, y[1] * f, y[2] * f, y[3] * f);
          *(float4*)(sum_row + col + 4) = make_float4(y[4] * f, y[5] * f, y[6] * f, y[7] * f);
        } else if (col < p.d)
          *(u32x4*)(row + col) = u32x4{pack2(y[0] * f, y[1] * f), pack2(y[2] * f, y[3] * f), pack2(y[4] * f, y[5] * f), pack2(y[6] * f, y[7] * f)};
      }
    }
  };
  join(ak, p.scale, dk, 0);
  join(av, 1.f, dv, 1);
}

// More than 64 KB of dynamic LDS need an opt-in, once per kernel and device.
template <typename K>
void allow_lds(std::atomic<uint64_t>& done, K kernel, int bytes) {
  int dev = 0;
  (void)hipGetDevice(&dev);
  const uint64_t bit = 1ull << (dev & 63);
  if (done.load(std::memory_order_acquire) & bit) return;
  (void)hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  done.fetch_or(bit, std::memory_order_release);
}

// Keys of a workgroup of dk and dv.  128 (each tile of queries read by four waves, three stages) where there are workgroups enough for that,
// 64 otherwise.  Measured, backward alone, 128 and 64 keys, 16 heads over 8 KV heads of 128: one sequence of 4096 320 and 274 us, of 5000 405
// and 389, of 6000 521 and 521, of 7000 643 and 672, of 8192 833 and 880; 2 of 4096 441 and 473; 4 of 3000 507 and 531, of 4096 875 and 945;
// forward and backward: 4 of 2048 691 and 649; 32 of 1024 1568 and 1608; 16 of 97 to 1511 353 and 333.  The sides cross below both of the
// rule's bounds, at n = 375 for one sequence and between 512 and 750 for four; between there and the bounds it gives away up to 5 %.
bool many_keys(const PackedShape& p) {
  const int64_t n = (int64_t)p.total_k * p.nkv / 128;
  return n >= 1024 || (n >= 512 && p.n_seq <= 2);
}

template <int D>
void forward(hipStream_t s, const PackedShape& p, const bf16_t* q, const bf16_t* k, const bf16_t* v, bf16_t* o, float* lse) {
  static std::atomic<uint64_t> done;
  const int lds = 5 * BN * D * 2;
  allow_lds(done, attention_forward_kernel<D>, lds);
  attention_forward_kernel<D><<<(unsigned)(packed_tiles(p.total_q, p.n_seq, BM) * p.nq), 256, lds, s>>>(p, q, k, v, o, lse);
}
template <int D>
void backward(hipStream_t s, const PackedShape& p, const bf16_t* dout, const bf16_t* q, const bf16_t* k, const bf16_t* v, const bf16_t* o,
              const float* lse, bf16_t* dq, bf16_t* dk, bf16_t* dv, float* stats, const KeyParts& parts) {
  static std::atomic<uint64_t> done[3];
  const int lds = 4 * BN * D * 2;
  if (p.total_q > 0) {
    allow_lds(done[0], attention_dq_kernel<D>, lds);
    attention_dq_kernel<D><<<(unsigned)(packed_tiles(p.total_q, p.n_seq, BM) * p.nq), 256, lds, s>>>(p, dout, q, k, v, o, lse, dq, stats);
  }
  if (p.total_k > 0) {
    auto go = [&](auto blocks, auto stages) {
      constexpr int BLOCKS = decltype(blocks)::value, R = decltype(stages)::value, STREAMS = 8 / BLOCKS, KEYS = 32 * BLOCKS;
      constexpr int ring = STREAMS * R * (2 * 32 * D * 2 + 512) + KEYS * D * 2, sums = STREAMS * KEYS * (D + 4) * 4, bytes = ring > sums ? ring : sums;
      auto kernel = attention_dkv_kernel<D, BLOCKS, R>;
      allow_lds(done[BLOCKS / 2], kernel, bytes);
      kernel<<<dim3(packed_tiles(p.total_k, p.n_seq, KEYS) * p.nkv, parts.n), 512, bytes, s>>>(p, dout, q, k, v, stats, dk, dv, parts);
    };
    if (many_keys(p)) go(std::integral_constant<int, 4>(), std::integral_constant<int, 3>());
    else go(std::integral_constant<int, 2>(), std::integral_constant<int, D == 128 ? 2 : 3>());
  }
}

}  // namespace

bool attention_takes_mfma(const PackedShape& p, const void* q, const void* k, const void* v, const void* o, const void* dout) {
  // a sequence's rows behind one descriptor with 32-bit offsets; rows that do not overlap, so that the descriptor's end is the
  // last row's; 16-byte pieces
  const int64_t most = (1ll << 31) - (1 << 20);
  auto takes = [&](const void* x, int64_t ts, int64_t hs, int total) {
    return aligned16(x) && ts % 8 == 0 && hs % 8 == 0 && ts >= p.d && ts * 2 * ((int64_t)total + 2 * BN) < most;
  };
  // the backward pass divides by the scale
  return fabsf(p.scale) > 1e-30f && p.d % 8 == 0 && takes(q, p.qt, p.qh, p.total_q) && takes(k, p.kt, p.kh, p.total_k) && takes(v, p.vt, p.vh, p.total_k) &&
         takes(o, p.ot, p.oh, p.total_q) && takes(dout, p.ot, p.oh, p.total_q) && (int64_t)packed_tiles(p.total_q, p.n_seq, BM) * p.nq <= most_workgroups(256) &&
         (int64_t)packed_tiles(p.total_k, p.n_seq, 64) * p.nkv <= most_workgroups(512);
}

void launch_attention_mfma_forward(hipStream_t s, const PackedShape& p, const bf16_t* q, const bf16_t* k, const bf16_t* v, bf16_t* o,
                                   float* lse) {
  if (p.d <= 64) forward<64>(s, p, q, k, v, o, lse);
  else forward<128>(s, p, q, k, v, o, lse);
}
void launch_attention_mfma_backward(hipStream_t s, const PackedShape& p, const bf16_t* dout, const bf16_t* q, const bf16_t* k,
                                    const bf16_t* v, const bf16_t* o, const float* lse, bf16_t* dq, bf16_t* dk, bf16_t* dv,
                                    float* stats, const KeyParts& parts) {
  if (p.d <= 64) backward<64>(s, p, dout, q, k, v, o, lse, dq, dk, dv, stats, parts);
  else backward<128>(s, p, dout, q, k, v, o, lse, dq, dk, dv, stats, parts);
}
