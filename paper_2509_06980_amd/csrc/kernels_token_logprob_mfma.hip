// The products of the token log-probs and of their gradient in bf16 on matrix instructions.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "lds_load.h"
#include "token_logprob.h"

namespace {

// =============================================================================================
// One kernel for the four products, C[i, j] = sum_k A[i, k] B[j, k] over tiles of 64 MB rows i and 256 columns j, four waves of
// 32 MB x 128 on 32x32x16 matrix instructions:
//   logits          A = hidden rows            B = weights                epilogue: (max, sum) of a row's 256 logits, or dz
//   dz W            A = dz                     B = weights, k-strided     epilogue: a slice's sum in 32 bits
//   dz^T hidden     A = dz, k-strided          B = rows, k-strided        epilogue: bf16
// Bound by the matrix units (2 flops x rows x hidden x vocab each, 2.5 PFLOP/s peak, held by power below 1.5 for random data), for few
// rows by the weights' bytes.  A chunk of 32 k of both operands goes straight from memory into one of R stages in LDS, R - 1 ahead;
// operands are read 16 k ahead of the instructions that use them, one barrier a chunk.
// Operands as they lie in memory, no copy of the weights in another order:
//   k-contiguous: [row][32 k], 64 bytes a row.  The 16-byte piece p of row r is kept at p ^ (r / 4 % 4), so the 16 rows that a
//     read takes in one go lie in different banks.
//   k-strided (TA, TB): [32 k][256 columns], 512 bytes a k, read with the transposing LDS read: 16 lanes take 4 k x 16 columns, lane i
//     gets column i of the 4 k.  The 64-byte block b of row k is kept at b ^ (k % 4): the 4 k of a read lie in different banks.
// =============================================================================================
constexpr int BN = 256;      // columns of a tile
enum { EPI_STRIP, EPI_DZ, EPI_SLICE, EPI_OUT };

typedef __attribute__((address_space(3))) char lds_char;

struct Product {
  const bf16_t *a, *b;
  int64_t lda, ldb;
  int a_n, b_n;                  // rows of a, b in memory (k-strided: k that may be read)
  int tiles_i, tiles_j;          // tiles_i: upper bound where the count of kept rows decides
  int k, slices;                 // k = 0: the kept rows; slices: of k, upper bound
  int group;                     // row tiles that an XCD takes together
  KeptRows kept;
  // logits
  int vocab, v0;                 // v0: first token of the piece
  float scale, inv_t;            // log2(e) / T, 1 / T
  float2* part;
  int padded;
  float* zt;
  // results
  bf16_t* out;
  float* slice;
  size_t slice_stride;
  int64_t ldo;
  int out_rows, out_cols, first;
};

template <bool TA, bool TB, int MB, int R, int EPI>
__global__ __launch_bounds__(256, 1) void product_kernel(Product P) {
  constexpr bool SWAP = EPI != EPI_SLICE;        // a lane holds one row's values, else one column's
  constexpr int NA = 4 * MB, PW = MB + 4, BUF = (NA + 16) * 1024, F = PW / 2;
  static_assert(!TA || MB == 4, "a k-strided A has 256 columns");
  extern __shared__ u32x4 smem[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, wm = wave >> 1, wn = wave & 1;
  const int kept = __builtin_amdgcn_readfirstlane(*P.kept.count);
  // tiles that have work, numbered so that an XCD (workgroups are dealt to the 8 of them in turn) takes a compact block of one slice
  const int ti = EPI == EPI_OUT ? P.tiles_i : min(P.tiles_i, (kept + 64 * MB - 1) / (64 * MB)), tiles = ti * P.tiles_j;
  const int slices = EPI == EPI_SLICE ? __builtin_amdgcn_readfirstlane(P.kept.count[1]) : 1, total = tiles * slices;
  if ((int)blockIdx.x >= total) return;
  int i0, j0, z;
  {
    const int base = total >> 3, rem = total & 7, x = blockIdx.x & 7, vid = x * base + min(x, rem) + ((int)blockIdx.x >> 3);
    z = vid / tiles;
    const int v = vid - z * tiles, per = P.group * P.tiles_j, grp = v / per, first = grp * P.group, gm = min(P.group, ti - first), in = v - grp * per;
    // the divisions leave them in vector registers
    i0 = __builtin_amdgcn_readfirstlane(first + in % gm) * 64 * MB;
    j0 = __builtin_amdgcn_readfirstlane(in / gm) * BN;
    z = __builtin_amdgcn_readfirstlane(z);
  }
  const int k_all = EPI == EPI_OUT ? kept : P.k, per_slice = EPI == EPI_SLICE ? __builtin_amdgcn_readfirstlane(P.kept.count[2]) : k_all;
  const int k_lo = z * per_slice, c0 = k_lo >> 5, c1 = (min(k_all, k_lo + per_slice) + 31) >> 5;
  // operands behind these descriptors: what is read past their end arrives as zeros
  const u32x4 ra = TA ? buffer_rsrc(P.a + i0, (unsigned)(((int64_t)P.a_n * P.lda - i0) * 2))
                      : buffer_rsrc(P.a + (int64_t)i0 * P.lda, (unsigned)((int64_t)min(P.a_n - i0, 64 * MB) * P.lda * 2));
  const u32x4 rb = TB ? buffer_rsrc(P.b + j0, (unsigned)(((int64_t)P.b_n * P.ldb - j0) * 2))
                      : buffer_rsrc(P.b + (int64_t)j0 * P.ldb, (unsigned)((int64_t)min(P.b_n - j0, BN) * P.ldb * 2));
  const unsigned sa = TA ? (unsigned)P.lda * 64u : 64u, sb = TB ? (unsigned)P.ldb * 64u : 64u;      // bytes of a chunk's step
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
  int va[MB], vb[4];      // this lane's offset of each piece that its wave loads
  auto offset = [&](int piece, int64_t ld, bool strided) {
    const int n = piece * 4 + wave;
    if (strided) {
      const int k = n * 2 + (lane >> 5);
      return (int)(k * ld * 2) + ((((lane & 31) >> 2) ^ (k & 3)) << 6) + ((lane & 3) << 4);
    }
    return (int)((n * 16 + (lane >> 2)) * ld * 2) + (((lane & 3) ^ (lane >> 4 & 3)) << 4);
  };
#pragma unroll
  for (int j = 0; j < MB; j++) va[j] = offset(j, P.lda, TA);
#pragma unroll
  for (int j = 0; j < 4; j++) vb[j] = offset(j, P.ldb, TB);
  // piece j of this wave of a chunk; chunks behind the slice's end: the last one again, never read
  auto load = [&](int chunk, int j, int stage) {
    const unsigned dst = lds0 + (unsigned)stage * BUF + (unsigned)(j * 4 + wave) * 1024u, c = (unsigned)min(chunk, c1 - 1);
    if (j < MB) load_to_lds(dst, va[j], ra, c * sa);
    else load_to_lds(dst, vb[j - MB], rb, c * sb);
  };
  f32x16 acc[MB][4];
#pragma unroll
  for (int a = 0; a < MB; a++)
#pragma unroll
    for (int b = 0; b < 4; b++)
#pragma unroll
      for (int e = 0; e < 16; e++) acc[a][b][e] = 0.f;
  auto mfma = [&](const u32x4& row, const u32x4& col, f32x16& c) {
    c = SWAP ? __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, col), __builtin_bit_cast(bf16x8, row), c, 0, 0, 0)
             : __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, row), __builtin_bit_cast(bf16x8, col), c, 0, 0, 0);
  };
  // lane parts of the operand reads: k-contiguous by 16-k half, k-strided by 32-column block
  int la[TA ? 4 : 2], lb[TB ? 4 : 2];
  auto part = [&](int (&l)[4]) {
    const int s = lane >> 2 & 3;
#pragma unroll
    for (int x = 0; x < 4; x++) l[x] = ((lane >> 5) * 8 + s) * 512 + ((x ^ s) << 6) + ((lane >> 4 & 1) << 5) + ((lane & 3) << 3);
  };
  auto part2 = [&](int (&l)[2]) {
#pragma unroll
    for (int x = 0; x < 2; x++) l[x] = (lane & 31) * 64 + (((x * 2 + (lane >> 5)) ^ (lane >> 2 & 3)) << 4);
  };
  if constexpr (TA) part(la);
  else part2(la);
  if constexpr (TB) part(lb);
  else part2(lb);
  lds_char* const lds = (lds_char*)(__attribute__((address_space(3))) void*)smem;
  auto strided = [&](int at) {
    typedef __attribute__((address_space(3))) s16x4 l4;
    const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((l4*)(lds + at)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((l4*)(lds + at + 2048));
    return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  };
  auto read_a = [&](int x, int kb, int stage) {
    const int base = stage * BUF;
    if constexpr (TA) return strided(base + kb * 8192 + wm * 256 + la[x]);
    else return *(__attribute__((address_space(3))) u32x4*)(lds + base + (wm * MB + x) * 2048 + la[kb]);
  };
  auto read_b = [&](int x, int kb, int stage) {
    const int base = stage * BUF + NA * 1024;
    if constexpr (TB) return strided(base + kb * 8192 + wn * 256 + lb[x]);
    else return *(__attribute__((address_space(3))) u32x4*)(lds + base + (wn * 4 + x) * 2048 + lb[kb]);
  };
  if (c1 > c0) {
    u32x4 av[2][MB], bv[2][4];
#pragma unroll
    for (int c = 0; c < R - 1; c++)
#pragma unroll
      for (int j = 0; j < PW; j++) load(c0 + c, j, c);
#pragma unroll
    for (int j = 0; j < F; j++) load(c0 + R - 1, j, R - 1);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((R - 2) * PW + F) : "memory");
    __builtin_amdgcn_s_barrier();
#pragma unroll
    for (int x = 0; x < MB; x++) av[0][x] = read_a(x, 0, 0);
#pragma unroll
    for (int x = 0; x < 4; x++) bv[0][x] = read_b(x, 0, 0);
    int sc = 0, sl = R - 1;                  // stages of chunks c and c + R - 1 (that of chunk c - 1)
    for (int c = c0; c < c1; c++) {
      const int sn = sc + 1 == R ? 0 : sc + 1;
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int g = 0; g < 2 * MB; g++) {
        const int a = g % MB, st = g / MB;
        if (g == MB) {     // chunk c + 1 has landed for every wave, chunk c is read out by every wave
          asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((R - 2) * PW) : "memory");
          __builtin_amdgcn_s_barrier();
        }
        const int stage = st == 0 ? sc : sn, kb = 1 - st;
        // the operands of the next 16 k, in the order of their use
        constexpr int order[8] = {0, MB, MB + 1, MB + 2, MB + 3, 1, 2, 3};
#pragma unroll
        for (int q = 0; q < MB + 4; q++)
          if (q * MB / (MB + 4) == a) {
            const int x = order[q];
            if (x < MB) av[1 - st][x] = read_a(x, kb, stage);
            else bv[1 - st][x - MB] = read_b(x - MB, kb, stage);
          }
        // this step's share of the loads: the rest of chunk c + R - 1, then the first F pieces of chunk c + R
#pragma unroll
        for (int j = 0; j < PW; j++) {
          if (st == 0 && j >= F && (j - F) * MB / (PW - F) == a) load(c + R - 1, j, sl);
          if (st == 1 && j < F && j * MB / F == a) load(c + R, j, sc);
        }
#pragma unroll
        for (int b = 0; b < 4; b++) mfma(av[st][a], bv[st][b], acc[a][b]);
        __builtin_amdgcn_sched_barrier(0);
      }
      sl = sc;
      sc = sn;
    }
  }
  // all loads into LDS are done; results of the last instructions may be read by the assembly below
  asm volatile("s_waitcnt vmcnt(0)\n\ts_nop 15\n\ts_nop 15" ::: "memory");
  __syncthreads();                                      // and nobody reads the stages any more

  // one element of a result: read as a whole, the 16 registers of an accumulator would be copied and spill
  auto val = [&](int a, int b, int e) {
    if (MB == 2) return acc[a][b][e];
    float x;
    asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(acc[a][b][e]));
    return x;
  };
  if constexpr (EPI == EPI_SLICE) {
    float* const out = P.slice + z * P.slice_stride + (int64_t)i0 * P.ldo + j0;      // offsets inside a tile fit 32 bits
    const unsigned ld = (unsigned)P.ldo;
#pragma unroll
    for (int a = 0; a < MB; a++) {
#pragma unroll
      for (int b = 0; b < 4; b++) {
        const int j = wn * 128 + b * 32 + (lane & 31), r = (wm * MB + a) * 32 + 4 * (lane >> 5);
        if (j0 + j < P.out_cols) {
          const unsigned at = (unsigned)r * ld + j;
#pragma unroll
          for (int e = 0; e < 16; e++) {
            const int d = 8 * (e >> 2) + (e & 3);
            if (i0 + r + d >= kept) continue;
            float* p = out + (at + (unsigned)d * ld);
            __builtin_nontemporal_store(P.first ? val(a, b, e) : *p + val(a, b, e), p);
          }
        }
        __builtin_amdgcn_sched_barrier(0);      // one block's addresses at a time
      }
    }
    return;
  }
  const int jw = wn * 128 + 4 * (lane >> 5);      // column of register e of block b: jw + 32 b + 8 (e / 4) + e % 4
  const bool crosses = (EPI == EPI_STRIP || EPI == EPI_DZ) && P.v0 + j0 + BN > P.vocab;
  if constexpr (EPI == EPI_STRIP) {
    float2* half = (float2*)smem;
#pragma unroll
    for (int a = 0; a < MB; a++) {
      const int il = (wm * MB + a) * 32 + (lane & 31), i = i0 + il, y = i < kept ? P.kept.target[i] - j0 : -1;
      float top = -INFINITY, sum = 0.f;
      auto strip = [&](auto some) {      // some: a target or the vocabulary's end is in the tile
        auto at = [&](int b, int e) {
          const int j = jw + 32 * b + 8 * (e >> 2) + (e & 3);
          const float v = val(a, b, e);
          return decltype(some)::value && j0 + j >= P.vocab ? -INFINITY : v;
        };
#pragma unroll
        for (int b = 0; b < 4; b++)
#pragma unroll
          for (int e = 0; e < 16; e++) {
            const float v = at(b, e);
            if (decltype(some)::value && jw + 32 * b + 8 * (e >> 2) + (e & 3) == y) P.zt[i] = v * P.inv_t;
            top = fmaxf(top, v);
          }
        top = fmaxf(top, __shfl_xor(top, 32, 64));
        const float ref = top == -INFINITY ? 0.f : top * P.scale;
#pragma unroll
        for (int b = 0; b < 4; b++)
#pragma unroll
          for (int e = 0; e < 16; e++) sum += __builtin_amdgcn_exp2f(fmaf(at(b, e), P.scale, -ref));
        sum += __shfl_xor(sum, 32, 64);
      };
      if (crosses || __any(y >= 0 && y < BN)) strip(std::true_type());
      else strip(std::false_type());
      if (lane < 32) half[wn * 64 * MB + il] = make_float2(top, sum);
      __builtin_amdgcn_sched_barrier(0);      // one row block at a time
    }
    __syncthreads();
    if (tid < 64 * MB && i0 + tid < kept) {
      const float2 a = half[tid], b = half[64 * MB + tid];
      const float top = fmaxf(a.x, b.x), ref = top == -INFINITY ? 0.f : top;
      P.part[(size_t)(j0 / BN) * P.padded + i0 + tid] =
          make_float2(top * P.inv_t, a.y * exp2f((a.x - ref) * P.scale) + b.y * exp2f((b.x - ref) * P.scale));
    }
    return;
  }
  // bf16 tile through LDS: rows of 512 bytes, 16 apart
  constexpr int PITCH = BN * 2 + 16;
#pragma unroll
  for (int a = 0; a < MB; a++) {
    const int il = (wm * MB + a) * 32 + (lane & 31);
    if constexpr (EPI == EPI_DZ) {
      const int i = i0 + il, y = P.kept.target[i] - P.v0 - j0;
      const float g = P.kept.g[i], l = P.kept.lse[i] * 1.44269504f;
#pragma unroll
      for (int b = 0; b < 4; b++)
#pragma unroll
        for (int e = 0; e < 16; e++) acc[a][b][e] = -g * __builtin_amdgcn_exp2f(fmaf(acc[a][b][e], P.scale, -l));
      if (crosses || __any(y >= 0 && y < BN)) {
#pragma unroll
        for (int b = 0; b < 4; b++)
#pragma unroll
          for (int e = 0; e < 16; e++) {
            const int j = jw + 32 * b + 8 * (e >> 2) + (e & 3);
            if (j == y) acc[a][b][e] += g;
            if (P.v0 + j0 + j >= P.vocab) acc[a][b][e] = 0.f;
          }
      }
    }
    auto out = [&](int b, int e) { return EPI == EPI_DZ ? acc[a][b][e] : val(a, b, e); };
#pragma unroll
    for (int b = 0; b < 4; b++)
#pragma unroll
      for (int q = 0; q < 4; q++) {
        typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4;
        const bf16x4 w = {(__bf16)out(b, 4 * q), (__bf16)out(b, 4 * q + 1), (__bf16)out(b, 4 * q + 2), (__bf16)out(b, 4 * q + 3)};
        *(__attribute__((address_space(3))) bf16x4*)(lds + il * PITCH + (jw + 32 * b + 8 * q) * 2) = w;
        if (q == 3) __builtin_amdgcn_sched_barrier(0);
      }
  }
  __syncthreads();
  const int c = (tid & 31) * 8;
  if (j0 + c < P.out_cols) {
#pragma unroll 4
    for (int r = tid >> 5; r < 64 * MB; r += 8) {
      if (i0 + r >= P.out_rows) break;
      const u32x4 v = *(__attribute__((address_space(3))) u32x4*)(lds + r * PITCH + c * 2);
      __builtin_nontemporal_store(v, (u32x4*)(P.out + (int64_t)(i0 + r) * P.ldo + j0 + c));
    }
  }
}

template <bool TA, bool TB, int MB, int R, int EPI>
void go(const Product& p, hipStream_t s) {
  constexpr int ring = R * (4 * MB + 16) * 1024, tile = 64 * MB * (BN * 2 + 16);
  constexpr int lds = EPI != EPI_SLICE && tile > ring ? tile : ring;
  static std::atomic<uint64_t> done;      // more than 64 KB of LDS need an opt-in, once per kernel and device
  int dev = 0;
  (void)hipGetDevice(&dev);
  const uint64_t bit = 1ull << (dev & 63);
  if (!(done.load(std::memory_order_acquire) & bit)) {
    (void)hipFuncSetAttribute((const void*)product_kernel<TA, TB, MB, R, EPI>, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    done.fetch_or(bit, std::memory_order_release);
  }
  product_kernel<TA, TB, MB, R, EPI><<<(unsigned)(p.tiles_i * p.tiles_j * p.slices), 256, lds, s>>>(p);
}

// rows of up to 128 take tiles of 128
int row_blocks(int rows) { return rows <= 128 ? 2 : 4; }

}  // namespace

bool token_logprob_takes_mfma(int64_t padded, int ld, int hidden, int width, const void* weight, const void* dweight) {
  // 32-bit offsets into one descriptor: the rows as k-strided operand, dz, a piece of the weights
  const int64_t most = (1ll << 32) - (1 << 20);
  return hidden % 8 == 0 && aligned16(weight) && aligned16(dweight) && padded * ld * 2 < most && padded * width * 2 < most &&
         (int64_t)std::max(width, 256) * hidden * 2 < most / 2;
}

int token_logprob_tile_rows(int rows) { return 64 * row_blocks(rows); }

void launch_logits_strips_mfma(hipStream_t s, const bf16_t* h, int ld, int rows, int64_t padded, const bf16_t* w, int vocab, int hidden,
                               const KeptRows& kept, float inv_t, float2* part, float* zt) {
  Product p{};
  const int mb = row_blocks(rows);
  p.a = h, p.lda = ld, p.a_n = (int)padded;
  p.b = w, p.ldb = hidden, p.b_n = vocab;
  p.tiles_i = (rows + 64 * mb - 1) / (64 * mb), p.tiles_j = (vocab + BN - 1) / BN;
  p.k = (int)up(hidden, 32), p.slices = 1, p.group = 4;
  p.kept = kept, p.vocab = vocab, p.v0 = 0, p.scale = (float)(1.4426950408889634 * inv_t), p.inv_t = inv_t;
  p.part = part, p.padded = (int)padded, p.zt = zt;
  if (mb == 4) go<false, false, 4, 4, EPI_STRIP>(p, s);
  else go<false, false, 2, 6, EPI_STRIP>(p, s);
}

void launch_logits_gradient_mfma(hipStream_t s, const bf16_t* h, int ld, int rows, int64_t padded, const bf16_t* w, int vocab, int hidden,
                                 const KeptRows& kept, float inv_t, const VocabPiece& piece, bf16_t* dz) {
  Product p{};
  const int mb = row_blocks(rows);
  p.a = h, p.lda = ld, p.a_n = (int)padded;
  p.b = w + (int64_t)piece.v0 * hidden, p.ldb = hidden, p.b_n = vocab - piece.v0;
  p.tiles_i = (rows + 64 * mb - 1) / (64 * mb), p.tiles_j = (piece.width + BN - 1) / BN;
  p.k = (int)up(hidden, 32), p.slices = 1, p.group = 4;
  p.kept = kept, p.vocab = vocab, p.v0 = piece.v0, p.scale = (float)(1.4426950408889634 * inv_t), p.inv_t = inv_t;
  p.out = dz, p.ldo = piece.ld, p.out_rows = (int)padded, p.out_cols = (int)up(piece.width, BN);
  if (mb == 4) go<false, false, 4, 4, EPI_DZ>(p, s);
  else go<false, false, 2, 6, EPI_DZ>(p, s);
}

void launch_hidden_gradient_mfma(hipStream_t s, const bf16_t* dz, const VocabPiece& piece, int rows, int64_t padded, const bf16_t* w, int vocab,
                                 int hidden, const KeptRows& kept, int most_slices, float* dh, size_t slice_stride, bool first) {
  Product p{};
  const int mb = row_blocks(rows);
  p.a = dz, p.lda = piece.ld, p.a_n = (int)padded;
  p.b = w + (int64_t)piece.v0 * hidden, p.ldb = hidden, p.b_n = std::min(piece.ld, vocab - piece.v0);
  p.tiles_i = (rows + 64 * mb - 1) / (64 * mb), p.tiles_j = (hidden + BN - 1) / BN;
  p.k = piece.width, p.slices = most_slices, p.group = 4;
  p.kept = kept, p.slice = dh, p.slice_stride = slice_stride, p.ldo = hidden, p.out_cols = hidden, p.first = first;
  if (mb == 4) go<false, true, 4, 4, EPI_SLICE>(p, s);
  else go<false, true, 2, 6, EPI_SLICE>(p, s);
}

void launch_weight_gradient_mfma(hipStream_t s, const bf16_t* dz, const VocabPiece& piece, const bf16_t* h, int ld, int64_t padded, int hidden,
                                 const KeptRows& kept, bf16_t* dw) {
  Product p{};
  p.a = dz, p.lda = piece.ld, p.a_n = (int)padded;
  p.b = h, p.ldb = ld, p.b_n = (int)padded;
  p.tiles_i = (piece.width + 255) / 256, p.tiles_j = (hidden + BN - 1) / BN;
  p.k = 0, p.slices = 1, p.group = 4;
  p.kept = kept, p.out = dw + (int64_t)piece.v0 * hidden, p.ldo = hidden, p.out_rows = piece.width, p.out_cols = hidden;
  go<true, true, 4, 4, EPI_OUT>(p, s);
}
