// The products of the token log-probs and of their gradient on matrix instructions, operands straight from memory into LDS.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "lds_load.h"
#include "token_logprob.h"

namespace {

// =============================================================================================
// One kernel for the four products, C[i, j] = sum_k A[i, k] B[j, k] over tiles of 64 MB rows i and 64 NB columns j, four waves of
// 32 MB x 32 NB on 32x32x16 (fp32: 32x32x2) matrix instructions:
//   logits          A = hidden rows            B = weights                epilogue: (max, sum) of a tile's logits of a row, or dz
//   dz W            A = dz                     B = weights, k-strided     epilogue: a slice's sum in 32 bits
//   dz^T hidden     A = dz, k-strided          B = rows, k-strided        epilogue: rounded
// dz is rounded to the weights' type once, as the operand that it becomes; all sums are kept in 32 bits.
// Bound by the matrix units (2 flops x rows x hidden x vocab each; busy 60 to 63 % of the cycles) at the clock that the data leaves them, 1.71 to
// 1.77 GHz: of 2.5 PFLOP/s at the full clock a large library product of random data reaches 1.47, and operands of zeros run these 1.2 times as
// fast.  For few rows by the weights' bytes; fp32: 155 TFLOP/s.
// Measured in bf16 on two GPUs, 2744 rows x 2560 x 151936: logits 1.79 and 1.85 ms (1.19 and 1.15 PFLOP/s), dz 1.95 and 2.00 in two pieces,
// dz W 1.78 and 1.83 (1.20, 1.17), dz^T hidden 1.80 and 1.86 (1.19, 1.15); 4096 x 1024 x 151936, logits 1.20 and 1.23 ms (1.06, 1.04).
// A chunk of 64 bytes of k (32; fp32 16) of both operands goes straight from memory into one of R stages in LDS, R - 1 ahead;
// operands are read half a chunk ahead of the instructions that use them, one barrier a chunk.  A workgroup stays for all its tiles
// and its loads run on into the next one, so a tile ends with its epilogue alone (without that, the last-named logits 1.35 ms).
// 256 x 256 tiles with one wave a SIMD: a wave of 128 x 128 reads least from LDS for its flops; 128 x 256 with two workgroups a CU, whose
// epilogues overlap with the other's products, is slower for what it fetches (logits of 2744 rows 2.35 ms against 1.93 then).
// Operands as they lie in memory, no copy of the weights in another order:
//   k-contiguous: [row][32 k], 64 bytes a row.  The 16-byte piece p of row r is kept at p ^ (r / 4 % 4), so the 16 rows that a
//     read takes in one go lie in different banks.
//   k-strided (TA, TB): [k][columns].  bf16: read with the transposing LDS read, 16 lanes take 4 k x 16 columns, lane i gets column i of
//     the 4 k.  The 64-byte block b of row k is kept at b ^ (k % 4): the 4 k of a read lie in different banks.  fp32: read one by one, two
//     blocks of row k and two of row k + 4 at once, which are kept at b ^ 2 (k / 4 % 2).
// fp32 instructions take 2 k, of a lane's 16 bytes element e in step e: k = e and 4 + e of the eight, the same for both operands.
// =============================================================================================
enum { EPI_STRIP, EPI_DZ, EPI_SLICE, EPI_OUT };

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;

template <typename T>
struct Product {
  const T *a, *b;
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
  T* out;
  float* slice;
  size_t slice_stride;
  int64_t ldo;
  int out_rows, out_cols, first;
};

// What a tile's loads of one operand may reach, from element `begin` on: its rows (k-contiguous), or all of the operand behind its
// first column (k-strided).  Scalar offsets have to stay inside: the hardware compares a lane's offset with the size less the scalar one.
struct Reach {
  int64_t begin;
  unsigned bytes;
};
// The operand has n rows of ld elements, the tile begins at row (k-strided: column) `at` and has `rows` of them.  A tile of dz may begin behind
// the vocabulary (its columns go on to a multiple of 256): it reads the last row, and stores zeros.
template <typename T>
__host__ __device__ __forceinline__ Reach reach_of(bool strided, int64_t ld, int n, int at, int rows) {
  if (strided) return {at, (unsigned)((n * ld - at) * (int64_t)sizeof(T))};
  const int first = at < n ? at : n - 1, left = n - first;
  return {first * ld, (unsigned)((left < rows ? left : rows) * ld * (int64_t)sizeof(T))};
}
// Scalar offset of chunk c: that many times a chunk's step
__host__ __device__ __forceinline__ unsigned chunk_step(bool strided, int64_t ld) { return strided ? (unsigned)ld * 64u : 64u; }
// Chunks [first, end) of a slice of k
template <typename T>
__host__ __device__ __forceinline__ void chunks_of(int slice, int per_slice, int k_all, int& first, int& end) {
  constexpr int KC = 64 / sizeof(T);
  const int lo = slice * per_slice, hi = k_all < lo + per_slice ? k_all : lo + per_slice;
  first = lo / KC, end = (hi + KC - 1) / KC;
}

// LDS of a workgroup: the ring of stages, behind it what an epilogue takes, so that it does not touch the next tile's chunks
template <typename T, int MB, int NB, int R, int EPI>
struct Lds {
  static constexpr int RING = R * (MB + NB) * 4096;
  static constexpr int ROWS = (MB + 1) / 2, ARRAYS = EPI == EPI_STRIP ? 1 : EPI == EPI_DZ ? 3 : 0;      // of 256 bytes a wave: target; g, lse
  static constexpr int ROW_DATA = 4 * ARRAYS * ROWS * 256;
  static constexpr int SC = sizeof(T) == 2 ? 64 : 16, PITCH = SC * sizeof(T) + 16;                      // columns stored at a time
  static constexpr int BYTES = RING + ROW_DATA + (EPI == EPI_STRIP ? 2 * 64 * MB * 8 : EPI == EPI_SLICE ? 0 : 4 * 32 * PITCH);
};
template <typename T, bool TA, bool TB, int MB, int NB, int R, int EPI>
__global__ __launch_bounds__(256, MB * NB > 4 ? 1 : 2) void product_kernel(Product<T> P) {
  constexpr bool SWAP = EPI != EPI_SLICE;        // a lane holds one row's values, else one column's
  constexpr int BM = 64 * MB, BN = 64 * NB, EL = sizeof(T), KC = 64 / EL, V = 16 / EL;
  constexpr int NA = 4 * MB, PW = MB + NB, BUF = (NA + 4 * NB) * 1024, F = PW / 2;
  static_assert((!TA || BM * EL >= 256) && (!TB || BN * EL >= 256), "four blocks of 64 bytes a row");
  using L = Lds<T, MB, NB, R, EPI>;
  constexpr int RING = L::RING, ROWS = L::ROWS, ARRAYS = L::ARRAYS, ROW_DATA = L::ROW_DATA, SC = L::SC, PITCH = L::PITCH;
  extern __shared__ u32x4 smem[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, wm = wave >> 1, wn = wave & 1;
  const int kept = __builtin_amdgcn_readfirstlane(*P.kept.count);
  // tiles that have work, numbered so that an XCD (workgroups are dealt to the 8 of them in turn) takes a compact block of one slice
  const int ti = EPI == EPI_OUT ? P.tiles_i : min(P.tiles_i, (kept + BM - 1) / BM), tiles = ti * P.tiles_j;
  const int slices = EPI == EPI_SLICE ? __builtin_amdgcn_readfirstlane(P.kept.count[1]) : 1, total = tiles * slices;
  if ((int)blockIdx.x >= total) return;
  const int k_all = EPI == EPI_OUT ? kept : P.k, per_slice = EPI == EPI_SLICE ? __builtin_amdgcn_readfirstlane(P.kept.count[2]) : k_all;
  struct Place {
    int i0, j0, z, c0, c1;      // first row and column, slice, its chunks of k
  };
  auto place = [&](int id) {
    const int base = total >> 3, rem = total & 7, x = id & 7, vid = x * base + min(x, rem) + (id >> 3), slice = vid / tiles;
    const int v = vid - slice * tiles, per = P.group * P.tiles_j, grp = v / per, first = grp * P.group, gm = min(P.group, ti - first), in = v - grp * per;
    Place t;      // the divisions leave these in vector registers
    t.i0 = __builtin_amdgcn_readfirstlane(first + in % gm) * BM;
    t.j0 = __builtin_amdgcn_readfirstlane(in / gm) * BN;
    t.z = __builtin_amdgcn_readfirstlane(slice);
    chunks_of<T>(t.z, per_slice, k_all, t.c0, t.c1);
    return t;
  };
  const unsigned sa = chunk_step(TA, P.lda), sb = chunk_step(TB, P.ldb);
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
  int va[MB], vb[NB];      // this lane's offset of each piece that its wave loads
  auto offset = [&](int piece, int64_t ld, bool strided, int row_bytes) {
    const int n = piece * 4 + wave;
    if (strided) {
      const int lanes = row_bytes / 16, k = n * (64 / lanes) + lane / lanes, p = lane % lanes;
      const int block = (p >> 2) ^ (EL == 2 ? k & 3 : (k >> 2 & 1) << 1);
      return (int)(k * ld * EL) + (block << 6) + ((p & 3) << 4);
    }
    return (int)((n * 16 + (lane >> 2)) * ld * EL) + (((lane & 3) ^ (lane >> 4 & 3)) << 4);
  };
#pragma unroll
  for (int j = 0; j < MB; j++) va[j] = offset(j, P.lda, TA, BM * EL);
#pragma unroll
  for (int j = 0; j < NB; j++) vb[j] = offset(j, P.ldb, TB, BN * EL);
  // The loads run R - 1 chunks ahead of the products, from one tile of the workgroup into the next: tile `at`, its chunk c, operands
  // behind its descriptors (what is read past their end arrives as zeros).  Behind the last tile: its last chunk again, never read.
  u32x4 ra, rb;
  int at = (int)blockIdx.x - (int)gridDim.x, lc = 0, lend = 0;
  auto advance = [&]() {
    if (++lc < lend) return;
    for (at += gridDim.x; at < total; at += gridDim.x) {
      const Place t = place(at);
      if (t.c1 <= t.c0) continue;
      const Reach a = reach_of<T>(TA, P.lda, P.a_n, t.i0, BM), b = reach_of<T>(TB, P.ldb, P.b_n, t.j0, BN);
      ra = buffer_rsrc(P.a + a.begin, a.bytes);
      rb = buffer_rsrc(P.b + b.begin, b.bytes);
      lc = t.c0, lend = t.c1;
      settle(ra);
      settle(rb);
      return;
    }
    lc = lend - 1;
  };
  auto load = [&](int j, int stage) {      // piece j of this wave
    const unsigned dst = lds0 + (unsigned)stage * BUF + (unsigned)(j * 4 + wave) * 1024u;
    if (j < MB) load_to_lds(dst, va[j], ra, (unsigned)lc * sa);
    else load_to_lds(dst, vb[j - MB], rb, (unsigned)lc * sb);
  };
  f32x16 acc[MB][NB];
  auto mfma = [&](const u32x4& row, const u32x4& col, f32x16& c) {
    const u32x4 &x = SWAP ? col : row, &y = SWAP ? row : col;
    if constexpr (EL == 2) {
      c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, x), __builtin_bit_cast(bf16x8, y), c, 0, 0, 0);
    } else {
      const f32x4 u = __builtin_bit_cast(f32x4, x), w = __builtin_bit_cast(f32x4, y);
#pragma unroll
      for (int e = 0; e < 4; e++) c = __builtin_amdgcn_mfma_f32_32x32x2f32(u[e], w[e], c, 0, 0, 0);
    }
  };
  // lane parts of the operand reads: k-contiguous by half a chunk, k-strided by 32-column block
  int la[TA ? MB : 2], lb[TB ? NB : 2];
  auto part = [&](int x, int row_bytes) {
    if constexpr (EL == 2) {
      const int s = lane >> 2 & 3;
      return ((lane >> 5) * 8 + s) * row_bytes + ((x ^ s) << 6) + ((lane >> 4 & 1) << 5) + ((lane & 3) << 3);
    } else {
      return (lane >> 5) * 4 * row_bytes + (((2 * x) ^ (lane >> 5 << 1)) << 6) + ((lane & 31) << 2);
    }
  };
  auto part2 = [&](int x) { return (lane & 31) * 64 + (((x * 2 + (lane >> 5)) ^ (lane >> 2 & 3)) << 4); };
#pragma unroll
  for (int x = 0; x < (TA ? MB : 2); x++) la[x] = TA ? part(wm * MB + x, BM * EL) : part2(x);
#pragma unroll
  for (int x = 0; x < (TB ? NB : 2); x++) lb[x] = TB ? part(wn * NB + x, BN * EL) : part2(x);
  lds_char* const lds = (lds_char*)(__attribute__((address_space(3))) void*)smem;
  auto strided = [&](int at, auto row_bytes) {
    constexpr int RB = decltype(row_bytes)::value;
    if constexpr (EL == 2) {
      typedef __attribute__((address_space(3))) s16x4 l4;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((l4*)(lds + at)), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((l4*)(lds + at + 4 * RB));
      return __builtin_bit_cast(u32x4, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      u32x4 v;
#pragma unroll
      for (int e = 0; e < 4; e++) v[e] = *(__attribute__((address_space(3))) unsigned*)(lds + at + e * RB);
      return v;
    }
  };
  auto read_a = [&](int x, int kb, int stage) {
    const int base = stage * BUF;
    if constexpr (TA) return strided(base + kb * (KC / 2) * BM * EL + la[x], std::integral_constant<int, BM * EL>());
    else return *(__attribute__((address_space(3))) u32x4*)(lds + base + (wm * MB + x) * 2048 + la[kb]);
  };
  auto read_b = [&](int x, int kb, int stage) {
    const int base = stage * BUF + NA * 1024;
    if constexpr (TB) return strided(base + kb * (KC / 2) * BN * EL + lb[x], std::integral_constant<int, BN * EL>());
    else return *(__attribute__((address_space(3))) u32x4*)(lds + base + (wn * NB + x) * 2048 + lb[kb]);
  };
  advance();
  if (lend > 0) {
#pragma unroll 1
    for (int c = 0; c < R - 1; c++) {
#pragma unroll
      for (int j = 0; j < PW; j++) load(j, c);
      advance();
    }
#pragma unroll
    for (int j = 0; j < F; j++) load(j, R - 1);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((R - 2) * PW + F) : "memory");
    __builtin_amdgcn_s_barrier();
  }
  int sc = 0, sl = R - 1;                  // stages of chunks c and c + R - 1 (that of chunk c - 1)
  for (int id = blockIdx.x; id < total; id += gridDim.x) {
    const Place here = place(id);
    const int i0 = here.i0, j0 = here.j0, z = here.z;
    if constexpr (EPI == EPI_STRIP || EPI == EPI_DZ) {      // what the epilogue needs of the wave's rows
      auto fetch = [&](const void* p, int which) {
        const u32x4 r = buffer_rsrc(p, (unsigned)P.a_n * 4u);
#pragma unroll
        for (int m = 0; m < ROWS; m++)
          load_dword_to_lds(lds0 + RING + (unsigned)(wave * ARRAYS + which) * (ROWS * 256u) + m * 256u, lane * 4, r, (unsigned)(i0 + wm * 32 * MB + m * 64) * 4u);
      };
      fetch(P.kept.target, 0);
      if constexpr (EPI == EPI_DZ) {
        fetch(P.kept.g, 1);
        fetch(P.kept.lse, 2);
      }
    }
#pragma unroll
    for (int a = 0; a < MB; a++)
#pragma unroll
      for (int b = 0; b < NB; b++)
#pragma unroll
        for (int e = 0; e < 16; e++) acc[a][b][e] = 0.f;
    if (here.c1 > here.c0) {      // its first chunk has landed for every wave
      u32x4 av[2][MB], bv[2][NB];
#pragma unroll
      for (int x = 0; x < MB; x++) av[0][x] = read_a(x, 0, sc);
#pragma unroll
      for (int x = 0; x < NB; x++) bv[0][x] = read_b(x, 0, sc);
      for (int c = here.c0; c < here.c1; c++) {
        const int sn = sc + 1 == R ? 0 : sc + 1;
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int g = 0; g < 2 * MB; g++) {
          const int a = g % MB, st = g / MB;
          if (g == MB) {     // chunk c + 1 has landed for every wave, chunk c is read out by every wave
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((R - 2) * PW) : "memory");
            __builtin_amdgcn_s_barrier();
            advance();
          }
          const int stage = st == 0 ? sc : sn, kb = 1 - st;
          // the operands of the next 16 k, in the order of their use
#pragma unroll
          for (int q = 0; q < MB + NB; q++)
            if (q * MB / (MB + NB) == a) {
              const int x = q == 0 ? 0 : q <= NB ? MB + q - 1 : q - NB;
              if (x < MB) av[1 - st][x] = read_a(x, kb, stage);
              else bv[1 - st][x - MB] = read_b(x - MB, kb, stage);
            }
          // this step's share of the loads: the rest of chunk c + R - 1, then the first F pieces of chunk c + R
#pragma unroll
          for (int j = 0; j < PW; j++) {
            if (st == 0 && j >= F && (j - F) * MB / (PW - F) == a) load(j, sl);
            if (st == 1 && j < F && j * MB / F == a) load(j, sc);
          }
#pragma unroll
          for (int b = 0; b < NB; b++) mfma(av[st][a], bv[st][b], acc[a][b]);
          __builtin_amdgcn_sched_barrier(0);
        }
        sl = sc;
        sc = sn;
      }
    }
    // results of the last instructions may be read by the assembly below; the rows' data is older than the loads still under way, if
    // those are all of this tile
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");
    if ((EPI == EPI_STRIP || EPI == EPI_DZ) && here.c1 - here.c0 < R) asm volatile("s_waitcnt vmcnt(0)" ::: "memory");

    int ln = lane;
    asm volatile("" : "+v"(ln));      // or what follows from the lane alone is kept in registers through the products
    // one element of a result: read as a whole, the 16 registers of an accumulator would be copied and spill
    auto val = [&](int a, int b, int e) {
      if (MB * NB <= 8) return acc[a][b][e];
      float x;
      asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(acc[a][b][e]));
      return x;
    };
    auto row_data = [&](int a, int which) {
      return *(__attribute__((address_space(3))) unsigned*)(lds + RING + (wave * ARRAYS + which) * (ROWS * 256) + (a * 32 + (ln & 31)) * 4);
    };
    if constexpr (EPI == EPI_SLICE) {
      // rows up to the padding are written, kept or not; a piece behind the first adds to what is there
      float* const out = P.slice + z * P.slice_stride + (int64_t)i0 * P.ldo + j0;      // offsets inside a tile fit 32 bits
      const unsigned ld = (unsigned)P.ldo;
#pragma unroll
      for (int a = 0; a < MB; a++) {
#pragma unroll
        for (int b = 0; b < NB; b++) {
          const int j = wn * 32 * NB + b * 32 + (ln & 31), r = (wm * MB + a) * 32 + 4 * (ln >> 5);
          if (j0 + j < P.out_cols) {
            float* const p = out + ((unsigned)r * ld + j);
            float old[16];
#pragma unroll
            for (int e = 0; e < 16; e++) old[e] = 0.f;
            if (!P.first) {
#pragma unroll
              for (int e = 0; e < 16; e++) old[e] = p[(unsigned)(8 * (e >> 2) + (e & 3)) * ld];
            }
#pragma unroll
            for (int e = 0; e < 16; e++) __builtin_nontemporal_store(old[e] + val(a, b, e), p + (unsigned)(8 * (e >> 2) + (e & 3)) * ld);
          }
          __builtin_amdgcn_sched_barrier(0);      // one block's addresses at a time
        }
      }
      continue;
    }
    const int jw = wn * 32 * NB + 4 * (ln >> 5);      // column of register e of block b: jw + 32 b + 8 (e / 4) + e % 4
    const bool crosses = (EPI == EPI_STRIP || EPI == EPI_DZ) && P.v0 + j0 + BN > P.vocab;
    if constexpr (EPI == EPI_STRIP) {
      __attribute__((address_space(3))) f32x2* const half = (__attribute__((address_space(3))) f32x2*)(lds + RING + ROW_DATA);
#pragma unroll
      for (int a = 0; a < MB; a++) {
        const int il = (wm * MB + a) * 32 + (ln & 31), i = i0 + il, y = (int)row_data(a, 0) - j0;      // padding: negative
        float top = -INFINITY, sum = 0.f;
        auto strip = [&](auto some) {      // some: a target or the vocabulary's end is in the tile
          float x[NB][16];
          auto at = [&](int b, int e) {
            const int j = jw + 32 * b + 8 * (e >> 2) + (e & 3);
            const float v = val(a, b, e);
            return decltype(some)::value && j0 + j >= P.vocab ? -INFINITY : v;
          };
#pragma unroll
          for (int b = 0; b < NB; b++)
#pragma unroll
            for (int e = 0; e < 16; e++) {
              const float v = x[b][e] = at(b, e);
              if (decltype(some)::value && jw + 32 * b + 8 * (e >> 2) + (e & 3) == y) P.zt[i] = v * P.inv_t;
              top = fmaxf(top, v);
            }
          top = fmaxf(top, __shfl_xor(top, 32, 64));
          const float ref = top == -INFINITY ? 0.f : top * P.scale;
#pragma unroll
          for (int b = 0; b < NB; b++)
#pragma unroll
            for (int e = 0; e < 16; e++) sum += __builtin_amdgcn_exp2f(fmaf(x[b][e], P.scale, -ref));
          sum += __shfl_xor(sum, 32, 64);
        };
        if (crosses || __any(y >= 0 && y < BN)) strip(std::true_type());
        else strip(std::false_type());
        if (ln < 32) half[wn * BM + il] = f32x2{top, sum};
        __builtin_amdgcn_sched_barrier(0);      // one row block at a time
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_s_barrier();
      if (tid < BM && i0 + tid < kept) {
        const f32x2 a = half[tid], b = half[BM + tid];
        const float top = fmaxf(a[0], b[0]), ref = top == -INFINITY ? 0.f : top;
        P.part[(size_t)(j0 / BN) * P.padded + i0 + tid] =
            make_float2(top * P.inv_t, a[1] * exp2f((a[0] - ref) * P.scale) + b[1] * exp2f((b[0] - ref) * P.scale));
      }
      continue;
    }
    // 32 rows x SC columns at a time through LDS of the wave's own, rows 16 bytes apart, so that a row is stored in pieces of SC
    lds_char* const mine = lds + RING + ROW_DATA + wave * (32 * PITCH);
    auto store = [&](int a, auto out) {      // out(b, e): element e of block b
#pragma unroll
      for (int n = 0; n < 32 * NB / SC; n++) {
#pragma unroll
        for (int u = 0; u < SC / 8; u++) {
          const int b = (n * SC + 8 * u) / 32, e = (n * SC + 8 * u) % 32 / 2;
          lds_char* const to = mine + (ln & 31) * PITCH + (8 * u + 4 * (ln >> 5)) * EL;
          if constexpr (EL == 2) {
            typedef __attribute__((__vector_size__(4 * sizeof(__bf16)))) __bf16 bf16x4;
            *(__attribute__((address_space(3))) bf16x4*)to = bf16x4{(__bf16)out(b, e), (__bf16)out(b, e + 1), (__bf16)out(b, e + 2), (__bf16)out(b, e + 3)};
          } else {
            *(__attribute__((address_space(3))) f32x4*)to = f32x4{out(b, e), out(b, e + 1), out(b, e + 2), out(b, e + 3)};
          }
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        constexpr int LANES = SC / V;      // of a row
        const int c = wn * 32 * NB + n * SC + ln % LANES * V, r0 = (wm * MB + a) * 32;
#pragma unroll
        for (int r = ln / LANES; r < 32; r += 64 / LANES) {
          const u32x4 v = *(__attribute__((address_space(3))) u32x4*)(mine + r * PITCH + ln % LANES * 16);
          if (j0 + c < P.out_cols && i0 + r0 + r < P.out_rows)
            __builtin_nontemporal_store(v, (u32x4*)(P.out + (int64_t)(i0 + r0 + r) * P.ldo + j0 + c));
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
      }
    };
#pragma unroll
    for (int a = 0; a < MB; a++) {
      if constexpr (EPI == EPI_DZ) {
        const int y = (int)row_data(a, 0) - P.v0 - j0;
        const float g = __builtin_bit_cast(float, row_data(a, 1)), l = __builtin_bit_cast(float, row_data(a, 2)) * 1.44269504f;
        auto dz = [&](int b, int e) { return -g * __builtin_amdgcn_exp2f(fmaf(val(a, b, e), P.scale, -l)); };
        const bool twin = EL == 2 && MB == 2 && P.kept.twins && (wm * MB + a) * 32 + (ln & 31) >= P.kept.twins;      // all rows are in one tile then
        if (crosses || __any(y >= 0 && y < BN)) {
          store(a, [&](int b, int e) {
            const int j = jw + 32 * b + 8 * (e >> 2) + (e & 3);
            const float v = P.v0 + j0 + j >= P.vocab ? 0.f : j == y ? dz(b, e) + g : dz(b, e);
            return twin ? rounding_left(v) : v;
          });
        } else if (__any(twin)) {
          store(a, [&](int b, int e) { return twin ? rounding_left(dz(b, e)) : dz(b, e); });
        } else {
          store(a, dz);
        }
      } else {
        store(a, [&](int b, int e) { return val(a, b, e); });
      }
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // loads into this LDS
}

template <typename T, bool TA, bool TB, int MB, int NB, int R, int EPI>
void go(const Product<T>& p, hipStream_t s) {
  constexpr int lds = Lds<T, MB, NB, R, EPI>::BYTES;
  auto kernel = product_kernel<T, TA, TB, MB, NB, R, EPI>;
  static std::atomic<uint64_t> done;      // more than 64 KB of LDS need an opt-in, once per kernel and device
  int dev = 0;
  (void)hipGetDevice(&dev);
  const uint64_t bit = 1ull << (dev & 63);
  if (!(done.load(std::memory_order_acquire) & bit)) {
    (void)hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    done.fetch_or(bit, std::memory_order_release);
  }
  // as many workgroups as the 256 CUs hold at once
  kernel<<<(unsigned)std::min<int64_t>((int64_t)p.tiles_i * p.tiles_j * p.slices, MB * NB > 4 ? 256 : 512), 256, lds, s>>>(p);
}

// Tile of a product, in 64 rows and 64 columns.  bf16: 256 x 256; 128 x 128 where those would leave a quarter of the CUs idle (1024 x 4096, both
// directions: 100 rows 62 us, with the others 86; 288 rows 65 and 129; forward, 500 rows x 2560 x 20000 70 and 73, 500 x 1024 x 30000 50 and 48); 128 x 256 for up to 128 rows
// otherwise (1024 x 151936, forward: 100 rows 109 us, with 256 x 256 124; 200 rows 141 and 131).  fp32 (16 times the matrix time a byte): 128 x 128, and 64 x 64 where those would be fewer than two
// for each of the 512 workgroups that the card holds (both directions: 1000 rows x 256 x 4096 99 us, with 128 x 128 142; 1000 x 1024
// x 8192 434 and 468; 1500 x 1024 x 16384 1155 and 1027).
struct Tile { int mb, nb; };
template <typename T>
Tile tile_of(int64_t rows, int64_t columns, int64_t slices, bool gathered) {
  if (sizeof(T) == 2) {
    if ((rows + 255) / 256 * ((columns + 255) / 256) * slices < 192) return {2, 2};
    return {gathered && rows <= 128 ? 2 : 4, 4};
  }
  const bool small = (rows + 127) / 128 * ((columns + 127) / 128) * slices < 1024;
  return {small ? 1 : 2, small ? 1 : 2};
}
// Slices of a piece of the vocabulary that dz W may count on when it chooses a tile
template <typename T>
int64_t slices_in(int width) {
  return sizeof(T) == 2 ? std::min(std::max(width / 2048, 1), 64) : 16;
}
// A product of rows x columns with its tiles
template <typename T>
struct Planned {
  Product<T> p;
  Tile t;
  Planned(const Product<T>& product, const Tile& tile, int64_t rows, int64_t columns) : p(product), t(tile) {
    p.tiles_i = (int)((rows + 64 * t.mb - 1) / (64 * t.mb)), p.tiles_j = (int)((columns + 64 * t.nb - 1) / (64 * t.nb));
  }
};
template <typename T, bool TA, bool TB, int EPI>
void go(const Planned<T>& planned, hipStream_t s) {
  const Product<T>& p = planned.p;
  const Tile& t = planned.t;
  if constexpr (sizeof(T) == 2) {
    if (t.nb == 2) return go<T, TA, TB, 2, 2, 6, EPI>(p, s);
    if constexpr (!TA) {
      if (t.mb == 2) return go<T, TA, TB, 2, 4, 5, EPI>(p, s);
    }
    go<T, TA, TB, 4, 4, 4, EPI>(p, s);
  } else {
    if (t.mb == 1) go<T, TA, TB, 1, 1, 8, EPI>(p, s);
    else go<T, TA, TB, 2, 2, 4, EPI>(p, s);
  }
}

}  // namespace

template <typename T>
bool token_logprob_takes_mfma(int64_t padded, int ld, int hidden, int width, const void* weight, const void* dweight) {
  // 32-bit offsets into one descriptor: the rows as k-strided operand, dz, a piece of the weights
  const int64_t most = (1ll << 32) - (1 << 20), el = sizeof(T);
  return hidden % (16 / el) == 0 && aligned16(weight) && aligned16(dweight) && padded * ld * el < most && padded * width * el < most &&
         (int64_t)std::max(width, 256) * hidden * el < most / 2;
}

template <typename T>
void token_logprob_slice_tile(int rows, int hidden, int width, SliceRule& r) {
  // us of a tile's 32 k, fitted; fp32: two workgroups a CU share its matrix units.  2744 rows x 75968 x 2560: two slices, 0.94 ms a piece; nine,
  // which a time of 0.85 would choose: 1.18.
  const Tile t = tile_of<T>(rows, hidden, slices_in<T>(width), true);
  r.rows = 64 * t.mb;
  r.tiles_j = (hidden + 64 * t.nb - 1) / (64 * t.nb);
  r.chunk_us = sizeof(T) == 2 ? (t.mb == 4 ? 0.6f : t.nb == 4 ? 0.35f : 0.2f) : t.mb == 2 ? 2.4f : 0.6f;
}

namespace {

template <typename T>
Planned<T> logits_strips(const T* h, int ld, int rows, int64_t padded, const T* w, int vocab, int hidden, const KeptRows& kept, float inv_t,
                         float2* part, float* zt) {
  Product<T> p{};
  p.a = h, p.lda = ld, p.a_n = (int)padded;
  p.b = w, p.ldb = hidden, p.b_n = vocab;
  p.k = hidden, p.slices = 1, p.group = 4;
  p.kept = kept, p.vocab = vocab, p.v0 = 0, p.scale = (float)(1.4426950408889634 * inv_t), p.inv_t = inv_t;
  p.part = part, p.padded = (int)padded, p.zt = zt;
  return {p, tile_of<T>(rows, vocab, 1, true), rows, vocab};
}
template <typename T>
Planned<T> logits_gradient(const T* h, int ld, int rows, int64_t padded, const T* w, int vocab, int hidden, const KeptRows& kept, float inv_t,
                           const VocabPiece& piece, T* dz) {
  Product<T> p{};
  p.a = h, p.lda = ld, p.a_n = (int)padded;
  p.b = w + (int64_t)piece.v0 * hidden, p.ldb = hidden, p.b_n = vocab - piece.v0;
  p.k = hidden, p.slices = 1, p.group = 4;
  p.kept = kept, p.vocab = vocab, p.v0 = piece.v0, p.scale = (float)(1.4426950408889634 * inv_t), p.inv_t = inv_t;
  p.out = dz, p.ldo = piece.ld, p.out_rows = (int)padded, p.out_cols = (int)up(piece.width, 256);
  // whole multiples of 256 columns: the products behind it read beyond the vocabulary's end
  return {p, tile_of<T>(rows, piece.width, 1, true), rows, p.out_cols};
}
template <typename T>
Planned<T> hidden_gradient(const T* dz, const VocabPiece& piece, int rows, int64_t padded, const T* w, int vocab, int hidden,
                           const KeptRows& kept, int most_slices, float* dh, size_t slice_stride, bool first) {
  Product<T> p{};
  p.a = dz, p.lda = piece.ld, p.a_n = (int)padded;
  p.b = w + (int64_t)piece.v0 * hidden, p.ldb = hidden, p.b_n = std::min(piece.ld, vocab - piece.v0);
  p.k = piece.width, p.slices = most_slices, p.group = 4;
  p.kept = kept, p.slice = dh, p.slice_stride = slice_stride, p.ldo = hidden, p.out_cols = hidden, p.first = first;
  return {p, tile_of<T>(rows, hidden, slices_in<T>(piece.ld - 128), true), rows, hidden};
}
template <typename T>
Planned<T> weight_gradient(const T* dz, const VocabPiece& piece, const T* h, int ld, int64_t padded, int hidden, const KeptRows& kept, T* dw) {
  Product<T> p{};
  p.a = dz, p.lda = piece.ld, p.a_n = (int)padded;
  p.b = h, p.ldb = ld, p.b_n = (int)padded;
  p.k = 0, p.slices = 1, p.group = 4;
  p.kept = kept, p.out = dw + (int64_t)piece.v0 * hidden, p.ldo = hidden, p.out_rows = piece.width, p.out_cols = hidden;
  return {p, tile_of<T>(piece.width, hidden, 1, false), piece.width, hidden};
}

// How far the loads of a planned product reach beyond its operands and its stores beyond its results, with `kept` rows and `slices` of
// per_slice k on the device: the kernel's own arithmetic over all of its tiles.
template <typename T, bool TA, bool TB, int EPI>
void find_overreach(const Planned<T>& planned, int kept, int slices, int per_slice, const Extent& a, const Extent& b, const Extent& out,
                    LoadOverreach& most) {
  const Product<T>& P = planned.p;
  const int64_t el = sizeof(T), BM = 64 * planned.t.mb, BN = 64 * planned.t.nb;
  const int ti = EPI == EPI_OUT ? P.tiles_i : std::min<int64_t>(P.tiles_i, (kept + BM - 1) / BM), k_all = EPI == EPI_OUT ? kept : P.k;
  if (EPI != EPI_SLICE) slices = 1, per_slice = k_all;
  auto operand = [&](bool strided, const T* p, int64_t ld, int n, int tiles, int64_t size, const Extent& in) {
    for (int i = 0; i < tiles; i++) {
      const Reach r = reach_of<T>(strided, ld, n, (int)(i * size), (int)size);
      const int64_t at = ((int64_t)(uintptr_t)p - in.base) / el + r.begin;
      most.buffers = std::max({most.buffers, -at * el, at * el + r.bytes - in.bytes});
      for (int z = 0; z < slices; z++) {
        int c0, c1;
        chunks_of<T>(z, per_slice, k_all, c0, c1);
        if (c1 > c0) most.offsets = std::max(most.offsets, (int64_t)(c1 - 1) * chunk_step(strided, ld) + 1 - r.bytes);
      }
    }
  };
  operand(TA, P.a, P.lda, P.a_n, ti, BM, a);
  if (ti > 0) operand(TB, P.b, P.ldb, P.b_n, P.tiles_j, BN, b);
  // the last element that is stored
  const int64_t rows = std::min<int64_t>(ti * BM, EPI == EPI_DZ || EPI == EPI_OUT ? P.out_rows : ti * BM);
  if (rows == 0) return;
  int64_t end;
  if (EPI == EPI_STRIP) end = ((int64_t)(P.tiles_j - 1) * P.padded + std::min<int64_t>(rows, kept)) * (int64_t)sizeof(float2);
  else if (EPI == EPI_SLICE) end = ((slices - 1) * (int64_t)P.slice_stride + (rows - 1) * P.ldo + P.out_cols) * (int64_t)sizeof(float);
  else end = (int64_t)(uintptr_t)P.out - out.base + ((rows - 1) * P.ldo + P.out_cols) * el;
  most.stores = std::max(most.stores, end - out.bytes);
}

}  // namespace

template <typename T>
LoadOverreach token_logprob_overreach(const LogprobSizes& n) {
  const int64_t el = sizeof(T);
  // addresses that nothing is at: only distances count
  const Extent h{1ll << 44, n.padded * n.ld * el}, w{2ll << 44, (int64_t)n.vocab * n.hidden * el}, dz{3ll << 44, n.padded * n.ldz * el},
      dw{4ll << 44, (int64_t)n.vocab * n.hidden * el}, part{0, n.padded * n.strips * (int64_t)sizeof(float2)},
      dh{0, n.padded * n.hidden * (int64_t)sizeof(float) * n.most_slices};
  auto at = [](const Extent& x) { return (T*)(uintptr_t)x.base; };
  const KeptRows none{};
  LoadOverreach most{0, 0, 0};
  if (!n.backward) {
    find_overreach<T, false, false, EPI_STRIP>(logits_strips<T>(at(h), n.ld, n.rows, n.padded, at(w), n.vocab, n.hidden, none, 1.f, nullptr, nullptr),
                                               n.kept, 1, 0, h, w, part, most);
    return most;
  }
  for (int v0 = 0; v0 < n.vocab; v0 += n.width) {
    const VocabPiece piece{v0, std::min(n.width, n.vocab - v0), n.ldz};
    find_overreach<T, false, false, EPI_DZ>(logits_gradient<T>(at(h), n.ld, n.rows, n.padded, at(w), n.vocab, n.hidden, none, 1.f, piece, at(dz)),
                                            n.kept, 1, 0, h, w, dz, most);
    find_overreach<T, false, true, EPI_SLICE>(hidden_gradient<T>(at(dz), piece, n.rows, n.padded, at(w), n.vocab, n.hidden, none, n.most_slices, nullptr,
                                                                 (size_t)n.padded * n.hidden, v0 == 0),
                                              n.kept, n.slices, n.per_slice, dz, w, dh, most);
    find_overreach<T, true, true, EPI_OUT>(weight_gradient<T>(at(dz), piece, at(h), n.ld, n.padded, n.hidden, none, at(dw)), n.kept, 1, 0, dz, h, dw, most);
  }
  return most;
}

template <typename T>
int launch_logits_strips_mfma(hipStream_t s, const T* h, int ld, int rows, int64_t padded, const T* w, int vocab, int hidden,
                              const KeptRows& kept, float inv_t, float2* part, float* zt) {
  const Planned<T> p = logits_strips<T>(h, ld, rows, padded, w, vocab, hidden, kept, inv_t, part, zt);
  go<T, false, false, EPI_STRIP>(p, s);
  return p.p.tiles_j;
}
template <typename T>
void launch_logits_gradient_mfma(hipStream_t s, const T* h, int ld, int rows, int64_t padded, const T* w, int vocab, int hidden,
                                 const KeptRows& kept, float inv_t, const VocabPiece& piece, T* dz) {
  go<T, false, false, EPI_DZ>(logits_gradient<T>(h, ld, rows, padded, w, vocab, hidden, kept, inv_t, piece, dz), s);
}
template <typename T>
void launch_hidden_gradient_mfma(hipStream_t s, const T* dz, const VocabPiece& piece, int rows, int64_t padded, const T* w, int vocab, int hidden,
                                 const KeptRows& kept, int most_slices, float* dh, size_t slice_stride, bool first) {
  go<T, false, true, EPI_SLICE>(hidden_gradient<T>(dz, piece, rows, padded, w, vocab, hidden, kept, most_slices, dh, slice_stride, first), s);
}
template <typename T>
void launch_weight_gradient_mfma(hipStream_t s, const T* dz, const VocabPiece& piece, const T* h, int ld, int64_t padded, int hidden,
                                 const KeptRows& kept, T* dw) {
  go<T, true, true, EPI_OUT>(weight_gradient<T>(dz, piece, h, ld, padded, hidden, kept, dw), s);
}

#define RL_OF(T)                                                                                                                              \
  template bool token_logprob_takes_mfma<T>(int64_t, int, int, int, const void*, const void*);                                                \
  template LoadOverreach token_logprob_overreach<T>(const LogprobSizes&);                                                                     \
  template void token_logprob_slice_tile<T>(int, int, int, SliceRule&);                                                                         \
  template int launch_logits_strips_mfma<T>(hipStream_t, const T*, int, int, int64_t, const T*, int, int, const KeptRows&, float, float2*,    \
                                            float*);                                                                                          \
  template void launch_logits_gradient_mfma<T>(hipStream_t, const T*, int, int, int64_t, const T*, int, int, const KeptRows&, float,          \
                                               const VocabPiece&, T*);                                                                        \
  template void launch_hidden_gradient_mfma<T>(hipStream_t, const T*, const VocabPiece&, int, int64_t, const T*, int, int, const KeptRows&,   \
                                               int, float*, size_t, bool);                                                                    \
  template void launch_weight_gradient_mfma<T>(hipStream_t, const T*, const VocabPiece&, const T*, int, int64_t, int, const KeptRows&, T*);
RL_OF(float)
RL_OF(bf16_t)
#undef RL_OF
