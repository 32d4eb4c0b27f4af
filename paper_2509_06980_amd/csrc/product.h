// Matrix products on matrix instructions with what follows them in their epilogue: the kernel that the policy update's linear layers and
// the orthogonalised updates share.
#pragma once
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "lds_load.h"
#include "policy_common.h"

// =============================================================================================
// C[i, j] = sum over k of A[i, k] B[j, k] over tiles of 64 MB rows i and 64 NB columns j: four waves of 32 MB x 32 NB on 32x32x16 (fp32:
// 32x32x2) matrix instructions, sums in 32 bits.
// Operands as they lie in memory: k-contiguous ([row][k]) or k-strided (TA, TB: [k][column]).  A chunk of CB = 64 or 128 bytes of k of both goes
// straight from memory into one of R stages in LDS, R - 1 ahead; operands are read 32 bytes of k ahead of the instructions that use them, one barrier a
// chunk.  A workgroup stays for all its tiles and its loads run on into the next one.
//   k-contiguous: rows of CB bytes.  The 16-byte piece p of row r is kept at p ^ (r / 4 % 4), of 128 bytes at p ^ (r / 2 % 8), so the 16 rows that a read
//     takes in one go lie in different banks.
//   k-strided, 16-bit types: read with the transposing LDS read, 16 lanes take 4 k x 16 columns, lane i gets column i of the 4 k.  The 64-byte
//     block b of row k is kept at b ^ (k % 4).  fp32: read one by one; block b of row k is kept at b ^ 2 (k / 4 % 2).
// fp32 instructions take 2 k, of a lane's 16 bytes element e in step e: k = e and 4 + e of the eight, the same for both operands.
// k may come in segments (two pairs of operands whose products add up, or one pair that no 32-bit offset spans), tiles in batches and k in
// slices, whose sums in 32 bits a second kernel adds up in order before the epilogue.
// Nothing is read behind an operand's last row and column, and what a tile has too many (rows, columns, k) enters as zeros: a value that is
// no number reaches its own row and column of C only.
// Epilogue: 32 rows x 64 columns of a wave at a time through LDS of its own, so that rows are read and written in pieces of 8 columns (fp32: 4);
// the 16-byte piece p of row r is kept at p ^ (r % 16) (32 columns: r % 8).
//
// Tiles and stages, 16-bit types: 256 x 256, one workgroup a CU, with two stages of 128 bytes where both operands are k-contiguous and four of 64 where one is
// strided (two of 128 there: 0 to 10 % slower); 192 x 256 where that leaves fewer CUs without a tile (4096 x 2560 from k 9728: 220 tiles in 236 us; 160 of
// 256 x 256 by the estimate below 270); 128 x 128, two workgroups a CU, with two stages of 128 bytes (where there are no more tiles than CUs four): a CU asks
// the caches for twice as much there, and in requests of 64 bytes it gets 25 bytes a clock however many are under way (2560 x 9728 orthogonalised 1564 us
// with 64, 1420 with 128).  fp32: 128 x 128 and 64 x 64, two stages of 128 bytes (1024 x 1024 orthogonalised 373 us, 391 with 64).
// What bounds the large ones: the clock that the power of the matrix units leaves (8192 x 8192 x 8192 in bf16 takes 835 us, 1.32 PFLOP/s, operands strided as in the
// backward pass 819 to 826; of zeros 569), and that these are busy in 39 to 67 % of a launch's clocks in linear layers, 20 to 43 % in orthogonalised updates.  The rest of
// the clocks goes to last rounds with few tiles (4096 rows x 2560 -> 9728: 222 us, 0.92 PFLOP/s, 608 tiles in 2.4 rounds of the CUs), to epilogues with no products beside
// them and to what a chunk's schedule leaves open; LDS reads wait for a bank in 0 to 5 % of theirs.
// =============================================================================================
namespace product {

typedef __attribute__((address_space(3))) char lds_char;
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 f16x8;

__host__ __device__ __forceinline__ int64_t padded(int64_t n) { return (n + 7) / 8 * 8; }      // columns of a row of sums

// ---- elements: float, bf16_t, _Float16 ----------------------------------------------------------
__device__ __forceinline__ float wide(float v) { return v; }
__device__ __forceinline__ float wide(bf16_t v) { return bf2f(v); }
__device__ __forceinline__ float wide(_Float16 v) { return (float)v; }
template <typename T>
__device__ __forceinline__ T narrow(float v) {
  if constexpr (std::is_same<T, bf16_t>::value) return to_bf16(v);
  else return (T)v;
}
// N consecutive elements; `vec`: as pieces of 16 bytes (8 or 16 for N elements of 16 bits)
template <typename T, int N>
__device__ __forceinline__ void load_row(const T* p, bool vec, int left, float (&v)[N]) {
  if (vec) {
    struct alignas(N * sizeof(T) < 16 ? N * sizeof(T) : 16) Piece { T x[N]; };
    const Piece q = *(const Piece*)p;
#pragma unroll
    for (int e = 0; e < N; e++) v[e] = wide(q.x[e]);
  } else {
#pragma unroll
    for (int e = 0; e < N; e++) v[e] = e < left ? wide(p[e]) : 0.f;
  }
}
// STREAM: past the caches
template <typename T, int N, bool STREAM = false>
__device__ __forceinline__ void store_row(T* p, bool vec, int left, const float (&v)[N]) {
  if (vec) {
    struct alignas(N * sizeof(T) < 16 ? N * sizeof(T) : 16) Piece { T x[N]; } q;
#pragma unroll
    for (int e = 0; e < N; e++) q.x[e] = narrow<T>(v[e]);
    if constexpr (STREAM && N * sizeof(T) >= 16) {
      struct Words { u32x4 x[N * sizeof(T) / 16]; };
      const Words w = __builtin_bit_cast(Words, q);
#pragma unroll
      for (unsigned i = 0; i < N * sizeof(T) / 16; i++) __builtin_nontemporal_store(w.x[i], (u32x4*)p + i);
    } else {
      *(Piece*)p = q;
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; e++)
      if (e < left) p[e] = narrow<T>(v[e]);
  }
}

// f(0), f(1), .. f(N - 1) with constants: an array of accumulators indexed by anything else would leave the registers
template <int N, int I = 0, typename F>
__device__ __forceinline__ void each_part(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>());
    each_part<N, I + 1>(f);
  }
}

// One operand in memory: rows of ld elements, n of them (of one segment), `width` elements of a row used.  k-contiguous: rows are i (or j) and width
// is k; k-strided: rows are k.
template <typename T>
struct Operand {
  const T* p;
  int64_t ld, batch, segment;      // strides in elements: of a row, a batch, a segment
  int rows, last_rows, width, last_width;      // of every segment but the last; of the last
  int64_t elements;                // that lie from p on, for the check of the loads
};
template <typename T>
struct Product {
  Operand<T> a, b;
  int64_t b2;                     // gated: from B to the second matrix's rows, in elements
  const T* u;                     // where B's second matrix lies (gated) or its second segment, if that is a matrix of its own, and the elements from there on: for the check of
  int64_t u_elements;             // the loads
  int tiles_i, tiles_j, batches, segments, slices;
  int k, last_k;                  // of a segment; of the last
  int group;                      // row tiles that an XCD takes together
  int rows, cols;                 // of C
  float* part;                    // sums of slices [slice][batch][rows][padded(cols)], gated: twice the columns
};

// What a tile's loads of one operand may reach, from element `begin` on.  Scalar offsets stay inside: the hardware compares a lane's offset with the
// size less the scalar one.  A tile behind the operand, which no product has, reaches what the first
// one does: a size below 0 would be one of 4 GiB, and a size of 0 less a scalar offset too.
struct Reach {
  int64_t begin;
  unsigned bytes;
};
template <typename T>
__host__ __device__ __forceinline__ Reach reach_of(bool strided, int64_t ld, int n, int width, int at, int rows) {
  if (at >= (strided ? width : n)) at = 0;
  if (strided) return {at, (unsigned)(((n - 1) * ld + width - at) * (int64_t)sizeof(T))};
  const int left = n - at;
  return {at * ld, (unsigned)((((left < rows ? left : rows) - 1) * ld + width) * (int64_t)sizeof(T))};
}
__host__ __device__ __forceinline__ unsigned chunk_step(bool strided, int64_t ld, int bytes) { return (strided ? (unsigned)ld : 1u) * (unsigned)bytes; }
template <typename T>
constexpr int kPiece = sizeof(T) == 2 ? 8 : 4;      // columns that a lane of the epilogue takes
// Chunks of all segments, and those of a slice
template <typename T>
__host__ __device__ __forceinline__ int chunks(int k, int bytes) { return (k + bytes / (int)sizeof(T) - 1) / (bytes / (int)sizeof(T)); }
__host__ __device__ __forceinline__ int slice_begin(int slice, int slices, int n) { return (int)((int64_t)n * slice / slices); }

template <typename T, int MB, int NB, int R, int CB, bool GATED>
struct Lds {
  // of an epilogue: columns and rows of a part; of 128 x 128 tiles half as much, so that a CU holds two workgroups
  static constexpr bool HALF = NB == 2 && CB == 128;
  static constexpr int RING = R * (MB + NB) * CB * 64, W = NB == 1 || (HALF && !GATED) ? 32 : 64, ROWS = HALF && GATED ? 16 : 32, WAVE = ROWS * W * 4, BYTES = RING + 4 * WAVE;
};

// EPI: struct with GATED, SYMMETRIC (lower triangle of tiles only; the epilogue's values are stored a second time across the diagonal), and
//   void fetch(int batch, int row, int col, Extra&) const           what joins these sums from memory
//   void operator()(int batch, int row, int col, float (&v)[V], float (&u)[V], const Extra&) const
// which finishes V columns of a row: u holds the second matrix's sums where GATED.  UNROLL: short enough that it may stand there for every row, so that
// fetch runs a part of the tile ahead.  SLICED: in slices, tiles of up to so many blocks of 64 x 64 are built; larger ones are never the cheapest there.
template <typename T, typename EPI>
struct Arguments {
  Product<T> p;
  EPI epi;
};
template <typename T, bool TA, bool TB, int MB, int NB, int R, int CB, bool SLICED, typename EPI>
__global__ __launch_bounds__(256, MB * NB > 4 ? 1 : 2) void product_kernel(Arguments<T, EPI>) {
  // The arguments are read where they are used, by scalar loads: kept in registers through the products, they would push the descriptors of the loads out of
  // theirs, and one that a vector instruction brings back has to be waited for.
  auto arguments = [&]() {
    auto* p = (const __attribute__((address_space(4))) Arguments<T, EPI>*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(p));
    return (const Arguments<T, EPI>*)p;
  };
  constexpr int BM = 64 * MB, BN = 64 * NB, EL = sizeof(T), KC = CB / EL, V = kPiece<T>;
  constexpr int NS = CB / 32, KS = KC / NS, PR = CB / 16;      // steps of a chunk, their k; pieces of a row
  constexpr int PA = MB * (CB / 64), PB = NB * (CB / 64), PW = PA + PB, BUF = PW * 4096, F = PW / 2;      // pieces of 1 KB that a wave loads
  static_assert(CB == 64 || CB == 128, "chunks of a row");
  constexpr bool GATED = EPI::GATED, SYM = EPI::SYMMETRIC;
  constexpr int JN = GATED ? BN / 2 : BN;      // columns of C that a tile covers
  static_assert((!TA || BM * EL >= 256) && (!TB || BN * EL >= 256), "four blocks of 64 bytes a row");
  static_assert(!GATED || (!TB && NB >= 2), "rows of two matrices in a tile");
  static_assert(!SYM || MB == NB, "square tiles");
  using L = Lds<T, MB, NB, R, CB, GATED>;
  extern __shared__ u32x4 smem[];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, wm = wave >> 1, wn = wave & 1;
  const Product<T>& P = arguments()->p;
  const int per_batch = SYM ? P.tiles_i * (P.tiles_i + 1) / 2 : P.tiles_i * P.tiles_j, slices = SLICED ? P.slices : 1;
  const int tiles = per_batch * slices, total = tiles * P.batches;
  const int c_seg = chunks<T>(P.k, CB), c_all = c_seg * (P.segments - 1) + chunks<T>(P.last_k, CB);
  struct Place {
    int i0, j0, batch, slice, c0, c1;      // first row and column of C, batch, slice, its chunks of k
  };
  // numbered so that an XCD (workgroups are dealt to the 8 of them in turn) takes a compact block of one batch and slice
  auto place = [&](int id) {
    const Product<T>& P = arguments()->p;
    const int base = total >> 3, rem = total & 7, x = id & 7, vid = x * base + min(x, rem) + (id >> 3);
    const int batch = vid / tiles, in_batch = vid - batch * tiles, slice = SLICED ? in_batch / per_batch : 0, v = in_batch - slice * per_batch;
    int i, j;
    if constexpr (SYM) {
      i = (int)((__builtin_sqrtf(8.f * v + 1.f) - 1.f) * 0.5f);
      while ((i + 1) * (i + 2) / 2 <= v) i++;
      while (i * (i + 1) / 2 > v) i--;
      j = v - i * (i + 1) / 2;
    } else {
      const int per = P.group * P.tiles_j, grp = v / per, first = grp * P.group, gm = min(P.group, P.tiles_i - first), in = v - grp * per;
      i = first + in % gm, j = in / gm;
    }
    Place t;      // the divisions leave these in vector registers
    t.i0 = __builtin_amdgcn_readfirstlane(i) * BM;
    t.j0 = __builtin_amdgcn_readfirstlane(j) * JN;
    t.batch = __builtin_amdgcn_readfirstlane(batch);
    t.slice = __builtin_amdgcn_readfirstlane(slice);
    t.c0 = SLICED ? slice_begin(t.slice, slices, c_all) : 0;
    t.c1 = SLICED ? slice_begin(t.slice + 1, slices, c_all) : c_all;
    return t;
  };
  const unsigned sa = chunk_step(TA, P.a.ld, CB), sb = chunk_step(TB, P.b.ld, CB);
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) void*)smem;
  // k of the lane's piece of a k-contiguous row
  const int kpos = (CB == 64 ? (lane & 3) ^ (lane >> 4 & 3) : (lane & 7) ^ ((wave & 1) * 4 + (lane >> 4 & 3))) * (16 / EL);
  int va[PA], vb[PB];      // this lane's offset of each piece that its wave loads
  auto offset = [&](int kb, int64_t ld, bool strided, int row_bytes) {      // kb: the KB of the operand
    if (strided) {
      const int lanes = row_bytes / 16, k = kb * (64 / lanes) + lane / lanes, p = lane % lanes;
      const int block = (p >> 2) ^ (EL == 2 ? k & 3 : (k >> 2 & 1) << 1);
      return (int)(k * ld * EL) + (block << 6) + ((p & 3) << 4);
    }
    return (int)((kb * (64 / PR) + lane / PR) * ld * EL) + kpos * EL;
  };
#pragma unroll
  for (int j = 0; j < PA; j++) va[j] = offset(j * 4 + wave, P.a.ld, TA, BM * EL);
#pragma unroll
  // gated: a wave column's rows are half of the first matrix, half of the second: 64 and 64 (NB = 4) or 32 and 32
  for (int j = 0; j < PB; j++) {
    constexpr int KBS = CB / 64;      // of 16 rows
    const int n = j * 4 + wave, in = n / (4 * KBS), rest = n % (4 * KBS);      // group of 64 rows, KB of it
    vb[j] = offset(!GATED ? n : NB == 4 ? (in >> 1) * (4 * KBS) + rest : in * (2 * KBS) + rest % (2 * KBS), P.b.ld, TB, BN * EL);
  }
  // The loads run R - 1 chunks ahead of the products, from one tile of the workgroup into the next: tile `at`, its chunk lc (li in its segment), operands
  // behind its descriptors (what is read past their end arrives as zeros).  Behind the last tile: its last chunk again, never read.
  u32x4 ra, rb, rb2;
  int at = (int)blockIdx.x - (int)gridDim.x, lc = 0, lend = 0, li = 0, lseg_end = 0;
  Place next{};
  unsigned tail = 0;      // k-contiguous: pieces of the chunk behind the end of k lie out of reach
  int seg_k = 0;
  unsigned oa = 0, ob = 0;      // scalar offsets of the chunk
  auto enter = [&](int seg) {      // a segment of tile `next`
    const Product<T>& P = arguments()->p;
    const bool end = seg == P.segments - 1;
    const Reach a = reach_of<T>(TA, P.a.ld, end ? P.a.last_rows : P.a.rows, end ? P.a.last_width : P.a.width, next.i0, BM);
    const Reach b = reach_of<T>(TB, P.b.ld, end ? P.b.last_rows : P.b.rows, end ? P.b.last_width : P.b.width, next.j0, JN);
    const T* pa = P.a.p + next.batch * P.a.batch + seg * P.a.segment + a.begin;
    const T* pb = P.b.p + next.batch * P.b.batch + seg * P.b.segment + b.begin;
    ra = buffer_rsrc(pa, a.bytes);
    rb = buffer_rsrc(pb, b.bytes);
    if constexpr (GATED) rb2 = buffer_rsrc(pb + P.b2, b.bytes);
    seg_k = end ? P.last_k : P.k;
    lseg_end = end ? lend : min(lend, (seg + 1) * c_seg);
    li = lc - seg * c_seg;
    settle(ra);
    settle(rb);
    if constexpr (GATED) settle(rb2);
  };
  auto set_chunk = [&]() {
    if constexpr (!TA || !TB) tail = li * KC + kpos >= seg_k ? 0x80000000u : 0u;
    oa = (unsigned)li * sa, ob = (unsigned)li * sb;
    settle(oa, ob);
  };
  auto advance = [&]() {
    lc++, li++;
    if (lc >= lseg_end) {
      if (lc < lend) {
        enter(lc / c_seg);
      } else {
        at += gridDim.x;
        if (at < total) {
          next = place(at);
          lc = next.c0, lend = next.c1;
          enter(lc / c_seg);
        } else {
          lc--, li--;
          at -= gridDim.x;
        }
      }
    }
    set_chunk();
  };
  auto load = [&](int j, int stage) {      // piece j of this wave
    const unsigned dst = lds0 + (unsigned)stage * BUF + (unsigned)(j * 4 + wave) * 1024u;
    if (j < PA) {
      load_to_lds(dst, TA ? va[j] : (int)(va[j] | tail), ra, oa);
    } else {
      const int off = TB ? vb[j - PA] : (int)(vb[j - PA] | tail);
      const bool second = GATED && (NB == 4 ? (j - PA) / (CB / 64) & 1 : CB == 64 ? wave >> 1 : (j - PA) & 1);
      if (GATED && second) load_to_lds(dst, off, rb2, ob);
      else load_to_lds(dst, off, rb, ob);
    }
  };
  f32x16 acc[MB][NB];
  auto mfma = [&](const u32x4& row, const u32x4& col, f32x16& c) {      // a lane holds one row's values
    if constexpr (std::is_same<T, bf16_t>::value) {
      c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, col), __builtin_bit_cast(bf16x8, row), c, 0, 0, 0);
    } else if constexpr (EL == 2) {
      c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, col), __builtin_bit_cast(f16x8, row), c, 0, 0, 0);
    } else {
      const f32x4 u = __builtin_bit_cast(f32x4, col), w = __builtin_bit_cast(f32x4, row);
#pragma unroll
      for (int e = 0; e < 4; e++) c = __builtin_amdgcn_mfma_f32_32x32x2f32(u[e], w[e], c, 0, 0, 0);
    }
  };
  // lane parts of the operand reads: k-contiguous by half a chunk, k-strided by 32-column block
  int la[TA ? MB : NS], lb[TB ? NB : NS];
  auto part = [&](int x, int row_bytes) {
    if constexpr (EL == 2) {
      const int s = lane >> 2 & 3;
      return ((lane >> 5) * 8 + s) * row_bytes + ((x ^ s) << 6) + ((lane >> 4 & 1) << 5) + ((lane & 3) << 3);
    } else {
      return (lane >> 5) * 4 * row_bytes + (((2 * x) ^ (lane >> 5 << 1)) << 6) + ((lane & 31) << 2);
    }
  };
  auto part2 = [&](int x) { return (lane & 31) * CB + (((x * 2 + (lane >> 5)) ^ (CB == 64 ? lane >> 2 & 3 : lane >> 1 & 7)) << 4); };
#pragma unroll
  for (int x = 0; x < (TA ? MB : NS); x++) la[x] = TA ? part(wm * MB + x, BM * EL) : part2(x);
#pragma unroll
  for (int x = 0; x < (TB ? NB : NS); x++) lb[x] = TB ? part(wn * NB + x, BN * EL) : part2(x);
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
    if constexpr (TA) return strided(base + kb * KS * BM * EL + la[x], std::integral_constant<int, BM * EL>());
    else return *(__attribute__((address_space(3))) u32x4*)(lds + base + (wm * MB + x) * (32 * CB) + la[kb]);
  };
  auto read_b = [&](int x, int kb, int stage) {
    const int base = stage * BUF + PA * 4096;
    if constexpr (TB) return strided(base + kb * KS * BN * EL + lb[x], std::integral_constant<int, BN * EL>());
    else return *(__attribute__((address_space(3))) u32x4*)(lds + base + (wn * NB + x) * (32 * CB) + lb[kb]);
  };
  if ((int)blockIdx.x >= total) return;
  lc = -1, li = -1;
  advance();
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
  int sc = 0, sl = R - 1;                  // stages of chunks c and c + R - 1 (that of chunk c - 1)
  for (int id = blockIdx.x; id < total; id += gridDim.x) {
    const Place here = place(id);
#pragma unroll
    for (int a = 0; a < MB; a++)
#pragma unroll
      for (int b = 0; b < NB; b++)
#pragma unroll
        for (int e = 0; e < 16; e++) acc[a][b][e] = 0.f;
    {      // its first chunk has landed for every wave
      u32x4 av[2][MB], bv[2][NB];
#pragma unroll
      for (int x = 0; x < MB; x++) av[0][x] = read_a(x, 0, sc);
#pragma unroll
      for (int x = 0; x < NB; x++) bv[0][x] = read_b(x, 0, sc);
      for (int c = here.c0; c < here.c1; c++) {
        const int sn = sc + 1 == R ? 0 : sc + 1;
        __builtin_amdgcn_sched_barrier(0);
        // the instructions of a step (16 k), one memory instruction behind each: the operands of the next step first, then this step's share of the loads: in
        // the chunk's last step, which begins with the barrier, the first F pieces of chunk c + R; in its first the rest of chunk c + R - 1
        constexpr int S = MB * NB, Q = MB + NB;
#pragma unroll
        for (int g = 0; g < NS * MB; g++) {
          const int a = g % MB, st = g / MB, now = st & 1;
          if (g == (NS - 1) * MB) {     // chunk c + 1 has landed for every wave, chunk c is read out by every wave
            asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((R - 2) * PW) : "memory");
            __builtin_amdgcn_s_barrier();
          }
          const int stage = st < NS - 1 ? sc : sn, kb = st < NS - 1 ? st + 1 : 0, first = st == 0 ? F : 0, n = st == 0 ? PW - F : st == NS - 1 ? F : 0;
#pragma unroll
          for (int b = 0; b < NB; b++) {
            mfma(av[now][a], bv[now][b], acc[a][b]);
#pragma unroll
            for (int q = 0; q < Q; q++)      // in the order of their use
              if (q * S / (2 * Q) == a * NB + b) {
                const int x = q == 0 ? 0 : q <= NB ? MB + q - 1 : q - NB;
                if (x < MB) av[1 - now][x] = read_a(x, kb, stage);
                else bv[1 - now][x - MB] = read_b(x - MB, kb, stage);
              }
#pragma unroll
            for (int j = 0; j < PW; j++)
              if (j < n && (n > S / 2 ? j * S / n : S / 2 + j * (S - S / 2) / n) == a * NB + b) load(first + j, st == 0 ? sl : sc);
            if (g == MB - 1 && b == NB - 1) advance();
            __builtin_amdgcn_sched_barrier(0);
          }
        }
        sl = sc;
        sc = sn;
      }
    }
    asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");      // results of the last instructions may be read by the assembly below

    int ln = lane;
    asm volatile("" : "+v"(ln));      // or what follows from the lane alone is kept in registers through the products
    // one element of a result: read as a whole, the 16 registers of an accumulator would be copied and spill
    auto val = [&](int a, int b, int e) __attribute__((always_inline)) {
      if (MB * NB <= 8) return acc[a][b][e];
      float x;
      asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(x) : "a"(acc[a][b][e]));
      return x;
    };
    constexpr int W = L::W, PW_ROW = W / 4;      // columns through LDS at a time, 16-byte pieces of a row
    static_assert(!GATED || W == 64, "halves of two matrices");
    lds_char* const mine = lds + L::RING + wave * L::WAVE;
    auto piece = [&](int r, int p) { return mine + r * (W * 4) + ((p ^ (r & (PW_ROW - 1))) << 4); };
    constexpr int CN = GATED ? W / 2 : W, LANES = CN / V, PR = L::ROWS, PASSES = PR * LANES / 64;      // columns of C, lanes of a row, rows of a part
    constexpr int GROUPS = GATED ? NB / 2 : 32 * NB / W, SPLIT = 32 / PR, PARTS = MB * GROUPS * SPLIT;
    auto column = [&](int group) { return here.j0 + (GATED ? wn * 16 * NB + group * 32 : wn * 32 * NB + group * W) + ln % LANES * V; };
    // what joins the sums from memory is requested a part ahead
    using Extra = typename EPI::Extra;
    Extra extra[2][EPI::UNROLL ? PASSES : 1];
    auto fetch = [&](auto constant) __attribute__((always_inline)) {
      constexpr int part = decltype(constant)::value;
      if constexpr (EPI::UNROLL && !SLICED) {
        const Arguments<T, EPI>& all = *arguments();
        const int r0 = here.i0 + (wm * MB + part / SPLIT / GROUPS) * 32 + part % SPLIT * PR + ln / LANES, col = column(part / SPLIT % GROUPS);
#pragma unroll
        for (int i = 0; i < PASSES; i++)
          if (r0 + i * (64 / LANES) < all.p.rows && col < all.p.cols) all.epi.fetch(here.batch, r0 + i * (64 / LANES), col, extra[part & 1][i]);
      }
    };
    auto through = [&](auto constant) __attribute__((always_inline)) {      // block a of rows, blocks b0 and b1 (gated: of the second matrix) of columns
      constexpr int part = decltype(constant)::value, a = part / SPLIT / GROUPS, group = part / SPLIT % GROUPS, split = part % SPLIT, b0 = GATED ? group : W / 32 * group, b1 = GATED ? group + NB / 2 : b0 + 1;
      const Arguments<T, EPI>& all = *arguments();
      const Product<T>& P = all.p;
      const EPI& epi = all.epi;
      auto put = [&](int b, int half) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < 4; u++) {
          const f32x4 x = f32x4{val(a, b, 4 * u), val(a, b, 4 * u + 1), val(a, b, 4 * u + 2), val(a, b, 4 * u + 3)};
          if (SPLIT == 1 || (ln & 31) / PR == split) *(__attribute__((address_space(3))) f32x4*)piece(ln & (PR - 1), half * 8 + 2 * u + (ln >> 5)) = x;
        }
      };
      put(b0, 0);
      if constexpr (W == 64) put(b1, 1);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      const int r0 = here.i0 + (wm * MB + a) * 32 + split * PR, c = ln % LANES * V, col = column(group) - c;
      auto pass = [&](int r, const Extra* given) __attribute__((always_inline)) {
        float v[V], u[V];
        auto get = [&](int first, float (&to)[V]) __attribute__((always_inline)) {
#pragma unroll
          for (int q = 0; q < V / 4; q++) {
            const f32x4 x = *(__attribute__((address_space(3))) f32x4*)piece(r, first + q);
#pragma unroll
            for (int e = 0; e < 4; e++) to[4 * q + e] = x[e];
          }
        };
        get(c / 4, v);
        if constexpr (GATED) get(W / 8 + c / 4, u);
        if (r0 + r < P.rows && col + c < P.cols) {
          if constexpr (SLICED) {
            const int64_t ld = padded(P.cols);
            float* to = P.part + (((int64_t)here.slice * P.batches + here.batch) * P.rows + r0 + r) * (GATED ? 2 * ld : ld) + col + c;
            store_row<float, V>(to, true, V, v);
            if constexpr (GATED) store_row<float, V>(to + ld, true, V, u);
          } else if (given) {
            epi(here.batch, r0 + r, col + c, v, u, *given);
          } else {
            Extra own;
            epi.fetch(here.batch, r0 + r, col + c, own);
            epi(here.batch, r0 + r, col + c, v, u, own);
          }
        }
        if constexpr (SYM && !SLICED) {
          if (here.i0 != here.j0) {
#pragma unroll
            for (int q = 0; q < V / 4; q++)
              *(__attribute__((address_space(3))) f32x4*)piece(r, c / 4 + q) = f32x4{v[4 * q], v[4 * q + 1], v[4 * q + 2], v[4 * q + 3]};
          }
        }
      };
      if constexpr (EPI::UNROLL && !SLICED) {
#pragma unroll
        for (int i = 0; i < PASSES; i++) pass(ln / LANES + i * (64 / LANES), &extra[part & 1][i]);
      } else {
#pragma unroll 1
        for (int r = ln / LANES; r < PR; r += 64 / LANES) pass(r, nullptr);
      }
      if constexpr (SYM && !SLICED) {
        if (here.i0 != here.j0) {      // column c of these 32 rows is a part of row c across the diagonal
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll 1
          for (int n = ln; n < W * 32 / V; n += 64) {
            const int cc = n % W, r = n / W * V;
            float v[V];
#pragma unroll
            for (int e = 0; e < V; e++) v[e] = *(__attribute__((address_space(3))) float*)(piece(r + e, cc >> 2) + (cc & 3) * 4);
            if (col + cc < P.cols && r0 + r < P.rows) epi.across(here.batch, col + cc, r0 + r, v);
          }
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      __builtin_amdgcn_sched_barrier(0);
    };
    fetch(std::integral_constant<int, 0>());
    each_part<PARTS>([&](auto part) __attribute__((always_inline)) {
      constexpr int next = decltype(part)::value + 1;
      if constexpr (next < PARTS) fetch(std::integral_constant<int, next>());
      through(part);
    });
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // loads into this LDS
}

// Sums of the slices, then the epilogue: a thread takes V columns of a row.
template <typename T, typename EPI>
__global__ __launch_bounds__(256) void join_kernel(Product<T> P, EPI epi) {
  constexpr int V = kPiece<T>;
  const int64_t ld = padded(P.cols), row_ld = EPI::GATED ? 2 * ld : ld, per_row = (P.cols + V - 1) / V;
  const int64_t rows = (int64_t)P.batches * P.rows, n = rows * per_row;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / per_row;
    const int c = (int)(i - row * per_row) * V;
    float v[V], u[V];
#pragma unroll
    for (int e = 0; e < V; e++) v[e] = u[e] = 0.f;
    for (int s = 0; s < P.slices; s++) {
      const float* p = P.part + (s * rows + row) * row_ld + c;
      float x[V];
      load_row<float, V>(p, true, V, x);
#pragma unroll
      for (int e = 0; e < V; e++) v[e] += x[e];
      if constexpr (EPI::GATED) {
        load_row<float, V>(p + ld, true, V, x);
#pragma unroll
        for (int e = 0; e < V; e++) u[e] += x[e];
      }
    }
    typename EPI::Extra x;
    epi.fetch((int)(row / P.rows), (int)(row % P.rows), c, x);
    epi((int)(row / P.rows), (int)(row % P.rows), c, v, u, x);
  }
}

template <typename T>
constexpr int kJoinBlock = sizeof(T) == 2 ? 64 : 32;
// The same for a symmetric product, of which the slices hold the tiles on and under the diagonal: a workgroup takes B x B elements and stores them across too.
template <typename T, typename EPI>
__global__ __launch_bounds__(256) void join_symmetric_kernel(Product<T> P, EPI epi) {
  constexpr int V = kPiece<T>, B = kJoinBlock<T>;
  __shared__ float block[B][B + 1];
  const int v0 = blockIdx.x;
  int i = (int)((__builtin_sqrtf(8.f * v0 + 1.f) - 1.f) * 0.5f);
  while ((i + 1) * (i + 2) / 2 <= v0) i++;
  while (i * (i + 1) / 2 > v0) i--;
  const int j = v0 - i * (i + 1) / 2, batch = blockIdx.y, r0 = i * B, c0 = j * B;
  const int64_t ld = padded(P.cols), rows = (int64_t)P.batches * P.rows;
  for (int p = threadIdx.x; p < B * B / V; p += 256) {
    const int r = p / (B / V), c = p % (B / V) * V;
    if (r0 + r >= P.rows || c0 + c >= P.cols) continue;
    float v[V], u[V];
#pragma unroll
    for (int e = 0; e < V; e++) v[e] = u[e] = 0.f;
    for (int s = 0; s < P.slices; s++) {
      float x[V];
      load_row<float, V>(P.part + (s * rows + (int64_t)batch * P.rows + r0 + r) * ld + c0 + c, true, V, x);
#pragma unroll
      for (int e = 0; e < V; e++) v[e] += x[e];
    }
    typename EPI::Extra extra;
    epi.fetch(batch, r0 + r, c0 + c, extra);
    epi(batch, r0 + r, c0 + c, v, u, extra);
#pragma unroll
    for (int e = 0; e < V; e++) block[r][c + e] = v[e];
  }
  if (i == j) return;
  __syncthreads();
  for (int p = threadIdx.x; p < B * B / V; p += 256) {
    const int c = p % B, r = p / B * V;
    if (r0 + r >= P.rows || c0 + c >= P.cols) continue;
    float v[V];
#pragma unroll
    for (int e = 0; e < V; e++) v[e] = block[r + e][c];      // what is behind the last row is set to zero by the epilogue
    epi.across(batch, c0 + c, r0 + r, v);
  }
}

template <typename T, bool TA, bool TB, int MB, int NB, int R, int CB, bool SLICED, typename EPI>
const char* form_of() { return __PRETTY_FUNCTION__; }
template <typename T, bool TA, bool TB, int MB, int NB, int R, int CB, bool SLICED, typename EPI>
void go(const Product<T>& p, const EPI& epi, hipStream_t s) {
  constexpr int lds = Lds<T, MB, NB, R, CB, EPI::GATED>::BYTES;
  auto kernel = product_kernel<T, TA, TB, MB, NB, R, CB, SLICED, EPI>;
  static std::atomic<uint64_t> done;      // more than 64 KB of LDS need an opt-in, once per kernel and device
  int dev = 0;
  (void)hipGetDevice(&dev);
  const uint64_t bit = 1ull << (dev & 63);
  if (!(done.load(std::memory_order_acquire) & bit)) {
    (void)hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
    done.fetch_or(bit, std::memory_order_release);
  }
  const int64_t tiles = (EPI::SYMMETRIC ? (int64_t)p.tiles_i * (p.tiles_i + 1) / 2 : (int64_t)p.tiles_i * p.tiles_j) * p.slices * p.batches;
  // as many workgroups as the 256 CUs hold at once
  kernel<<<(unsigned)std::min<int64_t>(tiles, 256 * (160 * 1024 / lds)), 256, lds, s>>>(Arguments<T, EPI>{p, epi});
  if constexpr (SLICED && EPI::SYMMETRIC) {
    const unsigned n = (unsigned)(p.rows + kJoinBlock<T> - 1) / kJoinBlock<T>;
    join_symmetric_kernel<T, EPI><<<dim3(n * (n + 1) / 2, p.batches), 256, 0, s>>>(p, epi);
  } else if constexpr (SLICED) {
    const int64_t n = (int64_t)p.batches * p.rows * ((p.cols + kPiece<T> - 1) / kPiece<T>);
    join_kernel<T, EPI><<<(unsigned)std::min<int64_t>((n + 255) / 256, 4096), 256, 0, s>>>(p, epi);
  }
}

// ---- the plan of a product: tile and slices -----------------------------------------------------------------------------------
struct Plan { int mb, nb, slices; };
// The cheapest by estimate.  A round of tiles takes what its chunks take and some us to begin and end; what the epilogue reads and writes (`bytes` an
// element of C) goes at 4.5 TB/s, half of it beside the other workgroup's products where a CU holds two; sums of slices are written and read at that rate
// too.  us of a chunk fitted on products of 2744 to 4096 rows, K of 1024 to 9728, batches of 28: 256 x 256 (one workgroup a CU) 0.87, 192 x 256
// 0.79, 128 x 128 (two a CU) 0.54, gated 0.62; estimates within 15 % of what was measured, their order right in 13 of 14 pairs.  Slices of a symmetric product cost
// more than their join of 3 to 10 us, for their sums cross the diagonal once more: counted as 25 us in 16-bit types, 8 in fp32.  Orthogonalised updates with that | with 5 us |
// without such slices: 1024 x 1024 bf16 254 | 269 | 255 us, 2048 x 2048 405 | 448 | 406, 1024 x 4096 324 | 326 | 363, 512 x 8000 282 | 283 | 425, 2560 x 9728 1386 | 1418 | 1347,
// 2 x 2048 x 8192 1646 | 1626 | 1646; 1024 x 4096 fp32 780 | 780 | 950, 3 x 512 x 256 169 | 168 | 188.
struct Sizes {
  int64_t rows, cols, batches, n_chunks;
  bool symmetric, gated, strided;      // strided: one of the operands
  float bytes;
  int sliced = 16;                     // the epilogue's SLICED
};
template <typename T>
Plan plan_of(const Sizes& z) {
  struct Option { int mb, nb, resident; float chunk_us, gated_us; };      // resident: workgroups that a round has
  constexpr int N = sizeof(T) == 2 ? 3 : 2;
  static const Option half[] = {{4, 4, 256, 0.87f, 0.87f}, {3, 4, 256, 0.79f, 0.79f}, {2, 2, 512, 0.54f, 0.62f}}, full[] = {{2, 2, 512, 4.8f, 4.8f}, {1, 1, 768, 1.8f, 1.8f}};
  const float elements = (float)(z.batches * z.rows * z.cols);
  Plan best{0, 0, 1};
  float best_us = 3e38f;
  for (int i = 0; i < N; i++) {
    const Option& o = sizeof(T) == 2 ? half[i] : full[i];
    if ((z.gated && o.nb < 2) || (o.mb == 3 && z.strided) || (sizeof(T) == 2 && o.mb > 2 && z.symmetric)) continue;
    const int64_t ti = (z.rows + 64 * o.mb - 1) / (64 * o.mb), bn = z.gated ? 32 * o.nb : 64 * o.nb, tj = (z.cols + bn - 1) / bn;
    const int64_t tiles = (z.symmetric ? ti * (ti + 1) / 2 : ti * tj) * z.batches;
    const float epilogue = elements * z.bytes / 4.5e6f * (o.resident > 256 && tiles > o.resident ? 0.5f : 1.f);
    const int64_t most = o.mb * o.nb <= z.sliced ? std::min<int64_t>(std::max<int64_t>(z.n_chunks / 8, 1), 16) : 1;
    for (int s = 1; s <= most; s++) {
      const float sums = s == 1 ? 0.f : (z.symmetric ? sizeof(T) == 2 ? 25.f : 8.f : 5.f) + (float)s * elements * (z.gated ? 2.f : z.symmetric ? 0.5f : 1.f) * 8.f / 4.5e6f;
      const float us = (float)((tiles * s + o.resident - 1) / o.resident) * ((float)((z.n_chunks + s - 1) / s) * (z.gated ? o.gated_us : o.chunk_us) + 5.f) + epilogue + sums;
      if (us < best_us) best_us = us, best = {o.mb, o.nb, s};
    }
  }
  return best;
}
inline int64_t part_bytes(const Plan& p, int64_t rows, int64_t cols, int64_t batches, bool gated) {
  return p.slices > 1 ? p.slices * batches * rows * padded(cols) * (gated ? 2 : 1) * (int64_t)sizeof(float) : 0;
}
// By how many bytes the loads of a call's products reach beyond their operands, and their scalar offsets beyond their buffers: found with the kernel's own
// arithmetic over all tiles, in place of the launches, while a thread's `probe` is set.
struct Probe {
  int64_t buffers, offsets, products;
  struct Form {
    const char* kernel;
    int segments;
  } forms[8];                   // of the products that the call launches, the first eight
  int n_forms;
  void form(const char* kernel, int segments) {
    if (n_forms < 8) forms[n_forms++] = {kernel, segments};
  }
};
inline thread_local Probe* probe = nullptr;
template <typename T>
void find_overreach(const Product<T>& p, bool strided_a, bool strided_b, int rows_i, int rows_j, bool gated, int bytes) {
  const int64_t el = sizeof(T);
  probe->products++;
  auto operand = [&](bool strided, const Operand<T>& o, int tiles, int size, int64_t more, bool of_b, bool other) {
    for (int batch : {0, p.batches - 1})
      for (int seg = 0; seg < p.segments; seg++)
        for (int i = 0; i < tiles; i++) {
          const bool end = seg == p.segments - 1, second = of_b && p.u && (other || seg > 0);
          const Reach r = reach_of<T>(strided, o.ld, end ? o.last_rows : o.rows, end ? o.last_width : o.width, i * size, size);
          const int64_t at = batch * o.batch + seg * o.segment + r.begin + more - (second ? p.u - o.p : 0);
          const int n = chunks<T>(end ? p.last_k : p.k, bytes);
          probe->buffers = std::max({probe->buffers, -at * el, at * el + (int64_t)r.bytes - (second ? p.u_elements : o.elements) * el});
          // 64 bits beside what the kernel computes in 32
          const int64_t step = strided ? o.ld * bytes : bytes, rows = strided ? bytes / el : std::min<int64_t>(size, (end ? o.last_rows : o.rows) - i * size);
          const int64_t furthest = strided ? (bytes / el - 1) * o.ld * el + size * el : (rows - 1) * o.ld * el + bytes;
          if (furthest >= 1ll << 31 || (n - 1) * step >= 1ll << 32 || (int64_t)r.bytes < 0) probe->offsets = std::max<int64_t>(probe->offsets, 1ll << 32);
          probe->offsets = std::max(probe->offsets, (n - 1) * step + 1 - (int64_t)r.bytes);
        }
  };
  operand(strided_a, p.a, p.tiles_i, rows_i, 0, false, false);
  operand(strided_b, p.b, p.tiles_j, rows_j, 0, true, false);
  if (gated) operand(strided_b, p.b, p.tiles_j, rows_j, p.b2, true, true);
}
// A product by the plan's tile, or by the one that is built in its place: its tiles are counted for the kernel that runs, whatever the plan says.
template <typename T, bool TA, bool TB, typename EPI>
void launch(Product<T> p, const Plan& plan, const EPI& epi, hipStream_t s) {
  p.slices = plan.slices, p.group = 4;
  auto with = [&](auto mb, auto nb, auto r, auto cb) {
    constexpr int MB = decltype(mb)::value, NB = decltype(nb)::value, R = decltype(r)::value, CB = decltype(cb)::value, BM = 64 * MB, BN = EPI::GATED ? 32 * NB : 64 * NB;
    p.tiles_i = (p.rows + BM - 1) / BM, p.tiles_j = (p.cols + BN - 1) / BN;
    constexpr bool CUT = MB * NB <= EPI::SLICED;
    if (!CUT) p.slices = 1;
    if (probe) probe->form(p.slices > 1 ? form_of<T, TA, TB, MB, NB, R, CB, true, EPI>() : form_of<T, TA, TB, MB, NB, R, CB, false, EPI>(), p.segments);
    if (probe) return find_overreach(p, TA, TB, BM, BN, EPI::GATED, CB);
    if constexpr (CUT) {
      if (p.slices > 1) return go<T, TA, TB, MB, NB, R, CB, true>(p, epi, s);
    }
    go<T, TA, TB, MB, NB, R, CB, false>(p, epi, s);
  };
#define RL_I(x) std::integral_constant<int, x>()
  if constexpr (sizeof(T) == 2) {
    if constexpr (!EPI::SYMMETRIC) {
      if (plan.mb == 4) return with(RL_I(4), RL_I(4), std::integral_constant<int, TA || TB ? 4 : 2>(), std::integral_constant<int, TA || TB ? 64 : 128>());
    }
    if constexpr (!TA && !TB && !EPI::SYMMETRIC) {
      if (plan.mb == 3) return with(RL_I(3), RL_I(4), RL_I(4), RL_I(64));
    }
    // one workgroup a CU or fewer: nothing else covers the latency of its loads (512 x 512 orthogonalised 218 us with two stages, 209 with four; 1024 x 4096
    // 336 and 320, 2560 x 9728 1398 and 1374)
    const int64_t ti = (p.rows + 127) / 128, tj = (p.cols + (EPI::GATED ? 63 : 127)) / (EPI::GATED ? 64 : 128);
    if ((EPI::SYMMETRIC ? ti * (ti + 1) / 2 : ti * tj) * p.slices * p.batches <= 256) return with(RL_I(2), RL_I(2), RL_I(4), RL_I(128));
    with(RL_I(2), RL_I(2), RL_I(2), RL_I(128));
  } else {
    if constexpr (!EPI::GATED) {
      if (plan.mb == 1) return with(RL_I(1), RL_I(1), RL_I(2), RL_I(128));
    }
    with(RL_I(2), RL_I(2), RL_I(2), RL_I(128));
  }
#undef RL_I
}

}  // namespace product
