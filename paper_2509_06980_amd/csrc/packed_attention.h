// Attention over packed sequences: what its kernels share.
#pragma once
#include "policy_common.h"

// Sequence s: queries [cu_q[s], cu_q[s + 1]), keys [cu_k[s], cu_k[s + 1]).  Causal: query i of lq sees the keys j <= i + lk - lq,
// so the last query sees all of them and, where lq > lk, the first lq - lk see none.
struct PackedShape {
  const int32_t *cu_q, *cu_k;
  int n_seq, total_q, total_k;
  int nq, nkv, d;
  int64_t qt, qh, kt, kh, vt, vh, ot, oh;      // strides of token and head in elements; dO and the gradients are contiguous
  float scale;
  int causal;
};

// Tiles of `rows` rows of every sequence, numbered through without a list: the tiles of sequence s begin at floor(cu[s] / rows) + s,
// which leaves each sequence as many numbers as it needs (floor((a + n) / rows) + 1 >= floor(a / rows) + ceil(n / rows)) and some
// without a tile.  packed_tiles: how many numbers there are.  Whatever cu holds, what comes back lies inside [0, total].
struct PackedTile {
  int seq, first, len;      // first token of the sequence and its length, in the tiled tensor
  int row0;                 // first row of the tile within the sequence; >= len: no such tile
};
static inline __host__ __device__ int packed_tiles(int total, int n_seq, int rows) { return total / rows + n_seq; }
__device__ __forceinline__ int packed_bound(const int32_t* cu, int s, int total) {
  const int c = cu[s];
  return c < 0 ? 0 : c > total ? total : c;
}
__device__ __forceinline__ PackedTile packed_tile(const int32_t* cu, int n_seq, int total, int rows, int tile) {
  int lo = 0, hi = n_seq;      // sequence `lo` begins at or before the tile, `hi` behind it
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (packed_bound(cu, mid, total) / rows + mid <= tile) lo = mid;
    else hi = mid;
  }
  PackedTile t;
  t.seq = lo;
  t.first = packed_bound(cu, lo, total);
  const int end = packed_bound(cu, lo + 1, total);
  t.len = end > t.first ? end - t.first : 0;
  const int row0 = tile - (t.first / rows + lo);
  t.row0 = row0 < 0 ? t.len : row0 <= t.len / rows ? row0 * rows : t.len;
  return t;
}
// Tile `n` of up to 64 sequences, a lane each, those with most tiles of their sequence behind them first.
__device__ __forceinline__ PackedTile packed_tile_by_rest(const int32_t* cu, int n_seq, int total, int rows, int n) {
  const int lane = threadIdx.x & 63;
  const int first = lane < n_seq ? packed_bound(cu, lane, total) : 0, end = lane < n_seq ? packed_bound(cu, lane + 1, total) : 0;
  const int len = end > first ? end - first : 0, tiles = (len + rows - 1) / rows;
  int rest = tiles;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) rest = max(rest, __shfl_xor(rest, o, 64));
  PackedTile t{0, 0, 0, 0};
  for (rest = __builtin_amdgcn_readfirstlane(rest) - 1; rest >= 0; rest--) {
    const uint64_t on = __ballot(tiles > rest);
    const int count = __popcll(on);
    if (n < count) {
      const int s = __builtin_ctzll(__ballot((on >> lane & 1) && __popcll(on & ((1ull << lane) - 1)) == n));
      t.seq = s;
      t.first = __builtin_amdgcn_readlane(first, s);
      t.len = __builtin_amdgcn_readlane(len, s);
      t.row0 = (__builtin_amdgcn_readlane(tiles, s) - 1 - rest) * rows;
      break;
    }
    n -= count;
  }
  return t;
}

// Rows of no sequence, before the first one and behind the last: nothing was seen there and nothing depends on them, so o and the gradients are
// zeros and lse is -infinity.  All workgroups of a launch share them, whether they have a tile or not.  Two steps: the offsets are
// requested before the tile is looked up and waited for together with that (waited for on their own: 350 us for 16 sequences of
// 97 to 1511 in place of 346).
struct OutsideRows {
  int total, before, after;      // rows [0, before) and [after, total)
  __device__ __forceinline__ OutsideRows(const int32_t* cu, int n_seq, int all) : total(all), before(cu[0]), after(cu[n_seq]) {}
  // a (and b, unless null): contiguous rows of `width` elements; lse (unless null): [heads][total]
  template <typename T>
  __device__ __forceinline__ void clear(int width, T* a, T* b, float* lse, int heads) const {
    const int first = min(max(before, 0), total), behind = max(min(after, total), first);
    const uint64_t rows = (uint64_t)(first + (total - behind)), step = (uint64_t)gridDim.x * gridDim.y * gridDim.z;
    for (uint64_t i = blockIdx.x + (uint64_t)gridDim.x * (blockIdx.y + (uint64_t)gridDim.y * blockIdx.z); i < rows; i += step) {
      const int64_t t = (int64_t)i < first ? (int64_t)i : behind + ((int64_t)i - first);
      for (int c = threadIdx.x; c < width; c += blockDim.x) {
        st1(a + t * width + c, 0.f);
        if (b) st1(b + t * width + c, 0.f);
      }
      if (lse)
        for (int h = threadIdx.x; h < heads; h += blockDim.x) lse[(int64_t)h * total + t] = -INFINITY;
    }
  }
};

// dk and dv of few key tiles: each tile's (query head, query tile) pairs are dealt to `n` workgroups, whose sums another kernel adds up in
// their order.  sums: [n][dk, dv][total_k][nkv][d].
struct KeyParts {
  int n;
  float* sums;
  __device__ __forceinline__ float* of(const PackedShape& p, int part, int which) const {
    return sums + (int64_t)(part * 2 + which) * p.total_k * p.nkv * p.d;
  }
};
// Parts for about `workgroups` in all, each with eight pairs of 64 queries on average or more.
static inline int key_parts(const PackedShape& p, int workgroups) {
  const int64_t tiles = (int64_t)packed_tiles(p.total_k, p.n_seq, 64) * p.nkv;
  const int64_t pairs = (int64_t)(p.nq / p.nkv) * ((p.total_q / (p.n_seq > 0 ? p.n_seq : 1) + 63) / 64);
  const int64_t n = workgroups / (tiles > 0 ? tiles : 1) < pairs / 8 ? workgroups / (tiles > 0 ? tiles : 1) : pairs / 8;
  return n < 2 ? 1 : n < 32 ? (int)n : 32;
}

// bf16 on matrix instructions: head sizes in multiples of 8, 16-byte aligned rows, nothing beyond 2 GB in one tensor, no more (tile, head) than
// a launch takes (2^19 sequences of 32 heads; the other kernels have the heads in a dimension of their own).  o and dout are
// checked for their alignment alone (null: not in the call).
bool attention_takes_mfma(const PackedShape& p, const void* q, const void* k, const void* v, const void* o, const void* dout);
void launch_attention_mfma_forward(hipStream_t s, const PackedShape& p, const bf16_t* q, const bf16_t* k, const bf16_t* v, bf16_t* o,
                                   float* lse);
void launch_attention_mfma_backward(hipStream_t s, const PackedShape& p, const bf16_t* dout, const bf16_t* q, const bf16_t* k,
                                    const bf16_t* v, const bf16_t* o, const float* lse, bf16_t* dq, bf16_t* dk, bf16_t* dv,
                                    float* stats, const KeyParts& parts);      // stats: 2 floats a query and head
