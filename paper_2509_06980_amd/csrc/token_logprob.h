// Log-probs of tokens from hidden rows and the lm-head, and their gradient: what the kernels share.
#pragma once
#include "policy_common.h"

// K-slices of the product dz W: the device chooses them, since it alone knows how many rows are kept.
struct SliceRule {
  int rows, tiles_j, width, most;      // rows of a tile, tiles along hidden, vocabulary of a piece, slices that there is room for
  float chunk_us, slice_us;            // time of a tile's 32 k; of writing and reading a slice's sums of one row
};
// The number of slices that ends first: a round of tiles on 256 CUs takes what its k take and 6 us to begin and end.
static __host__ __device__ __forceinline__ int choose_slices(const SliceRule& r, int kept) {
  const int tiles = (kept + r.rows - 1) / r.rows * r.tiles_j;
  float best = 3e38f;
  int slices = 1;
  for (int s = 1; s <= r.most; s++) {
    const float t = (float)((tiles * s + 255) / 256) * ((float)r.width / (float)(32 * s) * r.chunk_us + 6.f) + (float)s * (float)kept * r.slice_us;
    if (t < best) best = t, slices = s;
  }
  return slices;
}
// Vocabulary of a slice
static __host__ __device__ __forceinline__ int slice_width(const SliceRule& r, int slices) { return ((r.width + slices - 1) / slices + 63) / 64 * 64; }
// The rows that take part are gathered to the front; how many there are only the device knows.
struct KeptRows {
  const int32_t* count;      // kept rows; backward also [1]: K-slices of dz W, [2]: vocabulary of one (multiple of 64)
  const int32_t* target;     // [rows padded] target of a kept row, -1 in the padding
  const float* lse;          // backward: log-sum-exp of a kept row
  const float* g;            // backward: gradient of its log-prob / temperature, 0 in the padding
  int twins;                 // backward: as twins_of says
};
// Backward in bf16 with up to 64 rows: row twins + r is row r once more and holds what the rounding of its dz left, so that both products
// behind see dz in 16 bits (relative error of both gradients 0.0017, that of their last rounding).  Without it they were 0.0020 to 0.0028
// off: few rows do not average the rounding of a row's largest element, its target's.  The bound of 64 is one of cost alone: twice as many
// rows still fit one tile and cost next to nothing (64 x 2560 x 20000, both directions, 152 us with and without; 30 x 4096 x 151936 1.12
// ms, without 1.08), beyond it they would double the products.  From 65 rows on the gradients are 0.0023 to 0.0024 off, less exact than those of
// 64.
static inline int twins_of(int rows, bool bf16) { return !bf16 || rows > 64 ? 0 : rows > 32 ? 64 : rows > 16 ? 32 : 16; }
static __device__ __forceinline__ float rounding_left(float v) {
  const float left = v - (float)(__bf16)v;
  return left == left ? left : 0.f;      // infinite or no number: in the row itself
}
// Padding of the kept rows: zeros up to a multiple of this.
const int kRowPad = 256;
// One product of the backward pass over `width` tokens of the vocabulary from v0 on; dz [row][ld] holds the gradients of its logits.
struct VocabPiece {
  int v0, width, ld;
};

// ---- matrix instructions with operands straight from memory: hidden in whole 16 bytes, 16-byte aligned weights, nothing beyond 4 GB in
// one operand -------------------------------------------------------------------------------------
// h: kept rows [padded][ld]; `rows`: an upper bound of how many they are.  width: row length of dz (forward: 0).
template <typename T>
bool token_logprob_takes_mfma(int64_t padded, int ld, int hidden, int width, const void* weight, const void* dweight);
// Returns how many strips of the vocabulary it leaves a (max, sum) pair for, 64 tokens each or more.
template <typename T>
int launch_logits_strips_mfma(hipStream_t s, const T* h, int ld, int rows, int64_t padded, const T* w, int vocab, int hidden,
                              const KeptRows& kept, float inv_t, float2* part, float* zt);
template <typename T>
void launch_logits_gradient_mfma(hipStream_t s, const T* h, int ld, int rows, int64_t padded, const T* w, int vocab, int hidden,
                                 const KeptRows& kept, float inv_t, const VocabPiece& piece, T* dz);
// Tile of dz W and its time
template <typename T>
void token_logprob_slice_tile(int rows, int hidden, int width, SliceRule& r);
template <typename T>
void launch_hidden_gradient_mfma(hipStream_t s, const T* dz, const VocabPiece& piece, int rows, int64_t padded, const T* w, int vocab, int hidden,
                                 const KeptRows& kept, int most_slices, float* dh, size_t slice_stride, bool first);
template <typename T>
void launch_weight_gradient_mfma(hipStream_t s, const T* dz, const VocabPiece& piece, const T* h, int ld, int64_t padded, int hidden,
                                 const KeptRows& kept, T* dw);

// ---- the same arithmetic on the host: what the loads and stores of a call's products would reach ------------------------------------
struct Extent { int64_t base, bytes; };
// By how many bytes at most, 0: not at all: buffers beyond their operands, scalar offsets beyond their buffers, stores beyond the results
struct LoadOverreach { int64_t buffers, offsets, stores; };
struct LogprobSizes {
  int rows, kept, hidden, vocab, backward;      // kept: as counted on the device
  int64_t padded;
  int ld, strips, width, ldz, most_slices, slices, per_slice;
};
template <typename T>
LoadOverreach token_logprob_overreach(const LogprobSizes& n);
