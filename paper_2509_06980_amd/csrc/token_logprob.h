// Log-probs of tokens from hidden rows and the lm-head, and their gradient: what the kernels share.
#pragma once
#include "policy_common.h"

// The rows that take part are gathered to the front; how many there are only the device knows.
struct KeptRows {
  const int32_t* count;      // kept rows
  const int32_t* target;     // [rows padded] target of a kept row, -1 in the padding
  const float* lse;          // backward: log-sum-exp of a kept row
  const float* g;            // backward: gradient of its log-prob / temperature, 0 in the padding
};
// Padding of the kept rows: zeros up to a multiple of this.
const int kRowPad = 256;
// One product of the backward pass over `width` tokens of the vocabulary from v0 on; dz [row][ld] holds the gradients of its logits.
struct VocabPiece {
  int v0, width, ld;
};

// ---- bf16 on matrix instructions: hidden in multiples of 8, 16-byte aligned weights, nothing beyond 4 GB in one operand ----------
// h: kept rows [padded][ld]; `rows`: an upper bound of how many they are.  width: vocabulary of a piece (forward: 0).
bool token_logprob_takes_mfma(int64_t padded, int ld, int hidden, int width, const void* weight, const void* dweight);
const int kStripMfma = 256;      // tokens of the vocabulary that one (max, sum) pair covers
void launch_logits_strips_mfma(hipStream_t s, const bf16_t* h, int ld, int rows, int64_t padded, const bf16_t* w, int vocab, int hidden,
                               const KeptRows& kept, float inv_t, float2* part, float* zt);
void launch_logits_gradient_mfma(hipStream_t s, const bf16_t* h, int ld, int rows, int64_t padded, const bf16_t* w, int vocab, int hidden,
                                 const KeptRows& kept, float inv_t, const VocabPiece& piece, bf16_t* dz);
// K-slices of dz W that suit `rows` rows
int token_logprob_slices(int rows, int hidden, int width);
void launch_hidden_gradient_mfma(hipStream_t s, const bf16_t* dz, const VocabPiece& piece, int rows, int64_t padded, const bf16_t* w, int vocab,
                                 int hidden, const KeptRows& kept, int slices, int per_slice, float* dh, size_t slice_stride, bool first);
void launch_weight_gradient_mfma(hipStream_t s, const bf16_t* dz, const VocabPiece& piece, const bf16_t* h, int ld, int64_t padded, int hidden,
                                 const KeptRows& kept, bf16_t* dw);
