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
