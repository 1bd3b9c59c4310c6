// Declarations shared by the translation units of the key cache and the
// selection (include/avsg_select.h).
#pragma once

#include "avsg_select.h"
#include "latent_internal.h"

namespace avsg {

constexpr int kIndexDim = AVSG_KEY_DIM;                   // codes of a key or query
constexpr int kKeyScaleAt = kIndexDim;                    // of a row: its scale
constexpr int kLanesPerKey = kIndexDim / 8;               // lanes that share a vector to quantise or read
constexpr int64_t kMostKeyVectors = kMostThreads / 256 * (256 / kLanesPerKey);

struct KeyAppendParams {
  CacheView cache;
  int64_t tokens, positions;
  const __bf16* key;
  int64_t key_stride;
  const int32_t* request;
  const int64_t* position;
  const float* angles;
  int32_t rope_at;          // -1: nothing is rotated
  int32_t heads;
  const __bf16* q;
  int64_t q_token_stride, q_head_stride;
  const float* weights;     // or nullptr
  int64_t weight_stride;
  int8_t* q_out;
  int64_t q_out_token_stride, q_out_head_stride;
  float* weights_out;
  int64_t weight_out_stride;
};

struct SelectParams {
  CacheView cache;
  int32_t n_q, heads, longest, topk;
  int32_t block_shift;      // log2 of the positions of a block
  int32_t first, recent;
  const int8_t* q;
  int64_t q_token_stride, q_head_stride;
  const float* weights;
  int64_t weight_stride;
  const int64_t* lens;      // or nullptr
  int32_t* index;
  float* out_scores;        // or nullptr
  float* scores;            // workspace: [tokens of a turn][score_stride]
  int64_t score_stride;     // blocks of a token's positions, rounded up to 16 bytes
  int32_t r0, g0, requests, tokens;   // a turn: tokens [g0, g0 + tokens) of requests [r0, r0 + requests)
};

// Positions that token g of request r sees.
__device__ __forceinline__ int seen_by(const SelectParams& p, int r, int g) {
  if (!p.lens) return p.longest;
  const int64_t n = p.lens[static_cast<int64_t>(r) * p.n_q + g];
  return n < 0 ? 0 : n < p.longest ? static_cast<int>(n) : p.longest;
}

hipError_t launch_key_append(const KeyAppendParams& p, int rope_style, hipStream_t s);
hipError_t launch_key_read(const ReadParams& p, hipStream_t s);
hipError_t launch_scores(const SelectParams& p, hipStream_t s);
hipError_t launch_best(const SelectParams& p, hipStream_t s);

}  // namespace avsg
