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

// How the scores of a turn are computed: by waves on their own (with `run` tiles of sixteen keys each), or by workgroups
// that share their keys (`run` stages of 64).
struct ScorePlan {
  bool shared;
  int32_t head_tiles;        // sixteen heads each: 1, 2, 4 or 8
  int32_t tokens;            // of a wave on its own, or of a workgroup
  int32_t groups;            // of so many tokens
  int32_t waves_on_tokens;   // waves of a workgroup that take different ones
  int32_t run, runs;         // what a wave or workgroup goes through, and how many of these the positions make
};

// The key that is read in place of `key` (a tile's or a stage's, of which some may lie past the last one that a token
// sees), and the tile of a run in whose page a tile's keys are read where none lies in two (tiles past the last are
// loaded, but not used).
__host__ __device__ inline int seen_key(int key, int most) { return key < most ? key : most - 1; }
__host__ __device__ inline int paged_tile(int tile, int tiles) { return tile < tiles ? tile : tiles - 1; }

hipError_t launch_key_append(const KeyAppendParams& p, int rope_style, hipStream_t s);
hipError_t launch_key_read(const ReadParams& p, hipStream_t s);
ScorePlan score_plan(int requests, int tokens, int heads, int longest);
hipError_t launch_scores(const SelectParams& p, hipStream_t s);
hipError_t launch_best(const SelectParams& p, hipStream_t s);

}  // namespace avsg

// score_plan for tests, which assert what their cases run: 100 * head_tiles + 10 * waves_on_tokens + tokens of a wave on
// its own, or 100 * head_tiles where they share their keys, in the low half, the run's length in the high one.  Not part of
// the ABI.
extern "C" int64_t avsg_internal_score_plan(int32_t requests, int32_t tokens, int32_t heads, int32_t longest);
// The position whose row lane `lane` of sixteen reads for tile `tile` of a run of `tiles` from first_key.  Likewise.
extern "C" int32_t avsg_internal_score_row(int32_t first_key, int32_t tiles, int32_t tile, int32_t lane, int32_t most, int32_t page_shift);
