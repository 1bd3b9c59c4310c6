// Host side of the key cache and the selection (include/avsg_select.h): argument
// checks, the tokens' turns where the workspace does not hold all scores, launches.
#include "avsg_select.h"

#include <algorithm>

#include "select_internal.h"

using namespace avsg;

namespace {

// A key cache's view; its fields are those of an avsg_cache.
avsg_status view_of(const avsg_key_cache* c, CacheView* v) {
  if (!c || !c->base) return fail(AVSG_E_INVAL, "null cache or cache base");
  const avsg_cache same{c->base, c->pages, c->page_stride, c->row_stride, 0, c->batch, c->page_rows, c->pages_per_request, c->d_page_table};
  return view_of(&same, AVSG_KEY_ROW_BYTES, 4, v);
}

bool codes16(const void* p, int64_t token_stride, int64_t head_stride) {
  return p && aligned(p, 16) && (token_stride & 15) == 0 && (head_stride & 15) == 0;
}

// floats of a token's block scores
int64_t score_floats(int32_t longest, int32_t block) { return (static_cast<int64_t>(longest) / block + 3) & ~int64_t{3}; }

constexpr int32_t kMostPositions = 1 << 30;

bool takes(int32_t longest, int32_t block) {
  return longest >= 1 && longest <= kMostPositions && block >= 1 && block <= 128 && (block & (block - 1)) == 0 && longest % block == 0;
}

// Scores of more tokens than these are worked through in turns, so that they stay in the last cache
// between the kernel that writes them and the one that reads them.
constexpr int64_t kTurnBytes = int64_t{128} << 20;
// Positions of all tokens of a turn: 2^12 a workgroup of scores, 2^22 workgroups and one per token.
constexpr int64_t kTurnPositions = int64_t{1} << 34;

}  // namespace

extern "C" {

avsg_status avsg_key_append_rows(const avsg_key_cache* cache, const avsg_key_append* a, void* stream) {
  KeyAppendParams p{};
  if (avsg_status st = view_of(cache, &p.cache); st != AVSG_OK) return st;
  if (!a) return fail(AVSG_E_INVAL, "null append");
  if (a->tokens < 0 || a->heads < 0 || a->positions < 0)
    return fail(AVSG_E_INVAL, "tokens, heads and positions must not be negative");
  if (a->rope_style != AVSG_ROPE_PAIRS && a->rope_style != AVSG_ROPE_HALVES)
    return fail(AVSG_E_INVAL, "unknown rope_style %d", a->rope_style);
  if (a->rope_at != 0 && a->rope_at != 64 && a->rope_at != -1) return fail(AVSG_E_INVAL, "rope_at must be 0, 64 or -1");
  if (a->tokens == 0) return AVSG_OK;
  if (!rows16(a->d_key, a->key_stride))
    return fail(AVSG_E_INVAL, "d_key must be 16-byte aligned with a stride in multiples of 8 elements");
  if (!a->d_request || !a->d_position) return fail(AVSG_E_INVAL, "d_request and d_position are needed");
  if (a->rope_at >= 0 && (!a->d_angles || !aligned(a->d_angles, 16)))
    return fail(AVSG_E_INVAL, "d_angles (16-byte aligned) is needed where columns are rotated");
  if (a->heads > 0) {
    if (!rows16(a->d_q, a->q_token_stride) || (a->q_head_stride & 7) != 0)
      return fail(AVSG_E_INVAL, "d_q must be 16-byte aligned with strides in multiples of 8 elements");
    if (!codes16(a->d_q_out, a->q_out_token_stride, a->q_out_head_stride))
      return fail(AVSG_E_INVAL, "d_q_out must be 16-byte aligned with strides in multiples of 16 bytes");
    if (!a->d_weights_out || !aligned(a->d_weights_out, 4) || !aligned(a->d_weights, 4))
      return fail(AVSG_E_INVAL, "d_weights_out is needed, and weights must be 4-byte aligned");
  }
  if (a->tokens > kMostKeyVectors / (1 + static_cast<int64_t>(a->heads)))
    return fail(AVSG_E_RANGE, "tokens * (1 + heads) must be at most %lld", static_cast<long long>(kMostKeyVectors));
  p.tokens = a->tokens;
  p.positions = a->positions;
  p.key = static_cast<const __bf16*>(a->d_key);
  p.key_stride = a->key_stride;
  p.request = a->d_request;
  p.position = a->d_position;
  p.angles = a->d_angles;
  p.rope_at = a->rope_at;
  p.heads = a->heads;
  p.q = static_cast<const __bf16*>(a->d_q);
  p.q_token_stride = a->q_token_stride;
  p.q_head_stride = a->q_head_stride;
  p.weights = a->d_weights;
  p.weight_stride = a->weight_stride;
  p.q_out = static_cast<int8_t*>(a->d_q_out);
  p.q_out_token_stride = a->q_out_token_stride;
  p.q_out_head_stride = a->q_out_head_stride;
  p.weights_out = a->d_weights_out;
  p.weight_out_stride = a->weight_out_stride;
  return launched(launch_key_append(p, a->rope_style, static_cast<hipStream_t>(stream)), "avsg_key_append_rows");
}

avsg_status avsg_key_read_rows(const avsg_key_cache* cache, int64_t n, const int32_t* d_request, const int64_t* d_position,
                               void* d_out, int64_t out_stride, void* stream) {
  ReadParams p{};
  if (avsg_status st = view_of(cache, &p.cache); st != AVSG_OK) return st;
  if (n < 0) return fail(AVSG_E_INVAL, "n must not be negative");
  if (n == 0) return AVSG_OK;
  if (n > kMostKeyVectors) return fail(AVSG_E_RANGE, "n must be at most %lld", static_cast<long long>(kMostKeyVectors));
  if (!d_request || !d_position) return fail(AVSG_E_INVAL, "d_request and d_position are needed");
  if (!rows16(d_out, out_stride))
    return fail(AVSG_E_INVAL, "d_out must be 16-byte aligned with a stride in multiples of 8 elements");
  p.n = n;
  p.request = d_request;
  p.position = d_position;
  p.out = static_cast<__bf16*>(d_out);
  p.out_stride = out_stride;
  return launched(launch_key_read(p, static_cast<hipStream_t>(stream)), "avsg_key_read_rows");
}

size_t avsg_select_workspace_least(int32_t longest, int32_t block) {
  return takes(longest, block) ? static_cast<size_t>(score_floats(longest, block)) * sizeof(float) : 0;
}

size_t avsg_select_workspace_bytes(int32_t batch, int32_t n_q, int32_t longest, int32_t block) {
  const int64_t token = static_cast<int64_t>(avsg_select_workspace_least(longest, block));
  if (batch < 1 || n_q < 1 || token == 0) return 0;
  const int64_t tokens = static_cast<int64_t>(batch) * n_q;
  return static_cast<size_t>(std::min(tokens, std::max<int64_t>(1, kTurnBytes / token)) * token);
}

avsg_status avsg_select(const avsg_key_cache* cache, const avsg_selection* a, void* d_workspace, size_t workspace_bytes,
                        void* stream) {
  SelectParams p{};
  if (avsg_status st = view_of(cache, &p.cache); st != AVSG_OK) return st;
  if (!a) return fail(AVSG_E_INVAL, "null selection");
  if (a->n_q < 1 || a->heads < 1 || a->topk < 0 || a->longest < 0 || a->first < 0 || a->recent < 0)
    return fail(AVSG_E_INVAL, "n_q and heads must be positive, topk, longest, first and recent not negative");
  if (a->heads > AVSG_SELECT_HEADS_MOST) return fail(AVSG_E_RANGE, "heads must be at most %d", AVSG_SELECT_HEADS_MOST);
  if (a->block < 1 || a->block > 128 || (a->block & (a->block - 1)) != 0)
    return fail(AVSG_E_NOTPOW2, "block must be a power of two, 1 to 128");
  if (a->longest % a->block != 0 || a->topk % a->block != 0)
    return fail(AVSG_E_RANGE, "longest and topk must be multiples of block");
  // (keys past a run's end are counted in 32 bits)
  if (a->longest > kMostPositions) return fail(AVSG_E_RANGE, "longest must be at most 2^30");
  if (a->topk > a->longest) return fail(AVSG_E_RANGE, "topk must be at most longest");
  if (a->longest > p.cache.capacity) return fail(AVSG_E_CAPACITY, "longest is more than the rows of a request");
  const int64_t tokens = static_cast<int64_t>(cache->batch) * a->n_q;
  if (tokens > (1 << 19)) return fail(AVSG_E_RANGE, "batch * n_q must be at most 2^19");
  if (a->topk == 0) return AVSG_OK;
  if (!codes16(a->d_q, a->q_token_stride, a->q_head_stride))
    return fail(AVSG_E_INVAL, "d_q must be 16-byte aligned with strides in multiples of 16 bytes");
  if (!a->d_weights || !aligned(a->d_weights, 4) || !a->d_index || !aligned(a->d_index, 4) || !aligned(a->d_scores, 4))
    return fail(AVSG_E_INVAL, "d_weights and d_index are needed, and 4-byte aligned like d_scores");
  const int64_t floats = score_floats(a->longest, a->block), room = static_cast<int64_t>(workspace_bytes / sizeof(float)) / floats;
  if (!d_workspace || !aligned(d_workspace, 16) || room < 1)
    return fail(AVSG_E_INVAL, "the workspace must be 16-byte aligned and hold %zu bytes", static_cast<size_t>(floats) * sizeof(float));
  p.n_q = a->n_q;
  p.heads = a->heads;
  p.longest = a->longest;
  p.topk = a->topk;
  p.block_shift = __builtin_ctz(static_cast<unsigned>(a->block));
  p.first = a->first;
  p.recent = a->recent;
  p.q = static_cast<const int8_t*>(a->d_q);
  p.q_token_stride = a->q_token_stride;
  p.q_head_stride = a->q_head_stride;
  p.weights = a->d_weights;
  p.weight_stride = a->weight_stride;
  p.lens = a->d_lens;
  p.index = a->d_index;
  p.out_scores = a->d_scores;
  p.scores = static_cast<float*>(d_workspace);
  p.score_stride = floats;
  // turns of whole requests, or of some tokens of one; no more than a launch takes
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const int64_t most = std::min(room, std::max<int64_t>(1, kTurnPositions / a->longest));
  p.tokens = static_cast<int32_t>(std::min<int64_t>(a->n_q, most));
  p.requests = p.tokens < a->n_q ? 1 : static_cast<int32_t>(std::min<int64_t>(cache->batch, most / a->n_q));
  const int32_t by_r = p.requests, by_g = p.tokens;
  for (p.r0 = 0; p.r0 < cache->batch; p.r0 += by_r) {
    p.requests = std::min(by_r, cache->batch - p.r0);
    for (p.g0 = 0; p.g0 < a->n_q; p.g0 += by_g) {
      p.tokens = std::min(by_g, a->n_q - p.g0);
      if (avsg_status st = launched(launch_scores(p, s), "avsg_select"); st != AVSG_OK) return st;
      if (avsg_status st = launched(launch_best(p, s), "avsg_select"); st != AVSG_OK) return st;
    }
  }
  return AVSG_OK;
}

int64_t avsg_internal_score_plan(int32_t requests, int32_t tokens, int32_t heads, int32_t longest) {
  const ScorePlan p = score_plan(requests, tokens, heads, longest);
  const int how = 100 * p.head_tiles + (p.shared ? 0 : 10 * p.waves_on_tokens + p.tokens);
  return static_cast<int64_t>(how) | static_cast<int64_t>(p.run) << 32;
}

}  // extern "C"
