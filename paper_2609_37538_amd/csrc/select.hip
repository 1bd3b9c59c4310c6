// Scores of the key cache's positions for a step's query tokens, and the best
// of them.
#include <algorithm>

#include "select_internal.h"

namespace avsg {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4_at_4 __attribute__((ext_vector_type(4), aligned(4)));

constexpr int kWaves = 4;      // of a workgroup of scores
constexpr int kTileKeys = 16;  // keys that a matrix instruction takes

struct F64Pair {
  double a, b;
};
// Exchanges the odd rows of sixteen lanes of a with the even rows of b, or (kHalf) a's upper half with b's lower one.
template <bool kHalf>
__device__ __forceinline__ F64Pair swap_rows(double a, double b) {
  const uint64_t x = __builtin_bit_cast(uint64_t, a), y = __builtin_bit_cast(uint64_t, b);
  uint32_t lo[2], hi[2];
  if constexpr (kHalf) {
    const auto l = __builtin_amdgcn_permlane32_swap(static_cast<uint32_t>(x), static_cast<uint32_t>(y), false, false);
    const auto h = __builtin_amdgcn_permlane32_swap(static_cast<uint32_t>(x >> 32), static_cast<uint32_t>(y >> 32), false, false);
    lo[0] = l[0], lo[1] = l[1], hi[0] = h[0], hi[1] = h[1];
  } else {
    const auto l = __builtin_amdgcn_permlane16_swap(static_cast<uint32_t>(x), static_cast<uint32_t>(y), false, false);
    const auto h = __builtin_amdgcn_permlane16_swap(static_cast<uint32_t>(x >> 32), static_cast<uint32_t>(y >> 32), false, false);
    lo[0] = l[0], lo[1] = l[1], hi[0] = h[0], hi[1] = h[1];
  }
  return {__builtin_bit_cast(double, static_cast<uint64_t>(hi[0]) << 32 | lo[0]),
          __builtin_bit_cast(double, static_cast<uint64_t>(hi[1]) << 32 | lo[1])};
}

// Sums over the four rows of sixteen lanes; row i gets that of x[i % kCount].
template <int kCount>
__device__ __forceinline__ double row_sums(const double (&x)[kCount]) {
  static_assert(kCount == 2 || kCount == 4);
  const F64Pair u = swap_rows<false>(x[0], x[1]);
  const double s = u.a + u.b;   // rows 0 and 2: halves of x[0], rows 1 and 3 of x[1]
  double t = s;
  if constexpr (kCount == 4) {
    const F64Pair w = swap_rows<false>(x[2], x[3]);
    t = w.a + w.b;
  }
  const F64Pair v = swap_rows<true>(s, t);
  return v.a + v.b;
}

// The largest over groups of 2^shift lanes (at most 16).
__device__ __forceinline__ float group_max(float x, int shift) {
  auto with = [&](auto other) { x = fmaxf(x, __builtin_bit_cast(float, other)); };
  const auto bits = [&] { return __builtin_bit_cast(int, x); };
  if (shift > 0) with(__builtin_amdgcn_update_dpp(0, bits(), 0xb1, 0xf, 0xf, true));    // lanes 1 0 3 2
  if (shift > 1) with(__builtin_amdgcn_update_dpp(0, bits(), 0x4e, 0xf, 0xf, true));    // lanes 2 3 0 1
  if (shift > 2) with(__builtin_amdgcn_update_dpp(0, bits(), 0x141, 0xf, 0xf, true));   // mirrored within eight
  if (shift > 3) with(__builtin_amdgcn_update_dpp(0, bits(), 0x140, 0xf, 0xf, true));   // mirrored within sixteen
  return x;
}

// A wave scores kTok tokens of a request against a run of keys, sixteen at a time.  The matrix instruction
// (16 x 64 by 64 x 16, 8-bit) multiplies sixteen heads' queries with sixteen keys: lane l holds head, or
// key, l % 16 and columns (l / 16) * 32 .. + 31 in two instructions, and gets the products of heads (l / 16) *
// 4 .. + 3 with key l % 16.  The queries and their weights (in 64 bits) stay in registers.
// kWhole: a tile's keys lie in one page.
template <int kTiles, int kTok, bool kWhole>
__global__ __launch_bounds__(kWaves * 64, 2) void score_kernel(SelectParams p, int run_tiles, int runs, int groups, int waves_on_tokens) {
  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int waves_on_keys = kWaves / waves_on_tokens, run_groups = (runs + waves_on_keys - 1) / waves_on_keys;
  const int token_groups = (groups + waves_on_tokens - 1) / waves_on_tokens;
  const int run = static_cast<int>(blockIdx.x % run_groups) * waves_on_keys + wave / waves_on_tokens;
  const int rest = static_cast<int>(blockIdx.x / run_groups);
  const int group = rest % token_groups * waves_on_tokens + wave % waves_on_tokens, r = p.r0 + rest / token_groups;
  if (run >= runs || group >= groups) return;
  int token[kTok], seen[kTok], most = 0;   // tokens past the last are its copies
#pragma unroll
  for (int t = 0; t < kTok; ++t) {
    token[t] = p.g0 + min(group * kTok + t, p.tokens - 1);
    seen[t] = seen_by(p, r, token[t]);
    most = max(most, seen[t]);
  }
  const int first_key = run * run_tiles * kTileKeys;
  const int tiles = min(run_tiles, (most - first_key + kTileKeys - 1) / kTileKeys);
  if (first_key >= most) return;

  i32x4 q[kTok][kTiles][2];
  double weight[kTok][kTiles][4];
#pragma unroll
  for (int t = 0; t < kTok; ++t) {
    const int64_t at = static_cast<int64_t>(r) * p.n_q + token[t];
    const int8_t* from = p.q + at * p.q_token_stride + quad * 32;
    const float* weights = p.weights + at * p.weight_stride;
#pragma unroll
    for (int x = 0; x < kTiles; ++x) {
      const int8_t* row = from + min(x * 16 + l16, p.heads - 1) * p.q_head_stride;
      q[t][x][0] = *reinterpret_cast<const i32x4*>(row);
      q[t][x][1] = *reinterpret_cast<const i32x4*>(row + 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int h = x * 16 + quad * 4 + i;
        const float w = weights[min(h, p.heads - 1)];
        weight[t][x][i] = h < p.heads ? static_cast<double>(w) : 0.0;
      }
    }
  }

  struct Keys {
    i32x4 codes[2];
    float scale;
    bool there;   // or it is not the row's
  };
  // A run has at most 64 tiles: where a tile lies in one page, lane l holds the page of tile l.
  const int64_t first_page = static_cast<int64_t>(r) * p.cache.pages_per_request;
  auto page_of = [&](int key) {
    const int64_t at = first_page + (key >> p.cache.page_shift);
    const int page = p.cache.table ? p.cache.table[at] : static_cast<int>(at);
    return page < p.cache.pages ? page : -1;
  };
  const int pages = kWhole ? page_of(min(first_key + lane * kTileKeys, most - 1)) : 0;
  const int64_t in_row = quad * 32, to_scale = kKeyScaleAt - quad * 32;
  // (No branch: a wave that may skip a load has to wait for all of them;
  // and nothing is done with a loaded value here, which would wait for it.  Keys past the last one that is seen read as
  // it; in place of rows that do not exist the pool's first one is read.)
  auto fetch = [&](int tile) {
    Keys k;
    const int key = min(first_key + tile * kTileKeys + l16, most - 1);
    const int page = kWhole ? __builtin_amdgcn_readlane(pages, min(tile, tiles - 1)) : page_of(key);
    const bool there = page >= 0;
    uint64_t row = p.cache.base + (there ? page * p.cache.page_stride : 0);
    row += (there ? key & p.cache.page_mask : 0) * p.cache.row_stride + in_row;
    k.codes[0] = load_global<i32x4_at_4>(row);
    k.codes[1] = load_global<i32x4_at_4>(row + 16);
    k.scale = load_global<float>(row + to_scale);
    k.there = there;
    return k;
  };
  // Of a pair of tiles, the lanes of row i of sixteen end up with token i % kTok and tile i / kTok % 2.
  const int mine = quad % kTok, my_tile = quad / kTok & 1, my_seen = kTok > 1 && mine ? seen[kTok - 1] : seen[0];
  const int shift = p.block_shift, in_token = group * kTok + mine;
  const bool stores = quad < 2 * kTok && in_token < p.tokens;
  float* const out = p.scores + (static_cast<int64_t>(r - p.r0) * p.tokens + min(in_token, p.tokens - 1)) * p.score_stride;
  float best = -__builtin_inff();   // of a block of more than sixteen positions
  auto meet = [&](const Keys (&pair)[2], int tile) {
    double sum[2 * kTok];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int t = 0; t < kTok; ++t) {
        i32x4 dot[kTiles];
#pragma unroll
        for (int x = 0; x < kTiles; ++x) dot[x] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q[t][x][0], pair[u].codes[0], i32x4{}, 0, 0, 0);
#pragma unroll
        for (int x = 0; x < kTiles; ++x) dot[x] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q[t][x][1], pair[u].codes[1], dot[x], 0, 0, 0);
        double& s = sum[u * kTok + t];
        s = 0.0;
#pragma unroll
        for (int x = 0; x < kTiles; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i) s = __builtin_fma(weight[t][x][i], static_cast<double>(max(dot[x][i], 0)), s);
      }
    const float scale = my_tile ? pair[1].scale : pair[0].scale;
    const bool there = my_tile ? pair[1].there : pair[0].there;
    // (zeros of either sign are one)
    float score = static_cast<float>(row_sums<2 * kTok>(sum) * static_cast<double>(scale)) + 0.0f;
    const int key = first_key + (tile + my_tile) * kTileKeys + l16;
    if (!there || !(score == score)) score = -__builtin_inff();
    if (key < p.first || key >= my_seen - p.recent) score = __builtin_inff();
    if (key >= my_seen) score = -__builtin_inff();
    if (shift == 0) {
      if (stores && key < most) out[key] = score;
      return;
    }
    score = group_max(score, shift);
    if (shift <= 4) {
      if (stores && (l16 & ((1 << shift) - 1)) == 0 && key < most) out[key >> shift] = score;
    } else {
      best = fmaxf(best, score);
      if (((tile + 2) & ((1 << (shift - 4)) - 1)) == 0 || tile + 2 >= tiles) {
        best = fmaxf(best, __shfl_xor(best, 16 * kTok));
        if (stores && my_tile == 0 && l16 == 0) out[key >> shift] = best;
        best = -__builtin_inff();
      }
    }
  };
  Keys one[2], two[2];
  one[0] = fetch(0), one[1] = fetch(1), two[0] = fetch(2), two[1] = fetch(3);
  for (int tile = 0; tile < tiles; tile += 4) {
    meet(one, tile);
    one[0] = fetch(tile + 4), one[1] = fetch(tile + 5);
    if (tile + 2 >= tiles) break;
    meet(two, tile + 2);
    two[0] = fetch(tile + 6), two[1] = fetch(tile + 7);
  }
}

// Chunks of a prompt: a workgroup scores kChunkWaves tokens of a request, one per wave, against a run of keys that
// they share in LDS, 64 keys at a time, while the next ones are on their way.
constexpr int kChunkWaves = 8;
constexpr int kStageKeys = 64;
constexpr int kStagedRow = 144;   // bytes of a row in LDS: its codes, its scale; sixteen rows' sixteen bytes are in banks of their own
template <int kTiles>
__global__ __launch_bounds__(kChunkWaves * 64, kTiles > 4 ? 2 : 4) void chunk_kernel(SelectParams p, int run_stages, int runs, int groups) {
  __shared__ __align__(16) unsigned char staged[2][kStageKeys * kStagedRow];
  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int run = static_cast<int>(blockIdx.x % runs), rest = static_cast<int>(blockIdx.x / runs);
  const int group = rest % groups, r = p.r0 + rest / groups;
  int most = 0, seen = 0;
  for (int w = 0; w < kChunkWaves; ++w) {
    const int t = group * kChunkWaves + w, n = t < p.tokens ? seen_by(p, r, p.g0 + t) : 0;
    most = max(most, n);
    if (w == wave) seen = n;   // none of a token past the last
  }
  const int first_key = run * run_stages * kStageKeys;
  if (first_key >= most) return;
  const int stages = min(run_stages, (most - first_key + kStageKeys - 1) / kStageKeys);
  const int in_token = min(group * kChunkWaves + wave, p.tokens - 1);

  i32x4 q[kTiles][2];
  double weight[kTiles][4];
  {
    const int64_t at = static_cast<int64_t>(r) * p.n_q + p.g0 + in_token;
    const int8_t* from = p.q + at * p.q_token_stride + quad * 32;
    const float* weights = p.weights + at * p.weight_stride;
#pragma unroll
    for (int x = 0; x < kTiles; ++x) {
      const int8_t* row = from + min(x * 16 + l16, p.heads - 1) * p.q_head_stride;
      q[x][0] = *reinterpret_cast<const i32x4*>(row);
      q[x][1] = *reinterpret_cast<const i32x4*>(row + 16);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int h = x * 16 + quad * 4 + i;
        const float w = weights[min(h, p.heads - 1)];
        weight[x][i] = h < p.heads ? static_cast<double>(w) : 0.0;
      }
    }
  }
  // eight threads per row
  static_assert(kChunkWaves * 64 == kStageKeys * 8);
  const int my_row = threadIdx.x / 8, my_part = threadIdx.x % 8 * 16;
  i32x4 part;
  float part_scale;
  bool part_there;
  auto load = [&](int stage) {
    const int key = min(first_key + stage * kStageKeys + my_row, most - 1);
    const int64_t at = static_cast<int64_t>(r) * p.cache.pages_per_request + (key >> p.cache.page_shift);
    const int page = p.cache.table ? p.cache.table[at] : static_cast<int>(at);
    part_there = page >= 0 && page < p.cache.pages;
    const uint64_t row = p.cache.base + (part_there ? page * p.cache.page_stride + (key & p.cache.page_mask) * p.cache.row_stride : 0);
    part = load_global<i32x4_at_4>(row + my_part);
    part_scale = load_global<float>(row + kKeyScaleAt);
  };
  auto leave = [&](int buffer) {
    unsigned char* const to = staged[buffer] + my_row * kStagedRow;
    *reinterpret_cast<i32x4*>(to + my_part) = part;
    if (my_part == 0) *reinterpret_cast<float*>(to + kKeyScaleAt) = part_there ? part_scale : __uint_as_float(0x7fc00000u);
  };
  auto meet_all = [&] {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
  };
  const int shift = p.block_shift;
  float* const out = p.scores + (static_cast<int64_t>(r - p.r0) * p.tokens + in_token) * p.score_stride;
  float best = -__builtin_inff();   // of a block of 128 positions
  load(0);
  leave(0);
  meet_all();
  for (int stage = 0; stage < stages; ++stage) {
    const int stage_key = first_key + stage * kStageKeys;
    load(stage + 1);
    if (stage_key < seen) {
      const unsigned char* const from = staged[stage & 1];
      double sum[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        i32x4 keys[2], dot[kTiles];
#pragma unroll
        for (int h = 0; h < 2; ++h)
          keys[h] = *reinterpret_cast<const i32x4*>(from + (u * kTileKeys + l16) * kStagedRow + quad * 32 + h * 16);
#pragma unroll
        for (int x = 0; x < kTiles; ++x) dot[x] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q[x][0], keys[0], i32x4{}, 0, 0, 0);
#pragma unroll
        for (int x = 0; x < kTiles; ++x) dot[x] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q[x][1], keys[1], dot[x], 0, 0, 0);
        sum[u] = 0.0;
#pragma unroll
        for (int x = 0; x < kTiles; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[u] = __builtin_fma(weight[x][i], static_cast<double>(max(dot[x][i], 0)), sum[u]);
      }
      // row i of sixteen lanes gets the sums of tile i: lane l has key l of the stage
      const float scale = *reinterpret_cast<const float*>(from + lane * kStagedRow + kKeyScaleAt);
      float score = static_cast<float>(row_sums<4>(sum) * static_cast<double>(scale)) + 0.0f;
      const int key = stage_key + lane;
      if (!(score == score)) score = -__builtin_inff();
      if (key < p.first || key >= seen - p.recent) score = __builtin_inff();
      if (key >= seen) score = -__builtin_inff();
      if (shift == 0) {
        if (key < seen) out[key] = score;
      } else {
        score = group_max(score, shift);
        if (shift > 4) score = fmaxf(score, __shfl_xor(score, 16));
        if (shift > 5) score = fmaxf(score, __shfl_xor(score, 32));
        if (shift <= 6) {
          if ((lane & ((1 << shift) - 1)) == 0 && key < seen) out[key >> shift] = score;
        } else {
          best = fmaxf(best, score);
          if ((stage & 1) != 0 || stage_key + kStageKeys >= seen || stage + 1 == stages) {
            if (lane == 0) out[key >> shift] = best;
            best = -__builtin_inff();
          }
        }
      }
    }
    leave((stage + 1) & 1);
    meet_all();
  }
}

// Bits that order as the floats do (none of which is NaN), and back.
__device__ __forceinline__ uint32_t ordered(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float unordered(uint32_t u) { return __uint_as_float(u ^ (u >> 31 ? 0x80000000u : 0xffffffffu)); }
constexpr uint32_t kLowest = 0x007fffffu, kHighest = 0xff800000u;   // ordered(-inf), ordered(inf)

constexpr int kBins = 2048;
constexpr int kFew = 512;   // scores of a bin that are compared with each other

// What a workgroup picks from: the scores of a token's blocks; those of a segment of them; or what the
// segments' workgroups left, in the blocks' order.
enum class From { kScores, kSegment, kSegments };

// The best blocks of a token, one workgroup per token (or segment).  The threshold lies in one of 2048 bins of
// equal width between the smallest and the largest finite score, the scores of that bin are compared
// with each other, and the blocks above the threshold, and the lowest of those at it, are written in
// their order.  Where the bin holds many, or the scores are too far apart for such bins, histograms of
// their bits narrow the range down until a bin holds one value or all that is wanted.
// kResident: the scores stay in registers, else every pass reads them again.
template <int kThreads, int kPer, bool kResident, From kFrom>
__global__ __launch_bounds__(kThreads) void best_kernel(SelectParams p) {
  constexpr int kWavesHere = kThreads / 64, kChunk = kThreads * kPer, kCounts = kPer * kWavesHere;
  static_assert(kCounts <= kThreads && kBins % kThreads == 0 && kFew <= kBins);
  __shared__ uint32_t hist[kBins];
  __shared__ uint32_t above_counts[kCounts], equal_counts[kCounts];
  __shared__ uint32_t parts[4][kWavesHere];
  __shared__ uint32_t found[3];
  __shared__ uint32_t few_count;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = kFrom == From::kSegment ? static_cast<int>(blockIdx.x) / p.segments : static_cast<int>(blockIdx.x);
  const int r = p.r0 + row / p.tokens, g = p.g0 + row % p.tokens;
  const int shift = p.block_shift, wanted = p.topk >> shift;   // of the token
  const uint32_t blocks = p.longest >> shift;
  const uint32_t first = kFrom == From::kSegment ? blockIdx.x % p.segments * p.segment : 0;
  const uint32_t n = kFrom == From::kSegments ? static_cast<uint32_t>(p.candidates) : kFrom == From::kSegment ? min(blocks - first, p.segment) : blocks;
  const uint32_t want = kFrom == From::kSegment ? min(n, static_cast<uint32_t>(wanted)) : wanted;
  const uint32_t in_reach = (static_cast<uint32_t>(seen_by(p, r, g)) + (1u << shift) - 1) >> shift;
  const uint32_t seen = kFrom == From::kSegments ? n : in_reach > first ? min(in_reach - first, n) : 0;
  const float* const scores = kFrom == From::kSegments ? p.candidate_scores + static_cast<int64_t>(row) * p.candidates
                                                       : p.scores + row * p.score_stride + first;
  const int chunks = kResident ? 1 : static_cast<int>((n + kChunk - 1) / kChunk);
  auto load = [&](int chunk, int j) {
    const uint32_t i = static_cast<uint32_t>(chunk) * kChunk + j * kThreads + tid;
    return i < seen ? ordered(scores[i]) : i < n ? kLowest : 0u;
  };
  uint32_t held[kPer];
  if constexpr (kResident) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) held[j] = load(0, j);
  }
  auto each = [&](auto f) {
    for (int chunk = 0; chunk < chunks; ++chunk)
#pragma unroll
      for (int j = 0; j < kPer; ++j) f(kResident ? held[j] : load(chunk, j));
  };
  // over the workgroup: smallest, largest, and two sums
  auto reduced = [&](uint32_t& lo, uint32_t& hi, uint32_t& x, uint32_t& y) {
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) {
      lo = min(lo, static_cast<uint32_t>(__shfl_xor(static_cast<int>(lo), d)));
      hi = max(hi, static_cast<uint32_t>(__shfl_xor(static_cast<int>(hi), d)));
      x += static_cast<uint32_t>(__shfl_xor(static_cast<int>(x), d));
      y += static_cast<uint32_t>(__shfl_xor(static_cast<int>(y), d));
    }
    __syncthreads();
    if (lane == 0) parts[0][wave] = lo, parts[1][wave] = hi, parts[2][wave] = x, parts[3][wave] = y;
    __syncthreads();
    lo = 0xffffffffu, hi = x = y = 0;
#pragma unroll
    for (int w = 0; w < kWavesHere; ++w)
      lo = min(lo, parts[0][w]), hi = max(hi, parts[1][w]), x += parts[2][w], y += parts[3][w];
  };
  // prefix sums over the workgroup of a value per thread, without its own
  auto before_me = [&](uint32_t x) {
    const uint32_t with_me = wave_inclusive_scan(x);
    __syncthreads();
    if (lane == 63) parts[0][wave] = with_me;
    __syncthreads();
    uint32_t before = with_me - x;
    for (int w = 0; w < wave; ++w) before += parts[0][w];
    return before;
  };
  // histogram of the bins that `bin` gives (or -1); found: the bin that holds the need-th, those before it, and its own
  auto find_bin = [&](uint32_t need, auto bin) {
    __syncthreads();
#pragma unroll
    for (int b = 0; b < kBins / kThreads; ++b) hist[b * kThreads + tid] = 0;
    if (tid == 0) few_count = 0;
    __syncthreads();
    each([&](uint32_t k) {
      const int at = bin(k);
      if (at < 0) return;
      // (many equal scores would queue up at one address)
      const int one = __builtin_amdgcn_readfirstlane(at);
      const uint64_t all = __ballot(true);
      if (__ballot(at == one) == all) {
        if (lane == __builtin_ctzll(all)) atomicAdd(&hist[one], static_cast<uint32_t>(__popcll(all)));
      } else {
        atomicAdd(&hist[at], 1u);
      }
    });
    __syncthreads();
    constexpr int kMine = kBins / kThreads;
    uint32_t bins[kMine], mine = 0;
#pragma unroll
    for (int b = 0; b < kMine; ++b) bins[b] = hist[tid * kMine + b], mine += bins[b];
    uint32_t before = before_me(mine);
#pragma unroll
    for (int b = 0; b < kMine; ++b) {
      if (before < need && need <= before + bins[b]) found[0] = tid * kMine + b, found[1] = before, found[2] = bins[b];
      before += bins[b];
    }
    __syncthreads();
  };

  uint32_t lo = 0xffffffffu, hi = 0, finite = 0, infinite = 0;
  each([&](uint32_t k) {
    const bool is_finite = k > kLowest && k < kHighest;
    lo = min(lo, is_finite ? k : 0xffffffffu);
    hi = max(hi, is_finite ? k : 0u);
    finite += is_finite;
    infinite += k == kHighest;
  });
  reduced(lo, hi, finite, infinite);

  uint32_t threshold, need;   // taken: all above the threshold, and the first `need` at it
  if (infinite >= want) {
    threshold = kHighest, need = want;
  } else if (infinite + finite <= want) {
    threshold = kLowest, need = want - infinite - finite;
  } else {
    need = want - infinite;
    const float top = unordered(hi), width = top - unordered(lo), by = (kBins - 1) / width;
    bool narrow = true;   // by bits
    if (width < 1e37f && by < 1e37f) {
      auto bin = [&](uint32_t k) {
        return k >= lo && k <= hi ? min(static_cast<int>((top - unordered(k)) * by), kBins - 1) : -1;
      };
      find_bin(need, bin);
      const int here = found[0];
      const uint32_t size = found[2];
      need -= found[1];
      if (size <= kFew) {
        // (before_me's barriers lie between the last reads of the histogram and this)
        each([&](uint32_t k) {
          if (bin(k) == here) hist[atomicAdd(&few_count, 1u)] = k;
        });
        __syncthreads();
        for (uint32_t i = tid; i < size; i += kThreads) {
          const uint32_t k = hist[i];
          uint32_t above = 0, equal = 0;
          for (uint32_t o = 0; o < size; ++o) {
            const uint32_t other = hist[o];
            above += other > k, equal += other == k;
          }
          if (above < need && need <= above + equal) found[0] = k, found[1] = above;   // (equal ones write the same)
        }
        __syncthreads();
        threshold = found[0], need -= found[1];
        narrow = false;
      } else {
        uint32_t low = 0xffffffffu, high = 0, none = 0, more = 0;
        each([&](uint32_t k) {
          const bool in = bin(k) == here;
          low = min(low, in ? k : 0xffffffffu);
          high = max(high, in ? k : 0u);
        });
        reduced(low, high, none, more);
        lo = low, hi = high;
      }
    }
    while (narrow) {
      const uint32_t span = hi - lo;
      const int low_bits = max(0, 32 - 11 - (span ? __builtin_clz(span) : 32));
      find_bin(need, [&](uint32_t k) { return k >= lo && k <= hi ? static_cast<int>((hi - k) >> low_bits) : -1; });
      const uint32_t high = hi - (found[0] << low_bits), size = (1u << low_bits) - 1;
      need -= found[1];
      lo = high - lo > size ? high - size : lo;
      hi = high;
      if (need == found[2]) {   // all that is left of the bin
        threshold = lo - 1, need = 0;
        break;
      }
      if (lo == hi) {
        threshold = lo;
        break;
      }
    }
  }

  const int64_t token = static_cast<int64_t>(r) * p.n_q + g;
  int32_t* index;
  float* out;
  if constexpr (kFrom == From::kSegment) {
    // every segment but the last has as many
    const int64_t at = static_cast<int64_t>(row) * p.candidates + static_cast<int64_t>(blockIdx.x % p.segments) * min(p.segment, static_cast<uint32_t>(wanted));
    index = p.candidate_blocks + at;
    out = p.candidate_scores + at;
  } else {
    index = p.index + token * p.topk;
    out = p.out_scores ? p.out_scores + token * wanted : nullptr;
  }
  const int32_t* const candidates = kFrom == From::kSegments ? p.candidate_blocks + static_cast<int64_t>(row) * p.candidates : nullptr;
  uint32_t above_base = 0, equal_base = 0;
  for (int chunk = 0; chunk < chunks; ++chunk) {
    if (chunk > 0) __syncthreads();
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t k = kResident ? held[j] : load(chunk, j);
      const uint64_t above = __ballot(k > threshold), equal = __ballot(k == threshold);
      if (lane == 0) above_counts[j * kWavesHere + wave] = __popcll(above), equal_counts[j * kWavesHere + wave] = __popcll(equal);
    }
    __syncthreads();
    const uint32_t above_here = tid < kCounts ? above_counts[tid] : 0, equal_here = tid < kCounts ? equal_counts[tid] : 0;
    const uint32_t above_before = before_me(above_here), equal_before = before_me(equal_here);
    if (tid < kCounts) above_counts[tid] = above_base + above_before, equal_counts[tid] = equal_base + equal_before;
    if (tid == kThreads - 1) found[0] = above_base + above_before + above_here, found[1] = equal_base + equal_before + equal_here;
    __syncthreads();
    above_base = found[0], equal_base = found[1];
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const uint32_t k = kResident ? held[j] : load(chunk, j);
      const uint32_t above_at = above_counts[j * kWavesHere + wave], equal_at = equal_counts[j * kWavesHere + wave];
      const uint64_t lower = (uint64_t{1} << lane) - 1;
      const uint64_t equal = __ballot(k == threshold);
      const bool taken = k > threshold || (k == threshold && equal_at + __popcll(equal & lower) < need);
      const uint64_t all = __ballot(taken);
      if (taken) {
        const uint32_t at = above_at + min(equal_at, need) + __popcll(all & lower);
        const int i = chunk * kChunk + j * kThreads + tid;
        if constexpr (kFrom == From::kSegment) {
          index[at] = static_cast<int>(first) + i;
          out[at] = unordered(k);
        } else {
          const int block = candidates ? candidates[i] : i;
          for (int x = 0; x < 1 << shift; ++x) index[(static_cast<int64_t>(at) << shift) + x] = (block << shift) + x;
          if (out) out[at] = unordered(k);
        }
      }
    }
  }
}

template <int kTiles, int kTok>
hipError_t run_scores(const SelectParams& p, hipStream_t s) {
  const int groups = (p.tokens + kTok - 1) / kTok;
  const int waves_on_tokens = groups >= kWaves ? kWaves : 1;
  const int64_t tiles = (static_cast<int64_t>(p.longest) + kTileKeys - 1) / kTileKeys;
  // runs in eights of tiles, the largest block
  const int64_t waves = 2048, per_group = std::max<int64_t>(1, waves / (static_cast<int64_t>(p.requests) * groups));
  int64_t run_tiles = std::max<int64_t>(8, (tiles + per_group - 1) / per_group);
  run_tiles = std::min<int64_t>(64, (run_tiles + 7) / 8 * 8);
  const int64_t runs = (tiles + run_tiles - 1) / run_tiles;
  const int64_t run_groups = (runs * waves_on_tokens + kWaves - 1) / kWaves, token_groups = (groups + waves_on_tokens - 1) / waves_on_tokens;
  const int64_t total = run_groups * token_groups * p.requests;
  const auto kernel = p.cache.page_shift >= 4 ? &score_kernel<kTiles, kTok, true> : &score_kernel<kTiles, kTok, false>;
  kernel<<<dim3(static_cast<unsigned>(total)), kWaves * 64, 0, s>>>(p, static_cast<int>(run_tiles), static_cast<int>(runs), groups,
                                                                    waves_on_tokens);
  return hipGetLastError();
}

template <int kTiles>
hipError_t run_chunk(const SelectParams& p, hipStream_t s) {
  const int groups = (p.tokens + kChunkWaves - 1) / kChunkWaves;
  const int64_t stages = (static_cast<int64_t>(p.longest) + kStageKeys - 1) / kStageKeys;
  // runs of up to 16 stages, in pairs of them (the largest block)
  const int64_t per_group = std::max<int64_t>(1, 1024 / (static_cast<int64_t>(p.requests) * groups));
  const int64_t run_stages = std::min<int64_t>(16, ((stages + per_group - 1) / per_group + 1) / 2 * 2);
  const int64_t runs = (stages + run_stages - 1) / run_stages;
  chunk_kernel<kTiles><<<dim3(static_cast<unsigned>(runs * groups * p.requests)), kChunkWaves * 64, 0, s>>>(
      p, static_cast<int>(run_stages), static_cast<int>(runs), groups);
  return hipGetLastError();
}

template <int kThreads, int kPer, bool kResident, From kFrom>
hipError_t run_best(const SelectParams& p, hipStream_t s) {
  const int64_t groups = static_cast<int64_t>(p.requests) * p.tokens * (kFrom == From::kSegment ? p.segments : 1);
  best_kernel<kThreads, kPer, kResident, kFrom><<<dim3(static_cast<unsigned>(groups)), kThreads, 0, s>>>(p);
  return hipGetLastError();
}

// From n scores each.
template <From kFrom>
hipError_t best_of(const SelectParams& p, int64_t n, hipStream_t s) {
  if (n <= 2048) return run_best<256, 8, true, kFrom>(p, s);
  if (n <= 8192) return run_best<512, 16, true, kFrom>(p, s);
  if (n <= 16384) return run_best<512, 32, true, kFrom>(p, s);
  if (n <= 32768) return run_best<1024, 32, true, kFrom>(p, s);
  if (n <= 65536) return run_best<1024, 64, true, kFrom>(p, s);
  return run_best<1024, 64, false, kFrom>(p, s);
}

}  // namespace

hipError_t launch_scores(const SelectParams& p, hipStream_t s) {
  const int tiles = (p.heads + 15) / 16;
  if (p.tokens >= 6) {
    if (tiles == 1) return run_chunk<1>(p, s);
    if (tiles == 2) return run_chunk<2>(p, s);
    if (tiles <= 4) return run_chunk<4>(p, s);
    return run_chunk<8>(p, s);
  }
  if (tiles > 4) return run_scores<8, 1>(p, s);
  if (p.tokens == 1) {
    if (tiles == 1) return run_scores<1, 1>(p, s);
    if (tiles == 2) return run_scores<2, 1>(p, s);
    return run_scores<4, 1>(p, s);
  }
  if (tiles == 1) return run_scores<1, 2>(p, s);
  if (tiles == 2) return run_scores<2, 2>(p, s);
  return run_scores<4, 2>(p, s);
}

hipError_t launch_best(const SelectParams& p, hipStream_t s) {
  if (p.segments > 1) {
    if (const hipError_t e = best_of<From::kSegment>(p, p.segment, s); e != hipSuccess) return e;
    return best_of<From::kSegments>(p, p.candidates, s);
  }
  return best_of<From::kScores>(p, p.longest >> p.block_shift, s);
}

}  // namespace avsg
