// Scores of the key cache's positions for a step's query tokens, and the best
// of them.
#include <algorithm>
#include <cfloat>

#include "select_internal.h"

namespace avsg {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4_at_4 __attribute__((ext_vector_type(4), aligned(4)));

constexpr int kWaves = 4;      // of a workgroup of scores
constexpr int kTileKeys = 16;  // keys that a matrix instruction takes

// Whole numbers become doubles without a conversion: as the low words of numbers whose high word is zero, which are
// the numbers times 2^-1074.  Weights are held times 2^890, so that sums are normal numbers, 2^-184 of what they stand for.
constexpr double kWeightUnit = 0x1p890, kSumUnit = 0x1p184;
typedef int i32x2 __attribute__((ext_vector_type(2)));
// Pairs of words with high words of zero, which the compiler does not know and so keeps.
template <int kCount>
struct LowWords {
  i32x2 pair[kCount];
  __device__ __forceinline__ LowWords() {
#pragma unroll
    for (int j = 0; j < kCount; ++j) {
      pair[j] = i32x2{0, 0};
      asm volatile("" : "+v"(pair[j]));
    }
  }
  __device__ __forceinline__ double operator()(int j, int x) {
    pair[j][0] = x;
    return __builtin_bit_cast(double, pair[j]);
  }
};

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

// A wave scores kTok tokens of a request against a run of keys, sixteen at a time.  128 tokens of 64 heads over 32768
// keys per two of them take 60 us, 280 MB at 4.7 TB/s.  The matrix instruction
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
        weight[t][x][i] = h < p.heads ? static_cast<double>(w) * kWeightUnit : 0.0;
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
  const int pages = kWhole ? page_of(seen_key(first_key + lane * kTileKeys, most)) : 0;
  const int64_t in_row = quad * 32, to_scale = kKeyScaleAt - quad * 32;
  // (No branch: a wave that may skip a load has to wait for all of them;
  // and nothing is done with a loaded value here, which would wait for it.  Keys past the last one that is seen read as
  // it; in place of rows that do not exist the pool's first one is read.)
  auto fetch = [&](int tile) {
    Keys k;
    const int key = seen_key(first_key + tile * kTileKeys + l16, most);
    const int page = kWhole ? __builtin_amdgcn_readlane(pages, paged_tile(tile, tiles)) : page_of(key);
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
  LowWords<4> low;
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
          for (int i = 0; i < 4; ++i) s = __builtin_fma(weight[t][x][i], low(i, max(dot[x][i], 0)), s);
      }
    const float scale = my_tile ? pair[1].scale : pair[0].scale;
    const bool there = my_tile ? pair[1].there : pair[0].there;
    // (zeros of either sign are one)
    float score = static_cast<float>(row_sums<2 * kTok>(sum) * kSumUnit * static_cast<double>(scale)) + 0.0f;
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
// 2048 tokens of 64 heads that see 14337 to 16384 keys each take 340 us, 1.5 POP/s; with 128 heads the selection takes
// 672 us in place of 378, with 80 heads 653 (they are taken in 1, 2, 4 or 8 sixteens).  What bounds it is the issue of instructions: per sixteen
// heads and keys two matrix instructions (each takes about two places of the others) and eight for the sums, relu and weight
// (sum in 64 bits: 32-bit sums would take as many), 63% of the cycles, and with the matrix instructions 78%.
// Reads of LDS without bank conflicts (9% of the cycles have one), 128 keys at a time, and other orders of the
// products and sums took as long.
constexpr int kStagedRow = 144;   // bytes of a row in LDS: its codes, its scale
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
        weight[x][i] = h < p.heads ? static_cast<double>(w) * kWeightUnit : 0.0;
      }
    }
  }
  // eight threads per row
  static_assert(kChunkWaves * 64 == kStageKeys * 8);
  const int my_row = threadIdx.x / 8, my_part = threadIdx.x % 8 * 16;
  i32x4 part;
  float part_scale;
  bool part_there;
  // (a row's page is looked up a stage before the row is loaded)
  int page;
  auto key_of = [&](int stage) { return seen_key(first_key + stage * kStageKeys + my_row, most); };
  auto page_of = [&](int stage) {
    const int64_t at = static_cast<int64_t>(r) * p.cache.pages_per_request + (key_of(stage) >> p.cache.page_shift);
    page = p.cache.table ? p.cache.table[at] : static_cast<int>(at);
  };
  auto load = [&](int stage) {
    const int key = key_of(stage);
    part_there = page >= 0 && page < p.cache.pages;
    const uint64_t row = p.cache.base + (part_there ? page * p.cache.page_stride + (key & p.cache.page_mask) * p.cache.row_stride : 0);
    part = load_global<i32x4_at_4>(row + my_part);
    part_scale = load_global<float>(row + kKeyScaleAt);
    page_of(stage + 1);
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
  LowWords<4> low;
  page_of(0);
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
          for (int i = 0; i < 4; ++i) sum[u] = __builtin_fma(weight[x][i], low(i, max(dot[x][i], 0)), sum[u]);
      }
      // row i of sixteen lanes gets the sums of tile i: lane l has key l of the stage
      const float scale = *reinterpret_cast<const float*>(from + lane * kStagedRow + kKeyScaleAt);
      float score = static_cast<float>(row_sums<4>(sum) * kSumUnit * static_cast<double>(scale)) + 0.0f;
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
constexpr int kFew = 512;             // scores of a bin that are compared with each other
constexpr uint32_t kSample = 4096, kSampleMost = 16384;   // (by 1024 threads)

// The best blocks of a token, one workgroup per token.  A sample of the scores gives a bound that a few more than those
// wanted reach; one pass over all scores keeps these; the threshold lies in one of 2048 bins of equal width of
// theirs, and the scores of that bin are compared with each other.  The blocks above the threshold, and those at it, are
// marked in bit maps, from whose prefix sums each finds its place in the result.
// 2048 of 131072 scores take 23 us by the clock of the workgroup: sample 5.7, its bins 2.0, the pass 7.6, what it kept
// 2.6, their bins 1.7, comparisons 1.2, marks 2.5; of 32768 (128 workgroups) 16: 3.7, 1.7, 2.9, 2.4, 1.7, 1.0, 3.0.
// Where that does not do (no bound that leaves few enough, as with many equal scores; more wanted than are
// kept, 7000 of 32768 already) histograms of all scores' bits narrow the threshold's range down until a bin holds one
// value or all that is wanted, reading the scores again for each.  That takes longer: selections of 128 tokens of 64 heads
// over 32768 positions 128 us in place of 79 (7000 wanted), 112 (all scores equal), 4 tokens over 131072 positions 244 in
// place of 41 (16384 wanted), 188 (all equal), 276 (one head, whose scores are zero for half of the keys).
// kMarks: blocks that are marked, and placed, at a time; kCandidates: scores that are kept from the one pass over all.
template <int kThreads, int kMarks, uint32_t kCandidates>
__global__ __launch_bounds__(kThreads) void best_kernel(SelectParams p) {
  constexpr int kWavesHere = kThreads / 64;
  constexpr int kWords = kMarks / 32;
  static_assert(kBins % kThreads == 0 && kWords % kThreads == 0);
  __shared__ uint32_t shared[kBins > 3 * kWords ? kBins : 3 * kWords];
  uint32_t *const hist = shared, *const above_marks = shared, *const equal_marks = shared + kWords, *const before_words = shared + 2 * kWords;
  __shared__ uint32_t kept[kCandidates], kept_block[kCandidates];
  __shared__ uint32_t parts[4][kWavesHere];
  __shared__ uint32_t found[3];
  __shared__ uint32_t count;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint64_t lower = (uint64_t{1} << lane) - 1;
  const int r = p.r0 + static_cast<int>(blockIdx.x) / p.tokens, g = p.g0 + static_cast<int>(blockIdx.x) % p.tokens;
  const int shift = p.block_shift;
  const uint32_t n = p.longest >> shift, want = p.topk >> shift;
  const uint32_t seen = (static_cast<uint32_t>(seen_by(p, r, g)) + (1u << shift) - 1) >> shift;
  const float* const scores = p.scores + static_cast<int64_t>(blockIdx.x) * p.score_stride;
  const int64_t token = static_cast<int64_t>(r) * p.n_q + g;
  int32_t* const index = p.index + token * p.topk;
  float* const out = p.out_scores ? p.out_scores + token * want : nullptr;
  auto put = [&](uint32_t at, uint32_t block, float score) {
    for (int x = 0; x < 1 << shift; ++x) index[(static_cast<int64_t>(at) << shift) + x] = static_cast<int>(block << shift) + x;
    if (out) out[at] = score;
  };

  if (seen <= want) {
    // all that is seen, and the lowest others
    for (uint32_t i = tid; i < want << shift; i += kThreads) index[i] = static_cast<int>(i);
    if (out)
      for (uint32_t i = tid; i < want; i += kThreads) out[i] = i < seen ? scores[i] : -__builtin_inff();
    return;
  }

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
  // a histogram of what `fill` adds; found: the bin that holds the need-th, those before it, and its own
  auto find_bin = [&](uint32_t need, auto fill) {
    __syncthreads();
#pragma unroll
    for (int b = 0; b < kBins / kThreads; ++b) hist[b * kThreads + tid] = 0;
    __syncthreads();
    fill([&](int at) {
      if (at >= 0) atomicAdd(&hist[at], 1u);
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
  auto is_finite = [](uint32_t k) { return k > kLowest && k < kHighest; };
  // bins of equal width from the largest down, of finite scores from lo to hi
  struct Bins {
    uint32_t lo, hi;
    float top, by;
    __device__ bool fine() const { return top - unordered(lo) < 1e37f && by < 1e37f; }
    __device__ int operator()(uint32_t k) const {
      return k >= lo && k <= hi ? min(static_cast<int>((top - unordered(k)) * by), kBins - 1) : -1;
    }
  };
  auto bins_of = [&](uint32_t lo, uint32_t hi) {
    const float top = unordered(hi);
    return Bins{lo, hi, top, (kBins - 1) / (top - unordered(lo))};
  };

  uint32_t threshold = 0, need = 0;   // taken: all above the threshold, and the first `need` at it
  bool done = false;
  uint32_t candidates = 0;
  if (want <= kCandidates) {
    // few are all kept
    const bool all = seen <= kCandidates;
    candidates = seen;
    if (!all) {
      float bound = -FLT_MAX;
      // Of the sample as many as are wanted of all, four and a half standard deviations and three more: too few in one
      // of 300000 tokens where a score does not depend on its position.  (Where it does, too few or too many may reach the
      // bound more often; then all scores are read again, below.)  It is larger where it would not hold 128 of those wanted.
      constexpr int kMine = kSampleMost / 1024;
      uint32_t sample = kSample;
      while (sample < kMine * kThreads && static_cast<uint64_t>(want) * sample < uint64_t{128} * seen) sample *= 2;
      uint32_t k[kMine], lo = 0xffffffffu, hi = 0, number = 0, none = 0;
#pragma unroll
      for (int j = 0; j < kMine; ++j) {
        if (j * kThreads >= sample) break;
        k[j] = ordered(scores[static_cast<uint64_t>(j * kThreads + tid) * seen / sample]);
        const bool in = is_finite(k[j]);
        lo = min(lo, in ? k[j] : 0xffffffffu);
        hi = max(hi, in ? k[j] : 0u);
        number += in;
      }
      reduced(lo, hi, number, none);
      const float share = static_cast<float>(want) / static_cast<float>(seen) * static_cast<float>(sample);
      const uint32_t rank = static_cast<uint32_t>(share + 4.5f * sqrtf(share) + 3.0f);
      const Bins bin = bins_of(lo, hi);
      if (rank <= number && bin.fine()) {
        find_bin(rank, [&](auto add) {
#pragma unroll
          for (int j = 0; j < kMine; ++j) {
            if (j * kThreads >= sample) break;
            add(bin(k[j]));
          }
        });
        bound = bin.top - static_cast<float>(found[0] + 1) / bin.by;
      }
      // where it is reached, in no order: 32 scores of a thread at a time, as bits
      if (tid == 0) count = 0;
      __syncthreads();
      for (uint32_t at = 0; at < seen; at += kThreads * 32) {
        f32x4 x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (at + j * kThreads * 4 >= seen) break;
          x[j] = *reinterpret_cast<const f32x4*>(scores + min(at + (j * kThreads + tid) * 4, (seen - 1) & ~3u));
        }
        uint32_t hits = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if (at + j * kThreads * 4 >= seen) break;
          const uint32_t i = at + (j * kThreads + tid) * 4, left = i < seen ? seen - i : 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) hits |= x[j][e] >= bound ? 1u << (4 * j + e) : 0;
          if (left < 4) hits &= ~(15u << (4 * j)) | ((1u << left) - 1) << (4 * j);
        }
        const uint32_t mine = __popc(hits), with_me = wave_inclusive_scan(mine);
        uint32_t to = 0;
        if (lane == 63 && with_me) to = atomicAdd(&count, with_me);
        to = __builtin_amdgcn_readlane(to, 63) + with_me - mine;
        while (hits) {
          const int b = __ffs(static_cast<int>(hits)) - 1;
          hits &= hits - 1;
          if (to < kCandidates) kept_block[to] = at + (b / 4 * kThreads + tid) * 4 + b % 4;
          ++to;
        }
      }
      __syncthreads();
      candidates = count;
    }
    if (candidates >= want && candidates <= kCandidates) {
      uint32_t lo = 0xffffffffu, hi = 0, infinite = 0, number = 0;
      for (uint32_t i = tid; i < candidates; i += kThreads) {
        if (all) kept_block[i] = i;
        const uint32_t k = ordered(scores[all ? i : kept_block[i]]);
        kept[i] = k;
        number += k > kLowest;
        lo = min(lo, is_finite(k) ? k : 0xffffffffu);
        hi = max(hi, is_finite(k) ? k : 0u);
        infinite += k == kHighest;
      }
      reduced(lo, hi, infinite, number);
      if (number < want) {
        // (then some of those at minus infinity are wanted)
      } else if (infinite >= want) {
        threshold = kHighest, need = want, done = true;
      } else if (const Bins bin = bins_of(lo, hi); bin.fine()) {
        need = want - infinite;
        find_bin(need, [&](auto add) {
          for (uint32_t i = tid; i < candidates; i += kThreads) add(bin(kept[i]));
        });
        const int here = found[0];
        const uint32_t before = found[1], size = found[2];
        if (size <= kFew) {
          need -= before;
          if (tid == 0) count = 0;
          __syncthreads();
          // (the histogram has been read)
          for (uint32_t i = tid; i < candidates; i += kThreads)
            if (bin(kept[i]) == here) hist[atomicAdd(&count, 1u)] = kept[i];
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
          threshold = found[0], need -= found[1], done = true;
        }
      }
    }
  }

  if (done) {
    uint32_t above_base = 0, equal_base = 0;
    for (uint32_t first = 0; first < seen; first += kMarks) {
      constexpr int kMine = kWords / kThreads;   // words per thread
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kMine; ++w) above_marks[w * kThreads + tid] = 0, equal_marks[w * kThreads + tid] = 0;
      __syncthreads();
      for (uint32_t i = tid; i < candidates; i += kThreads) {
        const uint32_t k = kept[i], block = kept_block[i] - first;
        if (k >= threshold && block < kMarks) atomicOr(&(k == threshold ? equal_marks : above_marks)[block / 32], 1u << (block & 31));
      }
      __syncthreads();
      // above and equal in one word: at most kCandidates each
      uint32_t words[kMine], both = 0;
#pragma unroll
      for (int w = 0; w < kMine; ++w) {
        words[w] = __popc(above_marks[tid * kMine + w]) + (__popc(equal_marks[tid * kMine + w]) << 16);
        both += words[w];
      }
      uint32_t before = before_me(both);
      if (tid == kThreads - 1) found[2] = before + both;
#pragma unroll
      for (int w = 0; w < kMine; ++w) {
        before_words[tid * kMine + w] = before;
        before += words[w];
      }
      __syncthreads();
      for (uint32_t i = tid; i < candidates; i += kThreads) {
        const uint32_t k = kept[i], block = kept_block[i] - first;
        if (k < threshold || block >= kMarks) continue;
        const uint32_t word = block / 32, below = (1u << (block & 31)) - 1, prior = before_words[word];
        const uint32_t above_at = above_base + (prior & 0xffff) + __popc(above_marks[word] & below);
        const uint32_t equal_at = equal_base + (prior >> 16) + __popc(equal_marks[word] & below);
        if (k > threshold || equal_at < need) put(above_at + min(equal_at, need), first + block, unordered(k));
      }
      above_base += found[2] & 0xffff, equal_base += found[2] >> 16;
    }
    return;
  }

  // all scores, again and again
  auto load = [&](uint32_t i) { return i < seen ? ordered(scores[i]) : i < n ? kLowest : 0u; };
  uint32_t lo = 0xffffffffu, hi = 0, number = 0, none = 0;
  for (uint32_t i = tid; i < seen; i += kThreads) {
    const uint32_t k = load(i);
    if (k > kLowest) lo = min(lo, k), hi = max(hi, k), ++number;
  }
  reduced(lo, hi, number, none);
  threshold = kLowest, need = want;
  if (number <= want) {
    need = want - number;
  } else {
    for (;;) {
      const uint32_t span = hi - lo;
      const int low_bits = max(0, 32 - 11 - (span ? __builtin_clz(span) : 32));
      find_bin(need, [&](auto) {
        for (uint32_t i = tid; i < seen; i += kThreads) {
          const uint32_t k = load(i);
          if (k < lo || k > hi) continue;
          const int at = (hi - k) >> low_bits;   // the largest scores in the first bins
          // (many equal scores would queue up at one address)
          const int one = __builtin_amdgcn_readfirstlane(at);
          const uint64_t all = __ballot(true);
          if (__ballot(at == one) == all) {
            if (lane == __builtin_ctzll(all)) atomicAdd(&hist[one], static_cast<uint32_t>(__popcll(all)));
          } else {
            atomicAdd(&hist[at], 1u);
          }
        }
      });
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
  uint32_t above_base = 0, equal_base = 0;
  for (uint32_t first = 0; first < n; first += kThreads) {
    const uint32_t k = load(first + tid);
    const uint64_t above = __ballot(k > threshold), equal = __ballot(k == threshold);
    __syncthreads();
    if (lane == 0) parts[0][wave] = __popcll(above), parts[1][wave] = __popcll(equal);
    __syncthreads();
    uint32_t above_at = above_base, equal_at = equal_base;
    for (int w = 0; w < kWavesHere; ++w) {
      if (w < wave) above_at += parts[0][w], equal_at += parts[1][w];
      above_base += parts[0][w], equal_base += parts[1][w];
    }
    const bool taken = k > threshold || (k == threshold && equal_at + __popcll(equal & lower) < need);
    const uint64_t all = __ballot(taken);
    if (taken) put(above_at + min(equal_at, need) + __popcll(all & lower), first + tid, unordered(k));
  }
}

template <int kTiles, int kTok>
hipError_t run_scores(const SelectParams& p, const ScorePlan& plan, hipStream_t s) {
  const int waves_on_keys = kWaves / plan.waves_on_tokens;
  const int64_t run_groups = (plan.runs + waves_on_keys - 1) / waves_on_keys;
  const int64_t token_groups = (plan.groups + plan.waves_on_tokens - 1) / plan.waves_on_tokens;
  const int64_t total = run_groups * token_groups * p.requests;
  const auto kernel = p.cache.page_shift >= 4 ? &score_kernel<kTiles, kTok, true> : &score_kernel<kTiles, kTok, false>;
  kernel<<<dim3(static_cast<unsigned>(total)), kWaves * 64, 0, s>>>(p, plan.run, plan.runs, plan.groups, plan.waves_on_tokens);
  return hipGetLastError();
}

template <int kTiles>
hipError_t run_chunk(const SelectParams& p, const ScorePlan& plan, hipStream_t s) {
  const int64_t total = static_cast<int64_t>(plan.runs) * plan.groups * p.requests;
  chunk_kernel<kTiles><<<dim3(static_cast<unsigned>(total)), kChunkWaves * 64, 0, s>>>(p, plan.run, plan.runs, plan.groups);
  return hipGetLastError();
}

template <int kThreads, int kMarks, uint32_t kCandidates>
hipError_t run_best(const SelectParams& p, hipStream_t s) {
  best_kernel<kThreads, kMarks, kCandidates><<<dim3(static_cast<unsigned>(p.requests) * p.tokens), kThreads, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

// By waves on their own or by workgroups that share their keys, by what a selection took (us, in a graph; 8192 positions):
//   requests x tokens x heads    alone   shared        requests x tokens x heads    alone   shared
//       16 x 2 x 64              18.8     26.3             64 x 6 x 64              72.8     57.5
//        8 x 4 x 64              18.8     20.2             64 x 4 x 16              36.3     27.0
//       64 x 4 x 64              41.7     44.8             64 x 8 x 16              51.7     34.1
//        8 x 6 x 64              23.5     22.0              1 x 64 x 64             24.1     22.5
// (a wave on its own holds two tokens, so few tokens waste less of it than of a workgroup for eight.)
ScorePlan score_plan(int requests, int tokens, int heads, int longest) {
  ScorePlan plan{};
  const int tiles = (heads + 15) / 16;
  plan.head_tiles = tiles == 1 ? 1 : tiles == 2 ? 2 : tiles <= 4 ? 4 : 8;
  plan.shared = tokens >= (tiles <= 2 ? 4 : 6);
  plan.tokens = plan.shared ? kChunkWaves : tiles > 4 || tokens == 1 ? 1 : 2;
  plan.groups = (tokens + plan.tokens - 1) / plan.tokens;
  plan.waves_on_tokens = plan.shared ? kChunkWaves : plan.groups >= kWaves ? kWaves : 1;
  const int64_t all = static_cast<int64_t>(requests) * plan.groups, unit = plan.shared ? kStageKeys : kTileKeys;
  const int64_t units = (longest + unit - 1) / unit, per_group = std::max<int64_t>(1, (plan.shared ? 1024 : 2048) / all);
  const int64_t run = (units + per_group - 1) / per_group;
  // runs of up to 16 stages in pairs of them, or of up to 64 tiles in eights: the largest block
  plan.run = static_cast<int>(plan.shared ? std::min<int64_t>(16, (run + 1) / 2 * 2) : std::min<int64_t>(64, std::max<int64_t>(8, (run + 7) / 8 * 8)));
  plan.runs = static_cast<int>((units + plan.run - 1) / plan.run);
  return plan;
}

hipError_t launch_scores(const SelectParams& p, hipStream_t s) {
  const ScorePlan plan = score_plan(p.requests, p.tokens, p.heads, p.longest);
  if (plan.shared) {
    if (plan.head_tiles == 1) return run_chunk<1>(p, plan, s);
    if (plan.head_tiles == 2) return run_chunk<2>(p, plan, s);
    if (plan.head_tiles == 4) return run_chunk<4>(p, plan, s);
    return run_chunk<8>(p, plan, s);
  }
  if (plan.head_tiles == 8) return run_scores<8, 1>(p, plan, s);
  if (plan.tokens == 1) {
    if (plan.head_tiles == 1) return run_scores<1, 1>(p, plan, s);
    if (plan.head_tiles == 2) return run_scores<2, 1>(p, plan, s);
    return run_scores<4, 1>(p, plan, s);
  }
  if (plan.head_tiles == 1) return run_scores<1, 2>(p, plan, s);
  if (plan.head_tiles == 2) return run_scores<2, 2>(p, plan, s);
  return run_scores<4, 2>(p, plan, s);
}

hipError_t launch_best(const SelectParams& p, hipStream_t s) {
  const int n = p.longest >> p.block_shift;
  const int want = p.topk >> p.block_shift;
  if (n <= 4096) return run_best<256, 8192, 4096>(p, s);
  if (n <= 16384 && want <= 2560) return run_best<512, 16384, 4096>(p, s);
  if (n <= 16384) return run_best<512, 16384, 8192>(p, s);
  return run_best<1024, 131072, 8192>(p, s);
}

}  // namespace avsg

int32_t avsg_internal_score_row(int32_t first_key, int32_t tiles, int32_t tile, int32_t lane, int32_t most, int32_t page_shift) {
  const int key = avsg::seen_key(first_key + tile * avsg::kTileKeys + lane, most);
  if (page_shift < 4 || page_shift > 30) return key;
  const int paged = avsg::seen_key(first_key + avsg::paged_tile(tile, tiles) * avsg::kTileKeys, most);
  return (paged >> page_shift << page_shift) + (key & ((1 << page_shift) - 1));
}
