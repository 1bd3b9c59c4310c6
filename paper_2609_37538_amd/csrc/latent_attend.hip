// Attention of a step's query tokens over latent cache rows:
//   out = sum_i w_i v_i / sum_i w_i,  w_i = exp(scale q . k_i),
// in one pass over the rows.  Every head of a token reads the same rows, and a
// row's latent part is key and value at once, so a row is brought in once per
// workgroup and serves up to 64 heads twice: 2 * (576 + 512) operations per row
// and head, on the matrix cores.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "latent_internal.h"

namespace avsg {
namespace {

// Values in LDS: rows of 1024 bytes.  Of every 256 bytes (all banks) row x has
// its 32-byte pieces exchanged by x mod 8 and the halves of a piece by bit 3 of
// x.  Sixteen lanes that write 16 bytes each of the same columns of 16 rows, and
// groups of 16 lanes that read 32 bytes each of four rows, then meet every
// bank equally often.
constexpr int kValueStride = kLatent * 2;
// Byte of a row's 256 at which 16-byte part `part` lies.
__device__ __forceinline__ unsigned value_part(unsigned row, unsigned part) {
  return ((part ^ ((row & 7) * 2 + ((row >> 3) & 1))) & 15) * 16;
}
// Weights are kept relative to a reference, the largest score so far raised by `above` powers of two.  It need
// not follow the maximum: only a score that passes the one it was made of by kSlack raises it, which saves the
// exchange of maxima between waves for nearly every tile.  `above` is kSlack and the logarithm of the number of
// entries, so that however many weights there are, they add up to 1 at most and their products with values to
// the largest value at most: what is finite in the rows stays finite in every sum.  A token's largest weight is
// never less than 2^-above (2^-39 for the longest contexts), and weights down to 2^-87 of that do not vanish.  The matrix
// instructions keep denormal sums, so values lose bits only below about 2^(above - 140).
constexpr float kSlack = 8.f;
// A weight takes part in the output product as a sum of two bfloat16, its eight highest bits and the
// rest: one alone would be off by up to 2^-8, as much as the result's own rounding.  Where LDS has no
// room for both, the rest is kept in 8 bits (e4m3: 4 significant ones, so that the weight has 12), in units that
// fit the largest weight, 2^(kSlack - above), whose rest is at most 2^-9 of it: 256 units.  Below 2^-6 of the weight
// that the reference's own score has, the rest has fewer bits, and is off by at most 2^-19 of that weight.
constexpr float kRestUnit = 0x1p-17f;   // of the largest weight
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// The order in which the compiler is to issue what stands before in a block:
// the next `n` instructions of a kind.
constexpr int kMatrix = 0x8, kLdsRead = 0x100;
#define kSchedule(kind, n) __builtin_amdgcn_sched_group_barrier(kind, n, 0)

// What the loads of entries that do not count read in place of a row.
__device__ __align__(16) const unsigned char zero_row[kRowBytesBf16] = {};

__device__ __forceinline__ float zero_if_none(float reference) { return reference == -INFINITY ? 0.f : reference; }

__device__ __forceinline__ bf16x4 rounded(f32x4 x) {
  return bf16x4{static_cast<__bf16>(x[0]), static_cast<__bf16>(x[1]), static_cast<__bf16>(x[2]), static_cast<__bf16>(x[3])};
}

// What `rounded` leaves of x.
__device__ __forceinline__ f32x4 rest_of(f32x4 x, bf16x4 high) {
  return f32x4{x[0] - static_cast<float>(high[0]), x[1] - static_cast<float>(high[1]), x[2] - static_cast<float>(high[2]),
               x[3] - static_cast<float>(high[3])};
}

typedef short s16x2 __attribute__((ext_vector_type(2)));
// Four rests in 8 bits each, and eight of them in bfloat16.
__device__ __forceinline__ uint32_t rest_encode(f32x4 x, float unit) {
  s16x2 c{};
  c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, x[0], x[1], unit, false);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(c, x[2], x[3], unit, true);
  return __builtin_bit_cast(uint32_t, c);
}
__device__ __forceinline__ bf16x8 rest_decode(u32x2 c, float unit) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[0], unit, false);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[0], unit, true);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[1], unit, false);
  const bf16x2 e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(c[1], unit, true);
  return bf16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
}

// A lane's number that the compiler takes for a new value: what is derived from
// it is computed where it is used and not kept in registers across the loop.
__device__ __forceinline__ int lane_here() {
  int x = threadIdx.x & 63;
  asm volatile("" : "+v"(x));
  return x;
}

// A workgroup's share of the work: a block of heads of one query token over a
// run of tiles of its entries.
struct Share {
  int64_t token, len;
  int request, head_block, split, first, tiles;   // `first` of its entries (where it has any)
  unsigned count;                                 // that can count
};

// Tiles of `entries`, which may be as many as 31 bits hold.
__host__ __device__ constexpr int tiles_of(int entries, int rows) { return entries / rows + (entries % rows != 0); }

__device__ __forceinline__ Share share_of(const AttendParams& p, int head_blocks, int tiles_per_split, int tile_rows) {
  Share w;
  // workgroups of one request lie next to each other on one XCD, whose L2 then
  // serves the rows that they share
  const unsigned total = gridDim.x, per = total / kXcds, more = total % kXcds, xcd = blockIdx.x % kXcds;
  const unsigned id = xcd * per + min(xcd, more) + blockIdx.x / kXcds;
  const unsigned share = head_blocks * p.plan.splits;
  w.token = id / share;
  w.head_block = (id % share) % head_blocks;
  w.split = (id % share) / head_blocks;
  w.request = static_cast<int>(w.token / p.n_q);
  w.len = p.lens ? p.lens[w.token] : INT64_MAX;
  // entries that can count: with their positions given, any
  const int limit = p.index ? p.topk : static_cast<int>(w.len < 0 ? 0 : w.len < p.topk ? w.len : p.topk);
  const int64_t most = static_cast<int64_t>(tiles_per_split) * tile_rows, first = w.split * most;
  w.first = static_cast<int>(first);
  w.count = static_cast<unsigned>(max(int64_t{0}, min(most, limit - first)));
  w.tiles = static_cast<int>((w.count + tile_rows - 1) / tile_rows);
  return w;
}

// Finds the row of an entry: what is read of it comes first, its address (0: it
// does not count) some tiles later.
struct RowFinder {
  int row, pos, page;   // of this lane's row of those looked at last

  // entry `n` of the share
  __device__ __forceinline__ void look(const AttendParams& p, const Share& w, unsigned n) {
    row = pos = page = -1;
    if (n >= w.count) return;
    const int i = w.first + static_cast<int>(n);
    row = p.rows ? p.rows[w.token * p.topk + i] : i;
    pos = p.index ? p.index[w.token * p.topk + i] : i;
    if (!p.rows && p.cache.table && i < p.cache.capacity)
      page = p.cache.table[static_cast<int64_t>(w.request) * p.cache.pages_per_request + (i >> p.cache.page_shift)];
  }
  // the address of that row, 0 where it does not count
  __device__ __forceinline__ uint64_t address(const AttendParams& p, const Share& w) const {
    const CacheView& c = p.cache;
    if (row < 0 || row >= c.capacity || pos < 0 || pos >= w.len) return 0;
    // one page per request, as slots have it
    if (!c.table && c.pages_per_request == 1)
      return c.base + w.request * c.page_stride + static_cast<uint64_t>(static_cast<uint32_t>(row)) * static_cast<uint64_t>(c.row_stride);
    int64_t at = page;
    if (p.rows || !c.table) {
      at = static_cast<int64_t>(w.request) * c.pages_per_request + (row >> c.page_shift);
      if (c.table) at = c.table[at];
    }
    if (at < 0 || at >= c.pages) return 0;
    return c.base + at * c.page_stride + (row & c.page_mask) * c.row_stride;
  }
};

typedef __attribute__((address_space(3))) bf16x4* lds_bf16x4;

// Operand of the output product: columns l % 16 of a 16-column tile, of rows
// quad * 4 .. + 3 of two 16-row tiles that follow each other.  `at`: this lane's
// place in the first.
__device__ __forceinline__ bf16x8 load_values(const unsigned char* lds, unsigned at) {
  const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)(lds + at));
  const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)(lds + at + 16 * kValueStride));
  return bf16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
}
// That place for a wave whose columns start at `col`, a multiple of 64.
__device__ __forceinline__ unsigned values_from(int lane, int col) {
  const unsigned row = (lane >> 4) * 4 + (lane & 15) / 4;
  return row * kValueStride + (col * 2 & ~255) + value_part(row, col / 8 % 16 + (lane & 3) / 2) + (lane & 1) * 8;
}

// Eight columns of a head's query (of head 0 in place of one that does not exist).
__device__ __forceinline__ u32x4 load_query(const AttendParams& p, const Share& w, int head, int col) {
  return *reinterpret_cast<const u32x4*>(p.q + w.token * p.q_token_stride + (head < p.heads ? head : 0) * p.q_head_stride + col);
}
// Queries take the scale's sign (or its zero), so that with a positive scale
// products compare like scores.  In bits, without a branch: behind one, every load of a
// kernel's eighteen would be waited for by itself.
__device__ __forceinline__ bf16x8 signed_query(const AttendParams& p, int head, u32x4 x) {
  const uint32_t keep = head < p.heads && p.scale != 0.f ? ~0u : 0u, sign = p.scale < 0.f ? 0x80008000u : 0u;
  return __builtin_bit_cast(bf16x8, (x & keep) ^ sign);
}

// The logarithm of the sum of exp(score) where weights relative to `reference` add up to `all`, 0 if there are none.
__device__ __forceinline__ float log_sum(const AttendParams& p, float reference, float all) {
  return all == 0.f ? -INFINITY : (zero_if_none(reference) - p.above + __builtin_amdgcn_logf(all * __builtin_amdgcn_exp2f(p.above))) * kLn2;
}

// Result of one head: four columns of every column tile of a wave, whose sum
// of weights is `all` relative to `reference`.
template <int kColTiles, typename Out>
__device__ __forceinline__ void store_head(const AttendParams& p, const Share& w, int head, int col, Out out, float reference,
                                           float all, bool first) {
  if (p.plan.splits > 1) {
    const int64_t part = (w.token * p.plan.splits + w.split) * p.heads + head;
    if (first) p.part_ml[part] = f32x2{reference, all};
#pragma unroll
    for (int c = 0; c < kColTiles; ++c) *reinterpret_cast<f32x4*>(p.part_out + part * kLatent + col + c * 16) = out(c);
    return;
  }
  const float by = all == 0.f ? 0.f : 1.f / all;
  __bf16* to = p.out + w.token * p.out_token_stride + head * p.out_head_stride + col;
#pragma unroll
  for (int c = 0; c < kColTiles; ++c) *reinterpret_cast<bf16x4*>(to + c * 16) = rounded(out(c) * by);
  if (p.lse && first)
    p.lse[w.token * p.heads + head] = log_sum(p, reference, all);
}

// Operands of the products, in both kernels below:
//   scores   A = keys     lane l: row l % 16, eight columns     B = queries  lane l: head l % 16, the same columns
//            result lane l: head l % 16, rows (l / 16) * 4 .. + 3
//   output   A = values^T lane l: column l % 16, eight rows     B = weights  lane l: head l % 16, the same rows
//            result lane l: head l % 16, columns (l / 16) * 4 .. + 3
// The eight rows of the second product are rows (l / 16) * 4 .. + 3 of two
// 16-row tiles: what a lane holds of the first one's result, so weights need no
// exchange within a wave.  Of the 4-bit latent columns a lane has blocks of 32
// (16 bytes, four products' eight columns each), of bfloat16 ones eight columns
// of every 32.

// 16 heads at a time: few heads, or few tokens.  Four waves score 16 rows each against
// all 576 columns, leave weights and expanded values in LDS, and take 128 of the 512
// columns each of the output.  So few heads make the rows' bytes count, and two
// workgroups per CU keep 50 KB of them in flight.  A call of one token takes 7 us,
// launch, three dependent loads (entry, row, next tile's) and one tile.  Or eight waves
// and tiles of 128 rows: 2.5 us each where a lone workgroup of four takes 1.7 for 64,
// and half the parts of two workgroups: 4 x 131072 rows of 400 bytes for 16 heads take
// 58 us, 3.6 TB/s, where a large copy moves 5.0.
template <bool kMx4, int kWaves>
__global__ __launch_bounds__(kWaves * 64, 2) void attend_kernel(AttendParams p, int head_blocks, int tiles_per_split) {
  constexpr int kRows = kWaves * 16, kCols = kLatent / kWaves, kColTiles = kCols / 16;
  constexpr int kPairs = kWaves / 2;   // of 16-row tiles, as the output product takes them
  constexpr int kLoads = kMx4 ? 4 : 16;
  extern __shared__ __align__(16) unsigned char lds[];
  unsigned char* const values = lds;
  unsigned char* const weights = lds + kRows * kValueStride;                     // [high, rest][kPairs][64 lanes] 16 bytes
  float* const wave_top = reinterpret_cast<float*>(weights + 2 * kPairs * 1024); // [kWaves][16]
  float* const reference = wave_top + kWaves * 16;                               // [16]
  int* const raised = reinterpret_cast<int*>(reference + 16);                    // [2]

  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Share w = share_of(p, head_blocks, tiles_per_split, kRows);
  const int head = w.head_block * 16 + l16;

  // every lane finds the row whose keys it loads, what is read of it two tiles ahead
  RowFinder finder;
  finder.look(p, w, wave * 16 + l16);
  if (threadIdx.x < 16) reference[threadIdx.x] = -INFINITY;
  if (threadIdx.x < 4) raised[threadIdx.x] = 0;
  u32x4 raw[18];
#pragma unroll
  for (int j = 0; j < 18; ++j)
    raw[j] = load_query(p, w, head, kMx4 && j < 16 ? (j / 4 * 4 + quad) * 32 + j % 4 * 8 : 32 * j + 8 * quad);

  u32x4 key[kLoads], scales{}, turned[2];
  unsigned counts = 0;   // bits of this lane's four rows (quad * 4 + i) that count
  auto load_keys = [&](int t) {
    const unsigned x = lane_here();
    uint64_t at = finder.address(p, w);
    finder.look(p, w, (t + 1u) * kRows + wave * 16 + (x & 15));
    counts = static_cast<unsigned>(__ballot(at != 0) >> (x / 16 * 4)) & 15u;
    if (at == 0) at = reinterpret_cast<uint64_t>(zero_row);
    if constexpr (kMx4) scales = load_global<u32x4>(at + kMx4CodeBytes);
    at += x / 16 * 16;
#pragma unroll
    for (int j = 0; j < kLoads; ++j) key[j] = load_global<u32x4>(at + 64 * j);
#pragma unroll
    for (int j = 0; j < 2; ++j) turned[j] = load_global<u32x4>(at + (kMx4 ? kMx4RopeAt : kLatent * 2) + 64 * j);
  };
  load_keys(0);
  __builtin_amdgcn_sched_barrier(0);   // the first keys are on their way before the queries are waited for
  bf16x8 query[18];
#pragma unroll
  for (int j = 0; j < 18; ++j) query[j] = signed_query(p, head, raw[j]);

  const float scale = p.scale == 0.f ? 1.f : fabsf(p.scale) * kLog2e;   // scores in powers of two
  const float per_scale = 1.f / scale;
  float ref = -INFINITY, sum = 0.f;
  f32x4 out[kColTiles];
#pragma unroll
  for (int c = 0; c < kColTiles; ++c) out[c] = f32x4{};

  for (int t = 0; t < w.tiles; ++t) {
    __syncthreads();   // every wave is done with the last tile's values and weights
    f32x4 part[2] = {};   // sums that alternate
    {
      const int x = lane_here();
      const unsigned to = (wave * 16 + (x & 15)) * kValueStride + value_part(x & 15, (kMx4 ? 4 : 1) * (x >> 4));
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        bf16x8 k;
        if constexpr (kMx4) k = mx4_decode8(key[j / 4][j % 4], mx4_unit((scales[j / 4] >> (x / 16 * 8)) & 255u));
        else k = __builtin_bit_cast(bf16x8, key[j]);
        *reinterpret_cast<bf16x8*>(values + (to ^ (j % 4 * (kMx4 ? 16 : 64))) + j / 4 * 256) = k;
        part[j & 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, query[j], part[j & 1], 0, 0, 0);
      }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
      part[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, turned[j]), query[16 + j], part[j], 0, 0, 0);
    const unsigned now = counts;
    if (t + 1 < w.tiles) load_keys(t + 1);

    f32x4 s = part[0] + part[1];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (!((now >> i) & 1)) s[i] = -INFINITY;
    // weights relative to the reference as it is; a score that raises it is noted
    float add;
    auto weigh = [&]() {
      const float base = zero_if_none(ref);
      f32x4 e;
#pragma unroll
      for (int i = 0; i < 4; ++i) e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i], scale, -base));
      add = (e[0] + e[1]) + (e[2] + e[3]);
      bf16x4* const to = reinterpret_cast<bf16x4*>(weights + (wave >> 1) * 1024 + lane * 16 + (wave & 1) * 8);
      const bf16x4 high = rounded(e);
      to[0] = high;
      to[kPairs * 128] = rounded(rest_of(e, high));
    };
    const float top = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
    weigh();
    if (__any(top > (ref - p.above + kSlack) * per_scale) && lane == 0) raised[t & 1] = t + 1;
    __syncthreads();
    if (raised[t & 1] == t + 1) {
      // some score raises its reference: all waves agree on new ones and
      // bring what they hold to them
      float high = top * scale + p.above;
      high = fmaxf(high, __shfl_xor(high, 16));
      high = fmaxf(high, __shfl_xor(high, 32));
      if (quad == 0) wave_top[wave * 16 + l16] = high;
      __syncthreads();
      high = reference[l16];
#pragma unroll
      for (int i = 0; i < kWaves; ++i) high = fmaxf(high, wave_top[i * 16 + l16]);
      // nothing is held yet where there is no reference
      const float by = ref == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ref - high);
#pragma unroll
      for (int c = 0; c < kColTiles; ++c) out[c] *= by;
      sum *= by;
      ref = high;
      weigh();
      __syncthreads();
      // read again after the next tile's barrier at the earliest
      if (wave == 0 && quad == 0) reference[l16] = ref;
    }
    sum += add;

    const unsigned from = values_from(lane_here(), wave * kCols);
    const unsigned char* const weight_from = weights + lane_here() * 16;
    bf16x8 e[2][kPairs];
#pragma unroll
    for (int i = 0; i < 2 * kPairs; ++i) e[i / kPairs][i % kPairs] = *reinterpret_cast<const bf16x8*>(weight_from + i * 1024);
    // operands are read four products ahead: left to itself the compiler waits for each
    auto load_step = [&](int n) {   // column tile n % kColTiles of rows n / kColTiles * 32 .. + 31
      return load_values(values, (from ^ (n % kColTiles * 32)) + n / kColTiles * 32 * kValueStride);
    };
    constexpr int kAhead = 4;
    bf16x8 v[kAhead];
#pragma unroll
    for (int n = 0; n < kAhead; ++n) v[n] = load_step(n);
#pragma unroll
    for (int n = 0; n < kPairs * kColTiles; ++n) {
      const bf16x8 x = v[n % kAhead];
      if (n + kAhead < kPairs * kColTiles) v[n % kAhead] = load_step(n + kAhead);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        out[n % kColTiles] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, e[i][n / kColTiles], out[n % kColTiles], 0, 0, 0);
    }
    kSchedule(kLdsRead, 2 * kPairs + 2 * kAhead);
#pragma unroll
    for (int n = 0; n < kPairs * kColTiles; ++n) {
      kSchedule(kMatrix, 2);
      kSchedule(kLdsRead, 2);
    }
  }

  // the waves' sums of weights
  __syncthreads();
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  if (quad == 0) wave_top[wave * 16 + l16] = sum;
  __syncthreads();
  if (head >= p.heads) return;
  float all = 0.f;
#pragma unroll
  for (int i = 0; i < kWaves; ++i) all += wave_top[i * 16 + l16];
  store_head<kColTiles>(p, w, head, wave * kCols + quad * 4, [&](int c) { return out[c]; }, reference[l16], all,
                        wave == 0 && quad == 0);
}

// 64 heads at a time, of many tokens.  Eight waves work on 32 rows in three stages,
// each a tile behind the one before, with one barrier per tile:
//   scores   wave (rg, kg) multiplies a quarter of the key columns of 16 rows with
//            the queries of all 64 heads (held in registers), and leaves the values that
//            it expanded on the way and its part of the other waves' scores in LDS;
//   weights  it adds up the four parts of its 16 rows' scores of 16 heads and leaves
//            their weights in LDS;
//   output   it multiplies all 32 rows' weights of all heads with 64 of the 512
//            columns of the values.
// Alone, each stage keeps one unit of a CU busy (matrix cores, LDS, conversion,
// exponentials) and then waits for the others' waves; in one stream they overlap.
// 128 tokens of 128 heads over 2048 rows each take 104 us, 1.4 us per 32 rows, of which
// the products take 1600 cycles, about half: 18 matrix instructions of scores per wave, 16 of the
// output and 16 for the weights' rests, without which it took 81 us.  Of the other half one part is
// known: every second tile the first wave reads the entries of two tiles at the end of a stage, and
// waits for them with its keys at the start of the next, where all waves then wait for it.
constexpr int kWideRows = 32;
constexpr int kWideHeads = 64;

template <bool kMx4>
__global__ __launch_bounds__(512, 2) void attend_wide_kernel(AttendParams p, int head_blocks, int tiles_per_split) {
  constexpr int kTiles = kWideHeads / 16, kColTiles = kLatent / 8 / 16;
  constexpr int kLoads = kMx4 ? 1 : 4;                     // 16 bytes each
  constexpr int kBufferBytes = kWideRows * kValueStride;
  extern __shared__ __align__(16) unsigned char lds[];
  unsigned char* const values = lds;                                                        // [3] tiles
  unsigned char* const weights = lds + 3 * kBufferBytes;                                    // [2][head tiles][64 lanes] 16 bytes
  unsigned char* const rests = weights + 2 * kTiles * 1024;                                 // [2][head tiles][64 lanes] 8 bytes
  f32x4* const parts = reinterpret_cast<f32x4*>(rests + 2 * kTiles * 512);                  // [2][2][4][3][64]
  uint64_t* const row_at = reinterpret_cast<uint64_t*>(parts + 2 * 2 * 4 * 3 * 64);         // [4] tiles: rows, 0 = none
  float* const group_top = reinterpret_cast<float*>(row_at + 4 * kWideRows);                // [2][heads]
  float* const reference = group_top + 2 * kWideHeads;                                      // [heads]
  int* const raised = reinterpret_cast<int*>(reference + kWideHeads);                       // [2]

  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rg = wave / 4, kg = wave % 4;
  const Share w = share_of(p, head_blocks, tiles_per_split, kWideRows);
  const int head0 = w.head_block * kWideHeads;

  // The head tile whose weights the wave makes comes first.  Of the two steps of
  // rotated columns it takes step kg % 2 for that one and the next.
  auto head_of = [&](int h) { return head0 + (h + kg) % kTiles * 16 + l16; };
  u32x4 raw[kTiles][4], raw_turned[2];
#pragma unroll
  for (int h = 0; h < kTiles; ++h)
#pragma unroll
    for (int j = 0; j < 4; ++j) raw[h][j] = load_query(p, w, head_of(h), kg * 128 + (kMx4 ? 32 * quad + 8 * j : 32 * j + 8 * quad));
#pragma unroll
  for (int h = 0; h < 2; ++h) raw_turned[h] = load_query(p, w, head_of(h), kLatent + kg % 2 * 32 + 8 * quad);

  // the first wave finds the rows of two tiles at a time, one per lane; their
  // addresses go to LDS, and all waves fetch their keys a tile ahead
  RowFinder finder{};
  auto leave = [&](const RowFinder& f, int t) { row_at[(t & 3) * kWideRows + lane_here()] = f.address(p, w); };
  if (wave == 0) {
    RowFinder second;
    finder.look(p, w, lane);
    second.look(p, w, 2 * kWideRows + lane);
    leave(finder, 0);
    finder.look(p, w, 4 * kWideRows + lane);
    leave(second, 2);
  }
  if (threadIdx.x < kWideHeads) reference[threadIdx.x] = -INFINITY;
  if (threadIdx.x < 2) raised[threadIdx.x] = 0;

  u32x4 key[kLoads], turned;
  uint32_t scales = 0;
  unsigned counts = 0;   // bits of this lane's rows (quad * 4 + i) that count, of the tile whose keys are held
  auto find_keys = [&](int t) { return row_at[(t & 3) * kWideRows + rg * 16 + l16]; };
  auto take_keys = [&](uint64_t& at) {
    counts = static_cast<unsigned>(__ballot(at != 0) >> (quad * 4)) & 15u;
    if (at == 0) at = reinterpret_cast<uint64_t>(zero_row);
  };
  auto load_part = [&](uint64_t at, int n) {   // of kLoads + 2 loads the n-th
    if (n < kLoads) key[n] = load_global<u32x4>(at + (quad * 16 + kg * (kMx4 ? 64 : 256)) + 64 * n);
    if (n == kLoads) turned = load_global<u32x4>(at + (quad * 16 + (kMx4 ? kMx4RopeAt : kLatent * 2) + kg % 2 * 64));
    if (kMx4 && n == kLoads + 1) scales = load_global<uint32_t>(at + (kMx4CodeBytes + 4 * kg));
  };
  __syncthreads();
  {
    uint64_t at = find_keys(0);
    take_keys(at);
#pragma unroll
    for (int n = 0; n < kLoads + 2; ++n) load_part(at, n);
  }
  __builtin_amdgcn_sched_barrier(0);   // the first keys are on their way before the queries are waited for
  bf16x8 query[kTiles][4], query_turned[2];
#pragma unroll
  for (int h = 0; h < kTiles; ++h)
#pragma unroll
    for (int j = 0; j < 4; ++j) query[h][j] = signed_query(p, head_of(h), raw[h][j]);
#pragma unroll
  for (int h = 0; h < 2; ++h) query_turned[h] = signed_query(p, head_of(h), raw_turned[h]);

  const float scale = p.scale == 0.f ? 1.f : fabsf(p.scale) * kLog2e;   // scores in powers of two
  const float per_scale = 1.f / scale;
  float ref = -INFINITY, sum = 0.f, add = 0.f;
  f32x4 mine{}, s{};            // the wave's own part of its scores, and those scores of the tile that is weighed
  unsigned now = 0;             // rows that count of the tile whose parts are in LDS
  f32x4 out[kColTiles][kTiles];
#pragma unroll
  for (int c = 0; c < kColTiles; ++c)
#pragma unroll
    for (int h = 0; h < kTiles; ++h) out[c][h] = f32x4{};

  // weights of s relative to the reference, for tile t
  auto weigh = [&](int t) {
    const float base = zero_if_none(ref);
    f32x4 e;
#pragma unroll
    for (int j = 0; j < 4; ++j) e[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[j], scale, -base));
    add = (e[0] + e[1]) + (e[2] + e[3]);
    const bf16x4 high = rounded(e);
    const unsigned to = (t & 1) * kTiles * 64 + kg * 64 + lane_here();
    *reinterpret_cast<bf16x4*>(weights + to * 16 + rg * 8) = high;
    *reinterpret_cast<uint32_t*>(rests + to * 8 + rg * 4) = rest_encode(rest_of(e, high), p.rest_unit);
  };
  // some score of tile t raises its reference: all waves agree on new
  // ones and bring what they hold to them
  auto raise = [&](int t) {
    const int x = lane_here(), x16 = x & 15;
    float high = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])) * scale + p.above;
    high = fmaxf(high, __shfl_xor(high, 16));
    high = fmaxf(high, __shfl_xor(high, 32));
    if (x < 16) group_top[rg * kWideHeads + kg * 16 + x16] = high;
    __syncthreads();
    auto fresh = [&](int head) { return fmaxf(reference[head], fmaxf(group_top[head], group_top[kWideHeads + head])); };
#pragma unroll
    for (int h = 0; h < kTiles; ++h) {
      const float old = reference[h * 16 + x16];
      // nothing is held yet where there is no reference
      const float by = old == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(old - fresh(h * 16 + x16));
#pragma unroll
      for (int c = 0; c < kColTiles; ++c) out[c][h] *= by;
    }
    high = fresh(kg * 16 + x16);
    if (ref != -INFINITY) sum *= __builtin_amdgcn_exp2f(ref - high);
    ref = high;
    weigh(t);
    __syncthreads();
    // read again after the next barrier at the earliest
    if (rg == 0 && x < 16) reference[kg * 16 + x16] = ref;
  };

  const unsigned lane16 = lane * 16;
  const unsigned v_to = (rg * 16 + l16) * kValueStride + kg * 256 + value_part(l16, (kMx4 ? 4 : 1) * quad);
  const unsigned v_from = values_from(lane, wave * 64);
  const int scale_shift = quad * 8;

  // one barrier's work: the output of tile t, weights of tile t + 1, scores of tile t + 2
  auto stages = [&](auto with_output, auto with_weights, auto with_scores, int t, int buffer) {
    constexpr bool kOutput = decltype(with_output)::value, kWeights = decltype(with_weights)::value,
                   kScores = decltype(with_scores)::value;
    // what the other stages read of LDS comes while the scores' products run
    int high = 0;
    const unsigned char* const v_lds = values + buffer * kBufferBytes;
    const unsigned char* const e_lds = weights + (t & 1) * kTiles * 1024 + lane16;
    constexpr int kAhead = 2;
    bf16x8 v[kColTiles], e[kTiles];
    if constexpr (kOutput) {
      high = raised[t & 1];
#pragma unroll
      for (int h = 0; h < kTiles; ++h) e[h] = *reinterpret_cast<const bf16x8*>(e_lds + h * 1024);
#pragma unroll
      for (int c = 0; c < kAhead; ++c) v[c] = load_values(v_lds, v_from ^ (c * 32));
    }
    uint64_t next_at = 0;
    if constexpr (kScores) next_at = find_keys(t + 3);
    f32x4 part[kTiles];
    unsigned counted = 0;
    if constexpr (kScores) {
      unsigned char* const to = values + (buffer == 0 ? 2 : buffer - 1) * kBufferBytes;
      const float unit = mx4_unit((scales >> scale_shift) & 255u);
      auto operand = [&](int j) {
        bf16x8 k;
        if constexpr (kMx4) k = mx4_decode8(key[0][j], unit);
        else k = __builtin_bit_cast(bf16x8, key[j]);
        return k;
      };
      // the operand of a step is expanded during the one before
      bf16x8 k = operand(0);
#pragma unroll
      for (int h = 0; h < kTiles; ++h) part[h] = f32x4{};
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        bf16x8 following{};
        if (j < 3) following = operand(j + 1);
        *reinterpret_cast<bf16x8*>(to + (v_to ^ (j * (kMx4 ? 16 : 64)))) = k;
#pragma unroll
        for (int h = 0; h < kTiles; ++h) part[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, query[h][j], part[h], 0, 0, 0);
        k = following;
      }
      counted = counts;
      // the next keys' loads start where registers are free, two here and the rest one by
      // one between the products below (all of them below: 5% longer)
      take_keys(next_at);
      load_part(next_at, 0);
      load_part(next_at, kMx4 ? 2 : 1);
#pragma unroll
      for (int h = 0; h < 2; ++h)
        part[h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, turned), query_turned[h], part[h], 0, 0, 0);
    }
    if constexpr (kOutput) {
      if (high == t + 1) {
        raise(t);
#pragma unroll
        for (int h = 0; h < kTiles; ++h) e[h] = *reinterpret_cast<const bf16x8*>(e_lds + h * 1024);
      }
      sum += add;
    }
    f32x4 theirs[3];
    if constexpr (kWeights) {
      const unsigned char* const from = reinterpret_cast<unsigned char*>(parts) + (((t + 1) & 1) * 8 + rg * 4 + kg) * 3 * 1024 + lane16;
#pragma unroll
      for (int n = 0; n < 3; ++n) theirs[n] = *reinterpret_cast<const f32x4*>(from + n * 1024);
    }
    unsigned char* const parts_to = reinterpret_cast<unsigned char*>(parts) + (((t + 2) & 1) * 8 + rg * 4) * 3 * 1024 + lane16;
#pragma unroll
    for (int c = 0; c < kColTiles; ++c) {
      if constexpr (kOutput) {
        if (c + kAhead < kColTiles) v[c + kAhead] = load_values(v_lds, v_from ^ ((c + kAhead) * 32));
#pragma unroll
        for (int h = 0; h < kTiles; ++h) out[c][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[c], e[h], out[c][h], 0, 0, 0);
      }
      if constexpr (kScores) {
        // the rest of the loads and the scores' way to the others, one by one between products
        if (kMx4 ? c == 0 : c < 3) load_part(next_at, kMx4 ? 1 : c + 2);
        if (c > 0) *reinterpret_cast<f32x4*>(parts_to + (kg + c) % 4 * 3 * 1024 + (c - 1) * 1024) = part[c];
      }
    }
    if constexpr (kOutput) {
      const unsigned char* const rest_from = rests + (t & 1) * kTiles * 512 + lane16 / 2;
      bf16x8 low[kTiles];
#pragma unroll
      for (int h = 0; h < kTiles; ++h) low[h] = rest_decode(*reinterpret_cast<const u32x2*>(rest_from + h * 512), p.rest_unit);
#pragma unroll
      for (int c = 0; c < kColTiles; ++c)
#pragma unroll
        for (int h = 0; h < kTiles; ++h) out[c][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v[c], low[h], out[c][h], 0, 0, 0);
    }
    if constexpr (kWeights) {
      s = (mine + theirs[0]) + (theirs[1] + theirs[2]);
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] = (now >> j) & 1 ? s[j] : -INFINITY;
    }
    if constexpr (kScores) {
      now = counted;
      mine = part[0];
    }
    if constexpr (kWeights) {
      weigh(t + 1);
      // a score that raises the reference is noted
      const float top = fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3]));
      if (__any(top > (ref - p.above + kSlack) * per_scale)) raised[(t + 1) & 1] = t + 2;
    }
    if constexpr (kScores) {
      if (wave == 0 && t >= 0 && (t & 1) == 0) {
        leave(finder, t + 4);
        finder.look(p, w, (t + 6u) * kWideRows + lane_here());
      }
    }
    __syncthreads();
  };
  const std::true_type yes{};
  const std::false_type no{};
  if (w.tiles > 0) {
    stages(no, no, yes, -2, 1);
    if (w.tiles > 1) {
      stages(no, yes, yes, -1, 2);
      int buffer = 0;
      for (int t = 0; t + 2 < w.tiles; ++t) {
        stages(yes, yes, yes, t, buffer);
        buffer = buffer == 2 ? 0 : buffer + 1;
      }
      stages(yes, yes, no, w.tiles - 2, buffer);
      stages(yes, no, no, w.tiles - 1, buffer == 2 ? 0 : buffer + 1);
    } else {
      stages(no, yes, no, -1, 2);
      stages(yes, no, no, 0, 0);
    }
  }

  // the waves' sums of weights
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  if (quad == 0) group_top[rg * kWideHeads + kg * 16 + l16] = sum;
  __syncthreads();
#pragma unroll
  for (int h = 0; h < kTiles; ++h) {
    const int head = head0 + h * 16 + l16;
    if (head >= p.heads) continue;
    store_head<kColTiles>(p, w, head, wave * 64 + quad * 4, [&](int c) { return out[c][h]; }, reference[h * 16 + l16],
                          group_top[h * 16 + l16] + group_top[kWideHeads + h * 16 + l16], wave == 0 && quad == 0);
  }
}

// Joins the parts of one (query token, head), kCols of its columns: the parts' factors
// are made once, then groups of threads share the parts, four columns per thread, with several
// parts in flight.  Fewer columns per workgroup are for few results of many parts:
// 16 results of 512 parts took 57 us with the attention before them, and 34 so.
constexpr int kMostSplits = 512;
template <int kCols>
__global__ __launch_bounds__(kMostSplits) void combine_kernel(AttendParams p) {
  constexpr int kLanes = kCols / 4, kGroups = kMostSplits / kLanes, kFirst = 8;
  __shared__ float factor[kMostSplits], per_wave[2][8];
  __shared__ f32x4 group_sum[kGroups - 1][kLanes];
  const int64_t token = blockIdx.x / p.heads;
  const int head = static_cast<int>(blockIdx.x - token * p.heads);
  const int64_t first = token * p.plan.splits * p.heads + head;
  const int tid = threadIdx.x, wave = tid / 64;
  const f32x2 ml = tid < p.plan.splits ? p.part_ml[first + static_cast<int64_t>(tid) * p.heads] : f32x2{-INFINITY, 0.f};
  // the first parts come while their factors are found
  const int group = tid / kLanes, col = blockIdx.y * kCols + tid % kLanes * 4;
  const float* part = p.part_out + first * kLatent + col;
  const int64_t stride = static_cast<int64_t>(p.heads) * kLatent;
  f32x4 early[kFirst];
#pragma unroll
  for (int i = 0; i < kFirst; ++i) {
    const int at = group + i * kGroups;
    early[i] = at < p.plan.splits ? *reinterpret_cast<const f32x4*>(part + at * stride) : f32x4{};
  }
  float top = ml[1] != 0.f ? ml[0] : -INFINITY;   // a part without a row that counts has no reference
#pragma unroll
  for (int d = 32; d > 0; d /= 2) top = fmaxf(top, __shfl_xor(top, d));
  if ((tid & 63) == 0) per_wave[0][wave] = top;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 8; ++i) top = fmaxf(top, per_wave[0][i]);
  const float base = zero_if_none(top);
  const float w = ml[1] != 0.f ? __builtin_amdgcn_exp2f(ml[0] - base) : 0.f;
  factor[tid] = w;
  float all = ml[1] != 0.f ? w * ml[1] : 0.f;
#pragma unroll
  for (int d = 32; d > 0; d /= 2) all += __shfl_xor(all, d);
  if ((tid & 63) == 0) per_wave[1][wave] = all;
  __syncthreads();
  all = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) all += per_wave[1][i];

  f32x4 o{};
#pragma unroll
  for (int i = 0; i < kFirst; ++i) {
    const int at = group + i * kGroups;
    if (at < p.plan.splits) o += early[i] * factor[at];
  }
#pragma unroll 8
  for (int i = group + kFirst * kGroups; i < p.plan.splits; i += kGroups)
    o += *reinterpret_cast<const f32x4*>(part + i * stride) * factor[i];
  if (group > 0) group_sum[group - 1][tid % kLanes] = o;
  __syncthreads();
  if (group > 0) return;
#pragma unroll
  for (int g = 0; g < kGroups - 1; ++g) o += group_sum[g][tid % kLanes];
  o *= all == 0.f ? 0.f : 1.f / all;
  *reinterpret_cast<bf16x4*>(p.out + token * p.out_token_stride + head * p.out_head_stride + col) = rounded(o);
  if (p.lse && tid == 0 && col == 0) p.lse[token * p.heads + head] = log_sum(p, top, all);
}

// The same for up to kMost parts, which is most calls: a thread makes the factors itself, without a barrier, and adds up
// four columns of a result (8192 results of 2 parts: 21 us by the kernel above, 8 us by this).
template <int kMost>
__global__ __launch_bounds__(256) void combine_few_kernel(AttendParams p) {
  const int64_t result = static_cast<int64_t>(blockIdx.x) * 2 + threadIdx.x / 128;
  const int64_t token = result / p.heads;
  if (token >= static_cast<int64_t>(p.cache.batch) * p.n_q) return;
  const int head = static_cast<int>(result - token * p.heads), col = threadIdx.x % 128 * 4;
  const int64_t first = token * p.plan.splits * p.heads + head;
  f32x4 part[kMost];
  f32x2 ml[kMost];
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const int64_t at = first + static_cast<int64_t>(min(i, p.plan.splits - 1)) * p.heads;
    ml[i] = p.part_ml[at];
    part[i] = i < p.plan.splits ? *reinterpret_cast<const f32x4*>(p.part_out + at * kLatent + col) : f32x4{};
  }
  float top = -INFINITY, all = 0.f;
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    if (i >= p.plan.splits) ml[i][1] = 0.f;
    if (ml[i][1] != 0.f) top = fmaxf(top, ml[i][0]);   // a part without a row that counts has no reference
  }
  const float base = zero_if_none(top);
  f32x4 o{};
#pragma unroll
  for (int i = 0; i < kMost; ++i) {
    const float w = ml[i][1] != 0.f ? __builtin_amdgcn_exp2f(ml[i][0] - base) : 0.f;
    all += w * ml[i][1];
    o += part[i] * w;
  }
  o *= all == 0.f ? 0.f : 1.f / all;
  *reinterpret_cast<bf16x4*>(p.out + token * p.out_token_stride + head * p.out_head_stride + col) = rounded(o);
  if (p.lse && col == 0) p.lse[token * p.heads + head] = log_sum(p, top, all);
}

int head_blocks_of(int heads, AttendKernel kernel) { return (heads + heads_of(kernel) - 1) / heads_of(kernel); }

template <bool kMx4, int kWaves>
hipError_t launch_narrow(const AttendParams& p, int64_t groups, int head_blocks, int tiles_per_split, hipStream_t s) {
  constexpr size_t lds = kWaves * 16 * kValueStride + kWaves * 1024 + (kWaves + 1) * 16 * 4 + 16;
  static_assert(8 / kWaves * lds <= 160 * 1024, "LDS of a CU's workgroups");
  if (const hipError_t e = allow_lds<&attend_kernel<kMx4, kWaves>>(lds); e != hipSuccess) return e;
  attend_kernel<kMx4, kWaves><<<dim3(static_cast<unsigned>(groups)), kWaves * 64, lds, s>>>(p, head_blocks, tiles_per_split);
  return hipGetLastError();
}

template <bool kMx4>
hipError_t launch_wide(const AttendParams& p, int64_t groups, int head_blocks, int tiles_per_split, hipStream_t s) {
  constexpr size_t lds = 3 * kWideRows * kValueStride + 2 * (kWideHeads / 16) * (1024 + 512) + 2 * 2 * 4 * 3 * 1024 + 4 * kWideRows * 8 +
                         3 * kWideHeads * 4 + 8;
  static_assert(lds <= 160 * 1024, "LDS of a workgroup");
  if (const hipError_t e = allow_lds<&attend_wide_kernel<kMx4>>(lds); e != hipSuccess) return e;
  attend_wide_kernel<kMx4><<<dim3(static_cast<unsigned>(groups)), 512, lds, s>>>(p, head_blocks, tiles_per_split);
  return hipGetLastError();
}

template <bool kMx4>
hipError_t launch_format(const AttendParams& p, hipStream_t s) {
  const AttendKernel kernel = p.plan.kernel;
  const int head_blocks = head_blocks_of(p.heads, kernel), rows = kernel == AttendKernel::k64Heads ? kWideRows : rows_of(kernel);
  const int tiles = tiles_of(p.topk, rows), each = tiles_of(tiles, p.plan.splits);
  const int64_t groups = static_cast<int64_t>(p.cache.batch) * p.n_q * head_blocks * p.plan.splits;
  switch (kernel) {
    case AttendKernel::k16Heads: return launch_narrow<kMx4, 4>(p, groups, head_blocks, each, s);
    case AttendKernel::k16HeadsAlone: return launch_narrow<kMx4, 8>(p, groups, head_blocks, each, s);
    default: return launch_wide<kMx4>(p, groups, head_blocks, each, s);
  }
}

// Time of a call in us, from ones that were timed in a graph: what a workgroup needs
// at its start and end, its tiles, and the parts written and joined.  920 calls
// of 1 to 128 tokens, 8 to 128 heads, 150 to 2048 rows and of long contexts, 3992 ways in all, took 5%
// more or less than this says, and the ways chosen by it 0.1% more than the best
// (6% at worst); their times are in profiles/latent_attend_choices.csv.
double attend_cost(bool mx4, AttendKernel kernel, int64_t tokens, int heads, int tiles, int splits) {
  const int64_t groups = tokens * head_blocks_of(heads, kernel) * splits;
  const int each = (tiles + splits - 1) / splits;
  auto rounds = [&](int64_t at_once) { return static_cast<double>((groups + at_once - 1) / at_once); };
  double at = 0;
  if (kernel == AttendKernel::k64Heads) at = rounds(256) * (5.9 + 0.09 * std::min(heads, 64) + 2.7 * each);
  else if (kernel == AttendKernel::k16HeadsAlone) at = rounds(256) * (8.2 + (mx4 ? 2.5 : 4.8) * each);
  else if (groups <= 256) at = 6. + (mx4 ? 1.7 : 2.5) * each;   // a CU has one workgroup and not two
  else at = rounds(512) * (7.9 + (mx4 ? 2.4 : 4.2) * each);
  if (splits == 1) return at;
  const double megabytes = static_cast<double>(tokens) * splits * heads * (kLatent * 4) / 1e6;
  return at + 2.0 + 0.6 * std::min(megabytes, 17.) + 0.1 * std::max(megabytes - 17., 0.);
}

}  // namespace

int64_t attend_threads(const AttendPlan& plan, int64_t tokens, int heads) {
  return tokens * head_blocks_of(heads, plan.kernel) * plan.splits * (plan.kernel == AttendKernel::k16Heads ? 256 : 512);
}

// Which kernel, and how many workgroups share a token's rows: the least of the times
// above for parts that give 128, 256 or 512 workgroups.  Measured (us, 4-bit rows; 16 heads
// with 64-row tiles in 256 and 512 workgroups, with 128-row tiles in 256, 64 heads
// in 128 and 256):
//   tokens x heads x rows    64 rows: 256    512    128 rows    64 heads: 128    256
//       1 x  64 x    256          9.9         9.8     12.8          16.5        16.4
//      33 x  40 x   1000         25.8        27.2     24.3          31.0        29.2
//      33 x  64 x   1000         34.4        32.1     28.9          35.4        32.4
//      64 x  64 x   2048         63.3        54.9     50.2          62.5        45.8
//     128 x  64 x    256         20.3        20.3     26.0          24.2        29.6
//     128 x 128 x   2048        162.0       162.0    193.7         105.2       105.3
//       4 x  16 x 131072         67.8        55.4     55.8
//       1 x  16 x 131072         27.6        32.1     27.0
//   the same in bfloat16:
//       1 x  64 x    256         10.9        10.9     15.5          17.4        17.4
//      16 x  64 x   2048         32.2        34.0     34.2          31.4        29.4
//      33 x  40 x   1000         31.1        31.8     32.8          30.4        27.0
AttendPlan attend_plan(int format, int batch, int n_q, int heads, int topk) {
  const int64_t tokens = static_cast<int64_t>(batch) * n_q;
  AttendPlan best{AttendKernel::k16Heads, 1};
  double least = INFINITY;
  for (AttendKernel kernel : {AttendKernel::k16Heads, AttendKernel::k16HeadsAlone, AttendKernel::k64Heads}) {
    if (kernel == AttendKernel::k64Heads && heads <= 16) break;
    const int64_t groups = tokens * head_blocks_of(heads, kernel);
    const int tiles = tiles_of(topk, rows_of(kernel));
    int last = 0;
    for (int64_t target : {128, 256, 512}) {
      if (target == 512 && kernel != AttendKernel::k16Heads) break;   // one workgroup per CU
      const int64_t want = std::max<int64_t>(1, std::min<int64_t>(target / groups, tiles));
      const int each = static_cast<int>((tiles + want - 1) / want);
      const int splits = each > 0 ? (tiles + each - 1) / each : 1;
      if (splits == last) continue;
      last = splits;
      const double cost = attend_cost(format == 1, kernel, tokens, heads, tiles, splits);
      if (cost < least) least = cost, best = {kernel, splits};
    }
  }
  return best;
}

hipError_t launch_attend(const AttendParams& call, int format, hipStream_t s) {
  AttendParams p = call;
  int bits = 0;   // of the number of entries
  while (bits < 31 && (int64_t{1} << bits) < p.topk) ++bits;
  p.above = kSlack + static_cast<float>(bits);
  p.rest_unit = std::ldexp(kRestUnit, -bits);
  hipError_t e = format == 1 ? launch_format<true>(p, s) : launch_format<false>(p, s);
  const int splits = p.plan.splits;
  if (e != hipSuccess || splits <= 1) return e;
  const int64_t results = static_cast<int64_t>(p.cache.batch) * p.n_q * p.heads;
  const unsigned pairs = static_cast<unsigned>((results + 1) / 2);
  if (splits <= 4) combine_few_kernel<4><<<pairs, 256, 0, s>>>(p);
  else if (splits <= 16) combine_few_kernel<16><<<pairs, 256, 0, s>>>(p);
  else if (results <= 128) combine_kernel<128><<<dim3(static_cast<unsigned>(results), 4), kMostSplits, 0, s>>>(p);
  else combine_kernel<512><<<dim3(static_cast<unsigned>(results)), kMostSplits, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace avsg
