// Attention of a step's query tokens over latent cache rows:
//   out = sum_i w_i v_i / sum_i w_i,  w_i = exp(scale q . k_i),
// in one pass over the rows.  Every head of a token reads the same rows, and a
// row's latent part is key and value at once, so a row is brought in once per
// workgroup and serves up to 64 heads twice: 2 * (576 + 512) operations per row
// and head, on the matrix cores.
#include "latent_internal.h"

namespace avsg {
namespace {

constexpr int kRowTile = 64;                  // rows of one pass through the loop
constexpr int kRowWaves = kRowTile / 16;      // waves that share them, 16 each
// LDS row of values: 1024 bytes and 32 more, so that the four rows whose
// columns one group of 16 lanes reads at once lie in different banks
constexpr int kValueStride = kLatent * 2 + 32;
constexpr int kValueBytes = kRowTile * kValueStride;
// Weights are kept relative to a reference that need not be the maximum: it is
// raised only when a score passes it by this much (in powers of two), which in
// float32 and bfloat16 costs no accuracy and saves the exchange of maxima
// between waves for nearly every tile.
constexpr float kSlack = 40.f;

__device__ __align__(16) const unsigned char zero_row[kRowBytesBf16] = {};

// What is known of a row before its address: loaded two tiles ahead.
struct RowMeta {
  int row, pos, page;
};

// kHeadTiles * 16 heads per workgroup; kKeyGroups groups of four waves.  In the
// first half of a tile wave (rt, kg) multiplies its share of the columns of the
// keys of its 16 rows with the queries (held in registers) and leaves the
// values that it expanded on the way in LDS.  With two groups the halves of a
// score meet in LDS, each group taking half of the heads.  Scores become weights,
// which go to LDS.  In the second half each wave multiplies all 64 rows' weights
// of all heads with its own range of the 512 columns of the values.  Operands of
// the products:
//   scores   A = keys     lane l: row l % 16, eight columns     B = queries  lane l: head l % 16, the same columns
//            result lane l: head l % 16, rows (l / 16) * 4 .. + 3
//   output   A = values^T lane l: column l % 16, eight rows     B = weights  lane l: head l % 16, the same rows
//            result lane l: head l % 16, columns (l / 16) * 4 .. + 3
// The eight rows of the second product are rows (l / 16) * 4 .. + 3 of two
// 16-row tiles: what a lane holds of the first one's result, so weights need no
// exchange within a wave.
// 64 heads: queries and output of a wave fill 208 of the 256 registers that two
// waves per SIMD leave; splitting the keys' columns (not the heads) between the
// groups leaves each wave half of the keys to load and to expand.
template <int kHeadTiles, int kKeyGroups, bool kMx4>
__global__ __launch_bounds__(256 * kKeyGroups, 2) void attend_kernel(AttendParams p, int head_blocks, int tiles_per_split) {
  constexpr int kTiles = kHeadTiles / kKeyGroups;              // head tiles whose weights a wave makes
  constexpr int kCols = kLatent / (kRowWaves * kKeyGroups);    // columns of a wave's output
  constexpr int kColTiles = kCols / 16;
  constexpr int kValueBuffers = kKeyGroups;
  constexpr int kWeightBytes = kHeadTiles * 2048;
  constexpr int kHalves = 2 / kKeyGroups;                      // of the key columns, a wave's share
  constexpr int kLoads = (kMx4 ? 2 : 8) * kHalves;             // 16 bytes each
  constexpr int kSteps = 8 * kHalves;                          // products over 32 latent columns
  constexpr int kChains = kHeadTiles == 1 ? 2 : 1;             // sums that a head tile's products alternate between
  extern __shared__ __align__(16) unsigned char lds[];
  unsigned char* const values = lds;
  unsigned char* const weights = lds + kValueBuffers * kValueBytes;
  float* const wave_top = reinterpret_cast<float*>(weights + kWeightBytes);   // [4][heads]
  float* const reference = wave_top + kRowWaves * kHeadTiles * 16;            // [heads]
  int* const raised = reinterpret_cast<int*>(reference + kHeadTiles * 16);    // [4]
  unsigned char* const halves = reinterpret_cast<unsigned char*>(raised + 4); // two groups: [4][2][kTiles][64] f32x4

  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  // A lane's number that the compiler takes for a new value: what is derived from
  // it is computed where it is used and not kept in registers across the loop.
  auto here = [&]() {
    int x = lane;
    asm volatile("" : "+v"(x));
    return x;
  };
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rt = wave % kRowWaves, kg = wave / kRowWaves;

  // workgroups of one request lie next to each other on one XCD, whose L2 then
  // serves the rows that they share
  const unsigned total = gridDim.x, per = total / kXcds, more = total % kXcds, xcd = blockIdx.x % kXcds;
  const unsigned id = xcd * per + min(xcd, more) + blockIdx.x / kXcds;
  const unsigned share = head_blocks * p.splits;
  const int64_t token = id / share;
  const int hb = (id % share) % head_blocks, split = (id % share) / head_blocks;
  const int r = static_cast<int>(token / p.n_q);
  const int head0 = hb * kHeadTiles * 16;

  const int64_t len = p.lens ? p.lens[token] : INT64_MAX;
  // entries that can count: with their positions given, any
  const int limit = p.index ? p.topk : static_cast<int>(len < 0 ? 0 : len < p.topk ? len : p.topk);
  const int tile0 = split * tiles_per_split;
  const int tiles = min(tiles_per_split, (limit + kRowTile - 1) / kRowTile - tile0);
  const int32_t* const rows = p.rows ? p.rows + token * p.topk : nullptr;
  const int32_t* const index = p.index ? p.index + token * p.topk : nullptr;

  for (int i = threadIdx.x; i < kHeadTiles * 16; i += blockDim.x) reference[i] = -INFINITY;
  if (threadIdx.x < 4) raised[threadIdx.x] = 0;

  auto load_meta = [&](int t) {
    RowMeta m{-1, -1, -1};
    const int i = (tile0 + t) * kRowTile + rt * 16 + (here() & 15);
    if (t < tiles && i < limit) {
      m.row = rows ? rows[i] : i;
      m.pos = index ? index[i] : i;
      if (!rows && p.cache.table && i < p.cache.capacity)
        m.page = p.cache.table[static_cast<int64_t>(r) * p.cache.pages_per_request + (i >> p.cache.page_shift)];
    }
    return m;
  };
  auto address = [&](const RowMeta& m) -> uint64_t {
    if (m.row < 0 || m.row >= p.cache.capacity || m.pos < 0 || m.pos >= len) return 0;
    int64_t page = m.page;
    if (rows || !p.cache.table) {
      page = static_cast<int64_t>(r) * p.cache.pages_per_request + (m.row >> p.cache.page_shift);
      if (p.cache.table) page = p.cache.table[page];
    }
    if (page < 0 || page >= p.cache.pages) return 0;
    return p.cache.base + page * p.cache.page_stride + (m.row & p.cache.page_mask) * p.cache.row_stride;
  };

  // A half is 256 columns in a row, eight steps of 32.  4-bit rows: of every four
  // steps a lane has one block of 32 columns, 16 bytes; bfloat16 rows: of every
  // step eight columns.
  u32x4 key[kLoads], turned[kHalves];
  u32x2 scales[kHalves];
  unsigned counts = 0;   // bits of this lane's four rows (quad * 4 + i) that count
  auto load_keys = [&](const RowMeta& m) {
    uint64_t at = address(m);
    const unsigned x = here() >> 4;
    counts = static_cast<unsigned>(__ballot(at != 0) >> (x * 4)) & 15u;
    if (at == 0) at = reinterpret_cast<uint64_t>(zero_row);
    const uint64_t a = at + (16 * x + kg * (kMx4 ? 128 : 512));
#pragma unroll
    for (int j = 0; j < kLoads; ++j) key[j] = load_global<u32x4>(a + 64 * j);
#pragma unroll
    for (int j = 0; j < kHalves; ++j) {
      if constexpr (kMx4) scales[j] = load_global<u32x2>(at + kMx4CodeBytes + 8 * (kg + j));
      turned[j] = load_global<u32x4>(at + (16 * x + (kMx4 ? kMx4RopeAt : kLatent * 2) + 64 * kg) + 64 * j);
    }
  };

  RowMeta next = load_meta(0);
  // a group's own head tiles come first
  bf16x8 query[kHeadTiles][kSteps + kHalves];
#pragma unroll
  for (int h = 0; h < kHeadTiles; ++h) {
    const int head = head0 + (h + kg * kTiles) % kHeadTiles * 16 + l16;
    const bool there = head < p.heads;
    const __bf16* q = p.q + token * p.q_token_stride + (there ? head : 0) * p.q_head_stride;
#pragma unroll
    for (int j = 0; j < kSteps + kHalves; ++j) {
      const int col = j >= kSteps ? kLatent + 32 * (kg + j - kSteps) + 8 * quad
                      : kMx4      ? kg * 256 + ((j / 4) * 4 + quad) * 32 + (j % 4) * 8
                                  : kg * 256 + 32 * j + 8 * quad;
      query[h][j] = *reinterpret_cast<const bf16x8*>(q + col);
      if (!there) query[h][j] = bf16x8{};
    }
  }
  load_keys(next);
  next = load_meta(1);

  const float scale = p.scale * 1.4426950408889634f;   // scores in powers of two
  float ref[kTiles], sum[kTiles];
#pragma unroll
  for (int h = 0; h < kTiles; ++h) ref[h] = -INFINITY, sum[h] = 0.f;
  f32x4 out[kColTiles][kHeadTiles];
#pragma unroll
  for (int c = 0; c < kColTiles; ++c)
#pragma unroll
    for (int h = 0; h < kHeadTiles; ++h) out[c][h] = f32x4{};

  __syncthreads();

  for (int t = 0; t < tiles; ++t) {
    unsigned char* const v_lds = values + (kValueBuffers == 2 ? t & 1 : 0) * kValueBytes;
    // one buffer: every wave is done with the last tile's
    if constexpr (kValueBuffers == 1) __syncthreads();

    unsigned char* value_to;
    int shift;
    {
      const int x = here();
      value_to = v_lds + (rt * 16 + (x & 15)) * kValueStride + (kMx4 ? 64 : 16) * (x >> 4) + 512 * kg;
      shift = (x >> 4) * 8;
    }
    f32x4 score[kHeadTiles][kChains];
#pragma unroll
    for (int h = 0; h < kHeadTiles; ++h)
#pragma unroll
      for (int j = 0; j < kChains; ++j) score[h][j] = f32x4{};
#pragma unroll
    for (int j = 0; j < kSteps; ++j) {
      bf16x8 k;
      if constexpr (kMx4) k = mx4_decode8(key[j / 4][j % 4], mx4_unit((scales[j / 8][(j / 4) % 2] >> shift) & 255u));
      else k = __builtin_bit_cast(bf16x8, key[j]);
      *reinterpret_cast<bf16x8*>(value_to + (kMx4 ? (j / 4) * 256 + (j % 4) * 16 : 64 * j)) = k;
#pragma unroll
      for (int h = 0; h < kHeadTiles; ++h)
        score[h][j % kChains] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k, query[h][j], score[h][j % kChains], 0, 0, 0);
    }
#pragma unroll
    for (int j = 0; j < kHalves; ++j)
#pragma unroll
      for (int h = 0; h < kHeadTiles; ++h)
        score[h][j % kChains] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, turned[j]), query[h][kSteps + j],
                                                                        score[h][j % kChains], 0, 0, 0);
    const unsigned now = counts;
    load_keys(next);
    next = load_meta(t + 2);

    f32x4 s[kTiles];
    if constexpr (kKeyGroups == 2) {
      f32x4* const mine = reinterpret_cast<f32x4*>(halves) + (rt * 2 + kg) * kTiles * 64 + here();
      const f32x4* const theirs = reinterpret_cast<const f32x4*>(halves) + (rt * 2 + (kg ^ 1)) * kTiles * 64 + here();
#pragma unroll
      for (int h = 0; h < kTiles; ++h) mine[h * 64] = score[kTiles + h][0];
      __syncthreads();
#pragma unroll
      for (int h = 0; h < kTiles; ++h) s[h] = score[h][0] + theirs[h * 64];
    } else {
#pragma unroll
      for (int h = 0; h < kTiles; ++h) s[h] = kChains == 2 ? score[h][0] + score[h][kChains - 1] : score[h][0];
    }

    unsigned char* const weight_to = weights + kg * kTiles * 2048 + (rt >> 1) * 1024 + here() * 16 + (rt & 1) * 8;
    // weights relative to the reference as it is; a score far above it is noted
    auto weigh = [&](int h) {
      const float base = ref[h] == -INFINITY ? 0.f : ref[h];
      bf16x4 w;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float e = __builtin_amdgcn_exp2f(s[h][i] - base);
        sum[h] += e;
        // rounded once; the sum keeps float32 weights, so the rounding errors
        // of many rows cancel in the output and do not touch the sum
        w[i] = static_cast<__bf16>(e);
      }
      *reinterpret_cast<bf16x4*>(weight_to + h * 2048) = w;
    };
    bool above = false;
    float before[kTiles];
#pragma unroll
    for (int h = 0; h < kTiles; ++h) {
      before[h] = sum[h];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        s[h][i] = (now >> i) & 1 ? s[h][i] * scale : -INFINITY;
        above |= s[h][i] > ref[h] + kSlack;
      }
      weigh(h);
    }
    if (__any(above) && lane == 0) raised[t & 1] = t + 1;
    __syncthreads();

    if (raised[t & 1] == t + 1) {
      const int x = here(), x16 = x & 15;
      // some score lies far above the reference: all waves agree on new ones and
      // bring what they hold to them
#pragma unroll
      for (int h = 0; h < kTiles; ++h) {
        float top = fmaxf(fmaxf(s[h][0], s[h][1]), fmaxf(s[h][2], s[h][3]));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        if (x < 16) wave_top[rt * kHeadTiles * 16 + (kg * kTiles + h) * 16 + x16] = top;
      }
      __syncthreads();
      auto fresh = [&](int head) {
        float top = reference[head];
#pragma unroll
        for (int w = 0; w < kRowWaves; ++w) top = fmaxf(top, wave_top[w * kHeadTiles * 16 + head]);
        return top;
      };
#pragma unroll
      for (int h = 0; h < kHeadTiles; ++h) {
        const float old = reference[h * 16 + x16];
        // nothing is held yet where there is no reference
        const float by = old == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(old - fresh(h * 16 + x16));
#pragma unroll
        for (int c = 0; c < kColTiles; ++c) out[c][h] *= by;
      }
#pragma unroll
      for (int h = 0; h < kTiles; ++h) {
        const float top = fresh((kg * kTiles + h) * 16 + x16);
        sum[h] = ref[h] == -INFINITY ? before[h] : before[h] * __builtin_amdgcn_exp2f(ref[h] - top);
        ref[h] = top;
        weigh(h);
      }
      __syncthreads();
      // read again after the next tile's barrier at the earliest
      if (rt == 0 && x < 16) {
#pragma unroll
        for (int h = 0; h < kTiles; ++h) reference[(kg * kTiles + h) * 16 + x16] = ref[h];
      }
    }

    const int x = here();
    const unsigned char* const weight_from = weights + x * 16;
    const unsigned value_from = ((x >> 4) * 4 + (x & 15) / 4) * kValueStride + (wave * kCols + (x & 3) * 4) * 2;
    typedef __attribute__((address_space(3))) bf16x4* lds_ptr;
    auto load_values = [&](int i) {   // column tile i % kColTiles of row pair i / kColTiles
      const unsigned at = value_from + i / kColTiles * 32 * kValueStride + i % kColTiles * 32;
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_ptr)(v_lds + at));
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_ptr)(v_lds + at + 16 * kValueStride));
      return bf16x8{lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
    };
    bf16x8 v = load_values(0), w[kHeadTiles];
#pragma unroll
    for (int i = 0; i < 2 * kColTiles; ++i) {
      const int c = i % kColTiles;
      if (c == 0) {
#pragma unroll
        for (int h = 0; h < kHeadTiles; ++h)
          w[h] = *reinterpret_cast<const bf16x8*>(weight_from + h * 2048 + i / kColTiles * 1024);
      }
      bf16x8 following{};
      if (i + 1 < 2 * kColTiles) following = load_values(i + 1);
      // 64 heads: the compiler is kept from reading further ahead than registers last
      if constexpr (kHeadTiles == 4) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int h = 0; h < kHeadTiles; ++h)
        out[c][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, w[h], out[c][h], 0, 0, 0);
      if constexpr (kHeadTiles == 4) __builtin_amdgcn_sched_barrier(0);
      v = following;
    }
  }

  // the waves' sums of weights
  __syncthreads();
#pragma unroll
  for (int h = 0; h < kTiles; ++h) {
    float x = sum[h];
    x += __shfl_xor(x, 16);
    x += __shfl_xor(x, 32);
    if (quad == 0) wave_top[rt * kHeadTiles * 16 + (kg * kTiles + h) * 16 + l16] = x;
  }
  __syncthreads();
#pragma unroll
  for (int h = 0; h < kHeadTiles; ++h) {
    const int head = head0 + h * 16 + l16;
    if (head >= p.heads) continue;
    float all = 0.f;
#pragma unroll
    for (int w = 0; w < kRowWaves; ++w) all += wave_top[w * kHeadTiles * 16 + h * 16 + l16];
    const float base = reference[h * 16 + l16];
    const int col = wave * kCols + quad * 4;
    if (p.splits > 1) {
      const int64_t part = (token * p.splits + split) * p.heads + head;
      if (wave == 0 && quad == 0) p.part_ml[part] = f32x2{base, all};
      if (all != 0.f) {
#pragma unroll
        for (int c = 0; c < kColTiles; ++c)
          *reinterpret_cast<f32x4*>(p.part_out + part * kLatent + col + c * 16) = out[c][h];
      }
      continue;
    }
    const float by = all == 0.f ? 0.f : 1.f / all;
    __bf16* to = p.out + token * p.out_token_stride + head * p.out_head_stride + col;
#pragma unroll
    for (int c = 0; c < kColTiles; ++c) {
      const f32x4 o = out[c][h] * by;
      *reinterpret_cast<bf16x4*>(to + c * 16) =
          bf16x4{static_cast<__bf16>(o[0]), static_cast<__bf16>(o[1]), static_cast<__bf16>(o[2]), static_cast<__bf16>(o[3])};
    }
    if (p.lse && wave == 0 && quad == 0)
      p.lse[token * p.heads + head] =
          all == 0.f ? -INFINITY : ((base == -INFINITY ? 0.f : base) + __builtin_amdgcn_logf(all)) * 0.6931471805599453f;
  }
}

// Joins the parts of one (query token, head): four columns per thread.  Parts
// without a row that counts hold no sums.
__global__ __launch_bounds__(kLatent / 4) void combine_kernel(AttendParams p) {
  const int64_t token = blockIdx.x / p.heads;
  const int head = static_cast<int>(blockIdx.x - token * p.heads), col = threadIdx.x * 4;
  const int64_t first = token * p.splits * p.heads + head;
  float top = -INFINITY;
  for (int i = 0; i < p.splits; ++i) {
    const f32x2 ml = p.part_ml[first + static_cast<int64_t>(i) * p.heads];
    if (ml[1] != 0.f) top = fmaxf(top, ml[0]);
  }
  const float base = top == -INFINITY ? 0.f : top;
  float all = 0.f;
  f32x4 o{};
  for (int i = 0; i < p.splits; ++i) {
    const int64_t part = first + static_cast<int64_t>(i) * p.heads;
    const f32x2 ml = p.part_ml[part];
    if (ml[1] == 0.f) continue;
    const float w = __builtin_amdgcn_exp2f(ml[0] - base);
    all += w * ml[1];
    o += *reinterpret_cast<const f32x4*>(p.part_out + part * kLatent + col) * w;
  }
  o *= all == 0.f ? 0.f : 1.f / all;
  *reinterpret_cast<bf16x4*>(p.out + token * p.out_token_stride + head * p.out_head_stride + col) =
      bf16x4{static_cast<__bf16>(o[0]), static_cast<__bf16>(o[1]), static_cast<__bf16>(o[2]), static_cast<__bf16>(o[3])};
  if (p.lse && threadIdx.x == 0)
    p.lse[token * p.heads + head] = all == 0.f ? -INFINITY : (base + __builtin_amdgcn_logf(all)) * 0.6931471805599453f;
}

// Head tiles of a workgroup: the fewest that hold the heads, at most four.
int head_tiles(int heads) { return heads <= 16 ? 1 : heads <= 32 ? 2 : 4; }

template <int kHeadTiles, int kKeyGroups, bool kMx4>
hipError_t launch_one(const AttendParams& p, hipStream_t s) {
  constexpr size_t lds = kKeyGroups * kValueBytes + kHeadTiles * 2048 + (kRowWaves + 1) * kHeadTiles * 16 * 4 + 16 +
                         (kKeyGroups == 2 ? kRowWaves * kHeadTiles * 1024 : 0);
  static_assert(lds <= 160 * 1024, "LDS of a workgroup");
  const auto kernel = &attend_kernel<kHeadTiles, kKeyGroups, kMx4>;
  static const hipError_t ready =
      hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(lds));
  if (ready != hipSuccess) return ready;
  const int head_blocks = (p.heads + kHeadTiles * 16 - 1) / (kHeadTiles * 16);
  const int tiles = (p.topk + kRowTile - 1) / kRowTile;
  const int64_t groups = static_cast<int64_t>(p.cache.batch) * p.n_q * head_blocks * p.splits;
  if (groups > INT32_MAX) return hipErrorInvalidValue;
  kernel<<<dim3(static_cast<unsigned>(groups)), 256 * kKeyGroups, lds, s>>>(p, head_blocks, (tiles + p.splits - 1) / p.splits);
  return hipGetLastError();
}

template <bool kMx4>
hipError_t launch_format(const AttendParams& p, hipStream_t s) {
  switch (head_tiles(p.heads)) {
    case 1: return launch_one<1, 1, kMx4>(p, s);
    case 2: return launch_one<2, 2, kMx4>(p, s);
    default: return launch_one<4, 2, kMx4>(p, s);
  }
}

}  // namespace

// Splits so that every CU has work (two workgroups of up to 32 heads, one of
// 64), but no part smaller than a tile.
int attend_splits(int batch, int n_q, int heads, int topk) {
  constexpr int64_t kCus = 256;
  const int per = head_tiles(heads);
  const int64_t groups = static_cast<int64_t>(batch) * n_q * ((heads + per * 16 - 1) / (per * 16));
  const int64_t want = (per == 4 ? kCus : 2 * kCus) / groups;
  const int tiles = (topk + kRowTile - 1) / kRowTile;
  if (want <= 1 || tiles <= 1) return 1;
  const int64_t each = (tiles + want - 1) / want;
  return static_cast<int>((tiles + each - 1) / each);
}

hipError_t launch_attend(const AttendParams& p, int format, hipStream_t s) {
  hipError_t e = format == 1 ? launch_format<true>(p, s) : launch_format<false>(p, s);
  if (e != hipSuccess || p.splits <= 1) return e;
  combine_kernel<<<dim3(static_cast<unsigned>(p.cache.batch * p.n_q * p.heads)), kLatent / 4, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace avsg
