// Product of two mx4 matrices, out = a b^T, with the matrix instruction that
// takes 4-bit operands and their scales:
//   16 x 128 by 128 x 16; lane l holds row l % 16 of either operand, columns
//   (l / 16) * 32 .. + 31 of the 128 (one block: 16 bytes of codes and their
//   scale), and of the result column l % 16, rows (l / 16) * 4 .. + 3.
// The 32 x 32 x 64 form of the instruction adds up less exactly: products of
// random codes with scales 2^-7 to 2^6 were off by 1.5e-5 of the result where this
// form is off by 2.6e-7.
#include <type_traits>

#include <algorithm>
#include <utility>

#include "latent_internal.h"

namespace avsg {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ i32x8 operand(u32x4 x) {
  return i32x8{static_cast<int>(x[0]), static_cast<int>(x[1]), static_cast<int>(x[2]), static_cast<int>(x[3]), 0, 0, 0, 0};
}

// The next `kCount` instructions of a kind, in the order in which the compiler is to issue a block.
constexpr int kMatrix = 0x8, kLdsRead = 0x100;
template <int kKind, int kCount>
__device__ __forceinline__ void schedule() {
  __builtin_amdgcn_sched_group_barrier(kKind, kCount, 0);
}

// f(0), f(1), ..., each with its number as a constant.
template <class F, int... kI>
__device__ __forceinline__ void each(std::integer_sequence<int, kI...>, F f) {
  (f(std::integral_constant<int, kI>{}), ...);
}
template <int kCount, class F>
__device__ __forceinline__ void each(F f) {
  each(std::make_integer_sequence<int, kCount>{}, f);
}

template <int kByteA, int kByteB>
__device__ __forceinline__ f32x4 multiply(u32x4 a, u32x4 b, f32x4 sum, uint32_t scales_a, uint32_t scales_b) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(a), operand(b), sum, 4, 4, kByteA, static_cast<int>(scales_a),
                                                         kByteB, static_cast<int>(scales_b));
}

// The product's operands change places, so that a lane holds four neighbouring
// columns of one row of the result: out[m][n .. n + 3], m = m0 + l % 16.
template <bool kF32>
__device__ __forceinline__ void store4(const Mx4Product& p, int64_t batch, int m, int n, f32x4 x) {
  if (m >= p.m) return;
  const int64_t at = batch * p.out_batch_stride + static_cast<int64_t>(m) * p.out_stride + n;
  if constexpr (kF32) {
    float* to = static_cast<float*>(p.out) + at;
    if (p.wide_stores && n + 3 < p.n) {
      *reinterpret_cast<f32x4*>(to) = x;
      return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (n + j < p.n) to[j] = x[j];
  } else {
    __bf16* to = static_cast<__bf16*>(p.out) + at;
    if (p.wide_stores && n + 3 < p.n) {
      *reinterpret_cast<bf16x4*>(to) =
          bf16x4{static_cast<__bf16>(x[0]), static_cast<__bf16>(x[1]), static_cast<__bf16>(x[2]), static_cast<__bf16>(x[3])};
      return;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (n + j < p.n) to[j] = static_cast<__bf16>(x[j]);
  }
}

// Eight neighbouring columns of a row in 16 bits.
__device__ __forceinline__ void store8(const Mx4Product& p, int64_t batch, int m, int n, f32x4 x, f32x4 y) {
  if (p.wide_stores && n + 7 < p.n) {
    if (m >= p.m) return;
    typedef __bf16 bf16x8_at_8 __attribute__((ext_vector_type(8), aligned(8)));
    *reinterpret_cast<bf16x8_at_8*>(static_cast<__bf16*>(p.out) + batch * p.out_batch_stride + static_cast<int64_t>(m) * p.out_stride + n) =
        bf16x8_at_8{static_cast<__bf16>(x[0]), static_cast<__bf16>(x[1]), static_cast<__bf16>(x[2]), static_cast<__bf16>(x[3]),
                    static_cast<__bf16>(y[0]), static_cast<__bf16>(y[1]), static_cast<__bf16>(y[2]), static_cast<__bf16>(y[3])};
  } else {
    store4<false>(p, batch, m, n, x);
    store4<false>(p, batch, m, n + 4, y);
  }
}

// Column of the result, and row of b, that is row l16 of tile y of the products'
// second operand.  Results of 16 bits take them such that a lane has eight
// neighbouring columns in two tiles, and four lanes 64 bytes.
template <bool kF32>
__device__ __forceinline__ constexpr int column_of(int y, int l16) {
  return kF32 ? y * 16 + l16 : y / 2 * 32 + l16 / 4 * 8 + y % 2 * 4 + l16 % 4;
}

template <bool kF32, int kM, int kN>
__device__ __forceinline__ void store_tiles(const Mx4Product& p, int64_t batch, int m, int n, int quad, f32x4 (&sum)[kM][kN]) {
  each<kM>([&](auto x) {
    if constexpr (kF32) {
      each<kN>([&](auto y) { store4<kF32>(p, batch, m + x * 16, n + y * 16 + quad * 4, sum[x][y]); });
    } else {
      each<kN / 2>([&](auto y) { store8(p, batch, m + x * 16, n + y * 32 + quad * 8, sum[x][2 * y], sum[x][2 * y + 1]); });
    }
  });
}

// Few rows of a (up to 16 * kRowTiles): what counts is how fast b streams by.  A
// workgroup takes 16 rows of b; its waves share the columns (wave w takes every
// kWaves-th step of 128), several steps' loads in flight, and add up in LDS.
template <int kRowTiles, int kWaves, bool kF32>
__global__ __launch_bounds__(kWaves * 64) void thin_kernel(Mx4Product p) {
  constexpr int kAhead = 4;
  __shared__ f32x4 sums[kWaves - 1][kRowTiles][64];
  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = blockIdx.x * 16 + l16, m0 = blockIdx.y * kRowTiles * 16;
  const int64_t i = blockIdx.z;
  const int blocks = p.k / kMx4Block;
  const bool in_b = n < p.n;
  const uint8_t* bc = p.b.codes + i * p.b.code_batch_stride + static_cast<int64_t>(in_b ? n : 0) * p.b.code_stride;
  const uint8_t* bs = p.b.scales + i * p.b.scale_batch_stride + static_cast<int64_t>(in_b ? n : 0) * p.b.scale_stride;
  const uint8_t *ac[kRowTiles], *as[kRowTiles];
#pragma unroll
  for (int r = 0; r < kRowTiles; ++r) {
    const int m = min(m0 + r * 16 + l16, p.m - 1);   // rows past the end are not stored
    ac[r] = p.a.codes + i * p.a.code_batch_stride + static_cast<int64_t>(m) * p.a.code_stride;
    as[r] = p.a.scales + i * p.a.scale_batch_stride + static_cast<int64_t>(m) * p.a.scale_stride;
  }
  f32x4 sum[kRowTiles] = {};
  const int steps = (blocks + 3) / 4;
  for (int s0 = wave; s0 < steps; s0 += kWaves * kAhead) {
    u32x4 a[kAhead][kRowTiles], b[kAhead];
    uint32_t sa[kAhead][kRowTiles], sb[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int k = (s0 + u * kWaves) * 4 + quad;
      const bool there = k < blocks;   // columns past the end are zeros
      const int at = there ? k : 0;
      b[u] = *reinterpret_cast<const u32x4*>(bc + 16 * static_cast<int64_t>(at));
      sb[u] = bs[at];
      if (!there) b[u] = u32x4{}, sb[u] = 127;
#pragma unroll
      for (int r = 0; r < kRowTiles; ++r) {
        a[u][r] = *reinterpret_cast<const u32x4*>(ac[r] + 16 * static_cast<int64_t>(at));
        sa[u][r] = as[r][at];
        if (!there) a[u][r] = u32x4{}, sa[u][r] = 127;
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u)
#pragma unroll
      for (int r = 0; r < kRowTiles; ++r) sum[r] = multiply<0, 0>(b[u], a[u][r], sum[r], sb[u], sa[u][r]);
  }
  if (wave > 0) {
#pragma unroll
    for (int r = 0; r < kRowTiles; ++r) sums[wave - 1][r][lane] = sum[r];
  }
  __syncthreads();
  if (wave > 0) return;
#pragma unroll
  for (int r = 0; r < kRowTiles; ++r) {
#pragma unroll
    for (int w = 0; w < kWaves - 1; ++w) sum[r] += sums[w][r][lane];
    store4<kF32>(p, i, m0 + r * 16 + l16, blockIdx.x * 16 + quad * 4, sum[r]);
  }
}

// Tiles of kTileM x kTileN outputs, kWavesM x kWavesN waves.  Operands come
// straight from global memory: a lane's 16 bytes are one row's block, so there is
// nothing to rearrange, and the waves that share rows find them in L1.  Steps of 128
// columns, loads and then products; nothing is fetched ahead, for with fewer than 256 columns
// there are one or two steps.  128 products of 128 x 512 x 128 take 9.8 us (22 MB, 17 of them
// results).
template <int kTileM, int kTileN, int kWavesM, int kWavesN, bool kF32>
__global__ __launch_bounds__(kWavesM * kWavesN * 64) void tile_kernel(Mx4Product p, int tiles_m, int tiles_n) {
  constexpr int kM = kTileM / kWavesM / 16, kN = kTileN / kWavesN / 16;
  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // tiles of eight rows of tiles follow each other down the columns, on one XCD,
  // so that its L2 holds the operands they share
  const unsigned total = gridDim.x, per = total / kXcds, more = total % kXcds, xcd = blockIdx.x % kXcds;
  const unsigned id = xcd * per + min(xcd, more) + blockIdx.x / kXcds;
  constexpr int kGroup = 8;
  const int in_group = kGroup * tiles_n, group = id / in_group, rows_here = min(kGroup, tiles_m - group * kGroup);
  const int tm = group * kGroup + (id - group * in_group) % rows_here, tn = (id - group * in_group) / rows_here;
  const int64_t i = blockIdx.y;
  const int blocks = p.k / kMx4Block;
  const int m0 = tm * kTileM + wave / kWavesN * (kM * 16), n0 = tn * kTileN + wave % kWavesN * (kN * 16);
  const uint8_t* ac = p.a.codes + i * p.a.code_batch_stride;
  const uint8_t* as = p.a.scales + i * p.a.scale_batch_stride;
  const uint8_t* bc = p.b.codes + i * p.b.code_batch_stride;
  const uint8_t* bs = p.b.scales + i * p.b.scale_batch_stride;
  int64_t ca[kM], cb[kN], xa[kM], xb[kN];
#pragma unroll
  for (int r = 0; r < kM; ++r) {
    const int64_t m = min(m0 + r * 16 + l16, p.m - 1);   // rows past the end are not stored
    ca[r] = m * p.a.code_stride, xa[r] = m * p.a.scale_stride;
  }
#pragma unroll
  for (int r = 0; r < kN; ++r) {
    const int64_t n = min(n0 + column_of<kF32>(r, l16), p.n - 1);
    cb[r] = n * p.b.code_stride, xb[r] = n * p.b.scale_stride;
  }
  f32x4 sum[kM][kN] = {};
  for (int k = quad; k - quad < blocks; k += 4) {
    const bool there = k < blocks;   // columns past the end are zeros
    const int at = there ? k : 0;
    u32x4 a[kM], b[kN];
    uint32_t sa[kM], sb[kN];
#pragma unroll
    for (int r = 0; r < kM; ++r) {
      a[r] = *reinterpret_cast<const u32x4*>(ac + ca[r] + 16 * at), sa[r] = as[xa[r] + at];
      if (!there) a[r] = u32x4{}, sa[r] = 127;
    }
#pragma unroll
    for (int r = 0; r < kN; ++r) {
      b[r] = *reinterpret_cast<const u32x4*>(bc + cb[r] + 16 * at), sb[r] = bs[xb[r] + at];
      if (!there) b[r] = u32x4{}, sb[r] = 127;
    }
#pragma unroll
    for (int x = 0; x < kM; ++x)
#pragma unroll
      for (int y = 0; y < kN; ++y) sum[x][y] = multiply<0, 0>(b[y], a[x], sum[x][y], sb[y], sa[x]);
  }
  store_tiles<kF32>(p, i, m0 + l16, n0, quad, sum);
}

// What columns past the end read in place of codes.
__device__ __align__(16) const unsigned char zero_block[16] = {};

// Bits of a row by which the staged blocks of 16 bytes are exchanged: the eight pairs
// of the sixteen rows that are read together differ in them.
__device__ __forceinline__ int exchange(int row, bool by_eights) {
  return by_eights ? (row >> 1 & 1) | (row >> 2 & 6) : row >> 1 & 7;
}

// Larger products: tiles of kTileM x kTileN outputs, kWavesM x kWavesN waves.
// Steps of 256 columns go from global memory to LDS without passing registers, the
// next step's while this one's products run: 64 matrix instructions per wave and step
// at 256 x 256.  In LDS a row has its 128 bytes of the step, its eight blocks exchanged by
// three bits of the row, so that the sixteen lanes that read one block of sixteen
// rows meet every bank; eight neighbouring lanes fetch a row's whole line.  kGroups groups
// of such waves share the columns, a run of steps each, and add up in LDS.
// 8192 x 4096 x 4096 takes 83 to 100 us, 2.7 to 3.3 PFLOP/s.  Its loop takes 4200 cycles
// per step where the products take 2048, and 2500 without the loads.  Each step waits for
// memory twice: after its first product or two, because the next step's scales are shifted where
// they are loaded, which waits for all loads in flight and so keeps most of the step's loads from
// starting before; and at its end, for the next step's codes.
template <int kTileM, int kTileN, int kWavesM, int kWavesN, int kGroups, bool kF32>
__global__ __launch_bounds__(kGroups * kWavesM * kWavesN * 64, kGroups * kWavesM * kWavesN / 4) void staged_kernel(Mx4Product p, int tiles_m, int tiles_n) {
  constexpr int kWaves = kWavesM * kWavesN, kThreads = kWaves * 64;
  constexpr int kM = kTileM / kWavesM / 16, kN = kTileN / kWavesN / 16;
  constexpr int kRows = kTileM + kTileN;                 // rows of a, then rows of b
  constexpr int kLoads = kRows / 8 / kWaves;             // eight rows each
  static_assert(kRows % (8 * kWaves) == 0 && kRows <= kThreads, "shares of the loads: a thread brings the scales of one row");
  constexpr int kStage = kRows * 136;                    // codes, then eight scales per row
  extern __shared__ __align__(16) unsigned char all_lds[];   // [kGroups][2][kStage], then the groups' sums
  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int group = kGroups > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads) : 0;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) - group * kWaves;
  unsigned char* const lds = all_lds + group * 2 * kStage;
  // tiles of eight rows of tiles follow each other down the columns, on one XCD,
  // so that its L2 holds the operands they share
  const unsigned total = gridDim.x, per = total / kXcds, more = total % kXcds, xcd = blockIdx.x % kXcds;
  const unsigned id = xcd * per + min(xcd, more) + blockIdx.x / kXcds;
  constexpr int kGroup = 8;
  const int in_band = kGroup * tiles_n, band = id / in_band, rows_here = min(kGroup, tiles_m - band * kGroup);
  const int tm = band * kGroup + (id - band * in_band) % rows_here, tn = (id - band * in_band) / rows_here;
  const int64_t i = blockIdx.y;
  const int blocks = p.k / kMx4Block, steps = (blocks + 7) / 8;

  // Row `r` of the tile's rows of a and b, as an offset from the first of them;
  // rows past the end are not stored, and read as the last.
  const uint8_t* const codes_a = p.a.codes + i * p.a.code_batch_stride + static_cast<int64_t>(tm) * kTileM * p.a.code_stride;
  const uint8_t* const codes_b = p.b.codes + i * p.b.code_batch_stride + static_cast<int64_t>(tn) * kTileN * p.b.code_stride;
  const int last_a = p.m - 1 - tm * kTileM, last_b = p.n - 1 - tn * kTileN;
  // eight rows are of one matrix
  auto from_a = [&](int j) { return (j * kWaves + wave) * 8 < kTileM; };
  uint32_t row_at[kLoads];
  static_assert(kWaves % 4 == 0, "all loads exchange blocks alike");
  const int block_a = (lane & 7) ^ exchange(wave * 8 + lane / 8, false), block_b = (lane & 7) ^ exchange(wave * 8 + lane / 8, !kF32);
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int r = (j * kWaves + wave) * 8 + lane / 8;
    row_at[j] = from_a(j) ? min(r, last_a) * static_cast<uint32_t>(p.a.code_stride)
                          : min(r - kTileM, last_b) * static_cast<uint32_t>(p.b.code_stride);
  }
  // The scales of a row: in LDS lane l of a wave's products finds its bytes, a
  // tile of 16 rows after the other, first and second half of the step, in one place.
  const int row = threadIdx.x % kRows, of_b = row - kTileM;
  const bool is_a = of_b < 0;
  const Mx4View& x = is_a ? p.a : p.b;
  const uint8_t* const scale_row = x.scales + i * x.scale_batch_stride +
                                   (is_a ? tm * kTileM + min(row, last_a) : tn * kTileN + min(of_b, last_b)) * x.scale_stride;
  const int share = is_a ? kM : kN, in_wave = (is_a ? row : of_b) % (share * 16);
  const int tile16 = is_a || kF32 ? in_wave / 16 : in_wave / 32 * 2 + (in_wave / 4 & 1);
  const int lane16 = is_a || kF32 ? in_wave % 16 : (in_wave / 8 & 3) * 4 + (in_wave & 3);
  const unsigned scales_at = kRows * 128 + (row - in_wave) * 8 + lane16 * (share * 2) + tile16 * 2;

  uint32_t scales[2];
  auto fetch = [&](int j, int step, int buffer) {
    // (the compiler would keep eight advancing 64-bit addresses)
    uint32_t row = row_at[j];
    asm volatile("" : "+v"(row));
    const int block = step * 8 + (from_a(j) ? block_a : block_b);
    const uint8_t* from = (from_a(j) ? codes_a : codes_b) + row + 16 * static_cast<uint32_t>(block);
    if (block >= blocks) from = zero_block;
    __builtin_amdgcn_global_load_lds(
        reinterpret_cast<const __attribute__((address_space(1))) void*>(reinterpret_cast<uint64_t>(from)),
        (__attribute__((address_space(3))) void*)(lds + buffer * kStage + (j * kWaves + wave) * 1024), 16, 0, 0);
  };
  // eight scales, of the last step the row's last eight moved down: where they
  // are zeros in place of scales, so are the codes
  auto fetch_scales = [&](int step) {
    const int within = min(step, steps - 1) * 8, first = min(within, blocks - 8), off = (within - first) * 8;
    uint64_t eight;
    __builtin_memcpy(&eight, scale_row + first, 8);
    eight >>= off;
    scales[0] = static_cast<uint32_t>(eight), scales[1] = static_cast<uint32_t>(eight >> 32);
  };
  auto leave_scales = [&](int buffer) {
    const uint32_t two[2] = {__builtin_amdgcn_perm(scales[1], scales[0], 0x05010400), __builtin_amdgcn_perm(scales[1], scales[0], 0x07030602)};
    if (kRows < kThreads && wave * 64 >= kRows) return;
    unsigned char* const to = lds + buffer * kStage + scales_at;
#pragma unroll
    for (int q = 0; q < 4; ++q) *reinterpret_cast<uint16_t*>(to + q * 16 * (share * 2)) = static_cast<uint16_t>(two[q / 2] >> (q % 2 * 16));
  };

  f32x4 sum[kM][kN] = {};
  const int wave_a = wave / kWavesN * (kM * 16), wave_b = wave % kWavesN * (kN * 16);
  const unsigned at_a = (wave_a + l16) * 128 + (quad ^ exchange(l16, false)) * 16;
  const int row_b = column_of<kF32>(0, l16);
  const unsigned at_b = (kTileM + wave_b + row_b) * 128 + (quad ^ exchange(row_b, !kF32)) * 16;
  auto from_row_b = [&](int y) { return (column_of<kF32>(y, l16) - row_b) * 128; };
  // a group's steps follow each other; what it takes past the last step are zeros
  const int first_step = group * ((steps + kGroups - 1) / kGroups), steps_here = (steps + kGroups - 1) / kGroups;
#pragma unroll
  for (int j = 0; j < kLoads; ++j) fetch(j, first_step, 0);
  fetch_scales(first_step);
  leave_scales(0);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  for (int step = 0; step < steps_here; ++step) {
    const int buffer = step & 1;
    // (after the last step too: without a branch the products stay where they are)
    const int next = first_step + step + 1;
    const unsigned char* const from = lds + buffer * kStage;
    uint32_t sa[kM / 2], sb[kN / 2];
    __builtin_memcpy(sa, __builtin_assume_aligned(from + kRows * 128 + wave_a * 8 + lane * (kM * 2), kM * 2), kM * 2);
    __builtin_memcpy(sb, __builtin_assume_aligned(from + kRows * 128 + (kTileM + wave_b) * 8 + lane * (kN * 2), kN * 2), kN * 2);
    // Both halves' operands are in registers of their own: the second half's are
    // read while the first half's products run, a tile of a at a time.
    u32x4 a[2][kM], b[2][kN];
    auto read_a = [&](int half, int x) { a[half][x] = *reinterpret_cast<const u32x4*>(from + x * 2048 + (at_a ^ (half * 64))); };
    auto read_b = [&](int half, int y) { b[half][y] = *reinterpret_cast<const u32x4*>(from + from_row_b(y) + (at_b ^ (half * 64))); };
#pragma unroll
    for (int y = 0; y < kN; ++y) read_b(0, y);
#pragma unroll
    for (int x = 0; x < kM; ++x) read_a(0, x);
    __builtin_amdgcn_sched_barrier(0);
    fetch_scales(next);
    each<2>([&](auto half) {
      each<kM>([&](auto x) {
        each<kN>([&](auto y) {
          sum[x][y] = multiply<y % 2 * 2 + half, x % 2 * 2 + half>(b[half][y], a[half][x], sum[x][y], sb[y / 2], sa[x / 2]);
        });
        if constexpr (half == 0) {
          if constexpr (x < kN) read_b(1, x);
          read_a(1, x);
          // spread over the half: all of them ahead of the products took 6% longer
          each<kLoads / kM>([&](auto j) { fetch(x * (kLoads / kM) + j, next, buffer ^ 1); });
        }
        __builtin_amdgcn_sched_barrier(0);
      });
    });
    leave_scales(buffer ^ 1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }
  if constexpr (kGroups > 1) {
    f32x4* const sums = reinterpret_cast<f32x4*>(all_lds);
    each<kM>([&](auto x) {
      each<kN>([&](auto y) {
        if (group > 0) sums[((group - 1) * kM * kN + x * kN + y) * kThreads + wave * 64 + lane] = sum[x][y];
      });
    });
    __syncthreads();
    if (group > 0) return;
    each<kM>([&](auto x) {
      each<kN>([&](auto y) {
        each<kGroups - 1>([&](auto g) { sum[x][y] += sums[(g * kM * kN + x * kN + y) * kThreads + wave * 64 + lane]; });
      });
    });
  }
  const int m0 = tm * kTileM + wave_a, n0 = tn * kTileN + wave_b;
  store_tiles<kF32>(p, i, m0 + l16, n0, quad, sum);
}

template <int kTile, int kWavesM, int kWavesN, int kGroups, bool kF32>
hipError_t launch_staged(const Mx4Product& p, int64_t tiles_m, int64_t tiles_n, hipStream_t s) {
  constexpr int kLds = kGroups * 2 * 2 * kTile * 136;
  static_assert(kLds <= 160 * 1024, "LDS of a workgroup");
  constexpr auto kernel = &staged_kernel<kTile, kTile, kWavesM, kWavesN, kGroups, kF32>;
  if (const hipError_t e = allow_lds<kernel>(kLds); e != hipSuccess) return e;
  kernel<<<dim3(static_cast<unsigned>(tiles_m * tiles_n), p.batch), kGroups * kWavesM * kWavesN * 64, kLds, s>>>(
      p, static_cast<int>(tiles_m), static_cast<int>(tiles_n));
  return hipGetLastError();
}

// Which kernel, by what each took (us, bfloat16 results, one call after the other in
// a graph).  With 256 columns or more, which is a step of the staged kernels:
//   rows x columns of out, k   thin   64, 2 groups   128, 2 groups    128    256
//       1 x  4096, 4096         4.3       7.9            12.9        18.7
//       1 x 32768, 4096        19.0      13.5            19.3        25.2
//      32 x  4096, 4096         7.6       8.7            13.1        19.1
//      64 x  4096, 4096        11.4       9.0            13.5        19.8
//     512 x  4096, 4096                  13.5            15.0        20.9
//    1024 x  4096, 4096                  24.9            17.3        22.6   34.0
//    1536 x  4096, 4096                  37.3            32.7        29.6   38.3
//    2304 x  4096, 4096                  55.6            50.8        51.6   39.0
//    8192 x  4096, 4096                                             112.9   83.2
//    2500 x  4096,  512                  19.8            16.3        12.8   12.1
// Two groups halve the steps that wait for memory one after the other, while a
// tile for each CU, or two, is all there is; large tiles read less per product.
// With fewer columns (heads x rows x columns, k):
//                              thin  straight from memory
//     16 x  32 x 512, 128       3.0       3.7
//      8 x 128 x 512, 224       4.2       5.2
//     64 x   8 x 512, 128       3.9       3.7
//    128 x 128 x 512, 128      25.5       7.2
template <bool kF32>
hipError_t launch(const Mx4Product& p, hipStream_t s) {
  auto tiles = [](int64_t rows, int64_t by) { return (rows + by - 1) / by; };
  const int64_t tiles_m = tiles(p.m, 128), tiles_n = tiles(p.n, 128), wide_m = tiles(p.m, 256), wide_n = tiles(p.n, 256);
  const int64_t small_m = tiles(p.m, 64), small_n = tiles(p.n, 64);
  // offsets within a tile's rows are held in 32 bits
  const int64_t longest = std::max(p.a.code_stride, p.b.code_stride);
  const bool staged = p.k >= 256 && p.a.code_stride >= 0 && p.b.code_stride >= 0 && longest * 256 + p.k < (int64_t{1} << 31);
  const int rows = p.m <= 16 ? 16 : p.m <= 32 ? 32 : 64;
  const int64_t pieces = tiles(p.n, 16) * tiles(p.m, rows) * (rows / 16) * p.batch;
  if (staged ? p.m <= 32 && pieces <= 512 : pieces <= 2048) {
    const dim3 grid(tiles(p.n, 16), tiles(p.m, rows), p.batch);
    if (rows == 16) thin_kernel<1, 8, kF32><<<grid, 512, 0, s>>>(p);
    else if (rows == 32) thin_kernel<2, 4, kF32><<<grid, 256, 0, s>>>(p);
    else thin_kernel<4, 4, kF32><<<grid, 256, 0, s>>>(p);
    return hipGetLastError();
  }
  if (staged) {
    const int64_t all = tiles_m * tiles_n * p.batch;
    if (small_m * small_n * p.batch <= 512) return launch_staged<64, 2, 2, 2, kF32>(p, small_m, small_n, s);
    if (all <= 256) return launch_staged<128, 2, 2, 2, kF32>(p, tiles_m, tiles_n, s);
    // (large tiles that few rows or columns leave half empty are no gain)
    if (all > 512 && wide_m * wide_n * p.batch * 4 <= all + all / 4) return launch_staged<256, 2, 4, 1, kF32>(p, wide_m, wide_n, s);
    return launch_staged<128, 2, 2, 1, kF32>(p, tiles_m, tiles_n, s);
  }
  tile_kernel<128, 128, 2, 2, kF32><<<dim3(static_cast<unsigned>(tiles_m * tiles_n), p.batch), 256, 0, s>>>(
      p, static_cast<int>(tiles_m), static_cast<int>(tiles_n));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_matmul(const Mx4Product& p, hipStream_t s) { return p.f32 ? launch<true>(p, s) : launch<false>(p, s); }

}  // namespace avsg
