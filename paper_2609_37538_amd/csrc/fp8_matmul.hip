// Product of two matrices in 8-bit floating point with a scale per 128 columns, out = a b^T.  The matrix
// instruction takes 128 columns at once:
//   16 x 128 by 128 x 16; lane l holds row l % 16 of either operand, columns (l / 16) * 32 .. + 31 (32
//   bytes), and of the result column l % 16, rows (l / 16) * 4 .. + 3.
// So a product of one block of columns is one instruction, whose result is added up times both
// scales.  The operands change places, so that a lane holds four neighbouring columns of one row of
// out, and with them one scale of a; b's is the same for 128 columns of out.
#include <algorithm>
#include <type_traits>
#include <utility>

#include "fp8_internal.h"

namespace avsg {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ f32x4 multiply(u32x4 b0, u32x4 b1, u32x4 a0, u32x4 a1) {
  const i32x8 b{static_cast<int>(b0[0]), static_cast<int>(b0[1]), static_cast<int>(b0[2]), static_cast<int>(b0[3]),
                static_cast<int>(b1[0]), static_cast<int>(b1[1]), static_cast<int>(b1[2]), static_cast<int>(b1[3])};
  const i32x8 a{static_cast<int>(a0[0]), static_cast<int>(a0[1]), static_cast<int>(a0[2]), static_cast<int>(a0[3]),
                static_cast<int>(a1[0]), static_cast<int>(a1[1]), static_cast<int>(a1[2]), static_cast<int>(a1[3])};
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a, f32x4{}, 0, 0, 0, 0, 0, 0);
}

// out[m][n .. n + 3]
template <bool kF32>
__device__ __forceinline__ void store4(const Fp8Product& p, int64_t batch, int m, int n, f32x4 x) {
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

// Few rows of a (up to 16 * kRowTiles a workgroup): what counts is how fast b streams by.  A workgroup takes
// 16 rows of b; its waves share the columns (wave w takes every kWaves-th block of 128), several
// blocks' loads in flight, and add up in LDS.  Any strides.
template <int kRowTiles, int kWaves, bool kF32>
__global__ __launch_bounds__(kWaves * 64) void thin_kernel(Fp8Product p) {
  constexpr int kAhead = 4;
  __shared__ f32x4 sums[kWaves - 1][kRowTiles][64];
  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n0 = blockIdx.x * 16, m0 = blockIdx.y * kRowTiles * 16;
  const int64_t i = blockIdx.z;
  const uint8_t* const bc = p.b.codes + i * p.b.code_batch_stride + static_cast<int64_t>(min(n0 + l16, p.n - 1)) * p.b.code_stride;
  const float* const bs = p.b.scales + i * p.b.scale_batch_stride + n0 / kFp8Block * p.b.scale_stride;
  const uint8_t* ac[kRowTiles];
  const float* as[kRowTiles];
#pragma unroll
  for (int r = 0; r < kRowTiles; ++r) {
    const int64_t m = min(m0 + r * 16 + l16, p.m - 1);   // rows past the end are not stored
    ac[r] = p.a.codes + i * p.a.code_batch_stride + m * p.a.code_stride;
    as[r] = p.a.scales + i * p.a.scale_batch_stride + m * p.a.scale_stride;
  }
  f32x4 sum[kRowTiles] = {};
  const int steps = (p.k + kFp8Block - 1) / kFp8Block;
  for (int s0 = wave; s0 < steps; s0 += kWaves * kAhead) {
    u32x4 a[kAhead][kRowTiles][2], b[kAhead][2];
    float sa[kAhead][kRowTiles], sb[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int step = s0 + u * kWaves, block = min(step, steps - 1);
      sb[u] = bs[block];
#pragma unroll
      for (int r = 0; r < kRowTiles; ++r) sa[u][r] = as[r][block];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int k = step * kFp8Block + quad * 32 + h * 16;
        const bool there = step < steps && k < p.k;   // columns past the end are zeros
        const int at = there ? k : 0;
        b[u][h] = *reinterpret_cast<const u32x4*>(bc + at);
        if (!there) b[u][h] = u32x4{};
#pragma unroll
        for (int r = 0; r < kRowTiles; ++r) {
          a[u][r][h] = *reinterpret_cast<const u32x4*>(ac[r] + at);
          if (!there) a[u][r][h] = u32x4{};
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (s0 + u * kWaves >= steps) break;
#pragma unroll
      for (int r = 0; r < kRowTiles; ++r) {
        const f32x4 x = multiply(b[u][0], b[u][1], a[u][r][0], a[u][r][1]);
        const float s = sa[u][r] * sb[u];
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[r][j] = __builtin_fmaf(x[j], s, sum[r][j]);
      }
    }
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
    store4<kF32>(p, i, m0 + r * 16 + l16, n0 + quad * 4, sum[r]);
  }
}

// What columns past the end read in place of codes.
__device__ __align__(16) const unsigned char zero_block[16] = {};

// Bits of a row by which its staged blocks of 16 bytes are exchanged: the eight pairs of the sixteen rows that are
// read together differ in them.
__device__ __forceinline__ int exchange(int row) { return row >> 1 & 7; }

// f(0), f(1), ..., each with its number as a constant.
template <class F, int... kI>
__device__ __forceinline__ void each(std::integer_sequence<int, kI...>, F f) {
  (f(std::integral_constant<int, kI>{}), ...);
}
template <int kCount, class F>
__device__ __forceinline__ void each(F f) {
  each(std::make_integer_sequence<int, kCount>{}, f);
}

// Larger products: tiles of kTile x kTile outputs, kWavesM x kWavesN waves.  Steps of 128 columns, a block, go from
// global memory to LDS without passing registers, the next step's while this one's products run.  In LDS a row
// has its 128 bytes of the step, its eight blocks of 16 exchanged by three bits of the row, so that the sixteen lanes that
// read one block of sixteen rows meet every bank; eight neighbouring lanes fetch a row's whole line.
// The rows' scales of the step follow, a's, then b's for each 128 rows.
// kGroups groups of such waves share the columns, a run of steps each, and add up in LDS.
// 8192 x 4096 x 4096 takes 127 us, 2.2 PFLOP/s, with 256 x 256: 4240 cycles per step, whose products take 2112; without
// the loads it takes 95, and without the sums' multiplications too 95: they hide behind the products, the loads'
// latency does not, with two buffers being all that LDS holds.  Lane l's 32 bytes are the blocks l / 16 and l / 16 + 4 of
// its row (the columns' order does not matter while both operands have the same): with two neighbouring ones
// 46% of LDS's cycles were bank conflicts, so there are none.
template <int kTile, int kWavesM, int kWavesN, int kGroups, bool kF32>
__global__ __launch_bounds__(kGroups * kWavesM * kWavesN * 64, kGroups * kWavesM * kWavesN / 4) void staged_kernel(Fp8Product p, int tiles_m, int tiles_n) {
  constexpr int kWaves = kWavesM * kWavesN, kThreads = kWaves * 64;
  constexpr int kM = kTile / kWavesM / 16, kN = kTile / kWavesN / 16;
  constexpr int kRows = 2 * kTile;                // rows of a, then rows of b
  constexpr int kLoads = kRows / 8 / kWaves;      // eight rows each
  constexpr int kScaleLoads = kTile / 64 + 1;     // 64 scales each: a's, and b's
  static_assert(kRows % (8 * kWaves) == 0 && kScaleLoads <= kWaves + 1);
  constexpr int kStage = kRows * 128 + kScaleLoads * 256;
  extern __shared__ __align__(16) unsigned char all_lds[];   // [kGroups][2][kStage], then the groups' sums
  const int lane = threadIdx.x & 63, l16 = lane & 15, quad = lane >> 4;
  const int group = kGroups > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / kThreads) : 0;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) - group * kWaves;
  unsigned char* const lds = all_lds + group * 2 * kStage;
  // tiles of eight rows of tiles follow each other down the columns, on one XCD, so that its L2 holds the operands
  // they share
  const unsigned total = gridDim.x, per = total / kXcds, more = total % kXcds, xcd = blockIdx.x % kXcds;
  const unsigned id = xcd * per + min(xcd, more) + blockIdx.x / kXcds;
  constexpr int kBand = 8;
  const int in_band = kBand * tiles_n, band = id / in_band, rows_here = min(kBand, tiles_m - band * kBand);
  const int tm = band * kBand + (id - band * in_band) % rows_here, tn = (id - band * in_band) / rows_here;
  const int64_t i = blockIdx.y;
  const int steps = (p.k + kFp8Block - 1) / kFp8Block;

  // Row `r` of the tile's rows of a and b, as an offset from the first of them; rows past the end are not stored, and read
  // as the last.
  const uint8_t* const codes_a = p.a.codes + i * p.a.code_batch_stride + static_cast<int64_t>(tm) * kTile * p.a.code_stride;
  const uint8_t* const codes_b = p.b.codes + i * p.b.code_batch_stride + static_cast<int64_t>(tn) * kTile * p.b.code_stride;
  const int last_a = p.m - 1 - tm * kTile, last_b = p.n - 1 - tn * kTile;
  auto from_a = [&](int j) { return (j * kWaves + wave) * 8 < kTile; };   // eight rows are of one matrix
  uint32_t row_at[kLoads];
  static_assert(kWaves % 2 == 0, "all loads exchange blocks alike");
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int r = (j * kWaves + wave) * 8 + lane / 8;
    row_at[j] = from_a(j) ? min(r, last_a) * static_cast<uint32_t>(p.a.code_stride)
                          : min(r - kTile, last_b) * static_cast<uint32_t>(p.b.code_stride);
  }
  const int my_block = (lane & 7) ^ exchange(wave * 8 + lane / 8);
  // a's scales by the first waves, b's by the one after them (or the first)
  constexpr int kWaveOfB = (kScaleLoads - 1) % kWaves;
  const float* const scales_a = p.a.scales + i * p.a.scale_batch_stride + (tm * kTile + min(wave * 64 + lane, last_a)) * p.a.scale_stride;
  const float* const scales_b =
      p.b.scales + i * p.b.scale_batch_stride + min(tn * kTile / kFp8Block + (lane & 1), (p.n - 1) / kFp8Block) * p.b.scale_stride;
  auto fetch = [&](int j, int step, unsigned char* to) {
    // (the compiler would keep advancing 64-bit addresses)
    uint32_t row = row_at[j];
    asm volatile("" : "+v"(row));
    const int at = step * kFp8Block + my_block * 16;
    const uint8_t* from = (from_a(j) ? codes_a : codes_b) + row + static_cast<uint32_t>(at);
    if (at >= p.k) from = zero_block;
    __builtin_amdgcn_global_load_lds(
        reinterpret_cast<const __attribute__((address_space(1))) void*>(reinterpret_cast<uint64_t>(from)),
        (__attribute__((address_space(3))) void*)(to + (j * kWaves + wave) * 1024), 16, 0, 0);
  };
  auto fetch_scales = [&](int step, unsigned char* to) {
    const int block = min(step, steps - 1);   // (past the end the codes are zeros)
    to += kRows * 128;
    if (wave < kTile / 64)
      __builtin_amdgcn_global_load_lds(
          reinterpret_cast<const __attribute__((address_space(1))) void*>(reinterpret_cast<uint64_t>(scales_a + block)),
          (__attribute__((address_space(3))) void*)(to + wave * 256), 4, 0, 0);
    if (wave == kWaveOfB)
      __builtin_amdgcn_global_load_lds(
          reinterpret_cast<const __attribute__((address_space(1))) void*>(reinterpret_cast<uint64_t>(scales_b + block)),
          (__attribute__((address_space(3))) void*)(to + kTile * 4), 4, 0, 0);
  };

  f32x4 sum[kM][kN] = {};
  const int wave_a = wave / kWavesN * (kM * 16), wave_b = wave % kWavesN * (kN * 16);
  const unsigned at_a = (wave_a + l16) * 128 + (quad ^ exchange(l16)) * 16;
  const unsigned at_b = (kTile + wave_b + l16) * 128 + (quad ^ exchange(l16)) * 16;
  // a wave's columns are of one block of b's rows
  static_assert(kFp8Block % (kN * 16) == 0);
  const unsigned at_scale_a = kRows * 128 + (wave_a + l16) * 4, at_scale_b = kRows * 128 + kTile * 4 + wave_b / kFp8Block * 4;
  // a group's steps follow each other; what it takes past the last step are zeros
  const int steps_here = (steps + kGroups - 1) / kGroups, first_step = group * steps_here;
  // The last tile's products of a step are added up in the next one.
  static_assert(kM % 2 == 0);
  f32x4 part[2][kN] = {};
  float prior_scale = 0.0f;
  // What a step reads and what it brings are different buffers.  (`__restrict__` says so: else every read of LDS would
  // wait for the loads into it.)
  auto run = [&](const unsigned char* __restrict__ from, unsigned char* __restrict__ to, int next) {
    u32x4 a[2][2], b[kN][2];
    float scale[2];
    auto read_a = [&](auto x) {
      each<2>([&](auto h) { a[x % 2][h] = *reinterpret_cast<const u32x4*>(from + x * 2048 + (at_a ^ (h * 64))); });
      scale[x % 2] = *reinterpret_cast<const float*>(from + at_scale_a + x * 64);
    };
    const float scale_b = *reinterpret_cast<const float*>(from + at_scale_b);
    each<kN>([&](auto y) {
      each<2>([&](auto h) { b[y][h] = *reinterpret_cast<const u32x4*>(from + y * 2048 + (at_b ^ (h * 64))); });
    });
    read_a(std::integral_constant<int, 0>{});
    fetch_scales(next, to);
    constexpr int kEach = (kLoads + kM - 1) / kM * 2;   // in the first half: spread over all of it took 5% longer
    each<kM>([&](auto x) {
      if constexpr (x + 1 < kM) read_a(std::integral_constant<int, x + 1>{});
      each<kEach>([&](auto j) {
        if constexpr (x * kEach + j < kLoads) fetch(x * kEach + j, next, to);
      });
      // the products of a tile of a, each followed by the sums of the tile before, whose products are done by then
      constexpr int kPrior = (x + kM - 1) % kM;
      each<kN>([&](auto y) {
        part[x % 2][y] = multiply(b[y][0], b[y][1], a[x % 2][0], a[x % 2][1]);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[kPrior][y][j] = __builtin_fmaf(part[(x + 1) % 2][y][j], prior_scale, sum[kPrior][y][j]);
      });
      prior_scale = scale[x % 2] * scale_b;
      each<kN>([&](auto) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x2, 4, 0);
      });
      __builtin_amdgcn_sched_barrier(0);
    });
  };
#pragma unroll
  for (int j = 0; j < kLoads; ++j) fetch(j, first_step, lds);
  fetch_scales(first_step, lds);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  for (int step = 0; step < steps_here; ++step) {
    const int buffer = step & 1;
    run(lds + buffer * kStage, lds + (buffer ^ 1) * kStage, first_step + step + 1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }
  each<kN>([&](auto y) {
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[kM - 1][y][j] = __builtin_fmaf(part[1][y][j], prior_scale, sum[kM - 1][y][j]);
  });
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
  each<kM>([&](auto x) {
    each<kN>([&](auto y) { store4<kF32>(p, i, tm * kTile + wave_a + x * 16 + l16, tn * kTile + wave_b + y * 16 + quad * 4, sum[x][y]); });
  });
}

int64_t tiles_of(int64_t rows, int64_t by) { return (rows + by - 1) / by; }

template <int kRowTiles, int kWaves, bool kF32>
hipError_t launch_thin(const Fp8Product& p, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(tiles_of(p.n, 16)), static_cast<unsigned>(tiles_of(p.m, kRowTiles * 16)), p.batch);
  thin_kernel<kRowTiles, kWaves, kF32><<<grid, kWaves * 64, 0, s>>>(p);
  return hipGetLastError();
}

template <int kTile, int kWavesM, int kWavesN, int kGroups, bool kF32>
hipError_t launch_staged(const Fp8Product& p, hipStream_t s) {
  constexpr int kLds = kGroups * 2 * (2 * kTile * 128 + (kTile / 64 + 1) * 256);
  static_assert(kLds <= 160 * 1024, "LDS of a workgroup");
  static_assert((kGroups - 1) * kTile * kTile * 4 <= kLds, "the groups' sums");
  constexpr auto kernel = &staged_kernel<kTile, kWavesM, kWavesN, kGroups, kF32>;
  if (const hipError_t e = allow_lds<kernel>(kLds); e != hipSuccess) return e;
  const int64_t tiles_m = tiles_of(p.m, kTile), tiles_n = tiles_of(p.n, kTile);
  kernel<<<dim3(static_cast<unsigned>(tiles_m * tiles_n), p.batch), kGroups * kWavesM * kWavesN * 64, kLds, s>>>(
      p, static_cast<int>(tiles_m), static_cast<int>(tiles_n));
  return hipGetLastError();
}

template <bool kF32>
hipError_t launch(const Fp8Product& p, hipStream_t s) {
  switch (fp8_plan(p)) {
    case Fp8Kernel::k16Rows: return launch_thin<1, 8, kF32>(p, s);
    case Fp8Kernel::k32Rows: return launch_thin<2, 4, kF32>(p, s);
    case Fp8Kernel::k64Rows: return launch_thin<4, 4, kF32>(p, s);
    case Fp8Kernel::k64TwoGroups: return launch_staged<64, 2, 2, 2, kF32>(p, s);
    case Fp8Kernel::k128TwoGroups: return launch_staged<128, 2, 2, 2, kF32>(p, s);
    case Fp8Kernel::k128: return launch_staged<128, 2, 2, 1, kF32>(p, s);
    case Fp8Kernel::k256: return launch_staged<256, 2, 4, 1, kF32>(p, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace

// Which kernel, by what each took (us, bfloat16 results, one call after the other in a graph):
//   rows x columns of out, k   thin   64, 2 groups   128, 2 groups    128    256
//       1 x  4096, 4096         5.2      11.7            17.9        25.8    44.1
//       1 x 32768, 4096        26.1      22.0            27.0        32.2    50.7
//      32 x  4096, 4096        10.1      12.0            18.1        26.1    44.8
//      64 x  4096, 4096        16.6      12.0            18.9        26.7    45.7
//     512 x  4096, 4096                  19.7            23.8        30.7    52.2
//    1024 x  4096, 4096                  37.3            27.2        34.0    53.6
//    1536 x  4096, 4096                  53.7            48.5        42.5    54.0
//    2304 x  4096, 4096                  81.1            71.4        68.9    54.8
//    8192 x  4096, 4096                                 187.7       175.7   128.9
// Two groups halve the steps that wait for memory one after the other, while a tile for each CU, or two, is
// all there is; large tiles read less per product.  Heads (rows x columns x products, k):
//      32 x 512 x  16, 128      3.0       3.9             5.4         4.2     5.3
//       8 x 512 x  64, 128      3.9       4.6             5.1         4.1     4.9
//     128 x 512 x 128, 128     26.4      16.4            12.9         9.8    10.0
Fp8Kernel fp8_plan(const Fp8Product& p) {
  // offsets within a tile's rows are held in 32 bits
  const int64_t longest = std::max(p.a.code_stride, p.b.code_stride);
  const bool staged = p.k > 0 && p.a.code_stride >= 0 && p.b.code_stride >= 0 && longest <= (INT32_MAX - p.k) / 256;
  const int rows = p.m <= 16 ? 16 : p.m <= 32 ? 32 : 64;
  const int64_t pieces = tiles_of(p.n, 16) * tiles_of(p.m, rows) * (rows / 16) * p.batch;
  if (!staged || (p.m <= 32 && pieces <= (p.k < 256 ? 2048 : 512)))
    return rows == 16 ? Fp8Kernel::k16Rows : rows == 32 ? Fp8Kernel::k32Rows : Fp8Kernel::k64Rows;
  const int64_t middle = tiles_of(p.m, 128) * tiles_of(p.n, 128) * p.batch, wide = tiles_of(p.m, 256) * tiles_of(p.n, 256) * p.batch;
  if (tiles_of(p.m, 64) * tiles_of(p.n, 64) * p.batch <= 512) return Fp8Kernel::k64TwoGroups;
  if (middle <= 256) return Fp8Kernel::k128TwoGroups;
  // (large tiles that few rows or columns leave half empty are no gain)
  return middle > 512 && wide * 4 <= middle + middle / 4 ? Fp8Kernel::k256 : Fp8Kernel::k128;
}

hipError_t launch_fp8_matmul(const Fp8Product& p, hipStream_t s) { return p.f32 ? launch<true>(p, s) : launch<false>(p, s); }

}  // namespace avsg
