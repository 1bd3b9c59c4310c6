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
// nothing to rearrange, and the waves that share rows find them in L1.
// Steps of 256 columns; the next step's loads are issued before this one's
// products.
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
    const int64_t n = min(n0 + r * 16 + l16, p.n - 1);
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
#pragma unroll
  for (int x = 0; x < kM; ++x)
#pragma unroll
    for (int y = 0; y < kN; ++y) store4<kF32>(p, i, m0 + x * 16 + l16, n0 + y * 16 + quad * 4, sum[x][y]);
}

// What columns past the end read in place of codes.
__device__ __align__(16) const unsigned char zero_block[16] = {};

// Larger products: tiles of kTileM x kTileN outputs, kWavesM x kWavesN waves.
// Steps of 256 columns go from global memory to LDS without passing registers, the
// next step's while this one's products run: 64 matrix instructions per wave and step
// at 256 x 256.  In LDS a row has its 128 bytes of the step, its eight blocks exchanged by
// bits 1..3 of the row, so that the sixteen lanes that read one block of sixteen
// rows meet every bank; eight neighbouring lanes fetch a row's whole line.
template <int kTileM, int kTileN, int kWavesM, int kWavesN, bool kF32>
__global__ __launch_bounds__(kWavesM * kWavesN * 64, kWavesM * kWavesN / 4) void staged_kernel(Mx4Product p, int tiles_m, int tiles_n) {
  constexpr int kWaves = kWavesM * kWavesN, kThreads = kWaves * 64;
  constexpr int kM = kTileM / kWavesM / 16, kN = kTileN / kWavesN / 16;
  constexpr int kRows = kTileM + kTileN;                 // rows of a, then rows of b
  constexpr int kLoads = kRows / 8 / kWaves;             // eight rows each
  constexpr int kScaleRows = kRows / kThreads;           // rows whose scales a thread brings
  static_assert(kRows % (8 * kWaves) == 0 && kRows % kThreads == 0, "shares of the loads");
  constexpr int kStage = kRows * 136;                    // codes, then eight scales per row
  extern __shared__ __align__(16) unsigned char lds[];   // [2]
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
  const int blocks = p.k / kMx4Block, steps = (blocks + 7) / 8;

  // Row `r` of the tile's rows of a and b, as an offset from the first of them;
  // rows past the end are not stored, and read as the last.
  const uint8_t* const codes_a = p.a.codes + i * p.a.code_batch_stride + static_cast<int64_t>(tm) * kTileM * p.a.code_stride;
  const uint8_t* const codes_b = p.b.codes + i * p.b.code_batch_stride + static_cast<int64_t>(tn) * kTileN * p.b.code_stride;
  const int last_a = p.m - 1 - tm * kTileM, last_b = p.n - 1 - tn * kTileN;
  // eight rows are of one matrix
  auto from_a = [&](int j) { return (j * kWaves + wave) * 8 < kTileM; };
  uint32_t row_at[kLoads];
  const int block_of = (lane & 7) ^ ((wave * 4 + lane / 16) & 7);
  static_assert(kWaves % 2 == 0, "block_of is the same for all loads");
#pragma unroll
  for (int j = 0; j < kLoads; ++j) {
    const int r = (j * kWaves + wave) * 8 + lane / 8;
    row_at[j] = from_a(j) ? min(r, last_a) * static_cast<uint32_t>(p.a.code_stride)
                          : min(r - kTileM, last_b) * static_cast<uint32_t>(p.b.code_stride);
  }
  const uint8_t* scale_row[kScaleRows];
#pragma unroll
  for (int j = 0; j < kScaleRows; ++j) {
    const int r = j * kThreads + threadIdx.x;
    const Mx4View& x = r < kTileM ? p.a : p.b;
    const int64_t row = r < kTileM ? tm * kTileM + min(r, last_a) : tn * kTileN + min(r - kTileM, last_b);
    scale_row[j] = x.scales + i * x.scale_batch_stride + row * x.scale_stride;
  }

  uint64_t scales[kScaleRows];
  auto fetch = [&](int step, int buffer) {
#pragma unroll
    for (int j = 0; j < kLoads; ++j) {
      // (the compiler would keep eight advancing 64-bit addresses)
      uint32_t row = row_at[j];
      asm volatile("" : "+v"(row));
      const int block = step * 8 + block_of;
      const uint8_t* from = (from_a(j) ? codes_a : codes_b) + row + 16 * static_cast<uint32_t>(block);
      if (block >= blocks) from = zero_block;
      __builtin_amdgcn_global_load_lds(
          reinterpret_cast<const __attribute__((address_space(1))) void*>(reinterpret_cast<uint64_t>(from)),
          (__attribute__((address_space(3))) void*)(lds + buffer * kStage + (j * kWaves + wave) * 1024), 16, 0, 0);
    }
    // eight scales, of the last step the row's last eight moved down: where they
    // are zeros in place of scales, so are the codes
    const int first = min(step * 8, blocks - 8), off = (step * 8 - first) * 8;
#pragma unroll
    for (int j = 0; j < kScaleRows; ++j) {
      __builtin_memcpy(&scales[j], scale_row[j] + first, 8);
      scales[j] >>= off;
    }
  };
  auto leave_scales = [&](int buffer) {
#pragma unroll
    for (int j = 0; j < kScaleRows; ++j)
      reinterpret_cast<uint64_t*>(lds + buffer * kStage + kRows * 128)[j * kThreads + threadIdx.x] = scales[j];
  };

  f32x4 sum[kM][kN] = {};
  const int a0 = wave / kWavesN * (kM * 16), b0 = kTileM + wave % kWavesN * (kN * 16);
  const unsigned at = (l16 * 128) + ((quad ^ (l16 >> 1 & 7)) * 16);
  fetch(0, 0);
  leave_scales(0);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  for (int step = 0; step < steps; ++step) {
    const int buffer = step & 1;
    const unsigned char* const from = lds + buffer * kStage;
    // (of the last step a second time: without a branch the products stay where they are)
    fetch(min(step + 1, steps - 1), buffer ^ 1);
    u32x2 sa[kM], sb[kN];
#pragma unroll
    for (int x = 0; x < kM; ++x) sa[x] = *reinterpret_cast<const u32x2*>(from + kRows * 128 + (a0 + x * 16 + l16) * 8) >> (quad * 8);
#pragma unroll
    for (int y = 0; y < kN; ++y) sb[y] = *reinterpret_cast<const u32x2*>(from + kRows * 128 + (b0 + y * 16 + l16) * 8) >> (quad * 8);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      // a block of b for all of a's, which come two ahead: left to itself the
      // compiler reads all of a step first and runs out of registers
      u32x4 a[kM], b[kN];
#pragma unroll
      for (int y = 0; y < kN; ++y) b[y] = *reinterpret_cast<const u32x4*>(from + b0 * 128 + y * 2048 + (at ^ (half * 64)));
#pragma unroll
      for (int x = 0; x < kM; ++x) a[x] = *reinterpret_cast<const u32x4*>(from + a0 * 128 + x * 2048 + (at ^ (half * 64)));
#pragma unroll
      for (int x = 0; x < kM; ++x)
#pragma unroll
        for (int y = 0; y < kN; ++y) sum[x][y] = multiply<0, 0>(b[y], a[x], sum[x][y], sb[y][half], sa[x][half]);
      schedule<kLdsRead, kN + 2>();
#pragma unroll
      for (int x = 0; x < kM; ++x) {
        schedule<kMatrix, kN>();
        schedule<kLdsRead, 1>();
      }
      __builtin_amdgcn_sched_barrier(0);
    }
    leave_scales(buffer ^ 1);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }
  const int m0 = tm * kTileM + a0, n0 = tn * kTileN + b0 - kTileM;
#pragma unroll
  for (int x = 0; x < kM; ++x)
#pragma unroll
    for (int y = 0; y < kN; ++y) store4<kF32>(p, i, m0 + x * 16 + l16, n0 + y * 16 + quad * 4, sum[x][y]);
}

template <int kTile, int kWavesM, int kWavesN, bool kF32>
hipError_t launch_staged(const Mx4Product& p, int64_t tiles_m, int64_t tiles_n, hipStream_t s) {
  constexpr int kLds = 2 * 2 * kTile * 136;
  static_assert(kLds <= 160 * 1024, "LDS of a workgroup");
  const auto kernel = &staged_kernel<kTile, kTile, kWavesM, kWavesN, kF32>;
  static const hipError_t ready =
      hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kLds);
  if (ready != hipSuccess) return ready;
  kernel<<<dim3(static_cast<unsigned>(tiles_m * tiles_n), p.batch), kWavesM * kWavesN * 64, kLds, s>>>(
      p, static_cast<int>(tiles_m), static_cast<int>(tiles_n));
  return hipGetLastError();
}

template <bool kF32>
hipError_t launch(const Mx4Product& p, hipStream_t s) {
  const int64_t tiles_m = (p.m + 127) / 128, tiles_n = (p.n + 127) / 128;
  const int64_t wide_m = (p.m + 255) / 256, wide_n = (p.n + 255) / 256;
  if (tiles_m * tiles_n > INT32_MAX) return hipErrorInvalidValue;
  constexpr int64_t kCus = 256;
  // offsets within a tile's rows are held in 32 bits
  const int64_t longest = std::max(p.a.code_stride, p.b.code_stride);
  const bool staged = p.k > 512 && p.a.code_stride >= 0 && p.b.code_stride >= 0 && longest * 256 + p.k < (int64_t{1} << 31);
  if (p.m <= 64 || tiles_m * tiles_n * p.batch < kCus / 2) {
    const int rows = p.m <= 16 ? 16 : p.m <= 32 ? 32 : 64;
    if ((p.m + rows - 1) / rows > 65535) return hipErrorInvalidValue;
    const dim3 grid((p.n + 15) / 16, (p.m + rows - 1) / rows, p.batch);
    if (rows == 16) thin_kernel<1, 8, kF32><<<grid, 512, 0, s>>>(p);
    else if (rows == 32) thin_kernel<2, 4, kF32><<<grid, 256, 0, s>>>(p);
    else thin_kernel<4, 4, kF32><<<grid, 256, 0, s>>>(p);
    return hipGetLastError();
  }
  if (staged && wide_m * wide_n * p.batch >= kCus) return launch_staged<256, 2, 4, kF32>(p, wide_m, wide_n, s);
  if (staged) return launch_staged<128, 2, 2, kF32>(p, tiles_m, tiles_n, s);
  tile_kernel<128, 128, 2, 2, kF32><<<dim3(static_cast<unsigned>(tiles_m * tiles_n), p.batch), 256, 0, s>>>(
      p, static_cast<int>(tiles_m), static_cast<int>(tiles_n));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_matmul(const Mx4Product& p, hipStream_t s) { return p.f32 ? launch<true>(p, s) : launch<false>(p, s); }

}  // namespace avsg
