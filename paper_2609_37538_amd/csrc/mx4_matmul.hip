// Product of two mx4 matrices, out = a b^T, with the matrix instruction that
// takes 4-bit operands and their scales:
//   16 x 128 by 128 x 16; lane l holds row l % 16 of either operand, columns
//   (l / 16) * 32 .. + 31 of the 128 (one block: 16 bytes of codes and their
//   scale), and of the result column l % 16, rows (l / 16) * 4 .. + 3.
// The 32 x 32 x 64 form of the instruction adds up less exactly: products of
// random codes with scales 2^-7 to 2^6 were off by 1.5e-5 of the result where this
// form is off by 2.6e-7.
#include <type_traits>

#include "latent_internal.h"

namespace avsg {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

__device__ __forceinline__ i32x8 operand(u32x4 x) {
  return i32x8{static_cast<int>(x[0]), static_cast<int>(x[1]), static_cast<int>(x[2]), static_cast<int>(x[3]), 0, 0, 0, 0};
}

template <int kByteA, int kByteB>
__device__ __forceinline__ f32x4 multiply(u32x4 a, u32x4 b, f32x4 sum, uint32_t scales_a, uint32_t scales_b) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(operand(a), operand(b), sum, 4, 4, kByteA, static_cast<int>(scales_a),
                                                         kByteB, static_cast<int>(scales_b));
}

template <typename T>
__device__ __forceinline__ void store(void* out, int64_t at, float x) {
  static_cast<T*>(out)[at] = static_cast<T>(x);
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
      for (int r = 0; r < kRowTiles; ++r) sum[r] = multiply<0, 0>(a[u][r], b[u], sum[r], sa[u][r], sb[u]);
  }
  if (wave > 0) {
#pragma unroll
    for (int r = 0; r < kRowTiles; ++r) sums[wave - 1][r][lane] = sum[r];
  }
  __syncthreads();
  if (wave > 0 || !in_b) return;
#pragma unroll
  for (int r = 0; r < kRowTiles; ++r) {
#pragma unroll
    for (int w = 0; w < kWaves - 1; ++w) sum[r] += sums[w][r][lane];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int m = m0 + r * 16 + quad * 4 + j;
      if (m < p.m)
        store<std::conditional_t<kF32, float, __bf16>>(p.out, i * p.out_batch_stride + static_cast<int64_t>(m) * p.out_stride + n, sum[r][j]);
    }
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
      for (int y = 0; y < kN; ++y) sum[x][y] = multiply<0, 0>(a[x], b[y], sum[x][y], sa[x], sb[y]);
  }
#pragma unroll
  for (int x = 0; x < kM; ++x)
#pragma unroll
    for (int y = 0; y < kN; ++y) {
      const int n = n0 + y * 16 + l16;
      if (n >= p.n) continue;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int m = m0 + x * 16 + quad * 4 + j;
        if (m < p.m)
          store<std::conditional_t<kF32, float, __bf16>>(p.out, i * p.out_batch_stride + static_cast<int64_t>(m) * p.out_stride + n, sum[x][y][j]);
      }
    }
}

template <bool kF32>
hipError_t launch(const Mx4Product& p, hipStream_t s) {
  if (p.m <= 64) {
    const dim3 grid((p.n + 15) / 16, 1, p.batch);
    if (p.m <= 16) thin_kernel<1, 8, kF32><<<grid, 512, 0, s>>>(p);
    else if (p.m <= 32) thin_kernel<2, 4, kF32><<<grid, 256, 0, s>>>(p);
    else thin_kernel<4, 4, kF32><<<grid, 256, 0, s>>>(p);
    return hipGetLastError();
  }
  const int64_t tiles_m = (p.m + 127) / 128, tiles_n = (p.n + 127) / 128;
  if (tiles_m * tiles_n > INT32_MAX) return hipErrorInvalidValue;
  tile_kernel<128, 128, 2, 2, kF32><<<dim3(static_cast<unsigned>(tiles_m * tiles_n), p.batch), 256, 0, s>>>(
      p, static_cast<int>(tiles_m), static_cast<int>(tiles_n));
  return hipGetLastError();
}

}  // namespace

hipError_t launch_mx4_matmul(const Mx4Product& p, hipStream_t s) { return p.f32 ? launch<true>(p, s) : launch<false>(p, s); }

}  // namespace avsg
