// Product of two matrices in 8-bit floating point with a scale per 128 columns, out = a b^T.  The matrix
// instruction takes 128 columns at once:
//   16 x 128 by 128 x 16; lane l holds row l % 16 of either operand, columns (l / 16) * 32 .. + 31 (32
//   bytes), and of the result column l % 16, rows (l / 16) * 4 .. + 3.
// So a product of one block of columns is one instruction, whose result is added up times both
// scales.  The operands change places, so that a lane holds four neighbouring columns of one row of
// out, and with them one scale of a; b's is the same for 128 columns of out.
#include <algorithm>

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

template <bool kF32>
hipError_t launch(const Fp8Product& p, hipStream_t s) {
  auto tiles = [](int64_t rows, int64_t by) { return static_cast<unsigned>((rows + by - 1) / by); };
  const int rows = p.m <= 16 ? 16 : p.m <= 32 ? 32 : 64;
  const dim3 grid(tiles(p.n, 16), tiles(p.m, rows), p.batch);
  if (rows == 16) thin_kernel<1, 8, kF32><<<grid, 512, 0, s>>>(p);
  else if (rows == 32) thin_kernel<2, 4, kF32><<<grid, 256, 0, s>>>(p);
  else thin_kernel<4, 4, kF32><<<grid, 256, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_fp8_matmul(const Fp8Product& p, hipStream_t s) { return p.f32 ? launch<true>(p, s) : launch<false>(p, s); }

}  // namespace avsg
