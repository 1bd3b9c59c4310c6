// 8-bit form of matrices (e4m3 codes, a float32 scale per 128 columns of a row or per 128 x 128),
// and back.
#include "fp8_internal.h"

namespace avsg {
namespace {

constexpr int kThreads = kFp8Threads;

template <bool kF32>
__device__ __forceinline__ void load8(const void* x, int64_t at, float (&v)[8]) {
  if constexpr (kF32) {
    const f32x4* from = reinterpret_cast<const f32x4*>(static_cast<const float*>(x) + at);
    const f32x4 a = from[0], b = from[1];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = a[j], v[4 + j] = b[j];
  } else {
    const bf16x8 a = *reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(x) + at);
#pragma unroll
    for (int j = 0; j < 8; ++j) v[j] = static_cast<float>(a[j]);
  }
}

// Bits of magnitudes order like the magnitudes, infinities and NaN above all others.
__device__ __forceinline__ uint32_t top_of(const float (&x)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
  return top;
}

__device__ __forceinline__ uint32_t row_max(uint32_t x) {
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0xb1, 0xf, 0xf, true)));    // lanes 1 0 3 2
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0x4e, 0xf, 0xf, true)));    // lanes 2 3 0 1
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, true)));   // mirrored within eight
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0x140, 0xf, 0xf, true)));   // mirrored within sixteen
  return x;
}

// Steps and scale of a block by the bits of its largest magnitude: 448 steps of the code to it.  Where
// 448 / magnitude would not be finite everything is zero; where the magnitude is not, the scale is NaN.
struct Steps {
  float steps, scale;
};
__device__ __forceinline__ Steps steps_of(uint32_t top) {
  const float a = __uint_as_float(top);
  if (top >= 0x7f800000u) return {0.0f, __uint_as_float(0x7fc00000u)};
  if (top < 0x05000000u) return {0.0f, 0.0f};   // 2^-117
  return {448.0f / a, a / 448.0f};
}

// The conversion rounds to the nearest code, ties to the even one; x * steps is at most 448 but for a rounding.
__device__ __forceinline__ u32x2 encode8(const float (&x)[8], float steps) {
  u32x2 c{};
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = steps == 0.0f ? 0.0f : x[4 * h + j] * steps;
    int word = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    word = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], word, true);
    c[h] = static_cast<uint32_t>(word);
  }
  return c;
}

// A block per sixteen lanes, eight columns each.  What bounds it is memory: 8192 x 4096 in bfloat16 take 19.0 us, 5.3 TB/s (one call
// after the other in a graph on the same 101 MB, like the figures below).
template <bool kF32>
__global__ __launch_bounds__(kThreads) void quantize_rows_kernel(Fp8Convert c) {
  const int s = threadIdx.x & 15, across = (c.cols + kFp8Block - 1) / kFp8Block;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * kFp8BlocksPerGroup + threadIdx.x / 16;
  if (item >= c.rows * across) return;
  const int64_t row = item / across;
  const int block = static_cast<int>(item - row * across), col = block * kFp8Block + 8 * s;
  const bool in = col < c.cols;
  float x[8] = {};
  if (in) load8<kF32>(c.plain, blockIdx.y * c.batch_stride + row * c.stride + col, x);
  const Steps st = steps_of(row_max(top_of(x)));
  if (in) *reinterpret_cast<u32x2*>(c.m.codes + blockIdx.y * c.m.code_batch_stride + row * c.m.code_stride + col) = encode8(x, st.steps);
  if (s == 0) c.m.scales[blockIdx.y * c.m.scale_batch_stride + row * c.m.scale_stride + block] = st.scale;
}

// A block of 128 x 128 per workgroup: sixteen rows at a time, sixteen lanes each; the values stay in registers between the
// magnitude and the codes.  8192 x 4096 in bfloat16 take 19.4 us, 5.2 TB/s, 4096 x 4096 10.2 us.
template <bool kF32>
__global__ __launch_bounds__(kThreads) void quantize_blocks_kernel(Fp8Convert c) {
  __shared__ uint32_t tops[kThreads / 64];
  const int s = threadIdx.x & 15, across = (c.cols + kFp8Block - 1) / kFp8Block;
  const int64_t down = blockIdx.x / across;
  const int block = static_cast<int>(blockIdx.x % across), col = block * kFp8Block + 8 * s;
  const int64_t first = down * kFp8Block + threadIdx.x / 16;
  float x[8][8];
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = first + 16 * i;
#pragma unroll
    for (int j = 0; j < 8; ++j) x[i][j] = 0.0f;
    if (row < c.rows && col < c.cols) load8<kF32>(c.plain, blockIdx.y * c.batch_stride + row * c.stride + col, x[i]);
    top = max(top, top_of(x[i]));
  }
  top = row_max(top);
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 16)));
  top = max(top, static_cast<uint32_t>(__shfl_xor(static_cast<int>(top), 32)));
  if ((threadIdx.x & 63) == 0) tops[threadIdx.x / 64] = top;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) top = max(top, tops[w]);
  const Steps st = steps_of(top);
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = first + 16 * i;
    if (row < c.rows && col < c.cols)
      *reinterpret_cast<u32x2*>(c.m.codes + blockIdx.y * c.m.code_batch_stride + row * c.m.code_stride + col) = encode8(x[i], st.steps);
  }
  if (threadIdx.x == 0) c.m.scales[blockIdx.y * c.m.scale_batch_stride + down * c.m.scale_stride + block] = st.scale;
}

// Sixteen lanes per 128 columns of a row, whatever its blocks.  8192 x 4096 to bfloat16 take 17.9 us, 5.6 TB/s.
template <bool kF32>
__global__ __launch_bounds__(kThreads) void dequantize_kernel(Fp8Convert c) {
  const int s = threadIdx.x & 15, across = (c.cols + kFp8Block - 1) / kFp8Block;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * kFp8BlocksPerGroup + threadIdx.x / 16;
  if (item >= c.rows * across) return;
  const int64_t row = item / across;
  const int block = static_cast<int>(item - row * across), col = block * kFp8Block + 8 * s;
  if (col >= c.cols) return;
  const float scale = c.m.scales[blockIdx.y * c.m.scale_batch_stride + row / c.m.block_rows * c.m.scale_stride + block];
  const u32x2 codes = *reinterpret_cast<const u32x2*>(c.m.codes + blockIdx.y * c.m.code_batch_stride + row * c.m.code_stride + col);
  float x[8];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(codes[h]), false);
    const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(static_cast<int>(codes[h]), true);
    x[4 * h] = a[0] * scale, x[4 * h + 1] = a[1] * scale, x[4 * h + 2] = b[0] * scale, x[4 * h + 3] = b[1] * scale;
  }
  const int64_t at = blockIdx.y * c.batch_stride + row * c.stride + col;
  if constexpr (kF32) {
    f32x4* to = reinterpret_cast<f32x4*>(static_cast<float*>(c.plain) + at);
    to[0] = f32x4{x[0], x[1], x[2], x[3]}, to[1] = f32x4{x[4], x[5], x[6], x[7]};
  } else {
    bf16x8 y;
#pragma unroll
    for (int j = 0; j < 8; ++j) y[j] = static_cast<__bf16>(x[j]);
    *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(c.plain) + at) = y;
  }
}

}  // namespace

hipError_t launch_fp8_quantize(const Fp8Convert& c, bool f32, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(fp8_groups(c.rows, c.cols, c.m.block_rows)), c.batch);
  if (c.m.block_rows == 1) {
    if (f32) quantize_rows_kernel<true><<<grid, kThreads, 0, s>>>(c);
    else quantize_rows_kernel<false><<<grid, kThreads, 0, s>>>(c);
  } else {
    if (f32) quantize_blocks_kernel<true><<<grid, kThreads, 0, s>>>(c);
    else quantize_blocks_kernel<false><<<grid, kThreads, 0, s>>>(c);
  }
  return hipGetLastError();
}

hipError_t launch_fp8_dequantize(const Fp8Convert& c, bool f32, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(fp8_groups(c.rows, c.cols, 1)), c.batch);
  if (f32) dequantize_kernel<true><<<grid, kThreads, 0, s>>>(c);
  else dequantize_kernel<false><<<grid, kThreads, 0, s>>>(c);
  return hipGetLastError();
}

}  // namespace avsg
