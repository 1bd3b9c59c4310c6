// The 4-bit microscaled form: quantisation and its inverse.  A value is read and
// written once and takes a few operations, so memory bounds large matrices: 8192 x 4096
// of bfloat16 are quantised in 19 to 21 us (85 MB, 4.2 TB/s; a large copy moves 5.0).
// 16384 x 512, which the caches hold, takes 5.5 us either way, one small matrix 2.
#include "latent_internal.h"

namespace avsg {
namespace {

constexpr int kThreads = 256;
static_assert(kMostChunks % kThreads == 0);

// Eight columns per thread: 16 bytes of bfloat16 (32 of float32) in, one word of
// codes out; four neighbouring lanes hold a block of 32 and agree on its scale.
// A thread past the end takes part in the exchange with zeros.
template <bool kF32>
__global__ __launch_bounds__(kThreads) void quantize_kernel(const void* x, int64_t chunks, uint32_t per_row,
                                                            int64_t x_stride, uint8_t* codes, uint8_t* scales) {
  const int64_t at = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  float f[8] = {};
  if (at < chunks) {
    const int64_t row = at / per_row;
    const int64_t from = row * x_stride + (at - row * per_row) * 8;
    if constexpr (kF32) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(static_cast<const float*>(x) + from);
      const f32x4 b = *reinterpret_cast<const f32x4*>(static_cast<const float*>(x) + from + 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) f[i] = a[i], f[i + 4] = b[i];
    } else {
      const bf16x8 a = *reinterpret_cast<const bf16x8*>(static_cast<const __bf16*>(x) + from);
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = static_cast<float>(a[i]);
    }
  }
  const uint32_t scale = mx4_scale(mx4_block_top(f));
  if (at >= chunks) return;
  reinterpret_cast<uint32_t*>(codes)[at] = mx4_encode8(f, mx4_unit(scale));
  if ((at & 3) == 0) scales[at >> 2] = static_cast<uint8_t>(scale);
}

template <bool kF32>
__global__ __launch_bounds__(kThreads) void dequantize_kernel(Mx4View x, int64_t chunks, uint32_t per_row, void* out,
                                                              int64_t out_stride) {
  const int64_t at = static_cast<int64_t>(blockIdx.x) * kThreads + threadIdx.x;
  if (at >= chunks) return;
  const int64_t row = at / per_row, c = at - row * per_row;
  const uint32_t code = *reinterpret_cast<const uint32_t*>(x.codes + row * x.code_stride + 4 * c);
  const float unit = mx4_unit(x.scales[row * x.scale_stride + c / 4]);
  const int64_t to = row * out_stride + 8 * c;
  if constexpr (kF32) {
    const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, unit, 0);
    const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, unit, 1);
    const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, unit, 2);
    const f32x2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, unit, 3);
    *reinterpret_cast<f32x4*>(static_cast<float*>(out) + to) = f32x4{a[0], a[1], b[0], b[1]};
    *reinterpret_cast<f32x4*>(static_cast<float*>(out) + to + 4) = f32x4{d[0], d[1], e[0], e[1]};
  } else {
    *reinterpret_cast<bf16x8*>(static_cast<__bf16*>(out) + to) = mx4_decode8(code, unit);
  }
}

}  // namespace

hipError_t launch_mx4_quantize(const void* x, bool f32, int64_t rows, int64_t cols, int64_t x_stride, uint8_t* codes,
                               uint8_t* scales, hipStream_t s) {
  const int64_t chunks = rows * (cols / 8);
  const int64_t blocks = (chunks + kThreads - 1) / kThreads;   // chunks <= kMostChunks
  const uint32_t per_row = static_cast<uint32_t>(cols / 8);
  const dim3 grid(static_cast<unsigned>(blocks));
  if (f32) quantize_kernel<true><<<grid, kThreads, 0, s>>>(x, chunks, per_row, x_stride, codes, scales);
  else quantize_kernel<false><<<grid, kThreads, 0, s>>>(x, chunks, per_row, x_stride, codes, scales);
  return hipGetLastError();
}

hipError_t launch_mx4_dequantize(const Mx4View& x, int64_t rows, int64_t cols, void* out, bool f32, int64_t out_stride,
                                 hipStream_t s) {
  const int64_t chunks = rows * (cols / 8);
  const int64_t blocks = (chunks + kThreads - 1) / kThreads;   // chunks <= kMostChunks
  const uint32_t per_row = static_cast<uint32_t>(cols / 8);
  const dim3 grid(static_cast<unsigned>(blocks));
  if (f32) dequantize_kernel<true><<<grid, kThreads, 0, s>>>(x, chunks, per_row, out, out_stride);
  else dequantize_kernel<false><<<grid, kThreads, 0, s>>>(x, chunks, per_row, out, out_stride);
  return hipGetLastError();
}

}  // namespace avsg
