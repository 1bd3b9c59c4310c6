// Product of two mx4 matrices, out = a b^T, with the matrix instruction that
// takes 4-bit operands and their scales.
#include "latent_internal.h"

namespace avsg {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int kThreads = 256;

// One wave per 16 x 16 outputs.  The instruction multiplies 16 x 128 by 128 x 16:
// lane l holds row l % 16 of either operand, columns (l / 16) * 32 .. + 31 of
// the 128 (one block: 16 bytes of codes and their scale), and of the result
// column l % 16, rows (l / 16) * 4 .. + 3.  Rows and blocks past the end are
// zeros.
__global__ __launch_bounds__(kThreads) void product_kernel(Mx4Product p) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = lane & 15, quad = lane >> 4;
  const int m0 = blockIdx.y * 16, n0 = (blockIdx.x * 4 + wave) * 16;
  if (n0 >= p.n) return;
  const int64_t i = blockIdx.z;
  const int blocks = p.k / kMx4Block;
  const bool in_a = m0 + row < p.m, in_b = n0 + row < p.n;
  const uint8_t* ac = p.a.codes + i * p.a.code_batch_stride + static_cast<int64_t>(m0 + row) * p.a.code_stride;
  const uint8_t* as = p.a.scales + i * p.a.scale_batch_stride + static_cast<int64_t>(m0 + row) * p.a.scale_stride;
  const uint8_t* bc = p.b.codes + i * p.b.code_batch_stride + static_cast<int64_t>(n0 + row) * p.b.code_stride;
  const uint8_t* bs = p.b.scales + i * p.b.scale_batch_stride + static_cast<int64_t>(n0 + row) * p.b.scale_stride;
  f32x4 sum{};
  for (int k = quad; k - quad < blocks; k += 4) {
    u32x4 a{}, b{};
    uint32_t sa = 127, sb = 127;
    if (k < blocks && in_a) a = *reinterpret_cast<const u32x4*>(ac + 16 * k), sa = as[k];
    if (k < blocks && in_b) b = *reinterpret_cast<const u32x4*>(bc + 16 * k), sb = bs[k];
    const i32x8 A{static_cast<int>(a[0]), static_cast<int>(a[1]), static_cast<int>(a[2]), static_cast<int>(a[3]), 0, 0, 0, 0};
    const i32x8 B{static_cast<int>(b[0]), static_cast<int>(b[1]), static_cast<int>(b[2]), static_cast<int>(b[3]), 0, 0, 0, 0};
    sum = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(A, B, sum, 4, 4, 0, static_cast<int>(sa), 0, static_cast<int>(sb));
  }
  if (!in_b) return;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int m = m0 + quad * 4 + j;
    if (m >= p.m) continue;
    const int64_t to = i * p.out_batch_stride + static_cast<int64_t>(m) * p.out_stride + n0 + row;
    if (p.f32) static_cast<float*>(p.out)[to] = sum[j];
    else static_cast<__bf16*>(p.out)[to] = static_cast<__bf16>(sum[j]);
  }
}

}  // namespace

hipError_t launch_mx4_matmul(const Mx4Product& p, hipStream_t s) {
  if ((p.m + 15) / 16 > 65535) return hipErrorInvalidValue;
  const dim3 grid((p.n + 63) / 64, (p.m + 15) / 16, p.batch);
  product_kernel<<<grid, kThreads, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace avsg
