// Declarations shared by the translation units of the 8-bit matrices
// (include/avsg_fp8.h).
#pragma once

#include "avsg_fp8.h"
#include "latent_internal.h"

namespace avsg {

constexpr int kFp8Block = AVSG_FP8_BLOCK;

struct Fp8View {
  uint8_t* codes;
  float* scales;
  int64_t code_stride, code_batch_stride, scale_stride, scale_batch_stride;
  int32_t block_rows;
};

struct Fp8Convert {
  Fp8View m;
  void* plain;              // the other side
  int64_t stride, batch_stride;
  int64_t rows;
  int32_t cols, batch;
};

struct Fp8Product {
  Fp8View a, b;
  int32_t batch;
  int32_t m, n, k;
  void* out;
  bool f32;
  bool wide_stores;   // four neighbouring outputs can be stored at once
  int64_t out_stride, out_batch_stride;
};

// Rows of an operand of a product: 65535 tiles of 64 along a dimension of a launch.
constexpr int64_t kMostFp8Rows = 65535 * 64;

// Workgroups of a conversion's batch: 16 blocks of 1 x 128 or one of 128 x 128 each.
constexpr int kFp8Threads = 256, kFp8BlocksPerGroup = kFp8Threads / 16;
constexpr int64_t fp8_groups(int64_t rows, int64_t cols, int32_t block_rows) {
  const int64_t across = (cols + kFp8Block - 1) / kFp8Block;
  return block_rows == 1 ? (rows * across + kFp8BlocksPerGroup - 1) / kFp8BlocksPerGroup
                         : (rows + kFp8Block - 1) / kFp8Block * across;
}

// How a product is carried out.
enum class Fp8Kernel {
  k16Rows,          // up to 16 rows of a per workgroup, b streamed past them
  k32Rows,          // up to 32
  k64Rows,          // up to 64: what rows too far apart for 32-bit offsets take
  k64TwoGroups,     // tiles of 64 x 64 staged through LDS, two groups of waves that share the columns
  k128TwoGroups,    // tiles of 128 x 128, likewise
  k128,             // tiles of 128 x 128
  k256,             // tiles of 256 x 256
};

hipError_t launch_fp8_quantize(const Fp8Convert& c, bool f32, hipStream_t s);
hipError_t launch_fp8_dequantize(const Fp8Convert& c, bool f32, hipStream_t s);
// the kernel of a product, by its sizes and its operands' strides
Fp8Kernel fp8_plan(const Fp8Product& p);
hipError_t launch_fp8_matmul(const Fp8Product& p, hipStream_t s);

}  // namespace avsg

// fp8_plan for tests, which assert what their cases run.  Not part of the ABI.
extern "C" int32_t avsg_internal_fp8_plan(int32_t batch, int32_t m, int32_t n, int32_t k, int64_t a_stride, int64_t b_stride);
