// Host side of the 8-bit matrices (include/avsg_fp8.h): argument checks and launches.
#include "avsg_fp8.h"

#include "fp8_internal.h"

using namespace avsg;

namespace {

avsg_status view_of(const avsg_fp8* x, Fp8View* v) {
  if (!x || !x->d_codes || !x->d_scales) return fail(AVSG_E_INVAL, "null matrix, codes or scales");
  if (x->block_rows != 1 && x->block_rows != kFp8Block) return fail(AVSG_E_INVAL, "block_rows must be 1 or %d", kFp8Block);
  if (!aligned(x->d_codes, 16) || (x->code_stride & 15) != 0 || (x->code_batch_stride & 15) != 0 || !aligned(x->d_scales, 4))
    return fail(AVSG_E_INVAL, "codes and their rows must be 16-byte aligned, scales 4-byte aligned");
  *v = Fp8View{const_cast<uint8_t*>(static_cast<const uint8_t*>(x->d_codes)), const_cast<float*>(x->d_scales), x->code_stride,
               x->code_batch_stride, x->scale_stride, x->scale_batch_stride, x->block_rows};
  return AVSG_OK;
}

// What quantise and dequantise check alike; *nothing: there is nothing to do.
avsg_status convert_of(const avsg_fp8* m, const void* plain, int32_t type, int32_t batch, int64_t rows, int64_t cols, int64_t stride,
                       int64_t batch_stride, Fp8Convert* c, bool* nothing) {
  if (type != AVSG_BF16 && type != AVSG_F32) return fail(AVSG_E_INVAL, "unknown type %d", type);
  if (batch < 0 || rows < 0 || cols < 0) return fail(AVSG_E_INVAL, "batch, rows and cols must not be negative");
  if (cols % 16 != 0) return fail(AVSG_E_RANGE, "cols must be a multiple of 16");
  *nothing = batch == 0 || rows == 0 || cols == 0;
  if (*nothing) return AVSG_OK;
  if (avsg_status st = view_of(m, &c->m); st != AVSG_OK) return st;
  const int64_t unit = type == AVSG_F32 ? 3 : 7;
  if (!plain || !aligned(plain, 16) || (stride & unit) != 0 || (batch_stride & unit) != 0)
    return fail(AVSG_E_INVAL, "the plain matrix and its rows must be 16-byte aligned");
  // (rows of the smallest group of blocks, so that the product below does not overflow)
  if (batch > 65535 || cols > INT32_MAX - kFp8Block || rows > (int64_t{1} << 40) || fp8_groups(rows, cols, 1) > kMostThreads / kFp8Threads)
    return fail(AVSG_E_RANGE, "batch must be at most 65535, and a matrix have at most 16 * (2^24 - 1) blocks of 1 x 128");
  c->plain = const_cast<void*>(plain);
  c->stride = stride;
  c->batch_stride = batch_stride;
  c->rows = rows;
  c->cols = static_cast<int32_t>(cols);
  c->batch = batch;
  return AVSG_OK;
}

}  // namespace

extern "C" {

avsg_status avsg_fp8_quantize(const void* d_x, int32_t type, int32_t batch, int64_t rows, int64_t cols, int64_t x_stride,
                              int64_t x_batch_stride, const avsg_fp8* out, void* stream) {
  Fp8Convert c{};
  bool nothing = false;
  if (avsg_status st = convert_of(out, d_x, type, batch, rows, cols, x_stride, x_batch_stride, &c, &nothing); st != AVSG_OK || nothing) return st;
  return launched(launch_fp8_quantize(c, type == AVSG_F32, static_cast<hipStream_t>(stream)), "avsg_fp8_quantize");
}

avsg_status avsg_fp8_dequantize(const avsg_fp8* x, int32_t batch, int64_t rows, int64_t cols, void* d_out, int32_t type, int64_t out_stride,
                                int64_t out_batch_stride, void* stream) {
  Fp8Convert c{};
  bool nothing = false;
  if (avsg_status st = convert_of(x, d_out, type, batch, rows, cols, out_stride, out_batch_stride, &c, &nothing); st != AVSG_OK || nothing) return st;
  return launched(launch_fp8_dequantize(c, type == AVSG_F32, static_cast<hipStream_t>(stream)), "avsg_fp8_dequantize");
}

avsg_status avsg_fp8_matmul(const avsg_fp8* a, const avsg_fp8* b, int32_t batch, int64_t m, int64_t n, int64_t k, void* d_out, int32_t out_type,
                            int64_t out_stride, int64_t out_batch_stride, void* stream) {
  Fp8Product p{};
  if (out_type != AVSG_BF16 && out_type != AVSG_F32) return fail(AVSG_E_INVAL, "unknown out_type %d", out_type);
  if (batch < 0 || m < 0 || n < 0 || k < 0) return fail(AVSG_E_INVAL, "sizes must not be negative");
  if (k % 16 != 0) return fail(AVSG_E_RANGE, "k must be a multiple of 16");
  if (m > kMostFp8Rows || n > kMostFp8Rows || k > INT32_MAX / 2 || batch > 65535)
    return fail(AVSG_E_RANGE, "m and n must be at most %lld, k below 2^30 and batch at most 65535", static_cast<long long>(kMostFp8Rows));
  if ((m + 63) / 64 * ((n + 63) / 64) >= (int64_t{1} << 24)) return fail(AVSG_E_RANGE, "m x n must have fewer than 2^24 tiles of 64 x 64");
  if (batch == 0 || m == 0 || n == 0) return AVSG_OK;
  if (!d_out || !aligned(d_out, out_type == AVSG_F32 ? 4 : 2)) return fail(AVSG_E_INVAL, "d_out is null or misaligned");
  if (k > 0) {   // (without columns nothing of the matrices is read)
    if (avsg_status st = view_of(a, &p.a); st != AVSG_OK) return st;
    if (avsg_status st = view_of(b, &p.b); st != AVSG_OK) return st;
    if (p.a.block_rows != 1 || p.b.block_rows != kFp8Block)
      return fail(AVSG_E_UNSUPPORTED, "a must have blocks of 1 x 128 and b of 128 x 128");
  }
  p.batch = batch;
  p.m = static_cast<int32_t>(m);
  p.n = static_cast<int32_t>(n);
  p.k = static_cast<int32_t>(k);
  p.out = d_out;
  p.f32 = out_type == AVSG_F32;
  p.out_stride = out_stride;
  p.out_batch_stride = out_batch_stride;
  p.wide_stores = aligned(d_out, p.f32 ? 16 : 8) && (out_stride & 3) == 0 && (out_batch_stride & 3) == 0;
  return launched(launch_fp8_matmul(p, static_cast<hipStream_t>(stream)), "avsg_fp8_matmul");
}

int32_t avsg_internal_fp8_plan(int32_t batch, int32_t m, int32_t n, int32_t k, int64_t a_stride, int64_t b_stride) {
  Fp8Product p{};
  p.batch = batch, p.m = m, p.n = n, p.k = k;
  p.a.code_stride = a_stride, p.b.code_stride = b_stride;
  return static_cast<int32_t>(fp8_plan(p));
}

}  // extern "C"
