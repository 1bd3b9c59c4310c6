// Declarations shared by the translation units of the latent-cache operators
// (include/avsg_latent.h): cache addressing, the 4-bit format, launchers.
#pragma once

#include <atomic>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "avsg_internal.h"
#include "avsg_latent.h"

namespace avsg {

constexpr int64_t kMostThreads = (int64_t{1} << 32) - 1;   // of a launch, along a dimension

constexpr int kLatent = 512;           // latent values of a row: key and value
constexpr int kRope = 64;              // rotated values of a row: key only
constexpr int kKeyDim = kLatent + kRope;
constexpr int kMx4Block = 32;          // columns per scale
constexpr int kMx4CodeBytes = kLatent / 2;
constexpr int kMx4Scales = kLatent / kMx4Block;
constexpr int kMx4RopeAt = kMx4CodeBytes + kMx4Scales;
constexpr int kRowBytesBf16 = kKeyDim * 2;
constexpr int kRowBytesMx4 = kMx4RopeAt + kRope * 2;

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

// A cache as a kernel sees it (avsg_cache).
struct CacheView {
  uint64_t base;
  int64_t page_stride, row_stride;
  const int32_t* table;      // or nullptr
  int32_t pages;
  int32_t batch;
  int32_t pages_per_request;
  int32_t capacity;          // rows of a request
  int32_t page_shift;        // row >> page_shift is its page (31 for one page per request)
  int32_t page_mask;         // row & page_mask its place in the page
};

// Address of row `row` of request `r`, 0 where there is none.
__device__ __forceinline__ uint64_t cache_row(const CacheView& c, int r, int64_t row) {
  if (row < 0 || row >= c.capacity) return 0;
  const int64_t at = static_cast<int64_t>(r) * c.pages_per_request + (static_cast<int32_t>(row) >> c.page_shift);
  const int64_t page = c.table ? c.table[at] : at;
  if (page < 0 || page >= c.pages) return 0;
  return c.base + page * c.page_stride + (static_cast<int32_t>(row) & c.page_mask) * c.row_stride;
}

// The scale byte of a block whose largest magnitude has the float bits `top`:
// the power of two that brings it into [3.5, 7), where the nearest code is at
// most 6 (the quarter added to the mantissa carries into the exponent from 1.75
// on).  At least 2^-125, so that every value a code stands for is a normal
// number in bfloat16 and float32, and at most 2^125, so that it is finite there
// (magnitudes above 7 * 2^125 become 6 * 2^125); 255 for an infinity or a NaN.
__device__ __forceinline__ uint32_t mx4_scale(uint32_t top) {
  if (top >= 0x7f800000u) return 255u;
  const int e = static_cast<int>((top + 0x200000u) >> 23) - 2;
  return static_cast<uint32_t>(e < 2 ? 2 : e > 252 ? 252 : e);
}
// What a scale byte multiplies by, as the conversion instructions take it: they
// read the exponent field alone, so byte 0 is 2^-127 and 255 makes NaN.
__device__ __forceinline__ float mx4_unit(uint32_t scale) { return __uint_as_float(scale << 23); }

// Eight codes (a word, lowest column in the lowest half byte) of eight values.
// The conversion rounds to the nearest code, ties to the even one, and
// saturates at 6.
__device__ __forceinline__ uint32_t mx4_encode8(const float (&x)[8], float unit) {
  uint32_t c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], unit, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], unit, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], unit, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], unit, 3);
  return c;
}
// The eight values of a word of codes in bfloat16, which holds them exactly.
__device__ __forceinline__ bf16x8 mx4_decode8(uint32_t c, float unit) {
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 0);
  const bf16x2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 1);
  const bf16x2 d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 2);
  const bf16x2 e = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, unit, 3);
  return bf16x8{a[0], a[1], b[0], b[1], d[0], d[1], e[0], e[1]};
}

// The largest magnitude (float bits) of eight values and of the same in the
// other three lanes of a group of four: with eight columns per lane those hold
// one block.  Bits of magnitudes order like the magnitudes, infinities and NaN
// above all others.
__device__ __forceinline__ uint32_t mx4_block_top(const float (&x)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
  top = max(top, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, top, 0xb1, 0xf, 0xf, true)));   // lanes 1 0 3 2
  top = max(top, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, top, 0x4e, 0xf, 0xf, true)));   // lanes 2 3 0 1
  return top;
}

struct AppendParams {
  CacheView cache;
  int64_t tokens, positions;
  const __bf16* latent;
  const __bf16* rope;
  int64_t latent_stride, rope_stride;
  const int32_t* request;
  const int64_t* position;
  const float* angles;
  int32_t heads;
  const __bf16* q;
  int64_t q_token_stride, q_head_stride;
  __bf16* q_out;
  int64_t q_out_token_stride, q_out_head_stride;
};

struct ReadParams {
  CacheView cache;
  int64_t n;
  const int32_t* request;
  const int64_t* position;
  __bf16* out;
  int64_t out_stride;
};

// Rows that a launch of append or read takes: a wave each, four to a workgroup.
constexpr int64_t kMostRowWaves = kMostThreads / 256 * 4;
// Eight columns of a matrix that a launch of quantise or dequantise takes, a thread each.
constexpr int64_t kMostChunks = kMostThreads / 256 * 256;
// Heads' queries that one wave of append rotates.
constexpr int kHeadsPerWave = 8;

// How a call of attention is carried out.
enum class AttendKernel {
  k16Heads,        // 16 heads per workgroup, tiles of 64 rows, two workgroups per CU
  k16HeadsAlone,   // 16 heads, tiles of 128 rows, one workgroup per CU
  k64Heads,        // 64 heads, one workgroup per CU
};
constexpr int heads_of(AttendKernel k) { return k == AttendKernel::k64Heads ? 64 : 16; }
// the least part of a token's rows that a workgroup takes
constexpr int rows_of(AttendKernel k) { return k == AttendKernel::k16HeadsAlone ? 128 : 64; }

// Parts of results, of a head each, that the workgroups of a call leave: tokens * splits * heads
constexpr int64_t kMostParts = 256 * 64;

struct AttendPlan {
  AttendKernel kernel;
  int32_t splits;   // workgroups that share a query token's entries
};

struct AttendParams {
  CacheView cache;
  int32_t n_q, heads, topk;
  float scale;
  const __bf16* q;
  int64_t q_token_stride, q_head_stride;
  const int32_t* rows;
  const int32_t* index;
  const int64_t* lens;
  __bf16* out;
  int64_t out_token_stride, out_head_stride;
  float* lse;
  AttendPlan plan;
  float* part_out;      // [B n_q][splits][heads][512], splits > 1
  f32x2* part_ml;       // [B n_q][splits][heads]: reference and sum
  float above, rest_unit;   // of the weights; the launch sets them
};

struct Mx4View {
  const uint8_t* codes;
  const uint8_t* scales;
  int64_t code_stride, code_batch_stride, scale_stride, scale_batch_stride;
};

struct Mx4Product {
  Mx4View a, b;
  int32_t batch;
  int32_t m, n, k;
  void* out;
  bool f32;
  bool wide_stores;   // four neighbouring outputs can be stored at once
  int64_t out_stride, out_batch_stride;
};

// Host side, shared with the other operators around the step: the calling thread's error text, a
// launch's status, alignments, and a cache's view (its format is not looked at: rows of `row` bytes,
// addresses and strides in multiples of `align`).
avsg_status fail(avsg_status s, const char* fmt, ...);
avsg_status launched(hipError_t e, const char* what);
inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
// bfloat16 rows read or written 16 bytes at a time
inline bool rows16(const void* p, int64_t stride) { return p && aligned(p, 16) && (stride & 7) == 0; }
avsg_status view_of(const avsg_cache* c, size_t row, int align, CacheView* v);

// Lets a kernel have `bytes` of dynamic LDS, once on each GPU that is current in a call.
template <auto kKernel>
hipError_t allow_lds(size_t bytes) {
  static std::atomic<uint64_t> done{0};
  int gpu = 0;
  if (const hipError_t e = hipGetDevice(&gpu); e != hipSuccess) return e;
  const uint64_t bit = gpu < 64 ? uint64_t{1} << gpu : 0;
  if (done.load(std::memory_order_relaxed) & bit) return hipSuccess;
  const hipError_t e =
      hipFuncSetAttribute(reinterpret_cast<const void*>(kKernel), hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
  if (e == hipSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return e;
}

hipError_t launch_kv_append(const AppendParams& p, int format, int rope_style, hipStream_t s);
hipError_t launch_kv_read(const ReadParams& p, int format, hipStream_t s);
// threads of a call's attention kernel
int64_t attend_threads(const AttendPlan& plan, int64_t tokens, int heads);
// the kernel of a call of attention, and how many workgroups share a token
AttendPlan attend_plan(int format, int batch, int n_q, int heads, int topk);
hipError_t launch_attend(const AttendParams& p, int format, hipStream_t s);
hipError_t launch_mx4_quantize(const void* x, bool f32, int64_t rows, int64_t cols, int64_t x_stride, uint8_t* codes,
                               uint8_t* scales, hipStream_t s);
hipError_t launch_mx4_dequantize(const Mx4View& x, int64_t rows, int64_t cols, void* out, bool f32,
                                 int64_t out_stride, hipStream_t s);
hipError_t launch_mx4_matmul(const Mx4Product& p, hipStream_t s);

}  // namespace avsg

// attend_plan for tests, which assert what their cases run: the kernel in the low half, the parts in the high
// one.  Not part of the ABI.
extern "C" int64_t avsg_internal_attend_plan(int32_t format, int32_t batch, int32_t n_q, int32_t heads, int32_t topk);
