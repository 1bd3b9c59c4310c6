// Rows of the key cache: appending (rotation, 8-bit form), with the index queries
// of the same tokens, and reading back.
#include "select_internal.h"

namespace avsg {
namespace {

constexpr int kThreads = 256;
constexpr int kPerGroup = kThreads / kLanesPerKey;   // rows of sixteen lanes of a workgroup
constexpr int kHeadsPerRow = 4;
static_assert(kLanesPerKey == 16, "a row of lanes per vector");

typedef unsigned int u32x2_at_4 __attribute__((ext_vector_type(2), aligned(4)));

// The largest of a value over the sixteen lanes of a row.
__device__ __forceinline__ uint32_t row_max(uint32_t x) {
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0xb1, 0xf, 0xf, true)));    // lanes 1 0 3 2
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0x4e, 0xf, 0xf, true)));    // lanes 2 3 0 1
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0x141, 0xf, 0xf, true)));   // mirrored within eight
  x = max(x, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, x, 0x140, 0xf, 0xf, true)));   // mirrored within sixteen
  return x;
}

// Cosines and sines for the lane's columns: lane s of sixteen has columns 8s..8s+7, the lanes [first, first + 8) the 64
// rotated ones.  Pairs are neighbours (four of them, in the first half of t) or columns i and i + 32 (eight).
template <bool kHalves>
__device__ __forceinline__ void load_turns(f32x4 (&t)[4], const float* angles, int p) {
  const f32x4* at = reinterpret_cast<const f32x4*>(angles + (kHalves ? 16 * (p & 3) : 8 * p));
#pragma unroll
  for (int j = 0; j < (kHalves ? 4 : 2); ++j) t[j] = at[j];
}
// Turns the lane's eight columns, p being its place among the eight lanes that do (all sixteen take part in the exchange).
// Every product and sum is rounded to float32, so that the same steps elsewhere give the same codes.
template <bool kHalves>
__device__ __forceinline__ void turn(float (&x)[8], const f32x4 (&t)[4], int p) {
#pragma clang fp contract(off)
  const bool mine = p >= 0 && p < 8;
  if constexpr (kHalves) {
    float other[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) other[j] = __shfl_xor(x[j], 4, 16);   // columns i and i + 32 are four lanes apart
    if (!mine) return;
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float c = t[j][2 * i], d = t[j][2 * i + 1], mine_by_c = x[2 * j + i] * c, other_by_d = other[2 * j + i] * d;
        x[2 * j + i] = p < 4 ? mine_by_c - other_by_d : other_by_d + mine_by_c;
      }
  } else {
    if (!mine) return;
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float a = x[4 * j + 2 * i], b = x[4 * j + 2 * i + 1], c = t[j][2 * i], d = t[j][2 * i + 1];
        const float ac = a * c, bd = b * d, ad = a * d, bc = b * c;
        x[4 * j + 2 * i] = ac - bd;
        x[4 * j + 2 * i + 1] = ad + bc;
      }
  }
}

// Codes of the lane's eight values, and the vector's scale: 127 steps to its largest magnitude.  Where 127 /
// magnitude would not be finite everything is zero; where the magnitude is not, the scale is NaN.
__device__ __forceinline__ u32x2 encode(const float (&x)[8], float& scale) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
  top = row_max(top);
  const bool fine = top < 0x7f800000u, some = fine && top >= 0x04000000u;   // 2^-119
  const float a = __uint_as_float(top), steps = some ? 127.0f / a : 0.0f;
  scale = !fine ? __uint_as_float(0x7fc00000u) : some ? a / 127.0f : 0.0f;
  u32x2 codes{};
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int c = some ? static_cast<int>(rintf(x[j] * steps)) : 0;
    codes[j / 4] |= (static_cast<uint32_t>(c) & 255u) << (8 * (j & 3));
  }
  return codes;
}

// Sixteen lanes per vector, eight columns each: the keys of all tokens, one each, then kHeadsPerRow queries of a token, which
// share its angles.  5122 tokens of 64 queries take 28 us, 130 MB at 4.6 TB/s (with a query per row 37).
template <bool kHalves>
__global__ __launch_bounds__(kThreads) void append_kernel(KeyAppendParams p, int groups) {
  const int s = threadIdx.x % kLanesPerKey;
  int64_t item = static_cast<int64_t>(blockIdx.x) * kPerGroup + threadIdx.x / kLanesPerKey;
  const bool is_key = item < p.tokens;
  int64_t token = item;
  int head = 0;
  if (!is_key) {
    item -= p.tokens;
    if (groups == 0 || item >= p.tokens * groups) return;
    token = item / groups;
    head = static_cast<int>(item - token * groups) * kHeadsPerRow;
  }
  const int64_t pos = p.position[token];
  const bool known = pos >= 0 && (p.rope_at < 0 || pos < p.positions);
  const int place = s - p.rope_at / 8;   // among the lanes that turn
  f32x4 turns[4] = {};
  if (known && p.rope_at >= 0 && place >= 0 && place < 8) load_turns<kHalves>(turns, p.angles + pos * kRope, place);
  auto codes_of = [&](bf16x8 v, float& scale) {
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = static_cast<float>(v[j]);
    if (p.rope_at >= 0) turn<kHalves>(x, turns, place);
    return encode(x, scale);
  };
  if (is_key) {
    const int r = p.request[token];
    if (!known || r < 0 || r >= p.cache.batch) return;
    const uint64_t row = cache_row(p.cache, r, pos);
    if (row == 0) return;
    float scale;
    const u32x2 codes = codes_of(*reinterpret_cast<const bf16x8*>(p.key + token * p.key_stride + 8 * s), scale);
    store_global<u32x2_at_4>(row + 8 * s, codes);
    if (s == 0) store_global<float>(row + kKeyScaleAt, scale);
    return;
  }
  const int most = min(kHeadsPerRow, p.heads - head);
  bf16x8 v[kHeadsPerRow] = {};
#pragma unroll
  for (int h = 0; h < kHeadsPerRow; ++h)
    if (known && h < most) v[h] = *reinterpret_cast<const bf16x8*>(p.q + token * p.q_token_stride + (head + h) * p.q_head_stride + 8 * s);
#pragma unroll
  for (int h = 0; h < kHeadsPerRow; ++h) {
    if (h >= most) break;
    u32x2 codes{};
    float scale = 0.0f;
    if (known) codes = codes_of(v[h], scale);
    *reinterpret_cast<u32x2*>(p.q_out + token * p.q_out_token_stride + (head + h) * p.q_out_head_stride + 8 * s) = codes;
    if (s == 0)
      p.weights_out[token * p.weight_out_stride + head + h] =
          !known ? 0.0f : p.weights ? p.weights[token * p.weight_stride + head + h] * scale : scale;
  }
}

__global__ __launch_bounds__(kThreads) void read_kernel(ReadParams p) {
  const int s = threadIdx.x % kLanesPerKey;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * kPerGroup + threadIdx.x / kLanesPerKey;
  if (item >= p.n) return;
  const int r = p.request[item];
  const uint64_t row = r >= 0 && r < p.cache.batch ? cache_row(p.cache, r, p.position[item]) : 0;
  bf16x8 x{};
  if (row != 0) {
    const u32x2 codes = load_global<u32x2_at_4>(row + 8 * s);
    const float scale = load_global<float>(row + kKeyScaleAt);
#pragma unroll
    for (int j = 0; j < 8; ++j)
      x[j] = static_cast<__bf16>(static_cast<float>(static_cast<int8_t>(codes[j / 4] >> (8 * (j & 3)))) * scale);
  }
  *reinterpret_cast<bf16x8*>(p.out + item * p.out_stride + 8 * s) = x;
}

unsigned groups_of(int64_t vectors) { return static_cast<unsigned>((vectors + kPerGroup - 1) / kPerGroup); }

}  // namespace

hipError_t launch_key_append(const KeyAppendParams& p, int rope_style, hipStream_t s) {
  const int groups = (p.heads + kHeadsPerRow - 1) / kHeadsPerRow;
  const dim3 grid(groups_of(p.tokens * (1 + groups)));
  if (rope_style == AVSG_ROPE_HALVES) append_kernel<true><<<grid, kThreads, 0, s>>>(p, groups);
  else append_kernel<false><<<grid, kThreads, 0, s>>>(p, groups);
  return hipGetLastError();
}

hipError_t launch_key_read(const ReadParams& p, hipStream_t s) {
  read_kernel<<<dim3(groups_of(p.n)), kThreads, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace avsg
