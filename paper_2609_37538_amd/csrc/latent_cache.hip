// Rows of the latent cache: appending (rotation, 4-bit form) and reading back.
//
// Both move each value once and compute a few operations per value, so memory
// bounds them where there are many tokens and one launch's latency where there
// are few: appending the rows and 128 heads' queries of 128 tokens takes 3.4 us, 20 480
// tokens of four prompts in 4 bits 27 us and reading them back 9, together the
// 145 MB at 4.0 TB/s.
#include "latent_internal.h"

namespace avsg {
namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kGroup = 8;   // lanes that share one vector of 64 values to rotate
static_assert(kWaves == 4 && kGroup == kHeadsPerWave, "kMostRowWaves");

// Lane s of eight turns four pairs (a, b) of a 64-vector by the angles of its
// pairs 4s..4s+3: (a cos - b sin, a sin + b cos) in float32, rounded once.
// kHalves: pairs are columns i and i + 32, else 2i and 2i + 1.
template <bool kHalves>
__device__ __forceinline__ bf16x8 load_pairs(const __bf16* x, int s) {
  if constexpr (kHalves) {
    const bf16x4 a = *reinterpret_cast<const bf16x4*>(x + 4 * s);
    const bf16x4 b = *reinterpret_cast<const bf16x4*>(x + kRope / 2 + 4 * s);
    return bf16x8{a[0], b[0], a[1], b[1], a[2], b[2], a[3], b[3]};
  } else {
    return *reinterpret_cast<const bf16x8*>(x + 8 * s);
  }
}
template <bool kHalves>
__device__ __forceinline__ void store_pairs(__bf16* x, int s, bf16x8 v) {
  if constexpr (kHalves) {
    *reinterpret_cast<bf16x4*>(x + 4 * s) = bf16x4{v[0], v[2], v[4], v[6]};
    *reinterpret_cast<bf16x4*>(x + kRope / 2 + 4 * s) = bf16x4{v[1], v[3], v[5], v[7]};
  } else {
    *reinterpret_cast<bf16x8*>(x + 8 * s) = v;
  }
}
__device__ __forceinline__ bf16x8 rotate(bf16x8 x, f32x4 t0, f32x4 t1) {
  const float c[4] = {t0[0], t0[2], t1[0], t1[2]}, s[4] = {t0[1], t0[3], t1[1], t1[3]};
  bf16x8 y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = static_cast<float>(x[2 * i]), b = static_cast<float>(x[2 * i + 1]);
    y[2 * i] = static_cast<__bf16>(a * c[i] - b * s[i]);
    y[2 * i + 1] = static_cast<__bf16>(a * s[i] + b * c[i]);
  }
  return y;
}

// One wave per row (lane l has latent columns 8l..8l+7, so four lanes hold a
// block of 32; lanes 0..7 turn the rotated part), then one wave per eight query
// heads of a token (eight lanes each).
template <bool kMx4, bool kHalves>
__global__ __launch_bounds__(kThreads) void append_kernel(AppendParams p, int groups) {
  const int lane = threadIdx.x & 63;
  int64_t item = static_cast<int64_t>(blockIdx.x) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool is_row = item < p.tokens;
  int64_t token = item;
  int head = 0;
  if (!is_row) {
    item -= p.tokens;
    if (groups == 0 || item >= p.tokens * groups) return;
    token = item / groups;
    head = static_cast<int>(item - token * groups) * kGroup + lane / kGroup;
  }
  const int s = lane % kGroup;
  const int64_t pos = p.position[token];
  const bool known = pos >= 0 && pos < p.positions;
  f32x4 t0{}, t1{};
  if (known) {
    const float* t = p.angles + pos * kRope + 8 * s;
    t0 = *reinterpret_cast<const f32x4*>(t);
    t1 = *reinterpret_cast<const f32x4*>(t + 4);
  }
  if (!is_row) {
    if (head >= p.heads) return;
    bf16x8 y{};
    if (known) y = rotate(load_pairs<kHalves>(p.q + token * p.q_token_stride + head * p.q_head_stride, s), t0, t1);
    store_pairs<kHalves>(p.q_out + token * p.q_out_token_stride + head * p.q_out_head_stride, s, y);
    return;
  }
  const int r = p.request[token];
  if (!known || r < 0 || r >= p.cache.batch) return;
  const uint64_t row = cache_row(p.cache, r, pos);
  if (row == 0) return;
  const bf16x8 x = *reinterpret_cast<const bf16x8*>(p.latent + token * p.latent_stride + 8 * lane);
  bf16x8 turned{};
  if (lane < kGroup) turned = rotate(load_pairs<kHalves>(p.rope + token * p.rope_stride, s), t0, t1);
  if constexpr (kMx4) {
    float f[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = static_cast<float>(x[i]);
    const uint32_t scale = mx4_scale(mx4_block_top(f));
    store_global<uint32_t>(row + 4 * lane, mx4_encode8(f, mx4_unit(scale)));
    if ((lane & 3) == 0) store_global<uint8_t>(row + kMx4CodeBytes + lane / 4, static_cast<uint8_t>(scale));
  } else {
    store_global<bf16x8>(row + 16 * lane, x);
  }
  constexpr int kRopeAt = kMx4 ? kMx4RopeAt : kLatent * 2;
  if (lane < kGroup) store_pairs<kHalves>(reinterpret_cast<__bf16*>(row + kRopeAt), s, turned);
}

// One wave per row: lane l brings latent columns 8l..8l+7, lanes 0..7 the rotated part.
template <bool kMx4>
__global__ __launch_bounds__(kThreads) void read_kernel(ReadParams p) {
  const int lane = threadIdx.x & 63;
  const int64_t item = static_cast<int64_t>(blockIdx.x) * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (item >= p.n) return;
  const int r = p.request[item];
  const uint64_t row = r >= 0 && r < p.cache.batch ? cache_row(p.cache, r, p.position[item]) : 0;
  bf16x8 x{}, y{};
  if (row != 0) {
    if constexpr (kMx4) {
      const uint32_t c = load_global<uint32_t>(row + 4 * lane);
      x = mx4_decode8(c, mx4_unit(load_global<uint8_t>(row + kMx4CodeBytes + lane / 4)));
    } else {
      x = load_global<bf16x8>(row + 16 * lane);
    }
    if (lane < kGroup) y = load_global<bf16x8>(row + (kMx4 ? kMx4RopeAt : kLatent * 2) + 16 * lane);
  }
  __bf16* out = p.out + item * p.out_stride;
  *reinterpret_cast<bf16x8*>(out + 8 * lane) = x;
  if (lane < kGroup) *reinterpret_cast<bf16x8*>(out + kLatent + 8 * lane) = y;
}

}  // namespace

hipError_t launch_kv_append(const AppendParams& p, int format, int rope_style, hipStream_t s) {
  const int groups = (p.heads + kGroup - 1) / kGroup;
  const int64_t items = p.tokens * (1 + groups);
  const dim3 grid(static_cast<unsigned>((items + kWaves - 1) / kWaves));
  if (format == 1) {
    if (rope_style == 1) append_kernel<true, true><<<grid, kThreads, 0, s>>>(p, groups);
    else append_kernel<true, false><<<grid, kThreads, 0, s>>>(p, groups);
  } else {
    if (rope_style == 1) append_kernel<false, true><<<grid, kThreads, 0, s>>>(p, groups);
    else append_kernel<false, false><<<grid, kThreads, 0, s>>>(p, groups);
  }
  return hipGetLastError();
}

hipError_t launch_kv_read(const ReadParams& p, int format, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>((p.n + kWaves - 1) / kWaves));
  if (format == 1) read_kernel<true><<<grid, kThreads, 0, s>>>(p);
  else read_kernel<false><<<grid, kThreads, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace avsg
