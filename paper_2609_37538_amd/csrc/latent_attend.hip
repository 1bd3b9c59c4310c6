// Attention of a step's query tokens over latent cache rows.
#include "latent_internal.h"

namespace avsg {
namespace {

constexpr int kThreads = 256;
constexpr int kTile = 64;

// One workgroup per (query token, head): 64 entries at a time, each wave takes
// the scores of 16 of them (a lane has latent columns 8l..8l+7 and rotated
// column l), then every thread adds the 64 rows, weighted, to two columns of the
// output.  The sum is kept relative to the running maximum.
template <bool kMx4>
__global__ __launch_bounds__(kThreads) void attend_kernel(AttendParams p) {
  __shared__ float score[kTile];
  __shared__ uint64_t row_at[kTile];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t token = blockIdx.x;
  const int head = blockIdx.y, r = static_cast<int>(token / p.n_q);
  const __bf16* q = p.q + token * p.q_token_stride + head * p.q_head_stride;
  float ql[8], qr = static_cast<float>(q[kLatent + lane]);
  for (int i = 0; i < 8; ++i) ql[i] = static_cast<float>(q[8 * lane + i]);
  const int64_t len = p.lens ? p.lens[token] : INT64_MAX;
  float top = -INFINITY, total = 0.f, o[2] = {0.f, 0.f};
  for (int first = 0; first < p.topk; first += kTile) {
    __syncthreads();
    if (threadIdx.x < kTile) {
      const int i = first + threadIdx.x;
      uint64_t at = 0;
      if (i < p.topk) {
        const int64_t pos = p.index ? p.index[token * p.topk + i] : i;
        if (pos >= 0 && pos < len) at = cache_row(p.cache, r, p.rows ? p.rows[token * p.topk + i] : i);
      }
      row_at[threadIdx.x] = at;
    }
    __syncthreads();
    for (int i = wave * 16; i < wave * 16 + 16; ++i) {
      const uint64_t at = row_at[i];
      float s = 0.f;
      if (at != 0) {
        bf16x8 x;
        if constexpr (kMx4)
          x = mx4_decode8(load_global<uint32_t>(at + 4 * lane),
                          mx4_unit(load_global<uint8_t>(at + kMx4CodeBytes + lane / 4)));
        else
          x = load_global<bf16x8>(at + 16 * lane);
        for (int k = 0; k < 8; ++k) s += ql[k] * static_cast<float>(x[k]);
        s += qr * static_cast<float>(load_global<__bf16>(at + (kMx4 ? kMx4RopeAt : kLatent * 2) + 2 * lane));
      }
      for (int d = 32; d > 0; d /= 2) s += __shfl_xor(s, d);
      if (lane == 0) score[i] = at != 0 ? s * p.scale : -INFINITY;
    }
    __syncthreads();
    float high = top;
    for (int i = 0; i < kTile; ++i)
      if (row_at[i] != 0) high = fmaxf(high, score[i]);
    const float base = high == -INFINITY ? 0.f : high, keep = expf(top - base);
    if (top != -INFINITY) total *= keep, o[0] *= keep, o[1] *= keep;
    for (int i = 0; i < kTile; ++i) {
      const uint64_t at = row_at[i];
      if (at == 0) continue;
      const float w = expf(score[i] - base);
      total += w;
      bf16x2 v;
      if constexpr (kMx4)
        v = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(
            load_global<uint8_t>(at + threadIdx.x),
            mx4_unit(load_global<uint8_t>(at + kMx4CodeBytes + threadIdx.x / 16)), 0);
      else
        v = load_global<bf16x2>(at + 4 * threadIdx.x);
      o[0] += w * static_cast<float>(v[0]);
      o[1] += w * static_cast<float>(v[1]);
    }
    top = high;
  }
  const float by = total == 0.f ? 0.f : 1.f / total;
  __bf16* out = p.out + token * p.out_token_stride + head * p.out_head_stride + 2 * threadIdx.x;
  *reinterpret_cast<bf16x2*>(out) = bf16x2{static_cast<__bf16>(o[0] * by), static_cast<__bf16>(o[1] * by)};
  if (p.lse && threadIdx.x == 0) p.lse[token * p.heads + head] = total == 0.f ? -INFINITY : top + logf(total);
}

}  // namespace

int attend_splits(int batch, int n_q, int heads, int topk) {
  (void)batch, (void)n_q, (void)heads, (void)topk;
  return 1;
}

hipError_t launch_attend(const AttendParams& p, int format, hipStream_t s) {
  const dim3 grid(static_cast<unsigned>(p.cache.batch * p.n_q), static_cast<unsigned>(p.heads));
  if (format == 1) attend_kernel<true><<<grid, kThreads, 0, s>>>(p);
  else attend_kernel<false><<<grid, kThreads, 0, s>>>(p);
  return hipGetLastError();
}

}  // namespace avsg
