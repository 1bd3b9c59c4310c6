// Host side of the latent-cache operators (include/avsg_latent.h): argument
// checks, the kernels' view of caches, launches.  Nothing here allocates or
// keeps state beyond the calling thread's last error text.
#include "avsg_latent.h"

#include <algorithm>
#include <cstdarg>
#include <cstdio>

#include "latent_internal.h"

using namespace avsg;

namespace {

thread_local char g_error[256] = {0};

avsg_status fail(avsg_status s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(g_error, sizeof(g_error), fmt, ap);
  va_end(ap);
  return s;
}

avsg_status launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return AVSG_OK;
  return fail(AVSG_E_HIP, "%s: %s", what, hipGetErrorString(e));
}

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
// bfloat16 rows read or written 16 bytes at a time
bool rows16(const void* p, int64_t stride) { return p && aligned(p, 16) && (stride & 7) == 0; }

avsg_status view_of(const avsg_cache* c, CacheView* v) {
  if (!c || !c->base) return fail(AVSG_E_INVAL, "null cache or cache base");
  const size_t row = avsg_row_bytes(c->format);
  if (row == 0) return fail(AVSG_E_INVAL, "unknown row format %d", c->format);
  if (c->batch < 1 || c->pages_per_request < 1 || c->page_rows < 1 || c->pages < 1)
    return fail(AVSG_E_INVAL, "batch, pages, pages_per_request and page_rows must be positive");
  if (c->pages > INT32_MAX) return fail(AVSG_E_RANGE, "pages must be below 2^31");
  const bool power = (c->page_rows & (c->page_rows - 1)) == 0;
  if (!power && c->pages_per_request != 1)
    return fail(AVSG_E_NOTPOW2, "page_rows must be a power of two (or pages_per_request 1)");
  const int64_t capacity = static_cast<int64_t>(c->pages_per_request) * c->page_rows;
  if (capacity > INT32_MAX) return fail(AVSG_E_RANGE, "rows of a request must be below 2^31");
  if (!aligned(c->base, 16) || (c->row_stride & 15) != 0 || (c->page_stride & 15) != 0)
    return fail(AVSG_E_RANGE, "base, row_stride and page_stride must be multiples of 16 bytes");
  if (c->row_stride < static_cast<int64_t>(row)) return fail(AVSG_E_RANGE, "row_stride is less than a row's %zu bytes", row);
  if (c->row_stride > INT64_MAX / c->page_rows || c->page_stride < c->row_stride * c->page_rows ||
      c->page_stride > INT64_MAX / c->pages)
    return fail(AVSG_E_RANGE, "page_stride is less than the page's rows, or the pool's size overflows");
  if (!c->d_page_table && static_cast<int64_t>(c->batch) * c->pages_per_request > c->pages)
    return fail(AVSG_E_CAPACITY, "without a page table the pool needs batch * pages_per_request pages");
  v->base = reinterpret_cast<uint64_t>(c->base);
  v->page_stride = c->page_stride;
  v->row_stride = c->row_stride;
  v->table = c->d_page_table;
  v->pages = static_cast<int32_t>(c->pages);
  v->batch = c->batch;
  v->pages_per_request = c->pages_per_request;
  v->capacity = static_cast<int32_t>(capacity);
  if (c->pages_per_request == 1) {
    v->page_shift = 31;
    v->page_mask = INT32_MAX;
  } else {
    v->page_shift = __builtin_ctz(static_cast<unsigned>(c->page_rows));
    v->page_mask = c->page_rows - 1;
  }
  return AVSG_OK;
}

}  // namespace

extern "C" {

size_t avsg_row_bytes(int32_t format) {
  return format == AVSG_ROWS_BF16 ? kRowBytesBf16 : format == AVSG_ROWS_MX4 ? kRowBytesMx4 : 0;
}

const char* avsg_latent_last_error(void) { return g_error; }

avsg_status avsg_kv_append(const avsg_cache* cache, const avsg_append* a, void* stream) {
  AppendParams p{};
  if (avsg_status st = view_of(cache, &p.cache); st != AVSG_OK) return st;
  if (!a) return fail(AVSG_E_INVAL, "null append");
  if (a->tokens < 0 || a->heads < 0 || a->positions < 0)
    return fail(AVSG_E_INVAL, "tokens, heads and positions must not be negative");
  if (a->rope_style != AVSG_ROPE_PAIRS && a->rope_style != AVSG_ROPE_HALVES)
    return fail(AVSG_E_INVAL, "unknown rope_style %d", a->rope_style);
  if (a->tokens == 0) return AVSG_OK;
  if (!rows16(a->d_latent, a->latent_stride) || !rows16(a->d_rope, a->rope_stride))
    return fail(AVSG_E_INVAL, "d_latent and d_rope must be 16-byte aligned with strides in multiples of 8 elements");
  if (!a->d_request || !a->d_position || !a->d_angles || !aligned(a->d_angles, 16))
    return fail(AVSG_E_INVAL, "d_request, d_position and d_angles (16-byte aligned) are needed");
  if (a->heads > 0 && (!rows16(a->d_q, a->q_token_stride) || (a->q_head_stride & 7) != 0 ||
                       !rows16(a->d_q_out, a->q_out_token_stride) || (a->q_out_head_stride & 7) != 0))
    return fail(AVSG_E_INVAL, "d_q and d_q_out must be 16-byte aligned with strides in multiples of 8 elements");
  if (a->heads > 65536 || a->tokens > kMostRowWaves / (1 + (a->heads + kHeadsPerWave - 1) / kHeadsPerWave))
    return fail(AVSG_E_RANGE, "tokens * (1 + heads / 8, rounded up) must be at most %lld, heads at most 65536",
                static_cast<long long>(kMostRowWaves));
  p.tokens = a->tokens;
  p.positions = a->positions;
  p.latent = static_cast<const __bf16*>(a->d_latent);
  p.rope = static_cast<const __bf16*>(a->d_rope);
  p.latent_stride = a->latent_stride;
  p.rope_stride = a->rope_stride;
  p.request = a->d_request;
  p.position = a->d_position;
  p.angles = a->d_angles;
  p.heads = a->heads;
  p.q = static_cast<const __bf16*>(a->d_q);
  p.q_token_stride = a->q_token_stride;
  p.q_head_stride = a->q_head_stride;
  p.q_out = static_cast<__bf16*>(a->d_q_out);
  p.q_out_token_stride = a->q_out_token_stride;
  p.q_out_head_stride = a->q_out_head_stride;
  return launched(launch_kv_append(p, cache->format, a->rope_style, static_cast<hipStream_t>(stream)), "avsg_kv_append");
}

avsg_status avsg_kv_read(const avsg_cache* cache, int64_t n, const int32_t* d_request, const int64_t* d_position,
                         void* d_out, int64_t out_stride, void* stream) {
  ReadParams p{};
  if (avsg_status st = view_of(cache, &p.cache); st != AVSG_OK) return st;
  if (n < 0) return fail(AVSG_E_INVAL, "n must not be negative");
  if (n == 0) return AVSG_OK;
  if (n > kMostRowWaves) return fail(AVSG_E_RANGE, "n must be at most %lld", static_cast<long long>(kMostRowWaves));
  if (!d_request || !d_position) return fail(AVSG_E_INVAL, "d_request and d_position are needed");
  if (!rows16(d_out, out_stride))
    return fail(AVSG_E_INVAL, "d_out must be 16-byte aligned with a stride in multiples of 8 elements");
  p.n = n;
  p.request = d_request;
  p.position = d_position;
  p.out = static_cast<__bf16*>(d_out);
  p.out_stride = out_stride;
  return launched(launch_kv_read(p, cache->format, static_cast<hipStream_t>(stream)), "avsg_kv_read");
}

size_t avsg_attend_workspace_bytes(int32_t batch, int32_t n_q, int32_t heads, int32_t topk) {
  if (batch < 1 || n_q < 1 || heads < 1 || topk < 1) return 0;
  // of either row format, whichever has more parts
  const size_t splits = static_cast<size_t>(std::max(attend_plan(AVSG_ROWS_BF16, batch, n_q, heads, topk).splits,
                                                     attend_plan(AVSG_ROWS_MX4, batch, n_q, heads, topk).splits));
  if (splits <= 1) return 0;   // else at most 256 workgroups of 64 heads, or 512 of 16
  const size_t parts = static_cast<size_t>(batch) * n_q * splits * heads;
  return parts * (kLatent * sizeof(float) + sizeof(f32x2));
}

static_assert(AVSG_ATTEND_WORKSPACE_MOST == kMostParts * (kLatent * sizeof(float) + sizeof(f32x2)));

avsg_status avsg_attend(const avsg_cache* cache, const avsg_attention* a, void* d_workspace, size_t workspace_bytes,
                        void* stream) {
  AttendParams p{};
  if (avsg_status st = view_of(cache, &p.cache); st != AVSG_OK) return st;
  if (!a) return fail(AVSG_E_INVAL, "null attention");
  if (a->n_q < 1 || a->heads < 1 || a->topk < 0)
    return fail(AVSG_E_INVAL, "n_q and heads must be positive, topk not negative");
  if (!rows16(a->d_q, a->q_token_stride) || (a->q_head_stride & 7) != 0 || !rows16(a->d_out, a->out_token_stride) ||
      (a->out_head_stride & 7) != 0)
    return fail(AVSG_E_INVAL, "d_q and d_out must be 16-byte aligned with strides in multiples of 8 elements");
  const int64_t tokens = static_cast<int64_t>(cache->batch) * a->n_q;
  if (tokens > (1 << 19) || a->heads > 4096)
    return fail(AVSG_E_RANGE, "batch * n_q must be at most 2^19 and heads at most 4096");
  p.n_q = a->n_q;
  p.heads = a->heads;
  p.topk = a->topk;
  p.scale = a->scale;
  p.q = static_cast<const __bf16*>(a->d_q);
  p.q_token_stride = a->q_token_stride;
  p.q_head_stride = a->q_head_stride;
  p.rows = a->d_rows;
  p.index = a->d_index;
  p.lens = a->d_lens;
  p.out = static_cast<__bf16*>(a->d_out);
  p.out_token_stride = a->out_token_stride;
  p.out_head_stride = a->out_head_stride;
  p.lse = a->d_lse;
  p.plan = attend_plan(cache->format, cache->batch, a->n_q, a->heads, a->topk);
  if (attend_threads(p.plan, tokens, a->heads) > kMostThreads)
    return fail(AVSG_E_RANGE, "batch * n_q * heads is more than a launch takes");
  if (p.plan.splits > 1) {
    const size_t need = avsg_attend_workspace_bytes(cache->batch, a->n_q, a->heads, a->topk);
    if (!d_workspace || !aligned(d_workspace, 256) || workspace_bytes < need)
      return fail(AVSG_E_INVAL, "the workspace must be 256-byte aligned and hold %zu bytes", need);
    p.part_out = static_cast<float*>(d_workspace);
    p.part_ml = reinterpret_cast<f32x2*>(p.part_out + static_cast<size_t>(tokens) * p.plan.splits * p.heads * kLatent);
  }
  return launched(launch_attend(p, cache->format, static_cast<hipStream_t>(stream)), "avsg_attend");
}

int64_t avsg_internal_attend_plan(int32_t format, int32_t batch, int32_t n_q, int32_t heads, int32_t topk) {
  const AttendPlan plan = attend_plan(format, batch, n_q, heads, topk);
  return static_cast<int64_t>(plan.kernel) | static_cast<int64_t>(plan.splits) << 32;
}

avsg_status avsg_mx4_quantize(const void* d_x, int32_t type, int64_t rows, int64_t cols, int64_t x_stride, void* d_codes,
                              void* d_scales, void* stream) {
  if (type != AVSG_BF16 && type != AVSG_F32) return fail(AVSG_E_INVAL, "unknown type %d", type);
  if (rows < 0 || cols < 0) return fail(AVSG_E_INVAL, "rows and cols must not be negative");
  if (cols % kMx4Block != 0) return fail(AVSG_E_RANGE, "cols must be a multiple of %d", kMx4Block);
  if (rows == 0 || cols == 0) return AVSG_OK;
  if (!d_x || !aligned(d_x, 16) || (x_stride & (type == AVSG_F32 ? 3 : 7)) != 0)
    return fail(AVSG_E_INVAL, "d_x and its rows must be 16-byte aligned");
  if (!d_codes || !aligned(d_codes, 16) || !d_scales) return fail(AVSG_E_INVAL, "d_codes (16-byte aligned) and d_scales are needed");
  if (cols > INT32_MAX || rows > kMostChunks / (cols / 8)) return fail(AVSG_E_RANGE, "rows * cols must be at most 2^35 - 2048");
  return launched(launch_mx4_quantize(d_x, type == AVSG_F32, rows, cols, x_stride, static_cast<uint8_t*>(d_codes),
                                      static_cast<uint8_t*>(d_scales), static_cast<hipStream_t>(stream)),
                  "avsg_mx4_quantize");
}

avsg_status avsg_mx4_dequantize(const avsg_mx4* x, int64_t rows, int64_t cols, void* d_out, int32_t type,
                                int64_t out_stride, void* stream) {
  if (type != AVSG_BF16 && type != AVSG_F32) return fail(AVSG_E_INVAL, "unknown type %d", type);
  if (rows < 0 || cols < 0) return fail(AVSG_E_INVAL, "rows and cols must not be negative");
  if (cols % kMx4Block != 0) return fail(AVSG_E_RANGE, "cols must be a multiple of %d", kMx4Block);
  if (rows == 0 || cols == 0) return AVSG_OK;
  if (!x || !x->d_codes || !x->d_scales) return fail(AVSG_E_INVAL, "null matrix, codes or scales");
  if (!aligned(x->d_codes, 16) || (x->code_stride & 15) != 0)
    return fail(AVSG_E_INVAL, "codes and their rows must be 16-byte aligned");
  if (!d_out || !aligned(d_out, 16) || (out_stride & (type == AVSG_F32 ? 3 : 7)) != 0)
    return fail(AVSG_E_INVAL, "d_out and its rows must be 16-byte aligned");
  if (cols > INT32_MAX || rows > kMostChunks / (cols / 8)) return fail(AVSG_E_RANGE, "rows * cols must be at most 2^35 - 2048");
  const Mx4View v{static_cast<const uint8_t*>(x->d_codes), static_cast<const uint8_t*>(x->d_scales), x->code_stride,
                  x->code_batch_stride, x->scale_stride, x->scale_batch_stride};
  return launched(launch_mx4_dequantize(v, rows, cols, d_out, type == AVSG_F32, out_stride,
                                        static_cast<hipStream_t>(stream)),
                  "avsg_mx4_dequantize");
}

avsg_status avsg_mx4_matmul(const avsg_mx4* a, const avsg_mx4* b, int32_t batch, int64_t m, int64_t n, int64_t k,
                            void* d_out, int32_t out_type, int64_t out_stride, int64_t out_batch_stride, void* stream) {
  if (out_type != AVSG_BF16 && out_type != AVSG_F32) return fail(AVSG_E_INVAL, "unknown out_type %d", out_type);
  if (batch < 0 || m < 0 || n < 0 || k < 0) return fail(AVSG_E_INVAL, "sizes must not be negative");
  if (k % kMx4Block != 0) return fail(AVSG_E_RANGE, "k must be a multiple of %d", kMx4Block);
  if (m > INT32_MAX / 2 || n > INT32_MAX / 2 || k > INT32_MAX / 2 || batch > 65535)
    return fail(AVSG_E_RANGE, "m, n and k must be below 2^30 and batch at most 65535");
  if ((m + 127) / 128 * ((n + 127) / 128) > kMostThreads / 256)
    return fail(AVSG_E_RANGE, "m x n must have fewer than 2^24 tiles of 128 x 128");
  if (batch == 0 || m == 0 || n == 0) return AVSG_OK;
  if (!d_out || !aligned(d_out, out_type == AVSG_F32 ? 4 : 2)) return fail(AVSG_E_INVAL, "d_out is null or misaligned");
  const avsg_mx4* both[2] = {a, b};
  Mx4View v[2];
  for (int i = 0; i < 2; ++i) {
    const avsg_mx4* x = both[i];
    if (!x || (k > 0 && (!x->d_codes || !x->d_scales))) return fail(AVSG_E_INVAL, "null matrix, codes or scales");
    if (!aligned(x->d_codes, 16) || (x->code_stride & 15) != 0 || (x->code_batch_stride & 15) != 0)
      return fail(AVSG_E_INVAL, "codes and their rows must be 16-byte aligned");
    v[i] = Mx4View{static_cast<const uint8_t*>(x->d_codes), static_cast<const uint8_t*>(x->d_scales), x->code_stride,
                   x->code_batch_stride, x->scale_stride, x->scale_batch_stride};
  }
  Mx4Product p{};
  p.a = v[0];
  p.b = v[1];
  p.batch = batch;
  p.m = static_cast<int32_t>(m);
  p.n = static_cast<int32_t>(n);
  p.k = static_cast<int32_t>(k);
  p.out = d_out;
  p.f32 = out_type == AVSG_F32;
  p.out_stride = out_stride;
  p.out_batch_stride = out_batch_stride;
  p.wide_stores = aligned(d_out, p.f32 ? 16 : 8) && (out_stride & 3) == 0 && (out_batch_stride & 3) == 0;
  return launched(launch_mx4_matmul(p, static_cast<hipStream_t>(stream)), "avsg_mx4_matmul");
}

}  // extern "C"
