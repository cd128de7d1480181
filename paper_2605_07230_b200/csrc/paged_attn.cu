// Causal attention of every request's new tokens over its paged cache: checks and the choice of a kernel.
#include "paged.h"
#include "paged_attn.cuh"

constexpr int kMaxGroup = 128;  // query heads a key head: they share a row block
constexpr int kMaxKeys = INT32_MAX - 65535;  // so that a key's index rounded up to a tile stays in 32 bits

// Whether [out, out + out_bytes) meets one of `rows` rows of `width` bytes that start `stride` bytes apart.
static bool meets_rows(const void* rows_at, int64_t rows, int64_t stride, int64_t width, const void* out, int64_t out_bytes) {
  const int64_t d = (int64_t)(reinterpret_cast<uintptr_t>(out) - reinterpret_cast<uintptr_t>(rows_at));
  const int64_t first = d < width ? 0 : (d - width) / stride + 1;   // the first row that ends behind where `out` starts
  return first < rows && first * stride < d + out_bytes;
}

extern "C" int cascade_paged_attn(cascade_ctx* ctx, const cascade_paged_cache* cache, int32_t n_req, int32_t n_tok,
                                  const void* q, int64_t q_stride, const int32_t* q_begin, const int32_t* kv_len,
                                  int32_t max_q, int32_t max_kv, int32_t window, int32_t sinks, float softmax_scale,
                                  void* out, float* lse, void* stream) {
  if (ctx == nullptr || q == nullptr || q_begin == nullptr || kv_len == nullptr || out == nullptr) return CASCADE_ERR_INVALID_ARG;
  CASCADE_TRY(check_paged_cache(ctx, cache));
  const cascade_shape& sh = ctx->shape;
  const int es = sh.dtype == CASCADE_BF16 ? 2 : 4;
  if (cache->block_table == nullptr || cache->table_stride < 1) return CASCADE_ERR_INVALID_ARG;
  if (cache->table_width < 0 || cache->table_width > cache->table_stride) return CASCADE_ERR_INVALID_ARG;
  if (n_req < 1 || n_tok < 1 || max_q < 1 || max_kv < 0 || window < 0 || sinks < 0) return CASCADE_ERR_INVALID_ARG;
  if (!(softmax_scale > 0.f) || softmax_scale > 3e38f) return CASCADE_ERR_INVALID_ARG;
  if (q_stride < (int64_t)sh.Hq * sh.D || q_stride * es % 16 != 0) return CASCADE_ERR_INVALID_ARG;
  if (((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out)) & 15u) != 0 ||
      !aligned4(q_begin, kv_len, cache->block_table, lse))
    return CASCADE_ERR_INVALID_ARG;
  if (max_kv > kMaxKeys) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  if (n_req > CASCADE_MAX_REQUESTS || sh.Hq / sh.Hkv > kMaxGroup) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  if (meets_rows(q, n_tok, q_stride * es, (int64_t)sh.Hq * sh.D * es, out, (int64_t)n_tok * sh.Hq * sh.D * es))
    return CASCADE_ERR_INVALID_ARG;
  CASCADE_TRY(check_current_device(ctx));
  PagedAttnArgs a;
  a.n_req = n_req;
  a.n_tok = n_tok;
  a.Hq = sh.Hq;
  a.Hkv = sh.Hkv;
  a.page_size = cache->page_size;
  a.n_pages = cache->n_pages;
  a.table_stride = cache->table_stride;
  a.table_width = cache->table_width == 0 ? cache->table_stride : cache->table_width;
  a.max_q = max_q < n_tok ? max_q : n_tok;
  a.max_kv = max_kv;
  a.window = window;
  a.sinks = sinks;
  a.page_stride = cache->page_stride;
  a.q_stride = q_stride;
  a.q = q;
  a.k = cache->k_pages;
  a.v = cache->v_pages;
  a.out = out;
  a.lse = lse;
  a.q_begin = q_begin;
  a.kv_len = kv_len;
  a.block_table = cache->block_table;
  a.scale = softmax_scale;
  a.err = ctx->dev_error;
  a.wait_ns = ctx->wait_limit_ns;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  ctx->launches = 0;
  KernelScope ks(ctx, K_PAGED_ATTN, s);
  if (sh.dtype == CASCADE_BF16) return paged_attn_rows_takes(a) ? launch_paged_attn_rows(ctx, a, s) : launch_paged_attn_tc(ctx, a, s);
  return launch_paged_attn_f32(ctx, a, s);
}
