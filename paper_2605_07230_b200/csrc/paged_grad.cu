// The gradient of the attention over a paged cache: checks, the rows' statistics, and the choice of kernels.
#include <climits>

#include "overlap.h"
#include "paged.h"
#include "paged_grad_tc.cuh"

namespace {

using cascade_detail::Rows;

constexpr int kMaxGroup = 128;               // query heads a key head: they share a row block
constexpr int kMaxKeys = INT32_MAX - 65535;  // so that a key's index rounded up to a tile stays in 32 bits
constexpr int64_t kMostStride = 1ll << 40;
constexpr int kThreads = 256;

// stats[row,head] = (lse, sum_d d_out * out), the log-sum-exp in units of ln 2 for the 16-bit type: 16 bytes a lane.
template <typename E, int D>
__global__ void __launch_bounds__(kThreads) k_paged_grad_stats(const PagedGradArgs p, const float* __restrict__ lse) {
  constexpr int kVec = 16 / (int)sizeof(E), kLanes = D / kVec;       // lanes a row
  const long long rows = (long long)max(0, min(p.a.n_tok, p.a.q_begin[p.a.n_req])) * p.a.Hq;
  const long long step = (long long)gridDim.x * (kThreads / kLanes);
  const int lane = threadIdx.x % kLanes;
  for (long long row = (long long)blockIdx.x * (kThreads / kLanes) + threadIdx.x / kLanes; row - threadIdx.x / kLanes < rows; row += step) {
    float sum = 0.f;
    if (row < rows) {
      const E *o = static_cast<const E*>(p.a.out) + row * D + lane * kVec, *g = static_cast<const E*>(p.d_out) + row * D + lane * kVec;
      const uint4 x = *reinterpret_cast<const uint4*>(o), y = *reinterpret_cast<const uint4*>(g);
      const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (sizeof(E) == 4) {
          sum = fmaf(__uint_as_float(xs[i]), __uint_as_float(ys[i]), sum);
        } else {
          sum = fmaf(__uint_as_float(xs[i] << 16), __uint_as_float(ys[i] << 16), sum);
          sum = fmaf(__uint_as_float(xs[i] & 0xffff0000u), __uint_as_float(ys[i] & 0xffff0000u), sum);
        }
      }
    }
#pragma unroll
    for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (row < rows && lane == 0) p.stats[row] = make_float2(sizeof(E) == 2 ? lse[row] * paged::kLog2e : lse[row], sum);
  }
}

template <typename E, int D>
int launch_stats(cascade_ctx* ctx, const PagedGradArgs& p, const float* lse, cudaStream_t s) {
  constexpr int kRows = kThreads * 16 / (D * (int)sizeof(E));        // rows a block takes at once
  const long long blocks = ((long long)p.a.n_tok * p.a.Hq + kRows - 1) / kRows, most = 16ll * ctx->sm_count;
  KernelScope ks(ctx, K_PAGED_GRAD_STATS, s);
  k_paged_grad_stats<E, D><<<(unsigned)(blocks < most ? blocks : most), kThreads, 0, s>>>(p, lse);
  CASCADE_CUDA_TRY(cudaGetLastError());
  return CASCADE_OK;
}

}  // namespace

extern "C" int cascade_paged_attn_grad(cascade_ctx* ctx, const cascade_paged_cache* cache, int32_t n_req, int32_t n_tok, const void* q,
                                       int64_t q_stride, const int32_t* q_begin, const int32_t* kv_len, int32_t max_q, int32_t max_kv,
                                       int32_t window, int32_t sinks, float softmax_scale, const void* out, const float* lse,
                                       const void* d_out, float* scratch, void* dq, int64_t dq_stride, void* dk, int64_t dk_stride,
                                       void* dv, int64_t dv_stride, int32_t n_kv, const int32_t* k_begin, void* stream) {
  if (ctx == nullptr || q == nullptr || q_begin == nullptr || kv_len == nullptr || out == nullptr || lse == nullptr || d_out == nullptr ||
      scratch == nullptr || dq == nullptr || dk == nullptr || dv == nullptr)
    return CASCADE_ERR_INVALID_ARG;
  CASCADE_TRY(check_paged_cache(ctx, cache));
  const cascade_shape& sh = ctx->shape;
  const int64_t es = sh.dtype == CASCADE_BF16 ? 2 : 4, q_row = (int64_t)sh.Hq * sh.D, kv_row = (int64_t)sh.Hkv * sh.D;
  if (cache->block_table == nullptr || cache->table_stride < 1) return CASCADE_ERR_INVALID_ARG;
  if (cache->table_width < 0 || cache->table_width > cache->table_stride) return CASCADE_ERR_INVALID_ARG;
  if (n_req < 1 || n_tok < 1 || n_kv < 1 || max_q < 1 || max_kv < 0 || window < 0 || sinks < 0) return CASCADE_ERR_INVALID_ARG;
  if (!(softmax_scale > 0.f) || softmax_scale > 3e38f) return CASCADE_ERR_INVALID_ARG;
  for (const int64_t stride : {q_stride, dq_stride, dk_stride, dv_stride})
    if (stride * es % 16 != 0 || stride > kMostStride) return CASCADE_ERR_INVALID_ARG;
  if (q_stride < q_row || dq_stride < q_row || dk_stride < kv_row || dv_stride < kv_row) return CASCADE_ERR_INVALID_ARG;
  for (const void* x : {q, out, d_out, (const void*)scratch, (const void*)dq, (const void*)dk, (const void*)dv})
    if ((reinterpret_cast<uintptr_t>(x) & 15u) != 0) return CASCADE_ERR_INVALID_ARG;
  if (!aligned4(q_begin, kv_len, cache->block_table, k_begin) || !aligned4(lse)) return CASCADE_ERR_INVALID_ARG;
  if (max_kv > kMaxKeys || n_req > CASCADE_MAX_REQUESTS || sh.Hq / sh.Hkv > kMaxGroup) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  max_q = max_q < n_tok ? max_q : n_tok;
  if ((int64_t)max_q * (sh.Hq / sh.Hkv) > kMaxKeys) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  const Rows outputs[] = {{dq, n_tok, dq_stride * es, q_row * es}, {dk, n_kv, dk_stride * es, kv_row * es},
                          {dv, n_kv, dv_stride * es, kv_row * es}, {scratch, 1, 1, (int64_t)n_tok * sh.Hq * 8}};
  const int64_t pool = ((int64_t)(cache->n_pages - 1) * cache->page_stride + (int64_t)cache->page_size * kv_row) * es;
  const Rows inputs[] = {{q, n_tok, q_stride * es, q_row * es}, {out, 1, 1, n_tok * q_row * es}, {d_out, 1, 1, n_tok * q_row * es},
                         {lse, 1, 1, (int64_t)n_tok * sh.Hq * 4}, {cache->k_pages, 1, 1, pool}, {cache->v_pages, 1, 1, pool},
                         {cache->block_table, n_req, (int64_t)cache->table_stride * 4, (int64_t)cache->table_stride * 4},
                         {q_begin, 1, 1, (n_req + 1ll) * 4}, {kv_len, 1, 1, n_req * 4ll}, {k_begin, k_begin != nullptr, 1, n_req * 4ll}};
  for (int i = 0; i < 4; ++i) {
    for (const Rows& x : inputs)
      if (meet(outputs[i], x)) return CASCADE_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (meet(outputs[i], outputs[j])) return CASCADE_ERR_INVALID_ARG;
  }
  CASCADE_TRY(check_current_device(ctx));
  PagedGradArgs p;
  PagedAttnArgs& a = p.a;
  a.n_req = n_req;
  a.n_tok = n_tok;
  a.Hq = sh.Hq;
  a.Hkv = sh.Hkv;
  a.page_size = cache->page_size;
  a.n_pages = cache->n_pages;
  a.table_stride = cache->table_stride;
  a.table_width = cache->table_width == 0 ? cache->table_stride : cache->table_width;
  a.max_q = max_q;
  a.max_kv = max_kv;
  a.window = window;
  a.sinks = sinks;
  a.page_stride = cache->page_stride;
  a.q_stride = q_stride;
  a.q = q;
  a.k = cache->k_pages;
  a.v = cache->v_pages;
  a.out = const_cast<void*>(out);
  a.lse = nullptr;
  a.q_begin = q_begin;
  a.kv_len = kv_len;
  a.block_table = cache->block_table;
  a.scale = softmax_scale;
  a.err = ctx->dev_error;
  a.wait_ns = ctx->wait_limit_ns;
  p.d_out = d_out;
  p.stats = reinterpret_cast<float2*>(scratch);
  p.dq = dq;
  p.dk = dk;
  p.dv = dv;
  p.dq_stride = dq_stride;
  p.dk_stride = dk_stride;
  p.dv_stride = dv_stride;
  p.n_kv = n_kv;
  p.k_begin = k_begin;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  ctx->launches = 0;
  const bool wide = sh.D == 128;
  int status;
  if (sh.dtype == CASCADE_BF16)
    status = wide ? launch_stats<__nv_bfloat16, 128>(ctx, p, lse, s) : launch_stats<__nv_bfloat16, 64>(ctx, p, lse, s);
  else
    status = wide ? launch_stats<float, 128>(ctx, p, lse, s) : launch_stats<float, 64>(ctx, p, lse, s);
  CASCADE_TRY(status);
  return sh.dtype == CASCADE_BF16 ? launch_paged_grad_tc(ctx, p, s) : launch_paged_grad_f32(ctx, p, s);
}
