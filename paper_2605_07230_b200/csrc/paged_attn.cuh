// What the paged-attention kernels share: arguments, the visibility rule, and the attention of one row by one warp.
#pragma once
#include "cascade_internal.h"
#include "ptx.cuh"

struct PagedAttnArgs {
  int n_req, n_tok, Hq, Hkv, page_size, n_pages, table_stride, max_q, max_kv, window, sinks;
  long long page_stride, q_stride;
  const void *q, *k, *v;
  void* out;
  float* lse;
  const int32_t *q_begin, *kv_len, *block_table;
  float scale;
  int* err;
  unsigned long long wait_ns;
};

namespace paged {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// Request r: its first row, row count and key count.  False (and the error word) if they break the call's bounds.
struct Request {
  int q0, nq, kv;
};
__device__ __forceinline__ bool load_request(const PagedAttnArgs& a, int r, Request* q) {
  const int b = a.q_begin[r], e = a.q_begin[r + 1], kv = a.kv_len[r];
  q->q0 = b;
  q->nq = e - b;
  q->kv = kv;
  const bool ok = b >= 0 && e >= b && e <= a.n_tok && e - b <= a.max_q && kv >= 0 && kv <= a.max_kv &&
                  kv <= (long long)a.table_stride * a.page_size;
  if (!ok) atomicOr(a.err, CASCADE_DEV_ERR_BAD_PAGE);
  return ok;
}

// First key of the window of position x; a row sees [0, min(sinks, lo)) and [lo, x].
__device__ __forceinline__ int window_begin(int x, int window) { return window == 0 ? 0 : max(0, x - window + 1); }

__device__ __forceinline__ float load_elem(const float* p) { return *p; }
__device__ __forceinline__ float load_elem(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_elem(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_elem(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }

// One warp, one row and head, from the definition: only keys that the row sees are read, so that nothing else can reach
// the result.  Lane l holds elements l, l + 32, ...; fp32 throughout.
template <typename E, int D>
__device__ void attend_row(const PagedAttnArgs& a, int r, int row, int x, int head, int lane) {
  constexpr int kE = D / 32;
  const int kh = head / (a.Hq / a.Hkv);
  const E* q = static_cast<const E*>(a.q) + (long long)row * a.q_stride + head * D;
  float qv[kE], o[kE];
#pragma unroll
  for (int i = 0; i < kE; ++i) {
    qv[i] = load_elem(q + i * 32 + lane);
    o[i] = 0.f;
  }
  const int lo = window_begin(x, a.window), n_sink = min(a.sinks, lo);
  const int n = x < 0 ? 0 : n_sink + (x - lo + 1);
  float m = -INFINITY, l = 0.f;
  const float c = a.scale * kLog2e;
  for (int i = 0; i < n; ++i) {
    const int j = i < n_sink ? i : lo + (i - n_sink);
    const int page = a.block_table[(size_t)r * a.table_stride + j / a.page_size];
    if (page < 0 || page >= a.n_pages) {
      if (lane == 0) atomicOr(a.err, CASCADE_DEV_ERR_BAD_PAGE);
      continue;
    }
    const long long off = (long long)page * a.page_stride + ((long long)(j % a.page_size) * a.Hkv + kh) * D;
    const E* kp = static_cast<const E*>(a.k) + off;
    const E* vp = static_cast<const E*>(a.v) + off;
    float s = 0.f, vv[kE];
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      s = fmaf(qv[e], load_elem(kp + e * 32 + lane), s);
      vv[e] = load_elem(vp + e * 32 + lane);
    }
#pragma unroll
    for (int w = 16; w > 0; w >>= 1) s += __shfl_xor_sync(0xffffffffu, s, w);
    s *= c;
    const float m_new = fmaxf(m, s);
    const float corr = m == m_new ? 1.f : exp2f(m - m_new), p = exp2f(s - m_new);
    l = l * corr + p;
#pragma unroll
    for (int e = 0; e < kE; ++e) o[e] = o[e] * corr + p * vv[e];
    m = m_new;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  E* out = static_cast<E*>(a.out) + ((long long)row * a.Hq + head) * D;
#pragma unroll
  for (int e = 0; e < kE; ++e) store_elem(out + e * 32 + lane, l == 0.f ? 0.f : o[e] * inv);
  if (a.lse != nullptr && lane == 0) a.lse[(long long)row * a.Hq + head] = l == 0.f ? -INFINITY : m * kLn2 + logf(l);
}

}  // namespace paged

// paged_attn_tc.cu: row blocks on the tensor cores (bf16).  `takes`: the group of query heads fits into a block.
bool paged_attn_tc_takes(const PagedAttnArgs& a);
int launch_paged_attn_tc(cascade_ctx* ctx, const PagedAttnArgs& a, cudaStream_t s);
// paged_attn_rows.cu: at most 16 rows a key head, warp-level products straight from memory (bf16).
bool paged_attn_rows_takes(const PagedAttnArgs& a);
int launch_paged_attn_rows(cascade_ctx* ctx, const PagedAttnArgs& a, cudaStream_t s);
