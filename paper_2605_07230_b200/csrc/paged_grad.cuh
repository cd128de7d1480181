// What the kernels of the paged attention's gradient share: arguments, the rows and keys that belong together, and the gradient
// of one row or one key by one warp.
//
// With c the softmax scale, P_ij = exp(c q_i k_j - lse_i) where row i sees key j and 0 elsewhere, delta_i = <d_out_i, out_i>:
//     dV_j = sum_i P_ij d_out_i      dS_ij = P_ij (<d_out_i, v_j> - delta_i)      dQ_i = c sum_j dS_ij k_j      dK_j = c sum_i dS_ij q_i
// A key head's gradient sums over the query heads that read it: a row is (token, query head of the group), as in the forward pass.
// Queries' and keys' gradients come from two passes that both form P, so that no sum crosses blocks: seven products instead of
// five, but no atomics, no fp32 copy of dQ and the same bits every time.
#pragma once
#include "paged_attn.cuh"
#include "paged_range.h"

struct PagedGradArgs {
  PagedAttnArgs a;             // (a.out is read)
  const void* d_out;
  float2* stats;               // [n_tok,Hq]: lse (bf16: in units of ln 2) and delta
  void *dq, *dk, *dv;
  long long dq_stride, dk_stride, dv_stride;
  int n_kv;
  const int32_t* k_begin;
};

namespace paged {

// Request r with the row of dk, dv where its first key's gradient goes.
struct GradRequest : Request {
  int k0;
};
__device__ __forceinline__ bool load_request(const PagedGradArgs& p, int r, GradRequest* q) {
  bool ok = load_request(p.a, r, static_cast<Request*>(q));
  q->k0 = p.k_begin != nullptr ? p.k_begin[r] : q->q0;
  const bool fits = (p.k_begin != nullptr || q->kv == q->nq) && q->k0 >= 0 && (long long)q->k0 + q->kv <= p.n_kv;
  if (ok && !fits) {
    atomicOr(p.a.err, CASCADE_DEV_ERR_BAD_PAGE);
    ok = false;
  }
  return ok;
}

__device__ __forceinline__ bool sees(const PagedAttnArgs& a, int x, int j) {
  return j <= x && (a.window == 0 || j >= window_begin(x, a.window) || j < a.sinks);
}

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
  return x;
}
// exp(c s - lse) from what the element type's stats hold
template <typename E>
__device__ __forceinline__ float grad_weight(float s, float scale, float lse) {
  return sizeof(E) == 2 ? ptx::ex2(fmaf(s, scale * kLog2e, -lse)) : ptx::ex2(fmaf(s, scale, -lse) * kLog2e);
}
// Element offset of key j, -1 if its page lies outside the pool (reported).
__device__ __forceinline__ long long key_offset(const PagedAttnArgs& a, int r, int j, int kh, int D) {
  const int page = a.block_table[(size_t)r * a.table_stride + j / a.page_size];
  if (page < 0 || page >= a.n_pages) {
    atomicOr(a.err, CASCADE_DEV_ERR_BAD_PAGE);
    return -1;
  }
  return (long long)page * a.page_stride + ((long long)(j % a.page_size) * a.Hkv + kh) * D;
}

// One warp, one row and head, from the definition: only keys that the row sees are read.  Lane l holds elements l, l + 32, ..., of
// which those of groups e0 .. e1 - 1 are written.
template <typename E, int D>
__device__ void grad_row(const PagedGradArgs& p, int r, int row, int x, int head, int lane, int e0 = 0, int e1 = D / 32,
                         volatile uint64_t* alive = nullptr) {
  constexpr int kE = D / 32;
  const PagedAttnArgs& a = p.a;
  const int kh = head / (a.Hq / a.Hkv);
  const E* q = static_cast<const E*>(a.q) + (long long)row * a.q_stride + head * D;
  const E* g = static_cast<const E*>(p.d_out) + ((long long)row * a.Hq + head) * D;
  const float2 st = p.stats[(long long)row * a.Hq + head];
  float qv[kE], gv[kE], dq[kE];
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    qv[e] = load_elem(q + e * 32 + lane);
    gv[e] = load_elem(g + e * 32 + lane);
    dq[e] = 0.f;
  }
  const int lo = window_begin(x, a.window), n_sink = min(a.sinks, lo);
  const int n = x < 0 ? 0 : n_sink + (x - lo + 1);
  for (int i = 0; i < n; ++i) {
    if (alive != nullptr && i % 256 == 0) *alive = ptx::global_timer_ns();
    const long long off = key_offset(a, r, i < n_sink ? i : lo + (i - n_sink), kh, D);
    if (off < 0) continue;
    float s = 0.f, dp = 0.f, kv[kE];
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      kv[e] = load_elem(static_cast<const E*>(a.k) + off + e * 32 + lane);
      s = fmaf(qv[e], kv[e], s);
      dp = fmaf(gv[e], load_elem(static_cast<const E*>(a.v) + off + e * 32 + lane), dp);
    }
    const float ds = grad_weight<E>(warp_sum(s), a.scale, st.x) * (warp_sum(dp) - st.y);
#pragma unroll
    for (int e = 0; e < kE; ++e) dq[e] = fmaf(ds, kv[e], dq[e]);
  }
  E* to = static_cast<E*>(p.dq) + (long long)row * p.dq_stride + head * D;
#pragma unroll
  for (int e = 0; e < kE; ++e)
    if (e >= e0 && e < e1) store_elem(to + e * 32 + lane, a.scale * dq[e]);
}

// One warp, one key and key head, from the definition: only rows that see the key are read.  kDk, kDv: which gradients to write.
template <typename E, int D, bool kDk = true, bool kDv = true>
__device__ void grad_key(const PagedGradArgs& p, int r, const GradRequest& rq, int j, int kh, int lane, volatile uint64_t* alive = nullptr) {
  constexpr int kE = D / 32;
  const PagedAttnArgs& a = p.a;
  const int G = a.Hq / a.Hkv, x0 = rq.kv - rq.nq;
  const long long off = key_offset(a, r, j, kh, D);
  float kv[kE], vv[kE], dk[kE], dv[kE];
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    kv[e] = off < 0 ? 0.f : load_elem(static_cast<const E*>(a.k) + off + e * 32 + lane);
    vv[e] = off < 0 ? 0.f : load_elem(static_cast<const E*>(a.v) + off + e * 32 + lane);
    dk[e] = dv[e] = 0.f;
  }
  int lo, hi;
  tokens_that_see(a, x0, rq.nq, j, j, &lo, &hi);
  if (off < 0) hi = lo;
  for (int t = lo; t < hi; ++t) {
    if (alive != nullptr && t % 64 == 0) *alive = ptx::global_timer_ns();
    if (!sees(a, x0 + t, j)) continue;
    for (int g = 0; g < G; ++g) {
      const int row = rq.q0 + t, head = kh * G + g;
      const float2 st = p.stats[(long long)row * a.Hq + head];
      float s = 0.f, dp = 0.f, qv[kE], gv[kE];
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        qv[e] = load_elem(static_cast<const E*>(a.q) + (long long)row * a.q_stride + head * D + e * 32 + lane);
        gv[e] = load_elem(static_cast<const E*>(p.d_out) + ((long long)row * a.Hq + head) * D + e * 32 + lane);
        s = fmaf(qv[e], kv[e], s);
        dp = fmaf(gv[e], vv[e], dp);
      }
      const float w = grad_weight<E>(warp_sum(s), a.scale, st.x), ds = w * (warp_sum(dp) - st.y);
#pragma unroll
      for (int e = 0; e < kE; ++e) {
        dk[e] = fmaf(ds, qv[e], dk[e]);
        dv[e] = fmaf(w, gv[e], dv[e]);
      }
    }
  }
  const long long to = (long long)rq.k0 + j;
#pragma unroll
  for (int e = 0; e < kE; ++e) {
    if (kDk) store_elem(static_cast<E*>(p.dk) + to * p.dk_stride + kh * D + e * 32 + lane, a.scale * dk[e]);
    if (kDv) store_elem(static_cast<E*>(p.dv) + to * p.dv_stride + kh * D + e * 32 + lane, dv[e]);
  }
}

}  // namespace paged

// paged_grad_f32.cu: the fp32 type, three bf16 parts a number.
int launch_paged_grad_f32(cascade_ctx* ctx, const PagedGradArgs& p, cudaStream_t s);
