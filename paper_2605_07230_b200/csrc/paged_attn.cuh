// What the paged-attention kernels share: arguments, the visibility rule, and the attention of one row by one warp.
#pragma once
#include "cascade_internal.h"
#include "ptx_paged.cuh"

struct PagedAttnArgs {
  int n_req, n_tok, Hq, Hkv, page_size, n_pages, table_stride, table_width, max_q, max_kv, window, sinks;
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
                  kv <= (long long)a.table_width * a.page_size;
  if (!ok) atomicOr(a.err, CASCADE_DEV_ERR_BAD_PAGE);
  return ok;
}

// First key of the window of position x; a row sees [0, min(sinks, lo)) and [lo, x].
__device__ __forceinline__ int window_begin(int x, int window) { return window == 0 || x < window ? 0 : x - window + 1; }

__device__ __forceinline__ float load_elem(const float* p) { return *p; }
__device__ __forceinline__ float load_elem(const __nv_bfloat16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void store_elem(float* p, float v) { *p = v; }
__device__ __forceinline__ void store_elem(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }

// One warp, one row and head, from the definition: only keys that the row sees are read, so that nothing else can reach
// the result.  Lane l holds elements l, l + 32, ...; fp32 throughout.  *alive takes the global timer
// every 256 keys.
template <typename E, int D>
__device__ void attend_row(const PagedAttnArgs& a, int r, int row, int x, int head, int lane,
                           volatile uint64_t* alive = nullptr) {
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
  bool met = false;                              // a key, whatever its score
  const float c = a.scale * kLog2e;
  for (int i = 0; i < n; ++i) {
    if (alive != nullptr && i % 256 == 0) *alive = ptx::global_timer_ns();
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
    met = true;
    const float m_new = fmaxf(m, s);
    // (a score of -inf weighs nothing, the first ones too, whose reference is not finite yet)
    const float corr = m == m_new ? 1.f : exp2f(m - m_new), p = s == -INFINITY ? 0.f : exp2f(s - m_new);
    l = l * corr + p;
#pragma unroll
    for (int e = 0; e < kE; ++e) o[e] = o[e] * corr + p * vv[e];
    m = m_new;
  }
  if (met && m == -INFINITY) l = NAN;            // all scores -inf, or no numbers: 0 / 0
  const float inv = l == 0.f ? 0.f : 1.f / l;
  E* out = static_cast<E*>(a.out) + ((long long)row * a.Hq + head) * D;
#pragma unroll
  for (int e = 0; e < kE; ++e) store_elem(out + e * 32 + lane, l == 0.f ? 0.f : o[e] * inv);
  if (a.lse != nullptr && lane == 0) a.lse[(long long)row * a.Hq + head] = l == 0.f ? -INFINITY : m * kLn2 + logf(l);
}

// key / page_size by a multiplication, for keys below 2^31.
struct PageDiv {
  uint32_t mul;
  int shift;
  __device__ __forceinline__ int page(int key) const { return (int)(((unsigned long long)(uint32_t)key * mul) >> shift); }
};
inline PageDiv page_div(int page_size) {
  int lg = 0;
  while ((1ll << lg) < page_size) ++lg;
  return {(uint32_t)(((1ull << (31 + lg)) + (unsigned)page_size - 1) / (unsigned)page_size), 31 + lg};
}

__device__ __forceinline__ uint4 ld_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.L2::256B.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}

// Partial results of kernels whose splits are the CTAs of a cluster: [part][row][part_stride] floats in shared memory, a row
// being D un-normalised outputs, the reference (log2 units) and the sum of weights.
__host__ __device__ constexpr int part_stride(int D) { return D + 4; }

__device__ __forceinline__ void store4(float* p, const float4& v) { *reinterpret_cast<float4*>(p) = v; }
__device__ __forceinline__ void store4(__nv_bfloat16* p, const float4& v) {
  *reinterpret_cast<uint2*>(p) = make_uint2(ptx::pack_bf16x2(v.x, v.y), ptx::pack_bf16x2(v.z, v.w));
}

// Floats of shared memory for `rows` rows: the parts' results, then what the cluster's CTAs send each other.
__host__ __device__ constexpr int part_floats(int D, int parts, int rows) { return (parts * rows + rows + 8) * part_stride(D); }

// Ends such a kernel: merges the CTA's `kParts` partial results of rows row0 .. row0 + rows - 1 (row = token * G + query head
// of the group; x0 = position of the request's first new token) and sends every row to the CTA of the cluster that finishes
// it (row % splits), which stores outputs and lse and computes a row whose result is not finite, or whose sum is no number
// because a page was not there, again from the keys it sees alone.  max_rows: rows per part in s_part (part_floats(D, kParts, max_rows) floats), at most kMaxRows (<= 32).  splits <= 8.
// Every thread of every CTA of the cluster calls it, having arrived at the cluster's barrier (splits > 1) without waiting,
// with the partial results written but no barrier behind them yet.
template <typename E, int D, int kParts, int kMaxRows>
__device__ __forceinline__ void merge_and_store(const PagedAttnArgs& a, int r, int q0, int x0, int kh, int row0, int rows, int G, int splits,
                                                float* s_part, int max_rows) {
  constexpr int kX = part_stride(D), kMost = 8;
  static_assert(kMaxRows <= 32 && kParts <= kMost, "row bits, weights");
  __shared__ uint32_t s_odd;
  const int threads = (int)blockDim.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  float* s_in = s_part + kParts * max_rows * kX;   // [row / splits][split][kX]
  if (tid == 0) s_odd = 0u;
  __syncthreads();
  // four columns of a row from its parts, `stride` floats apart
  auto merge = [&](const float* part, int stride, int count, int col, float* ref, float* sum) {
    float m = -INFINITY, total = 0.f;
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int s = 0; s < count; ++s) m = fmaxf(m, part[s * stride + D]);
#pragma unroll 2
    for (int s = 0; s < count; ++s) {
      const float ms = part[s * stride + D], w = ms == -INFINITY ? 0.f : ptx::ex2(ms - m);
      const float4 v = *reinterpret_cast<const float4*>(part + s * stride + col);
      total += w * part[s * stride + D + 1];       // (a NaN sum stays one)
      // a part of weight 0 met nothing of the row: what it holds is 0, or NaN by a value nobody saw
      acc.x += w == 0.f ? 0.f : w * v.x;
      acc.y += w == 0.f ? 0.f : w * v.y;
      acc.z += w == 0.f ? 0.f : w * v.z;
      acc.w += w == 0.f ? 0.f : w * v.w;
    }
    *ref = m;
    *sum = total;
    return acc;
  };
  auto finish = [&](int row, int col, const float4& acc, float ref, float sum) {
    const int q_row = row0 + row, x = x0 + q_row / G;
    const long long at = (long long)(q0 + q_row / G) * a.Hq + kh * G + q_row % G;
    const float inv = x < 0 ? 0.f : 1.f / sum;
    const float4 v = x < 0 ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(acc.x * inv, acc.y * inv, acc.z * inv, acc.w * inv);
    store4(static_cast<E*>(a.out) + at * D + col, v);
    if (col == 0 && a.lse != nullptr) a.lse[at] = x < 0 ? -INFINITY : (ref + log2f(sum)) * kLn2;
    const float bad = v.x * 0.f + v.y * 0.f + v.z * 0.f + v.w * 0.f;   // NaN if any is not finite
    if (x >= 0 && (bad != 0.f || !(sum > 0.f))) atomicOr(&s_odd, 1u << row);
  };
  const int rank = splits == 1 ? 0 : (int)ptx::cluster_ctarank();
  const uint32_t in = ptx::smem_u32(s_in);
  if (splits > 1) ptx::cluster_wait();             // the others have started: their shared memory may be written
  for (int i = tid; i < rows * (D / 4); i += threads) {
    const int row = i / (D / 4), col = i % (D / 4) * 4;
    float ref, sum;
    const float4 acc = merge(s_part + row * kX, max_rows * kX, kParts, col, &ref, &sum);
    if (splits == 1) {
      finish(row, col, acc, ref, sum);
    } else {
      const uint32_t to = ptx::map_to_cta(in + (uint32_t)((row / splits * splits + rank) * kX) * 4u, (uint32_t)(row % splits));
      ptx::st_cluster_v4(to + col * 4u, acc);
      if (col == 0) {
        ptx::st_cluster_f32(to + D * 4u, ref);
        ptx::st_cluster_f32(to + D * 4u + 4u, sum);
      }
    }
  }
  if (splits > 1) {
    __syncwarp();
    ptx::cluster_arrive();
    ptx::cluster_wait();                           // all rows of this CTA are here
    const int mine = rows > rank ? (rows - rank + splits - 1) / splits : 0;
    for (int i = tid; i < mine * (D / 4); i += threads) {
      const int row = rank + i / (D / 4) * splits, col = i % (D / 4) * 4;
      float ref, sum;
      const float4 acc = merge(s_in + row / splits * splits * kX, kX, splits, col, &ref, &sum);
      finish(row, col, acc, ref, sum);
    }
  }
  __syncthreads();
  for (uint32_t left = s_odd; left != 0u; left &= left - 1u) {         // (only where rows were finished)
    const int row = __ffs(left) - 1, q_row = row0 + row;
    if (row % (threads / 32) == warp) attend_row<E, D>(a, r, q0 + q_row / G, x0 + q_row / G, kh * G + q_row % G, lane);
  }
}

}  // namespace paged

// paged_attn_tc.cu: row blocks on the tensor cores (bf16).
int launch_paged_attn_tc(cascade_ctx* ctx, const PagedAttnArgs& a, cudaStream_t s);
// paged_attn_rows.cu: at most 16 rows a key head, warp-level products straight from memory (bf16).
bool paged_attn_rows_takes(const PagedAttnArgs& a);
int launch_paged_attn_rows(cascade_ctx* ctx, const PagedAttnArgs& a, cudaStream_t s);
// paged_attn_f32.cu: the fp32 type.
int launch_paged_attn_f32(cascade_ctx* ctx, const PagedAttnArgs& a, cudaStream_t s);
