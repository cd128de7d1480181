// The paged KV cache's bookkeeping and its writer: block tables, slot map and free-page stack of the next pass from the
// requests' lengths, and rotary embedding + cache write of a pass's keys and values (queries rotated beside them).
#include <climits>
#include <cmath>
#include <cstring>

#include "cascade_internal.h"
#include "paged.h"
#include "paged_attn.cuh"
#include "ptx.cuh"

namespace {

constexpr int kTabThreads = 1024;
constexpr int kTabWarps = kTabThreads / 32;
static_assert(kTabWarps == 32, "one lane per warp in the scan of the warps' sums");
constexpr int kPerThread = CASCADE_MAX_REQUESTS / kTabThreads;  // requests per thread of the scan

struct TablesArgs {
  int n_req, n_tok, page_size, n_pages, table_stride;
  const int32_t *new_len, *kv_len, *free_count;
  int32_t *block_table, *free_pages, *kv_len_out, *free_count_out, *q_begin, *slot, *pos;
  int* err;
  paged::PageDiv div;
  // pages that n tokens fill (n >= 0)
  __device__ __forceinline__ int pages(int n) const { return n == 0 ? 0 : div.page(n - 1) + 1; }
};

// One cluster does the whole job.  Every CTA scans all requests (three exclusive sums: new tokens, pages needed, pages
// given back; a few kilobytes of lengths, cheaper to scan eight times than to exchange), all CTAs share the writes.  The
// cluster barrier parts the reads of what is updated in place (lengths, count, free list) and the pushes onto the free
// list from everything that is written or popped afterwards.  Latency-bound: 14.4 us for 512
// requests with about 110 thousand new tokens (1 MB), 5 us for two with one each (graph replays).
__global__ void __launch_bounds__(kTabThreads) k_paged_tables(const TablesArgs a) {
  extern __shared__ int smem[];
  int* s_q = smem;                     // [n_req + 1] exclusive sums of the new tokens
  int* s_need = s_q + a.n_req + 1;     // [n_req] exclusive sums of the pages needed
  int* s_back = s_need + a.n_req;      // [n_req] exclusive sums of the pages given back
  int* s_kv = s_back + a.n_req;        // [n_req] tokens held; -1 - tokens for a finished request
  __shared__ long long s_warp[3][kTabWarps];
  __shared__ int s_bad;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = (int)ptx::cluster_ctarank(), n_cta = (int)ptx::cluster_nctarank();
  const int P = a.page_size;
  const long long cap = min((long long)a.table_stride * P, (long long)INT_MAX);   // (a pool holds fewer tokens than 2^31)
  const int count = *a.free_count;
  if (tid == 0) s_bad = 0;
  __syncthreads();

  // each thread owns consecutive requests
  long long sum[3] = {0, 0, 0};
  int add[kPerThread], need[kPerThread], back[kPerThread];
  bool bad = count < 0 || count > a.n_pages;
  const int per = (a.n_req + kTabThreads - 1) / kTabThreads;
#pragma unroll
  for (int k = 0; k < kPerThread; ++k) {
    const int r = tid * per + k;
    add[k] = need[k] = back[k] = 0;
    if (k < per && r < a.n_req) {
      const int n = a.new_len[r], kv = a.kv_len[r];
      s_kv[r] = n < 0 ? -1 - kv : kv;
      if (kv < 0 || (long long)kv + (n > 0 ? n : 0) > cap) {
        bad = true;
      } else {
        const int had = a.pages(kv);
        if (n < 0) {
          back[k] = had;
        } else {
          add[k] = n;
          need[k] = a.pages(kv + n) - had;
        }
      }
      sum[0] += add[k];
      sum[1] += need[k];
      sum[2] += back[k];
    }
  }
  long long inc[3] = {sum[0], sum[1], sum[2]};
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      const long long t = __shfl_up_sync(0xffffffffu, inc[i], o);
      if (lane >= o) inc[i] += t;
    }
  }
  if (lane == 31)
    for (int i = 0; i < 3; ++i) s_warp[i][warp] = inc[i];
  if (bad) s_bad = 1;
  __syncthreads();
  long long total[3], run[3];
#pragma unroll
  for (int i = 0; i < 3; ++i) {   // every warp scans the warps' sums for itself
    const long long v = s_warp[i][lane];
    long long c = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long t = __shfl_up_sync(0xffffffffu, c, o);
      if (lane >= o) c += t;
    }
    total[i] = __shfl_sync(0xffffffffu, c, 31);
    run[i] = __shfl_sync(0xffffffffu, c - v, warp) + inc[i] - sum[i];
  }
  const long long count1 = (long long)count + total[2];
  const bool ok = s_bad == 0 && total[0] <= a.n_tok && count1 <= a.n_pages && total[1] <= count1;  // the same in every CTA
#pragma unroll
  for (int k = 0; k < kPerThread; ++k) {
    const int r = tid * per + k;
    if (k < per && r < a.n_req) {
      s_q[r] = ok ? (int)run[0] : 0;
      s_need[r] = (int)run[1];
      s_back[r] = (int)run[2];
      run[0] += add[k];
      run[1] += need[k];
      run[2] += back[k];
    }
  }
  if (tid == 0) s_q[a.n_req] = ok ? (int)total[0] : 0;
  __syncthreads();
  // pages of finished requests onto the stack, a warp per request
  if (ok)
    for (int r = rank * kTabWarps + warp; r < a.n_req; r += n_cta * kTabWarps) {
      if (s_kv[r] >= 0) continue;
      const int held = a.pages(-1 - s_kv[r]);
      for (int j = lane; j < held; j += 32) {
        const int page = a.block_table[(size_t)r * a.table_stride + j];
        if (page < 0 || page >= a.n_pages) atomicOr(a.err, CASCADE_DEV_ERR_BAD_PAGE);
        a.free_pages[count + s_back[r] + j] = page;
      }
    }
  __syncwarp();
  ptx::cluster_arrive();
  ptx::cluster_wait();

  // fresh pages behind the old ones, lengths
  for (int r = rank * kTabWarps + warp; r < a.n_req; r += n_cta * kTabWarps) {
    const bool done = s_kv[r] < 0;
    const int kv = done ? -1 - s_kv[r] : s_kv[r], n = s_q[r + 1] - s_q[r];
    if (ok && !done) {
      const int had = a.pages(kv), has = a.pages(kv + n);
      for (int j = had + lane; j < has; j += 32)
        a.block_table[(size_t)r * a.table_stride + j] = a.free_pages[count1 - 1 - s_need[r] - (j - had)];
    }
    if (lane == 0) {
      a.kv_len_out[r] = !ok ? a.kv_len[r] : (done ? 0 : kv + n);
      a.q_begin[r] = s_q[r];
    }
  }
  if (rank == 0 && tid == 0) {
    a.q_begin[a.n_req] = s_q[a.n_req];
    *a.free_count_out = ok ? (int)(count1 - total[1]) : count;
    if (!ok) atomicOr(a.err, CASCADE_DEV_ERR_OVERFLOW);
  }
  // slots and positions, four consecutive tokens a thread: one search, then a walk
  const int n_live = s_q[a.n_req];
  for (int t0 = 4 * (rank * kTabThreads + tid); t0 < a.n_tok; t0 += 4 * n_cta * kTabThreads) {
    int sl[4] = {-1, -1, -1, -1}, ps[4] = {-1, -1, -1, -1};
    if (t0 < n_live) {
      int lo = 0, hi = a.n_req;  // the request with s_q[r] <= t0 < s_q[r + 1]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (s_q[mid] <= t0)
          lo = mid;
        else
          hi = mid;
      }
      int r = lo, page_at = -1, page = -1;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int t = t0 + k;
        if (t >= n_live) break;
        while (t >= s_q[r + 1]) {
          ++r;
          page_at = -1;
        }
        const int x = s_kv[r] + t - s_q[r], pi = a.div.page(x);
        if (pi != page_at) {
          page_at = pi;
          const int had = a.pages(s_kv[r]);
          page = pi < had ? a.block_table[(size_t)r * a.table_stride + pi] : a.free_pages[count1 - 1 - s_need[r] - (pi - had)];
          if (page < 0 || page >= a.n_pages) {
            page = -1;
            atomicOr(a.err, CASCADE_DEV_ERR_BAD_PAGE);
          }
        }
        sl[k] = page < 0 ? -1 : page * P + (x - pi * P);
        ps[k] = x;
      }
    }
    if (t0 + 4 <= a.n_tok && ((reinterpret_cast<uintptr_t>(a.slot) | reinterpret_cast<uintptr_t>(a.pos)) & 15u) == 0) {
      *reinterpret_cast<int4*>(a.slot + t0) = make_int4(sl[0], sl[1], sl[2], sl[3]);
      *reinterpret_cast<int4*>(a.pos + t0) = make_int4(ps[0], ps[1], ps[2], ps[3]);
    } else {
      for (int k = 0; k < 4 && t0 + k < a.n_tok; ++k) {
        a.slot[t0 + k] = sl[k];
        a.pos[t0 + k] = ps[k];
      }
    }
  }
}

// ---- rotary embedding + cache write ---------------------------------------------------------------------------------

constexpr int kAppThreads = 256;
constexpr int kMaxHalf = 64;  // D / 2

struct AppendArgs {
  int n_tok, Hq, Hkv, page_size;
  long long n_slots, page_stride, q_stride, k_stride, v_stride, q_out_stride;
  const void *q, *k, *v;
  void *q_out, *k_pages, *v_pages;
  const int32_t *slot, *pos;
  int* err;
  double turns[kMaxHalf];  // rope_base^(-2i/D) / 2 pi: turns per position
};

template <typename E>
struct Vec16;
template <>
struct Vec16<float> {
  static constexpr int n = 4;
  static __device__ __forceinline__ void unpack(const uint4& u, float* f) {
    f[0] = __uint_as_float(u.x);
    f[1] = __uint_as_float(u.y);
    f[2] = __uint_as_float(u.z);
    f[3] = __uint_as_float(u.w);
  }
  static __device__ __forceinline__ uint4 pack(const float* f) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
};
template <>
struct Vec16<__nv_bfloat16> {
  static constexpr int n = 8;
  static __device__ __forceinline__ void unpack(const uint4& u, float* f) {
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = __uint_as_float(w[i] << 16);
      f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float* f) {
    return make_uint4(ptx::pack_bf16x2(f[0], f[1]), ptx::pack_bf16x2(f[2], f[3]), ptx::pack_bf16x2(f[4], f[5]),
                      ptx::pack_bf16x2(f[6], f[7]));
  }
};

// A CTA takes kTok tokens: their angles (one per token and pair, reduced to a fraction of a turn in 64 bits, so that far
// positions lose nothing) go to shared memory once, then every thread moves 2 x 16 bytes at a time -- elements i.. and
// i + D/2.. of a head, which turn together.  HBM-bound: every element is read and written once
// (19840 tokens of 3 x 32 heads of 128 in bf16: 155 us, 6.3 TB/s).
template <typename E, int D, bool kRope>
__global__ void __launch_bounds__(kAppThreads) k_paged_append(const __grid_constant__ AppendArgs a) {
  constexpr int kN = Vec16<E>::n, kHalf = D / 2, kVecs = kHalf / kN;  // 16-byte pieces in half a head
  constexpr int kTok = 2;
  __shared__ float2 s_cs[kTok][kHalf];
  const int t_base = blockIdx.x * kTok;
  if (kRope) {
    for (int i = threadIdx.x; i < kTok * kHalf; i += kAppThreads) {
      const int t = t_base + i / kHalf;
      if (t < a.n_tok) {
        const double turn = (double)a.pos[t] * a.turns[i % kHalf];
        float sn, cs;
        sincospif(2.f * (float)(turn - rint(turn)), &sn, &cs);
        s_cs[i / kHalf][i % kHalf] = make_float2(cs, sn);
      }
    }
    __syncthreads();
  }
  const int hq = a.q == nullptr ? 0 : a.Hq, heads = hq + 2 * a.Hkv;
#pragma unroll 1
  for (int tt = 0; tt < kTok; ++tt) {
    const int t = t_base + tt;
    if (t >= a.n_tok) break;
    const int slot = a.slot[t];
    if (slot == -1) continue;
    if (slot < 0 || slot >= a.n_slots) {
      if (threadIdx.x == 0) atomicOr(a.err, CASCADE_DEV_ERR_BAD_PAGE);
      continue;
    }
    const int page = slot / a.page_size, row = slot - page * a.page_size;
    const long long cache_off = (long long)page * a.page_stride + (long long)row * a.Hkv * D;
#pragma unroll 4
    for (int i = threadIdx.x; i < heads * kVecs; i += kAppThreads) {
      const int h = i / kVecs, e = (i % kVecs) * kN;
      const E* src;
      E* dst;
      bool turn = kRope;
      if (h < hq) {
        src = static_cast<const E*>(a.q) + (long long)t * a.q_stride + h * D;
        dst = static_cast<E*>(a.q_out) + (long long)t * a.q_out_stride + h * D;
      } else if (h < hq + a.Hkv) {
        src = static_cast<const E*>(a.k) + (long long)t * a.k_stride + (h - hq) * D;
        dst = static_cast<E*>(a.k_pages) + cache_off + (h - hq) * D;
      } else {
        src = static_cast<const E*>(a.v) + (long long)t * a.v_stride + (h - hq - a.Hkv) * D;
        dst = static_cast<E*>(a.v_pages) + cache_off + (h - hq - a.Hkv) * D;
        turn = false;
      }
      uint4 lo = *reinterpret_cast<const uint4*>(src + e), hi = *reinterpret_cast<const uint4*>(src + kHalf + e);
      if (turn) {
        float x[kN], y[kN], u[kN], w[kN];
        Vec16<E>::unpack(lo, x);
        Vec16<E>::unpack(hi, y);
#pragma unroll
        for (int k = 0; k < kN; ++k) {
          const float2 cs = s_cs[tt][e + k];
          u[k] = x[k] * cs.x - y[k] * cs.y;
          w[k] = y[k] * cs.x + x[k] * cs.y;
        }
        lo = Vec16<E>::pack(u);
        hi = Vec16<E>::pack(w);
      }
      *reinterpret_cast<uint4*>(dst + e) = lo;
      *reinterpret_cast<uint4*>(dst + kHalf + e) = hi;
    }
  }
}

template <typename E, int D>
void run_append(const AppendArgs& a, bool rope, cudaStream_t s) {
  const int grid = cascade_detail::ceil_div(a.n_tok, 2);
  if (rope)
    k_paged_append<E, D, true><<<grid, kAppThreads, 0, s>>>(a);
  else
    k_paged_append<E, D, false><<<grid, kAppThreads, 0, s>>>(a);
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace

int check_paged_cache(const cascade_ctx* ctx, const cascade_paged_cache* c) {
  if (c == nullptr || c->k_pages == nullptr || c->v_pages == nullptr) return CASCADE_ERR_INVALID_ARG;
  if (c->n_pages < 1 || c->page_size < 1) return CASCADE_ERR_INVALID_ARG;
  if (!aligned16(c->k_pages) || !aligned16(c->v_pages)) return CASCADE_ERR_INVALID_ARG;
  const cascade_shape& sh = ctx->shape;
  const int es = sh.dtype == CASCADE_BF16 ? 2 : 4;
  if (c->page_stride < (int64_t)c->page_size * sh.Hkv * sh.D || c->page_stride * es % 16 != 0) return CASCADE_ERR_INVALID_ARG;
  if (c->page_size % 8 != 0 || (int64_t)c->n_pages * c->page_size > INT32_MAX) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  return CASCADE_OK;
}

int check_current_device(const cascade_ctx* ctx) {
  int dev = -1;
  CASCADE_CUDA_TRY(cudaGetDevice(&dev));
  return dev == ctx->device ? CASCADE_OK : CASCADE_ERR_INVALID_ARG;
}

extern "C" {

int cascade_paged_tables(cascade_ctx* ctx, int32_t n_req, int32_t n_tok, int32_t page_size, int32_t n_pages,
                         const int32_t* new_len, const int32_t* kv_len, int32_t* block_table, int32_t table_stride,
                         int32_t* free_pages, const int32_t* free_count, int32_t* kv_len_out, int32_t* free_count_out,
                         int32_t* q_begin, int32_t* slot, int32_t* pos, void* stream) {
  if (ctx == nullptr || new_len == nullptr || kv_len == nullptr || block_table == nullptr || free_pages == nullptr ||
      free_count == nullptr || kv_len_out == nullptr || free_count_out == nullptr || q_begin == nullptr)
    return CASCADE_ERR_INVALID_ARG;
  if (n_req < 1 || n_tok < 0 || page_size < 1 || n_pages < 1 || table_stride < 1) return CASCADE_ERR_INVALID_ARG;
  if (n_tok > 0 && (slot == nullptr || pos == nullptr)) return CASCADE_ERR_INVALID_ARG;
  if (!aligned4(new_len, kv_len, block_table, free_pages, free_count, kv_len_out, free_count_out, q_begin, slot, pos))
    return CASCADE_ERR_INVALID_ARG;
  if (n_req > CASCADE_MAX_REQUESTS || page_size % 8 != 0 || (int64_t)n_pages * page_size > INT32_MAX)
    return CASCADE_ERR_UNSUPPORTED_SHAPE;
  if (n_tok > INT32_MAX - 65536) return CASCADE_ERR_UNSUPPORTED_SHAPE;  // the token loop's stride must not pass 32 bits
  CASCADE_TRY(check_current_device(ctx));
  TablesArgs a;
  a.n_req = n_req;
  a.n_tok = n_tok;
  a.page_size = page_size;
  a.n_pages = n_pages;
  a.table_stride = table_stride;
  a.new_len = new_len;
  a.kv_len = kv_len;
  a.free_count = free_count;
  a.block_table = block_table;
  a.free_pages = free_pages;
  a.kv_len_out = kv_len_out;
  a.free_count_out = free_count_out;
  a.q_begin = q_begin;
  a.slot = slot;
  a.pos = pos;
  a.err = ctx->dev_error;
  a.div = paged::page_div(page_size);
  const size_t smem = (size_t)(4 * n_req + 1) * sizeof(int);
  // (for every count: what a kernel gets unasked, 48 KB, has to hold its static arrays too)
  CASCADE_TRY(configure_smem(ctx, PAGED_CFG_TABLES, k_paged_tables, (4 * CASCADE_MAX_REQUESTS + 1) * (int)sizeof(int)));
  // a cluster of eight for few tokens too (against one CTA: two tokens 5.1 us either way, 2000 tokens of 32 requests 6.8 either
  // way, 4000 of 64 7.1 and 7.8, 256 requests of one token 6.7 and 9.4)
  constexpr int kCtas = 8;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kCtas);
  cfg.blockDim = dim3(kTabThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = static_cast<cudaStream_t>(stream);
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kCtas;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  ctx->launches = 0;
  KernelScope ks(ctx, K_PAGED_TABLES, cfg.stream);
  CASCADE_CUDA_TRY(cudaLaunchKernelEx(&cfg, k_paged_tables, a));
  return CASCADE_OK;
}

int cascade_paged_append(cascade_ctx* ctx, const cascade_paged_cache* cache, int32_t n_tok, const void* q, int64_t q_stride,
                         const void* k, int64_t k_stride, const void* v, int64_t v_stride, const int32_t* slot,
                         const int32_t* pos, float rope_base, void* q_out, int64_t q_out_stride, void* stream) {
  if (ctx == nullptr || k == nullptr || v == nullptr || slot == nullptr || pos == nullptr || n_tok < 1)
    return CASCADE_ERR_INVALID_ARG;
  CASCADE_TRY(check_paged_cache(ctx, cache));
  const cascade_shape& sh = ctx->shape;
  const int64_t kv_row = (int64_t)sh.Hkv * sh.D, q_row = (int64_t)sh.Hq * sh.D;
  const int es = sh.dtype == CASCADE_BF16 ? 2 : 4;
  const bool rope = rope_base != 0.f;
  if (rope && !(rope_base > 1.f && std::isfinite(rope_base))) return CASCADE_ERR_INVALID_ARG;
  if ((q == nullptr) != (q_out == nullptr) || (q != nullptr && !rope)) return CASCADE_ERR_INVALID_ARG;
  if (k_stride < kv_row || v_stride < kv_row || k_stride * es % 16 != 0 || v_stride * es % 16 != 0) return CASCADE_ERR_INVALID_ARG;
  if (!aligned16(k) || !aligned16(v) || !aligned16(q) || !aligned16(q_out) || !aligned4(slot, pos)) return CASCADE_ERR_INVALID_ARG;
  if (q != nullptr && (q_stride < q_row || q_out_stride < q_row || q_stride * es % 16 != 0 || q_out_stride * es % 16 != 0 ||
                       (q == q_out && q_stride != q_out_stride)))
    return CASCADE_ERR_INVALID_ARG;
  CASCADE_TRY(check_current_device(ctx));
  AppendArgs a;
  a.n_tok = n_tok;
  a.Hq = sh.Hq;
  a.Hkv = sh.Hkv;
  a.page_size = cache->page_size;
  a.n_slots = (long long)cache->n_pages * cache->page_size;
  a.page_stride = cache->page_stride;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_out_stride = q_out_stride;
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_out = q_out;
  a.k_pages = cache->k_pages;
  a.v_pages = cache->v_pages;
  a.slot = slot;
  a.pos = pos;
  a.err = ctx->dev_error;
  if (rope && ctx->rope_base != rope_base) {
    for (int i = 0; i < sh.D / 2; ++i) ctx->rope_turns[i] = std::pow((double)rope_base, -2.0 * i / sh.D) / 6.283185307179586476925;
    ctx->rope_base = rope_base;
  }
  if (rope) std::memcpy(a.turns, ctx->rope_turns, sizeof(double) * (sh.D / 2));
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  ctx->launches = 0;
  {
    KernelScope ks(ctx, K_PAGED_APPEND, s);
    if (sh.dtype == CASCADE_BF16) {
      if (sh.D == 128)
        run_append<__nv_bfloat16, 128>(a, rope, s);
      else
        run_append<__nv_bfloat16, 64>(a, rope, s);
    } else {
      if (sh.D == 128)
        run_append<float, 128>(a, rope, s);
      else
        run_append<float, 64>(a, rope, s);
    }
  }
  CASCADE_CUDA_TRY(cudaGetLastError());
  return CASCADE_OK;
}

}  // extern "C"
