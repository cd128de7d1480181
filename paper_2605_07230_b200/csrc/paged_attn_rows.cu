// Attention over a paged cache for few rows (bf16): single tokens, and short chunks, whose new tokens times the query
// heads of a key head are at most 16 rows.
//
// Memory-bound: every key and value is read once for all rows.  One CTA of four warps per (KV split, key head, request);
// a warp takes 16 keys at a time straight from memory into the operand registers of warp-level matrix products (m16n8k16).
// Keys and values stand on M and the rows on N, in blocks of eight: S^T = K Q^T and O^T = V^T P^T.  The sum over a head's
// elements does not care for their order, so a lane's 16-byte pieces of a key row serve as they come; the values' pieces
// give pairs of keys after one byte permute per register, and the weights turn with one 8 x 8 transpose per eight keys.
// No shared memory and no barrier in the loop: the keys of the next 16 are requested as soon as the scores have used the
// registers, the values as soon as the output has; with up to eight rows three CTAs fit an SM, 96 KB in flight.
// 48 single tokens over 256 to 2880 keys, 32 heads of 128: 196 us in graph replays, 6.6 TB/s of reads (a copy, half of it
// writes, runs at 6.45), 207 us called one by one; two over 385 keys: 8.2 and 10.2 us.
// (The 5th-generation tensor cores want 128 rows and operands in shared memory; here they would multiply padding.)
// Weights are 2^(s c - ref); ref is the running maximum, raised only when a score passes it by more than 2^8.  Weights are
// rounded to bf16 for the product with the bf16 values, sums and accumulators stay fp32.
// The warps' partial results meet in shared memory, the splits' (a thread-block cluster) through distributed shared memory.
#include "paged.h"
#include "paged_attn.cuh"

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kRows = 16;
constexpr int kChunk = 16;        // keys per step of a warp
constexpr float kLazy = 8.f;
constexpr int kSortMost = 256;    // requests that are ordered by length

struct RowArgs {
  PagedAttnArgs a;
  int G, splits, sorted, max_rows;
  paged::PageDiv div;
};

// 8 x 8 transpose of 16-bit elements across the warp.
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ void mma16816(float* c, const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// kNb: blocks of eight rows.
template <int D, int kNb>
__global__ void __launch_bounds__(kThreads, kNb == 1 ? 3 : 2) k_paged_attn_rows(const RowArgs p) {
  constexpr int kQ = D / 32;                     // 16-byte pieces of a key row per lane
  constexpr int kJ = D / 64;                     // 16-byte pieces of a value row per lane
  constexpr int kO = D / 16;                     // output products
  constexpr int kX = paged::part_stride(D);
  extern __shared__ __align__(16) float s_part[];  // [warp][row][kX], as many rows as the call has at most
  __shared__ bool s_lost[kWarps];                // the warp met a page outside the pool
  const PagedAttnArgs& a = p.a;
  const int part = p.max_rows * kX;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int split = blockIdx.x, kh = blockIdx.y;
  int r = blockIdx.z;
  if (p.sorted) {
    // several waves of CTAs: the longest requests go first, so that the last wave is short (the z-th longest is found by
    // counting who is longer; ties by index)
    __shared__ int s_len[kSortMost], s_r;
    for (int i = threadIdx.x; i < a.n_req; i += kThreads) s_len[i] = a.kv_len[i];
    __syncthreads();
    for (int i = threadIdx.x; i < a.n_req; i += kThreads) {
      const int mine = s_len[i];
      int rank = 0;
      for (int k = 0; k < a.n_req; ++k) rank += s_len[k] > mine || (s_len[k] == mine && k < i);
      if (rank == r) s_r = i;
    }
    __syncthreads();
    r = s_r;
  }
  paged::Request rq;
  const bool valid = paged::load_request(a, r, &rq);
  const int rows = valid ? rq.nq * p.G : 0;      // at most 8 kNb
  const int x0 = rq.kv - rq.nq;                  // position of the first new token
  if (rows == 0) return;                         // (the same in all CTAs of a cluster)
  if (p.splits > 1) ptx::cluster_arrive();       // (waited for in merge_and_store)
  if (lane == 0) s_lost[warp] = false;

  // 16-key steps that any row sees: [0, n_sink) and [n_sink + skip, ...)
  int n = 0, n_sink = 0, skip = 0;
  if (rq.kv > 0) {
    const int lo = paged::window_begin(x0, a.window), lo_c = lo / kChunk;
    n_sink = min((min(a.sinks, lo) + kChunk - 1) / kChunk, lo_c);
    skip = lo_c - n_sink;
    n = (rq.kv + kChunk - 1) / kChunk - skip;
  }
  const int per = (n + p.splits - 1) / p.splits;
  const int c_end = min(n, (split + 1) * per);
  int c = split * per + warp;

  // query fragments: lane (g, t) holds elements 32 j + 8 t .. + 7 of row 8 b + g
  uint32_t q[kNb][kQ][4];
#pragma unroll
  for (int b = 0; b < kNb; ++b) {
    const int row = 8 * b + g;
    const __nv_bfloat16* src = static_cast<const __nv_bfloat16*>(a.q);
    if (row < rows) src += (long long)(rq.q0 + row / p.G) * a.q_stride + (kh * p.G + row % p.G) * D;
#pragma unroll
    for (int j = 0; j < kQ; ++j) {
      const uint4 v = row < rows ? *reinterpret_cast<const uint4*>(src + 32 * j + 8 * t) : make_uint4(0, 0, 0, 0);
      q[b][j][0] = v.x;
      q[b][j][1] = v.y;
      q[b][j][2] = v.z;
      q[b][j][3] = v.w;
    }
  }
  int x_row[kNb][2];                             // positions of rows 8 b + 2 t + i; -1: no such row
#pragma unroll
  for (int b = 0; b < kNb; ++b)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int row = 8 * b + 2 * t + i;
      x_row[b][i] = row < rows ? x0 + row / p.G : -1;
    }

  const int32_t* table = a.block_table + (size_t)r * a.table_stride;
  const __nv_bfloat16* k_base = static_cast<const __nv_bfloat16*>(a.k) + kh * D;
  const __nv_bfloat16* v_base = static_cast<const __nv_bfloat16*>(a.v) + kh * D;
  const int row_elems = a.Hkv * D;
  auto first_key = [&](int i) { return (i < n_sink ? i : i + skip) * kChunk; };
  // element offset of a group of 8 keys (a group lies in one page); -1: nothing there
  auto page_off = [&](int key) -> long long {
    if (key >= rq.kv) return -1;
    const int pi = p.div.page(key);
    const int page = table[pi];
    if (page < 0 || page >= a.n_pages) {
      if (lane == 0) {
        atomicOr(a.err, CASCADE_DEV_ERR_BAD_PAGE);
        s_lost[warp] = true;
      }
      return -1;
    }
    return (long long)page * a.page_stride + (long long)(key - pi * a.page_size) * row_elems;
  };
  uint4 kr[2][kQ], vr[4][kJ];
  auto load_k = [&](int key0, const long long* off) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {                // keys g and 8 + g
      const bool there = off[h] >= 0 && key0 + 8 * h + g < rq.kv;
      const __nv_bfloat16* src = k_base + (there ? off[h] : 0) + (there ? g : 0) * row_elems + 8 * t;
#pragma unroll
      for (int j = 0; j < kQ; ++j) kr[h][j] = there ? paged::ld_stream(src + 32 * j) : make_uint4(0, 0, 0, 0);
    }
  };
  auto load_v = [&](int key0, const long long* off) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {                // keys 2t, 2t + 1, 2t + 8, 2t + 9
      const int in = 2 * t + (i & 1), h = i >> 1;
      const bool there = off[h] >= 0 && key0 + 8 * h + in < rq.kv;
      const __nv_bfloat16* src = v_base + (there ? off[h] : 0) + (there ? in : 0) * row_elems + 8 * g;
#pragma unroll
      for (int j = 0; j < kJ; ++j) vr[i][j] = there ? paged::ld_stream(src + 64 * j) : make_uint4(0, 0, 0, 0);
    }
  };

  float o[kNb][kO][4];
  float ref[kNb][2], l[kNb][2];                  // of rows 8 b + 2 t + i
#pragma unroll
  for (int b = 0; b < kNb; ++b) {
    ref[b][0] = ref[b][1] = -INFINITY;
    l[b][0] = l[b][1] = 0.f;
#pragma unroll
    for (int e = 0; e < kO; ++e) o[b][e][0] = o[b][e][1] = o[b][e][2] = o[b][e][3] = 0.f;
  }
  const float sc = a.scale * paged::kLog2e;

  long long off_next[2] = {-1, -1};
  int key0 = 0;
  if (c < c_end) {
    key0 = first_key(c);
    const long long off[2] = {page_off(key0), page_off(key0 + 8)};
    load_k(key0, off);
    load_v(key0, off);
    if (c + kWarps < c_end) {
      off_next[0] = page_off(first_key(c + kWarps));
      off_next[1] = page_off(first_key(c + kWarps) + 8);
    }
  }
  for (; c < c_end; c += kWarps) {
    const int next0 = c + kWarps < c_end ? first_key(c + kWarps) : 0;
    long long off_after[2] = {-1, -1};
    if (c + 2 * kWarps < c_end) {
      off_after[0] = page_off(first_key(c + 2 * kWarps));
      off_after[1] = page_off(first_key(c + 2 * kWarps) + 8);
    }
    // scores: s[b][2 h + i] is key key0 + 8 h + g, row 8 b + 2 t + i
    float s[kNb][4];
#pragma unroll
    for (int b = 0; b < kNb; ++b) s[b][0] = s[b][1] = s[b][2] = s[b][3] = 0.f;
#pragma unroll
    for (int j = 0; j < kQ; ++j) {
      const uint32_t a0[4] = {kr[0][j].x, kr[1][j].x, kr[0][j].y, kr[1][j].y};
      const uint32_t a1[4] = {kr[0][j].z, kr[1][j].z, kr[0][j].w, kr[1][j].w};
#pragma unroll
      for (int b = 0; b < kNb; ++b) {
        mma16816(s[b], a0, q[b][j][0], q[b][j][1]);
        mma16816(s[b], a1, q[b][j][2], q[b][j][3]);
      }
    }
    if (c + kWarps < c_end) load_k(next0, off_next);
    // steps behind the first token's position or at a window's edge look closer
    const bool edge = key0 + kChunk - 1 > x0 || (a.window > 0 && key0 < x0 + rq.nq - a.window);
    uint32_t w[kNb][2];                          // the weights as the B operand
#pragma unroll
    for (int b = 0; b < kNb; ++b) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float v = s[b][k] * sc;
        if (edge) {
          const int j = key0 + 8 * (k >> 1) + g, x = x_row[b][k & 1];
          const bool sees = j <= x && (j >= paged::window_begin(x, a.window) || j < a.sinks);
          v = sees ? v : -INFINITY;
        }
        s[b][k] = v;
      }
      // raise the reference where a score passes it by more than kLazy (or the row had none)
      float mx[2];
      bool raise = false;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        mx[i] = fmaxf(s[b][i], s[b][2 + i]);
        raise = raise || mx[i] > ref[b][i] + kLazy || (ref[b][i] == -INFINITY && mx[i] > -INFINITY);
      }
      if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
          for (int x = 4; x < 32; x <<= 1) mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], x));
          float alpha = 1.f;
          if (mx[i] > ref[b][i]) {
            alpha = ref[b][i] == -INFINITY ? 0.f : ptx::ex2(ref[b][i] - mx[i]);
            ref[b][i] = mx[i];
          }
          l[b][i] *= alpha;
#pragma unroll
          for (int e = 0; e < kO; ++e) {
            o[b][e][i] *= alpha;
            o[b][e][2 + i] *= alpha;
          }
        }
      }
      const float m0 = ref[b][0] == -INFINITY ? 0.f : ref[b][0], m1 = ref[b][1] == -INFINITY ? 0.f : ref[b][1];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float w0 = ptx::ex2(s[b][2 * h] - m0), w1 = ptx::ex2(s[b][2 * h + 1] - m1);
        l[b][0] += w0;
        l[b][1] += w1;
        w[b][h] = transpose8(ptx::pack_bf16x2(w0, w1));
      }
    }
    // outputs: product e holds elements 8 g + e and 64 + 8 g + e (D = 64: 8 g + e and 8 g + 4 + e) on its 16 rows
#pragma unroll
    for (int e = 0; e < kO; ++e) {
      const int e1 = D == 128 ? e : e + 4, j1 = kJ - 1;
      const uint32_t sel = (e & 1) ? 0x7632u : 0x5410u;
      auto word = [&](int i, int j, int x) { return (x >> 1) == 0 ? vr[i][j].x : (x >> 1) == 1 ? vr[i][j].y : (x >> 1) == 2 ? vr[i][j].z : vr[i][j].w; };
      const uint32_t av[4] = {__byte_perm(word(0, 0, e), word(1, 0, e), sel), __byte_perm(word(0, j1, e1), word(1, j1, e1), sel),
                              __byte_perm(word(2, 0, e), word(3, 0, e), sel), __byte_perm(word(2, j1, e1), word(3, j1, e1), sel)};
#pragma unroll
      for (int b = 0; b < kNb; ++b) mma16816(o[b][e], av, w[b][0], w[b][1]);
    }
    if (c + kWarps < c_end) load_v(next0, off_next);
    key0 = next0;
    off_next[0] = off_after[0];
    off_next[1] = off_after[1];
  }

  // ---- the warps' partial results -> one per CTA (in place of the first) -> one per cluster ----
  // (keys of a lost page went in as zeros: a sum that is no number has the rows computed again without them)
  __syncwarp();
  const bool lost = s_lost[warp];
#pragma unroll
  for (int b = 0; b < kNb; ++b)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
      for (int x = 4; x < 32; x <<= 1) l[b][i] += __shfl_xor_sync(0xffffffffu, l[b][i], x);
      const int row = 8 * b + 2 * t + i;
      if (row < rows) {
        float* x = s_part + warp * part + row * kX;
        float4* lo = reinterpret_cast<float4*>(x + 8 * g);
        if constexpr (D == 128) {
          float4* hi = reinterpret_cast<float4*>(x + 64 + 8 * g);
          lo[0] = make_float4(o[b][0][i], o[b][1][i], o[b][2][i], o[b][3][i]);
          lo[1] = make_float4(o[b][4][i], o[b][5][i], o[b][6][i], o[b][7][i]);
          hi[0] = make_float4(o[b][0][2 + i], o[b][1][2 + i], o[b][2][2 + i], o[b][3][2 + i]);
          hi[1] = make_float4(o[b][4][2 + i], o[b][5][2 + i], o[b][6][2 + i], o[b][7][2 + i]);
        } else {
          lo[0] = make_float4(o[b][0][i], o[b][1][i], o[b][2][i], o[b][3][i]);
          lo[1] = make_float4(o[b][0][2 + i], o[b][1][2 + i], o[b][2][2 + i], o[b][3][2 + i]);
        }
        if (g == 0) {
          x[D] = ref[b][i];
          x[D + 1] = lost ? NAN : l[b][i];
        }
      }
    }
  paged::merge_and_store<__nv_bfloat16, D, kWarps, 8 * kNb>(a, r, rq.q0, x0, kh, 0, rows, p.G, p.splits, s_part, p.max_rows);
}

}  // namespace

// 16 tokens, 32 key heads, 16 requests over 1000 to 2000 keys: 94 us here, 112 us in 128-row blocks on the 5th-generation
// tensor cores; 4 tokens of 4 query heads a key head: 34 / 36 us, two such requests over 300 to 400 keys 9.4 / 12.7 us.
bool paged_attn_rows_takes(const PagedAttnArgs& a) { return (long long)a.max_q * (a.Hq / a.Hkv) <= kRows && a.Hkv <= 65535; }

int launch_paged_attn_rows(cascade_ctx* ctx, const PagedAttnArgs& a, cudaStream_t s) {
  RowArgs p;
  p.a = a;
  p.G = a.Hq / a.Hkv;
  p.div = paged::page_div(a.page_size);
  // splits: as many as keep the resident CTAs (three an SM) busy at once, each with at least two steps a warp
  const long long units = (long long)a.n_req * a.Hkv;
  const int span = a.window > 0 && (long long)a.window + a.sinks + a.max_q < a.max_kv ? a.window + a.sinks + a.max_q : a.max_kv;
  const int steps = cascade_detail::ceil_div(span > 0 ? span : 1, kChunk * kWarps);
  p.max_rows = a.max_q * p.G;
  const bool two_blocks = p.max_rows > 8;
  const long long resident = (two_blocks ? 2ll : 3ll) * ctx->sm_count;
  p.splits = 1;
  while (p.splits < 8 && units * p.splits * 2 <= resident && steps >= 2 * p.splits) p.splits *= 2;
  p.sorted = units * p.splits > resident && a.n_req <= kSortMost;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.splits, a.Hkv, a.n_req);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = (size_t)paged::part_floats(ctx->shape.D, kWarps, p.max_rows) * sizeof(float);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = p.splits;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (ctx->shape.D == 128)
    CASCADE_CUDA_TRY(two_blocks ? cudaLaunchKernelEx(&cfg, k_paged_attn_rows<128, 2>, p) : cudaLaunchKernelEx(&cfg, k_paged_attn_rows<128, 1>, p));
  else
    CASCADE_CUDA_TRY(two_blocks ? cudaLaunchKernelEx(&cfg, k_paged_attn_rows<64, 2>, p) : cudaLaunchKernelEx(&cfg, k_paged_attn_rows<64, 1>, p));
  return CASCADE_OK;
}
