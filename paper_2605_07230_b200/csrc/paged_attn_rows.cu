// Attention over a paged cache for few rows (bf16): single tokens, and short chunks, whose new tokens times the query
// heads of a key head are at most 16 rows.
//
// Memory-bound: every key and value is read once for all rows.  One CTA of four warps per (KV split, key head, request);
// a warp takes 16 keys at a time straight from memory into the operand registers of warp-level matrix products
// (m16n8k16, the 16 rows on M): the sum over a head's elements does not care for their order, so a lane's 16-byte pieces
// of a key row serve as they come, and the values' 16-byte pieces give pairs of keys after one byte permute per register.
// No shared memory, no barrier in the loop: the keys of the next 16 are requested as soon as the scores have used the
// registers, the values as soon as the output has, and with three CTAs an SM keeps about 80 KB in flight.
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

struct RowArgs {
  PagedAttnArgs a;
  int G, splits;
  uint32_t page_mul;              // key / page_size = (key * page_mul) >> page_shift for keys below 2^31
  int page_shift;
};

__device__ __forceinline__ uint4 ld_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.L2::256B.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ void mma16816(float* c, const uint32_t* a, uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

template <int D>
__global__ void __launch_bounds__(kThreads, 3) k_paged_attn_rows(const RowArgs p) {
  constexpr int kQ = D / 32;                     // 16-byte pieces of a row per lane
  constexpr int kJ = D / 64;
  constexpr int kX = D + 4;                      // floats per row of a partial result: outputs, reference, sum
  __shared__ __align__(16) float s_part[kWarps][kRows][kX];
  __shared__ int s_odd;
  const PagedAttnArgs& a = p.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  const int split = blockIdx.x, kh = blockIdx.y, r = blockIdx.z;
  paged::Request rq;
  const bool valid = paged::load_request(a, r, &rq);
  const int rows = valid ? rq.nq * p.G : 0;      // at most kRows
  const int x0 = rq.kv - rq.nq;                  // position of the first new token
  if (threadIdx.x == 0) s_odd = 0;

  // 16-key steps that any row sees: [0, n_sink) and [n_sink + skip, ...)
  int n = 0, n_sink = 0, skip = 0;
  if (rows > 0 && rq.kv > 0) {
    const int lo = paged::window_begin(x0, a.window), lo_c = lo / kChunk;
    n_sink = min((min(a.sinks, lo) + kChunk - 1) / kChunk, lo_c);
    skip = lo_c - n_sink;
    n = (rq.kv + kChunk - 1) / kChunk - skip;
  }
  const int per = (n + p.splits - 1) / p.splits;
  const int c_end = min(n, (split + 1) * per);
  int c = split * per + warp;

  // query fragments: lane (g, t) holds elements 32 j + 8 t .. + 7 of rows g and g + 8
  uint32_t q_lo[kQ][4], q_hi[kQ][4];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int row = g + 8 * h;
    const __nv_bfloat16* q = static_cast<const __nv_bfloat16*>(a.q);
    if (row < rows) q += (long long)(rq.q0 + row / p.G) * a.q_stride + (kh * p.G + row % p.G) * D;
#pragma unroll
    for (int j = 0; j < kQ; ++j) {
      const uint4 v = row < rows ? *reinterpret_cast<const uint4*>(q + 32 * j + 8 * t) : make_uint4(0, 0, 0, 0);
      uint32_t* dst = h == 0 ? q_lo[j] : q_hi[j];
      dst[0] = v.x;
      dst[1] = v.y;
      dst[2] = v.z;
      dst[3] = v.w;
    }
  }
  const int x_row[2] = {g < rows ? x0 + g / p.G : -1, g + 8 < rows ? x0 + (g + 8) / p.G : -1};

  const int32_t* table = a.block_table + (size_t)r * a.table_stride;
  const __nv_bfloat16* k_base = static_cast<const __nv_bfloat16*>(a.k) + kh * D;
  const __nv_bfloat16* v_base = static_cast<const __nv_bfloat16*>(a.v) + kh * D;
  const int row_elems = a.Hkv * D;
  auto first_key = [&](int i) { return (i < n_sink ? i : i + skip) * kChunk; };
  // element offsets of the two groups of 8 keys of a step (a group lies in one page); -1: nothing there
  auto page_off = [&](int key) -> long long {
    if (key >= rq.kv) return -1;
    const int pi = (int)(((unsigned long long)(uint32_t)key * p.page_mul) >> p.page_shift);
    const int page = table[pi];
    if (page < 0 || page >= a.n_pages) {
      if (lane == 0) atomicOr(a.err, CASCADE_DEV_ERR_BAD_PAGE);
      return -1;
    }
    return (long long)page * a.page_stride + (long long)(key - pi * a.page_size) * row_elems;
  };
  uint4 kr[2][kQ], vr[4][kJ];
  auto load_k = [&](int key0, const long long* off) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const bool there = off[h] >= 0 && key0 + 8 * h + g < rq.kv;
      const __nv_bfloat16* src = k_base + (there ? off[h] : 0) + (there ? g : 0) * row_elems + 8 * t;
#pragma unroll
      for (int j = 0; j < kQ; ++j) kr[h][j] = there ? ld_stream(src + 32 * j) : make_uint4(0, 0, 0, 0);
    }
  };
  auto load_v = [&](int key0, const long long* off) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {   // keys 2t, 2t + 1, 2t + 8, 2t + 9
      const int in = 2 * t + (i & 1), h = i >> 1;
      const bool there = off[h] >= 0 && key0 + 8 * h + in < rq.kv;
      const __nv_bfloat16* src = v_base + (there ? off[h] : 0) + (there ? in : 0) * row_elems + 8 * g;
#pragma unroll
      for (int j = 0; j < kJ; ++j) vr[i][j] = there ? ld_stream(src + 64 * j) : make_uint4(0, 0, 0, 0);
    }
  };

  float o[kJ][8][4];
#pragma unroll
  for (int j = 0; j < kJ; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int k = 0; k < 4; ++k) o[j][e][k] = 0.f;
  float ref[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  const float sc = a.scale * paged::kLog2e;

  long long off[2] = {-1, -1}, off_next[2] = {-1, -1};
  int key0 = 0;
  if (c < c_end) {
    key0 = first_key(c);
    off[0] = page_off(key0);
    off[1] = page_off(key0 + 8);
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
    // scores: keys key0 + 8 h + (2t, 2t + 1), rows g and g + 8
    float s[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      s[h][0] = s[h][1] = s[h][2] = s[h][3] = 0.f;
#pragma unroll
      for (int j = 0; j < kQ; ++j) {
        const uint32_t a0[4] = {q_lo[j][0], q_hi[j][0], q_lo[j][1], q_hi[j][1]};
        const uint32_t a1[4] = {q_lo[j][2], q_hi[j][2], q_lo[j][3], q_hi[j][3]};
        mma16816(s[h], a0, kr[h][j].x, kr[h][j].y);
        mma16816(s[h], a1, kr[h][j].z, kr[h][j].w);
      }
    }
    if (c + kWarps < c_end) load_k(next0, off_next);
    // visibility: steps behind the first token's position or at a window's edge look closer
    const bool edge = key0 + kChunk - 1 > x0 || (a.window > 0 && key0 < x0 + rq.nq - a.window);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float v = s[h][k] * sc;
        if (edge) {
          const int j = key0 + 8 * h + 2 * t + (k & 1), x = x_row[k >> 1];
          const bool sees = j <= x && (j >= paged::window_begin(x, a.window) || j < a.sinks);
          v = sees ? v : -INFINITY;
        }
        s[h][k] = v;
      }
    // raise the reference where a score passes it by more than kLazy (or the row had none)
    float mx[2];
    bool raise = false;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      mx[i] = fmaxf(fmaxf(s[0][2 * i], s[0][2 * i + 1]), fmaxf(s[1][2 * i], s[1][2 * i + 1]));
      raise = raise || mx[i] > ref[i] + kLazy || (ref[i] == -INFINITY && mx[i] > -INFINITY);
    }
    if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 1));
        mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], 2));
        float alpha = 1.f;
        if (mx[i] > ref[i]) {
          alpha = ref[i] == -INFINITY ? 0.f : ptx::ex2(ref[i] - mx[i]);
          ref[i] = mx[i];
        }
        l[i] *= alpha;
#pragma unroll
        for (int j = 0; j < kJ; ++j)
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            o[j][e][2 * i] *= alpha;
            o[j][e][2 * i + 1] *= alpha;
          }
      }
    }
    uint32_t w[4];   // the weights as the A operand: rows g, g + 8; keys 2t.., 2t + 8..
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float m = ref[i] == -INFINITY ? 0.f : ref[i];
        const float w0 = ptx::ex2(s[h][2 * i] - m), w1 = ptx::ex2(s[h][2 * i + 1] - m);
        l[i] += w0 + w1;
        w[2 * h + i] = ptx::pack_bf16x2(w0, w1);
      }
    // outputs: n index g of product (j, e) is element 64 j + 8 g + e
#pragma unroll
    for (int j = 0; j < kJ; ++j) {
      const uint32_t v0[4] = {vr[0][j].x, vr[0][j].y, vr[0][j].z, vr[0][j].w}, v1[4] = {vr[1][j].x, vr[1][j].y, vr[1][j].z, vr[1][j].w};
      const uint32_t v2[4] = {vr[2][j].x, vr[2][j].y, vr[2][j].z, vr[2][j].w}, v3[4] = {vr[3][j].x, vr[3][j].y, vr[3][j].z, vr[3][j].w};
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t sel = (e & 1) ? 0x7632u : 0x5410u;
        mma16816(o[j][e], w, __byte_perm(v0[e >> 1], v1[e >> 1], sel), __byte_perm(v2[e >> 1], v3[e >> 1], sel));
      }
    }
    if (c + kWarps < c_end) load_v(next0, off_next);
    key0 = next0;
    off_next[0] = off_after[0];
    off_next[1] = off_after[1];
  }

  // ---- the warps' partial results -> one per CTA (in s_part[0]) -> one per cluster ----
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 1);
    l[i] += __shfl_xor_sync(0xffffffffu, l[i], 2);
    const int row = g + 8 * i;
    if (row < rows) {
      float* x = s_part[warp][row];
#pragma unroll
      for (int j = 0; j < kJ; ++j)
#pragma unroll
        for (int q = 0; q < 2; ++q)      // n = 2t + q: elements 64 j + 16 t + 8 q + e
#pragma unroll
          for (int e = 0; e < 8; e += 4)
            *reinterpret_cast<float4*>(x + 64 * j + 16 * t + 8 * q + e) =
                make_float4(o[j][e][2 * i + q], o[j][e + 1][2 * i + q], o[j][e + 2][2 * i + q], o[j][e + 3][2 * i + q]);
      if (t == 0) {
        x[D] = ref[i];
        x[D + 1] = l[i];
      }
    }
  }
  __syncthreads();
  // element i of the CTA's rows, from `count` partial results `get(s, row, column)`
  auto merge = [&](int row, int col, int count, auto get, float* ref_out, float* sum_out) {
    float m = -INFINITY;
    for (int s = 0; s < count; ++s) m = fmaxf(m, get(s, row, D));
    float acc = 0.f, sum = 0.f;
    for (int s = 0; s < count; ++s) {
      const float ms = get(s, row, D);
      const float w = ms == -INFINITY ? 0.f : ptx::ex2(ms - m);
      // a split that met nothing has no part in the row: what it holds is 0, or NaN by a value nobody saw
      acc += ms == -INFINITY ? 0.f : w * get(s, row, col);
      sum += w * get(s, row, D + 1);
    }
    *ref_out = m;
    *sum_out = sum;
    return acc;
  };
  auto here = [&](int s, int row, int col) { return s_part[s][row][col]; };
  const bool alone = p.splits == 1;
  auto finish = [&](int row, int col, float acc, float m, float sum) {
    const int x = x0 + row / p.G, tok = rq.q0 + row / p.G, head = kh * p.G + row % p.G;
    const long long at = (long long)tok * a.Hq + head;
    const float v = x < 0 ? 0.f : acc / sum;
    static_cast<__nv_bfloat16*>(a.out)[at * D + col] = __float2bfloat16(v);
    if (col == 0 && a.lse != nullptr) a.lse[at] = x < 0 ? -INFINITY : (m + log2f(sum)) * paged::kLn2;
    if (x >= 0 && !(fabsf(v) < INFINITY && sum > 0.f)) atomicOr(&s_odd, 1 << row);
  };
  if (alone) {
    for (int i = threadIdx.x; i < rows * D; i += kThreads) {
      float m, sum;
      const float acc = merge(i / D, i % D, kWarps, here, &m, &sum);
      finish(i / D, i % D, acc, m, sum);
    }
  } else {
    // merge the CTA's warps into s_part[0] (each thread reads a column of all four before it writes)
    float mine[kRows * D / kThreads], m_mine[kRows * D / kThreads], sum_mine[kRows * D / kThreads];
#pragma unroll
    for (int k = 0; k < kRows * D / kThreads; ++k) {
      const int i = k * kThreads + threadIdx.x;
      if (i < rows * D) mine[k] = merge(i / D, i % D, kWarps, here, &m_mine[k], &sum_mine[k]);
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kRows * D / kThreads; ++k) {
      const int i = k * kThreads + threadIdx.x;
      if (i < rows * D) {
        s_part[0][i / D][i % D] = mine[k];
        if (i % D == 0) {
          s_part[0][i / D][D] = m_mine[k];
          s_part[0][i / D][D + 1] = sum_mine[k];
        }
      }
    }
    __syncwarp();
    ptx::cluster_arrive();
    ptx::cluster_wait();
    if (ptx::cluster_ctarank() == 0) {
      const uint32_t base = ptx::smem_u32(&s_part[0][0][0]);
      auto there = [&](int s, int row, int col) { return ptx::ld_cluster_f32(ptx::map_to_cta(base + (uint32_t)(row * kX + col) * 4u, (uint32_t)s)); };
      for (int i = threadIdx.x; i < rows * D; i += kThreads) {
        float m, sum;
        const float acc = merge(i / D, i % D, p.splits, there, &m, &sum);
        finish(i / D, i % D, acc, m, sum);
      }
    }
    __syncwarp();
    ptx::cluster_arrive();   // nobody leaves while its shared memory may still be read
    ptx::cluster_wait();
  }
  __syncthreads();
  for (uint32_t left = (uint32_t)s_odd; left != 0u; left &= left - 1u) {   // (only where rows were finished)
    const int row = __ffs(left) - 1;
    if (row % kWarps == warp)
      paged::attend_row<__nv_bfloat16, D>(a, r, rq.q0 + row / p.G, x0 + row / p.G, kh * p.G + row % p.G, lane);
  }
}

}  // namespace

bool paged_attn_rows_takes(const PagedAttnArgs& a) { return (long long)a.max_q * (a.Hq / a.Hkv) <= kRows && a.Hkv <= 65535; }

int launch_paged_attn_rows(cascade_ctx* ctx, const PagedAttnArgs& a, cudaStream_t s) {
  RowArgs p;
  p.a = a;
  p.G = a.Hq / a.Hkv;
  int lg = 0;
  while ((1ll << lg) < a.page_size) ++lg;
  p.page_shift = 31 + lg;
  p.page_mul = (uint32_t)(((1ull << p.page_shift) + a.page_size - 1) / a.page_size);
  // splits: as many as keep the resident CTAs (three an SM) busy at once, each with at least two steps a warp
  const long long units = (long long)a.n_req * a.Hkv;
  const int span = a.window > 0 && (long long)a.window + a.sinks + a.max_q < a.max_kv ? a.window + a.sinks + a.max_q : a.max_kv;
  const int steps = cascade_detail::ceil_div(span > 0 ? span : 1, kChunk * kWarps);
  p.splits = 1;
  while (p.splits < 8 && units * p.splits * 2 <= 3ll * ctx->sm_count && steps >= 2 * p.splits) p.splits *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.splits, a.Hkv, a.n_req);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = p.splits;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  if (ctx->shape.D == 128)
    CASCADE_CUDA_TRY(cudaLaunchKernelEx(&cfg, k_paged_attn_rows<128>, p));
  else
    CASCADE_CUDA_TRY(cudaLaunchKernelEx(&cfg, k_paged_attn_rows<64>, p));
  return CASCADE_OK;
}
