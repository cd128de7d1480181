// Attention over a paged cache in fp32 on the tensor cores' 19-bit type, three products for one: every operand is split
// into its value rounded to that type and the remainder, and hi hi + hi lo + lo hi keeps about 22 bits.  (FMAs on tiles in
// shared memory, with far more instructions, took 25 us where this takes 20 us on 8 chunks of up to 130 tokens.)
//
// One CTA of four warps per (KV split, key head x row block, request), a row being (token, query head of the group).  As in
// the 16-bit kernel for few rows, a warp takes 16 keys at a time straight from memory into operand registers, keys and
// values on M, eight rows on N.  Single tokens and short chunks (up to eight rows) share the keys out between the warps;
// beyond that every warp has eight rows of its own and walks over all keys, which the four then share in the L1.
// 8 chunks of 47 to 122 tokens over 109 to 397 keys, 4 heads of 64: 20 us.  The case has four splits of at most 7 steps a warp,
// 1170 instructions a step with start and merge (operands are split by every warp for itself); 2.4 warps a scheduler use 31 % of
// the issue slots of active SMs, and an SM is active for 69 % of the time (512 uneven CTAs).
// D = 128 needs more than the 255 registers there are and spills some 60 words a thread; long chunks run at 13 to 16 TFLOP/s.
// The tensor cores add with truncation, so long sums stay out of them: the outputs of 16 keys are summed apart and added to
// the running fp32 outputs by ordinary additions, and scores are summed over at most 64 elements at a time.
// Splits of the keys are the CTAs of a cluster and meet through distributed shared memory.
#include <climits>

#include "paged.h"
#include "paged_attn.cuh"

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kChunk = 16;      // keys per step of a warp
constexpr int kRows = 8;        // rows of a warp
constexpr float kLazy = 8.f;

struct F32Args {
  PagedAttnArgs a;
  int G, splits, n_rb;          // query heads a key head; KV splits; row blocks of the longest request
  paged::PageDiv div;
};

// x = hi + lo, both of the 19-bit type up to what the products drop
__device__ __forceinline__ void split(uint32_t x, uint32_t* hi, uint32_t* lo) {
  asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(*hi) : "f"(__uint_as_float(x)));
  *lo = __float_as_uint(__uint_as_float(x) - __uint_as_float(*hi));
}
__device__ __forceinline__ void mma1688(float* c, const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 ld_shared_by_warps(const void* p) {   // through the L1: the other warps read it too
  uint4 v;
  asm volatile("ld.global.nc.L2::256B.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// kByRow: the warps have rows of their own (else: keys of their own).
template <int D, bool kByRow>
__global__ void __launch_bounds__(kThreads, D == 64 ? 3 : 2) k_paged_attn_f32(const F32Args p) {
  constexpr int kQ = D / 16;                     // 16-byte pieces of a key row per lane
  constexpr int kV = D / 32;                     // 16-byte pieces of a value row per lane
  constexpr int kO = D / 16;                     // output products
  constexpr int kX = paged::part_stride(D);
  constexpr int kStep = kByRow ? 1 : kWarps;
  constexpr int kBlock = kByRow ? kWarps * kRows : kRows;
  __shared__ __align__(16) float s_part[paged::part_floats(D, 1, kWarps * kRows)];   // (no fewer than kWarps parts of kRows need)
  __shared__ bool s_lost[kWarps];                // the warp met a page outside the pool
  const PagedAttnArgs& a = p.a;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
  // (the splits of one cluster lie side by side; x is the one dimension of a grid with room for long passes)
  const int unit = blockIdx.x / p.splits, split_i = blockIdx.x - unit * p.splits;
  const int kh = unit / p.n_rb, rb = unit % p.n_rb, r = blockIdx.y;
  paged::Request rq;
  const bool valid = paged::load_request(a, r, &rq);
  const int row0 = rb * kBlock;
  const int rows = valid ? max(0, min(kBlock, rq.nq * p.G - row0)) : 0;
  if (rows == 0) return;                         // (the same in all CTAs of a cluster)
  if (p.splits > 1) ptx::cluster_arrive();       // (waited for in merge_and_store)
  if (lane == 0) s_lost[warp] = false;
  const int w_row = kByRow ? warp * kRows : 0;                       // this warp's first row of the block
  const int w_rows = max(0, min(kRows, rows - w_row));
  const int x0 = rq.kv - rq.nq;                                      // position of the request's first new token
  const int x_first = x0 + (row0 + w_row) / p.G, x_last = w_rows > 0 ? x0 + (row0 + w_row + w_rows - 1) / p.G : -1;

  // 16-key steps that any row of the warp sees: [0, n_sink) and [n_sink + skip, ...)
  int n = 0, n_sink = 0, skip = 0;
  if (x_last >= 0) {
    const int lo = paged::window_begin(x_first, a.window), lo_c = max(lo, 0) / kChunk;
    n_sink = min((min(a.sinks, lo) + kChunk - 1) / kChunk, lo_c);
    skip = lo_c - n_sink;
    n = x_last / kChunk + 1 - skip;
  }

  const int per = (n + p.splits - 1) / p.splits;
  const int c_end = min(n, (split_i + 1) * per);
  int c = split_i * per + (kByRow ? 0 : warp);

  // queries: lane (g, t) holds elements 16 j + 4 t .. + 3 of row g
  uint32_t q[kQ][4];
  {
    const int row = row0 + w_row + g;
    const bool there = g < w_rows;
    const float* src = static_cast<const float*>(a.q);
    if (there) src += (long long)(rq.q0 + row / p.G) * a.q_stride + (kh * p.G + row % p.G) * D;
#pragma unroll
    for (int j = 0; j < kQ; ++j) {
      const uint4 v = there ? *reinterpret_cast<const uint4*>(src + 16 * j + 4 * t) : make_uint4(0, 0, 0, 0);
      q[j][0] = v.x;
      q[j][1] = v.y;
      q[j][2] = v.z;
      q[j][3] = v.w;
    }
  }
  int x_row[2];                                  // positions of rows 2 t + i; -1: no such row
#pragma unroll
  for (int i = 0; i < 2; ++i) x_row[i] = 2 * t + i < w_rows ? x0 + (row0 + w_row + 2 * t + i) / p.G : -1;

  const float* k_base = static_cast<const float*>(a.k) + kh * D;
  const float* v_base = static_cast<const float*>(a.v) + kh * D;
  const int row_elems = a.Hkv * D;
  const int32_t* table = a.block_table + (size_t)r * a.table_stride;
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
  auto fetch = [&](const float* src) { return kByRow ? ld_shared_by_warps(src) : paged::ld_stream(src); };
  uint4 kr[2][kQ], vr[4][kV];
  auto load_k = [&](int key0, const long long* off) {
#pragma unroll
    for (int h = 0; h < 2; ++h) {                // keys g and 8 + g
      const bool there = off[h] >= 0 && key0 + 8 * h + g < rq.kv;
      const float* src = k_base + (there ? off[h] : 0) + (there ? g : 0) * row_elems + 4 * t;
#pragma unroll
      for (int j = 0; j < kQ; ++j) kr[h][j] = there ? fetch(src + 16 * j) : make_uint4(0, 0, 0, 0);
    }
  };
  auto load_v = [&](int key0, const long long* off) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {                // keys t, t + 4, t + 8, t + 12
      const int in = t + 4 * (i & 1), h = i >> 1;
      const bool there = off[h] >= 0 && key0 + 8 * h + in < rq.kv;
      const float* src = v_base + (there ? off[h] : 0) + (there ? in : 0) * row_elems + 4 * g;
#pragma unroll
      for (int j = 0; j < kV; ++j) vr[i][j] = there ? fetch(src + 32 * j) : make_uint4(0, 0, 0, 0);
    }
  };

  float o[kO][4];
#pragma unroll
  for (int e = 0; e < kO; ++e) o[e][0] = o[e][1] = o[e][2] = o[e][3] = 0.f;
  float ref[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};   // of rows 2 t + i
  const float sc = a.scale * paged::kLog2e;

  long long off_next[2] = {-1, -1};
  int key0 = 0;
  if (c < c_end) {
    key0 = first_key(c);
    const long long off[2] = {page_off(key0), page_off(key0 + 8)};
    load_k(key0, off);
    load_v(key0, off);
    if (c + kStep < c_end) {
      off_next[0] = page_off(first_key(c + kStep));
      off_next[1] = page_off(first_key(c + kStep) + 8);
    }
  }
  for (; c < c_end; c += kStep) {
    const bool more = c + kStep < c_end;
    const int next0 = more ? first_key(c + kStep) : 0;
    long long off_after[2] = {-1, -1};
    if (c + 2 * kStep < c_end) {
      off_after[0] = page_off(first_key(c + 2 * kStep));
      off_after[1] = page_off(first_key(c + 2 * kStep) + 8);
    }
    // scores: s[2 h + i] is key key0 + 8 h + g, row 2 t + i
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int part = 0; part < D / 64; ++part) {
      float hh[4] = {0.f, 0.f, 0.f, 0.f}, mixed[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int j = 4 * part; j < 4 * part + 4; ++j) {
#pragma unroll
        for (int e = 0; e < 4; e += 2) {         // elements e and e + 1 of the pieces stand at k = t and t + 4
          uint32_t kh_[4], kl[4], qh[2], ql[2];
          split(word(kr[0][j], e), &kh_[0], &kl[0]);
          split(word(kr[1][j], e), &kh_[1], &kl[1]);
          split(word(kr[0][j], e + 1), &kh_[2], &kl[2]);
          split(word(kr[1][j], e + 1), &kh_[3], &kl[3]);
          split(q[j][e], &qh[0], &ql[0]);
          split(q[j][e + 1], &qh[1], &ql[1]);
          mma1688(hh, kh_, qh[0], qh[1]);
          mma1688(mixed, kh_, ql[0], ql[1]);
          mma1688(mixed, kl, qh[0], qh[1]);
        }
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) s[k] += hh[k] + mixed[k];
    }
    if (more) load_k(next0, off_next);
    // steps behind the first row's position or at a window's edge look closer
    const bool edge = key0 + kChunk - 1 > x_first || (a.window > 0 && key0 <= x_last - a.window);
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      float v = s[k] * sc;
      if (edge) {
        const int j = key0 + 8 * (k >> 1) + g, x = x_row[k & 1];
        const bool sees = j <= x && (j >= paged::window_begin(x, a.window) || j < a.sinks);
        v = sees ? v : -INFINITY;
      }
      s[k] = v;
    }
    // raise the reference where a score passes it by more than kLazy (or the row had none)
    float mx[2];
    bool raise = false;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      mx[i] = fmaxf(s[i], s[2 + i]);
      raise = raise || mx[i] > ref[i] + kLazy || (ref[i] == -INFINITY && mx[i] > -INFINITY);
    }
    if (__any_sync(0xffffffffu, raise)) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], x));
        float alpha = 1.f;
        if (mx[i] > ref[i]) {
          alpha = ref[i] == -INFINITY ? 0.f : exp2f(ref[i] - mx[i]);
          ref[i] = mx[i];
        }
        l[i] *= alpha;
#pragma unroll
        for (int e = 0; e < kO; ++e) {
          o[e][i] *= alpha;
          o[e][2 + i] *= alpha;
        }
      }
    }
    const float m[2] = {ref[0] == -INFINITY ? 0.f : ref[0], ref[1] == -INFINITY ? 0.f : ref[1]};
    float w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      w[k] = exp2f(s[k] - m[k & 1]);
      l[k & 1] += w[k];
    }
    // the weights as the B operand: row g, keys 8 h + t and 8 h + t + 4 (from lane (key, row / 2))
    uint32_t wh[4], wl[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int src = (t + 4 * (i & 1)) * 4 + (g >> 1), h = i >> 1;
      const float w0 = __shfl_sync(0xffffffffu, w[2 * h], src), w1 = __shfl_sync(0xffffffffu, w[2 * h + 1], src);
      split(__float_as_uint((g & 1) ? w1 : w0), &wh[i], &wl[i]);
    }
    // outputs: product (jj, e) holds elements 64 jj + 4 g + e and 64 jj + 32 + 4 g + e
#pragma unroll
    for (int jj = 0; jj < D / 64; ++jj)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          uint32_t vh[4], vl[4];
          split(word(vr[2 * h][2 * jj], e), &vh[0], &vl[0]);
          split(word(vr[2 * h][2 * jj + 1], e), &vh[1], &vl[1]);
          split(word(vr[2 * h + 1][2 * jj], e), &vh[2], &vl[2]);
          split(word(vr[2 * h + 1][2 * jj + 1], e), &vh[3], &vl[3]);
          mma1688(acc, vl, wh[2 * h], wh[2 * h + 1]);
          mma1688(acc, vh, wl[2 * h], wl[2 * h + 1]);
          mma1688(acc, vh, wh[2 * h], wh[2 * h + 1]);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) o[4 * jj + e][k] += acc[k];
      }
    if (more) load_v(next0, off_next);
    key0 = next0;
    off_next[0] = off_after[0];
    off_next[1] = off_after[1];
  }

  // ---- partial results: [warp][row] with keys shared out, [row of the block] with rows shared out ----
  // (keys of a lost page went in as zeros: a sum that is no number has the rows computed again without them)
  __syncwarp();
  const bool lost = s_lost[warp];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
#pragma unroll
    for (int x = 4; x < 32; x <<= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
    if (2 * t + i < w_rows) {
      float* x = s_part + (warp * kRows + 2 * t + i) * kX;
#pragma unroll
      for (int jj = 0; jj < D / 64; ++jj)
#pragma unroll
        for (int half = 0; half < 2; ++half)
          *reinterpret_cast<float4*>(x + 64 * jj + 32 * half + 4 * g) =
              make_float4(o[4 * jj][2 * half + i], o[4 * jj + 1][2 * half + i], o[4 * jj + 2][2 * half + i], o[4 * jj + 3][2 * half + i]);
      if (g == 0) {
        x[D] = ref[i];
        x[D + 1] = lost ? NAN : l[i];
      }
    }
  }
  paged::merge_and_store<float, D, kByRow ? 1 : kWarps, kBlock>(a, r, rq.q0, x0, kh, row0, rows, p.G, p.splits, s_part, kByRow ? kBlock : kRows);
}

template <int D, bool kByRow>
int launch(cascade_ctx* ctx, const PagedAttnArgs& a, cudaStream_t s) {
  F32Args p;
  p.a = a;
  p.G = a.Hq / a.Hkv;
  p.div = paged::page_div(a.page_size);
  constexpr int kBlock = kByRow ? kWarps * kRows : kRows;
  const long long row_blocks = ((long long)a.max_q * p.G + kBlock - 1) / kBlock;
  if (row_blocks * a.Hkv > INT_MAX / 8) return CASCADE_ERR_UNSUPPORTED_SHAPE;   // (the queries would not fit a GPU)
  p.n_rb = (int)row_blocks;
  // splits: up to four CTAs an SM, each with at least four steps a warp.  Three (D = 128: two) fit at once; the row blocks' work
  // is uneven, and a queue behind them fills the gaps: 8 chunks of up to 130 tokens, 4 heads of 64, take 20 us with up to four,
  // 29 with up to three or two, 26 with up to eight; 4 chunks of 30 to 60 tokens, 8 heads of 128, 47, 43, 42 and 47; 16 single
  // tokens over 1000 to 2000 keys, 8 heads of 128, 77, 76, 76 and 89.
  const long long units = (long long)a.n_req * a.Hkv * p.n_rb;
  const long long window = (long long)a.window + a.sinks + kBlock;
  const long long span = a.window > 0 && window < a.max_kv ? window : a.max_kv;
  const long long steps = (span + kChunk - 1) / kChunk / (kByRow ? 1 : kWarps);
  p.splits = 1;
  while (p.splits < 8 && units * p.splits * 2 <= 4ll * ctx->sm_count && steps >= 4ll * p.splits) p.splits *= 2;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.splits * a.Hkv * p.n_rb, a.n_req);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = p.splits;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  CASCADE_CUDA_TRY(cudaLaunchKernelEx(&cfg, k_paged_attn_f32<D, kByRow>, p));
  return CASCADE_OK;
}

}  // namespace

int launch_paged_attn_f32(cascade_ctx* ctx, const PagedAttnArgs& a, cudaStream_t s) {
  // 16 single tokens over 1000 to 2000 keys, 8 heads of 128: 78 us with keys of their own for the warps, 227 us by rows;
  // 8 tokens of 8 requests: 11 us either way
  const bool few = (long long)a.max_q * (a.Hq / a.Hkv) <= kRows;
  if (ctx->shape.D == 128) return few ? launch<128, false>(ctx, a, s) : launch<128, true>(ctx, a, s);
  return few ? launch<64, false>(ctx, a, s) : launch<64, true>(ctx, a, s);
}
