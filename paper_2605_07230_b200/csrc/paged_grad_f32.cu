// The gradient of the attention over a paged cache with ordinary multiply-adds: 64 x 64 tiles of scores in shared memory.
//
// Products run on packed pairs (two multiply-adds an instruction): scores sum over pairs of a head's elements, outputs hold pairs of
// them.  A CTA owns 64 keys or 64 rows and walks over the other side; both passes are one launch (8 short sequences, 4 heads of 64:
// 90 us, in two launches 150 us).  Four sequences of 1000 tokens, 8 heads: 18 TFLOP/s (five products) at D = 64 and 128, the multiply-add
// units 43 % busy and shared memory 66 %: what bounds it is the latency of either with four warps a scheduler.  Requesting a step's
// operands one ahead needs registers for half as many warps: 14 % slower at D = 64, the same at 128.
#include <climits>

#include "paged.h"
#include "paged_grad.cuh"

namespace {

constexpr int kT = 64;              // rows and keys of a tile
constexpr int kThreads = 256;
constexpr int kSp = kT + 4;         // row of a tile of weights in shared memory

template <int D>
struct Cfg {
  static constexpr int kRow = D + 4;
  static constexpr int kSmem = (4 * kT * kRow + 2 * kT * kSp + 2 * kT) * (int)sizeof(float);
};

struct F32Args {
  PagedGradArgs g;
  int G;                      // query heads a key head
  paged::PageDiv page, group; // (divisions by multiplication)
};

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
// s[i][j] = sum_d x[ty + 16 i][d] y[tx + 16 j][d]
template <int D>
__device__ __forceinline__ void scores(const float* x, const float* y, int tx, int ty, float (&s)[4][4]) {
  constexpr int kRow = Cfg<D>::kRow;
  uint64_t acc[4][4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) acc[i][j] = 0;
#pragma unroll 4
  for (int d = 0; d < D; d += 4) {
    ulonglong2 a[4], b[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      a[i] = *reinterpret_cast<const ulonglong2*>(x + (ty + 16 * i) * kRow + d);
      b[i] = *reinterpret_cast<const ulonglong2*>(y + (tx + 16 * i) * kRow + d);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] = ptx::fma2(a[i].y, b[j].y, ptx::fma2(a[i].x, b[j].x, acc[i][j]));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float lo, hi;
      ptx::unpack2(acc[i][j], &lo, &hi);
      s[i][j] = lo + hi;
    }
}

// o[i][.] += sum_t w[t][4 my + i] x[t][4 mx + 64 m ..]: four rows of outputs, D / 16 elements each, as pairs
template <int D>
__device__ __forceinline__ void outputs(const float* w, const float* x, int mx, int my, uint64_t (&o)[4][D / 32]) {
  constexpr int kRow = Cfg<D>::kRow;
#pragma unroll 4
  for (int t = 0; t < kT; ++t) {
    const float4 a = *reinterpret_cast<const float4*>(w + t * kSp + 4 * my);
    const uint64_t aa[4] = {ptx::pack2(a.x, a.x), ptx::pack2(a.y, a.y), ptx::pack2(a.z, a.z), ptx::pack2(a.w, a.w)};
#pragma unroll
    for (int m = 0; m < D / 64; ++m) {
      const ulonglong2 b = *reinterpret_cast<const ulonglong2*>(x + t * kRow + 64 * m + 4 * mx);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        o[i][2 * m] = ptx::fma2(aa[i], b.x, o[i][2 * m]);
        o[i][2 * m + 1] = ptx::fma2(aa[i], b.y, o[i][2 * m + 1]);
      }
    }
  }
}

template <int D>
struct Tile {
  float *a, *b, *c, *d;       // [kT][D + 4] each
  float *w, *e;               // [kT][kSp]: weights and their gradients
  float *lse, *delta;         // [kT]
  __device__ __forceinline__ explicit Tile(float* s) {
    constexpr int n = kT * Cfg<D>::kRow;
    a = s;
    b = a + n;
    c = b + n;
    d = c + n;
    w = d + n;
    e = w + kT * kSp;
    lse = e + kT * kSp;
    delta = lse + kT;
  }
};

// Rows first .. first + 63 of (token, head of the group) of a key head: queries and output gradients, zeros behind the last.
template <int D>
__device__ __forceinline__ void load_rows(const F32Args& f, int q0, int kh, int first, int n_rows, const Tile<D>& t) {
  const PagedGradArgs& p = f.g;
  const PagedAttnArgs& a = p.a;
  const int col = threadIdx.x % (D / 4) * 4;
#pragma unroll
  for (int k = 0; k < kT * (D / 4) / kThreads; ++k) {
    const int row = threadIdx.x / (D / 4) + k * (kThreads * 4 / D), rr = first + row;
    float4 q = make_float4(0.f, 0.f, 0.f, 0.f), g = q;
    if (rr < n_rows) {
      const int tok = f.group.page(rr), head = kh * f.G + rr - tok * f.G;
      const long long token = q0 + tok;
      q = load4(static_cast<const float*>(a.q) + token * a.q_stride + head * D + col);
      g = load4(static_cast<const float*>(p.d_out) + (token * a.Hq + head) * D + col);
      if (col == 0) {
        const float2 st = p.stats[token * a.Hq + head];
        t.lse[row] = st.x;
        t.delta[row] = st.y;
      }
    }
    paged::store4(t.a + row * Cfg<D>::kRow + col, q);
    paged::store4(t.b + row * Cfg<D>::kRow + col, g);
  }
}
// Keys first .. first + 63 of a request and their values, zeros where there is none; there[] tells which.
template <int D>
__device__ __forceinline__ void load_keys(const F32Args& f, int r, int kh, int first, int kv, const Tile<D>& t, uint8_t* there) {
  const PagedAttnArgs& a = f.g.a;
  const int col = threadIdx.x % (D / 4) * 4;
  const int32_t* table = a.block_table + (size_t)r * a.table_stride;
  constexpr int kN = kT * (D / 4) / kThreads;
  int at[kN];                                                // pages first: their loads go together
#pragma unroll
  for (int k = 0; k < kN; ++k) {
    const int j = first + (int)threadIdx.x / (D / 4) + k * (kThreads * 4 / D);
    at[k] = j < kv ? table[f.page.page(j)] : -1;
  }
#pragma unroll
  for (int k = 0; k < kN; ++k) {
    const int row = threadIdx.x / (D / 4) + k * (kThreads * 4 / D), j = first + row;
    const bool is = at[k] >= 0 && at[k] < a.n_pages;
    if (j < kv && !is && col == 0) atomicOr(a.err, CASCADE_DEV_ERR_BAD_PAGE);
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f), v = x;
    if (is) {
      const long long off = (long long)at[k] * a.page_stride + ((long long)(j - f.page.page(j) * a.page_size) * a.Hkv + kh) * D;
      x = load4(static_cast<const float*>(a.k) + off + col);
      v = load4(static_cast<const float*>(a.v) + off + col);
    }
    paged::store4(t.c + row * Cfg<D>::kRow + col, x);
    paged::store4(t.d + row * Cfg<D>::kRow + col, v);
    if (col == 0) there[row] = is;
  }
}

// Results of four rows a thread; a row that is not finite is noted in odd[].
template <int D>
__device__ __forceinline__ void store_out(float* to, long long stride, const uint64_t (&o)[4][D / 32], float by, int mx, int my, int n, uint32_t* odd) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 4 * my + i;
    if (row >= n) continue;
#pragma unroll
    for (int m = 0; m < D / 64; ++m) {
      float4 v;
      ptx::unpack2(o[i][2 * m], &v.x, &v.y);
      ptx::unpack2(o[i][2 * m + 1], &v.z, &v.w);
      if (v.x * 0.f + v.y * 0.f + v.z * 0.f + v.w * 0.f != 0.f) atomicOr(&odd[row >> 5], 1u << (row & 31));
      paged::store4(to + row * stride + 64 * m + 4 * mx, make_float4(v.x * by, v.y * by, v.z * by, v.w * by));
    }
  }
}

// A tile of keys.
template <int D>
__device__ __forceinline__ void keys_pass(const F32Args& f, float* smem) {
  const PagedGradArgs& p = f.g;
  __shared__ uint8_t there[kT];
  __shared__ uint32_t odd[2];
  const Tile<D> t(smem);
  const PagedAttnArgs& a = p.a;
  const int G = f.G, kh = blockIdx.x % a.Hkv, k_first = blockIdx.x / a.Hkv * kT, r = blockIdx.y;
  paged::GradRequest rq;
  if (!paged::load_request(p, r, &rq) || k_first >= rq.kv) return;
  const int n_keys = min(kT, rq.kv - k_first), x0 = rq.kv - rq.nq;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  if (threadIdx.x < 2) odd[threadIdx.x] = 0u;
  load_keys<D>(f, r, kh, k_first, rq.kv, t, there);
  uint64_t dk[4][D / 32], dv[4][D / 32];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int m = 0; m < D / 32; ++m) dk[i][m] = dv[i][m] = 0;
  int lo, hi;
  paged::tokens_that_see(a, x0, rq.nq, k_first, k_first + n_keys - 1, &lo, &hi);
  for (int first = lo * G; first < hi * G; first += kT) {
    __syncthreads();
    load_rows<D>(f, rq.q0, kh, first, hi * G, t);
    __syncthreads();
    float s[4][4], g[4][4];
    scores<D>(t.a, t.c, tx, ty, s);
    scores<D>(t.b, t.d, tx, ty, g);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = ty + 16 * i, x = x0 + f.group.page(first + row);
      const float lse = t.lse[row], delta = t.delta[row];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = tx + 16 * j;
        const bool see = first + row < hi * G && there[key] && paged::sees(a, x, k_first + key);
        const float w = see ? paged::grad_weight<float>(s[i][j], a.scale, lse) : 0.f;
        t.w[row * kSp + key] = w;
        t.e[row * kSp + key] = see ? w * (g[i][j] - delta) : 0.f;
      }
    }
    __syncthreads();
    outputs<D>(t.w, t.b, tx, ty, dv);
    outputs<D>(t.e, t.a, tx, ty, dk);
  }
  __syncthreads();
  const long long to = (long long)rq.k0 + k_first;
  store_out<D>(static_cast<float*>(p.dk) + to * p.dk_stride + kh * D, p.dk_stride, dk, a.scale, tx, ty, n_keys, odd);
  store_out<D>(static_cast<float*>(p.dv) + to * p.dv_stride + kh * D, p.dv_stride, dv, 1.f, tx, ty, n_keys, odd);
  __syncthreads();
  // (a value that is no number, or too large, at a row that another key of the tile sees)
  for (int key = threadIdx.x / 32; key < n_keys; key += kThreads / 32)
    if (odd[key >> 5] >> (key & 31) & 1u) paged::grad_key<float, D>(p, r, rq, k_first + key, kh, threadIdx.x % 32);
}

// A block of rows.
template <int D>
__device__ __forceinline__ void rows_pass(const F32Args& f, float* smem) {
  const PagedGradArgs& p = f.g;
  __shared__ uint8_t there[kT];
  __shared__ uint32_t odd[2];
  const Tile<D> t(smem);
  const PagedAttnArgs& a = p.a;
  const int G = f.G, kh = blockIdx.x % a.Hkv, first = blockIdx.x / a.Hkv * kT, r = blockIdx.y;
  paged::GradRequest rq;
  if (!paged::load_request(p, r, &rq) || first >= rq.nq * G) return;
  const int n_rows = min(kT, rq.nq * G - first), x0 = rq.kv - rq.nq;
  const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
  if (threadIdx.x < 2) odd[threadIdx.x] = 0u;
  load_rows<D>(f, rq.q0, kh, first, rq.nq * G, t);
  uint64_t dq[4][D / 32];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int m = 0; m < D / 32; ++m) dq[i][m] = 0;
  const int x_first = x0 + first / G, x_last = x0 + (first + n_rows - 1) / G;
  const int begin = paged::window_begin(max(x_first, 0), a.window), sink_end = min(a.sinks, begin);
  for (int k_first = sink_end > 0 ? 0 : begin / kT * kT; k_first <= x_last;) {
    __syncthreads();
    load_keys<D>(f, r, kh, k_first, rq.kv, t, there);
    __syncthreads();
    float s[4][4], g[4][4];
    scores<D>(t.a, t.c, tx, ty, s);
    scores<D>(t.b, t.d, tx, ty, g);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = ty + 16 * i, x = x0 + f.group.page(first + row);
      const float lse = t.lse[row], delta = t.delta[row];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int key = tx + 16 * j;
        const bool see = row < n_rows && there[key] && paged::sees(a, x, k_first + key);
        t.e[key * kSp + row] = see ? paged::grad_weight<float>(s[i][j], a.scale, lse) * (g[i][j] - delta) : 0.f;
      }
    }
    __syncthreads();
    outputs<D>(t.e, t.c, tx, ty, dq);
    k_first += kT;
    if (k_first >= sink_end) k_first = max(k_first, begin / kT * kT);
  }
  // rows four by four: row index inside the block -> token and head
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = 4 * ty + i;
    if (row >= n_rows) continue;
    float* to = static_cast<float*>(p.dq) + (long long)(rq.q0 + (first + row) / G) * p.dq_stride + (kh * G + (first + row) % G) * D;
#pragma unroll
    for (int m = 0; m < D / 64; ++m) {
      float4 v;
      ptx::unpack2(dq[i][2 * m], &v.x, &v.y);
      ptx::unpack2(dq[i][2 * m + 1], &v.z, &v.w);
      if (v.x * 0.f + v.y * 0.f + v.z * 0.f + v.w * 0.f != 0.f) atomicOr(&odd[row >> 5], 1u << (row & 31));
      paged::store4(to + 64 * m + 4 * tx, make_float4(v.x * a.scale, v.y * a.scale, v.z * a.scale, v.w * a.scale));
    }
  }
  __syncthreads();
  for (int row = threadIdx.x / 32; row < n_rows; row += kThreads / 32)
    if (odd[row >> 5] >> (row & 31) & 1u)
      paged::grad_row<float, D>(p, r, rq.q0 + (first + row) / G, x0 + (first + row) / G, kh * G + (first + row) % G, threadIdx.x % 32);
}

template <int D>
__global__ void __launch_bounds__(kThreads, D == 64 ? 2 : 1) k_paged_grad_f32(const F32Args p) {
  extern __shared__ __align__(16) float smem[];
  if (blockIdx.z == 0)
    keys_pass<D>(p, smem);
  else
    rows_pass<D>(p, smem);
}

template <int D>
int launch(cascade_ctx* ctx, const PagedGradArgs& p, cudaStream_t s) {
  const PagedAttnArgs& a = p.a;
  const int G = a.Hq / a.Hkv;
  const F32Args f = {p, G, paged::page_div(a.page_size), paged::page_div(G)};
  const long long kv_blocks = ((long long)a.max_kv + kT - 1) / kT * a.Hkv, q_blocks = ((long long)a.max_q * G + kT - 1) / kT * a.Hkv;
  const long long blocks = kv_blocks > q_blocks ? kv_blocks : q_blocks;
  if (blocks > INT_MAX) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  CASCADE_TRY(configure_smem(ctx, PAGED_CFG_GRAD_F32, k_paged_grad_f32<D>, Cfg<D>::kSmem));   // (a context has one D)
  KernelScope ks(ctx, K_PAGED_GRAD, s);
  k_paged_grad_f32<D><<<dim3((unsigned)blocks, a.n_req, 2), kThreads, Cfg<D>::kSmem, s>>>(f);
  CASCADE_CUDA_TRY(cudaGetLastError());
  return CASCADE_OK;
}

}  // namespace

int launch_paged_grad_f32(cascade_ctx* ctx, const PagedGradArgs& p, cudaStream_t s) {
  return ctx->shape.D == 128 ? launch<128>(ctx, p, s) : launch<64>(ctx, p, s);
}
