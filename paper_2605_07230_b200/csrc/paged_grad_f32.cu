// The gradient of the attention over a paged cache in 32 bits, on the tensor cores.
//
// A 32-bit number is the sum of three bf16 numbers h + m + l (8 bits each, to the last bit: m up to 2^-8 of it, l up to 2^-17); of a
// product's nine terms six are formed, ll, ml and lm are left out (2^-24 of the product).  They go into the accumulator the smallest first,
// so that what the tensor cores' additions cut off counts at the size of hh alone; products of one step start from zero and are added
// up in registers.
//
// A CTA owns 128 keys, or 128 rows (token, query head of the group), and walks over the other side 64 (D = 64) or 32 lines at a time:
//     S = X1 Y1^T    P = exp(c S - lse)    dP = X2 Y2^T    dS = P (dP - delta)        keys: dV += P Y2, dK += dS Y1;  rows: dQ += dS Y1
// with X1, X2 its own keys and values (queries and output gradients), Y1, Y2 the others'.  A lane of the tensor memory is one of its
// own lines, so all that a thread sums belongs to one line.  P and dS are the products' operands from the tensor memory, where the l
// of X1 and X2 stay too (there is no room for them beside two steps of Y).  Both passes are one launch.
//
// 8 sequences of 47 to 450 tokens, 4 heads of 64: 31 us (64 x 64 tiles of multiply-adds: 90 us).  4 of 1000 tokens, 8 heads: 141 us at
// D = 64, 289 us at 128, 71 TFLOP/s of the five products that have to be (multiply-adds: 18); 42 products of that size are formed for
// them, 600 TFLOP/s.  A step of 64 takes 5600 cycles where its 96 products, issued one by one, take 4300; loads, splits and weights of
// the next step lie beside them.
#include <climits>

#include "paged.h"
#include "paged_grad.cuh"

namespace {

constexpr int kOwn = 128;
constexpr int kComputeWarps = 8, kProducts = kComputeWarps;            // the last warp issues products
// A launch's 168 registers a thread are dealt out anew: 224 for the eight warps that compute, 56 for four of which one is at work
// (nine warps of 168: 38 and 156 us for the two cases above that take 31 and 141).
constexpr int kThreads = (kComputeWarps + 4) * 32;

template <int D>
struct Cfg {
  static constexpr int kStep = D == 64 ? 64 : 32;                                // lines walked over at a time
  static constexpr int kCols = kStep / 2;                                        // of them a thread's
  static constexpr int kLinesAtOnce = kComputeWarps * 32 * 8 / D, kN = kStep / kLinesAtOnce;   // loads: 8 elements a thread of kN lines
  // bytes: h and m of X1 and X2, two buffers of h, m, l of Y1 and Y2
  static constexpr int kOwnPart = kOwn * D * 2, kStepPart = kStep * D * 2, kStepTile = 3 * kStepPart;
  static constexpr int kX2 = 2 * kOwnPart, kY = 4 * kOwnPart, kTiles = kY + 4 * kStepTile;
  // columns of the tensor memory: S and dP (P and dS as operands, 3 kStep / 2 columns, over them), results, l of X1 and X2
  static constexpr int kS = 0, kDp = 2 * kStep, kOut = 4 * kStep, kXl = 384;
  static_assert(kOut + 2 * D <= kXl && kXl + D <= 512, "tensor memory");
};

struct Shared {
  uint64_t s_full, dp_full, out_full, p_full, ds_full, y_full, alive;
  int abort_flag;
  uint32_t tmem;
  uint32_t odd[kOwn / 32];                               // own lines with a result that is not finite
  __align__(16) float lse[2][64], delta[2][64];          // of the rows walked over
  uint8_t there[2][64], own_there[kOwn];                 // keys whose pages are in the pool
};

struct F32Args {
  PagedGradArgs g;
  int G;                      // query heads a key head
  int split_keys, split_rows; // CTAs (a cluster) that share the walk of a tile in either pass
  paged::PageDiv page, group; // (divisions by multiplication)
};

// Lines of one (request, key head): keys and values, or queries and output gradients (of rows (token, head)), up to `end`.
template <bool kKeys>
struct Lines {
  const F32Args& f;
  const int32_t* table;
  int head, q0, end;
  __device__ __forceinline__ int page(int j) const { return kKeys && j < end ? table[f.page.page(j)] : -1; }
  // -> where line j's elements are; false: there is none (zeros)
  __device__ __forceinline__ bool find(int j, int page, int D, const float** first, const float** second) const {
    const PagedGradArgs& p = f.g;
    const PagedAttnArgs& a = p.a;
    if (j >= end) return false;
    if (kKeys) {
      if (page < 0 || page >= a.n_pages) {
        atomicOr(a.err, CASCADE_DEV_ERR_BAD_PAGE);
        return false;
      }
      const long long off = (long long)page * a.page_stride + ((long long)(j - f.page.page(j) * a.page_size) * a.Hkv + head) * D;
      *first = static_cast<const float*>(a.k) + off;
      *second = static_cast<const float*>(a.v) + off;
    } else {
      const int tok = f.group.page(j);
      const long long token = q0 + tok, h = head * f.G + j - tok * f.G;
      *first = static_cast<const float*>(a.q) + token * a.q_stride + h * D;
      *second = static_cast<const float*>(p.d_out) + (token * a.Hq + h) * D;
    }
    return true;
  }
};

// A pair of numbers as three pairs of bf16.
__device__ __forceinline__ void split2(float x0, float x1, uint32_t* h, uint32_t* m, uint32_t* l) {
  auto rest = [&](uint32_t part) {
    x0 -= __uint_as_float(part << 16);
    x1 -= __uint_as_float(part & 0xffff0000u);
  };
  *h = ptx::pack_bf16x2(x0, x1);
  rest(*h);
  *m = ptx::pack_bf16x2(x0, x1);
  rest(*m);
  *l = ptx::pack_bf16x2(x0, x1);
}
// Eight elements of a line -> their 16 bytes of the three parts.
__device__ __forceinline__ void store_parts(uint32_t h_at, uint32_t m_at, uint32_t l_at, const float4& x, const float4& y) {
  uint32_t h[4], m[4], l[4];
  split2(x.x, x.y, &h[0], &m[0], &l[0]);
  split2(x.z, x.w, &h[1], &m[1], &l[1]);
  split2(y.x, y.y, &h[2], &m[2], &l[2]);
  split2(y.z, y.w, &h[3], &m[3], &l[3]);
  ptx::st_shared_v4(h_at, h[0], h[1], h[2], h[3]);
  ptx::st_shared_v4(m_at, m[0], m[1], m[2], m[3]);
  ptx::st_shared_v4(l_at, l[0], l[1], l[2], l[3]);
}
// Place of the 16 bytes `chunk` of a line in a tile whose rows are swizzled over 128 bytes.
template <int kLines>
__device__ __forceinline__ uint32_t place(int line, int chunk) {
  return (chunk >> 3) * (kLines * 128) + line * 128 + (((chunk & 7) ^ (line & 7)) << 4);
}

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ void ld_shared_v4(uint32_t addr, uint32_t* x) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ bool elect_one() {
  uint32_t is;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
  return is != 0;
}
__device__ __forceinline__ uint64_t plus(uint64_t desc, uint32_t bytes) { return desc + (bytes >> 4); }
// The terms from the smallest to the largest, l h, h l, m m, m h, h m, h h: the parts of A and of B.
__device__ __forceinline__ int part_a(int term) { return (0x001102 >> (4 * term)) & 15; }
__device__ __forceinline__ int part_b(int term) { return (0x010120 >> (4 * term)) & 15; }

// acc[128 x kStep] = X Y^T, h and m of X in shared memory, l in the tensor memory
template <int D>
__device__ __forceinline__ void scores(uint32_t acc, uint32_t x, uint32_t xl, uint32_t y) {
  constexpr int kStep = Cfg<D>::kStep;
  const uint32_t idesc = ptx::umma_idesc_bf16(kOwn, kStep);
  const uint64_t dx = ptx::umma_desc_sw128(x), dy = ptx::umma_desc_sw128(y);
  auto own = [](int ks) { return (ks >> 2) * (kOwn * 128) + (ks & 3) * 32; };
  auto other = [](int ks) { return (ks >> 2) * (kStep * 128) + (ks & 3) * 32; };
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) ptx::umma_bf16_ts(acc, xl + ks * 8, plus(dy, other(ks)), idesc, ks != 0);
#pragma unroll 1
  for (int t = 1; t < 6; ++t) {
    const uint64_t a = plus(dx, part_a(t) * Cfg<D>::kOwnPart), b = plus(dy, part_b(t) * Cfg<D>::kStepPart);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks) ptx::umma_bf16(acc, plus(a, own(ks)), plus(b, other(ks)), idesc, 1);
  }
}
// acc[128 x D] = W Y with W [128][kStep] in the tensor memory, kStep / 2 columns a part
template <int D>
__device__ __forceinline__ void results(uint32_t acc, uint32_t w, uint32_t y) {
  constexpr int kStep = Cfg<D>::kStep;
  const uint32_t idesc = ptx::umma_idesc_bf16_b_mn(kOwn, D);
  const uint64_t dy = ptx::umma_desc_sw128_strides(y, kStep * 128, 1024);
#pragma unroll 1
  for (int t = 0; t < 6; ++t) {
    const uint64_t b = plus(dy, part_b(t) * Cfg<D>::kStepPart);
#pragma unroll
    for (int ks = 0; ks < kStep / 16; ++ks)
      ptx::umma_bf16_ts(acc, w + part_a(t) * (kStep / 2) + ks * 8, plus(b, ks * 2048), idesc, ks != 0 || t != 0);
  }
}

// Columns of the tensor memory (after the wait).
__device__ __forceinline__ void load(uint32_t taddr, float (&v)[16]) { ptx::tmem_ld16(taddr, v); }
__device__ __forceinline__ void load(uint32_t taddr, float (&v)[32]) { ptx::tmem_ld32(taddr, v); }
// Weights of a lane as an operand's columns of each part, `gap` columns apart.
template <int kCols>
__device__ __forceinline__ void store_operand(uint32_t taddr, int gap, const float (&w)[kCols]) {
  uint32_t x[3][kCols / 2];
#pragma unroll
  for (int k = 0; k < kCols / 2; ++k) split2(w[2 * k], w[2 * k + 1], &x[0][k], &x[1][k], &x[2][k]);
#pragma unroll
  for (int part = 0; part < 3; ++part) {
    if (kCols == 32)
      ptx::tmem_st16_async(taddr + part * gap, x[part]);
    else
      ptx::tmem_st8_async(taddr + part * gap, x[part]);
  }
  ptx::tmem_wait_st();
}
// Bits lo .. hi - 1 of a word.
__device__ __forceinline__ uint32_t bits(int lo, int hi) {
  auto below = [](int n) { return n >= 32 ? 0xffffffffu : (1u << max(n, 0)) - 1u; };
  return below(hi) & ~below(lo);
}

__device__ __forceinline__ void cluster_meet() {
  __syncwarp();
  ptx::cluster_arrive();
  ptx::cluster_wait();
}

// One CTA's tile of keys (kKeys) or block of rows; of a cluster of `splits` each takes every splits-th step, and their results
// are added up by pairs, pairs of pairs and so on.  Per step:
//   warps 0-7   | loads of the next step   P   results of the last step added up   next step into shared memory   dS
//   products    | last dK or dQ   dP                                               dV   next S
// Every wait of a compute warp is made, in vain too, so that the two warps of 32 lines stay beside each other.
template <int D, bool kKeys>
__device__ __forceinline__ void pass(const F32Args& f, uint8_t* smem, Shared& sh) {
  using C = Cfg<D>;
  constexpr int kStep = C::kStep, kCols = C::kCols, kN = C::kN, kAtOnce = C::kLinesAtOnce;
  const PagedGradArgs& p = f.g;
  const PagedAttnArgs& a = p.a;
  const int splits = kKeys ? f.split_keys : f.split_rows, rank = blockIdx.x % splits, tile = blockIdx.x / splits;
  const int G = f.G, head = tile % a.Hkv, r = blockIdx.y;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  paged::GradRequest rq;
  if (!paged::load_request(p, r, &rq)) return;
  const int x0 = rq.kv - rq.nq, lines = kKeys ? rq.kv : rq.nq * G;
  int own = tile / a.Hkv;                                        // the longest first: keys in order, rows from the end
  if (!kKeys) own = (lines + kOwn - 1) / kOwn - 1 - own;
  const int first = own * kOwn;
  if (first < 0 || first >= lines) return;
  const int n_own = min(kOwn, lines - first);

  // what is walked over: rows [walk, end) that see any of the keys, or keys up to the last that a row sees
  int walk, end, begin = 0, sink_end = 0;
  if (kKeys) {
    paged::rows_that_see(a, x0, rq.nq, G, first, first + n_own - 1, &walk, &end);
  } else {
    begin = paged::window_begin(max(x0 + first / G, 0), a.window) / kStep * kStep;
    sink_end = min(a.sinks, begin);
    walk = sink_end > 0 ? 0 : begin;
    end = x0 + (first + n_own - 1) / G + 1;
  }
  auto step = [&](int at) {
    at += kStep;
    return kKeys || at < sink_end ? at : max(at, begin);
  };
  auto next = [&](int at) {
    for (int i = 0; i < splits && at < end; ++i) at = step(at);
    return at;
  };
  for (int i = 0; i < rank && walk < end; ++i) walk = step(walk);
  if (tid == 0) {
    for (uint64_t* b : {&sh.s_full, &sh.dp_full, &sh.out_full}) ptx::mbar_init(b, 1);
    for (uint64_t* b : {&sh.p_full, &sh.ds_full, &sh.y_full}) ptx::mbar_init(b, kComputeWarps);
    ptx::fence_mbar_init();
    sh.abort_flag = 0;
    sh.alive = 0;
  }
  if (tid < kOwn / 32) sh.odd[tid] = 0u;
  if (warp == kProducts) {
    ptx::tmem_alloc(&sh.tmem, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = sh.tmem, base = ptx::smem_u32(smem);
  auto y_tile = [&](int buf, int which) { return base + C::kY + (2 * buf + which) * C::kStepTile; };
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    const bool ok = __all_sync(0xffffffffu, ptx::mbar_wait_short(bar, parity & 1u, &sh.abort_flag, a.err, a.wait_ns, &sh.alive));
    ptx::tc_fence_after();
    return ok;
  };
  bool ok = true;

  if (warp >= kComputeWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
    int at = warp == kProducts ? walk : end, buf = 0;
    if (at < end && (ok = wait(&sh.y_full, 0)) && elect_one()) {
      scores<D>(tmem + C::kS, base, tmem + C::kXl, y_tile(0, 0));
      ptx::umma_commit(&sh.s_full);
      scores<D>(tmem + C::kDp, base + C::kX2, tmem + C::kXl + D / 2, y_tile(0, 1));
      ptx::umma_commit(&sh.dp_full);
    }
    for (int i = 0; ok && at < end; ++i, buf ^= 1) {
      at = next(at);
      const bool more = at < end;
      if (!(ok = wait(&sh.p_full, i))) break;
      if (kKeys && elect_one()) results<D>(tmem + C::kOut + D, tmem + C::kS, y_tile(buf, 1));
      if (more) {
        if (!(ok = wait(&sh.y_full, i + 1))) break;
        if (elect_one()) {
          scores<D>(tmem + C::kS, base, tmem + C::kXl, y_tile(buf ^ 1, 0));
          ptx::umma_commit(&sh.s_full);
        }
      }
      if (!(ok = wait(&sh.ds_full, i))) break;
      if (elect_one()) {
        results<D>(tmem + C::kOut, tmem + C::kDp, y_tile(buf, 0));
        ptx::umma_commit(&sh.out_full);
        if (more) {
          scores<D>(tmem + C::kDp, base + C::kX2, tmem + C::kXl + D / 2, y_tile(buf ^ 1, 1));
          ptx::umma_commit(&sh.dp_full);
        }
      }
    }
    __syncwarp();
    if (!__syncthreads_and(ok)) __nanosleep(1000000);                  // products still in flight
    for (int n = 1; n < splits; n *= 2) cluster_meet(), cluster_meet();
    __syncthreads();
    ptx::tc_fence_after();
    if (warp == kProducts) ptx::tmem_dealloc(tmem, 512);
    return;
  }
  asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");

  const int32_t* table = a.block_table + (size_t)r * a.table_stride;
  const Lines<kKeys> mine = {f, table, head, rq.q0, lines};
  const Lines<!kKeys> others = {f, table, head, rq.q0, kKeys ? end : rq.kv};
  auto all = [] { asm volatile("bar.sync 1, %0;" ::"n"(kComputeWarps * 32) : "memory"); };          // the compute warps
  auto both = [&] { asm volatile("bar.sync %0, 64;" ::"r"(2 + (warp & 3)) : "memory"); };            // the two warps of 32 lines
  const int chunk = tid % (D / 8), line0 = tid / (D / 8);              // a thread's 8 elements of lines line0, line0 + kAtOnce, ...
  const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
  float4 y[kN][4];                                                     // a step's elements on their way: Y1, Y2
  float2 st[kN];                                                       // its rows' statistics, or whether its keys are there
  int page[kN];                                                        // the pages of the step after that
  auto pages = [&](int at) {
#pragma unroll
    for (int k = 0; k < kN; ++k) page[k] = others.page(at + line0 + k * kAtOnce);
  };
  auto request = [&](int at) {
#pragma unroll
    for (int k = 0; k < kN; ++k) {
      const int j = at + line0 + k * kAtOnce;
      const float *y1 = nullptr, *y2 = nullptr;
      const bool is = others.find(j, page[k], D, &y1, &y2);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[k][e] = is ? load4((e < 2 ? y1 : y2) + 8 * chunk + 4 * (e & 1)) : zero;
      st[k] = make_float2(is, 0.f);
      if (kKeys && is && chunk == 0) {
        const int tok = f.group.page(j);
        st[k] = p.stats[(long long)(rq.q0 + tok) * a.Hq + head * G + j - tok * G];
      }
    }
  };
  auto put = [&](int buf) {
#pragma unroll
    for (int k = 0; k < kN; ++k) {
      const int line = line0 + k * kAtOnce;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t at = y_tile(buf, e) + place<kStep>(line, chunk);
        store_parts(at, at + C::kStepPart, at + 2 * C::kStepPart, y[k][2 * e], y[k][2 * e + 1]);
      }
      if (chunk != 0) continue;
      if (kKeys)
        sh.lse[buf][line] = st[k].x, sh.delta[buf][line] = st[k].y;
      else
        sh.there[buf][line] = st[k].x != 0.f;
    }
    ptx::fence_proxy_async_smem();
    ptx::tc_fence_before();
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(&sh.y_full);
  };

  // ---- X1 and X2; their l by way of the steps' place into the tensor memory ----
  const int half = warp >> 2, mine_line = tid & (kOwn - 1), n_mine = first + mine_line;
  const uint32_t at_lane = tmem + ((uint32_t)((warp & 3) * 32) << 16);
  constexpr int kOwnN = kOwn / kAtOnce;
  int own_page[kOwnN];
#pragma unroll
  for (int k = 0; k < kOwnN; ++k) own_page[k] = mine.page(first + line0 + k * kAtOnce);
  pages(walk);
  if (walk < end) {
    request(walk);
    pages(next(walk));
  }
#pragma unroll
  for (int k0 = 0; k0 < kOwnN; k0 += 2) {
    float4 x[2][4];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int line = line0 + (k0 + k) * kAtOnce;
      const float *x1 = nullptr, *x2 = nullptr;
      const bool is = mine.find(first + line, own_page[k0 + k], D, &x1, &x2);
#pragma unroll
      for (int e = 0; e < 4; ++e) x[k][e] = is ? load4((e < 2 ? x1 : x2) + 8 * chunk + 4 * (e & 1)) : zero;
      if (kKeys && chunk == 0) sh.own_there[line] = is;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const uint32_t at = base + place<kOwn>(line0 + (k0 + k) * kAtOnce, chunk);
        store_parts(at + e * C::kX2, at + e * C::kX2 + C::kOwnPart, at + C::kY + e * C::kOwnPart, x[k][2 * e], x[k][2 * e + 1]);
      }
  }
  all();
#pragma unroll
  for (int e = 0; e < 2; ++e)
#pragma unroll
    for (int q = 0; q < D / 64; ++q) {
      uint32_t l[16];
#pragma unroll
      for (int k = 0; k < 4; ++k)
        ld_shared_v4(base + C::kY + e * C::kOwnPart + place<kOwn>(mine_line, half * (D / 16) + 4 * q + k), l + 4 * k);
      ptx::tmem_st16_async(at_lane + C::kXl + e * (D / 2) + half * (D / 4) + 16 * q, l);
    }
  ptx::tmem_wait_st();
  // rows [see_lo, see_hi) see this lane's key, or this lane's row at position x sees the keys from x_begin to x and the first ones
  int see_lo = 0, see_hi = 0, x = -1, x_begin = 0;
  float lse = 0.f, delta = 0.f;
  if (kKeys) {
    if (mine_line < n_own && sh.own_there[mine_line]) paged::rows_that_see(a, x0, rq.nq, G, n_mine, n_mine, &see_lo, &see_hi);
  } else if (mine_line < n_own) {
    const int tok = f.group.page(n_mine);
    x = x0 + tok;
    x_begin = paged::window_begin(x, a.window);
    const float2 mine_stats = p.stats[(long long)(rq.q0 + tok) * a.Hq + head * G + n_mine - tok * G];
    lse = mine_stats.x;
    delta = mine_stats.y;
  }
  all();                                                               // (the l are read)
  if (walk < end) put(0);

  float out[kKeys ? 2 : 1][D / 2];                                     // this lane's half of the columns: dK or dQ, dV
#pragma unroll
  for (int o = 0; o < (kKeys ? 2 : 1); ++o)
#pragma unroll
    for (int k = 0; k < D / 2; ++k) out[o][k] = 0.f;
  int buf = 0, steps = 0;
  auto add = [&] {                                                     // the results of the step before
    ok = wait(&sh.out_full, steps - 1) && ok;
#pragma unroll
    for (int o = 0; o < (kKeys ? 2 : 1); ++o)
#pragma unroll
      for (int q = 0; q < D / 32; ++q) {
        float z[16];
        load(at_lane + C::kOut + o * D + half * (D / 2) + 16 * q, z);
#pragma unroll
        for (int k = 0; k < 16; ++k) out[o][16 * q + k] += z[k];
      }
  };
#pragma unroll 1
  for (int at = walk; at < end; ++steps, buf ^= 1) {
    const int col = at + half * kCols;
    at = next(at);
    const bool more = at < end;
    if (more) {
      request(at);
      pages(next(at));
    }
    ok = wait(&sh.y_full, steps) && ok;                                    // (statistics and marks of this step)
    uint32_t see;
    if (kKeys) {
      see = bits(see_lo - col, see_hi - col);
    } else {
      const uint32_t there = __ballot_sync(0xffffffffu, lane < kCols && sh.there[buf][half * kCols + lane % kCols]);
      see = there & bits(0, x + 1 - col) & (bits(x_begin - col, 32) | bits(0, a.sinks - col));
    }
    // (loads and weights of unseen pairs too: a branch a pair took 3400 cycles a step)
    float lses[kCols], deltas[kCols];
    auto stats = [&](const float* from, float (&to)[kCols]) {
#pragma unroll
      for (int k = 0; k < kCols; k += 4) *reinterpret_cast<float4*>(to + k) = load4(from + half * kCols + k);
    };
    if (kKeys) stats(sh.lse[buf], lses);
    // ---- P ----
    float w[kCols], v[kCols];
    ok = wait(&sh.s_full, steps) && ok;
    load(at_lane + C::kS + half * kCols, v);
    if (kKeys) {
      ptx::tc_fence_before();
      both();                                                          // (S is read: P goes over it)
      ptx::tc_fence_after();
    }
#pragma unroll
    for (int k = 0; k < kCols; ++k) {
      const float weight = paged::grad_weight<float>(v[k], a.scale, kKeys ? lses[k] : lse);
      w[k] = (see >> k) & 1u ? weight : 0.f;
    }
    if (steps > 0) add();
    if (kKeys) store_operand(at_lane + C::kS + half * (kCols / 2), kStep / 2, w);
    ptx::tc_fence_before();
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(&sh.p_full);
    if (more) put(buf ^ 1);
    // ---- dS ----
    if (kKeys) stats(sh.delta[buf], deltas);
    ok = wait(&sh.dp_full, steps) && ok;
    load(at_lane + C::kDp + half * kCols, v);
    ptx::tc_fence_before();
    both();
    ptx::tc_fence_after();
#pragma unroll
    for (int k = 0; k < kCols; ++k) {
      const float ds = w[k] * (v[k] - (kKeys ? deltas[k] : delta));
      w[k] = (see >> k) & 1u ? ds : 0.f;
    }
    store_operand(at_lane + C::kDp + half * (kCols / 2), kStep / 2, w);
    ptx::tc_fence_before();
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(&sh.ds_full);
  }
  if (steps > 0) add();
  ptx::tc_fence_before();
  __syncwarp();
  ok = __syncthreads_and(ok);
  if (splits > 1) {
    constexpr int kValues = (kKeys ? 2 : 1) * (D / 2);
    static_assert(kValues * kComputeWarps * 32 * 4 <= C::kY, "place of another CTA's results");
    for (int n = 1; n < splits; n *= 2) {
      cluster_meet();                                                  // the place is free: products are done, results of before added up
      if (rank % (2 * n) == n) {
        const uint32_t to = ptx::map_to_cta(base, rank - n) + tid * 16;
#pragma unroll
        for (int k = 0; k < kValues; k += 4) {
          const float* z = &out[k / (D / 2)][k % (D / 2)];
          ptx::st_cluster_v4(to + k * (kComputeWarps * 32 * 4), make_float4(z[0], z[1], z[2], z[3]));
        }
      }
      cluster_meet();
      if (rank % (2 * n) == 0) {
#pragma unroll
        for (int k = 0; k < kValues; k += 4) {
          uint32_t z[4];
          ld_shared_v4(base + tid * 16 + k * (kComputeWarps * 32 * 4), z);
#pragma unroll
          for (int e = 0; e < 4; ++e) out[k / (D / 2)][k % (D / 2) + e] += __uint_as_float(z[e]);
        }
      }
    }
    all();                                                             // (the results go the same way)
  }
  if (ok && rank == 0) {
    // ---- by way of the own lines' place, 32 columns of a warp's lines at a time: 128 bytes of a row by 8 lanes ----
    constexpr int kParts = (kKeys ? 2 : 1) * (D / 64);
    static_assert(kComputeWarps * kParts * 4096 <= C::kY, "place of results");
    const uint32_t stage = base + warp * (kParts * 4096);
    float bad = 0.f;
#pragma unroll
    for (int part = 0; part < kParts; ++part)
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        const float* z = &out[part / (D / 64)][part % (D / 64) * 32 + 4 * k];
        const float by = part < D / 64 ? a.scale : 1.f;
        bad += z[0] * 0.f + z[1] * 0.f + z[2] * 0.f + z[3] * 0.f;
        ptx::st_shared_v4(stage + part * 4096 + lane * 128 + ((k ^ (lane & 7)) << 4), __float_as_uint(z[0] * by), __float_as_uint(z[1] * by),
                          __float_as_uint(z[2] * by), __float_as_uint(z[3] * by));
      }
    __syncwarp();
#pragma unroll 2
    for (int k = 0; k < 8; ++k) {
      const int line = 4 * k + (lane >> 3), j = first + (warp & 3) * 32 + line;
      if (j >= lines) continue;
      float* to[2];
      if (kKeys) {
        const long long row = (long long)rq.k0 + j;
        to[0] = static_cast<float*>(p.dk) + row * p.dk_stride + head * D;
        to[1] = static_cast<float*>(p.dv) + row * p.dv_stride + head * D;
      } else {
        const int tok = f.group.page(j);
        to[0] = static_cast<float*>(p.dq) + (long long)(rq.q0 + tok) * p.dq_stride + (head * G + j - tok * G) * D;
      }
#pragma unroll
      for (int part = 0; part < kParts; ++part) {
        uint32_t z[4];
        ld_shared_v4(stage + part * 4096 + line * 128 + (((lane & 7) ^ (line & 7)) << 4), z);
        *reinterpret_cast<uint4*>(to[part / (D / 64)] + half * (D / 2) + part % (D / 64) * 32 + 4 * (lane & 7)) = make_uint4(z[0], z[1], z[2], z[3]);
      }
    }
    if (bad != 0.f && mine_line < n_own) atomicOr(&sh.odd[mine_line >> 5], 1u << (mine_line & 31));
    all();
    // (a value that is no number, or too large, at a line that another line of the tile sees)
    if ((sh.odd[0] | sh.odd[1] | sh.odd[2] | sh.odd[3]) != 0u) {
#pragma unroll 1
      for (int line = warp; line < n_own; line += kComputeWarps) {
        if (!(sh.odd[line >> 5] >> (line & 31) & 1u)) continue;
        const int j = first + line, tok = j / G;
        if (kKeys)
          paged::grad_key<float, D>(p, r, rq, j, head, lane);
        else
          paged::grad_row<float, D>(p, r, rq.q0 + tok, x0 + tok, head * G + j - tok * G, lane);
      }
    }
  }
  __syncthreads();
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1) k_paged_grad_f32(const F32Args p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  Shared& sh = *reinterpret_cast<Shared*>(smem + Cfg<D>::kTiles);
  if ((ptx::smem_u32(smem) & 1023u) != 0) {                            // the tiles' swizzle counts from there (the same in all threads)
    if (threadIdx.x == 0) atomicOr(p.g.a.err, CASCADE_DEV_ERR_WAIT);
    return;
  }
  if (blockIdx.z == 0)
    pass<D, true>(p, smem, sh);
  else
    pass<D, false>(p, smem, sh);
}

template <int D>
int launch(cascade_ctx* ctx, const PagedGradArgs& p, cudaStream_t s) {
  constexpr int kSmem = Cfg<D>::kTiles + (int)sizeof(Shared);
  static_assert(kSmem <= 232448, "shared memory of a CTA");
  const PagedAttnArgs& a = p.a;
  const int G = a.Hq / a.Hkv;
  F32Args f = {p, G, 1, 1, paged::page_div(a.page_size), paged::page_div(G)};
  const int max_kv = a.max_kv < p.n_kv ? a.max_kv : p.n_kv;            // (longer requests are left out)
  const long long kv_blocks = ((long long)max_kv + kOwn - 1) / kOwn * a.Hkv, q_blocks = ((long long)a.max_q * G + kOwn - 1) / kOwn * a.Hkv;
  const long long blocks = kv_blocks > q_blocks ? kv_blocks : q_blocks;
  if (blocks > INT_MAX) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  CASCADE_TRY(configure_smem(ctx, PAGED_CFG_GRAD_F32, k_paged_grad_f32<D>, kSmem));   // (a context has one D)
  // While there are SMs left, the steps of a tile are shared out in the pass with the longer walk, or in both, such that the longest
  // walk is shortest; setting up a tile takes as long as two steps, adding up another CTA's results one and a half.
  // (1000 tokens, one head of 64: 34 us, without 58 us; 2 x 500, 8 query heads of 128 on one key head: 84 us, without 403 us.)
  long long rows_seen = a.max_q, keys_seen = max_kv;
  if (a.window > 0) {
    if (keys_seen > (long long)a.window + a.sinks + kOwn) keys_seen = (long long)a.window + a.sinks + kOwn;
    if (a.sinks == 0 && rows_seen > (long long)a.window + kOwn) rows_seen = (long long)a.window + kOwn;
  }
  const double steps_keys = (double)rows_seen * G / Cfg<D>::kStep, steps_rows = (double)keys_seen / Cfg<D>::kStep;
  double best = 1e300;
  int cluster = 1;
  for (int n = 1, levels = 0; n <= 8; n *= 2, ++levels)
    for (int which = 1; which <= 3; ++which) {
      const int sk = which & 1 ? n : 1, sr = which & 2 ? n : 1;
      if (n > 1 && (kv_blocks * sk + q_blocks * sr) * a.n_req > ctx->sm_count) continue;
      const double keys = 2 + steps_keys / sk + (sk > 1 ? 1.5 * levels : 0), rows = 2 + steps_rows / sr + (sr > 1 ? 1.5 * levels : 0), time = keys > rows ? keys : rows;
      if (time >= 0.95 * best) continue;
      best = time;
      cluster = n;
      f.split_keys = sk;
      f.split_rows = sr;
    }
  const long long x = kv_blocks * f.split_keys > q_blocks * f.split_rows ? kv_blocks * f.split_keys : q_blocks * f.split_rows;
  KernelScope ks(ctx, K_PAGED_GRAD, s);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((x + cluster - 1) / cluster * cluster), a.n_req, 2);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  CASCADE_CUDA_TRY(cudaLaunchKernelEx(&cfg, k_paged_grad_f32<D>, (const F32Args)f));
  return CASCADE_OK;
}

}  // namespace

int launch_paged_grad_f32(cascade_ctx* ctx, const PagedGradArgs& p, cudaStream_t s) {
  return ctx->shape.D == 128 ? launch<128>(ctx, p, s) : launch<64>(ctx, p, s);
}
