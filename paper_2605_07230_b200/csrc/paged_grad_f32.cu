// The gradient of the attention over a paged cache in 32 bits, on the tensor cores.
//
// A 32-bit number is the sum of three bf16 numbers h + m + l (8 bits each, to the last bit); of a product's nine terms the six from
// 2^-17 up are formed, ll, ml and lm are left out (2^-26 of the product).  A product's terms go into the accumulator the smallest first,
// so that what the tensor cores' additions cut off counts at the size of hh alone; products of one step start from zero and are added
// up in registers.
//
// A CTA owns 128 keys, or 128 rows (token, query head of the group), and walks over the other side 64 at a time:
//     S = X1 Y1^T    P = exp(c S - lse)    dP = X2 Y2^T    dS = P (dP - delta)        keys: dV += P Y2, dK += dS Y1;  rows: dQ += dS Y1
// with X1, X2 its own keys and values (queries and output gradients), Y1, Y2 the others'.  A lane of the tensor memory is one of its
// own lines, so all that a thread sums belongs to one line.  P and dS are the products' operands from the tensor memory.
#include <climits>

#include "paged.h"
#include "paged_grad.cuh"

namespace {

constexpr int kOwn = 128, kStep = 64;
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

template <int D>
struct Cfg {
  static constexpr bool kShare = D == 128;               // X1 and X2 take turns in one place, Y1 and Y2 have one place each
  static constexpr int kOwnPart = kOwn * D * 2, kOwnTile = 3 * kOwnPart;        // bytes
  static constexpr int kStepPart = kStep * D * 2, kStepTile = 3 * kStepPart;
  static constexpr int kX2 = kShare ? 0 : kOwnTile, kY = kShare ? kOwnTile : 2 * kOwnTile;
  static constexpr int kTiles = kY + (kShare ? 2 : 4) * kStepTile;
};
// columns of the tensor memory: S, dP (dS as an operand over them), P as an operand, results
constexpr int kS = 0, kDp = 64, kDsOp = 0, kPOp = 128, kOut = 224;
static_assert(kOut + 2 * 128 <= 512, "tensor memory");

struct Shared {
  uint64_t s_full, dp_full, out_full, alive;
  int abort_flag;
  uint32_t tmem;
  uint32_t odd[kOwn / 32];                               // own lines with a result that is not finite
  float2 stats[2][kStep];                                // of the rows walked over
  uint8_t there[2][kStep], own_there[kOwn];              // keys whose pages are in the pool
};

struct F32Args {
  PagedGradArgs g;
  int G;                      // query heads a key head
  paged::PageDiv page, group; // (divisions by multiplication)
};

// Lines of one (request, key head): keys and values, or queries and output gradients (of rows (token, head) up to `end`).
struct Lines {
  const F32Args& f;
  const int32_t* table;
  int head, q0, end;
  // -> where line j's elements are; false: there is none (zeros)
  template <bool kKeys>
  __device__ __forceinline__ bool find(int j, int D, const float** first, const float** second) const {
    const PagedGradArgs& p = f.g;
    const PagedAttnArgs& a = p.a;
    if (j >= end) return false;
    if (kKeys) {
      const int in = f.page.page(j), page = table[in];
      if (page < 0 || page >= a.n_pages) return false;
      const long long off = (long long)page * a.page_stride + ((long long)(j - in * a.page_size) * a.Hkv + head) * D;
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
__device__ __forceinline__ void store_parts(uint32_t at, int part_bytes, const float4& x, const float4& y) {
  uint32_t h[4], m[4], l[4];
  split2(x.x, x.y, &h[0], &m[0], &l[0]);
  split2(x.z, x.w, &h[1], &m[1], &l[1]);
  split2(y.x, y.y, &h[2], &m[2], &l[2]);
  split2(y.z, y.w, &h[3], &m[3], &l[3]);
  ptx::st_shared_v4(at, h[0], h[1], h[2], h[3]);
  ptx::st_shared_v4(at + part_bytes, m[0], m[1], m[2], m[3]);
  ptx::st_shared_v4(at + 2 * part_bytes, l[0], l[1], l[2], l[3]);
}
// Place of the 16 bytes `chunk` of a line in a tile whose rows are swizzled over 128 bytes.
template <int kLines>
__device__ __forceinline__ uint32_t place(int line, int chunk) {
  return (chunk >> 3) * (kLines * 128) + line * 128 + (((chunk & 7) ^ (line & 7)) << 4);
}

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ bool elect_one() {
  uint32_t is;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
  return is != 0;
}
__device__ __forceinline__ uint64_t plus(uint64_t desc, uint32_t bytes) { return desc + (bytes >> 4); }
// The six terms, the smallest first: parts of A and of B.
__device__ __forceinline__ int part_a(int term) { return (0x001102 >> (4 * term)) & 15; }   // l h m m h h
__device__ __forceinline__ int part_b(int term) { return (0x010120 >> (4 * term)) & 15; }   // h l m h m h

// acc[128 x 64] = X Y^T
template <int D>
__device__ __forceinline__ void scores(uint32_t acc, uint32_t x, uint32_t y) {
  const uint32_t idesc = ptx::umma_idesc_bf16(kOwn, kStep);
  const uint64_t dx = ptx::umma_desc_sw128(x), dy = ptx::umma_desc_sw128(y);
#pragma unroll 1
  for (int t = 0; t < 6; ++t) {
    const uint64_t a = plus(dx, part_a(t) * Cfg<D>::kOwnPart), b = plus(dy, part_b(t) * Cfg<D>::kStepPart);
#pragma unroll
    for (int ks = 0; ks < D / 16; ++ks)
      ptx::umma_bf16(acc, plus(a, (ks >> 2) * (kOwn * 128) + (ks & 3) * 32), plus(b, (ks >> 2) * (kStep * 128) + (ks & 3) * 32), idesc,
                     ks != 0 || t != 0);
  }
}
// acc[128 x D] = W Y with W [128][64] in the tensor memory, 32 columns a part
template <int D>
__device__ __forceinline__ void results(uint32_t acc, uint32_t w, uint32_t y) {
  const uint32_t idesc = ptx::umma_idesc_bf16_b_mn(kOwn, D);
  const uint64_t dy = ptx::umma_desc_sw128_strides(y, kStep * 128, 1024);
#pragma unroll 1
  for (int t = 0; t < 6; ++t) {
    const uint64_t b = plus(dy, part_b(t) * Cfg<D>::kStepPart);
#pragma unroll
    for (int ks = 0; ks < kStep / 16; ++ks) ptx::umma_bf16_ts(acc, w + part_a(t) * 32 + ks * 8, plus(b, ks * 2048), idesc, ks != 0 || t != 0);
  }
}

// 32 columns (after the wait).
__device__ __forceinline__ void load32(uint32_t taddr, float (&v)[32]) {
  uint32_t r[32];
  ptx::tmem_ld32_async(taddr, r);
  ptx::tmem_wait_ld();
#pragma unroll
  for (int k = 0; k < 32; ++k) {
    asm volatile("" : "+r"(r[k]));                                     // no use before the wait
    v[k] = __uint_as_float(r[k]);
  }
}
// 32 weights of a lane as an operand's 16 columns of each part.
__device__ __forceinline__ void store_operand(uint32_t taddr, const float (&w)[32]) {
  uint32_t h[16], m[16], l[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) split2(w[2 * k], w[2 * k + 1], &h[k], &m[k], &l[k]);
  ptx::tmem_st16_async(taddr, h);
  ptx::tmem_st16_async(taddr + 32, m);
  ptx::tmem_st16_async(taddr + 64, l);
  ptx::tmem_wait_st();
}
// Bits lo .. hi - 1 of a word.
__device__ __forceinline__ uint32_t bits(int lo, int hi) {
  auto below = [](int n) { return n >= 32 ? 0xffffffffu : (1u << max(n, 0)) - 1u; };
  return below(hi) & ~below(lo);
}

// One CTA's tile of keys (kKeys) or block of rows.
template <int D, bool kKeys>
__device__ __forceinline__ void pass(const F32Args& f, uint8_t* smem, Shared& sh) {
  using C = Cfg<D>;
  const PagedGradArgs& p = f.g;
  const PagedAttnArgs& a = p.a;
  const int G = f.G, head = blockIdx.x % a.Hkv, r = blockIdx.y;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  paged::GradRequest rq;
  if (!paged::load_request(p, r, &rq)) return;
  const int x0 = rq.kv - rq.nq, lines = kKeys ? rq.kv : rq.nq * G;
  int own = blockIdx.x / a.Hkv;                                        // the longest first: keys in order, rows from the end
  if (!kKeys) own = (lines + kOwn - 1) / kOwn - 1 - own;
  const int first = own * kOwn;
  if (first < 0 || first >= lines) return;
  const int n_own = min(kOwn, lines - first);

  // what is walked over: rows [walk, end) that see any of the keys, or keys up to the last that a row sees
  int walk, end, begin = 0, sink_end = 0;
  if (kKeys) {
    int lo, hi;
    paged::tokens_that_see(a, x0, rq.nq, first, first + n_own - 1, &lo, &hi);
    walk = lo * G;
    end = hi * G;
  } else {
    begin = paged::window_begin(max(x0 + first / G, 0), a.window) / kStep * kStep;
    sink_end = min(a.sinks, begin);
    walk = sink_end > 0 ? 0 : begin;
    end = x0 + (first + n_own - 1) / G + 1;
  }
  auto next = [&](int at) {
    at += kStep;
    return kKeys || at < sink_end ? at : max(at, begin);
  };
  const int32_t* table = a.block_table + (size_t)r * a.table_stride;
  const Lines mine = {f, table, head, rq.q0, lines}, others = {f, table, head, rq.q0, kKeys ? end : rq.kv};

  const uint32_t base = ptx::smem_u32(smem);
  const int chunk = tid % (D / 8), line0 = tid / (D / 8);              // a thread's 8 elements of every kThreads / (D / 8)-th line
  constexpr int kLinesAtOnce = kThreads * 8 / D;
  // X1 and X2, or one of them
  auto load_own = [&](bool one, bool two) {
#pragma unroll 4
    for (int line = line0; line < kOwn; line += kLinesAtOnce) {
      const float *x1 = nullptr, *x2 = nullptr;
      const bool is = mine.find<kKeys>(first + line, D, &x1, &x2);
      const float4 zero = make_float4(0.f, 0.f, 0.f, 0.f);
      if (kKeys && one && chunk == 0) {
        sh.own_there[line] = is;
        if (!is && first + line < lines) atomicOr(a.err, CASCADE_DEV_ERR_BAD_PAGE);
      }
      const uint32_t at = base + place<kOwn>(line, chunk);
      if (one) store_parts(at, C::kOwnPart, is ? load4(x1 + 8 * chunk) : zero, is ? load4(x1 + 8 * chunk + 4) : zero);
      if (two) store_parts(at + C::kX2, C::kOwnPart, is ? load4(x2 + 8 * chunk) : zero, is ? load4(x2 + 8 * chunk + 4) : zero);
    }
  };
  constexpr int kN = kStep / kLinesAtOnce;
  float4 y[kN][4];                                                     // a step's elements on their way: Y1, Y2
  auto request = [&](int at, int buf) {
#pragma unroll
    for (int k = 0; k < kN; ++k) {
      const int line = line0 + k * kLinesAtOnce;
      const float *y1 = nullptr, *y2 = nullptr;
      const bool is = others.find<!kKeys>(at + line, D, &y1, &y2);
#pragma unroll
      for (int e = 0; e < 4; ++e) y[k][e] = is ? load4((e < 2 ? y1 : y2) + 8 * chunk + 4 * (e & 1)) : make_float4(0.f, 0.f, 0.f, 0.f);
      if (chunk != 0) continue;
      if (kKeys) {
        float2 st = make_float2(0.f, 0.f);
        if (is) {
          const int tok = f.group.page(at + line);
          st = p.stats[(long long)(rq.q0 + tok) * a.Hq + head * G + at + line - tok * G];
        }
        sh.stats[buf][line] = st;
      } else {
        sh.there[buf][line] = is;
        if (!is && at + line < rq.kv) atomicOr(a.err, CASCADE_DEV_ERR_BAD_PAGE);
      }
    }
  };
  auto y_tile = [&](int buf, int which) { return base + C::kY + ((C::kShare ? 0 : 2 * buf) + which) * C::kStepTile; };
  auto put = [&](int buf) {
#pragma unroll
    for (int k = 0; k < kN; ++k)
#pragma unroll
      for (int e = 0; e < 2; ++e)
        store_parts(y_tile(buf, e) + place<kStep>(line0 + k * kLinesAtOnce, chunk), C::kStepPart, y[k][2 * e], y[k][2 * e + 1]);
  };

  if (tid == 0) {
    for (uint64_t* b : {&sh.s_full, &sh.dp_full, &sh.out_full}) ptx::mbar_init(b, 1);
    ptx::fence_mbar_init();
    sh.abort_flag = 0;
    sh.alive = 0;
  }
  if (tid < kOwn / 32) sh.odd[tid] = 0u;
  if (warp == 0) {
    ptx::tmem_alloc(&sh.tmem, 512);
    ptx::tmem_relinquish();
  }
  if (walk < end) request(walk, 0);
  load_own(true, !C::kShare);
  if (walk < end) put(0);
  ptx::fence_proxy_async_smem();
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = sh.tmem;
  auto wait = [&](uint64_t* bar, uint32_t parity) { return ptx::mbar_wait_short(bar, parity & 1u, &sh.abort_flag, a.err, a.wait_ns, &sh.alive); };
  auto issue_scores = [&](int buf, bool one, bool two) {
    if (warp != 0 || !elect_one()) return;
    if (one) {
      scores<D>(tmem + kS, base, y_tile(buf, 0));
      ptx::umma_commit(&sh.s_full);
    }
    if (two) {
      scores<D>(tmem + kDp, base + C::kX2, y_tile(buf, 1));
      ptx::umma_commit(&sh.dp_full);
    }
  };
  // all threads' stores to shared or tensor memory are there and all their loads done, for the products that warp 0 issues next
  auto meet = [&](bool ok) {
    ptx::tc_fence_before();
    ok = __syncthreads_and(ok);
    ptx::tc_fence_after();
    return ok;
  };

  const int half = warp >> 2, mine_line = tid & (kOwn - 1), n_mine = first + mine_line;
  const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16, at_lane = tmem + lane_addr;
  // rows [see_lo, see_hi) see this lane's key, or this lane's row at position x sees the keys from x_begin to x and the first ones
  int see_lo = 0, see_hi = 0, x = -1, x_begin = 0;
  float lse = 0.f, delta = 0.f;
  if (kKeys) {
    if (mine_line < n_own && sh.own_there[mine_line]) {
      int lo, hi;
      paged::tokens_that_see(a, x0, rq.nq, n_mine, n_mine, &lo, &hi);
      see_lo = lo * G;
      see_hi = hi * G;
    }
  } else if (mine_line < n_own) {
    const int tok = f.group.page(n_mine);
    x = x0 + tok;
    x_begin = paged::window_begin(x, a.window);
    const float2 st = p.stats[(long long)(rq.q0 + tok) * a.Hq + head * G + n_mine - tok * G];
    lse = st.x;
    delta = st.y;
  }
  float out[kKeys ? 2 : 1][D / 2];                                     // this lane's half of the columns: dK or dQ, dV
#pragma unroll
  for (int o = 0; o < (kKeys ? 2 : 1); ++o)
#pragma unroll
    for (int k = 0; k < D / 2; ++k) out[o][k] = 0.f;

  bool ok = true;
  if (walk < end) issue_scores(0, true, !C::kShare);
  int buf = 0;
#pragma unroll 1
  for (int at = walk, i = 0; at < end; ++i) {
    const int then = next(at), col = at + half * 32;
    uint32_t see;
    if (kKeys) {
      see = bits(see_lo - col, see_hi - col);
    } else {
      const uint32_t there = __ballot_sync(0xffffffffu, sh.there[buf][half * 32 + lane]);
      see = there & bits(0, x + 1 - col) & (bits(x_begin - col, 32) | bits(0, a.sinks - col));
    }
    if (!C::kShare && then < end) request(then, buf ^ 1);
    // ---- P ----
    float w[32], v[32];
    ok = wait(&sh.s_full, i) && ok;
    ptx::tc_fence_after();
    __syncwarp();
    load32(at_lane + kS + 32 * half, v);
    const float2* stats = &sh.stats[buf][half * 32];
#pragma unroll
    for (int k = 0; k < 32; ++k) w[k] = (see >> k) & 1u ? paged::grad_weight<float>(v[k], a.scale, kKeys ? stats[k].x : lse) : 0.f;
    if (kKeys) store_operand(at_lane + kPOp + 16 * half, w);
    if (C::kShare) {
      load_own(false, true);
      ptx::fence_proxy_async_smem();
    }
    if (kKeys || C::kShare) {
      ok = meet(ok);
      if (!ok) break;
      if (C::kShare) issue_scores(buf, false, true);
      if (kKeys && warp == 0 && elect_one()) results<D>(tmem + kOut + D, tmem + kPOp, y_tile(buf, 1));
    }
    // ---- dS ----
    ok = wait(&sh.dp_full, i) && ok;
    ptx::tc_fence_after();
    __syncwarp();
    load32(at_lane + kDp + 32 * half, v);
#pragma unroll
    for (int k = 0; k < 32; ++k) w[k] = (see >> k) & 1u ? w[k] * (v[k] - (kKeys ? stats[k].y : delta)) : 0.f;
    ok = meet(ok);                                                     // (S and dP are read: dS goes over them)
    if (!ok) break;
    store_operand(at_lane + kDsOp + 16 * half, w);
    ok = meet(ok);
    if (warp == 0 && elect_one()) {
      results<D>(tmem + kOut, tmem + kDsOp, y_tile(buf, 0));
      ptx::umma_commit(&sh.out_full);
    }
    if (!C::kShare && then < end) {                                    // the next step's products queue up behind
      put(buf ^ 1);
      ptx::fence_proxy_async_smem();
      meet(true);
      issue_scores(buf ^ 1, true, true);
    }
    // ---- results ----
    ok = wait(&sh.out_full, i) && ok;
    ptx::tc_fence_after();
    __syncwarp();
#pragma unroll
    for (int o = 0; o < (kKeys ? 2 : 1); ++o)
#pragma unroll
      for (int q = 0; q < D / 64; ++q) {
        load32(at_lane + kOut + o * D + half * (D / 2) + 32 * q, v);
#pragma unroll
        for (int k = 0; k < 32; ++k) out[o][32 * q + k] += v[k];
      }
    at = then;
    if (C::kShare && at < end) {
      request(at, buf ^ 1);
      load_own(true, false);
      put(buf ^ 1);
      ptx::fence_proxy_async_smem();
      ok = meet(ok);
      if (!ok) break;
      issue_scores(buf ^ 1, true, false);
    }
    buf ^= 1;
  }
  if (!__syncthreads_and(ok)) {
    __nanosleep(1000000);                                              // products still in flight
  } else {
    if (mine_line < n_own) {
      float* to[2];
      if (kKeys) {
        const long long row = (long long)rq.k0 + n_mine;
        to[0] = static_cast<float*>(p.dk) + row * p.dk_stride + head * D;
        to[1] = static_cast<float*>(p.dv) + row * p.dv_stride + head * D;
      } else {
        const int tok = f.group.page(n_mine);
        to[0] = static_cast<float*>(p.dq) + (long long)(rq.q0 + tok) * p.dq_stride + (head * G + n_mine - tok * G) * D;
      }
      float bad = 0.f;
#pragma unroll
      for (int o = 0; o < (kKeys ? 2 : 1); ++o) {
        const float by = o == 0 ? a.scale : 1.f;
#pragma unroll
        for (int k = 0; k < D / 2; k += 4) {
          const float4 z = make_float4(out[o][k] * by, out[o][k + 1] * by, out[o][k + 2] * by, out[o][k + 3] * by);
          bad += out[o][k] * 0.f + out[o][k + 1] * 0.f + out[o][k + 2] * 0.f + out[o][k + 3] * 0.f;
          paged::store4(to[o] + half * (D / 2) + k, z);
        }
      }
      if (bad != 0.f) atomicOr(&sh.odd[mine_line >> 5], 1u << (mine_line & 31));
    }
    __syncthreads();
    // (a value that is no number, or too large, at a line that another line of the tile sees)
    for (int line = warp; line < n_own; line += kWarps) {
      if (!(sh.odd[line >> 5] >> (line & 31) & 1u)) continue;
      const int j = first + line, tok = j / G;
      if (kKeys)
        paged::grad_key<float, D>(p, r, rq, j, head, lane);
      else
        paged::grad_row<float, D>(p, r, rq.q0 + tok, x0 + tok, head * G + j - tok * G, lane);
    }
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  if (warp == 0) ptx::tmem_dealloc(tmem, 512);
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
  const F32Args f = {p, G, paged::page_div(a.page_size), paged::page_div(G)};
  const long long kv_blocks = ((long long)a.max_kv + kOwn - 1) / kOwn * a.Hkv, q_blocks = ((long long)a.max_q * G + kOwn - 1) / kOwn * a.Hkv;
  const long long blocks = kv_blocks > q_blocks ? kv_blocks : q_blocks;
  if (blocks > INT_MAX) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  CASCADE_TRY(configure_smem(ctx, PAGED_CFG_GRAD_F32, k_paged_grad_f32<D>, kSmem));   // (a context has one D)
  KernelScope ks(ctx, K_PAGED_GRAD, s);
  k_paged_grad_f32<D><<<dim3((unsigned)blocks, a.n_req, 2), kThreads, kSmem, s>>>(f);
  CASCADE_CUDA_TRY(cudaGetLastError());
  return CASCADE_OK;
}

}  // namespace

int launch_paged_grad_f32(cascade_ctx* ctx, const PagedGradArgs& p, cudaStream_t s) {
  return ctx->shape.D == 128 ? launch<128>(ctx, p, s) : launch<64>(ctx, p, s);
}
