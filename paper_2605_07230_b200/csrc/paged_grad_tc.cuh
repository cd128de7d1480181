// What the two tensor-core passes of the paged attention's gradient share: work items, the queue that hands them out, loads of
// keys by page, masks and products.
#pragma once
#include "paged.h"
#include "paged_grad.cuh"
#include "tmap.h"

namespace grad_tc {

constexpr int kTile = 128;        // rows and keys of a tile
constexpr int kComputeWarps = 8;  // two per 32 lanes of tensor memory, each with half the columns
constexpr int kWarps = kComputeWarps + 3;   // and one for loads, one for products, one for the rows' statistics
constexpr int kThreads = kWarps * 32;
constexpr int kLoads = kComputeWarps, kProducts = kLoads + 1, kStats = kLoads + 2;

template <int D>
struct Cfg {
  static constexpr int kHalves = D / 64;                 // 64-element column blocks of a tile
  static constexpr int kTileBytes = kTile * D * 2;
  static constexpr int kTiles = 7;
};
// Shared memory: the tiles, what both passes share, then a pass's own.  The tiles' swizzle wants 1024-byte boundaries, which dynamic
// shared memory has where a kernel has no other; a kernel that finds it elsewhere reports and leaves.
struct Common {
  uint64_t alive;
  int abort_flag;
  uint32_t tmem;
};

// Place of the next use in a ring of kN stages, and its parity.
template <int kN>
struct Ring {
  uint32_t stage = 0, ph = 0;
  __device__ __forceinline__ void step() {
    if (++stage == kN) {
      stage = 0;
      ph ^= 1u;
    }
  }
};

struct Args {
  PagedGradArgs g;
  int G, tpb, box_rows;           // query heads a key head; tokens per row block; rows of a page box
  int n_cta_keys;                 // CTAs that begin with the keys' pass
  int split;                      // of them (a cluster) share the row blocks of an item
  bool both;                      // a CTA whose pass has no more items goes on with the other
  int* taken;                     // items of either pass handed out beyond the CTAs' own, CTAs that are done; zero between launches
};

// The items that a CTA takes: its own index first, then what the launch's counter gives.  The loading warp finds an item's request
// and tiles and tells the other warps, at most kSlots items ahead.
struct Item : paged::GradRequest {
  int r, head, line;              // request, key head, its tile of keys or block of rows
  int n, first, skip;             // steps (row blocks or key tiles; -1: no more items), see the passes
  bool lost;                      // its loads met a page outside the pool: known when the next item is told
};
constexpr int kSlots = 4;
struct Queue {
  Item item[kSlots];
  uint64_t full[kSlots], empty[kSlots];
};

__device__ __forceinline__ void cluster_meet() {
  __syncwarp();
  ptx::cluster_arrive();
  ptx::cluster_wait();
}

// A waiting warp's view of the CTA: where waits give up.
struct Waits {
  volatile int* abort_flag;
  volatile uint64_t* alive;
  int* err;
  uint64_t ns;
  __device__ __forceinline__ bool operator()(uint64_t* bar, uint32_t parity) const {
    return ptx::mbar_wait_short(bar, parity & 1u, abort_flag, err, ns, alive);
  }
};

// One warp's turns through the queue; false behind the last item, or where a wait gave up.
struct Turns {
  uint32_t turn = 0;
  __device__ __forceinline__ bool next(Queue& q, const Waits& wait, bool* ok) {
    *ok = __all_sync(0xffffffffu, *ok && wait(&q.full[turn % kSlots], turn / kSlots));
    return *ok && static_cast<volatile Item&>(q.item[turn % kSlots]).n >= 0;
  }
  // (the loading warp's side) false where the wait gave up
  __device__ __forceinline__ bool tell(Queue& q, const Waits& wait, const Item& it, int lane, bool* ok) {
    *ok = __all_sync(0xffffffffu, *ok && wait(&q.empty[turn % kSlots], (turn / kSlots) ^ 1u));
    if (*ok && lane == 0) {
      q.item[turn % kSlots] = it;
      ptx::mbar_arrive(&q.full[turn % kSlots]);
    }
    ++turn;
    return *ok;
  }
  __device__ __forceinline__ Item& last(Queue& q) const { return q.item[(turn - 1) % kSlots]; }   // the one told last
  __device__ __forceinline__ bool next_is_told(Queue& q, const Waits& wait) const {
    return wait(&q.full[(turn + 1) % kSlots], (turn + 1) / kSlots);
  }
  __device__ __forceinline__ const Item& item(Queue& q) const { return q.item[turn % kSlots]; }
  __device__ __forceinline__ void done(Queue& q, int lane) {       // the item is not looked at any more
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(&q.empty[turn % kSlots]);
    ++turn;
  }
};

// Items of the requests in order: kKeys: tiles of keys, else blocks of rows, of every key head; a whole warp walks forward through
// them, 32 requests at a time.  Of a request the longest come first, all heads beside each other.
template <bool kKeys>
struct Cursor {
  int chunk = -32, lane_items = 0, lane_first = 0, base = 0, total = 0;
  paged::GradRequest lane_rq;

  // -> request, head and line of the item, or false behind the last
  __device__ __forceinline__ bool find(const Args& p, int item, int lane, Item* it) {
    const PagedAttnArgs& a = p.g.a;
    const int unit = kKeys ? kTile : p.tpb;
    while (chunk < 0 || item >= base + total) {
      base += total;
      chunk += 32;
      if (chunk >= a.n_req) return false;
      lane_items = 0;
      if (chunk + lane < a.n_req && paged::load_request(p.g, chunk + lane, &lane_rq))
        lane_items = a.Hkv * (((kKeys ? lane_rq.kv : lane_rq.nq) + unit - 1) / unit);
      int inc = lane_items;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
      }
      lane_first = inc - lane_items;
      total = __shfl_sync(0xffffffffu, inc, 31);
    }
    const int x = item - base;
    const int who = __ffs(__ballot_sync(0xffffffffu, x >= lane_first && x < lane_first + lane_items)) - 1;
    const int local = x - __shfl_sync(0xffffffffu, lane_first, who);
    it->r = chunk + who;
    it->q0 = __shfl_sync(0xffffffffu, lane_rq.q0, who);
    it->nq = __shfl_sync(0xffffffffu, lane_rq.nq, who);
    it->kv = __shfl_sync(0xffffffffu, lane_rq.kv, who);
    it->k0 = __shfl_sync(0xffffffffu, lane_rq.k0, who);
    const int n = ((kKeys ? it->kv : it->nq) + unit - 1) / unit, round = local / a.Hkv;
    it->line = kKeys ? round : n - 1 - round;
    it->head = local - round * a.Hkv;
    return true;
  }
};

// Bits lo .. hi - 1 of a word.
__device__ __forceinline__ uint32_t bits(int lo, int hi) {
  auto below = [](int n) { return n >= 32 ? 0xffffffffu : (1u << max(n, 0)) - 1u; };
  return below(hi) & ~below(lo);
}

__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// 2^x of a pair.  kPoly: on the multiply-add units, 1 + r (c1 + r (c2 + r (c3 + r c4))) with r = x - round(x) in [-1/2, 1/2] (least
// largest error of that form: 2.9e-6 relative, where the weights are rounded to 2^-8), times 2^round(x); below -127 exactly 0, no
// number stays none.  A third of the weights goes there: 16 exponentials a cycle and SM take 1024 cycles a 128 x 128 tile.
template <bool kPoly>
__device__ __forceinline__ uint64_t pow2(uint64_t x) {
  float x0, x1;
  ptx::unpack2(x, &x0, &x1);
  if (!kPoly) return ptx::pack2(ptx::ex2(x0), ptx::ex2(x1));
  auto both = [](float v) { return ptx::pack2(v, v); };
  asm("max.NaN.f32 %0, %0, 0fC2FE0000;" : "+f"(x0));       // -127
  asm("max.NaN.f32 %0, %0, 0fC2FE0000;" : "+f"(x1));
  x = ptx::pack2(x0, x1);
  const uint64_t t = ptx::add2(x, both(12582912.f));       // 1.5 2^23: the integer part in the last bits
  const uint64_t r = ptx::fma2(ptx::add2(t, both(-12582912.f)), both(-1.f), x);
  uint64_t y = ptx::fma2(both(0.009582853f), r, both(0.055906426f));
  y = ptx::fma2(y, r, both(0.24024099f));
  y = ptx::fma2(y, r, both(0.69312418f));
  y = ptx::fma2(y, r, both(1.f));
  float t0, t1;
  ptx::unpack2(t, &t0, &t1);
  return mul2(y, ptx::pack2(__int_as_float(__float_as_int(t0) * (1 << 23) + 0x3f800000), __int_as_float(__float_as_int(t1) * (1 << 23) + 0x3f800000)));
}

__device__ __forceinline__ uint64_t full_desc(uint32_t lo, uint64_t d) { return (uint64_t)lo | (d & 0xffffffff00000000ull); }

// The issuing warps walk their loops as a whole, so that descriptors stay in registers which the warp shares, and one lane (the same
// each time) issues products and commits: 40 cycles a product of 16 columns where predicated instructions took 51.
__device__ __forceinline__ bool elect_one() {
  uint32_t is;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
  return is != 0;
}
// acc[128 x 128] = A B^T, both tiles [128][D] in shared memory (low words of their descriptors).
template <int D>
__device__ __forceinline__ void product_ss(uint32_t acc, uint32_t a_lo, uint32_t b_lo, uint64_t desc, uint32_t idesc) {
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) {
    const uint32_t off = ((ks >> 2) * (kTile * 128) + (ks & 3) * 32) >> 4;
    ptx::umma_bf16(acc, full_desc(a_lo + off, desc), full_desc(b_lo + off, desc), idesc, ks != 0);
  }
}
// acc[128 x 128] = A B^T with A [128][D] in tensor memory (two elements a column), B a tile [128][D].
template <int D>
__device__ __forceinline__ void product_ts_k(uint32_t acc, uint32_t a_tmem, uint32_t b_lo, uint64_t desc, uint32_t idesc) {
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks)
    ptx::umma_bf16_ts(acc, a_tmem + ks * 8, full_desc(b_lo + (((ks >> 2) * (kTile * 128) + (ks & 3) * 32) >> 4), desc), idesc, ks != 0);
}
// acc[128 x D] += A B with A [128][128] in tensor memory, its halves kGap columns apart, B a tile [128][D].
template <int kGap>
__device__ __forceinline__ void product_ts(uint32_t acc, uint32_t a_tmem, uint32_t b_lo, uint64_t desc, uint32_t idesc, bool first) {
#pragma unroll
  for (int ks = 0; ks < kTile / 16; ++ks)
    ptx::umma_bf16_ts(acc, a_tmem + (ks >> 2) * kGap + (ks & 3) * 8, full_desc(b_lo + ks * (2048 >> 4), desc), idesc, ks != 0 || !first);
}

// 32 columns of tensor memory as 16 pairs (after the wait).
__device__ __forceinline__ void load32(uint32_t taddr, uint32_t (&v)[32]) {
  ptx::tmem_ld32_async(taddr, v);
  ptx::tmem_wait_ld();
#pragma unroll
  for (int k = 0; k < 32; ++k) asm volatile("" : "+r"(v[k]));   // no use before the wait
}

__device__ __forceinline__ void inval(uint64_t* bar) { asm volatile("mbarrier.inval.shared::cta.b64 [%0];" ::"r"(ptx::smem_u32(bar)) : "memory"); }
__device__ __forceinline__ void ld_shared_v4(uint32_t addr, uint32_t* x) {
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(addr) : "memory");
}

// `other` where the bit of a column is not set.
__device__ __forceinline__ void mask32(uint32_t (&v)[32], uint32_t see, uint32_t other) {
#pragma unroll
  for (int k = 0; k < 32; ++k) v[k] = (see >> k) & 1u ? v[k] : other;
}
constexpr uint32_t kMinusInf = 0xff800000u;

// 32 columns of a lane's row, times `by`, as bf16: four lanes exchange their 16-byte pieces, so that they write 64 bytes of one
// row after the other.  to[m]: where the columns of row m of the four go; null: nowhere.  False if a value is not finite.
__device__ __forceinline__ bool store_32_columns(const uint32_t (&v)[32], float by, __nv_bfloat16* const (&to)[4], int lane) {
  uint32_t x[4][4];
  uint64_t bad[2] = {0, 0};
  const uint64_t by2 = ptx::pack2(by, by);
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const uint64_t y = mul2(ptx::pack2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1])), by2);
    bad[k & 1] = ptx::fma2(y, 0, bad[k & 1]);                         // NaN if any is not finite
    float lo, hi;
    ptx::unpack2(y, &lo, &hi);
    x[k >> 2][k & 3] = ptx::pack_bf16x2(lo, hi);
  }
#pragma unroll
  for (int round = 1; round <= 2; round <<= 1) {                      // 4 x 4 transpose of pieces
    const bool upper = lane & round;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (k & round) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t got = __shfl_xor_sync(0xffffffffu, upper ? x[k][e] : x[k + round][e], round);
        x[k][e] = upper ? got : x[k][e];
        x[k + round][e] = upper ? x[k + round][e] : got;
      }
    }
  }
#pragma unroll
  for (int m = 0; m < 4; ++m)
    if (to[m] != nullptr) *reinterpret_cast<uint4*>(to[m] + 8 * (lane & 3)) = make_uint4(x[m][0], x[m][1], x[m][2], x[m][3]);
  float b0, b1;
  ptx::unpack2(ptx::add2(bad[0], bad[1]), &b0, &b1);
  return b0 + b1 == 0.f;
}

// Zeros in rows first .. last - 1 of a tile in shared memory, by the compute warps.
template <int D>
__device__ __forceinline__ void clear_rows(uint32_t tile, int first, int last, int tid) {
  for (int i = tid; i < (last - first) * (D / 8); i += kComputeWarps * 32) {
    const int row = first + i / (D / 8), chunk = i % (D / 8);
    ptx::st_shared_v4(tile + (chunk >> 3) * (kTile * 128) + row * 128 + (chunk & 7) * 16, 0, 0, 0, 0);
  }
}

// One lane's box of a tile of keys: page and row, page -1 where there is none (or, reported, outside the pool).  A tile has no
// more than 32 boxes (8 rows of 64 elements and more).
struct Box {
  int i, half, n;                 // box along the keys, 64-element half, boxes a tile
  __device__ __forceinline__ Box(const Args& p, int lane) : i(lane % (kTile / p.box_rows)), half(lane / (kTile / p.box_rows)), n(kTile / p.box_rows) {}
  __device__ __forceinline__ int page(const Args& p, const int32_t* table, int first_key, int kv, int halves, int* row, bool* bad) const {
    const int key = first_key + i * p.box_rows;
    *row = key % p.g.a.page_size;
    if (half >= halves || key >= kv) return -1;
    const int at = table[key / p.g.a.page_size];
    if (at >= 0 && at < p.g.a.n_pages) return at;
    atomicOr(p.g.a.err, CASCADE_DEV_ERR_BAD_PAGE);
    *bad = true;
    return -1;
  }
};

// Tensor maps of [n_tok][Hkv][G][D] rows (boxes of tpb tokens of one key head) and of the page pools.
inline bool row_map(CUtensorMap* m, const Args& p, int D, const void* base, long long stride) {
  const PagedAttnArgs& a = p.g.a;
  const uint64_t d[4] = {(uint64_t)D, (uint64_t)p.G, (uint64_t)a.Hkv, (uint64_t)a.n_tok};
  const uint64_t s[3] = {(uint64_t)D, (uint64_t)p.G * D, (uint64_t)stride};
  const uint32_t b[4] = {64, (uint32_t)p.G, 1, (uint32_t)p.tpb};
  return make_tmap_4d_bf16(m, base, d, s, b);
}
inline const CUtensorMap* page_map(cascade_ctx* ctx, const Args& p, int D, const void* base) {
  const PagedAttnArgs& a = p.g.a;
  const uint64_t d[4] = {(uint64_t)D, (uint64_t)a.Hkv, (uint64_t)a.page_size, (uint64_t)a.n_pages};
  const uint64_t s[3] = {(uint64_t)D, (uint64_t)a.Hkv * D, (uint64_t)a.page_stride};
  const uint32_t b[4] = {64, 1, (uint32_t)p.box_rows, 1};
  return get_tmap_4d_bf16(ctx, base, d, s, b);
}

}  // namespace grad_tc

// paged_grad_tc.cu: both passes in one launch (bf16).
int launch_paged_grad_tc(cascade_ctx* ctx, const PagedGradArgs& g, cudaStream_t s);
