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
// Shared memory: the tiles, then what S holds.  The tiles' swizzle wants 1024-byte boundaries, which dynamic shared memory has
// where a kernel has no other; a kernel that finds it elsewhere reports and leaves.
template <int D, typename S>
constexpr int smem_bytes() {
  return Cfg<D>::kTiles * Cfg<D>::kTileBytes + (int)sizeof(S);
}

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
  int* taken;                     // [0] items handed out beyond the blocks' own, [1] blocks that are done; zero between launches
};

// The items that a CTA takes: its own index first, then what the launch's counter gives; the loading warp asks one item ahead.
struct Queue {
  int answer[2];
  bool lost[2];                   // the item before met a page outside the pool
  uint64_t full[2], empty[2];
};

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

// Items of the requests in order: kKeys: tiles of keys, else blocks of rows, of every key head; a whole warp walks forward through
// them, 32 requests at a time.  Of a request the longest come first, all heads beside each other.
template <bool kKeys>
struct Cursor {
  int chunk = -32, lane_items = 0, lane_first = 0, base = 0, total = 0;
  paged::GradRequest lane_rq;

  // -> request and its place in line, or false behind the last
  __device__ __forceinline__ bool find(const Args& p, int item, int lane, paged::GradRequest* rq, int* r, int* head, int* line) {
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
    *r = chunk + who;
    rq->q0 = __shfl_sync(0xffffffffu, lane_rq.q0, who);
    rq->nq = __shfl_sync(0xffffffffu, lane_rq.nq, who);
    rq->kv = __shfl_sync(0xffffffffu, lane_rq.kv, who);
    rq->k0 = __shfl_sync(0xffffffffu, lane_rq.k0, who);
    const int n = ((kKeys ? rq->kv : rq->nq) + unit - 1) / unit, round = local / a.Hkv;
    *line = kKeys ? round : n - 1 - round;
    *head = local - round * a.Hkv;
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

__device__ __forceinline__ uint64_t full_desc(uint32_t lo, uint64_t d) { return (uint64_t)lo | (d & 0xffffffff00000000ull); }

// acc[128 x 128] = A B^T, both tiles [128][D] in shared memory (low words of their descriptors).
template <int D>
__device__ __forceinline__ void product_ss(uint32_t acc, uint32_t a_lo, uint32_t b_lo, uint64_t desc, uint32_t idesc) {
#pragma unroll
  for (int ks = 0; ks < D / 16; ++ks) {
    const uint32_t off = ((ks >> 2) * (kTile * 128) + (ks & 3) * 32) >> 4;
    ptx::umma_bf16(acc, full_desc(a_lo + off, desc), full_desc(b_lo + off, desc), idesc, ks != 0);
  }
}
// acc[128 x D] += A B: A in tensor memory as left by the compute warps (columns 0 .. 31 and 64 .. 95), B a tile [128][D].
__device__ __forceinline__ void product_ts(uint32_t acc, uint32_t a_tmem, uint32_t b_lo, uint64_t desc, uint32_t idesc, bool first) {
#pragma unroll
  for (int ks = 0; ks < kTile / 16; ++ks)
    ptx::umma_bf16_ts(acc, a_tmem + (ks >> 2) * 64 + (ks & 3) * 8, full_desc(b_lo + ks * (2048 >> 4), desc), idesc, ks != 0 || !first);
}

// 32 columns of tensor memory as 16 pairs (after the wait).
__device__ __forceinline__ void load32(uint32_t taddr, uint32_t (&v)[32]) {
  ptx::tmem_ld32_async(taddr, v);
  ptx::tmem_wait_ld();
#pragma unroll
  for (int k = 0; k < 32; ++k) asm volatile("" : "+r"(v[k]));   // no use before the wait
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

// paged_grad_kv.cu, paged_grad_q.cu: the two passes on the tensor cores (bf16).
int launch_paged_grad_kv(cascade_ctx* ctx, const grad_tc::Args& p, cudaStream_t s);
int launch_paged_grad_q(cascade_ctx* ctx, const grad_tc::Args& p, cudaStream_t s);
