// Causal attention of new tokens over a paged cache on the tensor cores (bf16): prompts and chunks.
//
// A work item is two blocks of up to 128 query rows of one (request, key head), a row being (token, query head of the group),
// with all the key tiles (128 keys) that any of the rows sees.  One CTA an SM works through items that a counter hands out.
//   * warp 8 loads: every lane owns one box of a tile (8 to 128 rows of one page and 64 elements), looks its page up one
//     tile ahead and issues its own TMA copy; keys and values share a ring of four 32 KB stages;
//   * warps 9 and 10 issue the products of block 0 and block 1, in halves of a tile: S_w = Q_w K^T (128 x 64) and
//     O_w += P_w V with P_w taken from tensor memory.  A block has two halves of scores in tensor memory, so that the next
//     scores are formed while the softmax works: 450 us for 8 prompts of 2480 tokens and 32 heads where whole tiles took
//     591, although a product with 64 keys takes 53 cycles where one with 128 takes 64 (both operands in shared memory);
//   * warps 0-3 and 4-7: softmax of block 0 and block 1, one row per thread.  The weights 2^(s c - ref) go back as bf16 over
//     the scores' own columns.  ref starts as the first half's maximum and is raised one half late, when the sum of a half's
//     weights passes 2^8: then the row's accumulator is rescaled in place (rare), and no maximum has to be taken.
// What bounds it: the products take 0.5 million of 0.77 million cycles an SM there; the rest is the softmax's latency beside
// them (exponentials: half of the special-function unit's time) and the start and end of 17 items.  450 us are 893 TFLOP/s of
// 1709 measured, in short bursts; calls back to back for seconds run at the 1 kW power cap and take 530 us, 760 TFLOP/s.
// Weights are rounded to bf16 for the product (the tensor cores take both operands in one type, and the values are bf16); the
// sums and accumulators stay fp32.  Root-mean-square error against 64 bits 0.0021 to 0.0023 of the outputs', where outputs
// rounded once have 0.0016 to 0.0017; a product with the weights' remainders beside it would halve the rate of P V.
// Rows of the last tile behind the request's last key hold whatever the page held before: their scores are masked, and
// their values are set to zero in shared memory, since 0 x NaN would reach the sum.  A row whose result is not finite all
// the same (a non-finite value at a key that another row of the block sees), and every row of an item that met a page
// outside the pool, is computed again by one warp from the keys it sees alone.
// Every wait is bounded (error word, normal teardown).
#include "paged.h"
#include "paged_attn.cuh"
#include "tmap.h"

namespace {

constexpr int kTile = 128;        // keys per tile (a stage of the ring), rows per block
constexpr int kHalf = 64;         // keys per step of the softmax: half a tile
constexpr int kThreads = 352;
constexpr int kStages = 4;         // keys and values of two tiles
constexpr float kLazy = 256.f;    // a sum of a half's weights from which the reference is raised
constexpr float kFar = 0x1p96f;   // and from which the row is computed again

template <int D>
struct Cfg {
  static constexpr int kHalves = D / 64;                 // 64-element column blocks of a tile
  static constexpr int kTileBytes = kTile * D * 2;
  static constexpr int kOut = (2 + kStages) * kTileBytes;  // place of the results on their way out: 32 rows of 128 bytes a warp
  static constexpr int kSmem = kOut + 8 * 4096 + 1024;
};

struct TcArgs {
  PagedAttnArgs a;
  int G, tpb, box_rows;           // query heads a key head; tokens per row block; rows of a page box
  int* taken;                     // [0] items handed out beyond the blocks' own, [1] blocks that are done; zero between launches
};

// Items of the requests in order, Hkv x pairs of row blocks each; a whole warp walks forward through them, 32 requests
// at a time.
struct Item;
struct Cursor {
  int chunk = -32, lane_items = 0, lane_first = 0, base = 0, total = 0;
  paged::Request lane_rq = {0, 0, 0};
  __device__ __forceinline__ bool find(const TcArgs& p, int item, int lane, Item* it);
};

// The items that a CTA takes: its own index first, then what the launch's counter gives.  The loading warp asks one item
// ahead; every warp reads the answers in turn.  (8 prompts of 2480 tokens: a fixed share of items took 507 us where the
// hardware's own scheduler, with a block per item, took 486 and the counter 1 % more; but that scheduler takes 0.8 ms for one
// chunk beside 511 requests without tokens, the counter 18 us.)
struct Queue {
  int answer[2];
  bool lost[2];               // the item before met a page outside the pool
  uint64_t full[2], empty[2];
};
constexpr int kWarps = kThreads / 32;

struct Item {
  int r, head, q0, nq, kv;    // request, key head, the request's first row, rows, keys
  int tok[2];                 // first token of each block
  int n[2], n_tiles;          // half tiles of keys each block needs, tiles loaded
  int n_sink, skip;           // tile i is i (i < n_sink) or i + skip
  __device__ __forceinline__ int tile(int i) const { return i < n_sink ? i : i + skip; }
  // (a block chosen at run time: an index would put the struct into local memory)
  __device__ __forceinline__ int first(int w) const { return w == 0 ? tok[0] : tok[1]; }
  __device__ __forceinline__ int count(int w) const { return w == 0 ? n[0] : n[1]; }
};

__device__ __forceinline__ bool Cursor::find(const TcArgs& p, int item, int lane, Item* it) {
  while (chunk < 0 || item >= base + total) {
    base += total;
    chunk += 32;
    if (chunk >= p.a.n_req) return false;
    const int n_rows = p.a.q_begin[p.a.n_req];
    lane_items = 0;
    if (chunk + lane < p.a.n_req && paged::load_request(p.a, chunk + lane, &lane_rq))
      lane_items = p.a.Hkv * ((lane_rq.nq + 2 * p.tpb - 1) / (2 * p.tpb));
    if (__shfl_sync(0xffffffffu, lane_rq.q0, 0) == n_rows) return false;   // no tokens from here on
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
  const int pairs = (it->nq + 2 * p.tpb - 1) / (2 * p.tpb);
  // the longest rows of all heads first: 0.99 of the SMs' time is used on 8 prompts of 2480 tokens by a model of the queue,
  // 0.94 with one head after the other
  const int round = local / p.a.Hkv, pair = pairs - 1 - round;
  it->head = local - round * p.a.Hkv;
  const int x0 = it->kv - it->nq;               // position of the request's first new token
  it->tok[0] = pair * 2 * p.tpb;
  it->tok[1] = it->tok[0] + p.tpb;
  const int lo = paged::window_begin(x0 + it->tok[0], p.a.window);
  const int lo_tile = max(lo, 0) / kTile;
  it->n_sink = min((min(p.a.sinks, lo) + kTile - 1) / kTile, lo_tile);
  it->skip = lo_tile - it->n_sink;
  it->n_tiles = 0;
#pragma unroll
  for (int w = 0; w < 2; ++w) {
    it->n[w] = 0;
    if (it->tok[w] < it->nq) {
      const int last = x0 + min(it->nq, it->tok[w] + p.tpb) - 1;   // position of the block's last token
      if (last >= 0) it->n[w] = last / kHalf + 1 - 2 * it->skip;
    }
    it->n_tiles = max(it->n_tiles, (it->n[w] + 2 - 1) / 2);
  }
  return true;
}

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
k_paged_attn_tc(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                const __grid_constant__ CUtensorMap tm_v, const TcArgs p) {
  using C = Cfg<D>;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t q_full[2], q_empty[2], kv_full[kStages], kv_empty[kStages], s_full[2][2], p_full[2][2],
      o_full[2], o_empty[2];
  __shared__ Queue queue;
  __shared__ uint32_t s_tmem_base;
  __shared__ int s_abort;
  __shared__ uint64_t s_alive;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem = smem_raw + (smem_base - ptx::smem_u32(smem_raw));
  const uint32_t q_addr = smem_base, ring = smem_base + 2 * C::kTileBytes;
  volatile int* abort_flag = &s_abort;
  volatile uint64_t* alive = &s_alive;   // (when a row was last computed again, see below)
  int* err = p.a.err;
  const uint64_t wait_ns = p.a.wait_ns;

  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      ptx::mbar_init(&kv_full[i], 1);
      ptx::mbar_init(&kv_empty[i], 2);
    }
    for (int w = 0; w < 2; ++w) {
      ptx::mbar_init(&q_full[w], 1);
      ptx::mbar_init(&q_empty[w], 1);
      for (int b = 0; b < 2; ++b) {
        ptx::mbar_init(&s_full[w][b], 1);
        ptx::mbar_init(&p_full[w][b], 4);
      }
      ptx::mbar_init(&o_full[w], 1);
      ptx::mbar_init(&o_empty[w], 4);
    }
    for (int i = 0; i < 2; ++i) {
      ptx::mbar_init(&queue.full[i], 1);
      ptx::mbar_init(&queue.empty[i], kWarps);
    }
    s_abort = 0;
    s_alive = 0;
    ptx::fence_mbar_init();
  }
  if (warp == 8 && lane == 0) {
    ptx::prefetch_tmap(&tm_q);
    ptx::prefetch_tmap(&tm_k);
    ptx::prefetch_tmap(&tm_v);
  }
  if (warp == 9) {
    ptx::tmem_alloc(&s_tmem_base, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t tmem = s_tmem_base;   // S of block w and half b at 128 w + 64 b; O0, O1 at 256, 384

  if (blockIdx.x == gridDim.x - 1)                              // requests without tokens are checked here alone
    for (int r = threadIdx.x; r < p.a.n_req; r += kThreads) {
      paged::Request rq;
      paged::load_request(p.a, r, &rq);
    }
  Cursor cur;
  Item it;
  uint32_t turn = 0;                                            // items that this warp has taken
  bool lost = false;                                            // the item that was left for this one met a bad page
  auto next = [&]() {                                           // the next item
    const uint32_t slot = turn & 1u, use = turn >> 1;
    ++turn;
    const bool here = ptx::mbar_wait_short(&queue.full[slot], use & 1u, abort_flag, err, wait_ns, alive);
    const int item = here ? *static_cast<volatile int*>(&queue.answer[slot]) : INT_MAX;
    lost = here && *static_cast<volatile bool*>(&queue.lost[slot]);
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(&queue.empty[slot]);
    return __shfl_sync(0xffffffffu, item, 0);
  };
  if (warp == 8) {
    // ---------------- loads ----------------
    const int n_box = kTile / p.box_rows;                       // boxes of a tile along the keys
    const int box_i = lane % n_box, half = lane / n_box;        // this lane's box
    const bool has_box = half < C::kHalves;
    const uint32_t box_bytes = (uint32_t)p.box_rows * 128u;
    int items[2] = {0, 0};
    uint32_t ph = 0;                                            // bit j: parity of the next use of stages 2 j, 2 j + 1
    bool ok = true;
    for (int item = blockIdx.x; ok && cur.find(p, item, lane, &it); item = next()) {
      bool met_bad = false;
      const int granted = lane == 0 ? (int)gridDim.x + atomicAdd(p.taken, 1) : 0;   // (told at the end: the answer takes its time)
#pragma unroll
      for (int w = 0; w < 2; ++w) {
        if (it.n[w] == 0) continue;
        if (items[w] > 0) ok = ok && ptx::mbar_wait_short(&q_empty[w], (items[w] - 1) & 1u, abort_flag, err, wait_ns, alive);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        ++items[w];
        if (lane == 0) {
          ptx::mbar_arrive_expect_tx(&q_full[w], (uint32_t)(p.tpb * p.G) * 128u * C::kHalves);
          for (int h = 0; h < C::kHalves; ++h)
            ptx::tma_load_4d(smem + w * C::kTileBytes + h * (kTile * 128), &tm_q, h * 64, 0, it.head, it.q0 + it.tok[w], &q_full[w]);
        }
      }
      const int32_t* table = p.a.block_table + (size_t)it.r * p.a.table_stride;
      auto page_of = [&](int i, int* row) {                     // this lane's page in tile i (-1: nothing to load)
        const int key = it.tile(i) * kTile + box_i * p.box_rows;
        *row = key % p.a.page_size;
        return has_box && key < it.kv ? table[key / p.a.page_size] : -1;
      };
      int row = 0, next_row = 0;
      int page = it.n_tiles > 0 ? page_of(0, &row) : -1;
      bool wanted = has_box && it.n_tiles > 0 && it.tile(0) * kTile + box_i * p.box_rows < it.kv;
      for (int i = 0; ok && i < it.n_tiles; ++i) {
        int next = -1;
        bool next_wanted = false;
        if (i + 1 < it.n_tiles) {
          next = page_of(i + 1, &next_row);
          next_wanted = has_box && it.tile(i + 1) * kTile + box_i * p.box_rows < it.kv;
        }
        const bool load = wanted && page >= 0 && page < p.a.n_pages;
        if (wanted && !load) {
          atomicOr(err, CASCADE_DEV_ERR_BAD_PAGE);
          met_bad = true;                                       // (its place keeps what it held: the rows are computed again)
        }
        const uint32_t bytes = box_bytes * (uint32_t)__popc(__ballot_sync(0xffffffffu, load));
        for (int kv = 0; kv < 2; ++kv) {
          const int stage = 2 * (i & 1) + kv;
          ok = ptx::mbar_wait_short(&kv_empty[stage], ((ph >> (i & 1)) & 1u) ^ 1u, abort_flag, err, wait_ns, alive);
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          if (lane == 0) ptx::mbar_arrive_expect_tx(&kv_full[stage], bytes);
          __syncwarp();
          if (load)
            ptx::tma_load_4d(smem + (2 + stage) * C::kTileBytes + half * (kTile * 128) + box_i * box_bytes, kv == 0 ? &tm_k : &tm_v,
                             half * 64, it.head, row, page, &kv_full[stage]);
        }
        ph ^= 1u << (i & 1);
        page = next;
        row = next_row;
        wanted = next_wanted;
      }
      const uint32_t slot = turn & 1u, use = turn >> 1;
      if (use > 0) ok = ok && ptx::mbar_wait_short(&queue.empty[slot], (use - 1) & 1u, abort_flag, err, wait_ns, alive);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      met_bad = __any_sync(0xffffffffu, met_bad);
      if (lane == 0) {
        *static_cast<volatile int*>(&queue.answer[slot]) = granted;
        *static_cast<volatile bool*>(&queue.lost[slot]) = met_bad;
        ptx::mbar_arrive(&queue.full[slot]);
      }
    }
    // every stage and query tile has been given back before the CTA may end (the arrivals are asynchronous)
    for (int i = 0; ok && i < kStages; ++i)
      ok = ptx::mbar_wait_short(&kv_empty[i], ((ph >> (i >> 1)) & 1u) ^ 1u, abort_flag, err, wait_ns, alive);
#pragma unroll
    for (int w = 0; w < 2; ++w)
      if (ok && items[w] > 0) ok = ptx::mbar_wait_short(&q_empty[w], (items[w] - 1) & 1u, abort_flag, err, wait_ns, alive);
  } else if (warp >= 9) {
    // ---------------- products ----------------
    // One lane issues, a warp for each block: one warp for both took 800 us where two take 526.  Only the halves are known at
    // compile time; with stages and blocks as constants too the code leaves the instruction cache (720 us), with rolled
    // loops the issue is too slow (667 us).  Offsets go to the descriptors' low words alone (2 %).
    const uint32_t idesc_s = ptx::umma_idesc_bf16(128, kHalf);
    const uint32_t idesc_o = ptx::umma_idesc_bf16_b_mn(128, D);
    const uint64_t q_desc = ptx::umma_desc_sw128(q_addr), k_desc = ptx::umma_desc_sw128(ring),
                   v_desc = ptx::umma_desc_sw128_strides(ring, kTile * 128, 1024);
    int used = 0;                              // items of the block so far
    uint32_t p_ph = 0, kv_ph = 0;              // bit b: parity of the next weights; bit j: of the next use of stages 2 j, 2 j + 1
    bool ok = true;
    auto wait = [&](uint64_t* bar, uint32_t parity) { return ok = ptx::mbar_wait_short(bar, parity & 1u, abort_flag, err, wait_ns, alive); };
    const int w = warp - 9;
    auto full = [](uint32_t lo, uint64_t d) { return (uint64_t)lo | (d & 0xffffffff00000000ull); };
    auto scores = [&](int b, int st) {
      const uint32_t kl = (uint32_t)k_desc + st * (C::kTileBytes >> 4) + b * (kHalf * 128 >> 4);
      const uint32_t ql = (uint32_t)q_desc + w * (C::kTileBytes >> 4);
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks) {
        const uint32_t off = ((ks >> 2) * (kTile * 128) + (ks & 3) * 32) >> 4;
        ptx::umma_bf16(tmem + w * 128 + b * kHalf, full(ql + off, q_desc), full(kl + off, k_desc), idesc_s, ks != 0);
      }
    };
    auto outputs = [&](int b, int st, bool first) {
      const uint32_t vl = (uint32_t)v_desc + st * (C::kTileBytes >> 4) + b * (kHalf / 16) * (2048 >> 4);
#pragma unroll
      for (int ks = 0; ks < kHalf / 16; ++ks)
        ptx::umma_bf16_ts(tmem + 256 + w * 128, tmem + w * 128 + b * kHalf + ks * 8,
                          full(vl + ks * (2048 >> 4), v_desc), idesc_o, ks != 0 || !first);
    };
    // the products that follow the weights of tile i (j = i & 1)
    auto tile = [&](int i, int n, int n_tiles) {
      const int j = i & 1, kV = 2 * j + 1, kK = 2 * (j ^ 1);
      if (!wait(&kv_full[kV], kv_ph >> j)) return;
      kv_ph ^= 1u << j;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int h = 2 * i + b;
        if (h >= n) {
          if (b == 0 && i + 1 < n_tiles && !wait(&kv_full[kK], kv_ph >> (j ^ 1))) return;
          break;
        }
        if (b == 0 && h == 0 && used > 0 && !wait(&o_empty[w], used - 1)) return;
        if (!wait(&p_full[w][b], p_ph >> b)) return;
        p_ph ^= 1u << b;
        ptx::tc_fence_after();
        outputs(b, kV, h == 0);
        if (h + 1 == n) {
          ptx::umma_commit(&o_full[w]);
          if (b == 0 && i + 1 < n_tiles && !wait(&kv_full[kK], kv_ph >> (j ^ 1))) return;
          break;
        }
        if (b == 0 && i + 1 < n_tiles && !wait(&kv_full[kK], kv_ph >> (j ^ 1))) return;
        if (h + 2 < n) scores(b, kK);
        ptx::umma_commit(&s_full[w][b]);     // (behind the last scores: tells that the product is done)
        if (h + 2 + 1 == n) ptx::umma_commit(&q_empty[w]);
      }
      ptx::umma_commit(&kv_empty[kV]);
      if (i + 1 < n_tiles) ptx::umma_commit(&kv_empty[kK]);
    };
    auto block = [&](int n, int n_tiles) {
      if (!wait(&kv_full[0], kv_ph)) return;
      if (n > 0) {
        if (!wait(&q_full[w], used)) return;
#pragma unroll 1
        for (int b = 0; b < 2 && b < n; ++b) {
          scores(b, 0);
          ptx::umma_commit(&s_full[w][b]);
        }
        if (n <= 2) ptx::umma_commit(&q_empty[w]);
      }
      ptx::umma_commit(&kv_empty[0]);
#pragma unroll 1
      for (int i = 0; ok && i < n_tiles; ++i) tile(i, n, n_tiles);
      used += n > 0;
    };
    for (int item = blockIdx.x; ok && cur.find(p, item, lane, &it); item = next()) {
      if (it.n_tiles == 0) continue;
      if (lane == 0) block(it.count(w), it.n_tiles);
      ok = __shfl_sync(0xffffffffu, ok, 0);
    }
  } else {
    // ---------------- softmax, one row per thread ----------------
    const int w = warp >> 2, rr = threadIdx.x & 127;           // row block, row
    const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t t_s = tmem + w * 128 + lane_addr, t_o = tmem + 256 + w * 128 + lane_addr;
    const int my_tok = rr / p.G, my_g = rr % p.G;
    const bool in_block = rr < p.tpb * p.G;
    const float c = p.a.scale * paged::kLog2e;
    int used = 0, kv_used[2] = {0, 0};                         // items of this block; tiles of all items by the stages they used
    uint32_t s_ph = 0;                                         // bit b: parity of the next scores of half b
    bool ok = true;
    for (int item = blockIdx.x; ok && cur.find(p, item, lane, &it);) {
      const int tok = it.first(w) + my_tok;
      const bool live = in_block && tok < it.nq;
      // position (below 0: sees nothing); a place without a row sees everything, which spares its warp the masks
      const int x = live ? it.kv - it.nq + tok : INT_MAX / 2;
      const int lo = live ? paged::window_begin(x, p.a.window) : 0, n_sink = p.a.sinks;
      const int n = it.count(w);
      float ref = -INFINITY, next_ref = -INFINITY, l = 0.f;
      bool odd = false;                                        // to be computed again from the keys the row sees alone
      // halves in which every row of the warp sees every key: those before h_end, from h_begin on or before h_sink
      const int x_min = __reduce_min_sync(0xffffffffu, x), lo_max = __reduce_max_sync(0xffffffffu, lo);
      const int moved = 2 * it.skip, split = 2 * it.n_sink;     // (halves from `split` on lie `moved` further)
      const int end_key = (x_min + 1) / kHalf, lo_key = lo_max > 0 ? (lo_max - 1) / kHalf + 1 : 0;
      const int h_end = end_key <= split ? end_key : max(end_key - moved, split);
      const int h_begin = max(lo_key - moved, lo_key <= split ? lo_key : split), h_sink = min(n_sink / kHalf, split);
      const int h_kv = it.kv / kHalf - moved;                    // (the last key is behind the moved halves)
      const bool waits_first = live && x >= 0;
      for (int h = 0; h < n; ++h) {
        const int b = h & 1;
        const uint32_t t_h = t_s + b * kHalf;
        ok = ptx::mbar_wait_short(&s_full[w][b], (s_ph >> b) & 1u, abort_flag, err, wait_ns, alive);
        const bool raise = next_ref > ref, none = ref == -INFINITY && waits_first;
        const bool special = !(h < h_end && (h >= h_begin || h < h_sink));
        s_ph ^= 1u << b;
        ptx::tc_fence_after();
        const int k0 = it.tile(h / 2) * kTile + b * kHalf;
        // bit k: this row sees key k0 + 32 q + k
        auto visible = [&](int q) {
          const int j0 = k0 + 32 * q;
          auto below = [](int n) { return n >= 32 ? 0xffffffffu : (1u << max(n, 0)) - 1u; };
          return below(x - j0 + 1) & (~below(lo - j0) | below(n_sink - j0));
        };
        if (__any_sync(0xffffffffu, raise || none || !ok)) {
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
          if (__any_sync(0xffffffffu, raise)) {
            // once the product of the half before is done (the next commit on the other half's scores), the accumulator is
            // at rest
            ok = ptx::mbar_wait_short(&s_full[w][b ^ 1], (s_ph >> (b ^ 1)) & 1u, abort_flag, err, wait_ns, alive);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) break;
            ptx::tc_fence_after();
            const float alpha = raise ? ptx::ex2(ref - next_ref) : 1.f;
            ref = fmaxf(ref, next_ref);
            l *= alpha;
#pragma unroll 1
            for (int q = 0; q < D / 16; ++q) {
              float t[16];
              ptx::tmem_ld16(t_o + 16 * q, t);
#pragma unroll
              for (int k = 0; k < 16; ++k) t[k] *= alpha;
              ptx::tmem_st16(t_o + 16 * q, t);
            }
          }
          if (__any_sync(0xffffffffu, none)) {
            // rows that have met no key yet take their reference from this half
            float m = -INFINITY;
#pragma unroll 1
            for (int q = 0; q < kHalf / 32; ++q) {
              uint32_t v[32];
              ptx::tmem_ld32_async(t_h + 32 * q, v);
              const uint32_t vis = visible(q);
              ptx::tmem_wait_ld();
#pragma unroll
              for (int k = 0; k < 32; ++k) asm volatile("" : "+r"(v[k]));
#pragma unroll
              for (int k = 0; k < 32; ++k) m = fmaxf(m, (vis >> k) & 1u ? __uint_as_float(v[k]) : -INFINITY);
            }
            if (none) next_ref = ref = m * c;
          }
        }
        const float minus = ref == -INFINITY ? 0.f : -ref;
        const uint64_t c2 = ptx::pack2(c, c), minus2 = ptx::pack2(minus, minus);
        uint64_t sum2 = 0;
        uint32_t v[2][32];
        ptx::tmem_ld32_async(t_h, v[0]);
#pragma unroll
        for (int q = 0; q < kHalf / 32; ++q) {
          uint32_t pk[16];
          ptx::tmem_wait_ld();
          uint32_t* vq = v[q & 1];
#pragma unroll
          for (int k = 0; k < 32; ++k) asm volatile("" : "+r"(vq[k]));   // no use of the scores before the wait
          if (q + 1 < kHalf / 32) ptx::tmem_ld32_async(t_h + 32 * (q + 1), v[(q + 1) & 1]);
          if (special) {
            const uint32_t vis = visible(q);
#pragma unroll
            for (int k = 0; k < 32; ++k) vq[k] = (vis >> k) & 1u ? vq[k] : 0xff800000u;
          }
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            const float s0 = __uint_as_float(vq[2 * k]), s1 = __uint_as_float(vq[2 * k + 1]);
            float e0, e1;
            const uint64_t x2 = ptx::fma2(ptx::pack2(s0, s1), c2, minus2);
            ptx::unpack2(x2, &e0, &e1);
            e0 = ptx::ex2(e0);
            e1 = ptx::ex2(e1);
            sum2 = ptx::add2(sum2, ptx::pack2(e0, e1));
            pk[k] = ptx::pack_bf16x2(e0, e1);
          }
          ptx::tmem_st16_async(t_h + 16 * q, pk);
        }
        float sa, sb;
        ptx::unpack2(sum2, &sa, &sb);
        sa += sb;
        l += sa;
        // no maximum is taken: the sum of a half's weights lies between the largest of them and 64 times it
        if (live && sa > kLazy) next_ref = ref + __log2f(sa);
        odd = odd || sa > kFar;
        // values behind the last key: zeros (both blocks write them, each ahead of its own product)
        if (h >= h_kv) {
          const int j = (h / 2) & 1, st = 2 * j + 1;
          const uint32_t st_ph = (uint32_t)((j == 0 ? kv_used[0] : kv_used[1]) + h / 4) & 1u;
          ok = ptx::mbar_wait_short(&kv_full[st], st_ph, abort_flag, err, wait_ns, alive);
          const int key = rr & (kHalf - 1);                    // two threads a key, each half of its values
          if (ok && k0 + key >= it.kv) {
            constexpr int kChunks = D / 16;
            for (int k = 0; k < kChunks; ++k) {
              const int at = (rr / kHalf) * kChunks + k;
              ptx::st_shared_v4(ring + st * C::kTileBytes + (at >> 3) * (kTile * 128) + (b * kHalf + key) * 128 + (at & 7) * 16, 0, 0, 0, 0);
            }
            ptx::fence_proxy_async_smem();
          }
          ok = __all_sync(0xffffffffu, ok);
          if (!ok) break;
        }
        ptx::tmem_wait_st();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&p_full[w][b]);
      }
      kv_used[0] += (it.n_tiles + 1) / 2;
      kv_used[1] += it.n_tiles / 2;
      if (!ok) break;
      if (n > 1) {                               // the commit without scores, behind the last product but one
        ok = ptx::mbar_wait_short(&s_full[w][n & 1], (s_ph >> (n & 1)) & 1u, abort_flag, err, wait_ns, alive);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        s_ph ^= 1u << (n & 1);
      }
      // ---- the rows' results ----
      const int row = it.q0 + tok, head = it.head * p.G + my_g;
      if (n > 0) {
        ok = ptx::mbar_wait_short(&o_full[w], used & 1u, abort_flag, err, wait_ns, alive);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        ptx::tc_fence_after();
        ++used;
      }
      const float inv = l > 0.f ? 1.f / l : 0.f;
      odd = live && x >= 0 && (odd || !(l > 0.f && l < INFINITY));   // (or a sum that is no number)
      // 64 columns at a time through shared memory, so that eight lanes write 128 consecutive bytes of a row
      uint8_t* place = smem + C::kOut + warp * 4096;
      const long long my_out = live ? (long long)row * p.a.Hq + head : -1;
#pragma unroll 1
      for (int q = 0; q < D / 64; ++q) {
        uint32_t o[64];
        if (n > 0) {
          ptx::tmem_ld32_async(t_o + 64 * q, o);
          ptx::tmem_ld32_async(t_o + 64 * q + 32, o + 32);
          ptx::tmem_wait_ld();
#pragma unroll
          for (int k = 0; k < 64; ++k) asm volatile("" : "+r"(o[k]));
        } else {
#pragma unroll
          for (int k = 0; k < 64; ++k) o[k] = 0u;
        }
        float bad = 0.f;
#pragma unroll
        for (int k = 0; k < 64; ++k) bad = fmaf(__uint_as_float(o[k]), 0.f, bad);   // NaN if any is not finite
        odd = odd || (live && x >= 0 && bad != 0.f);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          uint32_t v[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float a = __uint_as_float(o[8 * k + 2 * e]) * inv, b = __uint_as_float(o[8 * k + 2 * e + 1]) * inv;
            v[e] = x < 0 ? 0u : ptx::pack_bf16x2(a, b);
          }
          *reinterpret_cast<uint4*>(place + lane * 128 + ((k ^ (lane & 7)) << 4)) = make_uint4(v[0], v[1], v[2], v[3]);
        }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int r = 4 * k + (lane >> 3), chunk = lane & 7;
          const uint4 v = *reinterpret_cast<const uint4*>(place + r * 128 + ((chunk ^ (r & 7)) << 4));
          const long long to = __shfl_sync(0xffffffffu, my_out, r);
          if (to >= 0) *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(p.a.out) + to * D + 64 * q + 8 * chunk) = v;
        }
        __syncwarp();
      }
      if (n > 0) {
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&o_empty[w]);
      }
      if (live && p.a.lse != nullptr)
        p.a.lse[(long long)row * p.a.Hq + head] = x >= 0 ? (ref + log2f(l)) * paged::kLn2 : -INFINITY;
      __syncwarp();
      // the answer for the next item tells whether this one's keys were all there: the loads ended long ago
      item = next();
      odd = odd || (lost && live && x >= 0);
      // (0.6 us a key and row: whoever waits for this warp meanwhile starts its limit anew with every 256 keys)
      for (uint32_t left = __ballot_sync(0xffffffffu, odd); left != 0u; left &= left - 1u) {
        const int who = __ffs(left) - 1;
        paged::attend_row<__nv_bfloat16, D>(p.a, it.r, __shfl_sync(0xffffffffu, row, who), __shfl_sync(0xffffffffu, x, who),
                                            __shfl_sync(0xffffffffu, head, who), lane, alive);
      }
    }
  }
  __syncwarp();
  if (*abort_flag) __nanosleep(1000000);   // copies still in flight
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  if (threadIdx.x == 0 && atomicAdd(p.taken + 1, 1) == (int)gridDim.x - 1) p.taken[0] = p.taken[1] = 0;
  if (warp == 9) ptx::tmem_dealloc(tmem, 512);
}

template <int D>
int launch(cascade_ctx* ctx, const TcArgs& p, int n_items, cudaStream_t s) {
  const PagedAttnArgs& a = p.a;
  const uint64_t dq[4] = {(uint64_t)D, (uint64_t)p.G, (uint64_t)a.Hkv, (uint64_t)a.n_tok};
  const uint64_t sq[3] = {(uint64_t)D, (uint64_t)p.G * D, (uint64_t)a.q_stride};
  const uint32_t bq[4] = {64, (uint32_t)p.G, 1, (uint32_t)p.tpb};
  const uint64_t dk[4] = {(uint64_t)D, (uint64_t)a.Hkv, (uint64_t)a.page_size, (uint64_t)a.n_pages};
  const uint64_t sk[3] = {(uint64_t)D, (uint64_t)a.Hkv * D, (uint64_t)a.page_stride};
  const uint32_t bk[4] = {64, 1, (uint32_t)p.box_rows, 1};
  // the queries' map goes by the pass's token count, so none is kept: the list would grow by one a pass and every call on the
  // context walk through it (38 us of host time a call after 3500 lengths, 11 us with an empty list)
  CUtensorMap mq;
  const CUtensorMap* mk = get_tmap_4d_bf16(ctx, a.k, dk, sk, bk);
  const CUtensorMap* mv = get_tmap_4d_bf16(ctx, a.v, dk, sk, bk);
  if (mk == nullptr || mv == nullptr || !make_tmap_4d_bf16(&mq, a.q, dq, sq, bq)) return CASCADE_ERR_CUDA;
  CASCADE_TRY(configure_smem(ctx, PAGED_CFG_ATTN_TC, k_paged_attn_tc<D>, Cfg<D>::kSmem));   // (a context has one D)
  const int grid = n_items < ctx->sm_count ? n_items : ctx->sm_count;
  k_paged_attn_tc<D><<<grid, kThreads, Cfg<D>::kSmem, s>>>(mq, *mk, *mv, p);
  CASCADE_CUDA_TRY(cudaGetLastError());
  return CASCADE_OK;
}

}  // namespace

int launch_paged_attn_tc(cascade_ctx* ctx, const PagedAttnArgs& a, cudaStream_t s) {
  TcArgs p;
  p.a = a;
  p.G = a.Hq / a.Hkv;
  p.tpb = kTile / p.G;
  p.box_rows = 8;
  while (p.box_rows < kTile && a.page_size % (2 * p.box_rows) == 0) p.box_rows *= 2;
  // no more items than this: a request's pairs of row blocks are at most ceil(tokens / (2 tpb))
  const long long pairs = (long long)a.n_tok / (2 * p.tpb) + a.n_req;
  const long long by_length = (long long)a.n_req * ((a.max_q + 2 * p.tpb - 1) / (2 * p.tpb));
  const long long items = (pairs < by_length ? pairs : by_length) * a.Hkv;
  if (items > INT_MAX / 2) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  const int n_items = (int)items;
  p.taken = ctx->dev_error + 32;   // (cleared with the error word when the context is made; a line of its own)
  return ctx->shape.D == 128 ? launch<128>(ctx, p, n_items, s) : launch<64>(ctx, p, n_items, s);
}
