// Keys' and values' gradients of the paged attention on the tensor cores (bf16).
//
// A work item is a tile of 128 keys of one (request, key head) and all row blocks (128 rows: token, query head of the group) that
// see any of them.  One CTA an SM works through items that a counter hands out.  With rows on the columns, per block:
//     S^T = K Q^T      P^T = 2^(c S^T - lse)      dP^T = V dO^T      dS^T = P^T (dP^T - delta)      dV += P^T dO      dK += dS^T Q
// S^T, dP^T, dV and dK fill the tensor memory (4 x 128 columns at D = 128); P^T and dS^T go back as bf16 over their own scores
// and are the products' operand from there (both operands have one type: 2^-8 of a weight at most, which leaves an error of 0.0024 of the
// results' size where results rounded once have 0.0017).  The products of one block alternate with the next block's scores:
//     dV, S^T of the next block  beside the computation of dS^T;   dK, dP^T of the next block  beside that of P^T
//   * warp 8 loads keys and values once an item, queries through three stages (the next block's are wanted right behind the
//     product that frees a stage) and output gradients through two;
//   * warp 9 issues the products;  warp 10 brings the rows' statistics;
//   * warps 0-7: a key per lane, half of a block's rows each; P stays in registers between the two halves of the work.
//
// Few items with many row blocks (many query heads on one key head) are shared out: a cluster of `split` CTAs takes an item, a stretch of
// its blocks each, and adds up its results by pairs, pairs of pairs and so on, in the tensor memory of the first.
#pragma once
#include <climits>

#include "paged_grad_tc.cuh"

namespace grad_tc {

struct SharedKv {
  uint64_t kv_full, kv_empty, q_full[3], q_empty[3], do_full[2], do_empty[2], s_full, p_full, dp_full, ds_full, acc_full, acc_empty, stat_full[2],
      stat_empty[2];
  Queue queue;
  __align__(16) float lse[2][kTile], delta[2][kTile];                  // negated
};

// The results `acc` (a lane's columns in tensor memory; none yet: zeros) of a cluster's CTAs added up by pairs, by way of the tiles'
// place.  (A function of its own: beside the rest it costs registers.)
template <int D>
__device__ __noinline__ void join(uint32_t acc, uint32_t base, uint32_t place, int split, int rank, bool any) {
#pragma unroll 1
  for (int m = 1; m < split; m *= 2) {
    cluster_meet();                                                    // everywhere the products are done with the tiles
    if (rank % (2 * m) == m) {
      const uint32_t to = ptx::map_to_cta(base, rank - m) + place;
#pragma unroll 1
      for (int q = 0; q < D / 32; ++q) {
        uint32_t v[32];
        load32(acc + 32 * q, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          auto z = [&](int e) { return any ? __uint_as_float(v[4 * k + e]) : 0.f; };
          ptx::st_cluster_v4(to + (q * 8 + k) * (kTile * 16), make_float4(z(0), z(1), z(2), z(3)));
        }
      }
    }
    cluster_meet();
    if (rank % (2 * m) == 0) {
#pragma unroll 1
      for (int q = 0; q < D / 32; ++q) {
        uint32_t v[32];
        load32(acc + 32 * q, v);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          uint32_t z[4];
          ld_shared_v4(base + place + (q * 8 + k) * (kTile * 16), z);
#pragma unroll
          for (int e = 0; e < 4; ++e) v[4 * k + e] = __float_as_uint((any ? __uint_as_float(v[4 * k + e]) : 0.f) + __uint_as_float(z[e]));
        }
        ptx::tmem_st16_async(acc + 32 * q, v);
        ptx::tmem_st16_async(acc + 32 * q + 16, v + 16);
        ptx::tmem_wait_st();
      }
      any = true;
    }
  }
}

// The whole CTA; `cta` of `n_cta` that begin with this pass, the others (cta >= n_cta) take what its counter hands out.
template <int D>
__device__ __forceinline__ void pass_kv(const CUtensorMap& tm_q, const CUtensorMap& tm_do, const CUtensorMap& tm_k, const CUtensorMap& tm_v, const Args& p,
                                        uint8_t* smem, uint32_t base, uint32_t tmem, const Waits& wait, int cta, int n_cta) {
  using C = Cfg<D>;
  SharedKv& sh = *reinterpret_cast<SharedKv*>(smem + C::kTiles * C::kTileBytes + sizeof(Common));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // tiles: keys, values, queries of three stages, output gradients of two
  constexpr int kQ = 2, kDo = 5;
  auto tile = [&](int i) { return base + i * C::kTileBytes; };
  const PagedAttnArgs& a = p.g.a;
  int* taken = p.taken + 0;
  if (threadIdx.x == 0) {
    for (uint64_t* b : {&sh.kv_full, &sh.kv_empty, &sh.s_full, &sh.dp_full, &sh.acc_full}) ptx::mbar_init(b, 1);
    for (uint64_t* b : {&sh.p_full, &sh.ds_full, &sh.acc_empty}) ptx::mbar_init(b, kComputeWarps);
    for (int i = 0; i < 3; ++i) {
      ptx::mbar_init(&sh.q_full[i], 1);
      ptx::mbar_init(&sh.q_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      for (uint64_t* b : {&sh.do_full[i], &sh.do_empty[i], &sh.stat_full[i]}) ptx::mbar_init(b, 1);
      ptx::mbar_init(&sh.stat_empty[i], kComputeWarps);
    }
    for (int i = 0; i < kSlots; ++i) {
      ptx::mbar_init(&sh.queue.full[i], 1);
      ptx::mbar_init(&sh.queue.empty[i], kWarps - 1);
    }
    ptx::fence_mbar_init();
  }
  const int block_rows = p.tpb * p.G;
  if (block_rows < kTile && warp < kComputeWarps) {                    // rows that no load ever fills
    for (int i = kQ; i < C::kTiles; ++i) clear_rows<D>(tile(i), block_rows, kTile, threadIdx.x);
    ptx::fence_proxy_async_smem();
  }
  __syncthreads();
  const uint32_t t_s = tmem, t_dp = t_s + 128, t_dv = t_s + 256, t_dk = t_dv + D;

  const int rank = blockIdx.x % p.split;
  bool joined = p.split == 1;
  Turns turns;
  uint32_t used = 0, blk = 0;                                          // items with blocks, and blocks, so far
  Ring<3> ring;                                                        // the queries' stages
  bool ok = true;

  if (warp == kLoads) {
    const Box box(p, lane);
    const uint32_t box_bytes = (uint32_t)p.box_rows * 128u, row_bytes = (uint32_t)block_rows * 128u * C::kHalves;
    Cursor<true> cur;
    Item it = {};
    for (int item = cta < n_cta ? cta : INT_MIN;;) {
      if (item == INT_MIN) item = __shfl_sync(0xffffffffu, lane == 0 ? n_cta + atomicAdd(taken, 1) : 0, 0);
      // (a cluster has one item, whatever the requests' ranges)
      const bool more = cur.find(p, item, lane, &it) && (p.split == 1 || item < n_cta);
      int lo, hi;                                                      // tokens that see any of the keys -> row blocks
      paged::tokens_that_see(a, it.kv - it.nq, it.nq, it.line * kTile, min(it.kv, (it.line + 1) * kTile) - 1, &lo, &hi);
      it.first = lo / p.tpb;
      it.n = !more ? -1 : hi > lo ? (hi - 1) / p.tpb - it.first + 1 : 0;
      if (p.split > 1 && more) {
        const int each = (it.n + p.split - 1) / p.split, skip = min(it.n, rank * each);
        it.first += skip;
        it.n = min(it.n - skip, each);
      }
      if (!turns.tell(sh.queue, wait, it, lane, &ok) || !more) break;
      const int granted = lane == 0 ? n_cta + atomicAdd(taken, 1) : 0;
      auto load_rows = [&](int i, const CUtensorMap* m, uint64_t* full, uint64_t* empty, uint32_t ph, int to) {
        ok = __all_sync(0xffffffffu, ok && wait(empty, ph ^ 1u));
        if (ok && lane == 0) {
          ptx::mbar_arrive_expect_tx(full, row_bytes);
          for (int h = 0; h < C::kHalves; ++h)
            ptx::tma_load_4d(smem + to * C::kTileBytes + h * (kTile * 128), m, h * 64, 0, it.head, it.q0 + (it.first + i) * p.tpb, full);
        }
      };
      auto load_q = [&](int i) {
        load_rows(i, &tm_q, &sh.q_full[ring.stage], &sh.q_empty[ring.stage], ring.ph, kQ + ring.stage);
        ring.step();
      };
      if (it.n > 0) {
        int row;
        bool bad = false;
        const int page = box.page(p, a.block_table + (size_t)it.r * a.table_stride, it.line * kTile, it.kv, C::kHalves, &row, &bad);
        load_q(0);
        ok = __all_sync(0xffffffffu, ok && wait(&sh.kv_empty, used ^ 1u));
        if (!ok) break;
        const uint32_t bytes = 2u * box_bytes * (uint32_t)__popc(__ballot_sync(0xffffffffu, page >= 0));
        if (lane == 0) ptx::mbar_arrive_expect_tx(&sh.kv_full, bytes);
        __syncwarp();
        if (page >= 0)
          for (int kv = 0; kv < 2; ++kv)
            ptx::tma_load_4d(smem + kv * C::kTileBytes + box.half * (kTile * 128) + box.i * box_bytes, kv == 0 ? &tm_k : &tm_v, box.half * 64,
                             it.head, row, page, &sh.kv_full);
        ++used;
        for (int i = 0; ok && i < it.n; ++i) {
          if (i > 0) load_q(i);
          const uint32_t stage = (blk + i) & 1u;
          load_rows(i, &tm_do, &sh.do_full[stage], &sh.do_empty[stage], (blk + i) >> 1, kDo + stage);
        }
        if (!ok) break;
        blk += it.n;
      }
      item = __shfl_sync(0xffffffffu, granted, 0);
    }
    // everything has been given back before the CTA may end (the arrivals are asynchronous)
    ok = ok && wait(&sh.kv_empty, used ^ 1u);
    for (uint32_t i = 0; i < 2; ++i) ok = ok && wait(&sh.do_empty[(blk + i) & 1u], ((blk + i) >> 1) ^ 1u);
    for (uint32_t i = 0; i < 3; ++i, ring.step()) ok = ok && wait(&sh.q_empty[ring.stage], ring.ph ^ 1u);
  } else if (warp == kProducts) {
    const uint32_t idesc_s = ptx::umma_idesc_bf16(128, 128), idesc_o = ptx::umma_idesc_bf16_b_mn(128, D);
    const uint64_t desc = ptx::umma_desc_sw128(base), desc_mn = ptx::umma_desc_sw128_strides(base, kTile * 128, 1024);
    auto lo = [&](int i) { return (uint32_t)desc + i * (C::kTileBytes >> 4); };
    auto lo_mn = [&](int i) { return (uint32_t)desc_mn + i * (C::kTileBytes >> 4); };
    auto here = [&](uint64_t* bar, uint32_t parity) { return ok = __all_sync(0xffffffffu, wait(bar, parity)); };
    Ring<3> behind;                                                    // the stage of the block whose last product comes next
    // dV with the next S^T, and dK with the next dP^T, are one piece of code (this warp's instructions are fetched anew each time
    // beside the others' loops); between two products nothing is waited for that could be waited for earlier.
    auto work = [&](int n) {
      if (!here(&sh.kv_full, used)) return;
#pragma unroll 1
      for (int i = -2; i < 2 * n; ++i) {
        const bool second = i & 1, more = i < 2 * n - 2;
        const uint32_t b = blk + (i >> 1), next = b + 1;
        if (more && !here(second ? &sh.do_full[next & 1u] : &sh.q_full[ring.stage], second ? next >> 1 : ring.ph)) return;
        if (i >= 0) {
          if (i == 0 && !here(&sh.acc_empty, used ^ 1u)) return;
          if (!here(second ? &sh.ds_full : &sh.p_full, b)) return;
          ptx::tc_fence_after();
          if (elect_one()) {                                           // dV += P^T dO or dK += dS^T Q
            product_ts<64>(second ? t_dk : t_dv, second ? t_dp : t_s, lo_mn(second ? kQ + behind.stage : kDo + (b & 1u)), desc_mn, idesc_o, i < 2);
            ptx::umma_commit(second ? &sh.q_empty[behind.stage] : &sh.do_empty[b & 1u]);
          }
          if (second) behind.step();
        }
        if (more) {
          if (elect_one()) {                                           // S^T = K Q^T or dP^T = V dO^T
            product_ss<D>(second ? t_dp : t_s, lo(second), lo(second ? kDo + (next & 1u) : kQ + ring.stage), desc, idesc_s);
            ptx::umma_commit(second ? &sh.dp_full : &sh.s_full);
            if (i == 2 * n - 3) ptx::umma_commit(&sh.kv_empty);
          }
          if (!second) ring.step();
        }
      }
      if (elect_one()) ptx::umma_commit(&sh.acc_full);
    };
    while (turns.next(sh.queue, wait, &ok)) {
      const int n = __shfl_sync(0xffffffffu, turns.item(sh.queue).n, 0);
      turns.done(sh.queue, lane);
      if (n == 0) continue;
      work(n);
      if (!ok) break;
      ++used;
      blk += n;
    }
  } else if (warp == kStats) {
    int tok[kTile / 32], g[kTile / 32];                                // token and head of rows lane, lane + 32, ...
#pragma unroll
    for (int m = 0; m < kTile / 32; ++m) {
      tok[m] = (lane + 32 * m) / p.G;
      g[m] = (lane + 32 * m) % p.G;
    }
    while (turns.next(sh.queue, wait, &ok)) {
      // the blocks' tokens: how many, and how many stand in front of key 0 and see nothing
      const Item& it = turns.item(sh.queue);
      const int n = it.n, before = it.first * p.tpb, left = it.nq - before, unseeing = it.nq - it.kv - before;
      const float2* from = p.g.stats + (long long)(it.q0 + before) * a.Hq + it.head * p.G;
      turns.done(sh.queue, lane);
      for (int i = 0; ok && i < n; ++i, ++blk) {
        float2 st[kTile / 32];                                         // (zeros where there is no row, or one that sees no key)
#pragma unroll
        for (int m = 0; m < kTile / 32; ++m) {
          const int t = i * p.tpb + tok[m];
          st[m] = make_float2(0.f, 0.f);
          if (tok[m] < p.tpb && t < left && t >= unseeing) st[m] = from[(long long)t * a.Hq + g[m]];
        }
        ok = __all_sync(0xffffffffu, wait(&sh.stat_empty[blk & 1u], (blk >> 1) ^ 1u));
        if (!ok) break;
#pragma unroll
        for (int m = 0; m < kTile / 32; ++m) {
          sh.lse[blk & 1u][lane + 32 * m] = -st[m].x;
          sh.delta[blk & 1u][lane + 32 * m] = -st[m].y;
        }
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sh.stat_full[blk & 1u]);
      }
    }
  } else {
    const int part = warp >> 2, key = threadIdx.x & (kTile - 1);       // which half of the rows; this lane's key
    const int half_col = part * 64;
    const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t my_s = t_s + lane_addr + half_col, my_dp = t_dp + lane_addr + half_col;
    const float c = a.scale * paged::kLog2e;
    const uint64_t c2 = ptx::pack2(c, c);
    while (turns.next(sh.queue, wait, &ok)) {
      int n, left, rel, rel_end;                                       // blocks, their tokens, those of them that see this lane's key
      {
        const Item& it = turns.item(sh.queue);
        const int j = it.line * kTile + key;
        n = it.n;
        left = it.nq - it.first * p.tpb;
        rel = j - (it.kv - it.nq) - it.first * p.tpb;
        rel_end = a.window > 0 && j >= a.sinks ? (int)min((long long)rel + a.window, (long long)INT_MAX) : INT_MAX;
      }
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        const uint32_t b = blk + i;
        const int t0 = i * p.tpb, rows = min(p.tpb, left - t0) * p.G;
        // rows of the block that see this lane's key: lo .. hi - 1
        const int lo = min(max(rel - t0, 0), p.tpb) * p.G, hi = min(rows, min(max(rel_end - t0, 0), p.tpb) * p.G);
        const bool masked = __any_sync(0xffffffffu, lo > half_col || hi < half_col + 64);
        const uint32_t see[2] = {bits(lo - half_col, hi - half_col), bits(lo - half_col - 32, hi - half_col - 32)};
        // the rows' statistics come before the scores are waited for: loads from shared memory take long beside the products
        uint64_t w[32];                                                // weights of this lane's key, a pair of rows each
        ok = wait(&sh.stat_full[b & 1u], b >> 1);
        const ulonglong2* lse = reinterpret_cast<const ulonglong2*>(&sh.lse[b & 1u][half_col]);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          const ulonglong2 l = lse[k];
          w[2 * k] = l.x;
          w[2 * k + 1] = l.y;
        }
        ok = __all_sync(0xffffffffu, ok && wait(&sh.s_full, b));
        if (!ok) break;
        ptx::tc_fence_after();
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t v[32], pk[16];
          load32(my_s + 32 * q, v);
          if (masked) mask32(v, see[q], kMinusInf);
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            const uint64_t x = ptx::fma2(ptx::pack2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1])), c2, w[16 * q + k]);
            w[16 * q + k] = k % 3 == 1 ? pow2<true>(x) : pow2<false>(x);
            float e0, e1;
            ptx::unpack2(w[16 * q + k], &e0, &e1);
            pk[k] = ptx::pack_bf16x2(e0, e1);
          }
          ptx::tmem_st16_async(my_s + 16 * q, pk);
        }
        if (rows < block_rows) {                                       // what the load has brought behind the request's rows
          ok = wait(&sh.do_full[b & 1u], b >> 1);
          if (ok) {
            clear_rows<D>(tile(kDo + (b & 1u)), rows, block_rows, threadIdx.x);
            clear_rows<D>(tile(kQ + ring.stage), rows, block_rows, threadIdx.x);
            ptx::fence_proxy_async_smem();
          }
        }
        ptx::tmem_wait_st();
        ptx::tc_fence_before();
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (lane == 0) ptx::mbar_arrive(&sh.p_full);
        const ulonglong2* delta = reinterpret_cast<const ulonglong2*>(&sh.delta[b & 1u][half_col]);
        ulonglong2 d[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) d[k] = delta[k];
        ok = __all_sync(0xffffffffu, wait(&sh.dp_full, b));
        if (!ok) break;
        ptx::tc_fence_after();
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t v[32], pk[16];
          load32(my_dp + 32 * q, v);
          if (masked) mask32(v, see[q], 0u);                           // (beside rows that do not exist anything may stand)
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            const uint64_t x = ptx::add2(ptx::pack2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1])), k & 1 ? d[k / 2].y : d[k / 2].x);
            float e0, e1;
            ptx::unpack2(mul2(w[16 * q + k], x), &e0, &e1);
            pk[k] = ptx::pack_bf16x2(e0, e1);
            if (q == 0 && (k & 1)) d[k / 2] = delta[8 + k / 2];
          }
          ptx::tmem_st16_async(my_dp + 16 * q, pk);
        }
        ptx::tmem_wait_st();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          ptx::mbar_arrive(&sh.ds_full);
          ptx::mbar_arrive(&sh.stat_empty[b & 1u]);
        }
        ring.step();
      }
      if (!ok) break;
      // ---- results: values' gradients by one half of the warps, keys' by the other ----
      if (n > 0) {
        ok = __all_sync(0xffffffffu, wait(&sh.acc_full, used));
        if (!ok) break;
        ptx::tc_fence_after();
        ++used;
        blk += n;
      }
      if (p.split > 1) {
        joined = true;
        join<D>((part == 0 ? t_dv : t_dk) + lane_addr, base, (part * (D / 32) * 8 * kTile + key) * 16, p.split, rank, n > 0);
        if (rank != 0) {
          turns.done(sh.queue, lane);
          continue;
        }
        n = 1;
      }
      const Item it = turns.item(sh.queue);
      const int j = it.line * kTile + key;
      const int page = j < it.kv ? a.block_table[(size_t)it.r * a.table_stride + j / a.page_size] : 0;
      const long long stride = part == 0 ? p.g.dv_stride : p.g.dk_stride;
      const int quad = j & ~3;                                         // the first of the four keys whose columns this lane writes
      __nv_bfloat16* from = static_cast<__nv_bfloat16*>(part == 0 ? p.g.dv : p.g.dk) + ((long long)it.k0 + quad) * stride + it.head * D;
      const float by = part == 0 ? 1.f : a.scale;
      bool finite = true;
#pragma unroll 1
      for (int q = 0; q < D / 32; ++q) {
        uint32_t v[32];
        if (n > 0) {
          load32((part == 0 ? t_dv : t_dk) + lane_addr + 32 * q, v);
        } else {
#pragma unroll
          for (int k = 0; k < 32; ++k) v[k] = 0u;
        }
        __nv_bfloat16* to[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) to[m] = quad + m < it.kv ? from + m * stride + 32 * q : nullptr;
        finite = store_32_columns(v, by, to, lane) && finite;
      }
      if (n > 0) {
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sh.acc_empty);
      }
      // a value that is no number, or too large, at a row that another key of the tile sees; a page outside the pool
      const bool odd = j < it.kv && (page < 0 || page >= a.n_pages || !finite);
      __syncwarp();
      for (uint32_t again = __ballot_sync(0xffffffffu, odd); again != 0u; again &= again - 1u) {
        // (0.6 us a row: whoever waits meanwhile starts its limit anew)
        const int k = it.line * kTile + (warp & 3) * 32 + __ffs(again) - 1;
        if (part == 0)
          paged::grad_key<__nv_bfloat16, D, false, true>(p.g, it.r, it, k, it.head, lane, wait.alive);
        else
          paged::grad_key<__nv_bfloat16, D, true, false>(p.g, it.r, it, k, it.head, lane, wait.alive);
      }
      turns.done(sh.queue, lane);
    }
  }
  if (warp >= kComputeWarps || !joined)
    for (int m = 1; m < p.split; m *= 2) cluster_meet(), cluster_meet();
  __syncwarp();
  if (*wait.abort_flag) __nanosleep(1000000);                          // copies still in flight
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  if (threadIdx.x == 0)                                                // (the other pass lays its own barriers out here)
    for (uint64_t* b = reinterpret_cast<uint64_t*>(&sh); b < reinterpret_cast<uint64_t*>(&sh.queue); ++b) inval(b);
  if (threadIdx.x < kSlots) {
    inval(&sh.queue.full[threadIdx.x]);
    inval(&sh.queue.empty[threadIdx.x]);
  }
  __syncthreads();
}

}  // namespace grad_tc
