// Queries' gradients of the paged attention on the tensor cores (bf16).
//
// A work item is a block of 128 rows (token, query head of the group) of one (request, key head) with all the key tiles (128 keys)
// that any of them sees.  One CTA an SM works through items that a counter hands out.  Per tile:
//     S = Q K^T      P = 2^(c S - lse)      dP = dO V^T      dS = P (dP - delta)      dQ += dS K
// S, dP, dS (bf16), dQ and Q as an operand fill the tensor memory (512 columns at D = 128; with both operands in shared memory a
// product takes all of its bandwidth).  The next S and dP are formed as soon as these have been read, dQ behind dS:
//   * warp 8 loads queries and output gradients once an item, keys through three stages (they are used twice) and values through two;
//   * warp 9 issues S and dP, warp 10 dQ: a warp that issues is held up until the tensor cores have taken its products, and what
//     it waits for next should be looked at meanwhile;
//   * warps 0-7: a row per lane, half of a tile's keys each; P stays in registers.
#pragma once
#include <climits>

#include "paged_grad_tc.cuh"

namespace grad_tc {

constexpr int kOutputs = kStats;                                       // the warp that issues dQ (rows' statistics are read by their own lanes)

struct SharedQ {
  uint64_t q_full, q_empty, do_full, do_empty, a_full, k_full[3], k_empty[3], v_full[2], v_empty[2], s_full, s_empty, dp_full, dp_empty, ds_full,
      ds_empty, acc_full, acc_empty;
  Queue queue;
};

// The whole CTA; `cta` of `n_cta` that begin with this pass, the others (cta >= n_cta) take what its counter hands out.
template <int D>
__device__ __forceinline__ void pass_q(const CUtensorMap& tm_q, const CUtensorMap& tm_do, const CUtensorMap& tm_k, const CUtensorMap& tm_v, const Args& p,
                                        uint8_t* smem, uint32_t base, uint32_t tmem, const Waits& wait, int cta, int n_cta) {
  using C = Cfg<D>;
  SharedQ& sh = *reinterpret_cast<SharedQ*>(smem + C::kTiles * C::kTileBytes + sizeof(Common));
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  // tiles: queries, output gradients, keys of three stages, values of two
  constexpr int kK = 2, kV = 5;
  auto tile = [&](int i) { return base + i * C::kTileBytes; };
  const PagedAttnArgs& a = p.g.a;
  int* taken = p.taken + 1;
  if (threadIdx.x == 0) {
    for (uint64_t* b : {&sh.q_full, &sh.do_full, &sh.do_empty, &sh.s_full, &sh.dp_full, &sh.ds_empty, &sh.acc_full}) ptx::mbar_init(b, 1);
    for (uint64_t* b : {&sh.q_empty, &sh.a_full, &sh.s_empty, &sh.dp_empty, &sh.ds_full, &sh.acc_empty}) ptx::mbar_init(b, kComputeWarps);
    for (int i = 0; i < 3; ++i) {
      ptx::mbar_init(&sh.k_full[i], 1);
      ptx::mbar_init(&sh.k_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      for (uint64_t* b : {&sh.v_full[i], &sh.v_empty[i]}) ptx::mbar_init(b, 1);
    }
    for (int i = 0; i < kSlots; ++i) {
      ptx::mbar_init(&sh.queue.full[i], 1);
      ptx::mbar_init(&sh.queue.empty[i], kWarps - 1);
    }
    ptx::fence_mbar_init();
  }
  __syncthreads();
  const uint32_t t_s = tmem, t_dp = t_s + 128, t_ds = t_s + 256, t_q = t_s + 320, t_dq = t_s + 384;

  Turns turns;
  uint32_t used = 0, done = 0;                                         // items with tiles, and tiles, so far
  Ring<3> ring;                                                        // the keys' stages
  bool ok = true;
  // key tile i of an item: its first tiles reach over the first tokens, the others lie `skip` further
  auto first_key = [](const Item& it, int i) { return (i < it.first ? i : i + it.skip) * kTile; };

  if (warp == kLoads) {
    const Box box(p, lane);
    const uint32_t box_bytes = (uint32_t)p.box_rows * 128u, row_bytes = (uint32_t)(p.tpb * p.G) * 128u * C::kHalves;
    Cursor<false> cur;
    Item it = {};
    for (int item = cta < n_cta ? cta : INT_MIN;;) {
      if (item == INT_MIN) item = __shfl_sync(0xffffffffu, lane == 0 ? n_cta + atomicAdd(taken, 1) : 0, 0);
      const bool more = cur.find(p, item, lane, &it);
      {
        const int x0 = it.kv - it.nq, t0 = it.line * p.tpb, last = x0 + min(it.nq, t0 + p.tpb) - 1;
        const int lo = paged::window_begin(x0 + t0, a.window), lo_tile = lo / kTile;
        it.first = min((min(a.sinks, lo) + kTile - 1) / kTile, lo_tile);
        it.skip = lo_tile - it.first;
        it.n = !more ? -1 : last < 0 ? 0 : last / kTile + 1 - it.skip;
      }
      if (!turns.tell(sh.queue, wait, it, lane, &ok) || !more) break;
      const int granted = lane == 0 ? n_cta + atomicAdd(taken, 1) : 0;
      bool bad = false;
      if (it.n > 0) {
        const int32_t* table = a.block_table + (size_t)it.r * a.table_stride;
        auto rows = [&](int to, const CUtensorMap* m, uint64_t* full, uint64_t* empty) {
          ok = __all_sync(0xffffffffu, ok && wait(empty, used ^ 1u));
          if (ok && lane == 0) {
            ptx::mbar_arrive_expect_tx(full, row_bytes);
            for (int h = 0; h < C::kHalves; ++h)
              ptx::tma_load_4d(smem + to * C::kTileBytes + h * (kTile * 128), m, h * 64, 0, it.head, it.q0 + it.line * p.tpb, full);
          }
        };
        rows(0, &tm_q, &sh.q_full, &sh.q_empty);
        rows(1, &tm_do, &sh.do_full, &sh.do_empty);
        if (!ok) break;
        ++used;
        int row, next_row = 0;
        int page = box.page(p, table, first_key(it, 0), it.kv, C::kHalves, &row, &bad);
        for (int i = 0; i < it.n; ++i, ++done) {
          int next_page = -1;
          if (i + 1 < it.n) next_page = box.page(p, table, first_key(it, i + 1), it.kv, C::kHalves, &next_row, &bad);
          const uint32_t bytes = box_bytes * (uint32_t)__popc(__ballot_sync(0xffffffffu, page >= 0));
          auto load = [&](const CUtensorMap* m, uint64_t* full, uint64_t* empty, uint32_t ph, int to) {
            ok = __all_sync(0xffffffffu, ok && wait(empty, ph ^ 1u));
            if (!ok) return;
            if (lane == 0) ptx::mbar_arrive_expect_tx(full, bytes);
            __syncwarp();
            if (page >= 0)
              ptx::tma_load_4d(smem + to * C::kTileBytes + box.half * (kTile * 128) + box.i * box_bytes, m, box.half * 64, it.head, row, page, full);
          };
          load(&tm_k, &sh.k_full[ring.stage], &sh.k_empty[ring.stage], ring.ph, kK + ring.stage);
          load(&tm_v, &sh.v_full[done & 1u], &sh.v_empty[done & 1u], done >> 1, kV + (done & 1u));
          if (!ok) break;
          ring.step();
          page = next_page;
          row = next_row;
        }
        if (!ok) break;
      }
      bad = __any_sync(0xffffffffu, bad);
      if (bad && lane == 0) static_cast<volatile Item&>(turns.last(sh.queue)).lost = true;   // (before the next item is told)
      item = __shfl_sync(0xffffffffu, granted, 0);
    }
    // everything has been given back before the CTA may end (the arrivals are asynchronous)
    ok = ok && wait(&sh.q_empty, used ^ 1u) && wait(&sh.do_empty, used ^ 1u) && wait(&sh.ds_empty, done ^ 1u);
    for (uint32_t i = 0; i < 2; ++i) ok = ok && wait(&sh.v_empty[(done + i) & 1u], ((done + i) >> 1) ^ 1u);
    for (uint32_t i = 0; i < 3; ++i, ring.step()) ok = ok && wait(&sh.k_empty[ring.stage], ring.ph ^ 1u);
  } else if (warp == kProducts || warp == kOutputs) {
    const uint32_t idesc_s = ptx::umma_idesc_bf16(128, 128), idesc_o = ptx::umma_idesc_bf16_b_mn(128, D);
    const uint64_t desc = ptx::umma_desc_sw128(base), desc_mn = ptx::umma_desc_sw128_strides(base, kTile * 128, 1024);
    auto lo = [&](int i) { return (uint32_t)desc + i * (C::kTileBytes >> 4); };
    auto lo_mn = [&](int i) { return (uint32_t)desc_mn + i * (C::kTileBytes >> 4); };
    auto here = [&](uint64_t* bar, uint32_t parity) { return ok = __all_sync(0xffffffffu, wait(bar, parity)); };
    while (turns.next(sh.queue, wait, &ok)) {
      const int n = __shfl_sync(0xffffffffu, turns.item(sh.queue).n, 0);
      turns.done(sh.queue, lane);
      if (n == 0) continue;
      if (warp == kProducts) {
        if (!here(&sh.a_full, used) || !here(&sh.do_full, used)) break;
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
          const uint32_t t = done + i;
          if (!here(&sh.k_full[ring.stage], ring.ph) || !here(&sh.s_empty, t ^ 1u)) break;
          ptx::tc_fence_after();
          if (elect_one()) {
            product_ts_k<D>(t_s, t_q, lo(kK + ring.stage), desc, idesc_s);
            ptx::umma_commit(&sh.s_full);
          }
          ring.step();
          if (!here(&sh.v_full[t & 1u], t >> 1) || !here(&sh.dp_empty, t ^ 1u)) break;
          ptx::tc_fence_after();
          if (elect_one()) {
            product_ss<D>(t_dp, lo(1), lo(kV + (t & 1u)), desc, idesc_s);
            ptx::umma_commit(&sh.dp_full);
            ptx::umma_commit(&sh.v_empty[t & 1u]);
            if (i + 1 == n) ptx::umma_commit(&sh.do_empty);
          }
        }
        if (!ok) break;
      } else {
        if (!here(&sh.acc_empty, used ^ 1u)) break;
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
          if (!here(&sh.ds_full, done + i)) break;
          ptx::tc_fence_after();
          if (elect_one()) {
            product_ts<32>(t_dq, t_ds, lo_mn(kK + ring.stage), desc_mn, idesc_o, i == 0);
            ptx::umma_commit(&sh.ds_empty);
            ptx::umma_commit(&sh.k_empty[ring.stage]);                 // (its S is done, or there were no dS)
            if (i + 1 == n) ptx::umma_commit(&sh.acc_full);
          }
          ring.step();
        }
        if (!ok) break;
      }
      ++used;
      done += n;
    }
  } else {
    const int part = warp >> 2, rr = threadIdx.x & (kTile - 1);        // which half of the keys; this lane's row
    const int half_col = part * 64;
    const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t my_s = t_s + lane_addr + half_col, my_dp = t_dp + lane_addr + half_col, my_ds = t_ds + lane_addr + part * 32;
    const float c = a.scale * paged::kLog2e;
    const uint64_t c2 = ptx::pack2(c, c);
    const int my_tok = rr / p.G, my_g = rr % p.G;
    while (turns.next(sh.queue, wait, &ok)) {
      int n, x, lo, kv, first, skip;
      uint64_t lse2, delta2;
      {
        const Item& it = turns.item(sh.queue);
        const int tok = it.line * p.tpb + my_tok;
        const bool live = my_tok < p.tpb && tok < it.nq;
        n = it.n;
        kv = it.kv;
        first = it.first;
        skip = it.skip;
        // position (below 0: sees nothing); a place without a row sees everything, which spares its warp the masks
        x = live ? kv - it.nq + tok : INT_MAX / 2;
        lo = live ? paged::window_begin(x, a.window) : 0;
        const bool sees = live && x >= 0;
        const float2 st = sees ? p.g.stats[(long long)(it.q0 + tok) * a.Hq + it.head * p.G + my_g] : make_float2(0.f, 0.f);
        lse2 = ptx::pack2(-st.x, -st.x);
        delta2 = ptx::pack2(-st.y, -st.y);
      }
      if (n > 0) {                                                     // half of this lane's row of Q into tensor memory
        ok = __all_sync(0xffffffffu, wait(&sh.q_full, used));
        if (!ok) break;
#pragma unroll
        for (int k = 0; k < D / 64; ++k) {
          uint32_t y[16];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int piece = part * (D / 16) + 4 * k + e;
            ld_shared_v4(tile(0) + rr * 128 + (piece >> 3) * (kTile * 128) + (((piece & 7) ^ (rr & 7)) << 4), &y[4 * e]);
          }
          ptx::tmem_st16_async(t_q + lane_addr + part * (D / 4) + 16 * k, y);
        }
        ptx::tmem_wait_st();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          ptx::mbar_arrive(&sh.a_full);
          ptx::mbar_arrive(&sh.q_empty);
        }
      }
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        const uint32_t t = done + i;
        const int tile_key = (i < first ? i : i + skip) * kTile, k0 = tile_key + half_col;
        // bit k: this row sees key k0 + 32 q + k
        uint32_t see[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const int j0 = k0 + 32 * q;
          see[q] = bits(INT_MIN, x - j0 + 1) & (bits(lo - j0, 32) | bits(INT_MIN, a.sinks - j0));
        }
        const bool masked = __any_sync(0xffffffffu, (see[0] & see[1]) != 0xffffffffu);
        ok = __all_sync(0xffffffffu, wait(&sh.s_full, t));
        if (!ok) break;
        ptx::tc_fence_after();
        uint64_t w[32];                                                // weights of this lane's row, a pair of keys each
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t v[32];
          load32(my_s + 32 * q, v);
          if (q == 1) {                                                // the next tile's may come
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&sh.s_empty);
          }
          if (masked) mask32(v, see[q], kMinusInf);
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            const uint64_t y = ptx::fma2(ptx::pack2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1])), c2, lse2);
            w[16 * q + k] = k % 3 == 1 ? pow2<true>(y) : pow2<false>(y);
          }
        }
        if (tile_key + kTile > kv) {                                   // keys behind the last: whatever the page held before
          ok = wait(&sh.k_full[ring.stage], ring.ph);
          if (ok) {
            clear_rows<D>(tile(kK + ring.stage), kv - tile_key, kTile, threadIdx.x);
            ptx::fence_proxy_async_smem();
          }
        }
        ok = __all_sync(0xffffffffu, ok && wait(&sh.ds_empty, t ^ 1u) && wait(&sh.dp_full, t));
        if (!ok) break;
        ptx::tc_fence_after();
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t v[32], pk[16];
          load32(my_dp + 32 * q, v);
          if (q == 1) {
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&sh.dp_empty);
          }
          if (masked) mask32(v, see[q], 0u);                           // (beside keys that do not exist anything may stand)
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            const uint64_t y = ptx::add2(ptx::pack2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1])), delta2);
            float e0, e1;
            ptx::unpack2(mul2(w[16 * q + k], y), &e0, &e1);
            pk[k] = ptx::pack_bf16x2(e0, e1);
          }
          ptx::tmem_st16_async(my_ds + 16 * q, pk);
        }
        ptx::tmem_wait_st();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sh.ds_full);
        ring.step();
      }
      if (!ok) break;
      // ---- results: half of a row's elements each ----
      if (n > 0) {
        ok = __all_sync(0xffffffffu, wait(&sh.acc_full, used));
        if (!ok) break;
        ptx::tc_fence_after();
        ++used;
        done += n;
      }
      const Item it = turns.item(sh.queue);
      const int tok = it.line * p.tpb + my_tok, row = it.q0 + tok, q_head = it.head * p.G + my_g;
      const bool live = my_tok < p.tpb && tok < it.nq;
      __nv_bfloat16* mine = live ? static_cast<__nv_bfloat16*>(p.g.dq) + (long long)row * p.g.dq_stride + q_head * D + part * (D / 2) : nullptr;
      __nv_bfloat16* to[4];                                            // of the four rows whose columns this lane writes
#pragma unroll
      for (int m = 0; m < 4; ++m)
        to[m] = reinterpret_cast<__nv_bfloat16*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(mine), (lane & ~3) + m));
      bool finite = true;
#pragma unroll 1
      for (int q = 0; q < D / 64; ++q) {
        uint32_t v[32];
        if (n > 0) {
          load32(t_dq + lane_addr + part * (D / 2) + 32 * q, v);
        } else {
#pragma unroll
          for (int k = 0; k < 32; ++k) v[k] = 0u;
        }
        finite = store_32_columns(v, a.scale, to, lane) && finite;
#pragma unroll
        for (int m = 0; m < 4; ++m)
          if (to[m] != nullptr) to[m] += 32;
      }
      if (n > 0) {
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sh.acc_empty);
      }
      __syncwarp();
      // where the next item is told the loads of this one have ended: whether its keys were all there is known
      ok = __all_sync(0xffffffffu, turns.next_is_told(sh.queue, wait));
      if (!ok) break;
      const bool lost = static_cast<const volatile Item&>(turns.item(sh.queue)).lost;
      // (rows that see no key too: beside a key that holds no number their zeros became none)
      const bool odd = live && (!finite || lost);
      // (0.6 us a key and row: whoever waits meanwhile starts its limit anew; each warp sees to its half of the row's elements)
      for (uint32_t again = __ballot_sync(0xffffffffu, odd); again != 0u; again &= again - 1u) {
        const int who = __ffs(again) - 1;
        paged::grad_row<__nv_bfloat16, D>(p.g, it.r, __shfl_sync(0xffffffffu, row, who), __shfl_sync(0xffffffffu, x, who),
                                          __shfl_sync(0xffffffffu, q_head, who), lane, part * (D / 64), (part + 1) * (D / 64), wait.alive);
      }
      turns.done(sh.queue, lane);
    }
  }
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
