// Queries' gradients of the paged attention on the tensor cores (bf16).
//
// A work item is a block of 128 rows (token, query head of the group) of one (request, key head) with all the key tiles (128 keys)
// that any of them sees.  One CTA an SM works through items that a counter hands out.  Per tile:
//     S = Q K^T      P = 2^(c S - lse)      dP = dO V^T      dS = P (dP - delta)      dQ += dS K
// Two buffers of S, dP and dQ fill the tensor memory (4 x 128 columns at D = 128); dS goes back as bf16 over its own scores, so that
// the next tile's S and dP are formed while this one's dS is:
//   * warp 8 loads queries and output gradients once an item, keys through three stages (they are used twice) and values through two;
//   * warp 9 issues the products;  warps 0-7: a row per lane, half of a tile's keys each.
#include <climits>

#include "paged_grad_tc.cuh"

namespace {

using namespace grad_tc;

constexpr int kQWarps = kProducts + 1, kQThreads = kQWarps * 32;     // (rows' statistics are read by their own lanes)

struct Shared {
  uint64_t q_full, q_empty, k_full[3], k_empty[3], v_full[2], v_empty[2], s_full[2], ds_full[2], dp_full, dp_empty, acc_full, acc_empty;
  Queue queue;
  uint64_t alive;
  int abort_flag;
  uint32_t tmem;
};

template <int D>
__global__ void __launch_bounds__(kQThreads, 1)
k_paged_grad_q(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_do, const __grid_constant__ CUtensorMap tm_k,
               const __grid_constant__ CUtensorMap tm_v, const Args p) {
  using C = Cfg<D>;
  extern __shared__ __align__(1024) uint8_t smem[];
  Shared& sh = *reinterpret_cast<Shared*>(smem + C::kTiles * C::kTileBytes);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = ptx::smem_u32(smem);
  // tiles: queries, output gradients, keys of three stages, values of two
  constexpr int kK = 2, kV = 5;
  auto tile = [&](int i) { return base + i * C::kTileBytes; };
  const PagedAttnArgs& a = p.g.a;
  if ((base & 1023u) != 0) {                                           // (the same in all threads of all CTAs)
    if (threadIdx.x == 0) atomicOr(a.err, CASCADE_DEV_ERR_WAIT);
    return;
  }
  const Waits wait = {&sh.abort_flag, &sh.alive, a.err, a.wait_ns};

  if (threadIdx.x == 0) {
    for (uint64_t* b : {&sh.q_full, &sh.q_empty, &sh.dp_full, &sh.acc_full}) ptx::mbar_init(b, 1);
    for (uint64_t* b : {&sh.dp_empty, &sh.ds_full[0], &sh.ds_full[1], &sh.acc_empty}) ptx::mbar_init(b, kComputeWarps);
    for (int i = 0; i < 3; ++i) {
      ptx::mbar_init(&sh.k_full[i], 1);
      ptx::mbar_init(&sh.k_empty[i], 1);
    }
    for (int i = 0; i < 2; ++i) {
      for (uint64_t* b : {&sh.v_full[i], &sh.v_empty[i], &sh.s_full[i], &sh.queue.full[i]}) ptx::mbar_init(b, 1);
      ptx::mbar_init(&sh.queue.empty[i], kQWarps);
    }
    sh.abort_flag = 0;
    sh.alive = 0;
    ptx::fence_mbar_init();
  }
  if (warp == kLoads && lane == 0) {
    ptx::prefetch_tmap(&tm_q);
    ptx::prefetch_tmap(&tm_do);
    ptx::prefetch_tmap(&tm_k);
    ptx::prefetch_tmap(&tm_v);
  }
  if (warp == kProducts) {
    ptx::tmem_alloc(&sh.tmem, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  const uint32_t t_s = sh.tmem, t_dp = t_s + 256, t_dq = t_s + 384;    // (S of an odd tile at 128)

  Cursor<false> cur;
  paged::GradRequest rq = {};
  int r = 0, head = 0, line = 0;
  uint32_t turn = 0;                                                   // items that this warp has taken
  bool lost = false;                                                   // the item that was left for this one met a bad page
  auto next = [&]() {
    const uint32_t slot = turn & 1u, use = turn >> 1;
    ++turn;
    const bool here = wait(&sh.queue.full[slot], use);
    const int item = here ? *static_cast<volatile int*>(&sh.queue.answer[slot]) : INT_MAX;
    lost = here && *static_cast<volatile bool*>(&sh.queue.lost[slot]);
    __syncwarp();
    if (lane == 0) ptx::mbar_arrive(&sh.queue.empty[slot]);
    return __shfl_sync(0xffffffffu, item, 0);
  };
  // the item's key tiles: tile i is i (i < n_sink) or i + skip
  int n_sink = 0, skip = 0;
  auto tiles = [&]() {
    const int x0 = rq.kv - rq.nq, t0 = line * p.tpb, last = x0 + min(rq.nq, t0 + p.tpb) - 1;
    const int lo = paged::window_begin(x0 + t0, a.window), lo_tile = lo / kTile;
    n_sink = min((min(a.sinks, lo) + kTile - 1) / kTile, lo_tile);
    skip = lo_tile - n_sink;
    return last < 0 ? 0 : last / kTile + 1 - skip;
  };
  auto first_key = [&](int i) { return (i < n_sink ? i : i + skip) * kTile; };
  uint32_t used = 0, done = 0;                                         // items with tiles, and tiles, so far
  Ring<3> ring;                                                        // the keys' stages
  bool ok = true;

  if (warp == kLoads) {
    const Box box(p, lane);
    const uint32_t box_bytes = (uint32_t)p.box_rows * 128u, row_bytes = (uint32_t)(p.tpb * p.G) * 128u * C::kHalves;
    for (int item = blockIdx.x; ok && cur.find(p, item, lane, &rq, &r, &head, &line); item = next()) {
      const int granted = lane == 0 ? (int)gridDim.x + atomicAdd(p.taken, 1) : 0;
      const int n = tiles();
      bool bad = false;
      if (n > 0) {
        const int32_t* table = a.block_table + (size_t)r * a.table_stride;
        ok = ok && wait(&sh.q_empty, used ^ 1u);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        if (lane == 0) {
          ptx::mbar_arrive_expect_tx(&sh.q_full, 2u * row_bytes);
          for (int h = 0; h < C::kHalves; ++h) {
            ptx::tma_load_4d(smem + h * (kTile * 128), &tm_q, h * 64, 0, head, rq.q0 + line * p.tpb, &sh.q_full);
            ptx::tma_load_4d(smem + C::kTileBytes + h * (kTile * 128), &tm_do, h * 64, 0, head, rq.q0 + line * p.tpb, &sh.q_full);
          }
        }
        ++used;
        int row, next_row = 0;
        int page = box.page(p, table, first_key(0), rq.kv, C::kHalves, &row, &bad);
        for (int i = 0; i < n; ++i, ++done) {
          int next_page = -1;
          if (i + 1 < n) next_page = box.page(p, table, first_key(i + 1), rq.kv, C::kHalves, &next_row, &bad);
          const uint32_t bytes = box_bytes * (uint32_t)__popc(__ballot_sync(0xffffffffu, page >= 0));
          auto load = [&](const CUtensorMap* m, uint64_t* full, uint64_t* empty, uint32_t ph, int to) {
            ok = ok && wait(empty, ph ^ 1u);
            ok = __all_sync(0xffffffffu, ok);
            if (!ok) return;
            if (lane == 0) ptx::mbar_arrive_expect_tx(full, bytes);
            __syncwarp();
            if (page >= 0)
              ptx::tma_load_4d(smem + to * C::kTileBytes + box.half * (kTile * 128) + box.i * box_bytes, m, box.half * 64, head, row, page, full);
          };
          load(&tm_k, &sh.k_full[ring.stage], &sh.k_empty[ring.stage], ring.ph, kK + ring.stage);
          load(&tm_v, &sh.v_full[done & 1u], &sh.v_empty[done & 1u], done >> 1, kV + (done & 1u));
          if (!ok) break;
          ring.step();
          page = next_page;
          row = next_row;
        }
      }
      const uint32_t slot = turn & 1u, use = turn >> 1;
      ok = ok && wait(&sh.queue.empty[slot], use ^ 1u);
      ok = __all_sync(0xffffffffu, ok);
      if (!ok) break;
      bad = __any_sync(0xffffffffu, bad);
      if (lane == 0) {
        *static_cast<volatile int*>(&sh.queue.answer[slot]) = granted;
        *static_cast<volatile bool*>(&sh.queue.lost[slot]) = bad;
        ptx::mbar_arrive(&sh.queue.full[slot]);
      }
    }
    // everything has been given back before the CTA may end (the arrivals are asynchronous)
    ok = ok && wait(&sh.q_empty, used ^ 1u);
    for (uint32_t i = 0; i < 2; ++i) ok = ok && wait(&sh.v_empty[(done + i) & 1u], ((done + i) >> 1) ^ 1u);
    for (uint32_t i = 0; i < 3; ++i, ring.step()) ok = ok && wait(&sh.k_empty[ring.stage], ring.ph ^ 1u);
  } else if (warp == kProducts) {
    const uint32_t idesc_s = ptx::umma_idesc_bf16(128, 128), idesc_o = ptx::umma_idesc_bf16_b_mn(128, D);
    const uint64_t desc = ptx::umma_desc_sw128(base), desc_mn = ptx::umma_desc_sw128_strides(base, kTile * 128, 1024);
    auto lo = [&](int i) { return (uint32_t)desc + i * (C::kTileBytes >> 4); };
    auto lo_mn = [&](int i) { return (uint32_t)desc_mn + i * (C::kTileBytes >> 4); };
    Ring<3> behind;                                                    // the stage of the tile whose last product comes next
    auto scores = [&](uint32_t t) {
      if (!(ok = wait(&sh.k_full[ring.stage], ring.ph))) return;
      product_ss<D>(t_s + (t & 1u) * 128, lo(0), lo(kK + ring.stage), desc, idesc_s);
      ptx::umma_commit(&sh.s_full[t & 1u]);
      ring.step();
    };
    auto d_weights = [&](uint32_t t) {
      if (!(ok = wait(&sh.v_full[t & 1u], t >> 1)) || !(ok = wait(&sh.dp_empty, t ^ 1u))) return;
      ptx::tc_fence_after();
      product_ss<D>(t_dp, lo(1), lo(kV + (t & 1u)), desc, idesc_s);
      ptx::umma_commit(&sh.dp_full);
      ptx::umma_commit(&sh.v_empty[t & 1u]);
    };
    auto work = [&](int n) {
      if (!(ok = wait(&sh.q_full, used))) return;
      scores(done);
      if (!ok) return;
      d_weights(done);
      if (!ok) return;
      if (n == 1) ptx::umma_commit(&sh.q_empty);
#pragma unroll 1
      for (int i = 0; i < n; ++i) {
        const uint32_t t = done + i;
        if (i + 1 < n) {
          scores(t + 1);
          if (!ok) return;
          d_weights(t + 1);
          if (!ok) return;
          if (i + 2 == n) ptx::umma_commit(&sh.q_empty);
        }
        if (i == 0 && !(ok = wait(&sh.acc_empty, used ^ 1u))) return;
        if (!(ok = wait(&sh.ds_full[t & 1u], t >> 1))) return;         // (the next tile's may come before this is looked at)
        ptx::tc_fence_after();
        product_ts(t_dq, t_s + (t & 1u) * 128, lo_mn(kK + behind.stage), desc_mn, idesc_o, i == 0);
        ptx::umma_commit(&sh.k_empty[behind.stage]);
        behind.step();
      }
      ptx::umma_commit(&sh.acc_full);
    };
    for (int item = blockIdx.x; ok && cur.find(p, item, lane, &rq, &r, &head, &line); item = next()) {
      const int n = tiles();
      if (n == 0) continue;
      if (lane == 0) work(n);
      ok = __shfl_sync(0xffffffffu, ok, 0);
      ++used;
      done += n;
    }
  } else {
    const int part = warp >> 2, rr = threadIdx.x & (kTile - 1);        // which half of the keys; this lane's row
    const uint32_t lane_addr = (uint32_t)((warp & 3) * 32) << 16, half_col = part * 64;
    const uint32_t my_s = t_s + lane_addr + half_col, my_dp = t_dp + lane_addr + half_col;
    const float c = a.scale * paged::kLog2e;
    const uint64_t c2 = ptx::pack2(c, c);
    const int my_tok = rr / p.G, my_g = rr % p.G;
    for (int item = blockIdx.x; ok && cur.find(p, item, lane, &rq, &r, &head, &line);) {
      const int n = tiles(), tok = line * p.tpb + my_tok;
      const bool live = my_tok < p.tpb && tok < rq.nq;
      // position (below 0: sees nothing); a place without a row sees everything, which spares its warp the masks
      const int x = live ? rq.kv - rq.nq + tok : INT_MAX / 2;
      const int lo = live ? paged::window_begin(x, a.window) : 0;
      const long long at = (long long)(rq.q0 + tok) * a.Hq + head * p.G + my_g;
      const float2 st = live ? p.g.stats[at] : make_float2(0.f, 0.f);
      const uint64_t lse2 = ptx::pack2(-st.x, -st.x), delta2 = ptx::pack2(-st.y, -st.y);
      for (int i = 0; i < n; ++i) {
        const uint32_t t = done + i;
        const uint32_t ms = my_s + (t & 1u) * 128;
        const int k0 = first_key(i) + (int)half_col;
        // bit k: this row sees key k0 + 32 q + k
        uint32_t see[2];
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          const int j0 = k0 + 32 * q;
          see[q] = bits(INT_MIN, x - j0 + 1) & (bits(lo - j0, 32) | bits(INT_MIN, a.sinks - j0));
        }
        const bool masked = __any_sync(0xffffffffu, (see[0] & see[1]) != 0xffffffffu);
        ok = wait(&sh.s_full[t & 1u], t >> 1);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        ptx::tc_fence_after();
        uint64_t w[32];                                                // weights of this lane's row, a pair of keys each
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t v[32];
          load32(ms + 32 * q, v);
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            float e0, e1;
            ptx::unpack2(ptx::fma2(ptx::pack2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1])), c2, lse2), &e0, &e1);
            w[16 * q + k] = ptx::pack2(ptx::ex2(e0), ptx::ex2(e1));
          }
        }
        if (first_key(i) + kTile > rq.kv) {                            // keys behind the last: whatever the page held before
          ok = wait(&sh.k_full[ring.stage], ring.ph);
          if (ok) {
            clear_rows<D>(tile(kK + ring.stage), rq.kv - first_key(i), kTile, threadIdx.x);
            ptx::fence_proxy_async_smem();
          }
        }
        ok = ok && wait(&sh.dp_full, t);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        ptx::tc_fence_after();
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          uint32_t v[32], pk[16];
          load32(my_dp + 32 * q, v);
          if (q == 1) {                                                // the next tile's may come
            ptx::tc_fence_before();
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&sh.dp_empty);
          }
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            const uint64_t ds = mul2(w[16 * q + k], ptx::add2(ptx::pack2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1])), delta2));
            float e0, e1;
            ptx::unpack2(ds, &e0, &e1);
            if (masked) {
              e0 = (see[q] >> (2 * k)) & 1u ? e0 : 0.f;
              e1 = (see[q] >> (2 * k + 1)) & 1u ? e1 : 0.f;
            }
            pk[k] = ptx::pack_bf16x2(e0, e1);
          }
          ptx::tmem_st16_async(ms + 16 * q, pk);
        }
        ptx::tmem_wait_st();
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sh.ds_full[t & 1u]);
        ring.step();
      }
      if (!ok) break;
      // ---- results: half of a row's elements each ----
      if (n > 0) {
        ok = wait(&sh.acc_full, used);
        ok = __all_sync(0xffffffffu, ok);
        if (!ok) break;
        ptx::tc_fence_after();
        ++used;
        done += n;
      }
      const int row = rq.q0 + tok, q_head = head * p.G + my_g;
      __nv_bfloat16* to = static_cast<__nv_bfloat16*>(p.g.dq) + (long long)row * p.g.dq_stride + q_head * D + part * (D / 2);
      float bad = 0.f;
#pragma unroll 1
      for (int q = 0; q < D / 64; ++q) {
        uint32_t v[32];
        if (n > 0) {
          load32(t_dq + lane_addr + part * (D / 2) + 32 * q, v);
        } else {
#pragma unroll
          for (int k = 0; k < 32; ++k) v[k] = 0u;
        }
#pragma unroll
        for (int k = 0; k < 32; ++k) bad = fmaf(__uint_as_float(v[k]), 0.f, bad);   // NaN if any is not finite
        if (live) {
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint32_t y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              y[e] = ptx::pack_bf16x2(__uint_as_float(v[8 * k + 2 * e]) * a.scale, __uint_as_float(v[8 * k + 2 * e + 1]) * a.scale);
            *reinterpret_cast<uint4*>(to + 32 * q + 8 * k) = make_uint4(y[0], y[1], y[2], y[3]);
          }
        }
      }
      if (n > 0) {
        ptx::tc_fence_before();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sh.acc_empty);
      }
      __syncwarp();
      // the answer for the next item tells whether this one's keys were all there: the loads ended long ago
      const int r_was = r;
      item = next();
      const bool odd = live && x >= 0 && (bad != 0.f || lost);
      // (0.6 us a key and row: whoever waits meanwhile starts its limit anew; each warp sees to its half of the row's elements)
      for (uint32_t left = __ballot_sync(0xffffffffu, odd); left != 0u; left &= left - 1u) {
        const int who = __ffs(left) - 1;
        paged::grad_row<__nv_bfloat16, D>(p.g, r_was, __shfl_sync(0xffffffffu, row, who), __shfl_sync(0xffffffffu, x, who),
                                          __shfl_sync(0xffffffffu, q_head, who), lane, part * (D / 64), (part + 1) * (D / 64), &sh.alive);
      }
    }
  }
  __syncwarp();
  if (*wait.abort_flag) __nanosleep(1000000);                          // copies still in flight
  ptx::tc_fence_before();
  __syncthreads();
  ptx::tc_fence_after();
  if (threadIdx.x == 0 && atomicAdd(p.taken + 1, 1) == (int)gridDim.x - 1) p.taken[0] = p.taken[1] = 0;
  if (warp == kProducts) ptx::tmem_dealloc(t_s, 512);
}

template <int D>
int launch(cascade_ctx* ctx, const Args& p, int grid, cudaStream_t s) {
  const PagedAttnArgs& a = p.g.a;
  CUtensorMap mq, mo;
  const CUtensorMap *mk = page_map(ctx, p, D, a.k), *mv = page_map(ctx, p, D, a.v);
  if (mk == nullptr || mv == nullptr || !row_map(&mq, p, D, a.q, a.q_stride) || !row_map(&mo, p, D, p.g.d_out, (long long)a.Hq * D))
    return CASCADE_ERR_CUDA;
  constexpr int kSmem = smem_bytes<D, Shared>();
  CASCADE_TRY(configure_smem(ctx, PAGED_CFG_GRAD_Q, k_paged_grad_q<D>, kSmem));   // (a context has one D)
  KernelScope ks(ctx, K_PAGED_GRAD, s);
  k_paged_grad_q<D><<<grid, kQThreads, kSmem, s>>>(mq, mo, *mk, *mv, p);
  CASCADE_CUDA_TRY(cudaGetLastError());
  return CASCADE_OK;
}

}  // namespace

int launch_paged_grad_q(cascade_ctx* ctx, const grad_tc::Args& p, cudaStream_t s) {
  const PagedAttnArgs& a = p.g.a;
  // no more items than this: a request's blocks are at most ceil(tokens / tpb)
  const long long blocks = (long long)a.n_tok / p.tpb + a.n_req, by_length = (long long)a.n_req * ((a.max_q + p.tpb - 1) / p.tpb);
  const long long items = (blocks < by_length ? blocks : by_length) * a.Hkv;
  if (items > INT_MAX / 2) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  const int grid = (int)(items < ctx->sm_count ? items : ctx->sm_count);
  return ctx->shape.D == 128 ? launch<128>(ctx, p, grid, s) : launch<64>(ctx, p, grid, s);
}
