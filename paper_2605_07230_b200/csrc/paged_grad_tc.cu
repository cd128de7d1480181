// The gradient of the attention over a paged cache on the tensor cores (bf16): keys' and queries' passes side by side in one launch.
//
// A CTA an SM; some begin with the keys' pass, the rest with the queries' (a step of 128 x 128 takes 4.1 and 2.9 thousand cycles, of
// which the products alone need 2.0 and 1.5).  Where there are many items a CTA that finds no more goes on with the other pass.
//
// 8 sequences of 2480 tokens, 32 heads of 128: 1.57 to 1.72 ms, 590 to 640 TFLOP/s of the five products that have to be, 820 to 900 of the
// seven that are formed (the card's best: 1694); 2 of 640 tokens: 63 us; 12 of 100 to 1144, 20 heads of 64: 168 us.  On 2 sequences of
// 2480 tokens (393 us) the tensor cores are busy 53 % of the time.  What holds them up: the first and last steps of an item, which nothing
// lies beside (7 and 9 thousand cycles an item), and weights and their gradients on the way through the registers.
#include "paged_grad_kv.cuh"
#include "paged_grad_q.cuh"

namespace {

using namespace grad_tc;

template <int D>
constexpr int kSmem = Cfg<D>::kTiles * Cfg<D>::kTileBytes + (int)sizeof(Common) +
                      (int)(sizeof(SharedKv) > sizeof(SharedQ) ? sizeof(SharedKv) : sizeof(SharedQ));
static_assert(kSmem<128> <= 232448, "shared memory of a CTA");
static_assert(sizeof(Common) % 16 == 0, "alignment of what follows");

template <int D>
__global__ void __launch_bounds__(kThreads, 1)
k_paged_grad_tc(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_do, const __grid_constant__ CUtensorMap tm_k,
                const __grid_constant__ CUtensorMap tm_v, const Args p) {
  extern __shared__ __align__(1024) uint8_t smem[];
  Common& sh = *reinterpret_cast<Common*>(smem + Cfg<D>::kTiles * Cfg<D>::kTileBytes);
  const uint32_t base = ptx::smem_u32(smem);
  if ((base & 1023u) != 0) {                                           // (the same in all threads of all CTAs)
    if (threadIdx.x == 0) atomicOr(p.g.a.err, CASCADE_DEV_ERR_WAIT);
    return;
  }
  const int warp = threadIdx.x >> 5;
  const Waits wait = {&sh.abort_flag, &sh.alive, p.g.a.err, p.g.a.wait_ns};
  if (threadIdx.x == 0) {
    sh.abort_flag = 0;
    sh.alive = 0;
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
  const uint32_t tmem = sh.tmem;
  const bool keys_first = (int)blockIdx.x < p.n_cta_keys;
  const int n_q = (int)gridDim.x - p.n_cta_keys;
#pragma unroll 1
  for (int k = 0; k < (p.both ? 2 : 1) && !*wait.abort_flag; ++k) {
    const bool keys = keys_first == (k == 0);
    const int cta = k != 0 ? INT_MAX : keys ? (int)blockIdx.x / p.split : (int)blockIdx.x - p.n_cta_keys;
    if (keys)
      pass_kv<D>(tm_q, tm_do, tm_k, tm_v, p, smem, base, tmem, wait, cta, p.n_cta_keys / p.split);
    else
      pass_q<D>(tm_q, tm_do, tm_k, tm_v, p, smem, base, tmem, wait, cta, n_q);
  }
  if (threadIdx.x == 0 && atomicAdd(p.taken + 2, 1) == (int)gridDim.x - 1) p.taken[0] = p.taken[1] = p.taken[2] = 0;
  if (warp == kProducts) ptx::tmem_dealloc(tmem, 512);
}

template <int D>
int launch(cascade_ctx* ctx, const Args& p, int grid, cudaStream_t s) {
  const PagedAttnArgs& a = p.g.a;
  CUtensorMap mq, mo;
  const CUtensorMap *mk = page_map(ctx, p, D, a.k), *mv = page_map(ctx, p, D, a.v);
  if (mk == nullptr || mv == nullptr || !row_map(&mq, p, D, a.q, a.q_stride) || !row_map(&mo, p, D, p.g.d_out, (long long)a.Hq * D))
    return CASCADE_ERR_CUDA;
  CASCADE_TRY(configure_smem(ctx, PAGED_CFG_GRAD_TC, k_paged_grad_tc<D>, kSmem<D>));   // (a context has one D)
  KernelScope ks(ctx, K_PAGED_GRAD, s);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kSmem<D>;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = p.split;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  CASCADE_CUDA_TRY(cudaLaunchKernelEx(&cfg, k_paged_grad_tc<D>, mq, mo, *mk, *mv, p));
  return CASCADE_OK;
}

// No more items than this: a request's tiles are at most ceil(length / unit).
long long most_items(const PagedAttnArgs& a, long long total, int most, int unit) {
  const long long pieces = total / unit + a.n_req, by_length = (long long)a.n_req * ((most + unit - 1) / unit);
  return (pieces < by_length ? pieces : by_length) * a.Hkv;
}

}  // namespace

int launch_paged_grad_tc(cascade_ctx* ctx, const PagedGradArgs& g, cudaStream_t s) {
  const PagedAttnArgs& a = g.a;
  Args p;
  p.g = g;
  p.G = a.Hq / a.Hkv;
  p.tpb = kTile / p.G;
  p.box_rows = 8;
  while (p.box_rows < kTile && a.page_size % (2 * p.box_rows) == 0) p.box_rows *= 2;
  p.taken = ctx->dev_error + 40;   // (cleared with the error word when the context is made)
  const long long keys = most_items(a, g.n_kv, a.max_kv, kTile), rows = most_items(a, a.n_tok, a.max_q, p.tpb), sms = ctx->sm_count;
  if (keys > INT_MAX / 2 || rows > INT_MAX / 2) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  // All items at once if there are no more than SMs; else the SMs in proportion to the passes' time: thousands of cycles an item and
  // a step, of which there are as many in both, estimated from the requests' mean lengths.  (2 x 640 tokens, 32 heads of 128: 64 us; by
  // 41 : 29 an item, which is right for long rows alone, 67 us.)
  const bool wide = ctx->shape.D == 128;
  double seen = ((double)g.n_kv - 0.5 * a.n_tok) / a.n_req;            // keys that a row sees
  if (a.window > 0 && seen > (double)a.window + a.sinks) seen = (double)a.window + a.sinks;
  const double steps = (seen > 0 ? seen / kTile + 0.5 : 0.5) * rows, item_keys = wide ? 7 : 4, item_rows = wide ? 8.8 : 4.2;
  const double time_keys = item_keys * (double)keys + 4.05 * steps, time_rows = item_rows * (double)rows + 2.9 * steps;
  if (keys + rows <= sms) {
    p.n_cta_keys = (int)keys;
  } else {
    const long long share = (long long)(sms * time_keys / (time_keys + time_rows) + 0.5), most = keys < sms - 1 ? keys : sms - 1;
    p.n_cta_keys = (int)(keys == 0 ? 0 : share < 1 ? 1 : share > most ? most : share);
  }
  // Few tiles of keys with many row blocks each: the blocks of a tile are shared out where that shortens the longest walk or wait by a
  // tenth.  Adding up another CTA's results takes 16 (D = 64: 8) thousand cycles.  (2 x 500 tokens, 8 query heads of 128 on one key
  // head: 40 us, without 74 us; 2000 tokens, 8 heads of 64 on one: 68 us, without 198 us.)
  p.split = 1;
  if (keys > 0) {
    double blocks = (double)((a.max_q + p.tpb - 1) / p.tpb);
    if (a.window > 0 && a.sinks == 0 && blocks > ((double)a.window + kTile) / p.tpb + 1) blocks = ((double)a.window + kTile) / p.tpb + 1;
    const double row_item = item_rows + 2.9 * (a.window > 0 && (double)a.max_kv > (double)a.window + a.sinks ? ((double)a.window + a.sinks) / kTile + 1
                                                                                                             : (double)a.max_kv / kTile);
    auto longest = [](double x, double y) { return x > y ? x : y; };
    double best = 0.9 * longest(longest(item_keys + 4.05 * blocks, row_item), (time_keys + time_rows) / sms);
    for (int n = 2, levels = 1; n <= 8 && keys * n < sms; n *= 2, ++levels) {
      const long long for_rows = rows < sms - keys * n ? rows : sms - keys * n;
      const double time = longest(longest(item_keys + 4.05 * blocks / n + levels * (wide ? 16 : 8), row_item), time_rows / for_rows);
      if (time >= best) continue;
      best = time;
      p.split = n;
      p.n_cta_keys = (int)keys * n;
    }
  }
  const long long left = sms - p.n_cta_keys;
  int grid = p.n_cta_keys + (int)(rows < left ? rows : left);
  grid = (grid + p.split - 1) / p.split * p.split;                     // (whole clusters; the last ones may find no rows)
  p.both = p.split == 1 && keys + rows > 4 * sms;
  return ctx->shape.D == 128 ? launch<128>(ctx, p, grid, s) : launch<64>(ctx, p, grid, s);
}
