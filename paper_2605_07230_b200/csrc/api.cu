// Host side of the C ABI: argument validation, context and tree descriptors, and the composition of
// the kernels into the exported calls.
#include <atomic>
#include <cstdio>
#include <cstring>
#include <new>

#include "cascade_internal.h"
#include "gemm_tc.h"
#include "operand.cuh"
#include "tmap.h"

namespace cascade_detail {
static thread_local cudaError_t g_last_cuda_error = cudaSuccess;
void note_cuda_error(cudaError_t e) {
  g_last_cuda_error = e;
  (void)cudaGetLastError();  // clear the sticky-free error so later calls start clean
}
}  // namespace cascade_detail

using cascade_detail::align_up;
using cascade_detail::ceil_div;

namespace {

struct Carver {
  int64_t off = 0;
  char* base = nullptr;
  template <typename T>
  void take(T*& p, int64_t count) {
    off = align_up(off, 256);
    if (base != nullptr) p = reinterpret_cast<T*>(base + off);
    off += count * (int64_t)sizeof(T);
  }
};

int elem_size(const cascade_shape& s) { return s.dtype == CASCADE_BF16 ? 2 : 4; }

// Every state a tree descriptor ever holds gets its own number: a recorded step can be told from a step on a
// descriptor that was destroyed and re-created at the same address, or updated in place.
uint64_t next_tree_uid() {
  static std::atomic<uint64_t> counter{0};
  return ++counter;
}

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// Lays out every scratch region; with base == nullptr it only measures.
int64_t carve(cascade_ctx* c, char* base) {
  const cascade_shape& s = c->shape;
  const int R = 2 * s.B, T = s.T_max;
  const int64_t BT = (int64_t)s.B * T;
  Carver cv;
  cv.base = base;
  cv.take(c->dev_error, 64);
  cv.take(c->gemm_flags, 1024);
  cv.take(c->tail_counters, s.B);
  c->head_m_pad = (int)align_up(BT, 128);
  if (s.dtype == CASCADE_BF16) {
    cv.take(c->head_a, operand_elems((int)BT, s.h));
    c->head_max_tiles = ceil_div(s.V, 128);
    cv.take(c->head_part, (int64_t)c->head_max_tiles * c->head_m_pad);
    cv.take(c->gemm_scratch, gemm_tc_scratch_floats(c->sm_count));
  } else {
    cv.take(c->head_a_f32, BT * s.h);
  }
  cv.take(c->feat, BT * s.h);
  cv.take(c->feat_norm, BT);
  cv.take(c->row_lse, BT);
  cv.take(c->cand_parent, BT);
  cv.take(c->cand_gparent, BT);
  c->max_pairs = T * (CASCADE_MAX_CHILDREN + 1) / 2 + T;
  cv.take(c->scores, (int64_t)s.B * c->max_pairs);
  cv.take(c->q_relaxed, BT);
  cv.take(c->tvd_out, BT);
  if (s.ffn > 0) {
    // decoder layers: residual stream, GEMM operands, per-slice projection outputs, rotated q/k/v
    const int64_t RT = (int64_t)R * T;
    const int64_t k_max = s.h > s.ffn ? s.h : s.ffn;
    const int es = elem_size(s);
    cv.take(c->x, RT * s.h);
    if (s.dtype == CASCADE_BF16) {
      cv.take(c->act, operand_elems((int)RT, (int)align_up(k_max, 64)));
    } else {
      cv.take(c->act_f32, RT * k_max);
    }
    int64_t need = 0;
    const int shapes[4][2] = {{(s.Hq + 2 * s.Hkv) * s.D, s.h}, {s.h, s.Hq * s.D}, {2 * s.ffn, s.h}, {s.h, s.ffn}};
    for (const auto& nk : shapes) {
      int S = s.dtype == CASCADE_BF16 ? gemm_tc_pick_splits(c->sm_count, (int)RT, nk[0], nk[1], c->layer_max_splits) : 1;
      if (s.dtype == CASCADE_BF16) {  // the balanced mode of the gate/up projection may cut a tile once more
        const SliceMap map = gemm_tc_balanced_map(c, (int)RT, nk[0], nk[1]);
        if (map.balanced && map.n_slices > S && map.n_slices <= c->layer_max_splits) S = map.n_slices;
      }
      const int64_t f = (int64_t)S * RT * nk[0];
      if (f > need) need = f;
    }
    c->gemm_out_floats = need;
    cv.take(c->gemm_out, need);
    char* p = nullptr;
    cv.take(p, RT * s.Hq * s.D * es);
    c->q_rot = p;
    cv.take(p, RT * s.Hkv * s.D * es);
    c->k_rot = p;
    cv.take(p, RT * s.Hkv * s.D * es);
    c->v_rot = p;
    cv.take(p, s.dtype == CASCADE_BF16 ? operand_elems((int)RT, s.Hq * s.D) * 2 : RT * s.Hq * s.D * es);
    c->attn_out = p;
  }
  c->st_in_bytes = 3 * BT * 4;
  c->st_out_bytes = align_up(BT, 4) + (int64_t)s.B * (T + 1) * 4 + (int64_t)s.B * 4;
  cv.take(c->st_in, c->st_in_bytes);
  cv.take(c->st_out, c->st_out_bytes);
  return align_up(cv.off, 256);
}

int validate_shape(const cascade_shape* s) {
  if (s == nullptr) return CASCADE_ERR_INVALID_ARG;
  if (s->dtype != CASCADE_F32 && s->dtype != CASCADE_BF16) return CASCADE_ERR_INVALID_ARG;
  if (s->B < 1 || s->T_max < 1 || s->P_max < 0 || s->h < 1 || s->Hq < 1 || s->Hkv < 1 || s->D < 1 || s->V < 1 ||
      s->ffn < 0)
    return CASCADE_ERR_INVALID_ARG;
  if (s->T_max > CASCADE_MAX_TREE_ROWS) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  if (s->D != 64 && s->D != 128) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  if (s->Hq % s->Hkv != 0) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  if (s->h % 64 != 0 || s->V % 8 != 0 || s->ffn % 8 != 0) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  if (s->dtype == CASCADE_BF16 && s->ffn % 64 != 0) return CASCADE_ERR_UNSUPPORTED_SHAPE;  // GEMM K blocks of 64
  if ((int64_t)s->B * s->T_max > (1 << 20)) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  return CASCADE_OK;
}

cudaStream_t as_stream(void* s) { return static_cast<cudaStream_t>(s); }

}  // namespace

extern "C" {

const char* cascade_strerror(int status) {
  switch (status) {
    case CASCADE_OK: return "ok";
    case CASCADE_ERR_INVALID_ARG: return "invalid argument";
    case CASCADE_ERR_BAD_TREE: return "parent[] is not a BFS-ordered tree with contiguous sibling groups";
    case CASCADE_ERR_WORKSPACE: return "could not allocate the context's device scratch";
    case CASCADE_ERR_UNSUPPORTED_SHAPE: return "shape not supported by the kernels";
    case CASCADE_ERR_CUDA: return "a CUDA call failed";
    case CASCADE_ERR_TIMEOUT: return "a bounded device-side wait gave up";
    case CASCADE_ERR_OVERFLOW: return "a KV cache has no room for the accepted path";
    case CASCADE_ERR_BAD_PAGE: return "a page, slot or length outside what the paged call was given";
    default: return "unknown status";
  }
}

const char* cascade_kernel_name(int32_t id) {
  static const char* names[] = {"tree_attn", "tree_attn_f32", "final_norm_mix", "gemm_head",
                                "head_f32", "row_stats", "row_lse", "similarity", "accept", "tail", "select_path",
                                "embed_norm", "gemm_qkv", "rope_split", "gemm_o", "resid_norm", "gemm_gate_up",
                                "swiglu", "gemm_down", "gemm_f32", "resid_add", "kv_append", "bonus_token", "filter_logits", "wait_probe", "build_tree",
                                "paged_tables", "paged_append", "paged_attn", "sample"};
  static_assert(sizeof(names) / sizeof(names[0]) == K_KERNEL_ID_END, "one name per kernel id");
  if (id < 0 || id >= K_KERNEL_ID_END) return nullptr;
  return names[id];
}

int cascade_timing_enable(cascade_ctx* ctx, int32_t on) {
  if (ctx == nullptr) return CASCADE_ERR_INVALID_ARG;
  ctx->timing = on != 0;
  return CASCADE_OK;
}

int cascade_timing_read(cascade_ctx* ctx, float* ms_total, int32_t* launches) {
  if (ctx == nullptr || ms_total == nullptr || launches == nullptr) return CASCADE_ERR_INVALID_ARG;
  int status = CASCADE_OK;
  for (const TimedLaunch& t : ctx->timed) {
    float ms = 0.f;
    if (cudaEventSynchronize(t.stop) != cudaSuccess || cudaEventElapsedTime(&ms, t.start, t.stop) != cudaSuccess) {
      (void)cudaGetLastError();
      status = CASCADE_ERR_CUDA;
    } else {
      ms_total[t.id] += ms;
      launches[t.id] += 1;
    }
    ctx->event_pool.push_back(t.start);
    ctx->event_pool.push_back(t.stop);
  }
  ctx->timed.clear();
  return status;
}

int cascade_create(cascade_ctx** out, const cascade_shape* shape) {
  if (out == nullptr) return CASCADE_ERR_INVALID_ARG;
  CASCADE_TRY(validate_shape(shape));
  cascade_ctx* c = new (std::nothrow) cascade_ctx();
  if (c == nullptr) return CASCADE_ERR_WORKSPACE;
  c->shape = *shape;
  if (cudaGetDevice(&c->device) != cudaSuccess ||
      cudaDeviceGetAttribute(&c->sm_count, cudaDevAttrMultiProcessorCount, c->device) != cudaSuccess) {
    (void)cudaGetLastError();
    delete c;
    return CASCADE_ERR_CUDA;
  }
  c->ws_bytes = carve(c, nullptr);
  if (cudaMalloc(&c->ws, (size_t)c->ws_bytes) != cudaSuccess) {
    (void)cudaGetLastError();
    delete c;
    return CASCADE_ERR_WORKSPACE;
  }
  carve(c, c->ws);
  if (cudaMemset(c->ws, 0, (size_t)c->ws_bytes) != cudaSuccess ||
      cudaMallocHost(&c->host_error, 64) != cudaSuccess ||
      cudaMallocHost(&c->host_stage, (size_t)(c->st_in_bytes + c->st_out_bytes)) != cudaSuccess) {
    (void)cudaGetLastError();
    cudaFree(c->ws);
    if (c->host_error != nullptr) cudaFreeHost(c->host_error);
    delete c;
    return CASCADE_ERR_CUDA;
  }
  *c->host_error = 0;
  *out = c;
  return CASCADE_OK;
}

int cascade_destroy(cascade_ctx* ctx) {
  if (ctx == nullptr) return CASCADE_ERR_INVALID_ARG;
  for (const TimedLaunch& t : ctx->timed) {
    cudaEventDestroy(t.start);
    cudaEventDestroy(t.stop);
  }
  for (cudaEvent_t e : ctx->event_pool) cudaEventDestroy(e);
  cudaFree(ctx->ws);
  cudaFreeHost(ctx->host_error);
  cudaFreeHost(ctx->host_stage);
  for (auto& g : ctx->host_graphs)
    if (g.exec != nullptr) cudaGraphExecDestroy(g.exec);
  free_tmap_cache(ctx);
  delete ctx;
  return CASCADE_OK;
}

int64_t cascade_workspace_bytes(const cascade_ctx* ctx) { return ctx ? ctx->ws_bytes : 0; }

int cascade_last_launch_count(const cascade_ctx* ctx) { return ctx ? ctx->launches : 0; }

int cascade_set_wait_limit(cascade_ctx* ctx, int64_t limit_ns) {
  if (ctx == nullptr || limit_ns < 1000) return CASCADE_ERR_INVALID_ARG;
  ctx->wait_limit_ns = (unsigned long long)limit_ns;
  return CASCADE_OK;
}

int cascade_check(cascade_ctx* ctx, void* stream) {
  if (ctx == nullptr) return CASCADE_ERR_INVALID_ARG;
  cudaStream_t s = as_stream(stream);
  CASCADE_CUDA_TRY(cudaMemcpyAsync(ctx->host_error, ctx->dev_error, sizeof(int), cudaMemcpyDeviceToHost, s));
  CASCADE_CUDA_TRY(cudaStreamSynchronize(s));
  const int word = *ctx->host_error;
  if (word != 0) {
    CASCADE_CUDA_TRY(cudaMemsetAsync(ctx->dev_error, 0, sizeof(int), s));
    CASCADE_CUDA_TRY(cudaStreamSynchronize(s));
    if (word & CASCADE_DEV_ERR_WAIT) return CASCADE_ERR_TIMEOUT;
    if (word & CASCADE_DEV_ERR_BAD_TREE) return CASCADE_ERR_BAD_TREE;
    return (word & CASCADE_DEV_ERR_BAD_PAGE) ? CASCADE_ERR_BAD_PAGE : CASCADE_ERR_OVERFLOW;
  }
  return CASCADE_OK;
}

// ---- tree ---------------------------------------------------------------------------------------------

// Everything the descriptor holds, built on the host from parent[]; nothing is touched on failure.
namespace {
struct HostTree {
  int T = 0, depth_max = 0, n_pairs = 0;
  std::vector<int32_t> parent, depth, child_begin, child_count, pair_a, pair_b, sib_base;
  std::vector<uint64_t> anc;
};

int build_host_tree(const cascade_ctx* ctx, int32_t T, const int32_t* parent, HostTree* h) {
  if (T > ctx->shape.T_max) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  if (parent[0] != -1) return CASCADE_ERR_BAD_TREE;
  h->T = T;
  h->parent.assign(parent, parent + T);
  h->depth.assign(T, 0);
  h->child_begin.assign(T, 0);
  h->child_count.assign(T, 0);
  h->sib_base.assign(T, 0);
  for (int j = 1; j < T; ++j) {
    const int p = parent[j];
    if (p < 0 || p >= j) return CASCADE_ERR_BAD_TREE;
    h->depth[j] = h->depth[p] + 1;
    if (h->depth[j] < h->depth[j - 1]) return CASCADE_ERR_BAD_TREE;   // BFS order
    if (j > 1 && p < parent[j - 1]) return CASCADE_ERR_BAD_TREE;      // groups contiguous
    if (h->child_count[p] == 0) h->child_begin[p] = j;
    h->child_count[p]++;
    if (h->child_count[p] > CASCADE_MAX_CHILDREN) return CASCADE_ERR_UNSUPPORTED_SHAPE;
    h->depth_max = h->depth[j];
  }
  // pair list: edge (parent[j], j) at index j-1, then the sibling pairs of each parent in order
  for (int j = 1; j < T; ++j) {
    h->pair_a.push_back(parent[j]);
    h->pair_b.push_back(j);
  }
  for (int p = 0; p < T; ++p) {
    h->sib_base[p] = (int)h->pair_a.size();
    const int cb = h->child_begin[p], k = h->child_count[p];
    for (int x = 0; x < k; ++x)
      for (int y = x + 1; y < k; ++y) {
        h->pair_a.push_back(cb + x);
        h->pair_b.push_back(cb + y);
      }
  }
  h->n_pairs = (int)h->pair_a.size();
  if (h->n_pairs > ctx->max_pairs) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  h->anc.assign((size_t)T * 4, 0);
  for (int j = 0; j < T; ++j)
    for (int i = j; i >= 0; i = parent[i]) h->anc[(size_t)j * 4 + (i >> 6)] |= 1ull << (i & 63);
  return CASCADE_OK;
}

// Copies a host descriptor into the tree's device arrays (sized for the context's limits) and takes it over.
int install_host_tree(cascade_tree* t, HostTree&& h, cudaStream_t s, bool async) {
  bool ok = true;
  auto up = [&](void* dst, const void* src, size_t n) {
    if (n == 0) return;
    const cudaError_t e = async ? cudaMemcpyAsync(dst, src, n, cudaMemcpyHostToDevice, s)
                                : cudaMemcpy(dst, src, n, cudaMemcpyHostToDevice);
    if (e != cudaSuccess) ok = false;
  };
  const int T = h.T;
  up(t->d_parent, h.parent.data(), sizeof(int32_t) * T);
  up(t->d_depth, h.depth.data(), sizeof(int32_t) * T);
  up(t->d_child_begin, h.child_begin.data(), sizeof(int32_t) * T);
  up(t->d_child_count, h.child_count.data(), sizeof(int32_t) * T);
  up(t->d_sib_base, h.sib_base.data(), sizeof(int32_t) * T);
  up(t->d_pair_a, h.pair_a.data(), sizeof(int32_t) * h.n_pairs);
  up(t->d_pair_b, h.pair_b.data(), sizeof(int32_t) * h.n_pairs);
  up(t->d_anc, h.anc.data(), sizeof(uint64_t) * h.anc.size());
  if (!ok) {
    (void)cudaGetLastError();
    return CASCADE_ERR_CUDA;
  }
  t->T = h.T;
  t->depth_max = h.depth_max;
  t->n_pairs = h.n_pairs;
  t->uid = next_tree_uid();
  t->device_built = false;
  t->parent = std::move(h.parent);
  t->depth = std::move(h.depth);
  t->child_begin = std::move(h.child_begin);
  t->child_count = std::move(h.child_count);
  t->pair_a = std::move(h.pair_a);
  t->pair_b = std::move(h.pair_b);
  t->sib_base = std::move(h.sib_base);
  return CASCADE_OK;
}
}  // namespace

int cascade_tree_create(cascade_ctx* ctx, int32_t T, const int32_t* parent, cascade_tree** out) {
  if (ctx == nullptr || parent == nullptr || out == nullptr || T < 1) return CASCADE_ERR_INVALID_ARG;
  HostTree h;
  CASCADE_TRY(build_host_tree(ctx, T, parent, &h));
  cascade_tree* t = new (std::nothrow) cascade_tree();
  if (t == nullptr) return CASCADE_ERR_WORKSPACE;
  t->ctx = ctx;
  // device arrays sized for the context's limits, so that cascade_tree_update never allocates
  const int64_t T_cap = ctx->shape.T_max, pairs_cap = ctx->max_pairs > 0 ? ctx->max_pairs : 1;
  Carver cv;
  auto layout = [&](char* base) {
    cv = Carver();
    cv.base = base;
    cv.take(t->d_parent, T_cap);
    cv.take(t->d_depth, T_cap);
    cv.take(t->d_child_begin, T_cap);
    cv.take(t->d_child_count, T_cap);
    cv.take(t->d_sib_base, T_cap);
    cv.take(t->d_pair_a, pairs_cap);
    cv.take(t->d_pair_b, pairs_cap);
    cv.take(t->d_anc, T_cap * 4);
    cv.take(t->d_meta, 4);
    return align_up(cv.off, 256);
  };
  const int64_t bytes = layout(nullptr);
  if (cudaMalloc(&t->dev, (size_t)bytes) != cudaSuccess) {
    (void)cudaGetLastError();
    delete t;
    return CASCADE_ERR_WORKSPACE;
  }
  layout(t->dev);
  const int rc = install_host_tree(t, std::move(h), nullptr, false);
  if (rc != CASCADE_OK) {
    cudaFree(t->dev);
    delete t;
    return rc;
  }
  *out = t;
  return CASCADE_OK;
}

int cascade_tree_update(cascade_tree* tree, int32_t T, const int32_t* parent, void* stream) {
  if (tree == nullptr || parent == nullptr || T < 1) return CASCADE_ERR_INVALID_ARG;
  HostTree h;
  CASCADE_TRY(build_host_tree(tree->ctx, T, parent, &h));  // an invalid tree leaves the old one in place
  return install_host_tree(tree, std::move(h), as_stream(stream), true);
}

int cascade_tree_update_device(cascade_tree* tree, int32_t T, int32_t depth_cap, int32_t pairs_cap,
                               const int32_t* parent_dev, void* stream) {
  if (tree == nullptr || parent_dev == nullptr || T < 1 || depth_cap < 0) return CASCADE_ERR_INVALID_ARG;
  cascade_ctx* ctx = tree->ctx;
  if (T > ctx->shape.T_max) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  if (T > 1 && depth_cap < 1) return CASCADE_ERR_INVALID_ARG;
  if (depth_cap > T - 1) depth_cap = T - 1;
  if (pairs_cap <= 0 || pairs_cap > ctx->max_pairs) pairs_cap = ctx->max_pairs;
  ctx->launches = 0;
  CASCADE_TRY(launch_build_tree(ctx, tree, T, depth_cap, pairs_cap, parent_dev, as_stream(stream)));
  tree->T = T;
  tree->depth_max = depth_cap;
  tree->n_pairs = pairs_cap;
  tree->device_built = true;
  tree->uid = next_tree_uid();
  return CASCADE_OK;
}

int cascade_tree_destroy(cascade_tree* tree) {
  if (tree == nullptr) return CASCADE_ERR_INVALID_ARG;
  // steps recorded by the host-buffer entry point into this descriptor's device arrays
  if (tree->ctx != nullptr) {
    auto& graphs = tree->ctx->host_graphs;
    for (size_t i = graphs.size(); i-- > 0;)
      if (graphs[i].tree == tree) {
        if (graphs[i].exec != nullptr) cudaGraphExecDestroy(graphs[i].exec);
        graphs.erase(graphs.begin() + (long)i);
      }
  }
  cudaFree(tree->dev);
  delete tree;
  return CASCADE_OK;
}

int cascade_tree_download(const cascade_tree* tree, int32_t* parent, int32_t* depth, int32_t* child_begin,
                          int32_t* child_count, uint64_t* anc) {
  if (tree == nullptr) return CASCADE_ERR_INVALID_ARG;
  const size_t n = sizeof(int32_t) * (size_t)tree->T;
  if (parent != nullptr) CASCADE_CUDA_TRY(cudaMemcpy(parent, tree->d_parent, n, cudaMemcpyDeviceToHost));
  if (depth != nullptr) CASCADE_CUDA_TRY(cudaMemcpy(depth, tree->d_depth, n, cudaMemcpyDeviceToHost));
  if (child_begin != nullptr) CASCADE_CUDA_TRY(cudaMemcpy(child_begin, tree->d_child_begin, n, cudaMemcpyDeviceToHost));
  if (child_count != nullptr) CASCADE_CUDA_TRY(cudaMemcpy(child_count, tree->d_child_count, n, cudaMemcpyDeviceToHost));
  if (anc != nullptr)
    CASCADE_CUDA_TRY(cudaMemcpy(anc, tree->d_anc, sizeof(uint64_t) * 4 * (size_t)tree->T, cudaMemcpyDeviceToHost));
  return CASCADE_OK;
}

int32_t cascade_tree_rows(const cascade_tree* tree) { return tree ? tree->T : 0; }
int32_t cascade_tree_depth(const cascade_tree* tree) { return tree ? tree->depth_max : 0; }
int32_t cascade_tree_num_pairs(const cascade_tree* tree) { return tree ? tree->n_pairs : 0; }
int cascade_tree_pairs(const cascade_tree* tree, int32_t* pair_a, int32_t* pair_b) {
  if (tree == nullptr || pair_a == nullptr || pair_b == nullptr) return CASCADE_ERR_INVALID_ARG;
  if (tree->device_built) {
    // the list lives on the device only: fetched with blocking copies (the caller has synchronised the stream
    // of the update); entries beyond the tree's pair count are -1
    int32_t meta[4] = {0, 0, 0, 0};
    CASCADE_CUDA_TRY(cudaMemcpy(meta, tree->d_meta, sizeof(meta), cudaMemcpyDeviceToHost));
    const int n = meta[0] < tree->n_pairs ? meta[0] : tree->n_pairs;
    CASCADE_CUDA_TRY(cudaMemcpy(pair_a, tree->d_pair_a, sizeof(int32_t) * n, cudaMemcpyDeviceToHost));
    CASCADE_CUDA_TRY(cudaMemcpy(pair_b, tree->d_pair_b, sizeof(int32_t) * n, cudaMemcpyDeviceToHost));
    for (int i = n; i < tree->n_pairs; ++i) pair_a[i] = pair_b[i] = -1;
    return CASCADE_OK;
  }
  std::memcpy(pair_a, tree->pair_a.data(), sizeof(int32_t) * tree->n_pairs);
  std::memcpy(pair_b, tree->pair_b.data(), sizeof(int32_t) * tree->n_pairs);
  return CASCADE_OK;
}

// ---- (a) ------------------------------------------------------------------------------------------------

static int tree_attn_impl(cascade_ctx* ctx, const cascade_tree* tree, const void* q, const void* k_prefix,
                          const void* v_prefix, int32_t prefix_cap, const int32_t* prefix_len,
                          const void* k_tree, const void* v_tree, void* out, float softmax_scale,
                          cudaStream_t s) {
  if (ctx == nullptr || tree == nullptr || q == nullptr || prefix_len == nullptr || k_tree == nullptr ||
      v_tree == nullptr || out == nullptr)
    return CASCADE_ERR_INVALID_ARG;
  if (tree->ctx != ctx) return CASCADE_ERR_INVALID_ARG;
  if (prefix_cap < 0 || prefix_cap > ctx->shape.P_max) return CASCADE_ERR_INVALID_ARG;
  if (prefix_cap > 0 && (k_prefix == nullptr || v_prefix == nullptr)) return CASCADE_ERR_INVALID_ARG;
  if (!(softmax_scale > 0.f)) return CASCADE_ERR_INVALID_ARG;
  if (!aligned16(q) || !aligned16(k_prefix) || !aligned16(v_prefix) || !aligned16(k_tree) || !aligned16(v_tree) ||
      !aligned16(out))
    return CASCADE_ERR_INVALID_ARG;
  if (ctx->shape.dtype == CASCADE_BF16)
    return launch_tree_attn_bf16(ctx, tree, (const __nv_bfloat16*)q, (const __nv_bfloat16*)k_prefix,
                                 (const __nv_bfloat16*)v_prefix, prefix_cap, prefix_len,
                                 (const __nv_bfloat16*)k_tree, (const __nv_bfloat16*)v_tree, (__nv_bfloat16*)out,
                                 false, softmax_scale, s);
  return launch_tree_attn_f32(ctx, tree, (const float*)q, (const float*)k_prefix, (const float*)v_prefix,
                              prefix_cap, prefix_len, (const float*)k_tree, (const float*)v_tree, (float*)out,
                              softmax_scale, s);
}

int cascade_tree_attn(cascade_ctx* ctx, const cascade_tree* tree, const void* q, const void* k_prefix,
                      const void* v_prefix, int32_t prefix_cap, const int32_t* prefix_len,
                      const void* k_tree, const void* v_tree, void* out, float softmax_scale, void* stream) {
  if (ctx != nullptr) ctx->launches = 0;
  return tree_attn_impl(ctx, tree, q, k_prefix, v_prefix, prefix_cap, prefix_len, k_tree, v_tree, out,
                        softmax_scale, as_stream(stream));
}

// ---- (b) ------------------------------------------------------------------------------------------------

// fold_lse: also fold the head's per-tile partials into row_lse_out here (stand-alone call); the fused
// step leaves that to its tail kernel.
static int lm_head_impl(cascade_ctx* ctx, const cascade_tree* tree, const void* hidden, const float* rms_gamma,
                        float eps, const void* w_head, float cfg_scale, float temperature, const int32_t* tok,
                        float* logits_out, float* feat_out, float* feat_norm_out, float* row_lse_out,
                        float* cand_parent_out, float* cand_gparent_out, bool fold_lse, bool hidden_f32,
                        const PendingAdd& add, cudaStream_t s) {
  if (ctx == nullptr || tree == nullptr || hidden == nullptr || rms_gamma == nullptr || w_head == nullptr)
    return CASCADE_ERR_INVALID_ARG;
  if (tree->ctx != ctx) return CASCADE_ERR_INVALID_ARG;
  if (!(temperature > 0.f) || !(eps >= 0.f)) return CASCADE_ERR_INVALID_ARG;
  if (tok != nullptr && (cand_parent_out == nullptr || cand_gparent_out == nullptr)) return CASCADE_ERR_INVALID_ARG;
  if (!aligned16(hidden) || !aligned16(w_head) || !aligned16(logits_out) || !aligned16(feat_out) ||
      !aligned16(rms_gamma))
    return CASCADE_ERR_INVALID_ARG;
  if (row_lse_out == nullptr) row_lse_out = ctx->row_lse;
  CASCADE_TRY(launch_final_norm_mix(ctx, tree->T, hidden, hidden_f32, add, rms_gamma, eps, cfg_scale, 1.f / temperature, feat_out,
                                    feat_norm_out, tok ? cand_parent_out : nullptr, tok ? cand_gparent_out : nullptr,
                                    s));
  if (ctx->shape.dtype == CASCADE_BF16) {
    CASCADE_TRY(launch_head_bf16(ctx, tree, (const __nv_bfloat16*)w_head, tok, logits_out, cand_parent_out,
                                 cand_gparent_out, s));
    if (!fold_lse) return CASCADE_OK;
    TailWork w;
    w.kernel_id = K_ROW_LSE;
    w.part = ctx->head_part;
    w.part_ld = ctx->head_max_tiles;
    w.n_tiles = ceil_div(ctx->shape.V, 128);
    w.row_lse = row_lse_out;
    return launch_tail(ctx, tree, w, s);
  }
  if (logits_out == nullptr) return CASCADE_ERR_INVALID_ARG;  // the fp32 path always materialises logits
  return launch_head_f32(ctx, tree, (const float*)w_head, tok, logits_out, row_lse_out, cand_parent_out,
                         cand_gparent_out, s);
}

int cascade_lm_head_cfg(cascade_ctx* ctx, const cascade_tree* tree, const void* hidden, const float* rms_gamma,
                        float eps, const void* w_head, float cfg_scale, float temperature, const int32_t* tok,
                        float* logits_out, float* feat_out, float* feat_norm_out, float* row_lse_out,
                        float* cand_parent_out, float* cand_gparent_out, void* stream) {
  if (ctx != nullptr) ctx->launches = 0;
  return lm_head_impl(ctx, tree, hidden, rms_gamma, eps, w_head, cfg_scale, temperature, tok, logits_out, feat_out,
                      feat_norm_out, row_lse_out, cand_parent_out, cand_gparent_out, true, false, PendingAdd{},
                      as_stream(stream));
}

// ---- (c) ------------------------------------------------------------------------------------------------

int cascade_similarity(cascade_ctx* ctx, const cascade_tree* tree, const float* feat, int32_t feat_dim,
                       const float* feat_norm, float* scores_out, void* stream) {
  if (ctx == nullptr || tree == nullptr || feat == nullptr || (scores_out == nullptr && tree->n_pairs > 0))
    return CASCADE_ERR_INVALID_ARG;
  if (tree->ctx != ctx || feat_dim < 4 || feat_dim % 4 != 0 || !aligned16(feat)) return CASCADE_ERR_INVALID_ARG;
  ctx->launches = 0;
  TailWork w;
  w.kernel_id = K_SIMILARITY;
  w.feat = feat;
  w.feat_dim = feat_dim;
  w.feat_norm = feat_norm;
  w.scores = scores_out;
  return launch_tail(ctx, tree, w, as_stream(stream));
}

static int validate_params(const cascade_params* p) {
  if (p == nullptr) return CASCADE_ERR_INVALID_ARG;
  if (!(p->tvd_budget >= 0.f)) return CASCADE_ERR_INVALID_ARG;  // also rejects NaN
  if (p->tau_pos != p->tau_pos || p->tau_seq != p->tau_seq) return CASCADE_ERR_INVALID_ARG;
  if (p->flags & ~(CASCADE_USE_I | CASCADE_USE_C | CASCADE_CONV_DIST_SELF)) return CASCADE_ERR_INVALID_ARG;
  return CASCADE_OK;
}

int cascade_relaxed_accept(cascade_ctx* ctx, const cascade_tree* tree, const float* scores, const float* logits,
                           const float* row_lse, const float* cand_parent, const float* cand_gparent,
                           const int32_t* tok, const float* draft_p, const float* uniforms,
                           const cascade_params* params, uint8_t* accept, float* q_relaxed, float* tvd_out,
                           int32_t* near_count, void* stream) {
  if (ctx == nullptr || tree == nullptr || tok == nullptr || draft_p == nullptr || uniforms == nullptr ||
      accept == nullptr)
    return CASCADE_ERR_INVALID_ARG;
  if (tree->ctx != ctx) return CASCADE_ERR_INVALID_ARG;
  if (scores == nullptr && tree->n_pairs > 0) return CASCADE_ERR_INVALID_ARG;
  CASCADE_TRY(validate_params(params));
  if (logits == nullptr && (row_lse == nullptr || cand_parent == nullptr || cand_gparent == nullptr))
    return CASCADE_ERR_INVALID_ARG;
  ctx->launches = 0;
  cudaStream_t s = as_stream(stream);
  if (logits != nullptr) {
    CASCADE_TRY(launch_row_stats_from_logits(ctx, tree, logits, tok, ctx->row_lse, ctx->cand_parent,
                                             ctx->cand_gparent, s));
    row_lse = ctx->row_lse;
    cand_parent = ctx->cand_parent;
    cand_gparent = ctx->cand_gparent;
  }
  TailWork w;
  w.kernel_id = K_ACCEPT;
  w.scores = const_cast<float*>(scores);
  w.row_lse = const_cast<float*>(row_lse);
  w.prm = params;
  w.cand_parent = cand_parent;
  w.cand_gparent = cand_gparent;
  w.tok = tok;
  w.draft_p = draft_p;
  w.uniforms = uniforms;
  w.accept = accept;
  w.q_relaxed = q_relaxed;
  w.tvd_out = tvd_out;
  w.near_count = near_count;
  return launch_tail(ctx, tree, w, s);
}

// ---- (d) ------------------------------------------------------------------------------------------------

int cascade_select_path(cascade_ctx* ctx, const cascade_tree* tree, const uint8_t* accept, const float* tvd_out,
                        int32_t mode, int32_t* path_nodes, int32_t* path_len, float* tvd_used, void* stream) {
  if (ctx == nullptr || tree == nullptr || accept == nullptr || path_nodes == nullptr || path_len == nullptr)
    return CASCADE_ERR_INVALID_ARG;
  if (tree->ctx != ctx) return CASCADE_ERR_INVALID_ARG;
  if (mode != CASCADE_SELECT_LONGEST && mode != CASCADE_SELECT_FIRST_ACCEPT) return CASCADE_ERR_INVALID_ARG;
  ctx->launches = 0;
  return launch_select_path(ctx, tree, accept, tvd_out, mode, path_nodes, path_len, tvd_used, as_stream(stream));
}

// ---- the whole step -----------------------------------------------------------------------------------------

static int verify_step_impl(cascade_ctx* ctx, const cascade_tree* tree, const cascade_step* st, cudaStream_t s) {
  if (ctx == nullptr || tree == nullptr || st == nullptr) return CASCADE_ERR_INVALID_ARG;
  if (tree->ctx != ctx) return CASCADE_ERR_INVALID_ARG;
  if (st->tok == nullptr || st->draft_p == nullptr || st->uniforms == nullptr || st->accept == nullptr ||
      st->path_nodes == nullptr || st->path_len == nullptr || st->gamma_final == nullptr || st->w_head == nullptr)
    return CASCADE_ERR_INVALID_ARG;
  CASCADE_TRY(validate_params(&st->params));
  if (st->select_mode != CASCADE_SELECT_LONGEST && st->select_mode != CASCADE_SELECT_FIRST_ACCEPT)
    return CASCADE_ERR_INVALID_ARG;
  if (st->n_layers < 0) return CASCADE_ERR_INVALID_ARG;
  if (st->n_layers == 0 && st->hidden_in == nullptr) return CASCADE_ERR_INVALID_ARG;
  const bool nucleus = st->top_p > 0.f && st->top_p < 1.f;
  const bool truncate = (st->top_k > 0 && st->top_k < ctx->shape.V) || nucleus;
  if (st->top_k < 0 || st->top_p < 0.f || st->top_p > 1.f || st->top_p != st->top_p) return CASCADE_ERR_INVALID_ARG;
  if (truncate && st->logits == nullptr) return CASCADE_ERR_INVALID_ARG;  // the truncation works on stored logits
  ctx->launches = 0;
  const void* hidden = st->hidden_in;
  PendingAdd pending;
  if (st->n_layers > 0) {
    CASCADE_TRY(run_layers(ctx, tree, st, &pending, s));
    hidden = ctx->x;
  } else if (st->q != nullptr) {
    CASCADE_TRY(tree_attn_impl(ctx, tree, st->q, st->k_prefix, st->v_prefix, st->prefix_cap, st->prefix_len,
                               st->k_tree, st->v_tree, st->attn_out, st->softmax_scale, s));
  }
  float* feat = st->feat ? st->feat : ctx->feat;
  float* row_lse = st->row_lse ? st->row_lse : ctx->row_lse;
  const bool bf16 = ctx->shape.dtype == CASCADE_BF16;
  CASCADE_TRY(lm_head_impl(ctx, tree, hidden, st->gamma_final, st->eps, st->w_head, st->cfg_scale, st->temperature,
                           st->tok, st->logits, feat, ctx->feat_norm, row_lse, ctx->cand_parent, ctx->cand_gparent, false,
                           st->n_layers > 0, pending, s));
  // cosines, row log-sum-exp (bf16: folded from the head's partials), the rule and the path: one launch
  if (truncate) {
    // truncate the stored logits, then take every row's log-sum-exp and candidate logits from what is left
    CASCADE_TRY(launch_filter_logits(ctx, st->logits, ctx->shape.B * tree->T, st->top_k, nucleus ? st->top_p : 1.f,
                                     nullptr, s));
    CASCADE_TRY(launch_row_stats_from_logits(ctx, tree, st->logits, st->tok, row_lse, ctx->cand_parent,
                                             ctx->cand_gparent, s));
  }
  TailWork w;
  w.feat = feat;
  w.feat_dim = ctx->shape.h;
  w.feat_norm = ctx->feat_norm;
  w.scores = st->scores ? st->scores : ctx->scores;
  if (bf16 && !truncate) {
    w.part = ctx->head_part;
    w.part_ld = ctx->head_max_tiles;
    w.n_tiles = ceil_div(ctx->shape.V, 128);
  }
  w.row_lse = row_lse;
  w.prm = &st->params;
  w.cand_parent = ctx->cand_parent;
  w.cand_gparent = ctx->cand_gparent;
  w.tok = st->tok;
  w.draft_p = st->draft_p;
  w.uniforms = st->uniforms;
  w.accept = st->accept;
  w.q_relaxed = st->q_relaxed ? st->q_relaxed : ctx->q_relaxed;
  w.tvd_out = st->tvd_out ? st->tvd_out : ctx->tvd_out;
  w.near_count = st->near_count;
  w.select_mode = st->select_mode;
  w.path_nodes = st->path_nodes;
  w.path_len = st->path_len;
  w.tvd_used = st->tvd_used;
  return launch_tail(ctx, tree, w, s);
}

int cascade_verify_step(cascade_ctx* ctx, const cascade_tree* tree, const cascade_step* step, void* stream) {
  return verify_step_impl(ctx, tree, step, as_stream(stream));
}

int cascade_verify_step_host(cascade_ctx* ctx, const cascade_tree* tree, const cascade_step* step,
                             const int32_t* tok_host, const float* draft_p_host, const float* uniforms_host,
                             uint8_t* accept_host, int32_t* path_nodes_host, int32_t* path_len_host,
                             void* stream) {
  if (ctx == nullptr || tree == nullptr || step == nullptr || tok_host == nullptr || draft_p_host == nullptr ||
      uniforms_host == nullptr || accept_host == nullptr || path_nodes_host == nullptr || path_len_host == nullptr)
    return CASCADE_ERR_INVALID_ARG;
  if (tree->ctx != ctx) return CASCADE_ERR_INVALID_ARG;  // also bounds T by the context's T_max (the pinned block's size)
  cudaStream_t s = as_stream(stream);
  const size_t BT = (size_t)ctx->shape.B * tree->T;
  // The three inputs are a few hundred bytes each: they are gathered into one pinned block and go to the device
  // with one copy, the three results come back the same way (every small copy costs microseconds on the stream).
  const size_t in_bytes = 3 * BT * 4;
  const size_t nodes_bytes = (size_t)ctx->shape.B * (tree->depth_max + 1) * 4, len_bytes = (size_t)ctx->shape.B * 4;
  const size_t acc_pad = (BT + 3) / 4 * 4, out_bytes = acc_pad + nodes_bytes + len_bytes;
  char* h_in = ctx->host_stage;
  char* h_out = ctx->host_stage + ctx->st_in_bytes;
  std::memcpy(h_in, tok_host, BT * 4);
  std::memcpy(h_in + BT * 4, draft_p_host, BT * 4);
  std::memcpy(h_in + 2 * BT * 4, uniforms_host, BT * 4);
  cascade_step st = *step;
  st.tok = reinterpret_cast<const int32_t*>(ctx->st_in);
  st.draft_p = reinterpret_cast<const float*>(ctx->st_in + BT * 4);
  st.uniforms = reinterpret_cast<const float*>(ctx->st_in + 2 * BT * 4);
  st.accept = reinterpret_cast<uint8_t*>(ctx->st_out);
  st.path_nodes = reinterpret_cast<int32_t*>(ctx->st_out + acc_pad);
  st.path_len = reinterpret_cast<int32_t*>(ctx->st_out + acc_pad + nodes_bytes);
  // everything the enqueued work depends on: the same bytes mean the same copies and launches
  auto enqueue = [&]() -> int {
    CASCADE_CUDA_TRY(cudaMemcpyAsync(ctx->st_in, h_in, in_bytes, cudaMemcpyHostToDevice, s));
    CASCADE_TRY(verify_step_impl(ctx, tree, &st, s));
    CASCADE_CUDA_TRY(cudaMemcpyAsync(h_out, ctx->st_out, out_bytes, cudaMemcpyDeviceToHost, s));
    return CASCADE_OK;
  };
  // A caller in a decode loop repeats the same call (same step structure, same tree, same stream) with new
  // inputs in the same host block: from the second such call on, the copies and the dozen launches are
  // recorded once as a CUDA graph and replayed with one launch.  Anything that does not record (the
  // legacy stream, a caller that is itself recording, per-kernel timing) runs as before.
  std::vector<unsigned char> key;
  {
    auto put = [&](const void* p, size_t n) {
      const unsigned char* b = static_cast<const unsigned char*>(p);
      key.insert(key.end(), b, b + n);
    };
    const void* tp = tree;
    put(&tp, sizeof(tp));
    put(&tree->uid, sizeof(tree->uid));
    put(&s, sizeof(s));
    unsigned long long stream_id = 0;  // a new stream that got a destroyed stream's handle has a new id
    if (s != nullptr && cudaStreamGetId(s, &stream_id) != cudaSuccess) (void)cudaGetLastError();
    put(&stream_id, sizeof(stream_id));
    put(&st, sizeof(st));
    if (st.n_layers > 0 && st.layers != nullptr) put(st.layers, sizeof(cascade_layer) * (size_t)st.n_layers);
  }
  cudaStreamCaptureStatus capturing = cudaStreamCaptureStatusNone;
  const bool may_record = s != nullptr && !ctx->timing &&
                          cudaStreamIsCapturing(s, &capturing) == cudaSuccess && capturing == cudaStreamCaptureStatusNone;
  if (!may_record) (void)cudaGetLastError();
  constexpr size_t kHostGraphs = 4;
  cascade_ctx::HostGraph* hg = nullptr;
  for (auto& g : ctx->host_graphs)
    if (g.key == key) hg = &g;
  if (hg == nullptr) {
    if (ctx->host_graphs.size() < kHostGraphs) {
      ctx->host_graphs.emplace_back();
      hg = &ctx->host_graphs.back();
    } else {  // replace the entry that has not been used for longest
      hg = &ctx->host_graphs[0];
      for (auto& g : ctx->host_graphs)
        if (g.last_use < hg->last_use) hg = &g;
      if (hg->exec != nullptr) cudaGraphExecDestroy(hg->exec);
      *hg = cascade_ctx::HostGraph();
    }
    hg->key = key;
    hg->tree = tree;
    hg->last_use = ++ctx->host_graph_clock;
    CASCADE_TRY(enqueue());  // first sight of this call: run it directly
  } else if (may_record && hg->state == 1) {
    hg->last_use = ++ctx->host_graph_clock;
    ctx->launches = hg->launches;
    CASCADE_CUDA_TRY(cudaGraphLaunch(hg->exec, s));
  } else if (may_record && hg->state == 0) {
    hg->last_use = ++ctx->host_graph_clock;
    cudaGraph_t graph = nullptr;
    int rc = CASCADE_ERR_CUDA;
    if (cudaStreamBeginCapture(s, cudaStreamCaptureModeThreadLocal) == cudaSuccess) {
      rc = enqueue();
      if (cudaStreamEndCapture(s, &graph) != cudaSuccess) rc = CASCADE_ERR_CUDA;
    }
    if (rc == CASCADE_OK && graph != nullptr && cudaGraphInstantiate(&hg->exec, graph, 0) == cudaSuccess) {
      hg->state = 1;
      hg->launches = ctx->launches;
    } else {
      (void)cudaGetLastError();
      hg->exec = nullptr;
      hg->state = -1;
    }
    if (graph != nullptr) cudaGraphDestroy(graph);
    if (hg->state == 1) {
      CASCADE_CUDA_TRY(cudaGraphLaunch(hg->exec, s));
    } else {
      CASCADE_TRY(enqueue());
    }
  } else {
    CASCADE_TRY(enqueue());
  }
  CASCADE_CUDA_TRY(cudaStreamSynchronize(s));
  std::memcpy(accept_host, h_out, BT);
  std::memcpy(path_nodes_host, h_out + acc_pad, nodes_bytes);
  std::memcpy(path_len_host, h_out + acc_pad + nodes_bytes, len_bytes);
  return CASCADE_OK;
}

}  // extern "C"
