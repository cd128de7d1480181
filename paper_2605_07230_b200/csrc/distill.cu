// The drafter's training loss (Section 4.3, Eq. 4) against the target's largest logits alone, and its gradient.
//
// With t_i, id_i the stored logits and tokens of a position, d the drafter's row, T the temperature and w the position's weight:
//     q_i = exp(t_i / T) / sum_j exp(t_j / T)      (or exp(t_i / T - target_lse): the target's mass outside is left out)
//     loss = - w sum_i q_i log softmax(d / T)[id_i] = w (Q log Z + sum_i q_i (m - d_id) / T)
//     grad = (w / T) (Q softmax(d / T) - sum_i q_i e_id)
// with m the row's maximum, Z = sum_v exp((d_v - m) / T), Q = sum_i q_i.  Every term of the loss is positive, so nothing cancels.
#include "cascade_internal.h"
#include "ptx_paged.cuh"

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kMaxSplits = 8;       // CTAs of one row (a cluster)

// Rows are walked in pieces of 16 bytes from the 16-byte boundary at or in front of their first element: element v of the row
// is place v + lead.  A piece that is not wholly inside is read and written element by element.
template <typename E>
struct Row {
  static constexpr int kVec = 16 / (int)sizeof(E);
  int lead, V;
  __device__ __forceinline__ Row(const E* row, int v) : lead((int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(E))), V(v) {}
  __device__ __forceinline__ int pieces() const { return (V + lead + kVec - 1) / kVec; }
  __device__ __forceinline__ bool whole(int piece) const { return piece * kVec >= lead && (piece + 1) * kVec <= V + lead; }
};

__device__ __forceinline__ void unpack(const uint4& r, float (&x)[4]) {
  x[0] = __uint_as_float(r.x);
  x[1] = __uint_as_float(r.y);
  x[2] = __uint_as_float(r.z);
  x[3] = __uint_as_float(r.w);
}
__device__ __forceinline__ void unpack(const uint4& r, float (&x)[8]) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ uint4 pack(const float (&x)[4]) {
  return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}
__device__ __forceinline__ uint4 pack(const float (&x)[8]) {
  return make_uint4(ptx::pack_bf16x2(x[0], x[1]), ptx::pack_bf16x2(x[2], x[3]), ptx::pack_bf16x2(x[4], x[5]), ptx::pack_bf16x2(x[6], x[7]));
}
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ void from_float(float* p, float x) { *p = x; }
__device__ __forceinline__ void from_float(__nv_bfloat16* p, float x) { *p = __float2bfloat16(x); }

// One piece; places outside the row get `fill`.
template <typename E>
__device__ __forceinline__ void load_piece(const E* row, const Row<E>& r, int piece, float fill, float (&x)[Row<E>::kVec]) {
  const int v0 = piece * Row<E>::kVec - r.lead;
  if (r.whole(piece)) {
    unpack(*reinterpret_cast<const uint4*>(row + v0), x);
  } else {
#pragma unroll
    for (int i = 0; i < Row<E>::kVec; ++i) x[i] = v0 + i >= 0 && v0 + i < r.V ? to_float(row[v0 + i]) : fill;
  }
}

// Running maximum and sum of exponentials relative to it (an empty one: -inf, 0).
struct Soft {
  float m, z;
};
__device__ __forceinline__ float scaled(float x, float m, float c) { return ptx::ex2((x - m) * c); }
__device__ __forceinline__ Soft join(const Soft& a, const Soft& b, float c) {
  const float m = fmaxf(a.m, b.m);
  const float wa = a.m == -INFINITY ? 1.f : scaled(a.m, m, c), wb = b.m == -INFINITY ? 1.f : scaled(b.m, m, c);
  return {m, a.z * wa + b.z * wb};     // (the sum of an empty part is 0, or NaN by a value that was no number)
}
template <int kN>
__device__ __forceinline__ void add(Soft& s, const float (&x)[kN], float c) {
  float m = x[0];
#pragma unroll
  for (int i = 1; i < kN; ++i) m = fmaxf(m, x[i]);
  if (m > s.m) {
    s.z *= s.m == -INFINITY ? 1.f : scaled(s.m, m, c);
    s.m = m;
  }
  const float ref = s.m == -INFINITY ? 0.f : s.m;
#pragma unroll
  for (int i = 0; i < kN; ++i) s.z += scaled(x[i], ref, c);
}

template <int kThreads>
__device__ __forceinline__ Soft block_join(Soft s, float c, Soft* red) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) s = join(s, {__shfl_xor_sync(0xffffffffu, s.m, o), __shfl_xor_sync(0xffffffffu, s.z, o)}, c);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
  __syncthreads();
  s = red[0];
  for (int i = 1; i < kThreads / 32; ++i) s = join(s, red[i], c);
  return s;
}

struct LossArgs {
  const void* draft;
  const float *top, *target_lse, *feat;
  const int32_t *ids, *seq;
  float *loss, *saved;
  long long stride;
  int K, V, n, h, splits;
  float temperature, tau, raised;
};

// One row a cluster of `splits` CTAs.  Memory-bound: the row, the stored logits and the hidden states are read once, the drafter's
// logits of the stored tokens again from the L2.
template <typename E, int kThreads>
__global__ void __launch_bounds__(kThreads) k_distill_loss(const LossArgs a) {
  constexpr int kVec = Row<E>::kVec, kBatch = 4, kHold = 4;
  __shared__ Soft red_d[kThreads / 32], red_t[kThreads / 32];
  __shared__ __align__(16) float4 s_soft[kMaxSplits];      // (m, Z, m_t, Z_t) of every CTA of the row
  __shared__ double s_part[kMaxSplits][5];                 // its sums: q (m - d), q, and the three of the cosine
  __shared__ double s_red[kThreads / 32][5];
  const int row = blockIdx.x / a.splits, rank = blockIdx.x % a.splits, tid = threadIdx.x;
  const float c = kLog2e / a.temperature, inv_t = 1.f / a.temperature;
  const int seq = a.seq == nullptr ? 0 : a.seq[row];
  if (seq < 0) {                                           // (the same in every CTA of the cluster)
    if (rank == 0 && tid == 0) {
      a.loss[row] = 0.f;
      reinterpret_cast<float4*>(a.saved)[row] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    return;
  }
  const E* d = static_cast<const E*>(a.draft) + row * a.stride;
  const float* top = a.top + (long long)row * a.n;
  const int32_t* ids = a.ids + (long long)row * a.n;
  // the stored entries of this CTA: the first few of a thread stay in registers
  const int per = (a.n + a.splits - 1) / a.splits, i0 = min(a.n, rank * per), i1 = min(a.n, i0 + per);
  float t[kHold];
  int id[kHold];
#pragma unroll
  for (int i = 0; i < kHold; ++i) {
    const int at = i0 + i * kThreads + tid;
    id[i] = at < i1 ? ids[at] : -1;
    t[i] = at < i1 ? top[at] : -INFINITY;
    if (id[i] < 0 || id[i] >= a.V) {
      id[i] = -1;
      t[i] = -INFINITY;
    }
  }
  auto each_more = [&](auto&& f) {                         // the others
    for (int at = i0 + kHold * kThreads + tid; at < i1; at += kThreads) {
      const int v = ids[at];
      if (v >= 0 && v < a.V) f(v, top[at]);
    }
  };
  // the row
  const Row<E> r(d, a.V);
  const int pieces = r.pieces(), share = (pieces + a.splits - 1) / a.splits, p1 = min(pieces, (rank + 1) * share);
  Soft sd = {-INFINITY, 0.f};
  for (int p = rank * share + tid; p < p1; p += kBatch * kThreads) {
    float x[kBatch][kVec];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      if (p + b * kThreads < p1) {
        load_piece(d, r, p + b * kThreads, -INFINITY, x[b]);
      } else {
#pragma unroll
        for (int i = 0; i < kVec; ++i) x[b][i] = -INFINITY;
      }
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) add(sd, x[b], c);
  }
  Soft st = {-INFINITY, 0.f};
  if (a.target_lse == nullptr) {
    add(st, t, c);
    each_more([&](int, float x) {
      const float one[1] = {x};
      add(st, one, c);
    });
  }
  sd = block_join<kThreads>(sd, c, red_d);
  st = block_join<kThreads>(st, c, red_t);
  if (a.splits > 1) {
    ptx::cluster_arrive();
    ptx::cluster_wait();                                   // all CTAs have started
    if (tid < a.splits)
      ptx::st_cluster_v4(ptx::map_to_cta(ptx::smem_u32(&s_soft[rank]), tid), make_float4(sd.m, sd.z, st.m, st.z));
    __syncwarp();
    ptx::cluster_arrive();
    ptx::cluster_wait();
    sd = {s_soft[0].x, s_soft[0].y};
    st = {s_soft[0].z, s_soft[0].w};
    for (int i = 1; i < a.splits; ++i) {
      sd = join(sd, {s_soft[i].x, s_soft[i].y}, c);
      st = join(st, {s_soft[i].z, s_soft[i].w}, c);
    }
  }
  // sums over the stored entries (64 bits: few of them), and those of the cosine with the next position's hidden state
  const bool given = a.target_lse != nullptr;
  const float t_lse = given ? a.target_lse[row] : 0.f, t_ref = st.m == -INFINITY ? 0.f : st.m;
  double sum[5] = {0.0, 0.0, 0.0, 0.0, 0.0};
  auto entry = [&](int v, float x) {
    const float q = given ? ptx::ex2(fmaf(x, inv_t, -t_lse) * kLog2e) : scaled(x, t_ref, c);
    if (q != 0.f) {
      sum[0] += (double)(q * (sd.m - to_float(d[v])));
      sum[1] += (double)q;
    }
  };
#pragma unroll
  for (int i = 0; i < kHold; ++i)
    if (id[i] >= 0) entry(id[i], t[i]);
  each_more(entry);
  const bool pair = a.feat != nullptr && row + 1 < a.K && (a.seq == nullptr || a.seq[row + 1] == seq);
  if (pair) {
    const float *fa = a.feat + (long long)row * a.h, *fb = fa + a.h;
    for (int i = rank * kThreads + tid; i < a.h; i += a.splits * kThreads) {
      const double x = fa[i], y = fb[i];
      sum[2] += x * y;
      sum[3] += x * x;
      sum[4] += y * y;
    }
  }
#pragma unroll
  for (int i = 0; i < 5; ++i) {
    for (int o = 16; o > 0; o >>= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
    if ((tid & 31) == 0) s_red[tid >> 5][i] = sum[i];
  }
  __syncthreads();
  if (tid < 5) {
    double x = 0.0;
    for (int w = 0; w < kThreads / 32; ++w) x += s_red[w][tid];
    if (a.splits > 1) {
      const uint32_t to = ptx::map_to_cta(ptx::smem_u32(&s_part[rank][tid]), 0);
      asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(to), "d"(x) : "memory");
    } else {
      s_part[0][tid] = x;
    }
  }
  if (a.splits > 1) {
    __syncwarp();
    ptx::cluster_arrive();
    ptx::cluster_wait();
  } else {
    __syncthreads();
  }
  if (rank == 0 && tid == 0) {
    double x[5] = {0.0, 0.0, 0.0, 0.0, 0.0};
    for (int s = 0; s < a.splits; ++s)
      for (int i = 0; i < 5; ++i) x[i] += s_part[s][i];
    const float w = pair && x[2] / (sqrt(x[3]) * sqrt(x[4])) >= (double)a.tau ? a.raised : 1.f;
    const double log_z = log((double)sd.z), z_t = given ? 1.0 : x[1];
    const bool any = x[1] != 0.0;                          // something stored weighs something (or is no number)
    const double mass = given ? x[1] : any ? x[1] / z_t : 0.0;
    const double ce = any ? mass * log_z + x[0] / z_t * (double)inv_t : 0.0;
    a.loss[row] = (float)(w * ce);
    const float lse_t = given ? t_lse : any ? (float)((double)t_ref * inv_t + log(z_t)) : 0.f;
    reinterpret_cast<float4*>(a.saved)[row] = make_float4((float)((double)sd.m * inv_t + log_z), lse_t, (float)mass, w);
  }
}

// total = sum of n values, in a fixed order.
__global__ void __launch_bounds__(1024) k_distill_total(const float* __restrict__ x, int n, float* __restrict__ out) {
  __shared__ double s_warp[32];
  double s = 0.0;
  for (int i = threadIdx.x; i < n; i += 1024) s += (double)x[i];
  for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) s_warp[threadIdx.x >> 5] = s;
  __syncthreads();
  if (threadIdx.x < 32) {
    s = s_warp[threadIdx.x];
    for (int o = 16; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    if (threadIdx.x == 0) *out = (float)s;
  }
}

struct GradArgs {
  const void* draft;
  const float *top, *saved, *up;
  const int32_t* ids;
  void* grad;
  long long stride, grad_stride;
  int K, V, n, splits;
  float temperature, scale;
};

// A row, or one of `splits` parts of it, a CTA, in stretches of kStretch places: the stored entries of a stretch go into shared
// memory, then one pass reads the drafter's logits and writes the gradient.  Memory-bound.
template <typename E, int kThreads, int kStretch>
__global__ void __launch_bounds__(kThreads) k_distill_grad(const GradArgs a) {
  constexpr int kVec = Row<E>::kVec, kBatch = kStretch / kVec / kThreads, kHold = 4;
  __shared__ __align__(16) float s_q[kStretch];
  __shared__ int s_twice;
  const int row = blockIdx.x / a.splits, part = blockIdx.x % a.splits, tid = threadIdx.x;
  // (row by row the logits may be where the gradient goes: every element is read before the same thread writes it)
  const E* d = static_cast<const E*>(a.draft) + row * a.stride;
  E* g = static_cast<E*>(a.grad) + row * a.grad_stride;
  const float4 saved = reinterpret_cast<const float4*>(a.saved)[row];      // lse, target lse, Q, weight
  const float inv_t = 1.f / a.temperature;
  const float f = saved.w * (a.up == nullptr ? 1.f : a.up[row]) * a.scale * inv_t;
  const Row<E> r(g, a.V);
  const bool same = r.lead == Row<E>(d, a.V).lead;         // both rows have their 16-byte boundaries at the same elements
  const int pieces = r.pieces(), share = ((pieces + a.splits - 1) / a.splits + 31) / 32 * 32;
  const int first = min(pieces, part * share), last = min(pieces, first + share);
  auto store = [&](int piece, const float (&x)[kVec]) {
    const int v0 = piece * kVec - r.lead;
    if (r.whole(piece)) {
      *reinterpret_cast<uint4*>(g + v0) = pack(x);
    } else {
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        if (v0 + i >= 0 && v0 + i < r.V) from_float(g + v0 + i, x[i]);
    }
  };
  if (f == 0.f) {                                          // padding: nothing of the row is looked at
    float zero[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) zero[i] = 0.f;
    for (int p = first + tid; p < last; p += kThreads) store(p, zero);
    return;
  }
  const float* top = a.top + (long long)row * a.n;
  const int32_t* ids = a.ids + (long long)row * a.n;
  auto weight = [&](float t) { return ptx::ex2(fmaf(t, inv_t, -saved.y) * kLog2e); };
  int place[kHold];
  float q[kHold];
#pragma unroll
  for (int i = 0; i < kHold; ++i) {
    const int at = i * kThreads + tid, v = at < a.n ? ids[at] : -1;
    place[i] = v >= 0 && v < a.V ? v + r.lead : -1;
    q[i] = place[i] >= 0 ? weight(top[at]) : 0.f;
  }
  if (tid == 0) s_twice = 0;
  for (int p0 = first; p0 < last; p0 += kStretch / kVec) {
    const int base = p0 * kVec, n_piece = min(last - p0, kStretch / kVec);
    float x[kBatch][kVec];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int p = b * kThreads + tid;
      if (p < n_piece) {
        if (same) {
          load_piece(d, r, p0 + p, 0.f, x[b]);
        } else {
          const int v0 = (p0 + p) * kVec - r.lead;
#pragma unroll
          for (int i = 0; i < kVec; ++i) x[b][i] = v0 + i >= 0 && v0 + i < a.V ? to_float(d[v0 + i]) : 0.f;
        }
      }
    }
    for (int i = tid; i < kStretch / 4; i += kThreads) reinterpret_cast<float4*>(s_q)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    __syncthreads();
    auto put = [&](int at, float w) {
      const int in = at - base;
      if (in >= 0 && in < n_piece * kVec && atomicExch(&s_q[in], w) != 0.f) s_twice = 1;
    };
#pragma unroll
    for (int i = 0; i < kHold; ++i)
      if (place[i] >= 0) put(place[i], q[i]);
    for (int at = kHold * kThreads + tid; at < a.n; at += kThreads) {
      const int v = ids[at];
      if (v >= 0 && v < a.V) put(v + r.lead, weight(top[at]));
    }
    __syncthreads();
    if (s_twice) {                                         // a token more than once: its entries in order, by the thread that owns it
      for (int i = tid; i < kStretch; i += kThreads) s_q[i] = 0.f;
      __syncthreads();
      for (int at = 0; at < a.n; ++at) {
        const int v = ids[at], in = v + r.lead - base;
        if (v >= 0 && v < a.V && in >= 0 && in < n_piece * kVec && in % kThreads == tid) s_q[in] += weight(top[at]);
      }
      __syncthreads();
      if (tid == 0) s_twice = 0;
    }
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int p = b * kThreads + tid;
      if (p < n_piece) {
        float y[kVec];
#pragma unroll
        for (int i = 0; i < kVec; ++i)
          y[i] = f * fmaf(saved.z, ptx::ex2(fmaf(x[b][i], inv_t, -saved.x) * kLog2e), -s_q[p * kVec + i]);
        store(p0 + p, y);
      }
    }
    __syncthreads();
  }
}

constexpr int kLossThreads = 512, kGradThreads = 512, kStretch = 8192;
constexpr int kMostValues = INT32_MAX - 65535;      // tokens and stored entries of a row: indexes stay in 32 bits beyond the last one
constexpr long long kMostStride = 1ll << 40;

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
  return n;
}

template <typename E>
int launch_loss(const LossArgs& in, cudaStream_t s) {
  LossArgs a = in;
  const int sms = sm_count();
  if (sms <= 0) return CASCADE_ERR_CUDA;
  // few rows: as many CTAs a row as fill the SMs, each with two batches of loads a thread at least
  const long long bytes = (long long)a.V * sizeof(E);
  a.splits = 1;
  while (a.splits < kMaxSplits && (long long)a.K * a.splits * 2 <= 2 * sms && bytes >= (long long)a.splits * kLossThreads * 64) a.splits *= 2;
  if ((long long)a.K * a.splits > INT32_MAX) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.K * a.splits));
  cfg.blockDim = dim3(kLossThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = a.splits;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  CASCADE_CUDA_TRY(cudaLaunchKernelEx(&cfg, k_distill_loss<E, kLossThreads>, a));
  return CASCADE_OK;
}

template <typename E>
int launch_grad(const GradArgs& in, cudaStream_t s) {
  GradArgs a = in;
  const int sms = sm_count();
  if (sms <= 0) return CASCADE_ERR_CUDA;
  const int stretches = cascade_detail::ceil_div(a.V, kStretch);
  a.splits = 1;
  while (a.splits * 2 <= stretches * 2 && (long long)a.K * a.splits * 2 <= 3 * sms) a.splits *= 2;
  if ((long long)a.K * a.splits > INT32_MAX) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  k_distill_grad<E, kGradThreads, kStretch><<<a.K * a.splits, kGradThreads, 0, s>>>(a);
  CASCADE_CUDA_TRY(cudaGetLastError());
  return CASCADE_OK;
}

bool off(const void* p, unsigned align) { return (reinterpret_cast<uintptr_t>(p) & (align - 1)) != 0; }

bool meets(const void* a, long long a_bytes, const void* b, long long b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a != nullptr && b != nullptr && x < y + b_bytes && y < x + a_bytes;
}

// Bytes from the first to the last element of K rows of V elements.
long long span(int K, int V, long long stride, int es) { return ((K - 1) * stride + V) * es; }

}  // namespace

extern "C" int cascade_distill_loss(const void* draft_logits, int32_t logits_dtype, int64_t row_stride, const float* top_logits,
                                    const int32_t* top_ids, int32_t n_top, const float* target_lse, const float* feat,
                                    const int32_t* seq, int32_t K, int32_t V, int32_t h, float temperature, float tau_seq, float c,
                                    float* loss_out, float* saved_out, float* total_out, void* stream) {
  if (draft_logits == nullptr || top_logits == nullptr || top_ids == nullptr || loss_out == nullptr || saved_out == nullptr)
    return CASCADE_ERR_INVALID_ARG;
  if (logits_dtype != CASCADE_F32 && logits_dtype != CASCADE_BF16) return CASCADE_ERR_INVALID_ARG;
  if (K < 1 || V < 1 || n_top < 1 || (feat != nullptr && h < 1) || row_stride < V || row_stride > kMostStride)
    return CASCADE_ERR_INVALID_ARG;
  if (V > kMostValues || n_top > kMostValues) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  if (!(temperature > 0.f && temperature <= 1e30f && temperature >= 1e-30f) || !(c > 0.f) || tau_seq != tau_seq) return CASCADE_ERR_INVALID_ARG;
  const int es = logits_dtype == CASCADE_BF16 ? 2 : 4;
  if (off(draft_logits, es) || off(top_logits, 4) || off(top_ids, 4) || off(target_lse, 4) || off(feat, 4) || off(seq, 4) ||
      off(loss_out, 4) || off(saved_out, 16) || off(total_out, 4))
    return CASCADE_ERR_INVALID_ARG;
  const struct {
    const void* at;
    long long bytes;
  } in[] = {{draft_logits, span(K, V, row_stride, es)}, {top_logits, 4ll * K * n_top}, {top_ids, 4ll * K * n_top}, {target_lse, 4ll * K},
            {feat, 4ll * K * h}, {seq, 4ll * K}},
    out[] = {{loss_out, 4ll * K}, {saved_out, 16ll * K}, {total_out, 4}};
  for (int i = 0; i < 3; ++i) {
    for (const auto& x : in)
      if (meets(out[i].at, out[i].bytes, x.at, x.bytes)) return CASCADE_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (meets(out[i].at, out[i].bytes, out[j].at, out[j].bytes)) return CASCADE_ERR_INVALID_ARG;
  }
  LossArgs a;
  a.draft = draft_logits;
  a.top = top_logits;
  a.target_lse = target_lse;
  a.feat = feat;
  a.ids = top_ids;
  a.seq = seq;
  a.loss = loss_out;
  a.saved = saved_out;
  a.stride = row_stride;
  a.K = K;
  a.V = V;
  a.n = n_top;
  a.h = h;
  a.temperature = temperature;
  a.tau = tau_seq;
  a.raised = c;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  CASCADE_TRY(logits_dtype == CASCADE_BF16 ? launch_loss<__nv_bfloat16>(a, s) : launch_loss<float>(a, s));
  if (total_out != nullptr) {
    k_distill_total<<<1, 1024, 0, s>>>(loss_out, K, total_out);
    CASCADE_CUDA_TRY(cudaGetLastError());
  }
  return CASCADE_OK;
}

extern "C" int cascade_distill_grad(const void* draft_logits, int32_t logits_dtype, int64_t row_stride, const float* top_logits,
                                    const int32_t* top_ids, int32_t n_top, const float* saved, const float* grad_loss, float scale,
                                    int32_t K, int32_t V, float temperature, void* grad_out, int64_t grad_stride, void* stream) {
  if (draft_logits == nullptr || top_logits == nullptr || top_ids == nullptr || saved == nullptr || grad_out == nullptr)
    return CASCADE_ERR_INVALID_ARG;
  if (logits_dtype != CASCADE_F32 && logits_dtype != CASCADE_BF16) return CASCADE_ERR_INVALID_ARG;
  if (K < 1 || V < 1 || n_top < 1 || row_stride < V || grad_stride < V || row_stride > kMostStride || grad_stride > kMostStride)
    return CASCADE_ERR_INVALID_ARG;
  if (V > kMostValues || n_top > kMostValues) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  if (!(temperature > 0.f && temperature <= 1e30f && temperature >= 1e-30f) || !(scale - scale == 0.f)) return CASCADE_ERR_INVALID_ARG;
  const int es = logits_dtype == CASCADE_BF16 ? 2 : 4;
  if (off(draft_logits, es) || off(grad_out, es) || off(top_logits, 4) || off(top_ids, 4) || off(saved, 16) || off(grad_loss, 4))
    return CASCADE_ERR_INVALID_ARG;
  const long long bytes = span(K, V, grad_stride, es);
  const bool in_place = grad_out == draft_logits && (grad_stride == row_stride || K == 1);
  if ((!in_place && meets(grad_out, bytes, draft_logits, span(K, V, row_stride, es))) || meets(grad_out, bytes, top_logits, 4ll * K * n_top) ||
      meets(grad_out, bytes, top_ids, 4ll * K * n_top) || meets(grad_out, bytes, saved, 16ll * K) || meets(grad_out, bytes, grad_loss, 4ll * K))
    return CASCADE_ERR_INVALID_ARG;
  GradArgs a;
  a.draft = draft_logits;
  a.top = top_logits;
  a.saved = saved;
  a.up = grad_loss;
  a.ids = top_ids;
  a.grad = grad_out;
  a.stride = row_stride;
  a.grad_stride = grad_stride;
  a.K = K;
  a.V = V;
  a.n = n_top;
  a.temperature = temperature;
  a.scale = scale;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  return logits_dtype == CASCADE_BF16 ? launch_grad<__nv_bfloat16>(a, s) : launch_grad<float>(a, s);
}
