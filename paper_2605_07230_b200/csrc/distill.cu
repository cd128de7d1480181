// The drafter's training loss (Section 4.3, Eq. 4) against the target's largest logits alone, and its gradient.
//
// With t_i, id_i the stored logits and tokens of a position, d the drafter's row, T the temperature and w the position's weight:
//     q_i = exp(t_i / T) / sum_j exp(t_j / T)      (or exp(t_i / T - target_lse): the target's mass outside is left out)
//     loss = - w sum_i q_i log softmax(d / T)[id_i] = w (Q log Z + sum_i q_i (m - d_id) / T)
//     grad = (w / T) (Q softmax(d / T) - sum_i q_i e_id)
// with m the row's maximum, Z = sum_v exp((d_v - m) / T), Q = sum_i q_i.
//
// Both are memory-bound and walk over a row once.  The loss looks the drafter's logits of the stored tokens up behind the row, from the
// L1 or L2.  (In front of it 292 to 322 us for 4608 rows of 65536 where this takes 246, since memory gives 64 bytes for 4; from shared
// memory, as the gradient does it, 494 us: too much work an element.)  The gradient goes in stretches: the stored entries that fall into one
// go into shared memory at their tokens' places, then the logits, already requested, are worked on beside them.
#include "cascade_internal.h"
#include "overlap.h"
#include "ptx_paged.cuh"

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr int kMaxSplits = 8;       // CTAs of one row of the loss (a cluster)
constexpr int kBatch = 4;           // pieces a thread of a stretch
constexpr int kHold = 4;            // stored entries that a thread holds in registers

// Rows are walked in pieces of 16 bytes from the 16-byte boundary at or in front of their first element: element v of the row
// is place v + lead.  The pieces that lie wholly inside are `first` .. `last` - 1; what is left at both ends goes element by element.
template <typename E>
struct Row {
  static constexpr int kVec = 16 / (int)sizeof(E);
  int lead, first, last, V, head, tail;                    // (elements in front of `head` and from `tail` on are the ends)
  __device__ __forceinline__ Row(const E* row, int v)
      : lead((int)((reinterpret_cast<uintptr_t>(row) & 15u) / sizeof(E))), first(lead > 0), last(max((v + lead) / kVec, first)), V(v),
        head(min(first * kVec - lead, v)), tail(max(last * kVec - lead, head)) {}
  // i = 0 .. 2 kVec - 1: an element of the ends, V or more for none
  __device__ __forceinline__ int edge(int i) const { return i >= kVec ? tail + i - kVec : i < head ? i : V; }
};

// The values of a piece as pairs.
__device__ __forceinline__ void unpack(const uint4& r, uint64_t (&x)[2]) {
  x[0] = (uint64_t)r.y << 32 | r.x;
  x[1] = (uint64_t)r.w << 32 | r.z;
}
__device__ __forceinline__ void unpack(const uint4& r, uint64_t (&x)[4]) {
  const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = ptx::pack2(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
}
__device__ __forceinline__ uint4 pack(const uint64_t (&x)[2]) {
  return make_uint4((uint32_t)x[0], (uint32_t)(x[0] >> 32), (uint32_t)x[1], (uint32_t)(x[1] >> 32));
}
__device__ __forceinline__ uint4 pack(const uint64_t (&x)[4]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float lo, hi;
    ptx::unpack2(x[i], &lo, &hi);
    w[i] = ptx::pack_bf16x2(lo, hi);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint64_t both(float x) { return ptx::pack2(x, x); }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ uint32_t bits_of(const float* p) { return __float_as_uint(*p); }
__device__ __forceinline__ uint32_t bits_of(const __nv_bfloat16* p) { return *reinterpret_cast<const uint16_t*>(p); }
__device__ __forceinline__ void from_float(float* p, float x) { *p = x; }
__device__ __forceinline__ void from_float(__nv_bfloat16* p, float x) { *p = __float2bfloat16(x); }

// A thread's pieces of the stretch that begins at piece p0.
template <typename E, int kThreads>
__device__ __forceinline__ void load_stretch(const E* d, int lead, bool aligned, int p0, int last, uint4 (&raw)[kBatch]) {
  constexpr int kVec = Row<E>::kVec;
#pragma unroll
  for (int b = 0; b < kBatch; ++b) {
    const int p = p0 + b * kThreads + (int)threadIdx.x;
    if (p >= last) break;
    if (aligned) {
      raw[b] = reinterpret_cast<const uint4*>(d - lead)[p];
    } else {
      const E* x = d + (p * kVec - lead);
      uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < kVec; ++i) w[i * (int)sizeof(E) / 4] |= bits_of(x + i) << (i * (int)sizeof(E) % 4 * 8);
      raw[b] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
}

// What is stored of a position: the first entries of a thread stay in registers.
template <int kThreads>
struct Stored {
  const float* top;
  const int32_t* ids;
  int n, V, token[kHold];
  float value[kHold];                                      // logits, then weights
  __device__ __forceinline__ Stored(const float* t, const int32_t* i, int count, int v) : top(t), ids(i), n(count), V(v) {
#pragma unroll
    for (int k = 0; k < kHold; ++k) {
      const int at = k * kThreads + (int)threadIdx.x;
      token[k] = at < n ? ids[at] : -1;
      value[k] = at < n ? top[at] : -INFINITY;
    }
#pragma unroll
    for (int k = 0; k < kHold; ++k)
      if (token[k] < 0 || token[k] >= V) {
        token[k] = -1;
        value[k] = -INFINITY;
      }
  }
  template <typename F>
  __device__ __forceinline__ void each_more(F&& f) const { // the entries beyond those
    for (int at = kHold * kThreads + (int)threadIdx.x; at < n; at += kThreads) {
      const int v = ids[at];
      if (v >= 0 && v < V) f(v, top[at]);
    }
  }
  // s_q[place] = the weight of the token there, for the places of a stretch (base: its first token) and, with `ends`, the elements at
  // the row's ends behind them.  Ends with a barrier; the next call wants one in front of it.
  template <typename W>
  __device__ __forceinline__ void scatter(float* s_q, int* s_twice, int base, int places, bool ends, int head, int tail, int vec, W&& weight) const {
    const int tid = threadIdx.x, slots = places + (ends ? 2 * vec : 0);
    auto place = [&](int v) {
      const int in = v - base;
      if (v < 0 || v >= V) return -1;
      if (in >= 0 && in < places) return in;
      return !ends ? -1 : v < head ? places + v : v >= tail ? places + vec + v - tail : -1;
    };
    for (int i = tid; i < slots / 4; i += kThreads) reinterpret_cast<float4*>(s_q)[i] = make_float4(0.f, 0.f, 0.f, 0.f);
    if (tid == 0) *s_twice = 0;
    __syncthreads();
    auto put = [&](int at, float w) {
      if (at >= 0 && atomicExch(&s_q[at], w) != 0.f) *s_twice = 1;
    };
#pragma unroll
    for (int k = 0; k < kHold; ++k) put(place(token[k]), value[k]);
    each_more([&](int v, float t) {
      const int at = place(v);
      if (at >= 0) put(at, weight(t));
    });
    __syncthreads();
    if (*s_twice) {                                        // a token more than once: its entries in order, by the thread that owns it
      for (int i = tid; i < slots; i += kThreads) s_q[i] = 0.f;
      __syncthreads();
      for (int at = 0; at < n; ++at) {
        const int in = place(ids[at]);
        if (in >= 0 && in % kThreads == tid) s_q[in] += weight(top[at]);
      }
      __syncthreads();
    }
  }
};

// Running maximum m and sum of 2^(c x - c m) with c m rounded once (an empty one: -inf, 0).
struct Soft {
  float m, z;
};
__device__ __forceinline__ float reference(float m, float c) { return m == -INFINITY ? 0.f : m * c; }
__device__ __forceinline__ float scaled(float x, float ref, float c) { return ptx::ex2(fmaf(x, c, -ref)); }
__device__ __forceinline__ Soft join(const Soft& a, const Soft& b, float c) {
  const float m = fmaxf(a.m, b.m), ref = reference(m, c);
  const float wa = a.m == -INFINITY ? 1.f : ptx::ex2(reference(a.m, c) - ref), wb = b.m == -INFINITY ? 1.f : ptx::ex2(reference(b.m, c) - ref);
  return {m, a.z * wa + b.z * wb};     // (the sum of an empty part is 0, or NaN by a value that was no number)
}
// `ref` = reference(s.m, c) goes along.
__device__ __forceinline__ void raise(Soft& s, float& ref, float m, float c) {
  if (m > s.m) {
    const float to = m * c;
    if (s.m != -INFINITY) s.z *= ptx::ex2(ref - to);
    s.m = m;
    ref = to;
  }
}
template <int kN>
__device__ __forceinline__ void add(Soft& s, float& ref, const uint64_t (&x)[kN], float c) {
  float m = -INFINITY;
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    float a, b;
    ptx::unpack2(x[i], &a, &b);
    m = fmaxf(m, fmaxf(a, b));
  }
  raise(s, ref, m, c);
  const uint64_t cc = both(c), minus = both(-ref);
  uint64_t sum = 0;
#pragma unroll
  for (int i = 0; i < kN; ++i) {
    float a, b;
    ptx::unpack2(ptx::fma2(x[i], cc, minus), &a, &b);
    sum = ptx::add2(sum, ptx::pack2(ptx::ex2(a), ptx::ex2(b)));
  }
  float a, b;
  ptx::unpack2(sum, &a, &b);
  s.z += a + b;
}
__device__ __forceinline__ Soft warp_join(Soft s, float c, int lanes) {
  for (int o = lanes / 2; o > 0; o >>= 1) s = join(s, {__shfl_xor_sync(0xffffffffu, s.m, o), __shfl_xor_sync(0xffffffffu, s.z, o)}, c);
  return s;
}
// The largest of `lanes` values that are -inf as a rule.
__device__ __forceinline__ float most_left_out(float x, int lanes) {
  if (__any_sync(0xffffffffu, x != -INFINITY))
    for (int o = lanes / 2; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
template <int kThreads>
__device__ __forceinline__ float block_max(float x, float* red) {
  constexpr int kWarps = kThreads / 32;
  for (int o = 16; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = x;
  __syncthreads();
  x = red[threadIdx.x & (kWarps - 1)];
  for (int o = kWarps / 2; o > 0; o >>= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
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

// One row a cluster of `splits` CTAs, a share of the row and of the stored entries each.
template <typename E, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) k_distill_loss(const LossArgs a) {
  constexpr int kVec = Row<E>::kVec, kWarps = kThreads / 32, kPieces = kBatch * kThreads;
  __shared__ float s_max[kWarps];
  __shared__ Soft s_warp[kWarps];
  __shared__ double s_sum[kWarps][5];
  __shared__ float s_out[kWarps];
  __shared__ __align__(16) float4 s_soft[kMaxSplits];      // (m, Z, largest stored logit, largest left out) of every CTA of the row
  __shared__ double s_part[kMaxSplits][5];                 // its sums: q d, q, and the three of the cosine
  asm volatile("griddepcontrol.launch_dependents;");       // (the kernel that adds the losses up waits for this one's end itself)
  const int row = blockIdx.x / a.splits, rank = blockIdx.x % a.splits, tid = threadIdx.x;
  const float c = kLog2e / a.temperature, inv_t = 1.f / a.temperature;
  const int seq = a.seq == nullptr ? 0 : a.seq[row], seq_next = a.seq == nullptr ? 0 : row + 1 < a.K ? a.seq[row + 1] : -1;
  // what comes first of everything is requested at once, padding's too
  const E* d = static_cast<const E*>(a.draft) + row * a.stride;
  const Row<E> r(d, a.V);
  const int share = (r.last - r.first + a.splits - 1) / a.splits, last = min(r.last, r.first + (rank + 1) * share);
  int p = r.first + rank * share;
  uint4 raw[kBatch];
  load_stretch<E, kThreads>(d, r.lead, true, p, last, raw);
  const int per = (a.n + a.splits - 1) / a.splits, i0 = min(a.n, rank * per);
  Stored<kThreads> stored(a.top + (long long)row * a.n + i0, a.ids + (long long)row * a.n + i0, min(a.n - i0, per), a.V);
  if (seq < 0) {                                           // (the same in every CTA of the cluster)
    if (rank == 0 && tid == 0) {
      a.loss[row] = 0.f;
      reinterpret_cast<float4*>(a.saved)[row] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    return;
  }
  if (a.splits > 1) ptx::cluster_arrive();                 // (waited for before anything is written to another CTA)
  // the sums of the cosine with the next position's hidden state (64 bits: it may lie next to the threshold)
  double sum[5] = {0.0, 0.0, 0.0, 0.0, 0.0};
  const bool pair = a.feat != nullptr && row + 1 < a.K && seq_next == seq;
  if (pair) {
    const float *fa = a.feat + (long long)row * a.h, *fb = fa + a.h;
    auto term = [&](float x, float y) {
      const double u = x, v = y;
      sum[2] += u * v;
      sum[3] += u * u;
      sum[4] += v * v;
    };
    const int step = a.splits * kThreads, from = rank * kThreads + tid;
    if ((a.h & 3) == 0 && (reinterpret_cast<uintptr_t>(a.feat) & 15u) == 0) {
      const float4 *va = reinterpret_cast<const float4*>(fa), *vb = reinterpret_cast<const float4*>(fb);
#pragma unroll 4
      for (int i = from; i < a.h / 4; i += step) {
        const float4 x = va[i], y = vb[i];
        term(x.x, y.x);
        term(x.y, y.y);
        term(x.z, y.z);
        term(x.w, y.w);
      }
    } else {
#pragma unroll 4
      for (int i = from; i < a.h; i += step) term(fa[i], fb[i]);
    }
  }
  // the row
  Soft sd = {-INFINITY, 0.f};
  float ref_d = 0.f;
  if (rank == 0 && tid < 2 * kVec && r.edge(tid) < a.V) {
    const uint64_t one[1] = {ptx::pack2(to_float(d[r.edge(tid)]), -INFINITY)};
    add(sd, ref_d, one, c);
  }
  for (; p < last; p += kPieces) {
    uint4 now[kBatch];
#pragma unroll
    for (int b = 0; b < kBatch; ++b) now[b] = raw[b];
    load_stretch<E, kThreads>(d, r.lead, true, p + kPieces, last, raw);
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      if (p + b * kThreads + tid >= last) break;
      uint64_t x[kVec / 2];
      unpack(now[b], x);
      add(sd, ref_d, x, c);
    }
  }
  // the drafter's logits of the stored tokens, from the L1 or L2
  float dv[kHold];
#pragma unroll
  for (int k = 0; k < kHold; ++k) dv[k] = stored.token[k] >= 0 ? to_float(d[stored.token[k]]) : 0.f;
  const bool given = a.target_lse != nullptr;
  const float t_lse = given ? a.target_lse[row] : 0.f;
  float most = -INFINITY;
  if (!given) {
#pragma unroll
    for (int k = 0; k < kHold; ++k) most = fmaxf(most, stored.value[k]);
    stored.each_more([&](int, float t) { most = fmaxf(most, t); });
    most = block_max<kThreads>(most, s_max);
  }
  // sums over the entries (64 bits: few of them, and maximum times weight less weight times logit cancels); of the entries whose token
  // the drafter leaves out (-inf) the largest logit: whether it weighs anything goes by the largest of the whole row
  auto weight = [&](float t, float ref) { return given ? ptx::ex2(fmaf(t, inv_t, -t_lse) * kLog2e) : scaled(t, ref, c); };
  const float ref_t = reference(most, c);
  float left_out = -INFINITY;
  auto entry = [&](float t, float y) {
    const float q = weight(t, ref_t);
    if (q != 0.f) {                                        // (a token that weighs nothing may have -inf)
      const bool out = y == -INFINITY;
      left_out = fmaxf(left_out, out ? t : -INFINITY);
      sum[0] += (double)q * (double)(out ? 0.f : y);
      sum[1] += (double)q;
    }
  };
#pragma unroll
  for (int k = 0; k < kHold; ++k)
    if (stored.token[k] >= 0) entry(stored.value[k], dv[k]);
  stored.each_more([&](int v, float t) { entry(t, to_float(d[v])); });
  sd = warp_join(sd, c, 32);
  left_out = most_left_out(left_out, 32);
#pragma unroll
  for (int i = 0; i < 5; ++i)
    for (int o = 16; o > 0; o >>= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
  if ((tid & 31) == 0) {
    s_warp[tid >> 5] = sd;
    s_out[tid >> 5] = left_out;
#pragma unroll
    for (int i = 0; i < 5; ++i) s_sum[tid >> 5][i] = sum[i];
  }
  __syncthreads();
  if (a.splits > 1) ptx::cluster_wait();                   // all CTAs have started
  if (tid < 32) {
    sd = warp_join(s_warp[tid & (kWarps - 1)], c, kWarps);
    left_out = most_left_out(s_out[tid & (kWarps - 1)], kWarps);
    const uint32_t to = a.splits > 1 ? ptx::map_to_cta(ptx::smem_u32(&s_part[rank][tid < 5 ? tid : 0]), 0) : ptx::smem_u32(&s_part[0][tid < 5 ? tid : 0]);
    if (tid < 5) {
      double y = 0.0;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) y += s_sum[w][tid];
      asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(to), "d"(y) : "memory");
    }
    if (tid == 5)
      ptx::st_cluster_v4(a.splits > 1 ? ptx::map_to_cta(ptx::smem_u32(&s_soft[rank]), 0) : ptx::smem_u32(&s_soft[0]), make_float4(sd.m, sd.z, most, left_out));
    __syncwarp();
  }
  if (a.splits > 1) {
    __syncwarp();
    ptx::cluster_arrive();
    ptx::cluster_wait();
  }
  if (rank == 0 && tid == 0) {
    double y[5] = {0.0, 0.0, 0.0, 0.0, 0.0};
    most = s_soft[0].z;
    left_out = s_soft[0].w;
    for (int s = 1; s < a.splits; ++s) {
      most = fmaxf(most, s_soft[s].z);
      left_out = fmaxf(left_out, s_soft[s].w);
    }
    for (int s = 0; s < a.splits; ++s) {
      const float4 x = s_soft[s];
      sd = s == 0 ? Soft{x.x, x.y} : join(sd, {x.x, x.y}, c);
      // (a CTA's weights are by its own largest entry)
      const double by = given || a.splits == 1 || x.z == -INFINITY ? 1.0 : (double)exp2f(reference(x.z, c) - reference(most, c));
      for (int i = 0; i < 5; ++i) y[i] += i < 2 ? by * s_part[s][i] : s_part[s][i];
    }
    if (left_out != -INFINITY && weight(left_out, reference(most, c)) != 0.f) y[0] = -INFINITY;
    // cosine >= tau, squared with its sign (zeros and infinities have no cosine)
    const double squares = y[3] * y[4], bound = (double)a.tau * fabs((double)a.tau) * squares;
    const float w = pair && squares > 0.0 && squares < (double)INFINITY && y[2] * fabs(y[2]) >= bound ? a.raised : 1.f;
    // log sum exp((d - m) / T): what c m was rounded by comes back
    const double log_z = (double)logf(sd.z) + ((double)reference(sd.m, c) - (double)sd.m * c) * (double)kLn2;
    const bool any = y[1] != 0.0;                          // something stored weighs something (or is no number)
    const double mass = given ? y[1] : any ? y[1] / y[1] : 0.0, gap = (double)sd.m * y[1] - y[0];
    const double ce = any ? mass * log_z + (given ? gap : gap / y[1]) * (double)inv_t : 0.0;
    a.loss[row] = (float)(w * ce);
    const float lse_t = given ? t_lse
                        : any ? (float)((double)most * inv_t + (double)logf((float)y[1]) + ((double)reference(most, c) - (double)most * c) * (double)kLn2)
                              : 0.f;
    reinterpret_cast<float4*>(a.saved)[row] = make_float4((float)((double)sd.m * inv_t + log_z), lse_t, (float)mass, w);
  }
}

// total = sum of n values, in a fixed order.
__global__ void __launch_bounds__(1024) k_distill_total(const float* __restrict__ x, int n, float* __restrict__ out) {
  __shared__ double s_warp[32];
  asm volatile("griddepcontrol.wait;" ::: "memory");       // the losses are there
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

// A row, or one of `splits` parts of it, a CTA.
template <typename E, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) k_distill_grad(const GradArgs a) {
  constexpr int kVec = Row<E>::kVec, kPieces = kBatch * kThreads;
  extern __shared__ __align__(16) float s_q[];             // [places of a stretch, then the elements at the row's ends]
  __shared__ int s_twice;
  const int row = blockIdx.x / a.splits, part = blockIdx.x % a.splits, tid = threadIdx.x;
  // (row by row the logits may be where the gradient goes: every element is read before the same thread writes it)
  const E* d = static_cast<const E*>(a.draft) + row * a.stride;
  E* g = static_cast<E*>(a.grad) + row * a.grad_stride;
  const float4 saved = reinterpret_cast<const float4*>(a.saved)[row];      // lse, target lse, Q, weight
  const float up = a.up == nullptr ? 1.f : a.up[row], inv_t = 1.f / a.temperature;
  const Row<E> r(g, a.V);                                  // (logits with other boundaries are read element by element)
  const bool aligned = r.lead == Row<E>(d, a.V).lead;
  const int share = ((r.last - r.first + a.splits - 1) / a.splits + 31) / 32 * 32;
  const int first = min(r.last, r.first + part * share), last = min(r.last, first + share);
  uint4* to = reinterpret_cast<uint4*>(g - r.lead);
  const int edge = part == 0 && tid < 2 * kVec ? r.edge(tid) : a.V;        // (the first part's)
  // what comes first is requested at once, padding's too
  uint4 raw[kBatch];
  load_stretch<E, kThreads>(d, r.lead, aligned, first, last, raw);
  Stored<kThreads> stored(a.top + (long long)row * a.n, a.ids + (long long)row * a.n, a.n, a.V);
  const float f = saved.w * up * a.scale * inv_t;
  // padding, or no entry weighs anything: zeros, whatever the row holds and whatever comes back from above
  if (f == 0.f || saved.w == 0.f || saved.z == 0.f) {
    for (int p = first + tid; p < last; p += kThreads) to[p] = make_uint4(0, 0, 0, 0);
    if (edge < a.V) from_float(g + edge, 0.f);
    return;
  }
  auto weight = [&](float t) { return ptx::ex2(fmaf(t, inv_t, -saved.y) * kLog2e); };
#pragma unroll
  for (int k = 0; k < kHold; ++k) stored.value[k] = weight(stored.value[k]);
  const uint64_t scale2 = both(inv_t), lse2 = both(-saved.x), log2e2 = both(kLog2e), mass2 = both(saved.z * f), minus2 = both(-f);
  for (int p0 = first;; p0 += kPieces) {
    // (requested here and not one stretch ahead: 387 us for 4608 rows of 65536, ahead 420 us; reads and writes in turn suit the memory)
    if (p0 != first) load_stretch<E, kThreads>(d, r.lead, aligned, p0, last, raw);
    const int n_piece = max(0, min(kPieces, last - p0));
    const bool ends = part == 0 && p0 == first;
    stored.scatter(s_q, &s_twice, p0 * kVec - r.lead, n_piece * kVec, ends, r.head, r.tail, kVec, weight);
    if (ends && edge < a.V)
      from_float(g + edge, saved.z * f * ptx::ex2(fmaf(to_float(d[edge]), inv_t, -saved.x) * kLog2e) - f * s_q[n_piece * kVec + tid]);
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
      const int at = b * kThreads + tid;
      if (at >= n_piece) break;
      uint64_t x[kVec / 2];
      unpack(raw[b], x);
      const ulonglong2* sq = reinterpret_cast<const ulonglong2*>(&s_q[at * kVec]);
#pragma unroll
      for (int i = 0; i < kVec / 2; ++i) {
        float lo, hi;
        ptx::unpack2(mul2(ptx::fma2(x[i], scale2, lse2), log2e2), &lo, &hi);
        const ulonglong2 qq = sq[i / 2];
        x[i] = ptx::fma2(ptx::pack2(ptx::ex2(lo), ptx::ex2(hi)), mass2, mul2(i & 1 ? qq.y : qq.x, minus2));
      }
      __stcs(to + p0 + at, pack(x));
    }
    if (p0 + kPieces >= last) break;
    __syncthreads();
  }
}

constexpr int kMostValues = INT32_MAX - 65535;      // tokens and stored entries of a row: indexes stay in 32 bits beyond the last one
constexpr long long kMostStride = 1ll << 40;

int sm_count() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) return 0;
  return n;
}

// Few rows are shared out until every SM has some, in parts of at least 4 pieces a thread of 128.  A part goes over all of its row's
// stored entries, once a stretch, so that it takes as many threads as hold them in registers (4608 rows of 16384, 2000 entries: 512
// threads 126 us, 256 171 us, 128 268 us).  128 threads are for many parts with few entries, of which more are on an SM at once
// (1153 bf16 rows of 10007, 333 entries: 14.5 us, 256 threads 18.4 us; 300 rows: 256 threads 14 us, 128 16 us; 4608 rows of 262144
// bytes: 370 us, 128 380 us).  Shared memory: the places of a stretch and the row's ends.
template <typename E>
int plan(int K, int V, int n, int* splits, int* threads, int* smem) {
  constexpr int kVec = 16 / (int)sizeof(E);
  const int sms = sm_count(), pieces = V / kVec;
  if (sms <= 0) return CASCADE_ERR_CUDA;
  *splits = 1;
  while (*splits * 4 * 128 < pieces && (long long)K * *splits * 2 <= 4 * sms) *splits *= 2;
  if ((long long)K * *splits > INT32_MAX) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  const int part = cascade_detail::ceil_div(pieces, *splits) + 32;
  *threads = n > kHold * 256 ? 512 : n > kHold * 128 || (long long)K * *splits <= 4 * sms || part > 8192 + 32 ? 256 : 128;
  *smem = ((part < kBatch * *threads ? part : kBatch * *threads) * kVec + 2 * kVec) * (int)sizeof(float);
  return CASCADE_OK;
}

template <typename E>
int launch_loss(const LossArgs& in, cudaStream_t s) {
  LossArgs a = in;
  const int sms = sm_count();
  if (sms <= 0) return CASCADE_ERR_CUDA;
  // few rows are shared out until every SM has some
  const long long bytes = (long long)a.V * sizeof(E);
  a.splits = 1;
  while (a.splits < kMaxSplits && bytes >= a.splits * 8192ll && (long long)a.K * a.splits * 2 <= 4 * sms) a.splits *= 2;
  if ((long long)a.K * a.splits > INT32_MAX) return CASCADE_ERR_UNSUPPORTED_SHAPE;
  // Many parts take 128 threads, more of them being on an SM at once (1153 bf16 rows of 10007, 300 entries: 16 us, 256 threads 21 us),
  // unless there are more stored entries than they hold in registers and the part is long: the logits of the entries should still be in
  // the L1 or L2 at its end, so that fewer rows are to be under way (4608 rows of 262144 bytes, 2000 entries: 512 threads 243 us, 256
  // 288 us, 128 336 us; 1000 entries: 233, 222, 257 us; rows of 131072 bytes, 2000 entries: 172, 157, 203 us; of 65536 bytes: 123, 113,
  // 113 us).  A few hundred rows leave room for 256 (400 rows of 65536, 300 entries: 27 us, 128 threads 35 us).
  const long long part = bytes / a.splits;
  const int n = (a.n + a.splits - 1) / a.splits;
  const int threads = a.splits == 1 && a.K <= 4 * sms                                         ? 256
                      : n <= kHold * 128 || (part <= 65536 && a.splits == 1)                    ? 128
                      : n <= kHold * 256 || part <= 131072                                    ? 256
                                                                                              : 512;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(a.K * a.splits));
  cfg.blockDim = dim3(threads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = a.splits;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  auto* f = threads == 128 ? k_distill_loss<E, 128> : threads == 256 ? k_distill_loss<E, 256> : k_distill_loss<E, 512>;
  CASCADE_CUDA_TRY(cudaLaunchKernelEx(&cfg, f, a));
  return CASCADE_OK;
}

template <typename E>
int launch_grad(const GradArgs& in, cudaStream_t s) {
  GradArgs a = in;
  int threads, smem;
  CASCADE_TRY(plan<E>(a.K, a.V, a.n, &a.splits, &threads, &smem));
  auto* f = threads == 128 ? k_distill_grad<E, 128> : threads == 256 ? k_distill_grad<E, 256> : k_distill_grad<E, 512>;
  // (the most that any call of this kernel asks for: calls of other threads may lie between this and the launch)
  CASCADE_CUDA_TRY(cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                        (kBatch * threads + 2) * (16 / (int)sizeof(E)) * (int)sizeof(float)));
  f<<<a.K * a.splits, threads, smem, s>>>(a);
  CASCADE_CUDA_TRY(cudaGetLastError());
  return CASCADE_OK;
}

bool off(const void* p, unsigned align) { return (reinterpret_cast<uintptr_t>(p) & (align - 1)) != 0; }

using cascade_detail::Rows;
// K rows of n elements of `es` bytes, `stride` elements apart (none where nothing is given).
Rows rows(const void* at, int64_t K, int64_t n, int64_t stride, int es) { return {at, at != nullptr ? K : 0, stride * es, n * es}; }
Rows dense(const void* at, int64_t K, int64_t n) { return rows(at, K, n, n, 4); }

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
  const Rows in[] = {rows(draft_logits, K, V, row_stride, es), dense(top_logits, K, n_top), dense(top_ids, K, n_top),
                     dense(target_lse, K, 1), dense(feat, K, h), dense(seq, K, 1)},
             out[] = {dense(loss_out, K, 1), dense(saved_out, K, 4), dense(total_out, 1, 1)};
  for (int i = 0; i < 3; ++i) {
    for (const Rows& x : in)
      if (meet(out[i], x)) return CASCADE_ERR_INVALID_ARG;
    for (int j = 0; j < i; ++j)
      if (meet(out[i], out[j])) return CASCADE_ERR_INVALID_ARG;
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
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(1);
    cfg.blockDim = dim3(1024);
    cfg.stream = s;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;   // it starts beside the losses' kernel and waits for its end
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    CASCADE_CUDA_TRY(cudaLaunchKernelEx(&cfg, k_distill_total, (const float*)loss_out, (int)K, total_out));
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
  const Rows out = rows(grad_out, K, V, grad_stride, es), logits = rows(draft_logits, K, V, row_stride, es);
  const bool in_place = grad_out == draft_logits && (grad_stride == row_stride || K == 1);
  if (!in_place && meet(out, logits)) return CASCADE_ERR_INVALID_ARG;
  for (const Rows& x : {dense(top_logits, K, n_top), dense(top_ids, K, n_top), dense(saved, K, 4), dense(grad_loss, K, 1)})
    if (meet(out, x)) return CASCADE_ERR_INVALID_ARG;
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
