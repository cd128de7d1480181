// One token per row of logits from a given uniform number, after temperature, top-k, nucleus and min-p.
//
//   w[v] = exp((l[v] - m) / T),  token = first v whose cumulative kept weight exceeds u * (total kept weight)
//
// One CTA per row.  The row's order-preserving 32-bit keys stay in shared memory as far as they fit (the rest is read again
// through the L2), so HBM sees each logit once.  Weights are formed in 64 bits (relative error 1e-12) and summed as 64-bit
// fixed point: sums do not depend on the order of additions, and a draw differs from exact arithmetic only where u falls
// within about 1e-11 of a boundary.
// Thresholds are exact.  A histogram over 2048 equal steps of the distance to the row's maximum (counts for top-k, weights
// for the nucleus) finds the step in which the threshold lies; the few tokens of that step are then ranked among each
// other.  Where a step holds too many different values (logits spread over more than 48 and the threshold far down, or
// infinities), the search goes over the keys' own range instead, 2048 steps at a time.
#include <cfloat>

#include "cascade_internal.h"
#include "paged.h"
#include "ptx.cuh"

namespace {

constexpr int kBins = 2048;                // steps of a histogram; groups of consecutive tokens with a weight sum each
constexpr int kList = 1024;                // tokens of one step that are ranked directly
constexpr float kReach = 48.f;             // how far below the maximum the histogram reaches (its last step takes the rest)

__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);  // larger float <=> larger key
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k); }
constexpr uint32_t kNoKey = 0u;            // -inf and NaN: never kept (the key of -inf would be 0x007fffff)
__device__ __forceinline__ uint32_t logit_key(float x) {
  return x > -INFINITY ? order_key(x + 0.f) : kNoKey;   // + 0: the two zeros are one value
}
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

template <int kThreads>
struct Shared {
  union {
    struct {
      uint32_t lo[kBins], hi[kBins];       // 64-bit sums as two words
    } hist;
    unsigned long long group[kBins];
  };
  unsigned long long list_w[kList];
  uint32_t list_k[kList];
  double table[32];                        // 2^(j/32)
  unsigned long long warp_sum[kThreads / 32];
  uint32_t red_lo[kThreads / 32], red_hi[kThreads / 32];
  unsigned long long before;               // result of find()
  int at;
  int n_list;
  uint32_t list_min, list_max;
  uint32_t floor_key;
  int token;
};

struct SampleArgs {
  const void* logits;
  long long row_stride;
  int V, n_res, fixed_bits, group_shift;   // keys kept in shared memory; log2 of the tokens in a group
  const float* temperature;
  const int32_t* top_k;
  const float *top_p, *min_p, *uniforms;
  int32_t* token;
  float* prob;
  int32_t* kept;
};

// exp((l - m) / T) * 2^bits, rounded to an integer.  x = (l - m) * 32 / (T ln 2) is split into whole octaves, one of 32
// table steps and a remainder |g| <= ln 2 / 64, whose exponential is its Taylor sum to g^4 (error g^5/120 < 2e-12).
struct Weight {
  double m, c;      // row maximum, 32 / (T ln 2)
  uint32_t m_key;
  int bits;
  const double* table;
  __device__ __forceinline__ unsigned long long operator()(uint32_t key) const {
    if (key == m_key) return 1ull << bits;
    const double x = ((double)key_value(key) - m) * c;
    if (!(x > -2048.0)) return 0ull;                         // below 2^-64 (and -inf, NaN of infinite maxima)
    const double magic = 6755399441055744.0;                 // 1.5 * 2^52: rounds to an integer
    const double k = x + magic;
    const int n = __double2loint(k);
    const double g = (x - (k - magic)) * 0.021660849392498290;  // ln 2 / 32
    const double e = 1.0 + g * (1.0 + g * (0.5 + g * (1.0 / 6.0 + g * (1.0 / 24.0))));
    const double w = e * table[n & 31];
    const int exponent = (n >> 5) + bits;                    // w * 2^exponent
    if (exponent < -1) return 0ull;
    const double scaled = __hiloint2double(__double2hiint(w) + (exponent << 20), __double2loint(w));
    return (unsigned long long)__double_as_longlong(scaled + 4503599627370496.0) & 0xfffffffffffffull;  // + 2^52: the integer is in the mantissa
  }
};

__device__ __forceinline__ unsigned long long warp_sum(unsigned long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Adds w to a 64-bit sum kept as two words (native 32-bit atomics; the carry goes with whoever caused it).
template <typename S>
__device__ __forceinline__ void hist_add(S& sh, int bin, unsigned long long w) {
  const uint32_t lo = (uint32_t)w;
  const uint32_t old = atomicAdd(&sh.hist.lo[bin], lo);
  const uint32_t hi = (uint32_t)(w >> 32) + (old + lo < old ? 1u : 0u);
  if (hi != 0u) atomicAdd(&sh.hist.hi[bin], hi);
}

template <typename E>
struct Row {
  const E* g;
  uint32_t* s;         // keys of the first n_res tokens
  int V, n_res;
  __device__ __forceinline__ uint32_t key(int i) const { return i < n_res ? s[i] : logit_key(to_float(g[i])); }
};

// f(index, key) for every token of the row, in strides of the CTA; four independent reads at a time.
template <int kThreads, typename E, typename F>
__device__ __forceinline__ void each(const Row<E>& row, F f) {
  int i = threadIdx.x;
  for (; i + 3 * kThreads < row.V; i += 4 * kThreads) {
    uint32_t k[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) k[q] = row.key(i + q * kThreads);
#pragma unroll
    for (int q = 0; q < 4; ++q) f(i + q * kThreads, k[q]);
  }
  for (; i < row.V; i += kThreads) f(i, row.key(i));
}

// The first entry at which the running sum of kBins entries get(i) passes `target` (> target); sh.at and sh.before = the sum
// in front of it.  target_of(total) is called with the sum of all entries.  sh.at = -1 if the total does not pass it.
template <int kThreads, typename Get, typename Target>
__device__ __forceinline__ unsigned long long find(Shared<kThreads>& sh, Get get, Target target_of) {
  constexpr int kPer = kBins / kThreads;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  unsigned long long v[kPer], sum = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    v[k] = get(threadIdx.x * kPer + k);
    sum += v[k];
  }
  unsigned long long inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long t = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += t;
  }
  if (lane == 31) sh.warp_sum[warp] = inc;
  if (threadIdx.x == 0) sh.at = -1;
  __syncthreads();
  // every warp scans the warps' sums for itself
  unsigned long long w = lane < kThreads / 32 ? sh.warp_sum[lane] : 0ull, winc = w;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long t = __shfl_up_sync(0xffffffffu, winc, o);
    if (lane >= o) winc += t;
  }
  const unsigned long long total = __shfl_sync(0xffffffffu, winc, 31);
  unsigned long long run = __shfl_sync(0xffffffffu, winc - w, warp) + inc - sum;
  const unsigned long long target = target_of(total);
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    if (run <= target && target < run + v[k]) {
      sh.at = threadIdx.x * kPer + k;
      sh.before = run;
    }
    run += v[k];
  }
  __syncthreads();
  return total;
}

// The key x among keys in [lo, hi] with W(> x) <= target < W(>= x), W the weight (1 each, or exp) of keys >= lo: the
// general search, 2048 steps of the keys' range at a time.  The whole CTA calls it with the same arguments.
template <bool kMass, int kThreads, typename E>
__device__ __noinline__ uint32_t descend(const Row<E>& row, const Weight& weight, uint32_t lo, uint32_t hi, unsigned long long target,
                                         Shared<kThreads>& sh) {
  while (true) {
    const uint32_t range = hi - lo;
    const int shift = range < (uint32_t)kBins ? 0 : 32 - __clz(range) - 11;  // (range >> shift) < 2048
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kThreads) sh.hist.lo[i] = sh.hist.hi[i] = 0u;
    __syncthreads();
    each<kThreads>(row, [&](int, uint32_t k) {
      if (k >= lo && k <= hi) {
        const int bin = kBins - 1 - (int)((k - lo) >> shift);   // largest first
        if (kMass)
          hist_add(sh, bin, weight(k));
        else
          atomicAdd(&sh.hist.lo[bin], 1u);
      }
    });
    __syncthreads();
    find<kThreads>(sh, [&](int i) { return ((unsigned long long)sh.hist.hi[i] << 32) | sh.hist.lo[i]; },
                   [&](unsigned long long) { return target; });
    if (sh.at < 0) return lo;                                    // all of it stays
    target -= sh.before;
    lo += (uint32_t)(kBins - 1 - sh.at) << shift;
    if (shift == 0) return lo;
    const uint32_t step_end = lo + ((1u << shift) - 1u);
    if (step_end < hi) hi = step_end;                            // (the last step may pass the row's largest key)
  }
}

// The same threshold by one histogram over the distance to the maximum.  target_of: from the total weight of keys >= floor.
template <bool kMass, int kThreads, typename E, typename Target>
__device__ uint32_t threshold(const Row<E>& row, const Weight& weight, float m, float steps_per_unit, uint32_t floor_key,
                              uint32_t k_max, Target target_of, Shared<kThreads>& sh) {
  const int tid = threadIdx.x;
  auto bin_of = [&](uint32_t k) { return min(kBins - 1, (int)((m - key_value(k)) * steps_per_unit)); };
  __syncthreads();
  for (int i = tid; i < kBins; i += kThreads) sh.hist.lo[i] = sh.hist.hi[i] = 0u;
  if (tid == 0) {
    sh.n_list = 0;
    sh.list_min = 0xffffffffu;
    sh.list_max = 0u;
  }
  __syncthreads();
  each<kThreads>(row, [&](int, uint32_t k) {
    if (k >= floor_key) {
      if (kMass)
        hist_add(sh, bin_of(k), weight(k));
      else
        atomicAdd(&sh.hist.lo[bin_of(k)], 1u);
    }
  });
  __syncthreads();
  unsigned long long target = 0;
  find<kThreads>(sh, [&](int i) { return ((unsigned long long)sh.hist.hi[i] << 32) | sh.hist.lo[i]; },
                 [&](unsigned long long total) { return target = target_of(total); });
  const int bin = sh.at;
  if (bin < 0) return floor_key;                                 // all of it stays
  const unsigned long long left = target - sh.before;            // of the step's own weight
  // the tokens of that step
  uint32_t lo = 0xffffffffu, hi = 0u;
  each<kThreads>(row, [&](int, uint32_t k) {
    if (k >= floor_key && bin_of(k) == bin) {
      const int at = atomicAdd(&sh.n_list, 1);
      if (at < kList) sh.list_k[at] = k;
      lo = min(lo, k);
      hi = max(hi, k);
    }
  });
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if ((tid & 31) == 0 && hi != 0u) {
    atomicMin(&sh.list_min, lo);
    atomicMax(&sh.list_max, hi);
  }
  __syncthreads();
  const int n = sh.n_list;
  lo = sh.list_min;
  hi = sh.list_max;
  if (lo == hi) return lo;                                       // ties
  if (n > kList) return descend<kMass>(row, weight, lo, hi, left, sh);
  if (kMass) {
    for (int i = tid; i < n; i += kThreads) sh.list_w[i] = weight(sh.list_k[i]);
    __syncthreads();
  }
  for (int i = tid; i < n; i += kThreads) {
    const uint32_t k = sh.list_k[i];
    unsigned long long above = 0, with = 0;
    for (int j = 0; j < n; ++j) {
      const unsigned long long w = kMass ? sh.list_w[j] : 1ull;
      above += sh.list_k[j] > k ? w : 0ull;
      with += sh.list_k[j] >= k ? w : 0ull;
    }
    if (above <= left && left < with) sh.floor_key = k;          // exactly one value; its ties agree
  }
  __syncthreads();
  return sh.floor_key;
}

template <typename E, int kThreads>
__global__ void __launch_bounds__(kThreads, 1024 / kThreads) k_sample(const SampleArgs a) {
  constexpr int kWarps = kThreads / 32;
  extern __shared__ __align__(16) uint8_t s_raw[];
  Shared<kThreads>& sh = *reinterpret_cast<Shared<kThreads>*>(s_raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = blockIdx.x;
  Row<E> row;
  row.g = static_cast<const E*>(a.logits) + (long long)r * a.row_stride;
  row.s = reinterpret_cast<uint32_t*>(s_raw + sizeof(Shared<kThreads>));
  row.V = a.V;
  row.n_res = min(a.V, a.n_res);
  if (tid < 32) sh.table[tid] = exp2((double)tid / 32.0);
  // the row's keys, largest and smallest of those that can be kept
  uint32_t k_max = kNoKey, k_min = 0xffffffffu;
  auto take = [&](int i, float x) {
    const uint32_t k = logit_key(x);
    if (i < row.n_res) row.s[i] = k;
    k_max = max(k_max, k);
    k_min = min(k_min, k - 1u);                                  // kNoKey - 1 wraps to the largest
  };
  constexpr int kVec = 16 / sizeof(E);
  int done = 0;
  if ((reinterpret_cast<uintptr_t>(row.g) & 15u) == 0) {
    const uint4* g16 = reinterpret_cast<const uint4*>(row.g);
    const int n16 = a.V / kVec;
    auto take16 = [&](int i, const uint4& v) {
      const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        if (sizeof(E) == 4) {
          take(i * kVec + q, __uint_as_float(w[q]));
        } else {
          take(i * kVec + 2 * q, __uint_as_float(w[q] << 16));
          take(i * kVec + 2 * q + 1, __uint_as_float(w[q] & 0xffff0000u));
        }
      }
    };
    int i = tid;
    for (; i + 3 * kThreads < n16; i += 4 * kThreads) {
      uint4 v[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = __ldg(g16 + i + q * kThreads);
#pragma unroll
      for (int q = 0; q < 4; ++q) take16(i + q * kThreads, v[q]);
    }
    for (; i < n16; i += kThreads) take16(i, __ldg(g16 + i));
    done = n16 * kVec;
  }
  for (int i = done + tid; i < a.V; i += kThreads) take(i, to_float(row.g[i]));
  k_max = __reduce_max_sync(0xffffffffu, k_max);
  k_min = __reduce_min_sync(0xffffffffu, k_min);
  if (lane == 0) {
    sh.red_hi[warp] = k_max;
    sh.red_lo[warp] = k_min;
  }
  if (tid == 0) sh.token = INT_MAX;
  __syncthreads();
  k_max = __reduce_max_sync(0xffffffffu, lane < kWarps ? sh.red_hi[lane] : kNoKey);
  k_min = __reduce_min_sync(0xffffffffu, lane < kWarps ? sh.red_lo[lane] : 0xffffffffu) + 1u;
  if (k_max == kNoKey) {   // nothing to draw from
    if (tid == 0) {
      a.token[r] = -1;
      if (a.prob != nullptr) a.prob[r] = 0.f;
      if (a.kept != nullptr) a.kept[r] = 0;
    }
    return;
  }
  const float T = a.temperature == nullptr ? 1.f : a.temperature[r];
  if (!(T > 0.f)) {        // the most likely token, lowest index first
    int best = INT_MAX;
    each<kThreads>(row, [&](int i, uint32_t k) {
      if (k == k_max) best = min(best, i);
    });
    best = __reduce_min_sync(0xffffffffu, best);
    if (lane == 0 && best != INT_MAX) atomicMin(&sh.token, best);
    __syncthreads();
    if (tid == 0) {
      a.token[r] = sh.token;
      if (a.prob != nullptr) a.prob[r] = 1.f;
      if (a.kept != nullptr) a.kept[r] = 1;
    }
    return;
  }
  const float m = key_value(k_max);
  Weight weight;
  weight.m = (double)m;
  weight.c = 46.166241308446828 / (double)T;   // 32 / ln 2
  weight.m_key = k_max;
  weight.bits = a.fixed_bits;
  weight.table = sh.table;
  uint32_t floor_key = k_min;
  const int top_k = a.top_k == nullptr ? 0 : a.top_k[r];
  const float top_p = a.top_p == nullptr ? 1.f : a.top_p[r];
  const float min_p = a.min_p == nullptr ? 0.f : a.min_p[r];
  const float reach = fminf(m - key_value(k_min), kReach);
  const float steps = (float)(kBins - 1) / reach;
  const bool even = reach > 1e-30f && m < INFINITY;              // the histogram over distances makes sense
  if (top_k > 0 && top_k < a.V) {
    const unsigned long long target = (unsigned long long)top_k - 1ull;
    if (even)
      floor_key = threshold<false>(row, weight, m, steps, floor_key, k_max, [&](unsigned long long) { return target; }, sh);
    else
      floor_key = descend<false>(row, weight, floor_key, k_max, target, sh);
  }
  if (top_p < 1.f) {
    // kept iff W(> x) < top_p z; for whole W: W(> x) <= ceil(top_p z) - 1
    auto target_of = [&](unsigned long long z) {
      const double t = ceil((double)top_p * (double)z);
      return t < 1.0 ? 0ull : (unsigned long long)t - 1ull;
    };
    if (even) {
      floor_key = threshold<true>(row, weight, m, steps, floor_key, k_max, target_of, sh);
    } else {
      unsigned long long z = 0;
      each<kThreads>(row, [&](int, uint32_t k) {
        if (k >= floor_key) z += weight(k);
      });
      z = warp_sum(z);
      __syncthreads();
      if (lane == 0) sh.warp_sum[warp] = z;
      __syncthreads();
      z = warp_sum(lane < kWarps ? sh.warp_sum[lane] : 0ull);
      floor_key = descend<true>(row, weight, floor_key, k_max, target_of(z), sh);
    }
  }
  if (min_p > 0.f) {
    // w >= min_p  <=>  l >= m + T ln(min_p)
    const double bound = weight.m + (double)T * log(min((double)min_p, 1.0));
    const float f = (float)bound;
    uint32_t k = logit_key((double)f >= bound ? f : nextafterf(f, INFINITY));
    if (!(f > -INFINITY)) k = floor_key;
    floor_key = max(floor_key, min(k, k_max));
  }
  // weight sums of groups of consecutive tokens, one warp per group
  const int n_groups = ((a.V - 1) >> a.group_shift) + 1;
  __syncthreads();                                               // the histogram's place becomes the groups'
  for (int i = n_groups + tid; i < kBins; i += kThreads) sh.group[i] = 0ull;
  unsigned int count = 0;
  for (int g = warp; g < n_groups; g += kWarps) {
    unsigned long long sum = 0;
    const int end = min(a.V, (g + 1) << a.group_shift);
    for (int i0 = g << a.group_shift; i0 < end; i0 += 128) {
      uint32_t k[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) k[q] = i0 + 32 * q + lane < end ? row.key(i0 + 32 * q + lane) : kNoKey;
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (k[q] >= floor_key) {                                 // (floor_key is above kNoKey)
          sum += weight(k[q]);
          ++count;
        }
    }
    sum = warp_sum(sum);
    if (lane == 0) sh.group[g] = sum;
  }
  count = __reduce_add_sync(0xffffffffu, count);
  if (lane == 0) sh.red_lo[warp] = count;
  __syncthreads();
  // the group in which the cumulative weight passes u * total (cumulative > u total <=> > floor(u total) for whole sums)
  float u = a.uniforms[r];
  u = u > 0.f ? fminf(u, 1.f - FLT_EPSILON / 2.f) : 0.f;         // NaN and negative: 0
  unsigned long long target = 0;
  const unsigned long long total = find<kThreads>(sh, [&](int i) { return sh.group[i]; }, [&](unsigned long long z) {
    return target = min((unsigned long long)((double)u * (double)z), z - 1ull);
  });
  if (warp != 0) return;
  const uint32_t n_kept = __reduce_add_sync(0xffffffffu, lane < kWarps ? sh.red_lo[lane] : 0u);
  // the token inside it; one warp
  unsigned long long run = sh.before;
  const int g_hit = sh.at, end = min(a.V, (g_hit + 1) << a.group_shift);
  for (int i0 = g_hit << a.group_shift; i0 < end; i0 += 32) {
    const int i = i0 + lane;
    const uint32_t k = i < end ? row.key(i) : kNoKey;
    const unsigned long long w = k >= floor_key ? weight(k) : 0ull;
    unsigned long long c = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned long long t = __shfl_up_sync(0xffffffffu, c, o);
      if (lane >= o) c += t;
    }
    const uint32_t hit = __ballot_sync(0xffffffffu, run + c > target);
    if (hit != 0u) {
      if (lane == __ffs(hit) - 1) {
        a.token[r] = i;
        if (a.prob != nullptr) a.prob[r] = (float)((double)w / (double)total);
        if (a.kept != nullptr) a.kept[r] = (int32_t)n_kept;
      }
      break;
    }
    run += __shfl_sync(0xffffffffu, c, 31);
  }
}

template <typename E, int kThreads>
int launch(cascade_ctx* ctx, SampleArgs& a, int n_rows, cudaStream_t s) {
  // what the row's keys may take: the CTA's share of an SM's 227 KB less its arrays (and 1 KB that the system takes)
  constexpr int kMost = (kThreads == 1024 ? 226 : 112) * 1024 - (int)sizeof(Shared<kThreads>);
  a.n_res = kMost / 4 < a.V ? kMost / 4 : a.V;
  const size_t smem = sizeof(Shared<kThreads>) + (size_t)a.n_res * 4;
  const uint32_t bit = PAGED_CFG_SAMPLE << ((sizeof(E) == 2 ? 2 : 0) + (kThreads == 1024 ? 1 : 0));
  CASCADE_TRY(configure_smem(ctx, bit, k_sample<E, kThreads>, (int)sizeof(Shared<kThreads>) + kMost));
  k_sample<E, kThreads><<<n_rows, kThreads, smem, s>>>(a);
  CASCADE_CUDA_TRY(cudaGetLastError());
  return CASCADE_OK;
}

}  // namespace

extern "C" int cascade_sample(cascade_ctx* ctx, const void* logits, int32_t logits_dtype, int64_t row_stride, int32_t n_rows,
                              const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                              const float* uniforms, int32_t* token_out, float* prob_out, int32_t* kept_out, void* stream) {
  if (ctx == nullptr || logits == nullptr || uniforms == nullptr || token_out == nullptr) return CASCADE_ERR_INVALID_ARG;
  if (logits_dtype != CASCADE_F32 && logits_dtype != CASCADE_BF16) return CASCADE_ERR_INVALID_ARG;
  const int V = ctx->shape.V;
  if (n_rows < 1 || row_stride < V) return CASCADE_ERR_INVALID_ARG;
  const bool bf16 = logits_dtype == CASCADE_BF16;
  if ((reinterpret_cast<uintptr_t>(logits) & (bf16 ? 1u : 3u)) != 0) return CASCADE_ERR_INVALID_ARG;
  CASCADE_TRY(check_current_device(ctx));
  SampleArgs a;
  a.logits = logits;
  a.row_stride = row_stride;
  a.V = V;
  int log_v = 0;
  while ((1ll << log_v) < V) ++log_v;
  a.fixed_bits = 62 - log_v < 50 ? 62 - log_v : 50;   // V weights of at most 1 stay below 2^62; one weight below 2^52
  a.group_shift = 7;
  while (((V - 1) >> a.group_shift) + 1 > kBins) ++a.group_shift;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.uniforms = uniforms;
  a.token = token_out;
  a.prob = prob_out;
  a.kept = kept_out;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  ctx->launches = 0;
  KernelScope ks(ctx, K_SAMPLE, s);
  const bool many = n_rows > ctx->sm_count;
  if (bf16) return many ? launch<__nv_bfloat16, 512>(ctx, a, n_rows, s) : launch<__nv_bfloat16, 1024>(ctx, a, n_rows, s);
  return many ? launch<float, 512>(ctx, a, n_rows, s) : launch<float, 1024>(ctx, a, n_rows, s);
}
