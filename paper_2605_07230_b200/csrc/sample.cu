// One token per row of logits from a given uniform number, after temperature, top-k, nucleus and min-p.
//
//   w[v] = exp((l[v] - m) / T),  token = first v whose cumulative kept weight exceeds u * (total kept weight)
//
// One CTA per row.  The row's order-preserving 32-bit keys stay in shared memory (what does not fit is read again from
// memory), so HBM sees each logit once.  Weights are formed in 64 bits (relative error 1e-12) and summed as 64-bit fixed
// point: sums do not depend on the order of additions, and a draw differs from exact arithmetic only where u falls
// within about 1e-11 of a boundary.  Thresholds are exact: a histogram over the range of keys still in question, 2048
// equal steps of the key at a time, until a step holds a single key value.
#include <cfloat>

#include "cascade_internal.h"
#include "paged.h"
#include "ptx.cuh"

namespace {

constexpr int kThreads = 1024;
constexpr int kWarps = kThreads / 32;
constexpr int kBins = 2048;
constexpr int kMaxGroups = 2048;           // groups of consecutive tokens with a weight sum each
constexpr int kResident = 48 * 1024;       // keys kept in shared memory

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

struct Shared {
  unsigned long long hist[kBins];
  unsigned long long group[kMaxGroups];
  unsigned long long red[kWarps];
  double table[32];                        // 2^(j/32)
  uint32_t red_lo[kWarps], red_hi[kWarps];
  unsigned long long above;
  int bin;
  int token;
};

struct SampleArgs {
  const void* logits;
  long long row_stride;
  int V, fixed_bits, group_shift;          // group_shift: log2 of the tokens in a group
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
__device__ unsigned long long block_sum(unsigned long long v, Shared& sh) {
  v = warp_sum(v);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) sh.red[threadIdx.x >> 5] = v;
  __syncthreads();
  unsigned long long t = 0;
  for (int i = 0; i < kWarps; ++i) t += sh.red[i];
  return t;
}

template <typename E>
struct Row {
  const E* g;
  const uint32_t* s;   // keys of the first n_res tokens
  int V, n_res;
  __device__ __forceinline__ uint32_t key(int i) const { return i < n_res ? s[i] : logit_key(to_float(g[i])); }
};

// The key x among keys in [lo, hi] with W(> x) < target <= W(>= x), W the weight (1 each, or exp) of keys >= lo; the
// whole CTA calls it with the same arguments.  Every pass narrows [lo, hi] to one of 2048 steps.
template <bool kMass, typename E>
__device__ uint32_t descend(const Row<E>& row, const Weight& weight, uint32_t lo, uint32_t hi, unsigned long long target,
                            Shared& sh) {
  unsigned long long above = 0;
  while (true) {
    const uint32_t range = hi - lo;
    const int shift = range < (uint32_t)kBins ? 0 : 32 - __clz(range) - 11;  // (range >> shift) < 2048
    __syncthreads();
    for (int i = threadIdx.x; i < kBins; i += kThreads) sh.hist[i] = 0ull;
    __syncthreads();
    for (int i = threadIdx.x; i < row.V; i += kThreads) {
      const uint32_t k = row.key(i);
      if (k >= lo && k <= hi) atomicAdd(&sh.hist[(k - lo) >> shift], kMass ? weight(k) : 1ull);
    }
    __syncthreads();
    if (threadIdx.x < 32) {
      const int lane = threadIdx.x;
      // lane L owns the 64 bins 2047 - 64 L ... , largest first
      unsigned long long sum = 0;
      for (int i = 0; i < 64; ++i) sum += sh.hist[kBins - 1 - 64 * lane - i];
      unsigned long long inc = sum;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long t = __shfl_up_sync(0xffffffffu, inc, o);
        if (lane >= o) inc += t;
      }
      const unsigned long long exc = inc - sum;
      const bool mine = above + exc < target && target <= above + inc;
      const uint32_t who = __ballot_sync(0xffffffffu, mine);
      if (who == 0u) {
        if (lane == 0) sh.bin = -1;   // the target lies beyond everything: all of it stays
      } else if (mine) {
        unsigned long long run = above + exc;
        for (int i = 0; i < 64; ++i) {
          const int b = kBins - 1 - 64 * lane - i;
          if (run + sh.hist[b] >= target) {
            sh.bin = b;
            break;
          }
          run += sh.hist[b];
        }
        sh.above = run;
      }
    }
    __syncthreads();
    const int bin = sh.bin;
    if (bin < 0) return lo;
    above = sh.above;
    lo += (uint32_t)bin << shift;
    if (shift == 0) return lo;
    const uint32_t step_end = lo + ((1u << shift) - 1u);
    if (step_end < hi) hi = step_end;   // (the last step may pass the row's largest key)
  }
}

template <typename E>
__global__ void __launch_bounds__(kThreads) k_sample(const SampleArgs a) {
  extern __shared__ uint32_t s_keys[];
  __shared__ Shared sh;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, r = blockIdx.x;
  Row<E> row;
  row.g = static_cast<const E*>(a.logits) + (long long)r * a.row_stride;
  row.s = s_keys;
  row.V = a.V;
  row.n_res = min(a.V, kResident);
  if (tid < 32) sh.table[tid] = exp2((double)tid / 32.0);
  // the row's keys, largest and smallest of those that can be kept
  uint32_t k_max = kNoKey, k_min = 0xffffffffu;
  for (int i = tid; i < a.V; i += kThreads) {
    const uint32_t k = logit_key(to_float(row.g[i]));
    if (i < row.n_res) s_keys[i] = k;
    k_max = max(k_max, k);
    if (k != kNoKey) k_min = min(k_min, k);
  }
  k_max = __reduce_max_sync(0xffffffffu, k_max);
  k_min = __reduce_min_sync(0xffffffffu, k_min);
  if (lane == 0) {
    sh.red_hi[warp] = k_max;
    sh.red_lo[warp] = k_min;
  }
  if (tid == 0) sh.token = INT_MAX;
  __syncthreads();
  for (int i = 0; i < kWarps; ++i) {
    k_max = max(k_max, sh.red_hi[i]);
    k_min = min(k_min, sh.red_lo[i]);
  }
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
    for (int i = tid; i < a.V; i += kThreads)
      if (row.key(i) == k_max) best = min(best, i);
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
  Weight weight;
  weight.m = (double)key_value(k_max);
  weight.c = 46.166241308446828 / (double)T;   // 32 / ln 2
  weight.m_key = k_max;
  weight.bits = a.fixed_bits;
  weight.table = sh.table;
  uint32_t floor_key = k_min;
  const int top_k = a.top_k == nullptr ? 0 : a.top_k[r];
  const float top_p = a.top_p == nullptr ? 1.f : a.top_p[r];
  const float min_p = a.min_p == nullptr ? 0.f : a.min_p[r];
  if (top_k > 0 && top_k < a.V) floor_key = descend<false>(row, weight, floor_key, k_max, (unsigned long long)top_k, sh);
  if (top_p < 1.f) {
    unsigned long long z = 0;
    for (int i = tid; i < a.V; i += kThreads) {
      const uint32_t k = row.key(i);
      if (k >= floor_key) z += weight(k);
    }
    z = block_sum(z, sh);
    // W(> x) < top_p z for whole W: target = ceil(top_p z), at least 1
    const double t = ceil((double)top_p * (double)z);
    const unsigned long long target = t < 1.0 ? 1ull : (unsigned long long)t;
    floor_key = descend<true>(row, weight, floor_key, k_max, target, sh);
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
  unsigned int count = 0;
  for (int g = warp; g < n_groups; g += kWarps) {
    unsigned long long sum = 0;
    const int end = min(a.V, (g + 1) << a.group_shift);
    for (int i = (g << a.group_shift) + lane; i < end; i += 32) {
      const uint32_t k = row.key(i);
      if (k != kNoKey && k >= floor_key) {
        sum += weight(k);
        ++count;
      }
    }
    sum = warp_sum(sum);
    if (lane == 0) sh.group[g] = sum;
  }
  const unsigned long long n_kept = block_sum(count, sh);   // also a barrier behind the group sums
  if (warp != 0) return;
  // the group in which the cumulative weight passes u * total, then the token inside it; one warp
  const int per = (n_groups + 31) / 32, g0 = min(n_groups, lane * per), g1 = min(n_groups, g0 + per);
  unsigned long long sum = 0;
  for (int g = g0; g < g1; ++g) sum += sh.group[g];
  unsigned long long inc = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long t = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += t;
  }
  const unsigned long long total = __shfl_sync(0xffffffffu, inc, 31);
  float u = a.uniforms[r];
  u = u > 0.f ? fminf(u, 1.f - FLT_EPSILON / 2.f) : 0.f;   // NaN and negative: 0
  // cumulative > u * total  <=>  cumulative > floor(u * total) for whole sums
  const unsigned long long target = min((unsigned long long)((double)u * (double)total), total - 1ull);
  const uint32_t past = __ballot_sync(0xffffffffu, inc > target);
  const int owner = __ffs(past) - 1;
  int g_hit = 0;
  unsigned long long run = 0;
  if (lane == owner) {
    run = inc - sum;
    for (g_hit = g0; g_hit < g1 - 1; ++g_hit) {
      if (run + sh.group[g_hit] > target) break;
      run += sh.group[g_hit];
    }
  }
  g_hit = __shfl_sync(0xffffffffu, g_hit, owner);
  run = __shfl_sync(0xffffffffu, run, owner);
  const int end = min(a.V, (g_hit + 1) << a.group_shift);
  for (int i0 = g_hit << a.group_shift; i0 < end; i0 += 32) {
    const int i = i0 + lane;
    const uint32_t k = i < end ? row.key(i) : kNoKey;
    const unsigned long long w = k != kNoKey && k >= floor_key ? weight(k) : 0ull;
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
  while (((V - 1) >> a.group_shift) + 1 > kMaxGroups) ++a.group_shift;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.uniforms = uniforms;
  a.token = token_out;
  a.prob = prob_out;
  a.kept = kept_out;
  const size_t smem = (size_t)(V < kResident ? V : kResident) * 4;
  cudaStream_t s = static_cast<cudaStream_t>(stream);
  if (smem > 8 * 1024) {
    const int most = kResident * 4;
    if (bf16)
      CASCADE_CUDA_TRY(cudaFuncSetAttribute(k_sample<__nv_bfloat16>, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
    else
      CASCADE_CUDA_TRY(cudaFuncSetAttribute(k_sample<float>, cudaFuncAttributeMaxDynamicSharedMemorySize, most));
  }
  ctx->launches = 0;
  {
    KernelScope ks(ctx, K_SAMPLE, s);
    if (bf16)
      k_sample<__nv_bfloat16><<<n_rows, kThreads, smem, s>>>(a);
    else
      k_sample<float><<<n_rows, kThreads, smem, s>>>(a);
  }
  CASCADE_CUDA_TRY(cudaGetLastError());
  return CASCADE_OK;
}
