// One token per row of logits from a given uniform number, after temperature, top-k, nucleus and min-p.
//
//   w[v] = exp((l[v] - m) / T),  token = first v whose cumulative kept weight exceeds u * (total kept weight)
//
// One CTA per row.  The row stays in shared memory as far as it fits (the rest is read again through the L2), so HBM sees
// each logit once.  Weights are formed in 64 bits (relative error 1e-10), rounded to multiples of 2^-b of the largest one,
// b = min(50, 62 - log2 V), log2 rounded up, and summed in 64-bit fixed point: sums do not depend on the order of additions.
// V roundings of at most half a unit each leave a sum within V 2^-(b+1) + 1e-10 of it (largest weight 1): 1.3e-10 for V = 16384,
// 5.7e-10 for 65536, 3.8e-9 for 131080, 1.2e-7 for 2^20, all of it only where most tokens weigh about half a unit.  A draw, and
// where the nucleus ends, differ from exact arithmetic only where u or top_p falls that close to a boundary.
// For the rounded weights thresholds are exact.  A histogram over 2048 equal steps of the distance to the row's maximum (counts
// for top-k, weights for the nucleus) finds the step in which the threshold lies; the few tokens of that step are then ranked
// among each other.  Where a step holds too many different values (logits spread over more than 48 and the threshold far down, or
// infinities), the search goes over the range of the values' ordered bit patterns instead, 2048 steps at a time.
// Once a truncation has left at most 4096 tokens, they are gathered and the later passes go over them alone.
// Bound by the instructions of two to four passes over the row: 148 rows of 65536 take 6 us for the most likely token (HBM),
// 24 to 31 us with top-k, 30 us without truncation, 51 us for a nucleus of 0.9; 488 rows with mixed settings 123 us; two rows
// of 16384, where the passes' latencies add up, 13.5 us (graph replays; 15.2 called one by one).
#include <cfloat>

#include "cascade_internal.h"
#include "paged.h"
#include "ptx.cuh"

namespace {

constexpr int kThreads = 1024;             // one CTA an SM: two of 512 took 186 us where this takes 164 (488 rows of 65536)
constexpr int kBins = 2048;                // steps of a histogram; groups of consecutive tokens with a weight sum each
constexpr int kList = 4096;                // kept tokens that are gathered
constexpr int kMaxSorted = 4096;           // rows that are handed out by expected work
static_assert(kThreads / 32 == 32, "one lane a warp in the scans of the warps' sums");
constexpr int kRank = 1024;                // tokens of one step that are ranked directly
constexpr float kReach = 48.f;             // how far below the maximum the histogram reaches (its last step takes the rest)

__device__ __forceinline__ uint32_t order_key(float x) {
  const uint32_t u = __float_as_uint(x);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);  // larger float <=> larger key
}
__device__ __forceinline__ float key_value(uint32_t k) { return __uint_as_float((k & 0x80000000u) ? (k & 0x7fffffffu) : ~k); }

struct alignas(16) Shared {                // (the row's logits follow it and are read 16 bytes at a time)
  union {
    struct {
      uint32_t lo[kBins], hi[kBins];       // 64-bit sums as two words
    } hist;
    unsigned long long group[kBins];
  };
  float list_l[kList];                     // gathered tokens: logit, index
  int list_i[kList];
  unsigned long long rank_w[kRank];        // tokens of one step: weight, logit, index
  float rank_l[kRank];
  int rank_i[kRank];
  double table[64];                        // 2^(j/64)
  unsigned long long warp_sum[kThreads / 32];
  float red_lo[kThreads / 32], red_hi[kThreads / 32];
  uint32_t red_n[kThreads / 32];
  unsigned long long before;               // result of find()
  int at;
  int n_list, n_rank;
  uint32_t key_min, key_max;               // of one step
  float floor;
  int token;
};

struct SampleArgs {
  const void* logits;
  long long row_stride;
  int n_rows, sorted;  // sorted: a block takes the row of its rank by expected work
  int V, n_res, fixed_bits, group_shift;   // logits kept in shared memory; log2 of the tokens in a group
  const float* temperature;
  const int32_t* top_k;
  const float *top_p, *min_p, *uniforms;
  int32_t* token;
  float* prob;
  int32_t* kept;
};

// exp((l - m) / T) * 2^bits, rounded to an integer, for l >= zero.  x = (l - m) * 64 / (T ln 2) is split into whole octaves,
// one of 64 table steps and a remainder |g| <= 1/2 of a step, whose exponential is its Taylor sum to the third power (error
// (ln 2 / 128)^4 / 24 < 4e-11).  The last product adds 2^52, which leaves the rounded integer in the mantissa.
struct Weight {
  float m, zero;    // row maximum; logits below weigh nothing
  double md, c;     // the maximum, 64 / (T ln 2)
  int bits;
  const double* table;
  __device__ __forceinline__ unsigned long long of(float l) const {
    constexpr double a1 = 0.010830424696249146, a2 = a1 * a1 / 2, a3 = a1 * a1 * a1 / 6;   // ln 2 / 64
    const double magic = 6755399441055744.0;                     // 1.5 * 2^52: rounds to an integer
    const double x = ((double)l - md) * c, k = x + magic;
    const int n = __double2loint(k);
    const double g = x - (k - magic);
    const double e = fma(g, fma(g, fma(g, a3, a2), a1), 1.0);
    const double t = table[n & 63];
    const double scaled = __hiloint2double(__double2hiint(t) + (((n >> 6) + bits) << 20), __double2loint(t));
    const unsigned long long w = (unsigned long long)__double_as_longlong(fma(e, scaled, 4503599627370496.0)) & 0xfffffffffffffull;
    return l == m ? 1ull << bits : w;                            // (the maximum may be infinite)
  }
  __device__ __forceinline__ unsigned long long operator()(float l) const { return l >= zero ? of(l) : 0ull; }
};

__device__ __forceinline__ unsigned long long warp_sum(unsigned long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}

// Adds w to a 64-bit sum kept as two words (native 32-bit atomics; the carry goes with whoever caused it).
__device__ __forceinline__ void add_pair(uint32_t* lo_word, uint32_t* hi_word, unsigned long long w) {
  const uint32_t lo = (uint32_t)w;
  const uint32_t old = atomicAdd(lo_word, lo);
  const uint32_t hi = (uint32_t)(w >> 32) + (old + lo < old ? 1u : 0u);
  if (hi != 0u) atomicAdd(hi_word, hi);
}

template <typename E>
struct Row {
  const E* g;
  float* s;            // the first n_res logits (a multiple of 4)
  int V, n_res;
  bool wide;           // four logits can be read at once
  __device__ __forceinline__ float at(int i) const {
    if (i < n_res) return s[i];
    if constexpr (sizeof(E) == 4)
      return g[i];
    else
      return __bfloat162float(g[i]);
  }
  __device__ __forceinline__ float4 from_memory(int i4) const {
    if constexpr (sizeof(E) == 4) {
      if (wide) return __ldg(reinterpret_cast<const float4*>(g) + i4);
      return make_float4(g[4 * i4], g[4 * i4 + 1], g[4 * i4 + 2], g[4 * i4 + 3]);
    } else {
      uint2 u;
      if (wide) {
        u = __ldg(reinterpret_cast<const uint2*>(g) + i4);
      } else {
        const unsigned short* h = reinterpret_cast<const unsigned short*>(g) + 4 * i4;
        u = make_uint2(h[0] | ((uint32_t)h[1] << 16), h[2] | ((uint32_t)h[3] << 16));
      }
      return make_float4(__uint_as_float(u.x << 16), __uint_as_float(u.x & 0xffff0000u), __uint_as_float(u.y << 16),
                         __uint_as_float(u.y & 0xffff0000u));
    }
  }
  __device__ __forceinline__ float4 four(int i4) const { return 4 * i4 < n_res ? reinterpret_cast<const float4*>(s)[i4] : from_memory(i4); }
};

// f(index, logit) for every token of the row, four at a time (V is a multiple of 8).
template <typename E, typename F>
__device__ __forceinline__ void each(const Row<E>& row, F f) {
  const int n4 = row.V / 4;
  auto take = [&](int i, const float4& v) {
    f(4 * i, v.x);
    f(4 * i + 1, v.y);
    f(4 * i + 2, v.z);
    f(4 * i + 3, v.w);
  };
  int i = threadIdx.x;
  for (; i + kThreads < n4; i += 2 * kThreads) {
    const float4 a = row.four(i), b = row.four(i + kThreads);
    take(i, a);
    take(i + kThreads, b);
  }
  if (i < n4) take(i, row.four(i));
}

// The tokens still in play: the gathered ones, or those of the row from `floor` up.
template <typename E, typename F>
__device__ __forceinline__ void each_kept(const Row<E>& row, const Shared& sh, bool gathered, float floor, F f) {
  if (gathered) {
    for (int i = threadIdx.x; i < sh.n_list; i += kThreads)
      if (sh.list_l[i] >= floor) f(sh.list_i[i], sh.list_l[i]);
  } else {
    each(row, [&](int i, float l) {
      if (l >= floor) f(i, l);
    });
  }
}

// The first entry at which the running sum of kBins entries get(i) passes `target` (> target); sh.at and sh.before = the sum
// in front of it.  target_of(total) is called with the sum of all entries.  sh.at = -1 if the total does not pass it.
template <typename Get, typename Target>
__device__ __forceinline__ unsigned long long find(Shared& sh, Get get, Target target_of) {
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

__device__ __forceinline__ void clear_hist(Shared& sh) {
  __syncthreads();
  for (int i = threadIdx.x; i < kBins; i += kThreads) sh.hist.lo[i] = sh.hist.hi[i] = 0u;
  __syncthreads();
}

// The value x among keys in [lo, hi] with W(> x) <= target < W(>= x), W the weight (1 each, or exp) of the tokens in play
// with a key >= lo: the general search, 2048 steps of the keys' range at a time.  The whole CTA calls it.
template <bool kMass, typename E>
__device__ __noinline__ float descend(const Row<E>& row, const Weight& weight, bool gathered, uint32_t lo, uint32_t hi,
                                      unsigned long long target, Shared& sh) {
  while (true) {
    const uint32_t range = hi - lo;
    const int shift = range < (uint32_t)kBins ? 0 : 32 - __clz(range) - 11;  // (range >> shift) < 2048
    clear_hist(sh);
    each_kept(row, sh, gathered, key_value(lo), [&](int, float l) {
      const uint32_t k = order_key(l + 0.f);                     // + 0: the two zeros are one value
      if (k >= lo && k <= hi) {
        const int bin = kBins - 1 - (int)((k - lo) >> shift);   // largest first
        if (kMass)
          add_pair(&sh.hist.lo[bin], &sh.hist.hi[bin], weight(l));
        else
          atomicAdd(&sh.hist.lo[bin], 1u);
      }
    });
    __syncthreads();
    find(sh, [&](int i) { return ((unsigned long long)sh.hist.hi[i] << 32) | sh.hist.lo[i]; },
                   [&](unsigned long long) { return target; });
    if (sh.at < 0) return key_value(lo);                         // all of it stays
    target -= sh.before;
    lo += (uint32_t)(kBins - 1 - sh.at) << shift;
    if (shift == 0) return key_value(lo);
    const uint32_t step_end = lo + ((1u << shift) - 1u);
    if (step_end < hi) hi = step_end;                            // (the last step may pass the row's largest key)
  }
}

// kept iff W(> x) < top_p z; for whole W: W(> x) <= ceil(top_p z) - 1
__device__ __forceinline__ unsigned long long nucleus_target(float top_p, unsigned long long z) {
  const double t = ceil((double)top_p * (double)z);
  return t < 1.0 ? 0ull : (unsigned long long)t - 1ull;
}

// *floor = l if the threshold is l: W(> l) <= left < W(>= l) among n values (w: their weights, null: 1 each).  That holds for
// exactly one value, or for none; its ties agree.
__device__ __forceinline__ void rank(const float* values, const unsigned long long* w, int n, float l, unsigned long long left,
                                     float* floor) {
  unsigned long long over = 0, with = 0;
  for (int j = 0; j < n; ++j) {
    const unsigned long long x = w == nullptr ? 1ull : w[j];
    over += values[j] > l ? x : 0ull;
    with += values[j] >= l ? x : 0ull;
  }
  if (over <= left && left < with) *floor = l;
}

// The same threshold, over the tokens in play from `floor` up, by one histogram over the distance to the maximum; `even`:
// that makes sense.  target_of: from the total weight.  Leaves what stays gathered (*gathered) if it is few enough.
// clean: the histogram, its counters and (unless gathered) the list are empty.
template <bool kMass, typename E, typename Target>
__device__ __forceinline__ float threshold(const Row<E>& row, const Weight& weight, bool* gathered, float floor, bool even,
                                           float steps, Target target_of, bool clean, Shared& sh) {
  const int tid = threadIdx.x;
  auto bin_of = [&](float l) { return min(kBins - 1, (int)((weight.m - l) * steps)); };
  auto bins = [&](int i) { return ((unsigned long long)sh.hist.hi[i] << 32) | sh.hist.lo[i]; };
  unsigned long long target = 0;
  if (!even) {
    unsigned long long z = 0;
    if (kMass) {
      each_kept(row, sh, *gathered, floor, [&](int, float l) { z += weight(l); });
      z = warp_sum(z);
      __syncthreads();
      if ((tid & 31) == 0) sh.warp_sum[tid >> 5] = z;
      __syncthreads();
      z = warp_sum((tid & 31) < kThreads / 32 ? sh.warp_sum[tid & 31] : 0ull);
    }
    return descend<kMass>(row, weight, *gathered, order_key(floor + 0.f), order_key(weight.m + 0.f), target_of(z), sh);
  }
  if (!clean) {
    if (tid == 0) {
      sh.n_rank = 0;
      sh.key_min = 0xffffffffu;
      sh.key_max = 0u;
      if (!*gathered) sh.n_list = 0;
    }
    clear_hist(sh);
  }
  each_kept(row, sh, *gathered, floor, [&](int, float l) {
    if (kMass) {
      if (l >= weight.zero) {
        const int bin = bin_of(l);
        add_pair(&sh.hist.lo[bin], &sh.hist.hi[bin], weight.of(l));
      }
    } else {
      atomicAdd(&sh.hist.lo[bin_of(l)], 1u);
    }
  });
  __syncthreads();
  find(sh, bins, [&](unsigned long long total) { return target = target_of(total); });
  const int bin = sh.at;
  if (bin < 0) return floor;                                     // all of it stays
  const unsigned long long left = target - sh.before;            // of the step's own weight
  // the tokens of that step; those above it are gathered unless everything in play is already
  uint32_t lo = 0xffffffffu, hi = 0u;
  const bool gather = !*gathered;
  each_kept(row, sh, *gathered, floor, [&](int i, float l) {
    const int b = bin_of(l);
    if (b < bin) {
      if (gather) {
        const int at = atomicAdd(&sh.n_list, 1);
        if (at < kList) {
          sh.list_l[at] = l;
          sh.list_i[at] = i;
        }
      }
    } else if (b == bin) {
      const int at = atomicAdd(&sh.n_rank, 1);
      if (at < kRank) {
        sh.rank_l[at] = l;
        sh.rank_i[at] = i;
      }
      const uint32_t k = order_key(l + 0.f);
      lo = min(lo, k);
      hi = max(hi, k);
    }
  });
  lo = __reduce_min_sync(0xffffffffu, lo);
  hi = __reduce_max_sync(0xffffffffu, hi);
  if ((tid & 31) == 0 && hi != 0u) {
    atomicMin(&sh.key_min, lo);
    atomicMax(&sh.key_max, hi);
  }
  __syncthreads();
  const int n = sh.n_rank, above = sh.n_list;
  lo = sh.key_min;
  hi = sh.key_max;
  if (n > kRank) {
    if (lo == hi) return key_value(lo);                          // ties
    return descend<kMass>(row, weight, *gathered, lo, hi, left, sh);
  }
  if (lo == hi) {
    floor = key_value(lo);
    __syncthreads();                                             // (n_list has been read by everybody)
  } else {
    if (kMass) {
      for (int i = tid; i < n; i += kThreads) sh.rank_w[i] = weight(sh.rank_l[i]);
      __syncthreads();
    }
    for (int i = tid; i < n; i += kThreads) rank(sh.rank_l, kMass ? sh.rank_w : nullptr, n, sh.rank_l[i], left, &sh.floor);
    __syncthreads();
    floor = sh.floor;
  }
  if (gather && above + n <= kList) {
    for (int i = tid; i < n; i += kThreads)
      if (sh.rank_l[i] >= floor) {
        const int at = atomicAdd(&sh.n_list, 1);
        sh.list_l[at] = sh.rank_l[i];
        sh.list_i[at] = sh.rank_i[i];
      }
    *gathered = true;
    __syncthreads();
  }
  return floor;
}

// The nucleus without a gathered list, in one pass over the weights: a histogram of counts and of the places inside the steps
// estimates each step's weight to about 1e-4 of itself, which leaves a band of few steps around the threshold.  The pass over
// the exact weights then sums all tokens, those above the band and their groups, and gathers the band, whose tokens are
// ranked among each other.  That the exact threshold lies in the band is checked with the exact sums: false where it does
// not, or where the band is too full, and then the groups' sums and *count mean nothing.  least: tokens below it are not
// drawn (min-p), though they count for the nucleus.
template <typename E>
__device__ __forceinline__ bool nucleus(const Row<E>& row, const Weight& weight, const SampleArgs& a, float* floor, float least,
                                        float top_p, float T, float steps, int n_groups, uint32_t* count, bool clean, Shared& sh) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const float from = *floor;
  if (!clean) {
    if (tid == 0) sh.n_list = 0;
    clear_hist(sh);
  }
  each_kept(row, sh, false, from, [&](int, float l) {
    const float d = (weight.m - l) * steps;
    const int bin = min(kBins - 1, (int)d);
    atomicAdd(&sh.hist.lo[bin], 1u);
    atomicAdd(&sh.hist.hi[bin], (uint32_t)fminf((d - (float)bin) * 256.f, 255.f));
  });
  __syncthreads();
  const float step = 1.f / (steps * T), per_step = 1.4426950f * step;   // nats, octaves
  auto mass = [&](int i) {
    const float n = (float)sh.hist.lo[i];
    if (n == 0.f) return 0ull;
    const float place = ((float)sh.hist.hi[i] / n + 0.5f) * (1.f / 256.f);
    return (unsigned long long)(n * exp2f(32.f - ((float)i + place) * per_step));
  };
  // a step's estimate is off by step^2 / 24 (its weights are not all the mean place's), by step / 512 (the places' steps) and
  // by what float rounds; taken a few times over
  const float slack = 0.1f * step * step + 0.01f * step + 1e-5f;
  find(sh, mass, [&](unsigned long long z) { return (unsigned long long)(fmaxf(top_p - slack, 0.f) * (double)z); });
  const int first = sh.at;
  __syncthreads();
  find(sh, mass, [&](unsigned long long z) { return (unsigned long long)((double)(top_p + slack) * (double)z); });
  const int last = sh.at < 0 ? kBins - 1 : sh.at;
  __syncthreads();                                               // the histogram's place becomes the groups'
  for (int i = n_groups + tid; i < kBins; i += kThreads) sh.group[i] = 0ull;
  unsigned long long all = 0, above = 0;
  for (int g = warp; g < n_groups; g += kThreads / 32) {
    unsigned long long sum = 0;
    const int end = min(a.V, (g + 1) << a.group_shift) / 4;
    for (int i = ((g << a.group_shift) >> 2) + lane; i < end; i += 32) {
      const float4 v = row.four(i);
      const float l[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (l[q] >= from) {
          const unsigned long long w = weight(l[q]);
          const int bin = min(kBins - 1, (int)((weight.m - l[q]) * steps));
          all += w;
          if (bin < first) {
            above += w;
            if (l[q] >= least) {
              sum += w;
              ++*count;
            }
          } else if (bin <= last) {
            const int at = atomicAdd(&sh.n_list, 1);
            if (at < kRank) {
              sh.list_l[at] = l[q];
              sh.list_i[at] = 4 * i + q;
            }
          }
        }
    }
    sum = warp_sum(sum);
    if (lane == 0) sh.group[g] = sum;
  }
  all = warp_sum(all);
  above = warp_sum(above);
  if (lane == 0) {
    sh.warp_sum[warp] = all;
    sh.rank_w[warp] = above;
  }
  if (tid == 0) sh.floor = NAN;
  __syncthreads();
  all = warp_sum(sh.warp_sum[lane]);
  above = warp_sum(sh.rank_w[lane]);
  const int n = sh.n_list;
  __syncthreads();
  const unsigned long long target = nucleus_target(top_p, all);
  if (first < 0 || n > kRank || above > target) return false;
  const unsigned long long left = target - above;
  for (int i = tid; i < n; i += kThreads) sh.rank_w[i] = weight(sh.list_l[i]);
  __syncthreads();
  for (int i = tid; i < n; i += kThreads) rank(sh.list_l, sh.rank_w, n, sh.list_l[i], left, &sh.floor);
  __syncthreads();
  const float x = sh.floor;
  if (!(x == x)) return false;
  *floor = fmaxf(x, least);
  for (int i = tid; i < n; i += kThreads)
    if (sh.list_l[i] >= *floor) {
      uint32_t* word = reinterpret_cast<uint32_t*>(&sh.group[sh.list_i[i] >> a.group_shift]);
      add_pair(word, word + 1, sh.rank_w[i]);
      ++*count;
    }
  return true;
}

// The row with rank `rank` when rows of a nucleus alone (51 us for 65536 tokens) come first, then the others (24 to 34 us),
// then those that only want the most likely token (6 us); in index order otherwise.  Every block finds its own row.
__device__ __forceinline__ int row_of_rank(const SampleArgs& a, int rank, Shared& sh) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int per = (a.n_rows + kThreads - 1) / kThreads;
  auto cheapness = [&](int r) {
    if (a.temperature != nullptr && !(a.temperature[r] > 0.f)) return 2;
    const int k = a.top_k == nullptr ? 0 : a.top_k[r];
    return a.top_p != nullptr && a.top_p[r] < 1.f && !(k > 0 && k < a.V) ? 0 : 1;
  };
  int kind[kMaxSorted / kThreads];
  uint32_t mine = 0;                                             // first kind below, second in the upper half
#pragma unroll
  for (int k = 0; k < kMaxSorted / kThreads; ++k) {
    const int r = tid * per + k;
    kind[k] = k < per && r < a.n_rows ? cheapness(r) : 3;
    mine += kind[k] == 0 ? 1u : (kind[k] == 1 ? 0x10000u : 0u);
  }
  uint32_t inc = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t t = __shfl_up_sync(0xffffffffu, inc, o);
    if (lane >= o) inc += t;
  }
  if (lane == 31) sh.red_n[warp] = inc;
  __syncthreads();
  uint32_t w = sh.red_n[lane], winc = w;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint32_t t = __shfl_up_sync(0xffffffffu, winc, o);
    if (lane >= o) winc += t;
  }
  const uint32_t total = __shfl_sync(0xffffffffu, winc, 31);
  uint32_t run = __shfl_sync(0xffffffffu, winc - w, warp) + inc - mine;
  const int n0 = (int)(total & 0xffffu), n1 = (int)(total >> 16);
#pragma unroll
  for (int k = 0; k < kMaxSorted / kThreads; ++k) {
    const int r = tid * per + k, b0 = (int)(run & 0xffffu), b1 = (int)(run >> 16);
    const int at = kind[k] == 0 ? b0 : (kind[k] == 1 ? n0 + b1 : n0 + n1 + r - b0 - b1);
    if (kind[k] < 3 && at == rank) sh.token = r;
    run += kind[k] == 0 ? 1u : (kind[k] == 1 ? 0x10000u : 0u);
  }
  __syncthreads();
  const int r = sh.token;
  __syncthreads();
  return r;
}

template <typename E>
__global__ void __launch_bounds__(kThreads, 1) k_sample(const SampleArgs a) {
  constexpr int kWarps = kThreads / 32;
  extern __shared__ __align__(16) uint8_t s_raw[];
  Shared& sh = *reinterpret_cast<Shared*>(s_raw);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int r = a.sorted ? row_of_rank(a, blockIdx.x, sh) : blockIdx.x;
  const float T = a.temperature == nullptr ? 1.f : a.temperature[r];
  const bool greedy = !(T > 0.f);
  const int top_k = a.top_k == nullptr ? 0 : a.top_k[r];
  const float top_p = a.top_p == nullptr ? 1.f : a.top_p[r];
  const float min_p = a.min_p == nullptr ? 0.f : a.min_p[r];
  float u = a.uniforms[r];
  u = u > 0.f ? fminf(u, 1.f - FLT_EPSILON / 2.f) : 0.f;         // NaN and negative: 0
  Row<E> row;
  row.g = static_cast<const E*>(a.logits) + (long long)r * a.row_stride;
  row.s = reinterpret_cast<float*>(s_raw + sizeof(Shared));
  row.V = a.V;
  row.n_res = a.n_res;
  row.wide = (reinterpret_cast<uintptr_t>(row.g) & (4 * sizeof(E) - 1)) == 0;
  if (tid < 64) sh.table[tid] = exp2((double)tid / 64.0);
  // for the first histogram, so that it need not wait
  for (int i = tid; i < kBins; i += kThreads) sh.hist.lo[i] = sh.hist.hi[i] = 0u;
  bool clean = true;
  // the row: largest logit and its first place, smallest that can be kept
  float m = -INFINITY, low = INFINITY;
  int best = INT_MAX;
  auto take = [&](int i4, const float4& v) {
    if (greedy) {
      const float l[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (l[q] > m) {
          m = l[q];
          best = 4 * i4 + q;
        }
    } else {
      if (4 * i4 < row.n_res) reinterpret_cast<float4*>(row.s)[i4] = v;
      m = fmaxf(fmaxf(m, fmaxf(v.x, v.y)), fmaxf(v.z, v.w));     // (NaN is passed over)
      low = fminf(low, v.x > -INFINITY ? v.x : INFINITY);
      low = fminf(low, v.y > -INFINITY ? v.y : INFINITY);
      low = fminf(low, v.z > -INFINITY ? v.z : INFINITY);
      low = fminf(low, v.w > -INFINITY ? v.w : INFINITY);
    }
  };
  {
    const int n4 = a.V / 4;
    int i = tid;
    for (; i + 3 * kThreads < n4; i += 4 * kThreads) {
      float4 v[4];
#pragma unroll
      for (int q = 0; q < 4; ++q) v[q] = row.from_memory(i + q * kThreads);
#pragma unroll
      for (int q = 0; q < 4; ++q) take(i + q * kThreads, v[q]);
    }
    for (; i < n4; i += kThreads) take(i, row.from_memory(i));
  }
  const float thread_m = m;
  m = warp_max(m);
  low = -warp_max(-low);
  if (lane == 0) {
    sh.red_hi[warp] = m;
    sh.red_lo[warp] = low;
  }
  if (tid == 0) {
    sh.token = INT_MAX;
    sh.n_list = sh.n_rank = 0;
    sh.key_min = 0xffffffffu;
    sh.key_max = 0u;
  }
  __syncthreads();
  m = warp_max(lane < kWarps ? sh.red_hi[lane] : -INFINITY);
  low = -warp_max(lane < kWarps ? -sh.red_lo[lane] : -INFINITY);
  if (greedy || m == -INFINITY) {
    // the most likely token, lowest index first; or nothing to draw from
    best = __reduce_min_sync(0xffffffffu, thread_m == m ? best : INT_MAX);
    if (lane == 0 && best != INT_MAX) atomicMin(&sh.token, best);
    __syncthreads();
    if (tid == 0) {
      const bool any = m != -INFINITY;
      a.token[r] = any ? sh.token : -1;
      if (a.prob != nullptr) a.prob[r] = any ? 1.f : 0.f;
      if (a.kept != nullptr) a.kept[r] = any ? 1 : 0;
    }
    return;
  }
  Weight weight;
  weight.m = m;
  weight.md = (double)m;
  weight.c = 92.332482616893656 / (double)T;   // 64 / ln 2
  weight.bits = a.fixed_bits;
  weight.table = sh.table;
  const float zero = m - T * (0.6931472f * (float)(a.fixed_bits + 2));
  weight.zero = zero == zero ? zero : m;       // (infinite maximum and temperature)
  float floor = low;
  bool gathered = false;
  const float reach = fminf(m - low, kReach);
  const float steps = (float)(kBins - 1) / reach;
  const bool even = reach > 1e-30f && m < INFINITY;              // the histogram over distances makes sense
  if (top_k > 0 && top_k < a.V) {
    floor = threshold<false>(row, weight, &gathered, floor, even, steps,
                             [&](unsigned long long) { return (unsigned long long)top_k - 1ull; }, clean, sh);
    clean = false;
  }
  float least = floor;
  if (min_p > 0.f) {
    // w >= min_p  <=>  l >= m + T ln(min_p); beside an infinite maximum nothing else weighs anything, at any temperature
    const double bound = m == INFINITY ? (double)m : weight.md + (double)T * log(min((double)min_p, 1.0));
    const float f = (float)bound;
    const float up = (double)f >= bound ? f : nextafterf(f, INFINITY);
    if (f > -INFINITY) least = fmaxf(least, fminf(up, m));
  }
  // weight sums of groups of consecutive tokens: with the nucleus, by the gathered tokens, or one warp per group
  const int n_groups = ((a.V - 1) >> a.group_shift) + 1;
  uint32_t count = 0;
  bool summed = false;
  if (top_p < 1.f) {
    if (even && !gathered) {
      summed = nucleus(row, weight, a, &floor, least, top_p, T, steps, n_groups, &count, clean, sh);
      if (!summed) count = 0;
      clean = false;
    }
    if (!summed)
      floor = threshold<true>(row, weight, &gathered, floor, even, steps,
                              [&](unsigned long long z) { return nucleus_target(top_p, z); }, clean, sh);
  }
  floor = fmaxf(floor, least);
  __syncthreads();                                               // the histogram's place becomes the groups'
  if (summed) {
  } else if (gathered) {
    for (int i = tid; i < kBins; i += kThreads) sh.group[i] = 0ull;
    __syncthreads();
    each_kept(row, sh, true, floor, [&](int i, float l) {
      uint32_t* word = reinterpret_cast<uint32_t*>(&sh.group[i >> a.group_shift]);
      add_pair(word, word + 1, weight(l));
      ++count;
    });
  } else {
    for (int i = n_groups + tid; i < kBins; i += kThreads) sh.group[i] = 0ull;
    for (int g = warp; g < n_groups; g += kWarps) {
      unsigned long long sum = 0;
      const int end = min(a.V, (g + 1) << a.group_shift) / 4;
      for (int i = ((g << a.group_shift) >> 2) + lane; i < end; i += 32) {
        const float4 v = row.four(i);
        const float l[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int q = 0; q < 4; ++q)
          if (l[q] >= floor) {
            sum += weight(l[q]);
            ++count;
          }
      }
      sum = warp_sum(sum);
      if (lane == 0) sh.group[g] = sum;
    }
  }
  count = __reduce_add_sync(0xffffffffu, count);
  if (lane == 0) sh.red_n[warp] = count;
  __syncthreads();
  // the group in which the cumulative weight passes u * total (cumulative > u total <=> > floor(u total) for whole sums)
  unsigned long long target = 0;
  const unsigned long long total = find(sh, [&](int i) { return sh.group[i]; }, [&](unsigned long long z) {
    return target = min((unsigned long long)((double)u * (double)z), z - 1ull);
  });
  if (warp != 0) return;
  const uint32_t n_kept = __reduce_add_sync(0xffffffffu, lane < kWarps ? sh.red_n[lane] : 0u);
  // the token inside it: one warp, four consecutive tokens a lane
  unsigned long long run = sh.before;
  const int g_hit = sh.at, end = min(a.V, (g_hit + 1) << a.group_shift);
  for (int i0 = g_hit << a.group_shift; i0 < end; i0 += 128) {
    const int i = i0 + 4 * lane;
    const float4 v = i < end ? row.four(i / 4) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    const float l[4] = {v.x, v.y, v.z, v.w};
    unsigned long long w[4], mine = 0;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      w[q] = l[q] >= floor ? weight(l[q]) : 0ull;
      mine += w[q];
    }
    unsigned long long c = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned long long t = __shfl_up_sync(0xffffffffu, c, o);
      if (lane >= o) c += t;
    }
    const uint32_t hit = __ballot_sync(0xffffffffu, run + c > target);
    if (hit != 0u) {
      if (lane == __ffs(hit) - 1) {
        unsigned long long at = run + c - mine;
        bool found = false;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          at += w[q];
          if (!found && at > target) {
            found = true;
            a.token[r] = i + q;
            if (a.prob != nullptr) a.prob[r] = (float)((double)w[q] / (double)total);
          }
        }
        if (a.kept != nullptr) a.kept[r] = (int32_t)n_kept;
      }
      break;
    }
    run += __shfl_sync(0xffffffffu, c, 31);
  }
}

template <typename E>
int launch(cascade_ctx* ctx, SampleArgs& a, int n_rows, cudaStream_t s) {
  // what the row's logits may take: a CTA's 227 KB less its arrays, and 1 KB to spare
  constexpr int kMost = (226 * 1024 - (int)sizeof(Shared)) / 16 * 16;
  static_assert(sizeof(Shared) % 16 == 0 && kMost % 16 == 0, "alignment of the row in shared memory");
  a.n_res = kMost / 4 < a.V ? kMost / 4 : a.V;
  const size_t smem = sizeof(Shared) + (size_t)a.n_res * 4;
  const uint32_t bit = sizeof(E) == 2 ? PAGED_CFG_SAMPLE_BF16 : PAGED_CFG_SAMPLE;
  CASCADE_TRY(configure_smem(ctx, bit, k_sample<E>, (int)sizeof(Shared) + kMost));
  k_sample<E><<<n_rows, kThreads, smem, s>>>(a);
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
  if (!aligned4(temperature, top_k, top_p, min_p, uniforms, token_out, prob_out, kept_out)) return CASCADE_ERR_INVALID_ARG;
  const void* arrays[] = {token_out, prob_out, kept_out, temperature, top_k, top_p, min_p, uniforms, logits};
  for (int i = 0; i < 3; ++i)
    for (int k = i + 1; k < 9; ++k)
      if (arrays[i] != nullptr && arrays[i] == arrays[k]) return CASCADE_ERR_INVALID_ARG;   // (a block may read others' rows)
  CASCADE_TRY(check_current_device(ctx));
  SampleArgs a;
  a.logits = logits;
  a.row_stride = row_stride;
  a.V = V;
  a.n_rows = n_rows;
  // (more rows than SMs: 488 mixed rows took 133 us in index order)
  a.sorted = n_rows > ctx->sm_count && n_rows <= kMaxSorted && (temperature != nullptr || top_p != nullptr);
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
  return bf16 ? launch<__nv_bfloat16>(ctx, a, n_rows, s) : launch<float>(ctx, a, n_rows, s);
}
