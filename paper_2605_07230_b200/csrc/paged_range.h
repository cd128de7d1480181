// Which tokens of a request see a range of its keys (host and device; nothing of CUDA, so that it can be tested alone).
#pragma once

#ifdef __CUDACC__
#define CASCADE_BOTH __host__ __device__ __forceinline__
#else
#define CASCADE_BOTH inline
#endif

namespace paged {

// Tokens of a request (first position x0, nq of them) that see any of the keys k_first .. k_last: [*lo, *hi), inside [0, nq] where
// nobody does too, so that counts of rows stay in 32 bits (a window may end millions of tokens in front).  A: has window, sinks.
template <typename A>
CASCADE_BOTH void tokens_that_see(const A& a, int x0, int nq, int k_first, int k_last, int* lo, int* hi) {
  *lo = k_first > x0 ? k_first - x0 : 0;
  *hi = nq;
  if (a.window > 0 && k_first >= a.sinks) {
    const long long end = (long long)k_last + a.window - x0;
    if (end < nq) *hi = end > *lo ? (int)end : *lo;
  }
}
// The same as rows (token, query head of a group of G).
template <typename A>
CASCADE_BOTH void rows_that_see(const A& a, int x0, int nq, int G, int k_first, int k_last, int* lo, int* hi) {
  tokens_that_see(a, x0, nq, k_first, k_last, lo, hi);
  *lo *= G;
  *hi *= G;
}

}  // namespace paged
