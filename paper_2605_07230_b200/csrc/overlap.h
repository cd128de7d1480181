// Whether arrays whose rows may lie apart share memory (host).
#pragma once
#include <cstdint>

namespace cascade_detail {

// `n` rows of `width` bytes that start `stride` bytes apart.
struct Rows {
  const void* at;
  int64_t n, stride, width;
  uintptr_t span() const {                                             // (more than any memory has counts as 2^62)
    const __int128 bytes = n == 0 ? 0 : (__int128)(n - 1) * stride + width;
    return bytes < (int64_t)1 << 62 ? (uintptr_t)bytes : (uintptr_t)1 << 62;
  }
};
// Whether two of them share a byte; rows that lie between each other may have one common stride.
inline bool meet(const Rows& a, const Rows& b) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a.at), y = reinterpret_cast<uintptr_t>(b.at);
  if (a.n == 0 || b.n == 0 || x >= y + b.span() || y >= x + a.span()) return false;
  if (a.stride != b.stride) return true;
  const int64_t d = (int64_t)(y > x ? (y - x) % a.stride : (a.stride - (x - y) % a.stride) % a.stride);   // b's rows behind a's
  return d < a.width || d + b.width > a.stride;
}

}  // namespace cascade_detail
