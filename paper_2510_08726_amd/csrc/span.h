// The bytes that operands span, for the checks of what a call writes (host only).
#pragma once

#include <cstdint>
#include <initializer_list>

namespace attn {

struct Span {
  uintptr_t begin, end;
};

inline Span span(const void* p, int64_t bytes) {
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  return {at, p ? at + (uintptr_t)bytes : at};
}

// Those of rows of D 16-bit elements, with strides of batches, heads and tokens of either sign.
inline Span span(const void* p, const long long* strides, int B, int H, int L, int D) {
  const int n[3] = {B, H, L};
  __int128 low = 0, high = D;
  for (int i = 0; i < 3; ++i) {
    const __int128 reach = (__int128)(n[i] - 1) * strides[i];
    (reach < 0 ? low : high) += reach;
  }
  const uintptr_t at = reinterpret_cast<uintptr_t>(p);
  return {at + (uintptr_t)(2 * low), at + (uintptr_t)(2 * high)};
}

// Whether `out`, which a call writes, lies apart from all the others.
inline bool apart(Span out, std::initializer_list<Span> others) {
  for (const Span& x : others)
    if (x.begin < out.end && out.begin < x.end) return false;
  return true;
}

inline bool misaligned(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) != 0; }

}  // namespace attn
