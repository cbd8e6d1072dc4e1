// Shared by the two softmax attentions: which tokens a token sees.
#pragma once
#include "tokens.hpp"

namespace nc {

// The tokens that token i sees, j <= i with i - j < window (0: all) or j < sinks:
// the first `first` and those from `near` to i, `count` of them in all.
struct Seen {
  int first, near, count;
  __device__ __forceinline__ int at(int x) const { return x < first ? x : x - first + near; }
};
__device__ __forceinline__ Seen seen_by(int i, int64_t window, int64_t sinks) {
  Seen s;
  s.near = window ? (int)max((int64_t)0, i + 1 - window) : 0;
  s.first = (int)min(sinks, (int64_t)s.near);
  s.count = s.first + i + 1 - s.near;
  return s;
}

}  // namespace nc
