// What the forward and the backward pass of the attention over packed sequences share on the device.
#pragma once

#include "encoder.hpp"
#include "tiles.hpp"

namespace lime {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// A user's slot of a packed tensor and the rows of it that are in use.  Offsets and lengths are cut to the tensor, so that
// what they hold never takes an access outside it.
struct Span {
  int64_t start;
  int slot, used;
};
__device__ __forceinline__ Span span_of(const int32_t* offsets, const int32_t* lens, int b, int64_t rows, int most) {
  const int64_t start = min(max(static_cast<int64_t>(offsets[b]), int64_t{0}), rows);
  const int64_t end = min(max(static_cast<int64_t>(offsets[b + 1]), start), rows);
  const int slot = static_cast<int>(min(end - start, static_cast<int64_t>(most)));
  return {start, slot, lens ? min(max(lens[b], 0), slot) : slot};
}

// How many keys query i of a user sees: all, or those up to its own place counted from the end.
__device__ __forceinline__ int keys_seen(int i, int n_q, int n_k, int causal) { return causal ? min(n_k, max(0, i + 1 + n_k - n_q)) : n_k; }

}  // namespace lime
