// What the forward and the backward pass of the attention over packed sequences share on the device.
#pragma once

#include "divisor.hpp"
#include "encoder.hpp"
#include "tiles.hpp"

namespace lime {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// Which rows of the packed tensors are whose.  Lengths that are not given point at the offsets, so that they can be read along.
struct Packing {
  const int32_t *q_offsets, *q_lens, *k_offsets, *k_lens;
  int q_rows, k_rows, max_q, max_k;
  bool has_q_lens, has_k_lens;
  Packing() = default;
  explicit Packing(const SequenceAttention& x)
      : q_offsets(x.q_offsets), q_lens(x.q_lens ? x.q_lens : x.q_offsets), k_offsets(x.k_offsets), k_lens(x.k_lens ? x.k_lens : x.k_offsets),
        q_rows(static_cast<int>(x.q_rows)), k_rows(static_cast<int>(x.k_rows)), max_q(x.max_q), max_k(x.max_k), has_q_lens(x.q_lens != nullptr),
        has_k_lens(x.k_lens != nullptr) {}
};

// A user's slot of a packed tensor and the rows of it that are in use.  Offsets and lengths are cut to the tensor, so that
// what they hold never takes an access outside it.
struct Span {
  int64_t start;
  int slot, used;
};
struct Spans {
  Span q, k;
};
__device__ __forceinline__ Spans spans_of(const Packing& p, int b) {
  // all of them asked for before any is looked at: one wait of a kernel's start instead of four
  const int q0 = p.q_offsets[b], q1 = p.q_offsets[b + 1], k0 = p.k_offsets[b], k1 = p.k_offsets[b + 1], ql = p.q_lens[b], kl = p.k_lens[b];
  auto span = [](int begin, int end, int len, bool has, int rows, int most) -> Span {
    begin = min(max(begin, 0), rows), end = min(max(end, begin), rows);
    const int slot = min(end - begin, most);
    return {begin, slot, has ? min(max(len, 0), slot) : slot};
  };
  return {span(q0, q1, ql, p.has_q_lens, p.q_rows, p.max_q), span(k0, k1, kl, p.has_k_lens, p.k_rows, p.max_k)};
}

// The user and key head of a workgroup, from a grid of (key heads, users, tiles).  Workgroups go to the eight XCDs in turn, so that
// where users times key heads is a multiple of eight a pair's tiles all land on one XCD and read its keys from one L2: right where all
// histories are as long, but where they are not the XCD with the longest users ends last.  Then every second tile moves on to the next
// pair's place.  (16 users of 2048 to 4096 events, two key heads: forward 131 -> 114 us; 16 of 4096: 159, and 165 if they moved.)
inline bool ragged(const SequenceAttention& x) {
  return x.q_lens != nullptr || x.k_lens != nullptr || x.k_rows < static_cast<int64_t>(x.B) * x.max_k || x.q_rows < static_cast<int64_t>(x.B) * x.max_q;
}
struct Deal {
  Divisor pairs, hk;
  bool moves;
  Deal() = default;
  Deal(const SequenceAttention& x, bool may_move) : pairs(static_cast<uint32_t>(x.B) * x.hk), hk(x.hk), moves(may_move && ragged(x)) {}
};
struct Pair {
  int b, kv, index;
};
__device__ __forceinline__ Pair pair_of(const Deal& d) {
  const int hk = d.hk.d, pair = blockIdx.y * hk + blockIdx.x;
  if (!d.moves) return {static_cast<int>(blockIdx.y), static_cast<int>(blockIdx.x), pair};
  const int moved = pair + blockIdx.z / 2, at = moved - d.pairs.divide(moved) * d.pairs.d, b = d.hk.divide(at);
  return {b, at - b * hk, at};
}

// f(width) for the narrowest width of products that holds heads of dh.
template <typename F>
hipError_t at_head_width(int dh, F f) {
  if (dh <= 32) return f(std::integral_constant<int, 32>{});
  if (dh <= 48) return f(std::integral_constant<int, 48>{});
  if (dh <= 64) return f(std::integral_constant<int, 64>{});
  if (dh <= 80) return f(std::integral_constant<int, 80>{});
  if (dh <= 96) return f(std::integral_constant<int, 96>{});
  return f(std::integral_constant<int, 128>{});
}

// How many keys query i of a user sees: all, or those up to its own place counted from the end.
__device__ __forceinline__ int keys_seen(int i, int n_q, int n_k, bool causal) { return causal ? min(n_k, max(0, n_k - n_q + (i + 1))) : n_k; }

}  // namespace lime
