// Folding what the chunks of a long axis have left in memory: D columns of a row, four a lane, the chunks dealt out to `groups`
// groups of D / 4 lanes that each take every groups-th chunk and meet in LDS.  One order of the sums, whatever the timing.
#pragma once

#include "tiles.hpp"

namespace lime {

// Groups of lanes for a row (a power of two, at most a workgroup of 256): enough that a lane takes about four chunks, whose loads
// are in flight together; a lane that walked all of them alone waited for memory once a chunk (512 chunks of a row: 274 us).
inline int fold_groups(int splits, int lanes) {
  int groups = 1;
  while (groups * 4 < splits && groups * lanes < 256) groups *= 2;
  return groups;
}

template <int D>
struct Folder {
  static constexpr int kLanes = D / 4;
  int t, group, row, rows;  // this lane's four columns, its group, the row of the workgroup's it works on, and how many they are
  __device__ explicit Folder(int groups) {
    t = threadIdx.x % kLanes;
    group = threadIdx.x / kLanes % groups;
    row = threadIdx.x / kLanes / groups;
    rows = 256 / kLanes / groups;
  }
  // The sum of the chunks' states at p, `step` floats apart, in every lane of group 0.  All threads of the workgroup call it.
  __device__ f32x4 sum(const float* p, int64_t step, int splits, int groups, bool live) const {
    return sum_of([&](int s) { return *reinterpret_cast<const f32x4*>(p + s * step + 4 * t); }, splits, groups, live);
  }
  // The sum of chunk(s) over the chunks s, in the same way.
  template <typename F>
  __device__ f32x4 sum_of(F chunk, int splits, int groups, bool live) const {
    __shared__ f32x4 met[256];
    f32x4 a = {0, 0, 0, 0};
    if (live) {
#pragma unroll 4
      for (int s = group; s < splits; s += groups) {
        const f32x4 x = chunk(s);
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] += x[j];
      }
    }
    for (int half = groups / 2; half; half /= 2) {
      __syncthreads();
      met[threadIdx.x] = a;
      __syncthreads();
      if (group < half) {
        const f32x4 x = met[threadIdx.x + half * kLanes];
#pragma unroll
        for (int j = 0; j < 4; ++j) a[j] += x[j];
      }
    }
    return a;
  }
};

template <typename T>
__device__ __forceinline__ void store_four(T* to, f32x4 v, int c, int width, bool quads) {
  if (quads) {
    if (c >= width) return;
    if constexpr (sizeof(T) == 2) {
      bf16x4 x;
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = static_cast<__bf16>(v[j]);
      *reinterpret_cast<bf16x4*>(to + c) = x;
    } else {
      *reinterpret_cast<f32x4*>(to + c) = v;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (c + j < width) store_as(to + c + j, v[j]);
  }
}

}  // namespace lime
