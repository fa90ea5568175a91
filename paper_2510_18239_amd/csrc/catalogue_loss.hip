// Softmax cross entropy of rows over a catalogue of items, with its gradients, the logits never in memory:
//   z_iv = scale <X_i, W_v>,   lse_i = log sum_v exp(z_iv),   loss_i = lse_i - z_i,target(i)
//   e_iv = dloss_i scale (exp(z_iv - lse_i) - [v = target(i)]),   dX_i = sum_v e_iv W_v,   dW_v = sum_i e_iv X_i.
// Rows without a target have no loss and no gradients, and nothing of them is read into any: the other rows are listed first and, where
// they are streamed and there are any to leave out, copied together (gather), so that padding costs no products.
// The forward pass and dX hold rows of X in registers and stream the items' tiles, with the catalogue cut into chunks whose sums
// are folded in ascending order; dW holds items and streams rows.  The other items' p and e are rounded to the storage type, as operands
// of the last products (half a step each, of terms that are summed in fp32); the target's e = p - 1, which may be small beside p, is formed in
// fp32 once a row, from the stored lse (whose own rounding is what is left of its error): for dX it stays out of the product and is added at the fold.
// Bound by the matrix units: 8192 rows over 131072 items, d = 256, bf16: forward 500 us, 1.1 PFLOP/s, both gradients 1830 us with the
// logits' products done again on either side, 1.2 PFLOP/s, where a library product of 16384^3 reaches 1.36.  (Logits kept for the
// gradients would be 2 GB written and read twice, as long as the product that they save.)
#include <algorithm>
#include <cmath>

#include "divisor.hpp"
#include "encoder.hpp"
#include "fold.hpp"

namespace lime {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

struct Args {
  const void *x, *w;
  const int32_t* targets;
  float *loss, *lse;
  const float* dloss;
  void *dx, *dw;
  int64_t rows;
  int items, d;
  float scale;
  bool x_pieces, w_pieces, quads;
  // workspace
  int32_t* live;      // [1 + rows]: how many rows have a target, and which they are
  void* packed;       // [rows][d] the rows with a target, written where some have none
  float *c_logit;             // forward, [rows] of the listed rows: <X_i, W_target>
  float *c_lse2, *c_g, *c_e;  // backward, [rows] of the listed rows: lse log2 e; dloss scale; e of the target
  int32_t *c_target, *c_place;  // [rows] the target, and its place among the tiles of items
  Divisor item_tiles;
  float* parts;       // forward [splits][rows][2], dX [splits][rows][padded d]
  float* item_parts;  // dW [item_splits][items][padded d]
  int splits, chunk;            // of the catalogue, for the kernels that hold rows
  int item_splits, item_chunk;  // of the rows, for those that hold items
};

// Which of the tiles of 128 items, and of its places, an item has: neighbours are dealt out to different tiles, because popular items
// are often neighbours, and the one workgroup that held them all would end last: it adds a term for every row that has one of them for
// its target.  (8192 rows over 131072 items, a tenth of the rows with a target below 128: dW 1060 us in order, 945 dealt out.)
__device__ __forceinline__ int place_of(const Args& a, int item) {
  const int at = a.item_tiles.divide(item);
  return (item - at * static_cast<int>(a.item_tiles.d)) * 128 + at;
}

// <X_i, W_target> of 32 rows, a lane pair each, with the very bits that the forward pass's stream of tiles gives it: the same instructions in the
// same order, of -X for a negative scale (a sum of opposite terms need not be the opposite), and the diagonal of the block.  Of a learnt target
// lse and the logit nearly cancel.  (300 rows over 1000 items, d = 256, p of the target from 0.6 to 0.9999, median errors with a sum in another
// order, and with this: loss 9e-5 of itself and 1e-5, in fp32 dX 2.4e-4 and 2.7e-5.)
template <typename T>
__device__ __forceinline__ float target_logits(const Args& a, int64_t row, int target, bool live, int lane) {
  const int n = lane & 31, g = lane >> 5;
  const T *x = static_cast<const T*>(a.x) + row * a.d, *w = static_cast<const T*>(a.w) + static_cast<int64_t>(target) * a.d;
  f32x16 s = zero_block();
#pragma unroll 4
  for (int c = 0; c < a.d; c += 16) {
    Fragment<T> xf[1], wf[1];
    load_row<T, 16>(x + c, (a.d - c) * sizeof(T), a.x_pieces, live, g, xf);
    load_row<T, 16>(w + c, (a.d - c) * sizeof(T), a.w_pieces, live, g, wf);
    if (a.scale < 0.f) negate(xf[0]);
    s = mma16(wf[0], xf[0], s);
  }
  float own = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) own = block_row(e, g) == n ? s[e] : own;
  own = pair_sum(own);
  return a.scale < 0.f ? -own : own;
}

constexpr int kGatherRows = 64, kGatherWaves = 16;  // rows a workgroup of the gather takes at a time

// Lists the rows with a target.  Every workgroup counts all targets by itself (they are few next to the products), so that no
// workgroup waits for another: large workgroups, one a compute unit, because they all read all targets.
template <typename T, bool BACKWARD>
__global__ __launch_bounds__(64 * kGatherWaves) void gather_kernel(Args a, int64_t each) {
  __shared__ int sums[kGatherWaves][2];
  __shared__ int place[kGatherRows], aim[kGatherRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t begin = blockIdx.x * each, end = min(begin + each, a.rows);
  auto named = [&](int target) { return static_cast<unsigned>(target) < static_cast<unsigned>(a.items); };
  int before = 0, all = 0;
  auto count = [&](int64_t i, int target) {
    const int x = named(target);
    all += x, before += i < begin ? x : 0;
  };
  const int64_t fours = reinterpret_cast<uintptr_t>(a.targets) % 16 == 0 ? a.rows / 4 : 0;
#pragma unroll 4
  for (int64_t i = tid; i < fours; i += 64 * kGatherWaves) {
    const i32x4 t = reinterpret_cast<const i32x4*>(a.targets)[i];
#pragma unroll
    for (int j = 0; j < 4; ++j) count(4 * i + j, t[j]);
  }
  for (int64_t i = 4 * fours + tid; i < a.rows; i += 64 * kGatherWaves) count(i, a.targets[i]);
  for (int o = 32; o; o >>= 1) before += __shfl_xor(before, o, 64), all += __shfl_xor(all, o, 64);
  if (lane == 0) sums[wave][0] = before, sums[wave][1] = all;
  __syncthreads();
  before = all = 0;
  for (int w = 0; w < kGatherWaves; ++w) before += sums[w][0], all += sums[w][1];
  if (blockIdx.x == 0 && tid == 0) a.live[0] = all;
  const bool whole = all == a.rows;
  for (int64_t at = begin; at < end; at += kGatherRows) {
    if (wave == 0) {  // 64 rows' places
      const int64_t i = at + lane;
      const int target = i < end ? a.targets[i] : -1;
      const bool x = named(target);
      const unsigned long long votes = __ballot(x);
      const int to = before + __popcll(votes & ((1ull << lane) - 1));
      before += __popcll(votes);
      place[lane] = x ? to : -1, aim[lane] = target;
      if (x) {
        a.live[1 + to] = static_cast<int>(i);
        if constexpr (BACKWARD) a.c_lse2[to] = a.lse[i] * kLog2e, a.c_g[to] = a.dloss[i] * a.scale, a.c_target[to] = target, a.c_place[to] = place_of(a, target);
      } else if (i < end) {
        if constexpr (!BACKWARD) a.loss[i] = 0.f, a.lse[i] = 0.f;
      }
    }
    if constexpr (!BACKWARD) continue;
    __syncthreads();
    const int here = static_cast<int>(min<int64_t>(kGatherRows, end - at));
    if (wave < 2) {  // e of the rows' own targets, dloss scale (p - 1): 32 rows a wave
      const int r = 32 * wave + (lane & 31), to = r < here ? place[r] : -1;
      const int64_t i = at + min(r, here - 1);
      const float lse = to >= 0 ? a.lse[i] : 0.f, weight = to >= 0 ? a.dloss[i] : 0.f;
      const float s = target_logits<T>(a, i, to >= 0 ? aim[r] : 0, to >= 0, lane);
      if (to >= 0 && lane < 32) a.c_e[to] = (__builtin_amdgcn_exp2f(fmaf(s, a.scale, -lse) * kLog2e) - 1.f) * weight * a.scale;
    }
#pragma unroll 4
    for (int r = wave; r < here; r += kGatherWaves) {  // a wave a row
      if (whole) continue;
      const T* from = static_cast<const T*>(a.x) + (at + r) * a.d;
      const int to = place[r];
      T* dst = to >= 0 ? static_cast<T*>(a.packed) + static_cast<int64_t>(to) * a.d : static_cast<T*>(a.dx) + (at + r) * a.d;
      if (to < 0 && a.dx == nullptr) continue;
      if (a.x_pieces && a.quads) {  // rows of whole 16-byte pieces: at most 64 of them
        const int c = lane * static_cast<int>(16 / sizeof(T));
        if (c < a.d) {
          u32x4 v = {0, 0, 0, 0};
          if (to >= 0) v = *reinterpret_cast<const u32x4*>(from + c);
          *reinterpret_cast<u32x4*>(dst + c) = v;
        }
      } else {
        for (int c = lane; c < a.d; c += 64) {
          T v{};
          if (to >= 0) v = from[c];
          dst[c] = v;
        }
      }
    }
    __syncthreads();
  }
}

// Few rows are listed by every wave of the forward pass for itself: a look at all targets, 64 at a time, takes less than another
// kernel.  The wave's 32 places from `first` on get the rows that stand there and their targets; returns how many rows are listed in all.
constexpr int kFewRows = 4096;
__device__ __forceinline__ int list_rows(const Args& a, int first, int lane, int2* places, bool zero_others) {
  int before = 0;
  const int rows = static_cast<int>(a.rows);
  for (int base = 0; base < rows; base += 512) {
    int target[8];  // loads in flight
#pragma unroll
    for (int j = 0; j < 8; ++j) target[j] = a.targets[min(base + 64 * j + lane, rows - 1)];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = base + 64 * j + lane;
      const bool x = i < rows && static_cast<unsigned>(target[j]) < static_cast<unsigned>(a.items);
      const unsigned long long votes = __ballot(x);
      const int to = before + __popcll(votes & ((1ull << lane) - 1)) - first;
      if (x && static_cast<unsigned>(to) < 32u) places[to] = {i, target[j]};
      if (zero_others && !x && i < rows) a.loss[i] = 0.f, a.lse[i] = 0.f;
      before += __popcll(votes);
    }
  }
  wave_lds_fence();
  return before;
}

// Running maximum and sum of a chunk of the catalogue for 32 rows a wave; the last workgroups, one a tile of rows, have the rows' own logits.
template <typename T, int C, int STEP>
__global__ __launch_bounds__(256) void catalogue_lse_kernel(Args a) {
  constexpr int D = tile_width(C);
  using Stage = Stages<T, D, STEP, 1>;
  using Loader = TileLoader<T, D, STEP, 4>;
  using Reader = TileReader<T, D, STEP>;
  constexpr int VB = STEP / 32, NK = C / 16;
  extern __shared__ __align__(1024) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, g = lane >> 5;
  const Reader read(lane);
  const int tiles = static_cast<int>((a.rows + 127) / 128), block = blockIdx.x;
  const bool streams = block < tiles * a.splits;
  const int split = streams ? block % a.splits : a.splits, tile = streams ? block / a.splits : block - tiles * a.splits, row = tile * 128 + 32 * wave + n;
  const int v0 = streams ? split * a.chunk : 0, v1 = streams ? min(a.items, v0 + a.chunk) : 0, steps = (v1 - v0 + STEP - 1) / STEP;
  const unsigned width = a.d * sizeof(T);
  const Rows wm{static_cast<const T*>(a.w) + static_cast<int64_t>(v0) * a.d, width, width, a.w_pieces};
  Loader wl;
  wl.init(wm, tid);
  if (streams) wl.issue(wm, 0, v1 - v0, Stage::tile(smem, 0, 0), tid);
  int count, from = 0, target = 0;
  if (a.rows <= kFewRows) {
    int2* places = reinterpret_cast<int2*>(smem + Stage::kTiles) + 32 * wave;  // (where the first step's tile does not arrive)
    count = list_rows(a, row - n, lane, places, split == 0 && tile == 0 && wave == 0);
    if (row < count) from = places[n].x, target = places[n].y;
    if (split == 0 && g == 0 && row < count) a.live[1 + row] = from;
    if (split == 0 && row == 0 && g == 0) a.live[0] = count;
  } else {
    count = a.live[0];
    if (row < count) from = a.live[1 + row];
    if (row < count && !streams) target = a.targets[from];
  }
  if (tile * 128 >= count) {
    wait_lds_loads<0>();
    return;
  }
  if (!streams) {
    const float s = target_logits<T>(a, from, target, row < count, lane);
    if (row < count && g == 0) a.c_logit[row] = s;
    return;
  }
  Fragment<T> x[NK];
  load_row<T, C>(static_cast<const T*>(a.x) + static_cast<int64_t>(from) * a.d, width, a.x_pieces, row < count, g, x);
  const float c = fmaxf(fabsf(a.scale) * kLog2e, 1e-37f);
  if (a.scale < 0.f) {
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) negate(x[kk]);
  }
  // Two blocks of 32 items a step.  Each block's products are issued among the exponentials of the block before, which the matrix and the
  // vector units then work on together.
  float m = -INFINITY, l = 0.f;
  auto absorb = [&](const f32x16& s) {
    float top = s[0];
#pragma unroll
    for (int e = 1; e < 16; ++e) top = fmaxf(top, s[e]);
    const float to = fmaxf(m, pair_max(top) * c), base = to == -INFINITY ? 0.f : to;
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 16; ++e) sum += __builtin_amdgcn_exp2f(fmaf(s[e], c, -base));
    l = fmaf(l, __builtin_amdgcn_exp2f(m - base), sum), m = to;
  };
  auto logits = [&](unsigned wt, int vb) {
    f32x16 s = zero_block();
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) s = mma16(read.row(wt, 32 * vb, kk), x[kk], s);
    return s;
  };
  f32x16 before;
#pragma unroll
  for (int e = 0; e < 16; ++e) before[e] = -INFINITY;
  auto arrived = [&](int i) -> unsigned {  // step i's tile; the next is asked for (past the last: nothing but zeros)
    Stage::template arrive<4>(smem, tid);
    wl.issue(wm, (i + 1) * STEP, v1 - v0, Stage::tile(smem, i + 1, 0), tid);
    return Stage::operand(smem, i, 0);
  };
  const int whole = (v1 - v0) / STEP;
  for (int i = 0; i < whole; ++i) {
    const unsigned wt = arrived(i);
#pragma unroll
    for (int vb = 0; vb < VB; ++vb) {
      const f32x16 s = logits(wt, vb);
      absorb(before);
      before = s;
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int e = 0; e < 16; ++e) __builtin_amdgcn_sched_group_barrier(0x008, 1, 0), __builtin_amdgcn_sched_group_barrier(0x100, 1, 0), __builtin_amdgcn_sched_group_barrier(0x002, 4, 0);
      }
    }
  }
  if (whole < steps) {
    const unsigned wt = arrived(whole);
#pragma unroll 1
    for (int vb = 0; vb < VB; ++vb) {
      absorb(before);
      before = logits(wt + 32 * vb * Reader::kRowBytes, 0);
#pragma unroll
      for (int e = 0; e < 16; ++e)
        if (v0 + whole * STEP + 32 * vb + block_row(e, g) >= v1) before[e] = -INFINITY;
    }
  }
  wait_lds_loads<0>();
  absorb(before);
  l = pair_sum(l);
  if (row < count && g == 0) {
    float* to = a.parts + (static_cast<int64_t>(split) * a.rows + row) * 2;
    to[0] = m, to[1] = l;
  }
}

// A wave a row: the chunks' states folded, and the target's logit taken off.
__global__ __launch_bounds__(256) void catalogue_loss_kernel(Args a) {
  const int lane = threadIdx.x & 63, row = blockIdx.x * 4 + (threadIdx.x >> 6), count = a.live[0];
  if (row >= count) return;
  float m = -INFINITY, l = 0.f;
  for (int s = lane; s < a.splits; s += 64) {
    const float* p = a.parts + (static_cast<int64_t>(s) * a.rows + row) * 2;
    const float to = fmaxf(m, p[0]), base = to == -INFINITY ? 0.f : to;
    l = l * __builtin_amdgcn_exp2f(m - base) + p[1] * __builtin_amdgcn_exp2f(p[0] - base);
    m = to;
  }
  float most = m;
  for (int o = 32; o; o >>= 1) most = fmaxf(most, __shfl_xor(most, o, 64));
  const float base = most == -INFINITY ? 0.f : most;
  const float sum = wave_sum(l * __builtin_amdgcn_exp2f(m - base));
  if (lane == 0) {
    // (off the maximum as it went into it, in base 2; lse from both with one rounding where the target has a good part of it)
    const int at = a.live[1 + row];
    const float s = a.c_logit[row], rest = __builtin_amdgcn_logf(sum), loss = (fmaf(-s, a.scale * kLog2e, most) + rest) * kLn2;
    a.lse[at] = loss < 1.f ? fmaf(s, a.scale, loss) : (most + rest) * kLn2, a.loss[at] = loss;
  }
}

// sum_v p_iv W_v, v other than target(i), over a chunk of the catalogue, 32 rows a wave.  (The target's p among them, rounded, would leave
// nothing of p - 1 where a row has learnt its target: from p = 0.998 on, dX was off by as much as itself.)
template <typename T, int C, int STEP>
__device__ __forceinline__ void rows_gradient(Args a, unsigned block, unsigned char* smem) {
  constexpr int D = tile_width(C);
  using Stage = Stages<T, D, STEP, 1>;
  using Loader = TileLoader<T, D, STEP, 4>;
  using Reader = TileReader<T, D, STEP>;
  constexpr int VB = STEP / 32, NK = C / 16, OB = C / 32;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, g = lane >> 5;
  const Reader read(lane);
  const int split = block % a.splits, tile = block / a.splits, count = a.live[0];
  if (tile * 128 >= count) return;
  const int row = tile * 128 + 32 * wave + n;
  const int v0 = split * a.chunk, v1 = min(a.items, v0 + a.chunk), steps = (v1 - v0 + STEP - 1) / STEP;
  const unsigned width = a.d * sizeof(T);
  const Rows wm{static_cast<const T*>(a.w) + static_cast<int64_t>(v0) * a.d, width, width, a.w_pieces};
  Loader wl;
  wl.init(wm, tid);
  wl.issue(wm, 0, v1 - v0, Stage::tile(smem, 0, 0), tid);
  Fragment<T> x[NK];
  load_row<T, C>(static_cast<const T*>(a.x) + static_cast<int64_t>(row < count ? a.live[1 + row] : 0) * a.d, width, a.x_pieces, row < count, g, x);
  const float c = a.scale * kLog2e, lse2 = row < count ? a.c_lse2[row] : 0.f;
  const int own = row < count ? a.c_target[row] - v0 - 4 * g : -8;  // the target, from the chunk's first item of this lane half
  f32x16 dx[OB];
#pragma unroll
  for (int ob = 0; ob < OB; ++ob) dx[ob] = zero_block();
  for (int i = 0; i < steps; ++i) {
    Stage::template arrive<4>(smem, tid);
    if (i + 1 < steps) wl.issue(wm, (i + 1) * STEP, v1 - v0, Stage::tile(smem, i + 1, 0), tid);
    const unsigned wt = Stage::operand(smem, i, 0);
#pragma unroll
    for (int vb = 0; vb < VB; ++vb) {
      f32x16 p = zero_block();
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) p = mma16(read.row(wt, 32 * vb, kk), x[kk], p);
#pragma unroll
      for (int e = 0; e < 16; ++e) p[e] = __builtin_amdgcn_exp2f(fmaf(p[e], c, -lse2));
      const int first = i * STEP + 32 * vb;
      // some row's target is in this block, or zero rows past the chunk, where p may be infinite
      if (__any(static_cast<unsigned>(own - first) < 32u) || first + 32 > v1 - v0) {
        seldom();
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (own - first == block_row(e, 0) || v1 - v0 - first - 4 * g <= block_row(e, 0)) p[e] = 0.f;
      }
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const Fragment<T> pf = half_fragment<T>(p, f);
#pragma unroll
        for (int ob = 0; ob < OB; ++ob) dx[ob] = mma16(read.column(wt, 32 * vb + 16 * f, 32 * ob), pf, dx[ob]);
      }
    }
  }
  if (row >= count) return;
  float* to = a.parts + (static_cast<int64_t>(split) * a.rows + row) * D;
#pragma unroll
  for (int ob = 0; ob < OB; ++ob) store_block(to, dx[ob], 1.f, 32 * ob, a.d, true, g);
}

// dX_i = dloss_i scale the chunks' sums + e_target W_target.
template <typename T, int D>
__device__ __forceinline__ void fold_rows(const Args& a, unsigned block, int groups) {
  const Folder<D> at(groups);
  const int row = block * at.rows + at.row, c = 4 * at.t;
  const bool live = row < a.live[0] && c < a.d;
  f32x4 sum = at.sum(a.parts + static_cast<int64_t>(row) * D, a.rows * D, a.splits, groups, live);
  if (!live || at.group != 0) return;
  const T* w = static_cast<const T*>(a.w) + static_cast<int64_t>(a.c_target[row]) * a.d + c;
  const float f = a.c_g[row], e = a.c_e[row];
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (c + j < a.d) sum[j] = fmaf(f, sum[j], e * to_float(w[j]));
  store_four(static_cast<T*>(a.dx) + static_cast<int64_t>(a.live[1 + row]) * a.d, sum, c, a.d, a.quads);
}

// sum_i e_iv X_i over a chunk of the listed rows, 32 items a wave.
template <typename T, int C, int STEP>
__device__ __forceinline__ void items_gradient(Args a, unsigned block, unsigned char* smem) {
  constexpr int D = tile_width(C);
  using Stage = Stages<T, D, STEP, 1, 4>;  // rows; lse2, dloss scale, target's place, its e
  using Loader = TileLoader<T, D, STEP, 4>;
  using Reader = TileReader<T, D, STEP>;
  constexpr int RB = STEP / 32, NK = C / 16, OB = C / 32;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, g = lane >> 5;
  const Reader read(lane);
  const int split = block % a.item_splits, tile = block / a.item_splits, count = a.live[0];
  const int place0 = tile * 128 + 32 * wave, place = place0 + n, item = (32 * wave + n) * static_cast<int>(a.item_tiles.d) + tile;
  const int i0 = split * a.item_chunk, i1 = min(count, i0 + a.item_chunk), steps = i1 > i0 ? (i1 - i0 + STEP - 1) / STEP : 0;
  const unsigned width = a.d * sizeof(T);
  const Rows xm{static_cast<const T*>(count == a.rows ? a.x : a.packed) + static_cast<int64_t>(i0) * a.d, width, width, a.x_pieces};
  Loader xl;
  xl.init(xm, tid);
  auto ask = [&](int i) {
    xl.issue(xm, i * STEP, i1 - i0, Stage::tile(smem, i, 0), tid);
    const int from = i0 + i * STEP;
    const void* words[4] = {a.c_lse2, a.c_g, a.c_place, a.c_e};
    words_to_lds(static_cast<const float*>(words[wave]) + from, min(STEP, i1 - from), Stage::words(smem, i, wave), lane);
  };
  if (steps > 0) ask(0);
  Fragment<T> w[NK];
  load_row<T, C>(static_cast<const T*>(a.w) + static_cast<int64_t>(item) * a.d, width, a.w_pieces, item < a.items, g, w);
  const float c = a.scale * kLog2e;
  f32x16 dw[OB];
#pragma unroll
  for (int ob = 0; ob < OB; ++ob) dw[ob] = zero_block();
  for (int i = 0; i < steps; ++i) {
    Stage::template arrive<4>(smem, tid);
    if (i + 1 < steps) ask(i + 1);
    const unsigned xt = Stage::operand(smem, i, 0);
    const float *lse2 = Stage::words(smem, i, 0), *weight = Stage::words(smem, i, 1), *own = Stage::words(smem, i, 3);
    const int32_t* target = reinterpret_cast<const int32_t*>(Stage::words(smem, i, 2));
    // which of the step's rows have one of the wave's items for their target (rows past the last: with the weight 0)
    const unsigned long long chosen = __ballot(lane < STEP && static_cast<unsigned>(target[lane % STEP] - place0) < 32u);
#pragma unroll(D < 256 ? RB : 1)
    for (int rb = 0; rb < RB; ++rb) {
      const unsigned block = xt + 32 * rb * Reader::kRowBytes;
      f32x16 e = zero_block();
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) e = mma16(read.row(block, 0, kk), w[kk], e);
      auto weigh = [&](auto with_targets) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int at = 32 * rb + 8 * j + 4 * g;
          const f32x4 l4 = *reinterpret_cast<const f32x4*>(lse2 + at), g4 = *reinterpret_cast<const f32x4*>(weight + at);
#pragma unroll
          for (int y = 0; y < 4; ++y) e[4 * j + y] = __builtin_amdgcn_exp2f(fmaf(e[4 * j + y], c, -l4[y])) * g4[y];
          if constexpr (with_targets) {
            const i32x4 t4 = *reinterpret_cast<const i32x4*>(target + at);
            const f32x4 o4 = *reinterpret_cast<const f32x4*>(own + at);
#pragma unroll
            for (int y = 0; y < 4; ++y) e[4 * j + y] = t4[y] == place ? o4[y] : e[4 * j + y];
          }
        }
      };
      if (static_cast<unsigned>(chosen >> (32 * rb)) == 0) weigh(std::false_type{});
      else weigh(std::true_type{});
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const Fragment<T> ef = half_fragment<T>(e, f);
#pragma unroll
        for (int ob = 0; ob < OB; ++ob) dw[ob] = mma16(read.column(block, 16 * f, 32 * ob), ef, dw[ob]);
      }
    }
    // A target's e is near its row's whole weight and, in a large catalogue, rarely has company in its sum: what rounding took of it is
    // added by itself.  (Popular items are chosen at nearly every step: sixteen rows without one of them are passed over.)
    if constexpr (sizeof(T) == 2) {
      if (chosen != 0)
#pragma unroll 1
      for (int k = 0; k < 2 * RB; ++k) {
        if ((chosen >> (16 * k) & 0xffff) == 0) continue;
        bf16x8 low;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const i32x4 t4 = *reinterpret_cast<const i32x4*>(target + 16 * k + 8 * j + 4 * g);
          const f32x4 o4 = *reinterpret_cast<const f32x4*>(own + 16 * k + 8 * j + 4 * g);
#pragma unroll
          for (int y = 0; y < 4; ++y)
            low[4 * j + y] = static_cast<__bf16>(t4[y] == place ? o4[y] - static_cast<float>(static_cast<__bf16>(o4[y])) : 0.f);
        }
#pragma unroll
        for (int ob = 0; ob < OB; ++ob) dw[ob] = mma16(read.column(xt + 16 * k * Reader::kRowBytes, 0, 32 * ob), low, dw[ob]);
      }
    }
  }
  if (item >= a.items) return;
  if (a.item_splits > 1) {
    float* to = a.item_parts + (static_cast<int64_t>(split) * a.items + item) * D;
#pragma unroll
    for (int ob = 0; ob < OB; ++ob) store_block(to, dw[ob], 1.f, 32 * ob, a.d, true, g);
  } else {
    T* to = static_cast<T*>(a.dw) + static_cast<int64_t>(item) * a.d;
#pragma unroll
    for (int ob = 0; ob < OB; ++ob) store_block(to, dw[ob], 1.f, 32 * ob, a.d, a.quads, g);
  }
}

template <typename T, int D>
__device__ __forceinline__ void fold_items(const Args& a, unsigned block, int groups) {
  const Folder<D> at(groups);
  const int64_t item = static_cast<int64_t>(block) * at.rows + at.row;
  const bool live = item < a.items && 4 * at.t < a.d;
  const f32x4 sum = at.sum(a.item_parts + item * D, static_cast<int64_t>(a.items) * D, a.item_splits, groups, live);
  if (live && at.group == 0) store_four(static_cast<T*>(a.dw) + item * a.d, sum, 4 * at.t, a.d, a.quads);
}

// Both gradients in one launch (neither needs the other): `item_blocks` workgroups hold items, the others rows.
template <typename T, int C, int STEP>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void catalogue_gradients_kernel(Args a, unsigned item_blocks) {
  extern __shared__ __align__(1024) unsigned char smem[];
  if (blockIdx.x < item_blocks) items_gradient<T, C, STEP>(a, blockIdx.x, smem);
  else rows_gradient<T, C, STEP>(a, blockIdx.x - item_blocks, smem);
}
template <typename T, int D>
__global__ __launch_bounds__(256) void catalogue_fold_kernel(Args a, unsigned item_blocks, int item_groups, int row_groups) {
  if (blockIdx.x < item_blocks) fold_items<T, D>(a, blockIdx.x, item_groups);
  else fold_rows<T, D>(a, blockIdx.x - item_blocks, row_groups);
}


// The streamed side cut into chunks so that the workgroups fill the chip: `tiles` of the side that stays, `length` of the other.
// But a chunk's sums, `floats` of them, are written and read again at some 4.5 TB/s: no more chunks than the square root of the steps'
// time over that of one chunk's sums, where the two times' sum is least, rounded down unless near the next.  (A step takes about
// D / 128 us in bf16, half as long again in fp32.  12093 rows over 293 items, d = 256: 82 us with a chunk for every step, 68 so; 1003
// over 20011 in fp32 142 and 132.)
struct Cut {
  int splits, chunk;
};
Cut cut(int64_t tiles, int64_t length, int step, int64_t want, int64_t floats, double step_us) {
  int64_t splits = tiles >= want ? 1 : (want + tiles - 1) / tiles;
  const int64_t steps = (length + step - 1) / step;
  const double sums_us = floats * 8 / 4.5e6, least = std::sqrt(steps * step_us / sums_us);
  splits = std::max<int64_t>(1, std::min({splits, steps, static_cast<int64_t>(std::min(least + 0.2, 1e6))}));
  int64_t chunk = (length + splits - 1) / splits;
  chunk = (chunk + step - 1) / step * step;
  return {static_cast<int>((length + chunk - 1) / chunk), static_cast<int>(chunk)};
}

struct Plan {
  Cut rows, items;  // of the kernels that hold rows (chunks of items), that hold items (chunks of rows)
  size_t live, packed, listed, parts, item_parts, bytes;
};
Plan plan_of(int64_t rows, int items, int d, int dtype, bool backward) {
  Plan p{};
  const int step = dtype == 1 ? 64 : 32, D = tile_width(d);
  // (up to 64 columns a unit has room for four workgroups, but for three of the gradients' at 33 to 64, whose registers the fourth waits for:
  // 20000 rows over 20000 items, d = 64, both directions, 369 us with two, 325 with four)
  const int64_t want = (D <= 64 ? 4 : 2) * static_cast<int64_t>(compute_units());
  const double step_us = D / 128. * (dtype == 1 ? 1 : 1.5);
  p.rows = cut((rows + 127) / 128, items, step, want, rows * (backward ? D : 2), step_us);
  p.items = cut((static_cast<int64_t>(items) + 127) / 128, rows, step, want, static_cast<int64_t>(items) * D, step_us);
  p.live = align_up((rows + 1) * sizeof(int32_t));
  p.packed = backward ? align_up(static_cast<size_t>(rows) * d * (dtype == 1 ? 2 : 4)) : 0;
  p.listed = align_up(rows * sizeof(float));
  p.parts = align_up(static_cast<size_t>(p.rows.splits) * rows * (backward ? D : 2) * sizeof(float));
  p.item_parts = backward && p.items.splits > 1 ? align_up(static_cast<size_t>(p.items.splits) * items * D * sizeof(float)) : 0;
  p.bytes = p.live + p.packed + (backward ? 5 : 1) * p.listed + p.parts + p.item_parts;
  return p;
}

bool multiple(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

Args args_of(const CatalogueLoss& x, const Plan& p, bool backward, void* workspace) {
  const size_t e = x.dtype == 1 ? 2 : 4;
  Args a{};
  a.x = x.X, a.w = x.W, a.targets = x.targets, a.loss = x.loss, a.lse = x.lse, a.dloss = x.dloss, a.dx = x.dX, a.dw = x.dW;
  a.item_tiles = Divisor((static_cast<uint32_t>(x.items) + 127) / 128);
  a.rows = x.rows, a.items = x.items, a.d = x.d, a.scale = x.scale;
  a.x_pieces = multiple(x.X, 16) && x.d * e % 16 == 0, a.w_pieces = multiple(x.W, 16) && x.d * e % 16 == 0;
  a.quads = x.d % 4 == 0 && multiple(x.dW, 16) && multiple(x.dX, 16);
  char* at = static_cast<char*>(workspace);
  a.live = reinterpret_cast<int32_t*>(at), at += p.live;
  a.packed = at, at += p.packed;
  if (backward) {
    a.c_lse2 = reinterpret_cast<float*>(at), at += p.listed;
    a.c_g = reinterpret_cast<float*>(at), at += p.listed;
    a.c_e = reinterpret_cast<float*>(at), at += p.listed;
    a.c_target = reinterpret_cast<int32_t*>(at), at += p.listed;
    a.c_place = reinterpret_cast<int32_t*>(at), at += p.listed;
  } else {
    a.c_logit = reinterpret_cast<float*>(at), at += p.listed;
  }
  a.parts = reinterpret_cast<float*>(at), at += p.parts;
  a.item_parts = reinterpret_cast<float*>(at);
  a.splits = p.rows.splits, a.chunk = p.rows.chunk, a.item_splits = p.items.splits, a.item_chunk = p.items.chunk;
  return a;
}

template <typename T, bool BACKWARD>
hipError_t gather(const Args& a, hipStream_t s) {
  const int64_t each = std::max<int64_t>(16, (a.rows + compute_units() - 1) / compute_units());
  hipLaunchKernelGGL((gather_kernel<T, BACKWARD>), dim3(static_cast<unsigned>((a.rows + each - 1) / each)), dim3(64 * kGatherWaves), 0, s, a, each);
  return hipGetLastError();
}

template <typename K, typename... A>
hipError_t launch(PerDevice& granted, K kernel, int64_t blocks, int lds, hipStream_t s, A... args) {
  if (hipError_t e = allow_lds(granted, reinterpret_cast<const void*>(kernel), lds); e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3(static_cast<unsigned>(blocks)), dim3(256), lds, s, args...);
  return hipGetLastError();
}

template <typename T, int C>
hipError_t forward(const Args& a, hipStream_t s) {
  constexpr int D = tile_width(C);
  constexpr int STEP = sizeof(T) == 2 ? 64 : 32;
  if (a.rows > kFewRows)
    if (hipError_t e = gather<T, false>(a, s); e != hipSuccess) return e;
  static PerDevice granted;
  if (hipError_t e = launch(granted, catalogue_lse_kernel<T, C, STEP>, (a.rows + 127) / 128 * (a.splits + 1), Stages<T, D, STEP, 1>::kBytes, s, a); e != hipSuccess) return e;
  hipLaunchKernelGGL(catalogue_loss_kernel, dim3(static_cast<unsigned>((a.rows + 3) / 4)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T, int C>
hipError_t backward(const Args& a, hipStream_t s) {
  constexpr int D = tile_width(C);
  constexpr int STEP = sizeof(T) == 2 ? 64 : 32;
  if (hipError_t e = gather<T, true>(a, s); e != hipSuccess) return e;
  const int64_t item_blocks = a.dw ? (static_cast<int64_t>(a.items) + 127) / 128 * a.item_splits : 0, row_blocks = a.dx ? (a.rows + 127) / 128 * a.splits : 0;
  constexpr int lds = Stages<T, D, STEP, 1, 4>::kBytes;
  static PerDevice granted;
  if (hipError_t e = launch(granted, catalogue_gradients_kernel<T, C, STEP>, item_blocks + row_blocks, lds, s, a, static_cast<unsigned>(item_blocks)); e != hipSuccess) return e;
  const int item_groups = fold_groups(a.item_splits, D / 4), row_groups = fold_groups(a.splits, D / 4);
  auto folds = [](int64_t rows, int groups) { const int64_t per = 256 / (D / 4) / groups; return (rows + per - 1) / per; };
  const int64_t item_folds = a.dw && a.item_splits > 1 ? folds(a.items, item_groups) : 0, row_folds = a.dx ? folds(a.rows, row_groups) : 0;
  if (item_folds + row_folds == 0) return hipSuccess;
  hipLaunchKernelGGL((catalogue_fold_kernel<T, D>), dim3(static_cast<unsigned>(item_folds + row_folds)), dim3(256), 0, s, a, static_cast<unsigned>(item_folds), item_groups,
                     row_groups);
  return hipGetLastError();
}

// f(width) for the narrowest width of products that there is for d columns.  (224 was made for d = 200; d from 129 to 192 have none of their
// own and do up to 56 % more products than they need.)
template <typename F>
hipError_t at_width(int d, F f) {
  if (d <= 32) return f(std::integral_constant<int, 32>{});
  if (d <= 64) return f(std::integral_constant<int, 64>{});
  if (d <= 96) return f(std::integral_constant<int, 96>{});
  if (d <= 128) return f(std::integral_constant<int, 128>{});
  if (d <= 224) return f(std::integral_constant<int, 224>{});
  return f(std::integral_constant<int, 256>{});
}

}  // namespace

bool catalogue_loss_fits(int64_t rows, int items) {  // 2^32 work items a launch
  return rows < (int64_t{1} << 25) && items <= (1 << 30);
}

size_t catalogue_loss_workspace(int64_t rows, int items, int d, int dtype, bool backward) { return plan_of(rows, items, d, dtype, backward).bytes; }

hipError_t catalogue_loss(const CatalogueLoss& x, void* workspace, hipStream_t s) {
  const Plan p = plan_of(x.rows, x.items, x.d, x.dtype, false);
  const Args a = args_of(x, p, false, workspace);
  return at_width(x.d, [&](auto width) { return x.dtype == 1 ? forward<bf16_t, width.value>(a, s) : forward<float, width.value>(a, s); });
}

hipError_t catalogue_loss_backward(const CatalogueLoss& x, void* workspace, hipStream_t s) {
  const Plan p = plan_of(x.rows, x.items, x.d, x.dtype, true);
  const Args a = args_of(x, p, true, workspace);
  return at_width(x.d, [&](auto width) { return x.dtype == 1 ? backward<bf16_t, width.value>(a, s) : backward<float, width.value>(a, s); });
}

}  // namespace lime
