// Softmax attention over packed sequences with grouped heads:
//   O_i = sum_j p_ij V_j,   p_ij = exp(scale <Q_i, K_j> - lse_i),   lse_i = log sum_j exp(scale <Q_i, K_j>)   over the keys j that i sees.
// One pass over the keys with a running maximum m and sum l (everything in base 2): S^T = K Q^T block by block, so that a lane
// holds one query row and the softmax's statistics are the lane's own and its partner's; p = exp2(S c - m) rounded to the storage
// type is, as it stands, the operand of O^T += V^T P^T.  The rows of a workgroup are pairs (query, head of the group) that share a
// key head, in memory order: a tile of keys and values is read once for a whole group, in a prompt as for a single query.
// (Half a step of each p, of terms that fp32 sums hold, over the sum of the unrounded ones: against 64 bits O is off by 0.0023 of itself
// where fp32 p would leave the 0.0017 of its own rounding.)
// Bound by the vector units (a step's exponentials, scalings, maxima and sums are 930 of their cycles beside 512 of the matrix units at
// d/h = 64) and, with few rows, by the latency of a step: 16 causal histories of 4096 events, four heads on two, d/h = 64 160 us,
// 860 TFLOP/s; d/h = 128 275 us, 1 PFLOP/s; four users' single events over up to 131072 keys, d/h = 128: 4.1 TB/s.
#include <algorithm>

#include "fold.hpp"
#include "sequences.hpp"

namespace lime {
namespace {

struct Args {
  const void *q, *k, *v;
  int64_t q_stride, k_stride, v_stride;  // elements
  Packing where;
  Deal deal;
  void* o;
  float* lse;
  float *part_o, *part_ml;  // splits > 1: [splits][B][hk][max_q group][padded dh], [...][2]
  Divisor group, splits;    // query heads of a key head; chunks of the keys
  int B, hq, hk, dh, tiles, chunk;
  float c;                  // |scale| log2 e
  bool negate, pieces, causal, quads;
};

// The running maximum is raised, and what has been summed scaled down, only where a row's logits have outgrown it by more than
// this (a factor of 2^8 in p, which neither fp32 sums nor the rounding of p mind): rarely after a row's first tiles.
constexpr float kHeadroom = 8.f;

// WAVES waves of 32 rows each; KEYS keys a step.
template <typename T, int C, int WAVES, int KEYS>
__global__ __launch_bounds__(WAVES * 64) void sequence_attention_kernel(Args a) {
  constexpr int DH = tile_width(C);
  using Stage = Stages<T, DH, KEYS, 2>;  // keys, values
  using Loader = TileLoader<T, DH, KEYS, WAVES>;
  using Reader = TileReader<T, DH, KEYS>;
  constexpr int KB = KEYS / 32, OB = (C + 31) / 32, NK = C / 16, ROWS = 32 * WAVES;
  extern __shared__ __align__(1024) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, g = lane >> 5;
  const Reader read(lane);
  // last tiles of rows first: under a causal mask the longest
  const auto [b, kv, pair] = pair_of(a.deal);
  const int pairs = a.deal.pairs.d, group = a.group.d, splits = a.splits.d;
  const int reversed = splits > 1 ? a.splits.divide(blockIdx.z) : blockIdx.z, split = blockIdx.z - reversed * splits, tile = a.tiles - 1 - reversed;
  const auto [qs, ks] = spans_of(a.where, b);
  const int r0 = tile * ROWS, slot_rows = qs.slot * group, used_rows = qs.used * group;
  if (r0 >= slot_rows) return;
  // this lane's row
  const int r = r0 + 32 * wave + n, query = a.group.divide(r), head = kv * group + r - query * group;
  const bool live = r < used_rows;
  const int n_q = qs.used, n_k = ks.used;
  const int limit = live ? keys_seen(query, n_q, n_k, a.causal) : 0;
  // the furthest any row of the wave, of the workgroup, sees, and the least that a live row of the wave does
  auto last_limit = [&, n_q = n_q, n_k = n_k](int rows_end) { return rows_end > 0 ? keys_seen(a.group.divide(rows_end - 1), n_q, n_k, a.causal) : 0; };
  const int w0 = r0 + 32 * wave, wave_most = w0 < used_rows ? last_limit(min(w0 + 32, used_rows)) : 0;
  const int wave_least = w0 + 32 <= used_rows ? keys_seen(a.group.divide(w0), n_q, n_k, a.causal) : 0;
  const int most = r0 < used_rows ? last_limit(min(r0 + ROWS, used_rows)) : 0;
  // (no sum a chunk past the last key: there may be nearly 2^31)
  const int k_begin = split * a.chunk, k_end = splits > 1 ? k_begin + min(most - k_begin, a.chunk) : most;
  const int steps = k_end > k_begin ? (k_end - k_begin + KEYS - 1) / KEYS : 0;

  const T* kp = static_cast<const T*>(a.k) + (ks.start + k_begin) * a.k_stride + kv * a.dh;
  const T* vp = static_cast<const T*>(a.v) + (ks.start + k_begin) * a.v_stride + kv * a.dh;
  const unsigned width = a.dh * sizeof(T);
  const Rows km{kp, static_cast<unsigned>(a.k_stride * sizeof(T)), width, a.pieces}, vm{vp, static_cast<unsigned>(a.v_stride * sizeof(T)), width, a.pieces};
  Loader kl, vl;
  kl.init(km, tid), vl.init(vm, tid);
  auto ask = [&](int i) {
    kl.issue(km, i * KEYS, k_end - k_begin, Stage::tile(smem, i, 0), tid);
    vl.issue(vm, i * KEYS, k_end - k_begin, Stage::tile(smem, i, 1), tid);
  };
  if (steps > 0) ask(0);

  Fragment<T> q[NK];
  const T* qp = static_cast<const T*>(a.q) + (qs.start + query) * a.q_stride + head * a.dh;
  load_row<T, C>(qp, width, a.pieces, live, g, q);
  if (a.negate) {
#pragma unroll
    for (int kk = 0; kk < NK; ++kk) negate(q[kk]);
  }
  f32x16 o[OB];
#pragma unroll
  for (int ob = 0; ob < OB; ++ob) o[ob] = zero_block();
  float m = -INFINITY, l = 0.f;  // of this lane's row; l of the lane half's keys

  for (int i = 0; i < steps; ++i) {
    Stage::template arrive<WAVES>(smem, tid);
    if (i + 1 < steps) ask(i + 1);
    const int key0 = k_begin + i * KEYS;
    if (key0 >= wave_most) continue;
    const unsigned kt = Stage::operand(smem, i, 0), vt = Stage::operand(smem, i, 1);
    f32x16 s[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      s[kb] = zero_block();
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) s[kb] = mma16(read.row(kt, 32 * kb, kk), q[kk], s[kb]);
    }
    if (key0 + KEYS > wave_least) {
      seldom();
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int x = 0; x < 16; ++x)
          if (key0 + 32 * kb + block_row(x, g) >= limit) s[kb][x] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int x = 0; x < 16; ++x) top = fmaxf(top, s[kb][x]);
    top = pair_max(top) * a.c;
    if (__any(top > m + kHeadroom)) {
      seldom();
      const float to = fmaxf(m, top), f = to == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - to);
      m = to, l *= f;
#pragma unroll
      for (int ob = 0; ob < OB; ++ob)
#pragma unroll
        for (int x = 0; x < 16; ++x) o[ob][x] *= f;
    }
    const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
#pragma unroll
      for (int x = 0; x < 16; ++x) {
        s[kb][x] = __builtin_amdgcn_exp2f(fmaf(s[kb][x], a.c, -base));
        l += s[kb][x];
      }
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const Fragment<T> p = half_fragment<T>(s[kb], f);
#pragma unroll
        for (int ob = 0; ob < OB; ++ob) o[ob] = mma16(read.column(vt, 32 * kb + 16 * f, 32 * ob), p, o[ob]);
      }
    }
  }
  l = pair_sum(l);
  if (r >= slot_rows) return;
  if (splits > 1) {
    const int64_t at = (static_cast<int64_t>(split) * pairs + pair) * (static_cast<int64_t>(a.where.max_q) * group) + r;
#pragma unroll
    for (int ob = 0; ob < OB; ++ob) store_block(a.part_o + at * DH, o[ob], 1.f, 32 * ob, a.dh, true, g);
    if (g == 0) a.part_ml[at * 2] = m, a.part_ml[at * 2 + 1] = l;
    return;
  }
  const float inverse = l == 0.f ? 0.f : 1.f / l;
  const int64_t row = (qs.start + query) * a.hq + head;
  T* op = static_cast<T*>(a.o) + row * a.dh;
#pragma unroll
  for (int ob = 0; ob < OB; ++ob) store_block(op, o[ob], inverse, 32 * ob, a.dh, a.quads, g);
  if (a.lse != nullptr && g == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// The chunks' states of a row folded (see fold.hpp).
template <typename T, int DH>
__global__ __launch_bounds__(256) void sequence_attention_merge_kernel(Args a, int groups) {
  __shared__ f32x4 met[256];
  __shared__ float met_m[256], met_l[256];
  const Folder<DH> at(groups);
  const int kv = blockIdx.x, b = blockIdx.y, pairs = a.deal.pairs.d, pair = b * a.hk + kv, group = a.group.d, splits = a.splits.d;
  const int r = blockIdx.z * at.rows + at.row;
  const Span qs = spans_of(a.where, b).q;
  const bool live = r < qs.slot * group && 4 * at.t < a.dh;
  const int64_t each = static_cast<int64_t>(a.where.max_q) * group, step = pairs * each, state = pair * each + r;
  float m = -INFINITY, l = 0.f;
  f32x4 o = {0, 0, 0, 0};
  auto add = [&](float m1, float l1, const f32x4& o1) {
    const float to = fmaxf(m, m1), base = to == -INFINITY ? 0.f : to;
    const float f0 = __builtin_amdgcn_exp2f(m - base), f1 = __builtin_amdgcn_exp2f(m1 - base);
    m = to, l = l * f0 + l1 * f1;
#pragma unroll
    for (int j = 0; j < 4; ++j) o[j] = o[j] * f0 + o1[j] * f1;
  };
  if (live) {
#pragma unroll 4
    for (int s = at.group; s < splits; s += groups) {
      const float2 ml = *reinterpret_cast<const float2*>(a.part_ml + (state + s * step) * 2);
      add(ml.x, ml.y, *reinterpret_cast<const f32x4*>(a.part_o + (state + s * step) * DH + 4 * at.t));
    }
  }
  for (int half = groups / 2; half; half /= 2) {
    __syncthreads();
    met[threadIdx.x] = o, met_m[threadIdx.x] = m, met_l[threadIdx.x] = l;
    __syncthreads();
    if (at.group < half) {
      const int other = threadIdx.x + half * Folder<DH>::kLanes;
      add(met_m[other], met_l[other], met[other]);
    }
  }
  if (!live || at.group != 0) return;
  const float inverse = l == 0.f ? 0.f : 1.f / l;
  const int query = a.group.divide(r);
  const int64_t row = (qs.start + query) * a.hq + kv * group + r - query * group;
#pragma unroll
  for (int j = 0; j < 4; ++j) o[j] *= inverse;
  store_four(static_cast<T*>(a.o) + row * a.dh, o, 4 * at.t, a.dh, a.quads);
  if (a.lse != nullptr && at.t == 0) a.lse[row] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Keys a step of four waves: as many as leave a compute unit four workgroups' registers and LDS.  (Up to 256 events of 64 users, d/h = 32:
// 8.9 us in steps of 64 keys, 8.5 of 128; 16 of 2048 to 4096 events, d/h = 64: 113 and 122.)
constexpr int keys_of(bool bf16, int dh) { return !bf16 ? 32 : dh <= 32 ? 128 : 64; }

struct Plan {
  int waves, keys, splits, chunk, dh;  // dh: padded
  int64_t tiles;  // (the workspace's size is answered also where they pass what a launch takes)
  size_t o_bytes, bytes;
};

// Rows that one wave holds take a workgroup of one wave.  Where the tiles of rows are too few to fill the chip, the keys are cut
// into chunks as well.  A lone wave needs about 1600 cycles for a step of 32 keys, most of them waiting for itself, and 4600 to start
// and to end: so eight waves a compute unit are wanted, but no more chunks than four steps (fp32, where a step takes 4 us at d/h = 128: one)
// go into the keys, and no more than 256 of a row, which have to be folded again.  (32 users, up to 4096 keys: 14.6 us in chunks of 128 keys, 15.8 of
// 256; four users of up to 131072: 53 us in 512 chunks, 49 in 256; fp32, two users, up to 249 keys: 27.9 us in chunks of 128, 12.5 of
// 32.  More tiles in flight take the LDS of the other waves: three 16.0, four 15.7 and 51.9.)  Of workgroups of four waves, two a
// compute unit, but no more chunks than 256 keys (fp32: 128) go into the keys.  Chunks are of whole steps and as long as each other but for the
// last, so that 257 keys in two are 192 and 65.  (8 users' up to 64 new events over up to 8192 keys: 17.6 us, 19.0 with one workgroup
// a unit or 512 keys, 23 with four and 128; five users' up to 501 events in fp32: 21.2 us, 24.5 with 256.)
Plan plan_of(const SequenceAttention& a) {
  const int64_t B = a.B, hk = a.hk, max_k = std::max(a.max_k, 1), rows = std::max<int64_t>(a.max_q, 1) * (a.hq / a.hk);
  const int dh = a.dh, dtype = a.dtype;
  Plan p{};
  p.dh = tile_width(dh);
  p.waves = rows <= 32 ? 1 : 4;
  p.keys = p.waves > 1 ? keys_of(dtype == 1, p.dh) : 32;
  p.tiles = (rows + 32 * p.waves - 1) / (32 * p.waves);
  const int64_t groups = B * hk * p.tiles;
  const int64_t want = (p.waves == 1 ? 8 : 2) * static_cast<int64_t>(compute_units());
  const int64_t least = p.waves == 1 ? std::max<int64_t>(dtype == 1 ? 128 : 32, (max_k + 255) / 256) : dtype == 1 ? 256 : 128;
  int64_t splits = groups >= want ? 1 : std::min((want + groups - 1) / groups, (max_k + least - 1) / least);
  int64_t chunk = (max_k + splits - 1) / splits;
  chunk = (chunk + p.keys - 1) / p.keys * p.keys;
  splits = (max_k + chunk - 1) / chunk;
  p.chunk = static_cast<int>(std::min<int64_t>(chunk, (int64_t{1} << 31) - 1)), p.splits = static_cast<int>(splits);
  if (p.splits > 1) {
    const size_t states = static_cast<size_t>(p.splits) * B * hk * rows;
    p.o_bytes = align_up(states * p.dh * sizeof(float));
    p.bytes = p.o_bytes + align_up(states * 2 * sizeof(float));
  }
  return p;
}

template <typename T, int C, int WAVES, int KEYS>
hipError_t launch(const Args& a, hipStream_t s) {
  constexpr int DH = tile_width(C);
  constexpr int lds = Stages<T, DH, KEYS, 2>::kBytes;
  static PerDevice granted;
  const auto kernel = sequence_attention_kernel<T, C, WAVES, KEYS>;
  if (hipError_t e = allow_lds(granted, reinterpret_cast<const void*>(kernel), lds); e != hipSuccess) return e;
  hipLaunchKernelGGL(kernel, dim3(a.hk, a.B, a.tiles * a.splits.d), dim3(WAVES * 64), lds, s, a);
  return hipGetLastError();
}

template <typename T, int C>
hipError_t run(const Args& a, const Plan& p, hipStream_t s) {
  constexpr int DH = tile_width(C), KEYS = keys_of(sizeof(T) == 2, DH);
  hipError_t e = p.waves == 1 ? launch<T, C, 1, 32>(a, s) : launch<T, C, 4, KEYS>(a, s);
  if (e != hipSuccess || a.splits.d == 1) return e;
  const int groups = fold_groups(a.splits.d, DH / 4);
  const int64_t rows = static_cast<int64_t>(a.where.max_q) * a.group.d, per = 256 / (DH / 4) / groups;
  hipLaunchKernelGGL((sequence_attention_merge_kernel<T, DH>), dim3(a.hk, a.B, static_cast<unsigned>((rows + per - 1) / per)), dim3(256), 0, s, a, groups);
  return hipGetLastError();
}

bool multiple(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

}  // namespace

constexpr int64_t kMostKeys = (int64_t{1} << 31) - 256;  // a step past them is still a number of 32 bits

bool sequence_attention_fits(const SequenceAttention& a) {  // 2^32 work items a launch, 65535 workgroups along the grid's third axis
  const int64_t rows = static_cast<int64_t>(a.max_q) * (a.hq / a.hk), pairs = static_cast<int64_t>(a.B) * a.hk;
  if (rows >= (int64_t{1} << 31) - 128 || pairs >= (int64_t{1} << 24) || a.max_k > kMostKeys) return false;
  const Plan p = plan_of(a);
  const int64_t deep = p.tiles * p.splits;
  return deep < 65536 && pairs * deep < (int64_t{1} << 26) / p.waves;  // (where keys are cut, pairs times rows are less than 2^17)
}

size_t sequence_attention_workspace(const SequenceAttention& a) { return std::max<size_t>(plan_of(a).bytes, 256); }

hipError_t sequence_attention(const SequenceAttention& x, void* workspace, hipStream_t s) {
  const Plan p = plan_of(x);
  const size_t e = x.dtype == 1 ? 2 : 4;
  Args a{};
  // (Chunks of a few rows move where a pair's would otherwise all land on one XCD.  Others stay: the merge reads their states from the
  // same L2.  32 users of two key heads, up to 4096 keys: 13.7 us, 14.5 unmoved; four users' chunks of up to 131072 keys, 50.5 and 48.9,
  // and of 64 events each 18.5 and 17.5.)
  a.q = x.Q, a.k = x.K, a.v = x.V, a.q_stride = x.q_stride, a.k_stride = x.k_stride, a.v_stride = x.v_stride;
  a.where = Packing(x), a.deal = Deal(x, p.splits == 1 || (p.waves == 1 && x.B * x.hk % 8 == 0)), a.o = x.O, a.lse = x.lse;
  a.part_o = static_cast<float*>(workspace), a.part_ml = reinterpret_cast<float*>(static_cast<char*>(workspace) + p.o_bytes);
  a.B = x.B, a.hq = x.hq, a.hk = x.hk, a.dh = x.dh;
  a.group = Divisor(x.hq / x.hk), a.splits = Divisor(p.splits), a.tiles = static_cast<int>(p.tiles), a.chunk = p.chunk;
  a.c = std::max(fabsf(x.scale) * kLog2e, 1e-37f), a.negate = x.scale < 0.f, a.causal = x.causal != 0;
  a.pieces = multiple(x.Q, 16) && multiple(x.K, 16) && multiple(x.V, 16) && x.dh * e % 16 == 0 && x.q_stride * e % 16 == 0 &&
             x.k_stride * e % 16 == 0 && x.v_stride * e % 16 == 0;
  a.quads = x.dh % 4 == 0 && multiple(x.O, 4 * e);
  return at_head_width(x.dh, [&](auto width) { return x.dtype == 1 ? run<bf16_t, width.value>(a, p, s) : run<float, width.value>(a, p, s); });
}

}  // namespace lime
