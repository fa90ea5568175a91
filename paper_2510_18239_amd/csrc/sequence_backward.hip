// Gradients of the attention over packed sequences, with the attention matrix recomputed from the forward pass's lse: for G = dL/dO,
//   p_ij = exp(scale <Q_i, K_j> - lse_i),  D_i = <G_i, O_i>,  e_ij = p_ij (<G_i, V_j> - D_i):
//   dQ_i = scale sum_j e_ij K_j,   dK_j = scale sum_i e_ij Q_i,   dV_j = sum_i p_ij G_i   (i over all heads that share the key head).
// Two kernels, each with one side's rows and sums in registers while the other side's tiles stream past, so that every sum has one
// owner and one order (no atomics): the first holds queries (rows as in the forward pass) and also leaves -D and lse, by head, for
// the second, which holds keys.  A kernel that kept both sides' sums would do five products of the tiles where these do seven or eight: the
// sums of the other side would have to meet in memory.  Where the workgroups of a side are too few for the chip, the side that streams past is
// cut into chunks whose sums a third kernel folds (fold.hpp).  p and e are rounded to the storage type, as operands of the last products
// (half a step of each, of terms that are summed in fp32).
// D is held in fp32, and an O of bf16 gives it only to 2^-8 of <|G|, |O|>, which may be more than all of e: of a row whose softmax is
// nearly decided, that sees few keys, or whose values have a large part in common.  (One key of 300 to 2000 with p up to 0.9999, or values
// of 8 + noise: dQ off by as much as itself to ten times that.)  So the first kernel takes e from that D, sums e on the way, gap_i = sum_j e_ij,
// which is what D lacks, and takes gap_i sum_j p_ij K_j off its sums at the end, one more product of the key tile that it has; the
// second gets the whole D.  (16 causal histories of 4096 events, four heads on two, d/h = 64, forward and gradients: 660 us without, 708 with.
// D from products of its own beforehand would be two more.)
// Bound by the two units waiting for each other: matrix cores busy 45 and 38 % of the time in the two kernels, the vector units about half
// (of the second, at d/h = 64: 512 cycles of products and some 620 of exponentials, products and rounding a block of 32 queries, which takes
// 1350; two waves a SIMD are not enough to cover for each other).  16 causal histories of 4096 events, four heads on two, d/h = 64
// 550 us, 1 PFLOP/s of the eight products, 625 TFLOP/s of the five; d/h = 128 1160 us, 945 and 590.
#include <algorithm>

#include "fold.hpp"
#include "sequences.hpp"

namespace lime {
namespace {

struct Args {
  const void *q, *k, *v, *o, *go;
  int64_t q_stride, k_stride, v_stride, dq_stride, dk_stride, dv_stride;  // elements
  Packing where;
  Deal deal;
  const float* lse;
  float *lse2, *less;  // [hq][q_rows]: lse log2 e, -D
  void *dq, *dk, *dv;
  float *part_q, *part_gap, *part_kv;  // chunks > 1: [q_splits][1 or 2][q_rows][hq][padded dh], [q_splits][q_rows][hq], [k_splits][2][k_rows][hk][padded dh]
  Divisor group, q_splits, k_splits;
  int hq, hk, dh, tiles;
  int q_chunk, k_chunk;  // chunks of keys (in keys), and of the steps over queries
  float scale;
  bool pieces, causal, quads;
};

// Whether O has been rounded to fewer bits than D is held in.
template <typename T>
constexpr bool kRounded = sizeof(T) == 2;
// Whether the kernel that holds queries has to save registers for a second wave a SIMD: block by block, and with D taken off <G, V> where its
// sums would start from a block of -D.  (16 causal histories of 4096 events, forward and gradients: d/h = 128 1518 us without, 1435 so;
// 96 1152 and 1062; at 64 there are two waves in any case, 708 and 730.)
template <typename T, int C>
constexpr bool kTight = sizeof(T) == 2 && C > 80;

template <typename T, int C, int WAVES, int KEYS>
__global__ __launch_bounds__(WAVES * 64, (kTight<T, C> ? 2 : 1)) void sequence_attention_dq_kernel(Args a) {
  constexpr int DH = tile_width(C);
  using Stage = Stages<T, DH, KEYS, 2>;  // keys, values
  using Loader = TileLoader<T, DH, KEYS, WAVES>;
  using Reader = TileReader<T, DH, KEYS>;
  constexpr int KB = KEYS / 32, OB = (C + 31) / 32, NK = C / 16, ROWS = 32 * WAVES;
  extern __shared__ __align__(1024) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, g = lane >> 5;
  const Reader read(lane);
  const auto [b, kv, pair] = pair_of(a.deal);
  const int group = a.group.d, splits = a.q_splits.d;
  const int reversed = splits > 1 ? a.q_splits.divide(blockIdx.z) : blockIdx.z, split = blockIdx.z - reversed * splits, tile = a.tiles - 1 - reversed;
  const auto [qs, ks] = spans_of(a.where, b);
  const int r0 = tile * ROWS, slot_rows = qs.slot * group, used_rows = qs.used * group;
  if (r0 >= slot_rows) return;
  const int r = r0 + 32 * wave + n, query = a.group.divide(r), head = kv * group + r - query * group;
  const bool live = r < used_rows;
  const int n_q = qs.used, n_k = ks.used;
  const int limit = live ? keys_seen(query, n_q, n_k, a.causal) : 0;
  auto last_limit = [&, n_q = n_q, n_k = n_k](int rows_end) { return rows_end > 0 ? keys_seen(a.group.divide(rows_end - 1), n_q, n_k, a.causal) : 0; };
  const int w0 = r0 + 32 * wave, wave_most = w0 < used_rows ? last_limit(min(w0 + 32, used_rows)) : 0;
  const int wave_least = w0 + 32 <= used_rows ? keys_seen(a.group.divide(w0), n_q, n_k, a.causal) : 0;
  const int most = r0 < used_rows ? last_limit(min(r0 + ROWS, used_rows)) : 0;
  const int k_begin = split * a.q_chunk, k_end = min(most, k_begin + a.q_chunk), steps = k_end > k_begin ? (k_end - k_begin + KEYS - 1) / KEYS : 0;

  const unsigned width = a.dh * sizeof(T);
  const Rows km{static_cast<const T*>(a.k) + (ks.start + k_begin) * a.k_stride + kv * a.dh, static_cast<unsigned>(a.k_stride * sizeof(T)), width, a.pieces};
  const Rows vm{static_cast<const T*>(a.v) + (ks.start + k_begin) * a.v_stride + kv * a.dh, static_cast<unsigned>(a.v_stride * sizeof(T)), width, a.pieces};
  Loader kl, vl;
  kl.init(km, tid), vl.init(vm, tid);
  auto ask = [&](int i) {
    kl.issue(km, i * KEYS, k_end - k_begin, Stage::tile(smem, i, 0), tid);
    vl.issue(vm, i * KEYS, k_end - k_begin, Stage::tile(smem, i, 1), tid);
  };
  if (steps > 0) ask(0);

  const int64_t row = (qs.start + query) * a.hq + head;
  Fragment<T> q[NK], go[NK];
  load_row<T, C>(static_cast<const T*>(a.q) + (qs.start + query) * a.q_stride + head * a.dh, width, a.pieces, live, g, q);
  load_row<T, C>(static_cast<const T*>(a.go) + row * a.dh, width, a.pieces, live, g, go);
  const float c = a.scale * kLog2e, lse2 = live ? a.lse[row] * kLog2e : 0.f;
  float delta = 0.f;
  {
    Fragment<T> o[NK];
    load_row<T, C>(static_cast<const T*>(a.o) + row * a.dh, width, a.pieces, live, g, o);
#pragma unroll
    for (int kk = 0; kk < NK; ++kk)
#pragma unroll
      for (int t = 0; t < 8; ++t) delta = fmaf(element(go[kk], t), element(o[kk], t), delta);
    delta = pair_sum(delta);
  }
  f32x16 dq[OB], mean[kRounded<T> ? OB : 1], less;  // less: -D, where the sums <G_i, V_j> - D_i start from
  float gap = 0.f;  // of the lane half's keys
#pragma unroll
  for (int ob = 0; ob < OB; ++ob) {
    dq[ob] = zero_block();
    if constexpr (kRounded<T>) mean[ob] = zero_block();
  }
#pragma unroll
  for (int x = 0; x < 16; ++x) less[x] = -delta;

  for (int i = 0; i < steps; ++i) {
    Stage::template arrive<WAVES>(smem, tid);
    if (i + 1 < steps) ask(i + 1);
    const int key0 = k_begin + i * KEYS;
    if (key0 >= wave_most) continue;
    const unsigned kt = Stage::operand(smem, i, 0), vt = Stage::operand(smem, i, 1);
    const bool partial = key0 + KEYS > wave_least;
#pragma unroll(kTight<T, C> ? 1 : KB)
    for (int kb = 0; kb < KB; ++kb) {
      f32x16 s = zero_block(), e = kTight<T, C> ? zero_block() : less;
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) {
        s = mma16(read.row(kt, 32 * kb, kk), q[kk], s);
        e = mma16(read.row(vt, 32 * kb, kk), go[kk], e);
      }
#pragma unroll
      for (int x = 0; x < 16; ++x) s[x] = __builtin_amdgcn_exp2f(fmaf(s[x], c, -lse2)), e[x] = (kTight<T, C> ? e[x] - delta : e[x]) * s[x];
      if (partial) {
        seldom();
#pragma unroll
        for (int x = 0; x < 16; ++x)
          if (key0 + 32 * kb + block_row(x, g) >= limit) s[x] = 0.f, e[x] = 0.f;
      }
      if constexpr (kRounded<T>) {
#pragma unroll
        for (int x = 0; x < 16; ++x) gap += e[x];
      }
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const Fragment<T> ef = half_fragment<T>(e, f), pf = half_fragment<T>(s, f);
#pragma unroll
        for (int ob = 0; ob < OB; ++ob) {
          const Fragment<T> k = read.column(kt, 32 * kb + 16 * f, 32 * ob);
          dq[ob] = mma16(k, ef, dq[ob]);
          if constexpr (kRounded<T>) mean[ob] = mma16(k, pf, mean[ob]);
        }
      }
    }
  }
  if (r >= slot_rows) return;
  gap = pair_sum(gap);
  if (live && g == 0 && split == 0) {
    const int64_t at = head * static_cast<int64_t>(a.where.q_rows) + qs.start + query;
    a.lse2[at] = lse2, a.less[at] = splits > 1 ? -delta : -delta - gap;  // (of chunks, the fold adds the gaps)
  }
  if (splits > 1) {
    const int64_t plane = static_cast<int64_t>(a.where.q_rows) * a.hq * DH;
    float* to = a.part_q + (kRounded<T> ? 2 : 1) * split * plane + row * DH;
#pragma unroll
    for (int ob = 0; ob < OB; ++ob) {
      store_block(to, dq[ob], 1.f, 32 * ob, a.dh, true, g);
      if constexpr (kRounded<T>) store_block(to + plane, mean[ob], 1.f, 32 * ob, a.dh, true, g);
    }
    if (kRounded<T> && g == 0) a.part_gap[static_cast<int64_t>(split) * a.where.q_rows * a.hq + row] = gap;
    return;
  }
  if constexpr (kRounded<T>) {
#pragma unroll
    for (int ob = 0; ob < OB; ++ob)
#pragma unroll
      for (int x = 0; x < 16; ++x) dq[ob][x] = fmaf(-gap, mean[ob][x], dq[ob][x]);
  }
  T* out = static_cast<T*>(a.dq) + (qs.start + query) * a.dq_stride + head * a.dh;
#pragma unroll
  for (int ob = 0; ob < OB; ++ob) store_block(out, dq[ob], a.scale, 32 * ob, a.dh, a.quads, g);
}

// (bf16, d/h = 128: kept to 256 registers, with eight of a wave's loaded again for every 32 queries, for a second wave a SIMD: 120 us less
// of the 1150 that 16 causal histories of 4096 events took with one, both kernels.)
template <typename T, int C, int STEP>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 2 : 1) void sequence_attention_dkv_kernel(Args a) {
  constexpr int DH = tile_width(C);
  using Stage = Stages<T, DH, STEP, 2, 2>;  // queries, output gradients; lse2, -D
  using Loader = TileLoader<T, DH, STEP, 4>;
  using Reader = TileReader<T, DH, STEP>;
  constexpr int QB = STEP / 32, OB = (C + 31) / 32, NK = C / 16, KEYS = 128;
  extern __shared__ __align__(1024) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, g = lane >> 5;
  const Reader read(lane);
  // first keys first: under a causal mask most queries see them
  const auto [b, kv, pair] = pair_of(a.deal);
  const int group = a.group.d, splits = a.k_splits.d;
  const int tile = splits > 1 ? a.k_splits.divide(blockIdx.z) : blockIdx.z, split = blockIdx.z - tile * splits;
  const auto [qs, ks] = spans_of(a.where, b);
  const int j0 = tile * KEYS;
  if (j0 >= ks.slot) return;
  const int key = j0 + 32 * wave + n, shift = ks.used - qs.used;
  const bool live = key < ks.used;
  // the first query that sees this lane's key; that sees any of the wave's; that sees all of them
  const int first = live ? (a.causal ? max(0, key - shift) : 0) : qs.used;
  const int w0 = j0 + 32 * wave, wave_first = w0 < ks.used ? (a.causal ? max(0, w0 - shift) : 0) : qs.used;
  const int wave_all = w0 + 32 <= ks.used ? (a.causal ? max(0, w0 + 31 - shift) : 0) : qs.used;
  const int begin = (a.causal ? max(0, j0 - shift) : 0) / STEP * STEP;
  const int each = j0 < ks.used && begin < qs.used ? (qs.used - begin + STEP - 1) / STEP : 0, all = each * group;
  const int begin_step = min(all, split * a.k_chunk), steps = min(all - begin_step, a.k_chunk);

  const unsigned width = a.dh * sizeof(T);
  Rows qm{static_cast<const T*>(a.q) + (qs.start + begin) * a.q_stride + kv * group * a.dh, static_cast<unsigned>(a.q_stride * sizeof(T)), width, a.pieces};
  Rows gm{static_cast<const T*>(a.go) + ((qs.start + begin) * a.hq + kv * group) * a.dh, static_cast<unsigned>(a.hq * a.dh * sizeof(T)), width, a.pieces};
  Loader ql, gl;
  ql.init(qm, tid), gl.init(gm, tid);
  // steps are asked for one head after the other
  int ask_head = each ? begin_step / each : 0, ask_at = each ? begin_step % each * STEP : 0, at = ask_at;  // at: this step's first query, from `begin`
  qm.base = static_cast<const char*>(qm.base) + ask_head * width, gm.base = static_cast<const char*>(gm.base) + ask_head * width;
  auto ask = [&](int i) {
    const int count = qs.used - begin - ask_at;
    ql.issue(qm, ask_at, qs.used - begin, Stage::tile(smem, i, 0), tid);
    gl.issue(gm, ask_at, qs.used - begin, Stage::tile(smem, i, 1), tid);
    if (wave < 2) {
      const float* from = (wave == 0 ? a.lse2 : a.less) + (kv * group + ask_head) * static_cast<int64_t>(a.where.q_rows) + qs.start + begin + ask_at;
      words_to_lds(from, min(count, STEP), Stage::words(smem, i, wave), lane);
    }
    ask_at += STEP;
    if (ask_at >= each * STEP) {
      ask_at = 0, ++ask_head;
      qm.base = static_cast<const char*>(qm.base) + width, gm.base = static_cast<const char*>(gm.base) + width;
    }
  };
  if (steps > 0) ask(0);

  Fragment<T> k[NK], v[NK];
  load_row<T, C>(static_cast<const T*>(a.k) + (ks.start + key) * a.k_stride + kv * a.dh, width, a.pieces, live, g, k);
  load_row<T, C>(static_cast<const T*>(a.v) + (ks.start + key) * a.v_stride + kv * a.dh, width, a.pieces, live, g, v);
  const float c = a.scale * kLog2e;
  f32x16 dk[OB], dv[OB];
#pragma unroll
  for (int ob = 0; ob < OB; ++ob) dk[ob] = dv[ob] = zero_block();

  for (int i = 0; i < steps; ++i) {
    Stage::template arrive<4>(smem, tid);
    if (i + 1 < steps) ask(i + 1);
    const int q0 = begin + at;
    at = at + STEP < each * STEP ? at + STEP : 0;
    if (q0 + STEP <= wave_first) continue;
    const unsigned qt = Stage::operand(smem, i, 0), gt = Stage::operand(smem, i, 1);
    const float *lse2 = Stage::words(smem, i, 0), *less = Stage::words(smem, i, 1);
    const bool partial = q0 < wave_all || q0 + STEP > qs.used;
#pragma unroll(DH < 128 ? QB : 1)
    for (int qb = 0; qb < QB; ++qb) {
      f32x16 p = zero_block(), e;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x4 d4 = *reinterpret_cast<const f32x4*>(less + 32 * qb + 8 * j + 4 * g);
#pragma unroll
        for (int x = 0; x < 4; ++x) e[4 * j + x] = d4[x];
      }
#pragma unroll
      for (int kk = 0; kk < NK; ++kk) {
        p = mma16(read.row(qt, 32 * qb, kk), k[kk], p);
        e = mma16(read.row(gt, 32 * qb, kk), v[kk], e);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x4 l4 = *reinterpret_cast<const f32x4*>(lse2 + 32 * qb + 8 * j + 4 * g);
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          p[4 * j + x] = __builtin_amdgcn_exp2f(fmaf(p[4 * j + x], c, -l4[x]));
          e[4 * j + x] *= p[4 * j + x];
        }
      }
      if (partial) {
        seldom();
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const int query = q0 + 32 * qb + block_row(x, g);
          if (query < first || query >= qs.used) p[x] = 0.f, e[x] = 0.f;
        }
      }
#pragma unroll
      for (int f = 0; f < 2; ++f) {
        const Fragment<T> pf = half_fragment<T>(p, f), ef = half_fragment<T>(e, f);
#pragma unroll
        for (int ob = 0; ob < OB; ++ob) {
          dv[ob] = mma16(read.column(gt, 32 * qb + 16 * f, 32 * ob), pf, dv[ob]);
          dk[ob] = mma16(read.column(qt, 32 * qb + 16 * f, 32 * ob), ef, dk[ob]);
        }
      }
    }
  }
  if (key >= ks.slot) return;
  if (splits > 1) {
    const int64_t plane = static_cast<int64_t>(a.where.k_rows) * a.hk * DH;
    float* to = a.part_kv + 2 * split * plane + ((ks.start + key) * a.hk + kv) * DH;
#pragma unroll
    for (int ob = 0; ob < OB; ++ob) store_block(to, dk[ob], 1.f, 32 * ob, a.dh, true, g), store_block(to + plane, dv[ob], 1.f, 32 * ob, a.dh, true, g);
    return;
  }
  T* dk_row = static_cast<T*>(a.dk) + (ks.start + key) * a.dk_stride + kv * a.dh;
  T* dv_row = static_cast<T*>(a.dv) + (ks.start + key) * a.dv_stride + kv * a.dh;
#pragma unroll
  for (int ob = 0; ob < OB; ++ob) {
    store_block(dk_row, dk[ob], a.scale, 32 * ob, a.dh, a.quads, g);
    store_block(dv_row, dv[ob], 1.f, 32 * ob, a.dh, a.quads, g);
  }
}

// The chunks' sums folded: of dQ by the first q_blocks workgroups of a user where its keys were cut, then of dK and dV where the queries were.
template <typename T, int DH>
__global__ __launch_bounds__(256) void sequence_attention_fold_kernel(Args a, unsigned q_blocks, int q_groups, int k_groups) {
  const bool of_q = blockIdx.x < q_blocks;
  const int groups = of_q ? q_groups : k_groups;
  const Folder<DH> at(groups);
  const int block = of_q ? blockIdx.x : blockIdx.x - q_blocks, heads = of_q ? a.hq : a.hk, each = of_q ? heads : 2 * heads;
  const int tile = block / each, h = block - tile * each, what = of_q ? 0 : h < heads ? 1 : 2, head = what == 2 ? h - heads : h;
  const int b = blockIdx.y, i = tile * at.rows + at.row, splits = of_q ? a.q_splits.d : a.k_splits.d;
  const Spans spans = spans_of(a.where, b);
  const Span span = what == 0 ? spans.q : spans.k;
  const bool live = i < span.slot && 4 * at.t < a.dh;
  const int64_t rows = what == 0 ? a.where.q_rows : a.where.k_rows, row = span.start + i, plane = rows * heads * DH;
  const float* p = (what == 0 ? a.part_q : a.part_kv) + (what == 2 ? plane : 0) + (row * heads + head) * DH;
  f32x4 sum = at.sum(p, what == 0 && !kRounded<T> ? plane : 2 * plane, splits, groups, live);
  if (kRounded<T> && what == 0) {  // (the same for the whole workgroup)
    const f32x4 mean = at.sum(p + plane, 2 * plane, splits, groups, live);
    const float gap = at.sum_of([&](int s) { return f32x4{a.part_gap[(s * rows + row) * heads + head], 0, 0, 0}; }, splits, groups, live)[0];
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] = fmaf(-gap, mean[j], sum[j]);
    if (i < span.used && at.t == 0 && at.group == 0) a.less[head * rows + row] -= gap;
  }
  if (!live || at.group != 0) return;
  const float factor = what == 2 ? 1.f : a.scale;
#pragma unroll
  for (int j = 0; j < 4; ++j) sum[j] *= factor;
  T* to = static_cast<T*>(what == 0 ? a.dq : what == 1 ? a.dk : a.dv) + row * (what == 0 ? a.dq_stride : what == 1 ? a.dk_stride : a.dv_stride) + head * a.dh;
  store_four(to, sum, 4 * at.t, a.dh, a.quads);
}

struct Plan {
  int dh, q_splits, q_chunk, k_splits, k_chunk;
  int64_t q_tiles, k_tiles;  // (the workspace's size is answered also where they pass what a launch takes)
  size_t stats, part_q, part_gap, part_kv, bytes;
};

// Two workgroups of four waves a compute unit are wanted, but no more chunks than 256 keys (bf16; 128: fp32) or four steps over queries
// go into the length; chunks are of whole steps and as long as each other but for the last.
// In bf16 the fold of dQ is a launch of its own, and up to 512 keys of heads up to 64 are not cut: three users of up to 500 events, d/h = 32, 38.4 us in
// chunks of 256 and 36.2 whole; eight of 512, 64, 54.8 and 50.9; but three of up to 500, 128, 76.8 and 79.3, and with chunks of 512 two of 1000, 128,
// 72.2 and 82.1, 64 new events over 8192, d/h = 64, 44.3 and 46.8.
// Of ragged users twice as many for the kernel that holds keys: its workgroups are few, and the longest user's first keys see all of that
// user's queries of all heads of the group.  (Four users of 79 to 3983 events, eight heads on two, d/h = 80: 775 us with two a unit, 553
// with four; 52 of up to 551, eight heads on one, 122 and 103; 16 of 3129 each 314 and 342; in fp32, where a unit holds one, 162 and 177.)
Plan plan_of(const SequenceAttention& a) {
  const int64_t group = a.hq / a.hk, pairs = static_cast<int64_t>(a.B) * a.hk, max_q = std::max(a.max_q, 1), max_k = std::max(a.max_k, 1);
  const int64_t want = 2 * static_cast<int64_t>(compute_units()), step = a.dtype == 1 ? 64 : 32;
  Plan p{};
  p.dh = tile_width(a.dh);
  p.q_tiles = (max_q * group + 127) / 128, p.k_tiles = (max_k + 127) / 128;
  auto cut = [&](int64_t tiles, int64_t length, int64_t least, int64_t want, int& splits, int& chunk) {
    const int64_t most = std::max<int64_t>(1, (length + least - 1) / least), n = std::min(most, std::max<int64_t>(1, (want + pairs * tiles - 1) / (pairs * tiles)));
    const int64_t c = ((length + n - 1) / n + step - 1) / step * step;
    chunk = static_cast<int>(std::min<int64_t>(c, (int64_t{1} << 31) - 1)), splits = static_cast<int>((length + c - 1) / c);
  };
  const bool whole = a.dtype == 1 && p.dh <= 64 && max_k <= 8 * step;  // not worth the fold
  cut(p.q_tiles, max_k, whole ? max_k : 4 * step, want, p.q_splits, p.q_chunk);
  const int64_t steps = (max_q + step - 1) / step * group;
  cut(p.k_tiles, steps * step, 4 * step, ragged(a) && a.dtype == 1 ? 2 * want : want, p.k_splits, p.k_chunk);
  p.k_chunk = static_cast<int>((p.k_chunk + step - 1) / step);
  p.stats = align_up(static_cast<size_t>(a.q_rows) * a.hq * sizeof(float));
  const size_t states = p.q_splits > 1 ? static_cast<size_t>(p.q_splits) * a.q_rows * a.hq * sizeof(float) : 0;
  p.part_q = align_up(states * p.dh * (a.dtype == 1 ? 2 : 1)), p.part_gap = a.dtype == 1 ? align_up(states) : 0;
  p.part_kv = p.k_splits > 1 ? align_up(static_cast<size_t>(p.k_splits) * 2 * a.k_rows * a.hk * p.dh * sizeof(float)) : 0;
  p.bytes = std::max<size_t>(256, 2 * p.stats + p.part_q + p.part_gap + p.part_kv);
  return p;
}

template <typename T, int C>
hipError_t run(Args a, const Plan& p, int users, hipStream_t s) {
  constexpr int DH = tile_width(C), STEP = sizeof(T) == 2 ? 64 : 32;
  const int max_q = a.where.max_q, max_k = a.where.max_k;
  if (max_q > 0) {
    constexpr int lds = Stages<T, DH, STEP, 2>::kBytes;
    static PerDevice granted;
    const auto kernel = sequence_attention_dq_kernel<T, C, 4, STEP>;
    if (hipError_t e = allow_lds(granted, reinterpret_cast<const void*>(kernel), lds); e != hipSuccess) return e;
    a.tiles = static_cast<int>(p.q_tiles);
    hipLaunchKernelGGL(kernel, dim3(a.hk, users, a.tiles * p.q_splits), dim3(256), lds, s, a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  const bool q_folds = p.q_splits > 1 && max_q > 0, k_folds = p.k_splits > 1 && max_k > 0;
  const int q_groups = fold_groups(p.q_splits, DH / 4), k_groups = fold_groups(p.k_splits, DH / 4);
  auto fold = [&](bool q, bool k) {
    auto blocks = [](int rows, int groups, int heads) { const int per = 256 / (DH / 4) / groups; return static_cast<unsigned>((rows + per - 1) / per * heads); };
    const unsigned q_blocks = q ? blocks(max_q, q_groups, a.hq) : 0, k_blocks = k ? blocks(max_k, k_groups, 2 * a.hk) : 0;
    hipLaunchKernelGGL((sequence_attention_fold_kernel<T, DH>), dim3(q_blocks + k_blocks, users), dim3(256), 0, s, a, q_blocks, q_groups, k_groups);
    return hipGetLastError();
  };
  if (kRounded<T> && q_folds)  // D is whole
    if (hipError_t e = fold(true, false); e != hipSuccess) return e;
  if (max_k > 0) {
    constexpr int lds = Stages<T, DH, STEP, 2, 2>::kBytes;
    static PerDevice granted;
    const auto kernel = sequence_attention_dkv_kernel<T, C, STEP>;
    if (hipError_t e = allow_lds(granted, reinterpret_cast<const void*>(kernel), lds); e != hipSuccess) return e;
    hipLaunchKernelGGL(kernel, dim3(a.hk, users, static_cast<unsigned>(p.k_tiles * p.k_splits)), dim3(256), lds, s, a);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  const bool q_left = q_folds && !kRounded<T>;
  return q_left || k_folds ? fold(q_left, k_folds) : hipSuccess;
}

bool multiple(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

}  // namespace

bool sequence_attention_backward_fits(const SequenceAttention& a) {  // 2^32 work items a launch, 65535 workgroups along the grid's third axis
  const int64_t rows = static_cast<int64_t>(a.max_q) * (a.hq / a.hk), pairs = static_cast<int64_t>(a.B) * a.hk;
  if (rows >= (int64_t{1} << 31) - 128 || pairs >= (int64_t{1} << 24)) return false;
  const Plan p = plan_of(a);
  const int64_t q_deep = p.q_tiles * p.q_splits, k_deep = p.k_tiles * p.k_splits;
  // (of a side that is cut, users times heads times rows are less than 2^18: a side with more has workgroups enough)
  return q_deep < 65536 && k_deep < 65536 && pairs * q_deep < (int64_t{1} << 24) && pairs * k_deep < (int64_t{1} << 24);
}

size_t sequence_attention_backward_workspace(const SequenceAttention& a) { return plan_of(a).bytes; }

hipError_t sequence_attention_backward(const SequenceAttention& x, void* workspace, hipStream_t s) {
  const Plan p = plan_of(x);
  const size_t e = x.dtype == 1 ? 2 : 4;
  Args a{};
  a.q = x.Q, a.k = x.K, a.v = x.V, a.o = x.O, a.go = x.dO, a.dq = x.dQ, a.dk = x.dK, a.dv = x.dV, a.lse = x.lse;
  a.q_stride = x.q_stride, a.k_stride = x.k_stride, a.v_stride = x.v_stride;
  a.dq_stride = x.dq_stride, a.dk_stride = x.dk_stride, a.dv_stride = x.dv_stride;
  a.where = Packing(x), a.deal = Deal(x, true);
  char* at = static_cast<char*>(workspace);
  a.lse2 = reinterpret_cast<float*>(at), at += p.stats;
  a.less = reinterpret_cast<float*>(at), at += p.stats;
  a.part_q = reinterpret_cast<float*>(at), at += p.part_q;
  a.part_gap = reinterpret_cast<float*>(at), at += p.part_gap;
  a.part_kv = reinterpret_cast<float*>(at);
  a.group = Divisor(x.hq / x.hk), a.q_splits = Divisor(p.q_splits), a.q_chunk = p.q_chunk, a.k_splits = Divisor(p.k_splits), a.k_chunk = p.k_chunk;
  a.hq = x.hq, a.hk = x.hk, a.dh = x.dh;
  a.scale = x.scale, a.causal = x.causal != 0;
  a.pieces = multiple(x.Q, 16) && multiple(x.K, 16) && multiple(x.V, 16) && multiple(x.O, 16) && multiple(x.dO, 16) && x.dh * e % 16 == 0 &&
             x.q_stride * e % 16 == 0 && x.k_stride * e % 16 == 0 && x.v_stride * e % 16 == 0;
  a.quads = x.dh % 4 == 0 && x.dq_stride % 4 == 0 && x.dk_stride % 4 == 0 && x.dv_stride % 4 == 0 && multiple(x.dQ, 4 * e) && multiple(x.dK, 4 * e) &&
            multiple(x.dV, 4 * e);
  return at_head_width(x.dh, [&](auto width) { return x.dtype == 1 ? run<bf16_t, width.value>(a, p, x.B, s) : run<float, width.value>(a, p, x.B, s); });
}

}  // namespace lime
