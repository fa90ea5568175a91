// Root-mean-square norm of every query and key head and its rotation by the row's position, in one pass:
//   n = x / sqrt(mean(x^2) + eps),  z = n * gamma,  (y_i, y_{i + h/2}) = (z_i, z_{i + h/2}) turned by position base^(-2 i / h)
// for a head of h elements, and the gradients
//   dz = dy turned back,  dgamma = sum over rows and heads of dz * n,  dx = (dn - n mean(dn * n)) / sqrt(mean(x^2) + eps),  dn = dz * gamma.
// A few lanes hold a head, each the same pieces of both halves, so that a pair is in one lane and a sum takes log2(lanes) exchanges.
// The angles of a row are the same for all its heads: a workgroup works them out once, in turns and in fp64 (at position 10^6 an
// fp32 angle would be off by 0.06 radians), and keeps the cosines and sines in LDS.  Bound by memory: every element is read and
// written once.  (65536 rows of eight heads of 64, bf16: forward 24 us in a loop, 5.6 TB/s with what stays in the last cache, where a
// large copy takes 4.8; backward 47 us, 4.3 TB/s, and 4 for the fold of the weights' gradients.)
#include <math.h>

#include <algorithm>

#include "encoder.hpp"
#include "tiles.hpp"

namespace lime {
namespace {

// The most rows of a workgroup's turn, forward and backward.  Forward, the second where the first would leave half of the lanes without a
// head of one side, and has no more heads of either than lanes for them: bf16, 131072 rows of 4 + 4 heads of 32 39 us with turns of 8, 28 of
// 16, 27 of 32; 65536 of 4 + 4 of 64 27.5, 24, 25; of 8 + 1 of 64 27.5 and 25.3; 160704 of 1 + 1 of 20 43, 30, 33.  (Where eight rows fill the
// lanes of both sides: 65536 of 8 + 8 of 64 50.5 us with turns of 8, 53.2 of 16; of 4 + 4 of 128 52.2 and 50.3; of 4 + 4 of 64 in fp32 43.9 and
// 47.1.  Fewer rows than a thousand workgroups have need the workgroups more: 10007 rows of 3 + 1 of 48, fp32, both directions 22.7 and 23.7.)
constexpr int kRows = 8, kMoreRows = 16, kBackRows = 32;
constexpr int64_t kManyRows = 16384;
constexpr int kMaxGroups = 1024; // workgroups of a backward pass: each leaves one partial sum of the weights' gradients
constexpr int kMaxHalf = kMaxRotaryHead / 2;

struct Args {
  const void* x[2];
  const void* dy[2];
  void* out[2];
  const void* gamma[2];
  int64_t x_stride[2], dy_stride[2], out_stride[2];
  int heads[2];
  const int32_t* positions;
  int64_t rows;
  int dh, lanes;    // lanes of a head, a power of two
  int turn;         // rows of a workgroup's turn
  float eps;
  float* partial;   // [2][dh][groups]
  double turns[kMaxHalf];  // base^(-2 i / dh) / (2 pi)
};

// VEC neighbouring elements (16 bytes, or one)
template <typename T, int VEC>
__device__ __forceinline__ void load_piece(const T* p, float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    v[0] = to_float(*p);
  } else if constexpr (sizeof(T) == 2) {
    const bf16x8 x = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = static_cast<float>(x[i]);
  } else {
    const f32x4 x = *reinterpret_cast<const f32x4*>(p);
#pragma unroll
    for (int i = 0; i < VEC; ++i) v[i] = x[i];
  }
}
template <typename T, int VEC>
__device__ __forceinline__ void store_piece(T* p, const float (&v)[VEC]) {
  if constexpr (VEC == 1) {
    store_as(p, v[0]);
  } else if constexpr (sizeof(T) == 2) {
    bf16x8 x;
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[i] = static_cast<__bf16>(v[i]);
    *reinterpret_cast<bf16x8*>(p) = x;
  } else {
    *reinterpret_cast<f32x4*>(p) = f32x4{v[0], v[1], v[2], v[3]};
  }
}
__device__ __forceinline__ float lanes_sum(float x, int lanes) {
  for (int o = 1; o < lanes; o *= 2) x += __shfl_xor(x, o, 64);
  return x;
}

// A lane's part of a head: PARTS pieces of VEC elements of the first half, and their partners.
template <typename T, int VEC, int PARTS, bool BACKWARD, int ROWS>
__global__ __launch_bounds__(256, BACKWARD ? 4 : 1) void norm_rotary_kernel(Args a) {
  __shared__ float2 turned[ROWS][kMaxHalf];  // cosine, sine
  __shared__ float sums[BACKWARD ? 4 : 1][2][kMaxRotaryHead];  // of the waves
  const int tid = threadIdx.x, half = a.dh / 2, t = tid % a.lanes, unit = tid / a.lanes, units = 256 / a.lanes;
  float dgamma[BACKWARD ? 2 : 1][2][PARTS][VEC] = {};  // side, half
  for (int64_t row0 = static_cast<int64_t>(blockIdx.x) * a.turn; row0 < a.rows; row0 += static_cast<int64_t>(gridDim.x) * a.turn) {
    const int count = static_cast<int>(min<int64_t>(a.turn, a.rows - row0));
    __syncthreads();  // everyone is done with the last rows' angles
    for (int i = tid; i < count * half; i += 256) {
      const int r = i / half, c = i % half;
      float2 v = {1.f, 0.f};
      if (a.positions) {
        const double turns = a.positions[row0 + r] * a.turns[c];
        sincospif(2.f * static_cast<float>(turns - rint(turns)), &v.y, &v.x);
      }
      turned[r][c] = v;
    }
    __syncthreads();
#pragma unroll
    for (int side = 0; side < 2; ++side) {
      const int heads = a.heads[side];
      float glo[PARTS][VEC], ghi[PARTS][VEC];
#pragma unroll
      for (int p = 0; p < PARTS; ++p) {
        const int c = (t + p * a.lanes) * VEC;
#pragma unroll
        for (int i = 0; i < VEC; ++i) glo[p][i] = ghi[p][i] = 1.f;
        if (a.gamma[side] && c < half) {
          load_piece<T, VEC>(static_cast<const T*>(a.gamma[side]) + c, glo[p]);
          load_piece<T, VEC>(static_cast<const T*>(a.gamma[side]) + half + c, ghi[p]);
        }
      }
      for (int u = unit; u < count * heads; u += units) {
        const int r = u / heads, head = u % heads;
        const T* x = static_cast<const T*>(a.x[side]) + (row0 + r) * a.x_stride[side] + head * a.dh;
        const T* dy = BACKWARD ? static_cast<const T*>(a.dy[side]) + (row0 + r) * a.dy_stride[side] + head * a.dh : nullptr;
        float lo[PARTS][VEC], hi[PARTS][VEC], ylo[BACKWARD ? PARTS : 1][VEC], yhi[BACKWARD ? PARTS : 1][VEC], square = 0.f;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          const int c = (t + p * a.lanes) * VEC;
          if (c >= half) continue;
          load_piece<T, VEC>(x + c, lo[p]), load_piece<T, VEC>(x + half + c, hi[p]);
          if constexpr (BACKWARD) load_piece<T, VEC>(dy + c, ylo[p]), load_piece<T, VEC>(dy + half + c, yhi[p]);
        }
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          if ((t + p * a.lanes) * VEC >= half) continue;
#pragma unroll
          for (int i = 0; i < VEC; ++i) square = fmaf(lo[p][i], lo[p][i], fmaf(hi[p][i], hi[p][i], square));
        }
        const float total = lanes_sum(square, a.lanes) / a.dh + a.eps;
        float inverse = 1.f / sqrtf(total);
        if (__any(!(total >= 0x1p-60f && total < INFINITY))) {
          seldom();  // squares past the range of fp32, at either end: again, of entries that are 2^70 times smaller or larger
          const float f = total < 1.f ? 0x1p70f : 0x1p-70f;
          square = 0.f;
#pragma unroll
          for (int p = 0; p < PARTS; ++p) {
            if ((t + p * a.lanes) * VEC >= half) continue;
#pragma unroll
            for (int i = 0; i < VEC; ++i) square = fmaf(lo[p][i] * f, lo[p][i] * f, fmaf(hi[p][i] * f, hi[p][i] * f, square));
          }
          const float again = f / sqrtf(lanes_sum(square, a.lanes) / a.dh + a.eps * f * f);
          if (!(total >= 0x1p-60f && total < INFINITY)) inverse = again;
        }
        float mean = 0.f;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          const int c = (t + p * a.lanes) * VEC;
          if (c >= half) continue;
          if constexpr (BACKWARD) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
              const float2 w = turned[r][c + i];
              const float dlo = fmaf(ylo[p][i], w.x, yhi[p][i] * w.y), dhi = fmaf(yhi[p][i], w.x, -ylo[p][i] * w.y);
              lo[p][i] *= inverse, hi[p][i] *= inverse;
              dgamma[side][0][p][i] = fmaf(dlo, lo[p][i], dgamma[side][0][p][i]);
              dgamma[side][1][p][i] = fmaf(dhi, hi[p][i], dgamma[side][1][p][i]);
              ylo[p][i] = glo[p][i] * dlo, yhi[p][i] = ghi[p][i] * dhi;  // dn
              mean = fmaf(ylo[p][i], lo[p][i], fmaf(yhi[p][i], hi[p][i], mean));
            }
          } else {
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
              const float2 w = turned[r][c + i];
              const float zlo = lo[p][i] * inverse * glo[p][i], zhi = hi[p][i] * inverse * ghi[p][i];
              lo[p][i] = fmaf(zlo, w.x, -zhi * w.y), hi[p][i] = fmaf(zhi, w.x, zlo * w.y);
            }
          }
        }
        if constexpr (BACKWARD) mean = lanes_sum(mean, a.lanes) / a.dh;
        T* out = static_cast<T*>(a.out[side]) + (row0 + r) * a.out_stride[side] + head * a.dh;
#pragma unroll
        for (int p = 0; p < PARTS; ++p) {
          const int c = (t + p * a.lanes) * VEC;
          if (c >= half) continue;
          if constexpr (BACKWARD) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) lo[p][i] = inverse * fmaf(-mean, lo[p][i], ylo[p][i]), hi[p][i] = inverse * fmaf(-mean, hi[p][i], yhi[p][i]);
          }
          store_piece<T, VEC>(out + c, lo[p]), store_piece<T, VEC>(out + half + c, hi[p]);
        }
      }
    }
  }
  if constexpr (BACKWARD) {  // the workgroup's sums: a wave's lanes that hold the same elements, then the four waves
    const int lane = tid & 63, wave = tid >> 6;
#pragma unroll
    for (int side = 0; side < 2; ++side)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int p = 0; p < PARTS; ++p)
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            float x = dgamma[side][h][p][i];
            for (int o = a.lanes; o < 64; o *= 2) x += __shfl_xor(x, o, 64);
            const int c = (t + p * a.lanes) * VEC + i;
            if (lane < a.lanes && c < half) sums[wave][side][h * half + c] = x;
          }
    __syncthreads();
    for (int i = tid; i < 2 * a.dh; i += 256) {
      const int side = i / a.dh, c = i % a.dh;
      a.partial[static_cast<int64_t>(i) * gridDim.x + blockIdx.x] = sums[0][side][c] + sums[1][side][c] + sums[2][side][c] + sums[3][side][c];
    }
  }
}

// dgamma of one side and element a wave: the workgroups' sums, in a fixed order.
template <typename T>
__global__ __launch_bounds__(256) void norm_rotary_fold_kernel(const float* partial, int groups, int dh, T* dq, T* dk) {
  const int at = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63, side = at / dh, c = at % dh;
  if (side > 1) return;
  T* to = side ? dk : dq;
  float total = 0.f;
#pragma unroll 8
  for (int i = lane; i < groups; i += 64) total += partial[static_cast<int64_t>(at) * groups + i];
  total = wave_sum(total);
  if (to && lane == 0) store_as(to + c, total);
}

bool multiple(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
// Few rows are spread over more workgroups, in shorter turns.
int back_turn(int64_t rows) { return static_cast<int>(std::clamp<int64_t>((rows + kMaxGroups - 1) / kMaxGroups, 4, kBackRows)); }
int64_t groups_of(int64_t rows) { return std::min<int64_t>(kMaxGroups, (rows + back_turn(rows) - 1) / back_turn(rows)); }

template <typename T, int VEC, int PARTS>
hipError_t launch(const Args& a, bool backward, hipStream_t s) {
  const int64_t groups = backward ? groups_of(a.rows) : (a.rows + a.turn - 1) / a.turn;
  if (backward) hipLaunchKernelGGL((norm_rotary_kernel<T, VEC, PARTS, true, kBackRows>), dim3(static_cast<unsigned>(groups)), dim3(256), 0, s, a);
  else if (a.turn > kRows) hipLaunchKernelGGL((norm_rotary_kernel<T, VEC, PARTS, false, kMoreRows>), dim3(static_cast<unsigned>(groups)), dim3(256), 0, s, a);
  else hipLaunchKernelGGL((norm_rotary_kernel<T, VEC, PARTS, false, kRows>), dim3(static_cast<unsigned>(groups)), dim3(256), 0, s, a);
  return hipGetLastError();
}

template <typename T>
hipError_t run(const NormRotary& x, void* workspace, bool backward, hipStream_t s) {
  Args a{};
  constexpr int e = sizeof(T), kVec = 16 / e;
  const int half = x.dh / 2;
  bool vectors = half * e % 16 == 0;
  for (int i = 0; i < 2; ++i) {
    a.heads[i] = x.heads[i];
    if (x.heads[i] == 0) continue;
    a.x[i] = x.x[i], a.dy[i] = x.dy[i], a.out[i] = x.out[i], a.gamma[i] = x.gamma[i];
    a.x_stride[i] = x.x_stride[i], a.dy_stride[i] = x.dy_stride[i], a.out_stride[i] = x.out_stride[i];
    vectors = vectors && multiple(x.x[i], 16) && multiple(x.dy[i], 16) && multiple(x.out[i], 16) && multiple(x.gamma[i], 16) &&
              x.x_stride[i] * e % 16 == 0 && x.dy_stride[i] * e % 16 == 0 && x.out_stride[i] * e % 16 == 0;
  }
  a.positions = x.positions, a.rows = x.rows, a.dh = x.dh, a.eps = x.eps, a.turn = backward ? back_turn(x.rows) : kRows, a.partial = static_cast<float*>(workspace);
  const long double ratio = powl(x.base, -2.0L / x.dh);
  long double f = 1.0L / (2.0L * 3.14159265358979323846264338327950288L);
  for (int i = 0; i < half; ++i, f *= ratio) a.turns[i] = static_cast<double>(f);
  const int pieces = vectors ? half / kVec : half;
  a.lanes = 1;
  while (a.lanes < pieces && a.lanes < 64) a.lanes *= 2;
  const int units = 256 / a.lanes, most = std::max(a.heads[0], a.heads[1]), least = a.heads[1] > 0 ? std::min(a.heads[0], a.heads[1]) : a.heads[0];
  if (!backward && a.rows > kManyRows && most * kRows <= units && 2 * least * kRows <= units) a.turn = kMoreRows;
  hipError_t err = vectors ? launch<T, kVec, 1>(a, backward, s) : launch<T, 1, 2>(a, backward, s);
  if (err != hipSuccess || !backward || (!x.dgamma[0] && !x.dgamma[1])) return err;
  hipLaunchKernelGGL(norm_rotary_fold_kernel<T>, dim3(static_cast<unsigned>((2 * x.dh + 3) / 4)), dim3(256), 0, s, a.partial, static_cast<int>(groups_of(x.rows)), x.dh,
                     static_cast<T*>(x.dgamma[0]), static_cast<T*>(x.dgamma[1]));
  return hipGetLastError();
}

}  // namespace

bool norm_rotary_fits(const NormRotary& a) { return (a.rows + kRows - 1) / kRows * 256 < (int64_t{1} << 32); }
size_t norm_rotary_backward_workspace(int64_t rows, int dh) { return align_up(static_cast<size_t>(groups_of(rows)) * 2 * dh * sizeof(float)); }

hipError_t norm_rotary(const NormRotary& a, hipStream_t s) { return a.dtype == 1 ? run<bf16_t>(a, nullptr, false, s) : run<float>(a, nullptr, false, s); }
hipError_t norm_rotary_backward(const NormRotary& a, void* workspace, hipStream_t s) {
  return a.dtype == 1 ? run<bf16_t>(a, workspace, true, s) : run<float>(a, workspace, true, s);
}

}  // namespace lime
