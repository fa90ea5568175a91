// Tiles of row-major matrices in LDS, streamed in straight from memory and read as matrix-instruction operands, for both
// storage types: what the history encoder's attention and the catalogue loss are built from.
//
// A tile is ROWS rows of DH columns (the operand's own width rounded up; columns past it are zero).  Its 16-byte pieces are
// permuted within a row by the row's number (swizzle), so that neither of the two ways it is read meets its own lanes in a bank:
//   row      lane (n, g), slot t = tile[r0 + n][16 kk + 8g + t]       (the columns are summed)
//   column   lane (n, g), slot t = tile[r0 + chain_k(g, t)][c0 + n]   (the rows are summed, in chained order)
// A product's 32 x 32 accumulator, rounded to the storage type half by half (half_fragment), is the other operand of the
// second: the two products of an attention step chain in registers.
// fp32 operands are cut into three bf16 parts of eight bits each, which is all of their 24 bits, and a product is the six products of
// parts that reach into them (the three left out are below 2^-24 of it): six bf16 instructions of 32 cycles where
// v_mfma_f32_32x32x2_f32 takes eight of 64.  An fp32 tile is cut once, by all waves of the workgroup together, into three tiles of
// bf16 (Stages).  (When every wave cut the fragments it read: 1003 rows over 20011 items with both gradients 161 us, now 152.)
// An operand that is not finite gives NaN (an infinite one too: its parts are it and what is left of it less itself); one below 2^-110
// loses its last parts to the instruction's range.
#pragma once

#include <type_traits>

#include "mfma.hpp"

namespace lime {

typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

struct Parts {  // an fp32 fragment: x = sum of its parts
  bf16x8 part[3];
};
template <typename T>
using Fragment = std::conditional_t<std::is_same_v<T, float>, Parts, bf16x8>;

__device__ __forceinline__ Parts in_parts(const f32x8& x) {
  u32x4 w[3];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    unsigned bits[3][2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {  // the leading eight bits, the next eight, the rest: no rounding
      const float v = x[2 * i + k];
      bits[0][k] = __float_as_uint(v) & 0xffff0000u;
      const float r = v - __uint_as_float(bits[0][k]);
      bits[1][k] = __float_as_uint(r) & 0xffff0000u;
      bits[2][k] = __float_as_uint(r - __uint_as_float(bits[1][k]));
    }
#pragma unroll
    for (int p = 0; p < 3; ++p) w[p][i] = __builtin_amdgcn_perm(bits[p][1], bits[p][0], 0x07060302);  // the upper halves
  }
  return {__builtin_bit_cast(bf16x8, w[0]), __builtin_bit_cast(bf16x8, w[1]), __builtin_bit_cast(bf16x8, w[2])};
}

__device__ __forceinline__ f32x16 mma16(bf16x8 a, bf16x8 b, f32x16 c) { return mfma32(a, b, c); }
__device__ __forceinline__ f32x16 mma16(const Parts& a, const Parts& b, f32x16 c) {
  c = mfma32(a.part[0], b.part[2], c);  // the small ones first
  c = mfma32(a.part[1], b.part[1], c);
  c = mfma32(a.part[2], b.part[0], c);
  c = mfma32(a.part[0], b.part[1], c);
  c = mfma32(a.part[1], b.part[0], c);
  return mfma32(a.part[0], b.part[0], c);
}
__device__ __forceinline__ float element(const bf16x8& f, int t) { return static_cast<float>(f[t]); }
__device__ __forceinline__ float element(const Parts& f, int t) { return static_cast<float>(f.part[0][t]) + (static_cast<float>(f.part[1][t]) + static_cast<float>(f.part[2][t])); }
__device__ __forceinline__ void negate(bf16x8& f) { f = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, f) ^ 0x80008000u); }
__device__ __forceinline__ void negate(Parts& f) {
#pragma unroll
  for (int p = 0; p < 3; ++p) negate(f.part[p]);
}
__device__ __forceinline__ f32x16 zero_block() {
  f32x16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}
// Registers 8f .. 8f + 7 of an accumulator as a fragment of the storage type (bf16: round to nearest even).
template <typename T>
__device__ __forceinline__ Fragment<T> half_fragment(const f32x16& d, int f) {
  if constexpr (sizeof(T) == 2) {
    return pack_half(d, f);
  } else {
    f32x8 r;
#pragma unroll
    for (int t = 0; t < 8; ++t) r[t] = d[8 * f + t];
    return in_parts(r);
  }
}
// Stands first in a branch that few tiles take (masks): keeps the compiler from computing it for all of them and selecting after,
// which cost as many vector instructions again as the softmax itself.
__device__ __forceinline__ void seldom() { asm volatile(""); }
// Row of a 32 x 32 accumulator that register i of lane half g holds.
__device__ __forceinline__ constexpr int block_row(int i, int g) { return 8 * (i >> 2) + 4 * g + (i & 3); }

// Tiles and chunks' sums are as wide as a power of two; products may be done for fewer columns, a multiple of 16.  (Columns of chunks' sums
// past those are neither written nor read.)
constexpr int tile_width(int c) { return c <= 32 ? 32 : c <= 64 ? 64 : c <= 128 ? 128 : 256; }

template <typename T, int DH, int ROWS>
struct Tile {
  static constexpr int kRowBytes = DH * static_cast<int>(sizeof(T)), kPieces = kRowBytes / 16, kBytes = ROWS * kRowBytes;
  static constexpr int kPerPiece = 16 / static_cast<int>(sizeof(T));
  static_assert(DH % 32 == 0 && ROWS % 16 == 0);
  // Which piece sits in slot s of row r: s ^ swizzle(r).  The 64 banks serve 256 bytes at a time: sixteen consecutive rows at one piece
  // (a row fragment) and four consecutive rows at four neighbouring pieces (half a wave's part of a column fragment).  Either falls on
  // 16 different slots of the 256 bytes, which hold one, two or four rows.  (Laid out for 128 bytes, half of the cycles were conflicts.)
  __device__ static constexpr int swizzle(int r) {
    return kPieces >= 16 ? ((r & 3) << 2) | ((r >> 2) & 3) : kPieces == 8 ? (((r >> 1) & 1) << 2) | ((r >> 2) & 3) : (r >> 2) & 3;
  }
};

// Where a lane's fragments lie in a tile (at an LDS offset that is a multiple of 256).  The swizzle is an exclusive or, so that one place
// a kind of fragment gives all of them: another column is another bit of the place, another sixteen rows an offset of the instruction.
// (With a place of its own for each fragment, the widest kernels had no registers left.)
template <typename T, int DH, int ROWS>
class TileReader {
  using Shape = Tile<bf16_t, DH, ROWS>;
  static constexpr int kSpan = Shape::kRowBytes < 256 ? Shape::kRowBytes : 256;  // bytes of a row that the swizzle permutes
  unsigned row_, column_;

  // `place` moved by `bytes` along its row
  __device__ static unsigned along(unsigned place, int bytes) { return (place ^ (bytes % kSpan)) + bytes / kSpan * kSpan; }
  __device__ static bf16x4 transposed(unsigned place) {
    return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<__attribute__((address_space(3))) s16x4*>(place)));
  }
  __device__ bf16x8 row_of(unsigned tile, int r0, int kk) const {
    return *reinterpret_cast<__attribute__((address_space(3))) const bf16x8*>(along(tile + row_, 32 * kk) + r0 * kRowBytes);
  }
  __device__ bf16x8 column_of(unsigned tile, int r0, int c0) const {
    const unsigned place = along(tile + column_, 2 * c0);
    const bf16x4 lo = transposed(place + r0 * kRowBytes), hi = transposed((place ^ (Shape::swizzle(8) * 16u)) + (r0 + 8) * kRowBytes);  // eight rows on
    return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }

 public:
  static constexpr int kRowBytes = Shape::kRowBytes;
  __device__ explicit TileReader(int lane) {
    const int n = lane & 31, g = lane >> 5;
    row_ = n * kRowBytes + (g ^ Shape::swizzle(n)) * 16;
    // ds_read_b64_tr_b16: each lane of a group of 16 gets a column of the 4 x 16 block whose rows the group's lanes point
    // at, four lanes a row
    const int r = 4 * g + (lane & 15) / 4, piece = 2 * ((lane >> 4) & 1) + (lane & 3) / 2;
    column_ = r * kRowBytes + (piece ^ Shape::swizzle(r)) * 16 + (lane & 1) * 8;
  }
  // r0 a multiple of 32
  __device__ Fragment<T> row(unsigned tile, int r0, int kk) const {
    if constexpr (sizeof(T) == 2) return row_of(tile, r0, kk);
    else return {row_of(tile, r0, kk), row_of(tile + Shape::kBytes, r0, kk), row_of(tile + 2 * Shape::kBytes, r0, kk)};
  }
  // r0 a multiple of 16, c0 of 32
  __device__ Fragment<T> column(unsigned tile, int r0, int c0) const {
    if constexpr (sizeof(T) == 2) return column_of(tile, r0, c0);
    else return {column_of(tile, r0, c0), column_of(tile + Shape::kBytes, r0, c0), column_of(tile + 2 * Shape::kBytes, r0, c0)};
  }
};

// The LDS of a kernel that streams TILES tiles and WORDS times 64 words a step.  bf16: two steps' worth, one in use and the other on its
// way.  fp32: the tiles as they arrive, their three parts, and two steps' words; the next tiles are on their way while the parts are in use.
template <typename T, int DH, int ROWS, int TILES, int WORDS = 0>
struct Stages {
  using Raw = Tile<T, DH, ROWS>;
  using Part = Tile<bf16_t, DH, ROWS>;
  static constexpr bool kCut = sizeof(T) == 4;
  static constexpr int kTiles = TILES * Raw::kBytes, kParts = TILES * 3 * Part::kBytes, kWords = WORDS * 256;
  static constexpr int kBytes = kCut ? kTiles + kParts + 2 * kWords : 2 * (kTiles + kWords);
  // where step i's tile t and words w arrive
  __device__ static unsigned char* tile(unsigned char* smem, int i, int t) { return smem + (kCut ? 0 : i % 2 * (kTiles + kWords)) + t * Raw::kBytes; }
  __device__ static float* words(unsigned char* smem, int i, int w) {
    return reinterpret_cast<float*>(smem + kTiles + (kCut ? kParts + i % 2 * kWords : i % 2 * (kTiles + kWords)) + w * 256);
  }
  // where a reader finds tile t, once it has arrived
  __device__ static unsigned operand(unsigned char* smem, int i, int t) { return lds_offset_of(kCut ? smem + kTiles + t * 3 * Part::kBytes : tile(smem, i, t)); }
  // Step i's tiles are there, for all waves, and everyone is done with those of the step before: the next may be asked for.
  template <int WAVES>
  __device__ static void arrive(unsigned char* smem, int tid) {
    wait_lds_loads<0>();
    lds_barrier();
    if constexpr (kCut) {
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        const unsigned char* from = smem + t * Raw::kBytes;
        unsigned char* to = smem + kTiles + t * 3 * Part::kBytes;
#pragma unroll 2
        for (int i = tid; i < ROWS * Part::kPieces; i += WAVES * 64) {
          const int r = i / Part::kPieces, piece = i % Part::kPieces;
          const f32x4 lo = *reinterpret_cast<const f32x4*>(from + r * Raw::kRowBytes + ((2 * piece) ^ Raw::swizzle(r)) * 16);
          const f32x4 hi = *reinterpret_cast<const f32x4*>(from + r * Raw::kRowBytes + ((2 * piece + 1) ^ Raw::swizzle(r)) * 16);
          const Parts x = in_parts(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
          for (int p = 0; p < 3; ++p) *reinterpret_cast<bf16x8*>(to + p * Part::kBytes + r * Part::kRowBytes + (piece ^ Part::swizzle(r)) * 16) = x.part[p];
        }
      }
      lds_barrier();
    }
  }
};

// Rows of a strided row-major matrix, `width` elements each: what a tile is filled from.
struct Rows {
  const void* base;   // the first row, at this head's first column; uniform over the workgroup
  unsigned stride;    // bytes from row to row, at least the width, below 2^24
  unsigned width;     // bytes of a row
  bool pieces;        // base, stride and width are multiples of 16 bytes
};

// Fills tiles by WAVES waves, 1 KiB a load, from memory straight to LDS.  Rows at or past the given count and columns past the
// width come out as zeros: the loads go through a buffer whose size ends with the last row, and what lies outside reads as zero.
// (The loads are not said to touch memory, so that the compiler may work on other tiles among them; who fills a tile has passed a
// barrier since its last use, and who reads it waits and passes one, and those are.)
template <typename T, int DH, int ROWS, int WAVES>
struct TileLoader {
  using Shape = Tile<T, DH, ROWS>;
  static constexpr int kLoads = Shape::kBytes / 1024 / WAVES;  // a wave's, for one tile
  static_assert(kLoads * WAVES * 1024 == Shape::kBytes && ROWS <= 128);
  static constexpr int kRowsALoad = WAVES * 1024 / Shape::kRowBytes;               // from one of a wave's loads to its next
  static constexpr int kOffsets = kRowsALoad >= 16 ? 1 : 16 / kRowsALoad < kLoads ? 16 / kRowsALoad : kLoads;  // the swizzle repeats after 16 rows
  unsigned offset[kOffsets];

  __device__ void init(const Rows& m, int tid) {
    const int lane = tid & 63, wave = tid >> 6;
#pragma unroll
    for (int i = 0; i < kOffsets; ++i) {
      const int at = (wave + WAVES * i) * 64 + lane, row = at / Shape::kPieces, piece = (at % Shape::kPieces) ^ Shape::swizzle(row);
      offset[i] = piece * 16u < m.width ? row * m.stride + piece * 16u : 0x80000000u;
    }
  }
  // Asks for rows row0 .. row0 + ROWS - 1, those at or past `rows` as zeros.  kLoads loads a wave (none where rows are not
  // made of whole pieces: then the tile is copied here and now, element by element).
  __device__ void issue(const Rows& m, int row0, int rows, unsigned char* tile, int tid) const {
    const char* first = static_cast<const char*>(m.base) + static_cast<int64_t>(row0) * m.stride;
    const int count = min(rows - row0, ROWS);
    if (m.pieces) {
      const uint64_t at = reinterpret_cast<uint64_t>(first);
      const unsigned size = count > 0 ? (count - 1) * m.stride + m.width : 0;
      u32x4 resource;
      resource[0] = __builtin_amdgcn_readfirstlane(static_cast<unsigned>(at));
      resource[1] = __builtin_amdgcn_readfirstlane(static_cast<unsigned>(at >> 32) & 0xffffu);
      resource[2] = __builtin_amdgcn_readfirstlane(size);
      resource[3] = 0x00020000u;
      const unsigned lds = __builtin_amdgcn_readfirstlane(lds_offset_of(tile) + (tid >> 6) * 1024);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        unsigned at_row;  // (added here, not by the compiler: it would keep all the sums in registers across the kernel's loop)
        asm volatile("s_mov_b32 m0, %1\n\tv_add_u32_e32 %0, %2, %3\n\tbuffer_load_dwordx4 %0, %4, 0 offen lds"
                     : "=&v"(at_row)
                     : "s"(lds + WAVES * 1024 * i), "s"(i / kOffsets * kOffsets * kRowsALoad * m.stride), "v"(offset[i % kOffsets]), "s"(resource)
                     : "m0");
      }
    } else {
      const unsigned columns = m.width / sizeof(T);
      for (unsigned i = tid; i < ROWS * DH; i += WAVES * 64) {
        const int r = i / DH, c = i % DH;
        T v{};
        if (r < count && c < static_cast<int>(columns)) v = *reinterpret_cast<const T*>(first + r * static_cast<int64_t>(m.stride) + c * sizeof(T));
        *reinterpret_cast<T*>(tile + r * Shape::kRowBytes + ((c / Shape::kPerPiece) ^ Shape::swizzle(r)) * 16 + c % Shape::kPerPiece * sizeof(T)) = v;
      }
    }
  }
};

// 64 words, those from `count` on as zeros, straight to LDS: one load of one wave.
__device__ __forceinline__ void words_to_lds(const void* from, int count, void* to, int lane) {
  const uint64_t at = reinterpret_cast<uint64_t>(from);
  u32x4 resource;
  resource[0] = __builtin_amdgcn_readfirstlane(static_cast<unsigned>(at));
  resource[1] = __builtin_amdgcn_readfirstlane(static_cast<unsigned>(at >> 32) & 0xffffu);
  resource[2] = __builtin_amdgcn_readfirstlane(count * 4u);
  resource[3] = 0x00020000u;
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds"
               : : "s"(__builtin_amdgcn_readfirstlane(lds_offset_of(to))), "v"(lane * 4u), "s"(resource) : "m0");
}

// The 16-deep fragments of one row of `width` bytes, straight from memory: lane half g's slots hold columns 16 kk + 8g .. + 7.
// A row that is not live, and columns past the width, are zeros.
template <typename T, int DH>
__device__ __forceinline__ void load_row(const void* row, unsigned width, bool pieces, bool live, int g, Fragment<T> (&f)[DH / 16]) {
#pragma unroll
  for (int kk = 0; kk < DH / 16; ++kk) {
    const int c = 16 * kk + 8 * g;
    const T* p = static_cast<const T*>(row) + c;
    if constexpr (sizeof(T) == 2) {
      u32x4 v = {0, 0, 0, 0};
      if (pieces) {
        if (live && c * 2u < width) v = *reinterpret_cast<const u32x4*>(p);
      } else if (live) {
#pragma unroll
        for (int t = 0; t < 8; ++t)
          if ((c + t) * 2u < width) v[t / 2] |= static_cast<unsigned>(p[t].bits) << (16 * (t & 1));
      }
      f[kk] = __builtin_bit_cast(bf16x8, v);
    } else {
      f32x8 v = {0, 0, 0, 0, 0, 0, 0, 0};
      if (pieces) {
        f32x4 lo = {0, 0, 0, 0}, hi = {0, 0, 0, 0};
        if (live && c * 4u < width) lo = *reinterpret_cast<const f32x4*>(p);
        if (live && (c + 4) * 4u < width) hi = *reinterpret_cast<const f32x4*>(p + 4);
        v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      } else if (live) {
#pragma unroll
        for (int t = 0; t < 8; ++t)
          if ((c + t) * 4u < width) v[t] = p[t];
      }
      f[kk] = in_parts(v);
    }
  }
}

// A transposed accumulator block (lane n = row, registers = columns block_row(i, g)) into that row, scaled; columns from `width`
// (elements) on are left out.  `quads`: four neighbouring elements may be stored at once.
template <typename T>
__device__ __forceinline__ void store_block(T* row, const f32x16& d, float factor, int c0, int width, bool quads, int g) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int c = c0 + 8 * j + 4 * g;
    if (quads) {
      if (c >= width) continue;
      if constexpr (sizeof(T) == 2) {
        bf16x4 v;
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = static_cast<__bf16>(d[4 * j + r] * factor);
        *reinterpret_cast<bf16x4*>(row + c) = v;
      } else {
        *reinterpret_cast<f32x4*>(row + c) = f32x4{d[4 * j] * factor, d[4 * j + 1] * factor, d[4 * j + 2] * factor, d[4 * j + 3] * factor};
      }
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (c + r < width) store_as(row + c + r, d[4 * j + r] * factor);
    }
  }
}

}  // namespace lime
