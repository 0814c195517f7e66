// 4-bit weight matrices with group scales: the tiled layout and its expansion to bf16
// matrix-core operands (gfx950).
//
// A matrix of N rows and K columns is W[n][k] = s[n][k / g] (q[n][k] - z[n][k / g]), q in
// 0..15, s bf16, z in 0..15 (8 where there are no zero points), g = 32, 64 or 128.  Rows are
// padded to 16 and columns to 128.  A tile of 16 rows x 128 columns is 1 KB in one piece:
// lane l of a wavefront owns bytes [16 l, 16 l + 16), which are four words, word j the eight
// codes of row l % 16, columns 32 j + 8 (l / 16) + 0..7 -- what the lane feeds into the j-th
// of four 16x16x32 products.  Nibble p of a word holds column 2 p (p < 4) or 2 (p - 4) + 1,
// so one shift and one mask give two neighbouring columns as the halves of a word.
// Tiles run along k, then along the rows: [N / 16][K / 128][1024 bytes].  Scales and zero
// points: [N / 16][K / g][16 rows].
#pragma once
#include "common.h"

namespace moe {

constexpr int kInt4Rows = 16;      // rows of a tile
constexpr int kInt4Cols = 128;     // columns of a tile
constexpr int kInt4TileBytes = kInt4Rows * kInt4Cols / 2;

__host__ __device__ inline int64_t int4_row_tiles(int64_t rows) { return (rows + kInt4Rows - 1) / kInt4Rows; }
__host__ __device__ inline int int4_col_tiles(int K) { return (K + kInt4Cols - 1) / kInt4Cols; }

// Eight codes -> eight bf16 values 128 + q: the code is put under the exponent of 128, whose
// last seven mantissa bits count in ones.  The offset leaves with the zero point:
// sum (q - z) x = sum (128 + q) x - (128 + z) sum x, the sums in fp32.
__device__ __forceinline__ bf16x8 int4_expand(uint32_t w) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = ((w >> (4 * i)) & 0x000F000Fu) | 0x43004300u;
  return __builtin_bit_cast(bf16x8, v);
}

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ bf16x8 bf16_ones() {
  const u32x4 v = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
  return __builtin_bit_cast(bf16x8, v);
}

// What a lane needs of one tile: its codes, and for each of the tile's 128 / g groups the
// scales and zero points of the four rows 4 (l / 16) + 0..3 whose sums it holds.
template <int GPT, bool ZEROS>
struct Int4Tile {
  u32x4 q;
  u32x2 s[GPT];
  uint32_t z[ZEROS ? GPT : 1];
};

template <int GPT, bool ZEROS>
__device__ __forceinline__ void int4_load(Int4Tile<GPT, ZEROS>& t, const uint8_t* codes, const uint16_t* scales,
                                          const uint8_t* zeros, int64_t tile, int lane) {
  t.q = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(codes + tile * kInt4TileBytes) + lane);
  const int64_t g = tile * GPT * kInt4Rows + 4 * (lane >> 4);
#pragma unroll
  for (int i = 0; i < GPT; ++i) {
    t.s[i] = *reinterpret_cast<const u32x2*>(scales + g + i * kInt4Rows);
    if (ZEROS) t.z[i] = *reinterpret_cast<const uint32_t*>(zeros + g + i * kInt4Rows);
  }
}

// acc += tile . x, for x's four operands xb (32 columns each) and the sums xs[i] of x over each
// group of the tile.
template <int GPT, bool ZEROS>
__device__ __forceinline__ void int4_accumulate(f32x4& acc, const Int4Tile<GPT, ZEROS>& t, const bf16x8 (&xb)[4],
                                                const float (&xs)[GPT]) {
#pragma unroll
  for (int i = 0; i < GPT; ++i) {
    f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = i * (4 / GPT); j < (i + 1) * (4 / GPT); ++j) d = mfma16(int4_expand(t.q[j]), xb[j], d);
    const float s[4] = {__uint_as_float(t.s[i][0] << 16), __uint_as_float(t.s[i][0] & 0xFFFF0000u),
                        __uint_as_float(t.s[i][1] << 16), __uint_as_float(t.s[i][1] & 0xFFFF0000u)};
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float z = ZEROS ? 128.0f + float((t.z[i] >> (8 * r)) & 0xFFu) : 136.0f;
      acc[r] += s[r] * (d[r] - z * xs[i]);
    }
  }
}

// Sums of x over each group of a tile's columns, for the lane's column of x: a product with ones.
template <int GPT>
__device__ __forceinline__ void int4_group_sums(float (&xs)[GPT], const bf16x8 (&xb)[4]) {
#pragma unroll
  for (int i = 0; i < GPT; ++i) {
    f32x4 d = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = i * (4 / GPT); j < (i + 1) * (4 / GPT); ++j) d = mfma16(bf16_ones(), xb[j], d);
    xs[i] = d[0];
  }
}

}  // namespace moe
