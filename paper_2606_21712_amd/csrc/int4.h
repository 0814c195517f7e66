// 4-bit weight matrices with group scales: the packed layout and its expansion to bf16
// matrix-core operands (gfx950).
//
// A matrix of N rows and K columns is W[n][k] = s[n][k / g] (q[n][k] - z[n][k / g]), q in
// 0..15, s bf16, z in 0..15 (8 where there are no zero points), g = 32, 64 or 128.  Rows are
// padded to 16 and columns to 128.  A tile of 16 rows x 128 columns is 1 KB in one piece:
// lane l of a wavefront owns bytes [16 l, 16 l + 16), which are four words, word j the eight
// codes of row l % 16, columns 32 j + 8 (l / 16) + 0..7 -- what the lane feeds into the j-th
// of four 16x16x32 products.  Nibble p of a word holds column 2 p (p < 4) or 2 (p - 4) + 1,
// so one shift and one mask give two neighbouring columns as the halves of a word.
// Tiles run along k, then along the rows: [N / 16][K / 128][1024 bytes].  Scales:
// [N / 16][K / 128][4][128 / g][4], for rows 4 a + 0..3 those of each group: lane group a (16 lanes)
// of the products' results holds these rows, and loads their scales one to a lane; a lane
// permute inside the row of 16 then gives every lane the one it needs, at the cost of unpacking
// it.  bf16 without zero points; with them words of which the upper half is the scale and
// the lower one 128 + z, in bf16 (exact), the number that the kernels need: a byte instead would
// be a sixteenth to a twentieth less to read for more instructions.
#pragma once
#include "weight_stream.h"

namespace moe {

constexpr int kInt4Rows = 16;      // rows of a tile
constexpr int kInt4Cols = 128;     // columns of a tile
constexpr int kInt4TileBytes = kInt4Rows * kInt4Cols / 2;

__host__ __device__ inline int64_t int4_row_tiles(int64_t rows) { return (rows + kInt4Rows - 1) / kInt4Rows; }
__host__ __device__ inline int int4_col_tiles(int K) { return (K + kInt4Cols - 1) / kInt4Cols; }

// Eight codes -> eight bf16 values 128 + q: the code is put under the exponent of 128, whose
// last seven mantissa bits count in ones.  The offset leaves with the zero point:
// sum (q - z) x = sum (128 + q) x - (128 + z) sum x, the sums in fp32.
__device__ __forceinline__ bf16x8 int4_expand(uint32_t w, uint32_t exponent) {
  u32x4 v;
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = ((w >> (4 * i)) & 0x000F000Fu) | exponent;
  return __builtin_bit_cast(bf16x8, v);
}
// The exponents, in a register: the and and the or are one instruction then (two constants are not).
__device__ __forceinline__ uint32_t int4_exponent() {
  uint32_t e = 0x43004300u;
  asm("" : "+v"(e));
  return e;
}

// 4-bit weights as the kernels walk them: a step is one tile of 128 columns.  GPT: groups of a tile.
// POLICY: of the loads of codes.
template <int GPT, bool ZEROS, int POLICY = kStream>
struct Int4Weights {
  static constexpr int kCols = kInt4Cols;               // columns of a step
  static constexpr int kTok = 16;                       // rows of activations that one operand holds
  static constexpr int kXRegs = 4;                      // operands of activations of a step: 32 columns each
  static constexpr int kAcc = 1;
  static constexpr int kScaleBytes = ZEROS ? 4 : 2;
  const uint8_t* codes;
  const uint8_t* scales;

  // A matrix: codes and scales, tiles of 16 rows along k, and the lane's places in a tile.
  struct View {
    Buffer c, s;
    int tiles, lane_at, scale_at, offset_at;
  };
  // What a lane loads of a tile: its codes, and the words of one scale each in two orders (below).
  struct Step {
    u32x4 q;
    uint32_t s, z;
  };
  static __device__ __forceinline__ Int4Weights pick(bool first, const Int4Weights& a, const Int4Weights& b) {
    return {pick_of(first, a.codes, b.codes), pick_of(first, a.scales, b.scales)};
  }
  __device__ __forceinline__ View view(int mat, int64_t rows, int K, int lane) const {
    const int64_t tiles = int4_row_tiles(rows) * int4_col_tiles(K);
    const int64_t sb = tiles * (GPT * kInt4Rows * kScaleBytes);
    const int i = lane >> 2, g = (lane >> 4) & (GPT - 1);
    return {buffer_of(codes + mat * tiles * kInt4TileBytes, tiles * kInt4TileBytes), buffer_of(scales + mat * sb, sb),
            int4_col_tiles(K), 16 * lane, ((lane >> 4) * (4 * GPT) + (lane & (4 * GPT - 1))) * kScaleBytes,
            (((i & 3) * GPT + g) * 4 + (lane & 3)) * kScaleBytes};
  }
  static __device__ __forceinline__ void load(Step& t, const View& v, int rt, int s, bool on) {
    const int tile = rt * v.tiles + s;
    t.q = load16<POLICY>(v.c, on, v.lane_at, tile * kInt4TileBytes);
    const int at = tile * (GPT * kInt4Rows * kScaleBytes);
    t.s = ZEROS ? load4<kCached>(v.s, on, v.scale_at, at) : load2<kCached>(v.s, on, v.scale_at, at);
    t.z = ZEROS ? load4<kCached>(v.s, on, v.offset_at, at) : load2<kCached>(v.s, on, v.offset_at, at);
  }
  static __device__ __forceinline__ int token(int lane) { return lane & 15; }
  static __device__ __forceinline__ int x_at(int lane) { return 16 * (lane >> 4); }
  // K % 32 == 0: columns past K read as zeros.
  static __device__ __forceinline__ void load_x(u32x4 (&x)[kXRegs], const Buffer& b, int lane_at, int s, int K,
                                                bool on) {
#pragma unroll
    for (int j = 0; j < kXRegs; ++j) {
      const int k0 = (s * kXRegs + j) * 32;
      x[j] = load16<kCached>(b, on && k0 < K, lane_at, k0 * 2);
    }
  }
  static __device__ __forceinline__ f32x4 finish(f32x4 v) { return v; }
  static __device__ __forceinline__ bool holds(int) { return true; }
  static __device__ __forceinline__ int row(int, int lane) { return 4 * (lane >> 4); }

  // With d[n][g] = sum of (128 + q) x over group g and X[g] the sum of x,
  //   y[n] = sum_g s[n][g] d[n][g] - sum_g (s[n][g] (128 + z[n][g])) X[g]:
  // the second sum is a product along g, one fp32 matrix-core product of 4 groups for a tile, for which
  // the lane holds the word of row l % 16, group l / 16.  For the first, the lane that holds d of rows
  // 4 (l / 16) + 0..3 takes their scales out of its 16 neighbours' words (row 4 (l / 16) + l % 4, group
  // (l / 4) % 4) by a lane permute.
  //
  // X comes from products with ones, group i's in rows 4 i + 0..3: so it lands in lane group i, which
  // is where the fp32 product wants group i.
  template <int C>
  struct Sums {
    float x[C];
  };
  template <int C>
  static __device__ __forceinline__ void sums(Sums<C>& t, const u32x4 (&xb)[C][kXRegs], int lane) {
    const int i = (lane & 15) >> 2;
    f32x4 d[C];
#pragma unroll
    for (int c = 0; c < C; ++c) d[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = 0; j < kXRegs; ++j) {
      const uint32_t one = i == j / (4 / GPT) ? 0x3F803F80u : 0u;
      const bf16x8 ones = as_bf16(u32x4{one, one, one, one});
#pragma unroll
      for (int c = 0; c < C; ++c) d[c] = mfma16(ones, as_bf16(xb[c][j]), d[c]);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) t.x[c] = d[c][0];
  }
  static __device__ __forceinline__ float scale_of(uint32_t w) {
    return __uint_as_float(ZEROS ? w & 0xFFFF0000u : w << 16);
  }
  template <int LANE>
  static __device__ __forceinline__ float of_lane(float w) {     // row_newbcast
    return __uint_as_float(uint32_t(__builtin_amdgcn_update_dpp(0, int(__float_as_uint(w)), 0x150 + LANE, 0xF, 0xF, true)));
  }
  template <int I, int C>
  static __device__ __forceinline__ void add_group(f32x4 (&acc)[C][kAcc], const Step& t, float s, uint32_t e,
                                                   const u32x4 (&xb)[C][kXRegs]) {
    f32x4 d[C];
#pragma unroll
    for (int c = 0; c < C; ++c) d[c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int j = I * (4 / GPT); j < (I + 1) * (4 / GPT); ++j) {
      const bf16x8 q = int4_expand(t.q[j], e);
#pragma unroll
      for (int c = 0; c < C; ++c) d[c] = mfma16(q, as_bf16(xb[c][j]), d[c]);
    }
    const float r[4] = {of_lane<4 * I>(s), of_lane<4 * I + 1>(s), of_lane<4 * I + 2>(s), of_lane<4 * I + 3>(s)};
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[c][0][i] = __builtin_fmaf(r[i], d[c][i], acc[c][0][i]);
  }
  // acc += tile . x for C operands of 16 rows of x each; codes are expanded, and scales permuted, once
  // for all.
  template <int C>
  static __device__ __forceinline__ void add(f32x4 (&acc)[C][kAcc], const Step& t, const u32x4 (&xb)[C][kXRegs],
                                             const Sums<C>& xs) {
    const uint32_t e = int4_exponent();
    const float z = -scale_of(t.z) * (ZEROS ? __uint_as_float(t.z << 16) : 136.0f);
#pragma unroll
    for (int c = 0; c < C; ++c) acc[c][0] = __builtin_amdgcn_mfma_f32_16x16x4f32(z, xs.x[c], acc[c][0], 0, 0, 0);
    const float s = scale_of(t.s);
    add_group<0, C>(acc, t, s, e, xb);
    if constexpr (GPT >= 2) add_group<1, C>(acc, t, s, e, xb);
    if constexpr (GPT >= 4) {
      add_group<2, C>(acc, t, s, e, xb);
      add_group<3, C>(acc, t, s, e, xb);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) keep(acc[c][0]);
  }
};

}  // namespace moe
