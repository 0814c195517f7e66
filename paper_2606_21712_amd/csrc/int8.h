// 8-bit integer matrices: the packed layout, and the codes of a row.
//
// Codes are -127..127 (any int8 is taken), the value of one is its row's scale times it.
//
// Packed: rows in tiles of 16, columns in steps of 64, [rows / 16][2 ceil(K / 128)][64 lanes][16]: the
// 16 bytes of lane l of a step are row l % 16, columns 16 (l / 16) .. + 15, which is one operand of
// a 16 x 16 x 64 product.  A step is 1 KB in one piece, for loads to registers as for loads to LDS.
// Rows are padded to 16 and columns to 128 with zeros: what the other operand has there does not count.
#pragma once
#include "common.h"
#include "tiling.h"

namespace moe {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x16 __attribute__((ext_vector_type(16)));

// Codes of a row whose largest magnitude has the bits `top` (NaN above infinity above the numbers):
// q = v * 127 / max, rounded to nearest even, the quotient rounded to fp32 first.  What is not
// finite makes the whole row NaN by its scale, its codes are 0.
struct RowCodes {
  float up, inverse;   // v * up * inverse; up is a power of two that keeps the quotient finite
  bool finite;
  float max;
  __device__ __forceinline__ explicit RowCodes(uint32_t top) {
    finite = top < 0x7F800000u;
    max = __uint_as_float(top);
    up = max < 0x1p-100f ? 0x1p100f : 1.0f;
    inverse = finite && max > 0.f ? 127.0f / (max * up) : 0.f;
  }
  __device__ __forceinline__ int code(float v) const { return int(rintf(v * up * inverse)); }
  // of eight values
  __device__ __forceinline__ u32x2 pack(const float (&v)[8]) const {
    u32x2 out = {0u, 0u};
    if (finite) {
#pragma unroll
      for (int i = 0; i < 8; ++i) out[i >> 2] |= (uint32_t(code(v[i])) & 255u) << (8 * (i & 3));
    }
    return out;
  }
  // The scale of the codes of values times `factor`.
  __device__ __forceinline__ float scale(float factor = 1.0f) const {
    return finite ? max / 127.0f * factor : __uint_as_float(0x7FC00000u);
  }
};

__device__ __forceinline__ void unpack_bf16(const u32x4& v, float (&f)[8]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[2 * i] = __uint_as_float(v[i] << 16);
    f[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
  }
}

__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }

}  // namespace moe
