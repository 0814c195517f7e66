// What the kernels of int8 products share: the tile list, the scales, and how results leave.
#pragma once
#include "int8.h"
#include "lds_stage.h"
#include "moe_internal.h"
#include "weight_stream.h"

namespace moe {

// A sum times its two scales, and with its bias.  No product is contracted with a sum (an fma rounds
// once): the result's bits are those of the formula, operation by operation, in every kernel.
__device__ __forceinline__ float scaled(int32_t sum, float sx, float sw) {
#pragma clang fp contract(off)
  return float(sum) * sx * sw;
}
__device__ __forceinline__ float biased(float v, float bias) {
#pragma clang fp contract(off)
  return v + bias;
}

// A result, from its sum, or (gated) its two.
template <bool GATED>
__device__ __forceinline__ float result(int32_t sum, int32_t up, float sx, float s0, float s1, bool bias) {
  const float v = scaled(sum, sx, s0);
  if (GATED) return silu(v) * scaled(up, sx, s1);
  return bias ? biased(v, s1) : v;
}

// The scale of channel n of w0, and of w1 or the bias; past the last channel its own.
template <bool GATED>
__device__ __forceinline__ void channel_scales(const Int8Product& p, int n, float& s0, float& s1) {
  n = min(n, p.N - 1);
  s0 = p.s0[n];
  s1 = GATED ? p.s1[n] : p.bias != nullptr ? bf16_to_f32(p.bias[n]) : 0.f;
}

// 16 bytes at any element of a row: rows of an odd number of channels begin anywhere.
typedef u32x4 __attribute__((aligned(2))) u32x4_any;

// Up to eight results, whole pieces where they are, to channels from n on of a row.
__device__ __forceinline__ void put_piece(uint16_t* row, int n, int N, const uint8_t* from) {
  if (n + 8 <= N) {
    *reinterpret_cast<u32x4_any*>(row + n) = *reinterpret_cast<const u32x4*>(from);
  } else {
    for (int k = 0; k < N - n; ++k) row[n + k] = reinterpret_cast<const uint16_t*>(from)[k];
  }
}

// Tile L of the list: four tiles of rows by eight of columns at a time, so that the tiles that an XCD works on
// share a few panels of both operands.
struct TileAt {
  int m, n;
};
__device__ __forceinline__ TileAt tile_at(int L, int mtiles, int ntiles) {
  const int mb = L / (4 * ntiles), rem = L - mb * 4 * ntiles;
  const int bm = min(4, mtiles - 4 * mb);
  const int ng = rem / (bm * 8), in = rem - ng * bm * 8;
  return {4 * mb + in % bm, ng * 8 + in / bm};
}

// 16 bytes a lane from global memory to 1 KB of LDS, or zeros.
template <int POLICY>
__device__ __forceinline__ void load_lds(const Buffer& b, bool on, uint8_t* to, int lane_at, int at) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(b.at(on), to, 16, lane_at, at, 0, POLICY);
}

// The order of a group: P products with R reads from LDS and V loads spread out between them.
template <int P, int R, int V, int I = 0>
struct Mix {
  static __device__ __forceinline__ void order() {
    if constexpr (I < P) {
      constexpr int r = (I + 1) * R / P - I * R / P, v = (I + 1) * V / P - I * V / P;
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      if constexpr (r > 0) __builtin_amdgcn_sched_group_barrier(0x100, r, 0);
      if constexpr (v > 0) __builtin_amdgcn_sched_group_barrier(0x020, v, 0);
      Mix<P, R, V, I + 1>::order();
    }
  }
};

// What the lanes of a wavefront wrote to LDS is read by others of them after this, and the other way about: they
// run together, only the compiler must not move either past it.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// s_waitcnt: every LDS read done, and all but the last n loads.
constexpr int wait_all_but(int n) { return 0x0070 | (n & 15) | ((n >> 4) << 14); }

}  // namespace moe
