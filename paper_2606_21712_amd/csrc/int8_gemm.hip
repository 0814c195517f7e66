// Products of 8-bit integer codes on gfx950: packing the weights, and
//   y[t, n] = s_x[t] s_w[n] sum_k q_x[t, k] q_w[n, k] (+ b[n]),
// plain, or the two products of a gated block with silu(g) u on top.
//
// The sums are exact in 32 bits (K <= kInt8MaxK), whatever their order, so how a product is cut up
// does not show in its result.
#include "int8.h"
#include "launch_rules.h"
#include "lds_stage.h"
#include "moe_internal.h"
#include "weight_stream.h"

namespace moe {
namespace {

__device__ __forceinline__ i32x4 mfma_i8(u32x4 a, u32x4 b, i32x4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// ------------------------------------------------------------------ pack
// One wavefront a step of 16 rows x 64 columns.
__global__ __launch_bounds__(64) void pack_int8_kernel(const int8_t* __restrict__ codes, int64_t rows, int K, int steps,
                                                       int8_t* __restrict__ out) {
  const int lane = threadIdx.x;
  const int64_t step = blockIdx.x;
  const int64_t row = step / steps * 16 + (lane & 15);
  const int k = int(step % steps) * 64 + 16 * (lane >> 4);
  u32x4 v = {0u, 0u, 0u, 0u};
  if (row < rows && k < K) v = *reinterpret_cast<const u32x4*>(codes + row * K + k);
  reinterpret_cast<u32x4*>(out)[step * 64 + lane] = v;
}

// A sum times its two scales.  No operation is contracted with the next: the result's bits are the formula's.
__device__ __forceinline__ float scaled(int32_t sum, float sx, float sw) {
  return __fmul_rn(__fmul_rn(float(sum), sx), sw);
}

// Four results of consecutive channels n .. n + 3 of a row that starts at `row`.
__device__ __forceinline__ void store4(uint16_t* row, int n, int N, const float (&v)[4]) {
  const uint32_t a = pack_bf16x2(v[0], v[1]), b = pack_bf16x2(v[2], v[3]);
  if (n + 4 <= N && (N & 3) == 0) {
    *reinterpret_cast<u32x2*>(row + n) = u32x2{a, b};
  } else {
    const uint16_t e[4] = {uint16_t(a), uint16_t(a >> 16), uint16_t(b), uint16_t(b >> 16)};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (n + i < N) row[n + i] = e[i];
  }
}

// ------------------------------------------------------------------ few rows of x
// A wavefront multiplies NT tiles of 16 weight rows (GATED: NT / 2 of either matrix) with 16 C rows of x:
// the weights are the first operand, streamed from memory into registers, x the second, from the caches.
// KS wavefronts deal the steps along k among themselves and add their sums in LDS; P steps are in flight.
template <bool GATED, int NT, int C, int KS, int P>
__global__ __launch_bounds__(64 * KS) void few_int8_kernel(Int8Product p) {
  __shared__ i32x4 part[KS][NT * C][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t0 = int(blockIdx.y) * 16 * C;
  constexpr int kTiles = GATED ? NT / 2 : NT;     // of a matrix
  const int steps = p.steps;
  const int mine = (steps - wave + KS - 1) / KS;
  const int tiles = (p.N + 15) / 16, rt = int(blockIdx.x) * kTiles;
  const int64_t tile_bytes = int64_t(steps) * 1024;
  Buffer bw[NT];
#pragma unroll
  for (int r = 0; r < NT; ++r) {
    const int tile = rt + r % kTiles;
    bw[r] = buffer_of((GATED && r >= kTiles ? p.w1 : p.w0) + tile * tile_bytes, tile < tiles ? tile_bytes : 0);
  }
  const auto bx = buffer_of(p.x + int64_t(t0) * p.K, int64_t(min(p.T - t0, 16 * C)) * p.K);
  int xat[C];
#pragma unroll
  for (int c = 0; c < C; ++c) xat[c] = (16 * c + (lane & 15)) * p.K + 16 * (lane >> 4);   // past the last row: zeros
  i32x4 acc[NT][C];
#pragma unroll
  for (int r = 0; r < NT; ++r)
#pragma unroll
    for (int c = 0; c < C; ++c) acc[r][c] = i32x4{0, 0, 0, 0};
  u32x4 w[P][NT], x[P][C];
  auto load = [&](int q, int i) {
    const int at = wave + i * KS;
#pragma unroll
    for (int r = 0; r < NT; ++r) w[q][r] = load16<kCached>(bw[r], i < mine, 16 * lane, at * 1024);
#pragma unroll
    for (int c = 0; c < C; ++c) x[q][c] = load16<kCached>(bx, i < mine, xat[c], at * 64);
  };
#pragma unroll
  for (int q = 0; q < P; ++q) load(q, q);
  for (int i = 0; i < mine; i += P) {
#pragma unroll
    for (int q = 0; q < P; ++q) {
#pragma unroll
      for (int r = 0; r < NT; ++r)
#pragma unroll
        for (int c = 0; c < C; ++c) acc[r][c] = mfma_i8(w[q][r], x[q][c], acc[r][c]);
      load(q, i + q + P);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
#pragma unroll
  for (int r = 0; r < NT; ++r)
#pragma unroll
    for (int c = 0; c < C; ++c) part[wave][r * C + c][lane] = acc[r][c];
  __syncthreads();
  for (int q = wave; q < kTiles * C; q += KS) {
    i32x4 s = part[0][q][lane], u = {0, 0, 0, 0};
#pragma unroll
    for (int i = 1; i < KS; ++i) s += part[i][q][lane];
    if (GATED) {
#pragma unroll
      for (int i = 0; i < KS; ++i) u += part[i][kTiles * C + q][lane];
    }
    const int t = t0 + 16 * (q % C) + (lane & 15);
    const int n = (rt + q / C) * 16 + 4 * (lane >> 4);
    if (t >= p.T || n >= p.N) continue;
    const float sx = p.x_scales[t];
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int ni = min(n + i, p.N - 1);
      v[i] = scaled(s[i], sx, p.s0[ni]);
      if (GATED)
        v[i] = silu(v[i]) * scaled(u[i], sx, p.s1[ni]);
      else if (p.bias != nullptr)
        v[i] = __fadd_rn(v[i], bf16_to_f32(p.bias[ni]));
    }
    store4(p.y + int64_t(t) * p.N, n, p.N, v);
  }
}

template <bool GATED>
void few(const Int8Product& p, hipStream_t s) {
  const int tiles = (p.N + 15) / 16;
  const char* name = GATED ? "gated_int8_few" : "matmul_int8_few";
  if (p.T <= 16)
    MOE_LAUNCH(name, (few_int8_kernel<GATED, GATED ? 2 : 1, 1, 8, 4>), dim3(tiles, 1), dim3(512), s, p);
  else
    MOE_LAUNCH(name, (few_int8_kernel<GATED, 2, 2, 8, 2>), dim3(GATED ? tiles : (tiles + 1) / 2, (p.T + 31) / 32),
               dim3(512), s, p);
}

}  // namespace

hipError_t launch_pack_int8(const int8_t* codes, int64_t rows, int K, int8_t* out, hipStream_t s) {
  const int steps = (K + 127) / 128 * 2;
  MOE_LAUNCH("pack_int8", pack_int8_kernel, dim3(unsigned((rows + 15) / 16 * steps)), dim3(64), s, codes, rows, K, steps,
             out);
  return hipGetLastError();
}

hipError_t launch_int8_product(const Int8Product& p, int num_cu, hipStream_t s) {
  if (p.w1 != nullptr)
    few<true>(p, s);
  else
    few<false>(p, s);
  return hipGetLastError();
}

}  // namespace moe
