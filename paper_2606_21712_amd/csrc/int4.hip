// 4-bit weights with group scales on gfx950: quantizing, packing, and products with a few rows.
#include "int4.h"
#include "moe_internal.h"

namespace moe {
namespace {

// ------------------------------------------------------------------ quantize
// One wavefront per 64 groups: a lane reads its group's g values and writes g / 2 bytes of
// codes, the scale and the zero point.  A set-up step, run once for a matrix.
template <int G>
__global__ __launch_bounds__(256) void quantize_int4_kernel(const uint16_t* __restrict__ src, int64_t groups,
                                                            uint8_t* __restrict__ codes,
                                                            uint16_t* __restrict__ scales,
                                                            uint8_t* __restrict__ zeros) {
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (i >= groups) return;
  const u32x4* in = reinterpret_cast<const u32x4*>(src + i * G);
  float lo = 0.f, hi = 0.f;
  for (int b = 0; b < G / 8; ++b) {
    const u32x4 v = in[b];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float x0 = __uint_as_float(v[w] << 16), x1 = __uint_as_float(v[w] & 0xFFFF0000u);
      lo = fminf(lo, fminf(x0, x1));
      hi = fmaxf(hi, fmaxf(x0, x1));
    }
  }
  // the step, rounded to bf16 before it is used: codes are of the scale that is stored
  const float step = zeros ? (hi - lo) / 15.0f : fmaxf(hi, 0.f - lo) / 7.0f;
  const uint16_t sb = uint16_t(pack_bf16x2(step, 0.f) & 0xFFFFu);
  const float s = bf16_to_f32(sb);
  const float z = !zeros ? 8.0f : s > 0.f ? fminf(rintf(-lo / s), 15.0f) : 0.0f;
  scales[i] = sb;
  if (zeros) zeros[i] = uint8_t(z);
  for (int b = 0; b < G / 8; ++b) {
    const u32x4 v = in[b];
    uint32_t out = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float x0 = __uint_as_float(v[w] << 16), x1 = __uint_as_float(v[w] & 0xFFFF0000u);
      const float q0 = s > 0.f ? rintf(x0 / s) + z : z, q1 = s > 0.f ? rintf(x1 / s) + z : z;
      out |= uint32_t(fminf(fmaxf(q0, 0.f), 15.f)) << (8 * w);
      out |= uint32_t(fminf(fmaxf(q1, 0.f), 15.f)) << (8 * w + 4);
    }
    reinterpret_cast<uint32_t*>(codes + i * (G / 2))[b] = out;
  }
}

// ------------------------------------------------------------------ pack
// One block of 64 lanes per tile of the output, in the order of the tiles.
__global__ __launch_bounds__(64) void pack_int4_kernel(const uint8_t* __restrict__ codes,
                                                       const uint16_t* __restrict__ scales,
                                                       const uint8_t* __restrict__ zeros, int64_t rows, int K, int g,
                                                       uint8_t* __restrict__ out_codes,
                                                       uint16_t* __restrict__ out_scales,
                                                       uint8_t* __restrict__ out_zeros) {
  const int lane = threadIdx.x;
  const int64_t tile = blockIdx.x;
  const int64_t ct = int4_col_tiles(K), rt = int4_row_tiles(rows);
  const int kt = int(tile % ct);
  const int64_t row0 = tile / ct % rt * kInt4Rows, mat = tile / (ct * rt);
  const int64_t row = row0 + (lane & 15);
  u32x4 v;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int k = kt * kInt4Cols + 32 * j + 8 * (lane >> 4);
    uint32_t w = 0x88888888u;                     // padding: never multiplied by anything but 0
    if (row < rows && k < K) {                    // K % 32 == 0: all eight or none
      const uint32_t in = *reinterpret_cast<const uint32_t*>(codes + (mat * rows + row) * (K / 2) + k / 2);
      w = 0;
#pragma unroll
      for (int c = 0; c < 8; ++c) w |= ((in >> (4 * c)) & 15u) << (4 * ((c >> 1) + 4 * (c & 1)));
    }
    v[j] = w;
  }
  reinterpret_cast<u32x4*>(out_codes + tile * kInt4TileBytes)[lane] = v;
  const int gpt = kInt4Cols / g;
  for (int i = lane; i < gpt * kInt4Rows; i += 64) {
    const int64_t r = row0 + i % kInt4Rows;
    const int grp = kt * gpt + i / kInt4Rows;
    const bool in = r < rows && grp < K / g;
    const int64_t at = (mat * rows + r) * (K / g) + grp;
    out_scales[tile * gpt * kInt4Rows + i] = in ? scales[at] : uint16_t(0);
    if (out_zeros) out_zeros[tile * gpt * kInt4Rows + i] = in ? zeros[at] : uint8_t(8);
  }
}

// ------------------------------------------------------------------ matrix times a few rows
// y[t][n] = sum_k W[n][k] x[t][k].  A wavefront multiplies one tile of 16 weight rows with up
// to 16 C rows of x on the matrix cores: the weights are the A operand, expanded in registers,
// x the B operand, read from the caches.  The workgroup's wavefronts deal the tiles along k
// among themselves and add their sums in LDS, in the order of the wavefronts.
constexpr int kMvWaves = 8;

template <int C, int GPT, bool ZEROS>
__global__ __launch_bounds__(64 * kMvWaves) void matvec_int4_kernel(const uint16_t* __restrict__ x,
                                                                    const uint8_t* __restrict__ codes,
                                                                    const uint16_t* __restrict__ scales,
                                                                    const uint8_t* __restrict__ zeros, int T, int N,
                                                                    int K, uint16_t* __restrict__ y) {
  __shared__ f32x4 part[kMvWaves][C][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int g4 = lane >> 4, col = lane & 15;
  const int t0 = int(blockIdx.y) * 16 * C;
  const int ct = int4_col_tiles(K);
  f32x4 acc[C];
#pragma unroll
  for (int c = 0; c < C; ++c) acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int kt = wave; kt < ct; kt += kMvWaves) {
    Int4Tile<GPT, ZEROS> w;
    int4_load(w, codes, scales, zeros, int64_t(blockIdx.x) * ct + kt, lane);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      bf16x8 xb[4];
      const int t = t0 + 16 * c + col;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int k = kt * kInt4Cols + 32 * j + 8 * g4;
        u32x4 v = {0u, 0u, 0u, 0u};
        if (t < T && k < K) v = *reinterpret_cast<const u32x4*>(x + int64_t(t) * K + k);
        xb[j] = __builtin_bit_cast(bf16x8, v);
      }
      float xs[GPT];
      int4_group_sums<GPT>(xs, xb);
      int4_accumulate<GPT, ZEROS>(acc[c], w, xb, xs);
    }
  }
#pragma unroll
  for (int c = 0; c < C; ++c) part[wave][c][lane] = acc[c];
  __syncthreads();
  for (int c = wave; c < C; c += kMvWaves) {
    f32x4 s = part[0][c][lane];
#pragma unroll
    for (int w = 1; w < kMvWaves; ++w) s += part[w][c][lane];
    const int t = t0 + 16 * c + col;
    const int n = int(blockIdx.x) * kInt4Rows + 4 * g4;
    if (t < T) {
      uint16_t* out = y + int64_t(t) * N + n;
      const uint32_t a = pack_bf16x2(s[0], s[1]), b = pack_bf16x2(s[2], s[3]);
      if (n + 4 <= N && (N & 3) == 0) {
        *reinterpret_cast<u32x2*>(out) = u32x2{a, b};
      } else {
        const uint16_t v[4] = {uint16_t(a), uint16_t(a >> 16), uint16_t(b), uint16_t(b >> 16)};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (n + i < N) out[i] = v[i];
      }
    }
  }
}

template <int C, int GPT>
hipError_t launch_mv(const uint16_t* x, const uint8_t* codes, const uint16_t* scales, const uint8_t* zeros, int T,
                     int N, int K, uint16_t* y, hipStream_t s) {
  const dim3 grid(unsigned(int4_row_tiles(N)), unsigned((T + 16 * C - 1) / (16 * C)));
  const dim3 block(64 * kMvWaves);
  if (zeros)
    MOE_LAUNCH("matvec_int4", (matvec_int4_kernel<C, GPT, true>), grid, block, s, x, codes, scales, zeros, T, N, K, y);
  else
    MOE_LAUNCH("matvec_int4", (matvec_int4_kernel<C, GPT, false>), grid, block, s, x, codes, scales, zeros, T, N, K, y);
  return hipGetLastError();
}

template <int C>
hipError_t launch_mv_g(const uint16_t* x, const uint8_t* codes, const uint16_t* scales, const uint8_t* zeros, int T,
                       int N, int K, int group, uint16_t* y, hipStream_t s) {
  if (group == 32) return launch_mv<C, 4>(x, codes, scales, zeros, T, N, K, y, s);
  if (group == 64) return launch_mv<C, 2>(x, codes, scales, zeros, T, N, K, y, s);
  return launch_mv<C, 1>(x, codes, scales, zeros, T, N, K, y, s);
}

}  // namespace

hipError_t launch_quantize_int4(const uint16_t* src, int64_t groups, int group, uint8_t* codes, uint16_t* scales,
                                uint8_t* zeros, hipStream_t s) {
  const dim3 grid(unsigned((groups + 255) / 256)), block(256);
  if (group == 32)
    MOE_LAUNCH("quantize_int4", (quantize_int4_kernel<32>), grid, block, s, src, groups, codes, scales, zeros);
  else if (group == 64)
    MOE_LAUNCH("quantize_int4", (quantize_int4_kernel<64>), grid, block, s, src, groups, codes, scales, zeros);
  else
    MOE_LAUNCH("quantize_int4", (quantize_int4_kernel<128>), grid, block, s, src, groups, codes, scales, zeros);
  return hipGetLastError();
}

hipError_t launch_pack_int4(const uint8_t* codes, const uint16_t* scales, const uint8_t* zeros, int64_t matrices,
                            int64_t rows, int K, int group, uint8_t* out_codes, uint16_t* out_scales,
                            uint8_t* out_zeros, hipStream_t s) {
  const dim3 grid(unsigned(matrices * int4_row_tiles(rows) * int4_col_tiles(K)));
  MOE_LAUNCH("pack_int4", pack_int4_kernel, grid, dim3(64), s, codes, scales, zeros, rows, K, group, out_codes,
             out_scales, out_zeros);
  return hipGetLastError();
}

hipError_t launch_matvec_int4(const uint16_t* x, const Int4Ref& w, int T, int N, int K, int group, uint16_t* y,
                              int num_cu, hipStream_t s) {
  (void)num_cu;
  if (T <= 16) return launch_mv_g<1>(x, w.codes, w.scales, w.zeros, T, N, K, group, y, s);
  if (T <= 32) return launch_mv_g<2>(x, w.codes, w.scales, w.zeros, T, N, K, group, y, s);
  return launch_mv_g<4>(x, w.codes, w.scales, w.zeros, T, N, K, group, y, s);
}

}  // namespace moe
