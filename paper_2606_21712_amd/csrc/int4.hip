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
  // (hi - lo in halves, the same bits: whole it may be past fp32)
  const float step = zeros ? (0.5f * hi - 0.5f * lo) / 7.5f : fmaxf(hi, 0.f - lo) / 7.0f;
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
                                                       uint8_t* __restrict__ out_scales) {
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
    const int64_t r = row0 + i / (4 * gpt) * 4 + i % 4;
    const int grp = kt * gpt + i / 4 % gpt;
    const bool in = r < rows && grp < K / g;
    const int64_t at = (mat * rows + r) * (K / g) + grp;
    const uint16_t sc = in ? scales[at] : uint16_t(0);
    const int64_t to = tile * gpt * kInt4Rows + i;
    if (zeros)
      reinterpret_cast<uint32_t*>(out_scales)[to] = uint32_t(sc) << 16 | 0x4300u | (in ? zeros[at] & 15u : 8u);
    else
      reinterpret_cast<uint16_t*>(out_scales)[to] = sc;
  }
}

// ------------------------------------------------------------------ matrix times a few rows
// y[t][n] = sum_k W[n][k] x[t][k].  A wavefront multiplies NT tiles of 16 weight rows with up to
// 16 C rows of x on the matrix cores: the weights are the A operand, expanded in registers, x the B
// operand, read from the caches.  KS wavefronts deal the tiles along k among themselves and add
// their sums in LDS, in their order; P steps of weights are in flight.
//
// Bound by the read of the weights where they are many: 8 x 28672 x 4096, 65 MB in 14.5 us of which
// some 4 are launch and ramp (loads that stay in the caches: 62 MB took 19.4 us with streaming ones
// against 19.0, 8 MB 6.8 against 6.2).  1 x 4096 x 4096 takes 5.1 us and 5 x 1003 x 7168 6.6: launch
// and latency.  From 17 rows on x passes through the L2 more often than the weights do.
template <int NT, int C, int KS, int GPT, bool ZEROS, int P>
__global__ __launch_bounds__(64 * KS, 4) void matvec_int4_kernel(const uint16_t* __restrict__ x,
                                                                 Int4Weights<GPT, ZEROS, kCached> w, int T, int N, int K,
                                                                 uint16_t* __restrict__ y) {
  using W = Int4Weights<GPT, ZEROS, kCached>;
  __shared__ f32x4 part[KS][NT * C][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g4 = lane >> 4, col = lane & 15;
  const int t0 = int(blockIdx.y) * 16 * C;
  const int steps = int4_col_tiles(K);
  const int mine = (steps - wave + KS - 1) / KS;
  const auto v = w.view(0, N, K, lane);
  const int tiles = int(int4_row_tiles(N)), rt = int(blockIdx.x) * NT;
  const auto bx = buffer_of(x + int64_t(t0) * K, int64_t(min(T - t0, 16 * C)) * K * 2);
  int xat[C];
#pragma unroll
  for (int c = 0; c < C; ++c) xat[c] = (16 * c + W::token(lane)) * K * 2 + W::x_at(lane);   // past the last row: zeros
  f32x4 acc[NT][C][1];
#pragma unroll
  for (int r = 0; r < NT; ++r)
#pragma unroll
    for (int c = 0; c < C; ++c) acc[r][c][0] = f32x4{0.f, 0.f, 0.f, 0.f};
  typename W::Step ws[P][NT];
  u32x4 xb[C][W::kXRegs];
  auto load_w = [&](int p, int i) {
#pragma unroll
    for (int r = 0; r < NT; ++r) W::load(ws[p][r], v, rt + r, wave + i * KS, i < mine && rt + r < tiles);
  };
  auto load_x = [&](int i) {
#pragma unroll
    for (int c = 0; c < C; ++c) W::load_x(xb[c], bx, xat[c], wave + i * KS, K, i < mine);
  };
#pragma unroll
  for (int p = 0; p < P; ++p) load_w(p, p);
  load_x(0);
  for (int i = 0; i < mine; i += P) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      typename W::template Sums<C> sums;
      W::template sums<C>(sums, xb, lane);
#pragma unroll
      for (int r = 0; r < NT; ++r) W::template add<C>(acc[r], ws[p][r], xb, sums);
      load_x(i + p + 1);
      load_w(p, i + p + P);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
#pragma unroll
  for (int r = 0; r < NT; ++r)
#pragma unroll
    for (int c = 0; c < C; ++c) part[wave][r * C + c][lane] = acc[r][c][0];
  __syncthreads();
  for (int q = wave; q < NT * C; q += KS) {
    f32x4 s = part[0][q][lane];
#pragma unroll
    for (int i = 1; i < KS; ++i) s += part[i][q][lane];
    const int t = t0 + 16 * (q % C) + col;
    const int n = (int(blockIdx.x) * NT + q / C) * kInt4Rows + 4 * g4;
    if (t < T) {
      uint16_t* out = y + int64_t(t) * N + n;
      const uint32_t a = pack_bf16x2(s[0], s[1]), b = pack_bf16x2(s[2], s[3]);
      if (n + 4 <= N && (N & 3) == 0) {
        *reinterpret_cast<u32x2*>(out) = u32x2{a, b};
      } else {
        const uint16_t e[4] = {uint16_t(a), uint16_t(a >> 16), uint16_t(b), uint16_t(b >> 16)};
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (n + i < N) out[i] = e[i];
      }
    }
  }
}

template <int NT, int C, int KS, int GPT, bool ZEROS, int P>
void mv(const uint16_t* x, const Int4Ref& w, int T, int N, int K, uint16_t* y, hipStream_t s) {
  const dim3 grid(unsigned((int4_row_tiles(N) + NT - 1) / NT), unsigned((T + 16 * C - 1) / (16 * C)));
  const Int4Weights<GPT, ZEROS, kCached> v = {w.codes, w.scales};
  MOE_LAUNCH("matvec_int4", (matvec_int4_kernel<NT, C, KS, GPT, ZEROS, P>), grid, dim3(64 * KS), s, x, v, T, N, K, y);
}

template <int GPT, bool ZEROS>
hipError_t mv_group(const uint16_t* x, const Int4Ref& w, int T, int N, int K, uint16_t* y, int num_cu, hipStream_t s) {
  // Row tiles that share the rows of x, which pass through the caches for every step: as many as leave
  // the compute units work.  us with 1, 2 and 4 of T x N x K: 1 x 4096 x 4096 6.2, 7.3, 9.3; 4 x 7168 x
  // 2048 8.6, 6.3, 7.3; 12 x 8192 x 8192 20, 13.8, 19.4; 7 x 12550 x 9088 32, 20, 17; 18 x 4096 x 4096
  // 9.7, 10.2, 11.6; 40 x 2261 x 4608 18.5, 14.3, 15.2; 32 x 28672 x 4096 60, 39, 25.  Rows past 32 are
  // another workgroup's: 64 x 4096 x 14336 took 55 us with all rows in one, and takes 35 with two.
  const int64_t units = int4_row_tiles(N) * ((T + 31) / 32);
  const int nt = units >= 3 * num_cu ? 4 : units > num_cu ? 2 : 1;
  if (T <= 16) {
    if (nt == 4)
      mv<4, 1, 8, GPT, ZEROS, 1>(x, w, T, N, K, y, s);
    else if (nt == 2)
      mv<2, 1, 8, GPT, ZEROS, 2>(x, w, T, N, K, y, s);
    else
      mv<1, 1, 8, GPT, ZEROS, 2>(x, w, T, N, K, y, s);
  }
  else if (nt == 4)
    mv<4, 2, 8, GPT, ZEROS, 1>(x, w, T, N, K, y, s);
  else if (nt == 2)
    mv<2, 2, 8, GPT, ZEROS, 1>(x, w, T, N, K, y, s);
  else
    mv<1, 2, 8, GPT, ZEROS, 2>(x, w, T, N, K, y, s);
  return hipGetLastError();
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
                            int64_t rows, int K, int group, uint8_t* out_codes, uint8_t* out_scales, hipStream_t s) {
  const dim3 grid(unsigned(matrices * int4_row_tiles(rows) * int4_col_tiles(K)));
  MOE_LAUNCH("pack_int4", pack_int4_kernel, grid, dim3(64), s, codes, scales, zeros, rows, K, group, out_codes,
             out_scales);
  return hipGetLastError();
}

hipError_t launch_matvec_int4(const uint16_t* x, const Int4Ref& w, int T, int N, int K, int group, bool zeros,
                              uint16_t* y, int num_cu, hipStream_t s) {
  if (group == 32)
    return zeros ? mv_group<4, true>(x, w, T, N, K, y, num_cu, s) : mv_group<4, false>(x, w, T, N, K, y, num_cu, s);
  if (group == 64)
    return zeros ? mv_group<2, true>(x, w, T, N, K, y, num_cu, s) : mv_group<2, false>(x, w, T, N, K, y, num_cu, s);
  return zeros ? mv_group<1, true>(x, w, T, N, K, y, num_cu, s) : mv_group<1, false>(x, w, T, N, K, y, num_cu, s);
}

}  // namespace moe
