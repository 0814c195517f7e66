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
// A wavefront multiplies NT tiles of 16 weight rows (GATED: one of either matrix) with 16 rows of x: the weights are
// the first operand, streamed from memory into registers, x the second, from the caches.  KS wavefronts deal the
// steps of 128 columns along k among themselves (both halves of a line of x to one of them) and add their sums in
// LDS; P steps are in flight.  More rows are other workgroups', which find the weights in the L2.
template <bool GATED, int NT, int KS, int P, int POLICY>
__global__ __launch_bounds__(64 * KS) void few_int8_kernel(Int8Product p) {
  __shared__ i32x4 part[KS][NT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t0 = int(blockIdx.y) * 16;
  constexpr int kTiles = GATED ? NT / 2 : NT;     // of a matrix
  const int pairs = p.steps / 2;
  const int mine = (pairs - wave + KS - 1) / KS;
  const int tiles = (p.N + 15) / 16, rt = int(blockIdx.x) * kTiles;
  const int64_t tile_bytes = int64_t(p.steps) * 1024;
  Buffer bw[NT];
#pragma unroll
  for (int r = 0; r < NT; ++r) {
    const int tile = rt + r % kTiles;
    bw[r] = buffer_of((GATED && r >= kTiles ? p.w1 : p.w0) + tile * tile_bytes, tile < tiles ? tile_bytes : 0);
  }
  const auto bx = buffer_of(p.x + int64_t(t0) * p.K, int64_t(min(p.T - t0, 16)) * p.K);
  const int chunk = 16 * (lane >> 4);
  const int xat = (lane & 15) * p.K + chunk;      // past the last row: zeros
  // what the wavefronts that finish a tile need besides: loaded first, not once the sums are there
  const int t = t0 + (lane & 15), n = (rt + wave) * 16 + 4 * (lane >> 4);
  const bool finish = wave < kTiles && t < p.T && n < p.N;
  float sx = 0.f, s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
  if (finish) {
    sx = p.x_scales[t];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int ni = min(n + i, p.N - 1);
      s0[i] = p.s0[ni];
      if (GATED)
        s1[i] = p.s1[ni];
      else if (p.bias != nullptr)
        s1[i] = bf16_to_f32(p.bias[ni]);
    }
  }
  i32x4 acc[NT];
#pragma unroll
  for (int r = 0; r < NT; ++r) acc[r] = i32x4{0, 0, 0, 0};
  u32x4 w[P][NT][2], x[P][2];
  auto load = [&](int q, int i) {
    const int at = wave + i * KS;
#pragma unroll
    for (int r = 0; r < NT; ++r)
#pragma unroll
      for (int h = 0; h < 2; ++h) w[q][r][h] = load16<POLICY>(bw[r], i < mine, 16 * lane, at * 2048 + h * 1024);
#pragma unroll
    for (int h = 0; h < 2; ++h)                   // columns past K: zeros, whatever the offset's range check counts
      x[q][h] = load16<kCached>(bx, i < mine, at * 128 + h * 64 + chunk < p.K ? xat : kPast, at * 128 + h * 64);
  };
#pragma unroll
  for (int q = 0; q < P; ++q) load(q, q);
  for (int i = 0; i < mine; i += P) {
#pragma unroll
    for (int q = 0; q < P; ++q) {
#pragma unroll
      for (int r = 0; r < NT; ++r)
#pragma unroll
        for (int h = 0; h < 2; ++h) acc[r] = mfma_i8(w[q][r][h], x[q][h], acc[r]);
      load(q, i + q + P);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
#pragma unroll
  for (int r = 0; r < NT; ++r) part[wave][r][lane] = acc[r];
  __syncthreads();
  if (!finish) return;
  i32x4 s = part[0][wave][lane], u = {0, 0, 0, 0};
#pragma unroll
  for (int i = 1; i < KS; ++i) s += part[i][wave][lane];
  if (GATED) {
#pragma unroll
    for (int i = 0; i < KS; ++i) u += part[i][kTiles + wave][lane];
  }
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[i] = scaled(s[i], sx, s0[i]);
    if (GATED)
      v[i] = silu(v[i]) * scaled(u[i], sx, s1[i]);
    else if (p.bias != nullptr)
      v[i] = biased(v[i], s1[i]);
  }
  store4(p.y + int64_t(t) * p.N, n, p.N, v);
}

template <bool GATED, int NT>
void few(const Int8Product& p, bool stream, hipStream_t s) {
  const int tiles = (p.N + 15) / 16, each = GATED ? NT / 2 : NT;
  const char* name = GATED ? "gated_int8_few" : "matmul_int8_few";
  const dim3 grid((tiles + each - 1) / each, (p.T + 15) / 16), block(512);
  if (stream)
    MOE_LAUNCH(name, (few_int8_kernel<GATED, NT, 8, 2, kStream>), grid, block, s, p);
  else
    MOE_LAUNCH(name, (few_int8_kernel<GATED, NT, 8, 2, kCached>), grid, block, s, p);
}

// ------------------------------------------------------------------ many rows of x
// Tiles of 64 MI rows of x by 64 NI weight rows (GATED: 32 NI of either matrix) for four wavefronts, 2 x 2, of
// 32 MI x 32 NI each.  A stage holds 128 columns of both operands in LDS, the weights in their packed pieces,
// x in rows of 128 bytes whose 16-byte chunks are permuted so that 16 rows of one column lie in different banks;
// global -> LDS loads fill a ring of NS stages.  A stage is four groups of 32 columns; a group's operands are
// read from LDS while the one before it is multiplied, also across the border of two stages: the barrier that
// hands over a stage stands before the last group, whose operands are in registers by then.
__device__ __forceinline__ i32x16 mfma32_i8(u32x4 a, u32x4 b, i32x16 c) {
  return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
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

template <bool GATED, int MI, int NI>
struct Int8Tile {
  static constexpr int kRows = 64 * MI;                      // of x
  static constexpr int kWRows = 64 * NI;                     // of weights
  static constexpr int kCols = GATED ? kWRows / 2 : kWRows;  // of y
  static constexpr int kXBytes = kRows * 128, kWBytes = kWRows * 128;
  static constexpr int kWaveCols = kCols / 2;                // of y, of a wavefront
  static constexpr int kPitch = kWaveCols * 2 + 16;          // of a row on its way out
  static_assert(2 * 32 * kPitch <= kWBytes && 8 * kCols <= kXBytes, "the results pass through the ring's places");
};

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

// 16 bytes at any element of a row: rows of an odd number of channels begin anywhere.
typedef u32x4 __attribute__((aligned(2))) u32x4_any;

// The results of 32 rows from tb on, NI x 32 sums a wavefront: a lane holds channels 8 b + 4 (lane / 32) + 0..3 of
// row lane % 32 of each 32 x 32.  They go through LDS of the wavefront's own, to leave as whole pieces of rows.
template <bool GATED, int NI>
__device__ __forceinline__ void put_rows(const Int8Product& p, const i32x16 (&acc)[NI], int tb, int nb, float sx,
                                         const float* scale0, const float* scale1, uint8_t* out, int lane) {
  constexpr int kCols = GATED ? 16 * NI : 32 * NI, kPitch = kCols * 2 + 16;
  const int r32 = lane & 31, half = lane >> 5;
#pragma unroll
  for (int nc = 0; nc < (GATED ? NI / 2 : NI); ++nc)
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int at = nc * 32 + 8 * b + 4 * half;
      const f32x4 s0 = *reinterpret_cast<const f32x4*>(scale0 + at);
      const f32x4 s1 = *reinterpret_cast<const f32x4*>(scale1 + at);
      float v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[i] = scaled(acc[GATED ? 2 * nc : nc][4 * b + i], sx, s0[i]);
        if (GATED)
          v[i] = silu(v[i]) * scaled(acc[GATED ? 2 * nc + 1 : 0][4 * b + i], sx, s1[i]);
        else if (p.bias != nullptr)
          v[i] = biased(v[i], s1[i]);
      }
      *reinterpret_cast<u32x2*>(out + r32 * kPitch + at * 2) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    }
  constexpr int kPieces = kCols / 8;                         // of a row
#pragma unroll
  for (int i = lane; i < 32 * kPieces; i += 64) {
    const int r = i / kPieces, n = nb + 8 * (i % kPieces);
    if (tb + r >= p.T) continue;
    const uint8_t* from = out + r * kPitch + (i % kPieces) * 16;
    uint16_t* to = p.y + int64_t(tb + r) * p.N + n;
    if (n + 8 <= p.N) {
      *reinterpret_cast<u32x4_any*>(to) = *reinterpret_cast<const u32x4*>(from);
    } else {
      for (int k = 0; k < p.N - n; ++k) to[k] = reinterpret_cast<const uint16_t*>(from)[k];
    }
  }
}

template <bool GATED, int MI, int NI, int XS, int WS, bool SPLIT, int POLICY>
__global__ __launch_bounds__(256, 1) void int8_gemm_kernel(Int8Product p, int mtiles, int ntiles, int parts) {
  using Tile = Int8Tile<GATED, MI, NI>;
  __shared__ __attribute__((aligned(1024))) uint8_t x0[Tile::kXBytes], x1[Tile::kXBytes], x2[XS > 2 ? Tile::kXBytes : 16],
      x3[XS > 3 ? Tile::kXBytes : 16], x4[XS > 4 ? Tile::kXBytes : 16];
  __shared__ __attribute__((aligned(1024))) uint8_t w0[Tile::kWBytes], w1[Tile::kWBytes], w2[WS > 2 ? Tile::kWBytes : 16],
      w3[WS > 3 ? Tile::kWBytes : 16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  if (p.steps < 0) {              // never taken: keeps the reads of what global -> LDS loads fill
    x0[tid] = x1[tid] = w0[tid] = w1[tid] = 0;
    x2[tid & 15] = x3[tid & 15] = x4[tid & 15] = w2[tid & 15] = w3[tid & 15] = 0;
  }
  // XCD n % 8 takes a contiguous part of the tiles
  const int tiles = mtiles * ntiles, total = tiles * parts, per = (total + 7) / 8;
  const int num = int(blockIdx.x), L = (num & 7) * per + (num >> 3);
  if (num >> 3 >= per || L >= total) return;
  const int part = SPLIT ? L / tiles : 0;
  const TileAt tile = tile_at(L - part * tiles, mtiles, ntiles);
  const int t0 = tile.m * Tile::kRows, n0 = tile.n * Tile::kCols;

  const int K = p.K, stages = p.steps / 2;
  const int first = SPLIT ? part * stages / parts : 0, KT = SPLIT ? (part + 1) * stages / parts : stages;
  const int rows = min(Tile::kRows, p.T - t0);
  const int64_t tile_bytes = int64_t(p.steps) * 1024;
  const int wtiles = min(Tile::kCols / 16, (p.N + 15) / 16 - n0 / 16);    // of either matrix
  const Buffer bx = buffer_of(p.x + int64_t(t0) * K, int64_t(rows) * K);
  const Buffer bw0 = buffer_of(p.w0 + (n0 / 16) * tile_bytes, wtiles * tile_bytes);
  const Buffer bw1 = buffer_of((GATED ? p.w1 : p.w0) + (n0 / 16) * tile_bytes, wtiles * tile_bytes);

  // A stage's loads.  x: eight rows a load, row 8 (wave + 4 i) + lane / 8, whose chunk c lies at place
  // c ^ (row / 2) % 8; rows past the tile's last lie past the buffer.  Weights: the two pieces of 16 rows.
  // Past the last stage a buffer of no bytes gives zeros, so that every step is the same code.
  const int chunk = (lane & 7) ^ ((4 * wave + (lane >> 4)) & 7);
  uint32_t xat[2 * MI], wat[NI];
#pragma unroll
  for (int i = 0; i < 2 * MI; ++i) xat[i] = uint32_t(8 * (wave + 4 * i) + (lane >> 3)) * uint32_t(K) + 16 * chunk;
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int tile16 = wave + 4 * i;
    wat[i] = uint32_t((GATED ? tile16 % (2 * NI) : tile16) * tile_bytes) + 16 * lane;
  }
  // a half of a stage's loads
  auto issue_x = [&](uint8_t* stage, int kt, int which) {
    const bool on = kt * 128 + 16 * chunk < K;                // columns past K: zeros
#pragma unroll
    for (int i = 0; i < MI; ++i)
      load_lds<kCached>(bx, kt < KT, stage + (wave + 4 * (which * MI + i)) * 1024, on ? int(xat[which * MI + i]) : kPast, kt * 128);
  };
  auto issue_w = [&](uint8_t* stage, int kt, int which) {
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int i = which * NI + j, tile16 = wave + 4 * (i >> 1);
      load_lds<POLICY>(GATED && tile16 >= 2 * NI ? bw1 : bw0, kt < KT, stage + tile16 * 2048 + (i & 1) * 1024, int(wat[i >> 1]),
               kt * 2048 + (i & 1) * 1024);
    }
  };

  // A group's operands.  x: row 32 mi + lane % 32 of the wavefront's, chunk 2 g + lane / 32.  Weights: of
  // the piece g / 2 the same chunk of 32 rows.
  const int r32 = lane & 31, half = lane >> 5;
  const int xrow = (wm * 32 * MI + r32) * 128, xswz = (r32 >> 1) & 7;
  const int wrow = (r32 >> 4) * 2048 + half * 256 + (r32 & 15) * 16;
  auto weight_tile = [&](int ni) {               // first of the two tiles of 16 rows
    return GATED ? (ni & 1 ? 2 * NI : 0) + wn * NI + (ni >> 1) * 2 : wn * 2 * NI + 2 * ni;
  };
  i32x16 acc[MI][NI];
#pragma unroll
  for (int mi = 0; mi < MI; ++mi)
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
#pragma unroll
      for (int q = 0; q < 16; ++q) acc[mi][ni][q] = 0;
  u32x4 xf[2][MI], wf[2][NI];
  auto read = [&](const uint8_t* xs, const uint8_t* ws, int g, int to) {
#pragma unroll
    for (int ni = 0; ni < NI; ++ni)
      wf[to][ni] = *reinterpret_cast<const u32x4*>(ws + wrow + weight_tile(ni) * 2048 + (g >> 1) * 1024 + (g & 1) * 512);
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
      xf[to][mi] = *reinterpret_cast<const u32x4*>(xs + xrow + mi * 4096 + ((2 * g + half) ^ xswz) * 16);
  };
  auto multiply = [&](int from) {
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
      for (int ni = 0; ni < NI; ++ni) acc[mi][ni] = mfma32_i8(wf[from][ni], xf[from][mi], acc[mi][ni]);
  };
  // Stage kt.  Each group issues a quarter of a stage's loads: the second half of the weights of stage kt + WS - 1
  // and the rows of x of stage kt + XS - 1 to the places of stage kt - 1, the first half of the weights of stage kt + WS
  // to its own.
  constexpr int kAll = 0x0070;                               // s_waitcnt: no LDS read pending
  constexpr int kAhead = (WS - 2) * (2 * MI + 2 * NI) + (XS - WS) * 2 * MI;   // later stages' loads that may be pending
  auto step = [&](uint8_t* xprev, uint8_t* xcur, uint8_t* xnxt, uint8_t* wprev, uint8_t* wcur, uint8_t* wnxt, int kt) {
    read(xcur, wcur, 1, 1);
    issue_w(wprev, kt + WS - 1, 1);
    if (XS == WS) issue_w(wprev, kt + WS - 1, 0);
    multiply(0);
    Mix<MI * NI, MI + NI, XS == WS ? 2 * NI : NI>::order();
    __builtin_amdgcn_sched_barrier(0);
    read(xcur, wcur, 2, 0);
    if (XS > WS) issue_x(xprev, kt + XS - 1, 0);
    multiply(1);
    Mix<MI * NI, MI + NI, XS == WS ? 0 : MI>::order();
    __builtin_amdgcn_sched_barrier(0);
    read(xcur, wcur, 3, 1);
    if (XS > WS) issue_x(xprev, kt + XS - 1, 1);
    multiply(0);
    Mix<MI * NI, MI + NI, XS == WS ? 0 : MI>::order();
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(kAll | (kAhead & 15) | ((kAhead >> 4) << 14));
    bare_barrier();
    __builtin_amdgcn_sched_barrier(0);
    read(xnxt, wnxt, 0, 0);
    if (XS > WS) {
      issue_w(wcur, kt + WS, 0);
    } else {
      issue_x(xcur, kt + XS, 0);
      issue_x(xcur, kt + XS, 1);
    }
    multiply(1);
    Mix<MI * NI, MI + NI, XS == WS ? 2 * MI : NI>::order();
    __builtin_amdgcn_sched_barrier(0);
  };

  // the scales of the wavefront's rows, and this thread's share of the columns': of w0; of w1, or the bias
  float sx[MI];
#pragma unroll
  for (int mi = 0; mi < MI; ++mi) sx[mi] = p.x_scales[min(t0 + (wm * MI + mi) * 32 + r32, p.T - 1)];
  float scale0 = 0.f, scale1 = 0.f;
  if (tid < Tile::kCols && n0 + tid < p.N) {
    scale0 = p.s0[n0 + tid];
    if (GATED)
      scale1 = p.s1[n0 + tid];
    else if (p.bias != nullptr)
      scale1 = bf16_to_f32(p.bias[n0 + tid]);
  }
  uint8_t* const xs[5] = {x0, x1, x2, x3, x4};
  uint8_t* const ws[4] = {w0, w1, w2, w3};
  __builtin_amdgcn_sched_barrier(0);
#pragma unroll
  for (int j = 0; j < XS; ++j) {                             // in the order of the steps before
    if (j < XS - 1 || XS == WS)
#pragma unroll
      for (int h = 0; h < 2; ++h) issue_x(xs[j], first + j, h);
    if (j < WS && (XS > WS || j < WS - 1)) issue_w(ws[j], first + j, 0);
    if (j < WS - 1) issue_w(ws[j], first + j, 1);
  }
  constexpr int kFirst = kAhead + (XS > WS ? NI : 2 * MI);
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(kAll | (kFirst & 15) | ((kFirst >> 4) << 14));
  bare_barrier();
  __builtin_amdgcn_sched_barrier(0);
  read(x0, w0, 0, 0);
  constexpr int kUnroll = XS == WS ? XS : XS * WS;
  int kt = first;
  for (; kt + kUnroll <= KT; kt += kUnroll) {
#pragma unroll
    for (int j = 0; j < kUnroll; ++j)
      step(xs[(j + XS - 1) % XS], xs[j % XS], xs[(j + 1) % XS], ws[(j + WS - 1) % WS], ws[j % WS], ws[(j + 1) % WS], kt + j);
  }
#pragma unroll
  for (int j = 0; j < kUnroll - 1; ++j)
    if (kt + j < KT)
      step(xs[(j + XS - 1) % XS], xs[j % XS], xs[(j + 1) % XS], ws[(j + WS - 1) % WS], ws[j % WS], ws[(j + 1) % WS], kt + j);
  __builtin_amdgcn_s_waitcnt(kAll);
  if constexpr (SPLIT) {
    i32x4* const to = p.partial + (int64_t(L) * 4 + wave) * (MI * NI * 256) + lane;
#pragma unroll
    for (int mi = 0; mi < MI; ++mi)
#pragma unroll
      for (int ni = 0; ni < NI; ++ni)
#pragma unroll
        for (int b = 0; b < 4; ++b)
          to[((mi * NI + ni) * 4 + b) * 64] =
              i32x4{acc[mi][ni][4 * b], acc[mi][ni][4 * b + 1], acc[mi][ni][4 * b + 2], acc[mi][ni][4 * b + 3]};
    return;
  }
  __syncthreads();

  float* const scales = reinterpret_cast<float*>(x0);
  if (tid < Tile::kCols) {
    scales[tid] = scale0;
    scales[Tile::kCols + tid] = scale1;
  }
  __syncthreads();
  uint8_t* const out = (wave < 2 ? w0 : w1) + (wave & 1) * 32 * Tile::kPitch;
#pragma unroll
  for (int mi = 0; mi < MI; ++mi) {
    const int tb = t0 + (wm * MI + mi) * 32;
    if (tb < p.T)
      put_rows<GATED, NI>(p, acc[mi], tb, n0 + wn * Tile::kWaveCols, sx[mi], scales + wn * Tile::kWaveCols,
                          scales + Tile::kCols + wn * Tile::kWaveCols, out, lane);
  }
}

// Adds the parts of tiles that were cut along k: one workgroup for 32 rows of each pair of the tile's wavefronts.
template <bool GATED, int MI, int NI>
__global__ __launch_bounds__(256) void int8_join_kernel(Int8Product p, int mtiles, int ntiles, int parts) {
  using Tile = Int8Tile<GATED, MI, NI>;
  __shared__ __attribute__((aligned(16))) float scales[2][Tile::kCols];
  __shared__ __attribute__((aligned(16))) uint8_t rows[4 * 32 * Tile::kPitch];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int64_t tiles = int64_t(mtiles) * ntiles;
  const int L = int(blockIdx.x / MI);
  const int mi = int(blockIdx.x % MI);
  const TileAt tile = tile_at(L, mtiles, ntiles);
  const int tb = tile.m * Tile::kRows + ((wave >> 1) * MI + mi) * 32, n0 = tile.n * Tile::kCols, wn = wave & 1;
  for (int i = tid; i < Tile::kCols; i += 256) {
    const int n = n0 + i;
    scales[0][i] = n < p.N ? p.s0[n] : 0.f;
    scales[1][i] = n >= p.N ? 0.f : GATED ? p.s1[n] : p.bias != nullptr ? bf16_to_f32(p.bias[n]) : 0.f;
  }
  const float sx = p.x_scales[min(tb + (lane & 31), p.T - 1)];
  i32x16 acc[NI];
#pragma unroll
  for (int ni = 0; ni < NI; ++ni)
#pragma unroll
    for (int q = 0; q < 16; ++q) acc[ni][q] = 0;
  if (tb < p.T) {
    const i32x4* from = p.partial + (int64_t(L) * 4 + wave) * (MI * NI * 256) + mi * NI * 256 + lane;
    for (int part = 0; part < parts; ++part, from += tiles * (4 * MI * NI * 256))
#pragma unroll
      for (int i = 0; i < 4 * NI; ++i) {
        const i32x4 v = from[i * 64];
#pragma unroll
        for (int q = 0; q < 4; ++q) acc[i >> 2][4 * (i & 3) + q] += v[q];
      }
  }
  __syncthreads();
  if (tb < p.T)
    put_rows<GATED, NI>(p, acc, tb, n0 + wn * Tile::kWaveCols, sx, &scales[0][wn * Tile::kWaveCols],
                        &scales[1][wn * Tile::kWaveCols], rows + wave * 32 * Tile::kPitch, lane);
}

template <bool GATED, int MI, int NI, int XS, int WS, bool SPLIT = false, int POLICY = kCached>
void gemm(const Int8Product& p, int parts, hipStream_t s) {
  using Tile = Int8Tile<GATED, MI, NI>;
  const int mtiles = (p.T + Tile::kRows - 1) / Tile::kRows, ntiles = (p.N + Tile::kCols - 1) / Tile::kCols;
  const int tiles = mtiles * ntiles;

  MOE_LAUNCH(GATED ? "gated_int8" : "matmul_int8", (int8_gemm_kernel<GATED, MI, NI, XS, WS, SPLIT, POLICY>), dim3(unsigned((int64_t(tiles) * parts + 7) / 8 * 8)), dim3(256), s, p,
             mtiles, ntiles, parts);
  if constexpr (SPLIT)
    MOE_LAUNCH("int8_join", (int8_join_kernel<GATED, MI, NI>), dim3(unsigned(tiles * MI)), dim3(256), s, p, mtiles, ntiles,
               parts);
}

template <bool GATED>
void product(const Int8Product& p, const Int8Plan& plan, hipStream_t s) {
  const int parts = plan.parts;
  switch (plan.form) {
    case Int8Form::kFew1:
      if constexpr (!GATED) return few<GATED, 1>(p, plan.stream, s);
      [[fallthrough]];
    case Int8Form::kFew2: return few<GATED, 2>(p, plan.stream, s);
    case Int8Form::k64x128:
      if (parts > 1) return gemm<GATED, 1, 2, 3, 3, true>(p, parts, s);
      return plan.stream ? gemm<GATED, 1, 2, 3, 3, false, kStream>(p, 1, s) : gemm<GATED, 1, 2, 3, 3>(p, 1, s);
    case Int8Form::k128x128:
      return parts > 1 ? gemm<GATED, 2, 2, 3, 3, true>(p, parts, s) : gemm<GATED, 2, 2, 3, 3>(p, 1, s);
    case Int8Form::k128x128Two: return gemm<GATED, 2, 2, 2, 2>(p, 1, s);
    case Int8Form::k192x256: return gemm<GATED, 3, 4, 3, 2>(p, 1, s);
    case Int8Form::k256x256: return gemm<GATED, 4, 4, 3, 2>(p, 1, s);
  }
}

}  // namespace

hipError_t launch_pack_int8(const int8_t* codes, int64_t rows, int K, int8_t* out, hipStream_t s) {
  const int steps = (K + 127) / 128 * 2;
  MOE_LAUNCH("pack_int8", pack_int8_kernel, dim3(unsigned((rows + 15) / 16 * steps)), dim3(64), s, codes, rows, K, steps,
             out);
  return hipGetLastError();
}

hipError_t launch_int8_product(const Int8Product& p, const Int8Plan& plan, hipStream_t s) {
  if (p.w1 != nullptr)
    product<true>(p, plan, s);
  else
    product<false>(p, plan, s);
  return hipGetLastError();
}

}  // namespace moe
