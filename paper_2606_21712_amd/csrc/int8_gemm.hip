// Products of 8-bit integer codes on gfx950: packing the weights, and
//   y[t, n] = s_x[t] s_w[n] sum_k q_x[t, k] q_w[n, k] (+ b[n]),
// plain, or the two products of a gated block with silu(g) u on top.
//
// The sums are exact in 32 bits (K <= kInt8MaxK), whatever their order, so how a product is cut up
// does not show in its result.
#include <type_traits>

#include "int8_product.h"
#include "launch_rules.h"

namespace moe {
namespace {

__device__ __forceinline__ i32x4 mfma_i8(u32x4 a, u32x4 b, i32x4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

// ------------------------------------------------------------------ pack
// One wavefront a step of 16 rows x 64 columns: 16 pieces of 64 bytes in, one of 1 KB out.  Bound by memory, once
// for each matrix.
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
// A wavefront multiplies NT tiles of 16 weight rows (GATED: one of either matrix) with C groups of 16 rows of x: the
// weights are the first operand, streamed from memory into registers, x the second, from the caches.  KS wavefronts deal
// the steps of 128 columns along k among themselves (both halves of a line of x to one of them) and add their sums in
// LDS; P steps are in flight.  More rows are other workgroups', which find the weights in the L2.
//
// Bound by the reads of the weights, after a launch and its ramp: one row, 4096 channels, K 14336 (59 MB) 10.0 us, 5.9
// TB/s; eight rows gated, 2048, 7168 (29 MB) 7.5; five rows, 6309, 16400 past the caches (103 MB) 20.2, 5.1 TB/s.  Two
// tiles a wavefront halve the reads of x, eight wavefronts and two steps keep 32 KB of a tile in flight (four steps: 16
// rows, 4096, 14336 14.4 us for 13.6).  Two groups read the weights once for both: 32 rows, 6144, 4096 8.0 us, 10.1 in
// two workgroups; four were faster nowhere (64 rows 11.9 us, 10.0 on the tiles below).
template <bool GATED, int NT, int C, int KS, int P, int POLICY>
__global__ __launch_bounds__(64 * KS) void few_int8_kernel(Int8Product p) {
  __shared__ i32x4 part[KS][NT][C][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int t0 = int(blockIdx.y) * 16 * C;
  constexpr int kTiles = GATED ? NT / 2 : NT;     // of a matrix
  static_assert(kTiles * C <= KS, "a wavefront finishes a tile");
  const int pairs = p.steps / 2;
  const int mine = (pairs - wave + KS - 1) / KS;
  const int tiles = (p.N + 15) / 16, rt = int(blockIdx.x) * kTiles;
  if (rt >= tiles) return;
  const int64_t tile_bytes = int64_t(p.steps) * 1024;
  Buffer bw[NT];
#pragma unroll
  for (int r = 0; r < NT; ++r) {
    const int tile = rt + r % kTiles;
    bw[r] = buffer_of((GATED && r >= kTiles ? p.w1 : p.w0) + tile * tile_bytes, tile < tiles ? tile_bytes : 0);
  }
  const auto bx = buffer_of(p.x + int64_t(t0) * p.K, int64_t(min(p.T - t0, 16 * C)) * p.K);
  const int chunk = 16 * (lane >> 4);
  int xat[C];                                     // past the last row: zeros
#pragma unroll
  for (int c = 0; c < C; ++c) xat[c] = (16 * c + (lane & 15)) * p.K + chunk;
  // what the wavefronts that finish a tile need besides: loaded first, not once the sums are there
  const int fr = wave % kTiles, fc = wave / kTiles;
  const int t = t0 + 16 * fc + (lane & 15), n = (rt + fr) * 16 + 4 * (lane >> 4);
  const bool finish = wave < kTiles * C && t < p.T && n < p.N;
  float sx = 0.f, s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
  if (finish) {
    sx = p.x_scales[t];
#pragma unroll
    for (int i = 0; i < 4; ++i) channel_scales<GATED>(p, n + i, s0[i], s1[i]);
  }
  i32x4 acc[NT][C];
#pragma unroll
  for (int r = 0; r < NT; ++r)
#pragma unroll
    for (int c = 0; c < C; ++c) acc[r][c] = i32x4{0, 0, 0, 0};
  u32x4 w[P][NT][2], x[P][C][2];
  auto load = [&](int q, int i) {
    const int at = wave + i * KS;
#pragma unroll
    for (int r = 0; r < NT; ++r)
#pragma unroll
      for (int h = 0; h < 2; ++h) w[q][r][h] = load16<POLICY>(bw[r], i < mine, 16 * lane, at * 2048 + h * 1024);
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int h = 0; h < 2; ++h)                 // columns past K: zeros, whatever the offset's range check counts
        x[q][c][h] = load16<kCached>(bx, i < mine, at * 128 + h * 64 + chunk < p.K ? xat[c] : kPast, at * 128 + h * 64);
  };
#pragma unroll
  for (int q = 0; q < P; ++q) load(q, q);
  for (int i = 0; i < mine; i += P) {
#pragma unroll
    for (int q = 0; q < P; ++q) {
#pragma unroll
      for (int r = 0; r < NT; ++r)
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
          for (int h = 0; h < 2; ++h) acc[r][c] = mfma_i8(w[q][r][h], x[q][c][h], acc[r][c]);
      load(q, i + q + P);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
#pragma unroll
  for (int r = 0; r < NT; ++r)
#pragma unroll
    for (int c = 0; c < C; ++c) part[wave][r][c][lane] = acc[r][c];
  __syncthreads();
  if (!finish) return;
  i32x4 s = part[0][fr][fc][lane], u = {0, 0, 0, 0};
#pragma unroll
  for (int i = 1; i < KS; ++i) s += part[i][fr][fc][lane];
  if (GATED) {
#pragma unroll
    for (int i = 0; i < KS; ++i) u += part[i][kTiles + fr][fc][lane];
  }
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = result<GATED>(s[i], u[i], sx, s0[i], s1[i], p.bias != nullptr);
  store4(p.y + int64_t(t) * p.N, n, p.N, v);
}

template <bool GATED, int NT, int C = 1>
void few(const Int8Product& p, bool stream, hipStream_t s) {
  const int tiles = (p.N + 15) / 16, each = GATED ? NT / 2 : NT;
  const char* name = GATED ? "gated_int8_few" : "matmul_int8_few";
  // all groups of rows of a tile of weights on one XCD, whose L2 has it: number n of a launch runs on XCD n % 8
  const dim3 grid(((tiles + each - 1) / each + 7) / 8 * 8, (p.T + 16 * C - 1) / (16 * C)), block(512);
  if (stream)
    MOE_LAUNCH(name, (few_int8_kernel<GATED, NT, C, 8, 2, kStream>), grid, block, s, p);
  else
    MOE_LAUNCH(name, (few_int8_kernel<GATED, NT, C, 8, 2, kCached>), grid, block, s, p);
}

// ------------------------------------------------------------------ more rows: weights past LDS
// Tiles of 16 A rows of x by 64 B weight rows (GATED: 32 B of either matrix), 16 B for each of four wavefronts: no
// two read the same weights, which go from memory straight to registers, in the packed pieces that are the
// products' operands as they lie.  x, which all four read, passes through LDS, in a ring of XS stages of 128 columns
// of the large tiles.  A step is 64 columns; a ring of 2 XS steps of weights is in flight.
//
// Bound by what passes into a compute unit, 64 bytes a clock: 333 rows, 6145 channels, K 4096 15.4 us on 96 x 128 (196
// tiles; 28 KB a stage are 0.20 us of its 0.26; matrix cores 41% busy; 17.5 with the weights through LDS too); gated
// 700, 1408, 2816 9.5 us on 64 x 128.  At 160 x 256 the matrix cores share it: 2003, 4608, 7168 61 us, 2.17 P
// operations/s, 57% busy (70 on 192 x 256 through LDS).  Longer rings and unrolled loops lost at short K to the fetch of
// instructions; k starts of each tile's own, so that rows of x a power of two apart do not meet, gained nothing.
template <int A, int B, int XS>
struct Direct {
  static constexpr int kRows = 16 * A, kWRows = 64 * B;
  static constexpr int kSlots = 2 * XS;                      // of weights
  static constexpr int kXLoads = A / 2;                      // a wavefront's share of a stage of x
};

// The results of 16 rows from tb on, B x 16 sums a wavefront: a lane holds channels 4 (lane / 16) + 0..3 of row lane % 16
// of each 16 x 16.  They go through LDS of the wavefront's own, to leave as pieces of rows.
template <bool GATED, int B>
__device__ __forceinline__ void put_strip(const Int8Product& p, const i32x4 (&acc)[B], int tb, int nb, float sx,
                                          const float (&s0)[GATED ? B / 2 : B][4], const float (&s1)[GATED ? B / 2 : B][4],
                                          uint8_t* out, int lane) {
  constexpr int kFrags = GATED ? B / 2 : B, kPitch = 32 * kFrags + 16;
#pragma unroll
  for (int f = 0; f < kFrags; ++f) {
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      v[i] = result<GATED>(acc[GATED ? 2 * f : f][i], acc[GATED ? 2 * f + 1 : 0][i], sx, s0[f][i], s1[f][i], p.bias != nullptr);
    *reinterpret_cast<u32x2*>(out + (lane & 15) * kPitch + f * 32 + (lane >> 4) * 8) =
        u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
  }
  wave_order();
  constexpr int kPieces = 2 * kFrags;                        // of a row
#pragma unroll
  for (int i = lane; i < 16 * kPieces; i += 64) {
    const int r = i / kPieces, piece = i % kPieces;
    if (tb + r < p.T) put_piece(p.y + int64_t(tb + r) * p.N, nb + 8 * piece, p.N, out + r * kPitch + piece * 16);
  }
  wave_order();
}

template <bool GATED, int A, int B, int XS, bool SPLIT, int POLICY>
__global__ __launch_bounds__(256, A * B <= 16 ? 2 : 1) void int8_direct_kernel(Int8Product p, int mtiles, int ntiles, int parts) {
  using Tile = Direct<A, B, XS>;
  constexpr int kXBytes = Tile::kRows * 128, kSlots = Tile::kSlots;
  constexpr int kFrags = GATED ? B / 2 : B, kPitch = 32 * kFrags + 16;
  __shared__ __attribute__((aligned(1024))) uint8_t x0[kXBytes], x1[kXBytes], x2[kXBytes],
      x3[XS > 3 ? kXBytes : 16];
  __shared__ __attribute__((aligned(16))) uint8_t s_out[4][16 * kPitch];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (p.steps < 0) {              // never taken: keeps the reads of what global -> LDS loads fill
    x0[tid] = x1[tid] = x2[tid] = 0;
    x3[tid & 15] = 0;
  }
  const int tiles = mtiles * ntiles, total = tiles * parts, per = (total + 7) / 8;
  const int num = int(blockIdx.x), L = (num & 7) * per + (num >> 3);
  if (num >> 3 >= per || L >= total) return;
  const int part = SPLIT ? L / tiles : 0;
  const TileAt tile = tile_at(L - part * tiles, mtiles, ntiles);
  constexpr int kCols = GATED ? 32 * B : 64 * B;             // of y
  const int t0 = tile.m * Tile::kRows, nb = tile.n * kCols + wave * (kCols / 4);
  const int K = p.K, stages = p.steps / 2;
  const int first = SPLIT ? part * stages / parts : 0, KT = SPLIT ? (part + 1) * stages / parts : stages;
  const int rows = min(Tile::kRows, p.T - t0);
  const int64_t tile_bytes = int64_t(p.steps) * 1024;
  const int n16 = nb / 16, wtiles = max(0, min(kFrags, (p.N + 15) / 16 - n16));   // of either matrix
  const Buffer bx = buffer_of(p.x + int64_t(t0) * K, int64_t(rows) * K);
  const Buffer bw0 = buffer_of(p.w0 + n16 * tile_bytes, wtiles * tile_bytes);
  const Buffer bw1 = buffer_of((GATED ? p.w1 : p.w0) + n16 * tile_bytes, wtiles * tile_bytes);

  float sx[A], s0[kFrags][4], s1[kFrags][4];
  if (!SPLIT) {
#pragma unroll
    for (int a = 0; a < A; ++a) sx[a] = p.x_scales[min(t0 + 16 * a + (lane & 15), p.T - 1)];
#pragma unroll
    for (int f = 0; f < kFrags; ++f)
#pragma unroll
      for (int i = 0; i < 4; ++i) channel_scales<GATED>(p, nb + 16 * f + 4 * (lane >> 4) + i, s0[f][i], s1[f][i]);
  }
  __builtin_amdgcn_sched_barrier(0);

  const int chunk = (lane & 7) ^ ((4 * wave + (lane >> 4)) & 7);
  uint32_t xat[Tile::kXLoads], wat[kFrags];
#pragma unroll
  for (int i = 0; i < Tile::kXLoads; ++i) xat[i] = uint32_t(8 * (wave + 4 * i) + (lane >> 3)) * uint32_t(K) + 16 * chunk;
#pragma unroll
  for (int f = 0; f < kFrags; ++f) wat[f] = uint32_t(f * tile_bytes) + 16 * lane;
  auto issue_x = [&](uint8_t* stage, int kt) {
    const bool on = kt * 128 + 16 * chunk < K;                // columns past K: zeros
#pragma unroll
    for (int i = 0; i < Tile::kXLoads; ++i)
      load_lds<kCached>(bx, kt < KT, stage + (wave + 4 * i) * 1024, on ? int(xat[i]) : kPast, kt * 128);
  };
  u32x4 w[kSlots][B];
  auto issue_w = [&](u32x4(&to)[B], int q) {                 // step q
#pragma unroll
    for (int b = 0; b < B; ++b)
      to[b] = load16<POLICY>(GATED && (b & 1) ? bw1 : bw0, q < 2 * KT, int(wat[GATED ? b >> 1 : b]), q * 1024);
  };
  const int r16 = lane & 15, xrow = r16 * 128, xswz = (r16 >> 1) & 7, quarter = lane >> 4;
  i32x4 acc[A][B];
#pragma unroll
  for (int a = 0; a < A; ++a)
#pragma unroll
    for (int b = 0; b < B; ++b) acc[a][b] = i32x4{0, 0, 0, 0};
  u32x4 xf[2][A];
  auto read = [&](const uint8_t* stage, int s, u32x4(&to)[A], int from = 0, int end = A) {
#pragma unroll
    for (int a = from; a < end; ++a)
      to[a] = *reinterpret_cast<const u32x4*>(stage + xrow + a * 2048 + ((4 * s + quarter) ^ xswz) * 16);
  };
  auto multiply = [&](const u32x4(&wf)[B], const u32x4(&x)[A], int from = 0, int end = A) {
#pragma unroll
    for (int a = from; a < end; ++a)
#pragma unroll
      for (int b = 0; b < B; ++b) acc[a][b] = mfma_i8(wf[b], x[a], acc[a][b]);
  };
  // The waits leave as many loads in flight as were sent after the next stage's x, so scheduling barriers part x from the
  // weights around it.
  constexpr int kGroup = 2 * B + Tile::kXLoads;               // loads of a step
  constexpr int kAhead = (XS - 2) * kGroup + 2 * B;
  constexpr int kFirst = (XS - 1) * kGroup + B;
  constexpr int kSplit = (A * Tile::kXLoads + B) / (B + Tile::kXLoads);      // rows of 16 that are multiplied while x is sent for
  // stage kt, whose steps are the slots 2 j and 2 j + 1
  auto step = [&](uint8_t* xcur, uint8_t* xnxt, u32x4(&wprev)[B], u32x4(&w0)[B], u32x4(&w1)[B], int kt) {
    read(xcur, 1, xf[1]);
    issue_w(wprev, 2 * kt - 1 + kSlots);
    multiply(w0, xf[0]);
    Mix<A * B, A, B>::order();
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(wait_all_but(kAhead));
    bare_barrier();
    __builtin_amdgcn_sched_barrier(0);
    read(xnxt, 0, xf[0], 0, kSplit);
    issue_x(xcur, kt + XS);
    multiply(w1, xf[1], 0, kSplit);
    Mix<kSplit * B, kSplit, Tile::kXLoads>::order();
    __builtin_amdgcn_sched_barrier(0);
    read(xnxt, 0, xf[0], kSplit, A);
    issue_w(w0, 2 * kt + kSlots);
    multiply(w1, xf[1], kSplit, A);
    Mix<(A - kSplit) * B, A - kSplit, B>::order();
    __builtin_amdgcn_sched_barrier(0);
  };
  // The last steps, fewer than a ring: what they would load lies past the end.  They do not count on loads of weights
  // that no step reads, which the compiler leaves out.
  auto last_step = [&](auto which, uint8_t* xcur, uint8_t* xnxt, u32x4(&w0)[B], u32x4(&w1)[B]) {
    constexpr int j = decltype(which)::value;
    read(xcur, 1, xf[1]);
    multiply(w0, xf[0]);
    Mix<A * B, A, 0>::order();
    __builtin_amdgcn_sched_barrier(0);
    if constexpr (j < XS - 2) {
      __builtin_amdgcn_s_waitcnt(wait_all_but((XS - 2 - j) * kGroup));
      bare_barrier();
      __builtin_amdgcn_sched_barrier(0);
      read(xnxt, 0, xf[0]);
    }
    multiply(w1, xf[1]);
    Mix<A * B, j < XS - 2 ? A : 0, 0>::order();
    __builtin_amdgcn_sched_barrier(0);
  };
  uint8_t* const xs[4] = {x0, x1, x2, x3};
#pragma unroll
  for (int j = 0; j < XS; ++j) {
    issue_x(xs[j], first + j);
    __builtin_amdgcn_sched_barrier(0);
    issue_w(w[2 * j], 2 * (first + j));
    if (j < XS - 1) issue_w(w[2 * j + 1], 2 * (first + j) + 1);
    __builtin_amdgcn_sched_barrier(0);
  }
  __builtin_amdgcn_s_waitcnt(wait_all_but(kFirst));
  bare_barrier();
  __builtin_amdgcn_sched_barrier(0);
  read(x0, 0, xf[0]);
  int kt = first;
  for (; kt + XS <= KT; kt += XS) {
#pragma unroll
    for (int j = 0; j < XS; ++j)
      step(xs[j], xs[(j + 1) % XS], w[(2 * j + kSlots - 1) % kSlots], w[2 * j], w[2 * j + 1], kt + j);
  }
  static_assert(XS == 3 || XS == 4, "last steps");
  if (kt < KT) last_step(std::integral_constant<int, 0>{}, x0, x1, w[0], w[1]);
  if (kt + 1 < KT) last_step(std::integral_constant<int, 1>{}, x1, x2, w[2], w[3]);
  if constexpr (XS > 3)
    if (kt + 2 < KT) last_step(std::integral_constant<int, 2>{}, x2, x3, w[4], w[5]);

  __builtin_amdgcn_s_waitcnt(wait_all_but(0));                // for the zeros that are on their way to LDS
  if constexpr (SPLIT) {
    i32x4* const to = p.partial + (int64_t(L) * 4 + wave) * (A * B * 64) + lane;
#pragma unroll
    for (int a = 0; a < A; ++a)
#pragma unroll
      for (int b = 0; b < B; ++b) to[(a * B + b) * 64] = acc[a][b];
    return;
  }
#pragma unroll
  for (int a = 0; a < A; ++a)
    if (t0 + 16 * a < p.T) put_strip<GATED, B>(p, acc[a], t0 + 16 * a, nb, sx[a], s0, s1, s_out[wave], lane);
}

// Adds the parts of tiles that were cut along k: one workgroup for 16 rows of a tile.  64 rows, 4096 channels, K 14336
// in eight parts: 5.0 us after the products' 11.8 (9 MB, mostly from the L2), the latency of one load and one store.
template <bool GATED, int A, int B>
__global__ __launch_bounds__(256) void int8_join_kernel(Int8Product p, int mtiles, int ntiles, int parts) {
  constexpr int kFrags = GATED ? B / 2 : B, kPitch = 32 * kFrags + 16;
  __shared__ __attribute__((aligned(16))) uint8_t s_out[4][16 * kPitch];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int L = int(blockIdx.x / A), a = int(blockIdx.x % A);
  const TileAt tile = tile_at(L, mtiles, ntiles);
  constexpr int kCols = GATED ? 32 * B : 64 * B;
  const int tb = tile.m * 16 * A + 16 * a, nb = tile.n * kCols + wave * (kCols / 4);
  if (tb >= p.T) return;
  const float sx = p.x_scales[min(tb + (lane & 15), p.T - 1)];
  float s0[kFrags][4], s1[kFrags][4];
#pragma unroll
  for (int f = 0; f < kFrags; ++f)
#pragma unroll
    for (int i = 0; i < 4; ++i) channel_scales<GATED>(p, nb + 16 * f + 4 * (lane >> 4) + i, s0[f][i], s1[f][i]);
  i32x4 acc[B];
#pragma unroll
  for (int b = 0; b < B; ++b) acc[b] = i32x4{0, 0, 0, 0};
  const i32x4* from = p.partial + (int64_t(L) * 4 + wave) * (A * B * 64) + a * B * 64 + lane;
  for (int part = 0; part < parts; ++part, from += int64_t(mtiles) * ntiles * (4 * A * B * 64))
#pragma unroll
    for (int b = 0; b < B; ++b) acc[b] += from[b * 64];
  put_strip<GATED, B>(p, acc, tb, nb, sx, s0, s1, s_out[wave], lane);
}

template <bool GATED, int A, int B, int XS, bool SPLIT = false, int POLICY = kCached>
void direct(const Int8Product& p, int parts, hipStream_t s) {
  constexpr int kCols = GATED ? 32 * B : 64 * B;
  const int mtiles = (p.T + 16 * A - 1) / (16 * A), ntiles = (p.N + kCols - 1) / kCols, tiles = mtiles * ntiles;
  MOE_LAUNCH(GATED ? "gated_int8" : "matmul_int8", (int8_direct_kernel<GATED, A, B, XS, SPLIT, POLICY>),
             dim3(unsigned((int64_t(tiles) * parts + 7) / 8 * 8)), dim3(256), s, p, mtiles, ntiles, parts);
  if constexpr (SPLIT)
    MOE_LAUNCH("int8_join", (int8_join_kernel<GATED, A, B>), dim3(unsigned(tiles * A)), dim3(256), s, p, mtiles, ntiles,
               parts);
}

// Whole tiles, or parts along k.
template <bool GATED, int A, int XS>
void tiles(const Int8Product& p, const Int8Plan& plan, hipStream_t s) {
  if (plan.parts > 1)
    direct<GATED, A, 2, XS, true>(p, plan.parts, s);
  else if (plan.stream)
    direct<GATED, A, 2, XS, false, kStream>(p, 1, s);
  else
    direct<GATED, A, 2, XS>(p, 1, s);
}

template <bool GATED>
void product(const Int8Product& p, const Int8Plan& plan, hipStream_t s) {
  switch (plan.form) {
    case Int8Form::kFew1:
      if constexpr (!GATED) return few<GATED, 1>(p, plan.stream, s);
      [[fallthrough]];
    case Int8Form::kFew2: return few<GATED, 2>(p, plan.stream, s);
    case Int8Form::kFew2x32: return few<GATED, 2, 2>(p, plan.stream, s);
    case Int8Form::k32x128: return tiles<GATED, 2, 4>(p, plan, s);
    case Int8Form::k64x128: return tiles<GATED, 4, 3>(p, plan, s);
    case Int8Form::k96x128: return tiles<GATED, 6, 3>(p, plan, s);
    case Int8Form::k128x128: return tiles<GATED, 8, 3>(p, plan, s);
    case Int8Form::k160x256: return direct<GATED, 10, 4, 3>(p, 1, s);
    case Int8Form::k192x256: return launch_int8_large(p, false, s);
    case Int8Form::k256x256: return launch_int8_large(p, true, s);
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
