// Products of 8-bit integer codes with many rows of x on gfx950: large tiles through LDS.
#include "int8_product.h"

namespace moe {
namespace {

// Tiles of 64 MI rows of x by 64 NI weight rows (GATED: 32 NI of either matrix) for four wavefronts, 2 x 2, of
// 32 MI x 32 NI each.  A stage holds 128 columns of both operands in LDS, the weights in their packed pieces,
// x in rows of 128 bytes whose 16-byte chunks are permuted so that 16 rows of one column lie in different banks;
// global -> LDS loads fill rings of three stages of x and two of weights, all of the LDS at MI = 4.  A stage is four
// groups of 32 columns; a group's operands are read from LDS while the one before it is multiplied, also across the
// border of two stages: the barrier that hands over a stage stands before the last group, whose operands are in
// registers by then.
//
// Bound by the matrix cores, at the clock that the board's power leaves: 16384 rows, 4096 channels, K 14336 712 to 743
// us (2.59 to 2.70 P operations/s; a large library product of this size 2.49), matrix cores 83% busy at 1.62 GHz; gated
// 8192, 14336, 4096 766 to 813 us (2.37 to 2.51 P), 71% at 1.70 GHz: a tile takes 1.55 us a stage and some 4 us at its
// ends.  The largest tile that registers hold moves the fewest bytes through LDS; 192 rows (813 us) fill the last
// round better where that counts.  Measured against (16384, 4096, 14336): two stages of x 760 us; a stage's loads in
// one of its groups, 832; workgroups that stay and load their next tile's first stages while this one's results
// leave, 750 (gated 830, for 785 then): they need registers that the sums take, and spill 20 (as it is, one of the gated
// form's is spilled, before the loop and after it).
__device__ __forceinline__ i32x16 mfma32_i8(u32x4 a, u32x4 b, i32x16 c) {
  return __builtin_amdgcn_mfma_i32_32x32x32_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
}

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
      for (int i = 0; i < 4; ++i)
        v[i] = result<GATED>(acc[GATED ? 2 * nc : nc][4 * b + i], acc[GATED ? 2 * nc + 1 : 0][4 * b + i], sx, s0[i], s1[i],
                             p.bias != nullptr);
      *reinterpret_cast<u32x2*>(out + r32 * kPitch + at * 2) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    }
  wave_order();
  constexpr int kPieces = kCols / 8;                         // of a row
#pragma unroll
  for (int i = lane; i < 32 * kPieces; i += 64) {
    const int r = i / kPieces, piece = i % kPieces;
    if (tb + r < p.T) put_piece(p.y + int64_t(tb + r) * p.N, nb + 8 * piece, p.N, out + r * kPitch + piece * 16);
  }
  wave_order();
}

template <bool GATED, int MI, int NI>
__global__ __launch_bounds__(256, 1) void int8_large_kernel(Int8Product p, int mtiles, int ntiles) {
  using Tile = Int8Tile<GATED, MI, NI>;
  __shared__ __attribute__((aligned(1024))) uint8_t x0[Tile::kXBytes], x1[Tile::kXBytes], x2[Tile::kXBytes];
  __shared__ __attribute__((aligned(1024))) uint8_t w0[Tile::kWBytes], w1[Tile::kWBytes];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave >> 1, wn = wave & 1;
  if (p.steps < 0) x0[tid] = x1[tid] = x2[tid] = w0[tid] = w1[tid] = 0;   // never taken: keeps the reads of what loads fill
  // XCD n % 8 takes a contiguous part of the tiles
  const int total = mtiles * ntiles, per = (total + 7) / 8;
  const int num = int(blockIdx.x), L = (num & 7) * per + (num >> 3);
  if (num >> 3 >= per || L >= total) return;
  const TileAt tile = tile_at(L, mtiles, ntiles);
  const int t0 = tile.m * Tile::kRows, n0 = tile.n * Tile::kCols;

  const int K = p.K, KT = p.steps / 2;
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
      load_lds<kCached>(bx, kt < KT, stage + (wave + 4 * (which * MI + i)) * 1024,
                        on ? int(xat[which * MI + i]) : kPast, kt * 128);
  };
  auto issue_w = [&](uint8_t* stage, int kt, int which) {
#pragma unroll
    for (int j = 0; j < NI; ++j) {
      const int i = which * NI + j, tile16 = wave + 4 * (i >> 1);
      load_lds<kCached>(GATED && tile16 >= 2 * NI ? bw1 : bw0, kt < KT, stage + tile16 * 2048 + (i & 1) * 1024,
                        int(wat[i >> 1]), kt * 2048 + (i & 1) * 1024);
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
  // Stage kt.  Each group issues a quarter of a stage's loads: the second half of the weights of the next stage and
  // the rows of x of the one after it to the places of the stage before, the first half of the weights of the stage
  // after the next to its own.
  constexpr int kAhead = 2 * MI;                             // loads of later stages that may be pending
  auto step = [&](uint8_t* xprev, uint8_t* xcur, uint8_t* xnxt, uint8_t* wcur, uint8_t* wnxt, int kt) {
    read(xcur, wcur, 1, 1);
    issue_w(wnxt, kt + 1, 1);
    multiply(0);
    Mix<MI * NI, MI + NI, NI>::order();
    __builtin_amdgcn_sched_barrier(0);
    read(xcur, wcur, 2, 0);
    issue_x(xprev, kt + 2, 0);
    multiply(1);
    Mix<MI * NI, MI + NI, MI>::order();
    __builtin_amdgcn_sched_barrier(0);
    read(xcur, wcur, 3, 1);
    issue_x(xprev, kt + 2, 1);
    multiply(0);
    Mix<MI * NI, MI + NI, MI>::order();
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(wait_all_but(kAhead));
    bare_barrier();
    __builtin_amdgcn_sched_barrier(0);
    read(xnxt, wnxt, 0, 0);
    issue_w(wcur, kt + 2, 0);
    multiply(1);
    Mix<MI * NI, MI + NI, NI>::order();
    __builtin_amdgcn_sched_barrier(0);
  };

  // the scales of the wavefront's rows, and this thread's share of the columns': of w0; of w1, or the bias
  float sx[MI];
#pragma unroll
  for (int mi = 0; mi < MI; ++mi) sx[mi] = p.x_scales[min(t0 + (wm * MI + mi) * 32 + r32, p.T - 1)];
  float scale0 = 0.f, scale1 = 0.f;
  if (tid < Tile::kCols) channel_scales<GATED>(p, n0 + tid, scale0, scale1);
  __builtin_amdgcn_sched_barrier(0);
  issue_x(x0, 0, 0);                                         // in the order of the steps before
  issue_x(x0, 0, 1);
  issue_w(w0, 0, 0);
  issue_w(w0, 0, 1);
  __builtin_amdgcn_sched_barrier(0);                         // the wait counts on the second stage's being the youngest
  issue_x(x1, 1, 0);
  issue_x(x1, 1, 1);
  issue_w(w1, 1, 0);
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_waitcnt(wait_all_but(kAhead + NI));
  bare_barrier();
  __builtin_amdgcn_sched_barrier(0);
  read(x0, w0, 0, 0);
  uint8_t* const xs[3] = {x0, x1, x2};
  uint8_t* const ws[2] = {w0, w1};
  int kt = 0;
  for (; kt + 6 <= KT; kt += 6) {
#pragma unroll
    for (int j = 0; j < 6; ++j) step(xs[(j + 2) % 3], xs[j % 3], xs[(j + 1) % 3], ws[j % 2], ws[(j + 1) % 2], kt + j);
  }
#pragma unroll
  for (int j = 0; j < 5; ++j)
    if (kt + j < KT) step(xs[(j + 2) % 3], xs[j % 3], xs[(j + 1) % 3], ws[j % 2], ws[(j + 1) % 2], kt + j);
  __builtin_amdgcn_s_waitcnt(wait_all_but(0));
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

template <bool GATED, int MI>
void large(const Int8Product& p, hipStream_t s) {
  using Tile = Int8Tile<GATED, MI, 4>;
  const int mtiles = (p.T + Tile::kRows - 1) / Tile::kRows, ntiles = (p.N + Tile::kCols - 1) / Tile::kCols;
  MOE_LAUNCH(GATED ? "gated_int8_large" : "matmul_int8_large", (int8_large_kernel<GATED, MI, 4>),
             dim3(unsigned((int64_t(mtiles) * ntiles + 7) / 8 * 8)), dim3(256), s, p, mtiles, ntiles);
}

}  // namespace

void launch_int8_large(const Int8Product& p, bool rows256, hipStream_t s) {
  if (p.w1 != nullptr)
    rows256 ? large<true, 4>(p, s) : large<true, 3>(p, s);
  else
    rows256 ? large<false, 4>(p, s) : large<false, 3>(p, s);
}

}  // namespace moe
