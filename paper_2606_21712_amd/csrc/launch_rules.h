// How the launches are sized: which form of a kernel a call takes.  Plain C++, no HIP
// dependency, so that the rules can be evaluated on a host.
#pragma once
#include <cmath>
#include <cstdint>

#include "tiling.h"

namespace moe {

// Grid of the kernels with one workgroup per tile: at least `tiles` workgroups, numbered
// y * kTileGridX + x, in eight parts (number n runs on XCD n % 8).  Two dimensions once one
// would pass the launch's limit of 2^32 threads along it (workgroups have at most 512): fp32
// gate/up tiles of a workspace of 137 GB are 2^24.
struct TileGrid {
  unsigned x, y;
};
constexpr unsigned kTileGridX = 1u << 22;
inline TileGrid tile_grid(int64_t tiles) {
  const int64_t n = (tiles + 7) / 8 * 8;
  if (n <= kTileGridX) return TileGrid{unsigned(n), 1};
  return TileGrid{kTileGridX, unsigned((n + kTileGridX - 1) / kTileGridX)};
}

// One-block permute (up to 16384 assignments): groups of 64 that each of its 16 wavefronts
// takes, a constant of the kernel: the next built size up.  Sizes 6 and 12 because a third
// of the groups empty shows: 8200 assignments over 256 experts take 21.1 us in 16 groups,
// 17.4 in 12, and 5000 13.0 in 8, 11.9 in 6.
inline int permute_small_iters(int64_t R) {
  for (int n : {1, 2, 4, 6, 8, 12})
    if (R <= int64_t(n) * 1024) return n;
  return 16;
}

// Sixteen-byte vectors of each row that a lane of combine loads at once: 32 loads in flight
// with k rows (k = 1, 2: 8 or 16).
constexpr int combine_unroll(int k) { return k == 1 || k == 2 || k == 4 ? 8 : 2; }

// Column split of combine: a token's row (nvec vectors) is cut into this many parts, one
// wavefront each, every one with a vector per lane at least.
//   Large batches run enough wavefronts with a few vectors per lane each (measured cold, %
//   of 8 TB/s: memory-constrained 71 -> 76 with 2 parts, Mixtral-shaped 32K tokens 75 -> 77
//   with 4, DeepSeek-shaped 65 -> 70 with 8).
//   Small ones are bound by the latency of a row.  Where a whole row is several passes of a
//   lane (loads, sums, store), up to 4096 wavefronts run them side by side (96 tokens, k 8,
//   H 7168: 16.9 -> 7.7 us cold; 2048: 53.4 -> 51.8).  Where it is one pass only the loads
//   per lane shrink, and that pays while the wavefronts stay under three per SIMD (509
//   tokens, H 4096, k 4: 9.8 us, 8.6 in 4 parts, 9.8 in 8); from 640 tokens whole rows are
//   the fastest or level (1024, H 4096, k 4: 12.0 us, 13.7 in 4; 2048, k 2: 9.4, in 2 11.7).
//   Batches between keep whole rows.
inline int combine_splits(int64_t T, int k, int nvec) {
  constexpr int kWave = 64;
  const bool one_pass = nvec <= kWave * combine_unroll(k);
  const int64_t small = !one_pass ? 4096 : T < 640 ? 2800 : 0;
  int splits = 1;
  if (T < 4096)
    while (splits < 16 && nvec / (2 * splits) >= kWave && T * (2 * splits) <= small) splits *= 2;
  else if (T >= 8192)
    while (splits < 8 && nvec / (2 * splits) >= kWave && T * splits < (int64_t(1) << 30) &&
           (nvec / splits > 4 * kWave || T * splits < 131072))
      splits *= 2;
  return splits;
}

// ---- the grouped GEMMs for small groups (ffn_stream.hip)

// Experts that R rows dealt evenly at random reach, and their average rows.
struct GroupLoad {
  double live;
  int64_t rows;
  GroupLoad(int64_t R, int E)
      : live(E > 1 ? E * -std::expm1(double(R) * std::log1p(-1.0 / E)) : 1.0), rows(int64_t(double(R) / live + 0.999)) {}
};

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Whether one GEMM of the grouped FFN (K wide, N outputs per row) is faster on the streaming
// kernels than on the large-batch ones, without a compute-unit budget.  Only the mean group is
// known here; loads differ, so each line lies where even loads and lognormal ones (sigma
// 0.5 and 1) are faster on average.  Time streaming / large-batch, each shape even, then the
// slower of the uneven (H / F / experts):
//   Few tiles leave the large-batch kernels' grid part empty, and there streaming wins far out.
//     MXFP8, tiles of 256 rows, fewer tiles than compute units: down 4096 / 4096 / 10 at 112
//       rows 0.85, 0.79, at 256 0.68, 0.71; 4096 / 14336 / 4 at 640 rows 0.72, 0.71.  A just full
//       grid: only up to 320 rows, where uneven loads spill into a second round (4096 / 14336 / 8
//       at 300 rows 1.14, 0.69; at 330 1.15, 1.13).
//     bf16, tiles of 320 rows, at most half as many tiles, as long as streaming's own tiles run
//       at once, one workgroup per compute unit: 4096 / 14336 / 8 down at 220 rows 0.77, 0.82,
//       256 0.73, 1.33, 300 1.20, 1.25; 4096 / 14336 / 4 down at 500 rows 0.70, 1.19.
//   Gate/up, bf16: 112 rows (7168 / 2048 / 64 0.87, 0.97; 4096 / 4096 / 64 0.87, 1.04); 144 while
//     the large-batch grid has less than four rounds, whose last is part empty (at 128 rows
//     4096 / 14336 / 8 0.78, 1.06; 5120 / 1536 / 32 0.83, 1.00; 2816 / 1408 / 60 0.88, 1.01);
//     beyond, it loses: 7168 / 2048 / 64 at 160 rows 1.15, 1.04.
//   Gate/up, MXFP8: 96 rows (7168 / 2048 / 64 0.85, 0.89; 4096 / 14336 / 8 0.91, 1.00; at 128 rows
//     1.09, 0.97 and 1.02, 1.09).
//   Down: as gate/up, except where the large-batch kernel is near its best rate:
//     more than four rounds of its tiles: 88 rows (7168 / 2048 / 64 at 80 rows 0.97, 1.06, MXFP8
//       0.96, 1.04, at 104 1.00, 1.07, MXFP8 at 96 0.98, 1.05), more than sixteen 32 (7168 / 2048 / 256 at 40 rows 1.00, 1.13);
//     short k loops, whose start and end a tile of few steps does not hide, once there are two
//       rounds: under 16 steps 40 rows, MXFP8 72 (2048 / 768 / 128 bf16 at 40 rows 0.96, 1.06, at
//       52 1.02, 1.10; MXFP8 2816 / 1408 / 60 at 64 rows 0.96, 0.97, at 96 1.01, 1.12), under 8
//       steps 24 (2048 / 768 / 128 MXFP8 at 24 rows 0.97, 1.04, at 52 1.11, 1.19).
inline bool stream_is_faster(int64_t R, int E, int K, int N, bool swiglu, bool fp8, int num_cu) {
  const GroupLoad l(R, E);
  const int64_t ntiles = ceil_div(N, swiglu ? kTileCols / 2 : kTileCols);
  const int64_t big = int64_t(l.live * double(ceil_div(l.rows, fp8 ? kTileRows : kTileRowsMax) * ntiles));
  const int steps = K * (fp8 ? 1 : 2) / 128;
  if (fp8) {
    if (big < num_cu || (big == num_cu && l.rows <= 320)) return true;
  } else if (2 * big <= num_cu) {
    // streaming tiles of 160 rows (from 321 rows 128); uneven groups have 0.4 more each than their mean says
    const int mr = l.rows <= 320 ? 160 : 128;
    const double mtiles = E == 1 ? double(ceil_div(l.rows, mr)) : double(l.rows) / mr + 0.4;
    if (l.live * mtiles * double(ntiles) <= num_cu) return true;
  }
  if (!swiglu) {
    if (big > 16 * num_cu) return l.rows <= 32;
    if (big > 4 * num_cu && l.rows > 88) return false;
    if (steps < 8 && big >= 2 * num_cu) return l.rows <= 24;
    if (steps < 16 && big >= 2 * num_cu) return l.rows <= (fp8 ? 72 : 40);
  }
  return l.rows <= (fp8 ? 96 : big < 4 * num_cu ? 144 : 112);
}

// The streaming kernels' tiles: 64 wn weight rows x mr activation rows, kg k groups, stages of the ring.
struct StreamTile {
  int wn, mr, kg, stages;
};

// Which tile.  More activation rows per tile read the weights fewer times and the
// activations less often, fewer give more workgroups; the lines lie where the mean group
// leaves its largest members inside one tile (a group cut in two reads its weights from L2
// twice).  Measured, us of one GEMM (M: H 4096, F 14336, 8 experts):
//   160 rows for means of 100 to 320: M down at 256 rows 289 (128 rows: 430); beyond that
//     128 rows (one expert, 2048 rows, H 7168, F 2048, gate/up: 114, 160 rows: 191);
//   fewer workgroups than two per compute unit: two k groups, which keep as many bytes in
//     flight on half the workgroups (M down at one row: 80 -> 52), and four on 64 weight
//     rows when even that leaves half the chip idle (one expert, F 2048, H 7168 at 8 rows,
//     gate/up: 31 -> 21).
inline StreamTile stream_tile(int64_t R, int E, int N, bool swiglu, bool fp8, int num_cu) {
  const GroupLoad l(R, E);
  auto workgroups = [&](int wn, int mr) {
    return int64_t(l.live * double(ceil_div(l.rows, mr)) * double(ceil_div(N, 64 * wn / (swiglu ? 2 : 1))));
  };
  if (!fp8 && l.rows > 100 && l.rows <= 320) {       // (three MXFP8 stages of 160 rows and their scales exceed the LDS)
    if (workgroups(4, 160) >= num_cu) return {4, 160, 1, 3};
    if (workgroups(2, 160) >= num_cu * 3 / 4) return {2, 160, 1, 4};
  }
  if (l.rows > 44) {
    if (workgroups(4, 128) >= num_cu) return {4, 128, 1, 3};
    if (workgroups(2, 128) >= num_cu * 3 / 4) return {2, 128, 1, 4};
  }
  const int mr = l.rows <= 16 ? 32 : 64;
  if (workgroups(2, mr) >= 2 * num_cu) return {2, mr, 1, 3};
  if (workgroups(2, mr) >= num_cu / 2) return {2, mr, 2, 3};
  return l.rows <= 16 ? StreamTile{1, 32, 4, 3} : StreamTile{1, 64, 2, 4};
}

// Whether a tile's weights bypass the caches (the nt policy): nothing reads them again soon when
// one m-tile holds the mean group.  Not for small weights, which the Infinity Cache may hold
// from one call to the next.  (Deciding per expert by its own m-tiles was slower: uneven
// loads gained 1 to 3% on average, but MXFP8 lost up to 10% in gate/up of H 7168, F 2048, 64
// experts at 80 to 120 rows, and 20% in down of H 4096, F 14336, 4 experts at 112 to 128.)
inline bool stream_nt(int64_t R, int E, int K, int N, bool swiglu, bool fp8, int mr) {
  const int64_t weight_bytes = int64_t(E) * N * K * (fp8 ? 1 : 2) * (swiglu ? 2 : 1);
  return weight_bytes >= (int64_t(128) << 20) && GroupLoad(R, E).rows <= mr;
}

// ---- rows that a workgroup keeps in registers (norm.hip)

// Threads of a workgroup, and vectors of 8 elements that each keeps of a row of n elements (n % 8 == 0, at
// most 131072).  A row for each compute unit or less: as many threads as vectors, its latency is all
// there is (one row of 4096: 3.2 us on 512 threads, 3.5 on 256).  More rows: two vectors a thread, which
// leaves registers for the row ahead (2003 x 7168: 24.6 us on 512 threads, 26.5 with four vectors on 256), and
// whole rows to a wavefront, without a barrier, while four vectors do it (16384 x 1024: 26.8 us, 33.7 on 256).
struct RowShape {
  int threads, vectors;
};
inline RowShape row_shape(int n, int64_t rows, int num_cu) {
  const int nvec = (n + 7) / 8;
  if (rows <= num_cu)
    for (int t : {64, 256, 512, 1024})
      if (nvec <= t) return {t, 1};
  for (int v : {1, 2, 4})
    if (nvec <= 64 * v) return {64, v};
  for (int t : {256, 512, 1024})
    if (nvec <= 2 * t) return {t, 2};
  return {1024, nvec <= 4096 ? 4 : 16};
}

// Workgroups of norm_join for each compute unit: rows of one wavefront, or 1024 threads' worth of others (of
// 2048 threads' worth half waits for registers, and the last rows come unevenly: 2003 x 7168 26 us).
inline int row_groups(const RowShape& f) { return f.threads == 64 ? 32 : 1024 / f.threads; }

// ---- products of 8-bit codes (int8_gemm.hip)

// The kernels: 16 rows of x with one or two tiles of 16 weight rows a wavefront, 32 with two, or tiles of rows of x by
// weight rows (gated: half of either matrix), the last two through LDS.
enum class Int8Form { kFew1, kFew2, kFew2x32, k32x128, k64x128, k96x128, k128x128, k160x256, k192x256, k256x256 };

struct Int8Plan {
  Int8Form form;
  int parts;              // that tiles are cut into along k, their sums joined by a second kernel
  int64_t tiles;
  size_t part_bytes;      // of the sums of one part of every tile
  bool stream;            // weights bypass the caches (the nt policy)
};

// Which kernel: the one that a model of their times, fitted to 21000 measurements of 1950 sizes (1 to 16384 rows, 200 to
// 30000 channels, K 256 to 16384, plain and gated, replayed in graphs), thinks the fastest.  On 400 sizes apart from
// these, of up to 128 rows, its choice takes 0.9% more than the fastest of all kernels on average, at most 22%; on 147
// fresh ones of more rows 17% on 129 to 160 rows (at most 87%), 5% on 161 to 512 (39%), 1% above (9%).  us; a stage is
// 128 columns.
//   The kernels for few rows end at 128 rows because their fit does.  With few channels they are the fastest up to
//   some 220 rows (133 rows, 287 channels, K 2720: 7.3 on the 32 x 128 that is picked, 3.9 with one tile a wavefront; 221,
//   236, 1616 gated: 5.3 and 3.9).
//   Tiles: rounds of as many workgroups as run at once.  A stage takes what its operands take to pass
//   through a compute unit, once for each workgroup there, and so does a tile's end; all operands and results move
//   once besides, and the weights a quarter more for each further tile of rows.
//   Parts: another launch, and the sums written and read.
//   Few rows: a wavefront's steps, what passes into a compute unit, and the weights from memory, a fifth of that
//   again for each further group of rows at the same time, half for a later one.
// (333 rows, 6145 channels, K 4096: 16.2 on 96 x 128, 18.8 on 128 x 128, 20.5 on 64 x 128, 70 on 192 x 256; 2003, 4608,
// 7168: 64 on 160 x 256, 70 on 192 x 256, 76 on 256 x 256, 83 on 128 x 128; 64, 4096, 14336: 18.2 on 64 x 128 in eight
// parts, 26.7 with few rows, 44 on 32 x 128 whole; 16384, 4096, 14336: 738 on 256 x 256, 813 on 192 x 256, 828 on 160 x
// 256; 32, 7168, 2048: 5.9 with 32 rows, 7.1 with 16; 16, 4096, 14336: 13.6 with one tile on 256 workgroups, 17.1 with two.)
inline Int8Plan int8_plan(int64_t T, int64_t N, int64_t K, bool gated, int num_cu) {
  struct Tile {
    Int8Form form;
    int rows, wrows, together;     // workgroups that a compute unit holds
    double alone, each, end, start;   // a stage of one workgroup, of several for each of them; a tile's end for each, its start
    int most_parts;
  };
  static constexpr Tile kTiles[] = {
      {Int8Form::k32x128, 32, 128, 4, 0.108, 0.160, 0.40, 0.91, 8},  {Int8Form::k64x128, 64, 128, 3, 0.160, 0.203, 0.63, 1.12, 8},
      {Int8Form::k96x128, 96, 128, 3, 0.200, 0.266, 0.84, 1.38, 4},  {Int8Form::k128x128, 128, 128, 2, 0.300, 0.330, 1.32, 1.51, 4},
      {Int8Form::k160x256, 160, 256, 1, 0.650, 0.765, 5.61, 0, 1}, {Int8Form::k192x256, 192, 256, 1, 0.800, 0.822, 7.78, 0, 1},
      {Int8Form::k256x256, 256, 256, 1, 1.086, 0.960, 10.07, 0, 1},
  };
  const auto beside = [](double a, double b, double both) { return std::fmax(a, b) + both * std::fmin(a, b); };
  const int64_t most = int64_t(1) << 23;     // workgroups of a launch
  const double mats = gated ? 2 : 1, weights = mats * double(N) * double(K);
  const double results = 2.0 * double(T) * double(N);
  const double stages = double(ceil_div(K, 128));
  Int8Plan best{Int8Form::k256x256, 1, 0, 0, false};
  double best_us = 1e300;
  int64_t rows = 0;
  for (const Tile& t : kTiles) {
    const int64_t mtiles = ceil_div(T, t.rows), tiles = mtiles * ceil_div(N, gated ? t.wrows / 2 : t.wrows);
    const double moved = (weights * (1 + 0.26 * double(mtiles - 1)) + double(T) * double(K) + results) / 9.2e6;
    for (int parts = 1; parts <= t.most_parts; parts *= 2) {
      const int64_t blocks = tiles * parts, round = int64_t(num_cu) * t.together;
      if (blocks > most && t.form != Int8Form::k256x256) continue;
      if (parts > 1 && (parts > stages || blocks > 4 * round || blocks > 1 << 20)) continue;
      const auto some = [&](int n) {         // of n workgroups on a compute unit
        return stages / parts * std::fmax(t.alone, n * t.each) + n * t.end;
      };
      double work = double(blocks / round) * some(t.together);
      if (blocks % round) work += some(int(ceil_div(blocks % round, num_cu))) + t.start;
      if (parts > 1) work += 3.1 + 1.06e-6 * mats * double(T) * double(N) * parts;
      const double us = 1.84 + beside(work, moved, 1.09);
      if (us < best_us) {
        best_us = us;
        best = {t.form, parts, tiles, size_t(tiles) * t.rows * t.wrows * 4, false};
        rows = t.rows;
      }
    }
  }
  struct Few {
    Int8Form form;
    int tiles, groups;             // of 16 weight rows, of 16 rows of x
  };
  static constexpr Few kFew[] = {{Int8Form::kFew1, 1, 1}, {Int8Form::kFew2, 2, 1}, {Int8Form::kFew2x32, 2, 2}};
  if (T <= 128)
    for (const Few& f : kFew) {
      if (gated && f.tiles == 1) continue;
      const int64_t more = ceil_div(T, 16 * f.groups), each = gated ? f.tiles / 2 : f.tiles;
      const int64_t blocks = ceil_div(ceil_div(ceil_div(N, 16), each), 8) * 8 * more;
      const double steps = double(ceil_div(int64_t(stages), 8)), units = double(blocks) / num_cu;
      const bool together = units <= 4;        // a later group's weights are in the L2
      const double load = together ? std::ceil(units) : units;               // workgroups of a compute unit
      const double alone = steps * 0.015 * f.groups + 0.65 + 0.31 * (f.groups - 1);
      const double moved = load * (steps * (0.165 * f.tiles + 0.202 / 16 * double(T) / double(more) + 0.014 * f.groups) + 0.184);
      const double memory = (weights * (1 + (together ? 0.20 : 0.47) * double(more - 1)) + results) / 8.0e6;
      // (of more than 32 rows by 32 the fit is short: 48, 7168, 2048 8.4 us, 6.7 on 32 x 128)
      const double us = (1.43 + beside(beside(alone, moved, 1.345), memory, 0.926)) * (f.groups > 1 && more > 1 ? 1.05 : 1.0);
      if (us < best_us) {
        best_us = us;
        best = {f.form, 1, 0, 0, false};
        rows = 16 * f.groups;
      }
    }
  // Weights that one workgroup reads and no other, and that are too many to be found in the Infinity Cache by the
  // next call: 8 rows, 28672 channels, K 4096 (117 MB, on 32 x 128) 22.7 us, 20.4 past the caches; 5 rows, 6309, 16400 (103
  // MB, two tiles a wavefront) 22.0, 20.2; 2 rows, 8441, 10928 (92 MB, one) 22.3, 20.3.  59 MB that come back after two
  // others 10.3, 12.5 past the caches.  (One row, 128256 channels, K 4096, beyond the channels of the fit: 80.0 on the 32 x
  // 128 that is picked, 76.6 with two tiles a wavefront; 152064, 3584: 80.3 and 82.4.)
  best.stream = best.parts == 1 && T <= rows && T <= 128 && weights >= double(64 << 20);
  return best;
}

}  // namespace moe
