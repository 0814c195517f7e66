// moe_kv8_attention: attention of a batch's new tokens over the paged 8-bit cache (gfx950).
//
// A tile is up to 16 R query rows of one sequence and kv head, a row being (new token, query
// head of the group): the heads of a group share every key and value that is read.  Four
// wavefronts share the tile and deal the sequence's tokens among themselves in chunks of 64,
// each with the running maximum and sum of its own softmax; a chunk is read once, from memory
// into the registers that the matrix cores read:
//
//   S^T = K Q^T    A operand: the codes of 16 keys x 128 dimensions as they are, with their blocks'
//                  exponents (the matrix cores apply them), B operand: the queries.  Row m of the
//                  t-th product is token 4 t + m % 4 of block m / 4 of the chunk, so lane group g
//                  (16 lanes) gets the scores of the 16 tokens of block g, for its query column.
//   O^T += V^T P^T A operand: 16 dimensions x 32 tokens, group g reading 16 bytes = the 16 tokens
//                  of block g for one dimension (the cache holds values transposed), used in
//                  two products; B operand: the probabilities, which lane group g already
//                  holds for block g.  No score moves between lanes.
//
// The first product takes 8-bit numbers on both sides: a query row is scaled by a power of two and
// written as the sum of two E4M3 numbers, which together hold the eight significant bits of bf16.  (Numbers
// 2^-9 below the row's largest and less are off by up to 2^-17 of it: that is half the second
// number's smallest step, 2^-9, where the largest is 2^7.)  Two 8-bit products cost what one
// in bf16 does, and the keys' codes need no expansion: an expansion costs the vector unit
// four times an ordinary instruction, and was what bound prompts.  The values' codes, times their
// block's power of two, are expanded to bf16 exactly (E4M3 has four significant bits).  Scores, maxima
// and outputs are fp32; probabilities are rounded to bf16 (2^-8 relative at most) for the second product.
// Their sum is one more row of that product, of ones: fp32 sums of the rounded probabilities, which is
// what the values are weighted with.
//
// Work is dealt by what the sequences hold, which only the device knows: every workgroup adds up the
// batch's chunks and takes the quota that gives `target` workgroups; a tile that spans more is
// cut into parts of equal length.  Parts write their sums, maxima and outputs to scratch, and
// kv8_join adds them up, in order.
//
// One token a sequence is bound by the read of the cache: 8 sequences of up to 40000 tokens, 32 heads on
// 8 of 128, 271 MB in 53.5 us (5.1 TB/s, the join's 4.6 us and some 6 us of each workgroup's start
// and end included); 50 of up to 4500, 32 heads on 4 in pages of 16, 138 MB in 40 us.  Prompts are
// bound by what a compute unit issues: 2048 new tokens of 10240 take 319 us, 970 TFLOP/s, vector
// instructions 60% of the cycles, matrix cores 45%.  There the four wavefronts share what they read through
// LDS, and the keys go into the products as they are: 421 us with neither, the load path and the
// expansion the bounds.
#include <algorithm>

#include "kv8.h"
#include "kv8_cut.h"
#include "lds_stage.h"
#include "mxfp8.h"

namespace moe {
namespace {

constexpr int kAttWaves = 4;
constexpr int kMinChunks = 2 * kAttWaves;     // of a part: a tile is not cut below this
constexpr float kSlack = 8.0f;
constexpr float kLow = -1e30f;                // below every score: the maximum before any token

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Eight E4M3 codes times a power of two -> bf16, exact down to bf16's smallest values.
__device__ __forceinline__ bf16x8 expand8(uint32_t lo, uint32_t hi, float scale) {
  u32x4 v;
  v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false));
  v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true));
  v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false));
  v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true));
  return __builtin_bit_cast(bf16x8, v);
}

__device__ __forceinline__ float exp2_of(uint32_t e) {        // 2^(e - 127); the conversion reads the exponent
  return __uint_as_float(e << 23);
}

// 16 x 16 products of 128 E4M3 numbers with a power of two (E8M0) for each row of a and column of b.
__device__ __forceinline__ f32x4 mfma8(i32x8 a, uint32_t ae, i32x8 b, uint32_t be, f32x4 c) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, c, 0, 0, 0, int(ae), 0, int(be));
}

__device__ __forceinline__ i32x8 both(u32x4 a, u32x4 b) {
  return i32x8{int(a[0]), int(a[1]), int(a[2]), int(a[3]), int(b[0]), int(b[1]), int(b[2]), int(b[3])};
}

// Maximum over the four lanes l, l ^ 16, l ^ 32, l ^ 48: exchanges of rows of 16 and of halves.
__device__ __forceinline__ float max_of_groups(float v) {
  const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

__device__ __forceinline__ int wave_sum(int v) {
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) v += __shfl_xor(v, d);
  return v;
}
__device__ __forceinline__ int wave_scan(int v, int lane) {   // inclusive
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const int u = __shfl_up(v, d);
    v += lane >= d ? u : 0;
  }
  return v;
}

// A sequence's first row, new tokens and tokens; its tiles, and the most chunks that one of them spans.
struct Cut {
  int row0, fresh, len, tiles, chunks;
};
__device__ __forceinline__ Cut cut_of(const Kv8Batch& b, const Kv8Attend& a, const Kv8Plan& p, int G, int seq) {
  Cut c = {0, 0, 0, 0, 0};
  if (seq >= b.sequences) return c;
  c.row0 = b.cu[seq];
  c.fresh = b.cu[seq + 1] - c.row0;
  c.len = min(b.lens[seq], p.capacity);
  if (c.fresh <= 0) return c;
  c.tiles = int(min((int64_t(c.fresh) * G + p.rows - 1) / p.rows, int64_t(p.tiles)));
  c.chunks = kv8_chunks(c.len);
  if (a.window > 0) c.chunks = min(c.chunks, int((int64_t(a.window) + p.rows) / kChunk + 2));
  return c;
}

// Which tile, and part of it, workgroup `id` is; seq < 0: none.  Workgroups of a sequence follow one
// another, its heads fastest: they go round the XCDs, and with as many heads as XCDs a head's
// tiles share one L2.  Later tiles, which see more, come first.
struct Work {
  int seq, row0, fresh, len, head, tile, part, parts;
};
__device__ __forceinline__ Work find_work(const Kv8Batch& b, const Kv8Attend& a, const Kv8Plan& p, int heads, int G,
                                          int id, int lane) {
  Cut c = cut_of(b, a, p, G, lane);
  int quota = 1 << 30;
  if (p.target > 0) {
    int sum = c.tiles * c.chunks;
    for (int s0 = kWave; s0 < b.sequences; s0 += kWave) {
      const Cut d = cut_of(b, a, p, G, s0 + lane);
      sum += d.tiles * d.chunks;
    }
    const int64_t total = int64_t(wave_sum(sum)) * heads;
    quota = int(max(int64_t(kMinChunks), (total + p.target - 1) / p.target));
  }
  int before = 0;
  for (int s0 = 0; s0 < b.sequences; s0 += kWave) {
    if (s0 > 0) c = cut_of(b, a, p, G, s0 + lane);
    const int parts = max(1, (c.chunks + quota - 1) / quota);
    const int n = c.tiles * parts * heads;
    const int upto = before + wave_scan(n, lane);
    const uint64_t m = __ballot(upto > id);
    if (m != 0) {
      const int at = __builtin_ctzll(m);
      Work w;
      w.seq = s0 + at;
      w.row0 = __builtin_amdgcn_readlane(c.row0, at);
      w.fresh = __builtin_amdgcn_readlane(c.fresh, at);
      w.len = __builtin_amdgcn_readlane(c.len, at);
      w.parts = __builtin_amdgcn_readlane(parts, at);
      const int local = id - __builtin_amdgcn_readlane(upto - n, at);
      w.head = local % heads;
      w.part = local / heads % w.parts;
      w.tile = __builtin_amdgcn_readlane(c.tiles, at) - 1 - local / heads / w.parts;
      return w;
    }
    before = __builtin_amdgcn_readlane(upto, kWave - 1);
  }
  return Work{-1, 0, 0, 0, 0, 0, 0, 1};
}

// What kv8_join has to know of a row: the workgroup of its first part (the others follow a head count
// apart), and its parts times 128 plus its place in the tile.
struct RowParts {
  int first, packed;
};

// A wavefront has 16 R query rows.  SHARED: the four wavefronts have rows of their own and walk the tokens
// together, through a ring of LDS stages that each fills a quarter of; otherwise all have the same
// rows and deal the tokens among themselves, straight from memory.  A wavefront takes 16 NW tokens at a time (NW = 4 or 2); a lane group has 4 NW of
// them, a block or half of one.  UNIFORM: a page holds whole steps, so that a step's page is one number.
template <int D, int R, int NW, int OCC, bool SHARED, bool UNIFORM>
__global__ __launch_bounds__(64 * kAttWaves, OCC) void kv8_attention_kernel(Kv8Cache c, Kv8Batch b, Kv8Attend a, Kv8Plan plan) {
  constexpr int QW = D == 64 ? 1 : D / 64;    // operands of 16 bytes a lane of one part of the queries
  constexpr int DT = D / 16;                  // tiles of 16 dimensions
  constexpr int kTok = 16 * NW, kHalf = 4 / NW;   // tokens of a step, lane groups of a block
  typedef uint32_t vwords __attribute__((ext_vector_type(NW)));
  __shared__ float ml[SHARED ? 1 : kAttWaves][2][16 * R];
  __shared__ f32x4 oo[SHARED ? 1 : kAttWaves / 2][SHARED ? 1 : DT * R][64];
  // the queries' two parts, as operands: in LDS, or in registers where there is room
  constexpr bool kHeld = SHARED && D <= 128;
  __shared__ u32x4 ql[SHARED && !kHeld ? kAttWaves : 1][kHeld ? 1 : R][kHeld ? 1 : 2][kHeld ? 1 : QW][64];
  u32x4 qh[kHeld ? R : 1][2][QW];
  // LDS stages: operands in the order of the lanes that read them, keys then values
  constexpr int kStages = D <= 128 ? 3 : 2, kKeys = NW * (D / 64), kPieces = kKeys + DT;
  __shared__ u32x4 ring[SHARED ? kStages : 1][SHARED ? kPieces : 1][64];
  static_assert(!SHARED || (NW == 4 && kPieces % kAttWaves == 0), "pieces of 16 bytes a lane");
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = lane >> 4, col = lane & 15;
  const int G = a.q_heads / c.heads;
  const Work w = find_work(b, a, plan, c.heads, G, blockIdx.x, lane);
  if (w.seq < 0) return;
  const int row0 = w.row0, fresh = w.fresh, len = w.len;
  const int in_tile = SHARED ? wave * 16 * R : 0;
  const int first_row = w.tile * (SHARED ? kAttWaves * 16 * R : 16 * R) + in_tile;
  const int rows = min(16 * R, int(min(int64_t(fresh) * G, int64_t(1) << 30)) - first_row);
  // positions of the first and the last row, of the wavefront's and of the tile's
  const int first_pos = len - fresh + first_row / G, last_pos = len - fresh + (first_row + rows - 1) / G;
  const int tile_row = w.tile * plan.rows, tile_rows = min(plan.rows, int(min(int64_t(fresh) * G, int64_t(1) << 30)) - tile_row);
  const int tile_first = len - fresh + tile_row / G, tile_last = len - fresh + (tile_row + tile_rows - 1) / G;
  const Kv8Steps steps = kv8_steps(tile_first, tile_last, a.window, w.part, w.parts, kTok);
  const int begin = steps.begin, end = steps.end;

  // queries: row r is token r / G, head r % G of the group
  int pos[R];                                 // position of the column's token; -1: sees nothing
  uint32_t qe[R];                             // its queries' exponent, 127 + e
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int local = 16 * r + col;
    const int row = first_row + local;
    const int64_t t = int64_t(row0) + row / G;
    const bool on = local < rows && uint64_t(t) < uint64_t(b.tokens);
    pos[r] = on ? len - fresh + row / G : -1;
    const uint16_t* p = a.q + (t * a.q_heads + w.head * G + row % G) * D + 16 * g;
    u32x4 v[QW][2];
    float mx = 0.f, odd = 0.f;                // odd: 0, or NaN where an element is not finite
#pragma unroll
    for (int s = 0; s < QW; ++s)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        v[s][h] = u32x4{0u, 0u, 0u, 0u};
        if (on) v[s][h] = *reinterpret_cast<const u32x4*>(p + 64 * s + 8 * h);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = __uint_as_float(v[s][h][i] << 16), y = __uint_as_float(v[s][h][i] & 0xFFFF0000u);
          mx = fmaxf(mx, fmaxf(fabsf(x), fabsf(y)));
          odd += 0.f * x + 0.f * y;
        }
      }
    mx = max_of_groups(mx);
    // power of two that takes the largest into [128, 256)
    const int e = min(max(int(__float_as_uint(mx) >> 23) - 7, 1), 253);
    qe[r] = uint32_t(e);
    if (!SHARED && r % kAttWaves != wave) continue;
    const float down = __uint_as_float(uint32_t(254 - e) << 23);
#pragma unroll
    for (int s = 0; s < QW; ++s) {
      u32x4 hi, lo;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w0 = v[s][i / 2][2 * (i % 2)], w1 = v[s][i / 2][2 * (i % 2) + 1];
        const float x[4] = {__uint_as_float(w0 << 16) * down, __uint_as_float(w0 & 0xFFFF0000u) * down,
                            __uint_as_float(w1 << 16) * down, __uint_as_float(w1 & 0xFFFF0000u) * down};
        int c8 = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
        c8 = __builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], c8, true);
        const auto a0 = __builtin_amdgcn_cvt_pk_f32_fp8(c8, false), a1 = __builtin_amdgcn_cvt_pk_f32_fp8(c8, true);
        int c9 = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] - a0[0], x[1] - a0[1], 0, false);
        c9 = __builtin_amdgcn_cvt_pk_fp8_f32(x[2] - a1[0], x[3] - a1[1], c9, true);
        // not finite: the lane's numbers are all NaN, and with them the row's scores
        hi[i] = odd == 0.f ? uint32_t(c8) : 0x7F7F7F7Fu;
        lo[i] = odd == 0.f ? uint32_t(c9) : 0x7F7F7F7Fu;
      }
      if constexpr (kHeld) {
        qh[r][0][s] = hi;
        qh[r][1][s] = lo;
      } else {
        ql[SHARED ? wave : 0][r][0][s][lane] = hi;
        ql[SHARED ? wave : 0][r][1][s][lane] = lo;
      }
    }
  }
  if (!SHARED) __syncthreads();
  auto query = [&](int r, int part, int s) {
    if constexpr (kHeld) return qh[r][part][s];
    else return ql[SHARED ? wave : 0][r][part][s][lane];
  };

  f32x4 o[DT][R], l[R];                       // l: the sum, in every element
  float m[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = kLow;
    l[r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d][r] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float scale = a.scale * 1.44269504088896f;            // scores in powers of two

  // Where a step's blocks are: the lane's of the keys (a row of the first product) and of the values.  A
  // page is looked up a step ahead of its loads.  Past the end of the sequence the last block stands in,
  // where a page does not hold the whole step.
  const int k_of = (col >> 2) / kHalf, v_of = g / kHalf;      // the lane's blocks of a step
  const int per_page = c.page / kKvBlock, last_block = max(len - 1, 0) / kKvBlock;
  const int32_t* table = b.table + int64_t(w.seq) * b.table_cols;
  const uint32_t page_blocks = uint32_t(c.heads) * uint32_t(per_page), head_blocks = uint32_t(w.head) * uint32_t(per_page);
  struct Block {
    int page, inside;
  };
  struct Place {
    Block k, v;                               // UNIFORM: k alone, of the step's first block
  };
  auto find = [&](int block) {
    // block / per_page, by the reciprocal rounded down: one too few at most
    int at = int(__umulhi(uint32_t(block), plan.inverse)), rest = block - at * per_page;
    const bool more = rest >= per_page;
    at += more ? 1 : 0;
    rest -= more ? per_page : 0;
    return Block{table[at], rest};
  };
  auto look_up = [&](int step) {
    Place x;
    if (UNIFORM) {
      x.k = find(NW * step);
    } else {
      x.k = find(min(NW * step + k_of, last_block));
      x.v = find(min(NW * step + v_of, last_block));
    }
    return x;
  };
  auto block_at = [&](const Block& x) {                       // among the cache's blocks
    // read where it is used: a load in flight until then, and scalar from here on
    const int at = UNIFORM ? __builtin_amdgcn_readfirstlane(x.page) : x.page;
    const uint32_t page = min(uint32_t(max(at, 0)), uint32_t(c.pages - 1));
    return uint64_t(page) * page_blocks + (head_blocks + uint32_t(x.inside));
  };
  // A read-once load where one tile reads what it sees: its heads share the rows.
  auto fetch = [&](const auto* p) {
    if constexpr (R == 1) return __builtin_nontemporal_load(p);
    else return *p;
  };

  u32x4 kc[SHARED ? 1 : NW][D / 64];
  vwords vc[SHARED ? 1 : DT];
  uint32_t ke, ve;
  int stage = 0;                                              // of the ring, that the step is in
  const uint32_t k_lane = ((col >> 2) % kHalf * (4 * NW) + (col & 3)) * D + 16 * g;   // inside a block
  const uint32_t v_lane = col * kKvBlock + g % kHalf * (4 * NW);
  auto k_at = [&](const Place& x) {
    return c.k_codes + block_at(x.k) * (kKvBlock * D) + (UNIFORM ? k_of * (kKvBlock * D) + k_lane : k_lane);
  };
  auto v_at = [&](const Place& x) {
    return c.v_codes + block_at(UNIFORM ? x.k : x.v) * (kKvBlock * D) + (UNIFORM ? v_of * (kKvBlock * D) + v_lane : v_lane);
  };
  auto load_k = [&](const Place& x) {
    const uint8_t* p = k_at(x);
#pragma unroll
    for (int t = 0; t < NW; ++t)
#pragma unroll
      for (int s = 0; s < D / 64; ++s) kc[t][s] = fetch(reinterpret_cast<const u32x4*>(p + 4 * t * D + 64 * s));
  };
  auto load_v = [&](const Place& x) {
    const uint8_t* p = v_at(x);
#pragma unroll
    for (int d = 0; d < DT; ++d) vc[d] = fetch(reinterpret_cast<const vwords*>(p + 16 * d * kKvBlock));
  };
  auto load_ke = [&](const Place& x) { return uint32_t(c.k_exps[block_at(x.k) + (UNIFORM ? k_of : 0)]); };
  auto load_ve = [&](const Place& x) { return uint32_t(c.v_exps[block_at(UNIFORM ? x.k : x.v) + (UNIFORM ? v_of : 0)]); };
  // This wavefront's quarter of a step's operands, from memory into stage `to`.
  auto fill = [&](const Place& x, int to) {
    const uint8_t *k = k_at(x), *v = v_at(x);
#pragma unroll
    for (int i = 0; i < kPieces / kAttWaves; ++i) {
      const int j = i * kAttWaves + wave;
      const uint8_t* p = j < kKeys ? k + (j / (D / 64)) * (4 * D) + j % (D / 64) * 64 : v + (j - kKeys) * (16 * kKvBlock);
      __builtin_amdgcn_global_load_lds(p, reinterpret_cast<uint8_t*>(&ring[to][j][0]), 16, 0, 0);
    }
  };
  auto keys = [&](int t, int s) {
    if constexpr (SHARED) return ring[stage][t * (D / 64) + s][lane];
    else return kc[t][s];
  };
  auto values = [&](int d) {
    if constexpr (SHARED) return __builtin_bit_cast(vwords, ring[stage][kKeys + d][lane]);
    else return vc[d];
  };

  auto scores = [&](f32x4 (&s)[NW][R]) {
#pragma unroll
    for (int t = 0; t < NW; ++t) {
#pragma unroll
      for (int r = 0; r < R; ++r) s[t][r] = f32x4{0.f, 0.f, 0.f, 0.f};
      if constexpr (D == 64) {                                // both parts of the queries in one product
        const i32x8 k8 = both(keys(t, 0), keys(t, 0));
#pragma unroll
        for (int r = 0; r < R; ++r) s[t][r] = mfma8(k8, ke, both(query(r, 0, 0), query(r, 1, 0)), qe[r], s[t][r]);
      } else {
#pragma unroll
        for (int k = 0; k < D / 128; ++k) {
          const i32x8 k8 = both(keys(t, 2 * k), keys(t, 2 * k + 1));
#pragma unroll
          for (int part = 0; part < 2; ++part)
#pragma unroll
            for (int r = 0; r < R; ++r)
              s[t][r] = mfma8(k8, ke, both(query(r, part, 2 * k), query(r, part, 2 * k + 1)), qe[r], s[t][r]);
        }
      }
    }
  };
  // Probabilities of a step as the operands of the second product; masked scores are -infinity.
  auto softmax = [&](const f32x4 (&s)[NW][R], bf16x8 (&p)[NW / 2][R]) {
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float mx = fmaxf(fmaxf(s[0][r][0], s[0][r][1]), fmaxf(s[0][r][2], s[0][r][3]));
#pragma unroll
      for (int t = 1; t < NW; ++t)
        mx = fmaxf(mx, fmaxf(fmaxf(s[t][r][0], s[t][r][1]), fmaxf(s[t][r][2], s[t][r][3])));
      // The reference of the exponentials need not be the maximum, only near it: it follows once a score
      // is kSlack above it (probabilities then reach 2^kSlack, in bf16 as exact as any others).  Held
      // to the maximum, some column of sixteen had a new one in half of the steps.
      mx = max_of_groups(mx) * scale;
      if (__ballot(mx > m[r] + kSlack) != 0) {
        const float mn = fmaxf(m[r], mx), f = __builtin_amdgcn_exp2f(m[r] - mn);
        l[r] *= f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d][r] *= f;
        m[r] = mn;
      }
      const float mn = m[r];
#pragma unroll
      for (int h = 0; h < NW / 2; ++h) {
        u32x4 v;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          v[i] = pack_bf16x2(
              __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * h + i / 2][r][2 * (i % 2)], scale, -mn)),
              __builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * h + i / 2][r][2 * (i % 2) + 1], scale, -mn)));
        p[h][r] = __builtin_bit_cast(bf16x8, v);
      }
    }
  };
  // In a step that some row does not see in full: values are anything, NaN or infinite too, where no row
  // sees their token, and where some row must not, and 0 times these is NaN.  What no row of the wavefront sees
  // is taken out, codes and, for a whole block, its exponent.  Of the rest, codes of NaN and of what
  // bf16 has no finite number for are taken out, and the rows that do see their token get a NaN score instead.
  const int seen_from = a.window > 0 ? max(max(first_pos, 0) - a.window + 1, 0) : 0;
  uint32_t keep[NW];                                          // bytes of the lane's words that some row sees
  uint32_t over;                                              // 0x80 less the first code taken out, in each byte
  auto clean = [&](uint32_t x, uint32_t keep, uint32_t& out) {
    x &= keep;
    out = ((x & 0x7F7F7F7Fu) + over) & 0x80808080u;
    return x & ~(out | (out - (out >> 7)));
  };
  auto mask = [&](int ch, f32x4 (&s)[NW][R]) {
    const int t0 = ch * kTok + 4 * NW * g;                    // first of the lane's tokens
    const int n1 = min(max(last_pos + 1 - t0, 0), 4 * NW), n0 = min(max(seen_from - t0, 0), n1);
    ve = n0 < n1 ? ve : 127u;
    // NaN is 0x7F.  At 2^120 codes from 2^8 = 0x78 on are past bf16's numbers, at each power more a power
    // less; an exponent byte of 255 is NaN
    over = ve < 247u ? 0x01010101u : ve < 255u ? (ve - 246u) * 0x08080808u : 0x80808080u;
    uint32_t bad[NW];                                         // bit 8 i + 7 of word t: its token 4 t + i
#pragma unroll
    for (int t = 0; t < NW; ++t) {
      const auto below = [](int n) { return n <= 0 ? 0u : n >= 4 ? 0xFFFFFFFFu : (1u << (8 * n)) - 1u; };
      keep[t] = below(n1 - 4 * t) & ~below(n0 - 4 * t);
      bad[t] = 0;
    }
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      const vwords v = values(d);
#pragma unroll
      for (int t = 0; t < NW; ++t) {
        uint32_t out;
        clean(v[t], keep[t], out);
        bad[t] |= out;
      }
    }
    ve = ve < 255u ? ve : 127u;
#pragma unroll
    for (int t = 0; t < NW; ++t)
#pragma unroll
      for (int i = 1; i < 16; i <<= 1) bad[t] |= uint32_t(__shfl_xor(int(bad[t]), i));
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
      for (int t = 0; t < NW; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int tok = t0 + 4 * t + i;
          float x = s[t][r][i];
          x = (bad[t] >> (8 * i + 7)) & 1u ? NAN : x;
          s[t][r][i] = tok > pos[r] || (a.window > 0 && pos[r] - tok >= a.window) ? -INFINITY : x;
        }
  };
  auto weigh = [&](const bf16x8 (&p)[NW / 2][R], bool edge) {
    const float vf = exp2_of(ve);
    const u32x4 ones = {0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u};
#pragma unroll
    for (int h = 0; h < NW / 2; ++h)
#pragma unroll
      for (int r = 0; r < R; ++r) l[r] = mfma16(__builtin_bit_cast(bf16x8, ones), p[h][r], l[r]);
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      vwords v = values(d);
      if (edge) {
#pragma unroll
        for (int t = 0; t < NW; ++t) {
          uint32_t out;
          v[t] = clean(v[t], keep[t], out);
        }
      }
#pragma unroll
      for (int h = 0; h < NW / 2; ++h) {
        const bf16x8 va = expand8(v[2 * h], v[2 * h + 1], vf);
#pragma unroll
        for (int r = 0; r < R; ++r) o[d][r] = mfma16(va, p[h][r], o[d][r]);
      }
    }
  };
  auto step = [&](int ch, auto&& after_scores) {
    f32x4 s[NW][R];
    scores(s);
    after_scores();
    bf16x8 p[NW / 2][R];
    const bool edge = ch * kTok + kTok - 1 > first_pos || (a.window > 0 && last_pos - ch * kTok >= a.window);
    if (edge) mask(ch, s);
    softmax(s, p);
    weigh(p, edge);
  };

  const int last = end - 1;
  if constexpr (SHARED) {
    // kStages - 1 steps in flight.  A stage is filled again after the barrier that follows its last reads.
    // All loads but the newest fills being done means that the step's own fill is.
    constexpr int kAhead = kStages - 1, kFill = kPieces / kAttWaves;
    static_assert(kAhead <= 2, "first fills");
    if (begin < end) {
      Place at[kAhead + 1];                                   // of the steps ch, ch + 1, ..
#pragma unroll
      for (int i = 0; i <= kAhead; ++i) at[i] = look_up(min(begin + i, last));
      uint32_t ke1 = load_ke(at[0]), ve1 = load_ve(at[0]);
      // in ring order: the waits below count on it
      constexpr int st0 = 0, st1 = 1;
      auto issue = [&](int to, int i) { fill(at[i], to); };
      __builtin_amdgcn_sched_barrier(0);
      issue(st0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if constexpr (kAhead == 2) issue(st1, 1);
      __builtin_amdgcn_sched_barrier(0);
      for (int ch = begin; ch < end; ++ch) {
        __builtin_amdgcn_s_waitcnt(wait_vm((kAhead - 1) * kFill) & ~0x0F00);   // and the LDS reads
        bare_barrier();
        ke = ke1;
        ve = ve1;
        ke1 = load_ke(at[1]);
        ve1 = load_ve(at[1]);
        const Place next = look_up(min(ch + kAhead + 1, last));
        fill(at[kAhead], stage == 0 ? kAhead : stage - 1);
#pragma unroll
        for (int i = 0; i < kAhead; ++i) at[i] = at[i + 1];
        at[kAhead] = next;
        // steps wholly after the wavefront's last row, or before its first one's window, are not its own
        if (rows > 0 && ch * kTok <= last_pos && !(a.window > 0 && first_pos - (ch * kTok + kTok - 1) >= a.window))
          step(ch, [] {});
        stage = stage == kAhead ? 0 : stage + 1;
      }
    }
    __builtin_amdgcn_s_waitcnt(wait_vm(0));                   // fills past the end: the LDS is handed back
    if (rows <= 0) return;
  } else {
    // The loads of the next step are issued as soon as the registers of this one's are free: the keys
    // after the scores, the values after the second product.
    int ch = begin + wave;
    if (ch < end) {
      Place at = look_up(ch);
      load_k(at);
      ke = load_ke(at);
      load_v(at);
      ve = load_ve(at);
      at = look_up(min(ch + kAttWaves, last));
      for (; ch < end; ch += kAttWaves) {
        Place next;
        step(ch, [&] {
          load_k(at);
          ke = load_ke(at);
          next = look_up(min(ch + 2 * kAttWaves, last));
        });
        load_v(at);
        ve = load_ve(at);
        at = next;
      }
    }
  }

  float total[R], top[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    total[r] = l[r][0];
    top[r] = m[r];
  }
  if constexpr (!SHARED) {
    // join the wavefronts: all maxima and sums, then the outputs of half the waves at a time
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (g == 0) {
        ml[wave][0][16 * r + col] = m[r];
        ml[wave][1][16 * r + col] = l[r][0];
      }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
      top[r] = kLow;
#pragma unroll
      for (int v = 0; v < kAttWaves; ++v) top[r] = fmaxf(top[r], ml[v][0][16 * r + col]);
      total[r] = 0.f;
#pragma unroll
      for (int v = 0; v < kAttWaves; ++v)
        total[r] += ml[v][1][16 * r + col] * __builtin_amdgcn_exp2f(ml[v][0][16 * r + col] - top[r]);
      const float f = __builtin_amdgcn_exp2f(m[r] - top[r]);
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d][r] *= f;
    }
#pragma unroll
    for (int half = kAttWaves / 2; half >= 1; half /= 2) {
      if (wave >= half && wave < 2 * half) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int r = 0; r < R; ++r) oo[wave - half][d * R + r][lane] = o[d][r];
      }
      __syncthreads();
      if (wave < half) {
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int r = 0; r < R; ++r) o[d][r] += oo[wave][d * R + r][lane];
      }
      __syncthreads();
    }
    if (wave != 0) return;
  }
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int local = 16 * r + col;
    if (local >= rows) continue;
    const int row = first_row + local;
    const int64_t t = int64_t(row0) + row / G;
    if (uint64_t(t) >= uint64_t(b.tokens)) continue;
    if (w.parts == 1) {
      if (plan.target > 0 && g == 0)
        reinterpret_cast<RowParts*>(a.ws)[t * a.q_heads + w.head * G + row % G] = RowParts{0, 128};
      const float inv = total[r] > 0.f ? 1.0f / total[r] : total[r] == 0.f ? 0.f : total[r];
      uint16_t* out = a.out + (t * a.q_heads + w.head * G + row % G) * D + 4 * g;
#pragma unroll
      for (int d = 0; d < DT; ++d)
        *reinterpret_cast<u32x2*>(out + 16 * d) =
            u32x2{pack_bf16x2(o[d][r][0] * inv, o[d][r][1] * inv), pack_bf16x2(o[d][r][2] * inv, o[d][r][3] * inv)};
    } else {
      if (g == 0 && w.part == 0)
        reinterpret_cast<RowParts*>(a.ws)[t * a.q_heads + w.head * G + row % G] = RowParts{int(blockIdx.x), w.parts * 128 + in_tile + local};
      // [workgroup][row][D + 4]: the sums, then the maximum and the sum of the softmax
      float* part = a.ws + plan.row_words + (int64_t(blockIdx.x) * plan.rows + in_tile + local) * (D + 4);
#pragma unroll
      for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(part + 16 * d + 4 * g) = o[d][r];
      if (g == 0) {
        part[D] = top[r];
        part[D + 1] = total[r];
      }
    }
  }
}

// Joins the parts of a row (token, query head) that has several: one workgroup a row, its wavefronts
// deal the parts among themselves, eight at a time in flight, and are joined in order.
template <int D>
__global__ __launch_bounds__(256) void kv8_join_kernel(Kv8Cache c, Kv8Batch b, Kv8Attend a, Kv8Plan plan) {
  constexpr int kPer = D / 64, kAhead = 8;
  __shared__ float acc4[4][D], ml[4][2];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t unit = blockIdx.x;
  // rows that no workgroup had (more new tokens than the caller said) have anything here
  const RowParts rp = reinterpret_cast<const RowParts*>(a.ws)[unit];
  const int first = rp.first, parts = rp.packed >> 7, in_tile = rp.packed & 127;
  if (parts <= 1 || first < 0 || in_tile >= plan.rows ||
      int64_t(first) + int64_t(parts - 1) * c.heads >= plan.workgroups)
    return;
  const float* part = a.ws + plan.row_words + (int64_t(first) * plan.rows + in_tile) * (D + 4);
  const int64_t stride = int64_t(c.heads) * plan.rows * (D + 4);
  float acc[kPer], total = 0.f, top = kLow;
#pragma unroll
  for (int i = 0; i < kPer; ++i) acc[i] = 0.f;
  for (int s0 = wave; s0 < parts; s0 += 4 * kAhead) {
    float m[kAhead], l[kAhead], v[kAhead][kPer];
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const float* p = part + int64_t(min(s0 + 4 * j, parts - 1)) * stride;
      m[j] = p[D];
      l[j] = p[D + 1];
#pragma unroll
      for (int i = 0; i < kPer; ++i) v[j][i] = p[lane * kPer + i];
    }
    __builtin_amdgcn_sched_barrier(0);                        // all loads first
    float mx = top;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) mx = fmaxf(mx, s0 + 4 * j < parts ? m[j] : kLow);
    const float old = __builtin_amdgcn_exp2f(top - mx);
    total *= old;
#pragma unroll
    for (int i = 0; i < kPer; ++i) acc[i] *= old;
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      const float f = s0 + 4 * j < parts ? __builtin_amdgcn_exp2f(m[j] - mx) : 0.f;
      total += l[j] * f;
#pragma unroll
      for (int i = 0; i < kPer; ++i) acc[i] += v[j][i] * f;
    }
    top = mx;
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) acc4[wave][lane * kPer + i] = acc[i];
  if (lane == 0) {
    ml[wave][0] = top;
    ml[wave][1] = total;
  }
  __syncthreads();
  if (threadIdx.x >= D / 2) return;
  const int d = 2 * threadIdx.x;
  float mx = kLow, sum = 0.f, x0 = 0.f, x1 = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) mx = fmaxf(mx, ml[w][0]);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const float f = __builtin_amdgcn_exp2f(ml[w][0] - mx);
    sum += ml[w][1] * f;
    x0 += acc4[w][d] * f;
    x1 += acc4[w][d + 1] * f;
  }
  const float inv = sum > 0.f ? 1.0f / sum : sum == 0.f ? 0.f : sum;
  *reinterpret_cast<uint32_t*>(a.out + unit * D + d) = pack_bf16x2(x0 * inv, x1 * inv);
}

template <int D, int R, int NW, int OCC, bool SHARED, bool UNIFORM>
hipError_t launch_as(const Kv8Cache& c, const Kv8Batch& b, const Kv8Attend& a, const Kv8Plan& p, hipStream_t s) {
  const dim3 grid(unsigned(p.workgroups)), block(64 * kAttWaves);
  MOE_LAUNCH("kv8_attention", (kv8_attention_kernel<D, R, NW, OCC, SHARED, UNIFORM>), grid, block, s, c, b, a, p);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess || p.target == 0) return err;
  MOE_LAUNCH("kv8_join", (kv8_join_kernel<D>), dim3(unsigned(b.tokens * a.q_heads)), dim3(256), s, c, b, a, p);
  return hipGetLastError();
}

template <int D, int R, int NW, int OCC, bool SHARED>
hipError_t launch(const Kv8Cache& c, const Kv8Batch& b, const Kv8Attend& a, const Kv8Plan& p, hipStream_t s) {
  if (c.page % (16 * NW) == 0) return launch_as<D, R, NW, OCC, SHARED, true>(c, b, a, p, s);
  return launch_as<D, R, NW, OCC, SHARED, false>(c, b, a, p, s);
}

template <int D>
hipError_t launch_rows(const Kv8Cache& c, const Kv8Batch& b, const Kv8Attend& a, const Kv8Plan& p, hipStream_t s) {
  if (p.rows == 16) {
    // pages that hold no whole step of 64 tokens are looked up lane by lane: shorter steps then (50
    // sequences of up to 4500 tokens, pages of 16: 42 us with 64 tokens, 39 with 32)
    if constexpr (D <= 128) {
      if (c.page % 64 == 0) return launch_as<D, 1, 4, 2, false, true>(c, b, a, p, s);
    }
    return launch<D, 1, 2, 2, false>(c, b, a, p, s);
  }
  if (p.rows == 32) return launch<D, 2, 2, D <= 128 ? 2 : 1, false>(c, b, a, p, s);
  return launch<D, 2, 4, D <= 128 ? 2 : 1, true>(c, b, a, p, s);
}

}  // namespace

Kv8Plan kv8_plan(int sequences, int q_heads, int heads, int dim, int max_new, int max_len, int window, int num_cu) {
  Kv8Plan p = {};
  const int64_t rows = int64_t(max_new) * (q_heads / heads);
  const int64_t seen = window > 0 ? std::min<int64_t>(max_len, int64_t(window) + max_new) : max_len;
  const auto tiles_of = [&](int of) { return int64_t(sequences) * heads * ((rows + of - 1) / of); };
  const auto work = [&](int of) { return tiles_of(of) * ((seen + kChunk - 1) / kChunk); };
  // Rows of a tile.  Large ones read a block for more rows, small ones give more workgroups and wait less
  // for each step: small ones while all steps together are few.  us with 16, 32 and 128: 4 x 218 new tokens
  // of 5 heads 10.8, 12.2, 18.3; 1 x 699 of 2 x 4 heads 21, 15.6, 20; 6 x 308 of 4 x 4 heads 29, 23, 20;
  // 4 x 2000 of 8 x 4 heads 488, 308, 190.  Up to 64 rows a tile of 128 is mostly empty (8 x 9 tokens of
  // 8 x 4 heads, with 32 and 128 rows: all 8000 long 46 and 49 us, of up to 8000 25 and 36).
  if (work(16) <= 8 * int64_t(num_cu))
    p.rows = 16;
  else if (rows > 16 && (rows <= 64 || work(32) <= 12 * int64_t(num_cu)))
    p.rows = 32;
  else
    p.rows = rows <= 16 ? 16 : 128;
  p.tiles = int((rows + p.rows - 1) / p.rows);
  // Few tiles are cut so that all parts together are at most the two workgroups that a compute unit has
  // place for at a time; more tiles, whose parts would then be of too few sizes, for four a unit (8
  // heads: 1 sequence of 40000 22.9 us so, 27.5 with four a unit; 8 of up to 40000 52.4 and 55; 20 of 4000 27
  // and 29; 4 heads, 50 of 4500 42 and 39).  They are not cut where there are enough of
  // them, nor where they are so short that the join, some 5 us or more, costs what is gained
  // (4 sequences of 8 x 4 heads of 128, uncut and cut with join: 1024 long 15 and 17 us, 1536 19 and
  // 17; of 256: 768 long 20.6 and 19.4; tiles of 128 rows of 256, 749 long: 60 and 83).
  const int64_t tiles = tiles_of(p.rows);
  const int64_t uncut = (dim <= 128 || p.rows == 128 ? 2 : 1) * kMinChunks * kChunk;
  if (tiles < 2 * int64_t(num_cu) && seen > uncut)
    p.target = 3 * tiles <= 2 * int64_t(num_cu) ? 2 * num_cu - int(tiles) : (p.rows == 32 ? 2 : 4) * num_cu;
  return p;
}

// Parts are never more than the tiles and the target together: a part but the last of a tile holds a
// quota of chunks, and `target` quotas hold them all.
int64_t kv8_workgroups(const Kv8Plan& p, int sequences, int heads) {
  return int64_t(sequences) * heads * p.tiles + p.target;
}

// [a RowParts for each row | the parts]
static int64_t row_words(int64_t tokens, int q_heads) { return (tokens * q_heads * 2 + 3) / 4 * 4; }

size_t kv8_workspace_bytes(const Kv8Plan& p, int64_t tokens, int sequences, int q_heads, int heads, int dim) {
  if (p.target == 0) return 0;
  return (size_t(row_words(tokens, q_heads)) + size_t(kv8_workgroups(p, sequences, heads)) * p.rows * (dim + 4)) *
         sizeof(float);
}

hipError_t launch_kv8_attention(const Kv8Cache& c, const Kv8Batch& b, const Kv8Attend& a, const Kv8Plan& plan,
                                hipStream_t s) {
  Kv8Plan p = plan;
  const uint32_t per_page = uint32_t(c.page / kKvBlock);
  p.inverse = per_page == 1 ? 0xFFFFFFFFu : uint32_t((uint64_t(1) << 32) / per_page);
  p.row_words = row_words(b.tokens, a.q_heads);
  p.capacity = int(std::min<int64_t>(int64_t(b.table_cols) * c.page, INT32_MAX));
  if (!kv8_counts_fit(int64_t(b.sequences) * p.tiles, p.capacity)) p.target = 0;
  p.workgroups = kv8_workgroups(p, b.sequences, c.heads);
  if (c.dim == 64) return launch_rows<64>(c, b, a, p, s);
  if (c.dim == 128) return launch_rows<128>(c, b, a, p, s);
  return launch_rows<256>(c, b, a, p, s);
}

}  // namespace moe
