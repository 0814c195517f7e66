// moe_kv8_attention: attention of a batch's new tokens over the paged 8-bit cache (gfx950).
//
// A tile is up to 16 R query rows of one sequence and kv head, a row being (new token, query
// head of the group): the heads of a group share every key and value that is read.  Four
// wavefronts share the tile and deal the sequence's tokens among themselves in chunks of 64,
// each with the running maximum and sum of its own softmax; a chunk is read once, from memory
// into the registers that the matrix cores read:
//
//   S^T = K Q^T    A operand: 16 keys x 32 dimensions, B operand: the queries.  Row m of the t-th
//                  product is token 4 t + m % 4 of block m / 4 of the chunk, so lane group g (16
//                  lanes) gets the scores of the 16 tokens of block g, for its query column:
//                  one block, one exponent.
//   O^T += V^T P^T A operand: 16 dimensions x 32 tokens, group g reading 16 bytes = the 16 tokens
//                  of block g for one dimension (the cache holds values transposed), used in
//                  two products; B operand: the probabilities, which lane group g already
//                  holds for block g.  No score moves between lanes.
//
// Codes are expanded to bf16 exactly (E4M3 has four significant bits); the keys' exponent goes
// into the scores and the values' into the probabilities, both powers of two.  Scores, maxima,
// sums and outputs are fp32; probabilities are rounded to bf16 (2^-9 relative) for the product.
#include <algorithm>

#include "kv8.h"

namespace moe {
namespace {

constexpr int kAttWaves = 4;
constexpr int kChunk = 64;                    // tokens that a wavefront takes at a time
constexpr float kLow = -1e30f;                // below every score: the maximum before any token

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Eight E4M3 codes -> bf16, exact.
__device__ __forceinline__ bf16x8 expand8(uint32_t lo, uint32_t hi) {
  u32x4 v;
  v[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false));
  v[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true));
  v[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false));
  v[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true));
  return __builtin_bit_cast(bf16x8, v);
}

__device__ __forceinline__ float exp2_of(uint32_t e) {        // 2^(e - 127), 0 for e = 0
  return __uint_as_float(e << 23);
}

// What a tile sees: the rows and the chunks of tokens of one part of it.
struct Span {
  int row0, fresh, len;     // the sequence's first row, new tokens and tokens
  int rows;                 // query rows of the tile (of 16 R)
  int begin, end;           // chunks
};

__device__ __forceinline__ Span span_of(const Kv8Batch& b, int seq, int G, int tile, int tile_rows, int split,
                                        int splits, int64_t window, int64_t capacity) {
  Span s;
  s.row0 = b.cu[seq];
  s.fresh = b.cu[seq + 1] - s.row0;
  s.len = int(min(int64_t(b.lens[seq]), capacity));
  const int first = tile * tile_rows;
  s.rows = int(min(int64_t(tile_rows), int64_t(s.fresh) * G - first));
  s.begin = s.end = 0;
  if (s.rows <= 0) return s;
  const int64_t past = int64_t(s.len) - s.fresh;
  const int64_t last = past + (first + s.rows - 1) / G;       // position of the last row
  const int64_t low = window > 0 ? max(past + first / G - window + 1, int64_t(0)) : 0;
  const int c0 = int(low / kChunk), c1 = last < 0 ? 0 : int(last / kChunk) + 1;
  if (c1 <= c0) return s;
  const int each = (c1 - c0 + splits - 1) / splits;
  s.begin = min(c0 + split * each, c1);
  s.end = min(s.begin + each, c1);
  return s;
}

template <int D, int R>
__global__ __launch_bounds__(64 * kAttWaves) void kv8_attention_kernel(Kv8Cache c, Kv8Batch b, Kv8Attend a,
                                                                       Kv8Plan plan) {
  constexpr int KS = D / 32;                  // products of 32 dimensions
  constexpr int DT = D / 16;                  // tiles of 16 dimensions
  __shared__ float ml[kAttWaves][2][16 * R];
  __shared__ f32x4 oo[kAttWaves / 2][DT * R][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int g = lane >> 4, col = lane & 15;
  int id = blockIdx.x;
  const int split = id % plan.splits;
  id /= plan.splits;
  const int tile = id % plan.tiles;
  id /= plan.tiles;
  const int head = id % c.heads, seq = id / c.heads;
  const int G = a.q_heads / c.heads;
  const int per_page = c.page / kKvBlock;
  const Span sp = span_of(b, seq, G, tile, 16 * R, split, plan.splits, a.window, int64_t(b.table_cols) * c.page);
  if (sp.rows <= 0) return;

  // queries: row r is token r / G, head r % G of the group
  bf16x8 q[R][KS];
  int pos[R];                                 // position of the column's token; -1: sees nothing
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int local = 16 * r + col;
    const int row = tile * 16 * R + local;
    const int64_t t = int64_t(sp.row0) + row / G;
    const bool on = local < sp.rows && t < b.tokens;
    pos[r] = on ? sp.len - sp.fresh + row / G : -1;
    const uint16_t* p = a.q + (t * a.q_heads + head * G + row % G) * D;
#pragma unroll
    for (int s = 0; s < KS; ++s) {
      u32x4 v = {0u, 0u, 0u, 0u};
      if (on) v = *reinterpret_cast<const u32x4*>(p + 64 * (s / 2) + 16 * g + 8 * (s % 2));
      q[r][s] = __builtin_bit_cast(bf16x8, v);
    }
  }
  const int first_pos = sp.len - sp.fresh + tile * 16 * R / G;
  const int last_pos = sp.len - sp.fresh + (tile * 16 * R + sp.rows - 1) / G;

  f32x4 o[DT][R];
  float m[R], l[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    m[r] = kLow;
    l[r] = 0.f;
#pragma unroll
    for (int d = 0; d < DT; ++d) o[d][r] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float scale = a.scale * 1.44269504088896f;            // scores in powers of two
  const int last_block = (sp.len - 1) / kKvBlock;

  // a block's index in the cache; past the end of the sequence the last block stands in
  auto locate = [&](int block) {
    block = min(block, last_block);
    const int page = b.table[int64_t(seq) * b.table_cols + block / per_page];
    const int64_t inside = min(max(int64_t(page), int64_t(0)), c.pages - 1);
    return kv_block(inside, head, block % per_page, c.heads, per_page);
  };

  for (int ch = sp.begin + wave; ch < sp.end; ch += kAttWaves) {
    const int64_t kb = locate(4 * ch + (col >> 2)), vb = locate(4 * ch + g);
    u32x4 kc[4][D / 64], vc[DT];
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int s = 0; s < D / 64; ++s)
        kc[t][s] = *reinterpret_cast<const u32x4*>(c.k_codes + kb * (kKvBlock * D) + (4 * t + (col & 3)) * D + 64 * s +
                                                   16 * g);
#pragma unroll
    for (int d = 0; d < DT; ++d)
      vc[d] = *reinterpret_cast<const u32x4*>(c.v_codes + vb * (kKvBlock * D) + (16 * d + col) * kKvBlock);
    const float kf = exp2_of(c.k_exps[vb]) * scale, vf = exp2_of(c.v_exps[vb]);

    const int t0 = ch * kChunk + kKvBlock * g;                // first token of the lane's block
    if (ch * kChunk + kChunk > sp.len) {                      // codes past the end: anything, NaN too
      const int n = min(max(sp.len - t0, 0), kKvBlock);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const int k = min(max(n - 4 * w, 0), 4);
        const uint32_t keep = k == 4 ? 0xFFFFFFFFu : (1u << (8 * k)) - 1u;
#pragma unroll
        for (int d = 0; d < DT; ++d) vc[d][w] &= keep;
      }
    }
    // In a chunk that some row does not see in full, a NaN among the values must not reach the rows
    // that do not see it, and 0 NaN is NaN: such codes are taken out, and the rows that see
    // their token get a NaN score instead.
    const bool edge = ch * kChunk + kChunk - 1 > first_pos || (a.window > 0 && last_pos - ch * kChunk >= a.window);
    uint32_t bad[4] = {0u, 0u, 0u, 0u};                       // bit 8 i + 7 of word t: token 4 t + i of the block
    if (edge) {
#pragma unroll
      for (int w = 0; w < 4; ++w) {
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const uint32_t n = ((vc[d][w] & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;
          vc[d][w] &= ~((n >> 7) * 0xFFu);
          bad[w] |= n;
        }
#pragma unroll
        for (int i = 1; i < 16; i <<= 1) bad[w] |= uint32_t(__shfl_xor(int(bad[w]), i));
      }
    }
    f32x4 s[4][R];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
#pragma unroll
      for (int r = 0; r < R; ++r) s[t][r] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const bf16x8 ka = expand8(kc[t][k / 2][2 * (k % 2)], kc[t][k / 2][2 * (k % 2) + 1]);
#pragma unroll
        for (int r = 0; r < R; ++r) s[t][r] = mfma16(ka, q[r][k], s[t][r]);
      }
    }
    bf16x8 p[2][R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      float mx = -INFINITY;
#pragma unroll
      for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float x = s[t][r][i] * kf;
          if (edge) {
            const int tok = t0 + 4 * t + i;
            if ((bad[t] >> (8 * i + 7)) & 1u) x = NAN;
            if (tok > pos[r] || (a.window > 0 && pos[r] - tok >= a.window)) x = -INFINITY;
          }
          s[t][r][i] = x;
          mx = fmaxf(mx, x);
        }
      mx = fmaxf(mx, __shfl_xor(mx, 16));
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float mn = fmaxf(m[r], mx);
      if (__ballot(mn > m[r]) != 0) {
        const float f = __builtin_amdgcn_exp2f(m[r] - mn);
        l[r] *= f;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d][r] *= f;
        m[r] = mn;
      }
      float sum = 0.f;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float e0 = __builtin_amdgcn_exp2f(s[2 * h + i / 2][r][2 * (i % 2)] - mn);
          const float e1 = __builtin_amdgcn_exp2f(s[2 * h + i / 2][r][2 * (i % 2) + 1] - mn);
          sum += e0 + e1;
          w[i] = pack_bf16x2(e0 * vf, e1 * vf);
        }
        p[h][r] = __builtin_bit_cast(bf16x8, w);
      }
      l[r] += sum;
    }
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const bf16x8 va = expand8(vc[d][2 * h], vc[d][2 * h + 1]);
#pragma unroll
        for (int r = 0; r < R; ++r) o[d][r] = mfma16(va, p[h][r], o[d][r]);
      }
  }

  // join the wavefronts: all maxima and sums, then the outputs of half the waves at a time
#pragma unroll
  for (int r = 0; r < R; ++r) {
    l[r] += __shfl_xor(l[r], 16);
    l[r] += __shfl_xor(l[r], 32);
    if (g == 0) {
      ml[wave][0][16 * r + col] = m[r];
      ml[wave][1][16 * r + col] = l[r];
    }
  }
  __syncthreads();
  float total[R], top[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    top[r] = kLow;
#pragma unroll
    for (int w = 0; w < kAttWaves; ++w) top[r] = fmaxf(top[r], ml[w][0][16 * r + col]);
    total[r] = 0.f;
#pragma unroll
    for (int w = 0; w < kAttWaves; ++w)
      total[r] += ml[w][1][16 * r + col] * __builtin_amdgcn_exp2f(ml[w][0][16 * r + col] - top[r]);
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
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const int local = 16 * r + col;
    if (local >= sp.rows) continue;
    const int row = tile * 16 * R + local;
    const int64_t t = int64_t(sp.row0) + row / G;
    if (t >= b.tokens) continue;
    if (plan.splits == 1) {
      const float inv = total[r] > 0.f ? 1.0f / total[r] : (total[r] == 0.f ? 0.f : total[r]);
      uint16_t* out = a.out + (t * a.q_heads + head * G + row % G) * D + 4 * g;
#pragma unroll
      for (int d = 0; d < DT; ++d)
        *reinterpret_cast<u32x2*>(out + 16 * d) =
            u32x2{pack_bf16x2(o[d][r][0] * inv, o[d][r][1] * inv), pack_bf16x2(o[d][r][2] * inv, o[d][r][3] * inv)};
    } else {
      // [tile][split][row][D + 2]: the sums, then the maximum and the sum of the softmax
      float* part = a.ws + ((int64_t(blockIdx.x)) * (16 * R) + local) * (D + 4);
#pragma unroll
      for (int d = 0; d < DT; ++d) *reinterpret_cast<f32x4*>(part + 16 * d + 4 * g) = o[d][r];
      if (g == 0) {
        part[D] = top[r];
        part[D + 1] = total[r];
      }
    }
  }
}

// Joins the parts of each row: one wavefront a row.
template <int D>
__global__ __launch_bounds__(256) void kv8_join_kernel(Kv8Cache c, Kv8Batch b, Kv8Attend a, Kv8Plan plan) {
  const int lane = threadIdx.x & 63;
  const int64_t unit = (int64_t(blockIdx.x) * 256 + threadIdx.x) / 64;
  const int local = int(unit % plan.rows);
  int64_t id = unit / plan.rows;
  const int64_t tile_id = id;
  const int tile = int(id % plan.tiles);
  id /= plan.tiles;
  const int head = int(id % c.heads);
  const int64_t seq = id / c.heads;
  if (seq >= b.sequences) return;
  const int G = a.q_heads / c.heads;
  const int row0 = b.cu[seq], fresh = b.cu[seq + 1] - row0;
  const int64_t row = int64_t(tile) * plan.rows + local;
  if (row >= int64_t(fresh) * G) return;
  const int64_t t = row0 + row / G;
  if (t >= b.tokens) return;
  const float* part = a.ws + (tile_id * plan.splits * plan.rows + local) * (D + 4);
  const int64_t stride = int64_t(plan.rows) * (D + 4);
  float top = kLow;
  for (int s = 0; s < plan.splits; ++s) top = fmaxf(top, part[s * stride + D]);
  constexpr int kPer = D / 64;
  float acc[kPer], total = 0.f;
#pragma unroll
  for (int i = 0; i < kPer; ++i) acc[i] = 0.f;
  for (int s = 0; s < plan.splits; ++s) {
    const float f = __builtin_amdgcn_exp2f(part[s * stride + D] - top);
    total += part[s * stride + D + 1] * f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) acc[i] += part[s * stride + lane * kPer + i] * f;
  }
  const float inv = total > 0.f ? 1.0f / total : (total == 0.f ? 0.f : total);
  uint16_t* out = a.out + (t * a.q_heads + head * G + row % G) * D + lane * kPer;
#pragma unroll
  for (int i = 0; i < kPer; ++i) out[i] = uint16_t(pack_bf16x2(acc[i] * inv, 0.f));
}

template <int D, int R>
hipError_t launch(const Kv8Cache& c, const Kv8Batch& b, const Kv8Attend& a, const Kv8Plan& p, hipStream_t s) {
  const int64_t tiles = int64_t(b.sequences) * c.heads * p.tiles;
  MOE_LAUNCH("kv8_attention", (kv8_attention_kernel<D, R>), dim3(unsigned(tiles * p.splits)), dim3(64 * kAttWaves), s,
             c, b, a, p);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess || p.splits == 1) return err;
  MOE_LAUNCH("kv8_join", (kv8_join_kernel<D>), dim3(unsigned((tiles * p.rows + 3) / 4)), dim3(256), s, c, b, a, p);
  return hipGetLastError();
}

template <int D>
hipError_t launch_rows(const Kv8Cache& c, const Kv8Batch& b, const Kv8Attend& a, const Kv8Plan& p, hipStream_t s) {
  if (p.rows == 16) return launch<D, 1>(c, b, a, p, s);
  if constexpr (D <= 128) {
    if (p.rows == 64) return launch<D, 4>(c, b, a, p, s);
  }
  return launch<D, 2>(c, b, a, p, s);
}

}  // namespace

Kv8Plan kv8_plan(int sequences, int q_heads, int heads, int dim, int max_new, int max_len, int64_t window, int num_cu) {
  Kv8Plan p;
  const int64_t rows = int64_t(max_new) * (q_heads / heads);
  p.rows = rows <= 16 ? 16 : rows <= 32 || dim > 128 ? 32 : 64;
  p.tiles = int((rows + p.rows - 1) / p.rows);
  // two workgroups a compute unit, and at least one chunk for each wavefront
  const int64_t tiles = int64_t(sequences) * heads * p.tiles;
  const int64_t seen = window > 0 ? std::min<int64_t>(max_len, window + max_new) : max_len;
  const int64_t chunks = (seen + kChunk - 1) / kChunk;
  const int64_t want = (2 * int64_t(num_cu) + tiles - 1) / std::max<int64_t>(tiles, 1);
  p.splits = int(std::max<int64_t>(1, std::min(want, chunks / kAttWaves)));
  return p;
}

size_t kv8_workspace_bytes(const Kv8Plan& p, int sequences, int heads, int dim) {
  if (p.splits <= 1) return 0;
  return size_t(sequences) * heads * p.tiles * p.splits * p.rows * (dim + 4) * sizeof(float);
}

hipError_t launch_kv8_attention(const Kv8Cache& c, const Kv8Batch& b, const Kv8Attend& a, const Kv8Plan& p,
                                hipStream_t s) {
  if (c.dim == 64) return launch_rows<64>(c, b, a, p, s);
  if (c.dim == 128) return launch_rows<128>(c, b, a, p, s);
  return launch_rows<256>(c, b, a, p, s);
}

}  // namespace moe
