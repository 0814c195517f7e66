// moe_kv8_append: position rotation of queries and keys, and keys and values written into the
// paged 8-bit cache (gfx950).
//
// One workgroup owns one block of 16 tokens of one kv head that receives new tokens: nothing
// else writes there, so the block's exponent, the rescaling of what it holds and the new codes
// need no atomics.  One half of its threads has the keys, the other the values: a thread holds
// 16 dimensions of one token, both halves of its rotation pairs among them, so every value is
// read once and the block's largest is one reduction.  The same threads rotate the queries of
// the block's tokens, for all of which their angles are read once.
//
// Bound by memory for prompts: 116 us for 23 thousand tokens of 32 query and 8 kv heads of 128
// (524 MB, 4.5 TB/s; a large copy reaches 4.9).  Eight dimensions a thread, which reads every
// pair twice and the angles for each head, took 145 us; one query head loaded at a time 136.  A
// step's few tokens are bound by the launch and the chain lengths - page - rows: 7 us.
#include "kv8.h"
#include "mxfp8.h"

namespace moe {
namespace {

// Smallest s in [-127, 127] with amax <= 448 2^s; -127 for 0.  448 = 1.75 2^8.  Infinity counts as
// the largest finite value: its code saturates.
__device__ __forceinline__ int kv_exponent(float amax) {
  const uint32_t u = min(__float_as_uint(amax), 0x7F7FFFFFu);
  const int e = int(u >> 23);
  if (e == 0) return -127;                                    // zero and subnormal
  const int s = e - 127 - 8 + ((u & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return s < -127 ? -127 : s;
}

__device__ __forceinline__ float pow2(int s) {                // s <= 127; 0 below the normal range
  return s < -126 ? 0.f : __uint_as_float(uint32_t(s + 127) << 23);
}

// E4M3 codes of eight values times 2^-s, rounded to nearest even, saturated; NaN stays NaN.
__device__ __forceinline__ u32x2 kv_codes(const float (&v)[8], int s) {
  const float f = pow2(-s);                                   // s >= -127: 2^127 at most
  float c[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = v[i] * f;
    c[i] = x == x ? __builtin_amdgcn_fmed3f(x, -448.0f, 448.0f) : x;
  }
  u32x2 r = {0u, 0u};
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(c[4 * i], c[4 * i + 1], 0, false);
    r[i] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(c[4 * i + 2], c[4 * i + 3], w, true));
  }
  return r;
}

__device__ __forceinline__ void kv_values(float (&v)[8], u32x2 c) {
  typedef float f32x2 __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(int(c[i]), false);
    const f32x2 b = __builtin_amdgcn_cvt_pk_f32_fp8(int(c[i]), true);
    v[4 * i] = a[0]; v[4 * i + 1] = a[1]; v[4 * i + 2] = b[0]; v[4 * i + 3] = b[1];
  }
}

// The two runs of eight dimensions that thread t of a token's D / 16 holds: the halves of pairs
// (i, i + rot / 2) of the rotated dimensions and 16 neighbours beyond them, or 16 neighbours
// everywhere where pairs are (2 i, 2 i + 1).  rot is a multiple of 16.  angle: the first of the
// eight pairs' angles, or -1.
struct Runs {
  int a, b, angle;
};
template <bool INTERLEAVED>
__device__ __forceinline__ Runs runs_of(int t, int rot) {
  const int half = rot / 2;
  if constexpr (INTERLEAVED) return {16 * t, 16 * t + 8, 16 * t < rot ? 8 * t : -1};
  if (8 * t < half) return {8 * t, 8 * t + half, 8 * t};
  return {16 * t, 16 * t + 8, -1};
}

struct Raw {                                                  // 16 bf16
  u32x4 a, b;
};
__device__ __forceinline__ Raw load_runs(const uint16_t* row, const Runs& r) {   // read once: not kept in L2
  return {__builtin_nontemporal_load(reinterpret_cast<const u32x4*>(row + r.a)),
          __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(row + r.b))};
}

// Rotated values.  Products and sums are rounded one by one (no fused multiply-add), so that the
// codes are those of the formula in fp32 whatever the compiler.
template <bool INTERLEAVED>
__device__ __forceinline__ void rotated(float (&v)[16], const Raw& w, const float (&cs)[16], bool rotates) {
#pragma clang fp contract(off)
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w.a[i] << 16);
    v[2 * i + 1] = __uint_as_float(w.a[i] & 0xFFFF0000u);
    v[8 + 2 * i] = __uint_as_float(w.b[i] << 16);
    v[9 + 2 * i] = __uint_as_float(w.b[i] & 0xFFFF0000u);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int p = INTERLEAVED ? 2 * i : i, q = INTERLEAVED ? 2 * i + 1 : 8 + i;
    const float a = v[p], b = v[q];
    const float ac = a * cs[i], bs = b * cs[8 + i], as = a * cs[8 + i], bc = b * cs[i];
    const float x = ac - bs, y = as + bc;
    v[p] = rotates ? x : a;
    v[q] = rotates ? y : b;
  }
}

template <int kFrom>
__device__ __forceinline__ u32x4 pack8(const float (&v)[16]) {
  return u32x4{pack_bf16x2(v[kFrom], v[kFrom + 1]), pack_bf16x2(v[kFrom + 2], v[kFrom + 3]),
               pack_bf16x2(v[kFrom + 4], v[kFrom + 5]), pack_bf16x2(v[kFrom + 6], v[kFrom + 7])};
}

// Codes of eight values, and codes again of codes whose exponent grew by s.
template <int kFrom>
__device__ __forceinline__ u32x2 codes8(const float (&v)[16], int s) {
  const float w[8] = {v[kFrom], v[kFrom + 1], v[kFrom + 2], v[kFrom + 3],
                      v[kFrom + 4], v[kFrom + 5], v[kFrom + 6], v[kFrom + 7]};
  return kv_codes(w, s);
}
__device__ __forceinline__ u32x2 rescaled(u32x2 c, int s) {
  float v[8];
  kv_values(v, c);
  return kv_codes(v, s);
}

// Workgroup (slot, head).  Slots are handed out to sequences from their rows alone: sequence b
// gets those from cu[b] / 16 + 2 b on, which are always enough for the blocks that it touches.
template <int D, bool INTERLEAVED>
__global__ __launch_bounds__(2 * D) void kv8_append_kernel(Kv8Cache c, Kv8Batch b, Kv8Append a) {
  constexpr int kPer = D / 16;                                // threads of a token
  constexpr int kWaves = D / 64;                              // waves of a half
  constexpr int kQ = 2;                                       // query heads loaded at once
  __shared__ uint32_t vt[D][5];                               // a dimension's 16 tokens; 5: rows in different banks
  __shared__ float red[2 * kWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) >> 6);
  const int side = wave / kWaves;                             // 0 keys, 1 values
  const int tid = threadIdx.x % D;
  const int slot = blockIdx.x, head = blockIdx.y;
  // the last sequence whose slots begin at or before this one
  int seq = -1, row0 = 0, stop = 0, len = 0;
  for (int s0 = 0; s0 < b.sequences; s0 += kWave) {
    const int s = min(s0 + lane, b.sequences - 1);
    const int from = b.cu[s], to = b.cu[s + 1], n = b.lens[s];
    const uint64_t m = __ballot(s0 + lane < b.sequences && from / kKvBlock + 2 * s <= slot);
    if (m != 0) {
      const int last = 63 - __builtin_clzll(m);
      seq = s0 + last;
      row0 = __builtin_amdgcn_readlane(from, last);
      stop = __builtin_amdgcn_readlane(to, last);
      len = __builtin_amdgcn_readlane(n, last);
    }
    if (m != ~uint64_t(0)) break;
  }
  if (seq < 0 || stop <= row0) return;                        // a sequence without rows is left as it is
  const int begin = len - (stop - row0);                      // position of the first new token
  const int first = max(begin, 0);                            // tokens before position 0 are not written
  const int blk = first / kKvBlock + (slot - (row0 / kKvBlock + 2 * seq));
  const int p0 = blk * kKvBlock;                              // position of the block
  if (p0 >= len) return;
  const int per_page = c.page / kKvBlock;
  const int column = blk / per_page;
  const int64_t page = column < b.table_cols ? b.table[int64_t(seq) * b.table_cols + column] : -1;
  const bool held = page >= 0 && page < c.pages;              // otherwise only queries are written
  const int64_t at = kv_block(held ? page : 0, head, blk % per_page, c.heads, per_page);

  const int fresh0 = max(first - p0, 0), fresh1 = min(len - p0, kKvBlock);   // the new tokens' places in the block
  const int place = tid / kPer;
  const int64_t row = int64_t(row0) + p0 - begin + place;
  const bool is_new = place >= fresh0 && place < fresh1 && uint64_t(row) < uint64_t(b.tokens);
  const Runs r = runs_of<INTERLEAVED>(tid % kPer, a.rot);
  uint8_t* kc = c.k_codes + at * (kKvBlock * D) + place * D;
  u32x4* vc = reinterpret_cast<u32x4*>(c.v_codes + at * (kKvBlock * D)) + tid;
  uint8_t* exps = (side == 0 ? c.k_exps : c.v_exps) + at;
  u32x4 old = {0u, 0u, 0u, 0u};                               // this token's codes; one dimension's of all 16 tokens
  int old_e = -127;
  if (held && fresh0 > 0) {                                   // the block holds earlier tokens
    old_e = int(*exps) - 127;
    if (side == 1) {
      old = *vc;
    } else if (place < fresh0) {
      const u32x2 lo = *reinterpret_cast<const u32x2*>(kc + r.a), hi = *reinterpret_cast<const u32x2*>(kc + r.b);
      old = u32x4{lo[0], lo[1], hi[0], hi[1]};
    }
  }
  float x[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) x[i] = 0.f;
  if (is_new) {
    const int G = a.q_heads / c.heads;
    const uint16_t* q = a.q + row * a.q_stride + int64_t(head) * G * D;
    uint16_t* qo = a.q_out + (row * a.q_heads + int64_t(head) * G) * D;
    Raw w[kQ];
#pragma unroll
    for (int i = 0; i < kQ; ++i) w[i] = load_runs(q + min(side + 2 * i, G - 1) * D, r);
    const Raw own = load_runs((side == 0 ? a.k + row * a.k_stride : a.v + row * a.v_stride) + int64_t(head) * D, r);
    float cs[16];
#pragma unroll
    for (int i = 0; i < 16; ++i) cs[i] = 0.f;
    const bool rotates = r.angle >= 0;
    if (rotates) {
      const float* p = a.cos_sin + min(int64_t(p0 + place), a.positions - 1) * a.rot + r.angle;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        cs[i] = p[i];
        cs[8 + i] = p[a.rot / 2 + i];
      }
    }
    rotated<INTERLEAVED>(x, own, cs, rotates && side == 0);
    for (int j = side; j < G; j += 2 * kQ) {
      if (j != side) {
#pragma unroll
        for (int i = 0; i < kQ; ++i) w[i] = load_runs(q + min(j + 2 * i, G - 1) * D, r);
      }
#pragma unroll
      for (int i = 0; i < kQ; ++i) {
        if (j + 2 * i >= G) break;
        float y[16];
        rotated<INTERLEAVED>(y, w[i], cs, rotates);
        *reinterpret_cast<u32x4*>(qo + (j + 2 * i) * D + r.a) = pack8<0>(y);
        *reinterpret_cast<u32x4*>(qo + (j + 2 * i) * D + r.b) = pack8<8>(y);
      }
    }
  }

  if (!held) return;                                          // all of the workgroup
  float m = 0.f;                                              // fmaxf passes over NaN
#pragma unroll
  for (int i = 0; i < 16; ++i) m = fmaxf(m, fabsf(x[i]));
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) m = fmaxf(m, __shfl_xor(m, s));
  if constexpr (kWaves > 1) {
    if (lane == 0) red[wave] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kWaves; ++i) m = fmaxf(m, red[side * kWaves + i]);
  }
  const int e = fresh0 > 0 ? max(kv_exponent(m), old_e) : kv_exponent(m);
  if (fresh0 > 0 && e != old_e) {
    const u32x2 lo = rescaled(u32x2{old[0], old[1]}, e - old_e), hi = rescaled(u32x2{old[2], old[3]}, e - old_e);
    old = u32x4{lo[0], lo[1], hi[0], hi[1]};
  }
  const u32x2 lo = codes8<0>(x, e), hi = codes8<8>(x, e);
  if (side == 0) {
    *reinterpret_cast<u32x2*>(kc + r.a) = is_new ? lo : u32x2{old[0], old[1]};
    *reinterpret_cast<u32x2*>(kc + r.b) = is_new ? hi : u32x2{old[2], old[3]};
  } else {
    uint8_t* col = reinterpret_cast<uint8_t*>(vt) + place;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      col[(r.a + i) * 20] = uint8_t(lo[i / 4] >> (8 * (i % 4)));
      col[(r.b + i) * 20] = uint8_t(hi[i / 4] >> (8 * (i % 4)));
    }
  }
  if (tid == 0) *exps = uint8_t(e + 127);
  __syncthreads();
  if (side == 1) {                                            // earlier tokens, new ones, zeros
    const auto below = [](int n) { return n <= 0 ? 0u : n >= 4 ? 0xFFFFFFFFu : (1u << (8 * n)) - 1u; };
    u32x4 out;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t held = below(fresh0 - 4 * i), upto = below(fresh1 - 4 * i);
      out[i] = (old[i] & held) | (vt[tid][i] & upto & ~held);
    }
    *vc = out;
  }
}

template <int D>
void launch(const Kv8Cache& c, const Kv8Batch& b, const Kv8Append& a, hipStream_t s) {
  const dim3 grid(unsigned(b.tokens / kKvBlock + 2 * b.sequences), unsigned(c.heads));
  if (a.interleaved)
    MOE_LAUNCH("kv8_append", (kv8_append_kernel<D, true>), grid, dim3(2 * D), s, c, b, a);
  else
    MOE_LAUNCH("kv8_append", (kv8_append_kernel<D, false>), grid, dim3(2 * D), s, c, b, a);
}

}  // namespace

hipError_t launch_kv8_append(const Kv8Cache& c, const Kv8Batch& b, const Kv8Append& a, hipStream_t s) {
  if (c.dim == 64)
    launch<64>(c, b, a, s);
  else if (c.dim == 128)
    launch<128>(c, b, a, s);
  else
    launch<256>(c, b, a, s);
  return hipGetLastError();
}

}  // namespace moe
