// moe_kv8_append: position rotation of queries and keys, and keys and values written into the
// paged 8-bit cache (gfx950).
//
// One workgroup owns one block of 16 tokens of one kv head that receives new tokens: nothing
// else writes there, so the block's exponent, the rescaling of what it holds and the new codes
// need no atomics.  Thread t holds eight neighbouring dimensions of one token: the maximum
// over the block's new tokens is one reduction, and each value is read once.
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
  u32x2 r;
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

__device__ __forceinline__ void load8(float (&v)[8], const uint16_t* p) {
  const u32x4 w = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[2 * i] = __uint_as_float(w[i] << 16);
    v[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}

// Dimensions d .. d + 7 of a head's row, rotated: pairs are (i, i + rot / 2), or (2 i, 2 i + 1)
// where interleaved.  Products and sums are rounded one by one (no fused multiply-add), so that
// the codes are those of the formula in fp32 whatever the compiler.
__device__ __forceinline__ void rotated8(float (&v)[8], const uint16_t* row, int d, const float* cs, int rot,
                                         int interleaved) {
#pragma clang fp contract(off)
  load8(v, row + d);
  if (d >= rot) return;
  const int half = rot / 2;
  if (interleaved) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float c = cs[d / 2 + i], s = cs[half + d / 2 + i];
      const float a = v[2 * i], b = v[2 * i + 1];
      const float ac = a * c, bs = b * s, as = a * s, bc = b * c;
      v[2 * i] = ac - bs;
      v[2 * i + 1] = as + bc;
    }
  } else {
    const bool low = d < half;
    float o[8];
    load8(o, row + (low ? d + half : d - half));
    const float* p = cs + (low ? d : d - half);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float c = p[i], s = p[half + i];
      const float own = v[i] * c, other = o[i] * s;
      v[i] = low ? own - other : other + own;
    }
  }
}

// Workgroup (slot, head).  Slots are handed out to sequences from their rows alone: sequence b
// gets those from cu[b] / 16 + 2 b on, which are always enough for the blocks that it touches.
template <int D>
__global__ __launch_bounds__(2 * D) void kv8_append_kernel(Kv8Cache c, Kv8Batch b, Kv8Append a) {
  constexpr int kPer = D / 8;                                 // threads of a token
  constexpr int kWavesHere = 2 * D / 64;
  __shared__ uint8_t vt[D][kKvBlock];
  __shared__ float red[2][kWavesHere];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int slot = blockIdx.x, head = blockIdx.y;
  // the last sequence whose slots begin at or before this one
  int before = 0;
  for (int s0 = 0; s0 < b.sequences; s0 += kWave) {
    const int s = s0 + lane;
    const uint64_t m = __ballot(s < b.sequences && b.cu[min(s, b.sequences - 1)] / kKvBlock + 2 * s <= slot);
    before += __popcll(m);
    if (m != ~uint64_t(0)) break;
  }
  const int seq = before - 1;
  if (seq < 0) return;
  const int row0 = b.cu[seq], fresh = b.cu[seq + 1] - row0;
  const int begin = b.lens[seq] - fresh;                      // position of the first new token
  const int first = max(begin, 0);                            // tokens before position 0 are not written
  const int blk = first / kKvBlock + (slot - (row0 / kKvBlock + 2 * seq));
  const int p = blk * kKvBlock + tid / kPer;                  // this thread's token
  const int d = tid % kPer * 8;
  if (blk * kKvBlock >= begin + fresh) return;
  const int per_page = c.page / kKvBlock;
  const int column = blk / per_page;
  if (column >= b.table_cols) return;
  const int64_t page = b.table[int64_t(seq) * b.table_cols + column];
  if (page < 0 || page >= c.pages) return;
  const int64_t at = kv_block(page, head, blk % per_page, c.heads, per_page);

  const int64_t row = int64_t(row0) + p - begin;
  const bool is_new = p >= first && p < begin + fresh && row < b.tokens;
  const bool is_old = p < first;                              // held before this call
  const float* cs = a.cos_sin + min(int64_t(max(p, 0)), a.positions - 1) * a.rot;
  float kv[8], vv[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) kv[i] = vv[i] = 0.f;
  if (is_new) {
    rotated8(kv, a.k + row * a.k_stride + int64_t(head) * D, d, cs, a.rot, a.interleaved);
    load8(vv, a.v + row * a.v_stride + int64_t(head) * D + d);
    const int G = a.q_heads / c.heads;
    for (int j = 0; j < G; ++j) {
      const int qh = head * G + j;
      float q[8];
      rotated8(q, a.q + row * a.q_stride + int64_t(qh) * D, d, cs, a.rot, a.interleaved);
      *reinterpret_cast<u32x4*>(a.q_out + (row * a.q_heads + qh) * D + d) =
          u32x4{pack_bf16x2(q[0], q[1]), pack_bf16x2(q[2], q[3]), pack_bf16x2(q[4], q[5]), pack_bf16x2(q[6], q[7])};
    }
  }
  float mk = 0.f, mv = 0.f;                                   // fmaxf passes over NaN
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    mk = fmaxf(mk, fabsf(kv[i]));
    mv = fmaxf(mv, fabsf(vv[i]));
  }
#pragma unroll
  for (int s = 1; s < kWave; s <<= 1) {
    mk = fmaxf(mk, __shfl_xor(mk, s));
    mv = fmaxf(mv, __shfl_xor(mv, s));
  }
  if (lane == 0) {
    red[0][wave] = mk;
    red[1][wave] = mv;
  }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < kWavesHere; ++w) {
    mk = fmaxf(mk, red[0][w]);
    mv = fmaxf(mv, red[1][w]);
  }
  int ek = kv_exponent(mk), ev = kv_exponent(mv);
  uint8_t* kc = c.k_codes + at * (kKvBlock * D) + (tid / kPer) * D + d;
  uint8_t* vc = c.v_codes + at * (kKvBlock * D);
  u32x2 kout = {0u, 0u}, vout = {0u, 0u};
  if (first > blk * kKvBlock) {                               // the block holds earlier tokens
    const int ok = int(c.k_exps[at]) - 127, ov = int(c.v_exps[at]) - 127;
    ek = max(ek, ok);
    ev = max(ev, ov);
    if (is_old) {
      float o[8];
      kout = *reinterpret_cast<const u32x2*>(kc);
      if (ek != ok) {
        kv_values(o, kout);
        kout = kv_codes(o, ek - ok);
      }
      u32x2 w;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t byte = vc[(d + i) * kKvBlock + tid / kPer];
        w[i / 4] = (i % 4 ? w[i / 4] : 0u) | (byte << (8 * (i % 4)));
      }
      vout = w;
      if (ev != ov) {
        kv_values(o, vout);
        vout = kv_codes(o, ev - ov);
      }
    }
  }
  if (is_new) {
    kout = kv_codes(kv, ek);
    vout = kv_codes(vv, ev);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) vt[d + i][tid / kPer] = uint8_t(vout[i / 4] >> (8 * (i % 4)));
  __syncthreads();                                            // also: every old byte has been read
  *reinterpret_cast<u32x2*>(kc) = kout;
  if (tid < D) reinterpret_cast<u32x4*>(vc)[tid] = reinterpret_cast<const u32x4*>(&vt[tid][0])[0];
  if (tid == 0) {
    c.k_exps[at] = uint8_t(ek + 127);
    c.v_exps[at] = uint8_t(ev + 127);
  }
}

}  // namespace

hipError_t launch_kv8_append(const Kv8Cache& c, const Kv8Batch& b, const Kv8Append& a, hipStream_t s) {
  const dim3 grid(unsigned(b.tokens / kKvBlock + 2 * b.sequences), unsigned(c.heads));
  if (c.dim == 64)
    MOE_LAUNCH("kv8_append", (kv8_append_kernel<64>), grid, dim3(128), s, c, b, a);
  else if (c.dim == 128)
    MOE_LAUNCH("kv8_append", (kv8_append_kernel<128>), grid, dim3(256), s, c, b, a);
  else
    MOE_LAUNCH("kv8_append", (kv8_append_kernel<256>), grid, dim3(512), s, c, b, a);
  return hipGetLastError();
}

}  // namespace moe
