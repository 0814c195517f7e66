// Helpers of the kernels that read weights once, straight from memory into the registers of the
// matrix-core products (gfx950): products of 16 weight rows with up to 16 rows of activations.
//
// A wavefront keeps the loads of its next P steps along k in flight in registers.  Loads go
// through buffer descriptors: a lane's place inside a step is a vector offset that never changes, a
// step's place a scalar one, so that a step costs no vector arithmetic.  A load that is off has a
// descriptor of no bytes, which gives zeros and fetches nothing: the last rounds of the ring need no
// branch, and lanes without a row (whose offset lies past every buffer) no mask.
#pragma once
#include "common.h"

namespace moe {

// An offset past every buffer (they are kept under 2 GiB).
constexpr int kPast = int(0x80000000u);

constexpr int kCached = 0, kStream = 2;   // cache policy of a load: as usual, or read once

// A buffer as it is carried along; the descriptor is made at each load, of scalars.
struct Buffer {
  uint64_t base;
  uint32_t bytes;
  __device__ __forceinline__ __amdgpu_buffer_rsrc_t at(bool on) const {
    return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>(base), 0, on ? int(bytes) : 0, 0x00020000);
  }
};

__device__ __forceinline__ Buffer buffer_of(const void* p, int64_t bytes) {
  return {reinterpret_cast<uint64_t>(p), uint32_t(bytes)};
}

template <int POLICY>
__device__ __forceinline__ u32x4 load16(const Buffer& b, bool on, int lane_at, int at) {
  return __builtin_amdgcn_raw_buffer_load_b128(b.at(on), lane_at, at, POLICY);
}
template <int POLICY>
__device__ __forceinline__ uint32_t load4(const Buffer& b, bool on, int lane_at, int at) {
  return __builtin_amdgcn_raw_buffer_load_b32(b.at(on), lane_at, at, POLICY);
}
template <int POLICY>
__device__ __forceinline__ uint32_t load2(const Buffer& b, bool on, int lane_at, int at) {
  return __builtin_amdgcn_raw_buffer_load_b16(b.at(on), lane_at, at, POLICY);
}

__device__ __forceinline__ bf16x8 as_bf16(u32x4 v) { return __builtin_bit_cast(bf16x8, v); }

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Keeps a step's sums where they are written: the compiler moves them behind the loads that follow
// otherwise, with every operand of several steps alive.
__device__ __forceinline__ void keep(f32x4& v) {
  asm volatile("" : "+v"(v));
}

// One of two pointers.  By masks: a choice between kernel arguments becomes one between their addresses in
// scratch memory, and what is loaded from there no longer counts as the same for all lanes.
template <typename T>
__device__ __forceinline__ const T* pick_of(bool first, const T* a, const T* b) {
  const uint64_t m = first ? ~uint64_t(0) : 0;
  return reinterpret_cast<const T*>((reinterpret_cast<uint64_t>(a) & m) | (reinterpret_cast<uint64_t>(b) & ~m));
}

// Row-major bf16 weights [rows, K], K % 64 == 0: a step is 16 rows x 64 columns, loaded as two times 8
// rows x 128 bytes, whole cache lines.  The products have 16 rows, 32 columns along k and 16 columns
// of activations; here row m of the first operand is weight row m % 8 in the k half m / 8, and
// column n of the second is token n % 8 in the k half n / 8.  Of the 16 x 16 results the two 8 x 8
// squares on the diagonal are the sums of the two halves, the other two mean nothing.  Half the
// products are thrown away, which costs nothing: memory is what bounds these kernels.  With 16
// rows x 64 bytes to a load instead (a lane's row l % 16, its columns 8 (l / 16)) each line is
// asked for twice: the Mixtral-shaped layer's first kernel for one token took 90 us with streaming
// loads and 84 with cached ones, against 74 (DeepSeek shape, 8 tokens: 538 and 445, against 386).
struct Bf16Weights {
  static constexpr int kCols = 64;            // columns of a step
  static constexpr int kTok = 8;              // rows of activations that one operand holds
  static constexpr int kXRegs = 1;            // operands of activations of a step
  static constexpr int kAcc = 2;              // results of 16 rows: rows 0..7, rows 8..15
  const uint16_t* w;
  // A matrix: its bytes, those of a row, and the lane's place in a step.
  struct View {
    Buffer c;
    int row, lane_at;
  };
  struct Step {
    u32x4 a[2];
  };
  static __device__ __forceinline__ Bf16Weights pick(bool first, const Bf16Weights& a, const Bf16Weights& b) {
    return {pick_of(first, a.w, b.w)};
  }
  static __device__ __forceinline__ int chunk(int lane) { return (lane >> 4) + ((lane & 8) >> 1); }
  __device__ __forceinline__ View view(int mat, int64_t rows, int K, int lane) const {
    return {buffer_of(w + mat * rows * K, rows * K * 2), 2 * K, ((lane & 7) * K + 8 * chunk(lane)) * 2};
  }
  // Step s of row tile rt.
  static __device__ __forceinline__ void load(Step& t, const View& v, int rt, int s, bool on) {
    const int at = rt * 16 * v.row + s * (kCols * 2);
    t.a[0] = load16<kStream>(v.c, on, v.lane_at, at);
    t.a[1] = load16<kStream>(v.c, on, v.lane_at, at + 8 * v.row);
  }
  // A lane's row of activations, and where in it its operand begins (bytes).
  static __device__ __forceinline__ int token(int lane) { return lane & 7; }
  static __device__ __forceinline__ int x_at(int lane) { return 16 * chunk(lane); }
  static __device__ __forceinline__ void load_x(u32x4 (&x)[kXRegs], const Buffer& b, int lane_at, int s, int,
                                                bool on) {
    x[0] = load16<kCached>(b, on, lane_at, s * (kCols * 2));
  }
  template <int C>
  struct Sums {};
  template <int C>
  static __device__ __forceinline__ void sums(Sums<C>&, const u32x4 (&)[C][kXRegs], int) {}
  // acc += step . x for C operands of 8 rows of x each.
  template <int C>
  static __device__ __forceinline__ void add(f32x4 (&acc)[C][kAcc], const Step& s, const u32x4 (&xb)[C][kXRegs],
                                             const Sums<C>&) {
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
      for (int i = 0; i < kAcc; ++i) {
        acc[c][i] = mfma16(as_bf16(s.a[i]), as_bf16(xb[c][0]), acc[c][i]);
        keep(acc[c][i]);
      }
  }
  // Joins the halves of finished sums.  Result i of a lane that `holds` one is rows row(i, lane) + 0..3 of
  // token(lane).
  static __device__ __forceinline__ f32x4 finish(f32x4 v) {
#pragma unroll
    for (int r = 0; r < 4; ++r) v[r] += __shfl_xor(v[r], 40);
    return v;
  }
  static __device__ __forceinline__ bool holds(int lane) { return (lane & 40) == 0; }
  static __device__ __forceinline__ int row(int i, int lane) { return 8 * i + 4 * (lane >> 4); }
};

}  // namespace moe
