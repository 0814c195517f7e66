// moe_norm_join on gfx950: what happens between two blocks of a layer, in one pass over the stream.
//
//   x' = x + alpha * gate * j,   j = norm(y) * (offset + w_post)  (or y)
//   z  = norm(x') * (offset + w_pre),   norm(v) = v / sqrt(mean(v^2) + eps)
//
// A workgroup keeps a row in registers: x, y (and a full gate) are read once, x' and z written once, and
// between them lie two sums over the row, of y^2 and of x'^2.  z is taken of x' before x' is rounded.
// Its 8-bit codes need no third pass: a row's codes are those of x' (offset + w_pre), whose largest
// magnitude is found along with the sum; the norm's factor goes into the scale alone.
#include <algorithm>

#include "int8.h"
#include "launch_rules.h"
#include "moe_internal.h"

namespace moe {
namespace {

// Eight elements of the stream as they are read.
template <bool F32>
struct Raw {
  u32x4 v[F32 ? 2 : 1];
  __device__ __forceinline__ void load(const void* row, int vec) {
    const u32x4* p = static_cast<const u32x4*>(row) + vec * (F32 ? 2 : 1);
#pragma unroll
    for (int i = 0; i < (F32 ? 2 : 1); ++i) v[i] = p[i];
  }
  __device__ __forceinline__ void values(float (&f)[8]) const {
    if (F32) {
#pragma unroll
      for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(v[F32 ? i >> 2 : 0][i & 3]);
    } else {
      unpack_bf16(v[0], f);
    }
  }
  static __device__ __forceinline__ void store(void* row, int vec, const float (&f)[8]) {
    u32x4* p = static_cast<u32x4*>(row) + vec * (F32 ? 2 : 1);
    if (F32) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        p[i] = u32x4{__float_as_uint(f[4 * i]), __float_as_uint(f[4 * i + 1]), __float_as_uint(f[4 * i + 2]),
                     __float_as_uint(f[4 * i + 3])};
    } else {
      p[0] = u32x4{pack_bf16x2(f[0], f[1]), pack_bf16x2(f[2], f[3]), pack_bf16x2(f[4], f[5]), pack_bf16x2(f[6], f[7])};
    }
  }
};

// Sum, and the largest of the magnitudes' bits, over a workgroup of NT threads.  `slot` is LDS that no
// thread still reads: calls take turns between two.
template <int NT>
__device__ __forceinline__ void block_sum(float& sum, uint32_t& top, float (*slot)[2]) {
#pragma unroll
  for (int d = 32; d >= 1; d >>= 1) {
    sum += __shfl_xor(sum, d);
    top = max(top, uint32_t(__shfl_xor(int(top), d)));
  }
  if (NT == kWave) return;
  if ((threadIdx.x & (kWave - 1)) == 0) {
    slot[threadIdx.x / kWave][0] = sum;
    slot[threadIdx.x / kWave][1] = __uint_as_float(top);
  }
  __syncthreads();
  sum = 0.f;
  top = 0u;
#pragma unroll
  for (int w = 0; w < NT / kWave; ++w) {
    sum += slot[w][0];
    top = max(top, __float_as_uint(slot[w][1]));
  }
}

// A workgroup walks rows; while it works on one, the next one's x and y are on their way.  Norm weights and a gate of
// the channels stay in registers (read again for each row, from the L2, they cost a third: 9001 x 7168 133 us
// against 102).  Rows of more than 16384 leave no registers for either, nor for the row ahead, and 8 to 40 registers of
// theirs spill.
//
// Bound by memory: 9001 x 7168 with a post norm (516 MB) 98 us, 5.3 TB/s (without the row ahead 102), with codes
// 85; with a full gate (645 MB), which is read once its row is worked on, 122, 5.3 TB/s; an f32 stream (774 MB) 150, 5.2
// TB/s.  2003 x 7168 24.6 (30.9); one row of 4096 3.3 us, the latency of a load, two sums and a store.  4000 x 32768 (1049
// MB) 228 us, 4.6 TB/s, f32 344; 520 rows of it 44, 3.1 TB/s: a row at a time, two rounds and the last 8 rows.
template <int NT, int V, bool F32, bool CODES>
__global__ __launch_bounds__(NT) void norm_join_kernel(NormJoin a) {
  constexpr int kElt = F32 ? 4 : 2;
  constexpr bool kRoom = NT * V <= 2048;
  __shared__ float s_part[4][NT / kWave][2];
  const int nvec = a.H / 8;
  const float per = 1.0f / float(a.H);
  const bool full = a.gate_kind == kGateFull, channel = a.gate_kind == kGateChannel;
  const char* const xs = static_cast<const char*>(a.x);
  auto weights = [&](const uint16_t* w, int vec) {
    const u32x4 zero = {0u, 0u, 0u, 0u};
    return vec < nvec && w != nullptr ? reinterpret_cast<const u32x4*>(w)[vec] : zero;
  };
  u32x4 w_post[V], w_pre[V], gate[V];
  if (kRoom) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int vec = int(threadIdx.x) + i * NT;
      w_post[i] = weights(a.w_post, vec);
      w_pre[i] = weights(a.w_pre, vec);
      if (channel) gate[i] = weights(a.gate, vec);
    }
  }
  // without weights the factors are 1
  const float post_add = a.w_post != nullptr ? a.offset : 1.0f, pre_add = a.w_pre != nullptr ? a.offset : 1.0f;
  Raw<F32> xr[V], xn[V];
  u32x4 yr[V], yn[V];
  auto fetch = [&](Raw<F32>(&x)[V], u32x4(&y)[V], int64_t r) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int vec = int(threadIdx.x) + i * NT;
      if (vec < nvec) {
        x[i].load(xs + r * a.x_stride * kElt, vec);
        if (a.y != nullptr) y[i] = reinterpret_cast<const u32x4*>(a.y + r * a.y_stride)[vec];
      }
    }
  };
  if (kRoom) fetch(xn, yn, blockIdx.x);
  int turn = 0;
  for (int64_t r = blockIdx.x; r < a.T; r += gridDim.x) {
    if (kRoom) {
#pragma unroll
      for (int i = 0; i < V; ++i) {
        xr[i] = xn[i];
        yr[i] = yn[i];
      }
      if (r + gridDim.x < a.T) fetch(xn, yn, r + gridDim.x);
    } else {
      fetch(xr, yr, r);
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int vec = int(threadIdx.x) + i * NT;
      if (full && vec < nvec) gate[i] = reinterpret_cast<const u32x4*>(a.gate + r * a.gate_stride)[vec];
      if (!kRoom && channel) gate[i] = weights(a.gate, vec);
    }
    float scale = a.alpha;
    if (a.gate_kind == kGateToken) {
      const float g = bf16_to_f32(a.gate[r * a.gate_stride]);
      scale *= a.sigmoid ? 1.0f / (1.0f + __expf(-g)) : g;
    }
    if (a.post) {
      float sum = 0.f;
      uint32_t none = 0u;
#pragma unroll
      for (int i = 0; i < V; ++i)
        if (int(threadIdx.x) + i * NT < nvec) {
          float f[8];
          unpack_bf16(yr[i], f);
#pragma unroll
          for (int k = 0; k < 8; ++k) sum = fmaf(f[k], f[k], sum);
        }
      block_sum<NT>(sum, none, s_part[turn]);
      scale *= rsqrtf(sum * per + a.eps);
    }
    float x[V][8];
    float sum = 0.f;
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int vec = int(threadIdx.x) + i * NT;
      if (vec >= nvec) continue;
      xr[i].values(x[i]);
      if (a.y != nullptr) {
        float f[8];
        unpack_bf16(yr[i], f);
        if (a.post) {
          float w[8];
          unpack_bf16(kRoom ? w_post[i] : weights(a.w_post, vec), w);
#pragma unroll
          for (int k = 0; k < 8; ++k) f[k] *= w[k] + post_add;
        }
        if (channel || full) {
          float g[8];
          unpack_bf16(gate[i], g);
#pragma unroll
          for (int k = 0; k < 8; ++k) f[k] *= a.sigmoid ? 1.0f / (1.0f + __expf(-g[k])) : g[k];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) x[i][k] = fmaf(scale, f[k], x[i][k]);
        Raw<F32>::store(static_cast<char*>(a.x_out) + r * a.x_out_stride * kElt, vec, x[i]);
      }
      float w[8];
      unpack_bf16(kRoom ? w_pre[i] : weights(a.w_pre, vec), w);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        sum = fmaf(x[i][k], x[i][k], sum);
        x[i][k] *= w[k] + pre_add;
        if (CODES) top = max(top, magnitude(x[i][k]));
      }
    }
    if (a.z != nullptr) {
      block_sum<NT>(sum, top, s_part[2 + turn]);
      const float inv = rsqrtf(sum * per + a.eps);
      const RowCodes codes(top);
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const int vec = int(threadIdx.x) + i * NT;
        if (vec >= nvec) continue;
        if (CODES) {
          *reinterpret_cast<u32x2*>(static_cast<int8_t*>(a.z) + r * a.H + vec * 8) = codes.pack(x[i]);
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) x[i][k] *= inv;
          Raw<false>::store(static_cast<uint16_t*>(a.z) + r * a.H, vec, x[i]);
        }
      }
      if (CODES && threadIdx.x == 0) a.z_scales[r] = codes.scale(inv);
    }
    turn ^= 1;
  }
}

// ------------------------------------------------------------------ rows to codes
// A row stays in registers between its largest magnitude and its codes: read once, written once.  Bound by memory:
// 8192 x 14336 (352 MB) 65.5 us, 5.4 TB/s; nine rows of 7168 3.3 us, the latency of a load, a maximum and a store.
template <int NT, int V>
__global__ __launch_bounds__(NT) void quantize_int8_kernel(const uint16_t* __restrict__ src, int64_t stride,
                                                           int64_t rows, int K, int8_t* __restrict__ codes,
                                                           float* __restrict__ scales) {
  __shared__ float s_part[2][NT / kWave][2];
  const int nvec = K / 8;
  int turn = 0;
  for (int64_t r = blockIdx.x; r < rows; r += gridDim.x) {
    u32x4 raw[V];
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int vec = int(threadIdx.x) + i * NT;
      if (vec < nvec) raw[i] = reinterpret_cast<const u32x4*>(src + r * stride)[vec];
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
      if (int(threadIdx.x) + i * NT >= nvec) continue;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        top = max(top, max((raw[i][k] << 16) & 0x7FFFFFFFu, raw[i][k] & 0x7FFF0000u));
    }
    float none = 0.f;
    block_sum<NT>(none, top, s_part[turn]);
    const RowCodes q(top);
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const int vec = int(threadIdx.x) + i * NT;
      if (vec >= nvec) continue;
      float f[8];
      unpack_bf16(raw[i], f);
      *reinterpret_cast<u32x2*>(codes + r * K + vec * 8) = q.pack(f);
    }
    if (threadIdx.x == 0) scales[r] = q.scale();
    turn ^= 1;
  }
}

template <int NT, int V>
void norm_join(const NormJoin& a, int grid, hipStream_t s) {
  if (a.f32) {
    if (a.codes)
      MOE_LAUNCH("norm_join", (norm_join_kernel<NT, V, true, true>), dim3(grid), dim3(NT), s, a);
    else
      MOE_LAUNCH("norm_join", (norm_join_kernel<NT, V, true, false>), dim3(grid), dim3(NT), s, a);
  } else if (a.codes) {
    MOE_LAUNCH("norm_join", (norm_join_kernel<NT, V, false, true>), dim3(grid), dim3(NT), s, a);
  } else {
    MOE_LAUNCH("norm_join", (norm_join_kernel<NT, V, false, false>), dim3(grid), dim3(NT), s, a);
  }
}

template <int NT, int V>
void quantize(const uint16_t* src, int64_t stride, int64_t rows, int K, int8_t* codes, float* scales, int grid,
              hipStream_t s) {
  MOE_LAUNCH("quantize_int8", (quantize_int8_kernel<NT, V>), dim3(grid), dim3(NT), s, src, stride, rows, K, codes,
             scales);
}

}  // namespace

// Of a launch, whatever the budget: under 2^32 threads.
constexpr int64_t kMostGroups = 1 << 21;

hipError_t launch_norm_join(const NormJoin& a, int num_cu, hipStream_t s) {
  const RowShape f = row_shape(a.H, a.T, num_cu);
  const int grid = int(std::min<int64_t>(std::min(a.T, kMostGroups), int64_t(num_cu) * row_groups(f)));
  switch (f.threads * 8 + f.vectors) {
    case 64 * 8 + 1: norm_join<64, 1>(a, grid, s); break;
    case 64 * 8 + 2: norm_join<64, 2>(a, grid, s); break;
    case 64 * 8 + 4: norm_join<64, 4>(a, grid, s); break;
    case 256 * 8 + 1: norm_join<256, 1>(a, grid, s); break;
    case 256 * 8 + 2: norm_join<256, 2>(a, grid, s); break;
    case 512 * 8 + 1: norm_join<512, 1>(a, grid, s); break;
    case 512 * 8 + 2: norm_join<512, 2>(a, grid, s); break;
    case 1024 * 8 + 1: norm_join<1024, 1>(a, grid, s); break;
    case 1024 * 8 + 2: norm_join<1024, 2>(a, grid, s); break;
    default: norm_join<1024, 4>(a, grid, s); break;
  }
  return hipGetLastError();
}

hipError_t launch_quantize_int8(const uint16_t* src, int64_t stride, int64_t rows, int K, int8_t* codes, float* scales,
                                int num_cu, hipStream_t s) {
  const RowShape f = row_shape(K, rows, num_cu);
  const int grid = int(std::min<int64_t>(std::min(rows, kMostGroups), int64_t(num_cu) * 2048 / f.threads));
  switch (f.threads * 32 + f.vectors) {
    case 64 * 32 + 1: quantize<64, 1>(src, stride, rows, K, codes, scales, grid, s); break;
    case 64 * 32 + 2: quantize<64, 2>(src, stride, rows, K, codes, scales, grid, s); break;
    case 64 * 32 + 4: quantize<64, 4>(src, stride, rows, K, codes, scales, grid, s); break;
    case 256 * 32 + 1: quantize<256, 1>(src, stride, rows, K, codes, scales, grid, s); break;
    case 256 * 32 + 2: quantize<256, 2>(src, stride, rows, K, codes, scales, grid, s); break;
    case 512 * 32 + 1: quantize<512, 1>(src, stride, rows, K, codes, scales, grid, s); break;
    case 512 * 32 + 2: quantize<512, 2>(src, stride, rows, K, codes, scales, grid, s); break;
    case 1024 * 32 + 1: quantize<1024, 1>(src, stride, rows, K, codes, scales, grid, s); break;
    case 1024 * 32 + 2: quantize<1024, 2>(src, stride, rows, K, codes, scales, grid, s); break;
    case 1024 * 32 + 4: quantize<1024, 4>(src, stride, rows, K, codes, scales, grid, s); break;
    default: quantize<1024, 16>(src, stride, rows, K, codes, scales, grid, s); break;
  }
  return hipGetLastError();
}

}  // namespace moe
