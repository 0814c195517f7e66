// The whole MoE layer for at most 16 tokens in two kernels (gfx950): the step of the few
// sequences that a batch ends on.
//
// With so few tokens the layer is the read of the chosen experts' weights, each used for a
// handful of rows.  Grouping the rows, and a launch for each step, cost more than they save:
// the token index itself is the column of the matrix-core products (16 columns are what the
// 16 x 16 x 32 products have), and a token that did not choose the expert has a column of
// zeros.  No row is moved, and no map is built.
//
//   few_up    every workgroup selects all tokens' experts from the logits (16 x E values), lists
//             the experts that got a token, and computes 16 features of one of them:
//             h[t, j] = w_tj silu(Wg x_t) (Wu x_t), rounded to bf16.  The gate weight goes in here,
//             in fp32, before h is rounded: the second kernel is then one plain sum.
//   few_down  16 columns of y for all tokens: the sum over all listed experts of Wd h, along one
//             long k axis (expert after expert, the shared expert last), dealt to the
//             wavefronts of the workgroup, whose sums are added in LDS in their order.
//
// Weights are the A operand of the products and go straight from memory into the registers
// that the matrix cores read: nothing is shared between wavefronts, so nothing passes through LDS.
#include <algorithm>

#include "int4.h"
#include "moe_internal.h"

namespace moe {
namespace {

constexpr int kFewT = 16;             // tokens
constexpr int kFewWaves = 8;          // wavefronts of a workgroup
constexpr int kMaxPairs = kFewT * kMaxTopK;

// The experts that got a token, ascending, and which slot of each token is theirs.
struct Chosen {
  int n;                              // experts
  int16_t expert[kMaxPairs];
  int8_t slot[kMaxPairs][kFewT];      // -1: the token did not choose it
  int16_t ids[kFewT][kMaxTopK];
  float w[kFewT][kMaxTopK];
  int16_t place[kMaxExperts];
};

// Top-k of one token by one wavefront, as moe_route selects: larger logit first, equal ones to
// the lower expert.  Lane l holds experts l V .. l V + V - 1.
template <int V>
__device__ __forceinline__ void select(const float* __restrict__ logits, int E, int k, int renorm, int lane,
                                       int16_t* ids, float* w) {
  float l[V];
  uint32_t key[V];
#pragma unroll
  for (int v = 0; v < V; ++v) {
    const int e = lane * V + v;
    l[v] = e < E ? logits[e] : 0.f;
    // 0 marks what is taken or no expert: real keys are above it whatever the logit, so that
    // every round finds an expert
    key[v] = e < E ? max(orderable(l[v]), 1u) : 0u;
  }
  float lmax = 0.f, denom = 0.f, mine = 0.f;
  for (int j = 0; j < k; ++j) {
    uint32_t m = key[0];
#pragma unroll
    for (int v = 1; v < V; ++v) m = max(m, key[v]);
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) m = max(m, uint32_t(__shfl_xor(int(m), d)));
    int has = V;
#pragma unroll
    for (int v = V - 1; v >= 0; --v) has = key[v] == m ? v : has;
    const int owner = __builtin_ctzll(__ballot(has < V));
    const int v0 = __builtin_amdgcn_readlane(has, owner);
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (lane == owner && v == v0) key[v] = 0u;
    const float x = from_orderable(m);
    if (j == 0) lmax = x;
    const float p = expf(x - lmax);
    denom += p;                                               // slot order
    if (lane == j) mine = p;
    if (lane == 0) ids[j] = int16_t(owner * V + v0);
  }
  if (!renorm) {
    denom = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (lane * V + v < E) denom += expf(l[v] - lmax);
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) denom += __shfl_xor(denom, d);
  }
  if (lane < k) w[lane] = mine / denom;
}

// ch.ids (and ch.w) are in place: lists the experts.  All threads of the workgroup call it.
__device__ __forceinline__ void list_experts(Chosen& ch, int T, int E, int k) {
  const int tid = threadIdx.x, lane = tid & 63;
  for (int e = tid; e < E; e += int(blockDim.x)) ch.place[e] = 0;
  __syncthreads();
  if (tid < T * k) ch.place[ch.ids[tid / k][tid % k]] = 1;
  __syncthreads();
  if (tid < kWave) {
    int n = 0;
    for (int e0 = 0; e0 < E; e0 += kWave) {
      const int e = e0 + lane;
      const bool on = e < E && ch.place[e] != 0;
      const uint64_t b = __ballot(on);
      const int a = n + __popcll(b & ((uint64_t(1) << lane) - 1));
      if (on) {
        ch.place[e] = int16_t(a);
        ch.expert[a] = int16_t(e);
      }
      n += __popcll(b);
    }
    if (lane == 0) ch.n = n;
  }
  __syncthreads();
  const int n = ch.n;
  for (int i = tid; i < n * kFewT; i += int(blockDim.x)) ch.slot[i / kFewT][i % kFewT] = -1;
  __syncthreads();
  if (tid < T * k) ch.slot[ch.place[ch.ids[tid / k][tid % k]]][tid / k] = int8_t(tid % k);
  __syncthreads();
}

__device__ __forceinline__ bf16x8 load_row8(const uint16_t* p, bool on) {
  u32x4 v = {0u, 0u, 0u, 0u};
  if (on) v = *reinterpret_cast<const u32x4*>(p);
  return __builtin_bit_cast(bf16x8, v);
}

__device__ __forceinline__ bf16x8 load_weight8(const uint16_t* p) {
  return __builtin_bit_cast(bf16x8, __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p)));
}

// Weights of one step along k: 64 columns of 16 bf16 rows, or a tile of 128 columns of 4-bit
// ones.  `mat` is the matrix (expert), `rt` its tile of 16 rows.
struct Bf16Weights {
  static constexpr int kCols = 64;
  static constexpr int kParts = 2;            // products of 32 columns
  const uint16_t* w;
  struct Step {
    bf16x8 a[kParts];
  };
  struct Sums {};
  __device__ __forceinline__ void load(Step& s, int mat, int rt, int64_t rows, int K, int kt, int lane) const {
    const uint16_t* p = w + (mat * rows + rt * 16 + (lane & 15)) * K + kt * kCols + 8 * (lane >> 4);
#pragma unroll
    for (int j = 0; j < kParts; ++j) s.a[j] = load_weight8(p + 32 * j);
  }
  static __device__ __forceinline__ void sums(Sums&, const bf16x8 (&)[kParts]) {}
  static __device__ __forceinline__ void add(f32x4& acc, const Step& s, const bf16x8 (&xb)[kParts], const Sums&) {
#pragma unroll
    for (int j = 0; j < kParts; ++j) acc = mfma16(s.a[j], xb[j], acc);
  }
};

template <int GPT, bool ZEROS>
struct Int4Weights {
  static constexpr int kCols = kInt4Cols;
  static constexpr int kParts = 4;
  const uint8_t* codes;
  const uint16_t* scales;
  const uint8_t* zeros;
  using Step = Int4Tile<GPT, ZEROS>;
  struct Sums {
    float x[GPT];
  };
  __device__ __forceinline__ void load(Step& s, int mat, int rt, int64_t rows, int K, int kt, int lane) const {
    int4_load(s, codes, scales, zeros, (mat * int4_row_tiles(rows) + rt) * int4_col_tiles(K) + kt, lane);
  }
  static __device__ __forceinline__ void sums(Sums& t, const bf16x8 (&xb)[kParts]) { int4_group_sums<GPT>(t.x, xb); }
  static __device__ __forceinline__ void add(f32x4& acc, const Step& s, const bf16x8 (&xb)[kParts], const Sums& t) {
    int4_accumulate<GPT, ZEROS>(acc, s, xb, t.x);
  }
};

// ------------------------------------------------------------------ gate, up and SwiGLU
// Unit u: 16 features of one listed expert (then of the shared one); KS wavefronts deal its k
// steps among themselves.  h: routed rows [T, k, F], then the shared expert's [T, Fs].
template <typename W, int KS, int V>
__global__ __launch_bounds__(64 * kFewWaves) void few_up_kernel(const uint16_t* __restrict__ x,
                                                                const float* __restrict__ logits, int T, int H, int E,
                                                                int k, int F, int Fs, int renorm, W wg, W wu, W sg,
                                                                W su, int32_t* __restrict__ ids,
                                                                float* __restrict__ wts, uint16_t* __restrict__ h) {
  constexpr int kUnits = kFewWaves / KS;
  __shared__ Chosen ch;
  __shared__ f32x4 part[KS > 1 ? kFewWaves : 1][2][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  for (int t = wave; t < T; t += kFewWaves) select<V>(logits + int64_t(t) * E, E, k, renorm, lane, ch.ids[t], ch.w[t]);
  __syncthreads();
  if (blockIdx.x == 0 && tid < T * k) {
    ids[tid] = ch.ids[tid / k][tid % k];
    wts[tid] = ch.w[tid / k][tid % k];
  }
  list_experts(ch, T, E, k);

  const int ks = wave % KS;
  const int u = int(blockIdx.x) * kUnits + wave / KS;
  const int per = F / 16;                      // units of an expert
  const int a = u / per;
  const bool shared = a >= ch.n;
  const int rt = shared ? u - ch.n * per : u % per;
  const bool on = !shared || rt < Fs / 16;
  const int col = lane & 15, g4 = lane >> 4;
  const int slot = !on || col >= T ? -1 : shared ? 0 : ch.slot[a][col];
  f32x4 ag = {0.f, 0.f, 0.f, 0.f}, au = ag;
  if (on) {
    const W& g = shared ? sg : wg;
    const W& up = shared ? su : wu;
    const int mat = shared ? 0 : ch.expert[a];
    const int64_t rows = shared ? Fs : F;
    const int steps = (H + W::kCols - 1) / W::kCols;
    const uint16_t* xr = x + int64_t(col) * H + 8 * g4;
    for (int s = ks; s < steps; s += KS) {
      typename W::Step wsg, wsu;
      g.load(wsg, mat, rt, rows, H, s, lane);
      up.load(wsu, mat, rt, rows, H, s, lane);
      bf16x8 xb[W::kParts];
#pragma unroll
      for (int j = 0; j < W::kParts; ++j) {
        const int k0 = s * W::kCols + 32 * j;
        xb[j] = load_row8(xr + k0, slot >= 0 && k0 + 8 * g4 < H);
      }
      typename W::Sums sums;
      W::sums(sums, xb);
      W::add(ag, wsg, xb, sums);
      W::add(au, wsu, xb, sums);
    }
  }
  if (KS > 1) {
    part[wave][0][lane] = ag;
    part[wave][1][lane] = au;
    __syncthreads();
    if (ks != 0) return;
#pragma unroll
    for (int i = 1; i < KS; ++i) {
      ag += part[wave + i][0][lane];
      au += part[wave + i][1][lane];
    }
  }
  if (slot < 0) return;
  const float w = shared ? 1.0f : ch.w[col][slot];
  float v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = w * silu(ag[i]) * au[i];
  uint16_t* out = (shared ? h + (int64_t(T) * k * F + int64_t(col) * Fs) : h + (int64_t(col) * k + slot) * F) +
                  rt * 16 + 4 * g4;
  *reinterpret_cast<u32x2*>(out) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
}

// ------------------------------------------------------------------ down and sum
// Workgroup b: columns 16 b .. 16 b + 15 of y.  The k axis is the listed experts' F columns one
// after the other, then the shared expert's Fs; wavefront w takes steps w, w + 8, ...
template <typename W>
__global__ __launch_bounds__(64 * kFewWaves) void few_down_kernel(const uint16_t* __restrict__ h,
                                                                  const int32_t* __restrict__ ids, int T, int H,
                                                                  int E, int k, int F, int Fs, W wd, W sd,
                                                                  uint16_t* __restrict__ y) {
  __shared__ Chosen ch;
  __shared__ f32x4 part[kFewWaves][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid < T * k) ch.ids[tid / k][tid % k] = int16_t(ids[tid]);
  __syncthreads();
  list_experts(ch, T, E, k);
  const int col = lane & 15, g4 = lane >> 4;
  const int rt = blockIdx.x;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  auto walk = [&](const W& w, int mat, int cols, int first, const uint16_t* row, bool on) {
    const int steps = (cols + W::kCols - 1) / W::kCols;
    for (int s = first; s < steps; s += kFewWaves) {
      typename W::Step ws;
      w.load(ws, mat, rt, H, cols, s, lane);
      bf16x8 xb[W::kParts];
#pragma unroll
      for (int j = 0; j < W::kParts; ++j) {
        const int k0 = s * W::kCols + 32 * j + 8 * g4;
        xb[j] = load_row8(row + k0, on && k0 < cols);
      }
      typename W::Sums sums;
      W::sums(sums, xb);
      W::add(acc, ws, xb, sums);
    }
  };
  const int steps = (F + W::kCols - 1) / W::kCols;
  const int n = ch.n;
  int first = wave;                           // of the wavefront's steps in the expert
  for (int a = 0; a < n; ++a) {
    const int slot = col < T ? ch.slot[a][col] : -1;
    walk(wd, ch.expert[a], F, first, h + (int64_t(col) * k + max(slot, 0)) * F, slot >= 0);
    first = (first - steps % kFewWaves + kFewWaves) % kFewWaves;
  }
  if (Fs) walk(sd, 0, Fs, first, h + (int64_t(T) * k * F + int64_t(col) * Fs), col < T);
  part[wave][lane] = acc;
  __syncthreads();
  if (wave != 0 || col >= T) return;
#pragma unroll
  for (int w = 1; w < kFewWaves; ++w) acc += part[w][lane];
  *reinterpret_cast<u32x2*>(y + int64_t(col) * H + rt * 16 + 4 * g4) =
      u32x2{pack_bf16x2(acc[0], acc[1]), pack_bf16x2(acc[2], acc[3])};
}

// Units of few_up at most: the experts that T tokens can choose, and the shared one.
int64_t up_units(int T, int E, int k, int F, int Fs) { return int64_t(std::min(T * k, E)) * (F / 16) + Fs / 16; }

template <typename W, int KS>
void up_ks(const FewShape& s, W wg, W wu, W sg, W su, hipStream_t stream) {
  const int64_t units = up_units(s.T, s.E, s.k, s.F, s.Fs);
  const dim3 grid(unsigned((units * KS + kFewWaves - 1) / kFewWaves)), block(64 * kFewWaves);
  if (s.E <= 64)
    MOE_LAUNCH("few_up", (few_up_kernel<W, KS, 1>), grid, block, stream, s.x, s.logits, s.T, s.H, s.E, s.k, s.F, s.Fs,
               s.renorm, wg, wu, sg, su, s.ids, s.wts, s.h);
  else
    MOE_LAUNCH("few_up", (few_up_kernel<W, KS, 4>), grid, block, stream, s.x, s.logits, s.T, s.H, s.E, s.k, s.F, s.Fs,
               s.renorm, wg, wu, sg, su, s.ids, s.wts, s.h);
}

template <typename W>
hipError_t launch(const FewShape& s, const W (&w)[6], hipStream_t stream) {
  up_ks<W, 8>(s, w[0], w[1], w[3], w[4], stream);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  MOE_LAUNCH("few_down", (few_down_kernel<W>), dim3(unsigned(s.H / 16)), dim3(64 * kFewWaves), stream, s.h, s.ids,
             s.T, s.H, s.E, s.k, s.F, s.Fs, w[2], w[5], s.y);
  return hipGetLastError();
}

template <int GPT, bool ZEROS>
hipError_t launch_int4(const FewShape& s, const Int4Ref (&w)[6], hipStream_t stream) {
  Int4Weights<GPT, ZEROS> v[6];
  for (int i = 0; i < 6; ++i) v[i] = {w[i].codes, w[i].scales, w[i].zeros};
  return launch(s, v, stream);
}

}  // namespace

hipError_t launch_few_bf16(const FewShape& s, const uint16_t* const (&w)[6], hipStream_t stream) {
  Bf16Weights v[6];
  for (int i = 0; i < 6; ++i) v[i].w = w[i];
  return launch(s, v, stream);
}

hipError_t launch_few_int4(const FewShape& s, const Int4Ref (&w)[6], int group, hipStream_t stream) {
  const bool z = w[0].zeros != nullptr;
  if (group == 32) return z ? launch_int4<4, true>(s, w, stream) : launch_int4<4, false>(s, w, stream);
  if (group == 64) return z ? launch_int4<2, true>(s, w, stream) : launch_int4<2, false>(s, w, stream);
  return z ? launch_int4<1, true>(s, w, stream) : launch_int4<1, false>(s, w, stream);
}

}  // namespace moe
