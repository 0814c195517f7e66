// The whole MoE layer for at most 16 tokens in two or three kernels (gfx950): the step of the few
// sequences that a batch ends on.
//
// With so few tokens the layer is the read of the chosen experts' weights, each used for a
// handful of rows.  Grouping the rows, and a launch for each step, cost more than they save:
// the token index itself is the column of the matrix-core products (16 columns are what the
// 16 x 16 x 32 products have), and a token that did not choose the expert has a column of
// zeros.  No row is moved, and no map is built.
//
//   few_up    every workgroup selects all tokens' experts from the logits (16 x E values), lists
//             the experts that got a token, and computes units of 16 or 32 features of one:
//             h[t, j] = w_tj silu(Wg x_t) (Wu x_t).  The gate weight goes in here: the second
//             kernel is then one plain sum.
//   few_down  16 columns of y for all tokens: the sum over all listed experts of Wd h, along one
//             long k axis (expert after expert, the shared expert last), dealt to the
//             wavefronts of the workgroup, whose sums are added in LDS in their order.
//   few_join  where that axis is long and the columns are few, it is cut into parts of a workgroup
//             each; their sums, in fp32, are added in the parts' order.  (A last workgroup that
//             adds them behind a fence saves the launch, but the fences cost 42 -> 289 us.)
//
// h goes between the kernels as two bf16 numbers, the rounded value and the rounded rest (16
// significant bits), so that y carries one rounding to bf16, its own.  Up to eight tokens the rest
// takes the other eight columns of the same products; more tokens take a second product.
//
// Bound by the read of the weights (bf16: few_up and few_down of the Mixtral shape for one token 72 +
// 38 us, 705 MB at 6.5 TB/s launches included; DeepSeek shape, 8 tokens 355 + 181 us, at 6.9).  Weights
// therefore go from memory into the registers that the matrix cores read, each once, in whole
// cache lines, with steps of loads always in flight.  4 bits, 13 tokens of 4 x F 4096, H 4096, groups of 64 with
// zero points: 126 + 80 + 5 us, 1 GB at 4.9 TB/s: vector instructions (58% of the cycles) and
// matrix cores (26 to 44%) run beside the loads, none of them full.  The smallest layer (1 token, H 256)
// takes 6 + 5 us, launch, routing and the latencies of one step.
#include <algorithm>

#include "int4.h"
#include "moe_internal.h"

namespace moe {
namespace {

constexpr int kFewT = 16;             // tokens
constexpr int kUpWaves = 8;           // wavefronts of a workgroup of few_up
constexpr int kMaxPairs = kFewT * kMaxTopK;

// The experts that got a token, ascending, and which slot of each token is theirs.
struct Chosen {
  uint64_t mask[kMaxExperts / 64];
  int16_t expert[kMaxPairs];
  int8_t slot[kMaxPairs][kFewT];      // -1: the token did not choose it
  int16_t ids[kFewT][kMaxTopK];
  float w[kFewT][kMaxTopK];
};

// Maximum over the wavefront: inside the rows of 16 lanes by lane permutes, then over the rows.
template <int CTRL>
__device__ __forceinline__ uint32_t permuted(uint32_t v) {
  return uint32_t(__builtin_amdgcn_update_dpp(0, int(v), CTRL, 0xF, 0xF, false));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max(v, permuted<0xB1>(v));                          // quad_perm [1, 0, 3, 2]
  v = max(v, permuted<0x4E>(v));                          // quad_perm [2, 3, 0, 1]
  v = max(v, permuted<0x141>(v));                         // mirrored halves of a row
  v = max(v, permuted<0x140>(v));                         // mirrored row
  const uint32_t a = __builtin_amdgcn_readlane(v, 0), b = __builtin_amdgcn_readlane(v, 16);
  const uint32_t c = __builtin_amdgcn_readlane(v, 32), d = __builtin_amdgcn_readlane(v, 48);
  return max(max(a, b), max(c, d));
}

// Top-k of one token by one wavefront, as moe_route selects: larger logit first, equal ones to
// the lower expert.  Lane l holds experts l V .. l V + V - 1.
template <int V>
__device__ __forceinline__ void select(Chosen& ch, int t, const float* __restrict__ logits, int E, int k, int renorm,
                                       int lane) {
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
  int id = 0;
  for (int j = 0; j < k; ++j) {
    uint32_t m = key[0];
#pragma unroll
    for (int v = 1; v < V; ++v) m = max(m, key[v]);
    m = wave_max(m);
    int has = V;
#pragma unroll
    for (int v = V - 1; v >= 0; --v) has = key[v] == m ? v : has;
    const int owner = __builtin_ctzll(__ballot(has < V));
    const int v0 = V == 1 ? 0 : __builtin_amdgcn_readlane(has, owner);
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (lane == owner && v == v0) key[v] = 0u;
    const float x = from_orderable(m);
    if (j == 0) lmax = x;
    if (lane == j) {
      mine = x;
      id = owner * V + v0;
    }
  }
  mine = expf(mine - lmax);
  for (int j = 0; j < k; ++j) denom += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine), j));  // slot order
  if (!renorm) {
    denom = 0.f;
#pragma unroll
    for (int v = 0; v < V; ++v)
      if (lane * V + v < E) denom += expf(l[v] - lmax);
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) denom += __shfl_xor(denom, d);
  }
  if (lane < k) {
    ch.ids[t][lane] = int16_t(id);
    ch.w[t][lane] = mine / denom;
    atomicOr(reinterpret_cast<unsigned long long*>(&ch.mask[id >> 6]), 1ull << (id & 63));
  }
}

// Before and after the experts are in ch.ids and ch.mask, each between barriers of the caller's.
__device__ __forceinline__ void clear_list(Chosen& ch, int T, int E, int k) {
  const int tid = threadIdx.x;
  if (tid < kMaxExperts / 64) ch.mask[tid] = 0;
  const int most = min(T * k, E);
  for (int i = tid; i < most; i += int(blockDim.x)) *reinterpret_cast<u32x4*>(ch.slot[i]) = u32x4{~0u, ~0u, ~0u, ~0u};
}
__device__ __forceinline__ void fill_list(Chosen& ch, int T, int k) {
  const int tid = threadIdx.x;
  if (tid < T * k) {
    const int t = tid / k, j = tid - t * k;
    const int e = ch.ids[t][j];
    int a = __popcll(ch.mask[e >> 6] & ((uint64_t(1) << (e & 63)) - 1));
    for (int i = 0; i < (e >> 6); ++i) a += __popcll(ch.mask[i]);
    ch.slot[a][t] = int8_t(j);
    ch.expert[a] = int16_t(e);
  }
}
__device__ __forceinline__ int listed(const Chosen& ch) {
  int n = 0;
#pragma unroll
  for (int i = 0; i < kMaxExperts / 64; ++i) n += __popcll(ch.mask[i]);
  return __builtin_amdgcn_readfirstlane(n);
}

// ------------------------------------------------------------------ gate, up and SwiGLU
// Unit u: 16 NU features of one listed expert, or of the shared one after them.  Workgroups take units in
// turn; the wavefronts of one deal a unit's k steps among themselves and add their sums in LDS, in their
// order.  P steps of weights and PX of activations are in flight, across units too: those of the next
// one load while a unit's sums are joined.  C operands hold the tokens' activations.  h: routed rows
// [T, k][2][F], then the shared expert's [T][2][Fs].
template <typename W, int NU, int C, int V, int P, int PX>
__global__ __launch_bounds__(64 * kUpWaves, 4) void few_up_kernel(const uint16_t* __restrict__ x,
                                                                  const float* __restrict__ logits, int T, int H,
                                                                  int E, int k, int F, int Fs, int renorm, W wg, W wu,
                                                                  W sg, W su, int32_t* __restrict__ ids,
                                                                  float* __restrict__ wts, uint16_t* __restrict__ h) {
  constexpr int kAcc = W::kAcc, kSums = NU * 2 * C * kAcc;
  __shared__ Chosen ch;
  __shared__ f32x4 part[kUpWaves][kSums][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  clear_list(ch, T, E, k);
  __syncthreads();
  for (int t = wave; t < T; t += kUpWaves) select<V>(ch, t, logits + int64_t(t) * E, E, k, renorm, lane);
  __syncthreads();
  fill_list(ch, T, k);
  if (blockIdx.x == 0 && tid < T * k) {
    ids[tid] = ch.ids[tid / k][tid % k];
    wts[tid] = ch.w[tid / k][tid % k];
  }
  __syncthreads();

  const int n = listed(ch);
  const int per = F / (16 * NU);               // units of an expert
  const int units = n * per + Fs / (16 * NU);
  const int steps = (H + W::kCols - 1) / W::kCols;
  const int mine = ((steps + kUpWaves - 1) / kUpWaves + P - 1) / P * P;   // a wavefront's steps of a unit
  const auto bx = buffer_of(x, int64_t(T) * H * 2);

  // A wavefront's place: step i of unit u.  Units start at different columns: their rows lie at equal
  // distances, and the same column of all rows in flight would ask the same few memory channels.
  struct Step {
    int u, i, a, rt, turn;
  };
  auto enter = [&](Step& p) {
    p.a = p.u / per;
    if (p.a > n) p.a = n;
    p.rt = p.u - p.a * per;
    p.turn = p.u * 5 % steps;
  };
  auto advance = [&](Step& p) {
    if (++p.i < mine) return false;
    p.i = 0;
    p.u += int(gridDim.x);
    enter(p);
    return true;
  };
  auto at = [&](const Step& p) {
    const int s = wave + p.i * kUpWaves + p.turn;
    return s >= steps ? s - steps : s;
  };
  auto on = [&](const Step& p) { return p.u < units && wave + p.i * kUpWaves < steps; };

  typename W::View vg, vu;                     // of the unit that loads weights
  auto view = [&](const Step& p) {
    const bool shared = p.a >= n;
    const int mat = shared ? 0 : __builtin_amdgcn_readfirstlane(ch.expert[p.a]);
    const int64_t rows = shared ? Fs : F;
    vg = W::pick(shared, sg, wg).view(mat, rows, H, lane);
    vu = W::pick(shared, su, wu).view(mat, rows, H, lane);
  };
  int xat[C];                                  // of the unit that loads activations
  auto rows_of = [&](const Step& p) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int t = c * W::kTok + W::token(lane);
      const bool has = t < T && (p.a >= n || ch.slot[p.a][t] >= 0);
      xat[c] = has ? t * H * 2 + W::x_at(lane) : kPast;
    }
  };
  f32x4 acc[NU][2][C][kAcc];                   // gate and up
  f32x4* flat = &acc[0][0][0][0];
  typename W::Step wsg[P][NU], wsu[P][NU];
  u32x4 xb[PX][C][W::kXRegs];
  Step pw = {int(blockIdx.x), 0, 0, 0, 0}, px;
  if (pw.u >= units) return;
  enter(pw);
  px = pw;
  view(pw);
  rows_of(px);
  auto load_w = [&](int p) {
    const int s = at(pw);
    const bool o = on(pw);
#pragma unroll
    for (int r = 0; r < NU; ++r) {
      W::load(wsg[p][r], vg, pw.rt * NU + r, s, o);
      W::load(wsu[p][r], vu, pw.rt * NU + r, s, o);
    }
    if (advance(pw) && pw.u < units) view(pw);
  };
  auto load_x = [&](int p) {
#pragma unroll
    for (int c = 0; c < C; ++c) W::load_x(xb[p][c], bx, xat[c], at(px), H, on(px));
    if (advance(px) && px.u < units) rows_of(px);
  };
#pragma unroll
  for (int p = 0; p < P; ++p) {
    if (p < PX) load_x(p);
    load_w(p);
  }
  for (int u = int(blockIdx.x); u < units; u += int(gridDim.x)) {
#pragma unroll
    for (int q = 0; q < kSums; ++q) flat[q] = f32x4{0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < mine; i += P) {
#pragma unroll
      for (int p = 0; p < P; ++p) {
        typename W::template Sums<C> sums;
        W::template sums<C>(sums, xb[p % PX], lane);
#pragma unroll
        for (int r = 0; r < NU; ++r) {
          W::template add<C>(acc[r][0], wsg[p][r], xb[p % PX], sums);
          W::template add<C>(acc[r][1], wsu[p][r], xb[p % PX], sums);
        }
        load_x(p % PX);
        load_w(p);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
    __syncthreads();                           // the last unit's sums have been read
#pragma unroll
    for (int q = 0; q < kSums; ++q) part[wave][q][lane] = flat[q];
    __syncthreads();
    const int a = min(u / per, n), rt = u - a * per;
    const bool shared = a >= n;
    const int width = shared ? Fs : F;
    for (int o = wave; o < NU * C * kAcc; o += kUpWaves) {
      const int i = o % kAcc, c = o / kAcc % C, r2 = o / kAcc / C;
      const int qg = ((r2 * 2) * C + c) * kAcc + i, qu = qg + C * kAcc;
      f32x4 g = part[0][qg][lane], up = part[0][qu][lane];
#pragma unroll
      for (int w = 1; w < kUpWaves; ++w) {
        g += part[w][qg][lane];
        up += part[w][qu][lane];
      }
      g = W::finish(g);
      up = W::finish(up);
      const int t = c * W::kTok + W::token(lane);
      const int slot = t >= T ? -1 : shared ? 0 : ch.slot[a][t];
      if (slot < 0 || !W::holds(lane)) continue;
      const float w = shared ? 1.0f : ch.w[t][slot];
      float v[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) v[r] = w * silu(g[r]) * up[r];
      uint16_t* out = h + (shared ? int64_t(T) * k * F * 2 + int64_t(t) * 2 * Fs : (int64_t(t) * k + slot) * 2 * F) +
                      (rt * NU + r2) * 16 + W::row(i, lane);
      const u32x2 hi = {pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
      *reinterpret_cast<u32x2*>(out) = hi;
      // an h that rounds to infinity has an infinite or NaN rest, which would make the sum of both NaN: any finite
      // number will do (of NaN, med3 gives one of the bounds)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        v[r] = __builtin_amdgcn_fmed3f(v[r] - __uint_as_float(r & 1 ? hi[r / 2] & 0xFFFF0000u : hi[r / 2] << 16), -1e38f, 1e38f);
      *reinterpret_cast<u32x2*>(out + width) = u32x2{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3])};
    }
  }
}

// ------------------------------------------------------------------ down and sum
// A wavefront's place in the long k axis: step s of listed expert a (a = n: the shared expert).
template <typename W, int C>
struct Place {
  int a, s, steps, cols;
  typename W::View v;
  int xat[C];
};

// Workgroup (g, p): columns 16 NT g .. 16 NT g + 16 NT - 1 of y, part p of the k axis, which is the
// listed experts' F columns one after the other, then the shared expert's Fs.  All wavefronts of the
// parts deal its steps among themselves in turn.  Rows of h pass through the caches for every
// step, zeros included; NT tiles of weights share them.  TS operands hold the tokens, once with
// h's rounded values and once with the rests; FOLD: one operand of 16 columns holds up to eight
// tokens and their rests.
//
// One part writes y; several write their sums to `partial` [parts, T, H], for few_join.
template <typename W, int NT, int WAVES, int TS, bool FOLD, int P, int PX>
__global__ __launch_bounds__(64 * WAVES, 4) void few_down_kernel(const uint16_t* __restrict__ h,
                                                                 const int32_t* __restrict__ ids, int T, int H, int E,
                                                                 int k, int F, int Fs, int parts, W wd, W sd,
                                                                 float* __restrict__ partial,
                                                                 uint16_t* __restrict__ y) {
  constexpr int C = FOLD ? 1 : 2 * TS, kAcc = W::kAcc, kSums = NT * TS * kAcc;
  __shared__ Chosen ch;
  __shared__ f32x4 part[WAVES][kSums][64];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  clear_list(ch, T, E, k);
  __syncthreads();
  if (tid < T * k) {
    const int e = ids[tid];
    ch.ids[tid / k][tid % k] = int16_t(e);
    atomicOr(reinterpret_cast<unsigned long long*>(&ch.mask[e >> 6]), 1ull << (e & 63));
  }
  __syncthreads();
  fill_list(ch, T, k);
  __syncthreads();
  const int rg = blockIdx.x / parts, pt = blockIdx.x - rg * parts;
  const int n = listed(ch);
  const int fsteps = (F + W::kCols - 1) / W::kCols, ssteps = (Fs + W::kCols - 1) / W::kCols;
  const int total = n * fsteps + ssteps;
  const int stride = parts * WAVES, begin = pt * WAVES + wave;
  const int mine = (total - begin + stride - 1) / stride;
  const auto bh = buffer_of(h, int64_t(T) * (int64_t(k) * F + Fs) * 4);

  using At = Place<W, C>;
  auto enter = [&](At& p, int lane) {           // sets what goes with p.a
    const bool shared = p.a >= n;
    const int mat = shared ? 0 : __builtin_amdgcn_readfirstlane(ch.expert[p.a]);
    p.steps = shared ? ssteps : fsteps;
    p.cols = shared ? Fs : F;
    p.v = W::pick(shared, sd, wd).view(mat, H, p.cols, lane);
#pragma unroll
    for (int c = 0; c < C; ++c) {
      const int col = W::token(lane);
      const int t = FOLD ? col & 7 : (c >> 1) * W::kTok + col, rest = FOLD ? col >> 3 : c & 1;
      const int slot = t >= T ? -1 : shared ? 0 : ch.slot[p.a][t];
      const int row = shared ? T * k * F * 2 + (2 * t + rest) * Fs : ((t * k + slot) * 2 + rest) * F;
      p.xat[c] = slot >= 0 ? row * 2 + W::x_at(lane) : kPast;
    }
  };
  auto carry = [&](At& p) {                     // steps past the end of an expert belong to the next one,
    while (p.s >= p.steps) {                    // past the last one to the first
      p.s -= p.steps;
      p.a = p.a < n ? p.a + 1 : 0;
      p.steps = p.a < n ? fsteps : ssteps;
    }
  };
  auto advance = [&](At& p, int lane) {
    p.s += stride;
    if (p.s >= p.steps) {
      carry(p);
      enter(p, lane);
    }
  };
  auto start = [&](At& p, int lane) {
    p.a = 0;
    p.s = begin + rg * 5 % total;               // workgroups start at different columns, as in few_up
    p.steps = fsteps;                           // T, k >= 1: an expert is listed
    carry(p);
    enter(p, lane);
  };
  At pw, px;
  start(pw, lane);
  px = pw;

  f32x4 acc[NT][C][kAcc];
#pragma unroll
  for (int q = 0; q < NT * C * kAcc; ++q) (&acc[0][0][0])[q] = f32x4{0.f, 0.f, 0.f, 0.f};
  typename W::Step ws[P][NT];
  u32x4 xb[PX][C][W::kXRegs];
  auto load_w = [&](int p, int i) {
#pragma unroll
    for (int r = 0; r < NT; ++r) W::load(ws[p][r], pw.v, rg * NT + r, pw.s, i < mine);
    advance(pw, lane);
  };
  auto load_x = [&](int p, int i) {
#pragma unroll
    for (int c = 0; c < C; ++c) W::load_x(xb[p][c], bh, px.xat[c], px.s, px.cols, i < mine);
    advance(px, lane);
  };
#pragma unroll
  for (int p = 0; p < P; ++p) {
    if (p < PX) load_x(p, p);
    load_w(p, p);
  }
  for (int i = 0; i < mine; i += P) {
#pragma unroll
    for (int p = 0; p < P; ++p) {
      typename W::template Sums<C> sums;
      W::template sums<C>(sums, xb[p % PX], lane);
#pragma unroll
      for (int r = 0; r < NT; ++r) W::template add<C>(acc[r], ws[p][r], xb[p % PX], sums);
      load_x(p % PX, i + p + PX);
      load_w(p, i + p + P);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // A weight that is not finite times the zeros of a token that did not choose its expert is NaN.  Where a sum is
  // not finite the wavefront walks its steps again, tile by tile, and the tokens that did not choose a
  // step's expert keep their sums.  (In every step instead, sums and their copies spill.)
  float odd = 0.f;                              // 0, or NaN
#pragma unroll
  for (int q = 0; q < 4 * NT * C * kAcc; ++q) odd += 0.f * (&acc[0][0][0])[q / 4][q % 4];
  auto put = [&](int lane, int r, const f32x4 (&v)[C][kAcc]) {
#pragma unroll
    for (int q = 0; q < TS * kAcc; ++q) {
      const int i = q % kAcc, t = q / kAcc;
      part[wave][r * TS * kAcc + q][lane] = FOLD ? v[t][i] : v[2 * t][i] + v[(2 * t + 1) % C][i];
    }
  };
  if (__ballot(odd != 0.f) == 0) {
#pragma unroll
    for (int r = 0; r < NT; ++r) put(lane, r, acc[r]);
  } else {
    // the lane asked for anew: kept through the loop, what hangs on it costs registers there (4 bits, groups of
    // 32, 13 tokens of 4 x F 4096, H 4096: 91 -> 116 us)
    const int lane = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0));
#pragma unroll 1
    for (int r = 0; r < NT; ++r) {
      f32x4 sum[C][kAcc], next[C][kAcc];
#pragma unroll
      for (int q = 0; q < C * kAcc; ++q) (&sum[0][0])[q] = f32x4{0.f, 0.f, 0.f, 0.f};
      start(pw, lane);
#pragma unroll 1
      for (int i = 0; i < mine; ++i) {
        bool chose[C];
#pragma unroll
        for (int c = 0; c < C; ++c) {
          W::load_x(xb[0][c], bh, pw.xat[c], pw.s, pw.cols, true);
          chose[c] = pw.xat[c] != kPast;
        }
        W::load(ws[0][0], pw.v, rg * NT + r, pw.s, true);
        typename W::template Sums<C> sums;
        W::template sums<C>(sums, xb[0], lane);
#pragma unroll
        for (int q = 0; q < C * kAcc; ++q) (&next[0][0])[q] = (&sum[0][0])[q];
        W::template add<C>(next, ws[0][0], xb[0], sums);
#pragma unroll
        for (int q = 0; q < C * kAcc; ++q) (&sum[0][0])[q] = chose[q / kAcc] ? (&next[0][0])[q] : (&sum[0][0])[q];
        advance(pw, lane);
      }
      put(lane, r, sum);
    }
  }
  __syncthreads();
  for (int q = wave; q < kSums; q += WAVES) {
    f32x4 s = part[0][q][lane];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) s += part[w][q][lane];
    s = W::finish(s);
    if (FOLD) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] += __shfl_xor(s[i], 8);
    }
    const int t = q / kAcc % TS * W::kTok + W::token(lane);   // FOLD: T <= 8, the rests' columns are past it
    const int col = (rg * NT + q / kAcc / TS) * 16 + W::row(q % kAcc, lane);
    if (t >= T || !W::holds(lane)) continue;
    if (parts == 1)
      *reinterpret_cast<u32x2*>(y + int64_t(t) * H + col) = u32x2{pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3])};
    else
      *reinterpret_cast<f32x4*>(partial + (int64_t(pt) * T + t) * H + col) = s;
  }
}

// y = the parts' sums, in their order.
__global__ __launch_bounds__(256) void few_join_kernel(const float* __restrict__ partial, int parts, int64_t n4,
                                                       uint16_t* __restrict__ y) {
  const int64_t i = int64_t(blockIdx.x) * 256 + threadIdx.x;
  if (i >= n4) return;
  const f32x4* p = reinterpret_cast<const f32x4*>(partial) + i;
  f32x4 s = p[0];
  for (int q = 1; q < parts; ++q) s += p[q * n4];
  reinterpret_cast<u32x2*>(y)[i] = u32x2{pack_bf16x2(s[0], s[1]), pack_bf16x2(s[2], s[3])};
}

// Tiles of 16 rows that share a wavefront's activations (of each of gate and up in few_up), workgroups
// of few_up for a compute unit (as many as stay there: one for each unit, in turn as places come free,
// took 123 us for a bf16 layer of 64 experts of 2048 x 1024 and 16 tokens, 84 this way), and
// steps in flight: of weights and of activations.  kCut: steps of a wavefront from which the k axis is
// cut into parts.
template <typename W>
struct Shape;
template <>
struct Shape<Bf16Weights> {
  static constexpr int kUpTiles = 1, kUp = 2, kUpX = 2;
  static constexpr int kDownTiles = 1, kDownWaves = 8, kDown = 2, kDownX = 2, kCut = 24;
};
template <int GPT, bool ZEROS>
struct Shape<Int4Weights<GPT, ZEROS>> {
  static constexpr int kUpTiles = 2, kUp = 1, kUpX = 1;
  static constexpr int kDownTiles = 4, kDownWaves = 8, kDown = 1, kDownX = 1, kCut = 8;
};

template <typename W, int C>
void up_c(const FewShape& s, const W (&w)[6], int64_t units, hipStream_t stream) {
  using S = Shape<W>;
  const dim3 grid(unsigned(std::min<int64_t>(units, 2 * int64_t(s.num_cu)))), block(64 * kUpWaves);
  if (s.E <= 64)
    MOE_LAUNCH("few_up", (few_up_kernel<W, S::kUpTiles, C, 1, S::kUp, S::kUpX>), grid, block, stream, s.x, s.logits,
               s.T, s.H, s.E, s.k, s.F, s.Fs, s.renorm, w[0], w[1], w[3], w[4], s.ids, s.wts, s.h);
  else
    MOE_LAUNCH("few_up", (few_up_kernel<W, S::kUpTiles, C, 4, S::kUp, S::kUpX>), grid, block, stream, s.x, s.logits,
               s.T, s.H, s.E, s.k, s.F, s.Fs, s.renorm, w[0], w[1], w[3], w[4], s.ids, s.wts, s.h);
}

template <typename W, int NT, int TS, bool FOLD>
void down_c(const FewShape& s, const W (&w)[6], hipStream_t stream) {
  using S = Shape<W>;
  constexpr int kWaves = S::kDownWaves;
  static_assert(16 * NT <= kFewMaxCols, "workspace");
  const int groups = s.H / (16 * NT);
  // Where the columns do not give the compute units a workgroup each, the k axis is cut for two a unit
  // with still two steps for every wavefront, if that saves more than few_join costs, some 4 us (bf16, H
  // 1536, 8 tokens of 3 x F 11584: 251 us whole, 144 cut; H 2048, 1 token of 8 x F 1024: 17.2 and 14.8;
  // 4 bits, H 1984, 3 tokens of 5 x F 512: 16.6 and 10.9).
  const int64_t steps = int64_t(std::min(s.T * s.k, s.E)) * ((s.F + W::kCols - 1) / W::kCols) +
                        (s.Fs + W::kCols - 1) / W::kCols;
  const int64_t all = std::min<int64_t>(2 * int64_t(s.num_cu), kFewParts);
  const int64_t want = std::min<int64_t>({(all + groups - 1) / groups, kFewMostParts, steps / (2 * kWaves)});
  const bool cut = groups < s.num_cu * 3 / 4 && steps >= S::kCut * kWaves;
  const int parts = cut ? int(std::max<int64_t>(1, want)) : 1;
  MOE_LAUNCH("few_down", (few_down_kernel<W, NT, kWaves, TS, FOLD, S::kDown, S::kDownX>),
             dim3(unsigned(groups * parts)), dim3(64 * kWaves), stream, s.h, s.ids, s.T, s.H, s.E, s.k, s.F, s.Fs,
             parts, w[2], w[5], s.partial, s.y);
  if (parts == 1) return;
  const int64_t n4 = int64_t(s.T) * s.H / 4;
  MOE_LAUNCH("few_join", few_join_kernel, dim3(unsigned((n4 + 255) / 256)), dim3(256), stream, s.partial, parts, n4,
             s.y);
}

template <typename W>
hipError_t launch(const FewShape& s, const W (&w)[6], hipStream_t stream) {
  // units of few_up at most: the experts that T tokens can choose, and the shared one
  constexpr int kRows = 16 * Shape<W>::kUpTiles;
  const int64_t units = int64_t(std::min(s.T * s.k, s.E)) * (s.F / kRows) + s.Fs / kRows;
  if (s.T > W::kTok)
    up_c<W, (kFewT > W::kTok ? 2 : 1)>(s, w, units, stream);
  else
    up_c<W, 1>(s, w, units, stream);
  hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;
  constexpr bool kFold = W::kTok == kFewT;
  constexpr int kTiles = Shape<W>::kDownTiles;
  if (s.T > 8) {
    down_c<W, kTiles, kFewT / W::kTok, false>(s, w, stream);
    return hipGetLastError();
  }
  // bf16: two tiles share the rows of h where that still leaves three quarters of the compute units a
  // workgroup (DeepSeek shape, 8 tokens, H 7168: 216 us with one tile, 193 with two; Mixtral shape,
  // 1 token, H 4096: 38 and 61)
  if constexpr (W::kTok < kFewT) {
    if (s.H / 32 >= s.num_cu * 3 / 4) {
      down_c<W, 2, 1, kFold>(s, w, stream);
      return hipGetLastError();
    }
  }
  down_c<W, kTiles, 1, kFold>(s, w, stream);
  return hipGetLastError();
}

template <int GPT, bool ZEROS>
hipError_t launch_int4(const FewShape& s, const Int4Ref (&w)[6], hipStream_t stream) {
  Int4Weights<GPT, ZEROS> v[6];
  for (int i = 0; i < 6; ++i) v[i] = {w[i].codes, w[i].scales};
  return launch(s, v, stream);
}

}  // namespace

hipError_t launch_few_bf16(const FewShape& s, const uint16_t* const (&w)[6], hipStream_t stream) {
  Bf16Weights v[6];
  for (int i = 0; i < 6; ++i) v[i].w = w[i];
  return launch(s, v, stream);
}

hipError_t launch_few_int4(const FewShape& s, const Int4Ref (&w)[6], int group, bool zeros, hipStream_t stream) {
  if (group == 32) return zeros ? launch_int4<4, true>(s, w, stream) : launch_int4<4, false>(s, w, stream);
  if (group == 64) return zeros ? launch_int4<2, true>(s, w, stream) : launch_int4<2, false>(s, w, stream);
  return zeros ? launch_int4<1, true>(s, w, stream) : launch_int4<1, false>(s, w, stream);
}

}  // namespace moe
