// C ABI of the MoE hot path (include/moe.h): validation, workspace carving,
// launches and error mapping.  No allocation, no synchronization.
#include <hip/hip_runtime.h>

#include <cstdio>
#include <atomic>
#include <mutex>
#include <string>

#include "../../include/moe.h"
#include "launch_rules.h"
#include "moe_internal.h"
#include "moe_validate.h"

namespace {

thread_local std::string g_last_error;

moe_status finish(const moe::Check& c) {
  g_last_error = c.msg;
  return c.status;
}

moe_status hip_status(const char* fn, hipError_t err) {
  if (err == hipSuccess) {
    g_last_error.clear();
    return MOE_OK;
  }
  g_last_error = std::string(fn) + ": " + hipGetErrorString(err);
  return MOE_ERR_HIP;
}

std::atomic<int> g_cu_budget{0};

// Compute units the persistent grids are sized for: the budget set with
// moe_set_cu_budget, else the current device's count (cached per device).
int cu_count(hipError_t* err) {
  const int budget = g_cu_budget.load(std::memory_order_relaxed);
  if (budget > 0) {
    *err = hipSuccess;
    return budget;
  }
  static std::mutex mu;
  static int cache[64] = {0};
  int dev = 0;
  *err = hipGetDevice(&dev);
  if (*err != hipSuccess) return 0;
  if (dev < 0 || dev >= 64) dev = 0;
  std::lock_guard<std::mutex> lock(mu);
  if (cache[dev] == 0) {
    int n = 0;
    *err = hipDeviceGetAttribute(&n, hipDeviceAttributeMultiprocessorCount, dev);
    if (*err != hipSuccess) return 0;
    cache[dev] = n > 0 ? n : 256;
  }
  return cache[dev];
}

hipStream_t stream_of(moe_stream s) { return reinterpret_cast<hipStream_t>(s); }

}  // namespace

namespace moe {
bool cu_budget_set() { return g_cu_budget.load(std::memory_order_relaxed) > 0; }
}  // namespace moe

extern "C" {

int moe_abi_version(void) { return MOE_ABI_VERSION; }

moe_status moe_set_cu_budget(int32_t n) {
  moe::Check c;
  if (n < 0) {
    c.status = MOE_ERR_INVALID_ARGUMENT;
    c.msg = "moe_set_cu_budget: n=" + std::to_string(n) + " is negative";
    return finish(c);
  }
  g_cu_budget.store(n, std::memory_order_relaxed);
  return finish(c);
}

const char* moe_status_string(int status) {
  switch (status) {
    case MOE_OK: return "MOE_OK";
    case MOE_ERR_INVALID_ARGUMENT: return "MOE_ERR_INVALID_ARGUMENT";
    case MOE_ERR_UNSUPPORTED: return "MOE_ERR_UNSUPPORTED";
    case MOE_ERR_WORKSPACE_TOO_SMALL: return "MOE_ERR_WORKSPACE_TOO_SMALL";
    case MOE_ERR_HIP: return "MOE_ERR_HIP";
    default: return "MOE_ERR_UNKNOWN_STATUS";
  }
}

const char* moe_last_error(void) { return g_last_error.c_str(); }

moe_status moe_route(const float* logits, int64_t T, int32_t E, int32_t k, int32_t renormalize,
                     int32_t* topk_ids, float* topk_weights, moe_stream stream) {
  moe::Check c = moe::validate_route(logits, T, E, k, renormalize, topk_ids, topk_weights);
  if (!c.ok() || T == 0) return finish(c);
  hipError_t err;
  const int ncu = cu_count(&err);
  if (err != hipSuccess) return hip_status("moe_route", err);
  return hip_status("moe_route",
                    moe::launch_route(logits, T, E, k, renormalize, topk_ids, topk_weights, ncu,
                                      stream_of(stream)));
}

moe_status moe_router_topk(const void* x, const void* w_router, int64_t T, int32_t E, int32_t k, int32_t H,
                           int32_t renormalize, float* logits, int32_t* topk_ids, float* topk_weights,
                           moe_stream stream) {
  moe::Check c = moe::validate_router_topk(x, w_router, T, E, k, H, renormalize, logits, topk_ids, topk_weights);
  if (!c.ok() || T == 0) return finish(c);
  hipError_t err;
  const int ncu = cu_count(&err);
  if (err != hipSuccess) return hip_status("moe_router_topk", err);
  return hip_status("moe_router_topk",
                    moe::launch_router_topk(static_cast<const uint16_t*>(x), static_cast<const uint16_t*>(w_router),
                                            T, E, k, H, renormalize, logits, topk_ids, topk_weights, ncu,
                                            stream_of(stream)));
}

size_t moe_permute_workspace_bytes(int64_t T, int32_t E, int32_t k) {
  return moe::permute_workspace_bytes(T, E, k);
}

moe_status moe_permute(const int32_t* topk_ids, const void* x, int64_t T, int32_t E, int32_t k,
                       int32_t H, moe_dtype dt, int32_t* expert_counts, int32_t* expert_offsets,
                       int32_t* sorted_token_ids, int32_t* dest_rows, void* x_perm, void* ws,
                       size_t ws_bytes, moe_stream stream) {
  moe::Check c = moe::validate_permute(topk_ids, x, T, E, k, H, dt, expert_counts, expert_offsets,
                                       sorted_token_ids, dest_rows, x_perm, ws, ws_bytes);
  if (!c.ok() || T == 0) return finish(c);
  const int64_t upad = (moe::permute_units(T * k) + 3) / 4 * 4;
  return hip_status("moe_permute",
                    moe::launch_permute(topk_ids, x, T, E, k, H, dt == MOE_DTYPE_F32 ? 4 : 2,
                                        expert_counts, expert_offsets, sorted_token_ids, dest_rows,
                                        x_perm, static_cast<int32_t*>(ws), upad, stream_of(stream)));
}

moe_status moe_permute_static(const int32_t* topk_ids, const void* x, int64_t T, int32_t E, int32_t k,
                              int32_t H, moe_dtype dt, int32_t* expert_counts, int32_t* expert_offsets,
                              int32_t* sorted_token_ids, int32_t* dest_rows, void* x_perm, moe_stream stream) {
  moe::Check c = moe::validate_permute_static(topk_ids, x, T, E, k, H, dt, expert_counts, expert_offsets,
                                              sorted_token_ids, dest_rows, x_perm);
  if (!c.ok() || T == 0) return finish(c);
  void* ws = nullptr;
  const hipError_t err = moe::permute_static_scratch(&ws);
  if (err != hipSuccess) return hip_status("moe_permute_static", err);
  const int64_t upad = (moe::permute_units(T * k) + 3) / 4 * 4;
  return hip_status("moe_permute_static",
                    moe::launch_permute(topk_ids, x, T, E, k, H, dt == MOE_DTYPE_F32 ? 4 : 2, expert_counts,
                                        expert_offsets, sorted_token_ids, dest_rows, x_perm,
                                        static_cast<int32_t*>(ws), upad, stream_of(stream)));
}

size_t moe_grouped_ffn_workspace_bytes(int64_t R, int32_t E, int32_t H, int32_t F, moe_dtype dt) {
  return moe::ffn_workspace_bytes(R, E, H, F, dt);
}

namespace {

moe_status run_ffn(const char* fn, const void* act, const int32_t* gather, int64_t T,
                   const int32_t* expert_offsets, int64_t R, int32_t E, int32_t H, int32_t F,
                   const void* w_gate, const void* w_up, const void* w_down, moe_dtype dt, void* y_perm,
                   void* ws, moe_stream stream) {
  auto* prefix = static_cast<int32_t*>(ws);
  auto* queues = reinterpret_cast<int32_t*>(static_cast<uint8_t*>(ws) + moe::ffn_queue_offset(E));
  void* h = static_cast<uint8_t*>(ws) + moe::ffn_h_offset(E);
  hipError_t err;
  const int ncu = cu_count(&err);
  if (err != hipSuccess) return hip_status(fn, err);
  if (dt == MOE_DTYPE_F32) {
    return hip_status(fn, moe::launch_ffn_f32(static_cast<const float*>(act), gather, expert_offsets, R, E,
                                              H, F, static_cast<const float*>(w_gate),
                                              static_cast<const float*>(w_up),
                                              static_cast<const float*>(w_down), static_cast<float*>(y_perm),
                                              static_cast<float*>(h), ncu, stream_of(stream)));
  }
  auto* partial = reinterpret_cast<float*>(static_cast<uint8_t*>(ws) + moe::ffn_partial_offset(R, E, F, dt));
  return hip_status(
      fn, moe::launch_ffn_bf16(static_cast<const uint16_t*>(act), gather, T, expert_offsets, R, E, H, F,
                               static_cast<const uint16_t*>(w_gate), static_cast<const uint16_t*>(w_up),
                               static_cast<const uint16_t*>(w_down), static_cast<uint16_t*>(y_perm), prefix,
                               queues, static_cast<uint16_t*>(h), partial, ncu, stream_of(stream)));
}

}  // namespace

moe_status moe_grouped_ffn(const void* x_perm, const int32_t* expert_offsets, int64_t R, int32_t E,
                           int32_t H, int32_t F, const void* w_gate, const void* w_up,
                           const void* w_down, moe_dtype dt, void* y_perm, void* ws,
                           size_t ws_bytes, moe_stream stream) {
  moe::Check c = moe::validate_ffn(x_perm, expert_offsets, R, E, H, F, w_gate, w_up, w_down, dt,
                                   y_perm, ws, ws_bytes);
  if (!c.ok() || R == 0) return finish(c);
  return run_ffn("moe_grouped_ffn", x_perm, nullptr, R, expert_offsets, R, E, H, F, w_gate, w_up, w_down,
                 dt, y_perm, ws, stream);
}

moe_status moe_grouped_ffn_gather(const void* x, const int32_t* sorted_token_ids,
                                  const int32_t* expert_offsets, int64_t T, int64_t R, int32_t E,
                                  int32_t H, int32_t F, const void* w_gate, const void* w_up,
                                  const void* w_down, moe_dtype dt, void* y_perm, void* ws,
                                  size_t ws_bytes, moe_stream stream) {
  moe::Check c = moe::validate_ffn_gather(x, sorted_token_ids, T, expert_offsets, R, E, H, F, w_gate,
                                          w_up, w_down, dt, y_perm, ws, ws_bytes);
  if (!c.ok() || R == 0) return finish(c);
  return run_ffn("moe_grouped_ffn_gather", x, sorted_token_ids, T, expert_offsets, R, E, H, F, w_gate,
                 w_up, w_down, dt, y_perm, ws, stream);
}

size_t moe_mxfp8_scale_bytes(int64_t rows, int32_t K) { return moe::mxfp8_scale_bytes(rows, K); }

moe_status moe_quantize_mxfp8(const void* src, const int32_t* row_map, int64_t rows_out, int64_t rows_src,
                              int32_t K, uint8_t* codes, uint8_t* scales, moe_stream stream) {
  moe::Check c = moe::validate_quantize_mxfp8(src, row_map, rows_out, rows_src, K, codes, scales);
  if (!c.ok() || rows_out == 0) return finish(c);
  hipError_t err;
  const int ncu = cu_count(&err);
  if (err != hipSuccess) return hip_status("moe_quantize_mxfp8", err);
  return hip_status("moe_quantize_mxfp8",
                    moe::launch_quantize_mxfp8(static_cast<const uint16_t*>(src), row_map, rows_out, K, codes,
                                               scales, ncu, stream_of(stream)));
}

size_t moe_grouped_ffn_mxfp8_workspace_bytes(int64_t R, int32_t E, int32_t H, int32_t F) {
  return moe::ffn_mxfp8_workspace_bytes(R, E, H, F);
}

namespace {

moe_status run_ffn_mxfp8(const char* fn, const uint8_t* x_codes, const uint8_t* x_scales, const int32_t* gather,
                         int64_t T, const int32_t* expert_offsets, int64_t R, int32_t E, int32_t H, int32_t F,
                         const uint8_t* wg_codes, const uint8_t* wg_scales, const uint8_t* wu_codes,
                         const uint8_t* wu_scales, const uint8_t* wd_codes, const uint8_t* wd_scales, void* y_perm,
                         void* ws, moe_stream stream) {
  hipError_t err;
  const int ncu = cu_count(&err);
  if (err != hipSuccess) return hip_status(fn, err);
  auto* base = static_cast<uint8_t*>(ws);
  auto* prefix = reinterpret_cast<int32_t*>(base);
  auto* queues = reinterpret_cast<int32_t*>(base + moe::ffn_queue_offset(E));
  uint8_t* h = base + moe::ffn_h_offset(E);
  uint8_t* hs = base + moe::ffn_mxfp8_h_scales_offset(R, E, F);
  auto* partial = reinterpret_cast<float*>(base + moe::ffn_mxfp8_partial_offset(R, E, F));
  return hip_status(fn, moe::launch_ffn_mxfp8(x_codes, x_scales, gather, T, expert_offsets, R, E, H, F, wg_codes,
                                              wg_scales, wu_codes, wu_scales, wd_codes, wd_scales,
                                              static_cast<uint16_t*>(y_perm), prefix, queues, h, hs, partial, ncu,
                                              stream_of(stream)));
}

}  // namespace

moe_status moe_grouped_ffn_mxfp8(const uint8_t* x_codes, const uint8_t* x_scales,
                                 const int32_t* expert_offsets, int64_t R, int32_t E, int32_t H, int32_t F,
                                 const uint8_t* wg_codes, const uint8_t* wg_scales, const uint8_t* wu_codes,
                                 const uint8_t* wu_scales, const uint8_t* wd_codes, const uint8_t* wd_scales,
                                 void* y_perm, void* ws, size_t ws_bytes, moe_stream stream) {
  moe::Check c = moe::validate_ffn_mxfp8(x_codes, x_scales, expert_offsets, R, E, H, F, wg_codes, wg_scales,
                                         wu_codes, wu_scales, wd_codes, wd_scales, y_perm, ws, ws_bytes);
  if (!c.ok() || R == 0) return finish(c);
  return run_ffn_mxfp8("moe_grouped_ffn_mxfp8", x_codes, x_scales, nullptr, R, expert_offsets, R, E, H, F,
                       wg_codes, wg_scales, wu_codes, wu_scales, wd_codes, wd_scales, y_perm, ws, stream);
}

moe_status moe_grouped_ffn_mxfp8_gather(const uint8_t* x_codes, const uint8_t* x_scales,
                                        const int32_t* sorted_token_ids, const int32_t* expert_offsets, int64_t T,
                                        int64_t R, int32_t E, int32_t H, int32_t F, const uint8_t* wg_codes,
                                        const uint8_t* wg_scales, const uint8_t* wu_codes,
                                        const uint8_t* wu_scales, const uint8_t* wd_codes,
                                        const uint8_t* wd_scales, void* y_perm, void* ws, size_t ws_bytes,
                                        moe_stream stream) {
  moe::Check c = moe::validate_ffn_mxfp8_gather(x_codes, x_scales, sorted_token_ids, T, expert_offsets, R, E, H,
                                                F, wg_codes, wg_scales, wu_codes, wu_scales, wd_codes, wd_scales,
                                                y_perm, ws, ws_bytes);
  if (!c.ok() || R == 0) return finish(c);
  return run_ffn_mxfp8("moe_grouped_ffn_mxfp8_gather", x_codes, x_scales, sorted_token_ids, T, expert_offsets, R,
                       E, H, F, wg_codes, wg_scales, wu_codes, wu_scales, wd_codes, wd_scales, y_perm, ws, stream);
}

moe_status moe_combine(const void* y_perm, const int32_t* dest_rows, const float* topk_weights,
                       const void* y_shared, int64_t T, int32_t k, int32_t H, moe_dtype dt, void* y,
                       moe_stream stream) {
  moe::Check c = moe::validate_combine(y_perm, dest_rows, topk_weights, y_shared, T, k, H, dt, y);
  if (!c.ok() || T == 0) return finish(c);
  return hip_status("moe_combine",
                    moe::launch_combine(y_perm, dest_rows, topk_weights, y_shared, T, k, H,
                                        dt == MOE_DTYPE_BF16, y, stream_of(stream)));
}

// ------------------------------------------------------------------ 4-bit weights
size_t moe_int4_code_bytes(int64_t rows, int32_t K) { return moe::int4_code_bytes(rows, K); }
size_t moe_int4_scale_bytes(int64_t rows, int32_t K, int32_t group, int32_t zeros) {
  return moe::int4_scale_bytes(rows, K, group, zeros);
}

moe_status moe_quantize_int4(const void* src, int64_t rows, int32_t K, int32_t group, uint8_t* codes,
                             uint16_t* scales, uint8_t* zeros, moe_stream stream) {
  moe::Check c = moe::validate_quantize_int4(src, rows, K, group, codes, scales, zeros);
  if (!c.ok() || rows == 0) return finish(c);
  return hip_status("moe_quantize_int4",
                    moe::launch_quantize_int4(static_cast<const uint16_t*>(src), rows * (K / group), group, codes,
                                              scales, zeros, stream_of(stream)));
}

moe_status moe_pack_int4(const uint8_t* codes, const uint16_t* scales, const uint8_t* zeros, int64_t matrices,
                         int64_t rows, int32_t K, int32_t group, uint8_t* out_codes, uint8_t* out_scales,
                         moe_stream stream) {
  moe::Check c = moe::validate_pack_int4(codes, scales, zeros, matrices, rows, K, group, out_codes, out_scales);
  if (!c.ok() || matrices == 0 || rows == 0) return finish(c);
  return hip_status("moe_pack_int4", moe::launch_pack_int4(codes, scales, zeros, matrices, rows, K, group, out_codes,
                                                           out_scales, stream_of(stream)));
}

moe_status moe_matvec_int4(const void* x, const uint8_t* codes, const uint8_t* scales, int32_t zeros, int64_t T,
                           int32_t N, int32_t K, int32_t group, void* y, moe_stream stream) {
  moe::Check c = moe::validate_matvec_int4(x, codes, scales, zeros, T, N, K, group, y);
  if (!c.ok() || T == 0) return finish(c);
  hipError_t err;
  const int ncu = cu_count(&err);
  if (err != hipSuccess) return hip_status("moe_matvec_int4", err);
  return hip_status("moe_matvec_int4",
                    moe::launch_matvec_int4(static_cast<const uint16_t*>(x), moe::Int4Ref{codes, scales}, int(T),
                                            N, K, group, zeros != 0, static_cast<uint16_t*>(y), ncu, stream_of(stream)));
}

// ------------------------------------------------------------------ the layer for few tokens
size_t moe_few_tokens_workspace_bytes(int64_t T, int32_t H, int32_t k, int32_t F, int32_t Fs) {
  return moe::few_workspace_bytes(T, H, k, F, Fs);
}

namespace {

moe::FewShape few_shape(const void* x, const float* logits, int64_t T, int32_t H, int32_t E, int32_t k, int32_t F,
                        int32_t Fs, int32_t renormalize, int32_t* ids, float* wts, void* ws, void* y, int ncu) {
  auto* base = static_cast<uint8_t*>(ws);
  return {static_cast<const uint16_t*>(x), logits, int(T), H, E, k, F, Fs, renormalize, ids, wts,
          reinterpret_cast<uint16_t*>(base), reinterpret_cast<float*>(base + moe::few_partial_offset(T, k, F, Fs)),
          static_cast<uint16_t*>(y), ncu};
}

}  // namespace

moe_status moe_few_tokens(const void* x, const float* logits, int64_t T, int32_t H, int32_t E, int32_t k, int32_t F,
                          int32_t Fs, int32_t renormalize, const void* w_gate, const void* w_up, const void* w_down,
                          const void* ws_gate, const void* ws_up, const void* ws_down, int32_t* topk_ids,
                          float* topk_weights, void* y, void* ws, size_t ws_bytes, moe_stream stream) {
  const void* const w[6] = {w_gate, w_up, w_down, ws_gate, ws_up, ws_down};
  moe::Check c = moe::validate_few(x, logits, T, H, E, k, F, Fs, renormalize, w, topk_ids, topk_weights, y, ws,
                                   ws_bytes);
  if (!c.ok() || T == 0) return finish(c);
  hipError_t err;
  const int ncu = cu_count(&err);
  if (err != hipSuccess) return hip_status("moe_few_tokens", err);
  const moe::FewShape s = few_shape(x, logits, T, H, E, k, F, Fs, renormalize, topk_ids, topk_weights, ws, y, ncu);
  const uint16_t* p[6];
  for (int i = 0; i < 6; ++i) p[i] = static_cast<const uint16_t*>(w[i]);
  return hip_status("moe_few_tokens", moe::launch_few_bf16(s, p, stream_of(stream)));
}

moe_status moe_few_tokens_int4(const void* x, const float* logits, int64_t T, int32_t H, int32_t E, int32_t k,
                               int32_t F, int32_t Fs, int32_t renormalize, int32_t group, int32_t zeros,
                               const moe_int4* weights,
                               int32_t* topk_ids, float* topk_weights, void* y, void* ws, size_t ws_bytes,
                               moe_stream stream) {
  moe::Check c = moe::validate_few_int4(x, logits, T, H, E, k, F, Fs, renormalize, group, zeros, weights, topk_ids,
                                        topk_weights, y, ws, ws_bytes);
  if (!c.ok() || T == 0) return finish(c);
  hipError_t err;
  const int ncu = cu_count(&err);
  if (err != hipSuccess) return hip_status("moe_few_tokens_int4", err);
  const moe::FewShape s = few_shape(x, logits, T, H, E, k, F, Fs, renormalize, topk_ids, topk_weights, ws, y, ncu);
  moe::Int4Ref p[6] = {};
  for (int i = 0; i < (Fs ? 6 : 3); ++i) p[i] = {weights[i].codes, weights[i].scales};
  return hip_status("moe_few_tokens_int4", moe::launch_few_int4(s, p, group, zeros != 0, stream_of(stream)));
}

// ------------------------------------------------------------------ the paged 8-bit cache
namespace {

moe::Kv8Cache cache_of(const moe_kv8_cache& c) {
  return {c.k_codes, c.v_codes, c.k_exps, c.v_exps, c.pages, c.page, c.heads, c.dim};
}

}  // namespace

moe_status moe_kv8_append(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                          int64_t v_stride, int64_t T, int32_t q_heads, const float* cos_sin, int64_t positions,
                          int32_t rot, int32_t interleaved, const moe_kv8_cache* cache, const int32_t* block_table,
                          int32_t table_cols, const int32_t* seq_lens, const int32_t* cu_tokens, int32_t B,
                          void* q_out, moe_stream stream) {
  moe::Check c = moe::validate_kv8_append(q, q_stride, k, k_stride, v, v_stride, T, q_heads, cos_sin, positions, rot,
                                          interleaved, cache, block_table, table_cols, seq_lens, cu_tokens, B, q_out);
  if (!c.ok() || T == 0) return finish(c);
  const moe::Kv8Batch b = {block_table, seq_lens, cu_tokens, B, table_cols, T};
  const moe::Kv8Append a = {static_cast<const uint16_t*>(q), static_cast<const uint16_t*>(k),
                            static_cast<const uint16_t*>(v), q_stride, k_stride, v_stride, cos_sin, positions, rot,
                            interleaved, q_heads, static_cast<uint16_t*>(q_out)};
  return hip_status("moe_kv8_append", moe::launch_kv8_append(cache_of(*cache), b, a, stream_of(stream)));
}

size_t moe_kv8_attention_workspace_bytes(int64_t T, int32_t B, int32_t q_heads, int32_t heads, int32_t dim, int32_t max_new,
                                         int32_t max_len, int32_t window) {
  if (T < 1 || T >= (1 << 24) || !moe::kv8_plan_sizes_ok(B, q_heads, heads, dim, max_new, max_len, window)) return 0;
  hipError_t err;
  const int ncu = cu_count(&err);
  if (err != hipSuccess) return 0;
  return moe::kv8_workspace_bytes(moe::kv8_plan(B, q_heads, heads, dim, max_new, max_len, window, ncu), T, B, q_heads,
                                  heads, dim);
}

moe_status moe_kv8_attention(const void* q, int64_t T, int32_t q_heads, const moe_kv8_cache* cache,
                             const int32_t* block_table, int32_t table_cols, const int32_t* seq_lens,
                             const int32_t* cu_tokens, int32_t B, int32_t max_new, int32_t max_len, int32_t window,
                             float scale, void* out, void* ws, size_t ws_bytes, moe_stream stream) {
  // the workspace's size depends on the device's compute units: looked at once all else is right
  const auto check = [&](size_t need) {
    return moe::validate_kv8_attention(q, T, q_heads, cache, block_table, table_cols, seq_lens, cu_tokens, B, max_new,
                                       max_len, window, scale, out, ws, ws_bytes, need);
  };
  moe::Check c = check(0);
  if (!c.ok() || T == 0) return finish(c);
  hipError_t err;
  const int ncu = cu_count(&err);
  if (err != hipSuccess) return hip_status("moe_kv8_attention", err);
  const moe::Kv8Plan plan = moe::kv8_plan(B, q_heads, cache->heads, cache->dim, max_new, max_len, window, ncu);
  c = check(moe::kv8_workspace_bytes(plan, T, B, q_heads, cache->heads, cache->dim));
  if (!c.ok()) return finish(c);
  const moe::Kv8Batch b = {block_table, seq_lens, cu_tokens, B, table_cols, T};
  const moe::Kv8Attend a = {static_cast<const uint16_t*>(q), q_heads, window, scale,
                            static_cast<uint16_t*>(out), static_cast<float*>(ws)};
  return hip_status("moe_kv8_attention", moe::launch_kv8_attention(cache_of(*cache), b, a, plan, stream_of(stream)));
}

// ------------------------------------------------------------------ the dense half in 8-bit integers
moe_status moe_norm_join(const void* x, int64_t x_stride, moe_dtype dt, const void* y, int64_t y_stride, int32_t post,
                         const void* w_post, const void* gate, int64_t gate_stride, int32_t gate_kind, int32_t sigmoid,
                         float alpha, const void* w_pre, float offset, float eps, int64_t T, int32_t H, void* x_out,
                         int64_t x_out_stride, int32_t z_codes, void* z, float* z_scales, moe_stream stream) {
  moe::Check c = moe::validate_norm_join(x, x_stride, dt, y, y_stride, post, w_post, gate, gate_stride, gate_kind,
                                         sigmoid, alpha, w_pre, offset, eps, T, H, x_out, x_out_stride, z_codes, z,
                                         z_scales);
  if (!c.ok() || T == 0) return finish(c);
  hipError_t err;
  const int ncu = cu_count(&err);
  if (err != hipSuccess) return hip_status("moe_norm_join", err);
  const moe::NormJoin a = {x, x_stride, dt == MOE_DTYPE_F32, static_cast<const uint16_t*>(y), y_stride, post != 0,
                           static_cast<const uint16_t*>(w_post), static_cast<const uint16_t*>(gate), gate_stride,
                           gate_kind, sigmoid != 0, alpha, static_cast<const uint16_t*>(w_pre), offset, eps, T, H,
                           x_out, x_out_stride, z_codes != 0, z, z_scales};
  return hip_status("moe_norm_join", moe::launch_norm_join(a, ncu, stream_of(stream)));
}

moe_status moe_quantize_int8(const void* src, int64_t src_stride, int64_t rows, int32_t K, int8_t* codes, float* scales,
                             moe_stream stream) {
  moe::Check c = moe::validate_quantize_int8(src, src_stride, rows, K, codes, scales);
  if (!c.ok() || rows == 0) return finish(c);
  hipError_t err;
  const int ncu = cu_count(&err);
  if (err != hipSuccess) return hip_status("moe_quantize_int8", err);
  return hip_status("moe_quantize_int8", moe::launch_quantize_int8(static_cast<const uint16_t*>(src), src_stride, rows, K,
                                                                   codes, scales, ncu, stream_of(stream)));
}

size_t moe_int8_code_bytes(int64_t rows, int32_t K) { return moe::int8_code_bytes(rows, K); }

moe_status moe_pack_int8(const int8_t* codes, int64_t rows, int32_t K, int8_t* out, moe_stream stream) {
  moe::Check c = moe::validate_pack_int8(codes, rows, K, out);
  if (!c.ok() || rows == 0) return finish(c);
  return hip_status("moe_pack_int8", moe::launch_pack_int8(codes, rows, K, out, stream_of(stream)));
}

namespace {

// The plan of a product, and the scratch that it needs.
hipError_t int8_plan_of(int64_t T, int32_t N, int32_t K, bool gated, moe::Int8Plan* plan, size_t* need) {
  hipError_t err;
  const int ncu = cu_count(&err);
  if (err != hipSuccess) return err;
  *plan = moe::int8_plan(T, N, K, gated, ncu);
  *need = plan->parts > 1 ? plan->parts * plan->part_bytes : 0;
  return err;
}

size_t int8_workspace_bytes(int64_t T, int32_t N, int32_t K, bool gated) {
  moe::Int8Plan plan;
  size_t need;
  if (!moe::int8_sizes_ok(T, N, K) || int8_plan_of(T, N, K, gated, &plan, &need) != hipSuccess) return 0;
  return need;
}

typedef int i32x4_t __attribute__((ext_vector_type(4)));

}  // namespace

size_t moe_matmul_int8_workspace_bytes(int64_t T, int32_t N, int32_t K) { return int8_workspace_bytes(T, N, K, false); }
size_t moe_gated_int8_workspace_bytes(int64_t T, int32_t F, int32_t K) { return int8_workspace_bytes(T, F, K, true); }

moe_status moe_matmul_int8(const int8_t* x, const float* x_scales, const int8_t* w, const float* w_scales,
                           const void* bias, int64_t T, int32_t N, int32_t K, void* y, void* ws, size_t ws_bytes,
                           moe_stream stream) {
  // the workspace's size depends on the device's compute units: looked at once all else is right
  moe::Check c = moe::validate_matmul_int8(x, x_scales, w, w_scales, bias, T, N, K, y);
  if (!c.ok() || T == 0) return finish(c);
  moe::Int8Plan plan;
  size_t need;
  const hipError_t err = int8_plan_of(T, N, K, false, &plan, &need);
  if (err != hipSuccess) return hip_status("moe_matmul_int8", err);
  c = moe::validate_int8_workspace("moe_matmul_int8", ws, ws_bytes, need);
  if (!c.ok()) return finish(c);
  const moe::Int8Product p = {x, x_scales, w, nullptr, w_scales, nullptr, static_cast<const uint16_t*>(bias),
                              static_cast<uint16_t*>(y), int(T), N, K, (K + 127) / 128 * 2, static_cast<i32x4_t*>(ws)};
  return hip_status("moe_matmul_int8", moe::launch_int8_product(p, plan, stream_of(stream)));
}

moe_status moe_gated_int8(const int8_t* x, const float* x_scales, const int8_t* wg, const float* wg_scales,
                          const int8_t* wu, const float* wu_scales, int64_t T, int32_t F, int32_t K, void* h, void* ws,
                          size_t ws_bytes, moe_stream stream) {
  moe::Check c = moe::validate_gated_int8(x, x_scales, wg, wg_scales, wu, wu_scales, T, F, K, h);
  if (!c.ok() || T == 0) return finish(c);
  moe::Int8Plan plan;
  size_t need;
  const hipError_t err = int8_plan_of(T, F, K, true, &plan, &need);
  if (err != hipSuccess) return hip_status("moe_gated_int8", err);
  c = moe::validate_int8_workspace("moe_gated_int8", ws, ws_bytes, need);
  if (!c.ok()) return finish(c);
  const moe::Int8Product p = {x, x_scales, wg, wu, wg_scales, wu_scales, nullptr, static_cast<uint16_t*>(h), int(T), F, K,
                              (K + 127) / 128 * 2, static_cast<i32x4_t*>(ws)};
  return hip_status("moe_gated_int8", moe::launch_int8_product(p, plan, stream_of(stream)));
}

}  // extern "C"
