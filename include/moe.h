/*
 * moe.h - C ABI of the MI355X (gfx950) MoE-layer hot path.
 *
 * One Mixture-of-Experts layer over an expert-level batch: the module the
 * paper's forward pass (Algorithm 1) runs on the hidden states COMBINEd from
 * many yielded sequences, h_out <- MoE(h, l).  The layer is the top-k
 * softmax-gated SwiGLU expert layer of the Mixtral and DeepSeek models the
 * paper evaluates (Section 6, Models); its motivation is sparse expert
 * activation with uneven expert popularity (Section 2.2, Insight 1) and the
 * large expert batch needed to saturate the GPU (Section 7, batch-size regime).
 *
 * Four calls, issued in order on one stream, make the layer:
 *   moe_route        logits -> top-k expert ids and gate weights
 *   moe_permute      ids, x -> per-expert counts, offsets, row maps, x_perm
 *   moe_grouped_ffn  x_perm -> y_perm, each expert's SwiGLU FFN on its rows
 *   moe_combine      y_perm -> y, gate-weighted sum of each token's k rows
 * A shared (always active) expert is one more moe_grouped_ffn call with E = 1
 * over x itself, whose output moe_combine adds with weight 1.
 *
 * Conventions (all calls)
 *   - Every pointer argument is a DEVICE pointer unless stated otherwise, owned
 *     by the caller.  The library never allocates, frees or synchronizes in
 *     these calls: work is enqueued on `stream` (a hipStream_t; NULL is the
 *     default stream) and the call returns.  Buffers must not overlap.
 *   - Row-major layouts.  Shapes are given as [rows, cols].
 *   - Every base pointer must be 16-byte aligned.
 *   - Validation is done on the host before anything is enqueued.  On an error
 *     nothing is written and nothing is launched; moe_last_error() then holds
 *     a message naming the argument.  T = 0 (or R = 0) returns MOE_OK and
 *     enqueues nothing; pointers may then be NULL.
 *   - Not checked (preconditions): finite logits; expert ids in [0, E) and
 *     distinct within a token (moe_route guarantees both); offsets consistent
 *     with R; buffers large enough for the stated shapes.
 *   - Device faults surface asynchronously at the caller's next synchronization.
 *   - Thread-safe; calls on different streams are independent.
 *   - Deterministic: identical inputs give bitwise-identical outputs (no atomics
 *     decide any result).
 */
#ifndef MOE_H
#define MOE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    MOE_OK = 0,
    MOE_ERR_INVALID_ARGUMENT = 1,    /* null pointer, bad size, misalignment */
    MOE_ERR_UNSUPPORTED = 2,         /* E > 256, k > 16, unknown dtype */
    MOE_ERR_WORKSPACE_TOO_SMALL = 3,
    MOE_ERR_HIP = 4                  /* a HIP runtime call or kernel launch failed */
} moe_status;

typedef enum {
    MOE_DTYPE_F32 = 0,               /* fp32 activations and weights, fp32 arithmetic */
    MOE_DTYPE_BF16 = 1               /* bf16 activations and weights, fp32 accumulation */
} moe_dtype;

typedef void* moe_stream;            /* hipStream_t */

#define MOE_ABI_VERSION 1
#define MOE_MAX_EXPERTS 256
#define MOE_MAX_TOPK 16
#define MOE_MAX_ROUTER_EXPERTS 64   /* moe_router_topk */
#define MOE_FEW_TOKENS 16           /* moe_few_tokens */
#define MOE_KV8_BLOCK 16            /* tokens of a cache block that share an exponent */

/* ABI version of the loaded library (MOE_ABI_VERSION). */
int moe_abi_version(void);

/* Static description of a status code; never NULL. */
const char* moe_status_string(int status);

/* Message of the last failed call on this host thread ("" if none).  The
 * pointer stays valid until the next call on the same thread. */
const char* moe_last_error(void);

/*
 * moe_route - top-k gating (the MoE gate the expert batch reaches; the paper's
 * Section 2.2 expert selection).
 *
 *   logits        f32 [T, E]   gating logits (the router GEMM is the caller's)
 *   topk_ids      i32 [T, k]   out: slot 0 holds the largest logit
 *   topk_weights  f32 [T, k]   out: gate weights
 *
 * Order: larger logit first; equal logits (including +0 and -0) go to the
 * lower expert id.  Selection compares the fp32 logits exactly.  Weights:
 * p_e = exp(l_e - l_max); renormalize = 1 gives p / sum over the k selected,
 * renormalize = 0 gives p / sum over all E.  exp and the division are fp32.
 * Errors: INVALID_ARGUMENT for T < 0, E < 1, k < 1, k > E, T*k > INT32_MAX,
 * renormalize not 0/1, null or misaligned pointers; UNSUPPORTED for E > 256 or
 * k > 16.
 */
moe_status moe_route(const float* logits, int64_t T, int32_t E, int32_t k, int32_t renormalize,
                     int32_t* topk_ids, float* topk_weights, moe_stream stream);

/*
 * moe_router_topk - the MoE gate with its router GEMM: logits = x . w_router^T
 * computed on the matrix cores (bf16 operands, fp32 accumulation), then the
 * selection and gate weights of moe_route on those fp32 logits (the MoE gate
 * whose batch Section 7 sizes).  The logits stay on chip unless `logits` is given.
 *
 *   x             bf16 [T, H]   hidden states
 *   w_router      bf16 [E, H]   router matrix, one K-contiguous row per expert
 *   logits        f32  [T, E]   optional out (NULL: not written)
 *   topk_ids, topk_weights      as moe_route
 *
 * Errors: as moe_route, plus INVALID_ARGUMENT for H not a positive multiple of
 * 64 and UNSUPPORTED for E > 64 (MOE_MAX_ROUTER_EXPERTS) or a router matrix of
 * 2 GiB or more.
 */
moe_status moe_router_topk(const void* x, const void* w_router, int64_t T, int32_t E, int32_t k, int32_t H,
                           int32_t renormalize, float* logits, int32_t* topk_ids, float* topk_weights,
                           moe_stream stream);

/*
 * moe_permute - group the T*k (token, slot) assignments by expert and gather
 * each assignment's hidden row (the expert-level batch built by COMBINE,
 * Section 4.2 and Algorithm 1, regrouped per expert).
 *
 *   topk_ids          i32 [T, k]      expert of each assignment (from moe_route)
 *   x                 dt  [T, H]      hidden states
 *   expert_counts     i32 [E]         out: rows per expert
 *   expert_offsets    i32 [E + 1]     out: exclusive prefix sum, offsets[E] = T*k
 *   sorted_token_ids  i32 [T*k]       out: source token of each grouped row
 *   dest_rows         i32 [T, k]      out: grouped row of assignment (t, j)
 *   x_perm            dt  [T*k, H]    out: x_perm[r] = x[sorted_token_ids[r]], or NULL:
 *                                     then only the maps are produced and x is not read
 *                                     (x may be NULL); moe_grouped_ffn_gather reads the
 *                                     rows through sorted_token_ids instead
 *   ws, ws_bytes      device scratch of at least moe_permute_workspace_bytes()
 *
 * Expert e owns rows offsets[e] .. offsets[e+1]-1, holding its tokens in
 * ascending token order (a stable counting sort).
 * Errors: as moe_route, plus INVALID_ARGUMENT for H < 64 or H % 64 != 0,
 * UNSUPPORTED for an unknown dtype, WORKSPACE_TOO_SMALL.
 */
size_t moe_permute_workspace_bytes(int64_t T, int32_t E, int32_t k);
moe_status moe_permute(const int32_t* topk_ids, const void* x, int64_t T, int32_t E, int32_t k,
                       int32_t H, moe_dtype dt, int32_t* expert_counts, int32_t* expert_offsets,
                       int32_t* sorted_token_ids, int32_t* dest_rows, void* x_perm,
                       void* ws, size_t ws_bytes, moe_stream stream);

/*
 * moe_permute_static - moe_permute for callers that cannot allocate: code under
 * HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  It
 * takes no workspace and allocates nothing: its scratch (per-expert counts of
 * blocks of assignments) is a static device array of
 * MOE_PERMUTE_STATIC_SCRATCH_BYTES that the library holds on every device it
 * runs on until the process ends.  Arguments, outputs and results are those of
 * moe_permute, bit for bit.
 *
 * Calls that overlap on one device (e.g. on two streams) share that array and
 * race; serialize them.  Nothing in the array needs clearing between calls.
 * Errors: as moe_permute, without WORKSPACE_TOO_SMALL; UNSUPPORTED when
 * moe_permute_workspace_bytes(T, E, k) exceeds MOE_PERMUTE_STATIC_SCRATCH_BYTES
 * (4 MiB: e.g. up to 2^24 assignments with 64 experts, 2^22 with 256); HIP when
 * the array's device address cannot be obtained.
 */
#define MOE_PERMUTE_STATIC_SCRATCH_BYTES (4u << 20)
moe_status moe_permute_static(const int32_t* topk_ids, const void* x, int64_t T, int32_t E, int32_t k,
                              int32_t H, moe_dtype dt, int32_t* expert_counts, int32_t* expert_offsets,
                              int32_t* sorted_token_ids, int32_t* dest_rows, void* x_perm, moe_stream stream);

/*
 * moe_grouped_ffn - every expert's SwiGLU FFN on its own rows, as one grouped
 * GEMM pair (the expert computation of the MoE module in Algorithm 1).
 *
 *   x_perm          dt  [R, H]     rows grouped by expert
 *   expert_offsets  i32 [E + 1]    DEVICE array; group e = rows offsets[e]..offsets[e+1]-1
 *   w_gate, w_up    dt  [E, F, H]  K-contiguous (each row is one output feature)
 *   w_down          dt  [E, H, F]  K-contiguous
 *   y_perm          dt  [R, H]     out: W_down[e] (silu(W_gate[e] x) * (W_up[e] x))
 *   ws, ws_bytes    device scratch of at least moe_grouped_ffn_workspace_bytes();
 *                   it holds the intermediate h [R, F] and (bf16) fp32 partial
 *                   sums of down-projection tiles split along k
 *
 * silu(z) = z / (1 + exp(-z)).  bf16: fp32 accumulation, h and y_perm rounded
 * to bf16 (nearest even).  f32: fp32 throughout.  Group sizes are read on the
 * device only (no host readback).  Results are deterministic for a given device
 * and compute-unit budget (moe_set_cu_budget): R, E, H, F and the budget choose the
 * kernel, and (large groups) when the last round of
 * down-projection tiles would leave the grid mostly idle, those tiles are
 * computed in pieces along k and their fp32 partial sums added in piece order,
 * so their rounding depends on the grid size.
 * Errors: INVALID_ARGUMENT for R < 0, E < 1, H or F not a positive multiple of
 * 64, R > INT32_MAX, null or misaligned pointers; UNSUPPORTED for E > 256 or
 * an unknown dtype; WORKSPACE_TOO_SMALL.
 */
size_t moe_grouped_ffn_workspace_bytes(int64_t R, int32_t E, int32_t H, int32_t F, moe_dtype dt);
moe_status moe_grouped_ffn(const void* x_perm, const int32_t* expert_offsets, int64_t R, int32_t E,
                           int32_t H, int32_t F, const void* w_gate, const void* w_up,
                           const void* w_down, moe_dtype dt, void* y_perm, void* ws,
                           size_t ws_bytes, moe_stream stream);

/*
 * moe_grouped_ffn_gather - moe_grouped_ffn reading each grouped row straight
 * from the token rows: row r of group e is x[sorted_token_ids[r]].  The same
 * result as moe_permute's x_perm followed by moe_grouped_ffn, bit for bit, but
 * the grouped copy of the activations (T*k rows) is never written or read.
 *
 *   x                 dt  [T, H]   token rows (any size)
 *   sorted_token_ids  i32 [R]      from moe_permute (R = T*k)
 *   other arguments as moe_grouped_ffn; the workspace size is
 *   moe_grouped_ffn_workspace_bytes(R, E, H, F, dt)
 *
 * Errors: as moe_grouped_ffn, plus INVALID_ARGUMENT for T < 0, R > 0 with
 * T = 0, a NULL or misaligned x or sorted_token_ids.  Token ids are not checked
 * (precondition: 0 <= id < T).
 */
moe_status moe_grouped_ffn_gather(const void* x, const int32_t* sorted_token_ids,
                                  const int32_t* expert_offsets, int64_t T, int64_t R, int32_t E,
                                  int32_t H, int32_t F, const void* w_gate, const void* w_up,
                                  const void* w_down, moe_dtype dt, void* y_perm, void* ws,
                                  size_t ws_bytes, moe_stream stream);

/*
 * MXFP8 expert GEMMs (the paper's MoE GEMMs are FP8: Section 5, the prefill
 * cost estimate with FP8 MoE GEMMs, and Section 5.6).  MXFP8 is the OCP
 * Microscaling format: E4M3 element codes (1 sign, 4 exponent bits with bias 7,
 * 3 mantissa bits; largest value 448) and one E8M0 scale 2^(s - 127) per 32
 * consecutive elements along k, which gfx950's block-scaled MFMA applies itself.
 *
 * Layout of an MXFP8 matrix with `rows` rows and K columns (K % 128 == 0):
 *   codes   u8 [rows, K]                 row-major E4M3 codes
 *   scales  u8 [K / 128][rows][4]        the scale of row r for k in
 *                                        [32 b, 32 b + 32) is the byte
 *                                        scales[((b / 4) * rows + r) * 4 + b % 4]
 * moe_mxfp8_scale_bytes(rows, K) = rows * K / 32.  An expert weight tensor
 * [E, N, K] is the matrix of E * N rows.
 */
size_t moe_mxfp8_scale_bytes(int64_t rows, int32_t K);

/*
 * moe_quantize_mxfp8 - bf16 rows to MXFP8.
 *
 *   src      bf16 [rows_src, K]
 *   row_map  i32 [rows_out] or NULL: output row r quantizes src row row_map[r]
 *            (e.g. sorted_token_ids from moe_permute gives x_perm's order);
 *            NULL requires rows_out <= rows_src and quantizes rows 0..rows_out-1
 *   codes    u8 [rows_out, K]  out;  scales  u8, moe_mxfp8_scale_bytes(rows_out, K)  out
 *
 * Per block of 32: shared exponent floor(log2(max |v|)) - 8 clamped to
 * [-127, 127] (-127 for an all-zero block); codes = v / 2^shared_exp rounded to
 * the nearest E4M3 value, ties to an even mantissa, clamped to +-448, sign bit
 * kept (-0 gives 0x80).  Inputs are finite (not checked).
 * Errors: INVALID_ARGUMENT for rows_out < 0, rows_src < 0, K not a positive
 * multiple of 128, rows_out > rows_src without a row_map, null or misaligned
 * pointers.  Row indices are not checked (precondition: 0 <= row_map[r] < rows_src).
 */
moe_status moe_quantize_mxfp8(const void* src, const int32_t* row_map, int64_t rows_out, int64_t rows_src,
                              int32_t K, uint8_t* codes, uint8_t* scales, moe_stream stream);

/*
 * moe_grouped_ffn_mxfp8 - moe_grouped_ffn with both GEMMs on MXFP8 operands.
 *
 *   x_codes, x_scales    MXFP8 [R, H]    grouped rows (moe_quantize_mxfp8 with row_map =
 *                                        sorted_token_ids)
 *   expert_offsets       i32 [E + 1]     DEVICE array, as moe_grouped_ffn
 *   wg_*, wu_*           MXFP8 [E * F, H] W_gate, W_up quantized along H
 *   wd_*                 MXFP8 [E * H, F] W_down quantized along F
 *   y_perm               bf16 [R, H]     out
 *   ws, ws_bytes         device scratch of at least moe_grouped_ffn_mxfp8_workspace_bytes();
 *                        it holds h [R, F] in MXFP8 and fp32 partial sums of
 *                        down-projection tiles split along k
 *
 * g and u accumulate in fp32 from the dequantized operands (the matrix cores
 * apply the block scales), h = silu(g) * u in fp32 is quantized to MXFP8 along F
 * as moe_quantize_mxfp8 does, and y_perm accumulates in fp32 and is rounded to
 * bf16 (nearest even).  Determinism as moe_grouped_ffn: for a given device and
 * compute-unit budget.
 * Errors: INVALID_ARGUMENT for R < 0, R > INT32_MAX, E < 1, H or F not a
 * positive multiple of 128, null or misaligned pointers; UNSUPPORTED for
 * E > 256 or when a scale array or an expert matrix reaches 2 GiB;
 * WORKSPACE_TOO_SMALL.
 */
size_t moe_grouped_ffn_mxfp8_workspace_bytes(int64_t R, int32_t E, int32_t H, int32_t F);
moe_status moe_grouped_ffn_mxfp8(const uint8_t* x_codes, const uint8_t* x_scales,
                                 const int32_t* expert_offsets, int64_t R, int32_t E, int32_t H, int32_t F,
                                 const uint8_t* wg_codes, const uint8_t* wg_scales, const uint8_t* wu_codes,
                                 const uint8_t* wu_scales, const uint8_t* wd_codes, const uint8_t* wd_scales,
                                 void* y_perm, void* ws, size_t ws_bytes, moe_stream stream);

/*
 * moe_grouped_ffn_mxfp8_gather - moe_grouped_ffn_mxfp8 reading each grouped row's
 * codes and scales straight from the token rows: row r of group e is token
 * sorted_token_ids[r] of x.  x is then quantized once per token (T rows, no
 * row_map) instead of once per assignment; the result equals quantizing with
 * row_map = sorted_token_ids and calling moe_grouped_ffn_mxfp8, bit for bit.
 *
 *   x_codes, x_scales  MXFP8 [T, H]   token rows (T * H < 2^31)
 *   sorted_token_ids   i32 [R]        from moe_permute
 *   other arguments as moe_grouped_ffn_mxfp8 (same workspace size)
 *
 * Errors: as moe_grouped_ffn_mxfp8, plus INVALID_ARGUMENT for T < 0, R > 0 with
 * T = 0, a NULL or misaligned sorted_token_ids; UNSUPPORTED when the codes of x
 * reach 2 GiB.  Token ids are not checked (precondition: 0 <= id < T).
 */
moe_status moe_grouped_ffn_mxfp8_gather(const uint8_t* x_codes, const uint8_t* x_scales,
                                        const int32_t* sorted_token_ids, const int32_t* expert_offsets, int64_t T,
                                        int64_t R, int32_t E, int32_t H, int32_t F, const uint8_t* wg_codes,
                                        const uint8_t* wg_scales, const uint8_t* wu_codes,
                                        const uint8_t* wu_scales, const uint8_t* wd_codes,
                                        const uint8_t* wd_scales, void* y_perm, void* ws, size_t ws_bytes,
                                        moe_stream stream);

/*
 * moe_combine - gate-weighted sum of each token's k expert outputs (the MoE
 * module's output h_out in Algorithm 1).
 *
 *   y_perm        dt  [T*k, H]  expert outputs in grouped order
 *   dest_rows     i32 [T, k]    grouped row of assignment (t, j) (from moe_permute)
 *   topk_weights  f32 [T, k]
 *   y_shared      dt  [T, H]    optional (NULL = none): added with weight 1
 *   y             dt  [T, H]    out: sum_j w[t,j] * y_perm[dest_rows[t,j]] (+ y_shared[t])
 *
 * The sum is formed in fp32 in slot order j = 0..k-1, the shared row added
 * last, then rounded once to dt.  Gather form: no atomics.
 * Errors: INVALID_ARGUMENT for T < 0, k < 1, k > 16 (UNSUPPORTED), H not a
 * positive multiple of 64, T*k > INT32_MAX, null or misaligned pointers.
 */
moe_status moe_combine(const void* y_perm, const int32_t* dest_rows, const float* topk_weights,
                       const void* y_shared, int64_t T, int32_t k, int32_t H, moe_dtype dt, void* y,
                       moe_stream stream);

/*
 * 4-bit weights with group scales, for products with few rows, whose time is the
 * read of the weights (the memory-constrained single-GPU setting of Section 7; the
 * FP8 decoding of a batch's last sequences goes the same way).
 *
 *   W[n][k] = scale[n][k / group] * (q[n][k] - zero[n][k / group])
 *
 * q and zero are integers 0..15, scale is bf16, group is 32, 64 or 128 and divides K.
 * Without zero points (NULL) zero is 8.  Two representations:
 *
 *   standard  codes u8 [rows, K / 2], the even column in the low nibble; scales bf16
 *             [rows, K / group]; zeros u8 [rows, K / group]
 *   packed    what the kernels read, rows padded to 16 and columns to 128: codes u8
 *             [rows / 16][K / 128][1024], a tile of 16 rows x 128 columns in one piece.
 *             Word j of the four words 16 l .. 16 l + 15 of a tile holds row l % 16, columns
 *             32 j + 8 (l / 16) + 0..7: nibble p column 2 p for p < 4, 2 (p - 4) + 1 for
 *             p >= 4.  Scales [rows / 16][K / 128][4][128 / group][4], the last for rows
 *             4 a + 0..3: bf16; with zero points 32-bit words, the upper half the scale, the
 *             lower half 128 + zero, both bf16.
 *
 * moe_int4_code_bytes and moe_int4_scale_bytes (zeros: 0 or 1) give the packed sizes of one
 * matrix.  An expert tensor [E, N, K] is E packed matrices one after the other.
 */
size_t moe_int4_code_bytes(int64_t rows, int32_t K);
size_t moe_int4_scale_bytes(int64_t rows, int32_t K, int32_t group, int32_t zeros);

/*
 * moe_quantize_int4 - bf16 rows to standard 4-bit codes.
 *
 *   src     bf16 [rows, K]
 *   codes, scales, zeros   standard form, out; zeros NULL: symmetric
 *
 * Symmetric: scale = bf16(max |v| / 7), q = round(v / scale) + 8.  With zeros: lo = min(v, 0),
 * hi = max(v, 0), scale = bf16((hi - lo) / 15), zero = round(-lo / scale), q = round(v / scale)
 * + zero.  Both clamped to 0..15, ties to even, the quotients by the scale as rounded.  A group
 * of zeros has scale 0.  Inputs are finite (not checked).
 * Errors: INVALID_ARGUMENT for rows < 0, an unknown group, K not a positive multiple of
 * the group, null or misaligned pointers; UNSUPPORTED for 2^31 groups or more.
 */
moe_status moe_quantize_int4(const void* src, int64_t rows, int32_t K, int32_t group, uint8_t* codes,
                             uint16_t* scales, uint8_t* zeros, moe_stream stream);

/*
 * moe_pack_int4 - standard to packed form, of `matrices` matrices of rows x K each; zeros may be
 * NULL (out_scales then without them).  Run once when weights are loaded.
 * Errors: as moe_quantize_int4, plus INVALID_ARGUMENT for matrices < 0; UNSUPPORTED for 2^26
 * tiles or more.
 */
moe_status moe_pack_int4(const uint8_t* codes, const uint16_t* scales, const uint8_t* zeros, int64_t matrices,
                         int64_t rows, int32_t K, int32_t group, uint8_t* out_codes, uint8_t* out_scales,
                         moe_stream stream);

/*
 * moe_matvec_int4 - y = x W^T for a 4-bit W and few rows of x.
 *
 *   x       bf16 [T, K]
 *   codes, scales   packed W [N, K], zeros 1 where it has zero points, else 0
 *   y       bf16 [T, N]   out
 *
 * Codes are multiplied as integers in bf16 (exact) on the matrix cores, sums of a group in
 * fp32, scaled and added up in fp32, rounded once.  The weights are read once for each 32
 * rows of x: any T is right, few rows are what it is for.  x finite: an infinite x gives NaN.
 * Errors: INVALID_ARGUMENT for T < 0, N < 1, an unknown group, K not a positive multiple of
 * the group, null or misaligned pointers; UNSUPPORTED for T > 2^20, K > 2^23 or 2 GiB of
 * codes or scales.
 */
moe_status moe_matvec_int4(const void* x, const uint8_t* codes, const uint8_t* scales, int32_t zeros, int64_t T,
                           int32_t N, int32_t K, int32_t group, void* y, moe_stream stream);

/*
 * moe_few_tokens - the whole layer (moe_route, the expert FFNs, the shared expert,
 * moe_combine) for at most MOE_FEW_TOKENS tokens in two kernels, three where the sums of y are
 * cut into parts: the step of the few sequences that a batch ends on (the paper's long tail: at
 * most 8 active sequences).
 * Nothing is grouped: the layer's time is one read of the chosen experts' weights.
 *
 *   x               bf16 [T, H]    T <= 16
 *   logits          f32  [T, E]
 *   w_gate, w_up    bf16 [E, F, H];  w_down bf16 [E, H, F]   as moe_grouped_ffn
 *   ws_gate, ws_up  bf16 [Fs, H];    ws_down bf16 [H, Fs]    shared expert; NULL with Fs = 0
 *   topk_ids i32, topk_weights f32 [T, k]   out, as moe_route
 *   y               bf16 [T, H]    out
 *   ws, ws_bytes    device scratch of at least moe_few_tokens_workspace_bytes(): the rows h
 *                   and the parts of y's sums; not to be shared by calls that overlap
 *
 * The gate weight multiplies silu(g) u in fp32; h is kept to 16 significant bits (two bf16
 * numbers), all sums are fp32, y is rounded once.  Deterministic for a given device and
 * compute-unit budget; the order of y's sums depends on the experts that the batch chose, so a
 * token's y may differ in its last bit with the tokens beside it.  Weights and scales that are
 * not finite reach the tokens that chose their expert alone, as in moe_grouped_ffn.
 * Errors: as moe_route and moe_grouped_ffn, plus INVALID_ARGUMENT for Fs < 0 or not a
 * multiple of 64; UNSUPPORTED for T > 16.
 *
 * moe_few_tokens_int4 takes 4-bit weights: `weights` is a HOST array of six packed tensors in
 * the order w_gate, w_up, w_down, ws_gate, ws_up, ws_down, of one group size, all with zero
 * points (zeros = 1) or all without (0).  H and F (and Fs) are multiples of the group.
 */
typedef struct {
    const uint8_t* codes;
    const uint8_t* scales;
} moe_int4;
size_t moe_few_tokens_workspace_bytes(int64_t T, int32_t H, int32_t k, int32_t F, int32_t Fs);
moe_status moe_few_tokens(const void* x, const float* logits, int64_t T, int32_t H, int32_t E, int32_t k, int32_t F,
                          int32_t Fs, int32_t renormalize, const void* w_gate, const void* w_up, const void* w_down,
                          const void* ws_gate, const void* ws_up, const void* ws_down, int32_t* topk_ids,
                          float* topk_weights, void* y, void* ws, size_t ws_bytes, moe_stream stream);
moe_status moe_few_tokens_int4(const void* x, const float* logits, int64_t T, int32_t H, int32_t E, int32_t k,
                               int32_t F, int32_t Fs, int32_t renormalize, int32_t group, int32_t zeros,
                               const moe_int4* weights,
                               int32_t* topk_ids, float* topk_weights, void* y, void* ws, size_t ws_bytes,
                               moe_stream stream);

/*
 * The paged 8-bit key-value cache of one attention layer (per-sequence KV quantisation,
 * Section 4; pages of 64 tokens in the paper's Section 5.6).  Keys and values are E4M3 codes; the
 * 16 tokens of a block share one exponent byte for each kv head, one for their keys and one
 * for their values:  value = code * 2^(e - 127).
 *
 *   k_codes          u8 [pages, heads, page, dim]
 *   v_codes          u8 [pages, heads, page / 16, dim, 16]   a block's values transposed
 *   k_exps, v_exps   u8 [pages, heads, page / 16]
 *
 * page is a multiple of 16, dim 64, 128 or 256.
 *
 * A batch over it, the same arguments for both calls:
 *   block_table  i32 [B, table_cols]  page of tokens [page i, page (i + 1)) of each sequence
 *   seq_lens     i32 [B]     tokens of each sequence, the new ones included
 *   cu_tokens    i32 [B + 1] rows of the new tokens: sequence b has rows cu[b] .. cu[b + 1] - 1,
 *                at positions seq_lens[b] - n_b .. seq_lens[b] - 1 (n_b its row count)
 *   T            rows, cu_tokens[B]
 * A sequence may have no rows: its pages are neither read nor written.  Rows at positions
 * below 0 (a slot of a captured graph whose sequence has ended: seq_lens[b] = 0) are left out:
 * nothing is appended for them, their attention output is 0.  All of these are device arrays
 * and are not checked beyond what keeps the kernels inside their buffers: a page outside
 * [0, pages) is not written, and read as the nearest inside; rows outside [0, T) are left out.
 */
typedef struct {
    uint8_t* k_codes;
    uint8_t* v_codes;
    uint8_t* k_exps;
    uint8_t* v_exps;
    int64_t pages;
    int32_t page;
    int32_t heads;
    int32_t dim;
} moe_kv8_cache;

/*
 * moe_kv8_append - rotate the new tokens' queries and keys by their positions and write
 * keys and values into the cache.
 *
 *   q, k, v     bf16, rows T of q_heads, heads, heads heads of dim; *_stride elements from a
 *               row to the next (a multiple of 8): slices of one projection's output will do
 *   cos_sin     f32 [positions, rot]   cos, then sin, of rot / 2 angles of each position
 *   rot         leading dimensions that are rotated, a multiple of 16, at most dim
 *   interleaved 0: pairs (i, i + rot / 2);  1: pairs (2 i, 2 i + 1)
 *   q_out       bf16 [T, q_heads, dim]   out: rotated queries
 *
 * (a, b) becomes (a cos - b sin, a sin + b cos), each operation rounded to fp32.  For each block
 * and kv head that gets tokens:  s = the smallest integer with max |v| <= 448 * 2^s over the new
 * tokens (-127 for zeros); if the block holds earlier tokens, s = max(s, the block's) and, where
 * that grew, their codes are rounded again to the new step; places after the last token are
 * set to 0.  Codes are rounded to nearest even.  An infinity saturates, NaN stays NaN and does
 * not count in s.  Calling again with the same arguments leaves the cache as it is.  Tokens
 * at positions of `positions` or more are rotated as the last one.  Queries of tokens whose page
 * is outside the cache or the table are rotated all the same; those of rows left out are not written.
 * Errors: INVALID_ARGUMENT for negative sizes, heads not dividing q_heads, a page not a positive
 * multiple of 16, a bad stride or rot, null or misaligned pointers; UNSUPPORTED for another dim,
 * T + 2 B of 2^24 or more, heads > 65535.
 */
moe_status moe_kv8_append(const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                          int64_t v_stride, int64_t T, int32_t q_heads, const float* cos_sin, int64_t positions,
                          int32_t rot, int32_t interleaved, const moe_kv8_cache* cache, const int32_t* block_table,
                          int32_t table_cols, const int32_t* seq_lens, const int32_t* cu_tokens, int32_t B,
                          void* q_out, moe_stream stream);

/*
 * moe_kv8_attention - causal attention of the new tokens over the cache.
 *
 *   q           bf16 [T, q_heads, dim]   rotated queries; head h reads kv head h / (q_heads / heads)
 *   max_new     at least every sequence's row count: rows beyond it are not computed
 *   max_len     the longest sequence (for the plan only; any value gives right results).  A loop
 *               whose batches change may pass the largest max_new and max_len each time: the
 *               workspace for these is then right for every step
 *   window      0, or how many tokens a row sees, itself included
 *   scale       factor of the scores, positive
 *   out         bf16 [T, q_heads, dim]   out
 *   ws, ws_bytes  device scratch of at least moe_kv8_attention_workspace_bytes() for the same sizes
 *
 * A row at position p sees tokens 0..p, with a window p - window + 1..p.  The products of queries
 * and keys are exact up to 2^-17 of a query row's largest element; scores, softmax and sums are
 * fp32, probabilities are rounded to bf16 for the product with the values and for their sum.  A
 * row that sees nothing is 0.  Cache contents past a sequence's end are not used, whatever they
 * are, and neither are those outside a row's window.  A NaN that a row sees shows as NaN in its
 * output: one in its query or a key in all dimensions, one in a value in that dimension at least.
 * So does a value of 2^128 or more, which bf16 does not hold (what an infinity was appended as):
 * infinity or NaN.  Values are summed in fp32, weighted by up to 2^8, and then divided by the
 * weights' sum: those under 2^100 do not overflow there.
 * Deterministic for a given plan (sizes, max_new, max_len, compute-unit budget).
 * Errors: as moe_kv8_append, plus INVALID_ARGUMENT for max_new < 1, max_len < 0, window < 0;
 * WORKSPACE_TOO_SMALL.
 */
size_t moe_kv8_attention_workspace_bytes(int64_t T, int32_t B, int32_t q_heads, int32_t heads, int32_t dim,
                                         int32_t max_new, int32_t max_len, int32_t window);
moe_status moe_kv8_attention(const void* q, int64_t T, int32_t q_heads, const moe_kv8_cache* cache,
                             const int32_t* block_table, int32_t table_cols, const int32_t* seq_lens,
                             const int32_t* cu_tokens, int32_t B, int32_t max_new, int32_t max_len, int32_t window,
                             float scale, void* out, void* ws, size_t ws_bytes, moe_stream stream);

/*
 * The dense half of a layer in 8-bit integers: what runs before, after and beside the experts when
 * every FLOP of a dense batch counts (Section 7's batch sizes; the shared experts and dense
 * feed-forward blocks of the models of Section 6).  moe_norm_join gives the codes that moe_matmul_int8 and
 * moe_gated_int8 read, moe_quantize_int8 those of any rows.
 *
 *   value[r][k] = scale[r] * code[r][k]      codes int8, a scale (f32) for each row
 *
 * A row is a token of the activations or an output channel of the weights.  Two representations:
 *
 *   row-major  i8 [rows, K]: activations, and weights as they are quantised
 *   packed     weights as the products read them, rows padded to 16 and columns to 128 with zeros:
 *              i8 [rows / 16][K / 64][1024]: byte 16 l + j of a piece is row l % 16, column
 *              16 (l / 16) + j.  moe_int8_code_bytes gives the size
 *
 * Codes of a row of values v with m = max |v|:  scale = m / 127, code = round(v * (127 / m)), ties to
 * even, each operation rounded to fp32 (rows with m < 2^-100 are multiplied by 2^100 first, so that
 * 127 / m is finite); a row of zeros has scale 0.  A row that holds an infinity or a NaN gets the scale NaN
 * and codes 0, so that its products show it.
 */

/*
 * moe_norm_join - the joint between two blocks, in one pass over the residual stream: a block's output is
 * normalised, gated, scaled and added to the stream, and the stream is normalised for the next block.
 *
 *   x'  = x + alpha * g * j       j = norm(y) * (offset + w_post) with post = 1, y with post = 0
 *   z   = norm(x') * (offset + w_pre)                   norm(v) = v / sqrt(mean(v^2) + eps)
 *
 *   x           dt [T, H]      the stream, bf16 or f32
 *   y           bf16 [T, H]    a block's output; NULL: x' = x, and post, w_post, gate and x_out are 0 or NULL
 *   w_post, w_pre  bf16 [H]    NULL: factors of 1 (without offset).  offset: 0, or 1 for weights stored less 1
 *   gate        bf16, by gate_kind: MOE_GATE_CHANNEL [H], MOE_GATE_TOKEN [T] (gate_stride elements
 *               apart, a column at any element), MOE_GATE_FULL [T, H]; with sigmoid = 1 a gate counts as
 *               1 / (1 + exp(-gate))
 *   x_out       dt [T, H]      out: x'; may be x itself (then x_out_stride = x_stride), and overlaps nothing else
 *   z           out: bf16 [T, H], or with z_codes = 1 int8 [T, H] and z_scales f32 [T].  NULL: not computed
 *   *_stride    elements from a row to the next, rows in whole 16-byte pieces
 *
 * Arithmetic is fp32, x' and z are rounded once; z is taken of x' before its rounding.  The codes of z
 * are those of x' (offset + w_pre), the norm's factor is in the scale alone; products take them where H % 16 == 0.
 * Squares are summed in fp32: a row (of y with post = 1, of x') whose squares sum to 2^128 or more counts as infinitely
 * long, its norm is 0, or NaN where a product with a weight overflows; with an eps below 2^-100 a row whose
 * largest magnitude is below 2^-50 is too short, its norm is off, and from 2^-75 down infinite or NaN.  A NaN or
 * infinity stays in its row.  The order of the sums depends on H, T and the compute-unit budget
 * (moe_set_cu_budget), on nothing else.
 * Errors: INVALID_ARGUMENT for H not a positive multiple of 8, T < 0, eps < 0, an
 * eps, alpha or offset beyond 1e30 or NaN, flags that are not 0 or 1, an unknown gate_kind, bad strides, arguments without the one they belong to,
 * null or misaligned pointers; UNSUPPORTED for H > 32768, T > 2^31 or an unknown dtype.
 */
typedef enum { MOE_GATE_NONE = 0, MOE_GATE_CHANNEL = 1, MOE_GATE_TOKEN = 2, MOE_GATE_FULL = 3 } moe_gate;
moe_status moe_norm_join(const void* x, int64_t x_stride, moe_dtype dt, const void* y, int64_t y_stride, int32_t post,
                         const void* w_post, const void* gate, int64_t gate_stride, int32_t gate_kind, int32_t sigmoid,
                         float alpha, const void* w_pre, float offset, float eps, int64_t T, int32_t H, void* x_out,
                         int64_t x_out_stride, int32_t z_codes, void* z, float* z_scales, moe_stream stream);

/*
 * moe_quantize_int8 - bf16 rows to row-major codes and their scales.
 *
 *   src     bf16 [rows, K], src_stride elements from a row to the next (a multiple of 8)
 *   codes   i8 [rows, K]  out;   scales  f32 [rows]  out
 *
 * Errors: INVALID_ARGUMENT for rows < 0, K not a positive multiple of 16, a bad stride, null or
 * misaligned pointers; UNSUPPORTED for K > 131056 or rows > 2^31.
 */
moe_status moe_quantize_int8(const void* src, int64_t src_stride, int64_t rows, int32_t K, int8_t* codes, float* scales,
                             moe_stream stream);

/*
 * moe_pack_int8 - row-major to packed codes.  Run once when weights are loaded.
 * Errors: as moe_quantize_int8; UNSUPPORTED for rows > 2^24 or 2^26 pieces of 1 KB.
 */
size_t moe_int8_code_bytes(int64_t rows, int32_t K);
moe_status moe_pack_int8(const int8_t* codes, int64_t rows, int32_t K, int8_t* out, moe_stream stream);

/*
 * moe_matmul_int8 - y = x W^T (+ bias) of 8-bit codes, for one row as for large batches.
 *
 *   x, x_scales   row-major codes [T, K], f32 [T]
 *   w, w_scales   packed codes [N, K], f32 [N]
 *   bias          bf16 [N], or NULL
 *   y             bf16 [T, N]  out:  (sum_k x[t][k] w[n][k]) * x_scales[t] * w_scales[n] + bias[n]
 *   ws, ws_bytes  device scratch of at least moe_matmul_int8_workspace_bytes(); not to be shared by
 *                 calls that overlap
 *
 * The integer sums are exact, so results depend neither on how a call is cut up (by its sizes and the
 * compute-unit budget, which the workspace's size depends on too) nor on the other rows;
 * scales and bias are applied in fp32 in this order, y is rounded once.  A token's NaN scale is
 * in its row alone.
 * Errors: INVALID_ARGUMENT for T < 0, N < 1, K not a positive multiple of 16, null or misaligned
 * pointers; UNSUPPORTED for K > 131056, T > 2^20, N > 2^24 or T N > 2^37; WORKSPACE_TOO_SMALL.
 *
 * moe_gated_int8 - both projections of a gated block, its activation and product:
 *   h[t][f] = silu(g) * u,   g = x Wg^T, u = x Wu^T as above, in fp32; h bf16 [T, F], rounded once.
 *   silu(g) = g / (1 + exp(-g)) is 0 for g below -87.3, where it is smaller than 1.03e-36
 *   wg, wu        packed codes [F, K]
 * Errors as moe_matmul_int8.
 */
size_t moe_matmul_int8_workspace_bytes(int64_t T, int32_t N, int32_t K);
moe_status moe_matmul_int8(const int8_t* x, const float* x_scales, const int8_t* w, const float* w_scales,
                           const void* bias, int64_t T, int32_t N, int32_t K, void* y, void* ws, size_t ws_bytes,
                           moe_stream stream);
size_t moe_gated_int8_workspace_bytes(int64_t T, int32_t F, int32_t K);
moe_status moe_gated_int8(const int8_t* x, const float* x_scales, const int8_t* wg, const float* wg_scales,
                          const int8_t* wu, const float* wu_scales, int64_t T, int32_t F, int32_t K, void* h, void* ws,
                          size_t ws_bytes, moe_stream stream);

/*
 * Per-kernel timing (a benchmarking aid, not part of the layer).
 *
 * moe_profiler_start(capacity) creates `capacity` pairs of HIP events on the
 * current device and enables recording: every kernel the library launches
 * afterwards is bracketed by one pair, recorded on its launch stream, until the
 * pool is used up or moe_profiler_stop() is called.  Creating the events is the
 * only allocation, and it happens here, not in the layer calls.  After the
 * caller synchronizes, moe_profiler_record(i, &name, &ms) returns the i-th
 * launch's kernel name (a static string) and its duration in milliseconds.
 * moe_profiler_select(name) restricts recording to launches of the kernel of
 * that name (as moe_profiler_record reports it, e.g. "ffn_gemm1_gate_up"), so
 * that timing one kernel leaves the others' launches untouched; NULL or ""
 * records every launch again.  It applies to launches made after the call.
 * Errors: INVALID_ARGUMENT for capacity < 1 or an index out of range; HIP for
 * an event failure (e.g. the record's stream has not completed).
 */
moe_status moe_profiler_start(int capacity);
moe_status moe_profiler_select(const char* name);
moe_status moe_profiler_stop(void);
int moe_profiler_count(void);
moe_status moe_profiler_record(int i, const char** name, float* ms);

/*
 * moe_set_cu_budget - compute units the library plans its persistent grids for
 * (a scheduling knob, not part of the layer).
 *
 * The bf16 and MXFP8 grouped GEMMs for large groups, route and the MXFP8 quantizer
 * launch one workgroup per compute unit (or a multiple of that) and share out their
 * work among them.  With n > 0 they plan for n compute units instead of the
 * device's count (values above the device's count are used as given), so a
 * caller can leave compute units to concurrent streams; the grouped GEMMs then run
 * these kernels for small groups too, where a kernel with one workgroup per tile is
 * otherwise faster.  The fp32 GEMMs, the fused router and moe_matvec_int4 choose their tiles
 * by it, as do moe_matmul_int8 and moe_gated_int8; moe_norm_join and moe_quantize_int8 share out their rows.  The first
 * kernel of moe_few_tokens is persistent too; its down projection, and
 * moe_kv8_attention over long sequences, are cut into parts for n compute units (with more
 * tiles than that, a workgroup for each tile).
 * n = 0 restores the device's count.  Results do not depend on it beyond fp32
 * rounding: the order of the GEMMs' sums depends on the kernel, and how the down
 * projection's last round of tiles is split along k on the grid.  (moe_kv8_attention's depend
 * on it by the rounding of its probabilities too, which are relative to a maximum of each part.)
 * Process-wide; set it between calls, not while other host threads launch.
 * Errors: INVALID_ARGUMENT for n < 0.
 */
moe_status moe_set_cu_budget(int32_t n);

#ifdef __cplusplus
}
#endif

#endif /* MOE_H */
