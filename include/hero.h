/* hero.h -- C ABI of libhero: the W8A8 transformer-layer forward of ZeroQuant-HERO
 * (arXiv 2310.17723) for AMD MI355X (gfx950).
 *
 * Common rules for every entry point
 *   - All data pointers are DEVICE pointers owned by the caller, 16-byte aligned, valid
 *     until the work enqueued by the call has finished.  Nothing is retained afterwards.
 *   - The library allocates no device memory and keeps no state between calls.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  Calls only
 *     enqueue work; they never synchronise with the host.
 *   - Arguments are validated on the host BEFORE anything is launched; on error nothing
 *     has been enqueued and a non-zero hero_status is returned.  No exceptions cross the ABI.
 *   - Sizes and strides are int64_t, in ELEMENTS.  Outputs must not alias inputs unless
 *     the entry point says so.
 *   - Numeric conventions (Sec. 2.1 quantizes symmetrically and uniformly to 8-bit integers): codes
 *     lie in [-127,127]; rounding is to nearest, ties to even; a dynamic scale is absmax/127 (1.0 for an
 *     all-zero row).  Integer contractions are exact in int32.  The DEFINITION of every quantization
 *     divides by the scale with IEEE fp32 division, and the entry points whose results are bit-exact
 *     against that definition compute exactly that: REQUANT / DEQUANT / raw GeMM^quant (their scales are
 *     multiplied, never divided by), LN^quant without LayerNorm (pure token-wise quantization), the
 *     weight preparation.  Three places multiply by a reciprocal instead, all behind fp32 transcendental
 *     or statistical arithmetic whose own rounding already differs from the definition's, so that their
 *     codes agree with it up to +-1 step on <= 0.1 % of the elements (the tolerance class of those paths):
 *     LN^quant behind a LayerNorm (v_rcp_f32 of the row scale, v_rsq_f32 of the variance), GELU^quant
 *     (1 / S_a[j]: v_rcp_f32 in the persistent kernel, the correctly rounded quotient in the others), and
 *     Softmax^quant (the normaliser and 1 / S_p are folded into the exponent).
 *   - The kernel an entry point runs is chosen from the problem size alone; the library reads no
 *     environment variable.  (include/hero_debug.h has test hooks that force a kernel.)
 */
#ifndef HERO_H
#define HERO_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    HERO_OK = 0,
    HERO_ERR_NULL = 1,        /* a required pointer is NULL                           */
    HERO_ERR_SHAPE = 2,       /* a size is negative / inconsistent                    */
    HERO_ERR_ALIGN = 3,       /* a pointer or leading dimension breaks 16-byte rule   */
    HERO_ERR_UNSUPPORTED = 4, /* valid request this build has no kernel for           */
    HERO_ERR_WORKSPACE = 5,   /* workspace missing or too small                       */
    HERO_ERR_LAUNCH = 6       /* the HIP runtime refused a launch                     */
} hero_status;

typedef enum { HERO_I8 = 0, HERO_U8 = 1, HERO_I32 = 2, HERO_F16 = 3, HERO_BF16 = 4, HERO_F32 = 5,
               HERO_F8E4M3 = 6 /* OCP E4M3: bias 7, max 448, no infinities */ } hero_dtype;

typedef enum {
    HERO_EPI_RAW_I32 = 0,      /* C = acc                                   (int32)        */
    HERO_EPI_DEQUANT = 1,      /* C = y (+ residual)                        (f16/bf16)     */
    HERO_EPI_DEQUANT_GELU = 2, /* C = GELU(y)                               (f16/bf16)     */
    HERO_EPI_REQUANT = 3,      /* C = sat(rne(y))                           (int8)         */
    HERO_EPI_GELU_REQUANT = 4  /* C = sat(rne(GELU(y) / out_col_scale[j]))  (int8; +-1 LSB class, see above) */
} hero_epilogue;

typedef enum { HERO_MASK_NONE = 0, HERO_MASK_PADDING = 1, HERO_MASK_CAUSAL = 2 } hero_mask;

const char* hero_strerror(hero_status s);

/* LN^quant: LayerNorm of the SUM of its inputs with a token-wise (TWQ) INT8 output.
 * Paper: Sec. 2.1 (TWQ is computed on the fly and fused into LayerNorm), Sec. 2.2.2 last
 * line of the quantized attention flow  S_out X_out,int8 = LN^quant(S_in X_in,int8, X_o,int8 S_o),
 * Sec. 2.2.3 last line of the quantized MLP flow.
 *
 *   s[i][j] = x[i][j] * x_row_scale[i] + r[i][j] * r_col_scale[j]
 *   y       = (s - mean_j s) / sqrt(var_j s + eps) * gamma[j] + beta[j]     (biased variance)
 *   y_scale[i] = max_j |y[i][j]| / 127 ;  y_q[i][j] = sat(rne(y[i][j] / y_scale[i]))
 *
 *   x        [M,D] row-major.  HERO_I8 with x_row_scale[M] (TWQ), or HERO_BF16/HERO_F16
 *            with x_row_scale == NULL.
 *   r        optional second addend [M,D] (NULL = none): HERO_I8 with r_col_scale[D] (FWQ),
 *            or HERO_BF16/HERO_F16 with r_col_scale == NULL.
 *   gamma, beta  f32[D].  gamma == NULL: no LayerNorm, the sum itself is quantized per
 *            token (then beta must be NULL too).  beta may be NULL (= 0).
 *   y_q [M,D] int8 and y_scale[M] f32 are always written.
 *   y_hp     optional [M,D] copy of y in y_hp_dt (HERO_BF16/HERO_F16) for a BF16 consumer.
 *   The 8-bit inputs may hold OCP E4M3 codes instead (x_dt / r_dt = HERO_F8E4M3, the same scales; the
 *   FP8 variant of Sec. 2.1); two 8-bit addends must be of one format (else HERO_ERR_UNSUPPORTED).
 * Constraints: D % 16 == 0, 16 <= D <= 8192 for INT8 x, <= 4096 for 16-bit x (a row lives in one
 * wavefront's registers; HERO_ERR_UNSUPPORTED beyond).  M == 0 is a no-op.
 * Statistics are fp32 (mean, then variance about the mean) with the row held in registers.
 */
hero_status hero_ln_quant(const void* x, hero_dtype x_dt, const float* x_row_scale,
                          const void* r, hero_dtype r_dt, const float* r_col_scale,
                          const float* gamma, const float* beta, float eps,
                          int64_t M, int64_t D,
                          int8_t* y_q, float* y_scale, void* y_hp, hero_dtype y_hp_dt, void* stream);

/* LN^quant with a token-wise FP8 output (Sec. 2.1: the 8-bit format may be FP8): everything as for
 * hero_ln_quant, except
 *   y_scale[i] = max_j |y[i][j]| / 448 ;  y_q[i][j] = e4m3(y[i][j] / y_scale[i])
 * (OCP E4M3 bytes, IEEE fp32 division, round to nearest even, saturated to +-448): the A operand and
 * a_row_scale of hero_fp8_gemm. */
hero_status hero_ln_quant_fp8(const void* x, hero_dtype x_dt, const float* x_row_scale,
                              const void* r, hero_dtype r_dt, const float* r_col_scale,
                              const float* gamma, const float* beta, float eps,
                              int64_t M, int64_t D,
                              void* y_q, float* y_scale, void* y_hp, hero_dtype y_hp_dt, void* stream);

/* Embedding LN^quant.  Paper: Sec. 2.2.1,
 *   S_emb X_emb,int8 = LN^quant(S_xt X_t,int8, X_p, X_s)
 * the token embedding is stored as INT8 codes with one TWQ scale per table row, the (small) position
 * and sentence-type tables stay in 16-bit floating point; the LayerNorm of their sum is quantized
 * per token exactly as in hero_ln_quant:
 *   h[i][j] = tok_scale[t] * tok_table[t][j] + pos_table[p][j] (+ type_table[s][j]),
 *             t = tok_ids[i], p = pos_ids[i], s = type_ids[i]
 *   y = LayerNorm_j(h) * gamma + beta ;  y_scale[i] = max_j |y| / 127 ;  y_q = sat(rne(y / y_scale[i]))
 *   tok_ids, pos_ids, type_ids   int32[T] (device).  An index outside its table cannot be reported
 *            from an asynchronous call: it is clamped into the table.
 *   tok_table [V,D] int8, tok_scale [V] f32;  pos_table [P,D], type_table [NT,D] in pt_dt
 *            (HERO_BF16 / HERO_F16);  type_table == NULL: no third addend (type_ids ignored).
 *   gamma [D] required, beta [D] or NULL;  y_q [T,D] int8 and y_scale [T] f32 are written.
 * Constraints: D % 16 == 0, 16 <= D <= 8192; tables and y_q 16-byte aligned.  T == 0 is a no-op.
 */
hero_status hero_embed_ln_quant(const int32_t* tok_ids, const int32_t* pos_ids, const int32_t* type_ids,
                                const int8_t* tok_table, const float* tok_scale, int64_t V,
                                const void* pos_table, int64_t P,
                                const void* type_table, int64_t NT, hero_dtype pt_dt,
                                const float* gamma, const float* beta, float eps,
                                int64_t T, int64_t D, int8_t* y_q, float* y_scale, void* stream);

/* GeMM^quant: INT8 x INT8 -> INT32 GEMM with the dequantization and the static FWQ/SQ
 * scales fused behind it.  Paper: Sec. 2.1 (Y = XW, column-wise weight scales, weights in
 * column-major format), Sec. 2.2.2 (dequantization and pre-determined scales fused into
 * the INT8 GeMM; X_q,int8 = Round(GeMM^quant(X_in,int8, W_q,int8, S_in, S_q)) once S_q is
 * folded into the weight), Sec. 2.2.3 (GELU^quant).
 *
 *   acc[i][j] = sum_k A[i][k] * Bt[j][k]                      exact int32
 *   t = float(acc);  t = t * a_row_scale[i]  (skipped if NULL);
 *   y = fma(t, b_col_scale[j], bias[j])      (bias NULL = 0)   -- this order, fp32
 *   then the epilogue `epi` (see hero_epilogue).  GELU is the exact erf form.
 *
 *   A   [M,K] int8 row-major, leading dimension lda.
 *   Bt  [N,K] int8, K contiguous (the paper's column-major W[K,N]), leading dimension ldb.
 *   residual  optional [M,N] HERO_BF16/HERO_F16 (DEQUANT only), leading dimension ldr; added
 *       in fp32 before the final rounding.  C may alias residual when ldc == ldr and the
 *       dtypes match (in-place residual stream).
 *   out_col_scale[N]  required for GELU_REQUANT (the FWQ scale S_a), ignored otherwise.
 *   C   [M,N] in c_dt, leading dimension ldc: HERO_I32 (RAW), HERO_F16/HERO_BF16 (DEQUANT*),
 *       HERO_I8 (REQUANT*).  Other pairs -> HERO_ERR_UNSUPPORTED.
 * Constraints: K % 64 == 0; lda, ldb multiples of 16; ldc, ldr multiples of 4; base
 * pointers 16-byte aligned; M, N arbitrary (>= 0; zero is a no-op); M < 2^23 (HERO_ERR_SHAPE beyond).
 * The tile shape is chosen from the problem size; every choice gives the same result.
 */
hero_status hero_int8_gemm(const int8_t* A, int64_t lda, const float* a_row_scale,
                           const int8_t* Bt, int64_t ldb, const float* b_col_scale,
                           const float* bias, const void* residual, hero_dtype res_dt, int64_t ldr,
                           hero_epilogue epi, const float* out_col_scale,
                           void* C, hero_dtype c_dt, int64_t ldc,
                           int64_t M, int64_t N, int64_t K, void* stream);

/* The same GeMM^quant (Sec. 2.1, 2.2.2, 2.2.3; identical arguments, results and constraints) with a
 * caller-owned scratch buffer for skinny problems with a long K (M <= 128, K >= 8192, N <= 8192:
 * the widest linear of a decode step): K is split over several workgroups per output tile so that
 * every CU streams a share of the weights; the exact
 * int32 partial sums go through the scratch and a second kernel adds them and applies the
 * epilogue, so the result does not depend on the split.
 *   hero_int8_gemm_workspace_bytes(M, N, K): bytes of scratch this shape can use (0: it would not
 *       split; any buffer, or none, is accepted then).
 *   workspace  device memory, 256-byte aligned (else HERO_ERR_WORKSPACE), at least that many bytes
 *       (NULL or smaller: the call runs like hero_int8_gemm).  Pure scratch: no initialisation is
 *       needed and nothing is kept between calls, so consecutive calls ON ONE STREAM can share it;
 *       calls that may overlap on the GPU (different streams) need buffers of their own.
 */
size_t hero_int8_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K);
hero_status hero_int8_gemm_ws(const int8_t* A, int64_t lda, const float* a_row_scale,
                              const int8_t* Bt, int64_t ldb, const float* b_col_scale,
                              const float* bias, const void* residual, hero_dtype res_dt, int64_t ldr,
                              hero_epilogue epi, const float* out_col_scale,
                              void* C, hero_dtype c_dt, int64_t ldc,
                              int64_t M, int64_t N, int64_t K,
                              void* workspace, size_t workspace_bytes, void* stream);

/* hero_int8_gemm for callers that cannot allocate or pass device scratch: code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc.  Arguments, results (bit for bit) and constraints are those of
 * hero_int8_gemm_ws; the split-K scratch is a fixed array of HERO_STATIC_SCRATCH_BYTES inside the library (one
 * copy per GPU, held until the process ends) instead of a caller's buffer.  The call allocates nothing.
 *   - A shape whose split needs more than HERO_STATIC_SCRATCH_BYTES (hero_int8_gemm_workspace_bytes(M, N, K))
 *     is refused with HERO_ERR_WORKSPACE before anything is launched; shapes that do not split need no scratch
 *     and always run.
 *   - Every call on one GPU shares that GPU's array: calls that may overlap on the GPU (different streams,
 *     concurrently replayed graphs) race on it.  Calls on one stream are ordered and safe.  The array is pure
 *     scratch: every plane is written before it is read, nothing needs clearing between calls.
 *   - The device current at the call must be the one `stream` belongs to. */
#define HERO_STATIC_SCRATCH_BYTES (16u << 20)
hero_status hero_int8_gemm_static(const int8_t* A, int64_t lda, const float* a_row_scale,
                                  const int8_t* Bt, int64_t ldb, const float* b_col_scale,
                                  const float* bias, const void* residual, hero_dtype res_dt, int64_t ldr,
                                  hero_epilogue epi, const float* out_col_scale,
                                  void* C, hero_dtype c_dt, int64_t ldc,
                                  int64_t M, int64_t N, int64_t K, void* stream);

/* The FP8 variant of GeMM^quant (Sec. 2.1 names FP8 as an 8-bit format the method applies to as well): the
 * same operation and epilogue as hero_int8_gemm with OCP E4M3 operands and fp32 accumulation on the
 * matrix cores.
 *   acc[i][j] = sum_k A[i][k] * Bt[j][k]     every product exact; the sum in fp32 (hardware order)
 *   then t = acc * a_row_scale[i] (skipped if NULL); y = fma(t, b_col_scale[j], bias[j]); epilogue:
 *   DEQUANT / DEQUANT_GELU -> C in HERO_F16 / HERO_BF16 (residual as for hero_int8_gemm);
 *   REQUANT -> e4m3(y), GELU_REQUANT -> e4m3(GELU(y) / out_col_scale[j]): C in HERO_F8E4M3, round
 *   to nearest even, saturated to +-448.  HERO_EPI_RAW_I32 does not exist here.
 *   A [M,K], Bt [N,K] E4M3 bytes, K contiguous.  Constraints as for hero_int8_gemm.
 * Token-wise FP8 activations use scale = max|x| / 448 per row; static scales fold as for INT8.
 * The order of the fp32 accumulation depends on the kernel the library picks for a shape (fixed for this entry point and
 * build; inside hero_layer_fwd a long K is split where its workspace has room for that), so results are reproducible but
 * not bit-identical across kernels. */
hero_status hero_fp8_gemm(const void* A, int64_t lda, const float* a_row_scale,
                          const void* Bt, int64_t ldb, const float* b_col_scale,
                          const float* bias, const void* residual, hero_dtype res_dt, int64_t ldr,
                          hero_epilogue epi, const float* out_col_scale,
                          void* C, hero_dtype c_dt, int64_t ldc,
                          int64_t M, int64_t N, int64_t K, void* stream);

/* INT8 attention: QK^T, Softmax^quant, PV.  Paper: Sec. 2.2.2 quantized flow
 *   A = S_q S_k X_q,int8 X_k,int8^T / sqrt(d)   (not quantized; d~ = S_q S_k / sqrt(d))
 *   S_p P_int8 = Softmax^quant(A)               (unsigned codes: softmax has no negatives)
 *   X_attn,int8 S_attn = S_p S_v P_int8 X_v,int8
 * Per (batch b, head h), query i, key k, channel e (j = h*Dh + e):
 *   a[i][k]  = float(sum_e q k) * qk_scale                 keys outside the mask are left out
 *   p        = softmax_k(a)   (fp32);   P[i][k] = sat_[0,255](rne(p / p_scale))
 *   acc[i][e]= sum_k P[i][k] * v[k][e]                     exact int32
 *   out_dt == HERO_I8 :  out[b*Sq+i][j] = sat(rne(float(acc) * out_col_scale[j]))
 *   out_dt == HERO_BF16/HERO_F16 :  out = float(acc) * out_col_scale[0]   (out_scale_is_scalar = 1)
 *
 *   q [B,Sq,H,Dh], k/v [B,Skv,H,Dh] int8 given by a base pointer and 4 element strides in
 *   the order (batch, position, head, channel); the channel stride must be 1 and the
 *   others multiples of 16, so the operands can be views into a fused [T,3d] QKV buffer
 *   or a [B,H,Smax,Dh] KV cache.
 *   mask: key k is visible to query i iff k < kv_len[b] (when kv_len != NULL; required for
 *   HERO_MASK_PADDING) and, for HERO_MASK_CAUSAL, k <= i + (len_b - Sq) with len_b =
 *   min(kv_len[b], Skv) (or Skv): the last query sees the last valid key.  With
 *   HERO_MASK_PADDING and Sq == Skv (self-attention over a padded batch) the positions
 *   i >= kv_len[b] are padding as queries too and see no key.  A query that sees no key
 *   outputs 0.  The same rules hold for every attention entry point of this header.
 *   out [B*Sq, H*Dh] row-major with leading dimension ldo.
 * Constraints: Dh in {64, 128}; B, H, Sq, Skv >= 0 (zero is a no-op).
 * The softmax is normalised BEFORE it is quantized, as the equation says, so the kernel
 * makes two passes over the keys (row max and sum first, codes and PV second).
 */
hero_status hero_int8_attn(const int8_t* q, const int64_t q_strides[4],
                           const int8_t* k, const int64_t k_strides[4],
                           const int8_t* v, const int64_t v_strides[4],
                           int64_t B, int64_t H, int64_t Sq, int64_t Skv, int64_t Dh,
                           float qk_scale, float p_scale, const float* out_col_scale, int out_scale_is_scalar,
                           hero_mask mask, const int32_t* kv_len,
                           void* out, hero_dtype out_dt, int64_t ldo, void* stream);

/* INT8 attention with an ONLINE Softmax^quant: a single-sweep VARIANT of the flow above, not the
 * equation of Sec. 2.2.2 (which normalises before it quantizes).  The probabilities are quantized
 * un-normalised, in blocks of 64 keys, against the running row maximum, and normalised once at the
 * end; the largest weight of a row always has code 255 whatever the sequence length.
 * Per (b, h), query i, visible keys 0 .. n-1 in blocks t = [64t, 64t + 64) (aligned to key 0):
 *   a[k]   = float(sum_e q k) * qk_scale_h[h]              one d~ per head (device array f32[H])
 *   m_t    = max(m_{t-1}, max_{k in t} a[k])               running maximum
 *   c[k]   = sat_[0,255](rne(255 exp(a[k] - m_t)))         unsigned codes of block t
 *   O[e]   = sum_t exp(m_t - m_T) sum_{k in t} c[k] v[k][e]   (integer inner sums, exact)
 *   L      = sum_t exp(m_t - m_T) sum_{k in t} c[k]
 *   y      = O[e] / L * out_col_scale[j] / p_scale ;  INT8: sat(rne(y)), 16-bit: y with
 *            out_col_scale[0]
 * out_col_scale and p_scale mean what they mean for hero_int8_attn (S_p S_v / S_attn[j] and S_p;
 * S_p cancels), so the two are interchangeable; masks, strides, constraints and errors are the
 * same, plus HERO_ERR_NULL without qk_scale_h.  Any Sq runs through the same kernel (a one-query
 * decode call is served but not specialised). */
hero_status hero_int8_attn_online(const int8_t* q, const int64_t q_strides[4],
                                  const int8_t* k, const int64_t k_strides[4],
                                  const int8_t* v, const int64_t v_strides[4],
                                  int64_t B, int64_t H, int64_t Sq, int64_t Skv, int64_t Dh,
                                  const float* qk_scale_h, float p_scale, const float* out_col_scale,
                                  int out_scale_is_scalar, hero_mask mask, const int32_t* kv_len,
                                  void* out, hero_dtype out_dt, int64_t ldo, void* stream);

/* FP8 attention: the quantized attention flow of Sec. 2.2.2 with E4M3 as the 8-bit format (Sec. 2.1
 * allows INT8 or FP8).  q, k, v hold OCP E4M3 bytes (device; the same shapes, element strides and
 * views as hero_int8_attn).  Per (b, h), query i, visible keys k:
 *   a[k]  = (sum_e q[i][e] k[k][e]) * qk_scale          fp32 accumulation on the matrix cores
 *   p     = softmax(a)                                   fp32, normalised BEFORE it is quantized
 *   P_f8  = e4m3(min(p / p_scale, 448))                  non-negative E4M3 codes; p_scale = 1/448 maps
 *                                                        p = 1 to the largest code
 *   acc[e] = sum_k P_f8[k] v[k][e]                       fp32 accumulation on the matrix cores
 *   out_dt HERO_F8E4M3: e4m3(sat(acc[e] * out_col_scale[h*Dh+e])), out_col_scale = S_p S_v / S_attn[j]
 *   out_dt HERO_F16 / HERO_BF16: acc[e] * out_col_scale[0]  (out_scale_is_scalar must be 1)
 * Masks, kv_len, constraints (Dh 64 or 128, strides multiples of 16, 16-byte aligned bases, ldo) and
 * errors as for hero_int8_attn; the 8-bit output type is HERO_F8E4M3 (HERO_I8 -> HERO_ERR_UNSUPPORTED).
 * A query with no visible key outputs 0.  A one-query call (Sq == 1, Skv <= 16384) takes the
 * cache-streaming kernel, as for INT8 (fp32 sums on the vector ALU there).  The matrix cores add the 8 products of a lane group with 13
 * fractional bits below the largest of them, so results agree with an exactly accumulated reference
 * up to an adjacent E4M3 code on a small fraction of the outputs, not bit for bit. */
hero_status hero_fp8_attn(const void* q, const int64_t q_strides[4],
                          const void* k, const int64_t k_strides[4],
                          const void* v, const int64_t v_strides[4],
                          int64_t B, int64_t H, int64_t Sq, int64_t Skv, int64_t Dh,
                          float qk_scale, float p_scale, const float* out_col_scale, int out_scale_is_scalar,
                          hero_mask mask, const int32_t* kv_len,
                          void* out, hero_dtype out_dt, int64_t ldo, void* stream);

/* ---- one transformer layer (Sec. 2.2.2 + 2.2.3 chained, Sec. 2.3 / Table 1 modes) ---- */

typedef enum { HERO_ARCH_POST_LN = 0, HERO_ARCH_PRE_LN = 1 } hero_arch;

/* mode_mask: one bit per switchable module (Sec. 2.3; the columns of Table 1 after "Embedding"); set = INT8,
 * clear = 16-bit.  Table 1's modes are HERO_MODE_M1 / M2 / M3; HERO_MODE_M0 (no module bit) is the all-16-bit
 * layer, the FP16 row of Table 2.  A 16-bit module hands 16-bit values on and the method has no stand-alone
 * quantization kernel, so: ATTN set needs QKV set (the INT8 attention reads SQ codes), ATTN_OUT set needs ATTN
 * set, FC2 set needs FC1 set (GELU^quant codes); any other subset is HERO_ERR_UNSUPPORTED.
 * HERO_M_F16: the 16-bit type of the layer -- switched modules, the 16-bit copies between them, the PRE_LN
 * residual stream h -- is FP16 instead of BF16.
 * HERO_M_FP8 (only together with all five module bits): the 8-bit format of the whole layer is OCP E4M3
 * instead of INT8 (Sec. 2.1).  Every int8_t* of hero_layer_weights / hero_layer_io then holds E4M3 bytes
 * (weights quantized column-wise to max|column| / 448, static scales calibrated to 448, p_scale = 1/448),
 * and the layer runs hero_ln_quant_fp8 / hero_fp8_gemm / hero_fp8_attn in place of the INT8 entry points. */
enum { HERO_M_QKV = 1, HERO_M_ATTN = 2, HERO_M_ATTN_OUT = 4, HERO_M_FC1 = 8, HERO_M_FC2 = 16, HERO_M_FP8 = 32,
       HERO_M_F16 = 64 };
#define HERO_MODE_M3 (HERO_M_QKV | HERO_M_ATTN | HERO_M_ATTN_OUT | HERO_M_FC1 | HERO_M_FC2)
#define HERO_MODE_M2 (HERO_M_QKV | HERO_M_ATTN | HERO_M_ATTN_OUT | HERO_M_FC1)
#define HERO_MODE_M1 (HERO_M_QKV | HERO_M_FC1)
#define HERO_MODE_M0 0

typedef struct {
    int32_t arch;       /* hero_arch                                          */
    int32_t d, H, Dh, f; /* hidden width, heads, head width (H*Dh == d), FFN width */
    float eps;          /* LayerNorm epsilon                                  */
    int32_t mask;       /* hero_mask                                          */
    uint32_t mode_mask; /* HERO_M_* bits                                      */
} hero_layer_desc;

/* Prepared (folded, column-quantized) parameters, all device pointers.  INT8 weights are
 * [N][K] (K contiguous); *_s are their f32 column scales; biases are f32 and already
 * folded with the output scale where the output is requantized.  A 16-bit module takes its
 * weight in *_bf16 / *_hp ([N][K] in the layer's 16-bit type -- bf16, or fp16 with HERO_M_F16 --,
 * unfolded) and ignores the INT8 fields. */
typedef struct {
    const int8_t* w_qkv; const float* w_qkv_s; const float* b_qkv;          /* [3d][d] */
    const int8_t* w_o;   const float* w_o_s;   const float* b_o;            /* [d][d]  */
    const int8_t* w_1;   const float* w_1_s;   const float* b_1;            /* [f][d]  */
    const int8_t* w_2;   const float* w_2_s;   const float* b_2;            /* [d][f]  */
    const void* w_o_bf16; const void* w_2_bf16;                             /* 16-bit attention-output / FC2 */
    const float* ln1_g; const float* ln1_b; const float* ln2_g; const float* ln2_b;
    const float* S_o;   /* [d] FWQ scale of X_o  (POST_LN, INT8 attention-output)      */
    const float* S_x2;  /* [d] FWQ scale of X_2  (POST_LN, INT8 FC2)                   */
    const float* S_a;   /* [f] FWQ scale of A = GELU(X_1) (INT8 FC2)                   */
    const float* attn_out_scale; /* [d] S_p S_v / S_attn[j] (INT8 attention-output) or
                                    1 float S_p S_v (16-bit attention-output)          */
    float qk_scale;     /* d~ = S_q S_k / sqrt(Dh)  (INT8 attention) or 1/sqrt(Dh) (16-bit) */
    float p_scale;      /* S_p                                                         */
    const void* w_qkv_hp; const void* w_1_hp;                               /* 16-bit QKV / FC1 */
} hero_layer_weights;

typedef struct {
    int64_t B, S;            /* sequences and new tokens per sequence; T = B*S rows    */
    /* POST_LN: TWQ input (read when the QKV module is INT8) and output (always written) */
    const int8_t* x_q; const float* x_scale;     /* [T,d] int8, [T] f32               */
    int8_t* out_q;     float* out_scale;         /* [T,d] int8, [T] f32               */
    /* PRE_LN: 16-bit residual stream, updated IN PLACE */
    void* h;                                     /* [T,d] bf16 (fp16 with HERO_M_F16)  */
    const int32_t* kv_len;   /* [B] visible keys per sequence INCLUDING this call's S tokens;
                                NULL = S for every sequence (no cache, no padding)     */
    /* optional INT8 KV cache [B,H,Smax,Dh] (PRE_LN or POST_LN; INT8 attention only): this call's K/V codes
       are written at positions kv_len[b]-S .. kv_len[b]-1 and attention reads the cache.   */
    int8_t* k_cache; int8_t* v_cache; int64_t Smax;
    /* POST_LN with a 16-bit QKV module: the layer input [T,d] in the layer's 16-bit type (x_q / x_scale are then
       not read).  out_hp (optional, any mode): the 16-bit copy of the layer output, i.e. the x_hp of a successor
       whose QKV module is 16-bit. */
    const void* x_hp; void* out_hp;
    /* optional hint (may be NULL / 0; never written, changes no result): device memory that the caller's NEXT call
       reads first, typically the next layer's w_qkv.  The layer's last GeMM^quant requests its lines while it runs, so
       that they wait in the cache hierarchy instead of in HBM when the next call's first tiles ask for them.  At most
       next_read_bytes bytes from next_read are read; 4-byte aligned; a region above 8 MB is ignored (it would not
       survive in the cache until it is used). */
    const void* next_read; size_t next_read_bytes;
} hero_layer_io;

/* Bytes of scratch hero_layer_fwd can use for T = B*S rows of this layer.  Part of it is scratch for the K split of the GEMMs,
 * which only some sizes have, so a smaller T may ask for more than a larger one.  Where E4M3 or 16-bit modules, or INT8 ones of more than
 * 128 rows, are what asks for that part, a workspace without it is accepted and they run in one pass (fp32 sums are then ordered
 * otherwise, INT8's are the same); INT8 modules of T <= 128 rows and K >= 8192 insist on theirs (of 32 rows and fewer only those
 * whose K is split all the same). */
size_t hero_layer_workspace_bytes(const hero_layer_desc* desc, int64_t B, int64_t S);

/* One W8A8 layer: enqueues LN^quant, the four GeMM^quant, the attention and (POST_LN) the
 * closing LN^quant on `stream`, with no host synchronisation.  Paper: Sec. 2.2.2, 2.2.3,
 * Sec. 2.3 Table 1.  `workspace` is device scratch of
 * hero_layer_workspace_bytes() bytes (see there for what may be missing), 256-byte aligned, owned by the caller; its contents
 * are undefined afterwards.  Supported mode masks: see mode_mask above. */
hero_status hero_layer_fwd(const hero_layer_desc* desc, const hero_layer_weights* w, const hero_layer_io* io,
                           void* workspace, size_t workspace_bytes, void* stream);

/* 16-bit side of a switched module (Sec. 2.3, Table 1: a module that is not INT8 runs in FP16 / BF16):
 * C = act(A Wt^T + bias) (+ residual).  dt = HERO_BF16 or HERO_F16 is the type of A [M,K] (lda), Wt [N][K] (ldb),
 * residual [M,N] or NULL (ldr; C may alias it) and C [M,N] (ldc); bias f32[N] or NULL; gelu != 0 applies erf-GELU
 * before the residual.  fp32 accumulation on the matrix cores.  Constraints: K % 32 == 0; lda, ldb multiples of 8,
 * ldc, ldr of 4; base pointers 16-byte aligned.  hero_bf16_gemm is hero_hp_gemm with dt = HERO_BF16. */
hero_status hero_hp_gemm(const void* A, int64_t lda, const void* Wt, int64_t ldb,
                         const float* bias, const void* residual, int64_t ldr, int gelu,
                         void* C, int64_t ldc, int64_t M, int64_t N, int64_t K, hero_dtype dt, void* stream);
hero_status hero_bf16_gemm(const void* A, int64_t lda, const void* Wt, int64_t ldb,
                           const float* bias, const void* residual, int64_t ldr, int gelu,
                           void* C, int64_t ldc, int64_t M, int64_t N, int64_t K, void* stream);

/* 16-bit attention core softmax(q k^T * scale) v with the same operand description and mask rules as
 * hero_int8_attn (strides multiples of 8 elements); q, k, v and out [B*Sq, H*Dh] in dt (HERO_BF16 / HERO_F16).
 * hero_bf16_attn is hero_hp_attn with dt = HERO_BF16. */
hero_status hero_hp_attn(const void* q, const int64_t q_strides[4],
                         const void* k, const int64_t k_strides[4],
                         const void* v, const int64_t v_strides[4],
                         int64_t B, int64_t H, int64_t Sq, int64_t Skv, int64_t Dh, float scale,
                         hero_mask mask, const int32_t* kv_len, void* out, int64_t ldo, hero_dtype dt, void* stream);
hero_status hero_bf16_attn(const void* q, const int64_t q_strides[4],
                           const void* k, const int64_t k_strides[4],
                           const void* v, const int64_t v_strides[4],
                           int64_t B, int64_t H, int64_t Sq, int64_t Skv, int64_t Dh, float scale,
                           hero_mask mask, const int32_t* kv_len, void* out, int64_t ldo, void* stream);

/* ---- a KV cache in 8 bits with a scale for each block of tokens and head ----
 *
 * The cache that a 16-bit attention reads (Sec. 2.3: the attention module switched to 16 bits; the SQ codes of the INT8
 * attention have ONE calibrated scale per tensor and a cache of their own, hero_layer_io).  Here no scale is calibrated:
 * each is the absmax of a block of `block` tokens of one head, taken as the tokens are written.
 *
 *   k, v              codes, HERO_I8 or HERO_F8E4M3 (dt): n_blocks blocks of `block` tokens, H heads of width Dh, given by a base
 *                     pointer and 4 element strides in the order (block, position in the block, head, channel); the channel
 *                     stride must be 1, the others multiples of 16 that are not negative.  [n_blocks, H, block, Dh] keeps a head's block
 *                     in one piece.  The blocks of K and of V lie apart from each other (two views of one buffer will do).
 *   k_scale, v_scale  f32 [n_blocks, H]: token t of a block stands for codes[t] * scale.  Nothing needs clearing: a write that
 *                     begins a block (its first position is the block's first) sets its scales, whatever was there.  V's scales are positive
 *                     where tokens lie, and V's E4M3 codes there are numbers (all that a write makes are; in a cache from elsewhere a NaN among
 *                     V's codes may also reach rows that do not see its token).  K's scales may have either sign.
 *   block_table       int32 [B, max_blocks] (device): positions [j block, (j + 1) block) of sequence b lie in block block_table[b][j].
 *                     NULL: in block b max_blocks + j (n_blocks >= B max_blocks then).  An index outside [0, n_blocks) is no block:
 *                     nothing is written there, its keys are left out of the attention, its positions read as 0.  Sequences may
 *                     share blocks that are only read; a block that is written belongs to one sequence, once.
 * Constraints: Dh in {64, 128}; block in {16, 32, 64, 128}; max_blocks * block <= 2^30; B, H <= 65535; n_blocks < 2^31;
 * block times the position stride < 2^31.  The pointers are device pointers as everywhere; the structure itself is read during the call only. */
typedef struct {
    void* k; void* v;
    float* k_scale; float* v_scale;
    int64_t k_strides[4]; int64_t v_strides[4];
    const int32_t* block_table;
    int64_t B, max_blocks, n_blocks;
    int32_t H, Dh, block, dt;
} hero_kv_cache;

/* Quantises this call's K and V rows as it writes them into the cache.  Sequence b holds kv_len[b] tokens WITH this call's;
 * row s < n (n = new_len[b] clamped to [0, S], or S without new_len) is the token at position kv_len[b] - n + s; positions
 * outside [0, max_blocks * block) are left out, and rows s >= n are not read.  For every block with a new token, per head, K and V apart:
 *   a     = max |x| over the block's new tokens
 *   s_new = max(|s_old|, a / qmax, 2^-64)        qmax 127 (INT8) or 448 (E4M3), IEEE fp32 division;
 *                                                s_old = 0 if the block holds no token from before this call
 *   code  = sat(rne(x / s_new)) or e4m3(x / s_new), saturated          IEEE fp32 division
 *   and, where s_new != s_old, the tokens from before are coded anew: the code of fl(code s_old) at s_new.
 * A scale never shrinks while its block fills, so tokens cost their block a new coding only when they raise its largest value.  Each new
 * coding rounds anew: a block filled token by token has 1.25 to 1.35 (INT8) or 1.35 to 1.45 times (E4M3) the rms error of one written at once where its
 * tokens are of one size, 1.6 to 2.5 times where they grow from first to last.  A NaN or
 * infinity among the new tokens makes the scale NaN, and what is read from that block and head is NaN until it is begun anew.
 *   k, v  [B, S, H, Dh] in dt (HERO_BF16 / HERO_F16), base pointer and 4 element strides (batch, token, head, channel);
 *         channel stride 1, the others multiples of 8 (views into a fused QKV buffer will do).  B is the cache's.
 *   kv_len int32 [B] (device), required; new_len int32 [B] (device) or NULL: a padded batch.
 * B == 0, S == 0 or H == 0 is a no-op. */
hero_status hero_kv_write(const hero_kv_cache* cache, const void* k, const int64_t k_strides[4],
                          const void* v, const int64_t v_strides[4], hero_dtype dt, int64_t S,
                          const int32_t* kv_len, const int32_t* new_len, void* stream);

/* Reads positions start[b] + i, 0 <= i < S, back: out[b][i] = code * scale, rounded once to out_dt (HERO_BF16, HERO_F16 or
 * HERO_F32).  Positions outside [0, min(kv_len[b], max_blocks block)) are left as they were in the output.
 *   k_out, v_out  [B, S, H, Dh], base pointers and 4 element strides (batch, token, head, channel); channel stride 1, the others
 *                 multiples of 8.  Either may be NULL (only the other is read).
 *   start  int32 [B] (device) or NULL (0 for every sequence); kv_len int32 [B] (device), required.
 * S * H <= 2^31 - 256 and S * H * Dh < 2^36 (else HERO_ERR_SHAPE). */
hero_status hero_kv_read(const hero_kv_cache* cache, void* k_out, const int64_t k_strides[4],
                         void* v_out, const int64_t v_strides[4], hero_dtype out_dt, int64_t S,
                         const int32_t* start, const int32_t* kv_len, void* stream);

/* 16-bit attention over the cache, its codes and scales taken apart inside the kernel:
 *   out[b][i][hq] = softmax_k(scale q[b][i][hq] . K[b][k][h]) V[b][k][h],   K, V = codes * scales,  h = hq / (Hq / H)
 *   q    [B, Sq, Hq, Dh] in dt (HERO_BF16 / HERO_F16), base pointer and 4 element strides (batch, token, head, channel); channel
 *        stride 1, the others multiples of 8.  Hq is a multiple of the cache's H: grouped heads share a head of the cache.
 *   out  [B*Sq, Hq*Dh] in dt, leading dimension ldo (a multiple of 4).
 *   kv_len int32 [B] (device), required: tokens of each sequence, this call's n queries among them (they are written before).
 *   new_len int32 [B] (device) or NULL: n = new_len[b] (clamped to [0, Sq]) queries of sequence b, Sq without it.
 *   mask HERO_MASK_NONE: query i < n sees the keys k < len = min(kv_len[b], max_blocks block);  HERO_MASK_CAUSAL: of those k <= i + len - n.
 *        (HERO_MASK_PADDING -> HERO_ERR_UNSUPPORTED: new_len says it.)  A query that sees no key, i >= n among them, outputs 0.
 * The scores, the softmax and all sums are fp32; the probabilities (times the V scale of their block) are rounded to FP16 for
 * the second product whatever dt is, behind a shift that keeps them normal numbers down to 2^-29 of the row's largest; BF16
 * queries go through FP16 as well, each row times a power of two (exact down to 2^-29 of the row's largest).  (A block whose
 * V scale is more than 2^100 times smaller than another's that the row sees may be taken for one that it does not see.)
 * Few rows (Sq * Hq / H) over many keys are split along the keys when `workspace` has room: hero_kv_attn_workspace_bytes(cache,
 * Hq, Sq) bytes (0: this size is not split), device memory, 256-byte aligned (else HERO_ERR_WORKSPACE).  NULL or smaller: one piece (slower, and
 * fp32 sums are ordered otherwise).  Kernel and split go by max_blocks * block, not by the lengths: a table that is much wider than its
 * sequences are long costs speed.  Pure scratch, nothing is kept between calls: calls that may overlap on the GPU need
 * their own.  The order of the sums depends on the sizes alone, so results are reproducible.
 * B * Sq * Hq < 2^31, and workgroups (B * H for every 16 rows, where rows are that few) for less than 2^32 threads: else HERO_ERR_SHAPE. */
size_t hero_kv_attn_workspace_bytes(const hero_kv_cache* cache, int64_t Hq, int64_t Sq);
hero_status hero_kv_attn(const hero_kv_cache* cache, const void* q, const int64_t q_strides[4], hero_dtype dt,
                         int64_t Hq, int64_t Sq, float scale, hero_mask mask, const int32_t* kv_len, const int32_t* new_len,
                         void* out, int64_t ldo, void* workspace, size_t workspace_bytes, void* stream);

/* hero_layer_fwd with a block-scaled cache: a layer whose attention module is 16-bit (HERO_M_ATTN clear; else HERO_ERR_UNSUPPORTED)
 * writes this call's K and V into `kv` and attends over it (hero_kv_write, hero_kv_attn with qk_scale and the layer's mask; HERO_MASK_PADDING
 * asks for the same as HERO_MASK_NONE here), so that it prefills and decodes.  Everything else as for hero_layer_fwd.
 *   kv       the layer's cache, for io->B sequences of desc->H heads of width desc->Dh (else HERO_ERR_SHAPE); io->k_cache and
 *            io->v_cache are NULL.  io->kv_len [B], required, counts this call's tokens.
 *   new_len  int32 [B] (device) or NULL: of the S rows of sequence b the first new_len[b] are tokens (a padded batch; the
 *            other rows are computed without a key to attend to).  Without it S tokens have to fit the cache's positions (else HERO_ERR_SHAPE).
 *   workspace: hero_layer_kv_workspace_bytes(desc, kv, S) bytes; what hero_layer_fwd accepts without is accepted without here,
 *            and the attention of few rows is then not split. */
size_t hero_layer_kv_workspace_bytes(const hero_layer_desc* desc, const hero_kv_cache* kv, int64_t S);
hero_status hero_layer_fwd_kv(const hero_layer_desc* desc, const hero_layer_weights* w, const hero_layer_io* io,
                              const hero_kv_cache* kv, const int32_t* new_len,
                              void* workspace, size_t workspace_bytes, void* stream);

/* ---- the operators of a mixture-of-experts MLP (Sec. 2.2.3's two linears, one pair of weights per expert; the router and the weighted
 * sum are not the paper's) ----
 *
 * A router gives every token k of E experts; the rows of an expert are computed together.  Nothing about which expert has how many rows is
 * known to the host: `offsets` lies on the device, a call is enqueued for R rows at most, and no call waits for another's result.
 *
 *   LN^quant (codes, scales and y_hp) -> router logits (hero_hp_gemm of y_hp) -> hero_moe_route -> first linear, GELU^quant
 *   (hero_int8_gemm_grouped, row_index = row_token) -> second linear (DEQUANT, no row_index) -> hero_moe_combine into the residual stream
 *
 * hero_moe_route: the experts of every token, and the order of their rows.
 *   l[t][e]  = logits[t][e] in fp32; a NaN counts as -infinity, +infinity as the largest finite number
 *   chosen   the (up to) top_k experts of the largest l[t][e] > -infinity, falling, ties to the lowest index:
 *            expert[t][0], expert[t][1], ..; what is left of the top_k is -1 (a padding token: all its logits -infinity)
 *   weight[t][j] = exp(l[t][expert[t][j]] - m) / sum exp(l[t][e] - m), m = max_e l[t][e]; the sum over the chosen experts (renorm != 0) or
 *            over all E (renorm == 0), in fp32;  0 where expert[t][j] is -1
 *   offsets  the rows of expert e are offsets[e] .. offsets[e + 1] - 1, in the order of t * top_k + j; offsets[E] is their number
 *   slot[t][j]    the row of choice j of token t, or -1
 *   row_token[r]  the token of row r, or -1 (r >= offsets[E])
 *   logits [T,E] in dt (HERO_F32 / HERO_BF16 / HERO_F16), leading dimension ldl.  expert, slot int32 [T,top_k]; weight f32 [T,top_k];
 *   row_token int32 [T*top_k]; offsets int32 [E+1]: all are written whole.
 *   workspace: hero_moe_route_workspace_bytes(T, E, top_k) bytes (0 for few tokens), 256-byte aligned, else HERO_ERR_WORKSPACE.  Pure scratch:
 *            calls that may overlap on the GPU need their own.
 * Constraints: 1 <= E <= 512, 1 <= top_k <= 16, top_k <= E; T * top_k < 2^31, T <= 2^28 - 16 (what a launch holds; else HERO_ERR_SHAPE).  T == 0: offsets are
 * written, all 0.
 * The results depend on the arguments alone (no order of atomics shows in them). */
size_t hero_moe_route_workspace_bytes(int64_t T, int64_t E, int64_t top_k);
hero_status hero_moe_route(const void* logits, hero_dtype dt, int64_t ldl, int64_t T, int64_t E, int64_t top_k, int renorm,
                           int32_t* expert, float* weight, int32_t* slot, int32_t* row_token, int32_t* offsets,
                           void* workspace, size_t workspace_bytes, void* stream);

/* GeMM^quant of E experts in one call (Sec. 2.1, 2.2.3): the product of hero_int8_gemm with the weights, the column vectors and the number
 * of rows of each expert.  For the rows offsets[e] <= r < offsets[e + 1]:
 *   i = row_index ? row_index[r] : r
 *   acc[r][j] = sum_k A[i][k] * Bt[e][j][k];  t = float(acc) * a_row_scale[i] (skipped if NULL)
 *   y = fma(t, b_col_scale[e][j], bias[e][j]) (bias NULL = 0);  then the epilogue with out_col_scale[e][j]
 *   A    [MA,K] int8 row-major, leading dimension lda; MA == R without row_index.  a_row_scale f32[MA] or NULL.
 *   Bt   E matrices [N,K], K contiguous, leading dimension ldb, expert_stride elements apart.
 *   b_col_scale, bias, out_col_scale  f32 [E,N], contiguous.
 *   C    [R,N] in c_dt, leading dimension ldc; rows r >= offsets[E] are left as they were.
 *   offsets  int32 [E+1] (device), rising from 0 to at most R.  (Others cannot be reported from an asynchronous call: each is taken
 *        as the largest of those up to it, within [0, R], and the rows in front of offsets[0] belong to no expert.)
 *   row_index int32 [R] (device) or NULL; an index outside [0, MA) is clamped.  It is read below offsets[E] only.
 *   epi  HERO_EPI_DEQUANT, HERO_EPI_DEQUANT_GELU (C HERO_BF16 / HERO_F16), HERO_EPI_REQUANT, HERO_EPI_GELU_REQUANT (C HERO_I8);
 *        no residual (hero_moe_combine adds it).
 * Constraints: E <= 512; R < 2^23; K % 64 == 0; lda, ldb, expert_stride multiples of 16, ldc of 4; base pointers of A, Bt, C 16-byte aligned;
 * R * N such that a launch holds it (else HERO_ERR_SHAPE).  R == 0, N == 0 or E == 0 is a no-op.
 * Which kernel runs is chosen by R (taken as the number of rows: room for many more than there are costs time), E, N and K; results of 8-bit
 * integer operands do not depend on it.  E4M3 and 16-bit operands: the order in which a row's products are added (fp32) depends on the kernel and
 * on where the row's tile lies, so on the numbers of rows of all experts: the same call gives the same bits again, but the same row between other
 * rows, or twice in one call, may differ by the rounding of its sum.
 * hero_fp8_gemm_grouped: the same with OCP E4M3 operands (hero_fp8_gemm; 8-bit results are HERO_F8E4M3).
 * hero_hp_gemm_grouped: 16-bit operands (hero_hp_gemm): C = act(A Bt[e]^T + bias[e]) in dt; K % 32 == 0, lda, ldb, expert_stride
 * multiples of 8. */
hero_status hero_int8_gemm_grouped(const int8_t* A, int64_t lda, int64_t MA, const float* a_row_scale, const int32_t* row_index,
                                   const int8_t* Bt, int64_t ldb, int64_t expert_stride, const float* b_col_scale, const float* bias,
                                   hero_epilogue epi, const float* out_col_scale, void* C, hero_dtype c_dt, int64_t ldc,
                                   const int32_t* offsets, int64_t E, int64_t R, int64_t N, int64_t K, void* stream);
hero_status hero_fp8_gemm_grouped(const void* A, int64_t lda, int64_t MA, const float* a_row_scale, const int32_t* row_index,
                                  const void* Bt, int64_t ldb, int64_t expert_stride, const float* b_col_scale, const float* bias,
                                  hero_epilogue epi, const float* out_col_scale, void* C, hero_dtype c_dt, int64_t ldc,
                                  const int32_t* offsets, int64_t E, int64_t R, int64_t N, int64_t K, void* stream);
hero_status hero_hp_gemm_grouped(const void* A, int64_t lda, int64_t MA, const int32_t* row_index,
                                 const void* Bt, int64_t ldb, int64_t expert_stride, const float* bias, int gelu,
                                 void* C, int64_t ldc, const int32_t* offsets, int64_t E, int64_t R, int64_t N, int64_t K,
                                 hero_dtype dt, void* stream);

/* The weighted sum of every token's rows:  out[t] = residual[t] + sum_j weight[t][j] * y[slot[t][j]], in fp32 (the choices in their
 * order, the residual last), rounded once; a choice whose slot lies outside [0, R) is left out, whatever its weight.
 *   The rows y are 16 bits, as the second linear leaves them: each has been rounded once before the sum, which is rounded once more (the dense layer, whose
 *   second linear adds the residual itself, rounds once).
 *   y [R,D], residual [T,D] or NULL (= 0), out [T,D] in dt (HERO_BF16 / HERO_F16), leading dimensions ldy, ldr, ldo; out may be the residual
 *   itself (ldo == ldr).  slot int32 [T,top_k], weight f32 [T,top_k].
 * Constraints: D and the leading dimensions multiples of 8, base pointers 16-byte aligned, 1 <= top_k <= 16; T * D such that a launch holds it
 * (else HERO_ERR_SHAPE).  T == 0 or D == 0 is a no-op. */
hero_status hero_moe_combine(const void* y, int64_t ldy, int64_t R, const int32_t* slot, const float* weight,
                             const void* residual, int64_t ldr, void* out, int64_t ldo,
                             int64_t T, int64_t top_k, int64_t D, hero_dtype dt, void* stream);

/* Model-load-time operators (not on the hot path): the pre-processing phase of the method on the GPU.
 *
 * hero_absmax_cols -- calibration statistic of the static scales (Sec. 2.1: FWQ / SQ scales are
 *   calibrated in a pre-processing phase; Sec. 3: ranges recorded over calibration batches):
 *     col_absmax[j] = max(col_absmax[j], max_i |x[i][j]|)
 *   x [T,D] HERO_F32 / HERO_BF16 / HERO_F16, leading dimension ldx; col_absmax f32[D] is a RUNNING
 *   maximum (in/out: zero it before the first batch).  An FWQ scale is col_absmax[j] / 127, an SQ
 *   scale the maximum over j divided by 127.  Exact (a maximum has no rounding).
 *
 * hero_weight_fold_quant -- scale folding (Sec. 2.2.2: W~_q = W_q / S_q, W~_o = S_attn W_o / S_o;
 *   Sec. 2.2.3: W~_2 = S_a W_2 / S_x2) and column-wise weight quantization (Sec. 2.1):
 *     W~[k][n] = row_mult[k] * W[k][n] / col_div[n]     fp64: multiply, then divide; one cast to fp32
 *     col_scale[n] = max_k |W~[k][n]| / 127  (1 for an all-zero column)
 *     Wt[n][k] = sat(rne(W~[k][n] / col_scale[n]))       IEEE fp32 division
 *   W [K,N] f32 row-major (the paper's W: input rows, output columns), leading dimension ldw;
 *   row_mult f32[K] or NULL (= 1), col_div f32[N] or NULL (= 1); Wt [N,K] int8, leading dimension
 *   ldwt (K contiguous: the operand layout of hero_int8_gemm); col_scale f32[N].
 *   hero_weight_fold_quant_fp8: the FP8 variant (Sec. 2.1): the same fold, col_scale[n] = max / 448 and
 *   Wt[n][k] = e4m3(W~[k][n] / col_scale[n]) (OCP E4M3 bytes: the operand of hero_fp8_gemm).
 * All return HERO_ERR_SHAPE / HERO_ERR_NULL / HERO_ERR_UNSUPPORTED before any launch. */
hero_status hero_absmax_cols(const void* x, hero_dtype x_dt, int64_t ldx, int64_t T, int64_t D,
                             float* col_absmax, void* stream);
hero_status hero_weight_fold_quant(const float* W, int64_t ldw, const float* row_mult, const float* col_div,
                                   int64_t K, int64_t N, int8_t* Wt, int64_t ldwt, float* col_scale, void* stream);
hero_status hero_weight_fold_quant_fp8(const float* W, int64_t ldw, const float* row_mult, const float* col_div,
                                       int64_t K, int64_t N, void* Wt, int64_t ldwt, float* col_scale, void* stream);

/* Library build identification: target architecture string, e.g. "gfx950". */
const char* hero_build_arch(void);

#ifdef __cplusplus
}
#endif
#endif /* HERO_H */
