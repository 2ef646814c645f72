/*
 * svdcache.h — C ABI of the B200-native SVD-Cache hot path (sm_100a).
 *
 * SVD-Cache ("Forecast the Principal, Stabilize the Residual") splits the hidden
 * feature F (N tokens x D) of a DiT block into a rank-k principal part in a fixed,
 * pre-computed right-singular basis V_k and an orthogonal residual, forecasts the
 * principal part with an exponential moving average and reuses the residual:
 *
 *   one-off        V_k  = top-k right singular vectors of a stack of features  (Eq. 4-7)
 *   full step      C    = F V_k                                                (Eq. 8-9)
 *                  R    = F - C V_k^T                                          (Eq. 10)
 *                  Chat = C  on the first full step, else beta Chat + (1-beta) C (Eq. 11)
 *   cached step    Fhat = Chat V_k^T + R                                       (Sec. 3.5)
 *
 * Conventions
 *   - Every function returns an int status: SVDCACHE_OK or a negative SVDCACHE_ERR_*.
 *     Nothing throws.  svdcache_status_string() gives text.
 *   - "device" pointers are CUDA device addresses owned by the caller; "host" pointers
 *     are ordinary host addresses.  The library allocates no device memory.
 *   - `stream` is a cudaStream_t passed as void* (NULL = the default stream).  The step
 *     and basis calls only enqueue work on it and return; they never synchronise.
 *     Calls that must hand a number back to the host say so.
 *   - Matrices are row-major.  `ld` is the row pitch in ELEMENTS (>= the row width).
 *   - dtype is the storage type of F, R and Fhat: SVDCACHE_F32 or SVDCACHE_BF16.
 *     Coefficients (C, Chat) are always fp32.  For SVDCACHE_BF16 the kernels read a
 *     bf16 copy of V_k (made by svdcache_basis_prepare) and accumulate in fp32; for
 *     SVDCACHE_F32 they read V_k in fp32 and accumulate in fp64.
 *   - Shape limits: 1 <= N, 8 <= D <= 16384, D % 8 == 0, 8 <= k <= 256, k % 8 == 0,
 *     k <= D.  F, R, Fhat, V_k and all library-defined buffers must be 16-byte aligned,
 *     and (ld * element size) % 16 == 0.  Violations return SVDCACHE_ERR_BAD_SHAPE /
 *     SVDCACHE_ERR_BAD_ALIGN before anything is launched.
 *   - NaN / Inf in the inputs propagate per IEEE-754 and are not errors.
 */
#ifndef SVDCACHE_H_
#define SVDCACHE_H_

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define SVDCACHE_API __attribute__((visibility("default")))
#else
#define SVDCACHE_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

#define SVDCACHE_OK                0
#define SVDCACHE_ERR_INVALID_ARG  (-1) /* NULL pointer, unknown dtype, bad scalar      */
#define SVDCACHE_ERR_BAD_SHAPE    (-2) /* N, D, k, ld outside the limits above          */
#define SVDCACHE_ERR_BAD_ALIGN    (-3) /* a pointer or pitch is not 16-byte aligned     */
#define SVDCACHE_ERR_STATE        (-4) /* cached step on a state that saw no full step  */
#define SVDCACHE_ERR_WORKSPACE    (-5) /* workspace / buffer smaller than required      */
#define SVDCACHE_ERR_TIMEOUT      (-6) /* a bounded in-kernel wait ran out              */
#define SVDCACHE_ERR_CUDA         (-7) /* a CUDA runtime / driver call failed           */
#define SVDCACHE_ERR_NOT_CONVERGED (-8) /* eigen-solver hit its iteration limit         */
#define SVDCACHE_ERR_SCRATCH_LIMIT (-9) /* problem needs more than the built-in scratch    */

#define SVDCACHE_F32   0
#define SVDCACHE_BF16  1
#define SVDCACHE_FP8   2   /* 8-bit matrices (below): only where a call says so */

/* Predictors of the principal coefficients on cached steps (Sec. 3.4; Sec. 5.3, Fig. 4(b)). */
#define SVDCACHE_PREDICT_EMA     0  /* the method's own: the EMA state of Eq. 11                          */
#define SVDCACHE_PREDICT_TAYLOR  1  /* Taylor expansion in the step offset, backward-difference derivatives */
#define SVDCACHE_PREDICT_NEWTON  2  /* polynomial through the last order+1 full steps (Newton backward form) */

/* Text for a status code (static storage, never NULL). */
SVDCACHE_API const char *svdcache_status_string(int status);

/* Text of the last CUDA error seen by the calling thread inside this library. */
SVDCACHE_API const char *svdcache_last_cuda_error(void);

/* ---------------------------------------------------------------------------------
 * Calibration: the "one-time SVD" of Sec. 3.3 (Eq. 4, Eq. 5, Eq. 7).
 *
 * The right singular vectors of a row-stack Fstack (M x D) are the eigenvectors of the
 * Gram matrix G = Fstack^T Fstack, and sigma_i^2 its eigenvalues.  The stack may be fed
 * in pieces: begin, accumulate (any number of times, any row counts), finish.
 *
 *   workspace  device, caller-owned scratch of at least
 *              svdcache_calibrate_workspace_bytes(D, k) bytes, 256-byte aligned; it
 *              carries G between the three calls and must not be touched in between.
 *   F          device, M x D rows of dtype `dtype` with pitch ld; only read.
 *   Vk         device, out: D x k fp32, orthonormal columns ordered by descending
 *              eigenvalue; in each column the entry of largest magnitude is positive.
 *   lambda     device, out, k doubles (eigenvalues of G = sigma_i^2), or NULL.
 *   trace      device, out, 1 double: trace(G) = |Fstack|_F^2 = sum of ALL sigma_i^2
 *              (the denominator of the energy criterion, Eq. 6), or NULL.
 *   info       host, out, 4 doubles or NULL: {multiplications by G done, largest
 *              relative eigen-residual |G v - lambda v| / lambda_1 over the k pairs,
 *              Ritz block width, Jacobi sweeps of the last Rayleigh-Ritz step}.
 *
 * begin and accumulate only enqueue work.  finish synchronises `stream` several times
 * (it reads convergence numbers back) and returns SVDCACHE_ERR_NOT_CONVERGED if the
 * residual target was not met within the iteration limit (outputs are still written).
 * G is accumulated in a fixed order: results are bit-reproducible run to run.  fp32 stacks,
 * narrow or short bf16 stacks are summed in fp64 throughout (eigenvalues good to ~1e-10
 * relative).  bf16 stacks of at least 2048 rows per accumulate call whose width is a
 * multiple of 128 go through the tensor cores: exact bf16 products, fp32 sums over chunks of
 * 2048 rows, fp64 across chunks.  The tensor cores truncate the fp32 running sum, so G comes
 * out smaller by a few 1e-6, almost uniformly: eigenvalues (and the trace) carry that
 * relative error, the eigenvectors are affected far below the 1e-4 principal-angle bound.
 * Chunks start at the first row of each accumulate call, so feeding the same stack in
 * different pieces changes the last bits on that path.
 * ------------------------------------------------------------------------------- */
SVDCACHE_API int svdcache_calibrate_workspace_bytes(int D, int k, size_t *bytes /* host, out */);
SVDCACHE_API int svdcache_calibrate_begin(int D, int k, void *workspace, size_t workspace_bytes, void *stream);
SVDCACHE_API int svdcache_calibrate_accumulate(const void *F, int64_t M, int D, int64_t ld, int dtype,
                                  void *workspace, size_t workspace_bytes, void *stream);
SVDCACHE_API int svdcache_calibrate_finish(int D, int k, float *Vk, double *lambda, double *trace,
                              double *info, void *workspace, size_t workspace_bytes,
                              void *stream);
/* One-shot form: begin + accumulate(Fstack) + finish. */
SVDCACHE_API int svdcache_calibrate(const void *Fstack, int64_t M, int D, int64_t ld, int dtype, int k,
                       float *Vk, double *lambda, double *trace, double *info,
                       void *workspace, size_t workspace_bytes, void *stream);

/* Where the Gram matrix sits in a calibration workspace (Eq. 4): D x D doubles, row-major, `offset`
 * bytes from the start, complete between the last accumulate and the finish.  Row-sharded
 * calibration over several GPUs: every rank begins and accumulates its own rows, the ranks sum
 * this region (one all-reduce of D x D doubles), every rank finishes on the sum. */
SVDCACHE_API int svdcache_calibrate_gram_region(int D, size_t *offset, size_t *bytes /* host, out */);

/* Stability of the decomposition across "prompts" (Fig. 1(b)): similarity = cosine similarity x
 * magnitude similarity (min / max of the two norms).  For the singular values sigma = sqrt(lambda)
 * of two calibrations A and B: out[0] = cos(sigma_A, sigma_B) * min(|sigma_A|, |sigma_B|) / max(..).
 * For the right singular vectors (unit columns, sign-free): column_cos[j] = |<v_j^A, v_j^B>|,
 * out[1] = their mean.  VkA, VkB device D x k fp32, lambda device k doubles, column_cos device k
 * doubles (out), out host 2 doubles.  Synchronises `stream`. */
SVDCACHE_API int svdcache_basis_similarity(const float *VkA, const double *lambdaA, const float *VkB,
                              const double *lambdaB, int D, int k, double *column_cos,
                              double *out, void *stream);

/* ---------------------------------------------------------------------------------
 * Calibration for callers that cannot allocate device memory.  (The paper has no
 * counterpart: this entry point exists for how the library gets embedded, not for the
 * method.)
 *
 * svdcache_calibrate wants a workspace, and a host program normally gets one from
 * cudaMalloc.  Some hosts may not call it where calibration has to run: a plugin inside
 * an inference server whose memory pool was sized and handed out at start-up, code that
 * runs between the launches of a latency-critical loop where an allocation would
 * synchronise the device, or a process whose allocator is simply owned by someone else.
 * For them the library carries SVDCACHE_BUILTIN_SCRATCH_BYTES of scratch inside its own
 * device image (every GPU that loads the library holds that much until the process exits)
 * and this call uses it in place of the workspace.  Same arguments, results and status
 * codes as svdcache_calibrate otherwise; inputs and outputs are still the caller's.
 *
 *   - Size limit: svdcache_calibrate_workspace_bytes(D, k) must not exceed
 *     SVDCACHE_BUILTIN_SCRATCH_BYTES (e.g. D = 512 with k = 64 fits, D = 1152 does not);
 *     beyond it the call returns SVDCACHE_ERR_SCRATCH_LIMIT and launches nothing.
 *   - It calls no cudaMalloc / cudaFree and no routine that allocates.
 *   - The first call on a device looks up the scratch's device address
 *     (cudaGetSymbolAddress, with that device current) and keeps it; make that first call
 *     before starting any stream capture.
 *   - There is ONE scratch array per device and every call uses it.  It still holds the
 *     previous call's contents when a call starts; the call clears what it accumulates into
 *     before use.  Two calls whose GPU work overlaps (different streams, different threads)
 *     would trample each other: keep them ordered, e.g. on one stream.
 *   - Like svdcache_calibrate it synchronises `stream` while it iterates.
 * ------------------------------------------------------------------------------- */
#define SVDCACHE_BUILTIN_SCRATCH_BYTES (4u << 20)
SVDCACHE_API int svdcache_calibrate_noalloc(const void *Fstack, int64_t M, int D, int64_t ld, int dtype, int k,
                               float *Vk, double *lambda, double *trace, double *info, void *stream);

/* Rank selection by energy threshold (Eq. 6): the smallest k' <= n with
 * sum_{i<=k'} lambda_i / trace >= tau; n if the n listed eigenvalues fall short.
 * lambda: HOST array of n descending eigenvalues.  Pure host arithmetic. */
SVDCACHE_API int svdcache_rank_for_energy(const double *lambda, int n, double trace, double tau,
                             int *k_out /* host, out */);

/* ---------------------------------------------------------------------------------
 * Basis buffer: the cached reference basis of Eq. 7 in the layouts the step kernels
 * read.  Layout (all sections 256-byte aligned, offsets from svdcache_basis_layout):
 *   header (256 B) | V fp32 [D x k] | V^T fp32 [k x D] | V bf16 [D x k] | V^T bf16 [k x D]
 * The two bf16 sections exist only for dtype = SVDCACHE_BF16; they hold V_k rounded to
 * nearest-even, and are the values the bf16 kernels multiply with.
 * ------------------------------------------------------------------------------- */
SVDCACHE_API int svdcache_basis_bytes(int D, int k, int dtype, size_t *bytes /* host, out */);
SVDCACHE_API int svdcache_basis_layout(int D, int k, int dtype,
                          size_t *v_f32_offset, size_t *vt_f32_offset,
                          size_t *v_bf16_offset, size_t *vt_bf16_offset /* host, out; may be NULL */);
/* Vk: device D x k fp32 (only read).  basis: device, out, >= svdcache_basis_bytes. */
SVDCACHE_API int svdcache_basis_prepare(const float *Vk, int D, int k, int dtype, void *basis,
                           size_t basis_bytes, void *stream);

/* ---------------------------------------------------------------------------------
 * Per-block cache state, a caller-owned flat device buffer (checkpoint = memcpy):
 *   header (256 B) | Chat fp32 [N x k] | Chat operand copy | R dtype [N x D]   (dense, no pitch)
 * The operand copy exists only for dtype = SVDCACHE_BF16: Chat as two bf16 arrays [N x k],
 * hi = bf16(Chat) and lo = bf16(Chat - hi), which every full step rewrites together with
 * Chat and the cached step feeds to the tensor cores as they are (hi + lo carries ~16
 * mantissa bits).  Offsets of Chat and R come from svdcache_state_layout.
 * The header counts the full steps the state has seen and carries a sticky device
 * status word.  svdcache_state_reset must be called once before first use (and again to
 * start a new sampling run): it clears the counter, so the next full step initialises
 * the EMA with Chat = C.
 * ------------------------------------------------------------------------------- */
SVDCACHE_API int svdcache_state_bytes(int64_t N, int D, int k, int dtype, size_t *bytes /* host, out */);
SVDCACHE_API int svdcache_state_layout(int64_t N, int D, int k, int dtype,
                          size_t *chat_offset, size_t *r_offset /* host, out */);
SVDCACHE_API int svdcache_state_reset(void *state, int64_t N, int D, int k, int dtype, void *stream);
/* Synchronises `stream`, then reads the header: full steps seen, device status word
 * (SVDCACHE_OK, SVDCACHE_ERR_STATE or SVDCACHE_ERR_TIMEOUT).  Outputs are host. */
SVDCACHE_API int svdcache_state_query(const void *state, void *stream, int64_t *full_steps, int *status);

/* ---------------------------------------------------------------------------------
 * Full step (Eq. 8 - Eq. 11), one fused pass: C = F V_k, R = F - C V_k^T stored into
 * the state, Chat updated in the state (Chat = C if the state has seen no full step
 * yet).  F passes through untouched: the sampler keeps using the true feature.
 *   F      device, N x D, pitch ld, only read
 *   basis  device, from svdcache_basis_prepare for the same D, k, dtype
 *   state  device, in/out
 *   C_out  device, out, N x k fp32 (this step's coefficients), or NULL
 *   beta   EMA weight in [0, 1] (the paper uses 0.9)
 * ------------------------------------------------------------------------------- */
SVDCACHE_API int svdcache_full_step(const void *F, int64_t ld, const void *basis, void *state,
                       float *C_out, int64_t N, int D, int k, int dtype, float beta,
                       void *stream);

/* ---------------------------------------------------------------------------------
 * Cached step (Sec. 3.5): Fhat = Chat V_k^T + R.  The EMA state changes only at full
 * steps, so every cached step until the next full step returns the same Fhat;
 * `steps_since_full` is ignored by the EMA (the predictors that use it are the
 * svdcache_cached_step_forecast calls below).  If the state has seen no full step the kernel writes nothing and records
 * SVDCACHE_ERR_STATE in the state header (read it with svdcache_state_query).
 *   Fhat   device, out, N x D, pitch ld
 * ------------------------------------------------------------------------------- */
SVDCACHE_API int svdcache_cached_step(const void *state, const void *basis, void *Fhat, int64_t ld,
                         int64_t N, int D, int k, int dtype, int steps_since_full,
                         void *stream);

/* ---------------------------------------------------------------------------------
 * Batched forms: the same operation on `nblocks` independent DiT blocks in ONE launch
 * (Eq. 8 - Eq. 11 / Sec. 3.5 per block).  Block b uses F + b*F_stride, basis +
 * b*basis_stride, state + b*state_stride, out + b*out_stride; all strides are in BYTES
 * and multiples of 256.  Shapes, dtype and beta are shared.
 * ------------------------------------------------------------------------------- */
SVDCACHE_API int svdcache_full_step_batched(int nblocks, const void *F, int64_t ld, size_t F_stride,
                               const void *basis, size_t basis_stride, void *state,
                               size_t state_stride, float *C_out, size_t C_stride,
                               int64_t N, int D, int k, int dtype, float beta, void *stream);
SVDCACHE_API int svdcache_cached_step_batched(int nblocks, const void *state, size_t state_stride,
                                 const void *basis, size_t basis_stride, void *Fhat,
                                 int64_t ld, size_t Fhat_stride, int64_t N, int D, int k,
                                 int dtype, int steps_since_full, void *stream);

/* ---------------------------------------------------------------------------------
 * Blocks of different rank in one call (Eq. 6: the rank follows each block's spectrum, see
 * svdcache_rank_for_energy).  k_per_block is a HOST array of nblocks ranks; block b's basis and
 * state buffers are laid out for k_per_block[b] and sit b * stride bytes from the first (the
 * strides must cover the largest of them; C_out rows are k_per_block[b] wide).  Consecutive
 * blocks of equal rank go out as one batched launch; everything else is as in the batched
 * forms above.
 * ------------------------------------------------------------------------------- */
SVDCACHE_API int svdcache_full_step_ranked_batched(int nblocks, const void *F, int64_t ld, size_t F_stride,
                                      const void *basis, size_t basis_stride, void *state,
                                      size_t state_stride, float *C_out, size_t C_stride, int64_t N,
                                      int D, const int *k_per_block, int dtype, float beta,
                                      void *stream);
SVDCACHE_API int svdcache_cached_step_ranked_batched(int nblocks, const void *state, size_t state_stride,
                                        const void *basis, size_t basis_stride, void *Fhat,
                                        int64_t ld, size_t Fhat_stride, int64_t N, int D,
                                        const int *k_per_block, int dtype, int steps_since_full,
                                        void *stream);

/* ---------------------------------------------------------------------------------
 * Other predictors on the principal coefficients (Sec. 5.3, Fig. 4(b)): the decomposition
 * paired with a predictor that extrapolates inside the interval.  The caller keeps the
 * coefficients C of the last order+1 full steps (the C_out of svdcache_full_step) and hands
 * them over newest first; the residual is still the stored R (Sec. 3.5):
 *     Fhat = (sum_j w_j C_{n-j}) V_k^T + R,      u = steps_since_full / interval,
 *     backward differences D^i of the history, and
 *     SVDCACHE_PREDICT_TAYLOR   sum_i u^i / i! D^i
 *     SVDCACHE_PREDICT_NEWTON   sum_i u (u+1) ... (u+i-1) / i! D^i   (exact for polynomials of degree <= order)
 *     SVDCACHE_PREDICT_EMA      ignores the history: the plain cached step.
 * order 0 of either is plain reuse of the newest coefficients (Eq. 3).  order <= 7.
 *   svdcache_forecast_weights  host: the order+1 weights w_j (newest first) into w
 *   svdcache_forecast_bytes    host: size of the forecast buffer for N x k coefficients
 *   C_hist     HOST array of order+1 DEVICE pointers, each N x k fp32 (block b at + b*C_stride bytes)
 *   forecast   device scratch, 256-byte aligned, >= svdcache_forecast_bytes (block b at
 *              + b*forecast_stride): receives the forecast (fp32, then its split-bf16 pair)
 * Two launches: the forecast (N k work), then the cached-step kernel reading it.  The state is
 * only read.  Errors as svdcache_cached_step.
 * ------------------------------------------------------------------------------- */
SVDCACHE_API int svdcache_forecast_weights(int predictor, int order, int steps_since_full, int interval,
                              double *w /* host, out, order+1 */);
SVDCACHE_API int svdcache_forecast_bytes(int64_t N, int k, size_t *bytes /* host, out */);
SVDCACHE_API int svdcache_cached_step_forecast_batched(int nblocks, const void *state, size_t state_stride,
                                          const void *basis, size_t basis_stride, void *Fhat,
                                          int64_t ld, size_t Fhat_stride, int64_t N, int D, int k,
                                          int dtype, const float *const *C_hist, size_t C_stride,
                                          int predictor, int order, int steps_since_full,
                                          int interval, void *forecast, size_t forecast_stride,
                                          void *stream);

/* ---------------------------------------------------------------------------------
 * Ablation of Sec. 4.5 (Fig. 4(c)): the stored residual as an EMA of the residuals,
 *     R <- F - C V_k^T on the first full step, else beta_r R + (1 - beta_r)(F - C V_k^T).
 * beta_r = 0 is svdcache_full_step itself (the method: the residual is reused as it is);
 * beta = beta_r = 0 is "reuse on both" (Eq. 3); beta, beta_r > 0 is "EMA on both".  With
 * beta_r > 0 the step reads the old R as well (N D more elements than the method's step): the
 * epilogue of the fused kernel loads it and blends before the one rounding to the I/O dtype.
 * Arguments as svdcache_full_step_batched.
 * ------------------------------------------------------------------------------- */
SVDCACHE_API int svdcache_full_step_residual_ema_batched(int nblocks, const void *F, int64_t ld,
                                            size_t F_stride, const void *basis, size_t basis_stride,
                                            void *state, size_t state_stride, float *C_out,
                                            size_t C_stride, int64_t N, int D, int k, int dtype,
                                            float beta, float beta_r, void *stream);

/* ---------------------------------------------------------------------------------
 * The cached singular values and the left factors of Eq. 7 - Eq. 8.
 *   svdcache_singular_values  sigma_i = sqrt(lambda_i) of the calibration spectrum (device arrays of k)
 *   svdcache_left_factors     U = C diag(sigma)^-1 (Eq. 8), C and U device N x k fp32; a column whose
 *                             sigma is 0 is set to 0.  (The step kernels never form U: sigma cancels
 *                             between Eq. 8 and Eq. 9.)
 * ------------------------------------------------------------------------------- */
SVDCACHE_API int svdcache_singular_values(const double *lambda, int k, double *sigma, void *stream);
SVDCACHE_API int svdcache_left_factors(const float *C, const double *sigma, int64_t N, int k, float *U,
                          void *stream);

/* ---------------------------------------------------------------------------------
 * The 8-bit linear path around a cached block (no counterpart in the paper's equations; its
 * Table 3 pairs the method with an 8-bit quantised model).  A full step needs the block's
 * feature F from the network's own linear layers: the quantiser and the product are these in 8 bits, for
 * any block.  The norm is what follows F or Fhat in models that add a block's feature to the residual
 * stream as it is and begin the next block with an RMS norm; it has no gate, shift or mean, so blocks with
 * a gated addition and a modulated layer norm form their norm's output themselves and quantise it.
 *
 * 8-bit matrix: rows of e4m3 values (one byte each, pitch ld in bytes) and a scale buffer.
 *   - Every 1 x 128 group of a row has one scale, a power of two 2^e held as the byte e + 127
 *     (E8M0).  e is the smallest integer with 448 * 2^e >= the group's largest finite magnitude
 *     (0 for a group of zeros; e >= -127).  value = e4m3(y / 2^e), round to nearest even.
 *   - Inf and NaN become the NaN code and stay with their element; the group's scale is that of
 *     its finite elements.
 *   - The scale buffer has svdcache_fp8_scale_bytes(rows, cols) bytes: pieces of 512 bytes for
 *     128 rows x 4 groups, [rows / 128][groups / 4] rounded up; the byte of row m, group g is
 *     byte (m % 32) * 16 + (m / 32 % 4) * 4 + g % 4 of piece (m / 128, g / 4).  Bytes of rows and
 *     groups that do not exist are never written and reach no result.
 *   - Limits: 0 <= rows < 2^31 - 256 (0 rows: nothing is launched), 1 <= cols <= 131072, values and
 *     scales 16-byte aligned, pitch a multiple of 16 bytes.  cols itself need not be.
 *
 *   svdcache_quantize_fp8   X (rows x cols of F32 or BF16, pitch ld) -> Q, S.  tile_rows 1: a scale
 *              per 1 x 128 group (activations); 128: one per 128 x 128 tile, written for each of
 *              its rows (weights).
 *   svdcache_residual_rmsnorm_fp8   h = H + X;  H_out = h;  y = h * rsqrt(mean(h^2) + eps) * weight;
 *              Q, S = y in 8 bits, a scale per 1 x 128 group.  fp32 arithmetic, y from the unrounded
 *              h.  X may be NULL (plain norm), H_out NULL (h not kept) or H itself (in place),
 *              weight (device, D fp32) NULL for ones.  Needs 8 <= D <= 16384, D % 8 == 0, eps >= 0.
 *              The sum of squares is fp32 as well: where it exceeds that type (one element of 1.8e19 is enough)
 *              the row's finite values become 0, and squares below 1e-45 count as 0 (which matters where eps is
 *              as small).
 *   svdcache_gemm_fp8       C = act(A B^T + bias): A (M x K) and B (N x K) 8-bit with scales SA and
 *              SB, bias device N fp32 or NULL, act SVDCACHE_ACT_NONE or SVDCACHE_ACT_GELU (tanh
 *              form).  C (M x N, pitch ldc in ELEMENTS) is F32, BF16 or FP8; FP8 writes its scales
 *              (a scale per 1 x 128 group) to SC, which is ignored otherwise.  Products are exact; sums are
 *              the tensor cores' fp32, which truncates: off by 3e-7 of the result at K = 3072, 1.5e-6 at 12288
 *              (2-norm; an fp32 library product: 1e-7, 2e-7).  gelu adds less than 2^-17 of its value.
 *              1 <= N, K <= 131072.
 *              status (device, one int32 that the caller sets to 0 once) receives
 *              SVDCACHE_ERR_TIMEOUT if a bounded in-kernel wait runs out; it is never cleared here.
 *   svdcache_gemm_fp8_status_word   the address of a status word that the library itself has on the
 *              current device, zero when the library is loaded, for callers that keep none (the
 *              Python binding's default); svdcache_gemm_fp8_status_query waits for the device and reads it.
 * The three calls only enqueue work on `stream`, and any of them may be the first in a process to be captured.  Results are bit-reproducible.
 * ------------------------------------------------------------------------------- */
#define SVDCACHE_ACT_NONE  0
#define SVDCACHE_ACT_GELU  1   /* x / (1 + exp(-2u)), u = sqrt(2 / pi) (x + 0.044715 x^3) */
SVDCACHE_API int svdcache_fp8_scale_bytes(int64_t rows, int cols, size_t *bytes /* host, out */);
SVDCACHE_API int svdcache_quantize_fp8(const void *X, int64_t rows, int cols, int64_t ld, int dtype, int tile_rows,
                          void *Q, int64_t ldq, void *S, void *stream);
SVDCACHE_API int svdcache_residual_rmsnorm_fp8(const void *H, int64_t ldh, const void *X, int64_t ldx, void *H_out,
                                  int64_t ldo, const float *weight, float eps, void *Q, int64_t ldq,
                                  void *S, int64_t rows, int D, int dtype, void *stream);
SVDCACHE_API int svdcache_gemm_fp8(const void *A, int64_t lda, const void *SA, const void *B, int64_t ldb,
                      const void *SB, const float *bias, int act, void *C, int64_t ldc, int out_dtype,
                      void *SC, int64_t M, int N, int K, int32_t *status, void *stream);
SVDCACHE_API int svdcache_gemm_fp8_status_word(int32_t **word /* host, out: a device address */);
SVDCACHE_API int svdcache_gemm_fp8_status_query(int32_t *status /* host, out */);

/* ---------------------------------------------------------------------------------
 * Low-rank adapters of many requests beside a shared 8-bit projection (no counterpart in the paper's equations):
 *     C[m] = act( A[m] B^T + bias + factor_a (A[m] down_a^T) up_a^T ),   a the adapter of row m's request, or none.
 * The adapters' term is summed in the product's own accumulator, before the activation and the rounding into 8 bits.
 *
 * A pool holds `count` adapters of rank up to `rank` (a multiple of 8, 8 .. 128; smaller ones end in zeros) for one projection
 * of K columns to N: down[a], an 8-bit matrix of rank rows x K with scales of its own (format above, pitch and distance
 * in bytes), up[a] of N x rank in bf16 (pitch and distance in elements), factor[a].  Everything device and 16-byte aligned, pitches
 * and distances multiples of 16 bytes.  Values of `up` have to be finite: an infinity or NaN there would reach other requests'
 * rows of the same tile (0 * inf).  svdcache_adapter_load sees to that.
 *
 * Requests are runs of rows: row_start (device, requests + 1 int32, not decreasing) and adapter (device, requests int32; values
 * outside 0 .. count - 1: none).  Rows before the first and behind the last run have no adapter.  Both are read when the
 * call runs, so a captured call serves other requests after they are rewritten.  (Where row_start decreases, rows hold
 * unspecified values; nothing outside the buffers is touched.)  Nothing of another request, its rows, its adapter or what these hold, reaches
 * a row.  The order in which a row's sums are rounded may differ with the sizes of the call and its workspace, the number of its requests and which of
 * them have an adapter; for the same of these a row is the same bit for bit.
 *
 *   svdcache_adapters_workspace_bytes  room for A down^T between the two kernels of a call, and for which tile has which
 *              adapters; 256-byte aligned, of one call at a time, nothing in it outlives the call.  The size serves any
 *              output type; (ceil(M / 256) + requests) * (ceil(rank / 32) * 32768 + 1024) bytes are always enough
 *              for two values (below); where less does not hold them it is refused
 *   svdcache_gemm_fp8_adapters  as svdcache_gemm_fp8 otherwise.  A down^T is summed in fp32 as the product is, times factor, and goes
 *              into the second product as a sum of two bf16 values for bf16 output (off by 2^-16
 *              of itself at most), of three for the others (2^-24).  Where the workspace is
 *              smaller than svdcache_adapters_workspace_bytes and does not hold three, 8-bit output takes two, and fp32 output three by lower
 *              tiles or several launches, which may take longer.  Kernel and
 *              tiles are those of the product alone (svdcache_gemm_fp8_plan), which with many requests are not always the fastest.  0 requests or count 0: svdcache_gemm_fp8.
 *   svdcache_adapter_load  puts an adapter into place `index` of a pool: down (r x K) into 8 bits with a scale per 1 x 128 group, up
 *              (N x r) into bf16, both F32 or BF16 (dtype) with 16-byte aligned rows (up: any pitch), r <= rank, factor.  In
 *              e4m3 a value of down is off by 2^-4 of itself at most, and A down^T by 2.6 % of its norm for normally distributed values (as much as
 *              A's own rounding does; 3.6 %, 2^-4 / sqrt(3), for any whose roundings are independent).  Where a value
 *              of up does not become a finite bf16 it is held as 0 and the adapter's factor as NaN: all rows that use it
 *              become NaN, and no others.
 * ------------------------------------------------------------------------------- */
typedef struct {
    void *down;
    int64_t down_ld, down_stride;       /* bytes */
    void *down_scales;
    int64_t scales_stride;              /* bytes, at least svdcache_fp8_scale_bytes(rank, K) */
    void *up;
    int64_t up_ld, up_stride;           /* elements */
    float *factor;
    int count, rank;
} svdcache_adapters;
SVDCACHE_API int svdcache_adapters_workspace_bytes(int64_t M, int rank, int requests, size_t *bytes /* host, out */);
SVDCACHE_API int svdcache_gemm_fp8_adapters(const void *A, int64_t lda, const void *SA, const void *B, int64_t ldb, const void *SB,
                               const float *bias, int act, void *C, int64_t ldc, int out_dtype, void *SC, int64_t M, int N, int K,
                               const svdcache_adapters *adapters, const int32_t *row_start, const int32_t *adapter, int requests,
                               void *workspace, size_t workspace_bytes, int32_t *status, void *stream);
SVDCACHE_API int svdcache_adapter_load(const svdcache_adapters *adapters, int index, const void *down, int64_t ldd, const void *up, int64_t ldu,
                          int r, float factor, int N, int K, int dtype, void *stream);

/* ---------------------------------------------------------------------------------
 * Queries and keys between the product that makes them and the attention that reads them (no counterpart in the
 * paper's equations): positions of several axes (time, height, width) as rotations, and the RMS norm of each head.
 *
 * Heads: [batch, tokens, heads, dim] of F32 or BF16 with any strides (in ELEMENTS; batch, token and head), the dim elements of
 * a head side by side: a packed projection, heads before tokens, or anything between.  8 <= dim <= 256, dim % 8 == 0,
 * data 16-byte aligned, strides multiples of 16 bytes and not negative, heads <= 65536, tokens < 2^31,
 * batch < 65536.
 * Output and input are the same heads (in place) or share no memory.
 *
 * Rotation: pair i < r / 2 of a head's first r elements (r % 8 == 0, 8 <= r <= dim) turns by the table's (cos, sin) of the
 * token: (a, b) -> (a cos - b sin, a sin + b cos).  Pair i is elements (2i, 2i + 1), or with SVDCACHE_ROTARY_HALVES (i, i + r / 2).
 * SVDCACHE_ROTARY_INVERSE turns back, which is the rotation's gradient as well.  Tokens [first, first + tokens) have rows
 * 0 .. tokens - 1 of the table; the others, and elements r .. dim - 1, are not rotated.
 *
 *   svdcache_rotary_table  table[n][i] = (cos, sin) of position[n][axis] * base^(-2 j / d): axes of even widths d = dims[axis], one
 *              after the other, j the pair's number on its axis.  positions (tokens x axes, pitch ld in elements) are int32, int64
 *              or fp32; dims and bases are HOST arrays (1 <= axes <= 8, the widths sum to r, r % 8 == 0, r <= 256; bases positive
 *              and finite).  table: fp32, 16-byte aligned, pitch ldt >= r floats (a multiple of 4).  cos and sin
 *              are within 2^-23 of those of the angle, which is formed in 64 bits (itself off by 2^-51 of its size, which counts from 2^28
 *              on, and beyond 2^51 is an angle of any size).  tokens < 2^31.
 *   svdcache_rotary        out = X rotated
 *   svdcache_qk_rmsnorm_rotary  x * rsqrt(mean(x^2) + eps) * weight for each head of Q and of K, then the rotation, in one launch.
 *              weights (device, dim fp32) NULL for ones; K and K_out NULL: queries alone; rotation NULL: norm alone.
 *              K may have another number of heads.  fp32 arithmetic with one rounding at the end; a sum of squares beyond
 *              fp32 (elements of 1.8e19) makes the head's finite values 0.
 * The calls only enqueue work on `stream`; 0 tokens or batches: nothing is launched.
 * ------------------------------------------------------------------------------- */
#define SVDCACHE_POSITION_I32  0
#define SVDCACHE_POSITION_I64  1
#define SVDCACHE_POSITION_F32  2
#define SVDCACHE_ROTARY_HALVES   1
#define SVDCACHE_ROTARY_INVERSE  2
#define SVDCACHE_ROTARY_MAX_DIM  256
#define SVDCACHE_ROTARY_MAX_AXES 8
typedef struct {
    void *data;                                         /* device */
    int64_t batch_stride, token_stride, head_stride;    /* in elements */
    int heads;
} svdcache_heads;
typedef struct {
    const float *table;                                 /* device, 16-byte aligned */
    int64_t batch_stride, token_stride;                 /* in floats, multiples of 4; batch_stride 0: one table for all */
    int64_t first, tokens;
    int r, flags;
} svdcache_rotation;
SVDCACHE_API int svdcache_rotary_table(const void *positions, int64_t tokens, int64_t ld, int position_type, int axes,
                          const int *dims /* host */, const double *bases /* host */, float *table, int64_t ldt, void *stream);
SVDCACHE_API int svdcache_rotary(const svdcache_heads *X, const svdcache_heads *out, int64_t batch, int64_t tokens, int dim, int dtype,
                    const svdcache_rotation *rotation, void *stream);
SVDCACHE_API int svdcache_qk_rmsnorm_rotary(const svdcache_heads *Q, const svdcache_heads *Q_out, const float *q_weight,
                               const svdcache_heads *K, const svdcache_heads *K_out, const float *k_weight, float eps,
                               int64_t batch, int64_t tokens, int dim, int dtype, const svdcache_rotation *rotation, void *stream);

/* ---------------------------------------------------------------------------------
 * Introspection for benchmarks and tests (host only).
 *   svdcache_kernel_launches: kernels this library has launched in this process.
 *   svdcache_set_path: a process-wide switch for tests and benchmarks (every later step call
 *                      of every thread sees it; not meant for production code).
 *                      0 = pick automatically, 1 = force the CUDA-core kernels,
 *                      2 = force the tcgen05 kernels (error if the shape is outside what
 *                      they support).  Returns the previous setting.
 *   svdcache_last_path: which kernel family the last step call used (1 or 2).
 * ------------------------------------------------------------------------------- */
SVDCACHE_API uint64_t svdcache_kernel_launches(void);
SVDCACHE_API int svdcache_set_path(int path);
SVDCACHE_API int svdcache_last_path(void);

/* Self-test of the time-out path (no counterpart in the paper).  Every wait inside the
 * tcgen05 kernels is bounded (~2 s): when one runs out the kernel stops, stores
 * SVDCACHE_ERR_TIMEOUT in the state header of block 0 together with which wait it was, and
 * returns, so the context stays usable.  This call launches one small CTA that waits, with the
 * same code, for an event that never comes, for `limit_cycles` SM cycles (1 .. 2e8): afterwards
 * svdcache_state_query on `state` (a reset state buffer, device, 256-byte aligned) must report
 * SVDCACHE_ERR_TIMEOUT, the word at byte 36 of the header reads 99 << 16 (wait site 99, CTA 0),
 * and svdcache_state_reset clears both.  Asynchronous on `stream`.  Nothing is faulted or hung. */
SVDCACHE_API int svdcache_selftest_wait_timeout(void *state, int64_t limit_cycles, void *stream);

/* How the 8-bit product is taken, for tests and benchmarks.  svdcache_gemm_fp8 chooses among two kernels and their tiles by a
 * model of their times; plan (host, four words) names a choice:
 *   {1, 128, 192 or 256, 2}            pairs of CTAs on tiles of 256 rows x that many columns (192: F32, BF16; 256: FP8)
 *   {0, 16, 32, 64 or 128, 1 .. 8}     tiles of so many rows x 128 columns, K shared by 1, 2, 3, 4, 6 or 8 CTAs
 * svdcache_gemm_fp8_plan tells the model's on the current device, and in the fourth word how many tiles follow one another on
 * an SM at most.  svdcache_selftest_gemm_fp8 is svdcache_gemm_fp8 by the given plan (three words);
 * SVDCACHE_ERR_INVALID_ARG if it is not one that the model may choose for such a product: tiles of the fewest rows that
 * hold M, of 64 or 128 above that; several CTAs only where all clusters run at the same time, with two groups of K each.
 * limit_cycles 0: an ordinary product.  1 .. 2e8: a test of the time-out path: no operand is loaded, every wait runs out
 * after so many SM cycles, the kernel returns with SVDCACHE_ERR_TIMEOUT in *status, and C holds nothing of use. */
SVDCACHE_API int svdcache_gemm_fp8_plan(int64_t M, int N, int K, int64_t lda, int64_t ldb, int out_dtype, int32_t *plan /* host, out */);
SVDCACHE_API int svdcache_selftest_gemm_fp8(const void *A, int64_t lda, const void *SA, const void *B, int64_t ldb,
                               const void *SB, const float *bias, int act, void *C, int64_t ldc, int out_dtype,
                               void *SC, int64_t M, int N, int K, int32_t *status, const int32_t *plan /* host */,
                               int64_t limit_cycles, void *stream);
/* the same for svdcache_gemm_fp8_adapters (which takes its projection as svdcache_gemm_fp8_plan says), with a request and an adapter at least, and room for
 * three values of t for fp32 output */
SVDCACHE_API int svdcache_selftest_gemm_fp8_adapters(const void *A, int64_t lda, const void *SA, const void *B, int64_t ldb, const void *SB,
                               const float *bias, int act, void *C, int64_t ldc, int out_dtype, void *SC, int64_t M, int N, int K,
                               const svdcache_adapters *adapters, const int32_t *row_start, const int32_t *adapter, int requests,
                               void *workspace, size_t workspace_bytes, int32_t *status, const int32_t *plan /* host */,
                               int64_t limit_cycles, void *stream);
/* How its two kernels, the narrow product's and the projection's, are launched on a device of so many SMs, where the projection is
 * taken by the given plan and takes little time (brief) or much: CTAs, CTAs of a cluster, columns of tensor memory and bytes
 * of dynamic shared memory of each, for the one and for the other.  Host only. */
SVDCACHE_API int svdcache_selftest_adapters_sizes(int64_t M, int N, int K, int rank, int requests, int out_dtype, const int32_t *plan /* host */,
                               int brief, int sms, int64_t *sizes /* host, out: 8 words */);
/* What its kernels find out about requests (all host pointers) of a launch over rows first .. first + M - 1 in tiles of 16, 32, 64, 128 or
 * 256 rows, by the same code on the host.  S = tiles + requests: tasks (S x 4) the tile, rows and adapter (-1: none) that each slot stands
 * for; tiles (tiles x 4) where a tile's slots are listed, how many they are, the first one's number and adapter; list (S x 2) those
 * lists, number and adapter, entries that no tile lists left as they were; tile_list (tiles x (1 + 2 tile_rows)) how many slots a
 * small tile takes and which. */
SVDCACHE_API int svdcache_selftest_adapters_slots(const int32_t *row_start, const int32_t *adapter, int requests, int64_t first, int64_t M, int count,
                               int tile_rows, int32_t *tasks, int32_t *tiles, int32_t *list, int32_t *tile_list);

#ifdef __cplusplus
}
#endif
#endif /* SVDCACHE_H_ */
