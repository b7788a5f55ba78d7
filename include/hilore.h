/*
 * hilore.h -- C ABI of the B200 (sm_100a) hot path of HiLoRe's GRPO actor update.
 *
 * Two parts (paper: Algorithm 1, lines "Coefficients", "Exposure", risk score, and the
 * capture / recovery of L units):
 *   1. the fused GRPO loss-coefficient pass and its reduction to one update-exposure score
 *      per recovery unit, available before backward (Prop. 1, Eq. "update-coefficient",
 *      Eq. "mlp-weighted-exposure");
 *   2. the low-precision store / recover path for saved bf16 activations
 *      (Eq. "fp8-roundtrip"), gated by the per-unit H / L / R plan
 *      (Eq. "available-recovery-actions").
 *
 * Conventions for every entry point
 *   - Returns an int status (HILORE_OK = 0).  Never throws, aborts or traps.
 *   - Every pointer is a DEVICE pointer owned by the caller, valid until the work enqueued
 *     by the call has finished, unless its comment says "host".
 *   - The library allocates nothing and keeps no data between calls (the one exception is stated at
 *     its declaration); it only remembers immutable device properties (SM count, CTAs per SM of its
 *     kernels) after the first call on a device.  Work is enqueued on `stream` (a cudaStream_t passed as
 *     void*; NULL = the legacy default stream) and the call returns without synchronising.
 *     HILORE_CUDA reports a launch error seen by cudaGetLastError, nothing asynchronous.
 *   - Tensors are row-major.  bf16 tensors are passed as void* (16-bit patterns).
 *   - Output buffers must not overlap inputs or each other.
 *   - Optional pointers say "opt" and may be NULL.
 */
#ifndef HILORE_H
#define HILORE_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* ---- status codes ---- */
enum {
    HILORE_OK = 0,
    HILORE_INVALID_ARG = 1, /* NULL where data is required, negative size, unknown enum value          */
    HILORE_SHAPE = 2,       /* cols % 16 != 0, cols % block != 0, n_resp % G != 0, ld < cols, ...       */
    HILORE_ALIGN = 3,       /* a pointer or leading dimension misses the alignment stated below       */
    HILORE_ZERO_NORM = 4,   /* the normaliser N is not positive and no device-side N was given         */
    HILORE_CUDA = 5,        /* kernel launch failed                                                    */
    HILORE_WORKSPACE = 6    /* workspace too small; see hilore_workspace_bytes                         */
};

/* ---- storage formats of the L (compress) action ---- */
enum {
    HILORE_FMT_E4M3FN_RAW = 0, /* the paper's codec, Eq. "fp8-roundtrip": unscaled cast to FP8 E4M3FN,
                                  one byte per element, no scales; values that round above 448 and
                                  non-finite values become the NaN code, as the cast the paper names does */
    HILORE_FMT_E4M3FN_BLK = 1, /* E4M3FN payload + one fp32 absmax scale per block of 64 elements of a
                                  row (the benchmark's block-scaled generalisation; not in the paper)    */
    HILORE_FMT_INT8_BLK = 2    /* INT8 payload (+-127) + one fp32 absmax scale per block of 64            */
};
#define HILORE_BLOCK 64 /* the only block size of the scaled formats */

/* ---- recovery actions; the numeric order is the paper's tie order R, H, L ---- */
enum { HILORE_ACT_R = 0, HILORE_ACT_H = 1, HILORE_ACT_L = 2 };

/* ---- phases of hilore_plan_apply ---- */
enum {
    HILORE_PHASE_DECIDE = 0,  /* risk score, threshold rule, availability -> action / recompute / bytes  */
    HILORE_PHASE_CAPTURE = 1, /* forward-time capture by candidate plan q: q = L compress (+ token RMS),
                                 q = H token RMS only (bf16 kept), q = R nothing                          */
    HILORE_PHASE_ENCODE = 2,  /* post-forward encoding: units with q = H that were assigned L           */
    HILORE_PHASE_RECOVER = 3  /* backward-time recovery: units with action L are decoded to bf16         */
};

struct hilore_unit; /* one recovery unit of a microbatch; defined with hilore_plan_apply below */

const char *hilore_status_string(int status);
/* Version of this ABI (major * 1000 + minor). */
int hilore_abi_version(void);

/*
 * N = sum_t m_t, the learner's normaliser (Eq. "grpo-objective": N = sum of the update mask; the
 * setup section normalises by all valid response tokens of the complete rollout batch).
 *   mask   [n] u8, 0 or 1.            count  one int64 on the device, overwritten with the sum.
 * The sum is an integer, so the result does not depend on the order of the additions.
 */
int hilore_mask_count(const uint8_t *mask, int64_t n, int64_t *count, void *stream);

/*
 * Group-relative advantages and per-token update coefficients omega_t = dL/ds_t
 * (Eq. "grpo-objective", Eq. "update-coefficient", K3 derivative in the proof of Prop. 1):
 *     A_j     = (R_j - mean_g) / (population_std_g + adv_eps); a group whose rewards are all equal
 *               has A = +0 exactly (setup section, "GRPO and optimization")
 *     r_t     = exp(s_t - s_old_t)
 *     chi_t   = 1[(A >= 0 and r_t <= 1 + clip_eps) or (A < 0 and r_t >= 1 - clip_eps)]   (fp32 compare)
 *     omega_t = -(m_t / N) chi_t r_t A  +  beta (m_t / N) (1 - exp(s_ref_t - s_t))
 * Group statistics are evaluated in fp64 per response, the per-token part in fp32.
 *
 *   rewards      [n_resp_total] fp32; the G responses of prompt p are rewards[p*G .. p*G+G-1].
 *                n_resp_total % G must be 0 (HILORE_SHAPE).
 *   resp_offset, n_rows   this call covers responses [resp_offset, resp_offset + n_rows), a microbatch
 *                of the rollout batch; a prompt group may straddle two calls.
 *   logp_new, logp_old, logp_ref   [n_rows, T] fp32, 16-byte aligned; logp_ref may be NULL iff beta == 0.
 *   mask         [n_rows, T] u8 (0 / 1), 4-byte aligned.  T % 4 must be 0 (HILORE_SHAPE).  With T % 8 == 0, the fp32
 *                tensors 32-byte aligned and the byte tensors 8-byte aligned the call takes its fast path (256-bit
 *                accesses, one warp per 512 slots); the results do not depend on the path.
 *   N_norm, N_norm_dev   the normaliser N: if N_norm_dev (one int64 on the device, e.g. written by
 *                hilore_mask_count earlier on the same stream) is not NULL it is read by the kernel and
 *                N_norm is ignored; a device value <= 0 yields omega = 0 everywhere.  Otherwise N_norm
 *                (host value) must be > 0 (HILORE_ZERO_NORM).
 *   adv_out      opt [n_rows] fp32, advantage of each response of this call.
 *   omega        [n_rows, T] fp32, 16-byte aligned.  Masked slots get 0.
 *   ratio        opt [n_rows, T] fp32 (r_t as computed, also at masked slots), 16-byte aligned.
 *   clip_mask    opt [n_rows, T] u8 (chi_t), 4-byte aligned.
 */
int hilore_grpo_coeffs(const float *rewards, int64_t n_resp_total, int32_t G, int64_t resp_offset,
                       int64_t n_rows, int64_t T, const float *logp_new, const float *logp_old,
                       const float *logp_ref, const uint8_t *mask, int64_t N_norm,
                       const int64_t *N_norm_dev, float clip_eps, float beta, float adv_eps, float *adv_out,
                       float *omega, float *ratio, uint8_t *clip_mask, void *stream);

/*
 * hilore_grpo_coeffs followed by hilore_unit_exposure as ONE sweep (Algorithm 1, "coefficients" and "exposure"
 * lines; Eqs. "update-coefficient", "mlp-weighted-exposure"): the coefficients are computed inside the exposure
 * reduction instead of being written and read back, which saves launches and the round trip of omega when the
 * microbatch is small enough for the call to be launch-bound (n_rows * T <= 2^18 slots and at most 62 responses
 * per 1024 slots; other shapes run the two passes in turn inside this call).  Results are bit for bit those of
 * the two calls: omega [n_rows, T] (REQUIRED here, it is written either way), exposure [U], sum_abs_omega (opt).
 * Arguments, status codes and workspace as in the two calls; adv_out, ratio and clip_mask are not produced.
 */
int hilore_coeffs_exposure(const float *rewards, int64_t n_resp_total, int32_t G, int64_t resp_offset, int64_t n_rows,
                           int64_t T, const float *logp_new, const float *logp_old, const float *logp_ref,
                           const uint8_t *mask, int64_t N_norm, const int64_t *N_norm_dev, float clip_eps, float beta,
                           float adv_eps, const float *row_rms, int32_t U, int64_t rms_ld, int32_t row_shift,
                           float eps_alpha, float *omega, float *exposure, float *sum_abs_omega, void *workspace,
                           size_t workspace_bytes, void *stream);

/*
 * The score refresh of one microbatch in ONE kernel launch: hilore_coeffs_exposure followed by
 * hilore_plan_apply(HILORE_PHASE_DECIDE) (Algorithm 1, lines "coefficients", "exposure", risk score and allocation;
 * Eqs. "update-coefficient", "mlp-weighted-exposure", "token-weighted-risk", "available-recovery-actions").  The CTAs of
 * a group of eight units -- one per tile of 1024 tokens -- add their partial sums in the fixed order of the two-kernel
 * form and one of them takes the plan decisions of the group's units, so omega, exposure, psi, action_io, recompute and
 * retained_bytes are bit for bit those of the separate calls.  At microbatch size (up to 16 tiles of 1024 tokens;
 * the cluster is the next power of two) the CTAs of a group are one thread-block cluster and hand the sums to its
 * first CTA through distributed shared memory; otherwise through the workspace, the CTA that finishes last (a
 * counter per group, cleared by a memset inside the call) doing the rest.  Between forward and backward of a
 * microbatch this is one launch instead of four.
 *   Arguments as in hilore_coeffs_exposure (omega REQUIRED, U > 0, n_rows * T > 0) and in the DECIDE phase of
 *   hilore_plan_apply (units_dev, kappa, ebar, avail, action_io REQUIRED; psi, recompute, retained_bytes opt; the
 *   unit table is only read for rows, cols and fmt, on the device).
 *   workspace   at least hilore_scores_plan_workspace_bytes(U, n_rows * T) bytes, 16-byte aligned: the partial sums
 *               and, behind them, the counters of finished CTAs (unused by the cluster form).
 *   Microbatches beyond the one-sweep form's limits (see hilore_coeffs_exposure) run the coefficient pass first and
 *   then the reduction + plan launch.
 */
int hilore_scores_plan(const float *rewards, int64_t n_resp_total, int32_t G, int64_t resp_offset, int64_t n_rows,
                       int64_t T, const float *logp_new, const float *logp_old, const float *logp_ref,
                       const uint8_t *mask, int64_t N_norm, const int64_t *N_norm_dev, float clip_eps, float beta,
                       float adv_eps, const float *row_rms, int32_t U, int64_t rms_ld, int32_t row_shift,
                       float eps_alpha, float *omega, float *exposure, float *sum_abs_omega,
                       const struct hilore_unit *units_dev, const float *kappa, const float *ebar, float tau_lo,
                       float tau_hi, const uint8_t *avail, uint8_t *action_io, float *psi, uint8_t *recompute,
                       uint64_t *retained_bytes, void *workspace, size_t workspace_bytes, void *stream);
size_t hilore_scores_plan_workspace_bytes(int32_t U, int64_t n_tok);

/*
 * The coefficient and exposure passes on the packed (padding-removed) layout of the paper's DSR-sub execution
 * setting (Table "execution-configurations": "padding removal").  The sequences of a microbatch -- prompt
 * followed by the generated response, no padding slots -- lie back to back: sequence i (response
 * resp_offset + i of the rollout batch) owns tokens cu_seqlens[i] .. cu_seqlens[i+1]-1; the activation
 * tensors of the microbatch have one row per packed token.  Arithmetic per token exactly as in
 * hilore_grpo_coeffs / hilore_unit_exposure; mask = 1 on generated response tokens, 0 on prompt tokens.
 *
 *   cu_seqlens   [n_seq + 1] int32 on the device, cu_seqlens[0] = 0, non-decreasing (empty sequences allowed),
 *                cu_seqlens[n_seq] = n_tok.  The contents are the caller's responsibility (they are not read on
 *                the host); whatever they hold, no kernel indexes outside [0, n_seq] or [0, n_tok).
 *   logp_*, omega, ratio [n_tok] fp32, 16-byte aligned;  mask, clip_mask [n_tok] u8, 4-byte aligned; n_tok need
 *                not be a multiple of 4 (n_tok < 2^31).  With 32-byte aligned fp32 tensors and 8-byte aligned masks
 *                the call takes its fast kernel (one warp per 512 tokens); the results are the same bits either way.
 *   adv_out      [n_seq] fp32, REQUIRED here: the per-sequence advantages are written by a first launch and read
 *                by the token kernel (2 launches; the second starts while the first runs and waits for it only
 *                before it uses an advantage).
 *   Exposure: the activation row of token k is k - row_shift; with row_shift = 1 a token whose source row
 *   would fall before the start of its own sequence carries no weight (it counts neither in the mean nor in E_u).
 *   Other arguments, status codes and workspace as in the dense calls.
 */
int hilore_grpo_coeffs_packed(const float *rewards, int64_t n_resp_total, int32_t G, int64_t resp_offset,
                              int64_t n_seq, const int32_t *cu_seqlens, int64_t n_tok, const float *logp_new,
                              const float *logp_old, const float *logp_ref, const uint8_t *mask, int64_t N_norm,
                              const int64_t *N_norm_dev, float clip_eps, float beta, float adv_eps, float *adv_out,
                              float *omega, float *ratio, uint8_t *clip_mask, void *stream);
int hilore_unit_exposure_packed(const float *omega, const uint8_t *mask, int64_t n_tok, const int32_t *cu_seqlens,
                                int64_t n_seq, const float *row_rms, int32_t U, int64_t rms_ld, int32_t row_shift,
                                float eps_alpha, float *exposure, float *sum_abs_omega, void *workspace,
                                size_t workspace_bytes, void *stream);

/*
 * Score variants of the component ablations (paragraph "Component ablations"): hilore_grpo_coeffs with one
 * more argument.  variant 0: omega as above.  variant 1 ("removing ratio/clipping"): chi_t r_t replaced by 1 in
 * the policy contribution, omega_t = -(m_t / N) A + beta (m_t / N)(1 - exp(s_ref - s)).  variant 2: the
 * advantage-only signal omega_t := m_t A, whose exposure is sum_t |A_t| alpha_t.  "Removing KL" is beta = 0;
 * "removing activation weighting" is the sum_abs_omega output of hilore_unit_exposure; "removing
 * susceptibility" is kappa = 1.  ratio and clip_mask are reported as in hilore_grpo_coeffs.
 */
int hilore_grpo_coeffs_variant(const float *rewards, int64_t n_resp_total, int32_t G, int64_t resp_offset,
                               int64_t n_rows, int64_t T, const float *logp_new, const float *logp_old,
                               const float *logp_ref, const uint8_t *mask, int64_t N_norm,
                               const int64_t *N_norm_dev, float clip_eps, float beta, float adv_eps, int32_t variant,
                               float *adv_out, float *omega, float *ratio, uint8_t *clip_mask, void *stream);

/*
 * Structural sparsity of one record of coefficients (paragraph "Structural sparsity in diagnostic replays",
 * Eq. "diagnostic-clipping").  Over the n = n_rows * T padded response slots:
 *   counts[0] padding slots (m = 0);  counts[1] valid slots with zero advantage;  counts[2] valid slots with
 *   nonzero advantage on a flat clipped branch, (A > 0 and r > 1 + eps) or (A < 0 and r < 1 - eps);
 *   counts[3] slots whose coefficient is zero (padding counts as zero);  counts[4] = n, the common denominator.
 *   top_share = share of sum |omega| carried by the ceil(0.1 n) slots of largest |omega| (exact: the k-th largest
 *   value is found by a radix select on the bit patterns; ties at the threshold contribute as many copies as the
 *   decile still needs).   sum_abs = sum |omega| over valid slots.
 *   adv [n_rows], ratio / omega [n_rows, T] fp32, mask [n_rows, T] u8 (device); counts [5] int64, top_share,
 *   sum_abs (opt) fp64 on the device, 8-byte aligned; workspace hilore_omega_diagnostics_workspace_bytes() bytes.
 * Integer histograms and fixed-slot fp64 partial sums: the result is deterministic.
 */
int hilore_omega_diagnostics(const float *adv, const float *ratio, const uint8_t *mask, const float *omega,
                             int64_t n_rows, int64_t T, float clip_eps, int64_t *counts, double *top_share,
                             double *sum_abs, void *workspace, size_t workspace_bytes, void *stream);
size_t hilore_omega_diagnostics_workspace_bytes(void);

/*
 * Operational update exposure of U units over one microbatch
 * (Eq. "activation-token-weights", Eq. "mlp-weighted-exposure"):
 *     T_b = slots with mask = 1;  abar_u = mean_{t in T_b} a_{t,u}
 *     alpha_{t,u} = (a_{t,u} + eps_alpha) / (abar_u + eps_alpha)
 *     E_u = sum_{t in T_b} |omega_t| alpha_{t,u};       |T_b| = 0  =>  E_u = 0
 * a_{t,u} is row_rms[u*rms_ld + i*T + t - row_shift] for slot (i, t): row_shift = 1 takes the
 * activation row of the source position that predicts token t (the paper's wording), 0 the
 * token's own row.  A slot with t - row_shift < 0 has no activation row in this grid and carries no
 * weight: it counts neither in abar_u nor in E_u (the weights of the other slots of T_b average to
 * one); sum_abs_omega still covers all of T_b.
 *
 *   omega, mask   [n_rows, T] fp32 / u8 of the microbatch.    row_rms  [U, rms_ld] fp32, rms_ld >= n_rows*T.
 *   exposure      [U] fp32.     sum_abs_omega  opt, one fp32: sum_{t in T_b} |omega_t|.
 *   workspace     scratch of at least hilore_workspace_bytes(U, n_rows*T) bytes, 16-byte aligned; its
 *                 contents are overwritten (HILORE_WORKSPACE if too small).  Partial sums are kept in fp64
 *                 in fixed slots and added in a fixed order: the result is run-to-run deterministic.
 *   Launches: up to 16 tiles of 1024 tokens the call is ONE launch (the CTAs of a group of eight units are a
 *   thread-block cluster and add their sums through its shared memory; the workspace is not touched); larger
 *   microbatches take a second, small launch that adds the partial sums of the workspace.  Same bits either way.  With
 *   HILORE_DISABLE_CLUSTER_LAUNCH set in the environment (to anything but "0") no call of this library launches
 *   thread-block clusters.
 */
int hilore_unit_exposure(const float *omega, const uint8_t *mask, int64_t n_rows, int64_t T,
                         const float *row_rms, int32_t U, int64_t rms_ld, int32_t row_shift, float eps_alpha,
                         float *exposure, float *sum_abs_omega, void *workspace, size_t workspace_bytes,
                         void *stream);
size_t hilore_workspace_bytes(int32_t U, int64_t n_tok);

/*
 * hilore_unit_exposure for callers that cannot provide a workspace.  (The paper has no counterpart:
 * this is a packaging variant of the same reduction, with the same results.)
 *
 * Who needs it: code that must not allocate at the point where the exposure refresh runs -- for example
 * a saved-tensor hook running where the framework's caching allocator may not be re-entered, a process
 * whose device memory is wholly owned by another pool, or a latency-critical loop in which cudaMalloc
 * (which may synchronise the device) is ruled out.  The call allocates nothing on host or device: the
 * fp64 partial sums go to a fixed 1 MiB array inside the library image (hilore_static_scratch_bytes()),
 * which every GPU context that loads the library holds until it exits.
 *
 *   Arguments and results as hilore_unit_exposure, minus the workspace.
 *   Limit: hilore_workspace_bytes(U, n_rows*T) must not exceed the built-in array, i.e.
 *   (U + 1) * ceil(n_rows*T / 1024) <= 65536; larger problems return HILORE_WORKSPACE and nothing is
 *   launched (use hilore_unit_exposure with your own workspace).
 *   First call on a device: looks up the array's device address (once per device, with that device
 *   current) -- make this first call outside any stream capture.
 *   The array is shared by all calls and keeps the previous call's contents; every slot a call reads it
 *   has written first, so nothing needs clearing.  Two calls that overlap on the GPU (different streams
 *   without ordering, or several host threads) race on the array: order them.
 */
int hilore_unit_exposure_static(const float *omega, const uint8_t *mask, int64_t n_rows, int64_t T,
                                const float *row_rms, int32_t U, int64_t rms_ld, int32_t row_shift,
                                float eps_alpha, float *exposure, float *sum_abs_omega, void *stream);
size_t hilore_static_scratch_bytes(void);

/*
 * Compress one bf16 unit (the L action at capture time; Eq. "fp8-roundtrip" for fmt RAW) and, fused
 * into the same pass, the tokenwise activation magnitude a_t = sqrt(mean_j X_{t,j}^2) of
 * Eq. "activation-token-weights" (fp32 accumulation per block of 64, fp64 across the blocks of a row;
 * a row whose squares leave the fp32 range yields Inf).
 *   fmt RAW : code = cast_E4M3FN(x): one RNE rounding from the bf16 value; |x| up to 464 -> at most 448,
 *             larger, +-Inf and NaN -> sign | 0x7F.  block must be 0, scales NULL.
 *   fmt BLK : per block of 64 consecutive elements of a row: amax = max |x_i| over its finite elements;
 *             s = inv = 1 if amax == 0, if no element is finite, or if Q / amax overflows fp32;
 *             else s = fl32(amax / Q), inv = fl32(Q / amax), Q = 448 (E4M3FN) or 127 (INT8);
 *             q_i = fl32(x_i * inv); E4M3FN: code_i = RNE(q_i) saturating at +-448, NaN -> sign|0x7F;
 *             INT8: code_i = RNE(q_i) clamped to +-127, NaN -> 0x80.  block must be 64.
 *
 *   x        [rows, ld] bf16, ld >= cols, 32-byte aligned, ld % 16 == 0.    cols % 16 == 0 (RAW),
 *            cols % 64 == 0 (BLK).
 *   codes    [rows, cols] u8, 16-byte aligned; NULL => statistics only (row_rms must then be given).
 *   scales   [rows, cols/64] fp32 (BLK only).          row_rms  opt [rows] fp32.
 */
int hilore_compress(const void *x, int64_t rows, int64_t cols, int64_t ld, int32_t fmt, int32_t block,
                    uint8_t *codes, float *scales, float *row_rms, void *stream);

/*
 * Recover a compressed unit to bf16 (the L action at backward time).
 *   fmt RAW : x_hat = cast_BF16(code), exact; the NaN codes become a bf16 NaN.
 *   fmt BLK : x_hat = bf16_rne(fl32(value(code) * s)).
 *   codes [rows, cols] u8, 16-byte aligned;  scales [rows, cols/64] fp32 (BLK);
 *   out   [rows, ld_out] bf16, 32-byte aligned, ld_out % 16 == 0, ld_out >= cols.
 */
int hilore_recover(const uint8_t *codes, const float *scales, int64_t rows, int64_t cols, int32_t fmt,
                   int32_t block, void *out, int64_t ld_out, void *stream);

/*
 * Joint H / L / R allocation: the paper's allocator (Section "Joint H/L/R Allocation", Eq. "joint-allocation";
 * Appendix "Joint Allocation and Schedule Validation", Eqs. "allocation-grid", "allocation-integer-costs",
 * "allocation-dp").  Maximise sum_u dtau_u(a_u) subject to sum_u dmem_u(a_u) <= M_res,
 * sum_u d_u(a_u) <= delta_b with d(H) = d(R) = 0 and d(L) = psi_u, and a_u in A_u(q_u), exactly on the
 * conservative grid: h_B = M_res / N, h_d = delta_b / N, b_u(a) = ceil(dmem_u(a) / h_B),
 * r_u(a) = ceil(d_u(a) / h_d) (costs rounded up, so every grid-feasible assignment is feasible);
 * F_0(0,0) = 0, F_i(j,k) = max_a F_{i-1}(j - b, k - r) + dtau_i(a), candidates in the order R, H, L (first
 * maximum wins); terminal ties favour the lower risk state, then the lower memory state.  M_res == 0 leaves
 * one memory state (only actions without memory cost); delta_b == 0 disables L.  A NaN or negative psi_u makes
 * L unavailable for unit u; negative memory costs count as 0; R always has utility 0 and costs 0.
 * FP64 utilities as in the paper.  Layer i of the DP is one data-parallel pass over the (N+1)^2 states.
 *
 *   psi      [U] fp32 (device), e.g. written by hilore_plan_apply(PHASE_DECIDE).
 *   dtau, dmem   [U, 3] fp64 (device), indexed by the action code (R, H, L); column R is ignored.
 *   avail    [U] u8: the candidate plan q_u.        M_res, delta_b  host scalars, >= 0 (else INVALID_ARG).
 *   n_intervals  N; the paper uses 1024.
 *   action   [U] u8 out.   recompute  opt [U] u8 (1 iff R).   totals  opt [3] fp64: utility, memory, risk of the
 *            selection (8-byte aligned).
 *   workspace    hilore_allocate_workspace_bytes(U, N) bytes, 256-byte aligned (two value tables and the
 *            predecessor table; 105 MB for U = 84, N = 1024).
 * hilore_risk_budget: the microbatch budget delta_b = delta * N_b / sum_b' N_b' (host arithmetic).
 */
int hilore_allocate(int32_t U, const float *psi, const double *dtau, const double *dmem, const uint8_t *avail,
                    double M_res, double delta_b, int32_t n_intervals, uint8_t *action, uint8_t *recompute,
                    double *totals, void *workspace, size_t workspace_bytes, void *stream);
size_t hilore_allocate_workspace_bytes(int32_t U, int32_t n_intervals);
double hilore_risk_budget(double delta, int64_t N_b, int64_t N_total);

/*
 * Calibration of the L action (initialisation time, on the calibration microbatches).
 *   hilore_relative_error: e^L = ||x_hat - x||_2 / (||x||_2 + 1e-8) of one unit, operands widened to fp32 before
 *   the subtraction and the norms (Eq. "calibration-metrics"); fp32 per 16 elements, fp64 across them, per-CTA
 *   partial sums in fixed workspace slots, added in a fixed order (deterministic).
 *     x, xhat  [rows, ld] / [rows, ld_hat] bf16, 32-byte aligned, ld % 16 == 0; cols % 16 == 0.
 *     e_out    one fp64 on the device.    norms2   opt [2] fp64 on the device: ||x_hat - x||^2, ||x||^2.
 *     workspace  hilore_relative_error_workspace_bytes() bytes, 16-byte aligned.
 *   The mean reconstruction error ebar_u^L is the plain average of e^L over the calibration microbatches.
 *   hilore_fit_kappa: kappa_c = argmin_{kappa >= 0} sum_i (y_i - kappa x_i)^2 = max(0, sum x y / sum x^2)
 *   (Eq. "susceptibility"), x_i = E_{u,b} e^L_{u,b}; HOST arrays, host arithmetic; 0 if every x_i is 0.
 */
int hilore_relative_error(const void *x, const void *xhat, int64_t rows, int64_t cols, int64_t ld, int64_t ld_hat,
                          double *e_out, double *norms2, void *workspace, size_t workspace_bytes, void *stream);
size_t hilore_relative_error_workspace_bytes(void);
/*
 * The same e^L for x_hat = recover(compress(x)) in format fmt, fused: x is read once (2 B per element), encoded
 * and decoded in registers with the routines of hilore_compress / hilore_recover (x_hat is bit for bit what
 * they would produce), nothing else is written.  Shape and alignment rules of hilore_compress; workspace,
 * outputs and determinism as hilore_relative_error.  A unit with NaN codes gives e^L = NaN.
 */
int hilore_codec_relative_error(const void *x, int64_t rows, int64_t cols, int64_t ld, int32_t fmt, int32_t block,
                                double *e_out, double *norms2, void *workspace, size_t workspace_bytes, void *stream);
double hilore_fit_kappa(const double *x, const double *y, int64_t n);

/* One recovery unit of a microbatch: where its bf16 bundle lives and where its L representation goes.
 * A DEVICE array of these is passed to hilore_plan_apply.  Field rules as in hilore_compress /
 * hilore_recover; `out` may equal `x` only if the caller no longer needs the original. */
typedef struct hilore_unit {
    const void *x;   /* [rows, ld] bf16 saved activation                         */
    uint8_t *codes;  /* [rows, cols] u8                                          */
    float *scales;   /* [rows, cols/64] fp32, NULL for fmt RAW                   */
    void *out;       /* [rows, ld] bf16 reconstruction target of RECOVER         */
    float *row_rms;  /* opt [rows] fp32 token magnitudes written by CAPTURE      */
    int64_t rows, cols, ld;
    int32_t fmt, block;
} hilore_unit;

/*
 * Risk score, H / L / R gating and the batched capture / encode / recover of all units of a microbatch
 * in ONE launch per phase and 96 units (a longer table runs as consecutive launches over slices of 96)
 * (Eq. "token-weighted-risk": psi_u = kappa_c(u) E_u ebar_u; Eq. "available-recovery-actions").  All decisions
 * stay on the device: the gating arrays are read by the kernels, so no phase needs a host synchronisation.
 *
 *   units_dev   [U] hilore_unit on the DEVICE.     units_host  the same table on the HOST (read during
 *               the call for validation and launch sizing; must match units_dev).
 *   avail       [U] u8: the candidate plan q_u in {R, H, L} fixed before forward.
 *   action_io   [U] u8: DECIDE writes it; the other phases read it.
 *   DECIDE:  if exposure != NULL: psi_u = fl32(fl32(kappa_u * E_u) * ebar_u); desired = L if psi < tau_lo,
 *            H if psi >= tau_hi, else R (NaN -> R) -- a threshold stand-in for the paper's knapsack
 *            allocator; if exposure == NULL the desired action is action_io[u] as given.
 *            Then action = desired if it is in A_u(q_u) (q = H: {H,L,R}; q = L: {L,R}; q = R: {R}), else R.
 *            Writes psi (opt), action_io, recompute[u] = (action == R), retained_bytes[u] = 2*rows*cols (H),
 *            rows*cols + 4*rows*cols/64 (L; no scale term for fmt RAW), 0 (R).
 *   CAPTURE: q = L: compress into codes / scales and write row_rms; q = H: row_rms only; q = R: untouched.
 *   ENCODE:  units with q = H and action = L are compressed (post-forward encoding).
 *   RECOVER: units with action = L are decoded into `out`; H and R units are untouched (H keeps its
 *            exact bundle, Prop. "exact recovery equivalence"; R is recomputed by the caller).
 */
int hilore_plan_apply(const hilore_unit *units_dev, const hilore_unit *units_host, int32_t U, int32_t phase,
                      const float *exposure, const float *kappa, const float *ebar, float tau_lo,
                      float tau_hi, const uint8_t *avail, uint8_t *action_io, float *psi, uint8_t *recompute,
                      uint64_t *retained_bytes, void *stream);

/* ================================================================================================================
 * The two ends of the actor update that touch the model: from logits to the log-probabilities that
 * hilore_grpo_coeffs reads, from its coefficients back to a gradient of the logits, and the optimizer step
 * (Algorithm 1, lines "Forward", "Backward", "OptimizerStep").  The paper leaves these to its learner; their
 * definitions are stated here.
 * ================================================================================================================ */

/* ---- element types of logits, parameters and gradients ---- */
enum { HILORE_BF16 = 0, HILORE_F32 = 1 };

/*
 * What was imposed on the logits of a row when its token was sampled.  A HOST struct of DEVICE pointers, read during
 * the call; every part is optional (NULL) and has one entry per row unless it says otherwise.  For token v with logit x
 * in row r:
 *     c_all = occurrences of v in the row's history, c_out = those in its generated part
 *     z = x;   c_all > 0:  z = x > 0 ? x / repetition : x * repetition
 *     z = z - frequency * c_out - (c_out > 0 ? presence : 0)
 *     z = z + bias of v
 *     z = z / temperature;      v denied by the grammar:  z = -inf (also where x is NaN or Inf)
 * evaluated in fp32, rounded once to the type of the result.
 *   temperature   [n_rows] fp32; a value that is not > 0 (0: greedy) leaves the row unscaled, Inf makes its allowed tokens alike.
 *   repetition, frequency, presence   [n_rows] fp32 each; NULL = 1, 0, 0.  repetition > 0.
 *   tokens        [n_tokens] int32, the sequences of the batch packed back to back.  Row r's history is
 *                 tokens[hist_begin[r] .. hist_end[r]-1], of which the part from resp_begin[r] on was generated, the
 *                 part before it is the prompt.  Rows may share and overlap: the slots of one training sequence are rows
 *                 with the same hist_begin and growing hist_end.  Any length, 0 included; ranges are clamped to
 *                 [0, n_tokens); entries outside [0, V) (padding) count nowhere.  tokens may be NULL iff n_tokens = 0.
 *   bias_tokens, bias_values   [n_bias] int32 / fp32;  bias_offsets [n_rows + 1] int64: row r's list is entries
 *                 bias_offsets[r] .. bias_offsets[r+1]-1.  Where a list names a token twice, the last entry counts.
 *   allow         [n_allow, allow_ld] 32-bit words, allow_ld >= ceil(V / 32): bit v % 32 of word v / 32 is 1 where the
 *                 grammar allows token v.   allow_row [n_rows] int32 selects the mask of a row; an index outside
 *                 [0, n_allow) (-1) leaves it free.  NULL = row r uses mask r (n_allow >= n_rows).
 */
typedef struct hilore_logit_rules {
    const float *temperature, *repetition, *frequency, *presence;
    const int32_t *tokens;
    int64_t n_tokens;
    const int64_t *hist_begin, *resp_begin, *hist_end;
    const int32_t *bias_tokens;
    const float *bias_values;
    int64_t n_bias;
    const int64_t *bias_offsets;
    const int32_t *allow;
    const int32_t *allow_row;
    int64_t n_allow, allow_ld;
} hilore_logit_rules;

/*
 * Applies the rules to n_rows rows of V logits (one row per sequence at a decoding step, one per slot of a training
 * microbatch), and the gradient of that: grad_in = grad_out * dz/dx, with dz/dx = 1 / temperature, times 1 / repetition
 * (x > 0) or repetition (x <= 0) for a token of the history, and 0 for a denied one (whatever grad_out holds there).
 *   logits       [n_rows, ld] of dtype (HILORE_BF16 or HILORE_F32), ld >= V: any ld and any address that the element
 *                type allows; rows whose addresses agree modulo 32 bytes with those of the output are the fast case.
 *   out          [n_rows, ld_out] of the same type; may be `logits` itself with the same ld (HILORE_SHAPE if they differ).
 *   grad_out, grad_in   [n_rows, ld_..] of the same type; grad_in may be grad_out with the same ld, but not `logits`
 *                (HILORE_INVALID_ARG).  Of `logits` only the entries of history tokens are read.
 *   Otherwise the output must not overlap an input.  Nothing is read or written between the rows.
 *   Limits: V and n_rows at most 2^31 - 2^16, and n_rows * ceil((V + 15) / 2048) below 2^31 (HILORE_SHAPE).
 */
int hilore_logits_apply(const void *logits, int32_t dtype, int64_t n_rows, int64_t V, int64_t ld,
                        const hilore_logit_rules *rules, void *out, int64_t ld_out, void *stream);
int hilore_logits_apply_backward(const void *logits, int32_t dtype, int64_t n_rows, int64_t V, int64_t ld,
                                 const hilore_logit_rules *rules, const void *grad_out, int64_t ld_grad_out,
                                 void *grad_in, int64_t ld_grad_in, void *stream);

/*
 * Log-probability of one token per row under the processed logits z (rules may be NULL: z = logits), the s_t of
 * Eq. "grpo-objective", in one pass over the logits:
 *     lse_r = ln sum_v exp(z_v);   logp_r = z_a - lse_r, a = targets[r];   entropy_r = lse_r - sum_v p_v z_v
 * with fp32 statistics relative to the row's running maximum.
 *   targets      [n_rows] int32; a row whose target lies outside [0, V) is a slot without a token: it is not read and
 *                its logp, lse and entropy are 0.
 *   logp         [n_rows] fp32.    lse  opt [n_rows] fp32, what hilore_token_logp_backward needs.
 *   entropy      opt [n_rows] fp32 (a statistic: the gradient below is that of logp alone).
 *   A denied target has logp = -inf.  A row in which nothing is allowed has logp = lse = -inf, entropy 0.  A NaN among
 *   the allowed logits makes the row NaN; +Inf gives lse = +Inf and entropy NaN.
 *   A row is the work of one CTA, or of a thread-block cluster of up to 8 when there are few rows (never with
 *   HILORE_DISABLE_CLUSTER_LAUNCH): logp, lse and entropy of a row depend in their last bits on that choice and on the
 *   row's address modulo 32 bytes, not on the other rows of the call; the same call gives the same bits.
 *
 * hilore_token_logp_backward: grad_v = omega_r (1[v = a] - exp(z_v - lse_r)) dz_v/dx_v, the gradient of sum_r omega_r
 * logp_r with respect to the logits, for the omega of hilore_grpo_coeffs.
 *   omega, lse   [n_rows] fp32.    grad  [n_rows, ld_grad] of dtype; may be `logits` with the same ld (HILORE_SHAPE if they differ).
 *   Rows with omega = 0, without a token, with a denied target or with lse <= -1e30 (nothing to choose from) get zeros
 *   and are not read.
 */
int hilore_token_logp(const void *logits, int32_t dtype, int64_t n_rows, int64_t V, int64_t ld,
                      const hilore_logit_rules *rules, const int32_t *targets, float *logp, float *lse, float *entropy,
                      void *stream);
int hilore_token_logp_backward(const void *logits, int32_t dtype, int64_t n_rows, int64_t V, int64_t ld,
                               const hilore_logit_rules *rules, const int32_t *targets, const float *lse,
                               const float *omega, void *grad, int64_t ld_grad, void *stream);

/* ---- storage of the optimizer's moments ---- */
enum {
    HILORE_STATE_F32 = 0,    /* m, v fp32                                                                  */
    HILORE_STATE_E4M3FN = 1  /* m and sqrt(v) as E4M3FN codes with one fp32 scale per 64 elements, the block
                                format of HILORE_FMT_E4M3FN_BLK: 2.125 bytes per element instead of 8        */
};
#define HILORE_PARAM_TILE 1024

/* One tensor of an optimizer step.  A DEVICE array of these is passed beside the same array on the HOST. */
typedef struct hilore_param {
    void *p;               /* [n] parameters of p_dtype, updated                                              */
    float *master;         /* opt [n] fp32 copy of a bf16 parameter: it is updated and p is its rounding (p is not read) */
    const void *g;         /* [n] gradients of g_dtype                                                        */
    void *m, *v;           /* [n] fp32 moments, or [n] u8 codes of m and of sqrt(v)                           */
    float *m_scale, *v_scale; /* [ceil(n / 64)] fp32 scales of HILORE_STATE_E4M3FN, else NULL                 */
    int64_t n;             /* elements; 0 is allowed                                                          */
    int64_t first;         /* sum of ceil(n / HILORE_PARAM_TILE) over the entries before this one (HILORE_SHAPE if not) */
    int32_t p_dtype, g_dtype, state;
    float weight_decay;
} hilore_param;

/*
 * Global norm of the gradients of a table, ||g|| = sqrt(sum over all tensors of g^2), and the factor that clips it:
 * scale = min(1, max_norm / (norm + 1e-6)), NaN where a gradient is not finite.  Squares are added in fp32 per 32
 * elements (fp64 where that overflows or loses bits to the smallest numbers) and in fp64 beyond, in a fixed order: run-to-run
 * deterministic.  A norm beyond fp32 is stored as Inf; its scale is right.
 *   Of the table only g, g_dtype, n and first are read.    max_norm >= 0 (Inf: no clipping).
 *   norm, scale   opt one fp32 each on the device, at least one of them.
 *   workspace     hilore_grad_norm_workspace_bytes() bytes, 16-byte aligned.
 */
int hilore_grad_norm(const hilore_param *params_dev, const hilore_param *params_host, int32_t n_params, double max_norm,
                     float *norm, float *scale, void *workspace, size_t workspace_bytes, void *stream);
size_t hilore_grad_norm_workspace_bytes(void);

/*
 * One AdamW step over all tensors of a table in ONE launch.  Per element, in fp32, with g = grad_scale * gradient:
 *     m = beta1 m + (1 - beta1) g;        v = beta2 v + (1 - beta2) g^2
 *     p = p - lr ( weight_decay p + (m / (1 - beta1^t)) / (sqrt(v / (1 - beta2^t)) + eps) )
 * m, v and the codes made from them take every operation rounded by itself, in this order ((1 - beta2) g first,
 * then times g), so they are the same bits in any evaluation that does so.  sqrt(v) of HILORE_STATE_E4M3FN is rounded to
 * nearest; below v = 2^-102 it may be the next number instead.  No result depends on a tensor's alignment or place in the
 * table, nor on the values of other blocks of 64.
 * The parameter (or its fp32 master copy) is rounded to its type to nearest even.
 *   HILORE_STATE_E4M3FN: the moments of the step enter the update in fp32; then, per block of 64 consecutive elements of
 *     a tensor (the last one may be shorter), m and sqrt(v) are stored as codes by the rule of HILORE_FMT_E4M3FN_BLK in
 *     hilore_compress (amax over finite elements, RNE; zeros and what is too small to be scaled get scale 1), with
 *     scale = fl32(amax * fl32(1 / 448)) and inv = fl32(448 * fl32(1 / amax)), and one addition: a positive sqrt(v)
 *     that would round to zero takes the smallest code, so that a later step never divides by eps alone where a
 *     gradient has been.  v and each of its two terms count as zero below 2^-126, and so does an eps below that.  Codes
 *     and scales of a first step are zeros.
 *   params_dev, params_host   the table, as for hilore_plan_apply: [n_params] on the device and the same on the host
 *             (read during the call for validation and launch sizing).  Tensors may be of different types, sizes and
 *             state formats.  Any alignment that the types allow; tensors whose p, master and g are 32-byte aligned and
 *             whose m and v are 32-byte (fp32) or 16-byte (codes) aligned move in vectors.  They must not overlap.
 *   lr, lr_dev       lr_dev (opt, one fp32 on the device) replaces lr.
 *   step, step_dev   t >= 1; step_dev (opt, one int64 on the device, >= 1) replaces it: with both, a captured graph can
 *             be replayed over a schedule.
 *   grad_scale       opt, one fp32 on the device, e.g. the scale of hilore_grad_norm.  Where it is not finite the step
 *             leaves parameters and moments as they are.
 */
int hilore_adamw_step(const hilore_param *params_dev, const hilore_param *params_host, int32_t n_params, double lr,
                      const float *lr_dev, double beta1, double beta2, double eps, int64_t step, const int64_t *step_dev,
                      const float *grad_scale, void *stream);

/* ================================================================================================================
 * From rewards to the gradient of the log-probabilities beyond hilore_grpo_coeffs: advantages and returns per token,
 * the clipped policy loss and the preference loss.  omega is dL/ds_t in all of them, what hilore_token_logp_backward
 * reads.  The paper has GRPO alone; the definitions are stated here.
 *
 * Sequences, in every call of this part:
 *   cu_seqlens   [n_seq + 1] int32 as in hilore_grpo_coeffs_packed, or NULL: n_seq rows of n_tok / n_seq slots each
 *                (n_tok % n_seq must be 0, HILORE_SHAPE).  cu_seqlens[0] counts as 0.  Tokens from cu_seqlens[n_seq] on
 *                belong to no sequence: whatever they hold changes nothing and nothing of theirs is written, so a captured call serves
 *                batches of any number of tokens up to n_tok (which the tensors have; blocks of 256 tokens are read whole).
 *                Whatever cu_seqlens holds, no kernel indexes outside [0, n_seq] or [0, n_tok).
 *   mask         opt [n_tok] u8 (0 / not 0); NULL: every token is valid.  Masked tokens (prompt, tool outputs, padding) may
 *                hold anything, NaN included: they change nothing and their outputs are 0.
 *   Tensors with an entry per token may have any address that their type allows; with fp32 at 32, bf16 at 16 and masks at 8
 *   bytes eight tokens move at a time.  Results do not depend on that, nor on scheduling: the same call gives the same bits.
 *   Where in a call a sequence lies decides in which order sums are added up: its results may differ in a last bit, no more, with the
 *   sequences around it.  Sums are fp64; the statistics of RATIO_TOKEN add eight neighbouring tokens in fp32 first.  n_seq and
 *   n_tok at most 2^31 - 2^16 (HILORE_SHAPE).
 *   Small policy losses (up to 16384 tokens, RATIO_TOKEN with MEAN_TOKENS) are one thread-block cluster, two launches with
 *   HILORE_DISABLE_CLUSTER_LAUNCH set in the environment.
 *   workspace    the bytes of the call's .._workspace_bytes, 16-byte aligned, overwritten.
 * ================================================================================================================ */

/*
 * Advantages and returns of every valid token, a gated linear recurrence from the end of the sequence.  Over its valid tokens
 * k = 1 .. n (masked ones are stepped over, so tool outputs do not part a response):
 *     A_k = r_k + q_k - V_k + gamma lambda c_k A_{k+1},   A_{n+1} = 0
 *     q_k = gamma V_{k+1} (k < n),   q_n = outcome + gamma bootstrap;        returns_k = A_k + V_k
 * Generalised advantage estimation at c = 1; discounted rewards to go at lambda = 1 without values.  fp64 inside, rounded once.
 *   rewards      opt [n_tok] fp32.    outcome  opt [n_seq] fp32, the reward of the whole response, earned at its last valid token.
 *   values       opt [n_tok] of values_dtype (HILORE_BF16 or HILORE_F32).    bootstrap  opt [n_seq] fp32, the value behind a
 *                response that was cut short.    trace  opt [n_tok] fp32: c_k, e.g. clipped importance ratios.
 *   gamma, lambda   in [0, 1].
 *   adv, returns    opt [n_tok] fp32.    moments  opt [2] fp32: mean and population standard deviation of the advantages of the call's
 *                valid tokens (0, 0 where there are none), in a fixed order of additions.  At least one of the three.
 *   What is not finite makes the tokens before it in its sequence NaN or infinite, and no others; so do products of trace beyond fp64.
 *   Time grows faster than the length of a single sequence beyond some ten million tokens: 16 M 0.2 ms, 60 M 1.4 ms, 240 M 27 ms.
 *
 * hilore_advantages_backward: the gradients of sum_k (grad_adv_k A_k + grad_returns_k returns_k),
 *     G_k = grad_adv_k + grad_returns_k + gamma lambda c_{k-1} G_{k-1};     d r_k = G_k
 *     d V_k = grad_returns_k - G_k + gamma G_{k-1};   d c_k = gamma lambda A_{k+1} G_k;   d outcome = G_n;   d bootstrap = gamma G_n
 * (0 for a sequence without a valid token).
 *   grad_adv, grad_returns   opt [n_tok] fp32 (NULL: zeros).    adv  [n_tok] fp32 as written by the forward call, needed for grad_trace.
 *   grad_rewards, grad_values, grad_trace   opt [n_tok] fp32.    grad_outcome, grad_bootstrap  opt [n_seq] fp32.
 */
int hilore_advantages(const float *rewards, const float *outcome, const void *values, int32_t values_dtype,
                      const float *bootstrap, const float *trace, const uint8_t *mask, const int32_t *cu_seqlens, int64_t n_seq,
                      int64_t n_tok, double gamma, double lambda, float *adv, float *returns, float *moments, void *workspace,
                      size_t workspace_bytes, void *stream);
int hilore_advantages_backward(const float *grad_adv, const float *grad_returns, const float *adv, const float *trace,
                               const uint8_t *mask, const int32_t *cu_seqlens, int64_t n_seq, int64_t n_tok, double gamma,
                               double lambda, float *grad_rewards, float *grad_outcome, float *grad_values,
                               float *grad_bootstrap, float *grad_trace, void *workspace, size_t workspace_bytes, void *stream);
size_t hilore_advantages_workspace_bytes(int64_t n_tok);

/* ---- ratios, means and KL estimators of the policy loss ---- */
enum { HILORE_RATIO_TOKEN = 0, HILORE_RATIO_SEQUENCE = 1 };
enum { HILORE_MEAN_TOKENS = 0, HILORE_MEAN_SEQUENCES = 1 };
enum { HILORE_KL_K1 = 1, HILORE_KL_K2 = 2, HILORE_KL_K3 = 3 };

/* What a policy loss is made of.  A HOST struct, read during the call. */
typedef struct hilore_policy_terms {
    double clip_low, clip_high; /* the ratio is held in [1 - clip_low, 1 + clip_high]; clip_low in [0, 1], clip_high >= 0, Inf: no bound */
    double dual_clip;           /* 0: none; c >= 1: at A < 0 the ratio counts as c at most                  */
    double beta;                /* weight of the KL term                                                    */
    double rollout_cap;         /* > 0; most that a rollout weight may be (Inf: no bound)                   */
    double adv_eps;             /* >= 0; added to the standard deviation where advantages are whitened      */
    int32_t ratio, mean, kl;    /* HILORE_RATIO_.., HILORE_MEAN_.., HILORE_KL_..                            */
    int32_t adv_per_token;      /* 1: adv has an entry per token, 0: per sequence (always 0 for HILORE_RATIO_SEQUENCE) */
} hilore_policy_terms;

/*
 * Clipped policy loss over the valid tokens of a call and its gradient, forward and backward in one call:
 *     rho = exp(s - s_old) per token, or exp(mean over the sequence's valid tokens of s - s_old) for HILORE_RATIO_SEQUENCE
 *     u   = A >= 0: min(rho, 1 + clip_high);   A < 0: min(max(rho, 1 - clip_low), dual_clip)
 *     i   = min(rollout_cap, exp(s_old - s_rollout)), of the sequence's mean likewise; a constant, 1 without logp_rollout
 *     kl  = with e = s_ref - s:  K1 -e,  K2 e^2 / 2,  K3 exp(e) - e - 1
 *     w   = 1 / N (HILORE_MEAN_TOKENS), 1 / (N |T_s|) with the sequence's valid tokens |T_s| (HILORE_MEAN_SEQUENCES)
 *     L   = sum_t w ( -i A u + beta kl );     omega_t = dL/ds_t * grad_loss
 * On a flat branch (u a bound) the policy term's gradient is exactly 0; rho on its bound is not beyond it.  Which side a
 * token is on is decided on s - s_old in fp64, so it is decided as the formula does.  An infinite advantage is on a flat branch like
 * any other; one that is NaN is on none, and makes its tokens' omega NaN.  exp(e), and for RATIO_TOKEN ratios and weights, are fp32:
 * from a logarithm of 88.7 on they are infinite where no bound holds them.  An A of 0 is nothing even there.
 *   logp, logp_old   [n_tok] fp32.    logp_ref  opt [n_tok] fp32, needed unless beta = 0.    logp_rollout  opt [n_tok] fp32,
 *                    what the engine that sampled reported.
 *   adv              [n_tok] or [n_seq] fp32.    adv_moments  opt [2] fp32 as written by hilore_advantages:
 *                    A = (adv - mean) / (standard deviation + adv_eps).
 *   N_norm, N_norm_dev   as in hilore_grpo_coeffs: the whole batch's valid tokens or its sequences, so that the losses and
 *                    gradients of microbatches add up.
 *   grad_loss        opt one fp32 on the device: the gradient of L itself (loss scaling).  1 if NULL.
 *   stats            [5] fp32, sums of this call: L; its policy term; sum w kl (0 without logp_ref); sum w over the tokens with A != 0
 *                    on a flat branch; sum w (s_old - s).
 *   omega            [n_tok] fp32.
 */
int hilore_policy_loss(const float *logp, const float *logp_old, const float *logp_ref, const float *logp_rollout,
                       const uint8_t *mask, const float *adv, const float *adv_moments, const int32_t *cu_seqlens, int64_t n_seq,
                       int64_t n_tok, const hilore_policy_terms *terms, int64_t N_norm, const int64_t *N_norm_dev,
                       const float *grad_loss, float *stats, float *omega, void *workspace, size_t workspace_bytes, void *stream);
size_t hilore_policy_loss_workspace_bytes(int64_t n_seq, int64_t n_tok);

enum { HILORE_PREF_SIGMOID = 0, HILORE_PREF_HINGE = 1, HILORE_PREF_SQUARE = 2 };

/* What a preference loss is made of.  A HOST struct, read during the call. */
typedef struct hilore_preference_terms {
    double beta;                  /* > 0, scale of the scores                                                    */
    double margin, margin_reward; /* the gap asked for: margin + margin_reward (R_w - R_l)                       */
    double smoothing;             /* in [0, 1], HILORE_PREF_SIGMOID alone: share of pairs taken the other way round */
    double nll;                   /* weight of the winners' negative log-likelihood                              */
    int32_t loss, length_mean;    /* HILORE_PREF_..; 1: scores are means over a response's tokens, 0: sums       */
} hilore_preference_terms;

/*
 * Preference loss on pairs of responses to the same prompt, and its gradient.  The G responses of prompt p are sequences
 * p*G .. p*G+G-1; each pair of them with R_w > R_l counts (G = 2 with rewards 1 and 0: chosen and rejected), unless one of
 * the two has no valid token or a reward is NaN:
 *     h  = beta * sum (or mean) over the valid tokens of s - s_ref
 *     z  = h_w - h_l - margin - margin_reward (R_w - R_l)
 *     l  = SIGMOID -(1 - smoothing) ln sigma(z) - smoothing ln sigma(-z), a logarithm of weight 0 left out;   HINGE max(0, 1 - z);
 *          SQUARE ((z - 1/2) / beta)^2
 *     L  = 1/N sum over pairs of ( l + nll * (-mean over the winner's valid tokens of s) );     omega_t = dL/ds_t * grad_loss
 *   logp         [n_tok] fp32.    logp_ref  opt [n_tok] fp32 (NULL: without a reference).    rewards  [n_seq] fp32.
 *                G in [1, 1024], n_seq % G must be 0 (HILORE_SHAPE).
 *   N_norm, N_norm_dev   pairs of the whole batch; N_norm = 0: those of this call.  A device value <= 0 gives omega = 0 and stats 0.
 *   scores       opt [n_seq] fp32: h (0 without a valid token).    pairs  opt one int64 on the device: the pairs of this call.
 *   stats        [4] fp32, each the sum over this call's pairs divided by N: L; pairs with h_w > h_l; h_w - h_l; the mean
 *                above, -mean s of the winner.  Responses in no pair have no part in them, losers none in the last.
 *   omega        [n_tok] fp32.    grad_loss as in hilore_policy_loss.
 */
int hilore_preference_loss(const float *logp, const float *logp_ref, const uint8_t *mask, const float *rewards, int32_t G,
                           const int32_t *cu_seqlens, int64_t n_seq, int64_t n_tok, const hilore_preference_terms *terms,
                           int64_t N_norm, const int64_t *N_norm_dev, const float *grad_loss, float *scores, int64_t *pairs,
                           float *stats, float *omega, void *workspace, size_t workspace_bytes, void *stream);
size_t hilore_preference_loss_workspace_bytes(int64_t n_seq, int64_t n_tok);

#ifdef __cplusplus
}
#endif
#endif /* HILORE_H */
