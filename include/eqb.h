/*
 * eqb.h - C ABI of the MI355X (gfx950) library for one MoE layer's routing
 * and Exact Quantile Balancing (EQB) statistics.
 *
 * Method: arXiv 2609.28053, "Exact Quantile Balancing and Load-Error Injection
 * for Mixture-of-Experts".  Notation follows the paper:
 *   z[T,E]   router logits (BF16), b[E] expert bias (binary32),
 *   I_t      = Top-K(z_t + b)                          (Sec. 2, Eq. 1)
 *   s_{t,e}  = sigmoid(z_{t,e}) for e in I_t, unbiased  (Sec. 2, Eq. 1)
 *   f_e      = #{t : e in I_t}                          (Sec. 2)
 *   tau_t    = (K+1)st largest entry of z_t + b         (Sec. 2, "Quantile Balancing")
 *   margin   = tau_t - z_{t,e} as a BF16 value, key kappa = (h, l) (Appendix C, Algorithm 1)
 *   r        = T*K/E, the rank of the balanced quantile  (Sec. 3)
 *   H_{p,e,u}, L_{p,e,v}  coarse / fine counts of partition p (Algorithm 1, steps 1 and 4)
 *
 * Conventions shared by every call
 * --------------------------------
 * Memory.  Every pointer is a DEVICE pointer except `part_off`, which is a
 *   HOST array read during the call.  The caller allocates and owns every
 *   buffer; the library allocates nothing and keeps no pointer after the call
 *   returns.  Calls only enqueue work on `stream` (a hipStream_t, NULL = the
 *   default stream) and never synchronise the host.
 * Layouts.  Row-major.  z is [T,E] BF16 bit patterns (uint16), 16-byte
 *   aligned.  topk_idx/topk_score are [T,K].  Count arrays are int32:
 *   loads [P,E], coarse/fine histograms [P,E,256] (slab p = partition p).
 * Partitions.  Tokens are split into P contiguous ranges
 *   [part_off[p], part_off[p+1]), standing in for P data-parallel ranks.
 *   part_off has P+1 entries, part_off[0] = 0, part_off[P] = T, non-decreasing
 *   (empty partitions are allowed).  part_off = NULL means P = 1.  Summing the
 *   slabs over p is the all-reduce of Algorithm 1, steps 2 and 5.
 * Accumulation.  Histogram and load outputs are ACCUMULATED (+=): zero them
 *   before the first call of a layer.  Every count must stay in [0, 2^31)
 *   before and after a call: the kernels may add to two adjacent int32
 *   counters with one 64-bit atomic, which is exact only while no counter
 *   wraps.  Counts are token counts, so T < 2^31 keeps them in range.
 * Numerics.  z + b and tau - z are single binary32 operations rounded to
 *   nearest even, with subnormals kept; a margin is rounded once to BF16
 *   (nearest, ties to even).  kappa(bits) = bits ^ (sign ? 0xFFFF : 0x8000),
 *   which orders BF16 values as IEEE totalOrder (-0 < +0).  Top-K ties go to
 *   the lower expert index (-0 and +0 are equal there); I_t is written in rank
 *   order (score descending, then index ascending).  Inputs must be finite.
 * Supported shapes.  E in {8, 16, 32, 64, 128, 256}; 1 <= K < E;
 *   0 <= T < 2^31; 1 <= P <= EQB_MAX_PARTITIONS.
 * Errors.  Every argument check runs before anything is enqueued, so a call
 *   that returns an error has left the stream untouched.  T = 0 returns
 *   EQB_OK and enqueues nothing.
 * Concurrency.  The library keeps no state between calls except a per-device
 *   cache of the compute-unit count (filled once, thread-safe) and the
 *   per-thread test cap of eqb_set_max_blocks.  Calls may be made from
 *   several host threads and on several streams at once; calls that write
 *   the same buffers must be ordered by the caller (same stream, or events).
 */
#ifndef EQB_H
#define EQB_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef int32_t eqb_status;

#define EQB_OK               0
#define EQB_ERR_INVALID_ARG  1   /* null pointer, bad K/T/P, bad partition table */
#define EQB_ERR_UNSUPPORTED  2   /* E outside the supported set, misaligned z */
#define EQB_ERR_RANK         3   /* r < 1 or r > number of counted margins */
#define EQB_ERR_HIP          4   /* the HIP runtime reported a launch error */
#define EQB_ERR_SCRATCH      5   /* eqb_layer_noalloc: the layer needs more than
                                    EQB_NOALLOC_SCRATCH_BYTES of working memory */

#define EQB_NBINS            256
#define EQB_MAX_PARTITIONS   256

/* Device status word written by eqb_select_quantile. */
#define EQB_DEV_OK                 0
#define EQB_DEV_RANK_EXCEEDS_COUNT 1   /* an expert holds fewer than r (or rho) counts */

/*
 * Routing (Sec. 2, Eq. 1 and "Quantile Balancing"), optionally fused with
 * the coarse pass of Algorithm 1 (step 1).
 *   z [T,E] bf16 bits, b [E] binary32                     (in)
 *   topk_idx [T,K] int32, topk_score [T,K] binary32,
 *   tau [T] binary32                                      (out)
 *   load [P,E] int32 (nullable)                           (+= f_{p,e})
 *   hist_hi [P,E,256] int32 (nullable)                    (+= H_{p,e,u}, u = h of the margin key)
 * tau_t carries the bit pattern of the entry at rank K (0-based).
 * Returns EQB_ERR_INVALID_ARG, EQB_ERR_UNSUPPORTED or EQB_ERR_HIP on failure.
 */
eqb_status eqb_route_topk(const uint16_t* z, const float* b, int64_t T, int32_t E, int32_t K,
                          int32_t* topk_idx, float* topk_score, float* tau,
                          const int64_t* part_off, int32_t P,
                          int32_t* load, int32_t* hist_hi, void* stream);

/*
 * Coarse pass alone (Algorithm 1, step 1): hist_hi[p,e,u] += #{t in p : h_{t,e} = u},
 * where (h, l) = kappa(bf16(tau_t - z_{t,e})).
 *   z [T,E] bf16 bits, tau [T] binary32 (in); hist_hi [P,E,256] int32 (+=).
 */
eqb_status eqb_margin_hist_pass1(const uint16_t* z, const float* tau, int64_t T, int32_t E,
                                 const int64_t* part_off, int32_t P, int32_t* hist_hi,
                                 void* stream);

/*
 * Selection (Algorithm 1, steps 2-3 for pass = 1; steps 5-6 for pass = 2).
 * Both passes first sum the P slabs of `hist` (the all-reduce, steps 2 and 5).
 * pass = 1: hist = H_p [P,E,256].  Writes sel_hi[e] = u_e = min{u : sum_{j<=u} H[e,j] >= r}
 *   and rank_in_bin[e] = rho_e = r - sum_{j<u_e} H[e,j].
 * pass = 2: hist = L_p [P,E,256], reads sel_hi and rank_in_bin.  Writes
 *   sel_lo[e] = v_e = min{v : sum_{j<=v} L[e,j] >= rho_e}, q_bf16[e] = kappa^-1(u_e, v_e)
 *   (the exact r-th smallest BF16 margin, b_hat_e) and, if b_next != NULL,
 *   the centred bias b_next[e] = b_hat_e - mean(b_hat) (Eq. 2): a binary64 sum in
 *   ascending e, divided by E, subtracted in binary64 and rounded once to binary32.
 *   r is the rank over the whole batch (all partitions), see eqb_rank.
 *   hist_sum [E,256] int32 (nullable): receives the summed counts.
 *   dev_status (nullable, int32): set to EQB_DEV_RANK_EXCEEDS_COUNT when some
 *   expert holds fewer than r (pass 1) or rho_e (pass 2) counts; it is never
 *   cleared by the library.  The affected sel_hi/sel_lo entries are -1 and
 *   q_bf16 is a NaN pattern.
 * Returns EQB_ERR_RANK if r < 1; other errors as above.
 */
eqb_status eqb_select_quantile(int32_t pass, const int32_t* hist, int32_t P, int32_t E, int64_t r,
                               int32_t* sel_hi, int64_t* rank_in_bin,
                               int32_t* sel_lo, uint16_t* q_bf16, float* b_next,
                               int32_t* hist_sum, int32_t* dev_status, void* stream);

/*
 * Fine pass (Algorithm 1, step 4): rescans z and tau and, for margins whose
 * high byte equals sel_hi[e] = u_e, hist_lo[p,e,v] += #{t in p : h_{t,e} = u_e, l_{t,e} = v}.
 *   z [T,E] bf16 bits, tau [T], sel_hi [E] int32 (in); hist_lo [P,E,256] int32 (+=).
 */
eqb_status eqb_margin_hist_pass2(const uint16_t* z, const float* tau, int64_t T, int32_t E,
                                 const int32_t* sel_hi, const int64_t* part_off, int32_t P,
                                 int32_t* hist_lo, void* stream);

/*
 * Expert loads (Sec. 2): load[p,e] += #{t in p : e in I_t} from topk_idx [T,K].
 * Entries outside [0, E) are not counted.
 */
eqb_status eqb_expert_load(const int32_t* topk_idx, int64_t T, int32_t K, int32_t E,
                           const int64_t* part_off, int32_t P, int32_t* load, void* stream);

/*
 * The statistics EQB is compared with (Sec. 2, after Eq. 2; Sec. 3).
 *
 * Rank-averaged QB: every shard (partition) takes the K/E quantile of its own
 * margins and the shards average them.  Each shard's quantile is exact, found
 * by the two passes of Algorithm 1 run on that shard's counts alone:
 *   eqb_select_quantile_local(1, hist_hi [P,E,256]) -> sel_hi, rank_in_bin [P,E]
 *     with r_p = ceil(|B_p| K / E) (no summing over partitions);
 *   eqb_margin_hist_pass2_local: like eqb_margin_hist_pass2, but partition p
 *     counts inside its own bin sel_hi[p,e];
 *   eqb_select_quantile_local(2, hist_lo [P,E,256]) -> sel_lo, q_bf16 [P,E]
 *     (q_bf16[p,e] = b_hat_{p,e}, shard p's r_p-th smallest BF16 margin);
 *   eqb_rank_average: b_avg[e] = sum over non-empty p (binary64, ascending p)
 *     of b_hat_{p,e}, divided by their number (nullable output), and b_next =
 *     b_avg - mean(b_avg), centred as in Eq. 2.
 * An empty partition gets sel = -1 and a NaN q_bf16 and is left out of the
 * average.  dev_status as for eqb_select_quantile.  T and part_off describe
 * the whole batch as in every other call; K < E.
 */
eqb_status eqb_select_quantile_local(int32_t pass, const int32_t* hist, int64_t T, int32_t K, int32_t E,
                                     const int64_t* part_off, int32_t P, int32_t* sel_hi,
                                     int64_t* rank_in_bin, int32_t* sel_lo, uint16_t* q_bf16,
                                     int32_t* dev_status, void* stream);
eqb_status eqb_margin_hist_pass2_local(const uint16_t* z, const float* tau, int64_t T, int32_t E,
                                       const int32_t* sel_hi, const int64_t* part_off, int32_t P,
                                       int32_t* hist_lo, void* stream);
eqb_status eqb_rank_average(const uint16_t* q_bf16, int64_t T, int32_t E, const int64_t* part_off,
                            int32_t P, double* b_avg, float* b_next, void* stream);

/*
 * Fixed-resolution histogram QB: margin counts over nbins uniform bins of
 * [lo, hi), summed over the shards, and the quantile read off the sum.
 *   eqb_margin_hist_uniform: hist[p,e,j] += #{t in p : bin(tau_t - z_{t,e}) = j},
 *     the margin being the binary32 difference (no BF16 rounding) and
 *     bin(m) = floor((m - lo) * s) clamped to [0, nbins-1], with
 *     s = nbins / (hi - lo), all in binary32.  hist [P,E,nbins] int32 (+=).
 *   eqb_select_uniform: sums the P slabs, finds the first bin j whose running
 *     count C_j reaches r and writes est[e] = lo + (j + (r - C_{j-1}) / H_j) *
 *     (hi - lo) / nbins in binary64 (linear within the bin), and, if b_next is
 *     not NULL, b_next = est - mean(est) centred as in Eq. 2.
 * 1 <= nbins <= 256 and lo < hi (finite) or EQB_ERR_INVALID_ARG.
 */
eqb_status eqb_margin_hist_uniform(const uint16_t* z, const float* tau, int64_t T, int32_t E,
                                   const int64_t* part_off, int32_t P, float lo, float hi, int32_t nbins,
                                   int32_t* hist, void* stream);
eqb_status eqb_select_uniform(const int32_t* hist, int32_t P, int32_t E, int32_t nbins, int64_t r, float lo,
                              float hi, double* est, float* b_next, int32_t* dev_status, void* stream);

/*
 * Balance metric (Sec. 5; Appendix E, "Balance metrics"):
 *   MaxVio(B) = max_e [ f_e(B) / fbar(B) - 1 ],  fbar(B) = K|B|/E  (Sec. 2).
 *   load [P,E] int32 (in): per-partition loads f_{p,e}, e.g. from eqb_route_topk.
 *   maxvio_global [1] binary64 (out): the whole batch, f_e = sum_p f_{p,e}, |B| = T
 *     ("Global MaxVio").
 *   maxvio_local [P] binary64 (out, nullable): partition p alone,
 *     |B| = part_off[p+1] - part_off[p]; NaN for an empty partition.
 *   maxvio_local_mean [1] binary64 (out, nullable): "Local MaxVio" as Appendix E
 *     reports it, the per-partition values averaged over the non-empty
 *     partitions (binary64 sum in ascending p, divided by their number).
 * Each value is (max_e f_e) * E / (K * |B|) - 1 in binary64: an exact integer
 * maximum, then one division and one subtraction, each rounded to nearest even.
 * T = 0 returns EQB_OK and writes nothing.
 */
eqb_status eqb_max_violation(const int32_t* load, int64_t T, int32_t K, int32_t E,
                             const int64_t* part_off, int32_t P, double* maxvio_global,
                             double* maxvio_local, double* maxvio_local_mean, void* stream);

/*
 * Load-Error Injection, the residual (Sec. 4, Eq. lei and the normalisation
 * that bounds it).  For each partition p (a local batch B_l):
 *   rho_{p,e} = f_{p,e} / fbar(B_p) - 1 = f_{p,e} E / (K |B_p|) - 1,
 *   with c > 0: xi_p = max_e |rho_{p,e}| / c and rho~ = rho * tanh(xi_p)/xi_p
 *   (tanh(xi)/xi := 1 at xi = 0); with c <= 0: rho~ = rho (unnormalised LEI);
 *   inj[p,e] = eta * rho~_{p,e}, computed in binary64, rounded once to binary32.
 *   load [P,E] int32 (in); inj [P,E] binary32 (out, 16-byte aligned for
 *   eqb_lei_inject).  An empty partition gets inj = 0.  Unlike the other calls,
 *   T = 0 still writes inj (all zero).  NaN eta or c is EQB_ERR_INVALID_ARG.
 */
eqb_status eqb_lei_residual(const int32_t* load, int64_t T, int32_t K, int32_t E,
                            const int64_t* part_off, int32_t P, double eta, double c, float* inj,
                            void* stream);

/*
 * Load-Error Injection, the gradient correction (Sec. 4, Eq. lei):
 *   grad_s[t,e] += inj[p,e] for every token t of partition p, one binary32
 *   addition each (round to nearest even).  LEI leaves routing and mixture
 *   weights unchanged; only the router-score gradient moves.
 *   grad_s [T,E] binary32 (in/out, 16-byte aligned); inj [P,E] binary32 (in,
 *   16-byte aligned), e.g. from eqb_lei_residual.
 */
eqb_status eqb_lei_inject(float* grad_s, const float* inj, int64_t T, int32_t E,
                          const int64_t* part_off, int32_t P, void* stream);

/*
 * Router backward with Load-Error Injection, fused (Sec. 2 Eq. 1; Sec. 4 Eq. lei):
 *   grad_z[t,e] = (g[t,e] + inj[p,e]) * sigmoid'(z[t,e])    for t in partition p,
 *   where g[t,e] = grad_score[t,k] if e = topk_idx[t,k] (the gradient of the
 *   loss w.r.t. the mixture weight s_{t,e} of a selected expert) and 0 for the
 *   other experts; inj [P,E] from eqb_lei_residual, or NULL for the plain
 *   router backward.  sigmoid'(z) = q - q^2, q = e/(1+e), e = exp(-|z|), in
 *   binary32 (a few ulp, whatever the size of z); the sum and product are single
 *   binary32 operations.
 *   z [T,E] bf16 bits (16-byte aligned), topk_idx [T,K] int32, grad_score
 *   [T,K] binary32 (in); grad_z [T,E] binary32 (out, 16-byte aligned).
 *   Index entries outside [0, E) are ignored.
 */
eqb_status eqb_lei_router_backward(const uint16_t* z, const int32_t* topk_idx, const float* grad_score,
                                   const float* inj, int64_t T, int32_t E, int32_t K, const int64_t* part_off,
                                   int32_t P, float* grad_z, void* stream);

/*
 * One whole layer in one call (Sec. 2, Eq. 1 and "Quantile Balancing";
 * Appendix C, Algorithm 1 steps 1-6; Eq. 2): routing with the fused coarse
 * counts, the coarse selection, the fine counts and the fine selection with
 * the centred bias, enqueued as four kernels on `stream`.  It computes what
 * eqb_route_topk, eqb_select_quantile(1), eqb_margin_hist_pass2 and
 * eqb_select_quantile(2) compute in sequence, with r = eqb_rank(T, K, E).
 *   z [T,E] bf16 bits, b [E] binary32                       (in)
 *   topk_idx [T,K] int32, topk_score [T,K] binary32, tau [T] (out)
 *   load [P,E] int32                                         (out, WRITTEN: f_{p,e})
 *   q_bf16 [E] (out: b_hat_e, BF16 bits), b_next [E] binary32 (out: Eq. 2)
 *   hist_hi_sum, hist_lo_sum [E,256] int32 (nullable out): the summed coarse
 *     counts H[e,u] and the summed fine counts L[e,v] inside u_e.
 *   dev_status [1] int32 (out, WRITTEN): EQB_DEV_OK, or
 *     EQB_DEV_RANK_EXCEEDS_COUNT when some expert's selection failed.
 *   workspace: device memory of at least eqb_layer_workspace_size(E, P)
 *     bytes, 256-byte aligned, owned by the caller.  Its first
 *     eqb_layer_workspace_zero_bytes(E, P) bytes hold the per-partition
 *     counts and the selections while the layer runs: they must be ALL ZERO
 *     when the call's work starts, and the call's work leaves them all zero
 *     again (each selection clears the counts it has summed).  The rest is
 *     scratch for the per-block count images of the routing and then of the
 *     fine pass, which every call overwrites before reading; its contents do not
 *     matter.  So a caller
 *     zeroes the workspace once after allocating it and may then run layer
 *     after layer with it.  After an error reported by the call or by the
 *     runtime while its work ran, zero it again before the next use.  Two
 *     calls whose work may overlap need two workspaces.
 *   marks (nullable): host array of 5 hipEvent_t handles, each nullable,
 *     recorded on `stream` before the route kernel, after it, after the
 *     coarse selection, after the fine pass and after the last kernel (for
 *     timing the stages of one layer without splitting the call).
 * Returns EQB_ERR_RANK when T = 0 (no quantile), EQB_ERR_INVALID_ARG for a
 * null pointer or a workspace that is too small, EQB_ERR_UNSUPPORTED for a
 * misaligned z or workspace; other errors as for the calls it chains.
 */
size_t eqb_layer_workspace_size(int32_t E, int32_t P);        /* host only; 0 for unsupported E or P */
size_t eqb_layer_workspace_zero_bytes(int32_t E, int32_t P);  /* host only; 0 for unsupported E or P */
eqb_status eqb_layer(const uint16_t* z, const float* b, int64_t T, int32_t E, int32_t K,
                     const int64_t* part_off, int32_t P, int32_t* topk_idx, float* topk_score, float* tau,
                     int32_t* load, uint16_t* q_bf16, float* b_next, int32_t* hist_hi_sum,
                     int32_t* hist_lo_sum, int32_t* dev_status, void* workspace, size_t workspace_bytes,
                     void* const* marks, void* stream);

/*
 * eqb_layer for callers that cannot allocate device memory (code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc): the
 * same layer, the same outputs and argument checks, but the working buffers
 * live in a library-owned device array of EQB_NOALLOC_SCRATCH_BYTES per GPU
 * (held until the process ends) instead of a caller workspace.  The call
 * allocates nothing; the caller still passes every input and output.
 *   The array holds the layer's counters only (routing and fine pass add all
 *   their counts to the partition slabs instead of storing per-block images).
 *   Limit: eqb_layer_workspace_zero_bytes(E, P) <= EQB_NOALLOC_SCRATCH_BYTES,
 *   i.e. P * E <= 4096 (E = 256: up to 16 partitions); larger layers return
 *   EQB_ERR_SCRATCH before anything is enqueued.
 *   Every call on one GPU shares that GPU's array: the call clears the part
 *   it uses (a fill kernel) before the layer runs, and calls whose work may
 *   overlap on one GPU (other streams, other threads) race on it and give
 *   wrong results.  Order them on one stream.
 */
#define EQB_NOALLOC_SCRATCH_BYTES ((size_t)(8u << 20) + (192u << 10))
eqb_status eqb_layer_noalloc(const uint16_t* z, const float* b, int64_t T, int32_t E, int32_t K,
                             const int64_t* part_off, int32_t P, int32_t* topk_idx, float* topk_score,
                             float* tau, int32_t* load, uint16_t* q_bf16, float* b_next,
                             int32_t* hist_hi_sum, int32_t* hist_lo_sum, int32_t* dev_status, void* stream);

/*
 * ------------------------------------------------------------------------
 * Training operators around the layer: the balance loss with its gradient,
 * the experts' rows, and the optimizer step.  The conventions above hold for
 * them too, except that every output is WRITTEN, not accumulated.
 * ------------------------------------------------------------------------
 */

/* Element types of rows, gradients and the like. */
#define EQB_DTYPE_F32        0
#define EQB_DTYPE_BF16       1
#define EQB_DTYPE_F16        2

/* What the balance loss takes as a token's probabilities p_{t,e}. */
#define EQB_SCORE_SIGMOID    0   /* sigmoid(z_{t,e}) / sum_e sigmoid(z_{t,e}) */
#define EQB_SCORE_SOFTMAX    1   /* exp(z_{t,e}) / sum_e exp(z_{t,e}) */

/*
 * The auxiliary balance loss (Sec. 2, "GShard"; App. D) of each balance group,
 * with the counts of every expert.  A group is a partition of the token batch:
 * a rank's local batch, or one sequence.  For group p with n_p valid tokens:
 *   f_{p,e}    = #{(t, k) : topk_idx[t,k] = e, t valid in p}
 *   prob_{p,e} = (1/n_p) sum over valid t of p_{t,e}
 *   loss_p     = alpha * sum_e F_{p,e} prob_{p,e},   F_{p,e} = E f_{p,e} / (K n_p)
 * so that an even load gives alpha.  A group without valid tokens has prob = 0
 * and loss = 0.
 *   z [T,E] bf16 bits (16-byte aligned).  Logits of -inf (masked experts) have
 *     probability 0; a row of nothing but -inf has p = 0 throughout.
 *   topk_idx [T,K] int32 (nullable): entries outside [0, E) are not counted.
 *     With NULL, `load` is an INPUT: counts that the routing gave (over the
 *     valid tokens).
 *   valid [T] uint8 (nullable: every token is valid): a token of 0 takes no part,
 *     whatever its logits hold (NaN included).
 *   load [P,E] int32 (out, or in without topk_idx); tokens [P] int32 (out: n_p);
 *   prob [P,E] binary32 (out); loss [P] binary32 (out).
 *   workspace: eqb_balance_workspace_size(E, P) bytes, 256-byte aligned, owned
 *     by the caller, zeroed once after allocation; each call leaves its leading
 *     counters zero again, wherever E and P put the rest, so that one workspace of
 *     the largest size serves calls of all sizes.  Two calls whose work may overlap
 *     need two.
 * A row's probabilities and a lane's sum over up to 128 of its rows are binary32, the
 * sums of those binary64 (handed from block to block in binary32); the result does not
 * depend on the order in which blocks run.  T = 0 writes zeros (`load` too, with or without topk_idx).
 */
size_t eqb_balance_workspace_size(int32_t E, int32_t P);     /* host only; 0 for unsupported E or P */
eqb_status eqb_balance_loss(const uint16_t* z, const int32_t* topk_idx, const uint8_t* valid, int64_t T,
                            int32_t E, int32_t K, const int64_t* part_off, int32_t P, int32_t score, double alpha,
                            int32_t* load, int32_t* tokens, float* prob, float* loss, void* workspace,
                            size_t workspace_bytes, void* stream);

/*
 * The gradient of the balance loss with respect to the logits, alone or in one
 * pass with the router backward and the load-error injection.  The loads are not
 * differentiated (the straight-through estimate of App. D):
 *   grad_z[t,e] = (alpha grad_loss_p / n_p) p_{t,e} q_{t,e} (F_{p,e} - sum_e' p_{t,e'} F_{p,e'})
 *                 + (g[t,e] + inj[p,e]) sigmoid'(z_{t,e})
 * with q = 1 - sigmoid(z) (EQB_SCORE_SIGMOID) or 1 (EQB_SCORE_SOFTMAX) and g, inj as
 * in eqb_lei_router_backward, sigmoid' too; a row of an invalid token is 0 throughout.
 *   load [P,E], tokens [P] int32 (in): from eqb_balance_loss.
 *   grad_loss [P] binary32 (in): the gradient that arrives at each loss_p.
 *   topk_idx [T,K], grad_score [T,K] (both or neither): g; inj [P,E] (nullable).
 *   grad_z [T,E] binary32 (out, 16-byte aligned).
 */
eqb_status eqb_balance_backward(const uint16_t* z, const int32_t* load, const int32_t* tokens,
                                const float* grad_loss, const int32_t* topk_idx, const float* grad_score,
                                const float* inj, const uint8_t* valid, int64_t T, int32_t E, int32_t K,
                                const int64_t* part_off, int32_t P, int32_t score, double alpha, float* grad_z,
                                void* stream);

/*
 * The order of the experts' rows (what Eq. 1's FFN_e work on): the routed pairs
 * (t, k) sorted by expert and within an expert by t*K + k.
 *   topk_idx [T,K] int32 (in): entries outside [0, E) are dropped pairs.
 *   offsets [E+1] int32 (out): expert e's rows are [offsets[e], offsets[e+1]).
 *   slot [T,K] int32 (out): the row of pair (t, k), -1 for a dropped pair.
 *   workspace: eqb_dispatch_workspace_size(T, K, E) bytes of scratch, 16-byte
 *     aligned (nullable where that is 0); what it holds does not matter.
 * T*K < 2^31.  T = 0 writes offsets of zeros.
 */
size_t eqb_dispatch_workspace_size(int64_t T, int32_t K, int32_t E);   /* host only */
eqb_status eqb_dispatch_plan(const int32_t* topk_idx, int64_t T, int32_t K, int32_t E, int32_t* offsets,
                             int32_t* slot, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Rows of `hidden` elements of type dtype (EQB_DTYPE_*), between the tokens' order
 * and the experts'.  `rows` tells how many rows the expert-ordered buffers hold;
 * a pair whose slot lies outside [0, rows) is dropped.  Buffers need the alignment
 * of their elements only, and those of one call must not overlap.  T*K < 2^31.
 *   eqb_dispatch: expert_rows[slot[t,k]] = x[t].  Rows that no slot names are left
 *     as they are.
 *   eqb_combine (Eq. 1): y[t] = sum over k of weight[t,k] expert_rows[slot[t,k]], in
 *     ascending k in binary32, rounded once.  weight = NULL stands for 1: then it is
 *     the gradient of eqb_dispatch.  Dropped pairs add nothing.
 *   eqb_combine_backward: grad_rows[slot[t,k]] = weight[t,k] grad_y[t] (rows that no
 *     slot names are left as they are) and grad_weight[t,k] = <grad_y[t],
 *     expert_rows[slot[t,k]]> (0 for a dropped pair), summed in binary32: the
 *     grad_score of eqb_lei_router_backward and eqb_balance_backward.
 */
eqb_status eqb_dispatch(const void* x, const int32_t* slot, int64_t T, int32_t K, int64_t rows, int32_t hidden,
                        int32_t dtype, void* expert_rows, void* stream);
eqb_status eqb_combine(const void* expert_rows, const int32_t* slot, const float* weight, int64_t T, int32_t K,
                       int64_t rows, int32_t hidden, int32_t dtype, void* y, void* stream);
eqb_status eqb_combine_backward(const void* grad_y, const void* expert_rows, const int32_t* slot,
                                const float* weight, int64_t T, int32_t K, int64_t rows, int32_t hidden,
                                int32_t dtype, void* grad_rows, float* grad_weight, void* stream);

/*
 * One AdamW step over n tensors (decoupled weight decay), in place:
 *   g = grad * grad_scale
 *   m = beta1 m + (1 - beta1) g
 *   v = beta2 v + ((1 - beta2) g) g
 *   param = param (1 - lr weight_decay)
 *           - (m / (sqrt(v) / sqrt(1 - beta2^step) + eps)) * (lr / (1 - beta1^step))
 * Every operation is one binary32 operation in the order written (a division by a
 * constant is a product with its reciprocal; constants are computed in binary64 and
 * rounded once), so the results are reproducible bit for bit.
 *
 * state_bits = 32: exp_avg = m and exp_avg_sq = v, binary32.
 * state_bits = 8: 8-bit codes (E4M3: sign, 4 exponent and 3 mantissa bits, largest
 *   448, no infinities) of m / s and sqrt(v) / s, where a scale s = max / 448 belongs to
 *   each block of EQB_ADAMW_BLOCK elements counted from the tensor's start.  (The square
 *   root of v needs half of v's range of exponents.)  A code is rounded up or down at
 *   random, up with the chance that makes it right on average, by 16 bits of a hash of
 *   seed, step, the tensor's place in the call and the element: v moves by a few
 *   thousandths per step, far less than half a code, so that rounding to nearest would
 *   freeze the proportions inside a block.  A sqrt(v) above 0 never becomes 0, or the
 *   divisor would fall to eps.  Blocks whose largest value is below 2^-100 are stored
 *   as 0.  A gradient that is no finite number spoils its block.
 *
 * tensors: HOST array of n descriptors, read during the call.
 *   param: binary32 weights; copy (nullable, in all tensors or in none): bf16 bits,
 *   receives the new weights rounded to nearest even; grad: grad_dtype (F32 or BF16);
 *   exp_avg, exp_avg_sq: numel elements of 4 bytes or of 1; exp_avg_scale,
 *   exp_avg_sq_scale: ceil(numel / EQB_ADAMW_BLOCK) binary32 scales (8 bits only).
 *   Pointers need the alignment of their elements; buffers must not overlap.
 *   numel = 0 is allowed (and its pointers may be null).
 * step >= 1: the number of this step.  grad_scale (nullable, device binary32):
 * a factor on every gradient (clipping, unscaling).  found_inf (nullable, device
 * binary32): where it is not 0 the call changes nothing.  The number of the next
 * step then stays the same, which the host does not know without waiting:
 * eqb_adamw_step_counted keeps it on the device, also for steps that are captured
 * in a graph and replayed.  counter: EQB_ADAMW_COUNTER_BYTES of device memory,
 * 8-byte aligned; its first 8 bytes are the steps taken so far (int64: zeroed once,
 * or set to go on from a saved state), the rest is scratch.  A call that is not
 * skipped adds one and is the step of that number; a skipped one changes nothing
 * there either.  Its constants are computed on the device, in binary64 as well.
 */
#define EQB_ADAMW_BLOCK      256
#define EQB_ADAMW_COUNTER_BYTES 64
typedef struct eqb_adamw_tensor {
  float* param;
  const void* grad;
  uint16_t* copy;
  void* exp_avg;
  void* exp_avg_sq;
  float* exp_avg_scale;
  float* exp_avg_sq_scale;
  int64_t numel;
  double weight_decay;
} eqb_adamw_tensor;
eqb_status eqb_adamw_step(const eqb_adamw_tensor* tensors, int32_t n, int32_t grad_dtype, int32_t state_bits,
                          int64_t step, double lr, double beta1, double beta2, double eps, uint64_t seed,
                          const float* grad_scale, const float* found_inf, void* stream);
eqb_status eqb_adamw_step_counted(const eqb_adamw_tensor* tensors, int32_t n, int32_t grad_dtype, int32_t state_bits,
                                  void* counter, double lr, double beta1, double beta2, double eps, uint64_t seed,
                                  const float* grad_scale, const float* found_inf, void* stream);

/*
 * ------------------------------------------------------------------------
 * Routing by scores, and the experts' products in 8 bits.  The conventions
 * above hold, every output is WRITTEN, and the buffers of one call must not
 * overlap.  Pointers need the alignment of their elements where nothing else
 * is said.
 * ------------------------------------------------------------------------
 */

/*
 * The experts of every token by their scores, and their weights.
 *   s_e = sigmoid(z_e) (EQB_SCORE_SIGMOID) or exp(z_e) / sum_e' exp(z_e') (EQB_SCORE_SOFTMAX)
 *   q_e = s_e + bias_e: what decides; an expert whose z_e or q_e is -inf or NaN is masked out of the
 *     row.  z_e = +inf counts as the largest finite number.
 *   groups > 1: the E experts are `groups` groups of E / groups neighbours.  A group's score is the
 *     sum of its group_top (1 or 2) largest q that are not masked (of the one it has, or -inf without
 *     any); only the experts of the top_groups groups of the largest scores take part.
 *   The K largest q are chosen, in that order.  Where masks leave fewer, the last entries are
 *     expert -1 of weight 0: dropped pairs to eqb_dispatch_plan.
 *   weight_k = scale s_k / (sum of the chosen s) (normalize; also where binary32 holds none of those s) or
 *     scale s_k, in binary32.  Scores below 2^-126, normalized weights below 2^-100 scale, may count as 0 there.
 * Ties go to the lower expert and to the lower group.  Which of two scores is larger is decided as
 * in binary64 (without a bias: by the logits), so that the choice does not depend on a rounding of
 * binary32.
 *   z [T,E] of type dtype (EQB_DTYPE_*), 16-byte aligned; bias [E] binary32 (nullable: 0).
 *   topk_idx [T,K] int32 (out); topk_weight [T,K] binary32 (out).
 * groups: a power of two up to E; 1 <= top_groups <= groups; group_top <= E / groups;
 * K <= top_groups E / groups; K < E.  T*K < 2^31.
 */
eqb_status eqb_route_scored(const void* z, const float* bias, int64_t T, int32_t E, int32_t K, int32_t groups,
                            int32_t top_groups, int32_t group_top, int32_t score, int32_t normalize, double scale,
                            int32_t dtype, int32_t* topk_idx, float* topk_weight, void* stream);

/*
 * The gradient of topk_weight with respect to the logits, the choice held fixed (the bias has none).
 * With S = sum of the chosen s and a_k = scale (g_k - sum_j g_j s_j / S) / S (normalize) or scale g_k:
 *   grad_z_e = (sum of a_k over the k that chose e) s_e (1 - s_e)                  (sigmoid)
 *   grad_z_e = s_e ((sum of a_k over the k that chose e) - sum_k a_k s_k)          (softmax)
 *   grad_weight [T,K] binary32 (in): the combine's grad_weight.  Entries whose topk_idx lies outside
 *     [0, E) take no part.
 *   grad_z [T,E] binary32 (out, 16-byte aligned).
 */
eqb_status eqb_route_scored_backward(const void* z, const int32_t* topk_idx, const float* grad_weight, int64_t T,
                                     int32_t E, int32_t K, int32_t score, int32_t normalize, double scale,
                                     int32_t dtype, float* grad_z, void* stream);

/*
 * Numbers in 8 bits: E4M3 codes (sign, 4 exponent and 3 mantissa bits, largest 448, no infinities)
 * with a power of two for each block of EQB_CODE_BLOCK.  A block's scale is 2^x with the least
 * x >= -126 for which no finite value exceeds 448 2^x; a code is value 2^-x rounded to nearest, ties
 * to even; infinities and NaN become NaN.  A scale is kept as the byte x + 127.
 *   A row of H elements is eqb_code_width(H) codes (H rounded up to whole blocks, zeros behind H) and
 *   eqb_scale_width(H) scale bytes (one per block, rounded up to a multiple of 4, zeros behind).
 * Codes and scales are 16-byte aligned.  1 <= H <= 2^24.
 *
 *   eqb_quantize_rows: codes [rows, eqb_code_width(hidden)], scales [rows, eqb_scale_width(hidden)] of
 *     x [rows, hidden].  count (nullable, device int32): only the first *count rows are read and
 *     written (the offsets[E] of a plan).
 *   eqb_dispatch_quantized: eqb_dispatch and eqb_quantize_rows in one: x [T, hidden] to the rows that
 *     slot names; rows that no slot names are left as they are.
 *   eqb_quantize_columns: the same values along the other axis, for eqb_experts_grad_weight: codes
 *     [hidden, W] with W = eqb_column_width(rows, E), scales [hidden, eqb_scale_width(W)].  Row
 *     offsets[e] + i of expert e is column 128 (offsets[e] / 128 + e) + i; zeros fill an expert's last
 *     block.  Columns of no expert's block are left as they are.
 *   eqb_quantize_weights: w [E,N,hidden] with one scale for each 128 x 128: codes
 *     [E,N,eqb_code_width(hidden)], scales [E, ceil(N/128), eqb_scale_width(hidden)], and the transposed
 *     codes_t [E,hidden,eqb_code_width(N)], scales_t [E, ceil(hidden/128), eqb_scale_width(N)], the same
 *     values for the gradient of the rows.  Either pair may be null.
 * Offsets are taken as if they lay in [0, rows].  1 <= E <= 256 here, not only powers of two.
 */
#define EQB_CODE_BLOCK       128
int64_t eqb_code_width(int64_t hidden);                      /* host only */
int64_t eqb_scale_width(int64_t hidden);                     /* host only */
int64_t eqb_column_width(int64_t rows, int32_t E);           /* host only */
eqb_status eqb_quantize_rows(const void* x, const int32_t* count, int64_t rows, int32_t hidden, int32_t dtype,
                             uint8_t* codes, uint8_t* scales, void* stream);
eqb_status eqb_dispatch_quantized(const void* x, const int32_t* slot, int64_t T, int32_t K, int64_t rows,
                                  int32_t hidden, int32_t dtype, uint8_t* codes, uint8_t* scales, void* stream);
eqb_status eqb_quantize_columns(const void* x, const int32_t* offsets, int64_t rows, int32_t E, int32_t hidden,
                                int32_t dtype, uint8_t* codes, uint8_t* scales, void* stream);
eqb_status eqb_quantize_weights(const void* w, int32_t E, int32_t N, int32_t hidden, int32_t dtype, uint8_t* codes,
                                uint8_t* scales, uint8_t* codes_t, uint8_t* scales_t, void* stream);

/*
 * The experts' products (what FFN_e of Eq. 1 is made of), in the codes above, summed in binary32 and
 * rounded once to dtype.
 *   eqb_experts_product: out[r,n] = sum_k x[r,k] w[e,n,k] for the rows r of expert e (offsets [E+1],
 *     device, as eqb_dispatch_plan writes them): codes and scales of x [rows, hidden] and of w
 *     [E,N,hidden].  Rows outside the experts' ranges are left as they are.  With the transposed weights
 *     it is the gradient of the rows: grad_x[r,k] = sum_n grad_out[r,n] w[e,n,k].
 *   eqb_experts_grad_weight: out[e,n,k] = sum over the rows r of expert e of grad[r,n] x[r,k], from the
 *     columns' codes of grad [rows, N] and of x [rows, hidden]; zeros for an expert without rows.  Columns
 *     of up to 2^24.
 * Results of 16 bits come from 8-bit matrix instructions, whose sum over a block of 128 cuts off what
 * lies 16 bits below the block's largest product: at most 2^-9 of that product a block, which may be
 * more than a sum whose terms cancel; results in binary32 from BF16 ones, which sum in full (and take
 * a code times its scale below 2^-133 as 0, from 2^128 on as infinite).
 */
eqb_status eqb_experts_product(const uint8_t* codes, const uint8_t* scales, const uint8_t* w_codes,
                               const uint8_t* w_scales, const int32_t* offsets, int64_t rows, int32_t E, int32_t N,
                               int32_t hidden, int32_t dtype, void* out, void* stream);
eqb_status eqb_experts_grad_weight(const uint8_t* grad_codes, const uint8_t* grad_scales, const uint8_t* codes,
                                   const uint8_t* scales, const int32_t* offsets, int64_t rows, int32_t E, int32_t N,
                                   int32_t hidden, int32_t dtype, void* out, void* stream);

/*
 * The gated activation between an expert's two products: x [rows, 2 hidden] holds a row's gate g and
 * then its u, h = g sigmoid(g) u.  Computed in binary32, rounded once.
 *   eqb_gated: h [rows, hidden] of x's type.  eqb_gated_quantize: h as eqb_quantize_rows leaves it,
 *   without a rounding in between.  eqb_gated_quantize_columns: h of x's type as eqb_quantize_columns
 *   leaves it, for the gradient of the second product's weights; what the type does not hold (above
 *   65504 in F16) is taken in binary32, as the second product had it.
 *   eqb_gated_backward: grad_x [rows, 2 hidden] from grad_h [rows, hidden]:
 *     grad_g = grad_h u s (1 + g (1 - s)), grad_u = grad_h g s, s = sigmoid(g).
 * count as in eqb_quantize_rows.
 */
eqb_status eqb_gated(const void* x, const int32_t* count, int64_t rows, int32_t hidden, int32_t dtype, void* h,
                     void* stream);
eqb_status eqb_gated_quantize(const void* x, const int32_t* count, int64_t rows, int32_t hidden, int32_t dtype,
                              uint8_t* codes, uint8_t* scales, void* stream);
eqb_status eqb_gated_quantize_columns(const void* x, const int32_t* offsets, int64_t rows, int32_t E, int32_t hidden,
                                      int32_t dtype, uint8_t* codes, uint8_t* scales, void* stream);
eqb_status eqb_gated_backward(const void* grad_h, const void* x, const int32_t* count, int64_t rows, int32_t hidden,
                              int32_t dtype, void* grad_x, void* stream);

/*
 * Test control (host only, no HIP call): caps the number of blocks of the
 * streaming kernels (routing, the margin passes, the LEI kernels, the balance
 * loss and its gradient, the experts' rows, their codes by rows, gates and
 * products) at max_blocks for the calls that
 * follow FROM THE CALLING HOST THREAD; calls made from other threads keep their
 * own setting (the default 0: a whole number of blocks per compute unit).
 * Results do not depend on it, but for the last bits of the balance loss's
 * binary32 sums; tests use it to run one block, or a block count that does not
 * divide the rows, against the same oracle.  Negative values are
 * EQB_ERR_INVALID_ARG.
 * eqb_get_max_blocks returns the calling thread's current cap.
 */
eqb_status eqb_set_max_blocks(int32_t max_blocks);
int32_t eqb_get_max_blocks(void);

/* Host helper: r = ceil(T*K/E) (Sec. 3; the paper assumes T*K/E is an
 * integer), or -1 for invalid arguments.  Host only, no HIP call. */
int64_t eqb_rank(int64_t T_total, int32_t K, int32_t E);

/* Host helper: a static string naming a status code. */
const char* eqb_status_string(eqb_status status);

#ifdef __cplusplus
}
#endif

#endif /* EQB_H */
