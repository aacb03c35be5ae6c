/*
 * sgemm_cube.h -- C ABI of the SGEMM-cube library for NVIDIA B200 (sm_100a).
 *
 * SGEMM-cube approximates an FP32 GEMM C = A * B (FP32 in, FP32 out) with FP16 tensor-core
 * products.  Every FP32 operand x is split into an FP16 high word and a scaled FP16 residual,
 *
 *      hi = fl16(x),     lo = fl16((x - hi) * 2^s)            (round-to-nearest-even)
 *
 * and C is rebuilt from three FP16 x FP16 -> FP32 products, dropping lo*lo:
 *
 *      C  ~=  hi_A hi_B  +  2^-s ( lo_A hi_B  +  hi_A lo_B )
 *
 * (paper: Sec. 3.3, the two-component representation, Eq. fp16_high_low; Sec. 4.2, residual
 *  scaling, Eq. sf_bounds; Sec. 4.3, Eq. recover_eqn; Sec. 4.5, the two accumulation orders,
 *  Eq. elementwise / Eq. termwise).
 *
 * Conventions shared by every entry point
 *   - All matrices are ROW-MAJOR with a leading dimension counted in elements.
 *   - Pointers named *_dev are DEVICE pointers on the handle's device; pointers named *_host are
 *     host pointers.  The caller owns every buffer it passes; the handle owns only its internal
 *     workspace.  No entry point takes ownership of or frees a caller's buffer.
 *   - `stream` is a cudaStream_t passed as void* (NULL = the default stream).  Device entry
 *     points enqueue work on it and return without synchronising.
 *   - Every function returns a status code (0 = success) and never throws or exits.  Argument
 *     errors are detected before anything is enqueued.  A failure inside a kernel (a bounded
 *     wait that ran out) is recorded in a device error word and reported by sgemm_cube_check().
 *   - FP16 matrices are passed as uint16_t bit patterns (IEEE binary16).
 *   - There is no CPU fallback: on a device that is not sm_100 sgemm_cube_create fails.
 */
#ifndef SGEMM_CUBE_H_
#define SGEMM_CUBE_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef struct sgemm_cube_ctx* sgemm_cube_handle;

/* status codes */
enum {
  SGEMM_CUBE_OK = 0,
  SGEMM_CUBE_INVALID_ARG = 1,      /* null pointer, negative size, ld too small, bad enum        */
  SGEMM_CUBE_MISALIGNED = 2,       /* pointer / leading dimension violates an alignment rule    */
  SGEMM_CUBE_CUDA_ERROR = 3,       /* a CUDA runtime or driver call failed                      */
  SGEMM_CUBE_DEVICE_TIMEOUT = 4,   /* a kernel gave up on a bounded wait (see sgemm_cube_check) */
  SGEMM_CUBE_UNSUPPORTED_ARCH = 5, /* device is not compute capability 10.x                     */
  SGEMM_CUBE_ALLOC_FAILED = 6,     /* workspace allocation failed                               */
  SGEMM_CUBE_TOO_LARGE = 7         /* problem exceeds the fixed scratch of the _static variant  */
};

/* accumulation order (paper Sec. 4.5) */
enum {
  SGEMM_CUBE_TERMWISE = 0,   /* Eq. termwise: streams summed separately, combined once at the end */
  SGEMM_CUBE_ELEMENTWISE = 1, /* Eq. elementwise: per k-block, products folded into one accumulator */
  /* The reordered elementwise order that Sec. 4.5 (last paragraph) proposes and leaves unmeasured:
   * per k-block the corrections are summed first, scaled, added to the block's hi*hi product, and
   * the block enters the accumulator once: acc = acc + ((R_A B + A R_B) / s_f + A B).  Uses the
   * elementwise k-block option.  Accepted wherever an accumulation order is.  For scale_exp <= 15
   * the block's value is formed inside the tensor core's accumulator (the instruction that adds
   * the first hi*hi product scales the accumulated corrections by 2^-s), which makes this the
   * fastest of the per-block orders: 450 against 340 TFLOP/s for the plain elementwise order at
   * 8192^3 (termwise 470). */
  SGEMM_CUBE_ELEMENTWISE_REORDERED = 2
};

/* options for sgemm_cube_set_option */
enum {
  /* Length, in k, of a chain accumulated inside the tensor core before it is added, in FP32 with
   * round-to-nearest, to the running sum held in registers (termwise: the hi*hi stream; the
   * correction stream is carried whole).  Multiple of 64, default 128.  This is the k-block g
   * of Sec. 4.5 as realised on this hardware.  The tensor core truncates (rounds toward zero)
   * each time it adds a 16-deep group of products to its accumulator; on data of one sign that
   * bias adds up along a chain, about 0.5 ulp per 16 k (measured Frobenius error on U[0,1)
   * inputs: 1.9e-7 / 4.7e-7 / 1.1e-6 for k-blocks 64 / 128 / 256, FP32 GEMM 4.3e-7; on
   * symmetric data 1.5e-7 / 2.1e-7 / 3.5e-7).  Shorter blocks cost throughput: about 2 % from
   * 256 to 128 and a further 5 % to 64 at 8192^3. */
  SGEMM_CUBE_OPT_TERMWISE_K_BLOCK = 0,
  /* Same for the elementwise order: the k-block of Eq. elementwise.  Multiple of 64, default 64. */
  SGEMM_CUBE_OPT_ELEMENTWISE_K_BLOCK = 1,
  /* 1: run the tensor-core kernels as clusters of two CTAs that share one
   * tcgen05.mma.cta_group::2 (256 x 256 tile per pair, each CTA loading half of the B tile);
   * 0: one CTA per 128 x 256 tile; 2 (default): the library chooses: pairs for the kernels that
   * read FP16 words (two-phase sgemm_cube, sgemm_cube_presplit, sgemm_cube_hgemm, ...) whenever
   * M > 128 and split-K (below, single CTAs only) does not apply, and for the fused converter
   * kernel whenever M > 128.  Same arithmetic, bit-identical results either way as long as
   * split-K does not apply.  (Pairs pull two thirds of the bytes of single CTAs from L2 into the SMs, which is
   * what bounds this kernel: 458 against 439 TFLOP/s at 8192^3, 407 against 378 at 4096^3.) */
  SGEMM_CUBE_OPT_CTA_PAIR = 2,
  /* How sgemm_cube computes (same arithmetic; same bracketing and bit-identical results except
   * where split-K, which only the two-phase strategy uses, re-brackets the k-block sums):
   * SGEMM_CUBE_STRATEGY_FUSED     one kernel; TMA stages FP32 tiles in shared memory, converter
   *                               warps split them there in place, no FP16 copy of A or B exists
   *                               in device memory, no workspace;
   * SGEMM_CUBE_STRATEGY_TWO_PHASE the split kernel writes the FP16 words of A and B once into the
   *                               handle's workspace (4 bytes per element of A and B, grown with
   *                               cudaMalloc on first use), then one kernel forms all three
   *                               products and the reconstruction;
   * SGEMM_CUBE_STRATEGY_AUTO      (default) TWO_PHASE when M*N*K >= 2^27 and the workspace can be
   *                               had, FUSED otherwise (measured crossover: 512^3). */
  SGEMM_CUBE_OPT_STRATEGY = 3,
  /* 1: sgemm_cube records CUDA events around its tensor-core kernel, for
   * sgemm_cube_last_kernel_ms and sgemm_cube_mean_kernel_ms.  Default 0. */
  SGEMM_CUBE_OPT_TIME_KERNEL = 4,
  /* 1 (default): when a problem has so few 128 x 256 tiles that more than half of the SMs would
   * idle and k is long enough, the three-product kernel (two-phase sgemm_cube,
   * sgemm_cube_presplit) cuts the k range into up to 16 slices of whole k-blocks, one work unit per
   * (tile, slice); the slices' sums go to a workspace (grown with cudaMalloc on first use) and a
   * reduction kernel adds them in slice order (termwise: hi*hi sums and correction sums
   * separately, combined once).  This is one more level of the blocked summation of Sec. 4.5 and
   * is deterministic.  0: never split.  (Orthogonalised updates split the k range of their products under the same option.) */
  SGEMM_CUBE_OPT_SPLIT_K = 5
};

enum {
  SGEMM_CUBE_STRATEGY_AUTO = 0,
  SGEMM_CUBE_STRATEGY_FUSED = 1,
  SGEMM_CUBE_STRATEGY_TWO_PHASE = 2
};

/* Create a handle bound to CUDA device `device`.  Allocates a small device error word; the
 * workspace of the unfused path and of the host-buffer path grows on demand.
 * Errors: INVALID_ARG (out == NULL), CUDA_ERROR, UNSUPPORTED_ARCH, ALLOC_FAILED. */
int sgemm_cube_create(sgemm_cube_handle* out, int device);

/* Synchronise the device, free the handle's workspace and the handle.  Returns DEVICE_TIMEOUT
 * if a kernel recorded a failure that was never collected by sgemm_cube_check. */
int sgemm_cube_destroy(sgemm_cube_handle h);

/* Set an option (see SGEMM_CUBE_OPT_*).  Errors: INVALID_ARG. */
int sgemm_cube_set_option(sgemm_cube_handle h, int option, int64_t value);

/* Operand split (paper Eq. recover_eqn, first two lines; Sec. 3.3; Sec. 4.2).
 *   hi[i,j] = fl16(X[i,j]);  lo[i,j] = fl16((X[i,j] - hi[i,j]) * 2^scale_exp)
 * RN-even conversions; the subtraction and the scaling are exact FP32 operations; FP16
 * subnormals are produced (gradual underflow is kept, nothing is flushed or clamped);
 * out-of-range inputs follow IEEE (|x| >= 65520 -> hi = inf, lo = NaN or inf).
 *   X_dev      rows x cols FP32, row-major, leading dimension ldx >= cols          (device, read)
 *   hi_dev/lo_dev  rows x cols FP16 bit patterns, leading dimension ldh >= cols    (device, written)
 *   scale_exp  s in [0, 24];  rows, cols >= 0 (nothing is done, and the pointers are not looked
 *   at, when either is 0)
 * Any alignment is accepted; 16-byte aligned pointers with ldx % 4 == 0 and ldh % 8 == 0 take
 * the vectorised path.  Errors: INVALID_ARG, CUDA_ERROR. */
int sgemm_cube_split(sgemm_cube_handle h, int rows, int cols,
                     const float* X_dev, int64_t ldx,
                     uint16_t* hi_dev, uint16_t* lo_dev, int64_t ldh,
                     int scale_exp, void* stream);

/* SGEMM-cube (paper Eq. recover_eqn with Eq. termwise or Eq. elementwise):
 *   C = hi_A hi_B + 2^-s (lo_A hi_B + hi_A lo_B),
 * hi = fl16(x), lo = fl16((x - hi) 2^s) as in sgemm_cube_split, FP16 x FP16 products on the tensor
 * cores with FP32 accumulation, the reconstruction in FP32; C overwritten (no alpha/beta).
 * The operand split runs either inside the product kernel (converter warps, no FP16 copy of A or
 * B in device memory) or once up front into the handle's workspace: see SGEMM_CUBE_OPT_STRATEGY.
 * Both give bit-identical C unless split-K applies (SGEMM_CUBE_OPT_SPLIT_K).
 *   A_dev  M x K FP32, lda >= K     (device, read)
 *   B_dev  K x N FP32, ldb >= N     (device, read)
 *   C_dev  M x N FP32, ldc >= N     (device, written)
 *   scale_exp s in [0, 24]; accumulation_order SGEMM_CUBE_TERMWISE, SGEMM_CUBE_ELEMENTWISE or
 *   SGEMM_CUBE_ELEMENTWISE_REORDERED
 * Alignment: A_dev, B_dev 16-byte aligned and lda % 4 == 0, ldb % 4 == 0 (else MISALIGNED).
 * C_dev may have any alignment.  M, N, K >= 0, any values (ragged edges are handled).  Empty
 * problems are valid in every GEMM entry point of this header: M == 0 or N == 0 does nothing,
 * K == 0 stores C = 0 (the empty sum; left alone by sgemm_cube_hgemm with accumulate != 0); an
 * operand without elements may be a null pointer.
 * Once the workspace for a problem size exists (after the first call at that size or a larger
 * one) the call only enqueues work on `stream`: it can be captured into a CUDA graph and replayed, also
 * after larger calls (a workspace that a captured call has used is kept until the handle is destroyed).
 * A handle's workspace is shared by its calls, so calls that may overlap on the GPU need one
 * handle per stream.
 * Errors: INVALID_ARG, MISALIGNED, CUDA_ERROR (ALLOC_FAILED only with the TWO_PHASE strategy
 * forced; AUTO falls back to the fused kernel when the workspace cannot be had). */
int sgemm_cube(sgemm_cube_handle h, int M, int N, int K,
               const float* A_dev, int64_t lda,
               const float* B_dev, int64_t ldb,
               float* C_dev, int64_t ldc,
               int scale_exp, int accumulation_order, void* stream);

/* Unfused ablation of the same computation (paper Sec. 5.4: one GEMM pipeline per term):
 * split A and B into FP16 words in the handle's workspace, run three FP16 GEMM passes
 * (hi_A hi_B -> D_hh; lo_A hi_B -> D_x; hi_A lo_B added to D_x), then C = D_hh + 2^-s D_x.
 * Termwise only (accumulation_order must be SGEMM_CUBE_TERMWISE).  Same arguments and
 * alignment-free inputs (the workspace copies are padded).  The workspace
 * (4 bytes x (M K + K N) + 8 bytes x M N, rounded up) is grown with cudaMalloc on first use;
 * Errors: INVALID_ARG, ALLOC_FAILED, CUDA_ERROR. */
int sgemm_cube_unfused(sgemm_cube_handle h, int M, int N, int K,
                       const float* A_dev, int64_t lda,
                       const float* B_dev, int64_t ldb,
                       float* C_dev, int64_t ldc,
                       int scale_exp, int accumulation_order, void* stream);

/* SGEMM-cube on operands that were split beforehand with sgemm_cube_split (all three products
 * and the reconstruction in one kernel; useful when an operand is reused across calls).
 *   Ahi_dev/Alo_dev  M x K FP16 bit patterns, leading dimension lda16 >= K   (device, read)
 *   Bhi_dev/Blo_dev  K x N FP16 bit patterns, leading dimension ldb16 >= N   (device, read)
 * Alignment: the four FP16 pointers 16-byte aligned, lda16 % 8 == 0, ldb16 % 8 == 0.
 * scale_exp must be the value used for the split.  Errors as sgemm_cube. */
int sgemm_cube_presplit(sgemm_cube_handle h, int M, int N, int K,
                        const uint16_t* Ahi_dev, const uint16_t* Alo_dev, int64_t lda16,
                        const uint16_t* Bhi_dev, const uint16_t* Blo_dev, int64_t ldb16,
                        float* C_dev, int64_t ldc,
                        int scale_exp, int accumulation_order, void* stream);

/* Plain FP16 x FP16 -> FP32 GEMM on the tensor cores, D = A16 B16 (or D += A16 B16 when
 * accumulate != 0): one pass of the unfused path, and the plain FP16 GEMM the paper
 * contrasts with (Sec. 6.2).
 *   A16_dev M x K FP16 (lda16 >= K), B16_dev K x N FP16 (ldb16 >= N), D_dev M x N FP32 (ldd >= N).
 * Alignment as sgemm_cube_presplit.  Errors as sgemm_cube. */
int sgemm_cube_hgemm(sgemm_cube_handle h, int M, int N, int K,
                     const uint16_t* A16_dev, int64_t lda16,
                     const uint16_t* B16_dev, int64_t ldb16,
                     float* D_dev, int64_t ldd, int accumulate, void* stream);

/* Host-buffer convenience around sgemm_cube: copies A and B from HOST memory to the handle's
 * device workspace, runs the computation of sgemm_cube there (same strategy choice, see
 * SGEMM_CUBE_OPT_STRATEGY), copies C back to HOST memory and synchronises the stream before
 * returning.  Pinned host memory makes the copies asynchronous to the host but the
 * call still returns only when C_host is complete.  For M >= 1024 and M*N*K >= 2^30 (and a
 * strategy other than FUSED) the call is pipelined: B is copied and split once, A and C move in
 * about eight row panels on two internal copy streams so that the upload of one panel, the
 * products of the previous one and the download of the one before overlap.  The result is
 * bit-identical to sgemm_cube on device copies of the same operands when split-K applies to
 * neither (a panel of a tall problem may have few enough tiles to be split where the whole problem
 * is not; both results pass the same error gates).
 *   A_host M x K (lda >= K), B_host K x N (ldb >= N), C_host M x N (ldc >= N), all FP32 HOST.
 * Errors: INVALID_ARG, ALLOC_FAILED, CUDA_ERROR, DEVICE_TIMEOUT. */
int sgemm_cube_host(sgemm_cube_handle h, int M, int N, int K,
                    const float* A_host, int64_t lda,
                    const float* B_host, int64_t ldb,
                    float* C_host, int64_t ldc,
                    int scale_exp, int accumulation_order, void* stream);

/* Four-term variant: the low-low product that SGEMM-cube drops (paper Sec. 4.3, bounded by
 * Eq. ll_bound) is kept, i.e. the full expansion of (hi_A + lo_A 2^-s)(hi_B + lo_B 2^-s):
 *   C = hi_A hi_B + 2^-s (lo_A hi_B + hi_A lo_B) + 2^-2s lo_A lo_B.
 * It exists to measure what dropping that term costs; it is not part of the paper's method.
 * Termwise only: each stream is summed in k-blocks (SGEMM_CUBE_OPT_TERMWISE_K_BLOCK) and
 *   C = S_hh + (2^-s S_x + 2^-2s S_ll),
 * the small terms combined first.  Runs as: the split of both operands, one FP16 GEMM pass lo_A lo_B into
 * the handle's workspace, the three-product kernel writing its raw sums, one reduction kernel.
 * Arguments, layouts and alignment-free inputs as sgemm_cube_unfused.  Workspace:
 * 4 bytes x (M K + K N) + 12 bytes x M N, rounded up, grown with cudaMalloc on first use.
 * Errors: INVALID_ARG, ALLOC_FAILED, CUDA_ERROR. */
int sgemm_cube_four_term(sgemm_cube_handle h, int M, int N, int K,
                         const float* A_dev, int64_t lda,
                         const float* B_dev, int64_t ldb,
                         float* C_dev, int64_t ldc,
                         int scale_exp, void* stream);

/* Exponent window of a matrix's FP16 high words (paper Sec. 4.2: e_min and e_max of
 * Eq. sf_bounds are the smallest and largest unbiased exponents E' - 15 of the finite high
 * components).  One pass over X on the device; the call synchronises `stream` and writes to HOST
 * memory:
 *   window_out[0] = e_min, window_out[1] = e_max over the NORMAL high words (127 / -127 if none),
 *   window_out[2] = number of entries whose high word is subnormal (|x| < 2^-14: the 22-bit
 *                   guarantee cannot be kept by scaling the residual alone, Sec. 4.2),
 *   window_out[3] = number of entries whose high word is inf or NaN (|x| >= 65520),
 *   window_out[4] = number of entries whose high word is zero.
 *   X_dev rows x cols FP32, ldx >= cols (device, read); window_out 5 x int64 (host, written).
 * Errors: INVALID_ARG, CUDA_ERROR. */
int sgemm_cube_exponent_window(sgemm_cube_handle h, int rows, int cols,
                               const float* X_dev, int64_t ldx,
                               int64_t* window_out, void* stream);

/* Residual-overflow detection (paper Sec. 4.2, Rule 2, which allows a larger scale only if
 * overflowing residuals are caught): the number of entries of a split operand whose high word is finite
 * while its scaled residual word is inf or NaN, i.e. for which (x - hi) 2^s left the FP16 range
 * (the paper's example: x = 32784 at s_b = 12).  A non-zero count means the chosen scale exponent
 * is too large for this operand; sgemm_cube_choose_scale_exp gives one that cannot overflow.
 * One pass over the two word matrices; the call synchronises `stream`.
 *   hi_dev, lo_dev  rows x cols FP16 bit patterns as written by sgemm_cube_split, ldh >= cols
 *   count_out       1 x int64 (host, written)
 * Errors: INVALID_ARG, CUDA_ERROR. */
int sgemm_cube_residual_overflow_count(sgemm_cube_handle h, int rows, int cols,
                                       const uint16_t* hi_dev, const uint16_t* lo_dev, int64_t ldh,
                                       int64_t* count_out, void* stream);

/* Scale exponent for a pair of operands from their exponent windows (host arithmetic only).
 * Eq. sf_bounds:  -3 - e_min <= s_b <= 26 - e_max  over both operands; Sec. 4.2 advises moving
 * the residuals as far above the underflow threshold as the largest entry allows, so the upper end
 * is taken, capped at 15:  *scale_exp_out = min(26 - e_max, 15).  Full normal FP16 range
 * (e_max = 15) gives 11, e_max <= 14 gives at least 12.
 * *protected_out (optional) = 1 if that value also satisfies the lower end and no high word is
 * subnormal, inf or NaN, i.e. if Eq. split_error holds for every entry; else 0.
 * Errors: INVALID_ARG. */
int sgemm_cube_choose_scale_exp(const int64_t* window_a, const int64_t* window_b,
                                int* scale_exp_out, int* protected_out);

/* ---- Whole-input scaling (explicit exponent management).
 * The paper notes (Sec. 4.2, after Rule 1) that once a high word is subnormal, |x| < 2^-14,
 * scaling the residual alone cannot keep 22 bits and that the whole input must be scaled, and
 * leaves that outside its scope (Sec. 7 lists it as future work).  These entry points are that
 * extension: operands are multiplied by powers of two before the split (exact) and the product
 * is multiplied by the inverse power afterwards (exact unless the FP32 result leaves the normal
 * range, then rounded once). */

/* Range of the exponents the FP16 high words of X would have if FP16 had unbounded exponent
 * range: the unbiased exponent of |x| rounded (RN-even) to an 11-bit significand, over the
 * non-zero finite entries.  One pass over X; the call synchronises `stream` and writes HOST memory:
 *   range_out[0] = e_min, range_out[1] = e_max (127 / -127 if no entry qualifies),
 *   range_out[2] = number of inf / NaN entries.
 *   X_dev rows x cols FP32, ldx >= cols (device, read); range_out 3 x int64 (host, written).
 * Errors: INVALID_ARG, CUDA_ERROR. */
int sgemm_cube_hi_exponent_range(sgemm_cube_handle h, int rows, int cols,
                                 const float* X_dev, int64_t ldx,
                                 int64_t* range_out, void* stream);

/* Scaling exponents for a pair of operands from their ranges (host arithmetic only):
 * p = 15 - e_max per operand (its largest high word lands in the top normal FP16 binade, nothing
 * overflows), clamped to [-126, 126]; an operand without non-zero finite entries gets p = 0.  The
 * scaled windows may then span the whole normal range, for which Eq. sf_bounds leaves
 * *scale_exp_out = 11.  *protected_out (optional) = 1 if every non-zero entry of both scaled
 * operands has a normal high word (e_min + p >= -14), i.e. each operand spans at most 30 binades,
 * and there is no inf / NaN; else 0 (the smallest entries then keep fewer than 22 bits).
 * Errors: INVALID_ARG. */
int sgemm_cube_choose_input_scaling(const int64_t* range_a, const int64_t* range_b,
                                    int* p_a_out, int* p_b_out, int* scale_exp_out,
                                    int* protected_out);

/* C = 2^-(p_a + p_b) * sgemm_cube(2^p_a A, 2^p_b B): the split kernels scale while they read, one
 * three-product kernel, one pass over C for the way back (skipped when p_a + p_b == 0).  Always
 * the two-phase route (FP16 words in the handle's workspace), so inputs need no alignment.
 * p_a, p_b in [-126, 126]; the other arguments and layouts as sgemm_cube.
 * Errors: INVALID_ARG, ALLOC_FAILED, CUDA_ERROR. */
int sgemm_cube_scaled(sgemm_cube_handle h, int M, int N, int K,
                      const float* A_dev, int64_t lda,
                      const float* B_dev, int64_t ldb,
                      float* C_dev, int64_t ldc,
                      int p_a, int p_b, int scale_exp, int accumulation_order, void* stream);

/* sgemm_cube_hi_exponent_range on A and B, sgemm_cube_choose_input_scaling, sgemm_cube_scaled in
 * one call.  Synchronises `stream` twice (the ranges are read on the host) before it enqueues the
 * product.  chosen_out (optional, host, 4 x int): p_a, p_b, scale exponent, protected flag.
 * Errors: as the three calls. */
int sgemm_cube_auto_scaled(sgemm_cube_handle h, int M, int N, int K,
                           const float* A_dev, int64_t lda,
                           const float* B_dev, int64_t ldb,
                           float* C_dev, int64_t ldc,
                           int accumulation_order, void* stream, int* chosen_out);

/* ---- Language-model operators on and around the split product.
 *
 * A linear layer with its gradients, layer normalisation with its gradients, log probabilities of
 * given tokens with their gradient, embedding with the table's gradient, softmax cross entropy over a vocabulary with its
 * gradients, and orthogonalised updates.  No call synchronises; once the handle's workspace has its size
 * the calls can be captured into a graph.  A graph keeps the workspace that its calls were captured with: a larger
 * call may follow, and the graph can be replayed until the handle is destroyed.  As everywhere, calls on one handle
 * that may overlap on the GPU, replays among them, need one handle per stream.  Sums, statistics and softmax sums are FP32 (the products' k-blocks as
 * sgemm_cube, termwise, unless said otherwise); every result is the same from call to call.
 * "Any alignment" below means any multiple of the element's size: a pointer that is not one, to a matrix or a vector,
 * is refused with INVALID_ARG, and so is a result in the place of an operand with another leading dimension.
 * Dimensions go to 2^31 - 2^16; above, INVALID_ARG.  Leading dimensions and byte offsets have 64 bits.
 */

/* Operand of a linear layer: a row-major FP32 matrix (f32_dev, ld), or, with f32_dev NULL, one packed by
 * sgemm_cube_pack (hi_dev, lo_dev, ld16, exp_dev).  Packing is what the layer does to an FP32 operand
 * in its workspace on every call; an operand that is used again (a weight that is served, an operand
 * of both the product and a gradient) is packed once by the caller instead.  4 bytes per element. */
typedef struct sgemm_cube_operand {
  const float* f32_dev;
  int64_t ld;
  const uint16_t* hi_dev;
  const uint16_t* lo_dev;
  int64_t ld16;
  const int32_t* exp_dev;
} sgemm_cube_operand;

/* Layout of a weight with K inputs and N outputs. */
enum {
  SGEMM_CUBE_WEIGHT_KN = 0,   /* K x N row-major, the B of sgemm_cube */
  SGEMM_CUBE_WEIGHT_NK = 1    /* N x K row-major, one row per output */
};

enum {
  SGEMM_CUBE_ACT_NONE = 0,
  SGEMM_CUBE_ACT_RELU = 1,       /* max(z, 0), slope 0 at 0 */
  SGEMM_CUBE_ACT_GELU = 2,       /* z Phi(z), Phi the normal distribution function */
  SGEMM_CUBE_ACT_GELU_TANH = 3,  /* z (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2 */
  SGEMM_CUBE_ACT_SILU = 4        /* z / (1 + exp(-z)) */
};
/* Errors of activations and slopes in units u = 2^-24 of their terms (value: z times a weight; slope: that weight plus z
 * times its derivative), A the argument of the exponential:  GELU 24 + 5 A, A = z^2 / 2;  GELU_TANH and SILU 12 + 3 A, A = 1.6
 * (|z| + 0.045 |z|^3) and |z|.  Exponentials below 2^-126 are zero. */

/* Scaling exponent and two-word split of a matrix, all on the device:
 *   p = 15 - e_max, clamped to [-126, 126]; e_max as in sgemm_cube_hi_exponent_range (p = 0 if every
 *   entry is zero, infinite or NaN); hi = fl16(2^p x), lo = fl16((2^p x - hi) 2^11).
 * An entry keeps 22 bits while it is within 2^-29 of the largest; below that its error is at most 2^-51
 * of the largest.  One infinite or NaN entry makes the results that depend on it NaN, no others.
 *   X_dev  rows x cols FP32, ldx >= cols, any alignment                        (device, read)
 *   hi_dev/lo_dev  rows x ld16 words each, 16-byte aligned, ld16 >= cols, ld16 % 8 == 0 (device, written;
 *                  columns past cols are zero up to the next multiple of 8)
 *   exp_dev  one int32                                                          (device, written)
 * Errors: INVALID_ARG, MISALIGNED, CUDA_ERROR. */
int sgemm_cube_pack(sgemm_cube_handle h, int rows, int cols,
                    const float* X_dev, int64_t ldx,
                    uint16_t* hi_dev, uint16_t* lo_dev, int64_t ld16, int32_t* exp_dev, void* stream);

/* Linear layer:  z = X W + b,  Y = act(z) + R.
 *   X  M x K;  W  K inputs, N outputs in weight_layout;  either may be FP32 or packed
 *   bias_dev N FP32 or NULL;  R_dev M x N FP32 (ldr >= N) or NULL, may be Y_dev itself (then ldr == ldy)
 *   Y_dev M x N FP32 (written);  Z_dev M x N FP32 or NULL: z is stored there for the backward pass
 *     (neither Y_dev nor R_dev).  Y and Z must not overlap X, W, bias or each other.
 * FP32 matrices may have any alignment.  The product is the three-product form of sgemm_cube on packed
 * operands, with two forms of its own for an FP32 X of few rows, which read W once and pack nothing ahead:
 * for a short batch (up to 64 rows, to 256 for small weights) X, and an FP32 W that starts its rows on 16 bytes,
 * are split inside the kernel with an exponent for every 64 inputs instead of one for the matrix, and the
 * sums are taken over k-blocks of 64; one to eight rows may be multiplied in FP32.  M, N, K >= 0; K == 0 gives
 * Y = act(b) + R.
 * Errors: INVALID_ARG, MISALIGNED (packed operands), ALLOC_FAILED, CUDA_ERROR. */
int sgemm_cube_linear(sgemm_cube_handle h, int M, int N, int K,
                      const sgemm_cube_operand* X, const sgemm_cube_operand* W, int weight_layout,
                      const float* bias_dev, const float* R_dev, int64_t ldr, int activation,
                      float* Y_dev, int64_t ldy, float* Z_dev, int64_t ldz, void* stream);

/* Gradients of the linear layer for dY = dL/dY:  with dz = dY act'(z),
 *   dX = dz W^T (M x K),  dW = X^T dz (in weight_layout),  dbias = column sums of dz (N).
 * Each output may be NULL and is then not computed; X is looked at for dW only, W for dX only.  Z_dev is
 * the z of the forward call (looked at unless activation is NONE).  The gradient of R is dY.  dz is
 * packed like the other operands, so gradients of any magnitude keep their bits.  Outputs must not
 * overlap the inputs or each other.  An empty sum (M == 0 for dW and dbias, N == 0 for dX) is zero.
 * Errors: INVALID_ARG, MISALIGNED (packed operands), ALLOC_FAILED, CUDA_ERROR. */
int sgemm_cube_linear_backward(sgemm_cube_handle h, int M, int N, int K,
                               const float* dY_dev, int64_t lddy, const float* Z_dev, int64_t ldz,
                               int activation, const sgemm_cube_operand* X, const sgemm_cube_operand* W,
                               int weight_layout, float* dX_dev, int64_t lddx, float* dW_dev, int64_t lddw,
                               float* dbias_dev, void* stream);

/* Element types of the operators below. */
enum {
  SGEMM_CUBE_F32 = 0,
  SGEMM_CUBE_F16 = 1,
  SGEMM_CUBE_BF16 = 2
};

/* Layer normalisation of each row:  y = (x - mean) rstd w + b,  rstd = 1 / sqrt(var + eps), var the mean of
 * (x - mean)^2.  Computed in FP32, rounded once to the element type.
 *   X_dev, Y_dev  rows x cols of `dtype`, row-major, any alignment (Y_dev may be X_dev with ldy == ldx)
 *   weight_dev, bias_dev  cols FP32 or NULL (1 and 0);  mean_dev, rstd_dev  rows FP32 or NULL (written,
 *   for the backward pass)
 * rows >= 0, cols >= 1, eps >= 0.  Errors: INVALID_ARG, CUDA_ERROR. */
int sgemm_cube_layer_norm(sgemm_cube_handle h, int rows, int cols, int dtype,
                          const void* X_dev, int64_t ldx, const float* weight_dev, const float* bias_dev,
                          float eps, void* Y_dev, int64_t ldy, float* mean_dev, float* rstd_dev, void* stream);

/* Its gradients for dY:  with u = dY w and n = (x - mean) rstd,
 *   dX = rstd (u - mean(u) - n mean(u n)),  dweight = sum over rows of dY n,  dbias = sum over rows of dY.
 * dX_dev rows x cols of `dtype` or NULL (may be dY_dev with lddx == lddy); dweight_dev, dbias_dev cols FP32
 * or NULL (zero when rows == 0).  mean_dev and rstd_dev are the forward call's; mean rstd has to be an FP32 number
 * (it is not in a constant row of 1e36 or more with eps = 1e-5: dX may be NaN there).
 * Errors: INVALID_ARG, ALLOC_FAILED, CUDA_ERROR. */
int sgemm_cube_layer_norm_backward(sgemm_cube_handle h, int rows, int cols, int dtype,
                                   const void* dY_dev, int64_t lddy, const void* X_dev, int64_t ldx,
                                   const float* weight_dev, const float* mean_dev, const float* rstd_dev,
                                   void* dX_dev, int64_t lddx, float* dweight_dev, float* dbias_dev,
                                   void* stream);

/* Log probabilities of given tokens under softmax(scale * logits), row by row, in one pass over the logits:
 *   logp_dev[r]     = scale x[r, t] - lse[r], t = tokens_dev[r]; 0 where t < 0 (no target), NaN where t >= vocab
 *   entropy_dev[r]  = - sum_j p_j log p_j, a probability of zero contributing nothing      (or NULL)
 *   stats_dev[r]    = {largest logit m, sum of exp(scale (x - m))}; lse = scale m + log of the second
 *                     (rows x 2 FP32, for the backward pass; or NULL)
 *   top_logp_dev, top_index_dev  rows x top_k: the largest log probabilities, descending, and their
 *                     columns; equal logits are ordered by column (both NULL iff top_k == 0)
 *   logits_dev      rows x vocab of `dtype`, row-major, any alignment; -inf marks a token that is not allowed
 *   tokens_dev      rows int64, or NULL with logp_dev NULL
 * 0 <= top_k <= 32 and <= vocab; vocab >= 1; 2^-30 <= scale <= 2^30.  A row whose every logit is -inf has no
 * distribution: logp and top_logp are -inf, entropy 0, top_index the first columns, stats {-inf, 0}, its
 * gradient zero.  A row that holds NaN or +inf gives NaN (top_index then names valid columns, no more).
 * Errors: INVALID_ARG, CUDA_ERROR. */
int sgemm_cube_token_logprobs(sgemm_cube_handle h, int rows, int vocab, int dtype,
                              const void* logits_dev, int64_t ld, const int64_t* tokens_dev, float scale,
                              float* logp_dev, float* entropy_dev, float* stats_dev,
                              int top_k, float* top_logp_dev, int64_t* top_index_dev, void* stream);

/* Gradient of the logits for dlogp and dentropy (each rows FP32 or NULL, not both NULL):
 *   dlogits[r, j] = scale (dlogp[r] (1[j == t] - p_j) - dentropy[r] p_j (log p_j + H))
 * with the forward call's stats and (for dentropy) entropy.  A row without target takes no part in dlogp.
 * dlogits_dev rows x vocab of `dtype`, may be logits_dev itself (then lddl == ld).
 * Errors: INVALID_ARG, CUDA_ERROR. */
int sgemm_cube_token_logprobs_backward(sgemm_cube_handle h, int rows, int vocab, int dtype,
                                       const void* logits_dev, int64_t ld, const int64_t* tokens_dev,
                                       float scale, const float* stats_dev, const float* entropy_dev,
                                       const float* dlogp_dev, const float* dentropy_dev,
                                       void* dlogits_dev, int64_t lddl, void* stream);

/* Embedding: row t = tokens_dev[i] of a table times a scale,  Y[i] = scale table[t];  zeros where t < 0 (padding), NaN where
 * t >= vocab.  Computed in FP32, rounded once to the element type.
 *   tokens_dev  rows int64;  table_dev  vocab x cols, Y_dev  rows x cols, both of `dtype`, row-major, any alignment
 * rows >= 0, vocab >= 1, cols >= 1; the scale is finite.  Y must not overlap the table.
 * Errors: INVALID_ARG, CUDA_ERROR. */
int sgemm_cube_embedding(sgemm_cube_handle h, int rows, int vocab, int cols, int dtype,
                         const int64_t* tokens_dev, const void* table_dev, int64_t ld, float scale,
                         void* Y_dev, int64_t ldy, void* stream);

/* Gradient of the table for dY:  dtable[v] = scale * sum of dY[i] over the rows with tokens_dev[i] == v, for all
 * v of the vocabulary (accumulate == 0: rows that no token names become zero), or that added to what dtable holds
 * (accumulate == 1: such rows are left alone).  Tokens outside [0, vocab) have no row and take no part.
 * The sums are FP32 over rows in their order, in pieces of at least 32 of the sorted rows: the same from call to call.
 *   dY_dev  rows x cols of `dtype`;  dtable_dev  vocab x cols FP32, ldd >= cols.  Any alignment, no overlap.
 * Workspace: 16 bytes a row, 1 byte a token of the vocabulary, and FP32 rows of cols: two for every 32 rows, 8192 at most.
 * Errors: INVALID_ARG, ALLOC_FAILED, CUDA_ERROR. */
int sgemm_cube_embedding_backward(sgemm_cube_handle h, int rows, int vocab, int cols, int dtype,
                                  const int64_t* tokens_dev, const void* dY_dev, int64_t lddy, float scale,
                                  int accumulate, float* dtable_dev, int64_t ldd, void* stream);

/* Softmax cross entropy of a linear layer over a vocabulary of N tokens, from the layer's inputs; the logits z = X W + b are no operand
 * and are not returned:
 *   lse_dev[r]  = log sum_j exp(z[r, j])
 *   loss_dev[r] = lse[r] - z[r, t], t = targets_dev[r]; 0 where t < 0 (no target), NaN where t >= N
 * Either may be NULL, not both.  X, W, weight_layout and bias as in sgemm_cube_linear, whose products these are (its forms for few rows
 * among them, and FP32 multiplication for up to 64 rows); a bias of -inf takes a token out.  A row whose every logit is -inf has lse -inf and, with a target, loss +inf.
 * M >= 0, N >= 1, K >= 1.  Workspace: what sgemm_cube_linear takes to pack its operands, and M N / 8 bytes: the logits stay in tiles.  Where
 * sgemm_cube_linear has forms for few rows (up to 64, of narrow layers up to 256) it holds the logits instead, 4 bytes each, and for an FP32 W
 * with rows off 16-byte boundaries a copy of it (4 bytes an entry) or, for 5 to 16 rows, parts of the logits' sums (another 4 bytes
 * a logit, and 5 MB).
 * Errors: INVALID_ARG, MISALIGNED (packed operands), ALLOC_FAILED, CUDA_ERROR. */
int sgemm_cube_cross_entropy(sgemm_cube_handle h, int M, int N, int K,
                             const sgemm_cube_operand* X, const sgemm_cube_operand* W, int weight_layout,
                             const float* bias_dev, const int64_t* targets_dev, float* loss_dev, float* lse_dev,
                             void* stream);

/* The same with its gradients for dloss (M FP32): with dz[r, j] = dloss[r] (exp(z[r, j] - lse[r]) - 1[j == t]), 0 where t < 0,
 *   dX = dz W^T (M x K),  dW = X^T dz (in weight_layout),  dbias = column sums of dz (N).
 * It forms the logits itself and needs no call before it: loss_dev and lse_dev are written as above.  Every output
 * may be NULL and is then not computed.  A row whose every logit is -inf has no gradient.  dz is packed with one exponent, from the largest
 * |dloss| of a row with a target, as sgemm_cube_linear_backward packs its dz.  Outputs must not overlap inputs or each
 * other.  M == 0: dW and dbias are zero.
 * Workspace: what sgemm_cube_linear takes to pack its operands, and 8 bytes for every logit (rows of them rounded up to 8), twice what a matrix
 * of them takes, but 2 GiB at the most (256 rows of them where those are more); more rows are taken in pieces, whose dW are added up.  Beside that for sums:
 * an eighth of a byte a logit, 12 bytes a row and, with dbias, 4 bytes a token for every 32 rows (or part of them) of a piece; for few rows as
 * above parts of the logits' sums, and of those of dX (4 bytes an entry, and 20 MB).
 * Errors: INVALID_ARG, MISALIGNED (packed operands), ALLOC_FAILED, CUDA_ERROR. */
int sgemm_cube_cross_entropy_backward(sgemm_cube_handle h, int M, int N, int K,
                                      const sgemm_cube_operand* X, const sgemm_cube_operand* W, int weight_layout,
                                      const float* bias_dev, const int64_t* targets_dev, const float* dloss_dev,
                                      float* loss_dev, float* lse_dev, float* dX_dev, int64_t lddx,
                                      float* dW_dev, int64_t lddw, float* dbias_dev, void* stream);

/* An update brought near the closest matrix with orthonormal rows (columns, where rows > cols) by Newton-Schulz products:
 *   X = G / (|G|_F + eps);   steps times:  X <- a X + b (X X^T) X + c (X X^T)^2 X;   O = scale X + beta R
 * The polynomial acts on the singular values alone: x -> a x + b x^3 + c x^5.
 *   G_dev  rows x cols of `dtype`, any alignment
 *   coefficients  3 * steps floats (HOST): a, b, c of every step; NULL: 3.4445, -4.7750, 2.0315 in all of them
 *   R_dev  rows x cols FP32 (ldr >= cols) or NULL (no second term): the weight that is updated, with beta = 1 - rate * decay and a scale
 *     of -rate times what the sizes ask for; may be O_dev itself (then ldr == ldo)
 *   O_dev  rows x cols FP32 (written); may be G_dev where that is FP32 (then ldo == ldg; G is read before O is written)
 * All matrices of the iteration are kept as two FP16 words (22 bits) with exponents that follow from the coefficients:
 * entries of X keep 22 bits down to 2^-29 of the largest singular value.  The products are those of sgemm_cube, termwise; the sum of
 * squares is FP64, so G may have any FP32 size.  An infinite or NaN entry makes every entry of X NaN.  Zeros give zeros.
 * rows, cols >= 0; 1 <= steps <= 64; eps >= 0; singular values must stay in [2^-20, 2^20] at their largest after every step.
 * Workspace: 8 bytes an entry, 8 bytes for every entry of the smaller Gram matrix.
 * Errors: INVALID_ARG, ALLOC_FAILED, CUDA_ERROR. */
int sgemm_cube_orthogonalize(sgemm_cube_handle h, int rows, int cols, int dtype, const void* G_dev, int64_t ldg,
                             int steps, const float* coefficients, float eps, float scale,
                             const float* R_dev, int64_t ldr, float beta, float* O_dev, int64_t ldo, void* stream);

/* Size in bytes of the fixed device scratch area used by sgemm_cube_unfused_static. */
#define SGEMM_CUBE_STATIC_SCRATCH_BYTES (32u << 20)

/* The unfused computation (same arithmetic, same kernels and same result as sgemm_cube_unfused,
 * termwise order) for callers that are not allowed to allocate device memory: code running inside
 * another framework's memory pool with a hard cap, real-time or safety-certified loops where
 * cudaMalloc/cudaFree (which may synchronise the whole device or fail late) are forbidden after
 * start-up, or a process whose remaining device memory is already committed.  The paper has no
 * counterpart of this entry point; it exists for such integrations only.
 *
 * It needs no handle and calls no cudaMalloc, cudaFree or other allocating routine.  Its scratch
 * (the FP16 words of A and B and two FP32 M x N partial results) lives in a fixed array of
 * SGEMM_CUBE_STATIC_SCRATCH_BYTES (32 MiB) that is part of the library's device image: every GPU
 * on which the library is loaded holds those 32 MiB until the process exits.
 *   Limit: 4*(M*K8 + K*N8) + 8*M*N4 bytes (K8, N8 = K, N rounded up to 8; N4 = N rounded up to 4;
 *   each of the six pieces rounded up to 256 bytes) must not exceed the array, e.g. up to
 *   1024 x 1024 x 1024 or 2048 x 512 x 1024.  Larger problems return SGEMM_CUBE_TOO_LARGE and
 *   enqueue nothing.
 *   Arguments, layouts and alignment as sgemm_cube_unfused, on the CURRENT device
 *   (A_dev, B_dev, C_dev must be on it).
 *   The first call on a device looks up the array's device address and configures the kernels;
 *   make that first call outside any stream capture, and at start-up: the 32 MiB are committed
 *   when the CUDA runtime loads the library's device code on that GPU, which with lazy module
 *   loading can be as late as this first call, so a process whose device memory is already
 *   exhausted gets CUDA_ERROR from it.  Later calls only launch and leave the amount of free
 *   device memory unchanged.
 *   All calls share the one array, which keeps whatever the last call left in it.  Every region a
 *   call reads is first overwritten by that call, so results never depend on earlier calls; but
 *   two calls that may overlap on the GPU (different streams without an ordering between them,
 *   whether from one host thread or several) race on the scratch and give undefined results.
 *   Host threads may call concurrently as far as the host side goes (enqueueing is serialised
 *   internally).
 *   A kernel-side bounded-wait failure (never expected) cannot be reported by this entry point;
 *   C is then unspecified.
 * Errors: INVALID_ARG, TOO_LARGE, UNSUPPORTED_ARCH, CUDA_ERROR. */
int sgemm_cube_unfused_static(int M, int N, int K,
                              const float* A_dev, int64_t lda,
                              const float* B_dev, int64_t ldb,
                              float* C_dev, int64_t ldc,
                              int scale_exp, void* stream);

/* Synchronise `stream` and report (then clear) the device error word.
 * Returns OK, DEVICE_TIMEOUT (detail in *detail_out if non-NULL: a code naming the wait that
 * gave up) or CUDA_ERROR. */
int sgemm_cube_check(sgemm_cube_handle h, void* stream, uint32_t* detail_out);

/* Number of kernels this handle has launched since creation (for launch accounting). */
int64_t sgemm_cube_launch_count(sgemm_cube_handle h);

/* Device time, in milliseconds, of the tensor-core kernel of the most recent sgemm_cube call
 * (requires SGEMM_CUBE_OPT_TIME_KERNEL = 1 before that call; waits for the kernel to finish).
 * Errors: INVALID_ARG (timing off, or no call yet), CUDA_ERROR. */
int sgemm_cube_last_kernel_ms(sgemm_cube_handle h, float* ms_out);

/* Mean device time, in milliseconds, of the tensor-core kernel over the sgemm_cube calls made
 * since SGEMM_CUBE_OPT_TIME_KERNEL was set to 1 or since the previous call of this function (at
 * most the 128 most recent ones: one CUDA event pair is kept per call); *calls_out (optional) =
 * how many calls were averaged.  Waits for those kernels to finish, then starts a new average.
 * Errors: INVALID_ARG (timing off, or no call since), CUDA_ERROR. */
int sgemm_cube_mean_kernel_ms(sgemm_cube_handle h, float* mean_ms_out, int* calls_out);

/* SM clock cycles and nanoseconds (device global timer) that the tensor-core kernel of the most
 * recent sgemm_cube call ran for, taken inside the kernel by its first CTA (requires
 * SGEMM_CUBE_OPT_TIME_KERNEL = 1 before that call; waits for the device to finish).  Their
 * quotient is the SM clock the kernel actually ran at, which under a power cap is well below the
 * clock that nvidia-smi shows between kernels; the three-GEMM roofline at that clock is
 * SMs x 8192 FP16 flop/clk x (cycles / ns) / 3.
 * Errors: INVALID_ARG (timing off), CUDA_ERROR. */
int sgemm_cube_last_kernel_clock(sgemm_cube_handle h, uint64_t* sm_cycles_out, uint64_t* ns_out);

/* ---- Diagnostics for the failure-reporting path (tests; nothing on the GEMM path calls them).
 * Every wait inside the kernels is bounded; a wait that runs out writes a code into the handle's
 * device error word, the CTA drains and exits, and sgemm_cube_check / sgemm_cube_destroy report
 * SGEMM_CUBE_DEVICE_TIMEOUT.  Neither function below makes a GEMM kernel fail.
 *
 * sgemm_cube_debug_inject_error: host-made failure.  Waits for the device, then copies `code`
 * into the error word, as if a kernel had recorded it; with 0x10C (the sorting of an embedding's gradient) it also leaves the
 * count of the blocks that had met, as that kernel does.
 * sgemm_cube_debug_wait_timeout: enqueues a one-CTA kernel in which one thread runs the kernels'
 * bounded wait, with a limit of `limit_clocks` SM clocks (1 .. 10^8), on a barrier that nothing
 * signals; the wait gives up after the limit and records code 0x1F0.  The kernel then ends
 * normally and the context stays usable.
 * Errors: INVALID_ARG, CUDA_ERROR. */
int sgemm_cube_debug_inject_error(sgemm_cube_handle h, uint32_t code);
int sgemm_cube_debug_wait_timeout(sgemm_cube_handle h, int64_t limit_clocks, void* stream);

/* Text for a status code (static storage; never NULL). */
const char* sgemm_cube_status_string(int status);

/* Library version: major * 10000 + minor * 100 + patch. */
int sgemm_cube_version(void);

#ifdef __cplusplus
}
#endif
#endif /* SGEMM_CUBE_H_ */
