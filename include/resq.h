/*
 * resq.h - C ABI of the MI355X (gfx950) ResQ mixed-precision linear layer.
 *
 * ResQ (arXiv 2412.14363) keeps r of the K input coefficients of a linear
 * layer in 8 bits and the other K - r in 4 bits, for activations and weights
 * alike, and evaluates the layer as two integer GEMMs between operands of the
 * same precision whose dequantized results are added (Section 4.1, Eq. 2-4).
 * This library is that inference path: per-token activation quantization,
 * offline weight quantization and packing, the fused two-GEMM kernel with its
 * dequantizing epilogue, and the online Hadamard transform of the down_proj
 * input (Section 4.3).
 *
 * Conventions common to every call
 *   - Columns [0, r) of the K axis are the high-precision (INT8) group, columns
 *     [r, K) the low-precision (INT4) group.  r = 0 and r = K are legal; the
 *     pointers of an empty group may be null.  K - r must be even.
 *   - The quantizer is the symmetric one of Section 3, Eq. 1: zero-point 0,
 *     scale = max|x| / (2^(N-1) - 1) over the group (127 for N = 8, 7 for
 *     N = 4), code = clip(round_half_even(x / scale)), fp32 IEEE division.
 *     A group that is all zero has scale 1.
 *   - Every pointer is a DEVICE pointer owned by the caller unless marked
 *     "host".  The library allocates nothing and never synchronizes: work is
 *     enqueued on `stream` (a hipStream_t passed as void*; null = the default
 *     stream) and results are ready when that stream reaches them.
 *   - Every function returns a resq_status.  Arguments are checked on the host
 *     before anything is launched; on any status other than RESQ_OK nothing
 *     was enqueued (RESQ_ERR_HIP excepted: the runtime refused a launch).
 *   - bf16 tensors are row-major with a leading dimension given in ELEMENTS.
 *   - Inputs are expected to be finite; NaN or infinity give unspecified codes.
 */
#ifndef RESQ_H
#define RESQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum resq_status {
    RESQ_OK = 0,
    RESQ_ERR_NULL = 1,   /* a required pointer is null                               */
    RESQ_ERR_SHAPE = 2,  /* M, N, K < 1, r outside [0, K], K - r odd, ld too small,
                            bad Hadamard block, size beyond a documented limit        */
    RESQ_ERR_ALIGN = 3,  /* a pointer or leading dimension breaks a stated alignment  */
    RESQ_ERR_BUFFER = 4, /* packed-weight buffer smaller than resq_packed_weight_bytes */
    RESQ_ERR_HIP = 5     /* the HIP runtime reported an error at launch               */
} resq_status;

/* Static, human-readable name of a status code (host pointer, never null). */
const char* resq_status_string(int status);

/*
 * Measurement aid: the next quantize, GEMM or Hadamard kernel that THIS host
 * thread launches through the library records the two events (hipEvent_t passed
 * as void*, created by the caller) exactly at the kernel's start and end, so
 * that hipEventElapsedTime(start, stop) is the kernel's own duration without
 * the gaps that events recorded around a launch include.  One-shot: the request
 * is consumed by that launch.  The helper kernels of resq_pack_weights and
 * resq_unpack_weights are not timed.
 */
int resq_time_next_kernel(void* start_event, void* stop_event);

/* ---- layout queries (pure host functions) ------------------------------- */

/*
 * Bytes per token row of the two activation code arrays written by
 * resq_quantize_act and read by resq_gemm_mixed.  High codes are int8, one per
 * byte, the row padded with zero codes to a multiple of 128 codes.  Low codes
 * are nibbles, two per byte: column r + 2j in bits 0..3 of byte j as code + 8
 * (offset binary, 1..15) and column r + 2j + 1 in bits 4..7 in two's
 * complement, so that each of the two can be widened for the int8 matrix cores
 * with a single AND; the row is padded with zero codes (bytes 0x08) to a
 * multiple of 256 codes.  Zero codes add nothing to Eq. 4's sums.  Both return
 * 0 for an empty group and -1 for an invalid (K, r).
 */
int64_t resq_act_hi_ld(int64_t K, int64_t r);
int64_t resq_act_lo_ld(int64_t K, int64_t r);

/*
 * Size in bytes of the packed weight buffer of an [N, K] layer with a high
 * group of width r; 0 for invalid arguments.  The layout is private to the
 * library (tiled for the matrix cores; read it back with resq_unpack_weights):
 * N is padded to a multiple of 256 rows, the high group to a multiple of 128
 * and the low group to a multiple of 256 codes, all with zero codes, followed
 * by two fp16 scale vectors and three int32 sums of codes per channel (16 bytes
 * per channel in all).
 */
size_t resq_packed_weight_bytes(int64_t N, int64_t K, int64_t r);

/*
 * Default block size of the online Hadamard transform over `width` columns:
 * the largest power of two that divides width, at most 8192 (Sylvester
 * Hadamard matrices exist only for powers of two, so a width such as
 * 12544 = 49 * 256 is covered by a block-diagonal transform, which is still
 * orthogonal).  Returns 0 for width < 1.
 */
int64_t resq_hadamard_block(int64_t width);

/* ---- the hot path -------------------------------------------------------- */

/*
 * Per-token mixed-precision activation quantization (Section 4.1 Eq. 2 with
 * the quantizer of Section 3 Eq. 1, per token as in Section 5.1).
 *   x      bf16 [M, ldx], ldx >= K                      (read)
 *   q_hi   int8  [M, resq_act_hi_ld(K, r)]              (written, padding zeroed)
 *   q_lo   uint8 [M, resq_act_lo_ld(K, r)]              (written, padding = zero codes)
 *   s_hi, s_lo   fp32 [M] scales of the two groups      (written)
 *   lo_sum int32 [M]: per token, the sum of the low codes of the odd columns
 *          r + 1, r + 3, ...                            (written)
 *          resq_gemm_mixed needs it to undo the offset of the nibbles that are
 *          stored as code + 8 (see resq_act_lo_ld)
 * One read of x; the absmax, the division, the rounding and the packing are
 * fused.  Alignment: none required; x 16-byte aligned with ldx, K and r
 * multiples of 8 selects the vectorized path.  q_hi and q_lo must be 16-byte
 * aligned.  Limits: K <= 2^20.
 */
int resq_quantize_act(const void* x, int64_t ldx, int64_t M, int64_t K, int64_t r,
                      int8_t* q_hi, uint8_t* q_lo, float* s_hi, float* s_lo, int32_t* lo_sum,
                      void* stream);

/*
 * The online Hadamard projection of the low group (Section 4.3, U_D; see
 * resq_online_hadamard) fused with resq_quantize_act: the codes, scales and
 * lo_sum are exactly those of
 *   resq_online_hadamard(x, t, ..., col_begin = r, col_end = K, block)
 *   resq_quantize_act(t, ...)
 * (same butterflies in the same order, same rounding of the rotated values to
 * bf16 before they are quantized), but the rotated row is not written to memory
 * and read back: one read of x in all.  Blocks of 256 (the Llama down_proj
 * inputs) take most of their sums on the bf16 matrix cores, in another order:
 * there a rotated value may be the neighbouring bf16 of the stand-alone
 * transform's (both within rounding of the exact transform), and the codes are
 * exactly those of resq_quantize_act on the rotated row that x_rot receives.
 *   block   power of two in [8, 512] dividing both r and K - r (a block is held
 *           by one wavefront); 0 selects resq_hadamard_block(K - r).  Other
 *           sizes: RESQ_ERR_SHAPE, use the two calls above.
 *   x_rot   null, or bf16 [M, ld_rot] (ld_rot >= K, 16-byte aligned, ld_rot a
 *           multiple of 8): receives columns [r, K) of the rotated rows, for
 *           inspection and parity checks; columns [0, r) are not touched.
 * Needs the vectorized path: x 16-byte aligned, ldx, K, r multiples of 8,
 * K <= 16384, or with blocks of 256 r <= 4096 and K - r <= 26624 (else
 * RESQ_ERR_ALIGN).  Other arguments as resq_quantize_act.
 */
int resq_hadamard_quantize_act(const void* x, int64_t ldx, int64_t M, int64_t K, int64_t r,
                               int64_t block, int8_t* q_hi, uint8_t* q_lo, float* s_hi,
                               float* s_lo, int32_t* lo_sum, void* x_rot, int64_t ld_rot,
                               void* stream);

/*
 * Per-token quantization with the ASYMMETRIC branch of Section 3 Eq. 1, the
 * setting of the paper's own experiments for activations (Section 5.1), applied
 * to each group separately:
 *   z = min(x), s = (max(x) - min(x)) / (2^N - 1), code = clip(round((x - z) / s), 0, 2^N - 1)
 * with x - z and the quotient in fp32 and the round half to even; a constant
 * group has s = 1.  Codes are STORED minus 2^(N-1) in the layouts of
 * resq_quantize_act (int8 for the high group; for the low group the plain code
 * 0..15 in bits 0..3 for even columns, a two's-complement nibble of code - 8 in
 * bits 4..7 for odd columns), so that the matrix cores see the operands they see
 * for symmetric codes; padding is the stored code 0.
 *   s_hi, s_lo   fp32 [M] scales                                     (written)
 *   c_hi, c_lo   fp32 [M]: z + 2^(N-1) s, the real value that the stored code 0
 *                stands for, i.e. x ~ stored * s + c                 (written)
 *   lo_sum       as in resq_quantize_act, over the stored values     (written)
 *   hadamard_block  0: none; > 0: the block Walsh-Hadamard transform of the low
 *                group first, in the same kernel, under the conditions of
 *                resq_hadamard_quantize_act; < 0: the same with the default block
 * Other arguments, alignment and limits as resq_quantize_act.  Feed the result
 * to resq_gemm_mixed_asym.
 */
int resq_quantize_act_asym(const void* x, int64_t ldx, int64_t M, int64_t K, int64_t r,
                           int64_t hadamard_block, int8_t* q_hi, uint8_t* q_lo, float* s_hi,
                           float* s_lo, float* c_hi, float* c_lo, int32_t* lo_sum, void* stream);

/*
 * resq_quantize_act_asym with the block Walsh-Hadamard transform of the low
 * group in front (the down_proj input with asymmetric codes, Sections 4.3 and
 * 5.1) and the optional inspection output of resq_hadamard_quantize_act:
 * block, x_rot, ld_rot as there, everything else as resq_quantize_act_asym.
 */
int resq_hadamard_quantize_act_asym(const void* x, int64_t ldx, int64_t M, int64_t K, int64_t r,
                                    int64_t block, int8_t* q_hi, uint8_t* q_lo, float* s_hi,
                                    float* s_lo, float* c_hi, float* c_lo, int32_t* lo_sum,
                                    void* x_rot, int64_t ld_rot, void* stream);

/*
 * Offline weight quantization and packing (Section 4.1 Eq. 3; per output
 * channel, symmetric, round-to-nearest, Section 5.1).
 *   w       bf16 [N, ldw], ldw >= K: (out_features, in_features)   (read)
 *   packed  resq_packed_weight_bytes(N, K, r) bytes, 256-byte aligned (written)
 * The per-channel scale of each group is stored as fp16, rounded toward +inf
 * from max|w| / qmax and clamped to [2^-14, 65504]; the codes are computed
 * with the stored value, so |w - code * scale| <= scale / 2 holds for it.
 * packed_bytes is the capacity of `packed`.
 */
int resq_pack_weights(const void* w, int64_t ldw, int64_t N, int64_t K, int64_t r,
                      void* packed, size_t packed_bytes, void* stream);

/*
 * Inverse of the packing, for inspection and parity checks: plain row-major
 * codes (one per byte) and the stored fp16 scale bit patterns.
 *   w_hi int8 [N, r]   w_lo int8 [N, K - r]   sw_hi, sw_lo uint16 [N]   (written)
 */
int resq_unpack_weights(const void* packed, int64_t N, int64_t K, int64_t r, int8_t* w_hi,
                        int8_t* w_lo, uint16_t* sw_hi, uint16_t* sw_lo, void* stream);

/*
 * The layer (Section 4.1 Eq. 4): for every token m and output channel n
 *   A_hi[m, n] = sum_{k <  r} q_hi[m, k] * w_hi[n, k]       (int8 x int8 -> int32)
 *   A_lo[m, n] = sum_{k >= r} q_lo[m, k] * w_lo[n, k]       (int4 x int4 -> int32)
 *   y[m, n]    = bf16( A_hi * s_hi[m] * sw_hi[n] + A_lo * s_lo[m] * sw_lo[n] )
 * Both sums run on the matrix cores inside one kernel (int8, the nibbles widened in
 * registers; on layers of more than one round of 128 x 128 tiles the low group as fp8
 * numbers, which hold the codes and their sums exactly); y is written once.  The integer sums are exact: the call
 * accepts r <= 132104 and K - r <= 2^20, so neither 128 * 127 * r (stored asymmetric
 * codes reach -128) nor the widened low sum 1680 * (K - r) can reach 2^31 (larger
 * groups: RESQ_ERR_SHAPE).
 *   q_hi, q_lo, s_hi, s_lo, lo_sum   as written by resq_quantize_act for the same K, r
 *   packed                   as written by resq_pack_weights for the same N, K, r
 *   y        bf16 [M, ldy], ldy >= N                         (written)
 *   dbg_acc_hi, dbg_acc_lo   int32 [M, N] each, or null: when given, the two
 *                            integer accumulators are written as well
 * Shapes with M <= 64 take weight-streaming kernels bound by HBM bandwidth
 * (the packed weights cross HBM once; the code rows of up to 16 tokens are
 * read as they are needed while they are short enough to stay in cache, else
 * and up to 64 tokens they are chunked through LDS; layers with
 * few output channels split the reduction axis over wavefronts), larger M the
 * tiled matrix-core kernel (128 x 128 tiles, or 64 x 128 where those are at
 * most 512), except that up to 1024 tokens go through the streaming kernel in
 * slices of 16 to 64 tokens where that is estimated faster (few tiles, each
 * walking the whole reduction axis alone); the integer accumulators are
 * identical.
 * Alignment: q_hi, q_lo 16 bytes; packed 256 bytes; y 2 bytes.
 */
int resq_gemm_mixed(const int8_t* q_hi, const uint8_t* q_lo, const float* s_hi,
                    const float* s_lo, const int32_t* lo_sum, int64_t M, const void* packed,
                    int64_t N, int64_t K,
                    int64_t r, void* y, int64_t ldy, int32_t* dbg_acc_hi, int32_t* dbg_acc_lo,
                    void* stream);

/*
 * Which kernel resq_gemm_mixed (and its variants) runs for a shape: host only,
 * no device call.  For callers that want to know, and for tests.
 *   kernel        0: weight-streaming kernel for at most 16 tokens
 *                 1: weight-streaming kernel with the activation codes chunked
 *                    through LDS, in slices of 16 * token_groups tokens (also
 *                    for 10 to 16 tokens on wide layers of 64 MB and more)
 *                 2: tiled matrix-core kernel, 128 x 128 tiles
 *                 3: tiled matrix-core kernel, 64 (tokens) x 128 tiles, where
 *                    those are at most 512                           (written)
 *   token_groups  1, 2 or 4 for kernel 1 (1 for kernel 0, 0 for kernels 2, 3) (written)
 *   runs          parts into which the reduction axis of a channel group (kernels
 *                 0, 1: 1..8) or of a tile (kernel 3: 2 where the tiles are at
 *                 most 256, else 1) is cut across wavefronts; 0 for kernel 2 (written)
 * Errors as resq_gemm_mixed for the shape; RESQ_ERR_NULL for a null output.
 */
int resq_gemm_mixed_plan(int64_t M, int64_t N, int64_t K, int64_t r, int* kernel, int* token_groups,
                         int* runs);
/*
 * Whether kernel 2 of that plan takes the low group as fp8 numbers for the shape (1) or int8 ones (0);
 * 0 for the other kernels and for sizes that resq_gemm_mixed refuses.  Host only.
 */
int resq_gemm_mixed_low_fp8(int64_t M, int64_t N, int64_t K, int64_t r);

/*
 * The layer in ONE call for the generation stage (a handful of tokens, Section 1:
 * memory-bound): resq_quantize_act (Section 4.1 Eq. 2) and resq_gemm_mixed
 * (Eq. 4) in one kernel.  Every workgroup of the weight-streaming kernel
 * quantizes the M token rows itself, straight into the LDS rows that the kernel
 * reads its activation codes from, while its first weight blocks are on their
 * way: the codes never go to memory and the launch of the quantizer is saved.
 * y is bit-identical to the two calls (same quantizer arithmetic, same integer
 * sums, same epilogue).
 *   x        bf16 [M, ldx], ldx >= K                          (read)
 *   M        1..16 tokens whose code rows fit LDS (M * (padded row bytes) <=
 *            140 KiB; K = 8192 with r = 1024 takes 16), else RESQ_ERR_SHAPE: use
 *            the two calls
 *   packed, N, K, r, y, ldy   as in resq_gemm_mixed
 * Alignment: x 16 bytes and ldx, K, r multiples of 8 (else RESQ_ERR_ALIGN); packed
 * 256 bytes; y 2 bytes.  Symmetric codes, no gated epilogue, no debug outputs.
 */
int resq_quantize_gemm_mixed(const void* x, int64_t ldx, int64_t M, const void* packed, int64_t N,
                             int64_t K, int64_t r, void* y, int64_t ldy, void* stream);

/*
 * The gate and up projections of an MLP block as ONE layer with the gated
 * activation in its epilogue, so that the down_proj input (which Section 4.3
 * transforms and quantizes next) is written directly instead of two [M, F]
 * tensors that another kernel would read back:
 *   y[m, c] = bf16( silu(z[m, 2c]) * z[m, 2c + 1] ),  silu(x) = x / (1 + exp(-x)),
 * z the dequantized output of resq_gemm_mixed (in fp32, not rounded to bf16 in
 * between).  `packed` holds N2 = 2 F channels packed by resq_pack_weights from a
 * weight matrix whose rows 2c and 2c + 1 are the gate row and the up row of
 * feature c (the caller interleaves them); y is bf16 [M, ldy], ldy >= N2 / 2.
 * Symmetric activation codes; no accumulator dump.  Other arguments, alignment
 * and kernel choice as resq_gemm_mixed.
 */
int resq_gemm_mixed_swiglu(const int8_t* q_hi, const uint8_t* q_lo, const float* s_hi,
                           const float* s_lo, const int32_t* lo_sum, int64_t M, const void* packed,
                           int64_t N2, int64_t K, int64_t r, void* y, int64_t ldy, void* stream);

/*
 * Offline construction of the projection basis (Section 4.2), three steps.
 *
 * 1. The covariance (Gram) matrix of calibration activations, accumulated over
 *    calls:  c[i][j] += sum_t x[t][i] x[t][j]   (fp32 accumulation of exact bf16
 *    products on the fp32 matrix cores; the caller zeroes c before the first
 *    call).  When the token axis is cut over workgroups their sums meet by
 *    atomic adds, so the last bits depend on the order of arrival.
 *      x   bf16 [T, ldx], ldx >= K        (read)    T = 0 does nothing
 *      c   fp32 [K, ldc], ldc >= K        (read and written)
 *    Alignment: x 16 bytes, ldx % 8 == 0, K % 8 == 0 (else RESQ_ERR_ALIGN).
 */
int resq_gram_accumulate(const void* x, int64_t ldx, int64_t T, int64_t K, float* c, int64_t ldc,
                         void* stream);

/*
 * 2. PCA: eigenvalues and eigenvectors of the symmetric matrix c (its symmetric
 *    part is taken), by cyclic Jacobi rotations in fp64.  eigvals[k] decrease
 *    with k and column k of p is the unit eigenvector of eigvals[k], so that the
 *    high-precision subspace P_h of Section 4.2 (largest eigenvalues) is the
 *    first r columns, as this library's column convention wants it (the paper
 *    orders them increasingly and keeps the last r).  Signs of the vectors, and
 *    bases inside a repeated eigenvalue, are whatever the rotations give.
 *      c        fp32 [K, ldc]                        (read)
 *      K        even, 2 .. 8192 (else RESQ_ERR_SHAPE; two fp64 rows sit in LDS)
 *      sweeps   Jacobi sweeps, 1 .. 64.  Convergence is quadratic at the end: 12
 *               sweeps bring every off-diagonal element of a K = 4096 covariance
 *               below 2^-40 of its diagonal neighbours.  The count is fixed so
 *               that the call never has to wait for the device; sweeps after one
 *               that found nothing to rotate are skipped (orders up to 128) or cost
 *               only their empty launches
 *      eigvals  fp32 [K]                             (written)
 *      p        fp32 [K, ldp], ldp >= K              (written)
 *               eigvals and p may lie on c's memory (c is lost then), not on each other's; orders
 *               up to 128 run in one launch on separate memory, and through the workspace in place
 *      workspace  device memory, 256-byte aligned, resq_sym_eig_workspace_bytes(K)
 *               bytes (else RESQ_ERR_BUFFER); contents meaningless afterwards
 */
size_t resq_sym_eig_workspace_bytes(int64_t K);
int resq_sym_eig(const float* c, int64_t ldc, int64_t K, int sweeps, float* eigvals, float* p,
                 int64_t ldp, void* workspace, size_t workspace_bytes, void* stream);

/*
 * resq_sym_eig for callers that cannot allocate device memory and have no workspace to pass
 * (code under HIP graph capture, serving loops and harnesses that forbid hipMalloc, a basis
 * refreshed between requests): the same kernels on the same arguments, with the workspace in
 * a device array that is part of the library (4.2 MB on every GPU the library has run this
 * call on, held until the process ends).  The call allocates and frees nothing.
 *   K   even, 2 .. 512 (head-size and small hidden-size bases); larger: RESQ_ERR_BUFFER,
 *       nothing is launched
 * Results are those of resq_sym_eig bit for bit.  Calls on one GPU that work on the array
 * (orders above 128, and any order with an output on c's memory) share the one array: those
 * that overlap (different streams or host threads) race, and its contents after a call are
 * meaningless (every call initializes what it reads).  Other calls do not touch it.
 * RESQ_ERR_HIP if the array's address cannot be obtained on the current device.
 */
int resq_sym_eig_static(const float* c, int64_t ldc, int64_t K, int sweeps, float* eigvals, float* p,
                        int64_t ldp, void* stream);

/*
 * 3. Rows expressed in a basis:  out[i][j] = sum_k a[i][k] u[k][j]  (exact
 *    products, fp32 accumulation: fp32 matrix cores for fp32 a and for K <= 16; else for bf16
 *    a the bf16 ones, u in three bf16 parts whose sum it is, up to what lies under 2^-133).
 *    Infinities and NaN go through as in a plain fp32 sum.  This one product serves every
 *    remaining step: U_h = P_h R_h and U_l = P_l R_l (the definition of U in
 *    Section 4.2: a = a column block of p, u = a random orthogonal matrix passed
 *    in by the caller, out = a column block of U), the folding of U into the
 *    weights W U (Section 4.3; W as [out_features, in_features]) and the
 *    projection X U of activations.
 *      a    bf16 or fp32 (a_is_bf16) [rows, lda], lda >= K      (read)
 *      u    fp32 [K, ldu], ldu >= J                             (read)
 *      out  bf16 (rounded to nearest even) or fp32 (out_is_bf16) [rows, ldo], ldo >= J
 *    Alignment: a, u 16 bytes; lda % 8 == 0, ldu % 8 == 0, J % 8 == 0.  rows = 0
 *    does nothing.
 */
int resq_project_rows(const void* a, int a_is_bf16, int64_t lda, int64_t rows, int64_t K,
                      const float* u, int64_t ldu, int64_t J, void* out, int out_is_bf16,
                      int64_t ldo, void* stream);

/*
 * Which kernel resq_project_rows runs for these arguments (addresses are compared, nothing is read):
 * host only, no device call.  For callers that want to know, and for tests.
 *   kernel  0: fp32 matrix cores
 *           1: bf16 matrix cores, 128 x 128 tiles
 *           2: bf16 matrix cores, 256 x 128 tiles, another order of the sum     (written)
 * Errors as resq_project_rows; RESQ_ERR_NULL for a null kernel.
 */
int resq_project_rows_plan(const void* a, int a_is_bf16, int64_t lda, int64_t rows, int64_t K,
                           const float* u, int64_t ldu, int64_t J, const void* out, int out_is_bf16,
                           int64_t ldo, int* kernel);

/*
 * The online projection of queries and keys onto the basis of the K/V cache
 * (Section 4.3: after the position embedding each head is multiplied by the
 * d_head x d_head matrix U_C, with 8-bit weights and 8-bit activations), as one
 * kernel: every row of x (one head of one token) is quantized to INT8 with its
 * own symmetric scale (Section 3 Eq. 1), multiplied by the INT8 codes of U_C
 * and dequantized (Section 4.1 Eq. 4 with every column in the high group).
 * The result equals resq_quantize_act followed by resq_gemm_mixed with
 * K = N = r = d_head; the activation codes never go to memory.
 *   x        bf16 [rows, ldx], ldx >= d_head                 (read)
 *   rows     tokens x heads; 0 is allowed and does nothing (no pointer is looked at)
 *   d_head   64 or 128 (else RESQ_ERR_SHAPE: use the two calls above)
 *   packed   resq_pack_weights of the [d_head, d_head] matrix whose row n is
 *            column n of U_C (the weight of output channel n), r = d_head
 *   y        bf16 [rows, ldy], ldy >= d_head                 (written)
 * Alignment: x 16 bytes and ldx % 8 == 0 (else RESQ_ERR_ALIGN); packed 256
 * bytes; y 2 bytes (rows aligned to d_head / 8 bytes are written with wider stores).
 */
int resq_project_heads(const void* x, int64_t ldx, int64_t rows, int64_t d_head, const void* packed,
                       void* y, int64_t ldy, void* stream);

/*
 * The layer for asymmetric activation codes (resq_quantize_act_asym): inserting
 * x ~ stored * s + c (Section 3 Eq. 1) and w ~ code * sw into Section 4.1 Eq. 4
 * gives, per group,
 *   y[m, n] += sw[n] * ( s[m] * A[m, n] + c[m] * wsum[n] ),
 * A the integer sum over the stored codes (what dbg_acc_* receive) and wsum[n]
 * the sum of channel n's weight codes of that group, which resq_pack_weights
 * keeps in the packed buffer.  Same kernels as resq_gemm_mixed plus one
 * multiply-add per group in the epilogue; all other arguments as there.
 */
int resq_gemm_mixed_asym(const int8_t* q_hi, const uint8_t* q_lo, const float* s_hi,
                         const float* s_lo, const float* c_hi, const float* c_lo,
                         const int32_t* lo_sum, int64_t M, const void* packed, int64_t N, int64_t K,
                         int64_t r, void* y, int64_t ldy, int32_t* dbg_acc_hi, int32_t* dbg_acc_lo,
                         void* stream);

/*
 * Mixed-precision K/V cache entries (Section 5.1 and Appendix C: keys and values are
 * quantized per head with the asymmetric quantizer of Section 3, Eq. 1, an eighth of the
 * channels of a head in 8 bits, the rest in 4), in a compact row per head of a token:
 *   bytes [0, r)                      8-bit codes 0..255 of channels [0, r)
 *   bytes [r, r + (d_head - r) / 2)   4-bit codes 0..15: channel r + 2j in bits 0..3 of
 *                                     byte j, channel r + 2j + 1 in bits 4..7
 *   then fp32 s_hi, z_hi, s_lo, z_lo  scale and zero-point of both groups: a reader
 *                                     reconstructs x ~ code * s + z (a group without
 *                                     channels has s = 1, z = 0)
 * resq_kv_cache_row_bytes = r + (d_head - r) / 2 + 16 (88 bytes for d_head = 128, r = 16,
 * against 256 bytes of bf16), or 0 for an invalid pair.  Codes, scales and zero-points are
 * those of resq_quantize_act_asym on rows of d_head columns (z = min, s = (max - min) /
 * (2^N - 1), round half to even), stored here as Eq. 1 defines them.
 *   x       bf16 [rows, ldx], ldx >= d_head; one row per token and head       (read / written)
 *   cache   [rows, row_bytes] bytes, row_bytes >= resq_kv_cache_row_bytes     (written / read)
 *   d_head  multiple of 8, 8 .. 512; r multiple of 8, 0 .. d_head (else RESQ_ERR_SHAPE);
 *           rows = 0 does nothing
 * resq_dequantize_kv_cache is the reader: x[m, k] = bf16(code * s + z), the multiply-add in
 * fp32.  Errors: RESQ_ERR_BUFFER for a row_bytes too small; RESQ_ERR_ALIGN unless x is
 * 16-byte aligned, ldx % 8 == 0, cache 4-byte aligned and row_bytes % 4 == 0.
 */
size_t resq_kv_cache_row_bytes(int64_t d_head, int64_t r);
int resq_quantize_kv_cache(const void* x, int64_t ldx, int64_t rows, int64_t d_head, int64_t r, void* cache,
                           int64_t row_bytes, void* stream);
int resq_dequantize_kv_cache(const void* cache, int64_t row_bytes, int64_t rows, int64_t d_head, int64_t r,
                             void* x, int64_t ldx, void* stream);

/*
 * ---- the generation step between the query/key/value projections and the output projection -------------------------------
 * The K/V cache in PAGES: a page holds page_size rows of compact entries (resq_quantize_kv_cache's rows) for each K/V head, keys
 * and values in two arrays alike in shape.  The row of head h in row i of page p is at byte
 *   p * page_stride + h * head_stride + i * row_stride
 * of its array (strides in bytes, multiples of 4, each at least resq_kv_cache_row_bytes; an axis of one entry has no stride;
 * rows do not overlap).  In pages r may also be an odd multiple of 4 below d_head <= 256: rows of r + (d_head - r) / 2 + 16 bytes
 * in the same order, addresses and strides multiples of 2.  A SLOT is p * page_size + i, num_pages * page_size <= 2^31 - 1.  A row of the BLOCK TABLE names the
 * pages of a sequence in order: its token t is in row t % page_size of page block_table[b][t / page_size].  Any strides do for the
 * attention; it reads fastest where page_size is a multiple of 16 and row_stride below 2^26.
 * Common to these calls: lengths, positions, slots and table entries are int32 (4-byte aligned); head vectors are bf16 with a
 * stride from token to token and one from head to head in elements (strides of inputs may be 0).  Calls of more rows than a launch
 * can count (about 2^26 of 512 channels, 2^28 of 128) are refused with RESQ_ERR_SHAPE.  resq_time_next_kernel times a call's first
 * kernel.
 *
 * The plan of a step, on the GPU: request b has lens[b] tokens in its pages and gets new_tokens[b] more (0 is fine).
 * Its new tokens follow those of the requests before it in the batch; pages that it lacks are taken off the front of the free
 * list, in the order of the requests, and entered into its row of the block table.
 *   lens, new_tokens   int32 [B]; B <= 65536                                             (read)
 *   free_pages         int32 [n_free] pages to hand out; taken: int32 [1], how many of them are gone already  (read)
 *   block_table        int32 [B, ld_table], `width` entries used of each row, width * page_size <= 2^31 - 1   (entries of new pages written)
 *   lens_out           int32 [B]: lens + new_tokens; may be lens                         (written)
 *   cu_tokens, cu_pages  int32 [B + 1]: new tokens, and new pages, of the requests before b        (written)
 *   positions, slots   int32 [max_tokens]: of each new token; behind the last one 0 and -1          (written)
 *   state              int32 [2]: entries of free_pages gone after the call (taken may be this one), and a status:
 *                      0: done; 1: too few free pages; 2: a table row too narrow; 3: more than max_tokens new tokens;
 *                      4: a negative length, count or taken (the highest that applies).  Unless it is 0 nothing is handed out:
 *                      lens_out = lens, the sums are 0, every slot is -1, the block table is as it was  (written)
 * A token whose page (from the table or the free list) is outside [0, num_pages) gets slot -1.  max_tokens <= 2^31 - 257.
 * The arrays do not overlap except as said.
 */
int resq_kv_slots(const int32_t* lens, const int32_t* new_tokens, int64_t B, int64_t page_size, int64_t num_pages,
                  const int32_t* free_pages, int64_t n_free, const int32_t* taken, int32_t* block_table, int64_t ld_table,
                  int64_t width, int64_t max_tokens, int32_t* lens_out, int32_t* cu_tokens, int32_t* cu_pages,
                  int32_t* positions, int32_t* slots, int32_t* state, void* stream);

/*
 * The frequencies of a rotary position embedding, on the HOST (no device call): radians per position of each pair of channels,
 * base^(-2i/rot), as they are or stretched for contexts longer than the original one.
 *   scaling  RESQ_ROPE_PLAIN   as they are
 *            RESQ_ROPE_LINEAR  all divided by factor
 *            RESQ_ROPE_BASE    base * factor^(rot / (rot - 2)) for base: the fastest as it is, the slowest divided by factor
 *            RESQ_ROPE_BANDS   pairs that make more than `high` turns over original_len as they are, those with fewer than `low`
 *                              divided by factor, a share of both between
 *            RESQ_ROPE_RAMP    the same with the share linear in the pair's number (YaRN, arXiv 2309.00071), and
 *                              *mscale = 0.1 ln(factor) + 1
 *   rot      even, 2 .. 512; base > 1; factor >= 1 and 0 < low < high, original_len >= 1 where they are used
 *   freq     HOST, double [rot / 2];  mscale  HOST, one float: what resq_rope_heads multiplies rotated channels by   (written)
 */
enum { RESQ_ROPE_PLAIN = 0, RESQ_ROPE_LINEAR = 1, RESQ_ROPE_BASE = 2, RESQ_ROPE_BANDS = 3, RESQ_ROPE_RAMP = 4 };
int resq_rope_frequencies(int64_t rot, double base, int scaling, double factor, double low, double high, int64_t original_len,
                          double* freq, float* mscale);

/*
 * The position embedding of query and key heads, in front of resq_project_heads (Section 4.3 projects them after it), with the
 * norm of each head in the same pass for models that have one:
 *   n = x * rsqrt(mean(x^2) + eps) * w   (w: w_q for heads [0, heads_q), w_k for the others; both null: n = x)
 *   y = n with each pair (a, b) of its first rot channels turned to mscale * (a cos - b sin, b cos + a sin) by the angle
 *       positions[token] * freq[pair]; pair i is channels (i, i + rot/2), or (2i, 2i + 1) where `interleaved` is not 0
 * in fp32 with one rounding to bf16 at the end; the angle is taken modulo a turn in pairs of fp64 numbers, before it is rounded to fp32,
 * so that it is as exact at position 2^31 - 1 as at 1.  Channels [rot, d_head) are n alone.
 *   x, y     bf16 [tokens, heads_q + heads_k, d_head] with strides (ldx, ldxh), (ldy, ldyh); y may be x with the same strides,
 *            else they do not overlap                                                    (read / written)
 *   d_head   even, 2 .. 512; rot even, 0 .. d_head (positions and freq may be null for 0); tokens = 0 does nothing
 *   w_q, w_k bf16 [d_head] or both null; eps >= 0                                        (read)
 *   positions int32 [tokens]; freq fp64 [rot / 2], 8-byte aligned, in DEVICE memory      (read)
 * Alignment: 2 bytes; rows of whole 16-byte pieces (x, y 16-byte aligned, strides and d_head multiples of 8, rot a multiple of
 * 16 unless interleaved) are the fastest.
 */
int resq_rope_heads(const void* x, int64_t ldx, int64_t ldxh, int64_t tokens, int64_t heads_q, int64_t heads_k, int64_t d_head,
                    const void* w_q, const void* w_k, float eps, const int32_t* positions, const double* freq, int64_t rot,
                    int interleaved, float mscale, void* y, int64_t ldy, int64_t ldyh, void* stream);

/*
 * The paged writer: K and V of new tokens, quantized as by resq_quantize_kv_cache (the same bytes), straight to their slots.
 *   k, v     bf16 [tokens, heads, d_head] with strides (ldk, ldkh), (ldv, ldvh)           (read)
 *   slots    int32 [tokens]; tokens whose slot is outside [0, num_pages * page_size) are left out; the others' slots differ
 *            from one another (a slot named twice is left with bytes of both tokens)      (read)
 *   k_pages, v_pages   the pages (above)                                                  (rows of the slots written, nothing else)
 *   d_head, r as resq_quantize_kv_cache, or r as said above; tokens = 0 does nothing
 * Errors: RESQ_ERR_BUFFER for strides below the row; RESQ_ERR_ALIGN unless k and v are 16-byte aligned, their strides multiples
 * of 8, the pages 4-byte aligned and their strides multiples of 4 (2 and 2 where r is no multiple of 8).
 *
 * resq_gather_kv_cache is the paged reader: the values of the tokens in `slots` (any order, repeats are fine) as
 * resq_dequantize_kv_cache gives them, zeros for slots outside the pages.  k and v are written, their rows do not overlap.
 */
int resq_append_kv_cache(const void* k, int64_t ldk, int64_t ldkh, const void* v, int64_t ldv, int64_t ldvh, int64_t tokens,
                         int64_t heads, int64_t d_head, int64_t r, const int32_t* slots, void* k_pages, void* v_pages,
                         int64_t num_pages, int64_t page_size, int64_t page_stride, int64_t head_stride, int64_t row_stride,
                         void* stream);
int resq_gather_kv_cache(const void* k_pages, const void* v_pages, int64_t num_pages, int64_t page_size, int64_t page_stride,
                         int64_t head_stride, int64_t row_stride, const int32_t* slots, int64_t tokens, int64_t heads,
                         int64_t d_head, int64_t r, void* k, int64_t ldk, int64_t ldkh, void* v, int64_t ldv, int64_t ldvh,
                         void* stream);

/*
 * Attention of one new token of each sequence over its pages (the new token's own K and V are there already, as its last row),
 * queries in 16 bits (Section 5.1), the K/V rows as they stand for: k = code * s + z, not rounded.  For query head h, K/V head
 * h / (heads_q / heads_k), over the tokens t < len:
 *   x_t = scale * q . k_t;  softcap > 0: softcap * tanh(x_t / softcap);  window > 0: only the last `window` tokens
 *   out = sum_t e^(x_t - lse) v_t (rounded to bf16 once),  lse = ln sum_t e^(x_t)
 * Tokens whose table entry is outside [0, num_pages) take no part.  Where none is left (an empty sequence) out is 0 and lse -inf.
 *   q, out   bf16 [B, heads_q, d_head] with strides (ldq, ldqh), (ldo, ldoh); rows of out do not overlap, out may be q with the
 *            same strides                                                                 (read / written)
 *   lens     int32 [B]; what is above width * page_size (or 2^30) is read as that, what is below 0 as 0     (read)
 *   block_table  int32 [B, ld_table], `width` entries used of each row                    (read)
 *   lse      fp32 [B, heads_q] or null                                                    (written)
 *   d_head   multiple of 8, 8 .. 256; r as for the writer; heads_q a multiple of heads_k; B, heads_q <= 65535
 *   scale    > 0; softcap 0 (none) or a normal number above; window >= 0 (0: none)
 *   B * heads_q < 2^24, and B * heads_k * ceil(heads_q / heads_k / 16) * (ceil(width * page_size / 128) + 3) < 2^31
 *   workspace  device memory, 256-byte aligned, resq_attend_kv_cache_workspace_bytes bytes (else RESQ_ERR_BUFFER); contents
 *            meaningless before and after; calls that overlap (different streams) need one each
 * The work is cut by the lengths that the GPU finds, so that a captured call serves any lengths.  The cuts, and with them the
 * order of fp32 sums, depend on all lengths of the call, not on timing: equal calls give equal bits.
 */
size_t resq_attend_kv_cache_workspace_bytes(int64_t B, int64_t heads_q, int64_t heads_k, int64_t d_head);
int resq_attend_kv_cache(const void* q, int64_t ldq, int64_t ldqh, int64_t B, int64_t heads_q, int64_t heads_k, int64_t d_head,
                         int64_t r, const int32_t* lens, const int32_t* block_table, int64_t ld_table, int64_t width,
                         const void* k_pages, const void* v_pages, int64_t num_pages, int64_t page_size, int64_t page_stride,
                         int64_t head_stride, int64_t row_stride, float scale, float softcap, int64_t window, void* out,
                         int64_t ldo, int64_t ldoh, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Attention over whole prompts: causal, sequences packed one after the other, on top of cached tokens or not.  Sequence b has
 * the queries cu_q[b] .. cu_q[b + 1] - 1 and the keys cu_k[b] .. cu_k[b + 1] - 1; its queries are the last ones of its keys' tokens (nk keys, nq
 * queries: query i stands at own = i + nk - nq).  For query head h, K/V head h / (heads_q / heads_k), over the keys j <= own:
 *   x_j = scale * q . k_j;  softcap > 0: softcap * tanh(x_j / softcap);  window > 0: only the last `window` keys, j > own - window
 *   out = sum_j e^(x_j - lse) v_j (rounded to bf16 once),  lse = ln sum_j e^(x_j)
 * Weights go into the products rounded to bf16 (off by 2^-8 of each at most), sums are fp32.  Where a query sees no key (more queries than keys) out is 0
 * and lse -inf.  What a query does not see has no part in its result, infinities and NaN neither.  (Infinities in a query or in
 * keys that it sees may make NaN of its result.)
 *   q, out   bf16 [tokens_q, heads_q, d_head] with strides (ldq, ldqh), (ldo, ldoh); rows of out do not overlap, out may be q with the
 *            same strides, else it lies on no other tensor of the call; rows outside of the sequences are left as they were  (read / written)
 *   k, v     bf16 [tokens_k, heads_k, d_head] with strides (ldk, ldkh), (ldv, ldvh): views of a projection's output, or what
 *            resq_gather_kv_cache wrote                                                  (read)
 *   cu_q, cu_k  int32 [B + 1], not decreasing, from resq_kv_slots' cu_tokens; may be one array.  What is below 0 or above tokens_q
 *            (tokens_k) is read as that; results of arrays that decrease are unspecified (no access leaves the tensors)  (read)
 *   lse      fp32 [tokens_q, heads_q] or null                                            (written)
 *   d_head   multiple of 8, 8 .. 256; heads_q a multiple of heads_k; 1 <= B <= 65535; tokens_q = 0 does nothing
 *   scale, softcap, window   as resq_attend_kv_cache; a capped score is off by 2^-19.9 of itself at most beside what it was before
 *   tokens_q, tokens_k <= 2^30, tokens_q * heads_q + 255 B heads_k < 2^31, the first of both < 2^31 - 65536; ldk, ldv < 2^24 (of one key: any)
 *   workspace  device memory, 256-byte aligned, resq_attend_prompts_workspace_bytes bytes (else RESQ_ERR_BUFFER); contents
 *            meaningless before and after; calls that overlap (different streams) need one each
 * Alignment: k and v 16 bytes, their strides multiples of 8 (else RESQ_ERR_ALIGN); the others their elements'.
 * How the keys of few queries are cut into parts depends on the sizes alone: equal calls give equal bits.
 */
size_t resq_attend_prompts_workspace_bytes(int64_t tokens_q, int64_t tokens_k, int64_t B, int64_t heads_q, int64_t heads_k, int64_t d_head);
int resq_attend_prompts(const void* q, int64_t ldq, int64_t ldqh, int64_t tokens_q, const void* k, int64_t ldk, int64_t ldkh, const void* v,
                        int64_t ldv, int64_t ldvh, int64_t tokens_k, const int32_t* cu_q, const int32_t* cu_k, int64_t B, int64_t heads_q,
                        int64_t heads_k, int64_t d_head, float scale, float softcap, int64_t window, void* out, int64_t ldo, int64_t ldoh,
                        float* lse, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Attention of one new token of each sequence, as resq_attend_kv_cache, behind a PREFIX that all sequences of the batch share (the
 * instructions in front of every request, the question that many answers are tried for): the tokens of sequence b are the
 * prefix's, then lens[b] of its own (its new token the last of them).  The prefix is read and made into numbers once for 256 queries
 * of a K/V head instead of once for each sequence; results are those of resq_attend_kv_cache on tables that name both in a row, but for the
 * roundings below (there codes are multiplied as they are).
 *   prefix_len    int32 [1]: tokens of the prefix; what is above prefix_width * page_size (or 2^30) is read as that, below 0 as 0  (read)
 *   prefix_table  int32 [prefix_width]: its pages                                        (read)
 *   lens          int32 [B]: own tokens; 0: the prefix alone; below 0: the sequence is not there, its out is 0 and its lse -inf  (read)
 *   block_table   the own tokens' pages; own tokens begin with a page of their own        (read)
 *   window        counts own tokens first
 *   workspace     resq_attend_kv_prefix_workspace_bytes bytes
 * Everything else as resq_attend_kv_cache, capped scores of the prefix as in resq_attend_prompts.  Rows of the prefix go into the products as fp16 numbers, k as two of them: k is off by 2^-22 of
 * itself at most, v by 2^-11, both or by 2^-38 of the largest number among those of a tile of 64 tokens (v: among all so far); weights by
 * 2^-11 of themselves or 2^-35 of the row's largest one.  A value of the prefix that is not finite makes the channels of its group (of r
 * or of the others) NaN in every row that sees it, and does nothing in others.
 * How the prefix is cut into parts depends on the sizes and its length alone, for the own tokens see above: equal calls give equal bits.
 */
size_t resq_attend_kv_prefix_workspace_bytes(int64_t B, int64_t heads_q, int64_t heads_k, int64_t d_head);
int resq_attend_kv_prefix(const void* q, int64_t ldq, int64_t ldqh, int64_t B, int64_t heads_q, int64_t heads_k, int64_t d_head, int64_t r,
                          const int32_t* prefix_len, const int32_t* prefix_table, int64_t prefix_width, const int32_t* lens,
                          const int32_t* block_table, int64_t ld_table, int64_t width, const void* k_pages, const void* v_pages,
                          int64_t num_pages, int64_t page_size, int64_t page_stride, int64_t head_stride, int64_t row_stride, float scale,
                          float softcap, int64_t window, void* out, int64_t ldo, int64_t ldoh, float* lse, void* workspace,
                          size_t workspace_bytes, void* stream);

/*
 * What stands between two blocks of a layer, in one pass: the norm behind the block, its gate, the residual scale and sum, and the
 * norm in front of the next block (whose output resq_quantize_act takes):
 *   a  = y * rsqrt(mean(y^2) + eps) * (w_offset + w_post)   (w_post null: a = y;  y null: a = 0, what a first block needs)
 *   h' = h + alpha * gate * a                               (gate null: 1)
 *   x  = h' * rsqrt(mean(h'^2) + eps) * (w_offset + w_pre)
 * in fp32 with one rounding of each output; x comes from h' as it was before its rounding.  (Squares are fp32 numbers too: what is above 1.8e19
 * in a row has none.)
 *   y, gate, x  bf16 [tokens, width] with strides ldy, ldg, ldx (ldg 0: one gate for all tokens)   (read / read / written)
 *   h, h_out  bf16, or fp32 (h_is_fp32), [tokens, width] with strides ldh, ldho          (read / written)
 *            h_out may be h and x may be y, with the same strides; else outputs lie on no other tensor of the call, and rows of
 *            an output do not overlap.  h_out or x may be null (not both): not written, w_pre is not read without x
 *   w_pre, w_post  bf16 [width]; w_offset 0, or 1 for weights that are stored as their distance from 1             (read)
 *   width    1 .. 32768; tokens < 2^22 (more of narrow rows), 0 does nothing; eps >= 0; w_offset, alpha finite; gate and w_post need y
 * Alignment: that of the elements; rows of whole 16-byte pieces are the fastest.
 */
int resq_norm_residual(const void* y, int64_t ldy, const void* gate, int64_t ldg, const void* h, int64_t ldh, int h_is_fp32, int64_t tokens,
                       int64_t width, const void* w_pre, const void* w_post, float w_offset, float eps, float alpha, void* h_out,
                       int64_t ldho, void* x, int64_t ldx, void* stream);

/*
 * Online Hadamard projection of the down_proj input (Section 4.3, U_D):
 *   y[m, c0 + g*b + j] = (1/sqrt(b)) * sum_i x[m, c0 + g*b + i] * H_b[i, j]
 * for each block g of b columns in [col_begin, col_end), H_b the Sylvester
 * (natural-order) Hadamard matrix; other columns are copied.  fp32 butterflies,
 * bf16 in and out; y may alias x (in place).
 *   x, y   bf16 [M, ld], ld >= K
 *   block  power of two dividing col_end - col_begin, <= 8192;
 *          0 selects resq_hadamard_block(col_end - col_begin)
 * Errors: RESQ_ERR_ALIGN unless x and y are 16-byte aligned and ld, col_begin and
 * col_end - col_begin are multiples of 8 (rows are moved 16 bytes per lane).
 */
int resq_online_hadamard(const void* x, void* y, int64_t ld, int64_t M, int64_t K,
                         int64_t col_begin, int64_t col_end, int64_t block, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* RESQ_H */
