/*
 * heal.h -- C ABI of libheal.so: the bf16x3 algebraically compensated GEMM
 * for AMD Instinct MI355X (gfx950).
 *
 * The method (HEAL, Section 4 "Hybrid Error ALleviation", paragraph on GEMM
 * truncation, and its displayed expansion of GEMM(h, W^T) into 16-bit
 * products summed into an FP32 output) keeps a GEMM on 16-bit matrix units
 * while recovering the significand bits a single 16-bit cast would lose.
 * Here both FP32 operands are split into bfloat16 pairs
 *     hi = RNE_bf16(x),  lo = RNE_bf16(x - hi)
 * and the product is
 *     C = hiA*hiB + hiA*loB + loA*hiB
 * accumulated in FP32 by bf16 MFMA instructions and written as FP32 (the
 * output is never rounded to 16 bits: Appendix "HEAL Implementation", HEAL-Base
 * and HEAL-Full keep GEMM outputs in FP32).
 *
 * Reduction order.  For every output element the sum runs over K in 32-deep
 * chunks, k ascending, each chunk adding its three products into one FP32
 * accumulator in the order hiA*hiB, hiA*loB, loA*hiB; the K tail is padded
 * with zeros.  No product splits K across workgroups, nothing uses atomics, and
 * every kernel instance follows this order, so results are bitwise identical
 * run to run, for every M (a row's bits do not depend on the other rows), for
 * every N, and between the plain and batched entry points.
 *
 * Conventions for every entry point:
 *   - matrices are row-major FP32 with leading dimensions in ELEMENTS:
 *     A[i*lda + k], B[k*ldb + j] (or B[j*ldb + k] when transposed), C[i*ldc + j];
 *   - all pointers are DEVICE pointers owned by the caller; the library never
 *     allocates, frees or keeps device memory and holds no state beyond a
 *     per-device architecture check, so calls are thread-safe;
 *   - work is enqueued asynchronously on `stream` (0 = the null stream); the
 *     result is visible after the caller synchronises that stream;
 *   - C is write-only (beta = 0): its previous contents never matter; C must
 *     not overlap A or B (A and B may alias each other);
 *   - any 4-byte-aligned pointer and any leading dimension are accepted; the
 *     widest loads are used when alignment allows, and the result bits never
 *     depend on which load path ran;
 *   - a product whose output holds more than 2^21 blocks of 16 x 16 elements
 *     (over all its batch entries) is enqueued as several kernel launches,
 *     each on a range of batch entries, rows and columns, because a dispatch
 *     counts its work-items in 32 bits; the bits are those of one launch.
 * Errors: arguments are validated before any HIP call, so an invalid call
 * returns HEAL_ERR_INVALID_VALUE without touching the device.  The library
 * never aborts and never prints.
 */
#ifndef HEAL_H
#define HEAL_H

#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum heal_status_t {
    HEAL_OK = 0,
    HEAL_ERR_INVALID_VALUE = 1,      /* bad size, leading dimension, pointer or flag */
    HEAL_ERR_UNSUPPORTED_DEVICE = 2, /* the current device is not gfx950 */
    HEAL_ERR_LAUNCH = 3              /* a HIP call or kernel launch failed */
} heal_status_t;

/* Human-readable name of a status code (a static string; never NULL). */
const char *heal_status_string(heal_status_t status);

/* Library version as 10000*major + 100*minor + patch. */
int heal_version(void);

/* Identity of the sources this library was built from: 16 hex digits of a
 * SHA-256 over the kernel sources, this header and the compiler flags (a
 * static string; "unknown" if the build did not supply it).  A caller can
 * compare it with the same hash of the sources it expects, to refuse a stale
 * binary. */
const char *heal_build_id(void);

/*
 * heal_split_f32 -- the operand decomposition on its own (Section 4, GEMM
 * paragraph: the FP32 input is decomposed into a 16-bit head and residual).
 *   x   : n FP32 values (device, read-only).
 *   hi  : n bf16 bit patterns, hi[i] = RNE_bf16(x[i]) (device, written).
 *   lo  : n bf16 bit patterns, lo[i] = RNE_bf16(x[i] - hi[i]) evaluated in
 *         IEEE arithmetic (device, written).
 *   n   : number of elements, n >= 0 (n == 0 is a no-op).
 * The subtraction x - hi is exact, so |x - hi - lo| <= 2^-17 |x| for every
 * finite x with 2^-117 <= |x| that does not round to infinity; below 2^-117
 * lo can fall into bf16's subnormal range (step 2^-133) and the error is at
 * most 2^-134 in absolute terms.  hi and lo must not overlap x or each
 * other.  Non-finite inputs follow IEEE arithmetic: x = +/-inf gives
 * hi = x and lo = NaN; a finite x that rounds to infinity gives lo = -/+inf;
 * x = NaN gives NaN for both (payloads unspecified).  Any output of the GEMM
 * that such an element reaches is therefore NaN.
 */
heal_status_t heal_split_f32(const float *x, uint16_t *hi, uint16_t *lo, int64_t n,
                             hipStream_t stream);

/*
 * heal_gemm_f32 -- C = A * B with the compensated bf16x3 product (Section 4,
 * displayed GEMM expansion; FP32 accumulation and output).
 *   M, N, K : sizes, each >= 0.  M == 0 or N == 0 is a no-op; K == 0 writes +0.
 *   A       : M x K, row stride lda >= max(K, 1).
 *   B       : K x N, row stride ldb >= max(N, 1).
 *   C       : M x N, row stride ldc >= max(N, 1); written, never read.
 */
heal_status_t heal_gemm_f32(int64_t M, int64_t N, int64_t K,
                            const float *A, const float *B, float *C,
                            int64_t lda, int64_t ldb, int64_t ldc, hipStream_t stream);

/*
 * heal_gemm_f32_strided_batched -- batch independent products
 *     C_b = alpha * (A_b * op(B_b)),  b = 0 .. batch-1,
 * with A_b = A + b*strideA, B_b = B + b*strideB, C_b = C + b*strideC.
 *   trans_b = 0 : op(B) = B, B_b is K x N with row stride ldb >= max(N, 1);
 *   trans_b = 1 : op(B) = B^T, B_b is stored N x K (an nn.Linear weight, or
 *                 the keys of an attention score product) with row stride
 *                 ldb >= max(K, 1).
 *   alpha   : FP32 scale applied once to the FP32 accumulator in the epilogue
 *             (the attention 1/sqrt(d) scale), never folded into the inputs.
 *   strides : in elements, >= 0 (0 reuses the same matrix for every entry).
 *   batch   : >= 0.
 * With alpha == 1, trans_b == 0 and batch == 1 the result is bitwise equal to
 * heal_gemm_f32; with trans_b == 1 it is bitwise equal to trans_b == 0 on the
 * explicitly transposed B.
 */
heal_status_t heal_gemm_f32_strided_batched(int64_t M, int64_t N, int64_t K, float alpha,
                                            const float *A, int64_t lda, int64_t strideA,
                                            const float *B, int64_t ldb, int64_t strideB,
                                            int trans_b,
                                            float *C, int64_t ldc, int64_t strideC,
                                            int64_t batch, hipStream_t stream);

/*
 * Kernel instances.  heal_gemm_f32_instance forces one, for tests of
 * cross-instance bitwise equality and for tuning; every instance computes the
 * same bits.
 *   instance : one of heal_instance_t; HEAL_INSTANCE_AUTO chooses as usual, by
 *   sizes, layout and alignment, between these and two more kernels: the panel
 *   kernel for B stored N x K with K <= 128 (attention scores: bf16x3 with
 *   trans_b = 1, which the large and medium instances take too from 256 rows on
 *   where rows of C are whole 16-byte units, and the INT16 scores), where a panel
 *   of A stays in LDS while the workgroup walks the columns of C; and the direct-B
 *   kernel, whose smaller tiles fill the chip where the output has too few large
 *   ones.
 * Other arguments as heal_gemm_f32_strided_batched.
 */
typedef enum heal_instance_t {
    HEAL_INSTANCE_AUTO = 0,
    HEAL_INSTANCE_LARGE = 1,   /* 256 x 256 output tiles (the FP16 and pre-split
                                  products take 256 x 224 where that needs fewer
                                  rounds of workgroups; INT16 scores 128 x 256),
                                  compute-bound shapes */
    HEAL_INSTANCE_MEDIUM = 2,  /* 128 x 128 output tiles */
    HEAL_INSTANCE_SKINNY = 3,  /* M <= 64: decode and lm_head shapes, B streamed */
    HEAL_INSTANCE_COUNT = 4
} heal_instance_t;

heal_status_t heal_gemm_f32_instance(int instance, int64_t M, int64_t N, int64_t K, float alpha,
                                     const float *A, int64_t lda, int64_t strideA,
                                     const float *B, int64_t ldb, int64_t strideB,
                                     int trans_b,
                                     float *C, int64_t ldc, int64_t strideC,
                                     int64_t batch, hipStream_t stream);

/* The instance heal_gemm_f32 would choose for an M x N output by its size, where
 * neither the panel nor the direct-B kernel takes the product (no HIP call). */
int heal_gemm_select_instance(int64_t M, int64_t N);

/* The tile of the direct-B kernel, as 1000 * rows + columns, that a product of
 * dense, 16-byte aligned operands takes by itself, or 0 where another kernel
 * runs it: kind 0 HEAL-Base, 1 HEAL-Full, 3 pre-split, 4 bf16x3 (trans_b as in
 * heal_gemm_f32_strided_batched; the panel kernel is not considered).  For the
 * labels of measurements. */
int heal_gemm_direct_tile(int kind, int trans_b, int64_t M, int64_t N, int64_t K, int64_t batch);

/* ==========================================================================
 * FP16 forms of the method (HEAL-Base and HEAL-Full), the pre-split B
 * operand, and the INT16 Q/K score product (HEAL+).
 *
 * Packed operands.  A weight or B operand used many times is converted once
 * into a packed layout in MFMA fragment order: for each block of 16 columns
 * n (jb = n / 16) and 32-deep chunk of k (kc = k / 32), each plane p holds
 * 512 16-bit values at
 *     packed[((jb * KC + kc) * P + p) * 512 + lane * 8 + t],
 *     lane = (n % 16) + 16 * ((k % 32) / 8),  t = k % 8,  KC = ceil(K / 32),
 * positions beyond K or N holding +0.  heal_packed_size gives the number of
 * uint16 values (ceil(N/16) * KC * P * 512); the buffer must be 16-byte
 * aligned.  K is limited to 2^20 for packed operands.
 * ========================================================================== */

/*
 * heal_split_f16 -- the HEAL-Full activation pair on its own (Section 4, GEMM
 * paragraph: an FP32 activation h becomes h_hi + h_lo / 2^10 in FP16).
 *   hi[i] = RNE_f16(x[i]),  lo[i] = RNE_f16((x[i] - hi[i]) * 2^10),
 * as binary16 bit patterns, x - hi and the 2^10 shift exact in FP32.  For
 * finite |x| < 65520, |x - hi - lo / 2^10| <= 2^-22 |x| + 2^-35.  |x| >= 65520
 * gives hi = +/-inf and lo = -/+inf; x = +/-inf gives lo = NaN; NaN gives NaN.
 * Arguments as heal_split_f32.
 */
heal_status_t heal_split_f16(const float *x, uint16_t *hi, uint16_t *lo, int64_t n,
                             hipStream_t stream);

/* Number of uint16 values of a packed K x N operand with `planes` planes (1 or
 * 2), or -1 for invalid sizes (no HIP call). */
int64_t heal_packed_size(int64_t K, int64_t N, int planes);

/*
 * heal_maxabs_f32 -- max|x| over a rows x cols row-major FP32 matrix (row
 * stride ld >= max(cols, 1)), written as one float to *maxabs (device).  An
 * empty matrix gives +0.  A NaN element makes the result a NaN pattern.
 */
heal_status_t heal_maxabs_f32(const float *x, int64_t rows, int64_t cols, int64_t ld,
                              float *maxabs, hipStream_t stream);

/*
 * heal_f16_weight_exponent -- the per-matrix power-of-two weight scale
 * (Appendix "HEAL Implementation", HEAL-Base: weights are scaled by a power of
 * two before the FP16 GEMM and the output is scaled back).  *e (host) becomes
 * the largest integer with maxabs * 2^e <= 65504, so the scaled weights use
 * the top of the FP16 range and none overflows; maxabs == 0 gives e = 0.
 * maxabs is a host value (for example read back from heal_maxabs_f32); it must
 * be finite and >= 0.  No HIP call.
 */
heal_status_t heal_f16_weight_exponent(float maxabs, int32_t *e);

/*
 * heal_pack_f16_weight -- W16 = packed RNE_f16(W * 2^e), one plane, for the
 * FP16 GEMMs.  W is the FP32 weight of a linear layer, N x K row-major (row
 * stride ldw >= max(K, 1)), so the GEMM computes A * W^T.  |e| <= 300.  W16
 * holds heal_packed_size(K, N, 1) values.
 */
heal_status_t heal_pack_f16_weight(const float *W, int64_t N, int64_t K, int64_t ldw, int32_t e,
                                   uint16_t *W16, hipStream_t stream);

/*
 * heal_gemm_f16w -- FP16 GEMM with FP32 activations and FP32 output:
 *   products == 1 (HEAL-Base):  C = 2^-e * sum_k f16(a) w16
 *   products == 2 (HEAL-Full, Section 4 two-product expansion
 *       GEMM(h_hi, W) + GEMM(h_lo / 2^10, W)):
 *       C = 2^-e * sum_k (h_hi w16 + h_lo f16(w16 2^-10)),
 *       with (h_hi, h_lo) as heal_split_f16.  Both products go into ONE FP32
 *       accumulator, per 32-deep chunk the head product and then the
 *       residual product, and the residual's 2^-10 is applied to the FP16
 *       weight fragment.  w16 2^-10 is exact for |w16| >= 2^-4, that is for
 *       every weight above 2^-20 of the largest (the scaled weights reach
 *       2^15); a smaller weight's w16 2^-10 is rounded to FP16's subnormal
 *       step 2^-24, which moves its residual term by at most
 *       2^-25 |h_lo| <= 2^-26 |h| (before the 2^-e scale).
 *   A   : M x K FP32, row stride lda >= max(K, 1);
 *   W16 : packed FP16 weight from heal_pack_f16_weight (same N, K, e);
 *   C   : M x N FP32, row stride ldc >= max(N, 1); written, never read.
 * Reduction order: K in 32-deep chunks ascending, one FP16 MFMA per chunk and
 * product, so results are bitwise identical run to run and for every M.
 * FP16 overflow of an activation (|a| >= 65520) gives an infinite head and a
 * non-finite output, as the FP16 format implies.
 */
heal_status_t heal_gemm_f16w(int products, int64_t M, int64_t N, int64_t K, const float *A,
                             int64_t lda, const uint16_t *W16, int32_t e, float *C, int64_t ldc,
                             hipStream_t stream);
heal_status_t heal_gemm_f16w_instance(int instance, int products, int64_t M, int64_t N,
                                      int64_t K, const float *A, int64_t lda,
                                      const uint16_t *W16, int32_t e, float *C, int64_t ldc,
                                      hipStream_t stream);

/*
 * heal_presplit_b -- the B operand of heal_gemm_f32 split once (as
 * heal_split_f32) and packed with two planes (hi, lo).  B is K x N with row
 * stride ldb >= max(N, 1) (trans_b = 0), or N x K with ldb >= max(K, 1)
 * (trans_b = 1, a linear layer's weight).  Bp holds heal_packed_size(K, N, 2)
 * values: the same 4 bytes per element as the FP32 operand.
 *
 * heal_gemm_f32_presplit -- C = A * B from the pre-split operand: the same
 * bf16 MFMAs in the same order as heal_gemm_f32, so C is bitwise equal to
 * heal_gemm_f32(A, B) (and to the strided-batched form with trans_b = 1 on the
 * transposed storage); no B element is split on this path.
 */
heal_status_t heal_presplit_b(const float *B, int64_t K, int64_t N, int64_t ldb, int trans_b,
                              uint16_t *Bp, hipStream_t stream);
heal_status_t heal_gemm_f32_presplit(int64_t M, int64_t N, int64_t K, const float *A, int64_t lda,
                                     const uint16_t *Bp, float *C, int64_t ldc,
                                     hipStream_t stream);
heal_status_t heal_gemm_f32_presplit_instance(int instance, int64_t M, int64_t N, int64_t K,
                                              const float *A, int64_t lda, const uint16_t *Bp,
                                              float *C, int64_t ldc, hipStream_t stream);

/*
 * heal_quantize_i16 -- INT16 storage of a tensor (Section 4, Q/K/V
 * paragraph): q[i] = Round(32767 x[i] / m), m = max|x|, where Round takes the
 * real quotient to the nearest integer, ties to even.  The decision is exact
 * for every finite input and every m > 0 however small (it is taken on the
 * correctly rounded FP64 quotient of the exact product 32767 x, which cannot
 * cross a half-integer it does not equal); every code lies in
 * [-32767, 32767] and the extreme element gets +/-32767.  m is written to
 * *maxabs (device) and is the tensor's dequantisation scale
 * (x ~ q * m / 32767).  An all-zero tensor gives m = 0 and zero codes.  x
 * must be finite.  Two kernels are enqueued (the maximum, then the codes);
 * no host synchronisation.
 */
heal_status_t heal_quantize_i16(const float *x, int64_t n, int16_t *q, float *maxabs,
                                hipStream_t stream);

/*
 * heal_scores_i16 -- attention scores from INT16 Q and K with the dual-FP16
 * expansion (Section 4, displayed attention expansion):
 *   S_b = f * (Q_hi + Q_lo/2^10)(K_hi + K_lo/2^10)^T,
 *   f = alpha * (maxQ / 32767) * (maxK / 32767), the dequantisation of both
 *       codes, evaluated in FP64 and rounded once to FP32 (a factor below
 *       2^-126 lands in FP32's subnormal range and loses relative precision),
 * where each code q unpacks exactly into hi = RNE_f16(q) and
 * lo/2^10 = q - hi; all four products are accumulated in FP32 (per 32-deep
 * chunk: hi*hi, hi*lo, lo*hi, lo*lo), so the sum is the integer dot product
 * of the codes up to FP32 accumulation.
 *   Q_b  = Q + b*strideQ : M x K INT16, row stride ldq >= max(K, 1);
 *   K_b  = Kt + b*strideK: N x K INT16 (keys, one row per position), ldk >= max(K, 1);
 *   maxQ, maxK : device floats, the maxima written by heal_quantize_i16;
 *   S_b  = S + b*strideS : M x N FP32, row stride lds >= max(N, 1).
 */
heal_status_t heal_scores_i16(int64_t M, int64_t N, int64_t K, const int16_t *Q, int64_t ldq,
                              int64_t strideQ, const float *maxQ, const int16_t *Kt, int64_t ldk,
                              int64_t strideK, const float *maxK, float alpha, float *S,
                              int64_t lds, int64_t strideS, int64_t batch, hipStream_t stream);

/* ==========================================================================
 * Key/value cache: appending with the rotation, attention, and the choice of
 * the blocks that a query reads.
 *
 * The cache keeps the keys and values of many sequences in blocks of `block`
 * tokens.  A complete block is held as INT8 codes with one scale for its keys and
 * one for its values per head, as heal_quantize_i16 makes codes:
 *     m = max|x| over the block's rows of that head,
 *     code = Round(127 x / m), ties to even, decided exactly (m = 0: zeros),
 *     x ~ code * m / 127.
 * The rows of a sequence's last two blocks are also kept as they came, in FP32, in
 * a ring of 2 * block rows per sequence (its slot) and head.  A block that is not
 * complete is read from the ring; when its last token arrives it is quantised from
 * the ring's rows, once.  The cache therefore does not depend on how tokens were cut
 * into calls, and a sequence may be cut back (drafted tokens that were refused) by
 * passing a smaller length: as far as the beginning of the block before the last one
 * that it has reached, whose rows the ring still has, but not into blocks that were
 * appended with another slot, such as a beginning that it shares.
 *
 * Arrays (device, 16-byte aligned, owned by the caller, dense):
 *   k_codes  [blocks][heads][block][dim]
 *   v_codes  [blocks][heads][dim][block]; token 16 s + 4 g + i of a block (i, g < 4)
 *            is at place g * block / 4 + 4 s + i, the order in which a lane of a
 *            matrix instruction takes them
 *   scales   [blocks][heads][2]         m of the keys, m of the values; for a block that is
 *                                       not complete, of the rows it has
 *   k_mean   [blocks][heads][dim]       mean of the block's (rotated) keys, FP64 sum
 *                                       (both of the rows that the block had when it was
 *                                       last appended to: cutting back leaves them, and
 *                                       what reads an incomplete block goes by its rows)
 *   k_recent [slots][heads][2 * block][dim]    row of the token at place p: p % (2 * block)
 *   v_recent [slots][heads][dim][2 * block]
 * Nothing needs to be cleared before use.  A block holds one sequence's tokens for
 * heal_kv_append; sequences may share complete blocks that they only read.
 *
 * Sequences: sequence i owns the tokens cu[i] .. cu[i + 1] - 1 of a call's token
 * arrays, the last of its lens[i] tokens: token j of its n is at place
 * lens[i] - n + j.  Block b of the sequence is cache block table[i * table_ld + b].
 * These arrays are read on the device: a call does not wait for them and can be
 * captured; so what they hold is not refused but bounded:
 *   - table entries outside [0, blocks) and places past table_cols blocks hold no
 *     tokens: nothing is written for them, attention does not see them;
 *   - slots outside [0, slots): the FP32 rows are neither written nor seen;
 *   - places below 0 (lens[i] < n) are not stored; their queries see nothing;
 *   - cu is taken to ascend within [0, tokens]; tokens of no sequence are left alone,
 *     and so are their outputs.
 * ========================================================================== */

typedef struct heal_kv_cache_t {
    int64_t blocks, slots;  /* 1 .. 2^31 - 1 */
    int64_t heads;          /* key/value heads, 1 .. 1024 */
    int64_t dim;            /* 64, 96 or 128 */
    int64_t block;          /* tokens of a block: 16, 32, 64 or 128 */
    int8_t *k_codes, *v_codes;
    float *scales, *k_mean, *k_recent, *v_recent;
} heal_kv_cache_t;

typedef struct heal_kv_batch_t {
    int64_t seqs;           /* 0 .. 2^24 */
    int64_t tokens;         /* 0 .. 2^30: rows of the token arrays */
    const int32_t *cu;      /* [seqs + 1], or NULL: one token each (tokens == seqs) */
    const int32_t *lens;    /* [seqs]: lengths with the call's tokens */
    const int32_t *table;   /* [seqs][table_cols], row stride table_ld */
    int64_t table_ld, table_cols;   /* table_cols * block < 2^31 */
    const int32_t *slots;   /* [seqs], or NULL: sequence i has slot i */
} heal_kv_batch_t;

/*
 * heal_kv_append -- the tokens' keys and values enter the cache (and their queries
 * are rotated).
 *   k, v    : [tokens][heads][dim] FP32, strides of tokens and heads in elements,
 *             the last dimension dense; K and V may have strides of their own;
 *   cos, sin: [places][rot / 2] FP32, dense, or NULL with rot == 0: the first rot
 *             (even, <= dim) elements of a key at place p are rotated,
 *                 a' = a cos - b sin,  b' = b cos + a sin,
 *             the pairs (a, b) being elements j and j + rot / 2, or 2 j and 2 j + 1
 *             with interleaved = 1.  Products and sum are formed in FP64 (exactly, and
 *             with one rounding) and rounded to FP32.  A token whose place is not
 *             below `places` is taken as it is, without rotation;
 *   q, q_out: [tokens][heads_q][dim] or both NULL: queries rotated likewise; q_out
 *             may be q itself with the same strides, and must not overlap it otherwise.
 * Values are not rotated.
 *
 * A key or value that is not finite: while its block is not complete, a key makes the
 * whole output of the rows that see its token no number, a value the column that it is
 * in; other rows do not notice it, and nothing of it is left when the sequence is cut
 * back.  The codes of a complete block with such a row are no numbers, to all that see
 * any token of the block and when they are read back.
 */
heal_status_t heal_kv_append(const heal_kv_cache_t *cache, const heal_kv_batch_t *batch,
                             const float *k, int64_t k_token, int64_t k_head,
                             const float *v, int64_t v_token, int64_t v_head,
                             const float *cos, const float *sin, int64_t places, int64_t rot,
                             int interleaved,
                             const float *q, int64_t q_token, int64_t q_head, int64_t heads_q,
                             float *q_out, int64_t qo_token, int64_t qo_head, hipStream_t stream);

/*
 * heal_kv_read -- the cache's keys and values of the batch's tokens, back as FP32
 * rows: code * m / 127 (one FP32 product of the code and m / 127), or the FP32 rows
 * of a block that is not complete.  Tokens may be any number of a sequence's last
 * ones.  Rows that the cache does not hold are written as zeros.
 *   k, v : [tokens][heads][dim] FP32, dense; either may be NULL.
 */
heal_status_t heal_kv_read(const heal_kv_cache_t *cache, const heal_kv_batch_t *batch,
                           float *k, float *v, hipStream_t stream);

/*
 * heal_kv_select -- for each token and key/value head the blocks worth reading:
 * the first keep_first and the last keep_last blocks up to the token's own, and of
 * the others those that score highest,
 *     score(b) = max over the head's queries of  sum_d q_d k_mean[b]_d   (FP64),
 * equal scores by the lower block; a sum that is no number is left out, and a block
 * without any other, or that the cache does not hold, scores -infinity.
 *   q   : [tokens][heads_q][dim], heads_q a multiple of heads: head h has the queries
 *         h * heads_q / heads and on;
 *   sel : [tokens][heads][n_sel] int32, dense: block numbers of the sequence,
 *         ascending, -1 behind the last one;
 *   n_sel >= keep_first + keep_last, keep_first >= 0, keep_last >= 1,
 *   table_cols <= 16384.
 */
heal_status_t heal_kv_select(const heal_kv_cache_t *cache, const heal_kv_batch_t *batch,
                             const float *q, int64_t q_token, int64_t q_head, int64_t heads_q,
                             int64_t n_sel, int64_t keep_first, int64_t keep_last,
                             int32_t *sel, hipStream_t stream);

/*
 * heal_kv_attention -- attention of the tokens' queries over the cache:
 *     s_t = scale * q . k_t,  o = sum_t softmax(s)_t v_t,  lse = ln sum_t exp(s_t)
 * over the tokens t of the sequence with t <= place (causal = 1; all of them with
 * causal = 0) and, with window > 0 (causal = 1 only), t > place - window.  A row that sees nothing
 * gives o = 0 and lse = -infinity.  Codes are exact in FP16; queries and softmax
 * weights go to the matrix units as FP16 pairs (head and residual, scaled by powers
 * of two), FP32 rows of the cache likewise, all sums in FP32.  A pair is off by 2^-22 of
 * the value, or, where that is less, by
 *     an element of a query or of an FP32 key row   2^-38 of the row's largest,
 *     an element of an FP32 value row               2^-31 of the row's largest,
 *     a weight with its block's or row's values     2^-38 V,
 * V being the largest value of the complete blocks and FP32 rows that the output's row
 * sees.  So an output is FP32's in accuracy, not FP16's, in relation to V: beside the
 * relative errors it may be off by (2^-31 + 2^-38 n) V with n tokens seen, which is more
 * than FP32's last place only where the sum of p |v| is below (2^-7 + 2^-14 n) V, as in a
 * column far smaller than the others (and by 2^-146, in FP32's subnormal range).  Rows with
 * scores of 2^30 or more may be no numbers, and scores of query rows or keys that are below
 * 2^-100 throughout have fewer digits (which shows beside keys or queries above 2^100).
 *   sel  : NULL, or [tokens][heads][n_sel] int32, dense: only these blocks of the
 *          sequence are read for a token and head (a block listed twice counts
 *          twice; numbers outside the table hold nothing);
 *   tokens * heads_q / heads < 2^31;
 *   out  : [tokens][heads_q][dim], written; must not overlap q;
 *   lse  : [tokens][heads_q] dense, or NULL;
 *   chunk: 0, or a multiple of 64: each row's tokens are summed in chunks of so many
 *          from the first one it can see, joined in ascending order.  0 chooses by the
 *          call's sizes, so that a row's bits may depend on the batch it is in, and the
 *          time on table_cols: the lengths are not known to the host, so a table's width
 *          is best that of the longest sequence in the call; with a
 *          chunk of the caller's they depend on the row's own data only (in calls of
 *          one token per sequence, with cu NULL, or with sel).  Results are bitwise
 *          the same from run to run either way;
 *   workspace: heal_kv_attention_workspace bytes of device memory for the chunks'
 *          results, 16-byte aligned (NULL where that is 0).  It holds nothing between
 *          calls; calls that may run at the same time need one each.
 */
heal_status_t heal_kv_attention(const heal_kv_cache_t *cache, const heal_kv_batch_t *batch,
                                const float *q, int64_t q_token, int64_t q_head, int64_t heads_q,
                                float scale, int causal, int64_t window,
                                const int32_t *sel, int64_t n_sel,
                                float *out, int64_t out_token, int64_t out_head, float *lse,
                                int64_t chunk, void *workspace, int64_t workspace_bytes,
                                hipStream_t stream);

/* Bytes of workspace that heal_kv_attention needs for these arguments (which it reads
 * sizes of only: cache, batch, whether cu is NULL), or -1 where it would refuse them
 * (no HIP call). */
int64_t heal_kv_attention_workspace(const heal_kv_cache_t *cache, const heal_kv_batch_t *batch,
                                    int64_t heads_q, int64_t window, int64_t n_sel, int64_t chunk);

/* The rows (token, query of a head) of a tile that the call's kernel takes: 16, each
 * tile read by four waves side by side, or 128 for prompts; 0 where the call would be
 * refused (no HIP call).  For the labels of measurements. */
int heal_kv_attention_tile(const heal_kv_cache_t *cache, const heal_kv_batch_t *batch,
                           int64_t heads_q, int64_t window, int64_t n_sel, int64_t chunk);

#ifdef __cplusplus
}
#endif

#endif /* HEAL_H */
