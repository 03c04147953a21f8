/*
 * abq.h — C ABI of the MI355X (gfx950) arbitrary-precision quantized matmul
 *
 *      Y = dequant( A_q · W_pᵀ ),   p = weight bits, q = activation bits, both in 1..8
 *
 * after ABQ-LLM (arXiv 2408.08554), Sec. 3.4 "Custom Software Engine" and Appendix B
 * "Arbitrary Bit Matrix Calculation".  The integer accumulator is the paper's
 * Y = sum_{s<p} sum_{t<q} 2^(s+t) · BMMA(W^s, X^t)  with  w^s = (w >> s) & 1  (Appendix B),
 * i.e. exactly sum_k A[m,k]·W[n,k] over the unsigned codes; the epilogue applies the affine
 * quantizer of Eq. 3 backwards (value = Delta·(code − z); per output channel for weights,
 * per token for activations, Sec. 4.1).
 *
 * Conventions
 *  - Plain C, every call returns an int status (ABQ_OK or a negative ABQ_ERR_*), nothing is
 *    printed, no exception crosses the boundary.
 *  - Every data pointer is a DEVICE pointer (caller-owned; the library never allocates or
 *    frees device memory) and must be 16-byte aligned.  Sizes come from the *_bytes queries.
 *  - `stream` is a hipStream_t passed as void* (NULL = the default stream).  All work is
 *    enqueued asynchronously on it; no call synchronises unless its comment says so.
 *  - Argument validation happens before the first HIP call, so the error paths can be
 *    exercised on a host without a GPU.
 *  - Shapes: A is [M,K] row-major, W is [N,K] row-major (K contiguous on both), Y is [M,N]
 *    row-major.  Any M,N >= 1; 1 <= K <= ABQ_MAX_K and K·(2^p−1)·(2^q−1) <= INT32_MAX
 *    (the paper's "32-bit output"); K need not be a multiple of anything (packers pad with
 *    zero bits, which add nothing to any popcount).
 *  - Same inputs give bit-identical outputs from run to run.
 *
 * Packed operands are opaque blobs whose internal order is private to the kernels.  `layout`
 * says which representations a blob carries and must be the same value at pack time and at
 * every later call that reads the blob:
 *    ABQ_LAYOUT_PLANES  the paper's BitPacking (Sec. 3.4 step 1): [bits][rows][K] 1-bit planes;
 *                       consumed by the AND+popcount bit-serial kernels.
 *    ABQ_LAYOUT_FIELDS  bit-planes kept interleaved in groups of 1/2/4/8 planes (weights) or
 *                       as whole int8 codes (activations), tiled for the int8 MFMA kernels.
 *    ABQ_LAYOUT_BOTH    both of the above.
 *    ABQ_LAYOUT_AUTO    the library's default (currently FIELDS).
 */
#ifndef ABQ_H
#define ABQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define ABQ_OK            0
#define ABQ_ERR_NULL     (-1)  /* a required pointer is NULL */
#define ABQ_ERR_BITS     (-2)  /* p or q outside 1..8 */
#define ABQ_ERR_SHAPE    (-3)  /* M,N,K <= 0, K > ABQ_MAX_K, or K·(2^p−1)(2^q−1) > INT32_MAX */
#define ABQ_ERR_ALIGN    (-4)  /* a device pointer is not 16-byte aligned */
#define ABQ_ERR_SIZE     (-5)  /* a caller buffer is smaller than its size query */
#define ABQ_ERR_LAYOUT   (-6)  /* unknown layout value, or the blob lacks what the call needs */
#define ABQ_ERR_HIP      (-7)  /* a HIP call failed; see abq_last_hip_error() */

#define ABQ_LAYOUT_AUTO    0
#define ABQ_LAYOUT_PLANES  1
#define ABQ_LAYOUT_FIELDS  2
#define ABQ_LAYOUT_BOTH    3
#define ABQ_LAYOUT_FIELDS_G128 4   /* field-packed weights with a scale and zero-point per 128 values of K (abq_pack_weights_g128) */
/* abq_gemm only: OR one of these onto a BOTH layout to force a kernel family (A/B timing). */
#define ABQ_USE_PLANES     0x10
#define ABQ_USE_FIELDS     0x20

#define ABQ_MAX_K          131072

int         abq_version(void);                 /* major*10000 + minor*100 + patch */
const char* abq_status_string(int status);     /* static string, never NULL */
int         abq_last_hip_error(void);          /* hipError_t of the last failing HIP call on this thread */
/* Test hook: which decode kernel (Sec. 3.4, GEMV case) the last abq_gemm / abq_gemm_act_codes* call of this thread with
 * M <= 16 on field-packed operands launched; 0 before the first such call. */
#define ABQ_DECODE_DIRECT          1   /* A operand loaded into registers, one workgroup per tile */
#define ABQ_DECODE_STREAMING       2   /* A staged in LDS, ring of weight loads, workgroups walking tiles */
#define ABQ_DECODE_SHARED_OPERAND  3   /* one copy of A in LDS per workgroup of several tiles, every load up front */
int         abq_last_decode_kernel(void);

/* ------------------------------------------------------------------------------------------
 * Weights, offline (Sec. 3.4 step 1 "BitPacking"; "weight BitPacking is implemented offline").
 * ------------------------------------------------------------------------------------------ */

/* Bytes of the packed-weight blob; 0 on invalid arguments. */
size_t abq_packed_weight_bytes(int p, int N, int K, int layout);

/* Packs p-bit weight codes.  Also stores per-channel sum_k W[n,k] (needed by the zero-point
 * correction), w_scale and w_zero inside the blob.
 *   w_codes  [N,K] uint8, values < 2^p (higher bits are ignored)
 *   w_scale  [N] float, Delta_w per output channel
 *   w_zero   [N] int32, integer zero-point in 0..2^p−1
 *   packed_out / packed_bytes: caller buffer of at least abq_packed_weight_bytes(...) bytes;
 *   fully overwritten.  Inputs are not modified. */
int abq_pack_weights(int p, int N, int K,
                     const uint8_t* w_codes, const float* w_scale, const int32_t* w_zero,
                     int layout, void* packed_out, size_t packed_bytes, void* stream);

/* Per-group weight quantization (Appendix C: the method is orthogonal to group-wise weight scales; the
 * group runs along K and holds 128 values, "g128").  The blob is field-packed like ABQ_LAYOUT_FIELDS and
 * carries, per output channel and group, a binary16 scale and an integer zero-point:
 *   Y[m,n] = half_rne( a_scale[m] · sum_g w_scale[n,g] · sum_{k in group g} (A[m,k] − az[m])·(W[n,k] − wz[n,g]) )
 * with G = ceil(K/128) groups per channel, the last one short when 128 does not divide K.  The inner
 * sums are exact integers; the sum over groups is accumulated in binary32 (one rounding per group), so
 * the result carries a relative error of about G·2^-24 of the summed terms' size before the final
 * rounding to binary16.
 *   w_codes      [N,K] uint8, values < 2^p
 *   w_scale_fp16 [N,G] binary16 bit patterns (the precision deployed group formats store)
 *   w_zero       [N,G] int32 in 0..2^p−1
 *   packed_out / packed_bytes: at least abq_packed_weight_bytes(p, N, K, ABQ_LAYOUT_FIELDS_G128) bytes.
 * The order of that binary32 sum follows the launch plan (how K is split over waves), so the same problem
 * through different entry points agrees to this bound, not to the bit.
 * abq_gemm, abq_gemm_act_codes and abq_gemm_grouped take such a blob with w_layout =
 * ABQ_LAYOUT_FIELDS_G128.  Up to 16 rows of A run on the decode kernels, more rows on the prefill kernels (K-split,
 * block, tiled); all flush their integer accumulators through the group's scale every 128 k.  They cannot return the
 * raw integer accumulator: acc_i32 must be NULL (ABQ_ERR_LAYOUT otherwise).  abq_pack_weights rejects this layout value
 * (ABQ_ERR_LAYOUT). */
int abq_pack_weights_g128(int p, int N, int K,
                          const uint8_t* w_codes, const uint16_t* w_scale_fp16, const int32_t* w_zero,
                          void* packed_out, size_t packed_bytes, void* stream);

/* Test hook: recovers the codes from a blob.  `which` is ABQ_LAYOUT_PLANES or ABQ_LAYOUT_FIELDS
 * and selects the representation to decode (it must be present in the blob).
 *   w_codes_out [N,K] uint8. */
int abq_unpack_weights(int p, int N, int K, int layout, const void* packed, int which,
                       uint8_t* w_codes_out, void* stream);

/* ------------------------------------------------------------------------------------------
 * Activations, online (Fig. 3b "ReQuant" + "BitPacking": [M,K,q] -> [q,M,K]).
 * ------------------------------------------------------------------------------------------ */

size_t abq_packed_act_bytes(int q, int M, int K, int layout);

/* Per-token quantize + pack.  For each row m (all float steps in IEEE binary32):
 *   lo = min(min_k x, 0), hi = max(max_k x, 0), Delta = (hi−lo)/(2^q−1)  (Delta=1, z=0 if hi==lo)
 *   z = clamp(rint(−lo/Delta), 0, 2^q−1),  code = clamp(rint(x/Delta) + z, 0, 2^q−1)
 * (the clamp(round(x/Delta)+z) form of Eq. 3; the paper fixes only "per-token").  Stores the
 * codes, Delta, z and sum_k code inside the blob.  NaN/Inf inputs: undefined.
 *   x_fp16 [M,K] IEEE binary16 bit patterns. */
int abq_quant_pack_act(int q, int M, int K, const uint16_t* x_fp16,
                       int layout, void* packed_out, size_t packed_bytes, void* stream);

/* Packs activation codes that are already quantized.
 *   a_codes [M,K] uint8 (< 2^q; higher bits ignored), a_scale [M] float, a_zero [M] int32. */
int abq_pack_act_codes(int q, int M, int K,
                       const uint8_t* a_codes, const float* a_scale, const int32_t* a_zero,
                       int layout, void* packed_out, size_t packed_bytes, void* stream);

/* RMSNorm with the quantizer fused in (Sec. 3.4 / Fig. 3b: the online quantization of a linear layer's input
 * is folded into the operator in front of it; for the LLaMA models of the paper that operator is RMSNorm,
 * y = x / sqrt(mean(x^2) + eps) * gamma, whose formula the paper does not print).  Per token m:
 *   y[m,:] in binary16 (sum of squares exact, 1/sqrt in double rounded once to float, two float products,
 *   one rounding to binary16), then the quantizer of abq_quant_pack_act on y[m,:].
 *   x_fp16 [M,K], gamma_fp16 [K]: binary16 bit patterns;  eps >= 0
 *   a_codes_out [M,K] uint8, a_scale_out [M] float, a_zero_out [M] int32: the inputs of abq_gemm_act_codes
 *   y_fp16_out  [M,K] binary16, optional (NULL to skip): the normalized row before quantization
 * NaN/Inf inputs are undefined. */
int abq_rmsnorm_quant_act(int q, int M, int K, const uint16_t* x_fp16, const uint16_t* gamma_fp16, float eps,
                          uint8_t* a_codes_out, float* a_scale_out, int32_t* a_zero_out,
                          uint16_t* y_fp16_out, void* stream);

/* The same with the residual add in front (Sec. 3.4 / Fig. 3b again: the quantizer rides on the operator that
 * produces the linear layer's input; in the LLaMA block that operator adds a sub-layer's output to the hidden
 * state and normalizes the sum): h = half_rne(float(x) + float(residual)) — one binary32 addition, one rounding to binary16 —
 * then abq_rmsnorm_quant_act on h, all in one kernel.
 *   x_fp16, residual_fp16 [M,K] binary16;  sum_fp16_out [M,K] binary16, required: h, the next residual (it may be the
 *   buffer residual_fp16 itself, not x_fp16);  the other arguments as above. */
int abq_add_rmsnorm_quant_act(int q, int M, int K, const uint16_t* x_fp16, const uint16_t* residual_fp16,
                              const uint16_t* gamma_fp16, float eps,
                              uint8_t* a_codes_out, float* a_scale_out, int32_t* a_zero_out,
                              uint16_t* sum_fp16_out, uint16_t* y_fp16_out, void* stream);

/* SiLU(gate) * up with the quantizer fused in: the producer in front of down_proj in the LLaMA MLP (same passage).
 * Per element h = half_rne((g / (1 + exp(-g))) * up), exp taken as a fixed sequence of binary32 operations
 * (t = clamp(-g * log2 e, -126, 126), n = rint(t), 2^(t-n) by a degree-6 polynomial, scaled by 2^n: within
 * 2e-7 of exp, the same bits on every machine), then the quantizer of abq_quant_pack_act on h[m,:].
 *   gate_fp16, up_fp16 [M,K] binary16;  outputs as for abq_rmsnorm_quant_act (h_fp16_out optional). */
int abq_silu_mul_quant_act(int q, int M, int K, const uint16_t* gate_fp16, const uint16_t* up_fp16,
                           uint8_t* a_codes_out, float* a_scale_out, int32_t* a_zero_out,
                           uint16_t* h_fp16_out, void* stream);

/* Test hook: decodes an activation blob.  Any output pointer may be NULL.
 *   a_codes_out [M,K] uint8, a_scale_out [M] float, a_zero_out [M] int32, a_sum_out [M] int32. */
int abq_unpack_act(int q, int M, int K, int layout, const void* packed, int which,
                   uint8_t* a_codes_out, float* a_scale_out, int32_t* a_zero_out,
                   int32_t* a_sum_out, void* stream);

/* Load-time validation of a packed blob.  The matmul calls take a blob's geometry from their own arguments and
 * never read its header (that would cost a synchronising copy per call), so a p/q, N/M, K or layout value that
 * differs from pack time makes them read outside the blob.  This call is the check: it copies the blob's header
 * to the host — it SYNCHRONISES with `stream` — and compares magic, format version, bit width, rows, K and
 * layout with the arguments, and packed_bytes with the size query.
 *   kind: 0 = packed weights (bits = p, rows = N), 1 = packed activations (bits = q, rows = M)
 * ABQ_OK on a match; ABQ_ERR_LAYOUT on any mismatch (also for an unknown kind or layout value); ABQ_ERR_SIZE
 * when packed_bytes is smaller than the size query (checked before the first HIP call). */
int abq_check_packed(int kind, int bits, int rows, int K, int layout, const void* packed, size_t packed_bytes, void* stream);

/* ------------------------------------------------------------------------------------------
 * Matmul + bit reduction + fused dequant (Sec. 3.4 steps 2–6, Appendix B, Fig. 3b "DeQuant").
 * ------------------------------------------------------------------------------------------ */

/* Scratch bytes abq_gemm needs for this problem (may be 0). */
size_t abq_gemm_workspace_bytes(int p, int q, int M, int N, int K);

/* acc[m,n]  = sum_k A[m,k]·W[n,k]                                  (exact, int32)
 * acc'[m,n] = acc − wz[n]·sum_k A[m,k] − az[m]·sum_k W[n,k] + K·az[m]·wz[n]   (exact, int32)
 * Y[m,n]    = half_rne( float(acc') · a_scale[m] · w_scale[n] )
 *   packed_act, packed_w: blobs written by the pack calls above with the same q,M,K / p,N,K
 *   a_layout, w_layout: the layout value each blob was packed with; w_layout may carry an
 *                 ABQ_USE_* flag.  The kernel family is chosen from what both blobs carry.
 *   y_fp16    [M,N] binary16 bit patterns, required, fully overwritten
 *   acc_i32   [M,N] raw acc, optional (NULL to skip)
 *   workspace at least abq_gemm_workspace_bytes(...) bytes (may be NULL when that is 0);
 *             contents on entry are irrelevant, contents on return are unspecified. */
int abq_gemm(int p, int q, int M, int N, int K,
             const void* packed_act, int a_layout, const void* packed_w, int w_layout,
             uint16_t* y_fp16, int32_t* acc_i32,
             void* workspace, size_t workspace_bytes, void* stream);

/* Activation BitPacking fused into the matmul (Fig. 3b packs activations online on the way into
 * the kernel; Sec. 3.4 keeps that overhead down by fusing it into an existing operator).  Same
 * result, bit for bit, as abq_pack_act_codes followed by abq_gemm on the same arguments.
 *   a_codes [M,K] uint8 row-major, values < 2^q;  a_scale [M] float;  a_zero [M] int32  (device)
 *   packed_w, w_layout, y_fp16, acc_i32, stream: as for abq_gemm
 *   workspace at least abq_gemm_act_codes_workspace_bytes(...) bytes.  That query returns 0 when
 *             the call runs as ONE kernel: the decode shapes (M <= 16, or M <= 64 with few output
 *             tiles) on field-packed weights with K a multiple of 16 — the codes are offset to
 *             signed bytes and their row sums taken while the kernel stages them.  For every
 *             other problem the packed activations are written to the workspace and the two
 *             steps run back to back on the stream (few rows of another K, and more than 16 rows
 *             over few output tiles, run as one kernel all the same where that is faster; the
 *             workspace is still required, and unused).
 * Errors as abq_gemm (ABQ_ERR_NULL / ABQ_ERR_SIZE when a needed workspace is missing / too small). */
size_t abq_gemm_act_codes_workspace_bytes(int p, int q, int M, int N, int K, int w_layout);
int abq_gemm_act_codes(int p, int q, int M, int N, int K,
                       const uint8_t* a_codes, const float* a_scale, const int32_t* a_zero,
                       const void* packed_w, int w_layout,
                       uint16_t* y_fp16, int32_t* acc_i32,
                       void* workspace, size_t workspace_bytes, void* stream);

/* ReQuant fused into the matmul epilogue (Fig. 3b: the kernel's output is quantized again for the next layer; the last
 * paragraph of Sec. 3.4 folds quantization into neighbouring operators — this is the consumer side, the producers
 * above are the other).  abq_gemm_act_codes that also (or only) writes the next layer's activation codes.  A token's
 * own range is unknown before its whole output row exists, so Delta and z per token are the caller's (a calibrated or
 * previous-step range):
 *   code[m,n] = clamp( clamp(rint(Y[m,n] / out_scale[m]), -2^24, 2^24) + out_zero[m], 0, 2^q_out − 1 )
 * on the binary16 value Y[m,n] of abq_gemm, division and rint in IEEE binary32 (Eq. 3's clamp(round(x/Delta)+z)).
 *   q_out      1..8;  out_scale [M] float > 0;  out_zero [M] int32  (device)
 *   codes_out  [M,N] uint8, required: feeds the next abq_gemm_act_codes together with out_scale / out_zero
 *   y_fp16     [M,N] binary16, optional here (NULL to skip)
 *   the other arguments, the workspace and the errors as for abq_gemm_act_codes (same workspace query); ABQ_ERR_BITS
 *   also for q_out; ABQ_ERR_LAYOUT for ABQ_LAYOUT_FIELDS_G128 blobs (not built for them).  NaN/Inf outputs and
 *   out_scale <= 0 are undefined. */
int abq_gemm_act_codes_requant(int p, int q, int M, int N, int K,
                               const uint8_t* a_codes, const float* a_scale, const int32_t* a_zero,
                               const void* packed_w, int w_layout,
                               int q_out, const float* out_scale, const int32_t* out_zero, uint8_t* codes_out,
                               uint16_t* y_fp16, void* workspace, size_t workspace_bytes, void* stream);

/* abq_gemm_act_codes for callers that cannot allocate device memory or bring a workspace (code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc): the same call with no workspace argument.
 * Where abq_gemm_act_codes needs a workspace (the packed activations of its two-kernel path) this variant keeps
 * it in a buffer of ABQ_STATIC_SCRATCH_BYTES bytes that is part of the library's device image (every GPU the
 * library runs on holds it until the process ends).  It allocates nothing and frees nothing.
 * Same arguments, results (bit for bit) and errors as abq_gemm_act_codes; in addition ABQ_ERR_SIZE when
 * abq_gemm_act_codes_workspace_bytes(...) for the problem exceeds ABQ_STATIC_SCRATCH_BYTES (checked before
 * the first HIP call).  All calls on one GPU share that GPU's buffer: calls that may overlap on one GPU
 * (different streams, different host threads) race on it and must be serialized by the caller; calls on one
 * stream are safe.  The buffer needs no clearing between calls (each call writes what it reads). */
#define ABQ_STATIC_SCRATCH_BYTES (32u << 20)
int abq_gemm_act_codes_static(int p, int q, int M, int N, int K,
                              const uint8_t* a_codes, const float* a_scale, const int32_t* a_zero,
                              const void* packed_w, int w_layout,
                              uint16_t* y_fp16, int32_t* acc_i32, void* stream);

/* Very low bit widths on gfx950's 4-bit floating-point MFMA (Sec. 3.4 / Table 4: narrower operands should run faster;
 * Appendix B's sum over 1-bit planes is what makes that true on tensor cores that multiply bits).  For weights AND
 * activations of one or two bits the codes 0..3 are E2M1 values and the sums of their products are exact in the
 * instruction's binary32 accumulator for every K <= ABQ_MAX_K, so abq_f4_gemm returns the same int32 accumulator and
 * binary16 output as abq_gemm, at twice the matrix rate of the int8 path.  Both operands use one packed layout:
 *   abq_f4_packed_bytes(bits, rows, K)  size of the blob for a [rows][K] operand (0 for arguments out of range)
 *   abq_f4_pack_codes   codes u8 [rows][K] (device, row-major; bits above `bits` are dropped), scale f32 [rows] and
 *                       zero i32 [rows] (device; the zero-point of a `bits`-bit code, 0..2^bits-1: the matmul's
 *                       epilogue relies on it) -> blob `packed_out` (device, caller-owned, >= the size above);
 *                       for the weights rows = N, for the activations rows = M
 *   abq_f4_gemm         Y[M,N] = dequant(A . W^T) from two such blobs (p: bits of W, q: bits of A, both 1 or 2);
 *                       y_fp16 [M][N] device, acc_i32 [M][N] device or NULL
 * Device pointers 16-byte aligned; work is enqueued on `stream`; nothing is allocated.  ABQ_ERR_NULL, ABQ_ERR_BITS
 * (bits outside 1..2), ABQ_ERR_SHAPE, ABQ_ERR_ALIGN, ABQ_ERR_SIZE, ABQ_ERR_HIP as elsewhere.  The blobs are not
 * interchangeable with those of abq_pack_weights / abq_pack_act_codes. */
size_t abq_f4_packed_bytes(int bits, int rows, int K);
int abq_f4_pack_codes(int bits, int rows, int K, const uint8_t* codes, const float* scale, const int32_t* zero,
                      void* packed_out, size_t packed_bytes, void* stream);
int abq_f4_gemm(int p, int q, int M, int N, int K, const void* packed_act, const void* packed_w,
                uint16_t* y_fp16, int32_t* acc_i32, void* stream);

/* Launch-plan table (Appendix D, "auto kernel search": the engine picks, per problem size, the fastest of a
 * set of kernel configurations found by timing them).  The library chooses every launch plan from closed-form
 * rules; this table lets a tuner (paper_2408_08554_amd/tune.py times the candidates on the device) replace the
 * rule for exact problem sizes.  A field left 0 keeps the rule for that knob; a plan that does not fit the
 * problem (say, more waves than K has 512-blocks) is ignored and the rule applies.  Above 16 rows the rule may
 * choose a kernel without knobs.  A plan takes a problem from the K-split kernel by a K split of the decode kernel
 * where that kernel is the other choice (M <= 64, few output tiles), else by tiled_mt or tiled_ntw, and from the
 * block kernel (many output tiles) by any of the four tiled_ knobs: a plan found for the tiled kernel keeps it, so a
 * table older than the library is worth a new search.  Per-group blobs stay where the rule puts them.  Results never
 * depend on the plan (per-group weight scales: to their stated bound).  Process-wide, thread-safe; entries hold no
 * device state.
 *   skinny_waves    waves per workgroup of the decode kernel = K split of a tile: 1, 2, 4..8
 *   skinny_kgroups  K groups of the decode kernel: 1..4
 *   tiled_mt        rows of A per workgroup tile of the prefill kernel / 16: 4 or 8
 *   tiled_ntw       16-channel tiles of W per wave: 1, 2 or 4
 *   tiled_wd        operand steps in flight: 2 or 4 (4 exists for tiled_mt = 4 with tiled_ntw <= 2)
 *   tiled_band      row blocks of A per band of the tile order: >= 1
 *   direct_r        decode kernel for M <= 16: -1 the streaming kernel (A staged in LDS, load ring); 1, 2 or 4 the
 *                   direct kernel (A operand loaded into registers) with that many 512-k blocks per wave; -2 the
 *                   shared-operand kernel (one copy of A in LDS per workgroup of several tiles) where it fits, else the
 *                   streaming kernel
 * abq_plan_set: plan == NULL removes the entry.  ABQ_ERR_BITS / ABQ_ERR_SHAPE as abq_gemm; ABQ_ERR_LAYOUT for a
 * value outside the lists above.  abq_plan_get fills *out (all zero when there is no entry). */
typedef struct abq_plan {
    int skinny_waves, skinny_kgroups;
    int tiled_mt, tiled_ntw, tiled_wd, tiled_band;
    int direct_r;
} abq_plan;
int  abq_plan_set(int p, int q, int M, int N, int K, const abq_plan* plan);
int  abq_plan_get(int p, int q, int M, int N, int K, abq_plan* out);
void abq_plan_clear(void);

/* Grouped decode launch (Sec. 3.4: the engine replaces every linear layer of a decoder block; Table 4's
 * matmuls take microseconds each, so launching them one by one leaves the memory system idle between
 * them).  `count` independent problems that share p, q, M and the layouts, each with its own N, K,
 * weights, activations and outputs, are served by ONE kernel launch per eight problems when every
 * problem is decode-shaped: M <= 16, K >= 2048 (K a multiple of 16 for unpacked codes), up to 16 rows of
 * A fitting LDS ((M * (K + 528) below ~120 KB), field-packed weights.  Other groups with M <= 16 run as one
 * launch per length of K and eight problems too where that is faster (few bytes of A, no plan-table entry
 * for a member); otherwise the problems run one after the other exactly as abq_gemm / abq_gemm_act_codes
 * would run them.  Results are bit-identical to the single calls either way.
 *   host_problems: HOST array of `count` descriptors holding DEVICE pointers.  Each gives its activations
 *                  either packed (packed_act, a_codes = NULL) or as unpacked codes (a_codes, a_scale, a_zero,
 *                  packed_act = NULL); all problems of a call use the same form.  The array is read before the
 *                  call returns.
 *   workspace:     at least abq_gemm_grouped_workspace_bytes(...) bytes: 0 for packed activations and for groups of the
 *                  decode shape above, else the largest single call's need (required whichever way the group runs).
 * Errors as abq_gemm; ABQ_ERR_SHAPE also for count < 1, ABQ_ERR_LAYOUT for mixed activation forms. */
typedef struct abq_problem {
    int N, K;
    const void* packed_w;       /* abq_pack_weights(p, N, K, ..., w_layout) */
    const void* packed_act;     /* abq_pack_act_codes / abq_quant_pack_act (q, M, K, ..., a_layout), or NULL */
    const uint8_t* a_codes;     /* [M,K] uint8 codes < 2^q, or NULL */
    const float* a_scale;       /* [M], with a_codes */
    const int32_t* a_zero;      /* [M], with a_codes */
    uint16_t* y_fp16;           /* [M,N], required */
    int32_t* acc_i32;           /* [M,N] raw accumulator, may be NULL */
} abq_problem;
size_t abq_gemm_grouped_workspace_bytes(int p, int q, int M, int count, const abq_problem* host_problems,
                                        int a_layout, int w_layout);
int abq_gemm_grouped(int p, int q, int M, int count, const abq_problem* host_problems,
                     int a_layout, int w_layout, void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------
 * The attention half of a decoder block, for many requests at once: what lies between the q / k / v projections and the
 * output projection (rotation, paged cache, attention), and the requests' own low-rank adapters beside the projections.
 * All tensors are binary16, as the projections write them; queries, keys and values may be column ranges of one fused
 * projection's output (row strides in elements, a multiple of 8).
 * ------------------------------------------------------------------------------------------ */

/* Keys and values of one layer, in pages handed out to sequences by the caller.  Vector (page, head, offset) lies at
 * ((page * heads + head) * page_size + offset) * head_dim elements.
 *   kv_bits    16: binary16 values.  8: codes 0..255 (one byte each) with a scale and a zero-point per vector, the
 *              quantizer of abq_quant_pack_act with q = 8 on the binary16 vector; value = scale * (code - zero), scale > 0.
 *              (A vector of zeros has scale 2^-32: attention keeps what is 2^-24 of the largest weight times scale of V.)
 *   page_size  tokens per page: a power of two, 16..4096;  head_dim a multiple of 16, 16..256;  num_pages, heads >= 1,
 *              heads * head_dim < 2^20
 *   k, v       [num_pages][heads][page_size][head_dim] binary16 or uint8
 *   k_scale, v_scale [num_pages][heads][page_size] float;  k_zero, v_zero the same of uint8 (a zero-point of 8-bit codes
 *              fits a byte, and a decoding step reads one per vector).  NULL when kv_bits is 16. */
typedef struct abq_kv_cache {
    int kv_bits, num_pages, page_size, heads, head_dim;
    void *k, *v;
    float* k_scale;
    uint8_t* k_zero;
    float* v_scale;
    uint8_t* v_zero;
} abq_kv_cache;

/* The rows of one step: `rows` new tokens of `seqs` sequences, sequence s owning rows row_start[s] .. row_start[s+1] - 1.
 * Row i of a sequence with n rows stands at position lens[s] - n + i.
 *   row_start [seqs+1] int32, ascending from 0;  lens [seqs] int32: tokens of each sequence, the new ones among them
 *   pages     [seqs][max_pages] int32: token t of sequence s lies in page pages[s][t / page_size], at offset t % page_size
 *   max_new   no sequence has more rows in this step;  max_len: no sequence has more tokens.  They size the launches
 *             (abq_attn_paged): close bounds are faster ones.  1 <= max_new <= rows <= 2^22, 1 <= seqs <= 65535, 1 <= max_len.
 * The arrays are device memory and never checked on the host.  Whatever they hold, nothing outside the tensors is read or
 * written: rows behind row_start[seqs] are left as they were; a page number outside 0..num_pages-1 (-1, say) is a page
 * that is not there - nothing is appended to it and attention does not see its tokens; tokens beyond max_pages pages and
 * positions below 0 likewise.  abq_attn_paged leaves rows from max_new on as they were and sees no token from max_len on, nor
 * from 2^30 on. */
typedef struct abq_batch {
    int rows, seqs, max_pages, max_new, max_len;
    const int32_t *row_start, *lens, *pages;
} abq_batch;

/* Puts the rows' keys and values into the cache, at their positions, the keys rotated to them on the way, and rotates the
 * rows' queries (optional):
 *   (x[j], x[j + r/2]) -> (x[j] cos a - x[j + r/2] sin a, x[j + r/2] cos a + x[j] sin a),  a = position * inv_freq[j],  j < r/2
 * with r = rotary_dim (0: no rotation, inv_freq not read; elements from r on are kept); `interleaved`: the pairs are
 * (x[2j], x[2j+1]).  The angle is reduced from its exact value (positions are exact however far; angles up to 2^48), sine and cosine are
 * within 2^-23, products and sum in binary32, one rounding to binary16.  A cache of codes quantizes the rotated binary16
 * vector.
 *   heads_q    query heads (with q), a multiple of cache->heads, rows * heads_q <= 2^28, seqs * heads <= 2^21;  rotary_dim a multiple of 16, 0..head_dim
 *   q [rows][heads_q * head_dim] (NULL to skip), k, v [rows][heads * head_dim] with row strides ldq, ldk, ldv in elements
 *   inv_freq   [rotary_dim / 2] float
 *   q_out      [rows][heads_q * head_dim], contiguous; it may be q itself where that is contiguous too
 * Two rows of a call never name the same place unless two sequences share a page that both write (or a page stands twice in
 * a sequence); which of the rows' elements such a place then holds is unspecified.  NaN/Inf inputs: undefined for codes. */
int abq_kv_append(const abq_kv_cache* cache, const abq_batch* batch, int heads_q, int rotary_dim, int interleaved,
                  const float* inv_freq, const uint16_t* q, int ldq, const uint16_t* k, int ldk, const uint16_t* v, int ldv,
                  uint16_t* q_out, void* stream);

/* Reads vectors back out of the cache (exporting a prefix, checks): for each slot = page * page_size + offset the keys and
 * values of all heads as binary16, codes as half_rne(scale * (code - zero)).  A slot outside the cache reads as zeros.
 *   slots [count] int32 (device);  k_out, v_out [count][heads * head_dim];  page numbers up to INT32_MAX / page_size,
 *   count <= 2^22 */
int abq_kv_read(const abq_kv_cache* cache, int count, const int32_t* slots, uint16_t* k_out, uint16_t* v_out, void* stream);

/* Attention of the rows over what the cache holds of their sequences (the new tokens' keys and values among it: append
 * first).  Query head h reads key head h / (heads_q / heads):
 *   y[row,h,:] = half_rne( sum_t w_t v_t / sum_t w_t ),  w_t = exp(scale * q . k_t),  over the tokens t the row sees:
 *   all of its sequence up to its own position (causal), or all of its sequence (causal = 0).  A row that sees none is zero;
 *   one whose scores are all minus infinity (keys of a binary16 cache can be infinite) is 0 / 0, NaN.
 * Scores, running maximum, sums and the weighted sum are binary32.  For the product with the values the weights have 21 bits
 * or more where a sequence has few rows to a key head (new tokens times heads_q / heads: up to 16 or 32, by the sizes of the
 * step), and are rounded to binary16 in longer chunks.  What lies in pages beyond a sequence's length, or in tokens that a row does not see, does not reach its output
 * (NaN and infinities included).
 *   heads_q    as for abq_kv_append
 *   q [rows][heads_q * head_dim], row stride ldq;  y [rows][heads_q * head_dim], contiguous, not overlapping q
 *   workspace  at least abq_attn_paged_workspace_bytes(cache, batch, heads_q) bytes (may be 0): the parts of long sequences
 *              that several workgroups share.  Contents on entry are irrelevant; calls that may overlap need one each.
 * The order of the binary32 sums depends on max_new, max_len, rows and seqs, not on other sequences' contents. */
size_t abq_attn_paged_workspace_bytes(const abq_kv_cache* cache, const abq_batch* batch, int heads_q);
int abq_attn_paged(const abq_kv_cache* cache, const abq_batch* batch, int heads_q, const uint16_t* q, int ldq, float scale,
                   int causal, uint16_t* y, void* workspace, size_t workspace_bytes, void* stream);

/* Low-rank adapters beside a shared projection, one of many for each row:
 *   out[m,:] = half_rne( y[m,:] + scale[i] * B_i (A_i x[m,:]) ),  i = ids[m];   out[m,:] = y[m,:] where ids[m] is outside 0..adapters-1
 * x is the projection's input before quantization (y_fp16_out of the producers above), y its output.  A_i x is summed in
 * binary32 and enters the second product with 21 bits or more of its row's largest element.
 *   rank       1..256 (pad smaller adapters of a pool with zeros);  1 <= M <= 2^19, 1 <= N <= 2^28, 1 <= K <= ABQ_MAX_K
 *   x [M][K] row stride ldx;  ids [M] int32 (device);  a [adapters][rank][K], b [adapters][N][rank] binary16;
 *   scale [adapters] float;  y [M][N] row stride ldy;  out [M][N] row stride ldout: y itself (same stride), or no overlap
 *   (strides in elements, any value >= K or N)
 * A row's result does not depend on the other rows' adapters or inputs; infinities in its own come out as infinities or NaN.
 *   workspace  at least abq_lora_add_workspace_bytes(M, N, K, rank) bytes; contents on entry are irrelevant, calls that may
 *              overlap need one each. */
size_t abq_lora_add_workspace_bytes(int M, int N, int K, int rank);
int abq_lora_add(int M, int N, int K, int rank, int adapters, const uint16_t* x, int ldx, const int32_t* ids,
                 const uint16_t* a, const uint16_t* b, const float* scale, const uint16_t* y, int ldy, uint16_t* out, int ldout,
                 void* workspace, size_t workspace_bytes, void* stream);

/* ------------------------------------------------------------------------------------------
 * A layer of experts (a block's MLP as many small ones, a few of which each token goes through): the router's choice, the
 * products with the experts' quantized weights, and the weighted sum.  The pieces between are the calls above:
 * abq_rmsnorm_quant_act makes the codes that the up projections take, abq_silu_mul_quant_act those of the down projection.
 * A row is (token, choice), numbered token * top + choice ("slot"); rows sorted by expert have a place.
 * ------------------------------------------------------------------------------------------ */
#define ABQ_MOE_MAX_EXPERTS 1024
#define ABQ_MOE_MAX_TOP 16

/* The router: from each token's logits the `top` experts it goes to, their weights, and the rows sorted by expert.
 *   choice   the largest logits, largest first, ties to the lowest expert; with a bias the largest score + bias[e] (scores and sum in
 *            binary64).  An expert whose logit is minus infinity or NaN (or whose score + bias is) is not there: a token with
 *            fewer than `top` experts, a padding row with none, has -1 and weight 0 in its last choices.
 *   score    softmax over all of the token's experts (sigmoid = 0) or the sigmoid of the logit
 *   weight   score, with renormalize score / (sum of the chosen ones' scores); times scale.  Binary32, exponentials of differences from
 *            the largest logit.  (A logit of plus infinity makes NaN of its token's softmax weights, and with a bias its softmax
 *            scores too.)
 *   logits   [tokens][experts], row stride ld in elements, binary16 (logits_bits = 16) or float (32);  bias [experts] float or NULL
 *   ids, places [tokens][top] int32: expert, place of each choice (-1: none);  weights [tokens][top] float
 *   starts   [experts + 1] int32: expert e has the places starts[e] .. starts[e+1] - 1, in the order of their slots
 *   order    [tokens * top] int32: the slot at each place, -1 behind the last one
 *   1 <= experts <= ABQ_MOE_MAX_EXPERTS, 1 <= top <= min(experts, ABQ_MOE_MAX_TOP), tokens * top <= 2^22
 *   workspace at least abq_moe_route_workspace_bytes(...) bytes (0 for few tokens; never falls as tokens grow, so that one of the
 *            largest batch serves all); contents on entry are irrelevant, calls that may overlap need one each. */
size_t abq_moe_route_workspace_bytes(int tokens, int experts, int top);
int abq_moe_route(int tokens, int experts, int top, const void* logits, int logits_bits, int ld, const float* bias, int sigmoid,
                  int renormalize, float scale, int32_t* ids, float* weights, int32_t* starts, int32_t* order, int32_t* places,
                  void* workspace, size_t workspace_bytes, void* stream);

/* The weights of one linear layer of all experts: for each expert a blob of abq_pack_weights (the same bytes), `stride` bytes apart (a multiple of 16, at
 * least abq_packed_weight_bytes(p, N, K, layout)).  w_codes [experts][N][K], w_scale, w_zero [experts][N], device; per-channel layouts only. */
int abq_pack_experts(int p, int experts, int N, int K, const uint8_t* w_codes, const float* w_scale, const int32_t* w_zero, int layout,
                     void* packed_out, size_t stride, void* stream);

/* One linear layer of all experts: place r, which starts[e] <= r < starts[e+1] gives to expert e, is row r of Y:
 *   Y[r,:] = dequant( A[s] . W_e^T ),   s = order[r] / top, or r where order is NULL
 * with accumulator and epilogue of abq_gemm, to the bit (the int32 accumulator is not returned).
 *   a_codes  [tokens][K] uint8 (bits above q are dropped), a_scale [tokens] float, a_zero [tokens] int32
 *   packed_w of abq_pack_experts, or one blob of abq_pack_weights(p, N, K, ..., w_layout) for each expert, w_stride bytes apart (a multiple of 16, at least the
 *            blob's size); field-packed per-channel blobs (AUTO, FIELDS, BOTH), else ABQ_ERR_LAYOUT
 *   starts   [experts + 1] int32, ascending from 0 (device);  order [rows] int32 (device) or NULL, then tokens = rows
 *   y_fp16   [rows][N] binary16: rows from starts[experts] on are left as they were
 * starts and order are never checked on the host.  Whatever they hold, nothing outside the tensors is read or written; starts that do
 * not ascend, and entries of order that name no row of A, leave the rows concerned with unspecified contents.
 *   1 <= rows, tokens <= 2^22;  N <= 2^27;  tokens * K (K rounded up to 512) < 2^32;  (rows / 64 + experts) * ceil(N / 128) < 2^24;
 *   the rest as for abq_gemm.  Workspace: at least abq_moe_gemm_workspace_bytes(...) bytes (0 where an expert has few rows: the codes
 *   are packed on the way there; never falls as rows and tokens grow together); contents on entry are irrelevant, calls that may overlap need one each. */
size_t abq_moe_gemm_workspace_bytes(int p, int q, int rows, int N, int K, int tokens, int experts);
int abq_moe_gemm(int p, int q, int rows, int N, int K, int tokens, int experts, int top,
                 const uint8_t* a_codes, const float* a_scale, const int32_t* a_zero, const void* packed_w, size_t w_stride, int w_layout,
                 const int32_t* starts, const int32_t* order, uint16_t* y_fp16, void* workspace, size_t workspace_bytes, void* stream);

/* Back to one row a token:
 *   out[t,:] = half_rne( add[t,:] + sum_j weights[t,j] * y[places[t,j],:] ),   j < top in this order, in binary32
 * over the choices whose place is in 0..rows-1 (add NULL: without it; a shared expert's output, or the residual).
 *   y [rows][N] row stride ldy, add, out [tokens][N] row strides ldadd, ldout (binary16, strides in elements, any value >= N); out may be add
 *   itself (same stride), and overlaps nothing else;  weights [tokens][top] float, places [tokens][top] int32 (device)
 *   1 <= tokens, rows <= 2^22, 1 <= top <= ABQ_MOE_MAX_EXPERTS, 1 <= N <= 2^20, tokens * ceil(N / 2048) < 2^24 */
int abq_moe_combine(int tokens, int N, int rows, int top, const uint16_t* y, int ldy, const int32_t* places, const float* weights,
                    const uint16_t* add, int ldadd, uint16_t* out, int ldout, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* ABQ_H */
