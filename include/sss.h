/*
 * sss.h -- C ABI of the GB300 (sm_103a) signed-symmetric few-bit weight
 * library: group-wise q-bit weight quantization with a signed per-group scale
 * and no zero point, and the decode GEMV / prefill GEMM that consume the
 * packed codes with dequantisation fused in.
 *
 * Source of the operations: Colbert, Dash et al., "Signed Symmetric
 * Quantization for Few-Bit Integers": the integer quantizer (eq:quantizer,
 * Sec. 1), the min-max grid (eq:minmax) and absmax grid (eq:absmax) of
 * Sec. 3, the signed symmetric family (eq:signed_sym_quant) and the signed
 * absmax sign rule (eq:sign_rule), the direct-casting protocol (Appendix C.1)
 * and the deployed block formats and quantized GEMM expansion (Appendix B).
 *
 * Conventions for every entry point:
 *  - All tensor pointers are DEVICE pointers owned by the caller.  No entry
 *    point allocates device memory; the library keeps only small host-side
 *    per-device records (SM count, raised shared-memory limits of kernels).
 *  - `stream` is a cudaStream_t passed as void* (NULL = legacy default
 *    stream).  Every call is asynchronous on that stream; none synchronises.
 *  - The return value reports synchronous argument checks and launch errors.
 *    Data-dependent conditions (NaN/Inf weights, a scale that overflows
 *    fp16, a wait that timed out) are OR-ed as SSS_FLAG_* bits into the
 *    optional device word `dev_status` (uint32), which the caller zeroes and
 *    reads back after synchronising.
 *  - No C++ exception crosses the ABI.  Functions are thread-safe.
 *
 * Weight layout: W is row-major fp32 [n][k] (n = output features, k = input
 * features, the quantized axis); groups are `group` consecutive elements
 * along k, so group G = row*(k/group) + j starts at element G*group.
 * Packed codes are stored per group, groups back to back (codes of group G
 * start at byte G*group*q/8):
 *   q=4: element j in byte j>>1, low nibble for even j, high for odd j;
 *   q=2: element j in byte j>>2 at bits 2*(j&3);
 *   q=3: a plane of group/4 bytes holding (u & 3) in the q=2 layout, then a
 *        plane of group/8 bytes with bit (j&7) of byte (j>>3) = (u >> 2).
 * The stored code is u = c + 2^(q-1) for the symmetric grids (c in the signed
 * alphabet {-2^(q-1) .. 2^(q-1)-1}) and u = c in {0 .. 2^q-1} for ASYM.
 * scales: IEEE fp16 [n][k/group], the signed scale s = gamma*alpha for the
 * symmetric grids (Appendix B.1 lets the stored scale be negative), the step
 * for ASYM.
 * mins: fp16 [n][k/group], ASYM only (the stored minimum m; w^ = s*u + m).
 */
#ifndef SSS_H
#define SSS_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  SSS_GRID_UNSIGNED_SYM = 0, /* absmax grid, s = ||w||_inf / 2^(q-1) > 0 (eq:absmax)      */
  SSS_GRID_SIGNED_SYM = 1,   /* signed absmax, s = gamma* alpha (eq:signed_sym_quant,
                                eq:sign_rule); gamma = +1 when max w == -min w            */
  SSS_GRID_ASYM = 2          /* min-max grid on {0..2^q-1} (eq:minmax)                  */
} sss_grid_t;

typedef enum {
  SSS_OK = 0,
  SSS_E_ARG = 1,         /* a size or enum argument is out of range / NULL         */
  SSS_E_UNSUPPORTED = 2, /* a combination this build does not implement            */
  SSS_E_ALIGN = 3,       /* a pointer is not aligned as documented                 */
  SSS_E_CUDA = 4,        /* a CUDA runtime/driver call or launch failed            */
  SSS_E_WORKSPACE = 5    /* workspace too small (see sss_workspace_bytes)          */
} sss_status_t;

/* bits OR-ed into *dev_status by the kernels */
#define SSS_FLAG_NONFINITE 0x1u /* a weight group contains NaN or +-Inf; that group's
                                   codes/scale are placeholders (u = 2^(q-1) and s = +0
                                   for symmetric grids, u = 0 and s = +0 for ASYM);
                                   sss_kv_store_q4: a group of a head does             */
#define SSS_FLAG_RANGE 0x2u     /* sss_quantize: a stored fp16 scale or min is infinite
                                   (|s| >= 65520), or the fp32 ASYM step overflowed
                                   (codes then 0).  sss_gemv at batch 2..16 and
                                   sss_gemm: a group's fp16 weight operand may overflow
                                   (see those calls); their outputs may then hold
                                   inf or NaN.  sss_kv_store_q4, sss_attention_q4: see
                                   there                                               */
#define SSS_FLAG_TIMEOUT 0x4u   /* a bounded pipeline wait of sss_gemm (or
                                   sss_gemm_noalloc), sss_quantize,
                                   sss_quantize_rotated, sss_attention or
                                   sss_attention_q4 expired; the output is incomplete  */
#define SSS_FLAG_INDEX 0x8u     /* sss_page_plan, sss_qk_norm_rope, sss_attention, and the
                                   calls on the 4-bit cache and on shared pages: a length,
                                   position, slot, parent or page lies outside what the call's
                                   arguments allow; what the calls do then is said there */
#define SSS_FLAG_PAGES 0x10u    /* sss_page_plan, sss_page_fork: the free pages, or the
                                   table's columns, do not suffice                     */

typedef enum { SSS_OUT_F32 = 0, SSS_OUT_F16 = 1, SSS_OUT_BF16 = 2 } sss_dtype_t;

/* A packed weight tensor.  Plain descriptor; the library never frees it. */
typedef struct {
  int64_t n;         /* rows (output features), 0 .. 2^31                           */
  int64_t k;         /* columns (input features), 0 .. 2^31, multiple of `group`  */
  int32_t q;         /* bits per code: 2, 3 or 4                                   */
  int32_t group;     /* group size along k: 32, 64 or 128                          */
  int32_t grid;      /* sss_grid_t                                                 */
  int32_t reserved;  /* must be 0                                                  */
  uint8_t* codes;    /* [n][k*q/8] bytes, layout above                             */
  uint16_t* scales;  /* [n][k/group] fp16                                          */
  uint16_t* mins;    /* [n][k/group] fp16 for SSS_GRID_ASYM, else ignored (NULL)   */
} sss_qtensor_t;

/* Bytes of packed codes for an [n][k] tensor at q bits: n*k*q/8. */
size_t sss_codes_bytes(int64_t n, int64_t k, int32_t q);

/* Human-readable name of a status code (static storage). */
const char* sss_status_string(sss_status_t status);

/* Text of the last CUDA error seen by this thread inside the library
 * (static thread-local storage; "" if none). */
const char* sss_last_error(void);

/*
 * sss_quantize -- direct casting of an fp32 weight matrix (Appendix C.1):
 * for every group, M = ||w||_inf, the grid's scale (eq:absmax; eq:sign_rule
 * for SIGNED: gamma* = -sign(w_i*), so the dominant outlier lands exactly on
 * the code -2^(q-1); eq:minmax for ASYM), codes c = clip(RNE(w/s)) of the
 * exact quotient (ties to even), packed as above, and the fp16 scale (and
 * min).  Bit-exact with the reference definition.
 *
 *   w           [in]  device fp32 [n][k], 16-byte aligned, row-major contiguous.
 *   out         [in]  descriptor of the outputs (n, k, q, group, grid and the
 *                     device buffers codes (16-byte aligned), scales, mins);
 *                     not retained.
 *   clip_counts [out] nullable device uint8 [n][k/group][2]: for symmetric
 *                     grids {|C_gamma|, |C_-gamma|} (def:clipped-set): the
 *                     number of pre-clip codes equal to +2^(q-1) and to
 *                     -2^(q-1); for ASYM {0, 0}.
 *   dev_status  [out] nullable device uint32; SSS_FLAG_NONFINITE/RANGE OR-ed.
 * Errors: SSS_E_ARG (q, group, grid, k % group, NULL buffers), SSS_E_ALIGN
 * (w or codes not 16-byte aligned), SSS_E_CUDA.  n == 0 is a no-op.
 */
sss_status_t sss_quantize(const float* w, const sss_qtensor_t* out,
                          uint8_t* clip_counts, uint32_t* dev_status,
                          void* stream);

/*
 * sss_dequantize -- w^ = f16(s)*c (symmetric; exact in fp32) or
 * w^ = fl32(fl32(f16(s)*u) + f16(m)) (ASYM), the value eq:quantizer assigns
 * to each weight, written as [n][k] in out_dtype (fp16/bf16 outputs are the
 * round-to-nearest-even of the fp32 value).
 *   qt   [in]  packed tensor (device buffers).
 *   out  [out] device [n][k] of sss_dtype_t out_dtype, 16-byte aligned.
 * Errors: SSS_E_ARG, SSS_E_ALIGN, SSS_E_CUDA.
 */
sss_status_t sss_dequantize(const sss_qtensor_t* qt, void* out,
                            int32_t out_dtype, void* stream);

/*
 * sss_gemv -- decode GEMV y[b][r] = sum_k w^[r][k] * x[b][k] with the
 * dequantisation fused (Appendix B.3: y = sum_b s * (integer dot) for the
 * symmetric formats, plus the row-sum term sum_b m * sum_{k in b} x for
 * ASYM).  fp32 accumulation; deterministic (no atomics).
 * At batch 1 the integer codes meet the activations exactly and the group scale is
 * applied in fp32.  So it is at batch 2..16 for q = 2 and 4, and whenever k is not a
 * multiple of 256, with these limits:
 *   - an activation enters as fp16 x * 2^-p, p = 0, 2 or 4: exactly x for 2^-13 <=
 *     |x| <= 65504.  Smaller ones are rounded, to within 2^-21.  With larger or
 *     infinite ones, the outputs of their batch row are computed by plain fp32
 *     products of w^ and x, many times slower (q = 2 and 4, k a multiple of 256), or
 *     may be infinite or NaN (else);
 *   - the staged activations fit the shared memory: at batch 2..8, k up to 30720 at
 *     least (q = 4 ASYM, group 32; 38912 and more for the others); at batch 9..16
 *     k <= 12288 for q = 4 ASYM (17920 with group 128), 16384, 17920 or 21504 for q
 *     = 4 symmetric and 22528, 24576 or 28672 for q = 2 (group 32, 64 or 128).
 * Otherwise (k a multiple of 256 and q = 3 or a longer k) the batch fills the
 * tensor-core columns across groups, so each weight enters the product as w^
 * rounded once to fp16 (<= 2^-11 relative, as in sss_gemm), times 2^p (p = 0, 2 or
 * 4, the bit offset of the code's field).  That operand fits fp16 while |w^| * 2^p <
 * 65520; at batch 2..16 with k a multiple of 256, whatever q, every group whose
 * scale could break this raises SSS_FLAG_RANGE (checked per scale, conservatively:
 * |s| * 2^(q-1) * 16 >= 65520 for the symmetric grids, (|s| * (2^q - 1) + |m|) * 16
 * >= 65520 for ASYM).
 *   qt        [in]  packed tensor; codes 16-byte aligned, scales/mins 4-byte
 *                   aligned.
 *   x_bf16    [in]  device bf16 [batch][k], 16-byte aligned.
 *   batch     [in]  1..16.
 *   y         [out] device fp32 [batch][n].
 *   workspace [in]  device scratch of ws_bytes >= sss_workspace_bytes(qt,
 *                   batch, SSS_OP_GEMV) bytes, 16-byte aligned, or NULL when
 *                   that size is 0.  Its contents on entry are ignored.
 *   dev_status [out] nullable; SSS_FLAG_RANGE as above (batch 2..16).  The
 *                   GEMV kernels have no waits that could time out.
 * Errors: SSS_E_ARG, SSS_E_ALIGN, SSS_E_WORKSPACE, SSS_E_CUDA.
 */
sss_status_t sss_gemv(const sss_qtensor_t* qt, const uint16_t* x_bf16,
                      int32_t batch, float* y, void* workspace,
                      size_t ws_bytes, uint32_t* dev_status, void* stream);

/* flags of sss_gemv_multi */
#define SSS_GEMV_PDL 0x1u           /* launch as a programmatic dependent launch: the kernel
                                       may start while the preceding kernel in the stream
                                       drains; it reads x (and writes y) only after that
                                       kernel has completed                                */
#define SSS_GEMV_WEIGHTS_READY 0x2u /* with SSS_GEMV_PDL: the packed weights are not written
                                       by the preceding work in the stream, so they may be
                                       streamed in before it completes.  (What may still be
                                       running: the call before this one, and while that is
                                       a sss_gemv_multi with this flag, the call before it
                                       as well.)                                           */
#define SSS_GEMV_ACT_Q8 0x4u        /* quantize x to Q8_0 on the fly (see
                                       sss_quantize_act_q8) and multiply the packed
                                       weights with the Q8_0 values: y_j[r] =
                                       sum_blocks fl16(d) * sum_k w^_j[r][k] * q[k]; the
                                       integer dot of codes and int8 values is exact */

/*
 * sss_gemv_multi -- batch-1 decode GEMV of several packed matrices that
 * share one activation vector (e.g. the q/k/v or gate/up projections of a
 * layer) in one launch: y_j[r] = sum_k w^_j[r][k] * x[k] (same arithmetic as
 * sss_gemv).  Every lane loads the packed bytes it multiplies straight into
 * registers (a ring one unit ahead of its use); only the activations are
 * staged in shared memory.
 *   qts     [in]  count pointers to packed tensors with equal k, q, group and
 *                 grid; codes, scales (and mins) 16-byte aligned.
 *   ys      [out] count device fp32 pointers, y_j of length qts[j]->n.
 *   count   [in]  1..4.
 *   x_bf16  [in]  device bf16 [k], 16-byte aligned.
 *   flags   [in]  SSS_GEMV_* bits.
 *   dev_status [out] nullable; with SSS_GEMV_ACT_Q8 the Q8_0 flags of x
 *                 (the streaming kernel has no waits that could time out).
 * Shapes with k % 256 != 0 or k % (8*group) != 0, or unaligned buffers, run
 * as one sss_gemv per matrix (flags then have no effect, and SSS_GEMV_ACT_Q8
 * returns SSS_E_UNSUPPORTED).
 * Errors: SSS_E_ARG, SSS_E_ALIGN, SSS_E_UNSUPPORTED, SSS_E_CUDA.
 */
sss_status_t sss_gemv_multi(const sss_qtensor_t* const* qts, float* const* ys,
                            int32_t count, const uint16_t* x_bf16, uint32_t flags,
                            uint32_t* dev_status, void* stream);

/*
 * sss_gemm -- prefill GEMM Y[m][r] = sum_k w^[r][k] * X[m][k] (Appendix B.3;
 * prefill is the phase where the matrix products set the time), dequantising
 * weight tiles on chip and accumulating on the tcgen05 tensor cores in fp32
 * (tensor memory).  Tile operands are fp16: w^ rounded to fp16 and X
 * converted from bf16 (exact for 2^-17 <= |x| <= 65504).  The weight
 * operand fits fp16 while |w^| < 65520; every group whose scale could break
 * this raises SSS_FLAG_RANGE (checked per scale, conservatively: |s| *
 * 2^(q-1) >= 65520, or |s| * (2^q - 1) + |m| >= 65520 for ASYM).
 *   qt        [in]  packed tensor, symmetric grids or ASYM; k % 64 == 0;
 *                   codes 16-byte aligned.
 *   x_bf16    [in]  device bf16 [m][k], 16-byte aligned.
 *   m         [in]  0 .. 2^24 tokens.
 *   y         [out] device fp32 [m][n], 16-byte aligned, n % 4 == 0.
 *   workspace [in]  device scratch, 16-byte aligned, of ws_bytes >= m * k * 2
 *                   (rounded up to 256); sss_workspace_bytes(qt, m,
 *                   SSS_OP_GEMM) bytes enable split K (see there).  Its
 *                   contents on entry are ignored.
 *   dev_status [out] nullable; SSS_FLAG_TIMEOUT if a bounded wait expired,
 *                   SSS_FLAG_RANGE as above.
 * Errors: SSS_E_ARG, SSS_E_ALIGN, SSS_E_UNSUPPORTED, SSS_E_WORKSPACE, SSS_E_CUDA.
 */
sss_status_t sss_gemm(const sss_qtensor_t* qt, const uint16_t* x_bf16,
                      int64_t m, float* y, void* workspace, size_t ws_bytes,
                      uint32_t* dev_status, void* stream);

/*
 * sss_gemm_multi -- sss_gemm for several packed matrices that share one
 * activation matrix (e.g. the q/k/v or gate/up projections of a layer) in
 * one launch: Y_j[m][r] = sum_k w^_j[r][k] * X[m][k] (same arithmetic as
 * sss_gemm, Appendix B.3).  X is converted to fp16 once, and the output
 * tiles of all the matrices share one grid, so small matrices (k/v) fill
 * the SMs together with the others instead of splitting K.
 *   qts   [in]  count pointers to packed tensors with equal k, q, group and
 *               grid; each n % 4 == 0; codes 16-byte aligned.  Tensors with
 *               n == 0 are skipped.
 *   ys    [out] count device fp32 pointers, Y_j [m][n_j], 16-byte aligned.
 *   count [in]  1..4.
 *   x_bf16, m, workspace, ws_bytes, dev_status, stream: as sss_gemm, with
 *               the workspace sized by sss_gemm_multi_workspace_bytes (the
 *               fp16 copy of X, m*k*2 bytes, is enough to run unsplit).
 * Errors: SSS_E_ARG (count, mismatched tensors), SSS_E_ALIGN,
 * SSS_E_UNSUPPORTED, SSS_E_WORKSPACE, SSS_E_CUDA.
 */
sss_status_t sss_gemm_multi(const sss_qtensor_t* const* qts, float* const* ys,
                            int32_t count, const uint16_t* x_bf16, int64_t m,
                            void* workspace, size_t ws_bytes,
                            uint32_t* dev_status, void* stream);

/* Workspace bytes that let sss_gemm_multi take its preferred plan (0 for
 * invalid arguments or an empty call). */
size_t sss_gemm_multi_workspace_bytes(const sss_qtensor_t* const* qts,
                                      int32_t count, int64_t m);

/*
 * sss_gemm_q8 -- sss_gemm on Q8_0 activations: each token's X is quantized
 * per block of 32 (sss_quantize_act_q8) and the GEMM multiplies the packed
 * weights with fl16(fl16(d) * q), the fp16 operand of the tensor cores (one
 * rounding, <= 2^-11 relative).  This is the runtime pairing of few-bit
 * weights with 8-bit activations the paper deploys (Sec. 5 "Composition with
 * PTQ methods"; Appendix B.3 product).  Arguments, layouts, workspace and
 * errors as sss_gemm; dev_status also receives the activation flags of
 * sss_quantize_act_q8.
 */
sss_status_t sss_gemm_q8(const sss_qtensor_t* qt, const uint16_t* x_bf16,
                         int64_t m, float* y, void* workspace, size_t ws_bytes,
                         uint32_t* dev_status, void* stream);

/*
 * sss_quantize_act_q8 -- Q8_0 activations, the narrow-range 8-bit format the
 * paper pairs with its weight formats (Sec. 5 "Composition with PTQ
 * methods"; Appendix C "Algorithm details"): per block of 32 consecutive
 * values of a row, M = max |x|, d = fl32(M / 127), q = clip(RNE(x / d) of
 * the exact quotient, -127, 127), stored scale fl16(d).  A zero block gives
 * q = 0, d = +0; a block with NaN/Inf gives q = 0, d = +0 and
 * SSS_FLAG_NONFINITE; an fp16 overflow of d raises SSS_FLAG_RANGE.
 *   x_bf16 [in]  device bf16 [rows][k], 16-byte aligned; k % 32 == 0.
 *   q      [out] device int8 [rows][k], 8-byte aligned.
 *   d      [out] device fp16 [rows][k/32].
 * Errors: SSS_E_ARG, SSS_E_ALIGN, SSS_E_CUDA.
 */
sss_status_t sss_quantize_act_q8(const uint16_t* x_bf16, int64_t rows, int64_t k,
                                 int8_t* q, uint16_t* d, uint32_t* dev_status,
                                 void* stream);

/*
 * Normalized Hadamard rotation of the weights before quantization: the
 * mergeable rotations of the paper's PTQ pipeline (Sec. 5 "Composition with
 * PTQ methods"; Appendix C, the rotation graph), folded into the weights so
 * that the grids are computed on the rotated weights and the runtime path
 * is unchanged.  The transform of a block of b values (b a power of two,
 * 2 <= b <= 8192) is the normalized Walsh-Hadamard transform H_b/sqrt(b)
 * (Sylvester order) computed as the in-place fast transform in IEEE fp32:
 * strides h = 1, 2, ..., b/2, butterflies (a, c) -> (a + c, a - c), then
 * every value times the fp32 nearest to 1/sqrt(b).  H_b/sqrt(b) is
 * symmetric and orthogonal: W x = (W R)(R x) for R = I (x) H_b/sqrt(b).
 */
#define SSS_ROTATE_INPUT 0  /* W <- W R: every block of b consecutive values of a row (b | k,
                               k a multiple of 4)                                            */
#define SSS_ROTATE_OUTPUT 1 /* W <- R W: every block of b consecutive rows, per column
                               (b | n, and k a multiple of 8192/b)                          */

/*
 * sss_hadamard -- rotate the fp32 matrix w [n][k] into out [n][k] (out may
 * equal w).  Both 16-byte aligned.
 * Errors: SSS_E_ARG (block, side or shape), SSS_E_ALIGN, SSS_E_CUDA.
 */
sss_status_t sss_hadamard(const float* w, float* out, int64_t n, int64_t k,
                          int32_t block, int32_t side, void* stream);

/*
 * sss_quantize_rotated -- sss_quantize of the input-side rotation of w:
 * bit for bit sss_hadamard(w, tmp, n, k, block, SSS_ROTATE_INPUT) followed
 * by sss_quantize(tmp, out, ...), in one pass that never writes the rotated
 * fp32 weights (block | k).  Arguments and errors as sss_quantize.
 */
sss_status_t sss_quantize_rotated(const float* w, int32_t block, const sss_qtensor_t* out,
                                  uint8_t* clip_counts, uint32_t* dev_status,
                                  void* stream);

/*
 * sss_quantize_lsq -- symmetric-grid quantization with every group's scale
 * refined by LSQ steps (Sec. 5 "Composition with learned rotations and grid
 * parameters"; Appendix C: LSQ, the scale constrained to s != 0 for the
 * signed formats and s > 0 for the conventional ones).  The paper learns
 * the scales through the model loss on calibration data; this is the
 * data-free reading on each group's reconstruction loss L(s) =
 * sum (s c_i - w_i)^2, in IEEE fp32 without fused multiply-add:
 *   s_0 = gamma* alpha (SIGNED) or alpha (UNSIGNED), as sss_quantize;
 *   each step: v_i = w_i / s, c_i = clip(rint(v_i)), d_i = c_i - v_i inside
 *   the alphabet and the clip value outside (LSQ's straight-through
 *   derivative of w^_i = s c_i), t_i = (2 (s c_i - w_i)) d_i, G = the
 *   pairwise sum t_i <- t_i + t_{i+h} (h = g/2, ..., 1),
 *   s <- s - (lr / sqrt(g (2^(q-1) - 1))) G, and a step that would cross or
 *   reach zero halves s instead, so the sign is kept;
 *   then codes c = clip(RNE(w / s)) of the exact quotient and fp16 s, in the
 *   layout of sss_quantize.  steps = 0 reproduces sss_quantize.
 *   out   [in]  as sss_quantize; grid SIGNED_SYM or UNSIGNED_SYM.
 *   steps [in]  >= 0;  lr [in] >= 0.
 * Errors: SSS_E_ARG, SSS_E_ALIGN, SSS_E_UNSUPPORTED (ASYM), SSS_E_CUDA.
 */
sss_status_t sss_quantize_lsq(const float* w, const sss_qtensor_t* out, int32_t steps,
                              float lr, uint32_t* dev_status, void* stream);

/*
 * sss_sign_diagnostics -- the cardinality margin and the realised l2 gain of
 * the signed absmax sign rule on every group (Sec. 4, rem:cardinality-margin
 * and fig:theory-diagnostics), on any fp32 weights: for the sign gamma* of
 * eq:sign_rule and the clipped sets of def:clipped-set,
 *   margin m = |C_-gamma*| - |C_gamma*|            (in -group .. group)
 *   gain   g = ||w - Q_-gamma*(w)||^2 - ||w - Q_gamma*(w)||^2
 * with the weights each sign's stored fp16 scale dequantises to.  g is
 * exact (fp64).  Groups with NaN/Inf are skipped and raise
 * SSS_FLAG_NONFINITE; all-zero groups count as m = 0, g = 0.
 *   w      [in]  device fp32 [n][k], 16-byte aligned; k % group == 0.
 *   q      [in]  2, 3 or 4;  group 32, 64 or 128.
 *   margin [out] nullable device int16 [n][k/group].
 *   gain   [out] nullable device fp64 [n][k/group].
 *   hist   [in,out] nullable device uint64 [2*group+1][3], ADDED to: row
 *                m + group, column 0 (g < 0), 1 (g == 0) or 2 (g > 0).
 * Errors: SSS_E_ARG, SSS_E_ALIGN, SSS_E_CUDA.
 */
sss_status_t sss_sign_diagnostics(const float* w, int64_t n, int64_t k, int32_t q,
                                  int32_t group, int16_t* margin, double* gain,
                                  uint64_t* hist, uint32_t* dev_status, void* stream);

/*
 * Between a layer's {q, k, v} projection and its o_proj: a paged key/value
 * cache, what fills it and the attention that reads it.  The paper's path ends
 * at the projections (the weights are what it quantizes); these calls take
 * sss_gemm_multi's or sss_gemv's fp32 outputs to the bf16 activations that the
 * next projection reads.
 *
 * The cache of a layer is a matrix of slots, a slot per token: slot s holds the
 * token's keys (and values) of every key/value head.  A page is page_size
 * consecutive slots; request b's token at position p lies in slot
 * block_table[b][p / page_size] * page_size + p % page_size.
 */
typedef struct {
  void* k;           /* [slots][heads][dim], slots `stride` elements apart                 */
  void* v;           /* as k                                                               */
  int64_t slots;     /* 0 .. 2^31 - 1                                                      */
  int64_t stride;    /* >= heads * dim and a multiple of 8 (heads * dim where it is dense) */
  int32_t page_size; /* 16, 32, 64, 128 or 256 with a block table; else ignored            */
  int32_t heads;     /* key/value heads, 1 ..                                              */
  int32_t dim;       /* 64 or 128                                                          */
  int32_t dtype;     /* SSS_OUT_F16 or SSS_OUT_BF16                                        */
} sss_kv_cache_t;

/*
 * sss_page_plan -- a step's pages and slots from its requests' lengths: request
 * b holds the pages of past[b] tokens and gets fresh[b] new ones.  The
 * ceil((past + fresh) / page_size) - ceil(past / page_size) pages that it lacks
 * are taken from the front of free_pages, requests in order, and entered in its
 * row of the block table.  One launch; nothing is read back.
 *   past, fresh  [in]  device int32 [batch], >= 0.
 *   page_size    [in]  16, 32, 64, 128 or 256.
 *   free_pages   [in]  device int32 [free_count]: pages that no request holds.
 *   block_table  [in,out] device int32 [batch][table_width]: entries below
 *                      ceil(past / page_size) are read, the taken pages' written,
 *                      others left alone.
 *                      A partly filled last page is written to by the new tokens: no
 *                      other request may hold it (sss_page_fork sees to that).
 *   cu_q         [out] device int32 [batch + 1]: the first token of each request
 *                      among the step's, and their number.
 *   kv_len       [out] device int32 [batch]: past + fresh (of the tokens that cu_q has).
 *   positions    [out] device int32 [tokens]: each new token's position.
 *   slots        [out] device int32 [tokens]: its slot.  Rows past the step's
 *                      tokens get position 0 and slot -1 (a buffer may be larger
 *                      than the step, as in a captured graph).
 *   used         [out] device int32: how many of free_pages were taken (also for tokens
 *                      that are past `tokens` or past the table's columns).
 *   dev_status   [out] nullable.  SSS_FLAG_PAGES: free pages or table columns do
 *                      not suffice; the tokens without a page get slot -1 (and
 *                      the table -1).  SSS_FLAG_INDEX: a length is negative
 *                      (taken as 0), the new tokens are more than `tokens` (cu_q
 *                      ends there), or an entry of a held page is not one (slot
 *                      -1).
 * Errors: SSS_E_ARG, SSS_E_ALIGN, SSS_E_CUDA.
 */
sss_status_t sss_page_plan(const int32_t* past, const int32_t* fresh, int32_t batch,
                           int32_t page_size, const int32_t* free_pages, int32_t free_count,
                           int32_t* block_table, int32_t table_width, int32_t* cu_q,
                           int32_t* kv_len, int32_t* positions, int32_t* slots,
                           int64_t tokens, int32_t* used, uint32_t* dev_status,
                           void* stream);

#define SSS_ROPE_HALF 0  /* pairs (i, i + rot_dim / 2) */
#define SSS_ROPE_PAIRS 1 /* pairs (2i, 2i + 1)         */

/* The rotation of a model's heads, and their norm if it has one. */
typedef struct {
  const float* cos;    /* device fp32 [max_pos][rot_dim / 2]                             */
  const float* sin;    /* as cos                                                         */
  const float* q_norm; /* nullable device fp32 [dim]: the weights of the query heads' norm */
  const float* k_norm; /* nullable, of the key heads'                                    */
  int64_t max_pos;
  int32_t rot_dim;     /* values of a head that are rotated, from its first: 0 .. dim, a
                          multiple of 8                                                  */
  int32_t style;       /* SSS_ROPE_HALF or SSS_ROPE_PAIRS                                */
  float eps;           /* >= 0                                                           */
} sss_rope_t;

/*
 * sss_qk_norm_rope -- per head x of q and k: y = x / sqrt(mean(x^2) + eps) * w
 * (where the norm's weights are given), then each pair (a, b) of y's first
 * rot_dim values turned by the token's angle i: (a cos_i - b sin_i, b cos_i + a
 * sin_i).  q is rounded to q_out, k and the unchanged v to the token's slot of
 * the cache.  fp32 arithmetic, one rounding.
 *   q, k, v    [in]  device [tokens][heads * dim] and [tokens][cache->heads * dim]
 *                    of in_dtype (sss_dtype_t; fp32 is what the projections
 *                    write), rows q_stride, k_stride and v_stride elements apart
 *                    (multiples of 4: the three may be columns of one matrix);
 *                    16-byte aligned (16-bit types: 8).
 *   heads      [in]  query heads, any number.
 *   rope       [in]  16-byte aligned arrays; cos and sin may be NULL at rot_dim 0.
 *   positions  [in]  device int32 [tokens] (may be NULL at rot_dim 0).
 *   q_out      [out] device [tokens][heads][dim] of the cache's dtype, dense,
 *                    16-byte aligned.
 *   cache      [in]  written at the tokens' slots.
 *   slots      [in]  device int32 [tokens], no two alike; negative: the token's
 *                    key and value are not kept.  NULL: token t's slot is t (a
 *                    prompt whose keys are packed as its tokens are).
 *   dev_status [out] nullable.  SSS_FLAG_INDEX: a slot past the cache (not
 *                    written), or a position outside 0 .. max_pos - 1 (the
 *                    nearest is taken).
 * Errors: SSS_E_ARG, SSS_E_UNSUPPORTED (dim), SSS_E_ALIGN, SSS_E_CUDA.
 */
sss_status_t sss_qk_norm_rope(const void* q, int64_t q_stride, const void* k, int64_t k_stride,
                              const void* v, int64_t v_stride, int32_t in_dtype,
                              int64_t tokens, int32_t heads, const sss_rope_t* rope,
                              const int32_t* positions, void* q_out,
                              const sss_kv_cache_t* cache, const int32_t* slots,
                              uint32_t* dev_status, void* stream);

/*
 * sss_attention -- causal attention of each request's new tokens over its keys
 * and values: with n new tokens (cu_q[b] .. cu_q[b + 1] - 1) and kv_len[b] keys,
 * token i sees keys 0 .. kv_len - n + i, and
 *   o_i = sum_j p_ij v_j / sum_j p_ij,  p_ij = exp(scale q_i.k_j - max_j).
 * A whole prompt (kv_len = n), a chunk of one after what the cache holds, a
 * single token (n = 1) and drafted ones are the same call, and a batch may mix
 * them.  Query head h reads key/value head h / (heads / cache->heads).  A row
 * that sees no key (or none whose score is above minus infinity) is zero.  Scores, sums and outputs are held in fp32; p_ij is
 * rounded to the cache's type for its product with v_j (relative to a maximum
 * that may lie 8 powers of two below the row's own), the output once.
 * Keys and values that a row does not see have no part in it, whatever they
 * hold (infinities and NaN among them); what lies in the cache past kv_len is
 * never used.  An infinity that a row sees makes its output infinite, or NaN where
 * its p_ij is too small for the cache's type.
 *   q           [in]  device [tokens][heads][dim] of the cache's dtype, rows
 *                     q_stride elements apart (a multiple of 8, >= heads * dim);
 *                     16-byte aligned.
 *   heads       [in]  a multiple of cache->heads, at most 16384.
 *   cache       [in]  k and v 16-byte aligned.
 *   batch, tokens [in] at most 65535 and 2^24.
 *   cu_q        [in]  device int32 [batch + 1], cu_q[batch] <= tokens.  Rows of no
 *                     request are not written.
 *   kv_len      [in]  device int32 [batch].
 *   block_table [in]  device int32 [batch][table_width], or NULL: key j of request
 *                     b lies in slot cu_q[b] + j (keys packed as the queries;
 *                     kv_len may then be NULL: the request's new tokens).
 *   max_q, max_kv [in] bounds of a request's new tokens and keys; what is near
 *                     them is faster.  max_q may be any (above `tokens` it counts as
 *                     that), max_kv at most 2^30 - 1.
 *   scale       [in]  > 0, at most 2.3e38.
 *   out         [out] device [tokens][heads][dim] of the cache's dtype, dense,
 *                     16-byte aligned (bf16: the x_bf16 of the o_proj).
 *   workspace   [in]  device scratch of ws_bytes >=
 *                     sss_attention_workspace_bytes(...) bytes, 16-byte aligned,
 *                     or NULL when that size is 0.  Contents on entry are ignored.
 *   dev_status  [out] nullable.  SSS_FLAG_INDEX: cu_q, kv_len or the table point
 *                     outside what they may (a request past `tokens` is left
 *                     out, lengths are cut to max_q, max_kv, the table's width or
 *                     the request's own rows, a page that is none reads as zeros).
 *                     SSS_FLAG_TIMEOUT: a bounded wait ran out.
 * The result does not depend on timing, and a request's not on the others in the
 * batch but through `tokens`, max_q, max_kv and their number, by which the work is
 * split (a split changes the order of the sums, so the last bits).
 * Errors: SSS_E_ARG, SSS_E_UNSUPPORTED (dim; a driver without tensor maps),
 * SSS_E_ALIGN, SSS_E_WORKSPACE, SSS_E_CUDA.
 */
sss_status_t sss_attention(const void* q, int64_t q_stride, int32_t heads,
                           const sss_kv_cache_t* cache, const int32_t* cu_q,
                           const int32_t* kv_len, const int32_t* block_table,
                           int32_t table_width, int32_t batch, int64_t tokens,
                           int32_t max_q, int64_t max_kv, float scale, void* out,
                           void* workspace, size_t ws_bytes, uint32_t* dev_status,
                           void* stream);

/* Workspace bytes of that call (0 for invalid arguments, or if none are needed:
 * partial results where the keys of many rows are split over CTAs).  Fewer tokens
 * over the same keys may need more, as they are split where SMs would idle: a buffer
 * for several shapes is the largest of their sizes. */
size_t sss_attention_workspace_bytes(int64_t tokens, int32_t heads,
                                     const sss_kv_cache_t* cache, int32_t batch,
                                     int32_t max_q, int64_t max_kv);

/*
 * The same cache in 4 bits: keys and values on the signed symmetric grid of the
 * weights (eq:signed_sym_quant, eq:sign_rule), in groups of 32 consecutive values of a
 * head: M = max |x|, s = -M/8 where the dominant value is positive, else M/8 (so it lands
 * on the code -8), c = clip(RNE(x / s), -8, 7) of the exact quotient.  The value that is
 * held is fp16(s) c.  9/16 of a byte a value against 2: a decode step reads its keys and
 * values 3.6 times as fast.
 *
 * Pages are as above.  A page holds, per key/value head, page_size / 16 blocks of 16
 * slots; a block is 18 * dim bytes that lie together (one bulk copy brings a block):
 * the 16 keys' codes (8 * dim bytes, dim / 2 to a slot), their scales (fp16, dim / 32 to a
 * slot), then the values' codes and scales.  With W = dim / 8 words of 32 bits to a slot's
 * codes, word w holds as its nibble n = a + 4 h (the lowest is 0) the stored code c + 8
 * of dimension 2 W a + W h + w.  The values' words of slots whose number has bit 1 set
 * have their halves swapped where dim is 128 (word w lies at w ^ 8).
 */
typedef struct {
  void* blocks;        /* [pages][heads][page_size / 16][18 * dim] bytes, 16-byte aligned  */
  int64_t pages;       /* 0 .. 2^31 / page_size - 1                                        */
  int64_t page_stride; /* bytes from a page to the next: at least heads * page_size / 16 *
                          18 * dim, a multiple of 16                                       */
  int32_t page_size;   /* 16, 32, 64, 128 or 256                                           */
  int32_t heads;       /* key/value heads, 1 ..                                            */
  int32_t dim;         /* 64 or 128                                                        */
  int32_t reserved;    /* must be 0                                                        */
} sss_kv_cache_q4_t;

/*
 * sss_kv_store_q4 -- keys and values into the cache, in 4 bits (of sss_qk_norm_rope, say,
 * whose packed output the prompt attends to at full precision).
 *   k, v       [in]  device [tokens][heads * dim] of in_dtype (sss_dtype_t), rows k_stride
 *                    and v_stride elements apart (multiples of 8; fp32: of 4); 16-byte
 *                    aligned.
 *   slots      [in]  device int32 [tokens], no two alike; negative: the token is not kept.
 *                    NULL: token t's slot is t.
 *   dev_status [out] nullable.  SSS_FLAG_NONFINITE: a group holds an infinity or NaN; it is
 *                    stored as zeros.  SSS_FLAG_RANGE: a scale is 65520 or more and
 *                    stored as 65504.  SSS_FLAG_INDEX: a slot past the cache (not written).
 * Errors: SSS_E_ARG, SSS_E_UNSUPPORTED (dim), SSS_E_ALIGN, SSS_E_CUDA.
 */
sss_status_t sss_kv_store_q4(const void* k, int64_t k_stride, const void* v, int64_t v_stride,
                             int32_t in_dtype, int64_t tokens, const sss_kv_cache_q4_t* cache,
                             const int32_t* slots, uint32_t* dev_status, void* stream);

/*
 * sss_kv_fetch_q4 -- what the cache holds in the given slots, any number of times each:
 * fp16(s) c, exact in fp32, rounded once to a 16-bit out_dtype.
 *   slots      [in]  device int32 [count]; negative: the row is zeros.  NULL: row t is
 *                    slot t.
 *   k, v       [out] nullable device [count][heads][dim] of out_dtype, 16-byte aligned.
 *   dev_status [out] nullable.  SSS_FLAG_INDEX: a slot past the cache (zeros).
 * Errors: SSS_E_ARG, SSS_E_UNSUPPORTED (dim), SSS_E_ALIGN, SSS_E_CUDA.
 */
sss_status_t sss_kv_fetch_q4(const sss_kv_cache_q4_t* cache, const int32_t* slots, int64_t count,
                             void* k, void* v, int32_t out_dtype, uint32_t* dev_status,
                             void* stream);

/*
 * sss_attention_q4 -- sss_attention over the cache in 4 bits: the same requests, rows,
 * bounds and flags, always with a block table (so with kv_len).  The new tokens' own keys
 * and values are in the cache, as the others are.
 *   dtype [in]  of q and out: SSS_OUT_F16 or SSS_OUT_BF16.
 * A request's tokens times the heads of a group at most 64 (or single tokens): scores are
 * sums of q times the codes, scaled in fp32; p_ij times the value's scale is rounded to fp16
 * (for bf16 p_ij is rounded first) with a power of two taken off the row: below fp16's normal
 * range it is at most 2^-35 off, a row's largest p_ij being 1, as long as the scales that the
 * row sees are below 32, and 2^-39 of the largest scale from there on.
 * More: the keys and values are first written to the workspace as fp16 values, fp16(s) c
 * rounded once (and bf16 q as fp16 with a power of two taken off each row), and p_ij is rounded
 * to fp16 (a row's largest being 1 to 2^8; for bf16 with a power of two more, so lost below
 * 2^-32 only).  A key or value above 65504 in size counts as 65504 there: SSS_FLAG_RANGE.
 * That copy makes most of the workspace: 4 bytes a key and dimension of a key/value head, for
 * max_kv keys (whole pages, as the table has) of each request, or of more than one request for
 * the cache's slots where those are fewer.  It goes by the call as a whole: one request of
 * many tokens takes the others' keys with it, so in a step that mixes chunks of prompts with
 * single tokens, calls of their own for either (parts of cu_q, kv_len and the table's rows)
 * are smaller and faster (63 single tokens of 12000 to 16384 keys and a chunk of 512 after 4000:
 * 1508 us and 3.7 GB in one, 241 us and 0.12 GB in two).
 * Errors: as sss_attention; SSS_E_UNSUPPORTED also where batch times max_kv (whole pages, as the
 * table has) is 2^31 or more with many rows.
 */
sss_status_t sss_attention_q4(const void* q, int64_t q_stride, int32_t heads, int32_t dtype,
                              const sss_kv_cache_q4_t* cache, const int32_t* cu_q,
                              const int32_t* kv_len, const int32_t* block_table,
                              int32_t table_width, int32_t batch, int64_t tokens, int32_t max_q,
                              int64_t max_kv, float scale, void* out, void* workspace,
                              size_t ws_bytes, uint32_t* dev_status, void* stream);

/* Workspace bytes of that call (0 for invalid arguments, or if none are needed). */
size_t sss_attention_q4_workspace_bytes(int64_t tokens, int32_t heads,
                                        const sss_kv_cache_q4_t* cache, int32_t table_width,
                                        int32_t batch, int32_t max_q, int64_t max_kv);

/*
 * What else a serving loop does with pages, of either cache: the block table says all that
 * there is to know of them, and several of its rows may hold the same page.
 *
 * sss_page_fork -- the rows of a new block table from those of the old one: beams or
 * samples that go on from their parents.  Row r takes over the pages of past[p] tokens of
 * p = parents[r].  Full pages are shared.  A last page that is only partly filled is
 * written to by the tokens that follow, so one row alone may hold it: the first of the new rows
 * that end in it keeps it, unless a new row holds it as a full page; each other one gets a free
 * page in its place (from the front of free_pages, rows in order) and the entry (src[r],
 * dst[r]) for sss_page_copy.  So a length may be cut into a page that other rows share (a request
 * that is rolled back, drafted tokens that are rejected): fork the rows before they get new
 * tokens, each from itself (parents 0, 1, 2 ...) if nothing else changes.  sss_page_plan alone
 * would have them write to the shared page.  Pages of rows that nobody takes over are
 * found by sss_page_reclaim on the new table.
 *   parents      [in]  device int32 [rows]; negative: the row is empty.
 *   past         [in]  device int32 [batch].
 *   block_table  [in]  device int32 [batch][table_width].
 *   new_table    [out] device int32 [rows][table_width], not block_table itself: all of
 *                      it is written, -1 behind a row's pages.
 *   new_past     [out] device int32 [rows], not past itself.
 *   src, dst     [out] device int32 [rows]: -1 where nothing is to be copied.
 *   used         [out] device int32: how many of free_pages were taken.
 *   dev_status   [out] nullable.  SSS_FLAG_PAGES: free pages do not suffice (an entry of -1
 *                      is none): the row ends with its last full page, new_past says so.
 *                      SSS_FLAG_INDEX: a parent past the batch (the row is empty), a
 *                      negative length (taken as 0), one that the table's columns do not
 *                      hold (cut to them), or a last page to copy that is none (the row ends
 *                      before it).
 * Errors: SSS_E_ARG, SSS_E_ALIGN, SSS_E_CUDA.
 */
sss_status_t sss_page_fork(const int32_t* parents, int32_t rows, const int32_t* past,
                           int32_t batch, int32_t page_size, const int32_t* free_pages,
                           int32_t free_count, const int32_t* block_table, int32_t table_width,
                           int32_t* new_table, int32_t* new_past, int32_t* src, int32_t* dst,
                           int32_t* used, uint32_t* dev_status, void* stream);

/*
 * sss_page_reclaim -- the free pages, from the block table: those of 0 .. pages - 1 that no
 * row holds among its first ceil(past / page_size) entries, in ascending order (so pages of
 * requests that ended, or whose length was cut, are free again, and shared ones once the
 * last row has let go of them).
 * With `moves` it compacts as well: the i-th lowest free page takes the i-th highest held
 * one, while that is the higher and i < most_moves.  src and dst get the moves for
 * sss_page_copy, new_table the held entries after them, free_pages what is then free.
 *   past         [in]  device int32 [batch].
 *   block_table  [in]  device int32 [batch][table_width].
 *   pages        [in]  of the cache, 0 .. 2^20.
 *   free_pages   [out] device int32 [pages]: -1 behind the free ones (as sss_page_plan
 *                      and sss_page_fork take it whole).
 *   free_count   [out] device int32.
 *   new_table    [out] device int32 [batch][table_width] (with moves): only held entries
 *                      are written; may be block_table itself.
 *   src, dst     [out] device int32 [most_moves] (with moves): -1 behind them.
 *   moves        [out] nullable device int32: their number.
 *   dev_status   [out] nullable.  SSS_FLAG_INDEX: a length is negative (taken as 0) or past
 *                      the table's columns (cut to them), or a held entry is no page (left
 *                      as it is).
 * Errors: SSS_E_ARG, SSS_E_ALIGN, SSS_E_CUDA.
 */
sss_status_t sss_page_reclaim(const int32_t* block_table, int32_t table_width,
                              const int32_t* past, int32_t batch, int32_t page_size,
                              int32_t pages, int32_t* free_pages, int32_t* free_count,
                              int32_t* new_table, int32_t* src, int32_t* dst, int32_t most_moves,
                              int32_t* moves, uint32_t* dev_status, void* stream);

/*
 * sss_page_copy, sss_page_copy_q4 -- page src[i] to page dst[i] in each of the caches (the
 * layers of a model), keys and values, as they are.
 *   caches     [in]  host array of `count` descriptors, 0 .. 128; not retained.  All have the
 *                    same page_size, heads, dim and number of pages (slots / page_size).
 *   src, dst   [in]  device int32 [n].  Both negative: no copy.  No page is the destination
 *                    of two copies, nor the source of one and the destination of another.
 *   dev_status [out] nullable.  SSS_FLAG_INDEX: only one of the two is negative, or one is
 *                    past the cache (not copied).
 * Errors: SSS_E_ARG, SSS_E_UNSUPPORTED (dim), SSS_E_ALIGN, SSS_E_CUDA.
 */
sss_status_t sss_page_copy(const sss_kv_cache_t* const* caches, int32_t count, const int32_t* src,
                           const int32_t* dst, int32_t n, uint32_t* dev_status, void* stream);
sss_status_t sss_page_copy_q4(const sss_kv_cache_q4_t* const* caches, int32_t count,
                              const int32_t* src, const int32_t* dst, int32_t n,
                              uint32_t* dev_status, void* stream);

#define SSS_OP_GEMV 0
#define SSS_OP_GEMM 1
/* Workspace bytes sss_gemv (op SSS_OP_GEMV, m_or_batch = batch) or sss_gemm
 * (op SSS_OP_GEMM, m_or_batch = m) needs for this tensor; 0 if none (or an
 * invalid tensor).  For sss_gemm this is the size that lets the call take
 * its fastest plan: the fp16 copy of X (m * k * 2 bytes, rounded up to 256),
 * plus, when the weight tiles are fewer than the SMs, room for fp32 partial
 * tiles of K split across CTAs (summed in a fixed order, so the result does
 * not depend on timing).  sss_gemm runs with any workspace that holds the
 * fp16 copy of X, unsplit when the partials do not fit. */
size_t sss_workspace_bytes(const sss_qtensor_t* qt, int64_t m_or_batch,
                           int32_t op);

/*
 * sss_gemm_noalloc -- sss_gemm with its scratch (the fp16 copy of X, m*k*2
 * bytes) in a static 32 MiB device array of the library instead of a
 * caller workspace.  The paper has no counterpart: this is a library
 * convenience for callers that cannot allocate device memory when they
 * call, e.g. a plain C host with no device allocator, or a serving loop
 * that must not call cudaMalloc (it synchronises the device and can fail
 * under memory pressure).  Nothing is allocated at call time.
 *   Arguments, layouts and errors as sss_gemm, without workspace/ws_bytes.
 *   Limit: m * k * 2 <= sss_gemm_noalloc_max_scratch_bytes() (33554432);
 *          larger calls return SSS_E_WORKSPACE (sss_last_error() says why).
 *   The first call on each device looks up the array's device address with
 *   that device current (set-up); make that first call before any stream
 *   capture begins.  Nothing in the scratch needs to start at zero.
 *   All calls on a device share the one array: calls that overlap in time
 *   (other streams, other host threads) race on it; callers serialise them.
 */
sss_status_t sss_gemm_noalloc(const sss_qtensor_t* qt, const uint16_t* x_bf16,
                              int64_t m, float* y, uint32_t* dev_status,
                              void* stream);
size_t sss_gemm_noalloc_max_scratch_bytes(void);

/*
 * sss_test_set_stall -- test hook for the bounded waits; the paper has no
 * counterpart.  While a bit below is set, every later launch of that kernel
 * family leaves one mbarrier one arrive short: the GEMM on the first
 * stage's weight tile, the attention of many rows on its first value tile (of few
 * rows whose keys are split over a cluster: on what a CTA's peers store into it).  The decode GEMV kernels (batch 1 and batched) have no data-dependent waits (their
 * warps meet only at CTA-wide barriers), so their bits have no effect.  The wait
 * on that barrier then runs out after its bound (about one second), the kernel
 * raises SSS_FLAG_TIMEOUT in dev_status, lets its own copies and MMAs in flight
 * finish, releases its tensor memory and returns; its output is incomplete.
 * Nothing faults or hangs.  mask = 0 (the default) restores normal launches.
 * Process-wide; affects launches issued (or captured) after the call on every
 * thread.
 */
#define SSS_TEST_STALL_GEMV 0x1u       /* gemv_stream_kernel: no waits, no effect               */
#define SSS_TEST_STALL_GEMV_BATCH 0x2u /* gemv_batch_kernel: no waits, no effect                */
#define SSS_TEST_STALL_GEMM 0x4u       /* gemm_kernel (sss_gemm, sss_gemm_noalloc)             */
#define SSS_TEST_STALL_ATTENTION 0x8u  /* attn_prompt_kernel (sss_attention of many rows): the
                                          first value tile is never handed on              */
#define SSS_TEST_STALL_ATTENTION_ROWS 0x10u /* attn_rows_kernel, attn_rows_q4_kernel (of few
                                          rows), where a cluster shares the keys: each CTA
                                          expects 16 bytes too many                        */
void sss_test_set_stall(uint32_t mask);

#ifdef __cplusplus
}
#endif
#endif /* SSS_H */
