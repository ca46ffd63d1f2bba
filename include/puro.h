/*
 * puro.h -- C ABI of the MI355X (gfx950) FP8 linear-layer library (libpuro.so).
 *
 * The operations are those of an FP8 linear layer as the paper states it
 * (Section 3.2, "FP8 Mixed-Precision Training"; Appendix C, "FP8
 * implementation pipeline" and the precision-flow figure): BF16 inputs and
 * weights are quantised to FP8 immediately before each GEMM, with scales
 * computed online from the data; Fprop (Y = X W^T), Dgrad (dX = dY W) and
 * Wgrad (dW = dY^T X) run on FP8 operands; Y and dX are written in BF16 and
 * dW accumulates in FP32; the quantised input is kept for Wgrad.
 *
 * Conventions for every entry point:
 *  - All tensor pointers are DEVICE pointers owned by the caller. The library
 *    never allocates, frees or synchronises; scratch memory is a caller
 *    workspace (`ws`, `ws_bytes`) sized by the matching *_workspace_size().
 *  - BF16 tensors are passed as their uint16_t bit patterns, FP8 tensors as
 *    uint8_t codes (OCP E4M3 "E4M3FN" or E5M2), scales as float.
 *  - Matrices are row-major; `ld` is the row pitch in elements.
 *  - Arguments are validated on the host before anything is enqueued; an
 *    error status means nothing was launched. On success the work is
 *    enqueued on `stream` and the call returns without waiting.
 *  - Results are deterministic: the same inputs give the same bytes.
 *  - Calls on one stream are ordered; calls that share a workspace must not
 *    run concurrently on different streams.
 *
 * Encoding (readings of the paper, which fixes the formats but not the
 * rounding): a value x is encoded as FP8(fl32(x * r)) with round-to-nearest-
 * even, saturation of finite and infinite magnitudes above the format's
 * largest value (448 for E4M3, 57344 for E5M2) and every NaN mapped to 0x7F.
 * Per-tensor scales: s = fl32(amax / FMAX), r = fl32(FMAX / amax) (s = r = 1
 * when amax = 0). Power-of-two scales: s = 2^e, r = 2^-e with e the smallest
 * integer such that amax <= FMAX * 2^e, clamped to [-127, 127] (e = 0 for
 * amax = 0). The stored scale is always the dequantisation scale s.
 */
#ifndef PURO_H
#define PURO_H

#include <stddef.h>
#include <stdint.h>

#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    PURO_OK = 0,
    PURO_ERR_NULL = 1,        /* a required pointer is NULL                              */
    PURO_ERR_SHAPE = 2,       /* negative size, ld smaller than the row, mismatched dims */
    PURO_ERR_UNSUPPORTED = 3, /* format / mode / rounding combination not provided       */
    PURO_ERR_ALIGN = 4,       /* size or pointer not a multiple the kernels need         */
    PURO_ERR_WORKSPACE = 5,   /* ws_bytes below the matching *_workspace_size()          */
    PURO_ERR_HIP = 6          /* a kernel launch reported an error                       */
} puro_status;

typedef enum { PURO_E4M3 = 0, PURO_E5M2 = 1 } puro_fp8_format;

/* Scale granularity (Section 3.2: one scale per tensor, or groups of 128
 * consecutive values along a GEMM's reduction dimension for activations and
 * gradients, and 128x128 blocks for weights). */
typedef enum {
    PURO_SCALE_TENSOR = 0,        /* one scale                                          */
    PURO_SCALE_ROW_1x128 = 1,     /* one scale per row per 128 consecutive columns      */
    PURO_SCALE_COL_128x1 = 2,     /* one scale per column per 128 consecutive rows      */
    PURO_SCALE_BLOCK_128x128 = 3, /* one scale per 128x128 block                        */
    PURO_SCALE_KMAJOR = 0x100     /* layout flag of the grouped modes (below)           */
} puro_scale_mode;

/* PURO_SCALE_KMAJOR is a layout flag of the grouped modes, OR-ed into a puro_scale_mode argument
 * (the quantise calls) or into puro_fp8_operand.mode (the GEMM): the scale
 * array is stored k-block-major, the index of the 128-wide group along the
 * reduction dimension of the GEMM that reads the codes outermost. Without it
 * grouped scales are row-major. The GEMM then loads each k block's scales as
 * one contiguous run; the linear layer keeps its scales this way. Layouts:
 *   quantise ROW_1x128:     scale  [cols/128][rows], scaleT [rows/128][cols]
 *   quantise COL_128x1:     scaleT [rows/128][cols]
 *   quantise BLOCK_128x128: scale  [cols/128][rows/128], scaleT [rows/128][cols/128]
 *   GEMM operand [rows, K]: ROW_1x128 scale[(k/128) * rows + row],
 *                           BLOCK_128x128 scale[(k/128) * ceil(rows/128) + row/128]
 * With TENSOR it is PURO_ERR_UNSUPPORTED. */

/* Scale value rule. Section 3.2: block scales are powers of two (the
 * exponent-only E8M0 representation of MXFP8). */
typedef enum {
    PURO_SCALE_FP32 = 0, /* s = amax / FMAX in binary32 (per-tensor mode only) */
    PURO_SCALE_POW2 = 1, /* s = 2^e, the smallest power of two that avoids saturation */
    PURO_SCALE_POW2_FLOOR = 2 /* s = 2^(floor(log2 amax) - emax), the OCP-MX rule (emax 8 for
                                 E4M3, 15 for E5M2): the largest values of a group whose amax
                                 has a significand above 1.75 saturate. For comparison. */
} puro_scale_rounding;

typedef enum { PURO_OUT_BF16 = 0, PURO_OUT_FP32 = 1 } puro_out_dtype;

/* Static text for a status code (never NULL). */
const char* puro_status_string(puro_status status);

/* ---------------------------------------------------------------- amax ---
 * amax = max |x| over the [rows, cols] BF16 tensor x (row pitch ld), written
 * as one float to the device scalar `amax`. NaN if any element is NaN; 0 for
 * an empty tensor; -0 counts as 0. Section 3.2 computes scales online from
 * the data; this is the per-tensor statistic they come from.
 * Requirements: cols % 8 == 0, ld % 8 == 0, x 16-byte aligned (rows of whole
 * 16-byte vectors). ws: puro_amax_workspace_size(rows, cols) bytes. */
size_t puro_amax_workspace_size(int64_t rows, int64_t cols);
puro_status puro_amax(const uint16_t* x, int64_t rows, int64_t cols, int64_t ld,
                      float* amax, void* ws, size_t ws_bytes, hipStream_t stream);

/* ------------------------------------------------------------ quantise ---
 * Quantise the [rows, cols] BF16 tensor x (row pitch ld) to FP8 `fmt`.
 * Section 3.2: activations and activation gradients in 1x128 groups along the
 * reduction dimension, weights in 128x128 blocks, or one scale per tensor.
 *
 *  mode TENSOR: q [rows, cols] and/or qT [cols, rows] (the same codes,
 *      transposed); scale[0] = s. rnd FP32, POW2 or POW2_FLOOR. If amax_in is not NULL
 *      the device scalar *amax_in is used instead of the tensor's own amax
 *      (values beyond it saturate).
 *  mode ROW_1x128: q [rows, cols], scale [rows, cols/128]. If qT is not NULL
 *      the same read also writes the column-grouped copy: qT [cols, rows]
 *      with scaleT [cols, rows/128] (128x1 groups down each column, as
 *      Wgrad needs; quantised from the BF16 values, not from q).
 *  mode COL_128x1: only qT [cols, rows] and scaleT [cols, rows/128].
 *  mode BLOCK_128x128: q [rows, cols] with scale [rows/128, cols/128], and
 *      if qT is not NULL also qT [cols, rows] with scaleT [cols/128, rows/128]
 *      (the same codes and scales, transposed).
 *  Grouped modes require rnd == POW2 or POW2_FLOOR, and amax_in == NULL.
 *
 * Requirements: cols % 16 == 0 and ld % 8 == 0 with x 16-byte aligned;
 * ld < 2^23 (else PURO_ERR_SHAPE); rows % 16 == 0 when qT is written; the
 * grouped dimension(s) % 128 == 0.
 * Outputs are dense (row pitch = their column count). ws:
 * puro_quantize_workspace_size(rows, cols) bytes (used in TENSOR mode). */
size_t puro_quantize_workspace_size(int64_t rows, int64_t cols);
puro_status puro_quantize_fp8(const uint16_t* x, int64_t rows, int64_t cols, int64_t ld,
                              puro_fp8_format fmt, puro_scale_mode mode, puro_scale_rounding rnd,
                              const float* amax_in, uint8_t* q, float* scale,
                              uint8_t* qT, float* scaleT, void* ws, size_t ws_bytes,
                              hipStream_t stream);

/* For callers that cannot allocate (code under HIP graph capture, tight
 * serving loops, harnesses that forbid hipMalloc): puro_quantize_fp8 without
 * a workspace. The per-tensor mode's amax pass keeps its partial maxima in a
 * library-owned static device array of PURO_QUANTIZE_STATIC_SCRATCH_BYTES
 * (32 KiB) on each GPU it runs on, held until the process ends (its address is
 * looked up on the first such call on a device); nothing is allocated or freed.
 * Every call on one GPU shares that array: calls that overlap on one GPU (on
 * different streams, or from different threads without ordering) race and
 * may give wrong scales; order them on one stream. The partials are written
 * in full by each call, so nothing needs clearing. Sizes whose partials would
 * not fit return PURO_ERR_WORKSPACE (the quantiser uses at most 4096 partials,
 * which always fit). Arguments, outputs and errors otherwise as
 * puro_quantize_fp8; grouped modes and a supplied amax use no scratch. */
#define PURO_QUANTIZE_STATIC_SCRATCH_BYTES 32768
puro_status puro_quantize_fp8_static(const uint16_t* x, int64_t rows, int64_t cols, int64_t ld,
                                     puro_fp8_format fmt, puro_scale_mode mode, puro_scale_rounding rnd,
                                     const float* amax_in, uint8_t* q, float* scale, uint8_t* qT, float* scaleT,
                                     hipStream_t stream);

/* ------------------------------------------------- SwiGLU + quantise ---
 * The MLP of the paper's model (the Qwen3-1.7B architecture, Section 2)
 * computes down(silu(gate(x)) * up(x)); the hidden flow stays BF16 and the
 * down projection quantises its input right before its GEMM (Section 3.2,
 * Appendix C precision flow). This call fuses the two: from the fused
 * gate/up output gu [rows, 2 cols] (gate = columns [0, cols), up = columns
 * [cols, 2 cols), row pitch ld elements) it forms H = silu(gate) * up with
 * silu(g) = g / (1 + e^-g) in binary32, rounds H to BF16 (nearest even) and
 * quantises that H exactly as puro_quantize_fp8 would quantise a BF16 tensor
 * holding it, without writing H. The BF16 value of H can differ in its last
 * bit from another binary32 evaluation of exp; the codes and scales are
 * those of the H this call forms.
 *
 * Modes: TENSOR (q and/or qT; scale[0]; rnd FP32, POW2 or POW2_FLOOR; the
 * tensor's amax comes from a first pass over gu), ROW_1x128 (q, scale and
 * optionally the 128x1 column-grouped qT, scaleT) and COL_128x1 (qT,
 * scaleT), with the layouts of puro_quantize_fp8. BLOCK_128x128 returns
 * PURO_ERR_UNSUPPORTED (weights, not activations, take 128x128 blocks).
 *
 * Requirements: those of puro_quantize_fp8 with the BF16 matrix being gu
 * [rows, 2 cols] (ld >= 2 cols, ld % 8 == 0, ld < 2^23, gu 16-byte aligned)
 * and cols % 16 == 0. ws: puro_swiglu_quantize_workspace_size(rows, cols)
 * bytes (used in TENSOR mode). All pointers are device memory owned by the
 * caller; nothing is allocated or synchronised. */
size_t puro_swiglu_quantize_workspace_size(int64_t rows, int64_t cols);
puro_status puro_swiglu_quantize_fp8(const uint16_t* gu, int64_t rows, int64_t cols, int64_t ld,
                                     puro_fp8_format fmt, puro_scale_mode mode, puro_scale_rounding rnd,
                                     uint8_t* q, float* scale, uint8_t* qT, float* scaleT, void* ws,
                                     size_t ws_bytes, hipStream_t stream);

/* ---------------------------------------- SwiGLU backward + quantise ---
 * The gate/up projection's Dgrad and Wgrad take the gradient of its output
 * quantised (Section 3.2); that gradient is the SwiGLU's backward. From dH
 * [rows, cols] (the down projection's Dgrad output; row pitch ld_dh) and
 * the saved gate/up output gu [rows, 2 cols] (gate = columns [0, cols), up =
 * columns [cols, 2 cols); row pitch ld_gu) this call forms dgu [rows,
 * 2 cols] = [dg | du] with dg = dH * u * silu'(g), silu'(g) = s (1 + g (1 - s)),
 * s = 1 / (1 + e^-g), and du = dH * silu(g), each in binary32 rounded once to
 * BF16, and quantises dgu exactly as puro_quantize_fp8 would quantise a BF16
 * tensor holding it, without writing it: q [rows, 2 cols] for Dgrad and the
 * transposed qT [2 cols, rows] for Wgrad.
 *
 * Modes: TENSOR (q and/or qT; scale[0]; rnd FP32, POW2 or POW2_FLOOR),
 * ROW_1x128 (q, scale [rows, 2 cols / 128] and optionally the 128x1
 * column-grouped qT, scaleT) and COL_128x1 (qT, scaleT); BLOCK_128x128
 * returns PURO_ERR_UNSUPPORTED.
 *
 * Requirements: dH [rows, cols] and gu [rows, 2 cols] meet puro_quantize_fp8's
 * requirements for x; cols % 8 == 0 (2 cols % 16 == 0); the grouped
 * dimension(s) of dgu % 128 == 0. ws: puro_swiglu_bwd_quantize_workspace_size
 * (rows, cols) bytes (used in TENSOR mode). All pointers are device memory
 * owned by the caller; nothing is allocated or synchronised. */
size_t puro_swiglu_bwd_quantize_workspace_size(int64_t rows, int64_t cols);
puro_status puro_swiglu_bwd_quantize_fp8(const uint16_t* dh, int64_t ld_dh, const uint16_t* gu, int64_t ld_gu,
                                         int64_t rows, int64_t cols, puro_fp8_format fmt, puro_scale_mode mode,
                                         puro_scale_rounding rnd, uint8_t* q, float* scale, uint8_t* qT,
                                         float* scaleT, void* ws, size_t ws_bytes, hipStream_t stream);

/* ------------------------------------------------ RMSNorm + quantise ---
 * Every attention and MLP block of the paper's model (the Qwen3-1.7B
 * architecture, Section 2) starts with an RMSNorm whose output is the input
 * of the QKV or gate/up projection; the norm stays BF16 and the projection
 * quantises its input right before its GEMM (Section 3.2, Appendix C
 * precision flow). This call fuses the two: for x [rows, cols] (row pitch
 * ld elements) and the norm's weight gamma [cols] (BF16) it computes, per
 * row, rstd = 1 / sqrt(mean(x^2) + eps) in binary32 (written to rstd[rows],
 * float, for the norm's backward), forms y = x * rstd * gamma in binary32,
 * rounds y to BF16 (nearest even) and quantises that y exactly as
 * puro_quantize_fp8 would quantise a BF16 tensor holding it, without
 * writing y. The binary32 sum of squares is taken in this library's order;
 * another order can move rstd, and so y's last BF16 bit, slightly.
 *
 * Modes: TENSOR (q and/or qT; scale[0]; rnd FP32, POW2 or POW2_FLOOR),
 * ROW_1x128 (q, scale and optionally the 128x1 column-grouped qT, scaleT)
 * and COL_128x1 (qT, scaleT), with the layouts of puro_quantize_fp8.
 * BLOCK_128x128 returns PURO_ERR_UNSUPPORTED. eps must be finite and
 * >= 0 (else PURO_ERR_UNSUPPORTED).
 *
 * Requirements: those of puro_quantize_fp8 for x; cols > 0 when rows > 0;
 * gamma and rstd non-NULL and 16-byte aligned when rows > 0. ws:
 * puro_rmsnorm_quantize_workspace_size(rows, cols) bytes (used in TENSOR
 * mode). All pointers are device memory owned by the caller; nothing is
 * allocated or synchronised. */
size_t puro_rmsnorm_quantize_workspace_size(int64_t rows, int64_t cols);
puro_status puro_rmsnorm_quantize_fp8(const uint16_t* x, const uint16_t* gamma, int64_t rows, int64_t cols,
                                      int64_t ld, float eps, puro_fp8_format fmt, puro_scale_mode mode,
                                      puro_scale_rounding rnd, uint8_t* q, float* scale, uint8_t* qT,
                                      float* scaleT, float* rstd, void* ws, size_t ws_bytes,
                                      hipStream_t stream);

/* ------------------------- query / key norm with position rotation ---
 * Between the QKV projection and attention, the paper's model (the Qwen3-1.7B
 * architecture, Section 2) normalises every query and key head and turns it by
 * its position. For a head x of head_dim values, in binary32:
 *     n = x * gamma / sqrt(mean(x^2) + eps)       (gamma NULL: n = x)
 *     the pairs (a, b) of n's first R = rope->dim values become
 *     (a c - b s, b c + a s), (c, s) = the table's entry of the position and
 *     the pair; the values from R on stay (rope NULL or R = 0: all of them)
 * and one rounding to BF16. Pair i < R / 2 is (i, i + R / 2), or
 * (2 i, 2 i + 1) when interleaved.
 *
 * Heads in memory (puro_heads): head h of token s of sequence b starts
 * b * batch_stride + s * row_stride + h * head_stride elements after `data`,
 * its head_dim values are contiguous: views of the projection's output, packed
 * [T, H, D] tensors and heads-first [B, H, S, D] ones alike. Strides are
 * multiples of 8 and not negative, data 16-byte aligned; an output's heads may
 * not overlap each other. An output may be the corresponding input itself
 * (the same data and strides; backward: the incoming gradient), and must not
 * overlap any input otherwise.
 *
 * The rotation (puro_rope): table [len][dim / 2][2] binary32 (cos, sin) pairs,
 * 16-byte aligned, as puro_rope_table writes them or scaled in any way;
 * dim a multiple of 16 up to head_dim; positions [batch * seq] int32, or NULL:
 * token s of every sequence is at position s (then seq <= len). A position
 * outside [0, len) turns its token's first R values to NaN and reads nothing
 * outside the table.
 *
 * head_dim: a multiple of 8 from 8 to 256. heads_q and heads_k (heads_k also
 * counts the value heads of the backward): at most 65535; batch * seq at most 2^25.
 * batch * seq = 0 is a valid empty call. gamma_q, gamma_k: BF16 [head_dim],
 * 16-byte aligned. eps finite and >= 0 (with eps = 0 a head of zeros gives
 * NaN, as the formula does; any other head, down to the smallest values that
 * BF16 has, its norm); heads whose sum of squares overflows binary32 are
 * outside the statement. */
typedef struct {
    uint16_t* data;
    int64_t batch_stride, row_stride, head_stride;
} puro_heads;
typedef struct {
    const float* table;
    int64_t len;
    int dim;
    int interleaved;
    const int32_t* positions;
} puro_rope;

/* The table of angles p * theta^(-2 i / dim), position p in [0, len), pair
 * i < dim / 2: computed in double precision, rounded to binary32. dim a
 * multiple of 16 (0: nothing is written) up to 256, len < 2^31 of at most 2^31
 * pairs in all, theta > 0 and finite. */
puro_status puro_rope_table(float* table, int64_t len, int dim, double theta, hipStream_t stream);

puro_status puro_qk_norm_rope_fwd(int64_t batch, int64_t seq, int heads_q, int heads_k, int head_dim,
                                  const puro_heads* q, const puro_heads* k, const uint16_t* gamma_q,
                                  const uint16_t* gamma_k, float eps, const puro_rope* rope,
                                  const puro_heads* q_out, const puro_heads* k_out, hipStream_t stream);

/* Backward: from the gradients dq, dk of the outputs and the forward's inputs
 * q, k (read only where that kind of heads has a gamma; may be NULL otherwise)
 * the gradients of the inputs, rounded once to BF16, into dq_in and dk_in; with
 * dn the gradient turned back, r = 1 / sqrt(mean(x^2) + eps), h = x r,
 * g = dn gamma:  dx = r (g - h mean(g h)).  dgamma_q, dgamma_k (FP32
 * [head_dim], overwritten, either NULL: not wanted) = the sums over tokens and
 * heads of dn h, in a fixed order, in binary32 and, beyond 64 additions in a
 * row, in binary64. dv, dv_in (both or neither): the value heads' gradients,
 * copied, so that one call assembles the gradient of the projection's output.
 * The statistics are recomputed from the heads, which the call reads anyway:
 * nothing is kept from the forward but its inputs. ws: the matching
 * *_workspace_size bytes (for dgamma; 16-byte aligned). */
size_t puro_qk_norm_rope_bwd_workspace_size(int64_t batch, int64_t seq, int head_dim);
puro_status puro_qk_norm_rope_bwd(int64_t batch, int64_t seq, int heads_q, int heads_k, int head_dim,
                                  const puro_heads* dq, const puro_heads* dk, const puro_heads* dv,
                                  const puro_heads* q, const puro_heads* k, const uint16_t* gamma_q,
                                  const uint16_t* gamma_k, float eps, const puro_rope* rope,
                                  const puro_heads* dq_in, const puro_heads* dk_in, const puro_heads* dv_in,
                                  float* dgamma_q, float* dgamma_k, void* ws, size_t ws_bytes,
                                  hipStream_t stream);

/* The same backward with its result quantised: the matrix dqkv [batch * seq,
 * (heads_q + 2 heads_k) * head_dim] = [dq | dk | dv] of the projection's output
 * gradient (rounded to BF16), quantised exactly as puro_quantize_fp8 would
 * quantise a BF16 tensor holding it, without writing it: q8 for the QKV
 * projection's Dgrad, the transposed copy for its Wgrad. Modes TENSOR,
 * ROW_1x128 and COL_128x1 with puro_quantize_fp8's outputs, layouts and
 * requirements (rows = batch * seq, cols = the heads' width); BLOCK_128x128 is
 * PURO_ERR_UNSUPPORTED, and so is a head_dim other than 64 and 128 (a 128-column
 * tile then holds no whole heads: use the call above and puro_quantize_fp8).
 * batch * seq is at most 2^22 here; dv is required when heads_k > 0. ws: its *_workspace_size bytes, 16-byte
 * aligned (needed in TENSOR mode and for dgamma). */
size_t puro_qk_norm_rope_bwd_quantize_workspace_size(int64_t batch, int64_t seq, int heads_q, int heads_k,
                                                     int head_dim);
puro_status puro_qk_norm_rope_bwd_quantize_fp8(int64_t batch, int64_t seq, int heads_q, int heads_k, int head_dim,
                                               const puro_heads* dq, const puro_heads* dk, const puro_heads* dv,
                                               const puro_heads* q, const puro_heads* k, const uint16_t* gamma_q,
                                               const uint16_t* gamma_k, float eps, const puro_rope* rope,
                                               puro_fp8_format fmt, puro_scale_mode mode, puro_scale_rounding rnd,
                                               uint8_t* q8, float* scale, uint8_t* qT, float* scaleT,
                                               float* dgamma_q, float* dgamma_k, void* ws, size_t ws_bytes,
                                               hipStream_t stream);

/* ---------------------------------------------------------------- GEMM ---
 * D[m, n] = sum_k A[m, k] * B[n, k] with FP32 accumulation (Section 3.2:
 * the Fprop, Dgrad and Wgrad GEMMs of a linear layer run on FP8 operands).
 * Both operands are stored with the reduction index k contiguous: A is
 * [M, K] with row pitch A->ld bytes, B is [N, K] with row pitch B->ld bytes.
 * Fprop is A = Xq, B = Wq; Dgrad A = dYq, B = WqT; Wgrad A = dYqT, B = XqT.
 *
 * Operand scales (device memory, float):
 *   TENSOR:          scale[0]
 *   ROW_1x128:       scale[row * (K/128) + k/128]          ([rows, K/128])
 *   BLOCK_128x128:   scale[(row/128) * (K/128) + k/128]    ([ceil(rows/128), K/128])
 * Grouped scales must be powers of two in [2^-127, 2^127] (as written by
 * puro_quantize_fp8 with POW2); they are applied exactly inside the MFMA.
 * Per-tensor scales are applied once, in FP32, to the accumulated sum.
 *
 * D is BF16 (round-to-nearest-even) or FP32, row pitch ldd elements. With
 * accumulate != 0, D += result (the old value is read in D's type and the sum
 * formed in FP32). Requirements: K % 16 == 0 (K % 128 == 0 with grouped
 * scales), lda and ldb multiples of 16, operand pointers 16-byte aligned,
 * ldd >= N. ws: puro_fp8_gemm_workspace_size(M, N, K, d_type) bytes. */
typedef struct {
    const uint8_t* data;
    int64_t ld;
    puro_fp8_format fmt;
    puro_scale_mode mode;   /* TENSOR, ROW_1x128 or BLOCK_128x128; grouped ones may carry PURO_SCALE_KMAJOR */
    const float* scale;
} puro_fp8_operand;

size_t puro_fp8_gemm_workspace_size(int64_t M, int64_t N, int64_t K, puro_out_dtype d_type);
/* The execution plan puro_fp8_gemm chooses for this problem (host-side query;
 * enqueues nothing): the workgroup tile (tile_m x tile_n outputs), the depth
 * of its LDS ring (stages), the number of k ranges (splits > 1: FP32 partial
 * sums in ws plus a fixed-order reduction kernel) and the kernel launches
 * that makes. a_mode / b_mode are the operands' scale modes (the plan differs
 * with block scales). Outputs may be NULL. PURO_ERR_SHAPE for negative sizes,
 * PURO_ERR_UNSUPPORTED for a mode the GEMM does not take. For tests and
 * benchmarks that need to know which kernel configuration runs. */
puro_status puro_fp8_gemm_plan(int64_t M, int64_t N, int64_t K, puro_scale_mode a_mode,
                               puro_scale_mode b_mode, int* tile_m, int* tile_n, int* stages,
                               int* splits, int* launches);
puro_status puro_fp8_gemm(int64_t M, int64_t N, int64_t K,
                          const puro_fp8_operand* A, const puro_fp8_operand* B,
                          void* D, puro_out_dtype d_type, int64_t ldd, int accumulate,
                          void* ws, size_t ws_bytes, hipStream_t stream);

/* GEMM with the BF16 bias / residual epilogue of the linear layers around
 * the FP8 GEMMs: D = BF16(alpha * acc + bias[n] + residual[m, n]), the sum
 * in binary32 and one rounding (BF16 output only; either term may be NULL).
 * Qwen2's QKV projection carries a bias, and the attention output and MLP
 * down projections add into the residual stream, which stays BF16 (Appendix
 * C precision flow): fusing the add removes a BF16 read and write of Y.
 * bias: BF16 [N], 16-byte aligned. residual: BF16 [M, N] with row pitch
 * N <= ldr <= 2^22, ldr % 4 == 0, 16-byte aligned; it may be D itself (ldr == ldd,
 * an in-place residual add) but must not otherwise overlap D. Operands,
 * scales, workspace and errors as puro_fp8_gemm; accumulate is not offered. */
puro_status puro_fp8_gemm_epilogue(int64_t M, int64_t N, int64_t K, const puro_fp8_operand* A,
                                   const puro_fp8_operand* B, uint16_t* D, int64_t ldd, const uint16_t* bias,
                                   const uint16_t* residual, int64_t ldr, void* ws, size_t ws_bytes,
                                   hipStream_t stream);

/* -------------------------------------------------------- linear layer ---
 * Y = X W^T with X [M, K] and W [N, K] in BF16 (dense rows), and its backward
 * pass, as a sequence of the calls above (Section 3.2; Appendix C).
 *
 * Recipe: blockwise = 0 -> one scale per tensor (rule `rnd`); blockwise = 1
 * -> X and dY in 1x128 groups along each GEMM's reduction dimension (row
 * groups for Fprop and Dgrad, column groups for Wgrad), W in 128x128 blocks,
 * power-of-two scales (rule POW2_FLOOR if rnd says so, else POW2). */
typedef struct {
    puro_fp8_format x_fmt, w_fmt, dy_fmt;
    int blockwise;
    puro_scale_rounding rnd;
} puro_linear_recipe;

/* What the forward pass keeps for the backward pass (caller-allocated):
 * the quantised input, transposed for Wgrad (Section 3.2 keeps the quantised
 * input for Wgrad), and the quantised weight, transposed for Dgrad.
 *   xq_t    [K, M] FP8;  x_scale: per-tensor [1], blockwise [M/128, K]
 *   wq_t    [K, N] FP8;  w_scale: per-tensor [1], blockwise [N/128, K/128]
 * Blockwise scales are stored k-block-major (the group index along the
 * reduction dimension of the GEMM that reads them outermost): x_scale[b][k]
 * is the scale of xq_t row k, m in [128 b, 128 b + 128); w_scale[b][c] that
 * of the block of wq_t rows [128 c, 128 c + 128) and columns [128 b, ...).
 * The Wgrad and Dgrad GEMMs then read a k block's scales as one contiguous
 * run. (puro_quantize_fp8 and puro_fp8_gemm use the row-major layouts.)  */
typedef struct {
    uint8_t* xq_t;
    float* x_scale;
    uint8_t* wq_t;
    float* w_scale;
} puro_linear_saved;

/* Byte sizes of the four saved buffers (sizes[0..3] in the struct's order);
 * returns their sum. */
size_t puro_linear_saved_bytes(int64_t M, int64_t N, int64_t K, const puro_linear_recipe* recipe,
                               size_t sizes[4]);
size_t puro_linear_fwd_workspace_size(int64_t M, int64_t N, int64_t K, const puro_linear_recipe* recipe);
size_t puro_linear_bwd_workspace_size(int64_t M, int64_t N, int64_t K, const puro_linear_recipe* recipe);

/* Forward: quantise X and W, Y [M, N] (BF16) = Fprop, fill `saved`.
 * Requirements: M, N, K multiples of 16 (of 128 when blockwise) and at most
 * 2^22 (each is the row pitch of an FP8 operand of one of the three GEMMs);
 * larger sizes return PURO_ERR_SHAPE before anything is enqueued (this also
 * holds for the backward). */
puro_status puro_linear_fwd(const uint16_t* X, const uint16_t* W, int64_t M, int64_t N, int64_t K,
                            const puro_linear_recipe* recipe, uint16_t* Y,
                            const puro_linear_saved* saved, void* ws, size_t ws_bytes,
                            hipStream_t stream);

/* Backward: quantise dY [M, N]; dX [M, K] (BF16) = Dgrad and dW [N, K] (FP32)
 * = Wgrad (dW += when accumulate_dW != 0). dX or dW may be NULL to skip that
 * GEMM. */
puro_status puro_linear_bwd(const uint16_t* dY, const puro_linear_saved* saved,
                            int64_t M, int64_t N, int64_t K, const puro_linear_recipe* recipe,
                            uint16_t* dX, float* dW, int accumulate_dW,
                            void* ws, size_t ws_bytes, hipStream_t stream);

/* ------------------------------------- LM head with cross-entropy loss ---
 * Section 3.1.3 of the paper names the language-model head as the layer whose
 * cost sets the pipeline's last stage apart; Appendix C keeps it in BF16. For
 * hidden states X [M, K] and the output embedding W [V, K] (BF16, dense rows)
 * and one target vocabulary id per row, targets [M] (int32):
 *   forward:  z = X W^T; lse[m] = log sum_v exp(z[m, v]); loss[m] = lse[m] - z[m, t_m]
 *   backward: dz = g (exp(z - lse) - onehot(t)); dX = dz W (BF16 [M, K]);
 *             dW = dz^T X (FP32 [V, K], overwritten)
 * The logits are never stored: the forward reduces each 128-column block of
 * the GEMM's output tile to (max, sum exp) in its epilogue; the backward
 * recomputes the logits in chunks of 8192 vocabulary columns and writes only
 * the chunk's dz to the workspace (BF16; under PURO_LM_HEAD_FP8 its E4M3
 * copies, in 1x128 row and 128x1 column groups, made in the same epilogue).
 * g is the loss's upstream gradient (1 for the sum over tokens, 1/M for
 * their mean).
 * Recipes: PURO_LM_HEAD_BF16 (BF16 GEMMs with binary32 accumulation, dz
 * rounded to BF16), PURO_LM_HEAD_FP8 (Section 3.2's blockwise recipe: X in
 * 1x128 groups, W in 128x128 blocks, each dz chunk rounded to BF16 and then
 * in 1x128 + 128x1 groups; E4M3, power-of-two scales).
 * Requirements: M, V, K positive multiples of 128, at most 2^21; X, W, lse,
 * loss, dX, dW 16-byte aligned; targets in [0, V) (a row whose target lies
 * outside gets loss NaN and no onehot term). lse and loss are FP32 [M]. ws:
 * puro_lm_head_ce_workspace_size(M, V, K, recipe, backward) bytes (the
 * backward's includes the quantised or transposed operands and one chunk). All
 * pointers are device memory owned by the caller; nothing is allocated or
 * synchronised; invalid arguments return before anything is enqueued. */
typedef enum { PURO_LM_HEAD_BF16 = 0, PURO_LM_HEAD_FP8 = 1 } puro_lm_head_recipe;
size_t puro_lm_head_ce_workspace_size(int64_t M, int64_t V, int64_t K, puro_lm_head_recipe recipe, int backward);
puro_status puro_lm_head_ce_fwd(const uint16_t* X, const uint16_t* W, const int32_t* targets, int64_t M,
                                int64_t V, int64_t K, puro_lm_head_recipe recipe, float* lse, float* loss,
                                void* ws, size_t ws_bytes, hipStream_t stream);
puro_status puro_lm_head_ce_bwd(const uint16_t* X, const uint16_t* W, const int32_t* targets, const float* lse,
                                int64_t M, int64_t V, int64_t K, puro_lm_head_recipe recipe, float grad_scale,
                                uint16_t* dX, float* dW, void* ws, size_t ws_bytes, hipStream_t stream);

/* ----------------------------- LM head with a teacher's top logits ---
 * The LM head with distillation as its loss: the divergence of the student's
 * distribution over the vocabulary from a teacher's, known by its topk largest
 * entries per token. For hidden states X [M, K] and the output embedding
 * W [V, K] (BF16, dense rows), a temperature tau and, per row, topk token ids
 * [M, topk] (int32) with the teacher's values [M, topk] (FP32):
 *   z = X W^T, a = z / tau, lse[m] = log sum_v exp(a[m, v])
 *   q = softmax over the row's entries of value / tau   (PURO_DISTILL_LOGITS)
 *   q = value, a probability as stored, not negative      (PURO_DISTILL_PROBS)
 *   loss[m] = sum_j q_j (log q_j - a[m, id_j] + lse[m]),  0 log 0 = 0
 *   z_top[m, j] = z[m, id_j]
 *   backward, of grad_scale sum_m dloss[m] loss[m] (dloss NULL: ones):
 *     dz_v = (dloss grad_scale / tau) (Q exp(a_v - lse) - sum_{j: id_j = v} q_j),
 *     Q = sum_j q_j;  dX = dz W (BF16), dW = dz^T X (FP32 or BF16)
 * An entry whose id lies outside [0, V) (-1, say: fewer than topk are known)
 * does not count and has z_top 0; a row without entries (a padding token) has
 * loss 0 and gradient 0, and so has one whose teacher logits are all -infinity.
 * A row whose dloss is 0 or whose q are all 0 adds nothing to dW and has dX 0
 * whatever its hidden state holds, NaN included, and a row whose q are all 0
 * also whatever its dloss is. An id given twice counts twice: both q are added,
 * which also mixes a hard target into PURO_DISTILL_PROBS. A NaN among the
 * entries that count, or a teacher logit of +infinity, makes the row's loss and
 * gradient NaN. No teacher beyond the entries is assumed (PROBS need not add up
 * to 1). grad_scale and grad_scale / tau are finite; logits whose quotient by
 * tau overflows binary32 are outside the statement.
 *
 * The logits are never stored (as puro_lm_head_ce_*): the forward keeps lse and
 * z_top for the backward, which recomputes the logits and keeps two BF16 copies
 * of dz, of as many vocabulary columns at a time as 2.5 GiB each hold, in its
 * workspace. BF16 operands with binary32 accumulation, statistics and sums in
 * binary32; dz is rounded once to BF16, the operand type of its GEMMs. dX and
 * dW: either may be NULL to skip it. dw_type PURO_OUT_FP32, or PURO_OUT_BF16,
 * the type a gradient has when ranks exchange it (Appendix C); accumulate_dW
 * != 0 adds to an FP32 dW (with BF16: PURO_ERR_UNSUPPORTED).
 *
 * Any M >= 0 (0: dW is cleared), V >= 1, K a positive multiple of 8, each at
 * most 2^21, M V at most 2^39; topk from 1 to 1024; tau and 1 / tau positive
 * and normal; X, W, dX, dW and ws 16-byte aligned. Nothing is allocated or
 * synchronised. */
typedef enum { PURO_DISTILL_LOGITS = 0, PURO_DISTILL_PROBS = 1 } puro_distill_target;
size_t puro_lm_head_distill_workspace_size(int64_t M, int64_t V, int64_t K, int64_t topk, int backward);
puro_status puro_lm_head_distill_fwd(const uint16_t* X, const uint16_t* W, const int32_t* ids, const float* teacher,
                                     int64_t M, int64_t V, int64_t K, int64_t topk, puro_distill_target target,
                                     float temperature, float* lse, float* loss, float* z_top, void* ws,
                                     size_t ws_bytes, hipStream_t stream);
puro_status puro_lm_head_distill_bwd(const uint16_t* X, const uint16_t* W, const int32_t* ids, const float* teacher,
                                     const float* lse, const float* z_top, int64_t M, int64_t V, int64_t K,
                                     int64_t topk, puro_distill_target target, float temperature,
                                     const float* dloss, float grad_scale, uint16_t* dX, void* dW,
                                     puro_out_dtype dw_type, int accumulate_dW, void* ws, size_t ws_bytes,
                                     hipStream_t stream);

/* ------------------------------------------- 8-bit integer linear layers ---
 * The other 8-bit operand type of the matrix cores: a trained model served (or
 * trained on) with int8 weights and activations, a scale for each token and
 * each output channel instead of the FP8 recipe's groups. The paper trains in
 * FP8 (Section 3.2) and states no integer format; the readings here follow the
 * FP8 encoding above.
 *
 * Encoding of a row of values x with amax = max |x|:
 *     s = fl32(amax / 127),  r = fl32(127 / amax),  code = the integer nearest
 *     to x r (the exact product; ties to even), in [-127, 127];
 *     amax = 0: s = 1, codes 0;  a NaN or an infinity among x: s = NaN, codes 0
 *     (so that a product with the row is NaN). r does not overflow: rows below
 *     2^-100 are scaled by 2^64 with their amax first, which changes no code.
 *
 * puro_quantize_int8: of the BF16 tensor x [rows, cols] (row pitch ld) the codes
 * q [rows, cols] (dense) with a scale per row, scale [rows], and / or a transposed
 * copy with a scale per column: qT [cols, rows], row pitch ld_qT, scaleT [cols],
 * encoded from the BF16 values. The copy's columns from `rows` up to the next
 * multiple of 16 are filled with zeros, so that any number of tokens can be a
 * product's reduction dimension; what lies beyond is left alone. Either of q and
 * qT may be NULL (not wanted), each comes with its scales. An empty tensor writes
 * nothing.
 * Requirements: cols % 16 == 0, ld % 8 == 0, ld < 2^23, x, q and qT 16-byte
 * aligned, ld_qT % 16 == 0 and >= rows; rows at most 65535 * 128. ws (16-byte
 * aligned): *_workspace_size(rows, cols) bytes, needed for qT only. */
size_t puro_quantize_int8_workspace_size(int64_t rows, int64_t cols);
puro_status puro_quantize_int8(const uint16_t* x, int64_t rows, int64_t cols, int64_t ld, int8_t* q, float* scale,
                               int8_t* qT, int64_t ld_qT, float* scaleT, void* ws, size_t ws_bytes,
                               hipStream_t stream);

/* The same encoding of a linear layer's input where it is formed (the places of
 * puro_rmsnorm_quantize_fp8 and puro_swiglu_quantize_fp8), a scale per row:
 *   rmsnorm:  y = x rstd gamma, rstd = 1 / sqrt(mean(x^2) + eps) (written to
 *             rstd [rows] unless that is NULL), of x [rows, cols];
 *   swiglu:   h = silu(gate) up of gu [rows, 2 cols].
 * The values are encoded as binary32 has them, without a rounding to BF16
 * between. Requirements as puro_quantize_int8; gamma BF16 [cols], 16-byte
 * aligned; eps finite and >= 0 (with eps = 0 a row of zeros has scale NaN; any
 * other row has its norm, down to BF16's smallest values, its rstd infinity where
 * binary32 has no larger number); gu's pitch ld >= 2 cols. Rows whose sum of squares
 * overflows binary32 are outside the statement. */
puro_status puro_rmsnorm_quantize_int8(const uint16_t* x, const uint16_t* gamma, int64_t rows, int64_t cols,
                                       int64_t ld, float eps, int8_t* q, float* scale, float* rstd,
                                       hipStream_t stream);
puro_status puro_swiglu_quantize_int8(const uint16_t* gu, int64_t rows, int64_t cols, int64_t ld, int8_t* q,
                                      float* scale, hipStream_t stream);

/* D[m, n] = (sum_k A[m, k] B[n, k]) a_scale[m] b_scale[n] (+ bias[n] + residual[m, n])
 * of int8 codes A [M, K] (pitch lda) and B [N, K] (pitch ldb), a_scale [M] and
 * b_scale [N]. The sum is exact (32-bit integers; K at most 131056), rounded to
 * binary32, multiplied by a_scale and then by b_scale, the other terms added in
 * binary32, and rounded once to D's type (BF16 or FP32, pitch ldd). accumulate
 * != 0: D += result (FP32 only). bias: BF16 [N]; residual: BF16 [M, N], pitch ldr,
 * may be D itself (ldr == ldd) and must not overlap it otherwise; either may be
 * NULL; both for a BF16 D only. (Other combinations: PURO_ERR_UNSUPPORTED.)
 * A linear layer's three products have this form: Y from X's and W's rows,
 * dX from dY's rows and W's transposed copy, dW from the transposed copies of dY
 * and X (K then is the number of tokens rounded up to 16).
 * Requirements: K % 16 == 0; lda, ldb % 16 == 0, at least K and at most 2^22;
 * ldd, ldr % 4 == 0 and at least N, ldr at most 2^22; data pointers, a_scale and
 * b_scale 16-byte aligned; M and N at most 2^22, M N at most 2^36; ws (16-byte
 * aligned): puro_int8_gemm_workspace_size(M, N, K) bytes. M = 0 or N = 0 is a
 * valid empty call; K = 0 is an empty sum. */
size_t puro_int8_gemm_workspace_size(int64_t M, int64_t N, int64_t K);
puro_status puro_int8_gemm(int64_t M, int64_t N, int64_t K, const int8_t* A, int64_t lda, const float* a_scale,
                           const int8_t* B, int64_t ldb, const float* b_scale, void* D, puro_out_dtype d_type,
                           int64_t ldd, int accumulate, const uint16_t* bias, const uint16_t* residual, int64_t ldr,
                           void* ws, size_t ws_bytes, hipStream_t stream);

/* The int8 linear layer: Y = X W^T with X [M, K] and W [N, K] in BF16 (dense rows)
 * and its backward, as a sequence of the calls above: X and dY quantised per token
 * for the products that reduce over channels and per channel for the one that
 * reduces over tokens, W per output and per input channel.
 *   saved: xq_t [K, M16] (int8; M16 = M rounded up to 16, zeros behind the tokens),
 *   x_scale [K], wq_t [K, N], w_scale [K]: the transposed copies for the backward.
 * Forward: Y [M, N] (BF16); saved NULL: no backward follows, the copies are not made.
 * A backward reads W's copy for dX and X's for dW: of saved either, with its scales,
 * may be NULL where that gradient is not wanted.
 * Backward: dX [M, K] (BF16) and dW [N, K] (FP32; += when accumulate_dW != 0); either
 * may be NULL to skip it. M = 0 is valid (dW: zeros, or as it was), and K = 0 (Y: zeros).
 * Requirements: N and K multiples of 16 (else PURO_ERR_ALIGN), M, N and K at most
 * 131056; all pointers and ws 16-byte aligned; ws: the matching
 * *_workspace_size(M, N, K) bytes. */
size_t puro_int8_linear_fwd_workspace_size(int64_t M, int64_t N, int64_t K);
size_t puro_int8_linear_bwd_workspace_size(int64_t M, int64_t N, int64_t K);
puro_status puro_int8_linear_fwd(const uint16_t* X, const uint16_t* W, int64_t M, int64_t N, int64_t K, uint16_t* Y,
                                 const puro_linear_saved* saved, void* ws, size_t ws_bytes, hipStream_t stream);
puro_status puro_int8_linear_bwd(const uint16_t* dY, const puro_linear_saved* saved, int64_t M, int64_t N, int64_t K,
                                 uint16_t* dX, float* dW, int accumulate_dW, void* ws, size_t ws_bytes,
                                 hipStream_t stream);

/* --------------------------------------- verification of drafted tokens ---
 * A distilled student (puro_lm_head_distill_*) proposes tokens; the model itself
 * scores them all in one pass, and each is kept with the probability that leaves
 * the model's own distribution unchanged. For B sequences whose rows lie one
 * after another: sequence b has the target rows offsets[b] .. offsets[b + 1] - 1,
 * the i-th of them the target's prediction of the place where the draft put
 * draft_ids[offsets[b] + i]; the last row has no draft (its id is not read). The
 * draft's own predictions lie one after another in `draft`, a row for each draft:
 * for target row t of sequence b row t - (b - e), e the sequences before b that have
 * no rows (equal offsets); draft NULL: the drafts were chosen without probabilities
 * (q = 1 at the id).
 *     p, q: softmax of row / temperature (PURO_VERIFY_LOGITS), or the row as it
 *           stands, not negative (PURO_VERIFY_PROBS)
 *     draft i is kept while uniform[t] q[id] < p[id]; at the first that is not,
 *     or after all, the token drawn from max(p - q, 0) (from p in the last row,
 *     and where that is 0 everywhere): the least v with
 *     sum_{w <= v} rest[w] > uniform_sample[b] sum_w rest[w]
 *     (the last v with rest[v] > 0 where rounding leaves none). What is no more than
 *     2^-970 may count as 0.
 * tokens[offsets[b] ..]: the kept ids, the drawn token, then -1; accepted[b]: how
 * many were kept. temperature 0 (LOGITS): the row's largest logit, the lowest id
 * among equals, is the token, and a draft is kept where it is that; draft,
 * uniform and uniform_sample are not read then.
 * Exponentials (to 10^-10) and sums in binary64, in a fixed order: over 10^5
 * entries the drawn token moves with differences of 10^-8.
 * Special values: logits of -infinity have probability 0; an id outside [0, V) is
 * not kept, nor is one whose p or q is NaN; a row of logits with a NaN or a
 * +infinity, or with no probability at all, keeps nothing; a token that would be
 * drawn from such a row, or from one with a NaN or an infinity in its rest, is -1.
 * A sequence without rows (an idle slot, anywhere in the batch) has accepted 0, no
 * token and no row of the draft's; rows behind the last sequence are not written;
 * one whose offsets decrease or leave [0, T], that begins before an earlier
 * offset, or whose draft rows leave [0, draft_rows), has accepted -1 and no token.
 * tokens may be draft_ids itself (then the ids are replaced); tokens and accepted
 * overlap the ids and offsets in no other way (PURO_ERR_SHAPE).
 * dtype: PURO_OUT_BF16 or PURO_OUT_FP32 for both target [T, V] (pitch ld_target)
 * and draft [draft_rows, V] (pitch ld_draft); any V from 1 to 2^21 and pitches
 * from V to 2^22 (rows need no more than their element's alignment); T at
 * most 2^20, B at most 2^16, T V and B V at most 2^35, draft_rows at most T. offsets [B + 1], draft_ids [T],
 * tokens [T], accepted [B]: int32; uniform [T], uniform_sample [B]: FP32 in
 * [0, 1). temperature finite and >= 0, if not 0 between 2^-20 and 2^20 (PROBS:
 * not used). ws (16-byte aligned): *_workspace_size bytes. */
typedef enum { PURO_VERIFY_LOGITS = 0, PURO_VERIFY_PROBS = 1 } puro_verify_kind;
size_t puro_verify_drafts_workspace_size(int64_t B, int64_t T, int64_t draft_rows, int64_t V);
puro_status puro_verify_drafts(int64_t B, int64_t T, int64_t draft_rows, int64_t V, puro_verify_kind kind,
                               puro_out_dtype dtype, const void* target, int64_t ld_target, const void* draft,
                               int64_t ld_draft, const int32_t* draft_ids, const int32_t* offsets,
                               const float* uniform, const float* uniform_sample, double temperature,
                               int32_t* tokens, int32_t* accepted, void* ws, size_t ws_bytes, hipStream_t stream);

/* ---------------------------------------------------------------- MuonH ---
 * Section 3.3 (Hyperball Optimization), equation hyperball-update: a wrapped
 * matrix keeps its initial Frobenius radius R; with the Muon update u and the
 * weight learning rate eta,
 *     W~ = W - eta R u / ||u||_F,    W' = R W~ / ||W~||_F.
 * The paper takes Muon from its training framework; the Muon update here is
 * the published method's:
 *     buf' = mu buf + (1 - mu) G;  V = (1 - mu) G + mu buf' (nesterov) or buf'
 *     X_0 = V / (||V||_F + 1e-7), transposed when rows > cols;
 *     ns_steps times: A = X X^T, B = b A + c A A^T, X = a X + B X,
 *     (a, b, c) = (3.4445, -4.7750, 2.0315); u = X (turned back).
 * FP32 state (W, G, buf), each momentum product and sum rounded to binary32
 * in that order with (1 - mu) rounded first; Newton-Schulz in BF16 with
 * binary32 accumulation, each of A, B and X rounded once to BF16; the
 * hyperball step from the BF16 u in binary32 with double-precision norms.
 *
 * puro_muonh_step updates `count` matrices of one shape stored back to back:
 * W [count][rows][cols] (FP32, in place), buf (FP32, in place), G (FP32),
 * radius [count] (FP32 device array: each matrix's R). Optional outputs:
 * w_bf16 (BF16 copy of W'), u_out (BF16 u, W's layout). ns_steps: 5 in the
 * method; 0 applies the hyperball step to X_0 (a test hook). u = 0 (all of V
 * zero) leaves W's direction and only projects it. rows, cols: positive
 * multiples of 128, at most 2^21; count in [1, 65535]; pointers 16-byte
 * aligned device memory owned by the caller. ws:
 * puro_muonh_workspace_size(count, rows, cols) bytes. Matrices may not
 * overlap W, G, buf or the outputs.
 *
 * puro_newton_schulz_bf16 runs `steps` Newton-Schulz steps on X [count][r][c]
 * (BF16, r <= c, already normalised) into out (same layout); the steps of
 * puro_muonh_step, exposed for per-step checks. */
size_t puro_muonh_workspace_size(int64_t count, int64_t rows, int64_t cols);
puro_status puro_muonh_step(int64_t count, int64_t rows, int64_t cols, float* W, uint16_t* w_bf16, const float* G,
                            float* buf, const float* radius, float mu, int nesterov, float eta, int ns_steps,
                            uint16_t* u_out, void* ws, size_t ws_bytes, hipStream_t stream);
size_t puro_newton_schulz_workspace_size(int64_t count, int64_t r, int64_t c);
puro_status puro_newton_schulz_bf16(int64_t count, int64_t r, int64_t c, const uint16_t* X, int steps,
                                    uint16_t* out, void* ws, size_t ws_bytes, hipStream_t stream);

#ifdef __cplusplus
}
#endif

#endif /* PURO_H */
