/*
 * mixquant.h -- C ABI of the MI355X (gfx950) library for the prefill linear layer of
 * Mix-Quant run as NVFP4 W4A4 (Section 3.3, the paragraph on NVFP4 quantization of the
 * prefill phase): on-the-fly activation quantization (Eq. 2 then Eq. 1) followed by a
 * block-scaled FP4 GEMM against offline-quantized weights, plus a plain BF16 GEMM that
 * stands for the high-precision decode path the paper compares against.
 *
 * Conventions shared by every entry point
 *  - Every data pointer is a DEVICE pointer owned by the caller.  The library never
 *    allocates, frees or keeps a pointer, and never synchronises: each call enqueues its
 *    kernels on `stream` (a hipStream_t passed as void*; NULL = the default stream) and
 *    returns.  Calls on one stream execute in order.
 *  - Tensor-level scales (alpha in Eq. 1) are read from device memory, so a scale computed
 *    on the device needs no host round trip.
 *  - Return value: MQ_OK, or an mq_status error.  Arguments are validated on the host before
 *    anything is launched: with any status but MQ_ERR_HIP nothing has been enqueued.
 *    MQ_ERR_HIP means the HIP runtime refused a launch (mq_last_hip_error() returns its
 *    hipError_t); an entry point that launches several kernels (nvfp4_global_scale, a product
 *    cut into K slabs or into two parts of Y) may then have enqueued the earlier ones, and
 *    its outputs are undefined.
 *  - One-time set-up per device (kernel attributes, the address of the static scratch array):
 *    done by mq_init(), or else by the first product on that device.  A caller that captures
 *    streams into HIP graphs calls mq_init() once per device beforehand; after that no entry
 *    point does anything but enqueue kernels.
 *  - Outputs must not overlap inputs.
 *
 * NVFP4 tensor (Section 3.3): a [rows, K] matrix whose contraction index K is contiguous
 * (the scale blocks run along the GEMM's contraction dimension, Section 3.3, last sentence),
 * K % 16 == 0, stored as
 *    codes  : uint8 [rows, K/2]   element k of a row in byte k/2, even k in the low nibble;
 *                                 a code is E2M1: bit3 sign, bits2..1 exponent (bias 1),
 *                                 bit0 mantissa -> {0, .5, 1, 1.5, 2, 3, 4, 6}
 *    scales : uint8 [rows, K/16]  one FP8 E4M3 (OCP, max 448, no infinity) byte per block of
 *                                 g = 16 consecutive K elements
 *    alpha  : one float           the tensor-level scale
 * with value x_hat[r, k] = alpha * E4M3(scales[r, k/16]) * E2M1(code[r, k])   (Eq. 1, right).
 * Scale bytes are what Eq. 2 produces: non-negative and finite, 0x00 .. 0x7E.  The quantizers
 * emit nothing else; the products (nvfp4_gemm, nvfp4_matvec) given a byte with the sign bit set or the NaN
 * pattern 0x7F return unspecified values for the outputs that the block touches (never a fault).
 */
#ifndef MIXQUANT_H
#define MIXQUANT_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    MQ_OK = 0,
    MQ_ERR_NULL = 1,   /* a required pointer is NULL */
    MQ_ERR_SHAPE = 2,  /* rows/M/N < 0, K <= 0, K % 16 != 0 (K % 64 != 0 for MQ_LAYOUT_KTILE), ld too small */
    MQ_ERR_ALIGN = 3,  /* a pointer or leading dimension breaks the stated alignment */
    MQ_ERR_ARG = 4,    /* unknown enum value */
    MQ_ERR_HIP = 5,    /* kernel launch failed; see mq_last_hip_error() */
    MQ_ERR_SCRATCH = 6 /* nvfp4_gemm_noalloc: the problem wants more scratch than its static array holds;
                          nvfp4_matvec, mq_sample: than the workspace holds */
} mq_status;

typedef enum {
    MQ_OUT_BF16 = 0,   /* product path: FP32 accumulator rounded to BF16 (nearest even) */
    MQ_OUT_FP32 = 1    /* test path: the scaled FP32 accumulator itself */
} mq_out;

/*
 * Byte order of the two arrays of an NVFP4 tensor.
 * MQ_LAYOUT_LINEAR is the canonical order described at the top of this file.
 * MQ_LAYOUT_KTILE (needs K % 64 == 0) stores the same bytes K-step-major, so that the 64-wide
 * K step the GEMM consumes is contiguous over rows (one way to lay the blocks out along the
 * contraction dimension, which is all that Section 3.3 asks of the layout):
 *    codes_ktile [(t * rows + r) * 32 + j] = codes_linear [r * (K/2)  + t * 32 + j],  j < 32
 *    scales_ktile[(t * rows + r) * 4  + j] = scales_linear[r * (K/16) + t * 4  + j],  j < 4
 * for K step t = 0 .. K/64 - 1.  Sizes are the same in both layouts.
 */
typedef enum {
    MQ_LAYOUT_LINEAR = 0,
    MQ_LAYOUT_KTILE = 1
} mq_layout;

/*
 * One-time set-up of the current device (hipGetDevice): raises the dynamic-LDS limits of the
 * tiled kernels and looks up this device's copy of the static scratch array.  Idempotent,
 * thread-safe, launches nothing.  Optional except before stream capture (see above).
 */
int mq_init(void);

/* Sizes, in bytes, of the two byte arrays of an NVFP4 tensor (0 when K % 16 != 0). */
size_t mq_codes_bytes(int64_t rows, int64_t K);
size_t mq_scales_bytes(int64_t rows, int64_t K);

/*
 * Tensor-level scale (Section 3.3 gives it the role of setting the tensor's overall range and
 * no formula; the workloads use alpha = max|x| / (6 * 448)).
 * Writes alpha = max|x| / 2688 to *alpha_dev (1.0f when the tensor is all zero), all in
 * binary32.  x_bf16: [rows, K] BF16, row stride ldx elements (ldx >= K).  K % 16 == 0,
 * x_bf16 16-byte aligned, ldx % 8 == 0.  rows == 0 writes 1.0f.
 */
int nvfp4_global_scale(const void *x_bf16, int64_t rows, int64_t K, int64_t ldx,
                       float *alpha_dev, void *stream);

/*
 * NVFP4 quantizer for activations (per prefill batch) or weights (once, offline):
 * Eq. 2 gives each block's E4M3 scale from its largest magnitude, Eq. 1 the E2M1 codes.
 * Arithmetic, every step IEEE binary32, nearest-even, unfused, per block b of 16 elements:
 *    s = amax_b / (6 * alpha);  sigma_b = Pi_E4M3(s)   (ties to even, saturating at 448)
 *    r = 1 / (alpha * sigma_b); q_i = Pi_FP4(x_i * r)  (ties to even, clipped to +-6);
 *    sigma_b == 0 gives signed-zero codes.
 * x_bf16: [rows, K] BF16, row stride ldx elements; *alpha_dev finite and > 0, read on the
 * device.  codes: [rows, K/2], scales: [rows, K/16], dense.  Inputs must be finite (Inf
 * saturates, NaN gives unspecified codes; never a fault).
 * layout: mq_layout of the two output arrays.
 * K % 16 == 0; x_bf16 and codes 16-byte aligned (scales 4-byte aligned for MQ_LAYOUT_KTILE);
 * ldx % 8 == 0.  rows == 0 is a no-op.
 */
int nvfp4_quantize(const void *x_bf16, int64_t rows, int64_t K, int64_t ldx,
                   const float *alpha_dev, uint8_t *codes, uint8_t *scales, int layout,
                   void *stream);

/*
 * Quantizer fused with the operation that produces the activation (Section 3.3, last sentence:
 * the layout is chosen so that a backend can fuse quantization with its neighbours).  The paper
 * does not define the producers;
 * these are the two that feed the linear layers of the decoder blocks of the models it
 * evaluates (Section 4.1), by their textbook definitions.  In both, the producer's value is
 * computed in binary32, rounded once to BF16 (nearest even), and that BF16 tensor is quantized
 * exactly as nvfp4_quantize would: the BF16 activations never travel through memory.
 * p_bf16 / y_bf16 (may be NULL): if given, also receives the BF16 tensor that was quantized,
 * [rows, K] with row stride ldp / ldy elements (multiple of 8, 16-byte aligned base); the codes
 * and scales are then bit-identical to nvfp4_quantize applied to it.
 *
 * nvfp4_quantize_silu_mul: gated-MLP activation, the input of the down projection.
 *    p[r, k] = silu(g) * u,  g = gate_up[r, k],  u = gate_up[r, K + k],  silu(g) = g / (1 + exp(-g))
 * gate_up_bf16: [rows, 2K] BF16, row stride ld elements (ld >= 2K, ld % 8 == 0).  Gates below
 * about -88 (exp(-g) overflows binary32) give -0, as any binary32 evaluation does.
 * nvfp4_quantize_rmsnorm: root-mean-square normalisation, the input of the qkv and gate_up
 * projections.
 *    y[r, k] = x[r, k] / sqrt(mean_k(x[r, :]^2) + eps) * w[k]
 * x_bf16: [rows, K] BF16, row stride ldx; w_bf16: [K] BF16; eps >= 0; K % 64 == 0.
 * Other arguments, alignment and errors as in nvfp4_quantize.
 */
int nvfp4_quantize_silu_mul(const void *gate_up_bf16, int64_t rows, int64_t K, int64_t ld,
                            const float *alpha_dev, uint8_t *codes, uint8_t *scales, int layout,
                            void *p_bf16, int64_t ldp, void *stream);
int nvfp4_quantize_rmsnorm(const void *x_bf16, int64_t rows, int64_t K, int64_t ldx, const void *w_bf16,
                           float eps, const float *alpha_dev, uint8_t *codes, uint8_t *scales,
                           int layout, void *y_bf16, int64_t ldy, void *stream);

/*
 * Offline weight pre-pack (weights are static across requests: Section 3.3, the paragraph on
 * the disaggregated deployment): copy an NVFP4 tensor from one mq_layout to the other.  Pure byte
 * permutation by the index map given at mq_layout; src and dst must not overlap.
 * K % 64 == 0; code arrays 16-byte aligned, scale arrays 4-byte aligned; from_layout != to_layout.
 */
int nvfp4_relayout(const uint8_t *src_codes, const uint8_t *src_scales, uint8_t *dst_codes,
                   uint8_t *dst_scales, int64_t rows, int64_t K, int from_layout, int to_layout,
                   void *stream);

/*
 * Block-scaled FP4 GEMM (Section 3.3; the W4A4 linear layer of the prefill path):
 *    Y[m, n] = alpha_a * alpha_b * sum_k  sa[m, k/16] * qa[m, k] * sb[n, k/16] * qb[n, k]
 * A = quantized activations [M, K], B = quantized weights [N, K], both NVFP4 tensors as
 * described above.  Every product is formed exactly, sums are accumulated in FP32, the two
 * tensor-level scales are applied once to the accumulator, and the result is written as
 * BF16 (nearest even) or FP32.  y: [M, N], row stride ldy elements (ldy >= N).
 * K % 16 == 0; code arrays 16-byte aligned, scale arrays 4-byte aligned when K % 64 == 0;
 * y 16-byte aligned and ldy % 8 == 0 for BF16 (ldy % 4 == 0 for FP32).  M, N >= 0 arbitrary
 * (ragged batches); M == 0 or N == 0 is a no-op.  Results are bit-identical from run to run.
 * layout: mq_layout of all four operand arrays (both operands use the same one).
 */
int nvfp4_gemm(const uint8_t *a_codes, const uint8_t *a_scales, const float *a_alpha_dev,
               const uint8_t *b_codes, const uint8_t *b_scales, const float *b_alpha_dev,
               int64_t M, int64_t N, int64_t K, void *y, int64_t ldy, int out, int layout,
               void *stream);

/*
 * The same product (Section 3.3) with a caller-owned workspace.  A prefill chunk of a few
 * hundred tokens against a layer with a long K and a narrow N has fewer output tiles than the GPU
 * has compute units; with a workspace the K dimension is then cut into slabs across workgroups,
 * each writes FP32 partial sums to the workspace, and a second kernel adds the slabs in ascending
 * order, applies alpha_a * alpha_b and rounds.  Same arguments, requirements, tolerance and
 * run-to-run bit-identity as nvfp4_gemm; the summation order (and so the last bits) may differ
 * from nvfp4_gemm's where slabs are used.
 * workspace: device memory, 16-byte aligned, workspace_bytes >= 0 bytes, or NULL with 0; its
 * contents are undefined afterwards and it must not be used by other work on another stream
 * until this call's kernels have finished.  mq_gemm_workspace_bytes(M, N, K) (host function, no
 * GPU access) returns the size that lets the library choose freely: the most slabs it may take, for either
 * byte order and any number of compute units, * M * N * 4 bytes; never more than 4 MiB, and 0 where
 * slabs are never used (N % 4 != 0, K % 64 != 0, more than 128 output tiles of 64x64, or a K too
 * short for the second pass to pay: below about 7000).  How many of them a call takes, often none
 * (tiles of 32x32 occupy the GPU without), is decided by expected time.  A smaller workspace is
 * legal and only limits the number of slabs.
 */
int64_t mq_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K);
int nvfp4_gemm_ws(const uint8_t *a_codes, const uint8_t *a_scales, const float *a_alpha_dev,
                  const uint8_t *b_codes, const uint8_t *b_scales, const float *b_alpha_dev,
                  int64_t M, int64_t N, int64_t K, void *y, int64_t ldy, int out, int layout,
                  void *workspace, int64_t workspace_bytes, void *stream);

/*
 * The same product for callers that cannot allocate device memory and have no workspace to pass:
 * code under HIP graph capture, tight serving loops, harnesses that forbid hipMalloc.  Arguments,
 * requirements, results (bit-identical) and tolerance as nvfp4_gemm_ws given a workspace of
 * MQ_NOALLOC_SCRATCH_BYTES; the partial sums of the slab-split product go to a static device
 * array of that size inside the library, one copy per GPU, held until the process ends.  The
 * call allocates nothing and frees nothing.  A problem for which mq_gemm_workspace_bytes(M, N, K)
 * exceeds MQ_NOALLOC_SCRATCH_BYTES is rejected with MQ_ERR_SCRATCH before anything is enqueued.
 * Every call on a GPU uses that GPU's one array (nothing in it needs to start at zero: each
 * slab is written before it is read): calls that overlap in time on one GPU, from different
 * streams or threads, race on it; calls on one stream are ordered and safe.
 */
#define MQ_NOALLOC_SCRATCH_BYTES (4u << 20)
int nvfp4_gemm_noalloc(const uint8_t *a_codes, const uint8_t *a_scales, const float *a_alpha_dev,
                       const uint8_t *b_codes, const uint8_t *b_scales, const float *b_alpha_dev,
                       int64_t M, int64_t N, int64_t K, void *y, int64_t ldy, int out, int layout,
                       void *stream);

/*
 * High-precision baseline (the BF16 path that decoding keeps and that the paper's prefill
 * speed-up is measured against): Y = X . W^T, X [M, K] and W [N, K] BF16 with row strides
 * ldx, ldw elements, FP32 accumulation, output as in nvfp4_gemm.
 * K % 8 == 0; x, w 16-byte aligned; ldx % 8 == 0, ldw % 8 == 0; y as in nvfp4_gemm.
 * The same call on the same values gives the same bits.  The order of a row's FP32 sums may depend on its place in X
 * (from K = 4096 on it does in the larger tiles), so two equal rows of one X may differ in the last bits of Y.
 */
int bf16_gemm(const void *x_bf16, int64_t ldx, const void *w_bf16, int64_t ldw,
              int64_t M, int64_t N, int64_t K, void *y, int64_t ldy, int out, void *stream);

/*
 * The same product with a caller-owned workspace, for decode batches (the precision that the
 * decode phase keeps, Section 3.3): 33 to 64 tokens against a weight matrix with a long K and a narrow
 * N re-read the activations once per narrow tile of W, and more tokens with a K above 8192 both operands once per
 * tile; with a workspace the tiles can be wider, K being cut into slabs across workgroups (FP32 partial sums, added in ascending order by a second kernel:
 * bit-identical from run to run; the last bits may differ from bf16_gemm's).  Arguments and
 * requirements as bf16_gemm; workspace as in nvfp4_gemm_ws.
 * mq_bf16_gemm_workspace_bytes(M, N, K) (host function) returns a size that lets the library
 * choose freely: an upper bound of the slabs * M * N * 4 bytes (at most 16 MiB), 0 where slabs are never used:
 * M <= 32, N % 4 != 0, K % 64 != 0; up to 64 tokens also K % 128 != 0, K < 8192, N > 16256, or so few rows of W that even
 * with slabs half of the compute units would stay empty; more tokens K <= 8192, or two slabs of more than 16 MiB
 * (M * N > 2^21).
 */
int64_t mq_bf16_gemm_workspace_bytes(int64_t M, int64_t N, int64_t K);
int bf16_gemm_ws(const void *x_bf16, int64_t ldx, const void *w_bf16, int64_t ldw,
                 int64_t M, int64_t N, int64_t K, void *y, int64_t ldy, int out,
                 void *workspace, int64_t workspace_bytes, void *stream);

/*
 * BF16 activations times NVFP4 weights, for the few tokens of a decode step (W4A16; the prefill's weights, read as they are):
 *    Y[m, n] = alpha_w * sum_k x[m, k] * E4M3(w_scales[n, k/16]) * E2M1(w_codes[n, k])
 * Products are formed in FP16 of x * 2^e, e bringing the token's largest finite magnitude to 2^14 .. 2^15, and of the exact
 * weights: exact for every element of x down to 2^-29 of that magnitude, below that the element is off by at most 2^-38 of it
 * (K % 64 != 0: exact in FP32).  Sums are accumulated in FP32, alpha_w is applied once to the sum, and the result is written as
 * BF16 (nearest even) or FP32.  Bound by reading W up to about 64 tokens; more are computed 64 at a time, reading W again.
 * x: [M, K] BF16, row stride ldx.  K % 16 == 0 (K % 64 == 0 for MQ_LAYOUT_KTILE); x, w_codes 16-byte aligned, ldx % 8 == 0,
 * scale arrays 4-byte aligned when K % 64 == 0; any ldy >= N, y aligned to its element.  M <= 65535, N and K < 2^31.
 * workspace: device memory, 16-byte aligned, of mq_nvfp4_matvec_workspace_bytes(M, N, K) bytes (0 for up to four tokens, two
 * where N >= 8192, of at most 32768 elements in all, K rounded up to a multiple of 128, and where K % 64 != 0), or the call is
 * refused with MQ_ERR_SCRATCH; otherwise as in nvfp4_gemm_ws.
 * Results are bit-identical from run to run.
 */
int64_t mq_nvfp4_matvec_workspace_bytes(int64_t M, int64_t N, int64_t K);
int nvfp4_matvec(const void *x_bf16, int64_t ldx, const uint8_t *w_codes, const uint8_t *w_scales, const float *w_alpha_dev,
                 int64_t M, int64_t N, int64_t K, void *y, int64_t ldy, int out, int layout, void *workspace,
                 int64_t workspace_bytes, void *stream);

/*
 * The attention half of a decoder block over a paged 8-bit cache (the keys and values that a prefill worker leaves for the
 * decode worker, Section 3.3, the paragraph on the disaggregated deployment).
 *
 * The cache of one layer, all dense:
 *    k_codes, v_codes   : uint8 [pages, Hkv, P, D]  FP8 E4M3 (OCP); D is 64, 128 or 256, P (tokens a page) 16, 32, 64 or 128
 *    k_scales, v_scales : uint8 [pages, Hkv]        byte e + 127 for the scale 2^e, -112 <= e <= 119
 * with value code * 2^e.  Sequence b holds kv_lens[b] tokens, the i-th of them in place i % P of page page_table[b, i / P];
 * page_table: int32 [B, W], row stride pt_ld.  In a call the tokens cu_q[b] .. cu_q[b + 1] - 1 of T are the last of sequence
 * b's (kv_lens counts them; a sequence may have none).  cu_q: int32 [B + 1], kv_lens: int32 [B].  All of these are read on the
 * device.  A page number outside 0 .. pages - 1, or a place beyond the table's W * P, is no place: nothing is stored there and
 * no query sees it.  Tokens outside cu_q's ranges belong to no sequence, their outputs are unspecified.
 * W * P <= 2^30, T * Hq < 2^31.  All arrays of codes, BF16 tensors and the table 16-byte aligned, int32 arrays 4-byte aligned,
 * token strides (elements) multiples of 8; the heads of a token are adjacent.
 *
 * mq_rope_table: table[p, i] = gain * cos(p * f_i), table[p, R/2 + i] = gain * sin(p * f_i) for positions p < max_pos, i < R/2,
 * R = rot_dim a multiple of 16 up to 256, angles in binary64, with f_i = base^(-2i/R) (MQ_ROPE_PLAIN), that divided by factor
 * (MQ_ROPE_LINEAR), or between the two by how often the pair turns within original_max_pos (MQ_ROPE_YARN):
 *    f_i = (f_i / factor) * w_i + f_i * (1 - w_i),  w_i = clamp((i - low) / (high - low), 0, 1),
 *    low = floor(d(beta_fast)), high = ceil(d(beta_slow)), d(t) = R * ln(original_max_pos / (2 pi t)) / (2 ln base), both clamped to 0 .. R - 1
 *    (high = low + 0.001 where equal);  base > 1, factor >= 1, beta_fast >= beta_slow > 0.
 * gain multiplies both (what a scaling asks of the scores: 0.1 ln(factor) + 1 for YaRN); 1 otherwise.
 *
 * kv8_append: rotates queries and keys and appends keys and values.  The pairs (a, b) of a head's first rot_dim elements are
 * elements i and R/2 + i, or 2i and 2i + 1 where interleaved is not 0:
 *    a' = a * c_i - b * s_i,  b' = b * c_i + a * s_i     (each step binary32, unfused, the result rounded once to BF16)
 * with the table's row at positions[t], or, positions being NULL, at the token's place in its sequence; a position outside
 * 0 .. max_pos - 1 gives NaN.  q_out receives the queries, dense [T, Hq, D]; rot_dim == 0 (table may be NULL) copies them.
 * Keys (rotated, BF16) and values go to the cache: a page's e is the smallest of -112 .. 119 with which the largest finite
 * magnitude among its new tokens is at most 448 * 2^e, and at least what it was where the page holds earlier tokens of the
 * sequence; those tokens' codes are then brought to the new scale, each rounded once.  code = nearest E4M3 of x / 2^e, ties to
 * even, clipped to +-448; NaN stays NaN.  Pages that two sequences of the call share must not receive tokens.
 *
 * kv8_attention: y[t, h, :] = sum_j p_j v_j, p = softmax_j(sm_scale * (q[t, h, :] . k_j)) over the places j that token t sees:
 * 0 <= j <= pos, its own place, and j > pos - window where window > 0.  Query head h reads key head h / (Hq / Hkv).  A token that
 * sees nothing gets zeros (one that sees scores of -infinity alone NaN, as the formula).  Products of BF16 numbers, sums and the
 * softmax's maxima and sums in FP32, probabilities rounded to BF16 for the product with the values, y BF16 (nearest even),
 * [T, Hq, D] with token stride ldy.  Hq % Hkv == 0, sm_scale finite and > 0.  Places that no query of the call sees may hold
 * anything.  The sums of p_j v_j are divided by the sum of exponentials at the end: where the magnitudes of a row's values add up
 * to 2^119 or more they may overflow, and scores are to stay below 2^30 in magnitude.
 * workspace: as in nvfp4_gemm_ws; with mq_kv8_attention_workspace_bytes(...) bytes (at most 64 MiB; less counts as none) long
 * histories are cut across workgroups where the call has too few of them to fill the GPU twice, and a second kernel adds the
 * parts in ascending order: bit-identical from run to run.
 */
typedef enum {
    MQ_ROPE_PLAIN = 0,
    MQ_ROPE_LINEAR = 1,
    MQ_ROPE_YARN = 2
} mq_rope;
int mq_rope_table(float *table, int64_t max_pos, int rot_dim, double base, int scaling, double factor, int64_t original_max_pos,
                  double beta_fast, double beta_slow, double gain, void *stream);
int kv8_append(const void *q_bf16, int64_t ldq, const void *k_bf16, int64_t ldk, const void *v_bf16, int64_t ldv, void *q_out,
               uint8_t *k_codes, uint8_t *k_scales, uint8_t *v_codes, uint8_t *v_scales, int64_t pages, int P, int Hq, int Hkv, int D,
               const int32_t *page_table, int64_t pt_ld, int64_t W, const int32_t *cu_q, const int32_t *kv_lens, int64_t B, int64_t T,
               const float *table, int64_t max_pos, int rot_dim, const int32_t *positions, int interleaved, void *stream);
int64_t mq_kv8_attention_workspace_bytes(int64_t T, int64_t B, int Hq, int Hkv, int D);
int kv8_attention(const void *q_bf16, int64_t ldq, const uint8_t *k_codes, const uint8_t *k_scales, const uint8_t *v_codes,
                  const uint8_t *v_scales, int64_t pages, int P, int Hq, int Hkv, int D, const int32_t *page_table, int64_t pt_ld,
                  int64_t W, const int32_t *cu_q, const int32_t *kv_lens, int64_t B, int64_t T, float sm_scale, int64_t window,
                  void *y, int64_t ldy, void *workspace, int64_t workspace_bytes, void *stream);

/*
 * Decoding with drafted tokens over the same cache.  A drafter proposes a tree of tokens for each sequence; the model takes all of
 * them in one step, as the sequence's new tokens, and the path that its own choices confirm is kept.  One round, all of it on
 * the device:
 *    mq_draft_tree, then in every layer kv8_append (with the positions) and kv8_tree_attention, the logits of every
 *    token, mq_sample, mq_draft_accept, and in every layer kv8_compact.
 * cu_q and kv_lens as above: the new tokens are counted in kv_lens, and `start` is the first one's place, kv_lens[b] - n.  A token's
 * number is its place among its sequence's new ones.  parents: int32 [T], each the number of an earlier token of the sequence;
 * anything else (-1) makes a root.  Usually token 0 is the last one that was kept, and the root of all others.  int32 arrays 4-byte aligned.
 *
 * mq_draft_tree: tree [T, words] (dense): bit j % 32 of word j / 32 of a token is set where token number j is the token itself or above it,
 * and, where window > 0, fewer than `window` levels above.  positions [T]: start + the number of tokens above it.  1 <= words <= 32.  A
 * token whose own number is 32 * words or more gets no bits and its place as position.
 *
 * kv8_tree_attention: kv8_attention, but that of the new tokens a token sees those whose bits in its row of `tree` are set (none from
 * number 32 * words on), itself among them only if its bit is; and of the places before `start` all or, where window > 0, those
 * j > position - window.  positions: int32 [T], or NULL for the tokens' places; one below `start` counts as `start`.  Rows that see nothing,
 * precision, requirements and workspace as there.
 *
 * mq_sample: tokens[r] from row r of the logits [rows, V], BF16 or FP32 (type: MQ_OUT_BF16 or MQ_OUT_FP32), row stride ld >= V elements,
 * aligned to their elements.  The tokens of a row are ordered by falling logit, the lower index first among equals; w = exp((logit -
 * largest) / temperature).  Kept are the first top_k (all where top_k <= 0), of those the ones with less than top_p times their mass in
 * front of them (all where top_p >= 1), and of those the ones with w >= min_p (all where min_p <= 0); the first of the order always.  The
 * result is the lowest index up to which (and with it) the kept tokens' mass is more than uniform[r] times that of all kept ones; a draw of 1 or more counts
 * as one just below, one below 0 or NaN as 0.  A temperature that is not above 0 gives the first of the order, as a top_p or min_p of NaN does.  NaN
 * and -infinity are never chosen (-1 where a row has nothing else), +infinity has all the mass.  temperature, top_p, min_p: float
 * [rows], top_k: int32 [rows], each or NULL (1, none); uniform: float [rows].  Weights and sums in 64 bits, weights to 2^-34 of
 * their value (where |logit| is below 2^18 times the temperature) and top_p to 2^-32; those below 2^-43 of the largest may count as none.
 * Tokens of equal logits weigh the same: a border or a draw between two of them falls as defined.  rows, V <= 2^20.  Bit-identical from run to run.
 * workspace: as in nvfp4_matvec, of mq_sample_workspace_bytes(rows, V) bytes (0 for rows of at most 8192 logits).
 *
 * mq_draft_accept: sampled [T]: the token that the model chose behind each new token; tokens [T]: the drafted ones.  From token 0 on the path
 * goes to the lowest-numbered child whose token is the one sampled at its parent, while there is one.  path [T]: at cu_q[b] the numbers
 * of sequence b's path, then -1; counts [B]: its length (0 where the sequence has no new tokens); next [B]: the token
 * sampled at its end (-1 there); lens_out [B]: kv_lens - n + count, at least 0.
 *
 * kv8_compact: the places start + path[i] to start + i, i < counts[b], path strictly rising, 0 <= path[i] < n.  A page's exponent becomes the smallest
 * with which the finite magnitudes that come from other pages are at most 448 * 2^e, and at least what it was; codes that come, and
 * those in front of the first that moves, are brought to it with one rounding each as in kv8_append.  All other places
 * are left as they are.  A place that has no page is neither read nor written.  Pages that hold places
 * behind `start` of one sequence must not be another's.
 */
int mq_draft_tree(const int32_t *parents, const int32_t *cu_q, const int32_t *kv_lens, int64_t B, int64_t T, int words, int64_t window,
                  uint32_t *tree, int32_t *positions, void *stream);
int kv8_tree_attention(const void *q_bf16, int64_t ldq, const uint8_t *k_codes, const uint8_t *k_scales, const uint8_t *v_codes,
                       const uint8_t *v_scales, int64_t pages, int P, int Hq, int Hkv, int D, const int32_t *page_table, int64_t pt_ld,
                       int64_t W, const int32_t *cu_q, const int32_t *kv_lens, int64_t B, int64_t T, const uint32_t *tree, int words,
                       const int32_t *positions, float sm_scale, int64_t window, void *y, int64_t ldy, void *workspace,
                       int64_t workspace_bytes, void *stream);
int64_t mq_sample_workspace_bytes(int64_t rows, int64_t V);
int mq_sample(const void *logits, int64_t rows, int64_t V, int64_t ld, int type, const float *uniform, const float *temperature,
              const int32_t *top_k, const float *top_p, const float *min_p, int32_t *tokens, void *workspace, int64_t workspace_bytes,
              void *stream);
int mq_draft_accept(const int32_t *parents, const int32_t *tokens, const int32_t *sampled, const int32_t *cu_q, const int32_t *kv_lens,
                    int64_t B, int64_t T, int32_t *path, int32_t *counts, int32_t *next, int32_t *lens_out, void *stream);
int kv8_compact(uint8_t *k_codes, uint8_t *k_scales, uint8_t *v_codes, uint8_t *v_scales, int64_t pages, int P, int Hkv, int D,
                const int32_t *page_table, int64_t pt_ld, int64_t W, const int32_t *cu_q, const int32_t *kv_lens, int64_t B, int64_t T,
                const int32_t *path, const int32_t *counts, void *stream);

/* Human-readable name of an mq_status value (static storage). */
const char *mq_status_string(int status);

/* hipError_t of the most recent failed launch on the calling thread (0 if none). */
int mq_last_hip_error(void);

/* Library version, "major.minor". */
const char *mq_version(void);

#ifdef __cplusplus
}
#endif
#endif /* MIXQUANT_H */
