/*
 * sharq.h -- C ABI of the SharQ sparse-dense FP4 linear layer for AMD Instinct
 * MI355X (gfx950).
 *
 * SharQ (arXiv 2606.26587) approximates a linear layer Y = X W^T by splitting
 * the activation online into an N:M sparse FP4 backbone and a dense FP4
 * residual taken against the *dequantized* backbone, then summing two FP4
 * GEMMs that read one shared FP4 weight payload (Sec. 3.3 eqs.
 * "sharq-sparse-backbone", "sharq-quantized-backbone", "sharq-residual",
 * "sharq-output"; Sec. 3.4).  Between a decoder layer's qkv linear and its o
 * linear stand a paged key/value cache, in bf16, E4M3 or the library's MXFP4, and
 * the attention that reads it (sharq_kv_append, sharq_kv_read, sharq_attention).
 * Around them stand what a server does between two steps: the tables that these
 * calls take, from the requests' lengths (sharq_kv_assign), and beam search's choice
 * of the next tokens with the reordering of the cached states behind it
 * (sharq_beam_select, sharq_beam_reorder, sharq_kv_copy).
 *
 * Conventions for every entry point
 *   - Tensor pointers are DEVICE pointers owned by the caller; the library
 *     allocates nothing, keeps no global state and never synchronizes.  Calls that
 *     need scratch memory (sharq_attention, sharq_kv_assign, sharq_beam_select) take
 *     it as an argument.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream);
 *     all work is enqueued asynchronously on it.
 *   - Errors are returned, never thrown.  Arguments are validated before any
 *     launch: SHARQ_EINVAL (NULL pointer, negative size, K not a positive
 *     multiple of 32, K % m != 0, leading dimension < K or < N),
 *     SHARQ_EUNSUPPORTED (a format / pattern / dtype combination that is not
 *     built), SHARQ_EALIGN (a pointer not aligned as stated below),
 *     SHARQ_EHIP (the HIP runtime reported an error at launch).
 *   - Inputs must be finite; NaN or Inf inputs give unspecified results.
 *   - Row counts of 0 are valid and launch nothing; the buffers of an empty
 *     tensor may then be NULL.
 *
 * Numeric formats (App. A.1 of the paper)
 *   E2M1 element code: bit 3 = sign, bits 0-2 index {0, .5, 1, 1.5, 2, 3, 4, 6}.
 *   MXFP4: E2M1 + one E8M0 scale per 32 consecutive K values; E8M0 code c
 *          means 2^(c-127).  NVFP4: E2M1 + one E4M3 scale (bias 7, max 448)
 *          per block + one fp32 per-tensor scale.
 *   HiF4 (App. "HiFloat4 (HiF4) Data Format"): units of 64 K positions; each
 *          element an S1P2 code (bit 3 sign, bits 0-2 magnitude m, value
 *          m/4); per unit 4 metadata bytes [E6M2, E1_8, E1_16 low, E1_16
 *          high]: an E6M2 scale (6 exponent bits, bias 48, 2 mantissa bits,
 *          normal values only) and one-bit micro-exponents per 8 and per 4
 *          elements (bit j = group j); value = E6M2 * 2^(E1_8 + E1_16) *
 *          S1P2 (eq. "hif4-value").  The 4 bytes of a unit occupy the 2-byte
 *          scale slots of its two 32-position blocks.  K must be a multiple of
 *          64; built with the 2:4 pattern, SHARQ_MODE_SHARQ, no grouped form.
 *   Two 4-bit codes per byte, the element with the lower K index in the low
 *   nibble.
 *
 * Buffer layout: PANEL-MAJOR.  Every buffer below holds a fixed number of
 * bytes per 32 consecutive K positions of a row (its "row bytes").  K is cut
 * into panels of SHARQ_PANEL_K = 128 positions (the last panel is narrower
 * when K % 128 != 0); panel p stores the row bytes of ALL rows of the tensor
 * for K range [128 p, 128 p + width_p), row after row, and panels follow each
 * other.  Byte offset of (panel p, row r) in a buffer with b bytes per 32 K
 * positions and R rows: p * R * 4 b + r * (width_p / 32) * b.  A tile of
 * consecutive rows is thus one contiguous run per panel, which is how the
 * GEMM streams it; a single row is still addressable (row gathers).  The
 * total size equals the row-major size R * (K / 32) * b.
 */
#ifndef SHARQ_H
#define SHARQ_H

#define SHARQ_PANEL_K 128

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#ifndef SHARQ_API
#define SHARQ_API __attribute__((visibility("default")))
#endif

typedef enum {
  SHARQ_OK = 0,
  SHARQ_EINVAL = 1,
  SHARQ_EUNSUPPORTED = 2,
  SHARQ_EALIGN = 3,
  SHARQ_EHIP = 4
} sharq_status;

typedef enum { SHARQ_MXFP4 = 0, SHARQ_NVFP4 = 1, SHARQ_HIF4 = 2 } sharq_format;

typedef enum { SHARQ_BF16 = 0, SHARQ_F16 = 1, SHARQ_F32 = 2 } sharq_dtype;

/* N:M activation pattern: keep the n largest magnitudes of every m consecutive
 * K positions (eq. "dynamic-mask").  pairs = 1 selects in pairs, NVFP4's
 * "4:8 in pairs" (App. A.1.4; Fig. 2 "pair-topk"): the m positions of a group
 * are m/2 adjacent pairs (2i, 2i+1), and the n/2 pairs with the largest score
 * max(|y_2i|, |y_2i+1|) survive whole (ties -> lower pair).  Built: 2:4, 4:8
 * and 4:8 in pairs (with either format). */
typedef struct {
  int32_t n, m;
  int32_t pairs;   /* 0: element-wise top-n, 1: in pairs */
} sharq_pattern;

/*
 * E8M0 scale rule of MXFP4 (ablation flag).  SHARQ_SCALE_FLOOR, the default,
 * is the OCP Microscaling rule e = floor(log2 amax) - 2: a block peak above
 * 6 * 2^e saturates at 6.  SHARQ_SCALE_CEIL takes e = ceil(log2(amax / 6)),
 * the group scale amax / 6 of Sec. 3.1 eq. "group-quant" rounded up to a
 * power of two so that nothing clips (App. A.1.1: a power-of-two scale cannot
 * bring every block peak to the E2M1 maximum).  Both clamp at -127 and give
 * -127 to an all-zero block.  Built for MXFP4 in SHARQ_MODE_SHARQ.
 */
typedef enum { SHARQ_SCALE_FLOOR = 0, SHARQ_SCALE_CEIL = 1 } sharq_scale_rule;

/*
 * Path combination of a prepared activation (Sec. 4.4, table
 * "ablation-combination"; Sec. 3.1 eq. "direct-sparse-quant"; the
 * round-to-nearest FP4 rows of table "ablation-format").  Every mode has two
 * path slots: path 1 quantizes y, path 2 quantizes the residual of y against
 * path 1's dequantized values; the GEMM sums the paths' products into one
 * accumulator.  A sparse path keeps the top n of every m of ITS OWN input and
 * quantizes the kept values in blocks of 32 logical positions (the backbone
 * quantizer); a dense path is the format's plain quantizer (MXFP4 per 32,
 * NVFP4 per 16).  NVFP4 uses one per-tensor scale for both paths.
 *
 *   mode                       path 1   path 2
 *   SHARQ_MODE_SHARQ           sparse   dense     the method (default, 0)
 *   SHARQ_MODE_SPARSE          sparse   -         no residual compensation
 *   SHARQ_MODE_DENSE           -        dense     plain FP4 (RTN), i.e. n = 0
 *   SHARQ_MODE_DENSE_DENSE     dense    dense     two dense paths
 *   SHARQ_MODE_SPARSE_SPARSE   sparse   sparse    second mask chosen on |R|
 *
 * Only SHARQ_MODE_SHARQ is the method; the others exist for ablation.  They
 * run on generic (non-interleaved) GEMM kernels and are not built for the
 * grouped form or with the fused residual add.
 */
typedef enum {
  SHARQ_MODE_SHARQ = 0,
  SHARQ_MODE_SPARSE = 1,
  SHARQ_MODE_DENSE = 2,
  SHARQ_MODE_DENSE_DENSE = 3,
  SHARQ_MODE_SPARSE_SPARSE = 4
} sharq_mode;

/*
 * A prepared activation: the output of sharq_prepare, the input of
 * sharq_linear / sharq_linear_grouped.  One row per token; panel-major (see
 * above).  Row bytes per row are listed as [rows][...].  In SHARQ_MODE_SHARQ:
 *
 *   sp_codes [rows][K*n/m/2]  backbone E2M1 codes of the kept positions only,
 *                             in ascending K order (Sec. 3.4: "quantizes and
 *                             compresses it"); 16-byte aligned.
 *   sp_meta  [rows][K/8]      which positions were kept.  2:4: per group of 4
 *                             the two kept indices i0 < i1 as i0 | i1 << 2 (a
 *                             nibble), two groups per byte, even group low.
 *                             4:8 (also in pairs): per group of 8 an 8-bit
 *                             keep mask (bit p = position p kept).  4-byte
 *                             aligned.
 *   sp_scale [rows][K/32]     backbone block scale per 32 logical K positions
 *                             (Fig. 2 "sparse group-32 scales"): E8M0 (MXFP4)
 *                             or E4M3 (NVFP4); HiF4: [rows][K/16], the unit
 *                             metadata of each 64 logical positions.
 *   dn_codes [rows][K/2]      residual E2M1 codes, all positions; 16-byte aligned.
 *   dn_scale [rows][K/32] (MXFP4, E8M0) | [rows][K/16] (NVFP4, E4M3; HiF4,
 *                             unit metadata).
 *   tensor_scale              NVFP4: one fp32 per-tensor scale S (device); the
 *                             element value is code * block_scale * S.
 *                             MXFP4: unused (may be NULL).
 *   mode                      SHARQ_MODE_SHARQ (0).
 *   dn_meta                   unused (may be NULL).
 *   sp_dense [rows][K/2]      optional (NULL = none), MXFP4 and NVFP4 (not
 *                             HiF4): the backbone's codes at all K positions
 *                             (dropped positions code 0), laid out like
 *                             dn_codes, with the backbone's scales sp_scale;
 *                             16-byte aligned.  When given, the preparation
 *                             writes it beside the compressed form, and the
 *                             main kernels of sharq_linear and (MXFP4)
 *                             sharq_linear_grouped (K a multiple of 128) read
 *                             it instead of expanding sp_codes / sp_meta:
 *                             gfx950 has no sparse FP4 matrix instruction, so
 *                             the backbone runs dense anyway, and the copy
 *                             (K/2 more bytes per row) takes the expansion
 *                             out of every column tile.
 *                             Dense-only form: with sp_dense given, sp_codes
 *                             and sp_meta may both be NULL (K a multiple of
 *                             128, SHARQ_MODE_SHARQ); the preparation then
 *                             writes the backbone as the dense copy alone
 *                             (0.5 B per element instead of 0.375 + 0.5), and
 *                             every GEMM reads that copy.
 *   scale_rule                sharq_scale_rule of both paths' E8M0 scales
 *                             (MXFP4; SHARQ_SCALE_FLOOR = 0 by default).
 *   dbg_mask [rows][K/8]      optional (NULL = none) debug output of
 *                             sharq_prepare: the N:M keep mask, bit p of every
 *                             group of 8 positions set when position p was
 *                             kept, laid out like the 4:8 metadata (4 bytes
 *                             per 32 positions, panel-major); 4-byte aligned.
 *   dbg_r    [rows] fp32      optional debug output: the RMSNorm reciprocal r
 *                             of every row (written only when gamma is given).
 *                             Both are for parity triage; MXFP4 and NVFP4,
 *                             SHARQ_MODE_SHARQ.
 *
 * Other modes: path 1 lives in sp_codes / sp_meta / sp_scale and path 2 in
 * dn_codes / dn_meta / dn_scale.  A sparse path has the backbone layout above
 * (codes [rows][K*n/m/2], meta [rows][K/8], scale [rows][K/32]); a dense path
 * the residual layout (codes [rows][K/2], no meta, scale [rows][K/32] MXFP4 or
 * [rows][K/16] NVFP4); an absent path's buffers are unused and may be NULL.
 * sharq_act_buffer_bytes_mode gives every size (0 = unused).  Alignment as
 * above (dn_meta 4-byte aligned).
 */
typedef struct {
  int64_t rows, K;
  sharq_format fmt;
  sharq_pattern nm;
  uint8_t *sp_codes;
  uint8_t *sp_meta;
  uint8_t *sp_scale;
  uint8_t *dn_codes;
  uint8_t *dn_scale;
  float *tensor_scale;
  sharq_mode mode;
  uint8_t *dn_meta;
  uint8_t *sp_dense;
  sharq_scale_rule scale_rule;
  uint8_t *dbg_mask;
  float *dbg_r;
} sharq_act;

/*
 * A quantized weight: ONE shared FP4 payload for both paths with
 * path-specific scale views (Sec. 3.4 "Shared FP4 weights with path-specific
 * scales"; Fig. 2).  W is [N][K] (out-features x in-features), Y = X W^T;
 * each expert's buffers are panel-major over its N rows.
 * `experts` weights of identical shape may be stacked back to back (MoE);
 * expert e starts at codes + e*N*K/2 and scale + e*N*(K/32).
 *
 *   codes    [experts][N][K/2]   E2M1, 16-byte aligned.
 *   scale    [experts][N][K/32]  E8M0 (MXFP4, both paths) or E4M3 (NVFP4,
 *                                sparse view: one scale per 32).
 *   scale_dn [experts][N][K/16]  NVFP4 dense view: each per-32 scale repeated
 *                                for its two 16-element halves.  MXFP4: equal
 *                                to `scale`.
 *   HiF4: scale [experts][N][K/16] holds the unit metadata, one view for
 *   both paths (scale_dn unused, may equal `scale`).
 *   tensor_scale [experts]       NVFP4 per-tensor scale(s) S_w (device);
 *                                MXFP4: unused.
 *   scale_rule                   MXFP4: the sharq_scale_rule sharq_quantize_weight
 *                                applies (the GEMMs ignore it).
 */
typedef struct {
  int64_t N, K, experts;
  sharq_format fmt;
  uint8_t *codes;
  uint8_t *scale;
  uint8_t *scale_dn;
  float *tensor_scale;
  sharq_scale_rule scale_rule;
} sharq_weight;

/* Bytes of each buffer of a prepared activation / quantized weight (host-side
 * sizing helpers, no device work).  Return 0 for an invalid combination. */
SHARQ_API size_t sharq_act_buffer_bytes(int64_t rows, int64_t K, sharq_format fmt, sharq_pattern nm,
                              int32_t which /* 0 sp_codes, 1 sp_meta, 2 sp_scale, 3 dn_codes, 4 dn_scale */);
SHARQ_API size_t sharq_weight_buffer_bytes(int64_t N, int64_t K, sharq_format fmt,
                                 int32_t which /* 0 codes, 1 scale, 2 scale_dn */);
/* Buffer sizes of a prepared activation in a given mode; which 5 = dn_meta.
 * 0 for a buffer the mode does not use, or for an invalid combination. */
SHARQ_API size_t sharq_act_buffer_bytes_mode(int64_t rows, int64_t K, sharq_format fmt, sharq_pattern nm,
                                   sharq_mode mode, int32_t which);

/*
 * Quantize a weight W [N][K] (row stride ldw elements, dtype wdt = BF16 or
 * F32) once into the shared FP4 payload and its scale views (Fig. 2 "weight
 * preparation").  MXFP4: per row, per 32 K values, E8M0 = floor(log2 amax) - 2
 * (OCP rule, clamped at -127), codes = E2M1(w / 2^e), ties to even, saturating.
 * (out->scale_rule = SHARQ_SCALE_CEIL: ceil(log2(amax / 6)) instead).
 * NVFP4: S_w = amax(W)/2688 computed on the device, E4M3 per 32, dense view
 * duplicated per 16.  HiF4: units of 64 along K, the conversion of the HiF4
 * appendix (its algorithm "bf16-to-hif4") on the fp32 values.  `out` fields
 * N, K, fmt, scale_rule and the buffers must be set by the caller; experts
 * must be 1.  The format and the rule travel in `out` rather than as
 * arguments, so that the weight descriptor records what its bytes mean.
 */
SHARQ_API sharq_status sharq_quantize_weight(const void *W, sharq_dtype wdt, int64_t N, int64_t K, int64_t ldw,
                                   sharq_weight *out, void *stream);

/*
 * Fused activation preparation (Sec. 3.4 "Fused sparse-residual preparation";
 * Fig. 2): one kernel that, per row of X [M][K] (row stride ldx elements,
 * dtype xdt = BF16):
 *   1. if gamma != NULL (bf16 [K]): y = (x * r) * gamma with
 *      r = 1/sqrt(mean(x^2) + eps) (sum of squares as a balanced binary tree
 *      in fp32, r rounded from fp64); else y = x;
 *   2. keeps the n largest |y| of every group of m (ties -> lower index),
 *      or the n/2 best pairs when nm.pairs = 1;
 *   3. quantizes the kept values per 32 logical positions (backbone);
 *   4. forms the residual R = y - dequant(backbone) (eq. "sharq-residual");
 *   5. quantizes R densely.
 * NVFP4 additionally needs the per-tensor scale S: if tensor_scale_in is NULL
 * the library computes S = amax(y)/2688 over the whole call in a pre-pass
 * (one more read of X) and writes it to out->tensor_scale; otherwise
 * *tensor_scale_in (device) is used and copied there.
 * out->rows, K, fmt, nm and the buffers must match the arguments.
 * out->mode selects the path combination (see sharq_mode): steps 2-5 then
 * become path 1 on y, the residual R = y - dequant(path 1), and path 2 on R.
 * A mode with a sparse path needs a built pattern; SHARQ_MODE_DENSE and
 * SHARQ_MODE_DENSE_DENSE ignore nm (it must still be valid).
 */
SHARQ_API sharq_status sharq_prepare(const void *X, sharq_dtype xdt, int64_t M, int64_t K, int64_t ldx,
                           const void *gamma, float eps, sharq_pattern nm, sharq_format fmt,
                           const float *tensor_scale_in, sharq_act *out, void *stream);

/*
 * Preparation with the residual add that precedes a transformer block's
 * RMSNorm fused in on the producer side (Sec. 4.3: the preparation absorbs
 * the preprocessing steps of the data flow instead of running them as
 * separate operators).  Per element, h = bf16(x + residual): the two bf16
 * values added in fp32 and rounded to nearest even once.  h is written to
 * h_out (bf16 [M][K], row stride ldh; it may be `residual` itself, updated in
 * place, when ldh == ldr) and then prepared exactly as sharq_prepare prepares
 * X.  residual: bf16 [M][K], row stride ldr.  Both 16-byte aligned with
 * 16-byte row strides.  With NVFP4 and no tensor_scale_in the amax pre-pass
 * forms h as well.  Other arguments, errors and outputs as for sharq_prepare;
 * out->mode must be SHARQ_MODE_SHARQ (others: SHARQ_EUNSUPPORTED).
 */
SHARQ_API sharq_status sharq_prepare_residual(const void *X, const void *residual, void *h_out, sharq_dtype xdt,
                                    int64_t M, int64_t K, int64_t ldx, int64_t ldr, int64_t ldh,
                                    const void *gamma, float eps, sharq_pattern nm, sharq_format fmt,
                                    const float *tensor_scale_in, sharq_act *out, void *stream);

/*
 * Preparation of a down projection's input with the SiLU.mul that produces it
 * fused in on the producer side (Sec. 4.3: the preparation absorbs the
 * preprocessing steps of the data flow).  Per element,
 * h = bf16(SiLU(g) * u), SiLU(g) = g / (1 + exp(-g)), by one fixed fp32
 * recipe: t = e^-|g| (Cody-Waite argument reduction and the degree-7 Taylor
 * polynomial, within 2 ulp), s = g / (1 + t) for g >= 0 and g t / (1 + t)
 * below (correctly rounded division), h = bf16(s u) to nearest even.  h is
 * thus a fixed function of (g, u), within one bf16 step of the exactly
 * rounded value; inputs must keep s u finite.  h is prepared without RMSNorm
 * exactly as sharq_prepare prepares X, and written to h_out (bf16 [M][K], row stride ldh) when h_out is not NULL.
 * gate, up: bf16 [M][K], row strides ldg, ldu (e.g. the two halves of a
 * gate/up projection's output, ldg = ldu = 2K); 16-byte aligned with 16-byte
 * row strides.  With NVFP4 and no tensor_scale_in the amax pre-pass forms h
 * as well.  Modes other than SHARQ_MODE_SHARQ and HiF4: SHARQ_EUNSUPPORTED.
 * Other arguments, errors and outputs as for sharq_prepare.
 */
SHARQ_API sharq_status sharq_prepare_silu_mul(const void *gate, const void *up, void *h_out, sharq_dtype xdt,
                                    int64_t M, int64_t K, int64_t ldg, int64_t ldu, int64_t ldh,
                                    sharq_pattern nm, sharq_format fmt, const float *tensor_scale_in,
                                    sharq_act *out, void *stream);

/*
 * Two-path output (eq. "sharq-output"; Sec. 3.4 "Residual path compensation
 * by accumulation"): Y [rows][N] (row stride ldy, dtype ydt) =
 *   dequant(backbone) * dequant_sp(W)^T + dequant(residual) * dequant_dn(W)^T,
 * both products accumulated in one fp32 accumulator and written once.
 * The activation and weight formats must match.  MXFP4 runs on the
 * block-scaled FP4 matrix cores; NVFP4 (whose E4M3 block scales those cannot
 * apply) multiplies the exactly dequantized values q * d on 16-bit matrix
 * cores (in fp16 or bf16, both exact for every q * d; where the kernel for large
 * M adds the two paths' values before it multiplies, only where that sum is
 * exact too) and applies S_x * S_w once to the fp32 sums.  That choice is made
 * for 32 consecutive rows together, from their block scales: at the same M a
 * row's fp32 sums may be rounded in another order when other rows of its 32
 * change, within the same error bound.  NVFP4 needs
 * a->tensor_scale and w->tensor_scale.  For the other modes of a->mode, Y is the sum over the
 * mode's paths, each against the weight's view of its kind (sparse view for a
 * sparse path, dense view for a dense one).
 */
SHARQ_API sharq_status sharq_linear(const sharq_act *a, const sharq_weight *w, void *Y, sharq_dtype ydt,
                          int64_t ldy, void *stream);

/*
 * Preparation and two-path output in one call (Sec. 4.3: the fused
 * preparation, the shared weight and the accumulating residual path keep the
 * data flow close to a single linear kernel; Sec. 3.4; Sec. 3.3 eq.
 * "sharq-output"): exactly sharq_prepare(X ..., act) followed by
 * sharq_linear(act, w, Y ...), with every argument of both validated before
 * anything is launched.  For a few rows (decode: MXFP4, the method's path
 * combination, K a multiple of 128 up to 16384, M <= 4 when the prepared rows
 * fit in LDS) it runs as ONE kernel: each workgroup of the small-M GEMM
 * prepares the rows in its prologue and workgroup 0 writes them to `act`;
 * the outputs (act's buffers and Y) are bit-identical to the two calls.
 */
SHARQ_API sharq_status sharq_prepare_linear(const void *X, sharq_dtype xdt, int64_t M, int64_t K, int64_t ldx,
                                            const void *gamma, float eps, sharq_pattern nm, sharq_format fmt,
                                            const float *tensor_scale_in, sharq_act *act, const sharq_weight *w,
                                            void *Y, sharq_dtype ydt, int64_t ldy, void *stream);

/*
 * Grouped form for mixture-of-experts layers (the MoE configuration of the
 * paper's evaluation, Sec. 4.1-4.2, Qwen3-30B-A3B): the two-path output of
 * Sec. 3.3 eq. "sharq-output" applied per expert to the rows routed to it.
 * For every expert e and every i in [expert_offsets[e], expert_offsets[e+1]),
 *   Y[i] = SharQ(A[row_index ? row_index[i] : i], W_e).
 * The experts' weights are stacked in one sharq_weight (w->experts of them,
 * one shape) rather than passed as an array of descriptors, so that the
 * kernel reads every expert's payload from one base pointer.
 * expert_offsets: device int32 [w->experts + 1], non-decreasing, first 0,
 * last == total.  row_index: device int32 [total], each in [0, a->rows), or
 * NULL.  Y [total][N] (row stride ldy).  Offsets are read on the device; the
 * host never waits for them.  Built for MXFP4 in SHARQ_MODE_SHARQ; NVFP4 or
 * another mode returns SHARQ_EUNSUPPORTED.
 */
SHARQ_API sharq_status sharq_linear_grouped(const sharq_act *a, const int32_t *row_index,
                                  const int32_t *expert_offsets, int64_t total,
                                  const sharq_weight *w, void *Y, sharq_dtype ydt, int64_t ldy,
                                  void *stream);

/*
 * A paged key/value cache: what lies between the qkv projection's output and
 * the o projection's input of a decoder layer whose linears are the ones above.
 * A page holds page_size consecutive tokens of one sequence, for every
 * key/value head; a sequence's page table names its pages in order.
 *
 *   pages, page_size   pages of the pool; tokens of a page, a power of two in
 *                      [16, 1024].
 *   kv_heads, head_dim key/value heads; their width, 64 or 128.
 *                      pages * kv_heads * page_size is below 2^31.
 *   fmt                SHARQ_KV_BF16: k, v bf16 [pages][kv_heads][page_size][head_dim].
 *                      SHARQ_KV_MXFP4: k, v E2M1 codes (two a byte, the lower
 *                      index in the low nibble) [pages][kv_heads][page_size][head_dim/2]
 *                      and k_scale, v_scale E8M0 [pages][kv_heads][page_size][head_dim/32],
 *                      one per 32 consecutive values of a token's head.
 *                      SHARQ_KV_FP8: k, v E4M3 codes (OCP: bias 7, largest value 448,
 *                      0x7F and 0xFF NaN) [pages][kv_heads][page_size][head_dim] and
 *                      k_scale, v_scale E8M0 [pages][kv_heads][page_size/16], one for
 *                      16 consecutive tokens of a page and head: a block.  A value is
 *                      code * 2^(scale - 127), which is a bf16.
 *   scale_rule         MXFP4, FP8: the sharq_scale_rule that sharq_kv_append applies.
 *                      FP8: floor(log2 amax) - 8 (a peak above 448 * 2^e saturates), or
 *                      ceil(log2(amax / 448)), under which nothing does; both at
 *                      least -117.
 *   k, v 16-byte aligned, MXFP4's scales 4-byte aligned.
 */
typedef enum { SHARQ_KV_BF16 = 0, SHARQ_KV_MXFP4 = 1, SHARQ_KV_FP8 = 2 } sharq_kv_format;

typedef struct {
  int64_t pages;
  int32_t page_size, kv_heads, head_dim;
  sharq_kv_format fmt;
  void *k, *v;
  uint8_t *k_scale, *v_scale;
  sharq_scale_rule scale_rule;
} sharq_kv_cache;

/*
 * The sequences of a call.  Sequence s owns the rows [row_offsets[s],
 * row_offsets[s + 1]) of the call's row tensors and has lens[s] tokens in the
 * cache, its rows of this call among them, which are its last ones: row i of
 * its n is the token at position lens[s] - n + i.  A single new token is n = 1,
 * a whole prompt n = lens[s].
 *
 *   seqs, rows    sequences; rows of the row tensors, at least row_offsets[seqs].
 *                 Rows behind the last sequence are padding: neither looked at
 *                 nor written.
 *   max_rows      no sequence has more rows in this call.  (The attention's work is
 *                 split over the chip by max_rows and max_len: bounds far above the
 *                 sequences' own rows and lengths cost time, and workspace.)
 *   max_len       no sequence has more tokens; max_len <= ld_table * page_size
 *                 and at most 2^30.
 *   row_offsets   device int32 [seqs + 1], non-decreasing, first 0.
 *   lens          device int32 [seqs].
 *   page_table    device int32 [seqs][ld_table].  Entries of pages that hold no
 *                 token that the call reads or writes may hold anything.
 * The device arrays are read on the device; the host never waits for them.  An
 * entry of the page table outside [0, pages) is an absent page: its tokens are
 * not stored by sharq_kv_append, read as zeros by sharq_kv_read and invisible to
 * sharq_attention.  So are tokens at negative positions (more rows than
 * lens[s]).  Pages that a call writes belong to one sequence alone.
 */
typedef struct {
  int64_t seqs, rows, max_rows, max_len, ld_table;
  const int32_t *row_offsets, *lens, *page_table;
} sharq_kv_batch;

/* Bytes of each buffer of a cache (0 k, 1 v, 2 k_scale, 3 v_scale), from its
 * sizes and format alone.  0 for an unused buffer or invalid sizes. */
SHARQ_API size_t sharq_kv_buffer_bytes(const sharq_kv_cache *c, int32_t which);

/*
 * Rotates the rows' queries and keys by their positions and puts the keys and
 * values into the cache, in one pass over the qkv projection's output.
 *   Q [rows][q_heads * head_dim], K, V [rows][kv_heads * head_dim]: bf16, row
 *   strides ldq, ldk, ldv elements (slices of one qkv output, usually).
 *   q_heads may be 0 (Q, Q_out unused).
 *   cos, sin: fp32 [angles][head_dim / 2], the angle tables, row = position;
 *   16-byte aligned.  NULL, both of them: nothing is rotated.
 *   positions: device int32 [rows], the rows of the angle tables to use, or
 *   NULL: the tokens' positions in their sequences.
 * With h = head_dim / 2, y_j = x_j cos_j - x_{j+h} sin_j and
 * y_{j+h} = x_{j+h} cos_j + x_j sin_j for j < h, every product and sum rounded
 * to fp32 and the result once to bf16 (Q_out, row stride ldqo; it may be Q
 * itself with ldqo == ldq) or to the cache's format.  Values are not rotated.
 * A row at a negative position, or whose angle is not in the tables, is left
 * out: neither its query nor its key and value are written.
 * SHARQ_KV_FP8: a block's scale is the largest that its tokens have needed.  The
 * tokens before a sequence's first row of this call keep the scale that is there;
 * where the new ones need a larger one, their codes are rounded again to it (which
 * changes only values that become subnormal codes).  Bytes of the block's other
 * slots stay.  A value that is not finite is stored as NaN and does not count for
 * the scale.  Where all of a block's tokens have been left out so far (or their page
 * was absent) nothing has written its scale either, and the byte is what the page held
 * before.  One outside [10, 247] is no scale: the first tokens that are stored then get
 * one of their own.  A caller that leaves out a block's first rows clears the
 * scales (to 0) of pages that are used again; otherwise the byte found there counts.
 */
SHARQ_API sharq_status sharq_kv_append(const void *Q, const void *K, const void *V, sharq_dtype xdt, int64_t q_heads,
                                       int64_t ldq, int64_t ldk, int64_t ldv, const float *cos, const float *sin,
                                       int64_t angles, const int32_t *positions, const sharq_kv_cache *cache,
                                       const sharq_kv_batch *batch, void *Q_out, int64_t ldqo, void *stream);

/*
 * Reads the rows' keys and values back from the cache (keys as they were
 * stored, rotated): K, V [rows][kv_heads * head_dim] bf16, row strides ldk, ldv,
 * 16-byte aligned with 16-byte row strides.  An MXFP4 value E2M1 * 2^e is a
 * bf16, and so is an E4M3 code's, so nothing is rounded.  row_offsets that cover lens read whole sequences.
 */
SHARQ_API sharq_status sharq_kv_read(const sharq_kv_cache *cache, const sharq_kv_batch *batch, void *K, int64_t ldk,
                                     void *V, int64_t ldv, sharq_dtype ydt, void *stream);

/*
 * What a row sees of its sequence: the row at position p sees the tokens
 * t <= p with p - t < window (window 0: all of them) or t < sinks.
 *   scale         factor of the scores q.k, positive, from 2^-100 to 2^100.
 *   prefix_table, prefix_len
 *                 tokens that all sequences of the call share: those at the
 *                 positions below prefix_len (a multiple of page_size, at most
 *                 max_len) lie on the pages of prefix_table (device int32
 *                 [prefix_len / page_size]) for every sequence, whose own page
 *                 table entries for them are not looked at.  Their keys and
 *                 values are then read for all sequences together.  NULL and 0:
 *                 none.  The result is that of the same call without a shared
 *                 prefix whose page tables name these pages, but for the order
 *                 of fp32 sums.
 */
typedef struct {
  float scale;
  int64_t window, sinks;
  const int32_t *prefix_table;
  int64_t prefix_len;
} sharq_attn;

/* Bytes of workspace that sharq_attention needs for these sizes (the device
 * arrays are not looked at); 0: none needed, or invalid arguments. */
SHARQ_API size_t sharq_attention_workspace_bytes(const sharq_kv_cache *cache, const sharq_kv_batch *batch,
                                                 const sharq_attn *attn, int64_t q_heads);

/*
 * Causal attention of the rows over their cached sequences:
 *   O = softmax(scale Q K^T over the visible tokens) V,
 * K and V including the rows' own (appended before).  Query head h reads
 * key/value head h / (q_heads / kv_heads); q_heads is a multiple of kv_heads,
 * at most 128 times.  One call takes prompts, chunks of prompts and single
 * tokens, mixed.
 *   Q, O: bf16 [rows][q_heads * head_dim], row strides ldq, ldo, 16-byte aligned
 *   with 16-byte row strides; O overlaps neither Q nor the cache (O == Q is refused).
 *   lse: fp32 [rows][q_heads] or NULL: the natural logarithm of the sum of
 *   e^score of every row and head.
 *   workspace: device memory of at least sharq_attention_workspace_bytes,
 *   16-byte aligned; its contents before and after mean nothing.  Calls that may
 *   run at the same time need workspaces of their own.
 * A row that sees no token gets O = 0 and lse = -inf.  Cache slots that no row
 * of the call sees may hold anything; the keys, values and queries that are
 * seen must be finite, their scores too.  (A NaN that a row sees makes that row's
 * results NaN, a value's in its column; earlier rows of sequences that hold the
 * token may be NaN as well.)  Products are summed in fp32; the weights are rounded
 * to bf16 for the product with V, their sum is not.
 */
SHARQ_API sharq_status sharq_attention(const void *Q, sharq_dtype xdt, int64_t q_heads, int64_t ldq,
                                       const sharq_kv_cache *cache, const sharq_kv_batch *batch,
                                       const sharq_attn *attn, void *O, int64_t ldo, float *lse, void *workspace,
                                       size_t workspace_bytes, void *stream);

/*
 * Pages that no sequence holds, as a stack.
 *   pages        pages of the pool.
 *   free_pages   device int32 [pages]: the first *count entries are free pages; the
 *                last of them is given out first.
 *   count, count_out
 *                device int32 [1]: entries before and after a call (they may be
 *                the same word).
 */
typedef struct {
  int64_t pages;
  int32_t *free_pages;
  const int32_t *count;
  int32_t *count_out;
} sharq_kv_pool;

/*
 * The requests of a step, one for each sequence of the call that follows.
 *   seqs, rows, max_len, ld_table
 *                as in sharq_kv_batch; rows: entries of the row arrays.
 *   page_size    a power of two in [16, 1024].  seqs * ceil(max_len / page_size) is
 *                at most 2^30.
 *   keep         device int32 [seqs]: cached tokens that stay (0: the sequence is
 *                new, or has ended; fewer than there are: the last ones are dropped).
 *   add          device int32 [seqs]: tokens that this step brings.
 *   held         device int32 [seqs]: columns of its page table that are filled.
 *   held_out     device int32 [seqs]: the same after the call (it may be `held`).
 *   row_offsets  device int32 [seqs + 1], written.
 *   lens         device int32 [seqs], written (it may be `keep`).
 *   page_table   device int32 [seqs][ld_table]: new columns are written.
 *   own_table    device int32 [seqs][ld_table] or NULL: new columns are written
 *                there as well, and pages that go back are taken from it.  Needed for
 *                sequences whose page_table names pages of others (beams that share
 *                a prompt, any tables that sharq_beam_reorder has written): -1 in
 *                own_table where the page is another's.  With NULL, a page that several
 *                rows name would go back once for each of them.
 *   row_seq, positions, slots
 *                device int32 [rows] or NULL: of every row its sequence, its
 *                position and its slot in the pool, page * page_size + position %
 *                page_size, -1 without a page.
 *   missing      device int32 [1] or NULL: columns for which there was no page.
 */
typedef struct {
  int64_t seqs, rows, max_len, ld_table;
  int32_t page_size;
  const int32_t *keep, *add, *held;
  int32_t *held_out, *row_offsets, *lens, *page_table, *own_table;
  int32_t *row_seq, *positions, *slots, *missing;
} sharq_kv_requests;

/* Bytes of workspace that sharq_kv_assign needs; 0 for invalid sizes. */
SHARQ_API size_t sharq_kv_assign_workspace_bytes(const sharq_kv_requests *r);

/*
 * Builds a step's tables on the device: for sequence s, in order,
 *   n_s = add_s, cut where the call's rows end; row_offsets = exclusive sums of n;
 *   lens_s = keep_s + n_s; need_s = ceil(lens_s / page_size) columns.
 * Columns need_s .. held_s - 1 go back onto the stack, in the order of sequences
 * and columns (entries that are no page of the pool are passed over; the table
 * keeps them).  Then columns held_s .. need_s - 1 are given pages from the top of
 * the stack, in the same order; where it is empty they get -1, an absent page, and
 * `missing` counts them.  held_out_s = need_s.  row_offsets, lens and page_table are
 * those of a sharq_kv_batch.  Rows behind the last sequence are left as they were.
 * Calls on the same pool, and calls that share a workspace, run one after the other.
 * Values of the device arrays outside their range (negative, above max_len or the
 * table's columns) count as the nearest inside.  The result does not depend on the
 * order in which the device runs.  workspace: 4-byte aligned.
 */
SHARQ_API sharq_status sharq_kv_assign(const sharq_kv_pool *pool, const sharq_kv_requests *r, void *workspace,
                                       size_t workspace_bytes, void *stream);

/* Bytes of workspace that sharq_beam_select needs; 0 for invalid sizes. */
SHARQ_API size_t sharq_beam_workspace_bytes(int64_t groups, int64_t beams, int64_t vocab);

/*
 * Beam search's choice.  A group has `beams` (1 to 32) hypotheses with scores (sums of
 * log-probabilities), fp32 [groups][beams].  logits [groups * beams][vocab] (dtype
 * BF16, F16 or F32, row stride ld elements, element-aligned).  Candidate (b, v) has
 *   score_b + x_bv - lse_b,  lse_b = ln sum_v e^(x_bv);
 * a beam that is done has one, (b, eos), with score_b.  Of each group the `beams` best,
 * best first, equal ones by the lower b, and those of one beam by their logits, equal
 * ones by the lower v:
 *   scores_out  fp32 [groups][beams] (it may be `scores`)
 *   parents     int32 [groups][beams]: b
 *   tokens      int32 [groups][beams]: v
 *   done        uint8 [groups * beams] (0 or not) or NULL, with eos in [0, vocab)
 *   done_out    uint8 [groups * beams] (it may be `done`), NULL exactly if done is:
 *               done[b], or v == eos.
 *   eos         -1 where there is none (then done is NULL).
 * A logit of -inf is no candidate, nor is any of a beam whose score is not finite or
 * whose logits hold a NaN or +inf.  Where a group has fewer than `beams`
 * candidates, the places behind have score -inf, token -1 and themselves as parent.
 * Scores are compared in 64 bits, whatever their rounding to scores_out.  Exponentials and
 * the sums of 32 of them are fp32: lse_b is within 2^-19 (about 1e-8 measured), and only
 * candidates of different beams that lie closer than that may change places.
 * groups * beams is at most 2^20, beams * vocab at most 2^30.  workspace: 8-byte aligned;
 * calls that may run at the same time need workspaces of their own.
 */
SHARQ_API sharq_status sharq_beam_select(const void *logits, sharq_dtype dtype, int64_t ld, int64_t groups,
                                         int64_t beams, int64_t vocab, const float *scores, const uint8_t *done,
                                         int32_t eos, float *scores_out, int32_t *parents, int32_t *tokens,
                                         uint8_t *done_out, void *workspace, size_t workspace_bytes, void *stream);

/*
 * The states of groups of beams behind a choice.  Beam i of a group goes on from
 * parents[i], int32 [groups][beams].  The beams of a group have the same number of
 * cached tokens, lens (device int32 [groups * beams], the first of each group counts).
 *   table, table_out    device int32 [groups * beams][cols], row strides ldt, ldto (it
 *                       may be `table` with the same stride), or both NULL.
 *                       Whole pages are shared: table_out[i] names its parent's.  The
 *                       page that is partly filled goes to a parent's first child; each
 *                       further child takes over the page of a parent without children
 *                       (in order; there are as many).  Columns behind stay a beam's own.
 *                       Rows then share pages: sharq_kv_assign takes what goes back from
 *                       an own_table, which is not reordered, and a group's beams end
 *                       together.
 *   copies              device int32 [groups * beams][3], with table: (source page, destination
 *                       page, tokens) of what has to be copied into the pages taken over,
 *                       for sharq_kv_copy on the caches of all layers; -1s for
 *                       the others.
 *   tokens, ids, ids_out
 *                       chosen tokens, device int32 [groups][beams], and the sequences'
 *                       tokens, device int32 [groups * beams][id_cols], row strides ldi,
 *                       ldio (ids_out may be `ids`), or all NULL:
 *                       ids_out[i][t] = ids[parents[i]][t] for t < len,
 *                       ids_out[i][len] = tokens[i]; columns behind are left as they were.
 * Parents outside [0, beams) count as the nearest inside.  Outputs overlap inputs only where
 * they are the same array.  groups * beams is at most 2^20.
 */
SHARQ_API sharq_status sharq_beam_reorder(int64_t groups, int64_t beams, const int32_t *parents, const int32_t *lens,
                                          int32_t page_size, const int32_t *table, int64_t ldt, int32_t *table_out,
                                          int64_t ldto, int64_t cols, int32_t *copies, const int32_t *tokens,
                                          const int32_t *ids, int64_t ldi, int32_t *ids_out, int64_t ldio,
                                          int64_t id_cols, void *stream);

/*
 * Copies the first tokens of pages, keys and values of all heads, with their scales:
 * copies, device int32 [n][3]: (source page, destination page, tokens).  An entry whose
 * pages are the same or outside the pool is passed over; tokens above page_size
 * count as page_size.  No page is the destination of two entries, or the destination of
 * one and the source of another.
 */
SHARQ_API sharq_status sharq_kv_copy(const sharq_kv_cache *cache, const int32_t *copies, int64_t n, void *stream);

SHARQ_API const char *sharq_status_str(sharq_status s);

/* Library version string. */
SHARQ_API const char *sharq_version(void);

#ifdef __cplusplus
}
#endif

#endif /* SHARQ_H */
