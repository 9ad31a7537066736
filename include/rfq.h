/*
 * rfq.h -- C ABI of the GB300 (sm_103a) Residual Fallback Quantization
 * (RFQ) linear layer: "Activation Outliers Matter: Robust Recovery for
 * Quantized Multimodal LLMs", Sec. 3.2-3.3 (formats), Sec. 4.3 and
 * Algorithm 1 (method).
 *
 * The layer computes Y = X W for an activation X [M x K] (bf16) and a weight
 * W [K x N] (bf16) as
 *
 *     Y = Q(X) Q(W) + phi * Q(X - Q(X)) Q(W)                  (Eq. rfq)
 *
 * where Q is a block quantizer to a 4-bit format (MXFP4 or HiF4) along K.
 * The paper writes Z = X Y with X [P x R], Y [R x Q]; here P = M, R = K,
 * Q = N and the paper's Y is W.
 *
 * Conventions shared by every entry point:
 *   - Every pointer named "device" is CUDA device memory on the current
 *     device, allocated and owned by the caller; the library never allocates
 *     device memory and never frees a caller's buffer.
 *   - Every device pointer must be 16-byte aligned (RFQ_ERR_ALIGNMENT).
 *   - Calls are asynchronous: they validate the arguments on the host,
 *     enqueue kernels on `stream` (a cudaStream_t; NULL = legacy default
 *     stream) and return.  On any argument error nothing is launched.
 *   - bf16 inputs must be finite; non-finite inputs give unspecified codes
 *     but never a fault.
 *   - The library needs an sm_103 device (GB300); otherwise RFQ_ERR_DEVICE.
 *
 * Storage of a quantized matrix (rfq_qtensor), rows x k, quantized along k:
 *   codes   [rows][k/2] bytes; element 2j of a row in the low nibble of byte
 *           j, element 2j+1 in the high nibble.
 *   MXFP4   E2M1 codes (sign, 2 exponent bits, 1 mantissa bit, Sec. 3.2.2)
 *           with one E8M0 scale byte 2^(byte-127) per 32 elements
 *           (Sec. 3.2 Eq. 3-4).  Scale layouts:
 *             RFQ_SCALE_ROWMAJOR  [rows][k/32] bytes (k % 32 == 0)
 *             RFQ_SCALE_MMA       the tensor-core layout consumed by
 *               rfq_linear (k % 128 == 0): rows padded to a multiple of 128
 *               and split into 512-byte atoms of 128 rows x 4 k-blocks; the
 *               byte for (row m, k-block b) lives at
 *                 ((m/128) * (k/128) + b/4) * 512 + (m%32)*16 + ((m/32)%4)*4 + b%4
 *               Bytes of padding rows (m >= rows) are 0.
 *   HiF4    S1P2 codes (sign, 1 integer bit, 2 fraction bits) with one
 *           32-bit metadata word per 64 elements (Sec. 3.3):
 *           bits [7:0] UE6M2 macro scale (E in [7:2], bias 48; M in [1:0]),
 *           bits [15:8] E1_8 (bit g: group of 8 elements g),
 *           bits [31:16] E1_16 (bit j: sub-group of 4 elements j).
 *           Metadata layouts (k % 64 == 0):
 *             RFQ_SCALE_ROWMAJOR  [rows][k/64] uint32
 *             RFQ_SCALE_MMA       block-major [k/64][rows rounded up to 128]
 *                                 uint32, the layout rfq_linear consumes
 *   BF16    an exact bf16 expansion of a quantized matrix, [rows][k]
 *           (codes = the bf16 data, scales unused): rfq_dequant writes it,
 *           and rfq_linear takes the HiF4 weight in this form.
 *   MXFP8   E4M3 codes (Sec. 3.2.1: sign, 4 exponent bits with bias 7, 3
 *           mantissa bits; exponent field 0 subnormal; no infinity;
 *           S.1111.111 is NaN; largest finite 448), one byte per element:
 *           codes [rows][k]; one E8M0 scale byte per 32 elements with the
 *           MXFP4 scale layouts.  The block exponent is floor(log2 amax) - 8
 *           (clamped to [-127, 127]); elements round to nearest even and
 *           saturate at +-448.  An MXFP4 tensor re-encoded by rfq_convert is
 *           an MXFP8 tensor holding the same values.
 */
#ifndef RFQ_H
#define RFQ_H

#include <stddef.h>
#include <stdint.h>

#if defined(__GNUC__)
#define RFQ_API __attribute__((visibility("default")))
#else
#define RFQ_API
#endif

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    RFQ_OK = 0,
    RFQ_ERR_INVALID_ARG = 1, /* NULL pointer or an enum value out of range */
    RFQ_ERR_SHAPE = 2,       /* sizes violate the call's constraints */
    RFQ_ERR_ALIGNMENT = 3,   /* a device pointer is not 16-byte aligned */
    RFQ_ERR_UNSUPPORTED = 4, /* valid but unimplemented combination */
    RFQ_ERR_CUDA = 5,        /* a CUDA runtime call or a launch failed */
    RFQ_ERR_TIMEOUT = 6,     /* a kernel's bounded wait expired (device status) */
    RFQ_ERR_DEVICE = 7,      /* the current device is not an sm_103 GPU */
    RFQ_ERR_NONFINITE = 8    /* rfq_check_finite found an Inf or NaN (device status) */
} rfq_status;

typedef enum { RFQ_FMT_MXFP4 = 0, RFQ_FMT_HIF4 = 1, RFQ_FMT_BF16 = 2, RFQ_FMT_MXFP8 = 3 } rfq_format;

typedef enum { RFQ_SCALE_ROWMAJOR = 0, RFQ_SCALE_MMA = 1 } rfq_scale_layout;

/* Fallback indicator phi(p, r) of Sec. 4.3 over tiles of p_s rows x r_s
 * columns of X.  The paper gives no formula for it:
 *   RFQ_FALLBACK_NONE  phi = 0: plain W4A4, no residual pathway
 *   RFQ_FALLBACK_ALL   phi = 1 on every tile (the default; Sec. 1 describes
 *                      RFQ as working without threshold-based selection)
 *   RFQ_FALLBACK_AMAX  phi(p, r) = 1 iff max |x| over the tile > tau */
typedef enum {
    RFQ_FALLBACK_NONE = 0,
    RFQ_FALLBACK_ALL = 1,
    RFQ_FALLBACK_AMAX = 2
} rfq_fallback_mode;

typedef enum { RFQ_OUT_F32 = 0, RFQ_OUT_BF16 = 1 } rfq_out_dtype;

typedef struct {
    int32_t fmt;          /* rfq_format */
    int32_t scale_layout; /* rfq_scale_layout (ignored for RFQ_FMT_BF16) */
    int64_t rows;         /* M for an activation, N for a weight */
    int64_t k;            /* length of the quantized (reduction) axis */
    void *codes;          /* device, see "Storage" above */
    void *scales;         /* device, see "Storage" above */
} rfq_qtensor;

typedef struct {
    int32_t mode; /* rfq_fallback_mode */
    float tau;    /* threshold for RFQ_FALLBACK_AMAX */
    int32_t p_s;  /* tile rows (>= 1); rfq_linear reads phi tiles of 128 rows */
    int32_t r_s;  /* tile columns, a multiple of 32; rfq_linear needs a multiple of 128 */
} rfq_fallback;

/* Human-readable name of a status code (static string, never NULL). */
RFQ_API const char *rfq_status_string(rfq_status s);

/* Byte sizes of the code and scale arrays of a rows x k quantized matrix in
 * the given format and scale layout (host only, no device work).
 * Errors: RFQ_ERR_INVALID_ARG (NULL outputs, bad enums), RFQ_ERR_SHAPE
 * (rows < 0, k not a multiple of the layout's granule). */
RFQ_API rfq_status rfq_qtensor_bytes(int32_t fmt, int32_t scale_layout, int64_t rows, int64_t k,
                             size_t *codes_bytes, size_t *scale_bytes);

/* Weight quantization W~ = Q(W) (Sec. 4.3; Algorithm 1 quantizes every
 * weight block).  W: device bf16 [K][N] row-major.  out->fmt,
 * out->scale_layout, out->codes and out->scales are set by the caller and
 * out->rows must equal N, out->k must equal K; codes are written K-major
 * ([N][K/2]; MXFP8: [N][K]).  Formats: MXFP4, HiF4, MXFP8 (the W8A8
 * baseline of Table 1).  Meant to run once per weight, off the hot path.
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT,
 * RFQ_ERR_UNSUPPORTED, RFQ_ERR_CUDA, RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_quantize_weight(const void *w_bf16, int64_t K, int64_t N, rfq_qtensor *out,
                               void *stream);

/* RFQ activation decomposition in one pass over X (Sec. 4.3, Algorithm 1):
 *   X~ = Q(X), dX = X - X~, X^ = Q(dX) where phi = 1 (same format, Sec. 4.3),
 * with the E8M0 scale floor(log2 amax) - 2 clamped to [-127, 127] and
 * round-to-nearest-even, saturating element rounding (MXFP4); HiF4 per its
 * encoder.  X: device bf16 [M][K] row-major.  xq: main pathway output,
 * xr: residual pathway output (both with rows = M, k = K and the same fmt
 * and layout); xr may be NULL only when fb->mode == RFQ_FALLBACK_NONE.
 * Two more format combinations:
 *   xq MXFP4, xr MXFP8   the FP4-to-FP8 residual pathway named in Sec. 4.2:
 *                        X~ = Q_MXFP4(X), X^ = Q_MXFP8(X - X~) (E4M3 scale
 *                        floor(log2 amax) - 8), one pass over X;
 *   xq MXFP8, no residual (fb->mode == RFQ_FALLBACK_NONE; a residual
 *                        returns RFQ_ERR_UNSUPPORTED): X -> MXFP8, the
 *                        activation of the W4A8 / W8A8 baselines (Table 1).
 * Residual codes and scales of tiles with phi = 0 are written as zero.
 * phi: device bytes [ceil(M/p_s)][ceil(K/r_s)], may be NULL; fb may be
 * NULL (= RFQ_FALLBACK_ALL).  M may be 0 (nothing is launched).
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT,
 * RFQ_ERR_UNSUPPORTED, RFQ_ERR_CUDA, RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_quantize_act(const void *x_bf16, int64_t M, int64_t K, const rfq_fallback *fb,
                            rfq_qtensor *xq, rfq_qtensor *xr, uint8_t *phi, void *stream);

/* rfq_quantize_act that in the same pass over X also writes X~ (and X^) in
 * the form rfq_linear multiplies, replacing a separate conversion pass:
 *   xq, xr HiF4 (Sec. 3.3):  xq_op (and xr_op) receive the exact bf16 values
 *       of X~ (and X^), the products of rfq_dequant(xq) and rfq_dequant(xr):
 *       every HiF4 value has at most six significant bits and an exponent
 *       inside bf16's range.  RFQ_FMT_BF16 operands of rows = M, k = K
 *       (device bf16 [M][K] row-major, 16-byte aligned); xr_op is required
 *       with a residual and must be NULL when fb->mode == RFQ_FALLBACK_NONE.
 *       X^ values of phi = 0 tiles are zero.
 *   xq MXFP4, xr MXFP8 (the FP4-to-FP8 residual, Sec. 4.2):  xq_op receives
 *       X~ re-encoded as MXFP8 (RFQ_FMT_MXFP8, the layout of xq), the
 *       product of rfq_convert(xq): every E2M1 value is an E4M3 value, so
 *       the codes change and the scale bytes do not.  xr_op must be NULL
 *       (X^ is already MXFP8) and the mode must have a residual.
 * Other format combinations return RFQ_ERR_UNSUPPORTED.  xq, xr, phi and fb
 * as for rfq_quantize_act.  Asynchronous on `stream`.
 * Errors: as rfq_quantize_act. */
RFQ_API rfq_status rfq_quantize_act_expand(const void *x_bf16, int64_t M, int64_t K, const rfq_fallback *fb,
                                           rfq_qtensor *xq, rfq_qtensor *xr, uint8_t *phi, rfq_qtensor *xq_op,
                                           rfq_qtensor *xr_op, void *stream);

/* Bytes of device workspace rfq_linear needs (a status word, padded).  The
 * caller zeroes it.  Its int32 words: [0] the device status that
 * rfq_workspace_status reads; [1] the limit of the call's bounded waits in
 * microseconds (0: two seconds); [2] held start: when non-zero, the GEMM's
 * copy producers wait (within that limit) for word [3] to become non-zero
 * before their first copy and record RFQ_ERR_TIMEOUT if it stays zero -- a
 * way to run a kernel's timeout path with no copy or MMA in flight.  Every
 * GEMM entry point (rfq_linear, rfq_linear_fused, rfq_linear_grouped)
 * honours words [1] to [3]; leave them zero in normal use.  Bytes 32..95
 * receive rfq_linear_profile's counters.  With the environment variable
 * RFQ_DEBUG_SYNC set (to anything but "0") when the library first checks it,
 * every GEMM entry point synchronizes its stream after the launch and
 * returns the status the workspace then holds (as rfq_workspace_status
 * would), so a timeout surfaces at the call that caused it. */
RFQ_API size_t rfq_linear_workspace_bytes(void);

/* RFQ GEMM (Algorithm 1, Eq. rfq): Y = X~ W~ + phi X^ W~ with both products
 * accumulated into one fp32 accumulator per output tile, the weight tile read
 * once for both.  xq: [M x K] main codes; xr: [M x K] residual codes or NULL
 * (plain W4A4); phi: device bytes [ceil(M/128)][K/r_s] selecting the
 * residual k-tiles per 128-row tile, or NULL (= all ones); phi_r_s: the
 * column tile r_s of phi (a multiple of 128; ignored when phi is NULL).
 * The residual of every phi = 0 tile must be stored as zero, as
 * rfq_quantize_act writes it: phi only lets the GEMM skip residual loads and
 * products, at its own granularity (it may still include a phi = 0 tile that
 * shares a 256-row or 256-column block with a phi = 1 one).
 * wq: [N x K] weight.  MXFP4: every operand MXFP4 with RFQ_SCALE_MMA,
 * K % 128 == 0.  MXFP8: xq (and xr) MXFP8 (E4M3, kind::mxf8f6f4 MMAs)
 * with RFQ_SCALE_MMA, K % 128 == 0, and wq MXFP8 or MXFP4 -- the W8A8 and
 * W4A8 baselines and the FP4-to-FP8 RFQ (X~ re-encoded by rfq_convert, X^
 * from the MXFP8 residual pathway).  An MXFP4 wq (codes 32-byte aligned) is
 * multiplied as E2M1 (E4M3 x E2M1 MMAs) straight from its packed codes, half
 * the weight bytes of its E4M3 re-encoding, which gives the same Y.  HiF4 (Sec. 3.3): wq is the exact bf16 expansion of the HiF4
 * weight (RFQ_FMT_BF16, from rfq_dequant), K % 64 == 0, phi_r_s a multiple
 * of 64, and xq/xr are either HiF4 with RFQ_SCALE_MMA metadata (expanded
 * exactly to bf16 in shared memory inside the GEMM) or their exact bf16
 * expansions (RFQ_FMT_BF16, from rfq_dequant; faster when N spans several
 * tiles, since each activation tile is then expanded once instead of once
 * per output tile).  Both run on the bf16 tensor path.  N % 16 == 0, M >= 0.  y: device [M][N] row-major fp32 or bf16 (round-to-nearest-even
 * of the fp32 accumulator).  workspace: device, rfq_linear_workspace_bytes()
 * bytes, zeroed by the caller once; a kernel that gives up a bounded wait
 * records a timeout there (read it with rfq_workspace_status).  The record
 * is sticky: later calls with that workspace return without computing until
 * it is cleared.
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT,
 * RFQ_ERR_UNSUPPORTED, RFQ_ERR_CUDA, RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_linear(const rfq_qtensor *xq, const rfq_qtensor *xr, const uint8_t *phi,
                      int32_t phi_r_s, const rfq_qtensor *wq, void *y, int32_t out_dtype,
                      void *workspace, void *stream);

/* The RFQ linear layer end to end from host memory (Algorithm 1, Eq. rfq,
 * with X and Y in host memory): Y = X~ W~ + phi X^ W~ for a bf16 X on the
 * host.  The call copies X to the device, quantizes it (rfq_quantize_act,
 * MXFP4 main and residual pathways per fb), multiplies it by wq (rfq_linear)
 * and copies Y back, in chunks of chunk_rows rows: each chunk's
 * host-to-device copy runs on a copy stream of the library's, its two
 * kernels on `stream`, its device-to-host copy on a second copy stream, so
 * the copies of one chunk overlap the kernels and copies of the others.
 * `stream` then waits for the copy streams: y_host is complete once the
 * stream has passed the call (the call itself returns after enqueueing).
 * Y equals rfq_linear's on the same operands bit for bit (row chunking
 * does not change any output element's accumulation).
 *   x_host: host bf16 [M][K] row-major; page-locked memory lets the copies
 *           run asynchronously (pageable memory works, with copies that
 *           then block the host).
 *   y_host: host [M][N] row-major, bf16 or fp32 per out_dtype.
 *   fb: NULL (= RFQ_FALLBACK_ALL), RFQ_FALLBACK_NONE (plain W4A4; xr NULL)
 *       or RFQ_FALLBACK_AMAX with p_s = 128 and r_s a multiple of 128.
 *   wq: MXFP4 W~ [N x K] with RFQ_SCALE_MMA (device).
 *   chunk_rows: a multiple of 128; 0 selects 8192.  M = 0 does nothing
 *   (the host and device buffers may then be NULL).
 *   Device scratch, all the caller's (the library allocates no device
 *   memory; it creates two copy streams per device, kept for the process,
 *   and a few events per call): x_dev bf16 [M][K] (16-byte aligned); xq, xr
 *   MXFP4 qtensors of M x K with RFQ_SCALE_MMA (xr NULL exactly when fb is
 *   RFQ_FALLBACK_NONE); phi [ceil(M/128)][ceil(K/r_s)] bytes with
 *   RFQ_FALLBACK_AMAX, else ignored; y_dev [M][N]; workspace as for
 *   rfq_linear.  Nothing else may use these buffers until `stream` has
 *   passed the call.  Calls on one device share the two copy streams, so
 *   the copies of concurrent calls run one after another.
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT,
 * RFQ_ERR_UNSUPPORTED (other formats or layouts), RFQ_ERR_CUDA,
 * RFQ_ERR_DEVICE; every check happens before the first copy is enqueued. */
RFQ_API rfq_status rfq_linear_host(const void *x_host, int64_t M, int64_t K, const rfq_fallback *fb,
                                   const rfq_qtensor *wq, void *y_host, int32_t out_dtype, int64_t chunk_rows,
                                   void *x_dev, rfq_qtensor *xq, rfq_qtensor *xr, uint8_t *phi, void *y_dev,
                                   void *workspace, void *stream);

/* Workspace bytes rfq_linear_fused needs for an M x K activation and the
 * fallback mode fb (NULL = RFQ_FALLBACK_ALL); 0 for sizes it rejects
 * (K % 128 != 0).  For M <= 128 it is rfq_linear_workspace_bytes(); beyond,
 * it adds the kernel's counters and a scratch ring for the quantized X of
 * at most 12 blocks of 256 rows: 256 R K (1 + 1/16) bytes with the residual
 * for R = min(12, ceil(M / 256)) (half without) -- about 17 MB for K = 5120,
 * whatever M. */
RFQ_API size_t rfq_linear_fused_workspace_bytes(int64_t M, int64_t K, const rfq_fallback *fb);

/* RFQ linear layer with the activation quantizer fused into the GEMM (the
 * on-the-fly residual of Sec. 4.3): Y = Q(X) W~ + phi Q(X - Q(X)) W~ with X
 * read as bf16 and quantized inside the GEMM kernel, block by block, exactly
 * as rfq_quantize_act would (MXFP4: E8M0 scale floor(log2 amax) - 2, RNE
 * saturating E2M1 codes, exact residual): one launch, no separate
 * quantizer pass.  x_bf16: device bf16 [M][K] row-major (16-byte aligned).
 * wq: MXFP4 weight [N x K] with RFQ_SCALE_MMA scales.  fb: NULL or mode
 * RFQ_FALLBACK_ALL (residual on every block) or RFQ_FALLBACK_NONE (plain
 * W4A4); RFQ_FALLBACK_AMAX returns RFQ_ERR_UNSUPPORTED.  K % 128 == 0,
 * N % 16 == 0, M >= 0.  y, out_dtype: as for rfq_linear.
 * workspace: device, rfq_linear_fused_workspace_bytes(M, K, fb) bytes,
 * 16-byte aligned, zeroed by the caller once; its first 256 bytes are the
 * GEMM workspace of rfq_linear (status word, wait limit, held start).  For
 * M > 128 the GEMM runs on CTA pairs whose epilogue warps, between output
 * tiles, quantize X in units of 8 rows x 256 columns into the rest of the
 * workspace's ring, each element once; a stage's copies wait (bounded) until
 * its rows are quantized, a block of rows is written only once every output
 * tile has loaded the block its slot held before, and the kernel leaves its
 * counters zero for the next call.  Calls that overlap on the GPU must not
 * share a workspace.  For M <= 128 each output tile quantizes its rows of X itself in shared
 * memory (one row tile, so nothing is repeated across row tiles).
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT,
 * RFQ_ERR_UNSUPPORTED, RFQ_ERR_CUDA, RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_linear_fused(const void *x_bf16, int64_t M, int64_t K, const rfq_qtensor *wq,
                                    const rfq_fallback *fb, void *y, int32_t out_dtype, void *workspace,
                                    void *stream);

/* Grouped RFQ GEMM for mixture-of-experts layers (the MoE expert
 * projections that hold most of Qwen3-VL-30B's weights, Table 2): every
 * group g (an expert) computes
 *     Y[rows of g] = X~ W~_g + phi X^ W~_g             (Algorithm 1, Eq. rfq)
 * in one launch over all groups.  xq / xr: the activations of all groups
 * stacked along rows (rfq_qtensor as for rfq_linear, rows = the stacked
 * total); group_off: device int32 [groups + 1], rows [group_off[g],
 * group_off[g+1]) belong to group g; every group start must be a multiple
 * of 128 (pad each group's rows), the offsets non-decreasing and
 * group_off[groups] <= rows.  The offsets are read on the device (a router
 * may write them): a violation is recorded in the workspace, nothing is
 * computed, and rfq_workspace_status returns RFQ_ERR_SHAPE.  wq: the
 * weights of all groups stacked, rows = groups * N (group g's W~ rows
 * [g N, (g+1) N)), N % 128 == 0.  y: device [rows][N]; every row of a
 * group (the rows padding it to the next group's start included) is
 * written, rows before group_off[0] or from group_off[groups] on are not.  Operands MXFP4, or MXFP8
 * activations with an MXFP8 or MXFP4 (32-byte aligned) W~, as for rfq_linear; all with
 * RFQ_SCALE_MMA, K % 128 == 0; phi, phi_r_s, out_dtype and workspace as
 * for rfq_linear.  1 <= groups <= 128.
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT,
 * RFQ_ERR_UNSUPPORTED, RFQ_ERR_CUDA, RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_linear_grouped(const rfq_qtensor *xq, const rfq_qtensor *xr, const uint8_t *phi,
                                      int32_t phi_r_s, const int32_t *group_off, int32_t groups,
                                      const rfq_qtensor *wq, int64_t N, void *y, int32_t out_dtype,
                                      void *workspace, void *stream);

/* Exact re-encoding of an MXFP4 tensor as MXFP8 (every E2M1 value is an
 * E4M3 value): dst codes [rows][k] E4M3 bytes, dst scales = src scales.
 * src: fmt MXFP4; dst: fmt MXFP8, the same rows, k and scale layout; both
 * device, caller-owned.  Used for the weight of the W4A8 baseline and of
 * the FP4-to-FP8 RFQ (rfq_quantize_act_expand writes the activation's in
 * the quantizer's own pass).
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT,
 * RFQ_ERR_UNSUPPORTED (other formats), RFQ_ERR_CUDA, RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_convert(const rfq_qtensor *src, rfq_qtensor *dst, void *stream);

/* Checked mode for inputs: the quantizers and GEMMs take finite bf16 inputs
 * (non-finite ones give unspecified codes but never a fault); a caller that
 * cannot vouch for X runs this check first.  It scans the bf16 matrix
 * x [rows][k] (device, 16-byte aligned, k % 8 == 0) and, if any element is
 * Inf or NaN, records RFQ_ERR_NONFINITE in `workspace` (the GEMM workspace,
 * rfq_linear_workspace_bytes() bytes), where rfq_workspace_status reports
 * it.  Asynchronous on `stream`; one read of x.
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT, RFQ_ERR_CUDA,
 * RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_check_finite(const void *x_bf16, int64_t rows, int64_t k, void *workspace, void *stream);

/* Synchronizes `stream` and returns the device status left in a workspace by
 * earlier calls (RFQ_OK, RFQ_ERR_TIMEOUT, RFQ_ERR_SHAPE for group offsets
 * that break rfq_linear_grouped's contract, or RFQ_ERR_NONFINITE from
 * rfq_check_finite); clears it when `clear` != 0. */
RFQ_API rfq_status rfq_workspace_status(void *workspace, int32_t clear, void *stream);

/* Measurement of the ceiling the RFQ GEMM is held against: the dense
 * block-scaled FP4 tensor rate of this GPU (the kind::mxf4 MMA that carries
 * both products of Algorithm 1 / Eq. rfq), with MMAs alone.  Every SM
 * (cta_pair = 0: 128 x 256 x 64 MMAs, one CTA per SM) or every CTA pair
 * (cta_pair = 1: 256 x 256 x 64 cta_group::2 MMAs, the RFQ GEMM's form)
 * issues `iters` back-to-back MMAs from one shared-memory tile of
 * pseudo-random E2M1 codes (scales 2^0) into one TMEM accumulator; no
 * copies, scale writes or epilogue.  Time the launch on `stream` with
 * events; *flop_per_launch (host) receives its MMA work, 2 M N K per MMA
 * summed over the grid.  workspace: as for rfq_linear (a bounded final wait
 * that runs out records RFQ_ERR_TIMEOUT there).  iters in [1, 2^24].
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT,
 * RFQ_ERR_CUDA, RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_fp4_mma_peak(int32_t cta_pair, int64_t iters, void *workspace, double *flop_per_launch,
                                    void *stream);

/* RFQ GEMM with the FP4-to-FP8 residual at two rates (Sec. 4.2's FP4-to-FP8
 * pathway with the Sec. 3.2.1 format; Algorithm 1, Eq. rfq):
 *     Y = X~ W~ + phi X^ W~
 * with the main product X~ W~ on the FP4 tensor path (E2M1 x E2M1) and the
 * residual product X^ W~ on the FP8 one (E4M3 x E2M1), into one fp32
 * accumulator per output tile.  xq: X~, MXFP4 [M x K]; xr: X^, MXFP8 [M x K]
 * (rfq_quantize_act with an MXFP8 residual writes both); wq: W~, MXFP4
 * [N x K]: the kernel reads its packed codes once per k-stage and expands
 * them in shared memory to the one-byte-per-code form the residual MMAs
 * read (no second copy of W~ in memory).
 * Every operand with RFQ_SCALE_MMA scales; K % 128 == 0, N % 16 == 0,
 * M >= 0 (CTA pairs at every M).  phi, phi_r_s, y, out_dtype, workspace: as
 * for rfq_linear.  rfq_linear multiplies the same RFQ with X~ and W~
 * re-encoded as E4M3 (rfq_convert), both products then at the FP8 rate.
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT,
 * RFQ_ERR_UNSUPPORTED, RFQ_ERR_CUDA, RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_linear_mixed(const rfq_qtensor *xq, const rfq_qtensor *xr, const uint8_t *phi,
                                    int32_t phi_r_s, const rfq_qtensor *wq, void *y, int32_t out_dtype,
                                    void *workspace, void *stream);

/* Measurement of where the RFQ GEMM's tensor pipe idles: rfq_linear
 * (Algorithm 1, Eq. rfq) for MXFP4 operands with a residual and no phi,
 * M > 128 (the CTA-pair kernel), in a build of that kernel whose MMA-issuing
 * thread (one per CTA pair) counts, from its first wait to its final drain:
 * SM clock cycles, wall-clock nanoseconds, cycles waiting for a drained
 * accumulator, for a stage's operand copies and for a stage's scale words,
 * stages and tiles.  The sums over all pairs are added to the workspace's
 * 64-bit words 4..11 (bytes 32..95) in that order, with the number of pairs
 * in word 10: zero them before the call and read them after the stream has
 * synchronized.  Y is computed as by rfq_linear; the counters cost a few
 * instructions per stage, so time rfq_linear, not this call.
 * Errors: those of rfq_linear; RFQ_ERR_UNSUPPORTED for other operand forms. */
RFQ_API rfq_status rfq_linear_profile(const rfq_qtensor *xq, const rfq_qtensor *xr, const rfq_qtensor *wq, void *y,
                                      int32_t out_dtype, void *workspace, void *stream);

/* The debug build (librfq_debug.so, compiled with -DRFQ_DEBUG_BOUNDS): the
 * activation and weight quantizers and the CTA-pair GEMM check the index of
 * every direct global store against its buffer's extent (codes, scales, the
 * fused quantizer's ring, the grouped GEMM's row stores); an out-of-range
 * store is skipped and the source line of the first one is recorded.  This
 * call synchronizes the device and reports it: RFQ_OK (none, *line = 0) or
 * RFQ_ERR_SHAPE with *line set; clear != 0 resets the records.  The normal
 * build has no checks and returns RFQ_ERR_UNSUPPORTED.  The paper has no
 * counterpart: a debugging aid of this library.
 * Errors: RFQ_ERR_INVALID_ARG (line NULL), RFQ_ERR_CUDA. */
RFQ_API rfq_status rfq_debug_bounds(int32_t *line, int32_t clear);

/* Allocation-free variant of rfq_linear.  The paper has no counterpart: this
 * entry point exists for callers that cannot allocate device memory, such as
 * a serving loop that must not stall the device on cudaMalloc, a plug-in
 * whose host program owns every device buffer, or a runtime with no device
 * allocator of its own.  It takes the same arguments as rfq_linear except
 * the workspace and allocates nothing: no cudaMalloc, no cudaFree, no
 * allocating library routine.
 *
 * The GEMM's workspace (its status word) lives instead in a fixed 256-byte
 * __device__ array inside the library; every GPU that loads the library
 * holds it until the process exits.  If the GEMM ever needed more workspace
 * than 256 bytes the call would return RFQ_ERR_SHAPE; every size rfq_linear
 * accepts fits today.
 *
 * The first call on each device looks up the array's device address with
 * that device current; make that first call before any stream capture.  The
 * address is kept for the life of the process: a cudaDeviceReset reloads
 * the library's device code and makes it stale, so a caller of this entry
 * point does not reset the device.  A call passes rfq_linear's argument
 * checks first (a rejected call, or one with M == 0 or N == 0, leaves the
 * array untouched), then clears the array on `stream` before the GEMM runs,
 * because all calls share it and it keeps what the last call left.  Calls
 * that overlap on the GPU (other streams, other host threads) race on the
 * array.  A
 * timeout of a bounded wait is not reported by this variant (use rfq_linear
 * with a workspace to read it); Y is then left unwritten.
 * Errors: those of rfq_linear, and RFQ_ERR_SHAPE as above. */
RFQ_API rfq_status rfq_linear_noalloc(const rfq_qtensor *xq, const rfq_qtensor *xr, const uint8_t *phi,
                                      int32_t phi_r_s, const rfq_qtensor *wq, void *y, int32_t out_dtype,
                                      void *stream);

/* Dequantization x = code value * scale (Sec. 3.2 Eq. 4; Sec. 3.3 V_i) of a
 * quantized matrix (MXFP4 or HiF4) into device out[rows][k], fp32
 * (RFQ_OUT_F32) or bf16 (RFQ_OUT_BF16).  Every HiF4 value is exact in bf16;
 * MXFP4 values are exact in bf16 except below bf16's normal range.
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT,
 * RFQ_ERR_CUDA, RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_dequant(const rfq_qtensor *q, void *out, int32_t out_dtype, void *stream);

/* ---- Serving: one attention step on a 4-bit cache ------------------------
 * The entry points below carry a decoding step next to the linear layers
 * above: slots for the new tokens (rfq_slot_map), rotary positions
 * (rfq_rope), keys and values into a paged cache in MXFP4 or HiF4
 * (rfq_kv_append, rfq_kv_read), attention over that cache
 * (rfq_kv_attention), and products of a few tokens with a 4-bit weight
 * (rfq_matvec).  The paper's linear layer has no counterpart for them; the
 * formats are its own (Sec. 3.2.2, Sec. 3.3).  Arrays of int32, int64 and
 * fp32 need their natural alignment only; every other device pointer must be
 * 16-byte aligned, as above. */

/* Block tables, slot maps and positions of one serving step, built on the
 * GPU from the requests' lengths in one launch.  A cache is split into pages
 * of page_size tokens; request r holds its tokens in the pages
 * block_table[r][0 .. ceil(cached[r] / page_size)).  Free pages are a stack,
 * free_pages[0 .. *free_in).
 *   cached, added: device int32 [requests]: tokens in the cache, and tokens to
 *     add (> 0) or to drop from the end (< 0; more than cached drops all).
 *     after = max(cached + added, 0).
 *   1. Pages given back (those past ceil(after / page_size)) go on top of the
 *      stack, requests in order, each request's in the order of its table.
 *      Their table entries stay as they were.
 *   2. Pages wanted are taken from the top, requests in order.  The first
 *      request whose pages are not all there, and every later one that wants
 *      any, gets none: it is not served.  Requests that want none are served.
 *      A request whose pages exceed table_width (or whose cached is negative
 *      or exceeds it, or whose after passes int32) is not served either, takes
 *      and gives nothing, and the device status becomes RFQ_ERR_SHAPE.
 *   3. block_table (device int32 [requests][table_width], in place) gets the
 *      pages taken; free_out the stack's new height; lengths [requests] after,
 *      or cached where a request was not served.
 *   4. token_start [requests + 1]: prefix sums of max(added, 0), the rows of
 *      the step's tokens.  For token t = token_start[r] + i, positions[t] =
 *      cached[r] + i, and slots[t] = page * page_size + position % page_size,
 *      or -1 where request r was not served.  slots and positions hold
 *      `tokens` entries; those past token_start[requests] are -1 and 0 (a
 *      fixed-size step for a CUDA graph), and more tokens than that set the
 *      device status RFQ_ERR_SHAPE.
 * free_pages holds free_capacity entries; pages given back past it are
 * dropped (device status RFQ_ERR_SHAPE).  free_out may be free_in and lengths
 * may be cached; no other arrays overlap.  0 <= requests <= 8192,
 * page_size >= 1, table_width >= 1, requests * table_width < 2^31,
 * tokens >= 0.  workspace: device, 256 bytes zeroed by
 * the caller once, for the device status (rfq_workspace_status).
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT, RFQ_ERR_CUDA,
 * RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_slot_map(const int32_t *cached, const int32_t *added, int32_t requests, int32_t page_size,
                                int32_t *block_table, int32_t table_width, int32_t *free_pages,
                                int32_t free_capacity, const int32_t *free_in, int32_t *free_out, int32_t *lengths,
                                int32_t *token_start, int64_t *slots, int32_t *positions, int64_t tokens,
                                void *workspace, void *stream);

/* How the two elements of a rotary pair i of P lie in a head:
 *   RFQ_ROPE_HALF         elements i and i + P
 *   RFQ_ROPE_INTERLEAVED  elements 2i and 2i + 1 */
typedef enum { RFQ_ROPE_HALF = 0, RFQ_ROPE_INTERLEAVED = 1 } rfq_rope_pairing;

/* Rotary positions with several axes (time, height, width of images and
 * video; one axis for text).  For token t and pair i of every head,
 *     angle = positions[axis_of[i]][t] * inv_freq[i]
 *     (a, b) -> (a cos angle - b sin angle, b cos angle + a sin angle)
 * and with inverse != 0 by -angle: the gradient of the rotation.  Elements
 * past 2 pairs pass through unchanged, as does a pair whose axis_of is not in
 * [0, axes).
 *   x, out: device [tokens][heads][head_dim] of dtype (RFQ_OUT_F32 or
 *     RFQ_OUT_BF16) with the given strides in elements between tokens and
 *     heads (so queries and keys of a packed projection need no copy); out may
 *     be x with the same strides, and does not overlap it otherwise.  Strides
 *     and head_dim that are multiples of 16 bytes are read and written 16
 *     bytes at a time, others element by element.
 *   positions: device int32 [axes][tokens]; inv_freq: device fp32 [pairs];
 *   axis_of: device int32 [pairs].  The angle is reduced in fp64, so any
 *     int32 position keeps fp32 accuracy; the rotation is fp32, rounded once.
 * 1 <= head_dim <= 1024, 1 <= pairs <= head_dim / 2, axes >= 1, tokens >= 0,
 * heads >= 1.
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT, RFQ_ERR_CUDA,
 * RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_rope(const void *x, int64_t x_token_stride, int64_t x_head_stride, void *out,
                            int64_t out_token_stride, int64_t out_head_stride, int32_t dtype, int64_t tokens,
                            int32_t heads, int32_t head_dim, const int32_t *positions, int32_t axes,
                            const float *inv_freq, const int32_t *axis_of, int32_t pairs, int32_t pairing,
                            int32_t inverse, void *stream);

/* A paged cache of keys and values in 4 bits, quantized along head_dim.
 * Each (page, head) holds page_size tokens, and its bytes are contiguous:
 *   k_codes [pages][heads][page_size][head_dim / 2]: a token's row, its
 *     4-byte words transposed: the codes of elements 32 b + 8 c .. + 7 (element
 *     2j in the low nibble of byte j) are word c (head_dim / 32) + b.
 *   v_codes [pages][heads][page_size / 16][2][8][4][2][head_dim / 16]: token
 *     16 i + 8 h + 2 c + j of a page holds its elements g head_dim / 8 .. at
 *     [i][h][g][c][j].
 *   k_scales, v_scales: MXFP4 [pages][heads][page_size][head_dim / 32] E8M0
 *     bytes; HiF4 [pages][heads][page_size][head_dim / 64] metadata words.
 * This is the order in which the tensor cores' operands are loaded;
 * rfq_kv_read gives the values back in plain order.
 * fmt: RFQ_FMT_MXFP4 or RFQ_FMT_HIF4; head_dim: 64 or 128; page_size: a
 * multiple of 16 up to 4096.  Slot s is token s % page_size of page
 * s / page_size. */
typedef struct {
    int32_t fmt;       /* rfq_format */
    int32_t heads;     /* key / value heads */
    int32_t head_dim;
    int32_t page_size; /* tokens of a page */
    int64_t pages;
    void *k_codes;     /* device, see above */
    void *k_scales;
    void *v_codes;
    void *v_scales;
} rfq_kv_cache;

/* Byte sizes of each codes array and each scales array of a cache (host only).
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_UNSUPPORTED (head_dim). */
RFQ_API rfq_status rfq_kv_cache_bytes(int32_t fmt, int32_t heads, int32_t head_dim, int32_t page_size, int64_t pages,
                                      size_t *code_bytes, size_t *scale_bytes);

/* Quantizes the keys and values of `tokens` new tokens into the cache at
 * their slots, exactly as rfq_quantize_act would quantize the rows of one head
 * (RFQ_FALLBACK_NONE).  k, v: device bf16 [tokens][heads][head_dim] with
 * strides in elements (multiples of 8, so that every head starts on 16 bytes).
 * slots: device int64 [tokens]; a slot outside the cache (-1 of a token that
 * was not served) is skipped, and a slot given twice gets either token.
 * Non-finite inputs give unspecified codes.
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT,
 * RFQ_ERR_UNSUPPORTED, RFQ_ERR_CUDA, RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_kv_append(const void *k, int64_t k_token_stride, int64_t k_head_stride, const void *v,
                                 int64_t v_token_stride, int64_t v_head_stride, int64_t tokens, const int64_t *slots,
                                 const rfq_kv_cache *cache, void *stream);

/* The values of the cache's tokens at `slots` (device int64 [tokens]), keys
 * to k and values to v: device [tokens][heads][head_dim], fp32 or bf16 by
 * out_dtype (rounded to nearest even where bf16 does not hold a value: below
 * its normal range).  Rows of slots outside the cache are zero.
 * Errors: as rfq_kv_append. */
RFQ_API rfq_status rfq_kv_read(const rfq_kv_cache *cache, const int64_t *slots, int64_t tokens, void *k, void *v,
                               int32_t out_dtype, void *stream);

/* Bytes of device workspace rfq_kv_attention needs on the current device for
 * `heads` query heads of head_dim (whatever the lengths and requests). */
RFQ_API size_t rfq_kv_attention_workspace_bytes(int32_t heads, int32_t head_dim);

/* Attention over the paged 4-bit cache:
 *     o = softmax(scale q k^T) v
 * for the last tokens of every request over its cached keys (causal).  One
 * launch, or two with q_start: requests with more than 32 rows (new tokens times
 * heads / cache->heads) go through a kernel of their own, or if none can have as
 * many, rows of no request do.
 *   q: device bf16 [tokens][heads][head_dim], strides in elements (multiples
 *     of 8).  heads is a multiple of cache->heads: query head i reads key head
 *     i / (heads / cache->heads).
 *   q_start: device int32 [requests + 1]: rows q_start[r] .. q_start[r + 1] of
 *     q are the last tokens of request r (their keys are in the cache), or
 *     NULL: one token a request (tokens == requests).  Rows before q_start[0]
 *     and from q_start[requests] on belong to no request (the spare rows of a
 *     step of fixed size): they get o = 0 and lse = -inf.
 *   lengths: device int32 [requests]: keys of each request, its new tokens
 *     included.  Token i of n sees keys j <= length - n + i, and with
 *     window > 0 only j > length - n + i - window (window 0: all).  A row
 *     that sees no key gets o = 0 and lse = -inf.
 *   block_table: device int32 [requests][table_width] pages of each request.
 *   out: device bf16 [tokens][heads][head_dim], contiguous.
 *   lse: device fp32 [tokens][heads], the logarithm of the sum of
 *     exp(scale q k), or NULL.
 *   workspace: rfq_kv_attention_workspace_bytes bytes, zeroed by the caller
 *     once; calls that overlap on the GPU must not share it.
 * Scores, their maximum and sum and the accumulators are fp32; the codes enter
 * the tensor cores exactly, q as f16 scaled by a power of two per row, and the
 * softmax weights rounded to f16: by 2^-11 of themselves down to 2^-21 of the
 * row's largest, by 2^-32 of that one below.  Values whose block scale lies
 * 2^24 or more below the largest of the same head and dimensions in that request
 * may count as zero (HiF4, for a request with up to 32 rows: as anything up to
 * 2^-21 of the largest scale).  Keys with the smallest E8M0 scale (byte 0, 2^-127)
 * count as zero and, for a request with more than 32 rows, so may those with a
 * scale 2^24 or more below the largest key scale of the same head and request.
 * Block scales of 2^100 and more (keys) or 2^80 and more (values) may overflow.
 * q must be finite.
 * The same inputs give the same bits.
 * Lengths past table_width pages, rows outside q and pages outside the cache
 * set the device status RFQ_ERR_SHAPE (rfq_workspace_status); such requests'
 * rows are unspecified, and all rows are where q_start descends.  A bounded wait that runs out sets RFQ_ERR_TIMEOUT and
 * leaves NaN in the rows of out and lse that it concerns; int32 word 1 of the workspace is its
 * limit as for rfq_linear, and words 2 and 3 hold the start of the kernel for
 * more than 32 rows (of both in the debug build).
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT,
 * RFQ_ERR_UNSUPPORTED, RFQ_ERR_CUDA, RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_kv_attention(const void *q, int64_t q_token_stride, int64_t q_head_stride, int64_t tokens,
                                    int32_t heads, const int32_t *q_start, const int32_t *lengths, int32_t requests,
                                    const rfq_kv_cache *cache, const int32_t *block_table, int32_t table_width,
                                    float scale, int32_t window, void *out, float *lse, void *workspace,
                                    void *stream);

/* y = x W~^T for a few rows of x, x kept in bf16: the linear layer of a
 * decoding step, where the bytes of W~ bound the time (rfq_linear quantizes x
 * and is the call for more rows).
 *   x: device bf16 [rows][wq->k], x_row_stride in elements (a multiple of 8);
 *     0 <= rows <= 32.  x must be finite.
 *   wq: device, MXFP4 or HiF4 with either scale layout, any number of rows up
 *     to 2^21 (as rfq_quantize_weight writes it).
 *   y: device [rows][wq->rows], fp32 or bf16 by out_dtype.
 * Products and sums are fp32; W~ enters the tensor cores exactly and x as f16
 * scaled by a power of two per row and stretch of k, which keeps every bf16
 * bit down to 2^-28 of the stretch's maximum; blocks of W~ with the smallest
 * E8M0 scale (byte 0, 2^-127) count as zero, and scales of 2^100 and more may
 * overflow.  The same inputs give the same
 * bits.  Should a bounded wait run out, the sums that it concerns are NaN (the
 * call has no workspace, and so no device status).
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT,
 * RFQ_ERR_UNSUPPORTED (other formats), RFQ_ERR_CUDA, RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_matvec(const void *x, int64_t x_row_stride, int64_t rows, const rfq_qtensor *wq, void *y,
                              int32_t out_dtype, void *stream);

/* ---- Around a mixture-of-experts block ------------------------------------
 * The entry points below bring tokens to rfq_linear_grouped and back: norms in
 * front of a block (rfq_norm), the router (rfq_route), the pairs of tokens and
 * experts sorted into the groups of rows that the grouped product reads
 * (rfq_moe_sort), the tokens' rows brought there (rfq_moe_gather, or quantized
 * on the way: rfq_moe_quantize) and back (rfq_moe_combine), and the gradients
 * of all of them but the quantizer.  The paper's linear layer has no
 * counterpart for them; the format is its own (Sec. 3.2.2, Sec. 4.3).  Arrays
 * of int32 and fp32 results need their natural alignment only; every other
 * device pointer must be 16-byte aligned.  Rows whose strides and sizes are
 * multiples of 16 bytes are read and written 16 bytes at a time, others in
 * smaller steps.  A stride along an axis of one element is not looked at; along
 * others the rows of a result do not overlap (strides below their length are
 * refused, RFQ_ERR_SHAPE), while rows that are only read may.  The same call on
 * the same inputs and device gives the same bits; sizes, types and strides
 * choose the order of sums. */

/* RFQ_NORM_LAYER  y = (x - mean) rstd w + b,  rstd = 1 / sqrt(variance + eps)
 * RFQ_NORM_RMS    y = x rstd w + b,           rstd = 1 / sqrt(mean x^2 + eps) */
typedef enum { RFQ_NORM_LAYER = 0, RFQ_NORM_RMS = 1 } rfq_norm_kind;

/* Layer norm or RMS norm over the last axis.
 *   x, y: device [tokens][heads][dim] of dtype (RFQ_OUT_F32 or RFQ_OUT_BF16)
 *     with the given strides in elements between tokens and heads (so the heads
 *     of a packed projection need no copy; heads = 1 for plain rows); y may be x
 *     with the same strides, and does not overlap it otherwise.
 *   weight, bias: device [dim] of w_dtype, or NULL (1 and 0).
 *   mean, rstd: device fp32 [tokens][heads], what rfq_norm_grad needs, or NULL
 *     (with RFQ_NORM_RMS mean gets 0).
 * Mean, variance (from the differences to the mean) and everything between are
 * fp32; y is rounded once.  Squares that pass fp32 (elements beyond 1e18) give
 * rstd = 0.  A NaN makes its whole row NaN; in a layer norm so does an Inf, or a
 * sum of the row that passes fp32 (elements beyond 1e34 of one sign).  In an RMS
 * norm an Inf makes the squares' mean Inf and rstd = 0, which gives NaN in its own
 * place and b in the others.  No other row is affected.
 * 1 <= dim <= 16384, tokens * heads < 2^31, eps >= 0.
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT, RFQ_ERR_CUDA,
 * RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_norm(const void *x, int64_t x_token_stride, int64_t x_head_stride, void *y,
                            int64_t y_token_stride, int64_t y_head_stride, int32_t dtype, int64_t tokens,
                            int32_t heads, int32_t dim, int32_t kind, float eps, const void *weight, const void *bias,
                            int32_t w_dtype, float *mean, float *rstd, void *stream);

/* Bytes of device workspace rfq_norm_grad needs on the current device for rows
 * of dim elements (whatever their number); 0 for a dim it rejects. */
RFQ_API size_t rfq_norm_grad_workspace_bytes(int32_t dim);

/* Gradient of rfq_norm.  With h = (x - mean) rstd (RFQ_NORM_RMS: x rstd) and
 * g = dy w:
 *     dx = rstd (g - mean(g) - h mean(g h))      (RFQ_NORM_RMS: without mean(g))
 *     dweight = sum over rows of dy h,  dbias = sum over rows of dy
 *   dy, x, dx: device [tokens][heads][dim] of dtype, strided like rfq_norm's x;
 *     dx may be dy or x with the same strides.
 *   mean, rstd: device fp32 [tokens][heads] as rfq_norm wrote them (mean may be
 *     NULL with RFQ_NORM_RMS).
 *   weight: as rfq_norm got it, or NULL.
 *   dweight, dbias: device fp32 [dim], or NULL; written also when there are no
 *     rows (zeros).  The sums are fp32 in an order that the sizes, the type, the
 *     strides and the device decide, and nothing else: rows whose strides allow
 *     no 16-byte access are shared out in another way than those that do.
 *   workspace: rfq_norm_grad_workspace_bytes bytes, needed for dweight or dbias;
 *     calls that overlap on the GPU must not share it.  Its contents do not
 *     matter.
 * Errors: as rfq_norm. */
RFQ_API rfq_status rfq_norm_grad(const void *dy, int64_t dy_token_stride, int64_t dy_head_stride, const void *x,
                                 int64_t x_token_stride, int64_t x_head_stride, void *dx, int64_t dx_token_stride,
                                 int64_t dx_head_stride, int32_t dtype, int64_t tokens, int32_t heads, int32_t dim,
                                 int32_t kind, const float *mean, const float *rstd, const void *weight,
                                 int32_t w_dtype, float *dweight, float *dbias, void *workspace, void *stream);

/* The router: each token's top_k experts and their weights.  With
 * p = softmax(logits) over a token's experts,
 *     ids[t][j] = the expert of the j-th largest logit (of equal ones the lowest)
 *     weights[t][j] = p[ids[t][j]], or with normalize != 0 divided by their sum
 * (the softmax over the chosen logits alone).  A logit of -inf is never chosen:
 * a token with fewer than top_k others gets id -1 and weight 0 for the rest, and
 * one with none of them for all.  A row with a NaN or +inf gives NaN weights (its
 * ids are experts all the same, NaN counting as the largest).
 *   logits: device [tokens][experts] of dtype, row_stride in elements.
 *   ids: device int32 [tokens][top_k]; weights: device fp32 [tokens][top_k].
 * 1 <= experts <= 256, 1 <= top_k <= min(32, experts), tokens * top_k < 2^31.
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT, RFQ_ERR_CUDA,
 * RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_route(const void *logits, int64_t row_stride, int32_t dtype, int64_t tokens, int32_t experts,
                             int32_t top_k, int32_t normalize, int32_t *ids, float *weights, void *stream);

/* Gradient of rfq_route's weights in the logits: with d[i] = dweights[t][j]
 * where ids[t][j] = i, 0 for experts that were not chosen, and p the softmax over
 * all experts, or with normalize != 0 over the chosen ones (0 elsewhere),
 *     dlogits[t][i] = p[i] (d[i] - sum of p d).
 * ids outside [0, experts) and their dweights are not looked at; the others of a
 * token differ (of two that are equal one dweight counts).  dlogits: device
 * [tokens][experts] of dtype, every element written; it may be logits with the
 * same stride.  The rest as for rfq_route.
 * Errors: as rfq_route. */
RFQ_API rfq_status rfq_route_grad(const void *logits, int64_t row_stride, int32_t dtype, int64_t tokens,
                                  int32_t experts, int32_t top_k, int32_t normalize, const int32_t *ids,
                                  const float *dweights, void *dlogits, int64_t dlogits_row_stride, void *stream);

/* Rows that hold the groups of tokens * top_k pairs over the experts whatever
 * the ids, each group's rows rounded up to a multiple of align (host only);
 * -1 for sizes that rfq_moe_sort rejects. */
RFQ_API int64_t rfq_moe_rows(int64_t tokens, int32_t top_k, int32_t experts, int32_t align);

/* Pairs (token, choice) sorted by expert, in one launch.  Pair p = t top_k + j is
 * of expert ids[t][j]; the rows of expert e's pairs, in the order of the pairs,
 * are group_off[e], group_off[e] + 1, ...
 *   ids: device int32 [tokens][top_k]; a pair whose id is outside [0, experts) (of
 *     a place of the batch that holds no token) is of no group.
 *   group_off: device int32 [experts + 1], group_off[0] = 0; every group's rows are
 *     rounded up to a multiple of align (128 for rfq_linear_grouped).
 *   row_of: device int32 [tokens][top_k], the row of each pair, or -1.
 *   pair_of: device int32 [rows], the pair of each row, or -1 (rows that round a
 *     group up, and all from group_off[experts] on).
 *   rows: of the stacked matrix; rfq_moe_rows are always enough.  Pairs whose row
 *     is not among the first align * floor(rows / align) get none (row_of = -1),
 *     group_off is cut there, and the device status becomes RFQ_ERR_SHAPE.
 *   workspace: device, 256 bytes zeroed by the caller once, for the device status
 *     (rfq_workspace_status).
 * No two of the arrays overlap.
 * 1 <= experts <= 256, 1 <= top_k <= 32, 1 <= align <= 4096,
 * tokens * top_k + experts * align < 2^31, rows < 2^31.
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT, RFQ_ERR_CUDA,
 * RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_moe_sort(const int32_t *ids, int64_t tokens, int32_t top_k, int32_t experts, int32_t align,
                                int32_t *group_off, int32_t *row_of, int32_t *pair_of, int64_t rows, void *workspace,
                                void *stream);

/* The tokens' rows brought to their groups: out[row_of[t][j]] = x[t] for every
 * pair whose row is in [0, rows).
 *   x: device [tokens][dim] of dtype, x_row_stride in elements.
 *   row_of, pair_of: as rfq_moe_sort wrote them.  With pair_of, rows whose
 *     pair_of is negative are cleared, so that every row of out is written;
 *     without (NULL), rows of no pair are left as they were.
 *   out: device [rows][dim] of dtype, contiguous; not x.
 * rfq_moe_sort gives no row to two pairs; of a row that two name each element is
 * either token's.  Its gradient in x is rfq_moe_combine without weights.
 * 1 <= dim <= 65536, 1 <= top_k <= 32, tokens * top_k < 2^31, rows < 2^31.
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT, RFQ_ERR_CUDA,
 * RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_moe_gather(const void *x, int64_t x_row_stride, int32_t dtype, int64_t tokens, int32_t dim,
                                  const int32_t *row_of, int32_t top_k, const int32_t *pair_of, void *out,
                                  int64_t rows, void *stream);

/* The groups' rows brought back: out[t] = sum over j of
 * weights[t][j] y[row_of[t][j]], in the order of j, in fp32, rounded once; pairs
 * whose row is not in [0, rows) add nothing (out[t] = 0 where all are so).
 *   y: device [rows][dim] of dtype, contiguous.
 *   weights: device fp32 [tokens][top_k], or NULL (1).
 *   out: device [tokens][dim] of dtype, out_row_stride in elements; not y.
 * Sizes and errors: as rfq_moe_gather. */
RFQ_API rfq_status rfq_moe_combine(const void *y, int32_t dtype, int64_t rows, int32_t dim, const int32_t *row_of,
                                   const float *weights, int64_t tokens, int32_t top_k, void *out,
                                   int64_t out_row_stride, void *stream);

/* Gradients of rfq_moe_combine in y and in the weights: for every pair whose row
 * r is in [0, rows)
 *     dy[r] = weights[t][j] dout[t],  dweights[t][j] = <dout[t], y[r]>
 * and dweights[t][j] = 0 for the others.  With pair_of, rows of dy whose pair_of is
 * negative are cleared; without (NULL), rows of no pair are left as they were.
 *   dout: device [tokens][dim] of dtype, dout_row_stride in elements.
 *   y, dy: device [rows][dim] of dtype, contiguous; dy may be y if no two pairs
 *     name a row (rfq_moe_sort gives none to two: the second would multiply dout
 *     with the first one's gradient).
 *   dweights: device fp32 [tokens][top_k].
 * Of a row that two pairs name each element of dy is either one's gradient.
 * Sizes and errors: as rfq_moe_gather. */
RFQ_API rfq_status rfq_moe_combine_grad(const void *dout, int64_t dout_row_stride, const void *y, int32_t dtype,
                                        int64_t rows, int32_t dim, const int32_t *row_of, const int32_t *pair_of,
                                        const float *weights, int64_t tokens, int32_t top_k, void *dy,
                                        float *dweights, void *stream);

/* rfq_moe_gather that quantizes: the rows of xq and xr are what rfq_quantize_act
 * (RFQ_FALLBACK_ALL, or RFQ_FALLBACK_NONE without xr) would write for the gathered
 * rows, but each token is read and quantized once for all its pairs.
 *   x: device bf16 [tokens][xq->k], x_row_stride in elements (a multiple of 8).
 *   xq, xr: MXFP4 of the same rows and k with RFQ_SCALE_MMA, the operands of
 *     rfq_linear_grouped; xr may be NULL.  Scale bytes of the layout's padding
 *     rows (from xq->rows on) are zero.
 *   row_of, pair_of: as for rfq_moe_gather; a cleared row has zero codes and
 *     scales, and of a row that two pairs name the codes of 32 elements are one
 *     token's and the scales of 128 one token's, not the same one's.
 * k <= 65536; the other sizes as for rfq_moe_gather.
 * Errors: RFQ_ERR_INVALID_ARG, RFQ_ERR_SHAPE, RFQ_ERR_ALIGNMENT,
 * RFQ_ERR_UNSUPPORTED (other formats or layouts), RFQ_ERR_CUDA, RFQ_ERR_DEVICE. */
RFQ_API rfq_status rfq_moe_quantize(const void *x, int64_t x_row_stride, int64_t tokens, const int32_t *row_of,
                                    int32_t top_k, const int32_t *pair_of, rfq_qtensor *xq, rfq_qtensor *xr,
                                    void *stream);

#ifdef __cplusplus
}
#endif

#endif /* RFQ_H */
