/*
 * libaweq -- AWEQ (arXiv 2311.01305) per-linear-layer calibration + quantization path
 * for AMD MI355X (gfx950).  C ABI.
 *
 * Notation (the paper's): X[T x K] calibration activations (T tokens, K input channels),
 * W[N x K] the linear weight in PyTorch layout (the paper writes Y = X W with W as K x N,
 * Sec. 3.1 Eq. 3; its "channel i" is the column index k of both X and W here),
 * s[K] the equalization factors, Step / Z the quantizer's scale and zero point (Eq. 1-2).
 *
 * Conventions for every entry point
 *   - every pointer is a DEVICE pointer owned by the caller, unless marked "host";
 *     matrices are row-major with the K index contiguous and a leading dimension in
 *     elements; rows must start 16-byte aligned;
 *   - the library allocates nothing, frees nothing and never synchronises: each call
 *     enqueues kernels on `stream` (a hipStream_t passed as void*, NULL = default stream)
 *     and returns; scratch memory comes from the caller (`ws`, `ws_bytes`; ask
 *     aweq_workspace_size; 16-byte aligned; its contents need no initialisation), and may be
 *     reused by the next call on the same stream; entry points without a `ws` argument need none;
 *   - the return value is 0 or a negative AWEQ_ERR_* code found on the HOST before
 *     anything is launched (bad pointer, shape, dtype, alignment, workspace);
 *   - numeric conditions met on the device are OR-ed into the optional device word
 *     `status` (AWEQ_ST_* bits); inputs are expected to be finite;
 *   - an output must not overlap an input, another output or the workspace, except where an entry point says so;
 *   - calls on different streams must not share output or workspace buffers.
 */
#ifndef AWEQ_H
#define AWEQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { AWEQ_F32 = 0, AWEQ_F16 = 1, AWEQ_I8 = 2, AWEQ_BF16 = 3 } aweq_dtype;   /* AWEQ_BF16: where an entry point names it */

enum {
    AWEQ_OK = 0,
    AWEQ_ERR_NULL = -1,      /* a required pointer is NULL */
    AWEQ_ERR_SHAPE = -2,     /* a dimension is <= 0, a leading dimension is too small, K % 8 != 0 */
    AWEQ_ERR_DTYPE = -3,     /* dtype not supported by this entry point */
    AWEQ_ERR_BITS = -4,      /* bits not in {8, 4, 3} */
    AWEQ_ERR_GROUP = -5,     /* group does not divide K or is not a supported size */
    AWEQ_ERR_ALIGN = -6,     /* a pointer or row pitch is not 16-byte aligned */
    AWEQ_ERR_WORKSPACE = -7, /* ws is NULL or smaller than aweq_workspace_size says */
    AWEQ_ERR_LAUNCH = -8     /* the HIP runtime refused a launch */
};

/* bits of the device status word */
enum {
    AWEQ_ST_DEGENERATE = 1u, /* Eq. 2 gave a non-positive or non-finite Step; Step := 1 was used */
    AWEQ_ST_NONFINITE = 2u,  /* NaN / Inf seen in the input (results unspecified) */
    AWEQ_ST_BIGQUOT = 4u,    /* |x / Step| >= 2^24: quotient saturated */
    AWEQ_ST_SCALEGUARD = 8u, /* Eq. 10: a channel range was < 1e-5 (s := 1) or s was clamped to [1e-4, 1e4] */
    AWEQ_ST_ZEROPOINT = 16u, /* stage 4 de-quantisation met a zero point outside [0, 255] (a slice whose range does not
                                contain 0): its 32-bit integer part is exact only while it fits in 32 bits */
    AWEQ_ST_INDEX = 32u,     /* a page, slot or length on the device lies outside what the call was given: clamped or left out */
    AWEQ_ST_PAGES = 64u      /* aweq_step_plan: fewer pages are free than the step takes; nothing was changed */
};

typedef enum {
    AWEQ_OP_CALIB_STATS = 0,
    AWEQ_OP_EQUALIZE = 1,
    AWEQ_OP_QUANT_WEIGHT = 2,
    AWEQ_OP_W8A8_GEMM = 3,
    AWEQ_OP_BIAS_CORRECT = 4,
    AWEQ_OP_WONLY_GEMM = 5,
    AWEQ_OP_QUANT_ACT = 6,
    AWEQ_OP_CALIBRATE = 7
} aweq_op;

enum { AWEQ_BIAS_W8A8 = 0, AWEQ_BIAS_WEIGHT_ONLY = 1 };

/* values of aweq_equalize's enable_awe */
enum {
    AWEQ_SCALE_NONE = 0,   /* s = 1: equalization off (the ablation of Sec. 4.4) */
    AWEQ_SCALE_RANGE = 1,  /* Eq. 10 on the channel ranges: the method */
    AWEQ_SCALE_ABSMAX = 2  /* Eq. 10's form on the channels' maximum absolute values instead of their ranges: the
                              difficulty definition the method replaces (Sec. 1, Sec. 3.2), kept as a switch for
                              comparisons on the same layers */
};

/* Bytes of workspace the op needs for a [rows x K] input (rows = T or N as the op reads
 * it) and N output channels; 0 when it needs none.  Host function, no GPU needed. */
size_t aweq_workspace_size(aweq_op op, int64_t rows, int64_t K, int64_t N);

/* Name of an AWEQ_ERR_* code.  Host function. */
const char* aweq_status_string(int code);

/* ---- K-panel layout of the int8 GEMM operands (a storage format of this library, chosen so
 * that the matrix-core kernel of stage 4 reads whole cache lines: not part of the method).
 * An int8 matrix M[rows x K] is cut along K into ceil(K / 64) panels of 64 columns; panel p
 * stores bytes M[r][64 p .. 64 p + 63] of every row r back to back:
 *     byte offset of M[r][k] = ((k / 64) * rows + r) * 64 + k % 64,
 * columns past K in the last panel are zero.  xq (stage 4a / 4) and the 8-bit codes of stage 3
 * with group <= 0 use it.  aweq_panel_bytes: size of such a buffer (host function).
 * aweq_pack_panels_i8 / aweq_unpack_panels_i8 convert from / to a row-major [rows x K] int8
 * matrix of pitch ld bytes (K % 8 == 0, ld % 8 == 0, both pointers 8-byte aligned). */
size_t aweq_panel_bytes(int64_t rows, int64_t K);
int aweq_pack_panels_i8(const int8_t* src, int64_t rows, int64_t K, int64_t ld, int8_t* panels, void* stream);
int aweq_unpack_panels_i8(const int8_t* panels, int64_t rows, int64_t K, int8_t* dst, int64_t ld, void* stream);

/* ---- Stage 1: range statistics (Sec. 3.2: channel range = channel max - channel min,
 * tensor range = max - min over all channels, Eq. 4 p_i = r_i / R; Sec. 3.3: E[x] is
 * collected in the same pass).
 * M[rows x K] (F32 or F16, pitch ld) -> cmin[K], cmax[K] (exact), csum[K] (fp64 column
 * sums, nullable), count (uint64 scalar, nullable).  accumulate = 0 starts from
 * (+inf, -inf, 0, 0); accumulate = 1 merges into what the buffers hold (further
 * calibration batches; or a second weight sharing the same input: min of mins, max of
 * maxes).  finalize = 1 also writes r[K] = cmax - cmin, R[1] = max_k cmax - min_k cmin and
 * (nullable) p[K] = r / R.  Needs workspace. */
int aweq_calib_stats(const void* M, aweq_dtype dt, int64_t rows, int64_t K, int64_t ld,
                     float* cmin, float* cmax, double* csum, uint64_t* count,
                     int accumulate, int finalize, float* r, float* R, float* p,
                     void* ws, size_t ws_bytes, uint32_t* status, void* stream);

/* ---- Stage 1 for callers that cannot allocate or pass scratch memory (code under HIP graph capture
 * with a fixed argument list, tight serving loops, harnesses that forbid hipMalloc): the same
 * kernels and results as aweq_calib_stats, with the per-slice partial rows kept in a device array of
 * AWEQ_STATIC_SCRATCH_BYTES that is part of the library (every GPU the library runs on holds one
 * copy until the process ends) instead of a caller's workspace.  The call allocates nothing.
 * AWEQ_ERR_WORKSPACE when aweq_workspace_size(AWEQ_OP_CALIB_STATS, rows, K, 0) exceeds
 * AWEQ_STATIC_SCRATCH_BYTES (all configurations up to 262144 x 22016 binary16 fit).  The device
 * that owns `stream` must be the current device.  All calls on one GPU share that GPU's array:
 * calls that overlap on one GPU (different streams) race; calls on one stream do not. */
#define AWEQ_STATIC_SCRATCH_BYTES (16u << 20)
int aweq_calib_stats_static(const void* M, aweq_dtype dt, int64_t rows, int64_t K, int64_t ld,
                            float* cmin, float* cmax, double* csum, uint64_t* count,
                            int accumulate, int finalize, float* r, float* R, float* p,
                            uint32_t* status, void* stream);

/* ---- Stage 2: activation-weight equalization (Sec. 3.1 Eq. 3, Sec. 3.2 Eq. 10).
 * From the column statistics of X (xmin, xmax, xsum, host scalar count = T) and of W
 * (wmin, wmax): s[k] = sqrt(r_x r_w) / r_w evaluated in fp64 on the raw channel ranges,
 * inv_s[k] = 1 / s[k]  (enable_awe = AWEQ_SCALE_RANGE; AWEQ_SCALE_NONE: s = 1, the ablation switch of
 * Sec. 4.4; AWEQ_SCALE_ABSMAX: the same formula with m = max(|min|, |max|) of the channel in place of r).
 * Guards: a channel with r_x < 1e-5 or r_w < 1e-5 gets s = 1; s is clamped to [1e-4, 1e4].
 * Fold, weight side: W_hat[n,k] = W[n,k] * s[k], one fp32 multiply rounded to dt
 * (W has pitch ldw, W_hat pitch ldwh; W_hat may alias W when the pitches agree; W = NULL skips the
 * fold).  Activation side: the equalised
 * activation X_hat[t,k] = X[t,k] * inv_s[k] is never stored; its tensor range
 * xhat_range[2] = {min, max}, its mean mu_xhat[K] = (xsum / count) * inv_s and the static
 * int8 activation quantizer derived from that range by Eq. 2 (act_step[1], act_zero[1])
 * are written instead.  prev_scale[K] (nullable) is multiplied by inv_s so the caller can
 * fuse diag(s)^-1 into the preceding block.  mu_xhat / xsum nullable together.  s, inv_s, mu_xhat and prev_scale may
 * each replace xmin, xmax, wmin or wmax (the same address: channel k over channel k). */
int aweq_equalize(const float* xmin, const float* xmax, const double* xsum, uint64_t count,
                  const float* wmin, const float* wmax, int64_t K, int enable_awe,
                  float* s, float* inv_s,
                  const void* W, void* W_hat, aweq_dtype dt, int64_t N, int64_t ldw, int64_t ldwh,
                  float* prev_scale, float* xhat_range, float* mu_xhat,
                  float* act_step, int32_t* act_zero,
                  uint32_t* status, void* stream);

/* ---- Stage 3: weight quantizer, Eq. 1-2: Step = (max - min) / (2^b - 1),
 * Z = -round(min / Step), u = clamp(round(w / Step) + Z, 0, 2^b - 1); round-to-nearest
 * with ties to even, true fp32 division.  A slice with max == min uses Step = 1.
 * group = 0: one (Step, Z) per row n -> step[N], zero[N];
 * group = g > 0 (a power of two in [8, 512] dividing K): one per g consecutive k inside a
 *   row -> step/zero[N x K/g];
 * group = -1: one for the whole tensor -> step[1], zero[1] (needs workspace).
 * codes: bits 8 -> int8 u - 128; for group <= 0 in the K-panel layout (aweq_panel_bytes(N, K)
 * bytes: the weight operand of stage 4), for group > 0 row-major, N*K bytes; bits 4 -> two
 * codes per byte, even k in the low nibble, N*K/2 bytes; bits 3 -> per row a little-endian bit stream with code k in bits
 * [3k, 3k+3), N*3K/8 bytes (K % 32 == 0).  rowsum_w[N] = sum_k (u - 128), bits 8 only,
 * nullable. */
int aweq_quant_weight(const void* W_hat, aweq_dtype dt, int64_t N, int64_t K, int64_t ldw,
                      int bits, int group, void* codes, float* step, int32_t* zero,
                      int32_t* rowsum_w, void* ws, size_t ws_bytes,
                      uint32_t* status, void* stream);

/* ---- Stages 2b + 3 in one pass over W (per-row quantizer, group = 0): W_hat[n,k] = W[n,k] * s[k]
 * rounded to dt (Eq. 3; W_hat has pitch ldwh and may alias W when ldwh = ldw) is written and quantised from registers,
 * with the outputs of aweq_quant_weight(group = 0).  Same results as aweq_equalize's fold followed by
 * aweq_quant_weight; call aweq_equalize with W = NULL for the scales first. */
int aweq_fold_quant_weight(const void* W, aweq_dtype dt, int64_t N, int64_t K, int64_t ldw,
                           const float* s, void* W_hat, int64_t ldwh, int bits, void* codes, float* step,
                           int32_t* zero, int32_t* rowsum_w, uint32_t* status, void* stream);

/* ---- Stage 4a (helper, also run by aweq_w8a8_gemm): static per-tensor int8 activation
 * quantizer (Eq. 1 with b = 8) applied to X_hat = X * inv_s on the fly:
 * xq[t,k] = clamp(round((X[t,k] * inv_s[k]) / Step_x) + Z_x, 0, 255) - 128,
 * rowsum_x[T] = sum_k xq (int32, nullable), colsum_xq[K] = sum_t xq (int64, nullable).
 * xq is written in the K-panel layout (aweq_panel_bytes(T, K) bytes); xq = NULL computes the sums
 * only (one read of X, nothing written per element: what a calibration without the forward needs).
 * act_step / act_zero are the device scalars aweq_equalize wrote.  The sums are formed without
 * atomics, in a fixed order: per-slice partial sums in the workspace
 * (aweq_workspace_size(AWEQ_OP_QUANT_ACT, T, K, 0) bytes; needed when colsum_xq is asked for, or
 * rowsum_x with K > 512) and a merge kernel.  AWEQ_ST_BIGQUOT: some |X_hat / Step| reached 2^24
 * (Step and Z not from this data); the quotient is then rounded, saturated at +-2^30, and clamped
 * as Eq. 1 says.  colsum_xq, and with K > 512 rowsum_x, may overlap X and inv_s: the merge kernel writes them. */
int aweq_quant_act(const void* X, aweq_dtype dt, int64_t T, int64_t K, int64_t ldx,
                   const float* inv_s, const float* act_step, const int32_t* act_zero,
                   int8_t* xq, int32_t* rowsum_x, int64_t* colsum_xq,
                   void* ws, size_t ws_bytes, uint32_t* status, void* stream);

/* ---- Stage 4: W8A8 forward (Sec. 1-2: INT8 weights and activations).
 * x_dt F16 / F32: X is quantised into xq[T x K] first (stage 4a; xq, inv_s, act_step,
 * act_zero required).  x_dt I8: X already holds xq in the K-panel layout (ldx = K), stage 4a
 * is skipped.  wq[N x K]: the 8-bit codes of stage 3 (group <= 0), K-panel layout.
 * acc[t,n] = sum_k xq[t,k] wq[n,k], int8 x int8 -> int32 on the matrix cores (K <= 32768).
 * Outputs, each nullable: out_i32[T x N] (pitch ldo) the raw accumulator;
 * out_deq[T x N] (F16 or F32, pitch ldo) the de-quantised output
 *   Step_x Step_w[n] (acc - Z'x rowsum_w[n] - Z'w[n] rowsum_x[t] + K Z'x Z'w[n]) + bias[n],
 *   Z' = Z - 128 (needs rowsum_x, rowsum_w, step_w, zero_w; bias nullable);
 *   The integer in parentheses is formed in 32-bit arithmetic: exact whenever it fits, which zero
 *   points in [0, 255] (ranges that contain 0) guarantee for K <= 32768; other zero points are
 *   handled the same way and raise AWEQ_ST_ZEROPOINT;
 * colsum_acc[N] = sum_t acc[t,n] (int64; what stage 5 needs; always the sum of the accumulator
 *   itself, whatever the zero points).
 * w_group = 0: step_w[N] / zero_w[N] hold one entry per output channel (stage 3 with group = 0);
 * w_group = -1: step_w[1] / zero_w[1], one for the tensor (stage 3 with group = -1, the paper's
 * per-tensor setting, Sec. 3); rowsum_w[N] is per output channel in both cases.
 * With X F16 / F32, out_i32, out_deq and colsum_acc may overlap X and inv_s: the quantizer has read them before the GEMM
 * stores anything; colsum_xq and rowsum_x as in aweq_quant_act.
 * ws: the workspace of stage 4a when X is F16 / F32 (aweq_workspace_size(AWEQ_OP_W8A8_GEMM, T, K, N));
 * not needed (NULL) for x_dt = I8. */
int aweq_w8a8_gemm(const void* X, aweq_dtype x_dt, int64_t T, int64_t K, int64_t ldx,
                   const float* inv_s, const float* act_step, const int32_t* act_zero,
                   int8_t* xq, int32_t* rowsum_x, int64_t* colsum_xq,
                   const int8_t* wq, int64_t N, const float* step_w, const int32_t* zero_w, int w_group,
                   const int32_t* rowsum_w, const float* bias,
                   int32_t* out_i32, void* out_deq, aweq_dtype out_dt, int64_t ldo,
                   int64_t* colsum_acc, void* ws, size_t ws_bytes,
                   uint32_t* status, void* stream);

/* ---- Stage 4 with fused epilogues for the layer that consumes this one's output (statistics of
 * Sec. 3.2 / Sec. 3.3's E[x] and the quantizer of Eq. 1 applied where the output is produced
 * instead of in passes of their own over it).  The GEMM and the de-quantisation are those of
 * aweq_w8a8_gemm with x_dt = I8 and w_group = 0 (per-channel weight scales); y[t,n] = act(de-quantised output + bias) rounded to binary16,
 * act = 0 (none) or 1 (ReLU, OPT's fc1 -> fc2).  Outputs:
 *  out_f16[T x N] (pitch ldo, nullable): y itself;
 *  colsum_acc[N] (required): as in aweq_w8a8_gemm, for this layer's stage 5;
 *  statistics (ycmin non-NULL): ycmin[N], ycmax[N], ycsum[N] (nullable), ycount[1] (nullable) =
 *    what aweq_calib_stats(y, F16, rows = T, K = N, accumulate) returns on the stored output:
 *    extremes exact, sums exact (integer accumulation in units of 2^-24), independent of the
 *    launch; needs ws of aweq_workspace_size(AWEQ_OP_W8A8_GEMM, T, K, N) bytes;
 *  next-layer codes (yq non-NULL): yq[T x N] in the K-panel layout (aweq_panel_bytes(T, N) bytes),
 *    rowsum_y[T] (nullable), colsum_yq[N] (nullable) = what aweq_quant_act(y, F16, T, N, ...,
 *    next_inv_s[N], next_step[1], next_zero[1]) returns (true division).
 * At least one of the two.  Shapes the tiled kernel takes only: N % 4 == 0, 16-byte aligned
 * vectors and outputs (AWEQ_ERR_SHAPE / AWEQ_ERR_ALIGN otherwise). */
int aweq_w8a8_gemm_fused(const int8_t* xq, int64_t T, int64_t K, const int8_t* wq, int64_t N,
                         const float* act_step, const int32_t* act_zero,
                         const float* step_w, const int32_t* zero_w,
                         const int32_t* rowsum_x, const int32_t* rowsum_w, const float* bias, int act,
                         void* out_f16, int64_t ldo, int64_t* colsum_acc,
                         float* ycmin, float* ycmax, double* ycsum, uint64_t* ycount, int accumulate,
                         const float* next_inv_s, const float* next_step, const int32_t* next_zero,
                         int8_t* yq, int32_t* rowsum_y, int64_t* colsum_yq,
                         void* ws, size_t ws_bytes, uint32_t* status, void* stream);

/* ---- Stage 5: quantization bias correction (Sec. 3.3, Eq. 11-15).
 * delta[n] = mean over the calibration tokens of the FP output of the equalised layer
 * minus the mean output of the quantised layer; bias_out = bias_in + delta (the paper
 * subtracts E[y~ - y]).  enable_bc = 0 still writes delta but copies the bias unchanged.
 * mode AWEQ_BIAS_W8A8: mean FP output = W_hat mu_xhat (fp64 accumulation); mean int8-path
 *   output from colsum_acc, colsum_xq, rowsum_w, act_step/act_zero and step_w/zero_w (group = 0:
 *   [N], one per output channel; group = -1: [1], per tensor) as exact integers, count = T.  colsum_acc = NULL: the sums over tokens of the accumulator are
 *   formed from the weight codes instead (codes = the 8-bit per-row / per-tensor codes in the
 *   K-panel layout, bits = 8, group <= 0): sum_t acc[t,n] = sum_k wq[n,k] colsum_xq[k], the same
 *   integers, so the correction can be calibrated without running the forward.
 * mode AWEQ_BIAS_WEIGHT_ONLY (Eq. 12-15): delta[n] = -sum_k (W~[n,k] - W_hat[n,k]) mu_xhat[k]
 *   with W~ de-quantised from codes / bits / group / step_w / zero_w as laid out by
 *   aweq_quant_weight.
 * bias_in nullable (= zeros); delta, bias_out fp32[N]. */
int aweq_bias_correct(int mode, const void* W_hat, aweq_dtype dt, int64_t N, int64_t K, int64_t ldw,
                      const float* mu_xhat, uint64_t count,
                      const int64_t* colsum_acc, const int64_t* colsum_xq, const int32_t* rowsum_w,
                      const float* act_step, const int32_t* act_zero,
                      const void* codes, int bits, int group,
                      const float* step_w, const int32_t* zero_w,
                      const float* bias_in, float* delta, float* bias_out, int enable_bc,
                      uint32_t* status, void* stream);

/* ---- Weight-only forward (Sec. 4.2, Table 1: INT4 / INT3 weights, FP16 activations):
 * y[t,n] = sum_k x_hat[t,k] w~[n,k] + bias[n], w~ = Step (u - Z) the de-quantised weight of Eq. 1.
 * X_hat[T x K]: binary16 equalised activations, row-major, pitch ldx (the caller has folded
 * diag(s)^-1 into what produces them, Eq. 3); codes / step_w / zero_w: what aweq_quant_weight wrote
 * for bits in {4, 3} and the same group (group > 0: a multiple of 32 dividing K; 0: per row; -1: per
 * tensor); bias[N] fp32 nullable; out[T x N] F16 or F32, pitch ldo.  K % 64 == 0, N % 4 == 0,
 * ldo % 4 == 0, 16-byte aligned pointers.  Arithmetic: the weight operand is binary16,
 * w~_h = RN16((u - Z) * RN16(Step)), formed in registers, or written once per call into the workspace (N * K * 2 bytes:
 * aweq_workspace_size(AWEQ_OP_WONLY_GEMM, T, K, N); asked for in any case) where there are many tokens; products are exact in
 * fp32 and accumulated in fp32 on the matrix cores (summation order unspecified).  out may overlap codes, step_w and zero_w: the
 * weight is written to the workspace first then.  With N <= 256 a row of out may also lie over the same row of X_hat. */
int aweq_wonly_gemm(const void* X_hat, int64_t T, int64_t K, int64_t ldx,
                    const void* codes, int bits, int group,
                    const float* step_w, const int32_t* zero_w, int64_t N,
                    const float* bias, void* out, aweq_dtype out_dt, int64_t ldo,
                    void* ws, size_t ws_bytes, uint32_t* status, void* stream);

/* ---- Stages 1 - 5 in one call: the calibration of a layer, or of any number of layers that read the same activation (n_weights > 1:
 * one scale from the merged weight ranges, one activation quantizer; every weight has slices of its own, as `group` says).  The outputs are
 * those of the stage entry points called one after the other; the launches are fewer where the shapes allow (workspace of
 * aweq_workspace_size(AWEQ_OP_CALIBRATE, T, K, sum of the N); with less, down to what the stages ask for, they run one by one).
 * Sums in binary64 are added in another order than the stages add them, so that xsum and what is rounded from such sums (mu_xhat, delta,
 * bias_out) may differ from the stages' in the last place; everything else is the same to the bit.
 * Nullable: count, wcount, p_x, p_w, status; bias_in; rowsum_w without w8a8; xq, rowsum_x and colsum_acc without the
 * forward; out_i32 and out_deq.  W_hat may take the place of W (same pitch).  Output pitch N. */
typedef struct {
    const void* X;              /* [T x K], pitch ldx */
    aweq_dtype dt;              /* of X, every W and W_hat, and out_deq */
    int64_t T, K, ldx;
    float *xmin, *xmax;         /* stage 1 */
    double* xsum;
    uint64_t* count;
    float *r_x, *R_x, *p_x;
    float *wmin, *wmax;
    uint64_t* wcount;
    float *r_w, *R_w, *p_w;
    float *s, *inv_s;           /* stage 2 */
    float *xhat_range, *mu_xhat, *act_step;
    int32_t* act_zero;
    int8_t* xq;                 /* stage 4a */
    int32_t* rowsum_x;
    int64_t* colsum_xq;
    int enable_awe, enable_bc;
    int bits, group;            /* stage 3 */
    int w8a8, forward;          /* int8 path (8 bits, group 0 or -1; else weight-only); with the GEMM */
    int fused_weight_pass;      /* where the stages run one by one: aweq_fold_quant_weight (group = 0) */
    void* ws;
    size_t ws_bytes;
    uint32_t* status;
} aweq_calib_layer;

typedef struct {
    const void* W;              /* [N x K], pitch ldw */
    int64_t N, ldw;
    void* W_hat;                /* pitch ldwh */
    int64_t ldwh;
    void* codes;
    float* step_w;
    int32_t *zero_w, *rowsum_w;
    const float* bias_in;
    float *delta, *bias_out;
    int32_t* out_i32;
    void* out_deq;
    int64_t* colsum_acc;
} aweq_calib_weight;

int aweq_calibrate(const aweq_calib_layer* layer, const aweq_calib_weight* weights, int n_weights, void* stream);   /* both host structures */

/* ======== Around the quantised layers of a deployed decoder: a product whose tokens carry scales of their own, and the
 * attention block between the projections ========
 *
 * ---- Quantizer of Eq. 1-2 with b = 8 and a token as the slice.  x[t,k] = X[t,k] * inv_s[k] (one fp32 multiply; inv_s nullable: X is
 * equalised already).  The token's range is widened to contain 0, so that its zero point lies in [0, 255] and a 0 stays a 0:
 *   lo = min(0, min_k x), hi = max(0, max_k x), step_x[t] = (hi - lo) / 255 (1 for a token of zeros), zero_x[t] = -round(lo / step),
 *   xq[t,k] = clamp(round(x / step) + zero, 0, 255) - 128, rowsum_x[t] = sum_k xq        (true fp32 divisions, ties to even).
 * X[T x K] F32, F16 or BF16, pitch ldx; K <= 32768; xq in the K-panel layout (aweq_panel_bytes(T, K)).  A NaN or infinity raises
 * AWEQ_ST_NONFINITE (the results of that token are unspecified). */
int aweq_quant_tokens(const void* X, aweq_dtype dt, int64_t T, int64_t K, int64_t ldx, const float* inv_s,
                      int8_t* xq, float* step_x, int32_t* zero_x, int32_t* rowsum_x, uint32_t* status, void* stream);

/* ---- Product in 8-bit integers with a (Step, Z) for each token and each output channel.  X F32 / F16 / BF16 is quantised by
 * aweq_quant_tokens first (xq, step_x, zero_x, rowsum_x are written); X I8 (ldx = K) already is xq, and step_x, zero_x, rowsum_x
 * are inputs (zero_x in [0, 255], as aweq_quant_tokens writes them; outside: clamped, and AWEQ_ST_ZEROPOINT).  wq, step_w, zero_w, w_group, rowsum_w, bias (nullable): the
 * weight as in aweq_w8a8_gemm.
 *   out[t,n] = step_x[t] step_w[n] (acc - Z'x[t] rowsum_w[n] - Z'w[n] rowsum_x[t] + K Z'x[t] Z'w[n]) + bias[n],  Z' = Z - 128,
 * the integer exact in 32 bits (zero_w outside [0, 255]: AWEQ_ST_ZEROPOINT, as there), scaled in fp64, rounded to fp32 and from there to out_dt
 * (F32, F16, BF16; pitch ldo).  K % 8 == 0, K <= 32768, N % 4 == 0, ldo % 4 == 0, 16-byte aligned pointers. */
int aweq_w8a8_gemm_tokens(const void* X, aweq_dtype x_dt, int64_t T, int64_t K, int64_t ldx, const float* inv_s,
                          int8_t* xq, float* step_x, int32_t* zero_x, int32_t* rowsum_x,
                          const int8_t* wq, int64_t N, const float* step_w, const int32_t* zero_w, int w_group,
                          const int32_t* rowsum_w, const float* bias, void* out, aweq_dtype out_dt, int64_t ldo,
                          uint32_t* status, void* stream);

/* ---- Rotation by position.  The pair i of a head's first `rot` values turns by pos * freq[i], i < rot / 2: (x[i], x[i + rot / 2]), or with
 * interleaved (x[2i], x[2i + 1]).  aweq_rope_frequencies fills freq[rot / 2] (HOST memory, binary64) with base^(-2i / rot), scaled for contexts
 * `factor` times the trained length:
 *   AWEQ_ROPE_PLAIN   as it is
 *   AWEQ_ROPE_LINEAR  freq / factor (positions pressed together)
 *   AWEQ_ROPE_BASE    base * factor^(rot / (rot - 2)): the slowest pair turns factor times slower, the fastest as before (rot > 2)
 *   AWEQ_ROPE_PARTS   by the turns a pair makes over the trained length: above `high` as it is, below `low` freq / factor, between
 *                     them blended linearly in the turns.
 * Host function; AWEQ_ERR_SHAPE for rot odd or <= 0, base <= 0 (or not finite), factor <= 0, an unknown kind, or (PARTS) trained <= 0 or high <= low. */
enum { AWEQ_ROPE_PLAIN = 0, AWEQ_ROPE_LINEAR = 1, AWEQ_ROPE_BASE = 2, AWEQ_ROPE_PARTS = 3 };
int aweq_rope_frequencies(int64_t rot, double base, int kind, double factor, double trained, double low, double high, double* freq);

/* ---- Norm of every head of the queries and keys and their rotation, in one pass.  q[T][Hq][D], k[T][Hk][D] (F32, F16 or BF16; the heads
 * of a token side by side, pitch ldq / ldk from token to token: parts of the fused projection's rows will do); q or k nullable.
 *   y = x * w[d] / sqrt(mean_d x^2 + eps)   (q_norm / k_norm fp32[D]; NULL: y = x)
 *   rotated by pos[t] (int32, any sign) as above, cosine and sine times gain; values past rot are left as they are.
 * Norm, angle (reduced in binary64) and rotation are not rounded in between; outputs once, to dt (pitch ldqo, ldko).  q_out may be q, and k_out
 * k, with the same pitch.  rot = 0: the norms alone (pos and freq may be NULL); else rot <= D, a multiple of 16, or of 8 with interleaved.
 * D % 8 == 0, D <= 256; 16-byte aligned pointers and pitches (freq and pos: of their type). */
int aweq_qk_rope(const void* q, const void* k, aweq_dtype dt, int64_t T, int64_t Hq, int64_t Hk, int64_t D, int64_t ldq, int64_t ldk,
                 const int32_t* pos, const double* freq, int64_t rot, int interleaved, float gain,
                 const float* q_norm, const float* k_norm, float eps, void* q_out, int64_t ldqo, void* k_out, int64_t ldko, void* stream);

/* ---- A paged cache of keys and values.  k_cache and v_cache hold `pages` pages of Hk heads of page_size tokens of D values each,
 * [pages][Hk][page_size][D], in the queries' type (F16 or BF16), or as 8-bit codes (cache_dt = AWEQ_I8) with k_step and v_step
 * [pages][Hk][page_size] fp32: the value is code * step, step = max |x| / 127 of the token's head (the smallest normal number at least; 1 for a head of
 * zeros; always positive, or NaN), code = round(x / step).
 * (Symmetric, unlike the quantizers above: a zero point would cost a correction of every score.)  page_size: a power of two from 16 to 256.
 *
 * aweq_kv_append: aweq_qk_rope, with the keys, and the values v[T][Hk][D] (pitch ldv) as they are, going to the cache: token t to row slot[t] %
 * page_size of page slot[t] / page_size (int64; negative: the token is left out of the cache, a padded batch; past the last page: the
 * same, and AWEQ_ST_INDEX).  Tokens of one call must not share a slot.  An 8-bit code is made of the rotated value before any other rounding; a
 * head with a NaN or an infinity gets a step of NaN and raises AWEQ_ST_NONFINITE (a cache of the values' type holds them as they are). q
 * nullable (with q_out).  D % 8 == 0 and D <= 256; dt F16 or BF16. */
int aweq_kv_append(const void* q, const void* k, const void* v, aweq_dtype dt, int64_t T, int64_t Hq, int64_t Hk, int64_t D,
                   int64_t ldq, int64_t ldk, int64_t ldv, const int32_t* pos, const double* freq, int64_t rot, int interleaved, float gain,
                   const float* q_norm, const float* k_norm, float eps, void* q_out, int64_t ldqo,
                   void* k_cache, void* v_cache, float* k_step, float* v_step, aweq_dtype cache_dt, int64_t pages, int64_t page_size,
                   const int64_t* slot, uint32_t* status, void* stream);

/* ---- Attention of a batch over a prefix that all its sequences share and over each one's own pages.  q[T][Hq][D] (F16 or BF16, pitch
 * ldq): the new tokens of B sequences one after the other, those of sequence b from q_start[b] to q_start[b + 1] (int32[B + 1]; NULL: one each, T = B).
 * Query head h reads key head h / (Hq / Hk).  The keys of a token are
 *   the prefix: the first prefix_len tokens of the pages prefix_table[ceil(prefix_len / page_size)] (int32; prefix_len a HOST number, 0: none), and
 *   its sequence's own: lens[b] tokens (int32, 0 allowed) of the pages table[b][..] (int32, pitch table_ld), of which the last ones are its
 *   new tokens, appended before this call: new token i of m sees the first lens[b] - m + 1 + i of them.
 *   out[t][h] = sum_j p_j v_j,  p = softmax(scale * q k_j);   lse[t][h] (fp32, nullable) = log sum_j exp(scale * q k_j).
 * A token without any key gets zeros, and lse -inf; so does one whose scores all are -inf, and any key of such a score is left out.  A NaN in a query, in a key
 * that it sees or in that key's step, and a score of +inf, make the token's out and lse for that head NaN, however the keys are split; a
 * value that is not finite makes the out of the tokens that see it infinite or NaN where it stands, and has no part in any other's.  No status bit tells of it.  max_len and max_q (HOST): no lens[b] and no sequence's count of new tokens is larger; the launch is
 * laid out for them.  A page outside [0, pages), a length over max_len or over what table_ld pages hold, or rows of q_start out of order
 * raise AWEQ_ST_INDEX and are clamped (results unspecified, no access out of range).  Rows of out and lse past q_start[B] are unspecified.
 * The prefix is read once for all the batch's queries, which multiply its keys together; long key ranges are split between
 * workgroups whose partial results (fp32, in ws) a second launch joins.  Scores and softmax in fp32, with products of the stored
 * type exact in fp32; the probabilities are rounded to F16 / BF16 for the product with v (an 8-bit cache: both products in F16, BF16 queries scaled by a power
 * of two, and probabilities times their value's step by one for each token and head, which follows the largest step that it sees: a step says nothing of its
 * key's weight; a step of a value that is not finite makes the out of what sees it NaN).  D 64, 128 or 256; Hq a multiple of Hk; scale > 0, below 2^127; cache as
 * above (aweq_kv_append fills heads of other sizes too, which this does not read).  At most: T Hq 2^24 - 1, B Hk 2^24, B 2^20, Hq 2^16, prefix_len and
 * max_len 2^29, pages 2^31 - 1, workgroups of a launch (sequences or the prefix, key heads, ranges of keys, row tiles) 2^24 - 1; AWEQ_ERR_SHAPE beyond, and 0 from the two functions below.
 * ws: aweq_prefix_attention_ws(...) bytes, 16-byte aligned (host function; 0: none is needed).  A smaller call may need more, since fewer rows are split into
 * more ranges: aweq_prefix_attention_ws_most is enough for every call with no more of T, B, max_q, prefix_len and max_len whose T is at most its B max_q. */
size_t aweq_prefix_attention_ws(int64_t T, int64_t Hq, int64_t Hk, int64_t D, int64_t B, int64_t max_q, int64_t prefix_len, int64_t max_len);
size_t aweq_prefix_attention_ws_most(int64_t T, int64_t Hq, int64_t Hk, int64_t D, int64_t B, int64_t max_q, int64_t prefix_len, int64_t max_len);
int aweq_prefix_attention(const void* q, aweq_dtype dt, int64_t T, int64_t Hq, int64_t D, int64_t ldq,
                          const void* k_cache, const void* v_cache, const float* k_step, const float* v_step, aweq_dtype cache_dt,
                          int64_t pages, int64_t page_size, int64_t Hk, const int32_t* prefix_table, int64_t prefix_len,
                          const int32_t* table, int64_t table_ld, const int32_t* lens, const int32_t* q_start, int64_t B,
                          int64_t max_len, int64_t max_q, float scale, void* out, int64_t ldo, float* lse,
                          void* ws, size_t ws_bytes, uint32_t* status, void* stream);

/* ======== Projections in 4-bit floating point ========
 *
 * ---- Microscaled 4-bit format.  Each block of 32 values along K has a power of two 2^e, and a value's code stands for one of 0, 0.5, 1, 1.5, 2, 3, 4, 6
 * times that, with a sign (bit 3).  x[r,k] = X[r,k] * factor[k] (one fp32 multiply; factor nullable).  For a block with the largest magnitude m:
 *   e = floor(log2 m) - 2, at least -127 (a block of zeros: -127);  code = the nearest to x / 2^e, ties to the even code, 6 where that is larger.
 * A block with a NaN or an infinity gets the scale NaN, which every value of it then is, and raises AWEQ_ST_NONFINITE.
 * K % 32 == 0.  Codes: panels of 128 values, two a byte (even k low), rows back to back, zero fill past K:
 *     byte of M[r][k] = ((k / 128) * rows + r) * 64 + (k % 128) / 2;
 * scales e + 127 (255: NaN): 16 bytes for each row and four panels (512 values), block b = k % 128 / 32 of panel p = k / 128 at
 *     ((p / 4) * rows + r) * 16 + ((b % 2) * 2 + b / 2) * 4 + p % 4
 * (a matrix unit's lane then has the scales of four panels in one register), those of blocks past K in the last panel 127, of panels past it unspecified.
 * aweq_mx4_code_bytes, aweq_mx4_scale_bytes: sizes of the two buffers (host functions; 0 where the shape is none).
 * aweq_quant_mx4: X[rows x K] F32, F16 or BF16, pitch ldx.  aweq_mx4_values: the values that the codes stand for, to F32, F16 or BF16 (rounded; BF16 and
 * F32 hold them as they are), pitch ldo.  K <= 2^20, rows < 2^31; 16-byte aligned pointers and rows. */
size_t aweq_mx4_code_bytes(int64_t rows, int64_t K);
size_t aweq_mx4_scale_bytes(int64_t rows, int64_t K);
int aweq_quant_mx4(const void* X, aweq_dtype dt, int64_t rows, int64_t K, int64_t ldx, const float* factor, uint8_t* codes, uint8_t* scales,
                   uint32_t* status, void* stream);
int aweq_mx4_values(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t K, void* out, aweq_dtype out_dt, int64_t ldo, void* stream);

/* ---- Product of two such matrices: out[t,n] = sum_k x[t,k] w[n,k] + bias[n] (bias fp32, nullable).  X[T x K] (F32, F16, BF16; pitch ldx) is quantised as by
 * aweq_quant_mx4 first, and xq and x_scale are written; X NULL: they are inputs.  wq, w_scale: the weight's.  Products are exact, sums fp32 in an order that
 * depends on the shape alone, rounded once to out_dt (F32, F16, BF16; pitch ldo).  K % 32 == 0, K <= 2^20, N % 4 == 0, ldo % 4 == 0, T and N < 2^31;
 * 16-byte aligned pointers. */
int aweq_mx4_gemm_tokens(const void* X, aweq_dtype x_dt, int64_t T, int64_t K, int64_t ldx, const float* factor, uint8_t* xq, uint8_t* x_scale,
                         const uint8_t* wq, const uint8_t* w_scale, int64_t N, const float* bias, void* out, aweq_dtype out_dt, int64_t ldo,
                         uint32_t* status, void* stream);

/* ======== Drafted tokens: several of a sequence in one step, of which a part is kept ========
 *
 * ---- A step's plan, from what each of B sequences has and what it gets.  lens[b]: tokens in its pages; change[b] > 0: that many more, < 0: the last -change
 * of them go, 0: neither.  With page_size tokens to a page (as above) a sequence has ceil(lens / page_size) pages, the first entries of its row of `table`
 * ([B][table_pages], pitch table_ld).  free_pages[pages] is a stack of the pages that nobody has, *free_count of them.
 *   Pages that no longer hold a token are given back, in the order of the sequences and of their rows; they are the first that are taken, then the stack's
 *   from its top.  Sequences take theirs in order, into the entries behind those that they have.  What is left of those given back goes on the stack.
 *   lens_out[b] = lens + change, *count_out: pages on the stack;  q_start[B + 1]: the new tokens of each sequence, one sequence after the other;
 *   pos[t] = prefix_len + place in its sequence, slot[t] = where the token goes (aweq_kv_append), T of each; past q_start[B]: 0 and -1.
 * Where the pages do not suffice nothing is changed (lens_out = lens, *count_out = *free_count, q_start all 0, pos 0, slot -1) and AWEQ_ST_PAGES is raised; the same,
 * with AWEQ_ST_INDEX, for a length below 0, more taken away than there is, more tokens than T, a sequence longer than table_pages pages, a count
 * outside [0, pages], or more pages free and given back than there are.  lens_out must not be lens, nor count_out free_count (AWEQ_ERR_ALIGN for an output that overlaps an input): a step has the next one's inputs
 * beside its own.  B <= 8192, T <= 2^24,
 * pages < 2^31, table_pages <= 2^24, prefix_len <= 2^29, table_pages * page_size <= 2^29. */
int aweq_step_plan(const int32_t* lens, const int32_t* change, int64_t B, int64_t page_size, int64_t pages, int32_t* table, int64_t table_ld,
                   int64_t table_pages, int32_t* free_pages, const int32_t* free_count, int64_t prefix_len, int64_t T,
                   int32_t* lens_out, int32_t* count_out, int32_t* q_start, int32_t* pos, int64_t* slot, uint32_t* status, void* stream);

/* ---- Which of its sequence's new tokens a drafted token sees.  The new tokens of sequence b are the rows q_start[b] .. q_start[b + 1] - 1; parent[t] (int32) is
 * the place among them of the token that t goes on from, an earlier one, or -1: what the sequence has already (anything else: taken as -1, and
 * AWEQ_ST_INDEX).  mask[t] (words of 64 bits, pitch mask_ld words >= ceil(max_q / 64)): bit j says that t is new token j or goes on from it, however
 * far; bits of all ceil(max_q / 64) words are written.  pos[t] (nullable, with lens) = prefix_len + lens[b] - m + depth, m its sequence's new tokens, depth how
 * many of them come before t on its path.  max_q (HOST): no sequence has more; <= 4096.  Rows past q_start[B] are left as they are.  q_start out of
 * order, past T, or with more than max_q rows: AWEQ_ST_INDEX and clamped.  mask or pos over an input: AWEQ_ERR_ALIGN.  B <= 2^20, T <= 2^24. */
int aweq_tree_mask(const int32_t* parent, int64_t T, const int32_t* q_start, int64_t B, int64_t max_q, const int32_t* lens, int64_t prefix_len,
                   uint64_t* mask, int64_t mask_ld, int32_t* pos, uint32_t* status, void* stream);

/* ---- aweq_prefix_attention for new tokens that do not all see one another: of its sequence's lens[b] keys a token sees the first lens[b] - m, and of the m
 * new ones (the last m) those whose bit is set in mask[t] (pitch mask_ld words >= ceil(max_q / 64); any bits, its own or not).  All else, limits and scratch
 * memory (aweq_prefix_attention_ws, aweq_prefix_attention_ws_most) as there; a row without any key gets zeros and lse -inf, what a token does not
 * see has no part in its out, whatever it holds, and rows past q_start[B] (a batch that is filled up) are left as they are; q_start[0] is 0.  q_start is required, and table if max_len > 0; lens[b] < m: AWEQ_ST_INDEX (results of that sequence unspecified). */
int aweq_tree_attention(const void* q, aweq_dtype dt, int64_t T, int64_t Hq, int64_t D, int64_t ldq,
                        const void* k_cache, const void* v_cache, const float* k_step, const float* v_step, aweq_dtype cache_dt,
                        int64_t pages, int64_t page_size, int64_t Hk, const int32_t* prefix_table, int64_t prefix_len,
                        const int32_t* table, int64_t table_ld, const int32_t* lens, const int32_t* q_start, int64_t B,
                        int64_t max_len, int64_t max_q, const uint64_t* mask, int64_t mask_ld, float scale, void* out, int64_t ldo, float* lse,
                        void* ws, size_t ws_bytes, uint32_t* status, void* stream);

/* ---- After a step some of whose new tokens are kept: kept[b][j], j < count[b] (int32, pitch kept_ld >= every count; what lies behind them is not read), are their places among sequence
 * b's m new tokens, in strictly increasing order.  Their keys and values (and steps) move to the places 0 .. count - 1 of those, and change[b] = count - m is what
 * aweq_step_plan takes to drop the rest.  The tokens behind the kept ones are unspecified afterwards.  A count outside [0, min(m, kept_ld)], places out of
 * order or outside [0, m), lens[b] < m, or pages outside [0, pages): AWEQ_ST_INDEX, and nothing of that sequence is moved (change 0; a page outside: the
 * rows on it alone); so for a sequence longer than table_ld pages.  No two sequences may have a page of new tokens in common.  Caches as in aweq_kv_append;
 * T, q_start, lens, table: the step's.  change over an input, or among the min(kept_ld, T) entries from a row of kept on: AWEQ_ERR_ALIGN.  B <= 2^20, Hk < 2^16, B * Hk <= 2^24, T <= 2^24. */
int aweq_kv_keep(void* k_cache, void* v_cache, float* k_step, float* v_step, aweq_dtype cache_dt, int64_t pages, int64_t page_size, int64_t Hk, int64_t D,
                 const int32_t* table, int64_t table_ld, const int32_t* lens, const int32_t* q_start, int64_t B, int64_t T,
                 const int32_t* kept, int64_t kept_ld, const int32_t* count, int32_t* change, uint32_t* status, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* AWEQ_H */
