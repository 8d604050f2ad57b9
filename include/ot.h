/*
 * ot.h -- C ABI of libot, OutlierTune's per-channel-quantized linear layer
 * for AMD Instinct MI355X (gfx950).
 *
 * The library implements the inference path of OutlierTune (Wang et al.,
 * 2024): static per-channel calibration of the activations with a
 * symmetrization shift (Sec. 3.2, App. A), the offline fold of the
 * activation scale into the weights and of the shift into the bias
 * (Sec. 3.1 Eq. (e), Eq. (f), Sec. 3.2 Eq. (g)), runtime per-channel
 * quantization of the activations (Eq. (g)), and the integer GEMM with a
 * dequantizing epilogue (Eq. (f) right-hand side, Eq. (g)).
 *
 * Conventions shared by every entry point
 *  - Tensors are dense and row-major (leading dimension = inner size).
 *    X is [M x K] (tokens x input channels); the weight W is [N x K], the
 *    layout of a PyTorch nn.Linear weight, so the paper's W^T is its
 *    transpose.
 *  - Every tensor pointer is a DEVICE pointer owned by the caller.  The
 *    library never allocates, frees or retains caller memory and keeps no
 *    global state (apart from ot_qlinear_noalloc's fixed scratch array and a
 *    4 KiB block of pinned host memory, allocated by the first synchronous
 *    call, for their status words); calls on different streams are
 *    independent.
 *  - fp16 tensors are passed as uint16_t IEEE binary16 bit patterns.
 *  - bits is in [2, 8]; the quantizer is symmetric and signed with largest
 *    code q(bits) = 2^(bits-1) - 1 (127 for 8 bits, 31 for 6 bits).  Codes
 *    are stored in int8 whatever the bit-width.  Rounding is round half to
 *    even throughout.
 *  - stream is a hipStream_t passed as void* (NULL = the default stream).
 *  - Every argument check happens on the host before any launch: on an
 *    error status no kernel runs and no output is written, except where an
 *    entry point says otherwise.  A fault inside an asynchronous kernel
 *    surfaces as OT_EHIP from a later synchronous call or from the caller's
 *    own stream synchronization.
 */
#ifndef OT_H_
#define OT_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum ot_status {
  OT_OK = 0,
  OT_EINVAL = 1,     /* null pointer, bits outside [2, 8], negative size     */
  OT_ESHAPE = 2,     /* K not a multiple of 16, zero-sized where disallowed  */
  OT_ERANGE = 3,     /* K * qa * qw >= 2^31: the int32 accumulator could wrap */
  OT_ENONFINITE = 4, /* NaN or infinity in calibration data or weights       */
  OT_EHIP = 5,       /* a HIP runtime call failed                            */
  OT_ENOSCRATCH = 6  /* ot_qlinear_noalloc: the sizes need more scratch than  */
                     /* the library's fixed array holds                      */
} ot_status;

/* Static, human-readable description of a status code. */
const char *ot_strerror(int status);

/* Version of this ABI (bumped on any incompatible change). */
int ot_abi_version(void);

/* Static description of this build, "key=value" fields separated by ';':
 *   sources_sha256  SHA-256 of the sources and the release compiler flags
 *                   it was built from ("unknown" when built without the
 *                   recipe that computes it), so that a loaded library can
 *                   be matched against a source tree;
 *   arch            the GPU architecture of its device code;
 *   hip             the HIP version it was compiled against;
 *   header_sha256   SHA-256 of the ot.h it was compiled with ("unknown" as
 *                   above): code compiled against this header can tell
 *                   whether a library that it loads has the same signatures.
 * Never NULL; owned by the library. */
const char *ot_build_info(void);

/*
 * ot_calibrate -- static min-max calibration and symmetrization factors.
 * Sec. 3.2 (z = (max + min) / 2 per channel, X_hat = X - z) and App. A
 * (min-max calibration of the activations, done offline).
 *
 *   x       [rows x K] fp16 calibration activations (device).
 *   rows    >= 1.   K >= 1.
 *   a_bits  activation bit-width, in [2, 8]; qa = 2^(a_bits-1) - 1.
 *   first   nonzero: reset the running state before folding this batch in;
 *           zero: accumulate into the state left by earlier calls.
 *   minmax  [2K] fp32 running state (device): the K per-channel minima then
 *           the K maxima.  -0 is recorded as +0.
 *   z, s, inv_s  [K] fp32 outputs (device), rewritten from the running state
 *           on every call, so they are final after the last batch:
 *             z_k     = fp32((hi_k + lo_k) / 2)
 *             s_k     = fp32(((hi_k - lo_k) / 2) / qa), 1 if that is 0
 *             inv_s_k = fp32(1 / s_k)
 *           (fp64 arithmetic, each result rounded once to fp32).
 *
 * Synchronous: waits for the stream.  Returns OT_ENONFINITE if the running
 * state holds a NaN or an infinity (then z, s, inv_s are not written; the
 * state stays poisoned until a call with first != 0).
 */
ot_status ot_calibrate(const uint16_t *x, int64_t rows, int64_t K, int a_bits,
                       int first, float *minmax, float *z, float *s,
                       float *inv_s, void *stream);

/*
 * ot_scales_from_minmax -- z, s, 1/s from a calibration state (the minmax
 * that ot_calibrate keeps), for any bit-width, with or without the
 * symmetrization of Sec. 3.2 (the ablation of Sec. 4.4, Table 6):
 *   symmetrize != 0:  z_k = (hi_k + lo_k)/2,  s_k = ((hi_k - lo_k)/2)/qa
 *   symmetrize == 0:  z_k = 0,                s_k = max(|lo_k|, |hi_k|)/qa
 * fp64 math, fp32 storage, s_k = 1 where it would be 0, inv_s_k =
 * fp32(1/s_k).  With symmetrize != 0 and the calibration's own a_bits this
 * reproduces ot_calibrate's outputs exactly.
 *   minmax [2K] fp32 (device; the K minima then the K maxima, finite).
 *   z, s, inv_s [K] fp32 outputs (device).
 * Asynchronous on stream.
 */
ot_status ot_scales_from_minmax(const float *minmax, int64_t K, int a_bits,
                                int symmetrize, float *z, float *s,
                                float *inv_s, void *stream);

/*
 * ot_fold_weights -- the offline weight and bias transform.
 * Sec. 3.1 Eq. (e) (W_s = W scaled by s along the input channels), Eq. (f)
 * (per-output-channel quantization of W_s), Sec. 3.2 Eq. (g) (the shift z
 * moves into the bias, b' = z W^T + b), Implementation paragraph (the
 * weight quantization is done once, offline).
 *
 *   W       [N x K] fp16 weight (device).      b [N] fp16 bias or NULL.
 *   w_bits  weight bit-width in [2, 8]; qw = 2^(w_bits-1) - 1.
 *   z, s    [K] fp32 from ot_calibrate (device).
 *   Wq      [N x K] int8 output: clip(rne(W[n,k] s_k / sW_n), -qw, qw).
 *   sW      [N] fp32 output: fp32(max_k |W[n,k] s_k| / qw), 1 for a zero row.
 *   bprime  [N] fp32 output: fp32(sum_k z_k W[n,k] + b_n), summed in fp64
 *           (the summation order is unspecified, so it can differ from a
 *           sequential sum in the last fp32 place).
 *   The products W[n,k] s_k are exact in fp64, the division by sW_n is a
 *   correctly rounded fp64 division.
 *
 * Synchronous.  OT_ENONFINITE if W or b holds a NaN or an infinity; then
 * the contents of Wq, sW and bprime are unspecified.
 */
ot_status ot_fold_weights(const uint16_t *W, const uint16_t *b, int64_t N,
                          int64_t K, int w_bits, const float *z, const float *s,
                          int8_t *Wq, float *sW, float *bprime, void *stream);

/*
 * ot_quantize_act -- runtime symmetrize + per-channel quantize, Eq. (g):
 *   Xq[m,k] = clip(rne(fp32(fp32(x[m,k]) - z_k) * inv_s_k), -qa, qa)
 * with both fp32 operations rounded to nearest even (no fused multiply-add).
 * Values outside the calibrated range clip; NaN input gives unspecified
 * codes.
 *
 *   x      [M x K] fp16 (device).  M >= 0 (0 is a no-op), K >= 16, K % 16 == 0.
 *   z, inv_s  [K] fp32 (device).    Xq [M x K] int8 output (device).
 *
 * Asynchronous on stream.
 */
ot_status ot_quantize_act(const uint16_t *x, int64_t M, int64_t K, int a_bits,
                          const float *z, const float *inv_s, int8_t *Xq,
                          void *stream);

/*
 * ot_ln_quantize_act -- LayerNorm fused with symmetrization and Eq. (g)'s
 * per-channel quantization (Sec. 3.2: z is taken into the LayerNorm's bias,
 * Implementation paragraph: the quantization is fused with the LayerNorm
 * that precedes the linear).  Per row of h, with a_k = h_k 2^24 (an exact
 * integer for every fp16 value), S1 = sum_k a_k and S2 = sum_k a_k^2
 * (exact integers) and each float64 step rounded to nearest:
 *   mean = fl(fl(S1) / K) 2^-24
 *   var  = fl(fl(K S2 - S1^2) / K^2) 2^-48       (population variance)
 *   rstd = fl(1 / fl(sqrt(fl(var + eps))))
 * and per element, in fp32 rounded to nearest even (no fused multiply-add):
 *   Xq[m,k] = clip(rne((((h - fp32(mean)) * fp32(rstd)) * gamma_k
 *                       + (beta_k - z_k)) * inv_s_k), -qa, qa)
 * The codes are exactly these.  The kernel reaches fp32(mean) and
 * fp32(rstd) through float64 sums with a proven error bound, and through
 * the exact integer sums for the rows that bound cannot settle (a mean or
 * rstd within the bound of an fp32 rounding boundary, e.g. a mean of 0), so
 * such rows cost more.
 * The normalized fp16 activation is never written.
 *
 *   h      [M x K] fp16 LayerNorm input (device).  M >= 0 (0 is a no-op),
 *          16 <= K <= 65536, K % 16 == 0.  Finite values; a row of equal
 *          values with eps == 0 (and NaN or infinity anywhere in a row)
 *          gives unspecified codes for that row.
 *   gamma, beta  [K] fp16 LayerNorm weight and bias (device).
 *   eps    the LayerNorm epsilon, finite and >= 0.
 *   z, inv_s     [K] fp32 from ot_calibrate on the LayerNorm's output.
 *   Xq     [M x K] int8 output (device).
 *
 * Asynchronous on stream.
 */
ot_status ot_ln_quantize_act(const uint16_t *h, int64_t M, int64_t K,
                             const uint16_t *gamma, const uint16_t *beta,
                             float eps, int a_bits, const float *z,
                             const float *inv_s, int8_t *Xq, void *stream);

/*
 * ot_qlinear -- the quantized linear: integer GEMM (Eq. (f) right-hand side)
 * with the fused dequantizing epilogue of Eq. (g):
 *   acc[m,n] = sum_k Xq[m,k] Wq[n,k]                       (exact int32)
 *   Y[m,n]   = fp16(fp32(fp32(acc[m,n]) * sW_n) + bprime_n)
 * every conversion and operation rounded to nearest even, no fused
 * multiply-add.  Prefill shapes run on the int8 matrix cores; M <= 64 runs
 * a weight-streaming decode kernel.  Both give bit-identical results.
 *
 *   Xq [M x K] int8, Wq [N x K] int8, sW [N] fp32, bprime [N] fp32 (device).
 *   M >= 0 (0 is a no-op), N >= 1, K >= 16 with K % 16 == 0.
 *   a_bits, w_bits  the bit-widths the codes were made with; they bound the
 *           codes (|Xq| <= qa, |Wq| <= qw) and so the accumulator:
 *           OT_ERANGE if K * qa * qw >= 2^31.  Codes outside those bounds
 *           give unspecified results.
 *   Y      [M x N] fp16 output (device).
 *   acc_out  NULL, or [M x N] int32 (device) that also receives acc (for
 *           testing; costs extra memory traffic).
 *   workspace  NULL, or at least ot_qlinear_workspace_size(M, N, K) bytes of
 *           16-byte-aligned device memory the call may use as scratch; with
 *           NULL the call uses no scratch memory.  Results do not depend on
 *           it.  For 17..64 tokens, where the launch plan finds it faster
 *           (layers with few output channels per compute unit and long K),
 *           the call then splits K over more workgroups and adds their int32
 *           partial sums in a second kernel (the sums are exact, so the
 *           outputs are identical); ot_qlinear_workspace_size returns 0
 *           where it does not.  The contents need no initialization and
 *           are left unspecified; calls that overlap in time must not share
 *           a workspace.
 *
 * Asynchronous on stream; no synchronization, no allocation.
 */
ot_status ot_qlinear(const int8_t *Xq, const int8_t *Wq, const float *sW,
                     const float *bprime, int64_t M, int64_t N, int64_t K,
                     int a_bits, int w_bits, uint16_t *Y, int32_t *acc_out,
                     void *workspace, void *stream);

/*
 * Asymmetric weights, the paper's "Int8" setting (Sec. 4.1, App. A):
 * per-output-channel asymmetric quantization of W_s = W diag(s), Eq. (a)
 * with a zero point.  With L = 2^w_bits - 1, per output channel n:
 *   lo, hi = min(min_k W_s[n,k], 0), max(max_k W_s[n,k], 0)
 *   sW[n]  = fp32((hi - lo) / L)  (1 where 0);  zp = clip(rne(-lo/sW), 0, L)
 *   c[n,k] = clip(rne(W_s[n,k] / sW[n]) + zp, 0, L)   (fp64, correctly rounded)
 * stored shifted so that they fit int8: Wq = c - 2^(w_bits-1),
 * zW[n] = zp - 2^(w_bits-1).  bprime as for ot_fold_weights.
 *
 * ot_fold_weights_asym -- arguments as ot_fold_weights plus zW [N] int32
 * output.  Synchronous; OT_ENONFINITE as ot_fold_weights.
 */
ot_status ot_fold_weights_asym(const uint16_t *W, const uint16_t *b, int64_t N,
                               int64_t K, int w_bits, const float *z,
                               const float *s, int8_t *Wq, float *sW,
                               int32_t *zW, float *bprime, void *stream);

/*
 * ot_qlinear_asym -- the quantized linear with asymmetric weights:
 *   acc[m,n] = sum_k Xq[m,k] (Wq[n,k] - zW[n])   exact in int32
 *   Y[m,n]   = fp16(fp32(fp32(acc[m,n]) * sW[n]) + bprime[n])
 * The kernels compute sum_k Xq Wq and subtract zW[n] times the token's code
 * sum, which they take from the token fragments they already hold.
 * Arguments as ot_qlinear plus zW [N] int32 (device); acc_out receives acc.
 * OT_ERANGE when K * qa * 2^w_bits >= 2^31.
 */
ot_status ot_qlinear_asym(const int8_t *Xq, const int8_t *Wq, const float *sW,
                          const int32_t *zW, const float *bprime, int64_t M,
                          int64_t N, int64_t K, int a_bits, int w_bits,
                          uint16_t *Y, int32_t *acc_out, void *workspace,
                          void *stream);

/*
 * Per-token path.  The paper keeps the linears without activation outliers
 * (out and fc2, whose inputs are not LayerNorm outputs) on per-token
 * symmetric activation quantization, Eq. (c), and carries a symmetrized
 * residual stream back through their bias, Eq. (h) (Sec. 3.2, Sec. 4.1).
 *
 * ot_quantize_act_per_token -- dynamic per-token scales and codes:
 *   sX[m]    = fp32(max_k |x[m,k]| / qa)   (fp64 division; 1 for a zero row)
 *   Xq[m,k]  = clip(rne(fp32(x[m,k]) * fp32(1 / sX[m])), -qa, qa)
 *   x   [M x K] fp16 (device), finite.  M >= 0 (0 is a no-op),
 *       16 <= K <= 65536, K % 16 == 0.
 *   Xq  [M x K] int8 output, sX [M] fp32 output (device).
 * Asynchronous on stream.
 */
ot_status ot_quantize_act_per_token(const uint16_t *x, int64_t M, int64_t K,
                                    int a_bits, int8_t *Xq, float *sX,
                                    void *stream);

/*
 * ot_fold_weights_per_token -- offline weights of a per-token linear: no
 * activation scale is folded in (Eq. (c)).
 *   sW[n]     = fp32(max_k |W[n,k]| / qw)   (1 for a zero row)
 *   Wq[n,k]   = clip(rne(W[n,k] / sW[n]), -qw, qw)  (correctly rounded fp64)
 *   bprime[n] = fp32(b[n] + zres[n])        (fp64 sum; Eq. (h))
 *   W [N x K] fp16, b [N] fp16 or NULL, zres [N] fp32 or NULL: the shift z
 *   of the symmetrized residual stream that this linear's output is added
 *   to (NULL when the residual stream is not symmetrized).
 * Synchronous.  OT_ENONFINITE if W, b or zres hold a NaN or an infinity.
 */
ot_status ot_fold_weights_per_token(const uint16_t *W, const uint16_t *b,
                                    const float *zres, int64_t N, int64_t K,
                                    int w_bits, int8_t *Wq, float *sW,
                                    float *bprime, void *stream);

/*
 * ot_qlinear_per_token -- the quantized linear of Eq. (c) with the bias:
 *   Y[m,n] = fp16(fp32(fp32(fp32(acc[m,n]) * sX[m]) * sW[n]) + bprime[n])
 * with acc = Xq Wq^T exact in int32, each fp32 operation rounded to nearest
 * even.  Arguments as for ot_qlinear, plus sX [M] fp32 (device) from
 * ot_quantize_act_per_token; same kernels, same error codes.
 */
ot_status ot_qlinear_per_token(const int8_t *Xq, const int8_t *Wq,
                               const float *sX, const float *sW,
                               const float *bprime, int64_t M, int64_t N,
                               int64_t K, int a_bits, int w_bits, uint16_t *Y,
                               int32_t *acc_out, void *workspace, void *stream);

/*
 * ot_qlinear_noalloc -- ot_qlinear for callers that cannot allocate device
 * memory (code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc).  Same arguments, checks and results as ot_qlinear
 * without the workspace argument: where ot_qlinear would use a workspace
 * (split-K decode, 17..64 tokens), this call uses a fixed device array of
 * OT_NOALLOC_SCRATCH_BYTES that the library holds on every device it runs
 * on until the process ends (its address is looked up on the first call on
 * each device).  It calls no allocation routine.  OT_ENOSCRATCH if
 * ot_qlinear_workspace_size(M, N, K) exceeds OT_NOALLOC_SCRATCH_BYTES
 * (then nothing runs; ot_qlinear with a workspace serves such sizes).  On
 * a 256-CU device that cannot happen: a split plan runs at most one
 * workgroup per CU, runs x ceil(N / rows) <= 256 with rows <= 128, so it
 * needs at most 64 x 4 x (32768 + 8) bytes (8.0 MiB).
 * Calls that overlap in time on one device share the array and race:
 * serialize them (one stream, or events).  Asynchronous on stream.
 */
#define OT_NOALLOC_SCRATCH_BYTES (9u << 20)
ot_status ot_qlinear_noalloc(const int8_t *Xq, const int8_t *Wq,
                             const float *sW, const float *bprime, int64_t M,
                             int64_t N, int64_t K, int a_bits, int w_bits,
                             uint16_t *Y, int32_t *acc_out, void *stream);

/* Bytes of optional scratch that ot_qlinear, ot_qlinear_per_token,
 * ot_qlinear_asym and ot_qlinear_packed can use for these sizes on the
 * current device (0 if none; also 0 for sizes the calls reject).
 * Synchronous, no device work. */
size_t ot_qlinear_workspace_size(int64_t M, int64_t N, int64_t K);

/*
 * ot_qlinear_plan -- which kernel configuration the quantized-linear calls
 * (ot_qlinear and its per-token and asymmetric variants, or, with
 * packed != 0, ot_qlinear_packed) launch for these sizes on the current
 * device, given a workspace (with_workspace != 0) or not.  Writes a
 * NUL-terminated description into buf (at most len bytes, truncated if
 * longer): "none" for M == 0; "prefill <R>x<T>" (output channels x tokens
 * per workgroup: 320x256, 256x256, 192x256, 256x128, 192x128, 128x128,
 * 128x96, 64x128, 64x64, 32x64 or 32x32) above 64 tokens; "decode <layout>
 * <R>-row tiles", with " split-K <runs>" where K is split, up to 64 tokens.
 * OT_EINVAL for a NULL buf or len 0, OT_ESHAPE for sizes the calls reject.  Synchronous, no device work; for
 * introspection and tests (the results never depend on the plan).
 */
ot_status ot_qlinear_plan(int64_t M, int64_t N, int64_t K, int packed,
                          int with_workspace, char *buf, size_t len);

/*
 * Packed weights for decode.  The folded codes (Eq. (f) right-hand side,
 * fixed offline like the fold itself, Sec. 3.2) re-laid so that each 1 KiB
 * is one matrix-instruction operand of a wave, which the weight-streaming
 * kernel loads straight into registers: micro-tiles of 16 output channels
 * by 64 input channels,
 *   Wp[g][s][l][b] = Wq[16 g + (l mod 16)][64 s + 16 (l / 16) + b]
 * for g < ceil(N/16), s < ceil(K/64), lane l < 64, byte b < 16, and 0 where
 * the row is >= N or the column >= K (the lane order of the A operand of
 * the 16x16x64 int8 matrix instruction).  The codes are unchanged, so
 * ot_qlinear_packed gives ot_qlinear's results bit for bit.
 *
 * ot_packed_weights_size -- bytes of Wp: ceil(N/16) ceil(K/64) 1024 (0 for
 *   sizes ot_pack_weights rejects).  No device work.
 * ot_pack_weights -- Wq [N x K] int8 (device) -> Wp (device, 16-byte
 *   aligned, ot_packed_weights_size bytes).  N >= 1, K >= 16, K % 16 == 0.
 *   Asynchronous on stream.
 * ot_qlinear_packed -- ot_qlinear for M <= 64 tokens (OT_ESHAPE beyond)
 *   with Wp from ot_pack_weights for the same N and K; the other arguments,
 *   the workspace and the results as for ot_qlinear.
 */
size_t ot_packed_weights_size(int64_t N, int64_t K);
ot_status ot_pack_weights(const int8_t *Wq, int64_t N, int64_t K, int8_t *Wp,
                          void *stream);
ot_status ot_qlinear_packed(const int8_t *Xq, const int8_t *Wp, const float *sW,
                            const float *bprime, int64_t M, int64_t N, int64_t K,
                            int a_bits, int w_bits, uint16_t *Y,
                            int32_t *acc_out, void *workspace, void *stream);

/*
 * MX4: microscaled 4-bit floating point, for linears whose weights and
 * activations both take 4 bits.  A block of 32 consecutive input channels
 * holds an 8-bit scale byte b, worth 2^(b-127), and 32 4-bit codes: the sign
 * (bit 3) and one of the levels 0, 0.5, 1, 1.5, 2, 3, 4, 6 (bits 0..2).  With
 * E the exponent field of the largest fp32 magnitude in the block,
 *   b    = max(E - 2, 0), or 255 where E = 255
 *   code = the level nearest to |v| 2^(127-b), ties to the even code, 6 where
 *          that is larger; the sign is v's
 * A block with a NaN or an infinity has b = 255 and stands for 32 NaNs (its
 * codes are 0); every product with it is NaN.
 *
 * Codes and scales of a matrix [rows x K], K a multiple of 32:
 *   c  [rows x K/2] uint8, channel 2j in the low half of byte j, 2j+1 in the
 *      high half;
 *   e  [ceil(K/256) x rows x 8] uint8: e[t][row][i] is the scale of the row's
 *      block 8t + i, 0 past K.
 *
 * The per-channel shift and scale of Eq. (g) are kept: the activations are
 * symmetrized and scaled per channel before their blocks are formed, the scale
 * is folded into the weights and the shift into the bias, so that a channel
 * with outliers does not take its block's other channels' resolution.
 *
 * For all mx4 entry points: 32 <= K <= 2^22, K % 32 == 0 (OT_ESHAPE), rows
 * below 2^31, pointers 16-byte aligned (ot_fold_weights_mx4's b and bprime: to
 * their elements; OT_EINVAL).
 *
 * ot_quantize_act_mx4 -- runtime activations:
 *   v[m,k] = fp32(fp32(fp32(x[m,k]) - z_k) * inv_s_k), each rounded to nearest
 *   even; z and inv_s both NULL: v = x.
 *   x [M x K] fp16, z, inv_s [K] fp32 or NULL (device); Xc, Xe outputs (device).
 *   M >= 0 (0 is a no-op).  Asynchronous on stream.
 */
ot_status ot_quantize_act_mx4(const uint16_t *x, int64_t M, int64_t K,
                              const float *z, const float *inv_s, uint8_t *Xc,
                              uint8_t *Xe, void *stream);

/*
 * ot_ln_quantize_act_mx4 -- the LayerNorm fused with the MX4 quantizer:
 *   v[m,k] = ((((h - fp32(mean)) * fp32(rstd)) * gamma_k + (beta_k - z_k)) * inv_s_k)
 * in fp32 rounded to nearest even (no fused multiply-add), with mean and rstd
 * as defined for ot_ln_quantize_act.  A NaN or an infinity in a row of h makes
 * every block of that row NaN (b = 255), and so do equal values with eps == 0.
 * Arguments as there otherwise (K <= 65536), outputs as ot_quantize_act_mx4;
 * M < 2^22 (OT_ESHAPE).  Asynchronous on stream.
 */
ot_status ot_ln_quantize_act_mx4(const uint16_t *h, int64_t M, int64_t K,
                                 const uint16_t *gamma, const uint16_t *beta,
                                 float eps, const float *z, const float *inv_s,
                                 uint8_t *Xc, uint8_t *Xe, void *stream);

/*
 * ot_fold_weights_mx4 -- the offline transform of a layer's weights:
 *   v[n,k] = fp32(W[n,k] s_k)  (s NULL: W[n,k])
 *   bprime[n] = fp32(sum_k z_k W[n,k] + b_n)  (fp64; z NULL: b_n alone)
 *   W [N x K] fp16, b [N] fp16 or NULL, z, s [K] fp32 or NULL (device).
 *   Wc, We, bprime [N] fp32 outputs (device).  N >= 1.
 * Synchronous.  OT_ENONFINITE if a weight, a product with s or a bias is NaN or
 * infinite; then the outputs are unspecified.
 */
ot_status ot_fold_weights_mx4(const uint16_t *W, const uint16_t *b, int64_t N,
                              int64_t K, const float *z, const float *s,
                              uint8_t *Wc, uint8_t *We, float *bprime,
                              void *stream);

/*
 * ot_dequantize_mx4 -- the fp32 values that codes and scales stand for (exact;
 * NaN where the scale byte is 255).  c, e [rows x K] in MX4, y [rows x K] fp32
 * (device).  rows >= 0 (0 is a no-op).  Asynchronous on stream.
 */
ot_status ot_dequantize_mx4(const uint8_t *c, const uint8_t *e, int64_t rows,
                            int64_t K, float *y, void *stream);

/*
 * Packed MX4 weights: the order in which the products read them, laid out
 * once.  With T = ceil(K/256) and B = ceil(N/32), first the codes
 *   Wp[b][t][s][h][r][0..15] = the 16 bytes of block 8t + 4h + s of row 32b + r
 * for b < B, t < T, s < 4, h < 2, r < 32, then the scales
 *   We[t][32b + r][4h + s] at [t][b][h][r][s],
 * zeros past N and K.
 * ot_packed_weights_mx4_size -- its bytes, 4352 T B (0 for sizes that
 *   ot_pack_weights_mx4 rejects).  No device work.
 * ot_pack_weights_mx4 -- Wc, We (device) -> Wp (device).  N >= 1.
 *   Asynchronous on stream.
 */
size_t ot_packed_weights_mx4_size(int64_t N, int64_t K);
ot_status ot_pack_weights_mx4(const uint8_t *Wc, const uint8_t *We, int64_t N,
                              int64_t K, uint8_t *Wp, void *stream);

/*
 * ot_qlinear_mx4 -- the linear on MX4 operands:
 *   Y[m,n] = fp16(fp32(sum_k x[m,k] w[n,k]) + bprime_n)
 * with the values that the codes stand for; their products are exact, the sum
 * is in fp32.  Its order is unspecified, but fixed for given sizes on one kind
 * of device: the same call gives the same bits.  With a workspace the order is
 * another one than without, where the call uses it (ot_qlinear_mx4_plan tells).
 * Partial sums past fp32's largest value give an infinity or a NaN.
 *   Xc, Xe [M x K] and Wp of ot_pack_weights_mx4 for N x K, bprime [N] fp32
 *   (device).  M >= 0 (0 is a no-op), 1 <= N < 2^26 and
 *   ceil(M/256) ceil(N/256) < 2^23 (OT_ESHAPE).
 *   Y  [M x N] fp16 output (device).
 *   workspace  NULL, or at least ot_qlinear_mx4_workspace_size(M, N, K) bytes of
 *           scratch as for ot_qlinear, with which few tokens (from 17 on) on a
 *           long K are faster (K is shared between workgroups); up to 16 tokens
 *           none is used.  Calls that overlap in time must not share one.
 * Asynchronous on stream; no synchronization, no allocation.
 */
ot_status ot_qlinear_mx4(const uint8_t *Xc, const uint8_t *Xe, const uint8_t *Wp,
                         const float *bprime, int64_t M, int64_t N, int64_t K,
                         uint16_t *Y, void *workspace, void *stream);
/* Bytes of optional scratch that ot_qlinear_mx4 can use for these sizes on the
 * current device (0 if none, and for sizes it rejects).  No device work.
 * They are of these sizes alone: more tokens may use fewer bytes, or none, so a
 * buffer sized for the largest batch can be too small for a smaller one, and the
 * call, which is not told a size, would write past it. */
size_t ot_qlinear_mx4_workspace_size(int64_t M, int64_t N, int64_t K);
/* The most that ot_qlinear_mx4_workspace_size gives for 1 to M tokens: the size
 * of one buffer for calls of any of them (0 for sizes it rejects).  Host work of
 * up to a millisecond; no device work. */
size_t ot_qlinear_mx4_workspace_max(int64_t M, int64_t N, int64_t K);

/*
 * ot_qlinear_mx4_plan -- which kernel configuration ot_qlinear_mx4 launches for
 * these sizes on the current device, given a workspace or not; as
 * ot_qlinear_plan.  Writes "none" for M == 0, "decode <R> rows" (output channels
 * per workgroup: 16 or 32), or "tiles <R>x<T>" (output channels x tokens per
 * workgroup: 256x256, 192x256, 256x128, 192x128, 128x128, 64x128, 128x64
 * or 64x64), with " split-K <parts>" where K is shared between workgroups.
 */
ot_status ot_qlinear_mx4_plan(int64_t M, int64_t N, int64_t K, int with_workspace,
                              char *buf, size_t len);

/*
 * ot_moe_mx4 -- a whole mixture-of-experts layer for a few tokens on packed MX4
 * weights (a decode step).  An expert's rows of W1p and W2p are no packed weights
 * by themselves, since the scales of all experts lie behind all codes: larger
 * batches through ot_qlinear_mx4 need each expert's linears packed apart, as
 * copies of their own.  For token m, with its top_k largest logits (the lower expert
 * first among equals) and p the softmax over them,
 *   g_j  = W1_e x_m + b1_e             for its j-th expert e, in fp32
 *   h_j  = max(g_j, 0)                 OT_MOE_RELU, F1 = F
 *          silu(g_j[0..F)) g_j[F..2F)  OT_MOE_SWIGLU, F1 = 2F; silu(v) = v / (1 + e^-v)
 *   Y[m] = fp16(sum_j p_j (W2_e q(h_j) + b2_e)),  q: the values of h_j in MX4
 * A logit of -inf or NaN is never chosen: such a token takes fewer experts, and
 * one with no other logit gets Y = 0.  A NaN that the router should not have
 * made is therefore not seen in Y; a caller who wants to know looks at the logits.
 *   Xc, Xe [M x H] in MX4; logits [M x E] fp16 (device).
 *   W1p  packed weights of all experts' fc1 as one matrix [E F1 x H] (an
 *        expert's rows together; the gate's rows before the others).
 *   W2p  the same of fc2, [E H x F].
 *   b1 [E x F1], b2 [E x H] fp32, or NULL (device).
 *   M    0 (a no-op) .. OT_MOE_MAX_TOKENS.   E 1 .. OT_MOE_MAX_EXPERTS.
 *   top_k  1 .. min(E, OT_MOE_MAX_TOP_K).
 *   H, F   multiples of 32 up to 65536.
 *   Y    [M x H] fp16 output (device).
 *   workspace  ot_moe_mx4_workspace_size(M, H, F, E, top_k) bytes, 16-byte
 *        aligned (device).  Needs no initialization; calls that overlap in time
 *        must not share one.
 * OT_ESHAPE for sizes outside these.  The result does not depend on how calls
 * are scheduled: no atomics on sums.  Asynchronous on stream.
 */
#define OT_MOE_RELU 0
#define OT_MOE_SWIGLU 1
#define OT_MOE_MAX_TOKENS 64
#define OT_MOE_MAX_EXPERTS 256
#define OT_MOE_MAX_TOP_K 16
ot_status ot_moe_mx4(const uint8_t *Xc, const uint8_t *Xe,
                     const uint16_t *logits, const uint8_t *W1p,
                     const float *b1, const uint8_t *W2p, const float *b2,
                     int64_t M, int64_t H, int64_t F, int64_t E, int64_t top_k,
                     int act, uint16_t *Y, void *workspace, void *stream);
/* Bytes of the workspace (0 for M == 0 and for sizes it rejects). */
size_t ot_moe_mx4_workspace_size(int64_t M, int64_t H, int64_t F, int64_t E,
                                 int64_t top_k);

/*
 * KV8: a key/value cache in 8 bits, for the attention between the quantized qkv and
 * out linears.
 *
 * The cache is a pool of pages, each of OT_KV8_PAGE tokens of one sequence, for all
 * H key heads.  A page of a head holds one byte per value, b, worth (b - 128) s with
 * the page and head's fp32 scale s, for keys and for values apart:
 *   Kc  [num_pages x H x 64 x Dp] uint8     Ks  [num_pages x H] fp32
 *   Vc  [num_pages x H x Dp x 64] uint8     Vs  [num_pages x H] fp32
 * with Dp = ot_kv8_row_size(D): D rounded up to 64, 96, 128, 192 or 256.  Bytes past D
 * and past a page's tokens are unspecified and never seen.
 *
 * A batch is B sequences of a call's T rows and a page table:
 *   cu      [B + 1] int32: rows cu[b] .. cu[b+1] - 1 are sequence b's, in order (none
 *           where they are equal).  Rows from cu[B] on are padding: they are neither
 *           read nor written.
 *   kv_len  [B] int32: tokens that sequence b has once the call's are in the cache.
 *           Its n = cu[b+1] - cu[b] rows are its last n tokens, positions
 *           kv_len[b] - n .. kv_len[b] - 1.
 *   table   [B x max_pages] int32: token j of sequence b is in page
 *           table[b][j / 64], place j mod 64.  Entries past its tokens are not read.
 * All of them are in device memory, so that a captured graph can be replayed with
 * others.  They are not checked on the host; no value of them makes a call read or
 * write outside its tensors: what ot_kv8_append says of a page that is not in
 * 0 .. num_pages - 1, and what the others say, holds for positions past the table
 * (max_pages) too.  A cu that falls, or exceeds T, gives unspecified rows.
 *
 * For all kv8 entry points: 16 <= D <= 256, D % 16 == 0; 1 <= H <= 1024;
 * 0 <= B <= 65535; 0 <= T <= 2^24; 1 <= max_pages <= 2^24; 1 <= num_pages < 2^31
 * (OT_ESHAPE, as for calls too large for a launch).  B == 0 or T == 0 is a no-op.
 * fp16 tensors and codes 16-byte aligned, the others to their elements (OT_EINVAL).
 *
 * ot_kv8_row_size -- Dp (0 for a D that the calls reject).
 *
 * ot_kv8_append -- quantizes new tokens into their pages.  Per page and head, for keys
 * and for values apart, with a the largest magnitude of the call's tokens in it:
 *   s    = fp32(a / 127)   if the sequence has no earlier token in the page, or the
 *                          page's scale is 0
 *   s    = s_old 2^k       else, k >= 0 the least with a <= fp32(127.5 s_old) 2^k; where
 *                          k > 0 the earlier tokens' codes c become rne(c 2^-k)
 *   code = clip(rne(fp32(x fp32(1 / s))), -127, 127)   (0 where s is 0)
 * A token's error is at most s / 2 when written and below s ever after.  A NaN or an
 * infinity makes s, and with it all of the head's keys (or values) in the page, NaN
 * until a sequence begins the page anew.
 *   k, v   [T x H x D] fp16, token rows ldk and ldv elements apart (>= H D, multiples
 *          of 8: a qkv linear's output serves as it is).
 * Tokens of a page that the pool does not have (and of a position below 0) are left
 * out.  Two sequences of one call must not write to one page (pages of a shared prefix
 * are full ones, which are only read).  A call with the same tokens again changes
 * nothing.  Asynchronous on stream.
 */
#define OT_KV8_PAGE 64
int64_t ot_kv8_row_size(int64_t D);
ot_status ot_kv8_append(const uint16_t *k, int64_t ldk, const uint16_t *v,
                        int64_t ldv, int64_t T, int64_t B, int64_t H, int64_t D,
                        const int32_t *cu, const int32_t *kv_len,
                        const int32_t *table, int64_t max_pages,
                        int64_t num_pages, uint8_t *Kc, uint8_t *Vc, float *Ks,
                        float *Vs, void *stream);

/*
 * ot_kv8_read -- tokens of the cache as fp16(fp32(code s)), dense: rows cu[b] ..
 * cu[b+1] - 1 of k and v receive sequence b's tokens from position start[b] ([B]
 * int32) on.  Rows of a page that the pool does not have, and of positions below 0,
 * are NaN.  (A value near fp16's largest can come back as infinity: it is off by up to s.)
 *   k, v   [T x H x D] fp16 outputs (device).
 * Asynchronous on stream.
 */
ot_status ot_kv8_read(const uint8_t *Kc, const uint8_t *Vc, const float *Ks,
                      const float *Vs, int64_t num_pages, const int32_t *cu,
                      const int32_t *start, const int32_t *table,
                      int64_t max_pages, int64_t T, int64_t B, int64_t H,
                      int64_t D, uint16_t *k, uint16_t *v, void *stream);

/*
 * ot_attn_kv8 -- attention over the cache.  Query row i of sequence b (with
 * n = cu[b+1] - cu[b] of them) stands at position p = kv_len[b] - n + i; head g of Hq
 * goes with key head g / (Hq / Hkv).  With K_j and V_j the values that codes stand for,
 *   x_j = scale q . K_j     for j < kv_len[b], where causal != 0 only j <= p, and where
 *                           window > 0 (causal calls) only j > p - window
 *   Y   = sum_j e^x_j V_j / sum_j e^x_j,    lse = log sum_j e^x_j
 * A row without a key gets Y = 0 and lse = -inf.  Products are exact, sums and the
 * softmax's statistics in fp32; its weights, times their page's value scale (of a page
 * of zeros: 2^-31), are rounded to fp16 for the second product, by 2^-11 of themselves or
 * 2^-33 of the row's largest, whichever is more; its sum is in fp32, Y rounded once at the
 * end.  Keys behind the mask are never seen, also where they are NaN.  A NaN that a row
 * sees, among keys or values, makes its Y and its lse NaN; a page that the pool does not
 * have counts as NaN, and a kv_len past the table makes all of its sequence's rows NaN,
 * whatever they see of it.
 *   q      [T x Hq x D] fp16, rows ldq elements apart (>= Hq D, a multiple of 8).
 *   Hq     1 .. 16384, a multiple of Hkv.
 *   scale  finite (scores past fp32's range are unspecified, and those of a page whose
 *          scale times log2(e) scale is).   window  >= 0; 0: all keys (OT_EINVAL for
 *          others, and for a window without causal).
 *   max_q  1 .. T: no sequence has more rows than this (1 for decode).  Up to 32 rows to
 *          a key head (max_q Hq / Hkv) a kernel for few rows runs, which reads the cache
 *          at memory speed; rows of a sequence past max_q may be left as they were.  A
 *          prompt among many single tokens is faster as a call of its own where a key
 *          head has few query heads (a token takes a tile of 128 rows then; 63 tokens and
 *          a piece of 500, each over 1000 and more keys of 40 heads, take 194 us, in two
 *          calls 153).
 *   Y      [T x Hq x D] fp16 output, lse [T x Hq] fp32 output or NULL (device).
 *   workspace  NULL, or at least ot_attn_kv8_workspace_size(T, B, Hq, Hkv, D, max_q)
 *          bytes of 16-byte aligned scratch (device), with which a sequence's keys are
 *          shared between workgroups: few rows where tables have more than 16 pages,
 *          tiles where they would leave much of the device idle.  It needs no
 *          initialization; calls that overlap in time must not share one.
 * The order of the sums is fixed by the sizes, the lengths and whether there is a
 * workspace: the same call gives the same bits.  Asynchronous on stream; no
 * synchronization, no allocation.
 */
ot_status ot_attn_kv8(const uint16_t *q, int64_t ldq, int64_t T, int64_t B,
                      int64_t Hq, int64_t Hkv, int64_t D, const int32_t *cu,
                      const int32_t *kv_len, const int32_t *table,
                      int64_t max_pages, int64_t num_pages, const uint8_t *Kc,
                      const uint8_t *Vc, const float *Ks, const float *Vs,
                      float scale, int causal, int64_t window, int64_t max_q,
                      uint16_t *Y, float *lse, void *workspace, void *stream);
/* Bytes of optional scratch that ot_attn_kv8 can use for these sizes on the current
 * device (0 if none, and for sizes it rejects).  No device work. */
size_t ot_attn_kv8_workspace_size(int64_t T, int64_t B, int64_t Hq, int64_t Hkv,
                                  int64_t D, int64_t max_q);
/*
 * ot_attn_kv8_plan -- which kernel configuration ot_attn_kv8 launches for these sizes
 * on the current device, as ot_qlinear_plan: "none" (T or B == 0), "few <rows> rows"
 * (16 or 32 at a time), with ", <items> items" at most where a sequence's keys are shared
 * between workgroups, or "tiles <rows>" (128 or 256; small windows take 128), with
 * ", <parts> parts" at most where a tile's are.
 */
ot_status ot_attn_kv8_plan(int64_t T, int64_t B, int64_t Hq, int64_t Hkv,
                           int64_t D, int64_t max_q, int with_workspace,
                           char *buf, size_t len);

#ifdef __cplusplus
}
#endif

#endif /* OT_H_ */
