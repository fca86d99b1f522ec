/*
 * rdfft.h -- C ABI of the MI355X (gfx950) in-place real-domain FFT library.
 *
 * Implements the method of "Memory-Efficient Training with In-Place FFT
 * Implementation" (arXiv 2511.01385): a real FFT whose spectrum is written back
 * into the input's own n real slots (rdFFT), its inverse, and the
 * block-circulant linear layer (forward and backward) computed with them.
 *
 * Conventions shared by every entry point
 * --------------------------------------
 * - All pointers are DEVICE pointers on the current HIP device, 16-byte
 *   aligned.  The caller owns every buffer; the library keeps no pointer after
 *   the enqueued work completes.
 * - Every call validates its arguments on the host before any HIP call; on
 *   failure it returns a negative rdfft_status_t and enqueues nothing.
 * - Work is enqueued on `stream` (NULL = the default stream) and the call
 *   returns without synchronising.  Faults during execution surface at the
 *   caller's next synchronisation.
 * - No call allocates device memory.  The only device memory the library owns
 *   is a static table of twiddle factors (rdfft_table_bytes()), copied to each
 *   device the first time that device is used (or by rdfft_init()); that first
 *   use performs a synchronous copy and must not happen under stream capture.
 * - dtype selects the storage type of the transformed data; arithmetic is
 *   float32 throughout, bf16 and f16 values are widened exactly and rounded to
 *   nearest even on store (an f16 result beyond 65504 becomes an infinity).
 *
 * Packed spectrum layout ("pairs"), for a row of even length n:
 *   slot 0 = Y_0 (DC, real), slot 1 = Y_{n/2} (Nyquist, real),
 *   slots 2k, 2k+1 = Re Y_k, Im Y_k for 1 <= k < n/2,
 * where Y_k = sum_m x_m exp(-2 pi i k m / n)  (Sec. 3.1, Eq. (1), forward,
 * unnormalised).  The other half of the spectrum is conj-symmetric
 * (Sec. 3.1, Theorem 1) and DC/Nyquist are real (Sec. 4.1, "Squeeze N+2 into
 * N"), so these n reals hold the whole spectrum.
 */
#ifndef RDFFT_H
#define RDFFT_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#if defined(__GNUC__)
#define RDFFT_API __attribute__((visibility("default")))
#else
#define RDFFT_API
#endif

/* Same type as hipStream_t. */
struct ihipStream_t;
typedef struct ihipStream_t *rdfft_stream_t;

typedef enum {
  RDFFT_F32 = 0,  /* IEEE float32 storage */
  RDFFT_BF16 = 1, /* bfloat16 storage */
  RDFFT_F16 = 2   /* IEEE float16 storage */
} rdfft_dtype_t;

typedef enum {
  RDFFT_OK = 0,
  RDFFT_EINVAL = -1,       /* invalid argument (null/misaligned pointer, bad size, overlap) */
  RDFFT_EUNSUPPORTED = -2, /* valid but not implemented (n > 65536, n/2 with a prime factor
                              above 5 or beyond 16384 when not a power of two, p > 65536,
                              and the long-block limits of bca_forward / bca_backward) */
  RDFFT_ELAUNCH = -3,      /* HIP reported an error when enqueuing */
  RDFFT_EDEVICE = -4       /* no usable gfx950 device, or the twiddle table upload failed */
} rdfft_status_t;

/*
 * rdfft_forward -- in-place real FFT of `rows` rows (Sec. 4.1, rdFFT algorithm;
 * Sec. 3.1 Eq. (1), forward).
 *   buf   rows x n elements of `dtype`, row-major, row stride n.  On entry the
 *         real samples x_0..x_{n-1} of each row; on return the packed spectrum
 *         of that row in the layout above.
 *   rows  >= 0; rows == 0 is a no-op (buf may then be NULL).
 *   n     even, 2 <= n: a power of two up to 65536, or n = 2N with N = 2^a 3^b 5^c
 *         up to 16384 (mixed-radix rows: a row's points pass through LDS, twiddles
 *         computed on the fly).  Odd n -> RDFFT_EINVAL (no Nyquist bin,
 *         Theorem 1); any other even n -> RDFFT_EUNSUPPORTED.
 * No memory beyond buf is read or written (apart from the twiddle table).
 */
RDFFT_API int rdfft_forward(void *buf, int64_t rows, int64_t n, rdfft_dtype_t dtype, rdfft_stream_t stream);

/*
 * rdfft_inverse -- in-place inverse of rdfft_forward (Sec. 4.2; Sec. 3.1
 * Eq. (1), inverse, with the 1/n normalisation of Sec. 3.2):
 *   x_m = (1/n) sum_{k=0}^{n-1} Y_k exp(+2 pi i k m / n),  Y_{n-k} = conj(Y_k),
 * with the imaginary parts of Y_0 and Y_{n/2} taken as zero.  Any n reals are
 * a valid packed spectrum.  Arguments and errors as rdfft_forward.
 */
RDFFT_API int rdfft_inverse(void *buf, int64_t rows, int64_t n, rdfft_dtype_t dtype, rdfft_stream_t stream);

/*
 * rdfft_pairs_to_halfcomplex / rdfft_halfcomplex_to_pairs -- in-place change of
 * the packed layout of `rows` spectra between the pairs layout above and the
 * paper's halfcomplex layout (Sec. 4.1, "Memory Layout"):
 *   halfcomplex: slot k = Re Y_k for 0 <= k <= n/2, slot n-k = Im Y_k for
 *                1 <= k < n/2
 * (so pair slot k, i.e. elements 2k and 2k+1, maps to elements k and n-k, and
 * pair slot 0 to elements 0 and n/2).  Values are moved bit for bit; NaN
 * payloads included.  rdfft_inverse expects the pairs layout, so a spectrum
 * converted to halfcomplex must be converted back before it is inverted (or
 * inverted with rdfft_inverse_halfcomplex).
 * Arguments and errors as rdfft_forward.
 */
RDFFT_API int rdfft_pairs_to_halfcomplex(void *buf, int64_t rows, int64_t n, rdfft_dtype_t dtype, rdfft_stream_t stream);
RDFFT_API int rdfft_halfcomplex_to_pairs(void *buf, int64_t rows, int64_t n, rdfft_dtype_t dtype, rdfft_stream_t stream);

/*
 * rdfft_forward_halfcomplex / rdfft_inverse_halfcomplex -- the in-place transforms
 * with the spectrum in the halfcomplex layout above (Sec. 4.1, Memory Layout) instead
 * of pairs: the forward leaves Re Y_k at element k and Im Y_k at element n-k, the
 * inverse reads them from there.  The results equal rdfft_forward followed by
 * rdfft_pairs_to_halfcomplex (and rdfft_halfcomplex_to_pairs followed by
 * rdfft_inverse) bit for bit, in one pass over the data instead of two.  Arguments
 * and errors as rdfft_forward.
 */
RDFFT_API int rdfft_forward_halfcomplex(void *buf, int64_t rows, int64_t n, rdfft_dtype_t dtype, rdfft_stream_t stream);
RDFFT_API int rdfft_inverse_halfcomplex(void *buf, int64_t rows, int64_t n, rdfft_dtype_t dtype, rdfft_stream_t stream);

/* Gradient outputs of bca_backward. */
typedef struct {
  void *dx;  /* [tokens][d_in] in dtype: dL/dx */
  float *dc; /* [q][kb][p] float32: dL/dc, time-domain first columns, OVERWRITTEN (not accumulated) */
} bca_grads_t;

/*
 * bca_forward -- block-circulant layer y = W x per token (Sec. 3.3; Eq. (4)
 * per block: y_i = IFFT( sum_j FFT(c_ij) . FFT(x_j) )).
 *   W is d_out x d_in, tiled into q x kb circulant blocks of size p
 *   (q = d_out/p, kb = d_in/p); block (i, j) is the circulant matrix whose
 *   first column is c_ij, C[m][r] = c_ij[(m - r) mod p], and maps input segment
 *   j of a token to output segment i.
 *   x          [tokens][d_in] in dtype, read only.
 *   c_spectra  [q][kb][p] in dtype, read only: row (i, j) is the packed
 *              spectrum (rdfft_forward of c_ij).
 *   y          [tokens][d_out] in dtype, written.  y == x is allowed when
 *              d_in == d_out (a truly in-place layer, Sec. 5.1.1); any other
 *              overlap with x or c_spectra -> RDFFT_EINVAL.
 *   grads      reserved, must be NULL.
 *   dtype      RDFFT_F32, RDFFT_BF16 or RDFFT_F16: the storage of x, c_spectra and y
 *              (float32 arithmetic; 16-bit stores round to nearest even).
 *   p          power of two, 2 <= p <= 65536 (larger -> RDFFT_EUNSUPPORTED);
 *              must divide d_in and d_out (Table 1 marks such shapes N/A) -> else RDFFT_EINVAL.
 *   tokens     >= 0; 0 is a no-op (x and y may then be NULL).
 * Blocks beyond 8192 (p = 16384, 32768, 65536) run as passes over HBM with q * kb <= 65535
 * (else RDFFT_EUNSUPPORTED).  With kb <= q and kb <= 8 they stage the input spectra in y;
 * other shapes add each input block's contribution into y's spectra, one pass per block.
 * Either way the intermediate spectra are stored in dtype (for 16-bit storage, one more
 * rounding of each staged spectrum, or of each of the kb partial sums).  In place
 * (y == x) they need q = kb <= 8 (else RDFFT_EUNSUPPORTED).
 */
RDFFT_API int bca_forward(const void *x, const void *c_spectra, void *y, bca_grads_t *grads, int64_t d_in,
                int64_t d_out, int64_t p, int64_t tokens, rdfft_dtype_t dtype, rdfft_stream_t stream);

/*
 * bca_backward -- gradients of the block-circulant layer (Sec. 3.3, Eq. (5)):
 *   dx_j  = IFFT( sum_i conj(FFT(c_ij)) . FFT(g_i) )          per token,
 *   dc_ij = IFFT( sum_t conj(FFT(x_{t,j})) . FFT(g_{t,i}) )   summed over tokens,
 * with g = dL/dy.
 *   x          [tokens][d_in] in dtype, read only.
 *   c_spectra  [q][kb][p] in dtype, read only (as bca_forward).
 *   gy         [tokens][d_out] in dtype: the upstream gradient.  Its contents
 *              are unspecified on return (the layer may use it as work space,
 *              Sec. 5.1.1 "overwriting the grad_output").
 *   grads->dx  [tokens][d_in] in dtype, written; may equal gy when d_in == d_out.
 *              Blocks beyond 8192 stage the input spectra in dx while gy holds the
 *              upstream ones; with dx == gy (q = kb <= 8 there, else RDFFT_EUNSUPPORTED)
 *              each token's input spectra go straight into float32 atomic sums of dc.
 *   grads->dc  [q][kb][p] float32, written (overwritten, not accumulated).
 *              Summed with float32 atomics, so the last bits may vary run to run.
 *   Other arguments as bca_forward.  tokens == 0 writes dc = 0.
 * Any other overlap between the buffers -> RDFFT_EINVAL.
 */
RDFFT_API int bca_backward(const void *x, const void *c_spectra, void *gy, bca_grads_t *grads, int64_t d_in,
                 int64_t d_out, int64_t p, int64_t tokens, rdfft_dtype_t dtype, rdfft_stream_t stream);

/*
 * bca_backward_keep -- bca_backward that only reads gy, for a caller whose upstream gradient
 * must survive and who would else pass a copy of it.  dx must not overlap gy; gy may
 * share memory with x.  p up to 8192 (longer blocks transform gy in place:
 * RDFFT_EUNSUPPORTED).  dc is always summed with float32 atomics (the staging of partial
 * sums that bca_backward does in gy is not open to it).  Otherwise as bca_backward.
 */
RDFFT_API int bca_backward_keep(const void *x, const void *c_spectra, const void *gy, bca_grads_t *grads, int64_t d_in,
                 int64_t d_out, int64_t p, int64_t tokens, rdfft_dtype_t dtype, rdfft_stream_t stream);

/*
 * bca_forward_batched / bca_backward_batched -- `count` independent layers of one shape
 * (the same d_in, d_out, p, tokens and dtype, each with its own tensors), such as the query
 * and value adapters of every layer of an encoder (Sec. 5.1.2), in one call.  Square layers
 * of 128 <= p <= 512 with q = kb <= 4 (the ones whose transforms fit a wavefront) run the
 * layers side by side in the same launches, which fills the chip where one layer alone
 * cannot; the backward does so when every dx is apart from its gy.  Other batches run
 * their layers one after another.  Results equal those of bca_forward / bca_backward on
 * each layer (dc up to the order of its float32 sums).
 *   count      0 <= count <= 1024 (0: no-op); else RDFFT_EINVAL.
 *   x, c_spectra, y / gy
 *              host arrays of `count` device pointers, entry b as the argument of the
 *              single-layer call for layer b.
 *   grads      host array of `count` bca_grads_t (backward only).
 * Within a layer the aliasing rules of the single-layer calls hold.  Across layers, buffers
 * that are only read may be shared (one x for several layers), but nothing a layer writes
 * (y; gy, dx, dc) may overlap any buffer of another layer -> RDFFT_EINVAL.  All layers are
 * checked before anything is enqueued.
 */
RDFFT_API int bca_forward_batched(int count, const void *const *x, const void *const *c_spectra, void *const *y,
                                  int64_t d_in, int64_t d_out, int64_t p, int64_t tokens, rdfft_dtype_t dtype,
                                  rdfft_stream_t stream);
RDFFT_API int bca_backward_batched(int count, const void *const *x, const void *const *c_spectra, void *const *gy,
                                   const bca_grads_t *grads, int64_t d_in, int64_t d_out, int64_t p, int64_t tokens,
                                   rdfft_dtype_t dtype, rdfft_stream_t stream);

/* -------------------------------------------------------------------------------------------
 * The operators around the adapter in a fine-tuned layer: activations kept for the backward pass
 * in 8 bits, layer norm, and the dense product that the adapter is added to.
 *
 * They share the conventions above, with these differences:
 * - Tensors of `dtype` are rows of consecutive elements with a row stride of their own (in
 *   elements, at least the row's length), and start at any multiple of the element's size; rows that
 *   start at multiples of 16 bytes are the fast case.  Nothing outside a row's elements is
 *   read or written.
 * - A checkpoint is contiguous: codes [rows][n] and scales [rows][ceil(n/32)].
 * - A call that needs scratch memory takes it from the caller (16-byte aligned; its size from the
 *   matching _workspace call).  Its contents need not be kept between calls.
 * - Sums, means and variances are float32.  Results do not depend on the order in which the
 *   device executes (no atomics).
 * - An output overlaps no input unless said otherwise -> RDFFT_EINVAL.
 */

/*
 * The 8-bit format.  32 consecutive values of a row (the last block of a row may be short) share a power of
 * two 2^e, the least one with max|x| <= 127 * 2^e and e >= -127.  A value is held as the int8 code
 * rint(x / 2^e) (half to even) and stands for code * 2^e; the block's scale is the byte e + 127.
 * A block with an infinity or a NaN has scale byte 255, codes 0, and stands for NaN throughout.
 * The error of a value is at most 2^(e-1), 1/126 of the block's largest |x| (down to 2^-121).
 * Where |x| is within 1 % of the largest number M of its type, code * 2^e can be the power of two past M: +-64 * 2^10
 * made into float16, +-64 * 2^122 into any other type.  It stands for +-M, so finite values come back finite.
 */
typedef struct {
  int8_t *codes;
  uint8_t *scales;
} act8_t;

/* act8_quantize / act8_dequantize -- rows x n values into their checkpoint, and back (the values
 * that it stands for, rounded to dtype: a checkpoint of larger numbers than float16 has becomes infinities
 * there).  n >= 1; rows == 0 is a no-op. */
RDFFT_API int act8_quantize(const void *x, int64_t ldx, const act8_t *to, int64_t rows, int64_t n, rdfft_dtype_t dtype,
                            rdfft_stream_t stream);
RDFFT_API int act8_dequantize(const act8_t *from, void *out, int64_t ldo, int64_t rows, int64_t n, rdfft_dtype_t dtype,
                              rdfft_stream_t stream);

/*
 * layer_norm_forward -- per row, u = x (+ residual), y = (u - mean(u)) * rstd * weight + bias with
 * rstd = (mean((u - mean(u))^2) + eps)^(-1/2).  1 <= n <= 16384 (more -> RDFFT_EUNSUPPORTED).
 *   residual   may be null.  weight, bias: float32 [n]; bias may be null.
 *   y          may be x or residual itself (same pointer and stride).
 *   mean, rstd float32 [rows], written; either may be null.
 *   checkpoint of u (of the float32 sum where there is a residual), written; codes null: none.
 *   eps        >= 0.
 */
typedef struct {
  const void *x;
  int64_t ldx;
  const void *residual;
  int64_t ldr;
  const float *weight;
  const float *bias;
  void *y;
  int64_t ldy;
  float *mean;
  float *rstd;
  act8_t checkpoint;
} layer_norm_forward_t;
RDFFT_API int layer_norm_forward(const layer_norm_forward_t *a, int64_t rows, int64_t n, float eps, rdfft_dtype_t dtype,
                                 rdfft_stream_t stream);

/*
 * layer_norm_backward -- with xh = (u - mean) * rstd, g = dy * weight:
 *   dx = rstd * (g - mean(g) - xh * mean(g * xh)), the gradient of x and of residual,
 *   dweight = sum over rows of dy * xh,  dbias = sum over rows of dy  (float32 [n], overwritten).
 *   u          x (+ residual), or with x null (and residual null) what the checkpoint stands for.
 *   mean, rstd as layer_norm_forward left them.
 *   dx         may be dy itself (same pointer and stride).
 * rows == 0 writes zeros into dweight and dbias.
 */
typedef struct {
  const void *dy;
  int64_t ldg;
  const void *x;
  int64_t ldx;
  const void *residual;
  int64_t ldr;
  act8_t checkpoint;
  const float *weight;
  const float *mean;
  const float *rstd;
  void *dx;
  int64_t ldd;
  float *dweight;
  float *dbias;
  void *workspace;
  int64_t workspace_bytes;
} layer_norm_backward_t;
/* bytes (0: none is needed), or a negative rdfft_status_t */
RDFFT_API int64_t layer_norm_backward_workspace(int64_t rows, int64_t n);
RDFFT_API int layer_norm_backward(const layer_norm_backward_t *a, int64_t rows, int64_t n, rdfft_dtype_t dtype,
                                  rdfft_stream_t stream);

typedef enum {
  RDFFT_ACT_NONE = 0,
  RDFFT_ACT_RELU = 1,
  RDFFT_ACT_GELU = 2, /* z * Phi(z), Phi the normal distribution function */
  RDFFT_ACT_SILU = 3  /* z / (1 + exp(-z)) */
} rdfft_activation_t;

/*
 * linear_forward -- per token z = W x + bias, y = act(z) + residual.
 *   x [tokens][d_in], w [d_out][d_in], bias [d_out] or null, residual [tokens][d_out] or null, all in dtype.
 *   y          [tokens][d_out]; may be residual itself (same pointer and stride).
 *   checkpoint of z (of its float32 value), written, for linear_backward; codes null: none.
 * Products of dtype's values are summed in float32 (matrix cores); y is rounded once.
 * d_in, d_out >= 1, at most 2^20, strides at most 2^21 (a single row's is not looked at), tokens at most 2^22 (more
 * -> RDFFT_EUNSUPPORTED).
 */
typedef struct {
  const void *x;
  int64_t ldx;
  const void *w;
  int64_t ldw;
  const void *bias;
  const void *residual;
  int64_t ldr;
  void *y;
  int64_t ldy;
  act8_t checkpoint;
  void *workspace;
  int64_t workspace_bytes;
} linear_forward_t;
/* bytes (0: none is needed), or a negative rdfft_status_t */
RDFFT_API int64_t linear_forward_workspace(int64_t d_in, int64_t d_out, int64_t tokens, rdfft_dtype_t dtype);
RDFFT_API int linear_forward(const linear_forward_t *a, int64_t d_in, int64_t d_out, int64_t tokens,
                             rdfft_activation_t act, rdfft_dtype_t dtype, rdfft_stream_t stream);

/*
 * linear_backward -- with dz = dy * act'(z), z being what the checkpoint stands for:
 *   dx = dz W (+ add),  dw = dz^T x,  db = sum over tokens of dz.
 * Each of dx, dw, db is computed if its pointer is not null.  (The residual's gradient is dy.)
 *   checkpoint unused (and may be null) for RDFFT_ACT_NONE.  A positive z of less than half its block's step is held as
 *              zero, where RDFFT_ACT_RELU has slope 0: of normal z 0.6 % of the values, which puts dz 0.11 of its norm
 *              off the gradient at z itself.  GELU's and SILU's slopes, which have no jump, are off by less than 0.01.
 *   x          needed for dw only, w for dx only.
 *   add        [tokens][d_in] or null: a gradient that reaches x another way; dx may be add itself
 *              (same pointer and stride).
 *   dw [d_out][d_in], db [d_out] in dtype, overwritten.
 * As an operand of the products dz is rounded to dtype (act != RDFFT_ACT_NONE); db sums the float32 dz.
 * tokens == 0 writes zeros into dw and db.
 */
typedef struct {
  const void *dy;
  int64_t ldg;
  act8_t checkpoint;
  const void *x;
  int64_t ldx;
  const void *w;
  int64_t ldw;
  const void *add;
  int64_t lda;
  void *dx;
  int64_t ldd;
  void *dw;
  int64_t lddw;
  void *db;
  void *workspace;
  int64_t workspace_bytes;
} linear_backward_t;
/* for the gradients that are wanted (nonzero) */
RDFFT_API int64_t linear_backward_workspace(int64_t d_in, int64_t d_out, int64_t tokens, int dx, int dw, int db,
                                            rdfft_activation_t act, rdfft_dtype_t dtype);
RDFFT_API int linear_backward(const linear_backward_t *a, int64_t d_in, int64_t d_out, int64_t tokens,
                              rdfft_activation_t act, rdfft_dtype_t dtype, rdfft_stream_t stream);

/* -------------------------------------------------------------------------------------------
 * The same around a decoder's layer: RMS norm, and the dense product of operands in 8-bit floating point.  The conventions
 * of the section above hold.
 */

/*
 * The 8-bit floating point format.  128 consecutive values of a row (the last block of a row may be short), or the values of
 * a tile of 128 x 128 (those at the edges may be smaller), share a power of two 2^e, the least one with
 * max|x| <= 448 * 2^e and e >= -127.  A value is held as x / 2^e rounded to e4m3 (half to even), and stands for
 * code * 2^e; the block's scale is the byte e + 127.  A block with an infinity or a NaN has scale byte 255 and NaN codes.
 * An operand of a product has its blocks along the direction that is summed over.
 *   codes      rows of n codes, `ld` bytes apart (at least n), each starting at a multiple of 16 bytes.
 *   scales     rows of ceil(n/128) bytes, `lds` apart (at least that), each starting at a multiple of 4 bytes.
 *              (Strides of a single row are not looked at.)
 *   block_rows 1: a row of scales for each row of codes; 128: one for 128 rows of codes (tiles).
 * What follows a row's last value up to the next multiple of 16 codes (4 scales) may be read, but is of no account; it is
 * never written.
 */
typedef struct {
  uint8_t *codes;
  int64_t ld;
  uint8_t *scales;
  int64_t lds;
  int64_t block_rows;
} fp8_t;

/* fp8_quantize -- x [rows][n] into its 8-bit form: `held` [rows][n] and `columns` [n][rows], of x's transpose, with
 * blocks along x's columns.  Either may be null; both have the same block_rows (of a single row either will do), and
 * with tiles the same values.
 * fp8_dequantize -- the values that it stands for, rounded to dtype.  code * 2^e that is the power of two past the
 * type's largest number M (of values within 1/32 of M) comes back as +-M.
 * rows == 0 is a no-op; n >= 1, in fp8_quantize at most 2^29 (more -> RDFFT_EUNSUPPORTED). */
RDFFT_API int fp8_quantize(const void *x, int64_t ldx, const fp8_t *held, const fp8_t *columns, int64_t rows, int64_t n,
                           rdfft_dtype_t dtype, rdfft_stream_t stream);
RDFFT_API int fp8_dequantize(const fp8_t *from, void *out, int64_t ldo, int64_t rows, int64_t n, rdfft_dtype_t dtype,
                             rdfft_stream_t stream);

/*
 * rms_norm_forward -- per row, u = x (+ residual) rounded to dtype, y = u * rstd * weight with
 * rstd = (mean(u^2) + eps)^(-1/2).  1 <= n <= 16384 (more -> RDFFT_EUNSUPPORTED).
 *   residual   may be null.  weight: float32 [n].
 *   y, y8      the result in dtype and in 8-bit floating point (block_rows 1, from the float32 value); codes null: none.
 *              Either may be null.
 *   summed     u, written; may be null.
 *   y, summed  may be x or residual (same pointer and stride), but not each other.
 *   rstd       float32 [rows], written; may be null.  (With an eps of 0, infinite where it is 2^128 or more; y and y8 are
 *              right there all the same.)
 *   checkpoint of u, written; codes null: none.
 *   eps        >= 0.
 */
typedef struct {
  const void *x;
  int64_t ldx;
  const void *residual;
  int64_t ldr;
  const float *weight;
  void *y;
  int64_t ldy;
  void *summed;
  int64_t lds;
  float *rstd;
  act8_t checkpoint;
  fp8_t y8;
} rms_norm_forward_t;
RDFFT_API int rms_norm_forward(const rms_norm_forward_t *a, int64_t rows, int64_t n, float eps, rdfft_dtype_t dtype,
                               rdfft_stream_t stream);

/*
 * rms_norm_backward -- with xh = u * rstd, g = dy * weight:
 *   dx = rstd * (g - xh * mean(g * xh)) (+ add), the gradient of x and of residual,
 *   dweight = sum over rows of dy * xh  (float32 [n], overwritten; may be null).
 *   u          the norm's input, or with u null what the checkpoint stands for.
 *   rstd       as rms_norm_forward left it; where it is infinite dx and dweight are not finite.
 *   add        the gradient that reaches the sum another way (the residual stream); may be null.
 *   dx         may be dy or add itself (same pointer and stride).
 * rows == 0 writes zeros into dweight.
 */
typedef struct {
  const void *dy;
  int64_t ldg;
  const void *u;
  int64_t ldu;
  act8_t checkpoint;
  const float *weight;
  const float *rstd;
  const void *add;
  int64_t lda;
  void *dx;
  int64_t ldd;
  float *dweight;
  void *workspace;
  int64_t workspace_bytes;
} rms_norm_backward_t;
/* bytes (0: none is needed), or a negative rdfft_status_t */
RDFFT_API int64_t rms_norm_backward_workspace(int64_t rows, int64_t n);
RDFFT_API int rms_norm_backward(const rms_norm_backward_t *a, int64_t rows, int64_t n, rdfft_dtype_t dtype,
                                rdfft_stream_t stream);

/*
 * linear_fp8_forward -- per token z = W x + bias, y = act(z) + residual, as linear_forward.
 *   x [tokens][d_in], w [d_out][d_in] in 8-bit floating point, of either block_rows each.
 *   bias [d_out], residual [tokens][d_out] (null: none) and y [tokens][d_out] in dtype; y may be residual itself.
 *   checkpoint of z (of its float32 value), written, for linear_fp8_backward; codes null: none.
 * Sums are float32.  For a 16-bit dtype the 8-bit matrix instructions drop what lies about 16 bits below the largest product
 * that they add (1.5e-5 of the result's norm for normal values).  That moves about one code in a thousand of the checkpoint to
 * the next, and the backward's gradients with it.  With RDFFT_F32 every product counts in full, and a large product takes a
 * little over three times as long.  Sizes as for linear_forward; strides at most 2^21.
 */
typedef struct {
  fp8_t x;
  fp8_t w;
  const void *bias;
  const void *residual;
  int64_t ldr;
  void *y;
  int64_t ldy;
  act8_t checkpoint;
  void *workspace;
  int64_t workspace_bytes;
} linear_fp8_forward_t;
/* bytes (0: none is needed), or a negative rdfft_status_t */
RDFFT_API int64_t linear_fp8_forward_workspace(int64_t d_in, int64_t d_out, int64_t tokens, rdfft_dtype_t dtype);
RDFFT_API int linear_fp8_forward(const linear_fp8_forward_t *a, int64_t d_in, int64_t d_out, int64_t tokens,
                                 rdfft_activation_t act, rdfft_dtype_t dtype, rdfft_stream_t stream);

/*
 * linear_fp8_backward -- with dz = dy * act'(z), z being what the checkpoint stands for:
 *   dx = dz W (+ add),  dw = dz^T x,  db = sum over tokens of dz.
 * dz enters the products in 8-bit floating point, in blocks of 128 along d_out for dx and along the tokens for dw (from
 * the float32 value); db sums the float32 dz.  Each of dx, dw, db is computed if its pointer is not null.
 *   x          [d_in][tokens], the columns that fp8_quantize leaves of x; for dw only.
 *   w          [d_in][d_out], the columns that it leaves of W; for dx only.
 *   the rest   as for linear_backward.
 */
typedef struct {
  const void *dy;
  int64_t ldg;
  act8_t checkpoint;
  fp8_t x;
  fp8_t w;
  const void *add;
  int64_t lda;
  void *dx;
  int64_t ldd;
  void *dw;
  int64_t lddw;
  void *db;
  void *workspace;
  int64_t workspace_bytes;
} linear_fp8_backward_t;
/* for the gradients that are wanted (nonzero) */
RDFFT_API int64_t linear_fp8_backward_workspace(int64_t d_in, int64_t d_out, int64_t tokens, int dx, int dw, int db,
                                                rdfft_dtype_t dtype);
RDFFT_API int linear_fp8_backward(const linear_fp8_backward_t *a, int64_t d_in, int64_t d_out, int64_t tokens,
                                  rdfft_activation_t act, rdfft_dtype_t dtype, rdfft_stream_t stream);

/* Uploads the twiddle table to the current device (synchronously) if not done yet.
 * Optional: every entry point does it on first use.  Returns RDFFT_OK or RDFFT_EDEVICE. */
RDFFT_API int rdfft_init(void);

/* Bytes of the static twiddle table held on each device the library has used. */
RDFFT_API int64_t rdfft_table_bytes(void);

/* Human-readable name of a status code (static string). */
RDFFT_API const char *rdfft_status_string(int status);

#ifdef __cplusplus
}
#endif

#endif /* RDFFT_H */
