/*
 * oq.h -- C ABI of the MI355X (gfx950) W4A4 rotated-linear library.
 *
 * The library implements the inference hot path of the paper's W4A4 linear
 * layer: the online Hadamard half of the composite rotation R = R_SVD . H
 * (Section 4.1, eq:composite_rot, block-wise form eq:blockdiag, transform
 * eq:transform), the per-step DiT activation scale (Section 4.2,
 * eq:perstep_scale), symmetric per-token int4 activation quantization
 * (eq:scale, eq:quant), the packed-int4 x int4 product with int32
 * accumulation and the per-token x per-channel dequantization
 * (eq:lowbit_linear), plus a DiT denoising-step driver built from them
 * (Experimental Settings, Implementation Details).
 *
 * Conventions for every entry point
 * ---------------------------------
 *  - Device pointers point to memory of the current HIP device; host
 *    pointers are marked "host".  The caller allocates and owns every buffer;
 *    the stateless calls allocate nothing.
 *  - `stream` is a hipStream_t passed as void* (NULL = the null stream).
 *    Calls are asynchronous on that stream; outputs are valid after the
 *    stream is synchronized.
 *  - Every call validates its arguments before launching anything; a call
 *    that returns an error has launched nothing and written nothing.
 *  - Return value: OQ_OK (0) or a negative oq_status.  No exception crosses
 *    the ABI.  oq_status_string() names a code.
 *  - Stateless calls are thread-safe.  A DiT handle is used from one host
 *    thread / one stream at a time.
 *
 * Data layout
 * -----------
 *  X      fp16 activation, row-major [M][ldx], K used channels per row.  It is
 *         the linear's input already expressed in the SVD basis: the SVD
 *         factor of the composite rotation is folded into the producer and
 *         the weight offline; only the Hadamard half runs online.
 *  Xq     packed int4 codes, row-major [M][K/2] bytes; byte k/2 of a row
 *         holds channel k (even) in its low nibble and channel k+1 in its
 *         high nibble, two's complement.  Codes lie in [-7, 7]; 0x8 never
 *         occurs (q_max = 2^(4-1) - 1 = 7, eq:quant).
 *  x_scale fp32 [M]: per-token dequantization step, Delta_i / s_t.
 *  Wq     packed int4 weight codes, [N][K/2] bytes, same nibble order; row n
 *         is output channel n (the weight is stored output-major, so
 *         Y = X' . W'^T).
 *  w_scale fp32 [N]: per-output-channel step Delta_W'.
 */
#ifndef OQ_H
#define OQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  OQ_OK = 0,
  OQ_ERR_NULL = -1,      /* a required pointer is NULL                              */
  OQ_ERR_SHAPE = -2,     /* a size is out of range or inconsistent (see each call)  */
  OQ_ERR_ALIGN = -3,     /* a pointer or leading dimension is not aligned            */
  OQ_ERR_DEVICE = -4,    /* the current device is not gfx950                        */
  OQ_ERR_HIP = -5,       /* a HIP runtime call or kernel launch failed              */
  OQ_ERR_WORKSPACE = -6, /* DiT workspace missing or too small                      */
  OQ_ERR_ARG = -7        /* another invalid argument (enum value, step index, ...)  */
} oq_status;

/* Output element type of the dequantizing epilogue, and element type of the
 * attention and cache operands (OQ_OUT_F32: outputs of oq_kv4_gather and of the
 * MX4 operators, and residual rows). */
typedef enum { OQ_OUT_F16 = 0, OQ_OUT_BF16 = 1, OQ_OUT_F32 = 2 } oq_out_dtype;

/* Largest Hadamard block the rotation kernel accepts. */
#define OQ_MAX_HAD_BLOCK 16384

/* Human-readable name of a status code (static storage, never NULL). */
const char* oq_status_string(int status);

/* Library version string (static storage). */
const char* oq_version(void);

/*
 * oq_check_device -- OQ_OK if the current HIP device is gfx950, else
 * OQ_ERR_DEVICE (or OQ_ERR_HIP if the runtime cannot be queried).  Every
 * launching call performs the same check once per device.
 */
int oq_check_device(void);

/*
 * oq_rotate_quantize_act -- online Hadamard rotation, step scale and
 * per-token int4 quantization of one activation (Section 4.1 eq:transform
 * with the block-diagonal Hadamard of eq:blockdiag; Section 4.2 eq:scale,
 * eq:quant; the per-step scale of eq:perstep_scale in its per-(layer, step)
 * scalar form).
 *
 * For each row i:  y = X[i, 0:K] . blockdiag(H_b) / sqrt(b)   (Sylvester
 * order, H[r][c] = (-1)^popcount(r & c), blocks of b contiguous channels);
 * z = s_t * y;  Delta_i = max_k |z_k| / 7;  q_k = clamp(round_half_even(
 * z_k / Delta_i), -7, 7);  x_scale[i] = Delta_i / s_t.  A row of zeros gives
 * zero codes and x_scale 0.  s_t = s_table[t] when s_table is not NULL, else
 * 1; it is read on the host when the call is made.
 *
 * X        device fp16 [M][ldx]
 * M        rows (tokens), >= 0 (0 is a no-op)
 * K        channels, multiple of 8 and of had_block, <= 16384; K/8 must be a
 *          power of two times 1 or 3 (every hidden size used here is)
 * ldx      row stride of X in elements, >= K, multiple of 8
 * had_block Hadamard block b: power of two, 1 <= b <= OQ_MAX_HAD_BLOCK, b | K
 * s_table  host fp32 table or NULL; t indexes it (t >= 0)
 * Xq       device [M][K/2] bytes;  x_scale device fp32 [M]
 * Pointers X, Xq must be 16-byte aligned; x_scale 4-byte aligned.
 * Errors: OQ_ERR_NULL, OQ_ERR_SHAPE, OQ_ERR_ALIGN, OQ_ERR_ARG (t < 0),
 * OQ_ERR_DEVICE, OQ_ERR_HIP.
 */
int oq_rotate_quantize_act(const void* X, int64_t M, int64_t K, int64_t ldx,
                           int32_t had_block, const float* s_table, int32_t t,
                           uint8_t* Xq, float* x_scale, void* stream);

/*
 * oq_rotate_debug_f32 -- same computation as oq_rotate_quantize_act, but
 * writes the pre-rounding ratio r = z / Delta_i of every element as fp32
 * [M][K] (row-major, contiguous) together with x_scale, so that a code that
 * differs from a reference can be classified as a rounding-boundary case.
 * Arguments and errors as above; ratio must be 16-byte aligned.
 */
int oq_rotate_debug_f32(const void* X, int64_t M, int64_t K, int64_t ldx,
                        int32_t had_block, const float* s_table, int32_t t,
                        float* ratio, float* x_scale, void* stream);

/*
 * oq_w4a4_linear -- int4 x int4 product with int32 accumulation and the
 * fused dequantization epilogue (eq:lowbit_linear; all scales folded into
 * the dequantization as in the Implementation Details).
 *
 * acc[i][n] = sum_k q[i][k] * wq[n][k]           (exact, int32)
 * Y[i][n]   = round_to_out(float(acc) * x_scale[i] * w_scale[n] + bias[n])
 *
 * Xq, x_scale  device, as produced by oq_rotate_quantize_act, [M][K/2], [M]
 * Wq, w_scale  device, [N][K/2], [N] (oq_quantize_weights* produce them)
 * bias         device fp16 [N] or NULL
 * M >= 0, N >= 1, K >= 64 with K % 64 == 0, K <= 16384
 * Y            device [M][ldy] of out_dtype (oq_out_dtype), ldy >= N, ldy % 8 == 0
 * Xq, Wq, Y 16-byte aligned.  Errors: OQ_ERR_NULL, OQ_ERR_SHAPE,
 * OQ_ERR_ALIGN, OQ_ERR_ARG (out_dtype), OQ_ERR_DEVICE, OQ_ERR_HIP.
 */
int oq_w4a4_linear(const uint8_t* Xq, const float* x_scale, int64_t M,
                   const uint8_t* Wq, const float* w_scale, const void* bias,
                   int64_t N, int64_t K, void* Y, int64_t ldy, int32_t out_dtype,
                   void* stream);

/*
 * oq_w4a4_gemm_i32 -- the integer product alone: acc[i][n] (int32) written
 * to device [M][ldc], ldc >= N, ldc % 4 == 0.  Shapes and errors as
 * oq_w4a4_linear.  For parity checks of the accumulators.
 */
int oq_w4a4_gemm_i32(const uint8_t* Xq, int64_t M, const uint8_t* Wq, int64_t N,
                     int64_t K, int32_t* acc, int64_t ldc, void* stream);

/*
 * 16-row tiled token codes.  With few tokens (the DiT's action tokens, decode)
 * the product of eq:lowbit_linear is bound by how fast every workgroup can
 * re-read the token codes; this layout makes each 16-byte-per-lane load of a
 * 16-row operand fragment one contiguous kilobyte.  It holds the same codes
 * as Xq (K % 128 == 0):
 *   rows padded to R16 = 16 * ceil(R / 16); total R16 * K / 2 bytes;
 *   packed byte p (0 <= p < K/2) of row r is stored at byte
 *   ((r / 16) * (K / 128) + p / 64) * 1024 + ((p / 16) % 4) * 256
 *     + (r % 16) * 16 + p % 16.
 * Bytes of padding rows are never read into a result (they may hold anything).
 */

/*
 * oq_codes_to_tiled -- re-layout of packed codes Q [rows][K/2] (device) into
 * the tiled layout T (device, R16 * K / 2 bytes; padding rows written as 0).
 * rows >= 0, 128 <= K <= 16384, K % 128 == 0; Q, T 16-byte aligned.
 * Errors: OQ_ERR_NULL, OQ_ERR_SHAPE, OQ_ERR_ALIGN, OQ_ERR_DEVICE, OQ_ERR_HIP.
 */
int oq_codes_to_tiled(const uint8_t* Q, int64_t rows, int64_t K, uint8_t* T, void* stream);

/*
 * oq_rotate_quantize_act_tiled -- oq_rotate_quantize_act (the same rotation,
 * step scale and quantizer, identical codes and x_scale) writing the codes
 * in the tiled layout: Xt device, R16 * K / 2 bytes with R = M (padding rows
 * are left untouched).  Additionally K % 128 == 0.  Arguments and errors as
 * oq_rotate_quantize_act.
 */
int oq_rotate_quantize_act_tiled(const void* X, int64_t M, int64_t K, int64_t ldx,
                                 int32_t had_block, const float* s_table, int32_t t,
                                 uint8_t* Xt, float* x_scale, void* stream);

/*
 * oq_w4a4_linear_tiled / oq_w4a4_gemm_i32_tiled -- oq_w4a4_linear and
 * oq_w4a4_gemm_i32 (same results, bit for bit) with the token codes Xt in the
 * tiled layout (R = M); Wq stays [N][K/2].  Additionally K % 128 == 0.  Meant
 * for M <= 64; larger M is computed correctly in row groups of 64 but
 * without the large-tile kernel of the row-layout calls.  Arguments and
 * errors as the row-layout calls.
 */
int oq_w4a4_linear_tiled(const uint8_t* Xt, const float* x_scale, int64_t M,
                         const uint8_t* Wq, const float* w_scale, const void* bias,
                         int64_t N, int64_t K, void* Y, int64_t ldy, int32_t out_dtype,
                         void* stream);
int oq_w4a4_gemm_i32_tiled(const uint8_t* Xt, int64_t M, const uint8_t* Wq, int64_t N,
                           int64_t K, int32_t* acc, int64_t ldc, void* stream);

/*
 * Full composite rotation (Section 4.1, "Block-wise Implementation";
 * eq:blockdiag, eq:transform) with block size c = 64: X' = X P R_hat, where
 * P permutes the channels (zigzag over the blocks by descending weight
 * energy) and R_hat = BlockDiag(R_1 .. R_{K/64}), R_b = U_b H_64 / 8, U_b the
 * left singular vectors of the block's weight rows.  Unlike the entry points
 * above (whose input is already in the SVD basis, so only the Hadamard half
 * runs online), the whole transform runs online here.
 *
 * oq_rotate_quantize_act_composite -- for each row i:
 *   (X P)[i][k] = X[i][perm[k]];  y[i][64b + j] = sum_r (X P)[i][64b + r] R_b[r][j];
 *   z = s_t y;  Delta_i = max|z| / 7;  q = round_half_even(z / Delta_i)
 *   (|q| <= 7);  x_scale[i] = Delta_i / s_t.
 * X        device fp16 [M][ldx], ldx >= K, ldx % 8 == 0, 16-byte aligned
 * K        multiple of 64, 64 <= K <= 16384
 * perm     device int32 [K], a permutation of 0 .. K-1, 16-byte aligned
 *          (entries outside 0 .. K-1 are clamped into range; the result is
 *          then unspecified but every access stays in bounds); or NULL: X is
 *          already in the permuted channel order (P folded into the
 *          producer of X, as U is for the Hadamard path), so (X P) = X and
 *          no gather is needed
 * Rt       device fp16 [K/64][64][64], block b column-major:
 *          Rt[b][j][r] = R_b[r][j] (oq_block_rotations_host writes it), 16-byte
 *          aligned.  The products are formed from these fp16 values exactly
 *          and summed in fp32.
 * s_table, t  as oq_rotate_quantize_act
 * Xq       device [M][K/2] codes (16-byte aligned), x_scale device fp32 [M]
 * Above K = 4096 (and at K = 4096 with perm NULL and M > 1024) the rows are
 * split into channel chunks whose workgroups exchange their partial row maxima
 * through the rows of Xq before they store their codes there, so Xq holds other
 * values while the call runs; calls with outputs of their own may overlap.  A
 * token scale written as NaN reports that a chunk's exchange did not complete
 * (never expected; the codes of that row are then unspecified).
 * Errors: OQ_ERR_NULL, OQ_ERR_SHAPE, OQ_ERR_ALIGN, OQ_ERR_ARG, OQ_ERR_DEVICE,
 * OQ_ERR_HIP.
 */
int oq_rotate_quantize_act_composite(const void* X, int64_t M, int64_t K, int64_t ldx,
                                     const int32_t* perm, const void* Rt, const float* s_table,
                                     int32_t t, uint8_t* Xq, float* x_scale, void* stream);

/*
 * oq_zigzag_permutation_host -- perm (host int32 [K]) from per-channel weight
 * energies ||W_{j,:}||^2 (host double [K]; for a weight stored [N][K] the sum
 * of squares of column j): channels sorted by descending energy (ties keep
 * the lower index first) and dealt to the K / block blocks in snake order --
 * sorted position i goes to round r = i / n_blocks and block i % n_blocks
 * (r even) or n_blocks - 1 - i % n_blocks (r odd), slot r; perm[b block + r]
 * is that channel.  Errors: OQ_ERR_NULL, OQ_ERR_SHAPE.
 */
int oq_zigzag_permutation_host(const double* energy, int64_t K, int32_t block, int32_t* perm);

/*
 * oq_block_rotations_host -- Rt (host fp16 [K/block][block][block], each block
 * column-major) = round_to_fp16(U_b H_block / sqrt(block)) from the row-major
 * host double factors U [K/block][block][block].  block a power of two
 * <= 4096 dividing K (the online kernel takes block 64).
 * Errors: OQ_ERR_NULL, OQ_ERR_SHAPE.
 */
int oq_block_rotations_host(const double* U, int64_t K, int32_t block, uint16_t* Rt);

/*
 * oq_quantize_weights_composite_host -- the weight side of eq:transform in the
 * output-major storage: W'[n] = (W[n] P) R_hat with the fp16 block matrices
 * Rt as given (the same values the activation side uses), in float64, then
 * per-output-channel RTN (eq:scale, eq:quant): Wq host [N][K/2], w_scale host
 * fp32 [N].  W_u host double [N][K] row-major, perm host int32 [K], Rt host
 * fp16 as above.  Runs on the calling thread's process (std::thread workers).
 * Errors: OQ_ERR_NULL, OQ_ERR_SHAPE, OQ_ERR_ARG (perm entry out of range).
 */
int oq_quantize_weights_composite_host(const double* W_u, int64_t N, int64_t K, int32_t block,
                                       const int32_t* perm, const uint16_t* Rt, uint8_t* Wq,
                                       float* w_scale);

/*
 * oq_quantize_weights -- offline weight preparation on the device: fold the
 * Hadamard half of the rotation into the weight and quantize it per output
 * channel with round-to-nearest (eq:transform W' = R^T W in the output-major
 * storage used here: row n of W' is row n of W_u times blockdiag(H_b)/sqrt(b);
 * eq:scale / eq:quant per output channel; the DiT-side RTN solver of the
 * Implementation Details).  W_u is the weight already expressed in the SVD
 * basis (the SVD factor folded offline), device fp16 [N][ldw].  Identical to
 * oq_rotate_quantize_act with s_t = 1 applied to the weight rows; writes Wq
 * [N][K/2] and w_scale [N].  Shapes, alignment and errors as
 * oq_rotate_quantize_act.
 */
int oq_quantize_weights(const void* W_u, int64_t N, int64_t K, int64_t ldw,
                        int32_t had_block, uint8_t* Wq, float* w_scale, void* stream);

/*
 * oq_quantize_weights_host -- the same weight preparation on the host in
 * float64 from a float64 weight (for weights that are not fp16-exact).
 * W_u host [N][K] row-major; Wq host [N][K/2]; w_scale host fp32 [N].
 * Runs synchronously on the calling thread.  Errors: OQ_ERR_NULL,
 * OQ_ERR_SHAPE.
 */
int oq_quantize_weights_host(const double* W_u, int64_t N, int64_t K, int32_t had_block,
                             uint8_t* Wq, float* w_scale);

/* ------------------------------------------------------------------------ */
/* Offline preparation of the composite-rotation weight on the GPU           */
/* (Section 4.1: zigzag P, per-block SVD factor U_b, R_b = U_b H_64 / 8,      */
/* fold and RTN)                                                              */
/* ------------------------------------------------------------------------ */
/*
 * The weight W is device fp16 [N][ldw] (row n = output channel n, K input
 * channels); block b is input channels perm[64 b .. 64 b + 63].  The steps
 * can be called one by one or through oq_prepare_weights_composite.
 *
 * oq_channel_energy -- energy[j] = sum_n W[n][j]^2 in fp64 (device [K]); a
 *   fixed summation order, so equal columns give equal energies.
 *   Errors: OQ_ERR_NULL, OQ_ERR_SHAPE, OQ_ERR_ALIGN, OQ_ERR_DEVICE, OQ_ERR_HIP.
 *
 * oq_zigzag_permutation -- perm (device int32 [K]) from device energies: the
 *   descending order of the energy (ties to the lower channel index) dealt
 *   to K / block blocks in snake order: sorted position i goes to round
 *   r = i / n_b and to block i mod n_b on even rounds, n_b - 1 - (i mod n_b)
 *   on odd rounds, slot r; perm[b * block + r] is the source channel.
 *   K % block == 0, K <= 65536.
 *
 * oq_block_svd -- for each block (block must be 64): U (device fp64
 *   [K/64][64][64], row-major, U_b[r][i]) holds the left singular vectors of
 *   W_b (64 x N, the block's input-channel rows) as columns, ordered by
 *   descending singular value (ties to the lower index), each column's
 *   largest-magnitude entry (the first on ties) positive; sigma2 (device fp64
 *   [K/64][64]) the squared singular values.  Computed as the eigenvectors of
 *   the fp64 Gram matrix W_b W_b^T by cyclic Jacobi in fp64; vectors of
 *   (numerically) repeated singular values, including a null space when
 *   N < 64, are an orthonormal basis of their eigenspace, not unique.
 *   perm entries out of [0, K) are clamped.
 *
 * oq_block_rotations -- Rt (device fp16 [K/64][64][64], column-major blocks:
 *   Rt[b][j][r] = R_b[r][j]) with R_b = U_b H_64 / 8 evaluated in fp64 and
 *   rounded once to fp16 (half to even): the operand of
 *   oq_rotate_quantize_act_composite.
 *
 * oq_prepare_weights_composite -- all of the above, then the fold and RTN:
 *   Wq, w_scale = oq_rotate_quantize_act_composite(W, perm, Rt) with s_t = 1
 *   (the weight rows rotated by P R_hat and quantized per output channel).
 *   perm device int32 [K]; Rt device [K/64][64][64] fp16, 16-byte aligned;
 *   Wq device [N][K/2]; w_scale device fp32 [N]; work device, 16-byte
 *   aligned, at least oq_prepare_weights_workspace_bytes(K) = 528 K bytes.
 *   ldw % 8 == 0 and W 16-byte aligned (the fold's row loads).
 *   Errors: OQ_ERR_NULL, OQ_ERR_SHAPE (K % 64, K > 16384, workspace),
 *   OQ_ERR_ALIGN, OQ_ERR_DEVICE, OQ_ERR_HIP.
 */
int oq_channel_energy(const void* W, int64_t N, int64_t K, int64_t ldw, double* energy,
                      void* stream);
int oq_zigzag_permutation(const double* energy, int64_t K, int32_t block, int32_t* perm,
                          void* stream);
int oq_block_svd(const void* W, int64_t N, int64_t K, int64_t ldw, const int32_t* perm,
                 int32_t block, double* U, double* sigma2, void* stream);
int oq_block_rotations(const double* U, int64_t K, int32_t block, uint16_t* Rt, void* stream);
size_t oq_prepare_weights_workspace_bytes(int64_t K);
int oq_prepare_weights_composite(const void* W, int64_t N, int64_t K, int64_t ldw,
                                 int32_t* perm, uint16_t* Rt, uint8_t* Wq, float* w_scale,
                                 void* work, size_t work_bytes, void* stream);

/* ------------------------------------------------------------------------ */
/* W4A8: 8-bit per-token activations against the int4 weights (the paper's   */
/* deployment mode, Appendix: W4A8 real-quantization latency)                */
/* ------------------------------------------------------------------------ */
/*
 * oq_rotate_quantize_act_i8 -- oq_rotate_quantize_act with the symmetric
 * quantizer at 8 bits (eq:scale, eq:quant with k = 8): Delta_i = max|z_i| /
 * 127, codes in [-127, 127] (-128 never occurs), one signed byte per code.
 * Xq8 device int8 [M][K] row-major, 16-byte aligned; x_scale as before.
 * Arguments, limits and errors as oq_rotate_quantize_act.
 */
int oq_rotate_quantize_act_i8(const void* X, int64_t M, int64_t K, int64_t ldx,
                              int32_t had_block, const float* s_table, int32_t t,
                              int8_t* Xq8, float* x_scale, void* stream);

/*
 * oq_w4a8_linear / oq_w4a8_gemm_i32 -- oq_w4a4_linear / oq_w4a4_gemm_i32 with
 * the token operand in 8-bit codes (Xq8 [M][K], as written by
 * oq_rotate_quantize_act_i8) and the weight unchanged (packed int4 [N][K/2]):
 * acc[i][n] = sum_k q8[i][k] * wq[n][k] exactly in int32 (|acc| <= 889 K),
 * then the same epilogue.  Shapes, alignment and errors as the W4A4 calls.
 */
int oq_w4a8_linear(const int8_t* Xq8, const float* x_scale, int64_t M,
                   const uint8_t* Wq, const float* w_scale, const void* bias,
                   int64_t N, int64_t K, void* Y, int64_t ldy, int32_t out_dtype,
                   void* stream);
int oq_w4a8_gemm_i32(const int8_t* Xq8, int64_t M, const uint8_t* Wq, int64_t N, int64_t K,
                     int32_t* acc, int64_t ldc, void* stream);

/* ------------------------------------------------------------------------ */
/* W8A8: 8 bits on both sides, for linears that 4-bit weights cost too much    */
/* ------------------------------------------------------------------------ */
/*
 * oq_quantize_weights_i8 -- oq_quantize_weights at 8 bits (eq:scale, eq:quant
 * with k = 8): Wq8 device int8 [N][K] in [-127, 127], 16-byte aligned, w_scale
 * fp32 [N] = max / 127.  Identical to oq_rotate_quantize_act_i8 with s_t = 1 on
 * the weight's rows; arguments, limits and errors as there.
 */
int oq_quantize_weights_i8(const void* W_u, int64_t N, int64_t K, int64_t ldw, int32_t had_block,
                           int8_t* Wq8, float* w_scale, void* stream);

/*
 * oq_w8a8_linear / oq_w8a8_gemm_i32 -- the W4A8 calls with the weight in 8-bit
 * codes [N][K] too: acc[i][n] = sum_k q8[i][k] * wq8[n][k] exactly in int32
 * (any int8 codes: |acc| <= 2^14 K <= 2^28), Y[i][n] = round_to_out(float(acc) *
 * x_scale[i] * w_scale[n] + bias[n]).  Shapes, alignment and errors as the W4A4
 * calls.
 */
int oq_w8a8_linear(const int8_t* Xq8, const float* x_scale, int64_t M,
                   const int8_t* Wq8, const float* w_scale, const void* bias,
                   int64_t N, int64_t K, void* Y, int64_t ldy, int32_t out_dtype,
                   void* stream);
int oq_w8a8_gemm_i32(const int8_t* Xq8, int64_t M, const int8_t* Wq8, int64_t N, int64_t K,
                     int32_t* acc, int64_t ldc, void* stream);

/* ------------------------------------------------------------------------ */
/* Linears in microscaled 4-bit floating point, and what stands between them  */
/* ------------------------------------------------------------------------ */
/*
 * MX4 codes: blocks of 32 channels of a row share a step 2^s, s =
 * floor(log2 max|y|) - 2 clamped to [-127, 127] (0: -127); a channel's code is y /
 * 2^s rounded to the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 (ties to the even
 * code, past 6: 6), its index in bits 0 .. 2 and the sign in bit 3.  Unlike the
 * int4 codes above they need no step per token and channel in an epilogue: the
 * matrix cores take the steps.
 *   codes  uint8 [rows][K / 2], the even channel in the low nibble;
 *   steps  uint8 [rows][oq_mx4_step_bytes(K)], byte b of a row s + 127 of its
 *          channels 32 b .. 32 b + 31, 255: an infinity or a NaN among them (its
 *          codes are 0 and its values NaN).  The bytes of a row past K / 32 are
 *          neither written nor used.
 * K % 32 == 0, 32 <= K <= OQ_MX4_MAX_K; codes and steps 16-byte aligned.
 * The producers' codes are those of their formulas in 64 bits; a ratio within
 * about 2^-45 of a border between two codes may go either way.
 */
#define OQ_MX4_MAX_K 65536

/* Bytes from one row's steps to the next: 16 ceil(K / 512). */
size_t oq_mx4_step_bytes(int64_t K);

/*
 * oq_mx4_quantize -- codes and steps of rows of activations or weights, rotated
 * first if wanted: y = x . blockdiag(H_b) / sqrt(b) in blocks of b = had_block
 * channels (as oq_rotate_quantize_act; the two operands of a product need the
 * same b).
 * X         device fp16 or bf16 (dtype) [M][ldx], ldx >= K, % 8 == 0, 16-byte aligned
 * had_block 1 (none), 32, 64 or 128, dividing K
 * Xq, steps device, as above; may not overlap X
 * Errors: OQ_ERR_NULL, OQ_ERR_SHAPE, OQ_ERR_ALIGN, OQ_ERR_ARG, OQ_ERR_DEVICE,
 * OQ_ERR_HIP.
 */
int oq_mx4_quantize(const void* X, int64_t M, int64_t K, int64_t ldx, int32_t dtype, int32_t had_block,
                    uint8_t* Xq, uint8_t* steps, void* stream);

/*
 * oq_mx4_dequantize -- the values of rows of codes, X device [M][ldx] of
 * out_dtype (fp16, bf16, fp32; ldx >= K, % 8 == 0, 16-byte aligned).  fp32 and
 * bf16 hold every value but 3, 4 and 6 times 2^127 (infinite); fp16 rounds.
 * A rotation is not undone.  Errors as oq_mx4_quantize.
 */
int oq_mx4_dequantize(const uint8_t* Xq, const uint8_t* steps, int64_t M, int64_t K, void* X, int64_t ldx,
                      int32_t out_dtype, void* stream);

/*
 * oq_mx4_linear -- Y[i][n] = round_to_out(sum_k x[i][k] w[n][k] + bias[n]), x and
 * w the values of the codes, products exact and sums in fp32.
 * Xq, x_steps  device, [M] rows of K codes;  Wq, w_steps  device, [N] rows
 * bias         device fp16 [N] or NULL
 * M >= 0, N >= 1
 * Y            device [M][ldy] of out_dtype (fp16, bf16, fp32), ldy >= N, % 8 == 0,
 *              16-byte aligned; may not overlap the operands
 * A block with byte 255 makes its row's (column's) outputs NaN, no others.
 * Errors as oq_mx4_quantize.
 */
int oq_mx4_linear(const uint8_t* Xq, const uint8_t* x_steps, int64_t M, const uint8_t* Wq, const uint8_t* w_steps,
                  const void* bias, int64_t N, int64_t K, void* Y, int64_t ldy, int32_t out_dtype, void* stream);

/*
 * oq_gated_activation -- h = act(g) u of rows [g | u] as a gate|up linear writes
 * them, act(g) = g / (1 + e^-t), t = g (SiLU) or 2 sqrt(2 / pi) (g + 0.044715 g^3)
 * (GELU in its tanh form), in 16 bits or as the codes of the next linear.  (16 bits:
 * where e^-t is past 2^270, and no finite u makes half the smallest number of act(g) u, act(g)
 * counts as 0.)
 * GU       device fp16 or bf16 (dtype) [M][ld], g in columns 0 .. F - 1, u in F ..
 *          2 F - 1; ld >= 2 F, % 8 == 0, 16-byte aligned
 * F        % 8 == 0 (codes: % 32), 8 <= F <= OQ_MX4_MAX_K
 * H        device [M][ldh] of dtype (ldh >= F, % 8 == 0, 16-byte aligned), or NULL
 *          and Hq, steps: device codes of h (not rounded to dtype first)
 * Outputs may not overlap GU.  Errors as oq_mx4_quantize (OQ_ERR_ARG: act, both outputs).
 */
typedef enum { OQ_ACT_GELU_TANH = 0, OQ_ACT_SILU = 1 } oq_act;
int oq_gated_activation(const void* GU, int64_t M, int64_t F, int64_t ld, int32_t dtype, int32_t act, void* H,
                        int64_t ldh, uint8_t* Hq, uint8_t* steps, void* stream);

/*
 * oq_residual_norm -- the residual stream between two blocks, in one pass:
 *   r' = alpha R + gate[g] * post(Y),   h = pre(r') * (1 + scale[g]) + shift[g]
 * with post and pre each none, RMSNorm x / sqrt(mean(x^2) + eps) * gain + bias or
 * LayerNorm (x - mean) / sqrt(var + eps) * gain + bias (var of D values), and h
 * formed from the unrounded r'.
 * R        device [M][ldr] of r_dtype (fp32, or dtype), or NULL: 0
 * Y        device [M][ldy] of dtype (fp16 or bf16), the block's output, or NULL: 0
 * post     host, or NULL: none (y as it is)
 * pre      host, or NULL: none (no h)
 * gate, scale, shift  device [n_mod][ld_mod] of dtype, each may be NULL (1, 0, 0);
 *          ld_mod >= D, % 8 == 0 (so that they may be parts of one modulation row)
 * mod_row  device int32 [M]: row of these for each token (out of range: the
 *          token's outputs are left as they were), or NULL: row 0; without any of
 *          the three it is not used
 * R_out    device [M][ldro] of r_dtype, may be R (with ldro = ldr), or NULL: not wanted
 * H        device [M][ldh] of dtype, may be Y (with ldh = ldy), or NULL and Hq,
 *          steps: device MX4 codes of h (not rounded to dtype first)
 * D % 8 == 0 (codes: % 32), 8 <= D <= OQ_NORM_MAX_D; strides >= D, % 8 == 0; alpha
 * finite; pointers 16-byte aligned.  Other overlaps of outputs are not allowed.
 * Sums are fp32 over at most 32 values of a thread and fp64 beyond (finite if the values are
 * below 2^60 in magnitude); with codes all fp64.
 * Errors: as oq_mx4_quantize (OQ_ERR_ARG: kind, eps, alpha, h without pre, both
 * outputs; OQ_ERR_NULL: neither R nor Y, or no output).
 */
#define OQ_NORM_MAX_D 16384
typedef enum { OQ_NORM_NONE = 0, OQ_NORM_RMS = 1, OQ_NORM_LAYER = 2 } oq_norm_kind;
typedef struct {
  int32_t kind;      /* oq_norm_kind */
  float eps;         /* > 0, <= 1 */
  float gain_offset; /* the gain is gain_offset + gain (1 for gains stored about 0) */
  const void* gain;  /* device [D] of dtype, 16-byte aligned, or NULL: 1 */
  const void* bias;  /* device [D] of dtype, 16-byte aligned, or NULL: 0 */
} oq_norm;
int oq_residual_norm(const void* R, int64_t ldr, int32_t r_dtype, const void* Y, int64_t ldy, int32_t dtype,
                     int64_t M, int64_t D, const oq_norm* post, const oq_norm* pre, float alpha,
                     const void* gate, const void* scale, const void* shift, int64_t ld_mod, int64_t n_mod,
                     const int32_t* mod_row, void* R_out, int64_t ldro, void* H, int64_t ldh, uint8_t* Hq,
                     uint8_t* steps, void* stream);

/* ------------------------------------------------------------------------ */
/* Attention over packed prompts                                             */
/* ------------------------------------------------------------------------ */
/*
 * oq_attention_prompt -- softmax self-attention within each of n_seqs sequences
 * packed one behind the other: for token i of a sequence
 *   o_i = sum_j softmax_j(scale q_i . k_j) v_j
 * over its sequence's tokens j, with causal those up to i; query head h reads
 * kv head h / (n_heads / n_kv_heads).
 * Q, K, V  device fp16 or bf16 (dtype) [tokens][ldq / ldk / ldv], head h at columns
 *          h d .. of a row (so the three parts of a q|k|v linear's output serve
 *          as they lie); strides % 8 == 0 and at least heads * d; 16-byte aligned
 * cu_seqlens device int32 [n_seqs + 1], not decreasing: sequence s is rows
 *          cu_seqlens[s] .. cu_seqlens[s + 1] - 1 (clamped to [0, tokens]); rows
 *          of no sequence are left as they were, and what they hold is not used
 * head_dim d: 64, 128 or 256;  n_heads a multiple of n_kv_heads, n_heads <= 65535
 * scale    > 0, scale log2(e) finite
 * O        device [tokens][ldo] of dtype, ldo % 8 == 0; may not overlap Q, K, V
 * Probabilities are rounded to dtype for the second product (fp16: normal numbers
 * down to 2^-29 of a row's largest); sums and statistics are fp32.  Q, K and V of the
 * sequences' rows are finite, and so are their products q . k in fp32: one that is not may
 * show in any row of its sequence, and in no other sequence.  About tokens / 128 + n_seqs workgroups a head, of 2^32
 * threads at most together (OQ_ERR_SHAPE).
 * Errors: OQ_ERR_NULL, OQ_ERR_SHAPE, OQ_ERR_ALIGN, OQ_ERR_ARG, OQ_ERR_DEVICE,
 * OQ_ERR_HIP.
 */
int oq_attention_prompt(const void* Q, const void* K, const void* V, int64_t tokens, int64_t ldq,
                        int64_t ldk, int64_t ldv, int32_t dtype, const int32_t* cu_seqlens,
                        int32_t n_seqs, int32_t n_heads, int32_t n_kv_heads, int32_t head_dim,
                        int32_t causal, float scale, void* O, int64_t ldo, void* stream);

/* ------------------------------------------------------------------------ */
/* Static per-step, per-channel activation steps (Section 4.2,               */
/* eq:perstep_scale with the per-(layer, step, channel) table)               */
/* ------------------------------------------------------------------------ */
/*
 * The table holds Delta_{l,t,j} = sigma_hat(X'_{t,:,j}) / q_max for the
 * rotated activation X' of layer l at denoising step t, sigma_hat the
 * nearest-rank 99.9th percentile of the magnitudes over the calibration rows.
 * At inference the codes are q = clamp(round(y_j / Delta_j), -7, 7) (clipping
 * is live; round half to even) and the token scale is 1.  A per-channel step
 * cannot leave the sum over channels, so it is folded into the weight's input
 * channels per step: W''[n][j] = W'[n][j] Delta_j, quantized per output
 * channel (one weight copy per (layer, step)); the products are then the
 * ordinary oq_w4a4_linear / _tiled calls with x_scale = 1.
 */

/*
 * oq_rotate_act_f32 -- the rotated activation of eq:transform alone:
 * Y[i][k] = (x_i H_b / sqrt(b))[k] in fp32, Y device [M][K] contiguous,
 * 16-byte aligned (the calibration input of oq_calibrate_step_scales).
 * Arguments and shape limits as oq_rotate_quantize_act.  Errors: OQ_ERR_NULL,
 * OQ_ERR_SHAPE, OQ_ERR_ALIGN, OQ_ERR_DEVICE, OQ_ERR_HIP.
 */
int oq_rotate_act_f32(const void* X, int64_t M, int64_t K, int64_t ldx, int32_t had_block,
                      float* Y, void* stream);

/*
 * oq_calibrate_workspace_bytes -- device workspace needed by
 * oq_calibrate_step_scales for K channels (K * 1032 bytes).
 */
size_t oq_calibrate_workspace_bytes(int64_t K);

/*
 * oq_calibrate_step_scales -- delta[j] = v_j / qmax, v_j the nearest-rank
 * p-th percentile of |Y[:, j]| over the n rows: the k-th smallest magnitude
 * with k = ceil(p n / 100) clamped to [1, n], p taken to 1e-6 percent and
 * the product formed in integers (p = 99.9, n = 1000 gives k = 999, not the
 * maximum).  v_j is exact (an element of the column; selection over the bit
 * patterns, NaN ordered above +inf); the division is done in double and
 * rounded once to fp32.
 * Y device fp32 [n][ldy]; delta device fp32 [K]; work device, 16-byte
 * aligned, at least oq_calibrate_workspace_bytes(K) bytes, owned by the
 * caller and overwritten (calls that share it must not overlap).
 * p in (0, 100]; qmax > 0 (7 for int4 codes).
 * Errors: OQ_ERR_NULL, OQ_ERR_SHAPE (n == 0 with K > 0, ldy < K, workspace
 * too small), OQ_ERR_ARG (p, qmax), OQ_ERR_ALIGN, OQ_ERR_DEVICE, OQ_ERR_HIP.
 */
int oq_calibrate_step_scales(const float* Y, int64_t n, int64_t K, int64_t ldy, double p,
                             float qmax, float* delta, void* work, size_t work_bytes,
                             void* stream);

/*
 * oq_calibrate_step_scales_noalloc -- for callers that cannot allocate device
 * memory (code under HIP graph capture, tight serving loops, harnesses that
 * forbid hipMalloc): the same computation and results as
 * oq_calibrate_step_scales, bit for bit, with no workspace argument.  The
 * histogram, prefixes and ranks live in a device array inside the library
 * (16.9 MB per GPU, held until the process ends; its address is looked up
 * once per device on the first call with that device current).  The call
 * allocates nothing and clears what must start at zero with a kernel.
 * K <= 16384 columns; a larger K returns OQ_ERR_WORKSPACE and writes nothing.
 * The stream must belong to the current device.  Every call on one GPU
 * shares that GPU's array: calls that overlap on one GPU (other streams or
 * threads) race and must be serialized by the caller.
 * Errors: as oq_calibrate_step_scales, and OQ_ERR_WORKSPACE for K > 16384.
 */
int oq_calibrate_step_scales_noalloc(const float* Y, int64_t n, int64_t K, int64_t ldy, double p,
                                     float qmax, float* delta, void* stream);

/*
 * oq_rotate_quantize_act_static -- Hadamard rotation (as
 * oq_rotate_quantize_act) followed by the static quantizer with the step row
 * delta (device fp32 [K], 16-byte aligned: the table's row for this layer
 * and step): Xq[i][k] = clamp(round(y_ik / delta[k]), -7, 7), x_scale[i] = 1.
 * A channel whose step is zero, negative, NaN or infinite gets code 0.  The
 * ratio is formed in fp32 with the hardware reciprocal of delta (about one
 * ulp), so only ratios within a few ulps of a half integer can round
 * differently from exact arithmetic.
 * Errors: as oq_rotate_quantize_act; OQ_ERR_NULL (delta), OQ_ERR_ALIGN.
 */
int oq_rotate_quantize_act_static(const void* X, int64_t M, int64_t K, int64_t ldx,
                                  int32_t had_block, const float* delta, uint8_t* Xq,
                                  float* x_scale, void* stream);

/* The same with the codes in the 16-row tiled layout (K % 128 == 0). */
int oq_rotate_quantize_act_static_tiled(const void* X, int64_t M, int64_t K, int64_t ldx,
                                        int32_t had_block, const float* delta, uint8_t* Xt,
                                        float* x_scale, void* stream);

/*
 * oq_quantize_weights_step_host -- oq_quantize_weights_host with the step
 * folded in: row n of the quantized weight is RTN(W'[n][:] * delta[:]),
 * W' = W_u rotated by H_b / sqrt(b), in float64.  delta host fp32 [K], every
 * entry finite and >= 0.  Errors: OQ_ERR_NULL, OQ_ERR_SHAPE, OQ_ERR_ARG.
 */
int oq_quantize_weights_step_host(const double* W_u, int64_t N, int64_t K, int32_t had_block,
                                  const float* delta, uint8_t* Wq, float* w_scale);

/*
 * oq_quantize_weights_step -- the same fold on the device from an fp16
 * weight (as oq_quantize_weights, with channel j of each rotated row
 * multiplied by delta[j] before the row's maximum), in fp32.  delta device
 * fp32 [K], 16-byte aligned.  Errors: as oq_quantize_weights; OQ_ERR_NULL
 * (delta), OQ_ERR_ALIGN.
 */
int oq_quantize_weights_step(const void* W_u, int64_t N, int64_t K, int64_t ldw, int32_t had_block,
                             const float* delta, uint8_t* Wq, float* w_scale, void* stream);

/* ------------------------------------------------------------------------ */
/* Key/value cache in 4 bits (the per-token quantizer of eq:scale, eq:quant   */
/* on the rows of a backbone's keys and values), and attention over it         */
/* ------------------------------------------------------------------------ */
/*
 * A row is one token and kv head, head_dim channels x.  Its codes are q =
 * clamp(round_half_even(7 x / max|x|), -7, 7) (formed exactly: a quotient on a
 * half integer rounds to even, none beside one goes the wrong way; but in rotated bf16
 * rows whose nonzero elements span more than 2^34 one within 2^-42 of it may), its step
 * fp32 Delta = max|x| / 7, and the value it stands for q Delta; a row of
 * zeros has zero codes and step 0.  With rotate_k the keys are rotated first,
 * x = k H_d / sqrt(d) (d = head_dim, one Hadamard block per head); attention
 * then rotates its queries alike (q . k is unchanged) and oq_kv4_gather rotates
 * back.  A rotation of the values folds into the value and output projections.
 *
 * All buffers are the caller's.  Pages of page_tokens tokens:
 *   k_codes [n_pages][n_kv_heads][page_tokens][d / 2]: byte b of a row holds
 *     channel 2 b in its low nibble and 2 b + 1 in its high one (Xq's packing);
 *   v_codes [n_pages][n_kv_heads][page_tokens / 16][d / 2][16]: byte (b, t)
 *     holds channels 2 b and 2 b + 1 of token t of the 16;
 *   k_scale, v_scale fp32 [n_pages][n_kv_heads][page_tokens].
 * A slot is page * page_tokens + the token's place in the page.
 * head_dim 64, 128 or 256; page_tokens a multiple of 16, <= 65536; n_pages >= 1,
 * < 2^31; n_kv_heads 1 .. 65535; all four pointers 16-byte aligned.
 */
typedef struct {
  uint8_t* k_codes;
  uint8_t* v_codes;
  float* k_scale;
  float* v_scale;
  int64_t n_pages;
  int32_t page_tokens;
  int32_t n_kv_heads;
  int32_t head_dim;
  int32_t rotate_k; /* 0 or 1 */
} oq_kv4_cache;

/*
 * oq_kv4_append -- quantize n tokens' keys and values into their slots.
 * K, V     device fp16 or bf16 (dtype) [n][ldk], [n][ldv], head h of a token at
 *          columns h d .. h d + d - 1; ldk, ldv >= n_kv_heads d, % 8 == 0;
 *          16-byte aligned
 * slots    device int64 [n]: slot of each token; a slot below 0 or past the
 *          cache is skipped (padding tokens).  A slot may occur once in a call;
 *          of a repeated one the cache holds one of its tokens' bytes each.
 * Other slots are left as they were.  Input is finite.
 * Errors: OQ_ERR_NULL, OQ_ERR_SHAPE, OQ_ERR_ALIGN, OQ_ERR_ARG, OQ_ERR_DEVICE,
 * OQ_ERR_HIP.
 */
int oq_kv4_append(const oq_kv4_cache* cache, const void* K, const void* V, int64_t n, int64_t ldk,
                  int64_t ldv, int32_t dtype, const int64_t* slots, void* stream);

/*
 * oq_kv4_gather -- the values of n slots as dense rows (fp16, bf16 or fp32 by
 * dtype): K, V device [n][ldk], [n][ldv], laid out as oq_kv4_append's input;
 * keys in the basis in which they were appended.  A slot out of range gives
 * zeros.  For callers that need dense keys and values, as the prefix of
 * oq_dit_block (P slots give its prefix_k and prefix_v).
 * Errors: as oq_kv4_append.
 */
int oq_kv4_gather(const oq_kv4_cache* cache, const int64_t* slots, int64_t n, void* K, void* V,
                  int64_t ldk, int64_t ldv, int32_t dtype, void* stream);

/*
 * oq_attention_kv4 -- softmax attention of packed query tokens over a paged
 * cache: for sequence b with L = seq_lens[b] cached tokens and n query tokens
 * i = 0 .. n - 1 (its last n, whose keys are already in the cache),
 *   o_i = sum_j softmax_j(scale q_i . k_j) v_j,  j < L, and with causal
 *   j <= L - n + i
 * per query head; head h reads kv head h / (n_heads / n_kv_heads).  A query that
 * sees no key gives zeros.  One token per sequence is decoding; several are a
 * chunk of a prompt or a draft to verify.
 * Q        device fp16 / bf16 (dtype) [tokens][ldq], head h at columns h d ..;
 *          ldq >= n_heads d, % 8 == 0, 16-byte aligned.  O likewise (dtype, ldo); O may
 *          not overlap Q or the cache
 * cu_q     device int32 [n_seqs + 1]: sequence b's query tokens are rows
 *          cu_q[b] .. cu_q[b + 1] - 1; NULL: one each (tokens == n_seqs,
 *          max_q == 1).  Rows that no sequence has, and those past the first
 *          max_q of one, are left as they were.
 * max_q    1 .. 65535, at least the most query tokens of a sequence
 * block_table  device int32 [n_seqs][table_ld]: page of each page_tokens tokens
 *          of a sequence; tokens of an entry out of range are masked
 * seq_lens device int32 [n_seqs]; clamped to [0, max_len]
 * max_len  0 .. 2^30, at least the longest sequence; table_ld page_tokens >= max_len.
 *          It plans the split over the length: a tight one is faster.
 * scale    > 0, scale log2(e) finite
 * work     device, 16-byte aligned, at least oq_attention_kv4_workspace_bytes(the
 *          same sizes) bytes (0: may be NULL), written before it is read;
 *          calls that share it must not overlap
 * n_seqs n_kv_heads <= 65535, n_heads <= 65535, max_q n_heads / n_kv_heads <= 2^26.
 * Keys, steps and values past a sequence's end are not used, whatever they hold.
 * Queries are used as fp16 times a power of two (rotated ones as two such parts). A score's
 * fp32 sum starts at 72 sum(q) in units of the key's step, so its rounding is relative to 80
 * sum |q| of them; scores are finite in fp32. Probabilities are used as fp16 relative to the
 * largest contribution (a probability times a step; normal numbers down to 2^-29 of it, but
 * not below 2^-140), sums and statistics in fp32.
 * Errors: OQ_ERR_NULL, OQ_ERR_SHAPE, OQ_ERR_ALIGN, OQ_ERR_ARG,
 * OQ_ERR_WORKSPACE, OQ_ERR_DEVICE, OQ_ERR_HIP.
 */
size_t oq_attention_kv4_workspace_bytes(const oq_kv4_cache* cache, int64_t tokens, int32_t n_heads,
                                        int32_t n_seqs, int32_t max_q, int32_t max_len);
int oq_attention_kv4(const oq_kv4_cache* cache, const void* Q, int64_t tokens, int64_t ldq,
                     int32_t n_heads, int32_t dtype, const int32_t* cu_q, int32_t max_q,
                     const int32_t* block_table, int64_t table_ld, const int32_t* seq_lens,
                     int32_t n_seqs, int32_t max_len, int32_t causal, float scale, void* O,
                     int64_t ldo, void* work, size_t work_bytes, void* stream);

/* ------------------------------------------------------------------------ */
/* DiT denoising-step driver                                                 */
/* ------------------------------------------------------------------------ */

/*
 * One denoising step of a DiT action head whose every block linear is a
 * rotated W4A4 linear (Experimental Settings: W4A4 on all linears, RTN
 * weights and the per-step activation scale table on the DiT side, Euler
 * denoising steps).  Block structure, arch OQ_DIT_PI (Pi-0.5 action expert):
 *
 *   r   = x_t . W_in^T + b_in                                (fp32 residual)
 *   per block l, step t (modulation m = mod[l][t], scales s = s_table[l][t]):
 *     h   = fp16(rms(r) * g1 * (1 + m.sc1) + m.sh1)
 *     qkv = fp16(W4A4(h; Wqkv, s[0]))                        q|k|v along N
 *     o   = fp16(softmax(q k^T / sqrt(hd)) v) per head, keys = [prefix ; k]
 *     r  += m.gt1 * W4A4(o; Wo, s[1])
 *     h2  = fp16(rms(r) * g2 * (1 + m.sc2) + m.sh2)
 *     gu  = fp16(W4A4(h2; Wgu, s[2]))                        gate|up along N
 *     a   = fp16(gelu_tanh(gate) * up)
 *     r  += m.gt2 * W4A4(a; Wd, s[3])
 *   v   = fp16(rms(r) * g_f) . W_out^T + b_out ;  x_{t+1} = x_t + dt * v
 *
 * Arch OQ_DIT_GR00T (GR00T-N1.5 DiT; the Appendix on per-step scaling names
 * AdaLayerNorm -> attention q/k/v -> ... -> LayerNorm -> ff.net[0] -> GELU ->
 * ff.net[2]):
 *
 *   per block l, step t (m = mod[l][t], s = s_table[l][t]):
 *     h   = fp16(ln(r) * g1 * (1 + m.sc1) + m.sh1)           AdaLayerNorm
 *     even l (cross-attention):  q = fp16(W4A4(h; Wq, s[0])),
 *            k|v = fp16(W4A4(cond; Wkv, 1)) per sample, from
 *            oq_dit_set_condition (step-invariant, computed once)
 *     odd l (self-attention):    q|k|v = fp16(W4A4(h; Wqkv, s[0]))
 *     o   = fp16(softmax(q k^T / sqrt(hd)) v) per head and sample
 *     r  += W4A4(o; Wo, s[1])
 *     h2  = fp16(ln(r) * g2 + b2)                            LayerNorm
 *     f   = fp16(gelu_tanh(W4A4(h2; Wff0, s[2])))
 *     r  += W4A4(f; Wff2, s[3])
 *   v   = fp16(ln(r) * g_f) . W_out^T + b_out ;  x_{t+1} = x_t + dt * v
 *
 * rms(r) = r / sqrt(mean(r^2) + 1e-6), ln(r) = (r - mean) / sqrt(var + 1e-6),
 * dt = -1/steps (pi, tau 1 -> 0) or +1/steps (gr00t, tau 0 -> 1), the Hadamard
 * block of a linear is the largest power of two dividing its input size.
 */
typedef enum { OQ_DIT_PI = 0, OQ_DIT_GR00T = 1 } oq_dit_arch;

typedef struct {
  int32_t arch;        /* oq_dit_arch                                        */
  int32_t n_blocks;    /* >= 1                                               */
  int32_t hidden;      /* D, multiple of 64, <= 8192; = n_heads * head_dim  */
  int32_t mlp;         /* F, multiple of 64                                  */
  int32_t n_heads;
  int32_t head_dim;    /* <= 128, multiple of 16                             */
  int32_t tokens;      /* S action tokens per sample, <= 64                  */
  int32_t prefix;      /* pi: P prefix tokens per sample (keys before the S
                          own); gr00t: P conditioning tokens per sample      */
  int32_t batch;       /* B samples                                          */
  int32_t steps;       /* T denoising steps                                  */
  int32_t action_dim;  /* A, multiple of 8                                   */
} oq_dit_config;

/* A prepared W4A4 weight: device Wq [N][K/2] and w_scale fp32 [N]. */
typedef struct {
  const uint8_t* wq;
  const float* w_scale;
} oq_qweight;

/* Per-block device pointers (borrowed; the caller keeps them alive until
 * oq_dit_destroy).  All vectors fp16. */
typedef struct {
  const void* g1;          /* [D] norm gain before attention                   */
  const void* g2;          /* [D] norm gain before the MLP                     */
  oq_qweight qkv;          /* pi and odd gr00t blocks: q|k|v, N = 3D, K = D;
                              even gr00t blocks: q only, N = D, K = D          */
  oq_qweight o;            /* N = D,  K = D                                    */
  oq_qweight gate_up;      /* pi: gate|up, N = 2F; gr00t: ff0, N = F; K = D    */
  oq_qweight down;         /* N = D,  K = F                                    */
  const void* prefix_k;    /* pi: [B][P][D] fp16, step-invariant; gr00t: NULL  */
  const void* prefix_v;    /* pi: [B][P][D] fp16; gr00t: NULL                  */
  const void* b2;          /* gr00t: [D] LayerNorm bias before the MLP; pi: NULL */
  oq_qweight cross_kv;     /* even gr00t blocks: k|v of the conditioning
                              tokens, N = 2D, K = D; otherwise NULL            */
} oq_dit_block;

typedef struct {
  const void* w_in;        /* fp16 [D][A]                                      */
  const void* b_in;        /* fp16 [D]                                         */
  const void* w_out;       /* fp16 [A][D]                                      */
  const void* b_out;       /* fp16 [A]                                         */
  const void* g_f;         /* fp16 [D] final norm gain                         */
  const oq_dit_block* blocks; /* host array [n_blocks], copied by oq_dit_create */
  const void* mod;         /* fp16 device [n_blocks][steps][NM][D] per-step
                              modulation; pi: NM = 6 (sc1, sh1, gt1, sc2, sh2,
                              gt2), gr00t: NM = 2 (sc1, sh1)                   */
  const float* s_table;    /* host fp32 [n_blocks][steps][4], copied           */
} oq_dit_weights;

typedef struct oq_dit oq_dit;

/* Workspace size in bytes for a config (device memory the caller provides). */
int oq_dit_workspace_bytes(const oq_dit_config* cfg, size_t* bytes);

/* Validate cfg and weights and create a handle (host memory only).
 * Errors: OQ_ERR_NULL, OQ_ERR_SHAPE, OQ_ERR_ARG, OQ_ERR_DEVICE. */
int oq_dit_create(const oq_dit_config* cfg, const oq_dit_weights* w, oq_dit** out);

/* Attach caller-owned device workspace (256-byte aligned, at least
 * oq_dit_workspace_bytes).  Calls of one handle must not overlap in time (they
 * share the workspace).
 * Errors: OQ_ERR_NULL, OQ_ERR_WORKSPACE, OQ_ERR_ALIGN. */
int oq_dit_set_workspace(oq_dit* h, void* workspace, size_t bytes);

/* gr00t: compute every cross-attention block's conditioning k|v from cond
 * (device fp16 [B][P][D], read during the call only) into the workspace:
 * rotate-quantize with s = 1 and the W4A4 k|v linear, once per conditioning
 * input (it does not depend on the step).  Required before the first step
 * of a gr00t handle and again whenever the conditioning or the workspace
 * changes.  Errors: OQ_ERR_NULL, OQ_ERR_WORKSPACE, OQ_ERR_ARG (pi handle),
 * OQ_ERR_HIP. */
int oq_dit_set_condition(oq_dit* h, const void* cond, void* stream);

/* One Euler step t (0 <= t < steps) on x (device fp32 [B][S][A], in place).
 * Errors: OQ_ERR_NULL, OQ_ERR_WORKSPACE, OQ_ERR_ARG (bad t, or a gr00t handle
 * without a condition), OQ_ERR_HIP. */
int oq_dit_step(oq_dit* h, float* x, int32_t t, void* stream);

/* n_steps consecutive steps t = 0 .. n_steps-1 on x, in place. */
int oq_dit_denoise(oq_dit* h, float* x, int32_t n_steps, void* stream);

/* Run block l of step t alone on a residual (device fp32 [B*S][D], in place);
 * for per-block parity checks with a teacher-forced input. */
int oq_dit_run_block(oq_dit* h, int32_t l, int32_t t, float* resid, void* stream);

/* Parity check of the fused producers (each writes a linear's fp16 input and
 * quantizes it in the same kernel, eq:scale / eq:quant after the rotation of
 * eq:blockdiag): run block l of step t only up to and including the producer
 * of quantization site `site` (0: the q|k|v (q) input, 1: the o input, 2:
 * the gate|up (ff0) input, 3: the down (ff2) input).  That site's codes and
 * token scales are then in the workspace (oq_dit_intermediates.codes,
 * .x_scale).  Errors: as oq_dit_run_block; OQ_ERR_ARG for a bad site. */
int oq_dit_run_block_until(oq_dit* h, int32_t l, int32_t t, float* resid, int32_t site, void* stream);

/* Static per-step, per-channel steps inside the driver (eq:perstep_scale with
 * the per-(layer, step, channel) table; the scalar s_t of oq_dit_weights is
 * then unused for the four block sites).  delta: device fp32
 * [n_blocks][steps][3 D + F], 16-byte aligned: for block l and step t the step
 * rows of the q|k|v (q) input [D], the o input [D], the gate|up (ff0) input
 * [D] and the down (ff2) input [F], in that order.  step_weights: host array
 * [n_blocks][steps][4] of the same four linears folded with their step rows
 * (oq_quantize_weights_step: W''[n][j] = W'[n][j] Delta_j, RTN per output
 * channel), device pointers borrowed until the mode is cleared.  Each site's
 * producer then writes codes clamp(round(y_j / Delta_j), +-7) with token
 * scale 1 and each linear uses its step's folded weight.  delta = NULL
 * returns the handle to the per-token quantizer.  The array is copied; the
 * captured steps are dropped.  Not for the gr00t conditioning k|v linear
 * (step-invariant, computed once).  Errors: OQ_ERR_NULL, OQ_ERR_ALIGN. */
int oq_dit_set_static_steps(oq_dit* h, const float* delta, const oq_qweight* step_weights);

/* The step's in-projection alone: resid [M][D] fp32 = x W_in^T + b_in (the
 * residual at the input of block 0), for a caller that runs blocks one by
 * one (calibration rollouts).  Errors: OQ_ERR_NULL, OQ_ERR_ALIGN, OQ_ERR_HIP. */
int oq_dit_in_projection(oq_dit* h, const float* x, float* resid, void* stream);

/* The last stage of a step alone, on a caller residual (device fp32 [M][D],
 * 16-byte aligned, read only): v = fp16(norm(resid) g_f) W_out^T + b_out and
 * the Euler update x += dt v with dt = -1/T (pi) or +1/T (gr00t), x device
 * fp32 [B][S][A] in place (Experimental Settings: T Euler steps).  With
 * oq_dit_in_projection and oq_dit_run_block it rebuilds a step from its
 * parts, for checking oq_dit_step against them bit for bit.
 * Errors: OQ_ERR_NULL, OQ_ERR_ALIGN, OQ_ERR_HIP. */
int oq_dit_final_stage(oq_dit* h, const float* resid, float* x, void* stream);

/* Intermediate tensors of the most recent block the handle ran (fp16,
 * row-major, M = batch * tokens rows), for per-site parity checks: every
 * quantized linear's fp16 input and every fp16 output of the block can be
 * compared with the oracle fed the GPU's own upstream values.  Pointers into
 * the workspace, valid until the next call on the handle.  The fp16 linear
 * inputs h1, attn, h2 and act are written by oq_dit_run_block and
 * oq_dit_run_block_until only (oq_dit_step and oq_dit_denoise produce their
 * codes without storing them; gr00t's cross-attention output, which its
 * quantizer reads back, is the exception). */
typedef struct {
  const void* h1;        /* [M][D]  norm output, input of the q|k|v (q) linear  */
  const void* qkv;       /* [M][3D] q|k|v linear output (gr00t even: q, [M][D]) */
  const void* attn;      /* [M][D]  attention output, input of the o linear      */
  const void* h2;        /* [M][D]  norm output, input of the gate|up / ff0 linear */
  const void* gate_up;   /* pi: [M][2F] gate|up output; gr00t: not written (the
                            ff0 linear applies the GELU in its epilogue and
                            writes act directly)                              */
  const void* act;       /* [M][F]  input of the down / ff2 linear               */
  const float* resid;    /* [M][D]  fp32 residual of the last oq_dit_step after
                            its last block (oq_dit_run_block uses the caller's) */
  const void* cond_kv;   /* gr00t: k|v of the conditioning tokens of every
                            even block, head-major [n_blocks/2 rounded up][B]
                            [H][2 (k, v)][P][head_dim]; pi: NULL              */
  const void* codes;     /* packed codes of the last quantization site the
                            handle produced (its fp16 input is h1, attn, h2 or
                            act): [M][K/2], or the 16-row tiled layout when
                            codes_tiled is 1                                  */
  const float* x_scale;  /* [M] token scales of the same site                 */
  int32_t codes_tiled;   /* 1: codes in the 16-row tiled layout (M <= 64)      */
} oq_dit_intermediates;

/* Fill *out with the intermediate pointers.  Errors: OQ_ERR_NULL, OQ_ERR_WORKSPACE. */
int oq_dit_get_intermediates(const oq_dit* h, oq_dit_intermediates* out);

/* Free the handle (not the borrowed weights or the workspace). NULL is a no-op. */
void oq_dit_destroy(oq_dit* h);

#ifdef __cplusplus
}
#endif

#endif /* OQ_H */
