/*
 * basq.h -- C ABI of the MI355X (gfx950) W4A4 rotated linear layer of BASE-Q.
 *
 * The layer (paper Sec. 4, Eq. 14 and Eq. 15; row-vector form, R orthogonal, W' = W R given):
 *
 *     Y = Q_a( s^a (X R) - b^c ) . Q_w(W')^T + c ,      c = W_hat b^c + b   ("fused bias")
 *
 *   R      normalised Hadamard rotation applied online to each block of rot_size channels
 *          (Sec. 3.1: entries +-n^(-1/2); Sec. 4 "online rotations"), n = 2^t or 28 * 2^t
 *   Q_a    per-token asymmetric uniform quantiser with lower bound z and step s (Eq. 4; "per-token
 *          asymmetric dynamic quantization", Sec. 5), range [clip_lo*min, clip_hi*max]
 *   Q_w    per-output-channel asymmetric INT4 weights: W_hat[n,k] = sw[n] * (q_w[n,k] - zp[n])
 *
 * Conventions
 *   - Every pointer is a DEVICE pointer owned by the caller unless its comment says "host".
 *     The library never frees caller memory; hot calls allocate nothing and never synchronise.
 *   - `stream` is a hipStream_t passed as void* (NULL = the default stream).  All work of a call
 *     is enqueued on it in order.
 *   - bf16 tensors are passed as void* (16-bit storage, round-to-nearest-even on output).
 *   - Return value: BASQ_OK or a negative error code.  Arguments are validated on the host before
 *     anything is launched; a failing call launches nothing.  basq_last_error() gives the text of
 *     the calling thread's last error.
 *   - Packed INT4 ("canonical") layout: byte j of a row holds code k = 2j in its low nibble and
 *     code k = 2j+1 in its high nibble.
 *   - Alignment: X, Aq, meta, Wq, bias (b^c) and act_scale (s^a) base pointers 16-byte aligned (BASQ_EINVAL
 *     otherwise); K % 32 == 0; ldx % 8 == 0.  Y needs only its natural 2-byte alignment and any ldy >= N.
 */
#ifndef BASQ_H
#define BASQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define BASQ_OK            0
#define BASQ_EINVAL       (-1)  /* null pointer, bad shape, stride or alignment */
#define BASQ_EUNSUPPORTED (-2)  /* valid request the library does not implement (bits != 4, ...) */
#define BASQ_EWORKSPACE   (-3)  /* workspace too small */
#define BASQ_EHIP         (-4)  /* a HIP call or launch failed */

#define BASQ_W_CANONICAL 0      /* Wq is [N, K/2] in the canonical packed layout */
#define BASQ_W_DECODE16  1      /* Wq is in the weight-streaming layout written by basq_pack_decode */

/* Per-token quantisation record written by basq_rotate_quant and read by basq_w4a4_gemm.
 * x_hat[m,k] = scale * q[m,k] + lo   (Eq. 4 with z = lo);  rowsum = sum_k q[m,k]. */
typedef struct {
    float   scale;
    float   lo;
    int32_t rowsum;
    int32_t reserved;
} basq_tokmeta;

/* Library version (major*10000 + minor*100 + patch). */
int basq_version(void);

/* Text of the calling thread's most recent error ("" if none).  Host pointer, valid until the
 * thread's next failing call. */
const char* basq_last_error(void);

/*
 * Online rotation + bias + per-token quantisation (Sec. 3.1 rotation; Eq. 14 bias; Eq. 15 scale;
 * Eq. 4 quantiser; Fig. 6 "fused quant kernel").  For each token m:
 *
 *     r      = X[m,:] . (H_n / sqrt(n))     blockwise over K/rot_size blocks, fp32
 *     v_k    = r_k - bias_k                 (act_scale == NULL)
 *     v_k    = fma(r_k, act_scale_k, -bias_k)
 *     lo     = clip_lo * min_k v_k ;  hi = clip_hi * max_k v_k
 *     s      = (hi - lo) / 15  (1 if not a positive finite number) ;  inv = 1/s ;  nlo = -(lo*inv)
 *     q_k    = rint(min(max(fma(v_k, inv, nlo), 0), 15))        round-half-to-even, NaN -> 0
 *
 *   X          bf16 [M, ldx], row m at X + m*ldx, ldx >= K
 *   rot_size   n; K % n == 0; n = 2^t (t >= 1) or 28 * 2^t (t >= 1).  For n = 28 * 2^t the matrix is
 *              H_28 (x) H_(2^t) with the Paley type-I H_28 over GF(27) (see basq_hadamard28) and
 *              channel index k = i * 2^t + j, i the H_28 index.
 *   bias       fp32 [K] b^c in the rotated basis, or NULL (= 0)
 *   act_scale  fp32 [K] s^a, or NULL (= 1)
 *   bits       must be 4 (else BASQ_EUNSUPPORTED)
 *   group_size 0 or K: one range and one record per token (what basq_w4a4_gemm consumes).  Otherwise a
 *              multiple of 32 that divides K: every run of group_size consecutive channels gets its own
 *              range, steps 4-6 above and the record apply per group (per-head quantisation of q, k and
 *              the KV cache with rot_size = group_size = head_dim; Sec. 5 "Deployment Details").  Such
 *              codes are not an input of basq_w4a4_gemm; with group_size = 128 they are the input of
 *              basq_w4a4_gemm_grouped.
 *   Aq         out, uint8 [M, K/2] canonical packed codes.  May be NULL when Aq6 is given, with per-token ranges and
 *              rot_size == K in {4096, 8192, 14336} (the quantiser writes the fp6 form itself and then leaves the
 *              4-bit form out; elsewhere BASQ_EUNSUPPORTED)
 *   meta       out, [M, K/group_size] records, token-major (group_size 0 counts as K)
 *   rot_out    out, optional debug dump of r, fp32 [M, K]; NULL to skip
 *   Aq6        out, optional (NULL to skip): the same codes in the fp6 operand form described at
 *              basq_pack_fp6 (basq_fp6_bytes(M, K) bytes), 16-byte aligned; needs K % 128 == 0.  With per-token
 *              ranges and rot_size == K in {4096, 8192, 14336} the quantiser writes it itself; otherwise (other
 *              sizes, group-wise ranges) a packing pass follows on the same stream.
 * M == 0 is valid and does nothing.
 */
int basq_rotate_quant(const void* X, int64_t M, int32_t K, int64_t ldx, int32_t rot_size,
                      const float* bias, const float* act_scale,
                      float clip_lo, float clip_hi, int32_t bits, int32_t group_size,
                      uint8_t* Aq, basq_tokmeta* meta, float* rot_out, uint8_t* Aq6, void* stream);

/*
 * INT4 x INT4 GEMM with INT32 accumulation and fused de-quantisation (Sec. 5.2; Fig. 6
 * "de-quantisation" with the bias folded in; Eq. 14 fused bias):
 *
 *     ACC[m,n] = sum_k q_a[m,k] * q_w[n,k]
 *     Y[m,n]   = bf16( s_m * sw_n * (ACC[m,n] - zp_n * rowsum_m) + lo_m * w_sum_n + out_bias_n )
 *
 *   Aq, meta   as written by basq_rotate_quant, [M, K/2] and [M]
 *   Wq         uint8 [N, K/2] with w_layout = BASQ_W_CANONICAL, or the weight-streaming layout of
 *              basq_pack_decode with w_layout = BASQ_W_DECODE16.  The latter is read by the M <= 128 path
 *              only: with M > 128 it needs the fp6 operands (which replace Wq), else BASQ_EUNSUPPORTED.
 *   w_scale    bf16 [N] sw;  w_zero  bf16 [N] zp in code units (any real value)
 *   w_sum      fp32 [N] = sw_n * (sum_k q_w[n,k] - K * zp_n) = sum_k W_hat[n,k]
 *   out_bias   fp32 [N] c, or NULL (= 0)
 *   Y          out, bf16 [M, ldy], ldy >= N
 *   acc_out    out, optional debug dump of ACC, int32 [M, N]; NULL to skip
 *   Aq6, Wq6   optional, both or neither: the two code matrices in the fp6 operand form
 *              (basq_pack_fp6; Aq6 also straight from basq_rotate_quant).  With them, and M > 64 (from 33 on where
 *              the shape favours it), the
 *              product runs on the f8f6f4 matrix-core path at twice the int8 rate; ACC and Y are
 *              bit-identical to the int8 path.  Needs K % 128 == 0.
 * Any M >= 0, N >= 1; otherwise M <= 128 (decode, batched decode) takes a weight-streaming path, same results.
 */
int basq_w4a4_gemm(const uint8_t* Aq, const basq_tokmeta* meta, int64_t M, int32_t K,
                   const uint8_t* Wq, int32_t N, int32_t w_layout,
                   const void* w_scale, const void* w_zero, const float* w_sum, const float* out_bias,
                   void* Y, int64_t ldy, int32_t* acc_out,
                   const uint8_t* Aq6, const uint8_t* Wq6, void* stream);

/*
 * The same product for activations quantised in groups of 128 channels (basq_rotate_quant with group_size = 128:
 * every group g of token m has its own step s_mg, lower bound z_mg and code sum rowsum_mg; Eq. 4 per group):
 *
 *     ACC_g[m,n] = sum over the channels k of group g of q_a[m,k] * q_w[n,k]
 *     Y[m,n]     = bf16( sw_n * ( sum_g ( s_mg ACC_g[m,n] + z_mg w_gsum[g,n] )
 *                                 - zp_n * sum_g ( s_mg rowsum_mg + 128 z_mg ) ) + out_bias_n )
 *
 * which is sum_k x_hat[m,k] W_hat[n,k] + out_bias_n.  The integer products are exact; the sums over groups are
 * fp32 multiply-adds in group order.
 *   Aq, meta   as written by basq_rotate_quant with group_size = 128: [M, K/2] and [M, K/128] records
 *   group_size must be 128 (else BASQ_EUNSUPPORTED); K % 128 == 0
 *   Wq         uint8 [N, K/2] canonical;  w_scale, w_zero bf16 [N];  out_bias fp32 [N] or NULL
 *   w_gsum     int32 [K/128, N], group-major: w_gsum[g*N + n] = sum of the codes of row n in group g
 *              (basq_group_colsums)
 *   Y          out, bf16 [M, ldy]
 *   Aq6, Wq6   optional, both or neither: the same codes in the fp6 operand form (basq_rotate_quant's Aq6 output or
 *              basq_pack_fp6; basq_fp6_bytes each).  With them the product runs on the f8f6f4 matrix cores, about
 *              1.5 times as fast, with bit-identical Y.
 */
int basq_w4a4_gemm_grouped(const uint8_t* Aq, const basq_tokmeta* meta, int64_t M, int32_t K, int32_t group_size,
                           const uint8_t* Wq, int32_t N, const void* w_scale, const void* w_zero,
                           const int32_t* w_gsum, const float* out_bias, void* Y, int64_t ldy,
                           const uint8_t* Aq6, const uint8_t* Wq6, void* stream);

/* Offline: the per-group sums of the weight codes, w_gsum int32 [K/128, N] (see basq_w4a4_gemm_grouped). */
int basq_group_colsums(const uint8_t* Wq, int32_t N, int32_t K, int32_t group_size, int32_t* w_gsum, void* stream);

/*
 * The fp6 operand form of an INT4 code matrix (device-side repacking; offline for weights).
 * The matrix cores of this GPU multiply 6-bit floating-point operands (e2m3: sign, 2 exponent bits,
 * 3 mantissa bits) at twice their int8 rate.  Code q in 0..15 is stored as the e2m3 number q/8, which
 * is exact; S = sum_k (qa/8)(qb/8) is exact in the fp32 accumulator for K <= 32768 (longer rows run on the
 * int8 path whatever operands are given), and the INT32 accumulator of the INT4 GEMM (Sec. 5.2) is 64*S.
 * (The e2m3 bit pattern of q/8 is q itself.)
 *
 *   codes      device uint8 [rows, K/2], two codes per byte, low nibble first (as Aq and Wq)
 *   out6       out, device uint8, basq_fp6_bytes(rows, K) bytes, 16-byte aligned.  Blocks of 3072
 *              bytes, one per (chunk c of 128 codes along K, block rb of 32 rows), chunk-major: block
 *              (c, rb) at (c*ceil(rows/32) + rb)*3072.  Row r of the block, group f = 0..3 (codes
 *              128c + 32f .. +31) is a 24-byte little-endian string of 6-bit fields; its first 16 bytes
 *              sit at 64r + 16*(f ^ ((r>>2)&3)), its last 8 bytes at 2048 + 256f + 8r.  (The block is
 *              the image the GEMM keeps in LDS.)  Rows past the matrix in the last block stay unwritten.
 * K % 128 == 0.  basq_fp6_bytes returns ceil(rows/32)*32 * 3K/4 (0 for an unsupported K).
 */
size_t basq_fp6_bytes(int64_t rows, int32_t K);
int basq_pack_fp6(const uint8_t* codes, int64_t rows, int32_t K, uint8_t* out6, void* stream);

/*
 * The weight-streaming layout for decode-sized calls (M <= 128; such a call is one pass over the weights and
 * bound by memory bandwidth, the decode case of Sec. 5.2's speed measurement).  The matrix-core operand of
 * that path puts 16 different rows on the 16 lanes of a quarter wavefront, so canonical weights are read in
 * 16-byte pieces of 16 rows at a time; here the kilobyte one wavefront load consumes is contiguous instead.
 *
 *   Wq         device uint8 [N, K/2] canonical
 *   out        out, device uint8, basq_decode_bytes(N, K) = ceil(N/16)*16 * K/2 bytes, 16-byte aligned.
 *              Block nb (rows 16nb .. 16nb+15) at nb*16*K/2; inside it chunk c (bytes 64c .. 64c+63 of each
 *              row) is the KB at c*1024; inside that, the 16-byte piece at (16*s + r)*16, s = 0..3,
 *              r = 0..15, holds bytes 64c + 16s .. +15 of row 16nb + r.  Rows past N are zeros.
 * K % 128 == 0.  basq_decode_bytes returns 0 for an unsupported shape.
 */
size_t basq_decode_bytes(int32_t N, int32_t K);
int basq_pack_decode(const uint8_t* Wq, int32_t N, int32_t K, uint8_t* out, void* stream);

/* Bytes of workspace basq_linear_fused needs for this shape (activation codes, token records, and
 * the fp6 copy of the codes). */
size_t basq_workspace_bytes(int64_t M, int32_t K, int32_t N);

/*
 * The whole layer in one call: basq_rotate_quant then basq_w4a4_gemm on `stream`, the codes and
 * token records living in `workspace` (256-byte aligned, >= basq_workspace_bytes(M, K, N), else
 * BASQ_EWORKSPACE).  Arguments as in the two calls above; with Wq6, M > 128 takes the fp6 matrix-core path, and
 * so does M > 64 (from 33 on where the shape favours it) if the quantiser writes the fp6 form itself: rot_size == K in
 * {512, 1024, 2048, 4096, 8192, 14336}, or rot_size in {128, 256, 512} with K % 256 == 0 and K <= 16384.
 * group_size must be 0 or K here (BASQ_EUNSUPPORTED otherwise: groups go through basq_rotate_quant and
 * basq_w4a4_gemm_grouped).  With w_layout = BASQ_W_DECODE16 the whole layer is one kernel launch (same results bit for bit)
 * for at most 4 tokens of rot_size == K in {4096, 8192} with N <= 4096, and for few tokens of rot_size == K in
 * {512, 1024, 2048} (see basq_diag_one_launch).  Y may lie over X, bias or act_scale: the tokens are rotated and quantised
 * before the first output is written.  Nothing in this call allocates or synchronises, so it may be recorded in a HIP graph.
 */
int basq_linear_fused(const void* X, int64_t M, int32_t K, int64_t ldx, int32_t rot_size,
                      const float* bias, const float* act_scale,
                      float clip_lo, float clip_hi, int32_t bits, int32_t group_size,
                      const uint8_t* Wq, int32_t N, int32_t w_layout,
                      const void* w_scale, const void* w_zero, const float* w_sum, const float* out_bias,
                      void* Y, int64_t ldy, const uint8_t* Wq6,
                      void* workspace, size_t workspace_bytes, void* stream);

/*
 * basq_linear_fused for callers that cannot allocate a workspace or keep one alive: code recorded under HIP graph
 * capture, tight serving loops, harnesses in which hipMalloc is forbidden.  Same arguments, same kernels and
 * bit-identical results; the codes and token records live in a workspace of BASQ_STATIC_WORKSPACE_BYTES that is
 * part of the library's code object (every GPU the library runs on holds its own copy until the process ends).
 *   - basq_workspace_bytes(M, K, N) > BASQ_STATIC_WORKSPACE_BYTES returns BASQ_EWORKSPACE and launches nothing
 *     (8 MiB hold e.g. 192 tokens of K = 32768, 800 of K = 8192, 1632 of K = 4096).
 *   - The call allocates nothing, frees nothing and does not synchronise.  Its first call on a device looks the
 *     workspace's address up (hipGetSymbolAddress, which may load the code object): make that call outside stream
 *     capture.
 *   - All calls on one GPU share that GPU's workspace, which keeps the previous call's contents (the quantiser
 *     writes every byte the product reads, so nothing needs clearing).  Calls that overlap on one GPU - different
 *     streams, or threads - race on it; calls on one stream, or otherwise ordered, do not.
 */
#define BASQ_STATIC_WORKSPACE_BYTES (8u << 20)
int basq_linear_fused_static(const void* X, int64_t M, int32_t K, int64_t ldx, int32_t rot_size,
                             const float* bias, const float* act_scale,
                             float clip_lo, float clip_hi, int32_t bits, int32_t group_size,
                             const uint8_t* Wq, int32_t N, int32_t w_layout,
                             const void* w_scale, const void* w_zero, const float* w_sum, const float* out_bias,
                             void* Y, int64_t ldy, const uint8_t* Wq6, void* stream);

/* ---- offline helpers (not on the timed path) --------------------------------------------- */

/*
 * Offline weight rotation W' = W R (Sec. 4: the rotation of the activations is undone by folding R into the
 * weights; Eq. 14 writes the layer as (W R)(R^-1 x)): every row of W is rotated blockwise by H_n/sqrt(n) exactly
 * as basq_rotate_quant rotates a token (fp32), then rounded to bf16.
 *   W          bf16 [N, ldw], ldw >= K, ldw % 8 == 0, 16-byte aligned;  rot_size as in basq_rotate_quant
 *   W_rot      out, bf16 [N, K], 16-byte aligned
 *   workspace  >= N*K*4 bytes (the fp32 rotation), 16-byte aligned, else BASQ_EWORKSPACE
 */
int basq_rotate_weights(const void* W, int32_t N, int32_t K, int64_t ldw, int32_t rot_size, void* W_rot,
                        void* workspace, size_t workspace_bytes, void* stream);

/*
 * Round-to-nearest per-output-channel asymmetric INT4 quantisation of rotated-basis weights
 * (weights are quantised per channel, Sec. 5 "Deployment Details"; asymmetric with a bf16
 * zero-point per the workload definition).  Per row n, every operation one fp32 operation:
 *     lo, hi = min_k W', max_k W' ;  sw = bf16((hi - lo)/15)  (1 if not positive finite)
 *     zp = clamp(rint(-lo/sw), 0, 15) ;  q = clamp(rint(W'/sw) + zp, 0, 15)
 *     w_sum = fp32( double(sw) * (sum_k q - K*zp) )
 *   W_rot bf16 [N, ldw];  outputs Wq [N, K/2] canonical, w_scale bf16 [N], w_zero bf16 [N], w_sum fp32 [N].
 */
int basq_quantize_weights(const void* W_rot, int32_t N, int32_t K, int64_t ldw,
                          uint8_t* Wq, void* w_scale, void* w_zero, float* w_sum, void* stream);

/*
 * Fused bias of Eq. 14 from the dequantised weights:  out_bias[n] = sum_k W_hat[n,k] * bias[k]
 * + layer_bias[n], accumulated in fp64, stored fp32.  bias (b^c, fp32 [K]) and layer_bias
 * (fp32 [N]) may each be NULL (= 0).
 */
int basq_fused_bias(const uint8_t* Wq, int32_t N, int32_t K, const void* w_scale, const void* w_zero,
                    const float* bias, const float* layer_bias, float* out_bias, void* stream);

/*
 * Everything the hot calls need from already quantised weights, in one offline call (Eq. 14: the "fused bias"
 * W_hat b^c + b that undoes the channel bias after the product; and the weight sums that carry the activations'
 * lower bound through the product: with x_hat = s_m q_a + z_m and W_hat = sw_n (q_w - zp_n),
 * sum_k x_hat W_hat = s_m sw_n (ACC - zp_n rowsum_m) + z_m w_sum_n):
 *     w_sum[n]    = fp32( double(sw_n) * (sum_k q_w[n,k] - K * zp_n) )
 *     out_bias[n] = fp32( sum_k W_hat[n,k] * bias[k] + layer_bias[n] ),  accumulated in fp64
 *   Wq_canonical  uint8 [N, K/2], 16-byte aligned;  w_scale, w_zero bf16 [N]
 *   bias          fp32 [K] b^c in the rotated basis, or NULL (= 0);  layer_bias fp32 [N], or NULL (= 0)
 *   w_sum, out_bias   out, fp32 [N] each (the w_sum and out_bias arguments of the hot calls)
 *   Wq_prepacked  out, optional (NULL to skip): the weights in the fp6 operand form, basq_fp6_bytes(N, K) bytes,
 *                 16-byte aligned, K % 128 == 0 -- the Wq6 argument of the hot calls (see basq_pack_fp6)
 * Same results as basq_fused_bias and basq_pack_fp6, and the w_sum of basq_quantize_weights.
 */
int basq_prepare_weights(const uint8_t* Wq_canonical, int32_t N, int32_t K, const void* w_scale, const void* w_zero,
                         const float* bias, const float* layer_bias, float* w_sum, float* out_bias,
                         uint8_t* Wq_prepacked, void* stream);

/*
 * Channel bias calibration (Sec. 3.2: the bias cancels the per-channel means after rotation):
 *     bias_out[k] = mean_m ( s^a_k * r[m,k] ),  r the rotated calibration tokens; fp64 mean, fp32 out.
 * workspace: >= M*K*4 bytes (holds r), else BASQ_EWORKSPACE.
 */
int basq_calibrate_bias(const void* X, int64_t M, int32_t K, int64_t ldx, int32_t rot_size,
                        const float* act_scale, float* bias_out,
                        void* workspace, size_t workspace_bytes, void* stream);

/* The 28 x 28 matrix of +-1 used for rot_size = 28 * 2^t, row-major into a HOST buffer of 784
 * int8 (Paley type-I construction over GF(27) = GF(3)[t]/(t^3 + 2t + 1)). */
int basq_hadamard28(int8_t* out_host);

/* ---- around the linear layer: norm, rotary positions, INT4 cache, attention ------------------- */

/*
 * The residual's addition and the root-mean-square norm in front of a linear layer.  For each token m:
 *
 *     h_k = bf16(X[m,k] + residual[m,k])                             (X[m,k] without a residual)
 *     y_k = (h_k * rstd) * weight_k ,   rstd = 1 / sqrt(mean_k h_k^2 + eps)          fp32
 *     Y8[m,k] = e4m3(y_k / s_m) ,   s_m = max_k |y_k| / 448          fp32; s_m = 1 if not a positive finite number, quotients beyond
 *                                                                    +-448 are +-448, NaN stays NaN
 *
 *   X, residual  bf16 [M, ldx], [M, ldr]; residual may be NULL.   weight  bf16 [K]
 *   res_out      out, bf16 [M, ldro]: h, or NULL.  May be X or residual (with that one's stride)
 *   Y            out, bf16 [M, ldy], or NULL where Y8 is given.  May be X or residual
 *   Y8, y8_scale out, OCP e4m3 [M, ldy8] and fp32 [M] (for a projection that is kept in 8 bits), or NULL
 * K % 8 == 0, K <= 32768; strides multiples of 8; base pointers 16-byte aligned (Y8: 8, y8_scale: 4).  M == 0 does nothing.
 */
int basq_add_rms_norm(const void* X, const void* residual, const void* weight, int64_t M, int32_t K, int64_t ldx, int64_t ldr,
                      float eps, void* res_out, int64_t ldro, void* Y, int64_t ldy, uint8_t* Y8, int64_t ldy8, float* y8_scale,
                      void* stream);

/*
 * Cosines and sines for basq_rope_append, computed in fp64 (offline): row p holds cos(p f_j), j < rot_dim/2, then sin(p f_j),
 * with f_j = base^(-2j/rot_dim), and for long contexts
 *   BASQ_ROPE_LINEAR  f_j / factor
 *   BASQ_ROPE_BANDS   u f_j + (1 - u) f_j / factor, u = clamp((t_j - low) / (high - low), 0, 1), t_j = original_len f_j / 2 pi
 *                     the turns that pair j makes over the original length
 *   BASQ_ROPE_YARN    the same with u linear in j, between the pairs that make `high` and `low` turns (rounded outwards), and
 *                     cosines and sines times 0.1 ln(factor) + 1 (factor > 1)
 * factor is read by all but BASQ_ROPE_PLAIN; low, high and original_len by the last two.
 *   cos_sin   out, fp32 [positions, rot_dim]
 */
#define BASQ_ROPE_PLAIN  0
#define BASQ_ROPE_LINEAR 1
#define BASQ_ROPE_BANDS  2
#define BASQ_ROPE_YARN   3
int basq_rope_table(int32_t rot_dim, int64_t positions, double base, int32_t scaling, double factor, double low, double high,
                    double original_len, float* cos_sin, void* stream);

/*
 * The paged INT4 cache of keys and values (Sec. 5 "Deployment Details": per-head asymmetric INT4): uint8 [num_pages, kv_heads,
 * page_size * (head_dim + 16)].  With P = page_size, D = head_dim, one head of one page holds
 *     K codes [P, D/2] canonical | V codes [P, D/2] canonical | K ranges fp32 [P, 2] = (scale, lo) | V ranges fp32 [P, 2]
 * and stands for scale * code + lo.  Slot s of a layer's cache is token s % P of page s / P.
 * head_dim 64 or 128; page_size a power of two from 16 to 1024; fewer than 2^31 tokens in all pages; 16-byte aligned.
 * basq_kv_page_bytes: bytes of one page (all heads), 0 for an unsupported shape.
 */
size_t basq_kv_page_bytes(int32_t kv_heads, int32_t head_dim, int32_t page_size);

/*
 * New tokens' heads on their way into the cache: rotary positions and the online per-head Hadamard rotation of q and k (Sec. 4;
 * the rotation cancels in q . k), the INT4 quantisation of k and v (Eq. 4 per head, Sec. 5).  For each token t, in fp32, each
 * operation rounded on its own:
 *     rope     (a, b) -> (a cos - b sin, b cos + a sin) for the pairs of the first rot_dim channels: (i, i + rot_dim/2), or
 *              (2i, 2i + 1) where interleaved, with the cosines and sines of row positions[t]; the other channels stay
 *     rotate   sums and differences (a + b, a - b) of the channels 1, 2, 4, ... D/2 apart, then times fp32(1/sqrt(D)); a zero is positive
 *     k, v     lo, hi, s, q as in basq_rotate_quant, over each head; code and (s, lo) go to slots[t] of the cache
 *     k_hat, v_hat   bf16(fma(s, q, lo)), what the cache stands for (the prompt's own attention)
 *   q, k, v    bf16 [T, heads, D], [T, kv_heads, D] twice, heads side by side, token strides ldq, ldk, ldv (the three parts of one
 *              fused projection's output, say).  heads or kv_heads may be 0 (no q, or neither k nor v)
 *   positions  int32 [T]; a token whose position is negative or >= table_rows is padding: nothing of it is read or written.
 *              Not read where cos_sin is NULL (no rotary positions)
 *   cos_sin    fp32 [table_rows, rot_dim] (basq_rope_table); rot_dim a multiple of 16 up to D
 *   slots      int32 [T], each at most once; one that is negative or past the cache is not stored.  cache may be NULL (not stored)
 *   bits       must be 4 (else BASQ_EUNSUPPORTED)
 *   q_out      out, bf16 [T, heads, D], token stride ldqo; may be q.  k_hat, v_hat: out, bf16 [T, kv_heads, D], token stride ldh,
 *              or NULL; may be k and v
 * T == 0 does nothing.
 */
int basq_rope_append(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, int64_t T, int32_t heads,
                     int32_t kv_heads, int32_t head_dim, const int32_t* positions, const float* cos_sin, int64_t table_rows,
                     int32_t rot_dim, int32_t interleaved, int32_t rotate, float clip_lo, float clip_hi, int32_t bits,
                     const int32_t* slots, uint8_t* cache, int32_t num_pages, int32_t page_size, void* q_out, int64_t ldqo,
                     void* k_hat, void* v_hat, int64_t ldh, void* stream);

/*
 * Attention of the q_len newest tokens of each sequence over its cache, in which they are stored already.  With k_t, v_t what the
 * cache stands for, for new token j = 0 .. q_len - 1 of sequence b and each head (head h reads kv head h / (heads/kv_heads)):
 *     s_t = scale q . k_t ;   s_t = softcap tanh(s_t / softcap) where softcap > 0
 *     out = sum_t softmax(s)_t v_t ,   lse = ln sum_t e^(s_t)
 * over the tokens t < n, n = lengths[b] - (q_len - 1 - j), and t >= n - window where window > 0.  No token: out = 0, lse = -inf.
 *   q          bf16 [B * q_len, heads, D], token stride ldq (q_out of basq_rope_append)
 *   page_table int32 [B, table_stride]: token t of sequence b is token t % page_size of page page_table[b, t / page_size].  Entries
 *              past a length are not read; tokens of a page that is negative or >= num_pages count as not there
 *   lengths    int32 [B], the new tokens among them; more than max_len counts as max_len (negative as 0)
 *   max_len    host: the longest length there can be; the work is laid out for it.  At most table_stride * page_size, and 2^31 - 2^16
 *   q_len      up to 32768 (else BASQ_EUNSUPPORTED)
 *   out        out, bf16 [B * q_len, heads, D], token stride ldo; may be q.   lse   out, fp32 [B * q_len, heads], or NULL
 *   workspace  256-byte aligned (BASQ_EWORKSPACE where it is too small); NULL where basq_paged_attention_workspace_bytes is 0
 * The result does not depend on where pages lie.  B == 0 does nothing.
 * basq_paged_attention_workspace_bytes: what a call of this shape may need, and any with fewer sequences, new tokens or tokens, or a
 * shorter window (0 is the longest), of the same heads: a program asks once, for its largest.  At most 12.8 MB and 8 bytes for each
 * sequence, kv head and 16 of its query rows; 0 where no context is longer than 512 tokens, and for an unsupported shape.
 */
size_t basq_paged_attention_workspace_bytes(int32_t B, int32_t q_len, int32_t heads, int32_t kv_heads, int32_t head_dim,
                                            int32_t max_len, int32_t window);
int basq_paged_attention(const void* q, int64_t ldq, int32_t B, int32_t q_len, int32_t heads, int32_t kv_heads, int32_t head_dim,
                         int32_t bits, const uint8_t* cache, int32_t num_pages, int32_t page_size, const int32_t* page_table,
                         int64_t table_stride, const int32_t* lengths, int32_t max_len, float scale, float softcap, int32_t window,
                         void* out, int64_t ldo, float* lse, void* workspace, size_t workspace_bytes, void* stream);

/* ---- the ends of a step: places in the cache, embeddings, logits, tokens ------------------------ */

/*
 * Tokens in bf16 times 4-bit weights with a scale and a zero point for each group of channels: the output head, a layer whose
 * activations stay in 16 bits.  fp32 products and sums, one rounding at the end:
 *
 *     Y[m,n] = sum_g w_scale[n,g] * sum_{k in g} (q[n,k] - w_zero[n,g]) X[m,k]  +  bias[n]
 *
 *   X          bf16 [M, ldx], 16-byte aligned, ldx >= K, a multiple of 8, up to 2^23.  A token with a value that is not finite has
 *              outputs that are not finite, and one with values beyond 2^100 may have; they leave the others alone
 *   Wq         uint8 [N, K/2] canonical, or the layout of basq_pack_decode with w_layout = BASQ_W_DECODE16 (K % 128 == 0);
 *              16-byte aligned
 *   group_size channels of a group: a multiple of 32 that divides K; 0 counts as K.  (basq_quantize_weights makes such weights of
 *              [N, K] when called with N * K / group_size rows of group_size channels)
 *   w_scale, w_zero   bf16 [N, K / group_size], zero points in code units (any real value)
 *   bias       fp32 [N], or NULL (= 0)
 *   Y          out, [M, ldy], ldy >= N: fp32 where y_f32, otherwise bf16
 * K % 32 == 0.  Laid out for few tokens: the weights are read once for every 64.  K up to 2^20, N up to 2^28, M up to 1048560 (else
 * BASQ_EUNSUPPORTED); M == 0 does nothing.  Results do not change from call to call.
 */
int basq_w4a16_gemm(const void* X, int64_t M, int32_t K, int64_t ldx, const uint8_t* Wq, int32_t N, int32_t w_layout,
                    const void* w_scale, const void* w_zero, int32_t group_size, const float* bias, void* Y, int64_t ldy,
                    int32_t y_f32, void* stream);

/*
 * Rows of such a matrix in bf16: the embeddings of tokens, from the head's weights where the two are tied.
 *
 *     Y[t,k] = bf16( scale * (w_scale[n,g] * (q[n,k] - w_zero[n,g])) ) ,   n = ids[t]                       fp32
 *
 *   ids        int32 [T]; one that is negative or >= N (padding) gives a row of zeros
 *   Y          out, bf16 [T, ldy], 16-byte aligned, ldy >= K and a multiple of 8
 * The matrix as above.  T up to 2^30 (else BASQ_EUNSUPPORTED); T == 0 does nothing.
 */
int basq_w4a16_lookup(const int32_t* ids, int64_t T, const uint8_t* Wq, int32_t N, int32_t K, int32_t w_layout, const void* w_scale,
                      const void* w_zero, int32_t group_size, float scale, void* Y, int64_t ldy, void* stream);

/*
 * A token for each row of logits.  The tokens of a row are taken in the order of their logits, the largest first, equal ones by
 * their index; one whose logit is -inf or NaN is none.  With z_0 >= z_1 >= ... the logits in that order and weights
 * w_i = e^((z_i - z_0) / temperature) (1 where z_i = z_0), the first n tokens are kept, the least of
 *     top_k                                                 where top_k > 0
 *     the first n with  w_0 + ... + w_(n-1) >= top_p * S    where top_p < 1; S is the sum over the first top_k (over all without it); 1 at least
 *     the number of weights >= min(min_p, 1)                where min_p > 0
 * and 1 where temperature is not > 0 (the likeliest token).  The token is the first kept one at which
 * w_0 + ... + w_i > u * (sum of the kept weights).
 * Weights are computed in fp64, to 2^-36 of theirs or better, and summed as whole multiples of 2^-bits, bits = min(50, 62 - log2 V
 * rounded up), each rounded to one, or, of fp32 logits, the sum of some neighbours: a running sum is off by 2^-36 of it and V 2^-(bits + 1)
 * at most.  top_p * S and u * sum are fp64 products.  A weight below half of a step is never drawn, and the same call gives the same
 * tokens every time.
 *   logits     fp32 (f32 != 0) or bf16 [B, ldl], ldl >= V, aligned as their type is; ldl = 0: B draws from one row
 *   temperature, top_p, min_p   fp32 [B], top_k int32 [B]; each may be NULL (1; none).  A NaN among the last two is none
 *   u          fp64 [B], from [0, 1); what lies outside counts as the nearest of them, NaN as 0
 *   token      out, int32 [B]; -1 for a row without tokens
 *   logprob    out, fp32 [B] or NULL: ln of the token's share of the kept weights; -inf without tokens
 *   kept       out, int32 [B] or NULL: n
 *   workspace  256-byte aligned, >= basq_sample_workspace_bytes(B, V) (else BASQ_EWORKSPACE); NULL where that is 0, as for V up to
 *              32768.  A workspace for a call does for any with fewer rows or a smaller V.  bf16 logits need none: NULL, or any
 * V up to 2^22 (else BASQ_EUNSUPPORTED).  B == 0 does nothing.
 */
size_t basq_sample_workspace_bytes(int32_t B, int32_t V);
int basq_sample(const void* logits, int64_t ldl, int32_t B, int32_t V, int32_t f32, const float* temperature, const int32_t* top_k,
                const float* top_p, const float* min_p, const double* u, int32_t* token, float* logprob, int32_t* kept,
                void* workspace, size_t workspace_bytes, void* stream);

/*
 * The books of the paged cache, on the GPU: a batch's sequences grow, or lose their last tokens, and what basq_rope_append and
 * basq_paged_attention take is written.  Sequence b of the batch is row s = seqs[b] of the pool; with n = lengths[s], m = n +
 * new_tokens[b] and P = page_size it has ceil(n / P) pages and comes to have ceil(m / P):
 *     pages that go back   (new_tokens[b] < 0) are put behind the free ones, in the order of the batch, a sequence's in their order
 *     pages that are taken then come from the end of the free ones, in the order of the batch, into row s from entry ceil(n / P) on
 *     tokens               n .. m - 1 get positions and slots (page * P + token % P)
 *   lengths      int32 [rows];  lengths_out  out, int32 [rows]: m for the batch's rows, the others left as they are; may be lengths
 *   pool_table   int32 [rows, columns], row stride pool_stride, entries past a length may hold anything; in and out
 *   free_pages   int32 [capacity], the first free_count[0] are free; in and out.   free_out  out, int32 [1]; may be free_count
 *   seqs         int32 [B], none twice; NULL: the first B rows
 *   new_tokens   int32 [B]; NULL: q_len of each
 *   q_len        > 0: token places lie in B runs of q_len, T = B * q_len, and a sequence's new tokens are the last of its run
 *                0: they lie packed, sequence behind sequence, from 0 on
 *   positions, slots   out, int32 [T]; -1 for places without a token (padding to the operators that read them), slots also where the page
 *                      in the table or among the free ones is negative, or the slot would not be an int32
 *   starts       out, int32 [B + 1] or NULL, with q_len = 0: where each sequence's tokens start; the last is their number
 *   batch_table  out, int32 [B, columns], row stride batch_stride, or NULL: the pages of the batch's sequences; entries past them are
 *                left as they were
 *   batch_lengths   out, int32 [B] or NULL: m
 *   status       out, int32 [2]: (0, 0), or why nothing was done: all positions and slots are -1, batch_lengths and starts 0, the
 *                books as they were (free_out is free_count's value, lengths_out and batch_table are left)
 *                  BASQ_KV_SEQUENCE  (1, b): seqs[b] is no row, or was named before
 *                  BASQ_KV_LENGTH    (2, b): its length, before or after, is negative or more than columns * P, or q_len < new_tokens[b]
 *                  BASQ_KV_FREE      (3, free_count): the count is negative, or free_pages has no room for what goes back
 *                  BASQ_KV_PAGES     (4, pages): that many are missing
 *                  BASQ_KV_TOKENS    (5, tokens): that many more than T
 *   books        workspace, >= basq_kv_books_bytes(B), 16-byte aligned (else BASQ_EWORKSPACE); holds nothing between calls
 * page_size as in the cache; B up to 1024 and B * columns < 2^31 (else BASQ_EUNSUPPORTED).  But for the pairs named, nothing may
 * overlap.  B == 0: the padding, starts[0], free_out and status are written.
 */
#define BASQ_KV_SEQUENCE 1
#define BASQ_KV_LENGTH   2
#define BASQ_KV_FREE     3
#define BASQ_KV_PAGES    4
#define BASQ_KV_TOKENS   5
size_t basq_kv_books_bytes(int32_t B);
int basq_kv_extend(const int32_t* lengths, int32_t* pool_table, int64_t pool_stride, int32_t rows, int32_t columns, int32_t page_size,
                   int32_t* free_pages, int32_t capacity, const int32_t* free_count, const int32_t* seqs, const int32_t* new_tokens,
                   int32_t B, int32_t q_len, int32_t* positions, int32_t* slots, int64_t T, int32_t* starts, int32_t* batch_table,
                   int64_t batch_stride, int32_t* batch_lengths, int32_t* lengths_out, int32_t* free_out, int32_t* status,
                   void* books, size_t books_bytes, void* stream);

/* ---- diagnostics: what this machine sustains (used by the benchmark's measured ceilings), single tilings, bounds ---- */

/*
 * Pure streaming kernel with the access pattern of basq_rotate_quant (the paper's fused quant kernel,
 * Fig. 6, is bandwidth bound): one wavefront per token reads 2K bytes from src + m*2K and writes K/2
 * bytes to dst + m*K/2 and 16 bytes to meta + m*16.  K a multiple of 2048.  Moves tokens*(2.5K+16) bytes.
 */
int basq_diag_stream(const void* src, void* dst, void* meta, int64_t tokens, int32_t K, void* stream);

/*
 * Read-only streaming kernel with the access pattern of the decode-sized product (M <= 128: one pass over the
 * weights, bound by memory bandwidth): `blocks` workgroups walk `bytes` (a multiple of 32768) of src in 32 KB
 * spans, every lane requesting eight 16-byte pieces before it consumes any; out receives blocks*256 uint32
 * checksums.
 */
int basq_diag_read(const void* src, int64_t bytes, uint32_t* out, int32_t blocks, void* stream);

/*
 * Register-resident int8 MFMA loop (Sec. 5.2: the prefill GEMM is compute bound): `blocks` workgroups of
 * 4 waves, each wave issues 8*iters v_mfma_i32_32x32x32_i8 on 4-bit valued operands; out receives
 * blocks*256 int32 checksums.  Executes blocks*4*8*iters*65536 integer operations.
 */
int basq_diag_mfma_i8(int32_t* out, int32_t blocks, int32_t iters, void* stream);

/*
 * Such a loop on the f8f6f4 matrix-core path the prefill GEMM uses by default: each wave issues
 * 16*iters v_mfma_f32_16x16x128_f8f6f4, that GEMM's instruction, with fp6 (e2m3) operands that encode 4-bit codes;
 * out receives blocks*256 fp32 checksums.  Executes blocks*4*16*iters*65536 operations.
 */
int basq_diag_mfma_f6(float* out, int32_t blocks, int32_t iters, void* stream);

/*
 * The fp6 product of basq_w4a4_gemm has several tilings, of which it takes the one a cost table names for the shape.  For
 * checking and timing them one by one: the index of that tiling (0 .. BASQ_FP6_TILINGS - 1; -1 where basq_w4a4_gemm takes
 * another kernel though both fp6 operands are given), and the product on a given one, whatever M is (the bits do not
 * depend on it).  Arguments as in basq_w4a4_gemm; both fp6 operands are needed.
 * The same for the split tilings, in which two groups of waves share a tile's channels: basq_diag_fp6_split_tiling is the
 * index of the one that is taken instead of the tiling above (0 .. BASQ_FP6_SPLIT_TILINGS - 1), -1 where none is.
 */
#define BASQ_FP6_TILINGS 6
#define BASQ_FP6_SPLIT_TILINGS 6
int basq_diag_fp6_tiling(int64_t M, int32_t K, int32_t N);
int basq_diag_fp6_split_tiling(int64_t M, int32_t K, int32_t N);
int basq_diag_w4a4_gemm_fp6(int32_t tiling, const basq_tokmeta* meta, int64_t M, int32_t K, int32_t N,
                            const void* w_scale, const void* w_zero, const float* w_sum, const float* out_bias,
                            void* Y, int64_t ldy, int32_t* acc_out,
                            const uint8_t* Aq6, const uint8_t* Wq6, void* stream);
int basq_diag_w4a4_gemm_fp6_split(int32_t tiling, const basq_tokmeta* meta, int64_t M, int32_t K, int32_t N,
                                  const void* w_scale, const void* w_zero, const float* w_sum, const float* out_bias,
                                  void* Y, int64_t ldy, int32_t* acc_out,
                                  const uint8_t* Aq6, const uint8_t* Wq6, void* stream);

/*
 * The fp6 product of basq_w4a4_gemm_grouped has two tilings: 0, 128 x 128, and 1, 256 x 192, which needs N % 4 == 0, w_gsum on
 * a 16-byte boundary and K >= 384.  The one that is taken for a shape whose w_gsum is aligned (-1 where there is none), and the
 * product on a given one (the bits do not depend on it); arguments as in basq_w4a4_gemm_grouped, group_size = 128.
 */
int basq_diag_grouped_tiling(int64_t M, int32_t K, int32_t N);
int basq_diag_w4a4_gemm_grouped_fp6(int32_t tiling, const basq_tokmeta* meta, int64_t M, int32_t K, int32_t N,
                                    const void* w_scale, const void* w_zero, const int32_t* w_gsum, const float* out_bias,
                                    void* Y, int64_t ldy, const uint8_t* Aq6, const uint8_t* Wq6, void* stream);

/*
 * Whether basq_linear_fused takes a layer in one kernel launch: 1, or 0 where it takes several, as it does where Y lies over what the
 * rotation reads.  Arguments as there; known on the host, nothing is read or launched.
 */
int basq_diag_one_launch(const void* X, int64_t M, int32_t K, int64_t ldx, int32_t rot_size, const float* bias, const float* act_scale,
                         int32_t N, int32_t w_layout, const void* Y, int64_t ldy);

/*
 * The 256 x 192 tiling goes on requesting behind a workgroup's last tile, from lane offsets that the bounds check of the load drops.
 * Counted on the host with the kernel's own offsets: the requests of an M x K x N product that leave their table, or are not
 * dropped behind a last tile; 0 in a sound kernel, -1 for a shape that the tiling does not take.
 */
int64_t basq_diag_grouped_wide_strays(int64_t M, int32_t K, int32_t N);

/*
 * The blockwise rotations with per-token ranges request bias and act_scale without a test for the token's end.  Computed on the
 * host with the kernel's own index: one past the last channel that it requests of either, for a token of K channels, K a
 * multiple of 256 up to 16384 (otherwise BASQ_EINVAL); at most K.
 */
int basq_diag_block_vector_channels(int32_t K);

#ifdef __cplusplus
}
#endif
#endif /* BASQ_H */
