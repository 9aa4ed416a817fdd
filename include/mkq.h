/*
 * mkq.h -- C ABI of libmkq: the 4-bit (W4A4) quantized BERT linear layer of
 * MKQ-BERT (arXiv 2203.13483) for AMD MI355X (gfx950).
 *
 * Conventions that hold for every entry point unless it says otherwise
 *   - returns an int status: MKQ_OK (0) or a negative MKQ_ERR_* code; nothing
 *     throws, nothing prints;
 *   - every pointer is a DEVICE pointer owned by the caller (the library keeps
 *     no reference after the call is enqueued), except arguments whose names
 *     end in _host and the parameter structs themselves, which are read on the
 *     host during the call;
 *   - work is enqueued on `stream` (a hipStream_t passed as void*, NULL = the
 *     default stream); the call does not synchronise and does not allocate;
 *   - matrices are row-major and dense (row stride = number of columns) unless
 *     a leading dimension is given; device pointers must be 16-byte aligned;
 *   - argument errors are detected on the host before anything is enqueued, so
 *     a failing call has no effect on device memory.
 *
 * Packed int4 ("I4") tensors use the canonical nibble packing: element k of a
 * row is the low nibble of byte k/2 when k is even, the high nibble when k is
 * odd, two's complement, rows of K/2 bytes.
 */
#ifndef MKQ_H
#define MKQ_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

enum {
    MKQ_OK = 0,
    MKQ_ERR_NULL = -1,        /* a required pointer is NULL */
    MKQ_ERR_SHAPE = -2,       /* a dimension is negative / not a supported multiple */
    MKQ_ERR_ALIGN = -3,       /* a device pointer is not 16-byte aligned */
    MKQ_ERR_SCALE = -4,       /* a host-side step size is <= 0, NaN or Inf */
    MKQ_ERR_DTYPE = -5,       /* unknown / unsupported MKQ_* dtype or activation enum */
    MKQ_ERR_WORKSPACE = -6,   /* workspace NULL or smaller than the *_workspace_bytes value */
    MKQ_ERR_UNSUPPORTED = -7, /* valid request outside what the kernels cover (e.g. K >= 131072) */
    MKQ_ERR_HIP = -8          /* the HIP runtime reported an error at launch */
};

enum { MKQ_F32 = 0, MKQ_F16 = 1, MKQ_BF16 = 2, MKQ_I4 = 3, MKQ_I8 = 4 };
enum { MKQ_ACT_NONE = 0, MKQ_ACT_GELU = 1 };

const char *mkq_status_string(int status);
int mkq_version(void);

/* Quantizer of section 3.1, Eq. 1, integer part, 4 bits, one step for the whole
 * tensor (per-tensor scale):  code = round(clamp(x / s_x, -8, 7)), binary32
 * divide, round half to even, NaN -> 0.
 *   x      [M, K] of x_dtype (MKQ_F32 or MKQ_F16), row stride ldx elements
 *   q_out  [M, K/2] bytes, canonical packing
 * K must be a multiple of 32.  M == 0 is a no-op.
 * Errors: NULL, SHAPE (M<0, K<0, K%32, ldx<K), ALIGN, SCALE, DTYPE, HIP. */
int mkq_quantize(const void *x, int x_dtype, int64_t M, int64_t K, int64_t ldx, float s_x,
                 uint8_t *q_out, void *stream);

/* Abs-max calibration of section 3.1 (third paragraph):  s = max|x| / 7, written
 * to s_out[0] (per_row == 0) or s_out[m] for every row (per_row != 0).  An
 * all-zero tensor / row gets s = 1.  x_dtype MKQ_F32 or MKQ_F16.
 * Errors: NULL, SHAPE, ALIGN, DTYPE, HIP. */
int mkq_absmax_scale(const void *x, int x_dtype, int64_t M, int64_t K, int64_t ldx, int per_row,
                     float *s_out, void *stream);

/* Scale gradients of one tensor under one step (section 4.1):
 *     g_out[0] = sum_i ( round(x_i/s) - x_i/s )                 STE-based (4.1.1)
 *     g_out[1] = 2 sum_i ( Q[x_i] - x_i ) round(x_i/s)          MSE-based (4.1.2)
 * where round() is the code of Eq. 1 (clamp to the `bits`-bit range included, decided in
 * binary32 like the quantizer) and Q[x] = s * code.  Terms and sums are binary64; the
 * order of the partial sums is not fixed, so results agree to rounding only.
 *   x      [M, K] of x_dtype (MKQ_F32 or MKQ_F16), row stride ldx; K % 8 == 0, M > 0
 *   bits   4 or 8;  g_out  two doubles on the device (overwritten)
 * Errors: NULL, SHAPE, ALIGN, SCALE, DTYPE (x_dtype, bits), HIP. */
int mkq_scale_gradients(const void *x, int x_dtype, int64_t M, int64_t K, int64_t ldx, float s,
                        int bits, double *g_out, void *stream);

/* Percentile calibration of an activation step (section 3.1, third paragraph): the
 * clipping point T is the k-th largest |x_i|, k = max(1, floor(M*K * top_ppm / 10^6))
 * (top_ppm = 100 for the top 0.01 %), found exactly by radix selection over the bit
 * patterns of |x| (counting passes over x: two for binary16, three for binary32);
 * s_out[0] = T / (2^(bits-1) - 1), or 1 when T = 0.  NaN ranks as 0.  top_ppm = 0 gives abs-max calibration.
 *   workspace  at least mkq_percentile_scale_workspace_bytes() bytes, 16-byte aligned
 * M*K < 2^32.  Errors: NULL, SHAPE, ALIGN, DTYPE, WORKSPACE, UNSUPPORTED, HIP. */
size_t mkq_percentile_scale_workspace_bytes(void);
int mkq_percentile_scale(const void *x, int x_dtype, int64_t M, int64_t K, int64_t ldx,
                         int64_t top_ppm, int bits, float *s_out, void *workspace,
                         size_t workspace_bytes, void *stream);

/* Offline weight preparation (Eq. 1 with one step per row = per output channel;
 * abs-max calibration when s_w_in is NULL).
 *   W        [N, K] binary32, row n = output channel n
 *   s_w_in   [N] steps to use, or NULL to calibrate  s_w[n] = max_k |W[n,k]| / 7
 *            (all-zero row -> 1).  Given steps must be > 0 and finite (precondition;
 *            they live on the device and are not checked).
 *   s_w_out  [N] the steps actually used (may alias s_w_in)
 *   Wq_out   mkq_packed_weight_bytes(N, K) bytes in the layout the GEMM reads
 *            (currently the canonical packing, rows of K/2 bytes)
 * K must be a multiple of 32.
 * Errors: NULL, SHAPE, ALIGN, HIP. */
size_t mkq_packed_weight_bytes(int64_t N, int64_t K);
int mkq_pack_weights_int4(const float *W, int64_t N, int64_t K, const float *s_w_in,
                          float *s_w_out, uint8_t *Wq_out, void *stream);

/* Reduction lengths that are not a multiple of 32 (the 4-layer student of section 5.2 has hidden size
 * 312 and FFN size 1200): both operands are stored with rows padded to mkq_padded_k(K) codes, the
 * smallest multiple of 128 >= K (whole 64-byte stages of the tile kernels), the padding codes being
 * zero, which adds nothing to any dot product.  The padded variants of the quantizer and of the weight
 * preparation take K % 8 == 0, compute exactly what their plain counterparts compute on the K real
 * columns (abs-max over the real columns only) and write rows of mkq_padded_k(K) / 2 bytes;
 * mkq_linear_int4 is then called with K = mkq_padded_k(K) on pre-quantized activations.  Same errors
 * as the plain variants (SHAPE on K % 8 instead of K % 32). */
int64_t mkq_padded_k(int64_t K);
int mkq_quantize_padded(const void *x, int x_dtype, int64_t M, int64_t K, int64_t ldx, float s_x,
                        uint8_t *q_out, void *stream);
int mkq_pack_weights_int4_padded(const float *W, int64_t N, int64_t K, const float *s_w_in,
                                 float *s_w_out, uint8_t *Wq_out, void *stream);

/* Packs already-quantized int8 codes (values in [-8, 7]; higher bits are
 * discarded) of a [rows, K] matrix into the weight / activation layout. */
int mkq_pack_codes_int4(const int8_t *codes, int64_t rows, int64_t K, uint8_t *q_out, void *stream);

/* Inverse of the weight layout: int8 codes [N, K] (for tests and inspection). */
int mkq_unpack_weights_int4(const uint8_t *Wq, int64_t N, int64_t K, int8_t *codes_out,
                            void *stream);

/* Optional parts of the linear's epilogue. */
typedef struct mkq_epilogue {
    int act;              /* MKQ_ACT_*; applied after bias and residual (GELU: erf form, FFN of section 3.2; binary32
                             and bfloat16 results, and codes written beside them, come from a form that also keeps
                             values below 1e-7: within 1e-7 plus one unit in the last place of what binary16
                             results and code outputs are decided from) */
    const void *residual; /* NULL or [M, N] added after the bias */
    int residual_dtype;   /* MKQ_F32 or MKQ_F16 */
    float s_next;         /* step of the next layer's activation quantizer; used when out_dtype == MKQ_I4
                             or q_out != NULL */
    uint8_t *q_out;       /* NULL, or [M, N/2] packed codes of the binary32 result under s_next, written
                             in addition to a float `out` */
    int32_t *acc_out;     /* NULL, or [M, N] raw int32 accumulators (for parity checks) */
    void *splitk_scratch; /* NULL, or a scratch area prepared by mkq_splitk_scratch_init (see there): lets a
                             linear with few tokens split K across workgroups to fill the chip */
    size_t splitk_scratch_bytes;
    int64_t q_pitch;      /* codes per row of the code outputs (`out` of MKQ_I4 / MKQ_I8, q_out); 0 = N.  A
                             consumer whose reduction length is padded (mkq_padded_k) takes rows of that
                             many codes: give the padded length here; the columns N .. q_pitch - 1 of every
                             row are written as zero codes.  >= N, a multiple of 8, and N % 8 == 0. */
} mkq_epilogue;

/* Scratch of a K split across workgroups.  Few tokens against a weight matrix with few output channels
 * give too few workgroups to fill 256 compute units; the reduction over K is then cut into slices that
 * different workgroups sum (int32 addition is associative: the accumulators are the same bit for bit),
 * their partial sums meeting in this area.  It is device memory owned by the caller, at least
 * mkq_splitk_scratch_bytes() bytes (a constant: 16 KiB of ticket counters, then 16 MiB for partial sums),
 * 16-byte aligned.  mkq_splitk_scratch_init clears the counters and must have run once (on any stream,
 * ordered before the first linear that uses the area) after the area was allocated; every linear leaves the
 * counters cleared again.  Two linears that may run at the same time need two areas.  A linear given no
 * area, or whose partial sums would not fit, runs without the split -- same results, fewer workgroups.
 * Errors: NULL, ALIGN, WORKSPACE (area too small), HIP. */
size_t mkq_splitk_scratch_bytes(void);
int mkq_splitk_scratch_init(void *scratch, size_t scratch_bytes, void *stream);

/* Once-per-device setup of every kernel of the library (dynamic LDS limits, occupancy queries) for the
 * device that is current.  Optional: each kernel is otherwise set up, under a lock, the first time it is
 * launched on a device.  Call it before capturing launches into a HIP graph if no eager call has run yet.
 * Errors: HIP. */
int mkq_init(void);

/* The quantized linear layer  y = x W^T + b  with both operands in 4 bits
 * (the int4 matrix multiplication of sections 1 and 5.4 applied to the linears
 * of section 3.2):
 *     acc[m,n] = sum_k a[m,k] * w[n,k]                      (int32, exact)
 *     y[m,n]   = fma((float)acc, s_x * s_w[n], bias[n])     (binary32)
 *     y       += residual;  y = act(y)                      (optional)
 *     out      = narrow(y)  or  codes(y; s_next) packed     (Eq. 1 again)
 *   a        [M, K]: packed codes (a_dtype == MKQ_I4, rows of K/2 bytes) or float
 *            activations (MKQ_F32 / MKQ_F16), which are first quantized with s_x
 *            into `workspace`: by a launch of mkq_quantize's kernel that precedes the
 *            GEMM (inside one launch a hand-over between quantizing and multiplying
 *            workgroups cost more than the second launch), or, for a few sentences
 *            (K <= 1024, at most one 32x32 tile per CU), by the GEMM's own workgroups
 *   Wq, s_w  from mkq_pack_weights_int4;  bias [N] binary32 or NULL
 *   out      [M, N] of out_dtype (F32, F16, BF16) or [M, N/2] bytes (I4); may be
 *            NULL when epi->q_out or epi->acc_out is the only result wanted
 *   epi      NULL = no activation, no residual, no extra outputs
 *   workspace  at least mkq_linear_int4_workspace_bytes(M, N, K, a_dtype) bytes
 *              (0 for packed input: then workspace may be NULL)
 * K % 32 == 0, K < 131072; N even when codes are written.  M == 0 is a no-op.
 * Errors: NULL, SHAPE, ALIGN, SCALE (s_x, s_next), DTYPE, WORKSPACE, UNSUPPORTED, HIP. */
size_t mkq_linear_int4_workspace_bytes(int64_t M, int64_t N, int64_t K, int a_dtype);
int mkq_linear_int4(const void *a, int a_dtype, float s_x, const uint8_t *Wq, const float *s_w,
                    const float *bias, int64_t M, int64_t N, int64_t K, void *out, int out_dtype,
                    const mkq_epilogue *epi, void *workspace, size_t workspace_bytes, void *stream);

/* Few tokens (M <= 128): the linear is one pass over the weights and is bound by how fast they stream from
 * HBM.  Canonical rows, K/2 bytes apart, are a poorer stream (rows fetched side by side, a power-of-two
 * pitch apart, land on the same few memory channels), so large weights that serve few tokens can be kept in a
 * second layout (16 tokens, us, mkq_linear_int4 and this: K = N = 4096 4.9 and 9.2, 8192 9.5 and 12.8, 16384 28.4 and
 * 27.6, 32768 107 and 92; K = 8192, N = 28672 26 and 22.5, the other way round 25 and 27), in which the bytes that the chip reads at one moment lie next to each other: the 32 channels
 * of panel q (q = 0 .. P-1, P = ceil(N / 32)) and the 64 codes of k position g (g = 0 .. K/64 - 1) form a
 * block of 1 KiB = 64 pieces of 16 bytes; the block is number g P' + q, where P' = P if P is odd, else P + 1
 * (all panels of one k position, one unused block when P is even, then the next k position: an odd pitch keeps
 * the k positions that a wave has in flight off each other's memory channels); piece l of a block is bytes
 * [32 g + 16 (l / 32), + 16) of the canonical row of channel 32 q + r(l % 32), where
 * r(i) = 16 (i / 16) + 8 ((i / 4) % 2) + 4 ((i / 8) % 2) + i % 4; channels past N and the unused block are
 * zero.  mkq_stream_weight_bytes(N, K) = 32 P' K / 2.
 *   mkq_repack_weights_int4_stream   canonical (from mkq_pack_weights_int4) -> streaming layout; K % 64 == 0
 *   mkq_linear_int4_stream           mkq_linear_int4 on weights in the streaming layout: same arguments, same
 *                                    results bit for bit; M <= 128 and K % 256 == 0 (else UNSUPPORTED)
 * Errors: as mkq_linear_int4. */
size_t mkq_stream_weight_bytes(int64_t N, int64_t K);
int mkq_repack_weights_int4_stream(const uint8_t *Wq, int64_t N, int64_t K, uint8_t *Wq_stream_out, void *stream);
int mkq_linear_int4_stream(const void *a, int a_dtype, float s_x, const uint8_t *Wq_stream, const float *s_w,
                           const float *bias, int64_t M, int64_t N, int64_t K, void *out, int out_dtype,
                           const mkq_epilogue *epi, void *workspace, size_t workspace_bytes, void *stream);

/* For callers that cannot allocate device memory or carry a scratch area around -- code under HIP graph
 * capture, tight serving loops, harnesses that forbid hipMalloc: mkq_linear_int4_stream on packed codes
 * (a is [M, K/2] bytes; no workspace) with the scratch of the K split taken from an area that is part of
 * the library's code object (16 KiB of ticket counters + 16 MiB for partial sums, per GPU, held until the
 * process ends) instead of epi->splitk_scratch, which is ignored.  Nothing is allocated or freed.  Same
 * results as mkq_linear_int4_stream, bit for bit.  A problem whose K split would need more room for partial
 * sums than the area has (ceil(N / 128) * slices * 16 KiB * ceil(M / 32) rounded up to 1, 2 or 4 > 16 MiB,
 * or N > 524288) is refused with MKQ_ERR_UNSUPPORTED and nothing runs.  All calls on one GPU share the area:
 * calls that may overlap in time on one GPU (two streams, two threads) race; calls ordered on one stream
 * do not.  Other errors: as mkq_linear_int4. */
int mkq_linear_int4_stream_static(const uint8_t *a, float s_x, const uint8_t *Wq_stream, const float *s_w,
                                  const float *bias, int64_t M, int64_t N, int64_t K, void *out, int out_dtype,
                                  const mkq_epilogue *epi, void *stream);

/* The same linear with both operands in 8 bits (the int8 column of Table 2 in
 * section 5.4; the 8-bit layers of the mixed 4/8-bit models of section 4.2).  Eq. 1
 * with k = 8: codes in [-128, 127], one byte each, row-major, K-contiguous.
 *   mkq_quantize_int8      x [M, K] (F32 / F16, row stride ldx) -> int8 [M, K], per-tensor
 *                          step s_x; NaN -> 0.  K % 16 == 0.
 *   mkq_pack_weights_int8  W [N, K] binary32 -> int8 [N, K] and per-channel steps
 *                          s_w[n] = max_k |W[n,k]| / 127 (all-zero row -> 1) unless
 *                          s_w_in gives them.  K % 16 == 0.
 *   mkq_linear_int8        acc[m,n] = sum_k a[m,k] w[n,k] (int32, exact; |acc| <= K * 2^14),
 *                          y = fma((float)acc, s_x * s_w[n], bias[n]), then residual and
 *                          activation as in mkq_linear_int4.  a is int8 codes [M, K]
 *                          (quantize first; there is no workspace), out [M, N] of
 *                          F32 / F16 / BF16, or int8 codes of y under epi->s_next (MKQ_I8),
 *                          or NULL with epi->acc_out.  4-bit code outputs (out_dtype
 *                          MKQ_I4, epi->q_out) are not offered: UNSUPPORTED.
 *                          K % 64 == 0, K < 65536.  M == 0 is a no-op.
 * Errors: NULL, SHAPE, ALIGN, SCALE, DTYPE, UNSUPPORTED, HIP. */
int mkq_quantize_int8(const void *x, int x_dtype, int64_t M, int64_t K, int64_t ldx, float s_x,
                      int8_t *q_out, void *stream);
int mkq_pack_weights_int8(const float *W, int64_t N, int64_t K, const float *s_w_in,
                          float *s_w_out, int8_t *Wq_out, void *stream);
int mkq_linear_int8(const int8_t *a, float s_x, const int8_t *Wq, const float *s_w,
                    const float *bias, int64_t M, int64_t N, int64_t K, void *out, int out_dtype,
                    const mkq_epilogue *epi, void *stream);

/* Experimental: the 4-bit linear through the 6-bit float path of the matrix core.  Every code in [-8, 8]
 * is an E3M2 value (sign, 3 exponent bits with bias 3, 2 mantissa bits), products and sums of codes are
 * exact in binary32 while |sum| < 2^24, so the result is the same exact integer contraction as
 * mkq_linear_int4 -- with no widening and half the matrix instructions per k.  Operands are "containers":
 * 6 bits per code, rows of 3K/4 bytes made of groups of 64 codes = 48 bytes; the 32 codes of half h of a
 * group are a 192-bit little-endian stream (code i in bits [6i, 6i + 6)) stored as bytes [16h, 16h + 16)
 * and then [32 + 8h, 40 + 8h) of the group.  K % 64 == 0 for the containers, K % 128 == 0 and
 * K < 262144 for the linear.  The quantizer and the weight preparation are those of
 * mkq_quantize / mkq_pack_weights_int4 (Eq. 1, per-tensor / per-channel steps), written as containers;
 * mkq_pack_codes_e3m2 takes int8 codes in [-8, 8].  mkq_linear_int4_e3m2: arguments and epilogue as
 * mkq_linear_int4 with both operands given as containers (no workspace).
 * Errors: NULL, SHAPE, ALIGN, SCALE, DTYPE, UNSUPPORTED, HIP. */
int mkq_quantize_e3m2(const void *x, int x_dtype, int64_t M, int64_t K, int64_t ldx, float s_x,
                      uint8_t *q_out, void *stream);
int mkq_pack_codes_e3m2(const int8_t *codes, int64_t rows, int64_t K, uint8_t *q_out, void *stream);
int mkq_pack_weights_e3m2(const float *W, int64_t N, int64_t K, const float *s_w_in, float *s_w_out,
                          uint8_t *Wq_out, void *stream);
int mkq_linear_int4_e3m2(const uint8_t *a, float s_x, const uint8_t *Wq, const float *s_w,
                         const float *bias, int64_t M, int64_t N, int64_t K, void *out, int out_dtype,
                         const mkq_epilogue *epi, void *stream);

/* 16-bit float baseline linear (same epilogue, no quantizers):
 *   a [M, K] binary16, W [N, K] binary16, bias [N] binary32 or NULL, binary32
 *   accumulation, out [M, N] of out_dtype (F32 or F16), residual binary16 or NULL.
 * K % 64 == 0.  Errors: NULL, SHAPE, ALIGN, DTYPE, UNSUPPORTED, HIP. */
int mkq_linear_fp16(const void *a, const void *W, const float *bias, int64_t M, int64_t N,
                    int64_t K, void *out, int out_dtype, int act, const void *residual,
                    void *stream);

/* One post-LN BERT encoder layer (multi-head attention and feed-forward network
 * of section 3.2) with all six linears W4A4; LayerNorm, softmax and GELU are
 * computed in binary32 (section 5), the attention products in binary16 with
 * binary32 accumulation, hidden states are stored in binary16.
 *
 *   c0  = codes(h; sx_qkv)                      (or q_in, if the caller has them)
 *   qkv = Lin_qkv(c0)                           [M, 3*hidden], q | k | v
 *   ctx = softmax(q k^T / sqrt(d_k)) v          per sequence and head, d_k = hidden/heads
 *   u   = Lin_ao(codes(ctx; sx_ao)) + h
 *   h1  = LayerNorm1(u)
 *   d   = Lin_down(codes(GELU(Lin_up(codes(h1; sx_up))); sx_down)) + h1
 *   out = LayerNorm2(d)
 *
 * The struct lives on the host; the pointers inside are device pointers. */
typedef struct mkq_bert_layer_params {
    int64_t batch, seq, hidden, heads, ffn;
    const uint8_t *Wq_qkv, *Wq_ao, *Wq_up, *Wq_down; /* packed; qkv is [3*hidden, hidden] */
    const float *sw_qkv, *sw_ao, *sw_up, *sw_down;   /* per-output-channel steps */
    const float *b_qkv, *b_ao, *b_up, *b_down;       /* biases, binary32 */
    float sx_qkv, sx_ao, sx_up, sx_down;             /* learned per-tensor activation steps */
    const float *ln1_gamma, *ln1_beta, *ln2_gamma, *ln2_beta;
    float ln_eps;
    float s_out_next; /* > 0: also write codes(out; s_out_next) to q_out_next */
    int next_bits;    /* width of those codes: 4 (packed, [M, hidden/2] bytes), 8 ([M, hidden] bytes), or 0 =
                         this layer's own width; lets 4-bit and 8-bit layers follow each other in a mixed
                         model (section 4.2) */
    /* Padding-free batches (the "valid tokens" of Table 2, section 5.4): cu_seqlens is NULL, or a device
     * array [batch + 1] of row offsets, sequence b being rows cu_seqlens[b] .. cu_seqlens[b+1] - 1 of the
     * total_tokens rows of h_in / h_out; seq is then an upper bound of the lengths (<= 128, any value);
     * a longer sequence is a precondition violation (its rows beyond the bound are not computed). */
    const int32_t *cu_seqlens;
    int64_t total_tokens;
} mkq_bert_layer_params;

/* Byte offsets of the layer's intermediates inside its workspace (all 256-byte
 * aligned); tests read them back stage by stage. */
typedef struct mkq_bert_layer_workspace_layout {
    size_t c0;   /* [M, hidden/2]   codes of the input                     */
    size_t qkv;  /* [M, 3*hidden]   binary16                                */
    size_t c1;   /* [M, hidden/2]   codes of the attention context          */
    size_t u;    /* [M, hidden]     binary16, attention output + residual   */
    size_t h1;   /* [M, hidden]     binary16, LayerNorm1 output             */
    size_t c2;   /* [M, hidden/2]   codes of h1                             */
    size_t c3;   /* [M, ffn/2]      codes of GELU(FFN-up)                   */
    size_t d;    /* [M, hidden]     binary16, FFN output + residual         */
    size_t total;
} mkq_bert_layer_workspace_layout;

int mkq_bert_layer_workspace(const mkq_bert_layer_params *p_host,
                             mkq_bert_layer_workspace_layout *layout_host);

/*   h_in   [M, hidden] binary16 (h_dtype == MKQ_F16) or binary32, M = batch*seq
 *   q_in   NULL, or packed codes of h_in under sx_qkv (skips the first quantizer)
 *   h_out  [M, hidden] binary16
 *   q_out_next  [M, hidden/2] bytes (or [M, hidden] when next_bits == 8), required iff s_out_next > 0
 * hidden % 8 == 0, ffn % 8 == 0, hidden % heads == 0 (else SHAPE); d_k = hidden / heads even and <= 64,
 * seq <= 4096, hidden <= 8192 (else UNSUPPORTED).
 * A hidden or FFN size that is no multiple of 32 (the 4-layer student of section 5.2: 312 and 1200) is
 * carried padded: every 4-bit code buffer whose rows feed a linear of that reduction length -- q_in,
 * q_out_next, the workspace's c0..c3 -- has rows of mkq_padded_k(size) / 2 bytes with zero codes past the
 * real columns (every kernel of the layer that writes codes writes the padding too), and the weights come from
 * mkq_pack_weights_int4_padded.  Sizes that are a multiple of 32 are stored as they are.
 * Errors: NULL, SHAPE, ALIGN, SCALE, DTYPE, WORKSPACE, UNSUPPORTED, HIP. */
int mkq_bert_layer_int4(const mkq_bert_layer_params *p_host, const void *h_in, int h_dtype,
                        const uint8_t *q_in, void *h_out, uint8_t *q_out_next, void *workspace,
                        size_t workspace_bytes, void *stream);

/* The same layer in the 16-bit float baseline (no quantizers). */
typedef struct mkq_bert_layer_params_fp16 {
    int64_t batch, seq, hidden, heads, ffn;
    const void *W_qkv, *W_ao, *W_up, *W_down; /* binary16 [N, K] */
    const float *b_qkv, *b_ao, *b_up, *b_down;
    const float *ln1_gamma, *ln1_beta, *ln2_gamma, *ln2_beta;
    float ln_eps;
    const int32_t *cu_seqlens; /* as in mkq_bert_layer_params */
    int64_t total_tokens;
} mkq_bert_layer_params_fp16;

size_t mkq_bert_layer_fp16_workspace_bytes(const mkq_bert_layer_params_fp16 *p_host);
int mkq_bert_layer_fp16(const mkq_bert_layer_params_fp16 *p_host, const void *h_in /* binary16 */,
                        void *h_out /* binary16 */, void *workspace, size_t workspace_bytes,
                        void *stream);

/* The same encoder layer with every linear W8A8 (an 8-bit layer of a mixed 4/8-bit model,
 * section 4.2; the int8 column of Table 2): the params struct is the one above with
 * Wq_* = int8 codes [N, K] from mkq_pack_weights_int8 and sx_* the steps of the 8-bit
 * range; every code buffer (q_in, q_out_next, the c* intermediates) holds one byte per
 * code, so the workspace layout has c0, c1, c2 of M*hidden bytes and c3 of M*ffn bytes.
 * Shape limits and errors of mkq_bert_layer_int4, but hidden % 64 == 0 and ffn % 64 == 0 (no padding). */
int mkq_bert_layer_int8_workspace(const mkq_bert_layer_params *p_host,
                                  mkq_bert_layer_workspace_layout *layout_host);
int mkq_bert_layer_int8(const mkq_bert_layer_params *p_host, const void *h_in, int h_dtype,
                        const int8_t *q_in, void *h_out, int8_t *q_out_next, void *workspace,
                        size_t workspace_bytes, void *stream);

/* Building blocks of the layer, exported for stage-wise parity checks.
 * LayerNorm over the last dimension in binary32 (section 5); x binary16 [M, D];
 * y binary16 [M, D] (may be NULL); q_out (NULL or [M, D/2]) receives
 * codes(y_binary32; s_next).  D % 8 == 0, D <= 8192. */
int mkq_layernorm(const void *x, int64_t M, int64_t D, const float *gamma, const float *beta,
                  float eps, void *y, float s_next, uint8_t *q_out, void *stream);

/* Attention core of section 3.2 on a fused binary16 qkv buffer [batch*seq, 3*hidden]:
 * ctx binary16 [batch*seq, hidden] (may be NULL) and/or q_out packed codes under s_next.
 * Scores are scaled by 1/sqrt(d_k), d_k = hidden / heads; the softmax runs in binary32 and its normalized
 * probabilities are narrowed to binary16 before they multiply v.
 * d_k even and <= 64, hidden % 8 == 0, seq <= 4096 (anything else: UNSUPPORTED).  d_k == 64 with
 * seq <= 128 takes a kernel that holds all keys of a (sequence, head) at once, other sequences of up to 512
 * keys with d_k <= 32 or a multiple of 8 one that holds the scores of a query in registers; the rest (longer
 * sequences, heads of 34 to 62 that are no multiple of 8, and batches or rows beyond what the second can address
 * or be launched for) one that walks the keys in blocks of 128, twice (row maximum and denominator, then the
 * weighted sum). */
int mkq_attention(const void *qkv, int64_t batch, int64_t seq, int64_t hidden, int64_t heads,
                  void *ctx, float s_next, uint8_t *q_out, void *stream);

/* Attention over a padding-free batch: qkv [total_tokens, 3*hidden], sequence b = rows
 * cu_seqlens[b] .. cu_seqlens[b+1] - 1 (device array [batch + 1]), each at most max_seq <= 4096 rows
 * (any length; an empty sequence is skipped).  q_out: codes of q_bits (4: [total, hidden/2] bytes,
 * 8: [total, hidden] bytes) or NULL.  Errors as mkq_attention, plus DTYPE for q_bits. */
int mkq_attention_varlen(const void *qkv, const int32_t *cu_seqlens, int64_t batch, int64_t max_seq,
                         int64_t hidden, int64_t heads, void *ctx, float s_next, void *q_out,
                         int q_bits, void *stream);

/* The two building blocks with 8-bit code output: q_out int8 [M, D] / [batch*seq, hidden]. */
int mkq_layernorm_int8(const void *x, int64_t M, int64_t D, const float *gamma, const float *beta,
                       float eps, void *y, float s_next, int8_t *q_out, void *stream);
int mkq_attention_int8(const void *qkv, int64_t batch, int64_t seq, int64_t hidden, int64_t heads,
                       void *ctx, float s_next, int8_t *q_out, void *stream);

/* Group-scaled 4-bit weights: a step for every `group` (32, 64 or 128) neighbours of a row.  One such matrix serves as the
 * table of mkq_embedding_int4_group and, tied, as the weights of mkq_linear_int4_group.
 *   rows    ceil(K / 32) * 16 bytes: the canonical nibble packing, zero codes from K up to the next multiple of 32; any K > 0
 *   steps   s_w [N, ceil(K / group)] binary32, step g of a row for its codes g * group .. ; the last group may be short
 * mkq_pack_weights_int4_group: W [N, K] of w_dtype (F32, F16, BF16), row stride ldw; every group's step is its abs-max / 7
 * (all zeros -> 1) unless s_w_in gives them (then > 0 and below 2^120, a precondition; for weights below 2^122 its own are), its codes are Eq. 1 of section 3.1
 * under that step; s_w_out may alias s_w_in.  N == 0 is a no-op.  Steps and biases of what follows need only the alignment of
 * a binary32 value, so that rows of a table can be passed on their own.
 * Errors: NULL, SHAPE (N < 0, K <= 0, ldw < K, group), ALIGN, DTYPE, UNSUPPORTED (N or K from about 2^31 on), HIP. */
size_t mkq_group_weight_bytes(int64_t N, int64_t K);
int mkq_pack_weights_int4_group(const void *W, int w_dtype, int64_t N, int64_t K, int64_t ldw, int group,
                                const float *s_w_in, float *s_w_out, uint8_t *Wq_out, void *stream);

/* Linear of few tokens on group-scaled 4-bit weights, activations in floats (the head over the vocabulary, single linears
 * of decoding or of a classifier):
 *     y[m,n] = sum_g s_w[n,g] ( sum_{k in g} x[m,k] c[n,k] ) + bias[n],  + residual, act, narrowed once to out_dtype
 * Activations and codes enter the products exactly, all sums are binary32.  (A binary32 activation is a sum of three bfloat16 numbers:
 * exactly from 2^-110 up, off by less than 2^-133 below.  A group's sum of |x c| reaches 2^128 only with activations near the end of
 * binary32's or bfloat16's range, and is then an infinity or a NaN before its step is applied.)  Infinities and NaN in a row
 * of x reach that row of y, as in IEEE arithmetic on the dequantized weights (GELU as x Phi(x): +infinity stays one, -infinity gives a NaN).
 *   x     [M, K] of x_dtype (F32, F16, BF16), row stride ldx (any; K a multiple of 8 in rows of a multiple of 16 bytes is faster)
 *   Wq, s_w  from mkq_pack_weights_int4_group with the same group;  bias [N] binary32 or NULL
 *   out   [M, N] of out_dtype (F32, F16, BF16)
 *   epi   NULL, or act and residual (residual_dtype F32, F16 or BF16); its code and accumulator outputs: UNSUPPORTED
 * Any M (made for up to 128 tokens), N and K, up to about 2^34 results (UNSUPPORTED); M == 0 is a no-op.  No workspace.
 * Errors: NULL, SHAPE (group, ldx < K, ...), ALIGN, DTYPE, UNSUPPORTED, HIP. */
int mkq_linear_int4_group(const void *x, int x_dtype, int64_t ldx, const uint8_t *Wq, const float *s_w, int group,
                          const float *bias, int64_t M, int64_t N, int64_t K, void *out, int out_dtype,
                          const mkq_epilogue *epi, void *stream);

/* Token rows: out[i,:] = scale * table[tokens[i],:], one multiplication in binary32 and one rounding to out_dtype per value.
 * A token outside [0, V) gives a row of zeros.
 *   tokens  [M] whole numbers of token_bits (32 or 64) bits, aligned to their own size
 *   table   [V, D] of table_dtype (F32, F16, BF16), row stride ld_table; or group-scaled 4-bit rows and their steps from
 *           mkq_pack_weights_int4_group (N = V, K = D): then a value is scale * (code * step), both products in binary32
 *   out     [M, D] of out_dtype (F32, F16, BF16), row stride ld_out (what lies between the rows is left as it is)
 *   scale   finite (sqrt(D) in some models, else 1)
 * Any D; multiples of 8 in rows that are multiples of 16 bytes are faster.  M == 0 is a no-op.
 * Errors: NULL, SHAPE, ALIGN, SCALE, DTYPE (token_bits too), UNSUPPORTED (V or D from about 2^31 on), HIP. */
int mkq_embedding(const void *tokens, int token_bits, int64_t M, const void *table, int table_dtype, int64_t V, int64_t D,
                  int64_t ld_table, float scale, void *out, int out_dtype, int64_t ld_out, void *stream);
int mkq_embedding_int4_group(const void *tokens, int token_bits, int64_t M, const uint8_t *Wq, const float *s_w, int group,
                             int64_t V, int64_t D, float scale, void *out, int out_dtype, int64_t ld_out, void *stream);

/* Gradient of the lookup with respect to its float table:
 *     grad[v,:] = scale * sum_{i: tokens[i] = v} dy[i,:]        (accumulate == 0: all V rows are written, zeros without a token)
 *     grad[v,:] += the same                                     (accumulate != 0: rows without a token are left as they are)
 * Tokens outside [0, V) and those equal to padding_token (a negative one: none) count for nothing.  The positions are sorted
 * by token and every row is summed in binary32 in an order that the tokens alone decide: equal calls give equal bits.  One
 * rounding to grad_dtype, behind the scale and the addition.
 *   dy    [M, D] of dy_dtype (F32, F16, BF16), row stride ld_dy
 *   grad  [V, D] of grad_dtype (F32, F16, BF16), row stride ld_grad (what lies between the rows is left as it is)
 *   workspace  at least mkq_embedding_gradient_workspace_bytes(M, D) bytes, 16-byte aligned; no preparation.  Two calls that may
 *              run at the same time need two.
 * M == 0 writes the zeros only (no workspace needed).
 * Errors: NULL, SHAPE, ALIGN, SCALE, DTYPE, WORKSPACE, UNSUPPORTED, HIP. */
size_t mkq_embedding_gradient_workspace_bytes(int64_t M, int64_t D);
int mkq_embedding_gradient(const void *tokens, int token_bits, int64_t M, const void *dy, int dy_dtype, int64_t ld_dy,
                           int64_t V, int64_t D, float scale, int64_t padding_token, int accumulate, void *grad,
                           int grad_dtype, int64_t ld_grad, void *workspace, size_t workspace_bytes, void *stream);

/* Norm over the gradients of n tensors, and their clipping to it:
 *     norm = sqrt(sum over all tensors and values of g^2)       (squares and sums binary64, in a fixed order)
 *     out  = c g,  c = min(1, max_norm / (norm + 1e-6))          (mkq_clip_gradients; one rounding per value)
 *   grads_host, counts_host, dtypes_host   host arrays [n]: device pointers, numbers of values, F32 / F16 / BF16 each; a tensor
 *                 is contiguous and aligned to its own element size (16 bytes are faster); one without values may be NULL
 *   outs_host     host array [n] of device pointers; outs_host[t] == grads_host[t] clips in place, otherwise it overlaps no
 *                 gradient; no two of them overlap (a tensor that is in the list twice would be scaled twice): UNSUPPORTED
 *   norm_out      device, the norm before clipping, binary32
 *   max_norm      > 0 (infinity: copies only, whatever the norm is)
 *   workspace     at least mkq_gradient_norm_workspace_bytes(n) bytes, 16-byte aligned; no preparation.  Two calls that may run
 *                 at the same time need two.
 * A NaN among the gradients makes the norm and, under a finite max_norm, all results NaN; an infinity makes the norm infinite and, under
 * a finite max_norm, c = 0 and itself NaN.
 * n == 0: the norm is 0.  Errors: NULL, SHAPE, ALIGN, SCALE, DTYPE, WORKSPACE, UNSUPPORTED, HIP. */
size_t mkq_gradient_norm_workspace_bytes(int64_t n);
int mkq_gradient_norm(int64_t n, const void *const *grads_host, const int64_t *counts_host, const int32_t *dtypes_host,
                      float *norm_out, void *workspace, size_t workspace_bytes, void *stream);
int mkq_clip_gradients(int64_t n, const void *const *grads_host, void *const *outs_host, const int64_t *counts_host,
                       const int32_t *dtypes_host, float max_norm, float *norm_out, void *workspace, size_t workspace_bytes,
                       void *stream);

/* Log probabilities of given tokens under rows of scores (of mkq_linear_int4_group as a head, or any other), entropies and the most
 * probable alternatives, in one pass over the scores; and the gradient of the first two.  With z = scale * logits[m,:]:
 *     normalizers[m] = (max_j logits[m,j],  L = log sum_j exp(z_j - max z)),    log p_j = z_j - max z - L
 *     log_probs[m]   = log p_t, t = tokens[m];  0 for a token outside [0, V)
 *     entropies[m]   = -sum_j p_j log p_j
 *     top_tokens[m]  = the `top` tokens with the largest scores, equal scores (0 and -0 too) by the lower token, with their log p
 *     grad[m,j]      = scale ( d_log_probs[m] (delta_jt - p_j)  -  d_entropies[m] p_j (log p_j + entropies[m]) )
 * -infinity forbids a token: p = 0, and its gradient is 0 but for the given token's own part, scale d_log_probs.  A row of nothing else has no distribution: log probabilities and L are -infinity,
 * the entropy is 0, its gradient zeros.  A NaN or +infinity makes its row's results NaN (a NaN is ordered as -infinity).  A row whose d_log_probs
 * (or whose token is outside) and d_entropies are 0 has zeros for a gradient, whatever its scores are.  top_log_probs have no gradient here.
 *   logits  [M, V] of dtype (F32, F16, BF16), row stride ld: any, rows are read in aligned pieces of 16 bytes
 *   scale   1 / temperature, 2^-100 .. 2^100;  tokens [M] of token_bits (32 or 64) bits, aligned to their own size
 *   normalizers [M, 2] (8-byte aligned), log_probs [M], entropies [M], top_tokens and top_log_probs [M, top] (NULL if top == 0): binary32, int32
 *   top     0 .. min(V, 64)
 *   workspace  at least mkq_token_log_probs_workspace_bytes(M, V, top) bytes (0: may be NULL), 16-byte aligned; no preparation.  Two calls
 *              that may run at the same time need two.
 *   grad    [M, V] of grad_dtype (F32, F16, BF16), row stride ld_grad (what lies between the rows is left as it is); the logits themselves if type
 *           and stride are theirs, otherwise apart from them (else UNSUPPORTED).  Strides that differ by no multiple of 8 are slower.
 *   d_log_probs [M];  d_entropies [M], or NULL (then entropies may be NULL)
 * Exponents and sums are binary32 (a probability below 2^-126 counts as 0), log probabilities are off by about 1e-7 plus as much of their own size.
 * Equal calls give equal bits.
 * M == 0 is a no-op.  Errors: NULL, SHAPE (top > V too), ALIGN, SCALE, DTYPE (token_bits too), WORKSPACE, UNSUPPORTED (top > 64), HIP. */
size_t mkq_token_log_probs_workspace_bytes(int64_t M, int64_t V, int top);
int mkq_token_log_probs(const void *logits, int dtype, int64_t ld, int64_t M, int64_t V, float scale, const void *tokens, int token_bits,
                        float *normalizers, float *log_probs, float *entropies, int top, int32_t *top_tokens, float *top_log_probs,
                        void *workspace, size_t workspace_bytes, void *stream);
int mkq_token_log_probs_gradient(const void *logits, int dtype, int64_t ld, int64_t M, int64_t V, float scale, const void *tokens,
                                 int token_bits, const float *normalizers, const float *entropies, const float *d_log_probs,
                                 const float *d_entropies, void *grad, int grad_dtype, int64_t ld_grad, void *stream);

/* Activations kept in 8 bits from the forward pass to the backward, with a step for every `group` (32, 64 or 128) neighbours of a row.
 *   step  = max|x| / 127 of the group (binary32, between 2^-126 and the largest of which 127 are finite; all zeros -> 1);  a group with an infinity or a NaN: step NaN, codes 0
 *   code  = x / step rounded to the nearest whole number, ties to even, decided exactly
 *   codes mkq_checkpoint_bytes(M, K): rows of ceil(K / 32) * 32 bytes, zero codes past K;  steps [M, ceil(K / group)] binary32
 * mkq_checkpoint_int8           x [M, K] of x_dtype (F32, F16, BF16), row stride ldx -> codes, steps
 * mkq_checkpoint_restore        out = act(code * step) of out_dtype (MKQ_ACT_NONE, or MKQ_ACT_GELU: what stood behind it), row stride ld_out
 * mkq_checkpoint_gelu_gradient  dx = dy (Phi(x) + x phi(x)), x = code * step; dx may be dy if type and stride are its own, otherwise it is apart
 *                               from it (else UNSUPPORTED)
 * Codes and steps lie apart from each other, from x, and from out and dx (else UNSUPPORTED).
 * What lies between rows of out and dx is left as it is.  Any K; multiples of 8 in rows that are multiples of 16 bytes are faster.
 * mkq_low_rank_adapters_gradient reads such rows in the place of x.  M == 0 is a no-op.
 * Errors: NULL, SHAPE (group too), ALIGN, DTYPE (act too), UNSUPPORTED, HIP. */
size_t mkq_checkpoint_bytes(int64_t M, int64_t K);
int mkq_checkpoint_int8(const void *x, int x_dtype, int64_t M, int64_t K, int64_t ldx, int group, int8_t *codes, float *steps, void *stream);
int mkq_checkpoint_restore(const int8_t *codes, const float *steps, int group, int64_t M, int64_t K, int act, void *out, int out_dtype,
                           int64_t ld_out, void *stream);
int mkq_checkpoint_gelu_gradient(const int8_t *codes, const float *steps, int group, int64_t M, int64_t K, const void *dy, int dy_dtype,
                                 int64_t ld_dy, void *dx, int dx_dtype, int64_t ld_dx, void *stream);

/* Low-rank adapters of many requests beside a shared projection.  Row m of a batch has the adapter a = adapter[m]; outside [0, R): none.
 *     hidden[m] = down_a x[m]                 out[m] = base[m] + s_a up_a^T hidden[m]
 * and their gradients, of the same rows, with u[m] = s_a up_a dy[m]:
 *     dx[m] = dx_base[m] + down_a^T u[m]      d_down_a = sum_m u[m] x[m]^T      d_up_a = s_a sum_m hidden[m] dy[m]^T
 * base is what the projection gave (mkq_linear_int4_group or any other: out itself will do), or NULL; out without a base may be the `residual` of a
 * linear whose epilogue follows.  A row without an adapter has hidden 0 and out = base (0 without one); an adapter without a row has gradients 0.
 *   x, dy       [M, K], [M, N] of their dtype (F32, F16, BF16), row strides ldx, ld_dy (any; multiples of 16 bytes are faster)
 *               x of the gradient also MKQ_I8: what mkq_checkpoint_int8 kept of it, with its steps and group (ldx is not read)
 *   adapter     [M] int32.  Rows of one adapter are best side by side; a tile of rows is gone through once for each of its adapters
 *   down, up    [R, rank, K], [R, rank, N] of w_dtype: the long side in rows, of both;  scales [R] binary32, or NULL: 1.  A smaller adapter
 *               has zeros in its last rows
 *   base, out   [M, N] of out_dtype;  dx_base, dx [M, K] of dx_dtype; their row strides.  A base is its result if the strides are the same, otherwise
 *               apart from it; out is apart from x, but may be other columns of one matrix of wider rows; dx is apart from dy and x (else UNSUPPORTED).
 *               What lies between the rows is left as it is
 *   hidden      [M, rank] binary32: an output of the first, apart from x and out, or NULL; needed for d_up
 *   d_down, d_up  [R, rank, K], [R, rank, N] of grad_dtype (F32, F16, BF16); accumulate: added to what is there, with one rounding.  dx, d_down and
 *               d_up may be NULL, but not all of them; what only they need may be NULL then.  They lie apart from each other, dx, dy, x and hidden, and dx
 *               from hidden (else UNSUPPORTED)
 *   workspace   at least the *_workspace_bytes bytes (0, for few rows: may be NULL), 16-byte aligned; no preparation.  Two calls that may run at
 *               the same time need two
 * All sums and hidden are binary32.  Products are exact, but that binary32 with binary32 may leave out 2^-24 of a product, and hidden values (u for dx)
 * under 16-bit results 2^-17 of one, of either sign; binary32 numbers enter as multiples of 2^-133.  Equal calls give equal bits.  Infinities and NaN of a row or an adapter reach the rows and gradients that depend on it, as infinities or NaN, and no others.
 * rank 1 .. 256, R up to 2^22 - 1, rank K and rank N below 2^29, K and N from 8 and, as the strides of base, out, dx_base and dx, up to 2^25
 * (UNSUPPORTED).  The gradient: R rank (K + N) below about 2^32 and, for d_down and d_up, R M up to 2^40 (UNSUPPORTED): the rows of each of the R adapters
 * are found by reading all M numbers, which shows from about 2^26 on (R = 10^5, M = 8192: 0.7 ms).  M == 0: the first does nothing, the second writes its zeros.
 * Errors: NULL, SHAPE (x_group too), ALIGN, DTYPE, WORKSPACE, UNSUPPORTED, HIP. */
size_t mkq_low_rank_adapters_workspace_bytes(int64_t M, int64_t K, int64_t N, int rank, int64_t R);
int mkq_low_rank_adapters(const void *x, int x_dtype, int64_t ldx, const int32_t *adapter, int64_t M, int64_t K, int64_t N, int rank, int64_t R,
                          const void *down, const void *up, int w_dtype, const float *scales, const void *base, int64_t ld_base, void *out,
                          int out_dtype, int64_t ld_out, float *hidden, void *workspace, size_t workspace_bytes, void *stream);
size_t mkq_low_rank_adapters_gradient_workspace_bytes(int64_t M, int64_t K, int64_t N, int rank, int64_t R);
int mkq_low_rank_adapters_gradient(const void *dy, int dy_dtype, int64_t ld_dy, const void *x, int x_dtype, int64_t ldx, const float *x_steps,
                                   int x_group, const int32_t *adapter, const float *hidden, int64_t M, int64_t K, int64_t N, int rank, int64_t R,
                                   const void *down, const void *up, int w_dtype, const float *scales, const void *dx_base, int64_t ld_dx_base,
                                   void *dx, int dx_dtype, int64_t ld_dx, void *d_down, void *d_up, int grad_dtype, int accumulate,
                                   void *workspace, size_t workspace_bytes, void *stream);

#ifdef __cplusplus
}
#endif
#endif /* MKQ_H */
