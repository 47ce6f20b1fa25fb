/*
 * hago.h -- C ABI of libhago: the quantized-operator hot path of HAGO
 * (arXiv 2103.14949, "Automated Backend-Aware Post-Training Quantization")
 * as hand-written HIP kernels for AMD MI355X (gfx950).
 *
 * The library exports the operators the paper's realization pass produces and
 * its search loop executes:
 *   hago_simquant   -- simulated_quantize (Sec. 4.2; Eq. 3; Sec. 5.2)
 *   hago_qdense     -- integer dense, integer accumulate, fused requantize
 *   hago_qconv2d    -- integer conv2d (groups == 1 or depthwise), same epilogue
 *   hago_requantize -- the standalone requantize operator (Sec. 6.1, 6.2)
 *   hago_simquant_batched -- several candidate settings over one tensor (Sec. 6.3)
 *   hago_absmax     -- max-abs calibration thresholds (Eq. 2)
 *   hago_quantize, hago_dequantize -- fp32 <-> integer codes (Sec. 6.1; Eq. 3)
 *   hago_simquant_codes -- simulated_quantize plus its integer codes, one pass
 *   hago_simquant_wrap  -- simulated_quantize with the overflow of the simulated
 *                          integer type (Sec. 5.2)
 *   hago_mx_quantize, hago_mx_rmsnorm, hago_mx_silu_mul, hago_mx_dense,
 *   hago_mx_dense_grouped -- microscaled (block-scaled) 4- and 8-bit floating
 *                          point: a transformer's layers on codes
 *   hago_rope, hago_mx_cache_write, hago_mx_cache_read, hago_mx_attention --
 *                          rotary positions, a paged cache of keys and values
 *                          on microscaled codes, attention over it
 * and the operand / accumulator variants the paper names: int16 x int16
 * operands, 24-bit accumulators (Sec. 4.1), shift-only requantize for
 * power-of-two scales (Sec. 5.1).
 *
 * Conventions common to every call
 *   - Pointers marked "device" are GPU addresses valid on the current HIP
 *     device; "host" are ordinary pointers.  The caller owns every buffer it
 *     passes: the library never frees or keeps such a pointer after returning.
 *   - No entry point allocates, frees or keeps device memory, and none waits
 *     for the device.  The two operators that want scratch memory, the
 *     groups == 1 convolution (it rewrites its operands before the matrix
 *     cores read them) and the attention (runs of keys meet there), take it
 *     from the caller: hago_qconv2d_ws, hago_mx_attention.
 *   - A call is kernel launches on `stream` and nothing else, so it may be
 *     recorded into a HIP graph.  The first call that reaches a kernel with a
 *     large LDS footprint raises that kernel's limit on the current device
 *     (hipFuncSetAttribute): make one ordinary call of the same operator and
 *     geometry before capturing.
 *   - Tensors are dense and contiguous in the stated order.  `out` must not
 *     overlap any input.  A tensor with zero elements may be passed as NULL.
 *   - `stream` is the caller's hipStream_t (NULL = the default stream).  Calls
 *     enqueue work on it and return without synchronizing.
 *   - Every argument error is detected on the host BEFORE anything is
 *     launched and reported as a status code; nothing is written in that
 *     case.  The CONTENTS of device arrays (multiplier, shift, scale) cannot
 *     be inspected without a synchronizing copy and are the caller's
 *     contract: multiplier in [0, 2^31), shift in [0, 31], scale finite and
 *     non-zero.
 *   - Quantization parameters that the search varies (scales, zero points,
 *     multipliers, shifts, clip limits, effective bits) are runtime arguments,
 *     never compile-time constants (Sec. 6.3, batched search).
 */
#ifndef HAGO_H_
#define HAGO_H_

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  HAGO_OK = 0,
  HAGO_ERR_NULL = 1,      /* a required pointer is NULL                          */
  HAGO_ERR_SHAPE = 2,     /* negative/zero/inconsistent dimension, bad groups,
                             bad layout, a size beyond the 32-bit index range   */
  HAGO_ERR_DTYPE = 3,     /* operand / accumulator / output dtype combination
                             that the operator does not define                  */
  HAGO_ERR_BITS = 4,      /* effective bits < 1 or > container width, zero point
                             or clip range outside the container / bit range    */
  HAGO_ERR_PARAM = 5,     /* other invalid scalar parameter (flags, per_channel) */
  HAGO_ERR_ACC_BOUND = 6, /* HAGO_STRICT_ACC16 set and K*Amax*Wmax > 32767       */
  HAGO_ERR_DEVICE = 7,    /* the HIP runtime refused the launch                  */
  HAGO_ERR_SCRATCH = 8    /* hago_qconv2d_static: the rewritten operands exceed
                             HAGO_STATIC_SCRATCH_BYTES                          */
} hago_status;

/* Container data types.  "Effective bits" (Sec. 2, Sec. 5.3) may be fewer
 * than the container's width: a 6-bit value is still stored in an int8. */
typedef enum {
  HAGO_U8 = 0,
  HAGO_I8 = 1,
  HAGO_I16 = 2,
  HAGO_I32 = 3,
  HAGO_F32 = 4,
  HAGO_I24 = 5, /* accumulator type only (Sec. 4.1: accelerators with 24-bit
                   accumulation): 24-bit two's complement, held sign-extended
                   in an int32; also a simulated type of hago_simquant_wrap */
  HAGO_BF16 = 6, /* real types of the microscaled operators, beside HAGO_F32:  */
  HAGO_F16 = 7   /* bfloat16 and IEEE binary16                                 */
} hago_dtype;

typedef enum {
  HAGO_NCHW = 0, /* activations [B,C,H,W], weights [O,C/g,KH,KW], out [B,O,OH,OW] */
  HAGO_NHWC = 1  /* activations [B,H,W,C], weights [O,KH,KW,C/g], out [B,OH,OW,O] */
} hago_layout;

/* flags */
#define HAGO_STRICT_ACC16 1u /* refuse 16-bit (and 24-bit) accumulation unless
                                the declared operand ranges prove that it
                                cannot overflow */
#define HAGO_WS_WEIGHTS_READY 2u /* hago_qconv2d_ws only: the workspace still
                                holds this layer's rewritten weights from an
                                earlier call with the same w, geometry and
                                workspace; only the activations are rewritten.
                                B, the output, the accumulator, bias, rq and
                                the activations may differ between the two */

/* A quantized tensor type: container, effective bit count, signedness of the
 * effective range, zero point.  `bits` is a CONTRACT on the value range
 * (signed b bits: [-2^(b-1), 2^(b-1)-1]; unsigned: [0, 2^b-1]); kernels never
 * mask operands to it.  It bounds the zero point and clip limits and feeds the
 * int16-accumulation overflow check. */
typedef struct {
  hago_dtype dtype;
  int32_t bits;
  int32_t is_signed;
  int32_t zero_point;
} hago_qtype;

/* Requantize epilogue (Sec. 6.1 realization; Sec. 6.2 "integer-only
 * computations"): for an accumulator acc of output channel c
 *     r   = floor(acc * multiplier[c] / 2^(31 + shift[c]) + 1/2)
 *     out = clip(r + out.zero_point, clip_lo, clip_hi)  cast to out.dtype
 * evaluated exactly in 64-bit integers (single rounding, ties toward
 * +infinity).  With rounding == HAGO_ROUND_HALF_AWAY, r is instead the nearest
 * integer to acc * multiplier[c] / 2^(31 + shift[c]) with halves away from
 * zero (the two tie rules of the compiler stack the paper generates code
 * with; the results differ, by one, exactly on negative ties).  The fastest
 * kernel variants implement the first rule; the second takes each operator's
 * more general variant.  ReLU / ReLU6 are expressed through clip_lo /
 * clip_hi in the output's quantized domain (Sec. 6.1).
 * multiplier == NULL selects the form for power-of-two scales (Sec. 5.1:
 * thresholds rounded to powers of two "make it possible to use shifting to
 * replace multiplication"): r is acc / 2^shift[c] rounded by the same tie
 * rule, shift 0..31 (0: r = acc).  The standalone operator then runs a kernel
 * without a multiplication; the fused epilogues use the identity
 * acc / 2^s = acc * 2^30 / 2^(31 + s - 1). */
typedef enum { HAGO_ROUND_UPWARD = 0, HAGO_ROUND_HALF_AWAY = 1 } hago_rounding;

typedef struct {
  const int32_t* multiplier; /* device, [channels] or [1]; Q31; NULL: shift only */
  const int32_t* shift;      /* device, [channels] or [1]; 0..31                */
  int32_t per_channel;       /* 0: entry 0 serves every channel; 1: one each    */
  hago_qtype out;            /* dtype HAGO_I8 or HAGO_U8; bits; zero_point      */
  int32_t clip_lo, clip_hi;  /* inclusive; within out's effective-bit range     */
  int32_t rounding;          /* HAGO_ROUND_UPWARD or HAGO_ROUND_HALF_AWAY       */
} hago_requant;

/*
 * simulated_quantize (Sec. 4.2 "Simulated Quantize Operator"; Eq. 3;
 * rounding and saturation errors of Sec. 5.2).  Elementwise over
 * x[outer, channels, inner] (device, fp32):
 *     y = (clip(rint(x / s) + z, clip_lo, clip_hi) - z) * s
 * in IEEE binary32 with true division, round-half-to-even and a
 * compare-select clip (NaN stays NaN, +-inf saturates, no -0 results).
 * s = scale[c], z = zero_point[c] (device, [channels]) when per_channel != 0,
 * else entry 0.  q names the simulated container / effective bits and bounds
 * clip_lo/clip_hi and nothing else.  y (device) may equal x (in place).
 * Errors: NULL, SHAPE (negative dim), DTYPE (q.dtype not U8/I8/I16/I32),
 * BITS (clip range outside q), DEVICE.  Empty tensors are a no-op.
 */
hago_status hago_simquant(const float* x, float* y, int64_t outer,
                          int64_t channels, int64_t inner, const float* scale,
                          const int32_t* zero_point, int32_t per_channel,
                          hago_qtype q, int32_t clip_lo, int32_t clip_hi,
                          void* stream);

/*
 * Quantized dense (Introduction: u8 x i8 -> i32, i8 x i8 -> i16 and
 * i16 x i16 -> i32 operand triples; Sec. 6.2: dense on the fast integer
 * instruction):
 *     acc[m,n] = bias[n] + sum_k (a[m,k] - a_t.zero_point) * w[n,k]
 * reduced modulo 2^32 (acc_dtype HAGO_I32), modulo 2^16 and sign-extended
 * (HAGO_I16, the int16-accumulation mode of Sec. 8.4) or modulo 2^24 and
 * sign-extended (HAGO_I24, Sec. 4.1; raw results are int32).  With rq != NULL (host
 * pointer to the struct) each accumulator is requantized with channel = n and
 * out is [M,N] of rq->out.dtype; with rq == NULL the raw accumulators are
 * stored as [M,N] int32 / int16.
 * a: device [M,K], HAGO_U8 or HAGO_I8.  w: device [N,K] HAGO_I8, symmetric
 * (w_t.zero_point must be 0).  bias: device [N] int32 or NULL.
 * Or both operands HAGO_I16 (int16 data, acc_dtype HAGO_I32 or HAGO_I24): there
 * is no 16-bit matrix instruction, so this triple runs as four byte products.
 * Errors: NULL, SHAPE (negative dims, > 2^31-1), DTYPE, BITS, PARAM,
 * ACC_BOUND (flags & HAGO_STRICT_ACC16 and acc_dtype I16 / I24 and
 * K * max|a - z_a| * max|w| over the declared bit ranges > 2^15 - 1 /
 * 2^23 - 1), DEVICE.
 * M == 0 or N == 0 is a no-op; K == 0 yields the bias.
 */
hago_status hago_qdense(const void* a, hago_qtype a_t, const void* w,
                        hago_qtype w_t, const int32_t* bias, int64_t M,
                        int64_t N, int64_t K, hago_dtype acc_dtype,
                        const hago_requant* rq, void* out, uint32_t flags,
                        void* stream);

/*
 * Quantized conv2d (same operand triples; Sec. 6.2 conv2d; depthwise is the
 * memory-bound MobileNet case of Sec. 8.3).  Cross-correlation, dilation 1:
 *     acc[b,o,y,x] = bias[o] + sum_{c,ky,kx} (a[b,c,y*sh+ky-ph,x*sw+kx-pw] - z_a)
 *                                            * w[o,c,ky,kx]
 * where taps outside the image contribute exactly 0 (the input is padded with
 * its zero point).  OH = (H + 2*pad_h - KH) / stride_h + 1 (floor), same for
 * OW.  groups must be 1, or equal C and O (depthwise).  Accumulator width,
 * requantize (channel = o) and raw output as for hago_qdense.
 * Errors as for hago_qdense; additionally SHAPE for any other `groups`, a
 * kernel larger than the padded image, stride < 1, pad < 0; DTYPE for int16
 * operands with groups != 1.
 * This entry point uses no scratch memory.  Every geometry runs as one launch
 * that reads the caller's tensors directly.  Depthwise, 1x1 stride-1 (either
 * layout) and NCHW 3x3 stride-1 pad-1 convolutions with C a multiple of 32 up
 * to 128 and W a multiple of 4 up to 128 (configs 2 and 3) have kernels that
 * hago_qconv2d_ws runs too.  Of the other groups == 1 geometries, where they
 * have enough output to fill the chip, hago_qconv2d_ws goes through the
 * workspace for filters beyond 9 taps, for up to 9 taps beyond 64 to 128
 * channels (by layout, W and size), and on small maps for channel-last layers
 * of whole 16-channel chunks and for layers of up to 16 channels
 * (channel-last; NCHW with W a multiple of 4 and more than 64 output
 * channels).  It runs the others as this entry point does.
 */
hago_status hago_qconv2d(const void* a, hago_qtype a_t, const void* w,
                         hago_qtype w_t, const int32_t* bias,
                         hago_layout layout, int64_t B, int64_t C, int64_t H,
                         int64_t W, int64_t O, int32_t KH, int32_t KW,
                         int32_t stride_h, int32_t stride_w, int32_t pad_h,
                         int32_t pad_w, int32_t groups, hago_dtype acc_dtype,
                         const hago_requant* rq, void* out, uint32_t flags,
                         void* stream);

/*
 * The same operator with caller-owned scratch memory (Sec. 6.2: conv2d on the
 * fast integer instruction).  The matrix cores read 16 consecutive reduction
 * elements per lane, so a groups == 1 convolution first rewrites, in one
 * launch, the activations into a padded channel-last int8 copy and the
 * weights into [O][KH*KW][C rounded up to 16] inside `workspace`, then runs
 * the implicit GEMM over the copies.  (Calls for which hago_qconv2d has a
 * kernel that is at least as fast run that kernel here too.  Without
 * HAGO_WS_WEIGHTS_READY they still write the weight part, except in 1x1 and
 * NCHW 3x3 layers that have a kernel of their own: those leave the workspace
 * untouched and never read weights that an earlier call left there.)
 *   hago_qconv2d_workspace_bytes  (host only, launches nothing): bytes this
 *     geometry wants; 0 when it runs without scratch (depthwise, or shapes
 *     only the general kernel indexes); -1 for arguments hago_qconv2d would
 *     refuse with SHAPE.  The weight copy comes first and its size does not
 *     depend on B.
 *   hago_qconv2d_ws: `workspace` is device memory, 256-byte aligned, of
 *     `workspace_bytes` >= that count (NULL / 0 allowed when the count is 0).
 *     Its contents need not be initialised and are overwritten; the library
 *     keeps no pointer to it after the call's work has run.  Calls that share
 *     one workspace must be ordered on one stream; calls with distinct
 *     workspaces may overlap freely.  With HAGO_WS_WEIGHTS_READY the weight
 *     part is taken as written by an earlier call without the flag (weights
 *     are constants of a layer) and only the activations are rewritten; a call
 *     whose count is 0 (B == 0 among them) writes none.
 * Results are identical to hago_qconv2d's.  Errors as for hago_qconv2d;
 * additionally NULL (workspace needed but NULL) and PARAM (workspace too
 * small, misaligned, or negative size).
 */
int64_t hago_qconv2d_workspace_bytes(hago_layout layout, int64_t B, int64_t C,
                                     int64_t H, int64_t W, int64_t O,
                                     int32_t KH, int32_t KW, int32_t stride_h,
                                     int32_t stride_w, int32_t pad_h,
                                     int32_t pad_w, int32_t groups);
hago_status hago_qconv2d_ws(const void* a, hago_qtype a_t, const void* w,
                            hago_qtype w_t, const int32_t* bias,
                            hago_layout layout, int64_t B, int64_t C, int64_t H,
                            int64_t W, int64_t O, int32_t KH, int32_t KW,
                            int32_t stride_h, int32_t stride_w, int32_t pad_h,
                            int32_t pad_w, int32_t groups, hago_dtype acc_dtype,
                            const hago_requant* rq, void* out, void* workspace,
                            int64_t workspace_bytes, uint32_t flags,
                            void* stream);

/*
 * hago_qconv2d for callers that cannot allocate device memory and have no
 * workspace to hand over: code under HIP graph capture, tight serving loops,
 * harnesses that forbid hipMalloc.  Same arguments and results as
 * hago_qconv2d_ws, but the scratch is a fixed array of
 * HAGO_STATIC_SCRATCH_BYTES of static device memory inside the library (each
 * GPU the library runs on holds its own copy until the process ends).  The
 * call allocates and frees nothing and does not wait for the device.
 * A geometry whose hago_qconv2d_workspace_bytes exceeds the array is refused
 * with HAGO_ERR_SCRATCH before anything is launched (use hago_qconv2d_ws).
 * Every call on a GPU uses that GPU's one array, which is overwritten by each
 * call: calls that may run at the same time on one GPU (different streams,
 * different host threads) race and must be ordered by the caller; calls on
 * one stream are safe.
 */
#define HAGO_STATIC_SCRATCH_BYTES (64ll << 20)
hago_status hago_qconv2d_static(const void* a, hago_qtype a_t, const void* w,
                                hago_qtype w_t, const int32_t* bias,
                                hago_layout layout, int64_t B, int64_t C,
                                int64_t H, int64_t W, int64_t O, int32_t KH,
                                int32_t KW, int32_t stride_h, int32_t stride_w,
                                int32_t pad_h, int32_t pad_w, int32_t groups,
                                hago_dtype acc_dtype, const hago_requant* rq,
                                void* out, uint32_t flags, void* stream);

/*
 * simulated_quantize with the overflow of the simulated integer type (Sec. 5.2
 * "Model Simulation": besides the rounding and the saturation error there is
 * "the overflow error, possible when the output of quantized operator is beyond
 * the limit of output data type can represent").  As hago_simquant, but the
 * code rint(x / s) + z is first reduced modulo 2^w into the range of q.dtype's
 * container: w = 8 (HAGO_I8 two's complement, HAGO_U8 0..255), 16 (HAGO_I16),
 * 24 (HAGO_I24) or 32 (HAGO_I32); then clipped to clip_lo..clip_hi (within
 * q's effective bits and +-2^24) and dequantized.  With q the accumulator
 * type of a quantized operator this reproduces, in the simulated graph, what
 * hago_qdense / hago_qconv2d with that acc_dtype do to a sum that does not fit.
 * A code of magnitude >= 4e18 or an infinite one reduces to 0; NaN stays NaN.
 * Errors as for hago_simquant.
 */
hago_status hago_simquant_wrap(const float* x, float* y, int64_t outer,
                               int64_t channels, int64_t inner,
                               const float* scale, const int32_t* zero_point,
                               int32_t per_channel, hago_qtype q,
                               int32_t clip_lo, int32_t clip_hi, void* stream);

/*
 * Batched candidate evaluation of simulated_quantize (Sec. 6.3 "Batched GPU
 * Search": quantization parameters are runtime arguments, and a batch of
 * candidate settings is evaluated in one go).  The tensor x[outer, channels,
 * inner] (device, fp32) is read once; candidate b = 0..nbatch-1 (at most 16)
 * writes y[b, outer, channels, inner] (device, fp32) = hago_simquant(x) with
 * scale[b*P + c], zero_point[b*P + c] (device; P = channels if per_channel
 * else 1) and the clip range clip_lo[b]..clip_hi[b] (HOST arrays, read before
 * the call returns).  q bounds every clip range as in hago_simquant (use the
 * widest candidate's bits).  y must not overlap x.
 * Errors: NULL, SHAPE, DTYPE, BITS (some clip range outside q or +-2^24),
 * PARAM (per_channel not 0/1, nbatch > 16), DEVICE.  Empty is a no-op.
 */
hago_status hago_simquant_batched(const float* x, float* y, int64_t outer,
                                  int64_t channels, int64_t inner,
                                  int32_t nbatch, const float* scale,
                                  const int32_t* zero_point,
                                  int32_t per_channel, hago_qtype q,
                                  const int32_t* clip_lo,
                                  const int32_t* clip_hi, void* stream);

/*
 * quantize and dequantize (Sec. 6.1: the operators with which the realized
 * graph enters and leaves the integer domain; the two halves of Eq. 3).
 *     q = clip(rint(x / s) + z, clip_lo, clip_hi)      stored as qt.dtype
 *     y = ((float)q - (float)z) * s
 * x, y: device fp32 [outer, channels, inner]; q: device, container qt.dtype
 * (HAGO_I8, HAGO_U8, HAGO_I16 or HAGO_I32), same shape.  s, z as for
 * hago_simquant.  The code is formed exactly as in hago_simquant (binary32
 * division, round half to even, compare-select clip), so
 * hago_dequantize(hago_quantize(x)) equals hago_simquant(x) bit for bit; a NaN
 * input takes the code of real zero, clip(z).  clip_lo/clip_hi must lie within
 * qt's effective-bit range and within +-2^24.  hago_dequantize converts q to
 * binary32 first (exact for |q| <= 2^24).
 * Errors: NULL, SHAPE, DTYPE (qt.dtype HAGO_F32 or unknown), BITS, PARAM
 * (per_channel not 0/1), DEVICE.  Empty tensors are a no-op.
 */
hago_status hago_quantize(const float* x, void* q, int64_t outer,
                          int64_t channels, int64_t inner, const float* scale,
                          const int32_t* zero_point, int32_t per_channel,
                          hago_qtype qt, int32_t clip_lo, int32_t clip_hi,
                          void* stream);
hago_status hago_dequantize(const void* q, hago_qtype qt, float* y,
                            int64_t outer, int64_t channels, int64_t inner,
                            const float* scale, const int32_t* zero_point,
                            int32_t per_channel, void* stream);

/*
 * simulated_quantize that also emits the integer codes it passes through
 * (Sec. 6.1: realization replaces simulated_quantize by operators on q, so the
 * codes are what the realized graph carries where the simulated graph carries
 * q * s; Eq. 3).  One pass over x: y = hago_simquant(x) and q = hago_quantize(x)
 * with the same arguments, bit for bit (a NaN stays NaN in y and takes the
 * code of real zero in q).  x, y: device fp32 [outer, channels, inner]; q:
 * device, container qt.dtype, same shape; none of them may overlap.
 * Errors as for hago_quantize.  Empty tensors are a no-op.
 */
hago_status hago_simquant_codes(const float* x, float* y, void* q,
                                int64_t outer, int64_t channels, int64_t inner,
                                const float* scale, const int32_t* zero_point,
                                int32_t per_channel, hago_qtype qt,
                                int32_t clip_lo, int32_t clip_hi, void* stream);

/*
 * Max-abs calibration (Sec. 2, Eq. 2: threshold = max |x|; Sec. 5.1 statistics
 * collection): the thresholds that Eq. 1 turns into the scales of
 * simulated_quantize.  x[outer, channels, inner] (device, fp32);
 *     threshold[c] = max over o, i of |x[o, c, i]|      (per_channel != 0)
 *     threshold[0] = max over the whole tensor           (per_channel == 0)
 * threshold (device) has `channels` entries, or one.  NaN elements are ignored
 * (they never win a comparison); an empty reduction gives 0; the result is
 * never -0.  The result is exact (a maximum does not depend on the order).
 * Errors: NULL, SHAPE (negative dim or overflowing element count), PARAM
 * (per_channel not 0/1), DEVICE.
 */
hago_status hago_absmax(const float* x, int64_t outer, int64_t channels,
                        int64_t inner, int32_t per_channel, float* threshold,
                        void* stream);

/*
 * Standalone requantize (Sec. 6.1, 6.2): acc[outer, channels, inner] (device,
 * HAGO_I32 or HAGO_I16; int16 is sign-extended) -> out of rq->out.dtype with
 * the same shape, channel = axis 1.  rq must be non-NULL.
 */
hago_status hago_requantize(const void* acc, hago_dtype acc_dtype,
                            int64_t outer, int64_t channels, int64_t inner,
                            const hago_requant* rq, void* out, void* stream);

/*
 * Microscaled values.  A row of `cols` real numbers is held as codes of 4 bits
 * (HAGO_MX_FP4: E2M1; magnitudes 0 .5 1 1.5 2 3 4 6) or 8 bits (HAGO_MX_FP8:
 * E4M3, largest 448) and one scale byte per block of 32 columns (E8M0: byte b
 * stands for 2^(b - 127), 255 for NaN); a value is its code times its block's
 * scale.  Rows are held in whole blocks of 128 columns, C = cols rounded up to
 * 128:
 *   codes   [rows, C / 2] (two columns a byte, the even one in the lower four
 *           bits) or [rows, C]; 16-byte aligned
 *   scales  [rows, C / 32]; 4-byte aligned
 * Columns behind `cols` hold zero codes, and blocks without a column the scale
 * byte 0; the products rely on that.
 * Encoding a block of largest magnitude m: the scale is 2^e with
 * e = max(floor(log2 m) - emax, -127), emax 2 or 8 (m = 0: e = -127); the code
 * is the one nearest to x / 2^e, ties to the code with an even last bit,
 * and the largest one for magnitudes beyond it.  The sign of zero is kept.  A
 * block that holds a NaN or an infinity gets the scale 255 and zero codes: all
 * of it stands for NaN.
 */
typedef enum { HAGO_MX_FP4 = 0, HAGO_MX_FP8 = 1 } hago_mx_format;

/*
 * The operators by rows.  x_t: HAGO_F32, HAGO_BF16 or HAGO_F16, the type of
 * every real tensor of the call; arithmetic is binary32, the norm's sum and
 * its root binary64.  x[rows, cols] may have any row_stride (in elements) of
 * at least its columns; all else is dense.  `values`, unless NULL, takes the
 * values that the codes stand for, rounded to x_t once, as [rows, cols]: the
 * simulated quantization of the same numbers (hago_simquant_codes returns both
 * too).
 *   hago_mx_quantize: codes of x.
 *   hago_mx_rmsnorm: h = x + residual (NULL: h = x), codes of
 *     y = h * rsqrt(mean(h^2) + eps) * gamma[col] (NULL: 1); residual_out,
 *     unless NULL, takes h rounded to x_t (the norm is of h before that
 *     rounding).  It may be residual itself, or x itself where
 *     row_stride == cols.
 *   hago_mx_silu_mul: x[rows, 2 cols]; codes of g / (1 + exp(-g)) * u with g
 *     the first cols columns of a row and u the others, within a few units of
 *     the last place of binary32 (of a product far below g's own size too; an
 *     infinite g has what the formula makes of it: g * u, or NaN where it is
 *     negative).
 * Errors: NULL (x, codes or scales), SHAPE (negative or beyond 2^31 - 129
 * columns or 2^62 elements, row_stride below the columns), DTYPE (x_t), PARAM
 * (format; eps negative or not finite; codes, scales misaligned, or a real
 * tensor that its elements do not align), DEVICE.  Empty tensors are a no-op.
 */
hago_status hago_mx_quantize(const void* x, hago_dtype x_t, int64_t rows,
                             int64_t cols, int64_t row_stride,
                             hago_mx_format format, void* codes, void* scales,
                             void* values, void* stream);
hago_status hago_mx_rmsnorm(const void* x, const void* residual,
                            const void* gamma, hago_dtype x_t, int64_t rows,
                            int64_t cols, int64_t row_stride, float eps,
                            hago_mx_format format, void* residual_out,
                            void* codes, void* scales, void* values,
                            void* stream);
hago_status hago_mx_silu_mul(const void* x, hago_dtype x_t, int64_t rows,
                             int64_t cols, int64_t row_stride,
                             hago_mx_format format, void* codes, void* scales,
                             void* values, void* stream);

/*
 * Products of microscaled operands: activations a of either format, weights w
 * of HAGO_MX_FP4, results of out_t (HAGO_F32, HAGO_BF16 or HAGO_F16) rounded
 * once from a binary32 sum.
 *   hago_mx_dense:
 *     out[m,n] = bias[n] + sum_k a[m,k] * w[n,k]       a [M,K], w [N,K]
 *   hago_mx_dense_grouped (the experts of a layer): T result rows in groups,
 *     group e = rows offsets[e] .. offsets[e+1] - 1, of its own length, none
 *     among them:
 *     out[t,n] = bias[e,n] + sum_k a[r(t),k] * w[e,n,k]
 *     r(t) = row_index[t], or t where row_index is NULL.  a [a_rows,K],
 *     w [experts,N,K], offsets [experts + 1] and row_index [T] (device,
 *     int32), bias [experts,N].  offsets do not decrease and lie in 0..T,
 *     row_index in 0..a_rows - 1: the caller's contract, as device arrays'
 *     contents are (other values give wrong results, never an access out of
 *     bounds).  Rows in no group are not written.  Nothing waits for the
 *     device: the launch depends on T and experts alone.
 * bias: device, binary32, or NULL.
 * 4-bit products are added exactly up to the binary32 rounding of the running
 * sum, and so are those of 8-bit activations for HAGO_F32 results.  For 16-bit
 * results of 8-bit activations the matrix instruction's own sum is taken: of
 * 16 k at a time (0..7 and 16..23 of a block of 32, or the other half) it cuts
 * every product towards zero to a multiple of 2^(E - 13), E the largest sum of
 * two exponents among them.  On normally distributed rows that is 2^-17.8 of
 * the root of the sum of the squared terms (rms; 2^-14.2 the most of 16384
 * results), at worst 15 * 2^-13 of each largest term.
 * Errors: NULL, SHAPE (negative dimensions, beyond 2^31 - 1, K beyond 2^22,
 * more than 2^31 - 1 tiles; a_rows == 0 with T > 0; indexed activations of 2^31
 * bytes and more), DTYPE (out_t), PARAM (format, misaligned operands), DEVICE.
 * T, M or N == 0 is a no-op, K == 0 yields the bias.
 */
hago_status hago_mx_dense(const void* a_codes, const void* a_scales,
                          hago_mx_format a_format, const void* w_codes,
                          const void* w_scales, const float* bias, int64_t M,
                          int64_t N, int64_t K, hago_dtype out_t, void* out,
                          void* stream);
hago_status hago_mx_dense_grouped(const void* a_codes, const void* a_scales,
                                  hago_mx_format a_format, int64_t a_rows,
                                  const int32_t* row_index,
                                  const void* w_codes, const void* w_scales,
                                  const float* bias, const int32_t* offsets,
                                  int64_t T, int64_t experts, int64_t N,
                                  int64_t K, hago_dtype out_t, void* out,
                                  void* stream);

/*
 * Rotary positions.  x[T, heads, dim] -> out: the pairs j < `pairs` of every
 * row's columns (a, b) = (j, j + pairs), or (2j, 2j + 1) for
 * HAGO_ROPE_NEIGHBOURS, turned by t = positions[axis[j], row] * frequencies[j]:
 *     out[a] = x[a] cos t - x[b] sin t      out[b] = x[b] cos t + x[a] sin t
 * and the columns from 2 pairs on as they are.  positions [axes, T] (time,
 * height, width or any others), frequencies [pairs], axis [pairs] (NULL: all 0)
 * are device arrays; a pair whose axis is not below `axes` has position 0 (the
 * caller's contract is that there is none).  The angle, its turns and their
 * fraction are binary64, so positions may be far; cosines and sums are binary32,
 * rounded once to x_t (HAGO_F32, HAGO_BF16 or HAGO_F16).
 * Rows and heads of x and out may have any distance (in elements), so that the
 * queries and keys of one product's result are turned by one call.  out may be x
 * with the same strides, and not overlap it otherwise.
 * Errors: NULL, SHAPE (negative; dim above 4096, heads above 65536, T beyond
 * 2^31 - 1, 2 pairs above dim, axes < 1; strides negative, or such that rows or heads of
 * out overlap), DTYPE, PARAM (order; misaligned for its elements; out is x with
 * other strides), DEVICE.  Empty tensors are a no-op.
 */
typedef enum { HAGO_ROPE_HALVES = 0, HAGO_ROPE_NEIGHBOURS = 1 } hago_rope_order;
hago_status hago_rope(const void* x, hago_dtype x_t, int64_t T, int64_t heads,
                      int64_t dim, int64_t row_stride, int64_t head_stride,
                      const int32_t* positions, int64_t axes,
                      const float* frequencies, const int32_t* axis,
                      int64_t pairs, hago_rope_order order, void* out,
                      int64_t out_row_stride, int64_t out_head_stride,
                      void* stream);

/*
 * A paged cache of keys and values on microscaled codes.  The codes of a token's
 * key are those that hago_mx_quantize makes of it, in whole blocks of 32 columns
 * (B = dim rounded up to 32, zero codes behind dim):
 *   codes   [pages, kv_heads, page_size, B / 2 or B], 16-byte aligned
 *   scales  [pages, kv_heads, page_size, B / 32]
 * and the same for values; keys and values may differ in their format.  Codes of
 * 8 bits that are no number (0x7f, 0xff), which the operators here never write,
 * must not be in the pages of a sequence.
 */
typedef struct {
  void* k_codes;
  void* k_scales;
  void* v_codes;
  void* v_scales;
  hago_mx_format k_format, v_format;
  int64_t pages, kv_heads, page_size, dim;
} hago_mx_cache;

/*
 * The sequences of a call, and which of its T rows are whose.  Position p of
 * sequence s lies in page table[s * table_stride + p / page_size], at place
 * p % page_size.  Its rows are offsets[s] .. offsets[s + 1] - 1, the last n of
 * the lengths[s] tokens that it has with them: row i of n has position
 * lengths[s] - n + i.  table [seqs, table_cols], lengths [seqs] and offsets
 * [seqs + 1] are device arrays of int32; nothing waits for the device.
 * A position below 0, at or behind table_cols * page_size, or whose entry is not
 * below `pages` (a page that a window has left behind, say: -1) has no place: it is not
 * written, not read, and no query sees it.  offsets do not decrease and lie in
 * 0..T, and no two positions of a call share a place: the caller's contract, as
 * device arrays' contents are (other values give wrong results, never an access
 * out of bounds).  Rows in no sequence are left as they are.
 */
typedef struct {
  const int32_t* table;
  const int32_t* lengths;
  const int32_t* offsets;
  int64_t seqs, table_cols, table_stride;
} hago_mx_sequences;

/*
 *   hago_mx_cache_write: the keys and values of T tokens, k and v [T, kv_heads,
 *     dim] with rows and heads at any distance (in elements), into their places.
 *     k_values and v_values, unless NULL, take the values that the codes stand
 *     for, rounded to x_t once, as [T, kv_heads, dim] (also of tokens
 *     without a place).
 *   hago_mx_cache_read: the values of the rows' codes, rounded to out_t, into k
 *     and v [T, kv_heads, dim]; rows without a place are left as they are.
 * Real types are HAGO_F32, HAGO_BF16 and HAGO_F16.
 * Errors: NULL (a pointer; the structs), SHAPE (negative; dim above 256,
 * kv_heads above 65536, a cache of 2^62 bytes, pages, T or seqs beyond 2^31 - 1,
 * page_size < 1, table_cols * page_size beyond 2^31 - 2^16, table_stride below
 * table_cols; negative strides), DTYPE, PARAM (formats; misaligned), DEVICE.
 * No tokens, sequences, heads or columns are a no-op.
 */
hago_status hago_mx_cache_write(const hago_mx_cache* cache,
                                const hago_mx_sequences* sequences,
                                const void* k, int64_t k_row_stride,
                                int64_t k_head_stride, const void* v,
                                int64_t v_row_stride, int64_t v_head_stride,
                                hago_dtype x_t, int64_t T, void* k_values,
                                void* v_values, void* stream);
hago_status hago_mx_cache_read(const hago_mx_cache* cache,
                               const hago_mx_sequences* sequences,
                               hago_dtype out_t, int64_t T, void* k, void* v,
                               void* stream);

/*
 * Attention of new tokens (one a sequence, a chunk, a prompt) over the cache that
 * holds their keys and values already:
 *     out[t, h] = sum_j e^(s_j) v_j / sum_j e^(s_j),   s_j = scale * q[t, h] k_j
 * over the positions j of t's sequence that t sees: 0 <= j < lengths[s] that have
 * a place, j <= p where `causal`, and j > p - window where window > 0 (p: t's own
 * position).  Head h reads the cache's head h / (heads / kv_heads).  lse [T,
 * heads], unless NULL, takes log(sum_j e^(s_j)).  A row that sees nothing gives
 * zeros, and -infinity there.  q has rows and heads at any distance, out is dense.
 * Codes and their scales go into the products as bfloat16, which holds them
 * (below 2^-126 they may count as zero); queries as one, two or three bfloat16 numbers
 * for HAGO_BF16, HAGO_F16 and HAGO_F32, probabilities as two, two and three: 2^-16,
 * 2^-16 and 2^-24 of each.  HAGO_BF16 calls of many rows (T * heads / kv_heads 33 * seqs
 * or more) and up to 128 columns hold a probability to 2^-11, and those below 2^-27 of a
 * row's largest to 2^-38 of that.  Sums are binary32, of probabilities up to 2^6 where
 * values are large (values of 2^120, queries and scores of 2^127 and more may leave its
 * range).  Scores may be large otherwise: the largest of a row's counts.
 * workspace: device, 256-byte aligned, hago_mx_attention_workspace_bytes(...) bytes at
 * least, of any contents; calls that may run at the same time need one each.
 * Errors: as above, and SHAPE (heads not a multiple of kv_heads, T * heads beyond
 * 2^27, seqs * kv_heads beyond 2^22; window negative), PARAM (scale
 * NaN or beyond 2^100; workspace too small or misaligned).
 * hago_mx_attention_workspace_bytes returns -1 for what the call would refuse.  What
 * it returns does not fall where T or seqs rise: room for the largest call, in both,
 * serves every smaller one of the same heads and columns, whichever kernel that has.
 */
int64_t hago_mx_attention_workspace_bytes(int64_t T, int64_t seqs,
                                          int64_t heads, int64_t kv_heads,
                                          int64_t dim);
hago_status hago_mx_attention(const hago_mx_cache* cache,
                              const hago_mx_sequences* sequences, const void* q,
                              hago_dtype q_t, int64_t T, int64_t heads,
                              int64_t q_row_stride, int64_t q_head_stride,
                              float scale, int32_t causal, int64_t window,
                              void* out, float* lse, void* workspace,
                              int64_t workspace_bytes, void* stream);

/* Static, NUL-terminated description of a status code. */
const char* hago_status_string(hago_status s);

/*
 * The inclusive range of integer codes that `bits` effective bits hold
 * (Sec. 2: a b-bit data type has 2^b bins; Sec. 5.3: fewer effective bits than
 * the container): signed [-2^(bits-1), 2^(bits-1)-1], unsigned [0, 2^bits-1].
 * These are the widest clip limits a call accepts for that bit count and the
 * defaults a binding should pass.  lo, hi: host pointers.  Errors: NULL, BITS
 * (bits < 1, > 32, or 32 unsigned, which int32 cannot hold).
 */
hago_status hago_bit_range(int32_t bits, int32_t is_signed, int32_t* lo,
                           int32_t* hi);

/*
 * Measurement probes, not part of the operator set: what this chip delivers
 * when a kernel does nothing but the bounding operation, printed by the
 * benchmark beside the published peaks.
 *   hago_probe_mfma_i8: `workgroups` workgroups of four wavefronts each issue
 *     16 * iters int8 matrix instructions (32x32x32) back to back on the operands
 *     at `operands` (device, 8192 bytes, read once; real data matters, the clock
 *     under matrix-core load depends on it); 2 * 32*32*32 * 16 * iters *
 *     workgroups operations in all.  sink: device, 4 bytes, practically never
 *     written.
 *   hago_probe_copy: streaming copy of `bytes` (a multiple of 16, 16-byte aligned
 *     device pointers) with the elementwise kernels' access pattern.
 * Errors: NULL, SHAPE, PARAM (alignment), DEVICE.
 */
hago_status hago_probe_mfma_i8(const void* operands, void* sink,
                               int32_t workgroups, int32_t iters, void* stream);
hago_status hago_probe_copy(const void* src, void* dst, int64_t bytes,
                            void* stream);

/*
 * Test hook, not part of the operator set: forces which GEMM kernel family
 * and tile shape serve the following hago_qdense / hago_qconv2d* calls of
 * this process, so that tests can compare every variant with the oracle on
 * one shape.  Results never depend on it (but for the order in which the
 * microscaled products add, each kernel's own).  Keys:
 *   HAGO_HOOK_GEMM_PATH     0 automatic; 1 the general register-staged kernel;
 *                           2 the streaming kernel, skipping the one-launch
 *                           convolution kernels; 3 the general one-launch
 *                           convolution kernel; 4 the convolution kernels
 *                           without staging; 5 the streaming kernel on the
 *                           caller's channel-last tensor
 *   HAGO_HOOK_STREAM_TILE   -1 automatic; 0..6 a tile of the streaming dense kernels
 *                           (3 is 2)
 *   HAGO_HOOK_GENERAL_TILE  -1 automatic; 0..6 a tile of the general convolution
 *                           kernel (modulo 5: a form of the general dense kernel)
 *   HAGO_HOOK_MX_KERNEL     -1 automatic; 0.. a kernel of the microscaled products
 * Unknown keys are ignored.
 */
#define HAGO_HOOK_GEMM_PATH 0
#define HAGO_HOOK_STREAM_TILE 1
#define HAGO_HOOK_GENERAL_TILE 2
#define HAGO_HOOK_MX_KERNEL 3
void hago_set_test_hook(int32_t key, int32_t value);

#ifdef __cplusplus
}
#endif
#endif /* HAGO_H_ */
