/*
 * sdq_mx4.h -- C-ABI of the microscaled 4-bit operators: quantization and product of plain (not decomposed) matrices, and the
 * mixture-of-experts layer of a few tokens over experts in that format.  Conventions, status codes and ownership as in sdq.h.
 *
 * Formats.  An element is an E2M1 code (0, 0.5, 1, 1.5, 2, 3, 4, 6 and a sign).
 *   SDQ_FMT_MXFP4  one E8M0 scale 2^(c - 127) per 32 elements of a row; scale_rule as for the decomposition's Q-Vectors
 *                  (SDQ_SCALE_OCP_FLOOR, SDQ_SCALE_CEIL_NOSAT).
 *   SDQ_FMT_NVFP4  one unsigned E4M3 scale per 16 elements under one fp32 factor per row.  sdq_mx4_quantize chooses the factor
 *                  2^t, t the smallest integer >= -126 with the row's largest magnitude <= 2688 * 2^t (0 for a row of zeros), and as
 *                  scale the E4M3 value nearest to a / (6 * 2^t) (ties to even, at least 2^-9 unless a = 0); scale_rule is
 *                  ignored.  sdq_mx4_import takes any factors (a per-tensor factor is the same one for every row).
 * Elements are the E2M1 values nearest to x / (scale * factor), ties to even, saturating; both formats decide as the exact
 * quotient does.  Infinities count as the largest finite number of their type.  A block that holds a NaN gets the NaN scale code,
 * and every product with it is NaN.
 *
 * Sizes.  Any R, K >= 1 (rows that end inside a block are quantized over the elements they have).  Rows may be strided;
 * pointers are aligned to their element, buffers to 256 bytes.  Every call asks for the device that is current.
 */
#ifndef SDQ_MX4_H_
#define SDQ_MX4_H_

#include "sdq.h"

#ifdef __cplusplus
extern "C" {
#endif

enum { SDQ_FMT_MXFP4 = 0, SDQ_FMT_NVFP4 = 1 };
enum { SDQ_BF16 = 0, SDQ_FP16 = 1, SDQ_FP32 = 2 };            /* element types of unquantized operands */
enum { SDQ_ROUTE_SOFTMAX = 0, SDQ_ROUTE_SIGMOID = 1 };

/* Host-side descriptor of a quantized matrix, or of the stacked matrices of E experts (plain data, may be copied; `dev`
 * stays owned by the caller) */
typedef struct {
  void* dev;
  size_t bytes;
  int64_t E, R, K;      /* E = 0: a linear matrix [R, K]; else E matrices [R, K] in the experts' layout */
  int32_t fmt;
  int32_t reserved;
  size_t factors;       /* byte offset of the row factors (NVFP4) */
} sdq_mx4_t;

/* Bytes of the buffer of an R x K matrix. */
sdq_status_t sdq_mx4_size(int64_t R, int64_t K, int32_t fmt, size_t* bytes);

/* X (device) [R][ldx] of `dtype` -> codes and scales in `buf`, in the tiled layout sdq_mx4_linear streams (a weight matrix and a
 * batch of activations are stored alike).  One launch.  Asynchronous on `stream`. */
sdq_status_t sdq_mx4_quantize(const void* X, int32_t dtype, int64_t R, int64_t K, int64_t ldx, int32_t fmt, int32_t scale_rule,
                              void* buf, size_t bytes, sdq_mx4_t* out, void* stream);

/* Codes and scales as checkpoints hold them -> the tiled layout.  codes (device) [R][ceil(K/2)], two to a byte, the lower k in the
 * low nibble; scales (device) [R][ceil(K/32)] E8M0 or [R][ceil(K/16)] E4M3 (its sign bit is not looked at); factor (device) [R] fp32, NVFP4 only, NULL = 1. */
sdq_status_t sdq_mx4_import(const uint8_t* codes, const uint8_t* scales, const float* factor, int64_t R, int64_t K, int32_t fmt,
                            void* buf, size_t bytes, sdq_mx4_t* out, void* stream);

/* The reverse: plain arrays of the same shapes (factor may be NULL).  Also for experts: rows e * R + r. */
sdq_status_t sdq_mx4_export(const sdq_mx4_t* q, uint8_t* codes, uint8_t* scales, float* factor, void* stream);

/* The values that are held, rounded to `dtype` (bf16 and fp32 hold them exactly unless they leave their range):
 * out (device) [R][ldo], for experts [E * R][ldo]. */
sdq_status_t sdq_mx4_dequantize(const sdq_mx4_t* q, void* out, int32_t dtype, int64_t ldo, void* stream);

/* Y [M][ldy] (dtype) = Xq Wq^T + bias, Xq [M, K] and Wq [N, K] of one format, products and sums in fp32 on the tensor core, bias
 * (device) [N] of `dtype` or NULL; rounded once.  Errors: SHAPE where K differs, UNSUPPORTED where the formats do or an
 * operand has the experts' layout.  A wait that gives up sets the flag that sdq_device_status reports. */
sdq_status_t sdq_mx4_linear(const sdq_mx4_t* Xq, const sdq_mx4_t* Wq, const void* bias, int32_t dtype, void* Y, int64_t ldy, void* stream);

/* The experts' form: E stacked matrices [E][R][K] in MXFP4. */
sdq_status_t sdq_mx4_experts_size(int64_t E, int64_t R, int64_t K, size_t* bytes);
/* W (device) [E][R][K] contiguous, of `dtype` */
sdq_status_t sdq_mx4_experts_quantize(const void* W, int32_t dtype, int64_t E, int64_t R, int64_t K, int32_t scale_rule,
                                      void* buf, size_t bytes, sdq_mx4_t* out, void* stream);
sdq_status_t sdq_mx4_experts_import(const uint8_t* codes, const uint8_t* scales, int64_t E, int64_t R, int64_t K,
                                    void* buf, size_t bytes, sdq_mx4_t* out, void* stream);

/* Router: logits = X Wr^T over the H channels, X [T][ldx] and Wr [E][ldw] of `dtype`; score = softmax over the E experts or
 * sigmoid; every token's k experts are those of the largest score + bias (bias (device) [E] fp32 or NULL; of equal ones the lowest
 * index first), in descending order; weight = score of the chosen, divided by their sum where `renorm`, times `scale`.
 * Logits, scores and choices are formed in 64 bits from fp32 partial sums: a logit is within 32 * 2^-23 (16-bit operands, sums of 32 products) or
 * 8 * 2^-24 (fp32, sums of 8) of the sum of its products' magnitudes, and the choice does not depend on the order of the channels where the gaps are wider than
 * that.  ids (device) [T][k] int32, weights (device) [T][k] fp32.
 * 1 <= k <= E <= 1024, k <= 32. */
sdq_status_t sdq_moe_route(const void* X, int32_t dtype, int64_t T, int64_t H, int64_t ldx, const void* Wr, int64_t E, int64_t ldw,
                           const float* bias, int32_t k, int32_t scoring, int32_t renorm, float scale,
                           int32_t* ids, float* weights, void* stream);

/* Experts: Y[t] = sum_j weights[t][j] * W2[e](silu(W1[e] x_t) * W3[e] x_t), e = ids[t][j].  X [T][ldx], Y [T][ldy] bf16 or fp16;
 * w1, w3 [E, I, H], w2 [E, H, I] in the experts' layout.  The activations are not quantized: the tensor core multiplies the 4-bit weights by
 * six E2M1 pieces whose sum is x, exactly down to 2^-9 (fp16: 2^-6) of the largest magnitude of its 32 channels and to 2^-17 of that
 * below, and never finer than 2^-128; the same for silu(.) * (.) in fp32.  A pair whose id lies outside [0, E) adds nothing.  1 <= T <= 64, 1 <= k <= 32.  A token that
 * holds an infinity or a NaN gives NaN.
 * ws (device): scratch of sdq_mx4_moe_workspace_size bytes, needs no initialisation; calls that can overlap on the GPU must not
 * share it. */
sdq_status_t sdq_mx4_moe_workspace_size(int64_t T, int32_t k, int64_t H, int64_t I, size_t* bytes);
sdq_status_t sdq_mx4_moe(const void* X, int32_t dtype, int64_t T, int64_t H, int64_t ldx, const int32_t* ids, const float* weights, int32_t k,
                         const sdq_mx4_t* w1, const sdq_mx4_t* w3, const sdq_mx4_t* w2, void* Y, int64_t ldy,
                         void* ws, size_t ws_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif
