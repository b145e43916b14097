/*
 * compact_block.h -- C ABI of the operators that stand next to the compressed linear layers in a transformer
 * block, for NVIDIA B200 (sm_100a): RMS norm with the residual's addition, quantisation to 8-bit floating point
 * with a scale for each 128 values, matrix products of such operands, and rotary positions.
 *
 * The conventions of compact.h hold: row-major matrices with a leading dimension in ELEMENTS, device pointers owned by
 * the caller, `stream` a cudaStream_t, calls asynchronous on it, arguments checked on the host before any launch,
 * a compact_status_t from every call, nothing allocated.  In addition:
 *   - Sizes may be any positive number (no multiple is asked for); base pointers are 16-byte aligned and pitches times
 *     the element size are multiples of 16 bytes, exactly as for the layers.  Scales are 4-byte aligned.
 *   - Zero rows are a successful call that launches nothing (a gradient of the weight is zeroed unless it accumulates).
 *
 * 8-bit matrices.  An element is e4m3 (4 exponent bits, largest finite value 448) or e5m2 (largest 57344).  Each 128
 * columns of a row share a scale, a power of two held as its exponent plus 127 in one byte (E8M0): the value of element
 * (i, k) is data[i, k] * 2^(scale[i, k / 128] - 127).  The scale is the least power of two that brings the largest
 * magnitude of its block inside the type's range (at least 2^-127; 1 for a block of zeros).  Scaling a floating-point number by a power of
 * two is exact, so this loses nothing against a 32-bit scale except part of one binade at the bottom of the range,
 * and the tensor cores take such scales as operands.  A block that holds an infinity or a NaN gets the scale byte 255, which is
 * NaN: every sum that a value of the block enters is NaN.  (With the values themselves an infinity could stay one, and of a 128 x 128 block only
 * the rows that hold such a value would be touched, not all 128.)
 * Layout of the scales of a matrix of `rows` x `cols`: groups of four column blocks,
 *     byte scales[(g * lds + i) * 4 + j] scales columns 128 (4 g + j) .. 128 (4 g + j) + 127 of row i,
 * g < compact_fp8_scale_groups(cols), lds >= rows.  Bytes of column blocks past the last one are written as 127 (scale 1).
 */
#ifndef COMPACT_BLOCK_H_
#define COMPACT_BLOCK_H_

#include "compact.h"

#ifdef __cplusplus
extern "C" {
#endif

typedef enum { COMPACT_E4M3 = 0, COMPACT_E5M2 = 1 } compact_fp8_t;

/* ceil(cols / 512): groups of four scales per row. */
int64_t compact_fp8_scale_groups(int64_t cols);

/* Rows to 8 bits, a scale for each 128 columns of a row (activations, gradients).
 * X [rows x cols] is COMPACT_F32 or COMPACT_BF16; Q gets one byte per element, rounded to nearest even. */
compact_status_t compact_quantize_rows(int dtype, int64_t rows, int64_t cols, const void* X, int64_t ldx,
                                       int fp8, void* Q, int64_t ldq, void* scales, int64_t lds, void* stream);

/* Blocks of 128 x 128 to 8 bits (weights): one scale for all 128 rows of a block, written for each of its rows.  Q and
 * scales hold X; QT [cols x rows] and scales_t hold its transpose with the same values and scales, so that both
 * orientations of a weight can be the K-major operand of a product from one pass over it.  Either pair may be NULL. */
compact_status_t compact_quantize_blocks(int dtype, int64_t rows, int64_t cols, const void* X, int64_t ldx,
                                         int fp8, void* Q, int64_t ldq, void* scales, int64_t lds,
                                         void* QT, int64_t ldqt, void* scales_t, int64_t lds_t, void* stream);

/* RMS norm.  For each of `tokens` rows of n:
 *     h = x + residual            (rounded to the dtype; h = x when residual is NULL, and H must then be NULL)
 *     rstd = 1 / sqrt(mean(h^2) + eps)     (eps finite, not negative; a row of zeros with eps = 0 gives NaN)
 *     y = h * rstd * weight
 * Any of the outputs Y (dtype) and Q with scales (e4m3 or e5m2 of the unrounded y, a scale for each 128 columns) may be
 * NULL, and rstd (fp32, one per token, what the backward needs) too.  H may be the same memory as X or residual. */
compact_status_t compact_rms_norm_fwd(int dtype, int64_t tokens, int32_t n, float eps,
                                      const void* X, int64_t ldx, const void* residual, int64_t ldr,
                                      const void* weight, void* H, int64_t ldh, void* Y, int64_t ldy, float* rstd,
                                      int fp8, void* Q, int64_t ldq, void* scales, int64_t lds, void* stream);

/* Its gradient.  H is what the forward normed (x itself if it had no residual):
 *     dx = rstd * (dy * weight) - h * rstd^3 * mean(dy * weight * h) + residual_grad
 *     dweight (fp32, n) = sum over tokens of dy * h * rstd
 * dx is the gradient of x and of the residual alike.  residual_grad (the gradient that reaches h past the norm), dX
 * or dweight may be NULL.  dX may be the same memory as dY or residual_grad.  accumulate != 0 adds to dweight.  The
 * order of the sum over tokens is fixed by (dtype, tokens, n) and by whether residual_grad is passed: results of the same call are
 * bitwise reproducible, wherever its matrices lie and whichever outputs it has.
 * workspace: compact_rms_norm_bwd_workspace_bytes(dtype, tokens, n) bytes, not needed when dweight is NULL. */
size_t compact_rms_norm_bwd_workspace_bytes(int dtype, int64_t tokens, int32_t n);
compact_status_t compact_rms_norm_bwd(int dtype, int64_t tokens, int32_t n,
                                      const void* dY, int64_t lddy, const void* H, int64_t ldh, const void* weight,
                                      const float* rstd, const void* residual_grad, int64_t ldr,
                                      void* dX, int64_t lddx, float* dweight, int accumulate,
                                      void* workspace, size_t workspace_bytes, void* stream);
#define COMPACT_RMS_NORM_MAX_N 16384

/* Rotary positions.  The first rot_dim elements of every head are turned in pairs: pair i of a token at position p by
 * the angle p * w_i, and multiplied by attention_factor.  Pairs are (2 i, 2 i + 1) when interleaved, (i, i + rot_dim / 2)
 * otherwise; the rest of the head passes through.  w_i = base^(-2 i / rot_dim), then
 *     COMPACT_ROTARY_LINEAR:   w_i / factor
 *     COMPACT_ROTARY_BASE:     the base is base * factor^(rot_dim / (rot_dim - 2))
 *     COMPACT_ROTARY_BY_PARTS: t = clamp((trained_length * w_i / 2 pi - low) / (high - low), 0, 1); w_i (t + (1 - t) / factor)
 * Angles are kept as 64-bit fractions of a turn, so they are as exact at position 10^6 as at 1.  A factor that makes the base zero or
 * infinite, or a w_i infinite, is refused. */
typedef enum { COMPACT_ROTARY_NONE = 0, COMPACT_ROTARY_LINEAR = 1, COMPACT_ROTARY_BASE = 2, COMPACT_ROTARY_BY_PARTS = 3 } compact_rotary_scaling_t;
typedef struct {
  int32_t head_dim, rot_dim;  /* rot_dim even, 2 <= rot_dim <= head_dim <= 1024, rot_dim <= 512 */
  int32_t interleaved;
  int32_t scaling;            /* compact_rotary_scaling_t */
  double base, factor, low, high, trained_length;   /* those the scaling does not use are ignored */
  float attention_factor;     /* 1 for none */
} compact_rotary_config_t;
typedef struct compact_rotary compact_rotary_t;  /* opaque, host side, never changes: may be used from several threads */
compact_status_t compact_rotary_create(const compact_rotary_config_t* cfg, compact_rotary_t** out);
compact_status_t compact_rotary_destroy(compact_rotary_t* rot);
/* Q [tokens x heads x head_dim] and K [tokens x kv_heads x head_dim] in one launch; K may be NULL with kv_heads = 0.
 * *_token and *_head are the strides, in elements, between tokens and between heads.  positions: one per token, int64
 * (pos_bits = 64) or int32 (32); NULL: token t is at first_position + t.  back != 0 applies the transpose (the gradient).
 * Outputs may be the inputs themselves; they must not overlap them in another way, nor themselves: an output's strides are at least
 * head_dim long (of a single token or head they are not used).  Those of an input are free. */
compact_status_t compact_rotary_apply(const compact_rotary_t* rot, int dtype, int64_t tokens, int32_t heads, int32_t kv_heads,
                                      const void* Q, int64_t q_token, int64_t q_head, const void* K, int64_t k_token, int64_t k_head,
                                      const void* positions, int pos_bits, int64_t first_position, int back,
                                      void* Qout, int64_t qo_token, int64_t qo_head, void* Kout, int64_t ko_token, int64_t ko_head,
                                      void* stream);

/* C [M x N] = A B^T with A [M x K] and B [N x K] in 8 bits with their scales; sums in fp32, C (COMPACT_BF16 or
 * COMPACT_F32) rounded once.  For a layer: Y = X W with B the transpose of W, dX = dY W^T with B = W itself.  Results are
 * bitwise reproducible.  The handle holds the status word of the kernels' bounded waits, nothing else; like a layer's, it must not
 * be used from two threads at once.  Operand pitches that are multiples of 128 are read fastest. */
typedef struct compact_fp8_product compact_fp8_product_t;
compact_status_t compact_fp8_product_create(compact_fp8_product_t** out);
compact_status_t compact_fp8_product_destroy(compact_fp8_product_t* p);
compact_status_t compact_fp8_product_run(compact_fp8_product_t* p, int64_t M, int64_t N, int64_t K,
                                         int a_type, const void* A, int64_t lda, const void* a_scales, int64_t lds_a,
                                         int b_type, const void* B, int64_t ldb, const void* b_scales, int64_t lds_b,
                                         int c_dtype, void* C, int64_t ldc, void* stream);
/* COMPACT_ERR_DEVICE_TIMEOUT if one of the handle's kernels has given up on a wait since the last call (its C is then not valid), on whichever
 * device and stream it ran, replayed from a graph or not; COMPACT_OK otherwise.  Synchronises the devices that the handle has launched
 * on.  After the handle is destroyed there is nobody to tell: one whose products matter outlives them. */
compact_status_t compact_fp8_product_status(compact_fp8_product_t* p);
/* Selects the kernel: 0 = automatic, 1 = pairs of SMs, 2 = clusters that split K (the tests compare the two).  Returns
 * the previous value. */
int compact_fp8_product_set_kernel(int which);
/* Test hook for the bounded waits: the handle's next product loads only the first `k_steps` of the 128-column steps of each tile's K (rounded
 * up to the even number that share a barrier), and its waits give up after a few thousand polls.  With fewer steps than K has, the
 * kernel gives up as it would after a lost copy: it returns, C is not valid, compact_fp8_product_status reports
 * COMPACT_ERR_DEVICE_TIMEOUT once, and the context stays usable.  k_steps < 0 takes the request back. */
compact_status_t compact_debug_fp8_product_withhold(compact_fp8_product_t* p, int32_t k_steps);
/* Test hook that makes the choice of tiles observable, on the host alone: plan[0] the kernel of an automatic product (as above), and of
 * the pairs' kernel plan[1] the columns of a tile, plan[2] the number of tiles, plan[3] the k-steps to a barrier, plan[4] the panels of
 * column tiles that B is taken in. */
compact_status_t compact_debug_fp8_product_plan(int64_t M, int64_t N, int64_t K, int32_t plan[5]);

#ifdef __cplusplus
}
#endif
#endif /* COMPACT_BLOCK_H_ */
