/*
 * rudra_learner.h -- the learner's side of the parameter server's two messages, for learners that
 * compute on the same GPU as the server: weights in 4 bits and the product with them, activation
 * checkpoints in 8 bits and the backward pass that reads them.
 *
 * Beside them what a residual network's learner needs: weights and activations in 8-bit floating point and
 * the product with them, the norm in front of a layer with its backward pass, and the clipping of what is pushed.
 *
 * A learner of Section 2 (Gupta, Zhang, Wang, arXiv 1509.04210) pulls weights, runs a mini-batch
 * forward and backward and pushes a gradient.  With lambda learners to a GPU its memory and its
 * bandwidth are shared lambda ways, so what each learner holds is made small: the weights it
 * pulled take 4.25 bits each, the activations it keeps for its backward pass 8.25 bits.  One linear
 * layer of a learner is then
 *     pull      rudra_ps_pull_mx4 (as they stand, and transposed for the backward product)
 *     forward   rudra_act8_forward (RUDRA_ACT_NONE: keep x), rudra_mx4_linear
 *     backward  rudra_act8_weight_grad straight into the vector rudra_ps_push takes,
 *               rudra_mx4_linear on the transposed weights for the gradient of x,
 *               rudra_act8_backward through the activation function.
 *
 * Conventions are those of rudra_ps.h: plain C, codes < 0 with the reason in rudra_last_error(),
 * nothing thrown or aborted, all work enqueued on cuda_stream (NULL: the legacy default stream) of
 * the current device and asynchronous to the host, nothing allocated, no state between calls but which
 * streams rudra_learner_sync has told of what.
 * Matrices are row-major; ld is the distance between rows in elements (ld >= row length) and a
 * matrix of dtype may start at any multiple of its element size; rows on 32-byte boundaries are the
 * fastest.  What lies between the rows of a matrix that is read may be read too, but is not used;
 * what lies between the rows of a matrix that is written is left alone.  Sizes may be zero (a sum
 * over nothing is zero) and are at most RUDRA_MAX_DIM each.  Outputs must not overlap inputs, except
 * that rudra_act8_backward may write a gradient over dy where both have one layout.
 */
#ifndef RUDRA_LEARNER_H
#define RUDRA_LEARNER_H

#include "rudra_ps.h"

#ifdef __cplusplus
extern "C" {
#endif

#define RUDRA_F32  0   /* dtype of a matrix: float (RUDRA_GRAD_F32)      */
#define RUDRA_BF16 1   /* dtype of a matrix: bfloat16 (RUDRA_GRAD_BF16)  */
#define RUDRA_MAX_DIM 2147483520   /* most rows or columns of a matrix (2^31 - 128) */

/*
 * MX4: a matrix in microscaled 4-bit floating point (the OCP MXFP4 format).  32 consecutive values
 * of a row form a block (a row's last block may be short).  With E the exponent field of the block's
 * largest magnitude as a float, the block's scale byte is s = max(E - 2, 0) and stands for
 * 2^(s - 127); a value is the E2M1 number {0, 0.5, 1, 1.5, 2, 3, 4, 6} with a sign that is nearest
 * to x * 2^(127 - s), ties to the even code, magnitudes above 6 as 6.  A block that holds an infinity
 * or a NaN has s = 255, and all of it stands for NaN.  Values are exact in bf16.
 *
 * codes: rows of 16 * ceil(cols / 32) bytes, two codes to a byte, the lower column in the low half.
 * scales: the byte of row r, block b sits at
 *     ((r / 128) * ceil(nb / 4) + b / 4) * 512 + (r % 32) * 16 + (r % 128) / 32 * 4 + b % 4,
 * nb = ceil(cols / 32), which is the order the tensor cores take them in.  rudra_mx4_codes_bytes and
 * rudra_mx4_scales_bytes give the sizes; both arrays start on 32-byte boundaries.  Codes past cols
 * and scale bytes of blocks past nb are zero; scale bytes of rows past the last are never used.
 */
uint64_t rudra_mx4_codes_bytes(uint64_t rows, uint64_t cols);
uint64_t rudra_mx4_scales_bytes(uint64_t rows, uint64_t cols);

/* src (rows x cols of dtype) to MX4.  transpose != 0: the MX4 matrix is src's transpose (cols x
 * rows), with its blocks along src's columns: what the backward product needs, where the sum runs
 * over a layer's outputs. */
int rudra_mx4_quantize(const void* src_dev, int dtype, uint64_t rows, uint64_t cols, uint64_t ld, int transpose,
                       void* codes_dev, void* scales_dev, void* cuda_stream);

/* The values an MX4 matrix (rows x cols) stands for, as dtype. */
int rudra_mx4_dequantize(const void* codes_dev, const void* scales_dev, uint64_t rows, uint64_t cols, void* dst_dev,
                         int dtype, uint64_t ld, void* cuda_stream);

/* A pull in 4 bits: quantizes the rows x cols matrix (row-major, contiguous) that starts at weight
 * `offset` of the server's vector, as of every update issued so far, on the handle's stream, and
 * returns the weights' timestamp.  0.53 bytes per weight are written instead of a pull's 4.  The arrays are memory of
 * the handle's device; ordering other streams' use of them with the handle's stream is the caller's part. */
int64_t rudra_ps_pull_mx4(rudra_ps* ps, uint64_t offset, uint64_t rows, uint64_t cols, int transpose, void* codes_dev,
                          void* scales_dev);

/* The same for a caller that works on cuda_stream (of the handle's device): the arrays are written after all that
 * cuda_stream holds at the call, and what it is given later runs after they are written.  Both orders are kept on
 * the device; one stream for both costs nothing. */
int64_t rudra_ps_pull_mx4_on(rudra_ps* ps, uint64_t offset, uint64_t rows, uint64_t cols, int transpose, void* codes_dev,
                             void* scales_dev, void* cuda_stream);

/* The CUDA device a handle lives on (the one current at its creation). */
int rudra_ps_device(const rudra_ps* ps);

/* y[m][n] = sum over k of a[m][k] * b[n][k], a (m x k) and b (n x k) in MX4: products exact, sums in
 * 32 bits, one rounding to y's dtype.  A sum stays in one accumulator (a few where a tile is split), which the tensor
 * core cuts off where it adds to it: sums over 9 216 values came out within 2e-7 of themselves, over a million of
 * blocks whose scales differ by 2^11 within 4e-5.  The order of a sum depends on m, n, k and the device alone. */
int rudra_mx4_matmul(const void* a_codes_dev, const void* a_scales_dev, uint64_t m, const void* b_codes_dev,
                     const void* b_scales_dev, uint64_t n, uint64_t k, void* y_dev, int y_dtype, uint64_t ldy,
                     void* cuda_stream);

/* The same with a = x (m x k of x_dtype) brought to MX4 inside the call: a linear layer without
 * bias.  workspace_dev: rudra_mx4_linear_workspace(m, k) bytes (zero for few rows) on a 32-byte boundary,
 * free for other use once the call's work has run. */
uint64_t rudra_mx4_linear_workspace(uint64_t m, uint64_t k);
int rudra_mx4_linear(const void* x_dev, int x_dtype, uint64_t ldx, uint64_t m, const void* w_codes_dev,
                     const void* w_scales_dev, uint64_t n, uint64_t k, void* y_dev, int y_dtype, uint64_t ldy,
                     void* workspace_dev, uint64_t workspace_bytes, void* cuda_stream);

/*
 * ACT8: an activation matrix (tokens x channels) in 8 bits.  32 consecutive values of a row form a
 * block; with E as above the scale byte is s = max(E - 6, 0), a value is an integer of at most 127
 * in magnitude, the nearest (ties to even) to x * 2^(127 - s), and stands for itself times
 * 2^(s - 127).  s = 255 (an infinity or NaN in the block): the block stands for NaN.  Values are off
 * by at most 1/127 of the block's largest magnitude, and exact in bf16.
 *
 * codes: int8, rows of 32 * ceil(channels / 32) bytes, codes past channels zero; scales: rows of
 * 16 * ceil(channels / 512) bytes, one for each block and the rest unused.  Both arrays start on
 * 32-byte boundaries.
 */
uint64_t rudra_act8_codes_bytes(uint64_t tokens, uint64_t channels);
uint64_t rudra_act8_scales_bytes(uint64_t tokens, uint64_t channels);

#define RUDRA_ACT_NONE   0 /* f(x) = x: rudra_act8_forward keeps the checkpoint only (y_dev NULL)     */
#define RUDRA_ACT_RELU   1 /* max(x, 0), slope 0 at 0                                                 */
#define RUDRA_ACT_SILU   2 /* x / (1 + exp(-x))                                                       */
#define RUDRA_ACT_GELU   3 /* x / (1 + exp(-2u)), u = sqrt(2 / pi) (x + 0.044715 x^3)                 */
#define RUDRA_ACT_SWIGLU 4 /* silu(x) * up: two inputs, two checkpoints                               */

/* y = f(x), and the checkpoint of x, in one pass; y has x's dtype and is computed from x itself, in
 * 32 bits (a sigmoid of argument z is off by (8 + 4 |z|) * 2^-23 of itself at most, and 0 below 2^-126).  RUDRA_ACT_SWIGLU: up_dev (same dtype, shape and ld as x) is the second input and
 * up_codes_dev / up_scales_dev its checkpoint; NULL otherwise. */
int rudra_act8_forward(int act, const void* x_dev, const void* up_dev, int dtype, uint64_t tokens, uint64_t channels,
                       uint64_t ldx, void* y_dev, uint64_t ldy, void* codes_dev, void* scales_dev, void* up_codes_dev,
                       void* up_scales_dev, void* cuda_stream);

/* dx = dy * f'(xhat) with xhat from the checkpoint (RUDRA_ACT_NONE: dx = xhat, the checkpoint
 * expanded; dy_dev is NULL).  RUDRA_ACT_SWIGLU: dx = dy * uphat * silu'(xhat), dup = dy *
 * silu(xhat).  dy, dx and dup have one dtype; dx and dup have one ld. */
int rudra_act8_backward(int act, const void* dy_dev, int dtype, uint64_t tokens, uint64_t channels, uint64_t lddy,
                        const void* codes_dev, const void* scales_dev, const void* up_codes_dev,
                        const void* up_scales_dev, void* dx_dev, void* dup_dev, uint64_t lddx, void* cuda_stream);

/* dw[n][k] = sum over t of dy[t][n] * xhat[t][k] with xhat (tokens x k) from the checkpoint: the weight
 * gradient of a linear layer, written as dtype dw_dtype wherever the layer lies in the vector that
 * rudra_ps_push takes (lddw = k there).  Products are exact, sums in 32 bits; the result does not
 * depend on the run.  The tensor core cuts a sum off where it adds to it, every 16 tokens: f32 results are therefore gathered,
 * with rounding, every 512 tokens (128 for f32 dy), and so are bf16 results of more than 65 536 tokens (21 824 for f32 dy);
 * up to there positive terms add up to at most 2e-4 too little, a tenth of what the rounding to bf16 takes off.
 * dy of RUDRA_F32 is taken at full precision down to 2^-133; smaller parts of a value are cut off.  workspace_dev:
 * rudra_act8_weight_grad_workspace(...) bytes (zero where dy is bf16 with 16-byte-aligned rows) on a
 * 32-byte boundary. */
uint64_t rudra_act8_weight_grad_workspace(const void* dy_dev, int dy_dtype, uint64_t tokens, uint64_t n, uint64_t lddy);
int rudra_act8_weight_grad(const void* dy_dev, int dy_dtype, uint64_t lddy, uint64_t tokens, uint64_t n,
                           const void* codes_dev, const void* scales_dev, uint64_t k, void* dw_dev, int dw_dtype,
                           uint64_t lddw, void* workspace_dev, uint64_t workspace_bytes, void* cuda_stream);

/*
 * FP8: a matrix in 8-bit floating point with a scale for each block.  128 consecutive values of a row (or, square, 128 rows
 * of them) form a block (the last of a row may be short).  The block's scale byte s stands for 2^(s - 127),
 * the smallest power of two (s >= 0) under which its largest magnitude is at most 448; a value is the E4M3
 * number (largest 448, smallest 2^-9, three bits after the leading one) nearest to x * 2^(127 - s), ties to the even
 * code.  A block that holds an infinity or a NaN has s = 255, and all of it stands for NaN.  Values are off by at most 1/16 of
 * themselves or 2^-17 of the block's largest magnitude, whichever is more, and exact in float (magnitudes from 248 * 2^120 on
 * stand for 2^128, an infinity there); in bf16 too down to 2^-130.
 *
 * codes: rows of 128 * ceil(cols / 128) bytes, codes past cols zero.  scales: a byte for each row and block, square or not, in
 * the order that MX4 has them in, with nb = ceil(cols / 128).  Both arrays start on 32-byte boundaries; scale
 * bytes of blocks past nb are zero, those of rows past the last are never used.
 */
uint64_t rudra_fp8_codes_bytes(uint64_t rows, uint64_t cols);
uint64_t rudra_fp8_scales_bytes(uint64_t rows, uint64_t cols);

/* src (rows x cols of dtype) to FP8.  transpose != 0: the FP8 matrix is src's transpose (cols x rows).  square == 0: blocks run
 * along the rows of the result.  square != 0: blocks of 128 x 128, so that a matrix and its transpose have the same
 * values: for weights, which forward and backward pass both read. */
int rudra_fp8_quantize(const void* src_dev, int dtype, uint64_t rows, uint64_t cols, uint64_t ld, int transpose, int square,
                       void* codes_dev, void* scales_dev, void* cuda_stream);

/* The values an FP8 matrix (rows x cols) stands for, as dtype. */
int rudra_fp8_dequantize(const void* codes_dev, const void* scales_dev, uint64_t rows, uint64_t cols, void* dst_dev,
                         int dtype, uint64_t ld, void* cuda_stream);

/* rudra_ps_pull_mx4 and rudra_ps_pull_mx4_on with the matrix in FP8, its blocks square: 1.01 bytes per weight. */
int64_t rudra_ps_pull_fp8(rudra_ps* ps, uint64_t offset, uint64_t rows, uint64_t cols, int transpose, void* codes_dev,
                          void* scales_dev);
int64_t rudra_ps_pull_fp8_on(rudra_ps* ps, uint64_t offset, uint64_t rows, uint64_t cols, int transpose, void* codes_dev,
                             void* scales_dev, void* cuda_stream);

/* y[m][n] = sum over k of a[m][k] * b[n][k], a (m x k) and b (n x k) in FP8: products exact, sums in 32 bits, one rounding to
 * y's dtype.  With a transposed quantization of both factors it is a layer's weight gradient.  The tensor core cuts a sum off
 * where it adds to it, every 32 values; f32 results are gathered, with rounding, every 64 blocks or so: rows of 9 216 to 2^20 normal
 * values came out within 6e-7 of their sums' 2-norm, positive ones 5e-6 too little at most; bf16 results are gathered every
 * 512 blocks: positive values add up to at most 2e-4 too little however long the rows, a twentieth of what the rounding to bf16 takes off.
 * The order of a sum depends on m, n, k, y's dtype and the device alone. */
int rudra_fp8_matmul(const void* a_codes_dev, const void* a_scales_dev, uint64_t m, const void* b_codes_dev,
                     const void* b_scales_dev, uint64_t n, uint64_t k, void* y_dev, int y_dtype, uint64_t ldy,
                     void* cuda_stream);

/* The same with a = x (m x k of x_dtype) brought to FP8 inside the call, by pieces of rows.  workspace_dev:
 * rudra_fp8_linear_workspace(m, k) bytes (zero for few rows) on a 32-byte boundary, free for other use once
 * the call's work has run. */
uint64_t rudra_fp8_linear_workspace(uint64_t m, uint64_t k);
int rudra_fp8_linear(const void* x_dev, int x_dtype, uint64_t ldx, uint64_t m, const void* w_codes_dev,
                     const void* w_scales_dev, uint64_t n, uint64_t k, void* y_dev, int y_dtype, uint64_t ldy,
                     void* workspace_dev, uint64_t workspace_bytes, void* cuda_stream);

/*
 * Root-mean-square norm with the residual's addition, a row (token) at a time:
 *     s = x + residual, rounded to dtype;   y = s * weight / sqrt(mean(s^2) + eps)
 * computed from the rounded s in 32 bits (rows whose squares add up to 2^128 or more are out of range; squares below 2^-126 are
 * lost, which shows where eps is that small).  x, residual,
 * sum and y are tokens x channels of one dtype; weight holds `channels` values.  residual_dev NULL: s = x, and sum_dev is
 * NULL; otherwise sum_dev receives s, and may be x's or the residual's memory in the same layout.  y leaves as any of
 * y_dev (dtype; may be x's memory in the same layout where sum_dev is not), FP8 (blocks along the rows) and ACT8 (the
 * checkpoint that rudra_act8_weight_grad takes), the last two from y before it is rounded to dtype; what is NULL is not
 * wanted, but one is.  Outputs do not overlap each other.  eps >= 0.  The order of a row's sum depends on tokens, channels, dtype, the
 * outputs that are wanted, whether rows and weight all begin on 16-byte boundaries, and the device alone.
 */
int rudra_rms_norm(const void* x_dev, uint64_t ldx, const void* residual_dev, uint64_t ldr, int dtype, uint64_t tokens,
                   uint64_t channels, const void* weight_dev, int weight_dtype, float eps, void* sum_dev, uint64_t ldsum,
                   void* y_dev, uint64_t ldy, void* fp8_codes_dev, void* fp8_scales_dev, void* act8_codes_dev,
                   void* act8_scales_dev, void* cuda_stream);

/* The backward pass, from the s that went into the norm: with r = 1 / sqrt(mean(s^2) + eps),
 *     ds = r * (weight * dy - s * r^2 * mean(weight * dy * s)) + dsum,    dweight = sum over tokens of dy * s * r.
 * ds is the gradient of x and of the residual alike; dsum (NULL: zero) is what comes down the residual stream.  dy, s, dsum
 * and ds are tokens x channels of one dtype; ds may be dy's or dsum's memory in the same layout.  dweight is of
 * dweight_dtype, wherever it lies in the vector that rudra_ps_push takes; its sums are in 32 bits, in an order that
 * depends on tokens, channels, dtype, whether there is a dsum, whether rows and weight all begin on 16-byte boundaries, and the device
 * alone; so do those of a row.  workspace_dev:
 * rudra_rms_norm_backward_workspace(tokens, channels) bytes on a 32-byte boundary. */
uint64_t rudra_rms_norm_backward_workspace(uint64_t tokens, uint64_t channels);
int rudra_rms_norm_backward(const void* dy_dev, uint64_t lddy, const void* s_dev, uint64_t lds, const void* dsum_dev,
                            uint64_t lddsum, int dtype, uint64_t tokens, uint64_t channels, const void* weight_dev,
                            int weight_dtype, float eps, void* ds_dev, uint64_t ldds, void* dweight_dev,
                            int dweight_dtype, void* workspace_dev, uint64_t workspace_bytes, void* cuda_stream);

/*
 * The norm of `count` gradients together: the square root of the sum of all their squares, to *norm_dev (a float).  Gradient i
 * is sizes[i] consecutive values of dtypes[i]; the three lists are host memory, read before the call returns.  Squares of 16 values
 * are added in 32 bits, all beyond that, and squares a float does not hold, in 64; the order depends on the list alone: its
 * sizes, dtypes and how far past 32-byte boundaries the gradients begin.
 * workspace_dev: rudra_grad_norm_workspace(count) bytes on a 32-byte boundary.  A list has at most 2^24 gradients and
 * 2^43 values.
 */
uint64_t rudra_grad_norm_workspace(uint64_t count);
int rudra_grad_norm(const void* const* grads_dev, const int* dtypes, const uint64_t* sizes, uint64_t count, float* norm_dev,
                    void* workspace_dev, uint64_t workspace_bytes, void* cuda_stream);

/* outs[i] = grads[i] * (norm <= max_norm ? 1 : max_norm / norm): for instance into the layers' parts of the vector that
 * rudra_ps_push takes, in its dtype.  norm_known != 0: norm = *norm_dev (of the shards of several ranks together, say);
 * otherwise it is computed here and left in *norm_dev, as rudra_grad_norm does it and with its workspace; the sums of a
 * small list are added in another order, in 64 bits as well, so that the two floats may be one step apart.
 * outs_dev[i] may be grads_dev[i] with the same dtype; no two outputs, no output and another gradient, nor the norm and an
 * output (or, where it is computed, a gradient) may overlap, which is refused.  Where all are scaled in their place and norm <= max_norm nothing is written.  A norm that is
 * NaN makes every value NaN, an infinite one the finite values zero and the others NaN, unless max_norm is infinite
 * too.  max_norm >= 0. */
int rudra_grad_clip(const void* const* grads_dev, const int* dtypes, const uint64_t* sizes, uint64_t count, float* norm_dev,
                    int norm_known, float max_norm, void* const* outs_dev, const int* out_dtypes, void* workspace_dev,
                    uint64_t workspace_bytes, void* cuda_stream);

/* Waits for cuda_stream and reports asynchronous CUDA errors, and kernels of this header that gave up, as
 * RUDRA_E_CUDA.  The kernels of the products, and of the norm of many rows, wait on barriers inside a block or cluster; a wait
 * that lasts about two seconds (which no working GPU needs) ends, and its kernel with it: what such a call
 * wrote is not to be used.  The kernels count this per device, not per stream: one that gave up, on whichever stream, is
 * reported to every stream of the device that is asked about afterwards, and once told not again, so each learner on a
 * shared GPU hears of it from its own stream.  Waits for no other stream. */
int rudra_learner_sync(void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* RUDRA_LEARNER_H */
