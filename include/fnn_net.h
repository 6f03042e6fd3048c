/*
 * fnn_net.h -- the operators of the network that ends in the maps of fnn.h, on one AMD Instinct MI355X (gfx950).
 *
 * The Speedy MASt3R paper (arXiv 2503.10017) speeds up the matching (fnn.h) and the network before it: attention that
 * never writes the score matrix ("FlashMatch", section 3.4.1) and layers fused with what follows them ("GraphFusion", section
 * 3.4.2).  This header has the operators of a pre-norm transformer block over image tokens and of the matching head (section
 * 3.2.4: layers that end in one descriptor per pixel), with their gradients:
 *
 *   fnn_layer_norm   y = (x - mean) / sqrt(var + eps) * weight + bias          and fnn_layer_norm_backward
 *   fnn_linear       y = act(x w^T + bias) + residual                         and fnn_linear_backward
 *   fnn_attention    softmax(scale q k^T) v over packed sequences             and fnn_attention_backward
 *
 * and of the same block with its layers in 8 bits (e4m3 codes with a scale for each block of 128):
 *
 *   fnn_rms_norm     y = s / sqrt(mean(s^2) + eps) * weight, s = x + residual  and fnn_rms_norm_backward; y in 8 bits, too
 *   fnn_quantize     a matrix, or its transpose, in 8 bits
 *   fnn_linear_e4m3  fnn_linear of operands in 8 bits                          and fnn_linear_e4m3_backward
 *
 * Conventions: those of fnn.h (status codes; device pointers; caller-owned buffers and workspaces, the latter 256-byte
 * aligned; asynchronous on `stream`; argument errors before anything is enqueued; capturable in a HIP graph; no state between calls), and
 *  - A matrix is an fnn_map: n rows of d elements, row_stride >= d elements apart (the stride of fewer than two rows is not looked at);
 *    outputs are passed the same way and written through `data`.  Rows may start anywhere that their element type may (2 or 4 bytes);
 *    rows on 16-byte boundaries are faster.  A matrix of no elements needs no pointer.  Elements between the rows are neither read for
 *    their value nor written.  All matrices of a call have one dtype, unless said otherwise.
 *  - Outputs must not overlap inputs or each other; the exceptions are named.
 *  - A call that would need more workgroups than one launch takes ends in FNN_E_HIP (some 2^24: attention and its gradient where sequences, or
 *    tiles of 32 or 128 rows or keys, times key heads come to that; fnn_linear with 2^31 - 128 rows or 64 GB of copied operands).
 *  - Results do not depend on the order in which workgroups run: the same call gives the same bits.
 *  - Sums, products, statistics and activations are fp32; outputs are rounded once, to nearest even, to their type.  Infinities and NaN in the inputs
 *    reach the outputs that depend on them, and no others.
 */
#ifndef FNN_NET_H
#define FNN_NET_H

#include "fnn.h"

#ifdef __cplusplus
extern "C" {
#endif

#define FNN_MAX_NORM_WIDTH 16384

/*
 * Layer norm over the rows of x (n rows of d <= FNN_MAX_NORM_WIDTH elements, any dtype):
 *   mean = sum_k x[k] / d,  rstd = 1 / sqrt(sum_k (x[k] - mean)^2 / d + eps),  y[k] = (x[k] - mean) * rstd * weight[k] + bias[k]
 * weight and bias (device, d elements of weight_dtype, which is x's dtype or FNN_F32) may each be NULL: 1 and 0.
 * mean and rstd (device float[n]) may be NULL; the gradient takes them.  y may be x itself (same rows).  No workspace.
 * Errors: FNN_E_NULL, FNN_E_SHAPE (n > 2^31 - 64, d < 1 or too large, strides, x and y of different size), FNN_E_DTYPE, FNN_E_RANGE (eps
 * negative or not a number).
 */
int32_t fnn_layer_norm(const fnn_map* x, const void* weight, const void* bias, int32_t weight_dtype, float eps,
                       const fnn_map* y, float* mean, float* rstd, void* stream);

/*
 * Its gradient.  With h = (x - mean) * rstd and g = dy * weight:
 *   dx = rstd * (g - sum_k g / d - h * sum_k (g h) / d),  dweight = sum over the rows of dy * h,  dbias = sum over the rows of dy
 * mean and rstd are those of fnn_layer_norm.  dx, dweight and dbias (the latter two of weight_dtype, d elements) may each be
 * NULL: not wanted.  dx may be dy or x itself (same rows).
 */
size_t fnn_layer_norm_backward_workspace_bytes(int64_t n, int32_t d);
int32_t fnn_layer_norm_backward(const fnn_map* dy, const fnn_map* x, const float* mean, const float* rstd, const void* weight,
                                int32_t weight_dtype, const fnn_map* dx, void* dweight, void* dbias,
                                void* workspace, size_t workspace_bytes, void* stream);

/* Activations of fnn_linear. */
typedef enum {
    FNN_ACT_NONE = 0,
    FNN_ACT_RELU = 1,  /* max(p, 0) */
    FNN_ACT_GELU = 2,  /* p Phi(p), Phi the integral of the normal density */
    FNN_ACT_SILU = 3   /* p / (1 + exp(-p)) */
} fnn_act;

/*
 * A linear layer: p = x w^T + bias, y = act(p) + residual, for x [rows][inner], w [outer][inner], y, pre and residual
 * [rows][outer] and bias [outer], all of one dtype.  bias, residual and pre may be NULL; pre receives p, which the gradient
 * takes.  Sizes of 0 are fine (inner == 0: p = bias).  16-bit types multiply on the 16-bit matrix instructions, FNN_F32 on the
 * fp32 ones; sums are fp32.  y may be the residual itself (same rows).
 * The workspace is for few tiles with a long `inner`, whose products are split and joined in a fixed order, and for aligned copies of
 * the operands of large products whose `inner` is odd; fnn_linear_workspace_bytes may return 0, and returns 0 for invalid sizes.
 * Errors: FNN_E_NULL, FNN_E_SHAPE, FNN_E_DTYPE, FNN_E_RANGE (act), FNN_E_WORKSPACE.
 */
size_t fnn_linear_workspace_bytes(int64_t rows, int64_t inner, int64_t outer, int32_t dtype);
int32_t fnn_linear(const fnn_map* x, const fnn_map* w, const void* bias, int32_t act, const fnn_map* residual,
                   const fnn_map* y, const fnn_map* pre, void* workspace, size_t workspace_bytes, void* stream);

/*
 * Its gradient.  With q = dy * act'(pre) (act == FNN_ACT_NONE: q = dy, and pre is not looked at):
 *   dx = q w,  dw = q^T x,  dbias = sum over the rows of q
 * dx [rows][inner], dw [outer][inner] and dbias [outer] are of x's dtype and may each be NULL: not wanted.  The residual's gradient is dy itself.
 * In 16-bit types q is rounded to that type before the products, as their matrix instructions take it; dbias sums the
 * unrounded values.  FNN_ACT_RELU's slope at 0 is 0.
 */
size_t fnn_linear_backward_workspace_bytes(int64_t rows, int64_t inner, int64_t outer, int32_t dtype, int32_t act);
int32_t fnn_linear_backward(const fnn_map* dy, const fnn_map* x, const fnn_map* w, const fnn_map* pre, int32_t act,
                            const fnn_map* dx, const fnn_map* dw, void* dbias, void* workspace, size_t workspace_bytes,
                            void* stream);

#define FNN_MAX_HEAD_DIM 128

/* n tokens with `heads` vectors of d elements each: element e of head h of token t is data[t * row_stride + h * head_stride + e]. */
typedef struct {
    const void* data;
    int64_t n;
    int32_t heads;
    int32_t d;
    int32_t dtype;        /* fnn_dtype: FNN_F16 or FNN_BF16 */
    int32_t reserved;     /* must be zero */
    int64_t row_stride;   /* in elements */
    int64_t head_stride;  /* in elements */
} fnn_heads;

/*
 * Attention over `batch` sequences packed one after the other: queries cu_q[b] .. cu_q[b + 1] - 1 of q are those of sequence b, keys and values
 * cu_k[b] .. cu_k[b + 1] - 1 of k and v its keys (cu_q, cu_k: device int32[batch + 1], ascending; both NULL with batch == 1: one sequence of
 * everything).  Query i of lq sees key j of lk if !causal or j <= i + lk - lq: the last query sees every key, so queries at the end of
 * a cache, one token among them, need nothing else.
 *   out = sum_j softmax_j(scale <q, k_j>) v_j,   lse = log sum_j exp(scale <q, k_j>)   over the keys j that the query sees
 * A query that sees none has out = 0 and lse = minus infinity; one that sees some, each with a score of minus infinity, has no softmax: its out
 * is NaN.  q and out have `heads` heads, k and v a divisor of that: query head h reads key head h / (heads / key heads).
 * d <= FNN_MAX_HEAD_DIM; scale > 0.  lse (device float [q->n][heads]) may be NULL; the gradient takes it.  Strides are free (heads of
 * a token may also lie apart by more than a token); vectors on 16-byte boundaries are faster.  What lies outside the sequences is neither
 * read for its value nor written.  Neither do infinities and NaN of keys and values reach a query of a causal call that does not see them;
 * in the gradient they spoil what sees them.
 * Scores, softmax and sums are fp32; the weights are rounded to the values' type for the second product.
 * The workspace is for few queries with many keys, which are split and joined in a fixed order.
 * Errors: FNN_E_NULL, FNN_E_SHAPE, FNN_E_DTYPE, FNN_E_RANGE (scale, batch < 1), FNN_E_WORKSPACE.
 */
size_t fnn_attention_workspace_bytes(int64_t tokens_q, int64_t tokens_k, int32_t batch, int32_t heads, int32_t key_heads, int32_t d);
int32_t fnn_attention(const fnn_heads* q, const fnn_heads* k, const fnn_heads* v, int32_t batch, const int32_t* cu_q,
                      const int32_t* cu_k, int32_t causal, float scale, const fnn_heads* out, float* lse,
                      void* workspace, size_t workspace_bytes, void* stream);

/*
 * Its gradient, from dout and what the forward call was given and gave.  With p = exp(scale <q, k> - lse) where the query sees the key,
 * delta = sum_e dout out and ds = p (<dout, v> - delta):
 *   dq = scale sum_j ds k_j,   dk = scale sum_i ds q_i,   dv = sum_i p dout_i   (over all query heads of the key head)
 * dq, dk and dv may each be NULL: not wanted.  Keys of a sequence without queries get 0, and so do queries that see no key.
 * p and ds are rounded to the inputs' type for the products (in FNN_F16 times powers of two, so that neither dout's size nor long rows cost digits).  lse has 24 bits, so where it passes 2^12 in size p is less exact than the
 * inputs' type, and where it passes 2^22 p tells no more than that the gradient is finite.
 */
size_t fnn_attention_backward_workspace_bytes(int64_t tokens_q, int64_t tokens_k, int32_t batch, int32_t heads, int32_t key_heads, int32_t d);
int32_t fnn_attention_backward(const fnn_heads* dout, const fnn_heads* q, const fnn_heads* k, const fnn_heads* v, const fnn_heads* out,
                               const float* lse, int32_t batch, const int32_t* cu_q, const int32_t* cu_k, int32_t causal, float scale,
                               const fnn_heads* dq, const fnn_heads* dk, const fnn_heads* dv, void* workspace, size_t workspace_bytes,
                               void* stream);

/*
 * A matrix in 8 bits: n rows of d e4m3 codes (four bits of exponent, three of mantissa, no infinities: 1 S.1111.111 is NaN and 448 the largest value), row_stride
 * bytes apart, and an fp32 scale for each block of FNN_SCALED_BLOCK columns, of one row (block_rows == 1) or of a tile of 128 rows (block_rows == 128):
 *   element (r, k) = e4m3(data[r * row_stride + k]) * scale[(r / block_rows) * scale_row + (k / 128) * scale_block]
 * The last block of a row, and the last tile of rows, may be short.  scale_row and scale_block may have any values of at least 1; scales of one column of blocks next to each
 * other (scale_row == 1) and rows of codes on 16-byte boundaries are faster.  The strides of what there is one of, or none, are not looked at.
 */
#define FNN_SCALED_BLOCK 128
typedef struct {
    const void* data;
    const float* scale;
    int64_t n;
    int32_t d;
    int32_t block_rows;   /* 1 or 128 */
    int64_t row_stride;   /* of the codes, in bytes */
    int64_t scale_row;    /* in floats */
    int64_t scale_block;  /* in floats */
} fnn_scaled;

/*
 * x (any dtype) in 8 bits, or with `transposed` != 0 its transpose (q has x's columns as rows, and blocks run along x's rows):
 *   scale = max(m / 448, 2^-126) with m the largest finite magnitude of the block,  code = e4m3(value / scale)
 * The division is fp32's, and so is the quotient by 448; from there to e4m3 is rounded to nearest even.  Infinities and NaN become NaN, and do not enter the scale.
 * Neither codes between the rows nor scales between those of the blocks are written.
 * Errors: FNN_E_NULL, FNN_E_SHAPE (sizes, strides, block_rows), FNN_E_DTYPE.
 */
int32_t fnn_quantize(const fnn_map* x, int32_t transposed, const fnn_scaled* q, void* stream);

/*
 * Root-mean-square norm over the rows of s = x + residual (n rows of d <= FNN_MAX_NORM_WIDTH elements, any dtype; residual may be NULL: s = x):
 *   rstd = 1 / sqrt(sum_k s[k]^2 / d + eps),  y[k] = s[k] * rstd * weight[k]
 * weight (device, d elements of weight_dtype, which is x's dtype or FNN_F32) may be NULL: 1.  Outputs, each of which may be NULL: sum receives s, rounded to its type (y is of the
 * unrounded one), y, codes the same y (unrounded) in 8 bits as fnn_quantize does it (block_rows == 1), and rstd (device float[n]) what the gradient takes.  sum and y may be x or residual itself (same
 * rows), but not one matrix.  No workspace.
 * Errors: FNN_E_NULL, FNN_E_SHAPE (n > 2^31 - 64, d < 1 or too large, strides, matrices of different size, block_rows), FNN_E_DTYPE, FNN_E_RANGE (eps negative or not a number).
 */
int32_t fnn_rms_norm(const fnn_map* x, const fnn_map* residual, const void* weight, int32_t weight_dtype, float eps,
                     const fnn_map* sum, const fnn_map* y, const fnn_scaled* codes, float* rstd, void* stream);

/*
 * Its gradient, from dy, s (`sum`) and rstd as fnn_rms_norm gave them.  With h = s * rstd and g = dy * weight:
 *   dx = rstd * (g - h * sum_k (g h) / d) + dsum,  dweight = sum over the rows of dy * h
 * dsum (what reaches s by other ways, down the residual stream; NULL: 0) is added in fp32; dx is the gradient of x and of residual alike.  The rounding of y to 8 bits is not in it.  dx and
 * dweight (of weight_dtype, d elements) may each be NULL: not wanted.  dx may be dy, s or dsum itself (same rows).
 */
size_t fnn_rms_norm_backward_workspace_bytes(int64_t n, int32_t d);
int32_t fnn_rms_norm_backward(const fnn_map* dy, const fnn_map* sum, const float* rstd, const void* weight, int32_t weight_dtype, const fnn_map* dsum,
                              const fnn_map* dx, void* dweight, void* workspace, size_t workspace_bytes, void* stream);

/*
 * fnn_linear of operands in 8 bits: p = x w^T + bias, y = act(p) + residual for x [rows][inner], w [outer][inner], y, pre and residual [rows][outer] and bias
 * [outer], the latter four of one dtype, which may be any.  The products of a block of 128 are summed first, then multiplied by the product of the two scales (fp32, so this has to be a number that
 * fp32 has), and added to the fp32 sum over the blocks.  16-bit results take the matrix instructions for 8 bits, which cut each of eight products at 2^-13 of the largest of the eight before they
 * add them: an error of some 10^-5 of the sum's size (where the terms cancel: of theirs), below what the result is rounded by.  FNN_F32 results take exact products and fp32 sums, at half the rate or less.
 * The workspace is for few tiles with a long `inner`, whose products are split and joined in a fixed order, and for aligned copies of operands with an `inner` that is no multiple of 16;
 * fnn_linear_e4m3_workspace_bytes may return 0, and returns 0 for invalid sizes.  dtype: that of y.  y may be the residual itself (same rows).
 * Errors: FNN_E_NULL, FNN_E_SHAPE, FNN_E_DTYPE, FNN_E_RANGE (act), FNN_E_WORKSPACE.
 */
size_t fnn_linear_e4m3_workspace_bytes(int64_t rows, int64_t inner, int64_t outer, int32_t dtype);
int32_t fnn_linear_e4m3(const fnn_scaled* x, const fnn_scaled* w, const void* bias, int32_t act, const fnn_map* residual,
                        const fnn_map* y, const fnn_map* pre, void* workspace, size_t workspace_bytes, void* stream);

/*
 * The gradient of that layer, in 8 bits too, from dy, x as it was before its quantising, the layer's w (block_rows == 128: its transpose has the same codes and scales) and pre.  With
 * q = dy * act'(pre) (act == FNN_ACT_NONE: q = dy, and pre is not looked at) and Q(.) a matrix as fnn_quantize gives it, a scale for each block of 128 of a row:
 *   dx = Q(q) w,  dw = Q(q^T) Q(x^T)^T,  dbias = sum over the rows of q
 * dy, x, pre, dx, dw and dbias are of one dtype, dx [rows][inner], dw [outer][inner] and dbias [outer] may each be NULL: not wanted.  q is quantised, and summed, as it is in fp32.  With
 * GELU and SiLU q is off by what their slopes are (16-bit types: up to 4e-6 of dy), and in 16-bit types its quotient by the scale may be off by another two units in fp32's last place: a code
 * next to the border of two may be its neighbour there.  All other codes are fnn_quantize's to the bit.  The residual's gradient is dy itself.  Products as in fnn_linear_e4m3.
 */
size_t fnn_linear_e4m3_backward_workspace_bytes(int64_t rows, int64_t inner, int64_t outer, int32_t dtype);
int32_t fnn_linear_e4m3_backward(const fnn_map* dy, const fnn_map* x, const fnn_scaled* w, const fnn_map* pre, int32_t act,
                                 const fnn_map* dx, const fnn_map* dw, void* dbias, void* workspace, size_t workspace_bytes, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* FNN_NET_H */
