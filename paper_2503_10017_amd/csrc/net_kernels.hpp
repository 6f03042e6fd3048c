// What net_api.hip launches: arguments and launchers of the network's operators (fnn_net.h).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/fnn_net.h"

namespace fnn {

struct NormArgs {
    const void* x;
    const void* weight;
    const void* bias;
    void* y;
    float* mean;
    float* rstd;
    int64_t n, x_stride, y_stride;
    int32_t d;
    float eps;
};
hipError_t launch_layer_norm(const NormArgs& a, int dtype, int weight_dtype, hipStream_t s);

struct NormBackArgs {
    const void* dy;
    const void* x;
    const float* mean;
    const float* rstd;
    const void* weight;
    void* dx;
    void* dweight;
    void* dbias;
    float* partial;  // [workgroups][2][d]: a workgroup's share of dweight and dbias
    int64_t n, dy_stride, x_stride, dx_stride;
    int32_t d;
};
// Workgroups that the gradient is launched with: a function of the sizes alone, which the workspace and the order of its sums rest on.
int64_t layer_norm_backward_groups(int64_t n, int32_t d);
hipError_t launch_layer_norm_backward(const NormBackArgs& a, int dtype, int weight_dtype, hipStream_t s);

// C[m][n] = sum over k of A(m, k) B(n, k), then y = act(C + bias) + residual.
struct GemmArgs {
    const void* a;
    const void* b;
    int64_t lda, ldb;  // elements between rows
    int64_t m;
    int32_t n, k;
    int32_t k_a, k_b;  // what may be read of a row that runs along k, as of k elements or, where zeros follow them, more
    void* y;
    const void* bias;
    const void* residual;
    void* pre;         // C + bias is stored too
    int64_t ldy, ldr, ldp;
    int32_t act;
    float* partial;    // [splits][tiles_m * rows of a tile][tiles_n * columns of a tile]
    int32_t tiles_m, tiles_n, splits;
};
// Bytes of `partial` that a product of these sizes wants (0: none): a function of the sizes and layouts alone.
size_t gemm_workspace(int64_t m, int64_t n, int64_t k, int dtype, int layout_a, int layout_b);
hipError_t launch_gemm(GemmArgs a, int dtype, int layout_a, int layout_b, int trace_kind, hipStream_t s);

// Whether a product of these sizes (forward, or one of the two of a gradient) is worth copies of operands whose rows of `width` elements do not end on
// 16-byte boundaries.
bool copies_pay(int64_t m, int64_t n, int64_t k, int64_t width, int dtype, bool backward);
// to[r][0 .. stride) = from[r][0 .. width), then zeros; to and its rows lie on 16-byte boundaries.
hipError_t launch_copy_rows(const void* from, int64_t from_stride, int64_t rows, int64_t width, void* to, int64_t stride, int dtype, int trace_kind, hipStream_t s);

// p = dy * act'(pre), rounded to dy's type, and the column sums of p before that rounding, as shares of strips of rows.
struct SlopeArgs {
    const void* dy;
    const void* pre;
    void* p;          // rows of n elements and zeros up to a multiple of 16 bytes; NULL: not wanted
    float* partial;   // [strips][n]; NULL: not wanted
    int64_t m, dy_stride, pre_stride, p_stride;
    int32_t n, act;
};
int64_t slope_strips(int64_t m, int64_t n);
hipError_t launch_slope(const SlopeArgs& a, int dtype, hipStream_t s);

// Sums of the columns of partial [groups][width] into out[0 .. first) and more[0 .. width - first), either of which may be NULL.
hipError_t launch_column_sums(const float* partial, int64_t groups, int64_t width, int64_t first, void* out, void* more, int dtype, int trace_kind, hipStream_t s);

// Attention over packed sequences: strides in elements, `share` query heads to a key head.
struct AttentionArgs {
    const void* q;
    const void* k;
    const void* v;
    void* out;
    float* lse;            // [tq][heads]
    const int32_t* cu_q;   // NULL: one sequence of everything
    const int32_t* cu_k;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head, out_row, out_head;
    int32_t tq, tk, batch, heads, groups, share, d, causal;
    float scale;
    int32_t direct;        // keys and values lie on 16-byte boundaries
    int32_t row_tiles, splits, d_pad;
    int32_t part_tiles;    // tiles of keys in a part of a split call
    float* partial;
};
size_t attention_workspace(int64_t tq, int64_t tk, int64_t batch, int64_t heads, int64_t groups, int64_t d);
hipError_t launch_attention(AttentionArgs a, int dtype, hipStream_t s);

// Its gradient: `forward` has q, k, v, out, lse and the tables; dq, dk, dv may be NULL.
struct AttentionBackArgs {
    AttentionArgs forward;
    const void* dout;
    void* dq;
    void* dk;
    void* dv;
    float* stats;  // [2][tq][heads]: what each row's scores and dout v^T are lessened by, as the second pass takes them
    int64_t dout_row, dout_head, dq_row, dq_head, dk_row, dk_head, dv_row, dv_head;
    int32_t key_tiles;
    int32_t direct_rows;   // q and dout lie on 16-byte boundaries
};
hipError_t launch_attention_backward(AttentionBackArgs a, int dtype, hipStream_t s);

// ---- matrices in 8 bits with a scale for each block ----
constexpr int SCALED_BLOCK = 128;
__host__ __device__ constexpr int64_t scaled_blocks(int64_t n) { return (n + SCALED_BLOCK - 1) / SCALED_BLOCK; }

// One that a kernel writes: the places of its codes and scales, and their strides.  Without data it is not wanted.
struct CodesOut {
    uint8_t* data;
    float* scale;
    int64_t row, scale_row, scale_block;
};
hipError_t launch_quantize_rows(const void* x, int64_t x_stride, int64_t n, int32_t d, const CodesOut& out, int dtype, int trace_kind, hipStream_t s);

// Tiles of 128 x 128 of x: by rows, across (transposed), one scale per block of a row or per tile.  What is of x * act'(pre), and the sums, launch_gradient_operands takes.
struct QuantizeArgs {
    const void* x;
    const void* pre;
    CodesOut rows, across;
    float* partial;   // [tiles of rows][d]: the columns' sums; NULL: not wanted
    int64_t n, x_stride, pre_stride;
    int32_t d, act;
};
hipError_t launch_quantize_tiles(const QuantizeArgs& a, bool tiles, int dtype, int trace_kind, hipStream_t s);

// What the products of the gradient of a layer in 8 bits take: q = x * act'(pre) of `q` by rows, across and summed, `x` across, `w`'s codes transposed.  Without x (from) one is not wanted.
struct TransposeArgs {
    const uint8_t* from;
    uint8_t* to;
    int64_t from_stride, to_stride, n;
    int32_t d;
};
struct GradientOperands {
    QuantizeArgs q, x;
    TransposeArgs w;
    uint32_t tiles_q, tiles_x, first;  // the launch's first tile of all
};
hipError_t launch_gradient_operands(GradientOperands a, int dtype, int trace_kind, hipStream_t s);

// Root-mean-square norm of x + residual, and its gradient.
struct RmsArgs {
    const void* x;
    const void* residual;  // NULL: 0
    const void* weight;    // NULL: 1
    void* sum;             // outputs, each of which may be NULL
    void* y;
    CodesOut codes;
    float* rstd;
    int64_t n, x_stride, residual_stride, sum_stride, y_stride;
    int32_t d;
    float eps;
};
hipError_t launch_rms_norm(const RmsArgs& a, int dtype, int weight_dtype, hipStream_t s);
struct RmsBackArgs {
    const void* dy;
    const void* x;
    const void* dsum;      // NULL: 0
    const float* rstd;
    const void* weight;
    void* dx;
    void* dweight;
    float* partial;        // [workgroups][d]: a workgroup's share of dweight
    int64_t n, dy_stride, x_stride, dsum_stride, dx_stride;
    int32_t d;
};
int64_t rms_norm_backward_groups(int64_t n, int32_t d);
hipError_t launch_rms_norm_backward(const RmsBackArgs& a, int dtype, int weight_dtype, hipStream_t s);

// The product behind the layers in 8 bits: C[m][n] = sum over blocks of k of scale_a(m, block) scale_b(n, block) sum over the block of A(m, k) B(n, k).
struct ScaledGemmArgs {
    GemmArgs g;                                     // codes, sizes and epilogue
    const float* scale_a;
    const float* scale_b;
    int64_t sa_row, sa_block, sb_row, sb_block;     // strides of the scales
    int32_t shift_a, shift_b;                       // log2 of the rows that share a scale: 0 or 7
};
// `partial` is a workspace of these bytes: for the shares of a split product, with `copies` also for copies of operands that do not start on 16-byte boundaries.
size_t scaled_gemm_workspace(int64_t m, int64_t n, int64_t k, int dtype, bool copies);
hipError_t launch_scaled_gemm(const ScaledGemmArgs& a, int dtype, int trace_kind, hipStream_t s);  // with a workspace that has room for copies
// A gradient's two products (either may have no rows or columns) and, unless `sums` is NULL, sums[c] = the sum of column c of partial ([groups][columns]).
hipError_t launch_scaled_gradient(const ScaledGemmArgs& dx, const ScaledGemmArgs& dw, const float* partial, int64_t groups, int64_t columns, void* sums, int dtype, int trace_kind,
                                  hipStream_t s);

}  // namespace fnn
