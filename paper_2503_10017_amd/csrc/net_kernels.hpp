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

}  // namespace fnn
