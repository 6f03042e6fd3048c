// C entry points of the network's operators (see include/fnn_net.h): argument checks and workspace carving.  Nothing here
// synchronises with the device or allocates memory.
#include <hip/hip_runtime.h>
#include <math.h>
#include <string.h>

#include "fnn_kernels.hpp"
#include "net_kernels.hpp"
#include "trace.hpp"

using namespace fnn;

#define FNN_CHECK(call)                       \
    do {                                      \
        const int32_t status_ = (call);       \
        if (status_ != FNN_OK) return status_; \
    } while (0)

namespace {

bool valid_type(int32_t t) { return t == FNN_F32 || t == FNN_F16 || t == FNN_BF16; }

// Shape, then pointer, of a matrix; the stride of at most one row is not looked at.
int32_t check_matrix(const fnn_map* m) {
    if (!m) return FNN_E_NULL;
    if (m->n < 0 || m->n > MAX_SLOTS || m->d < 0 || (m->n > 1 && m->row_stride < m->d)) return FNN_E_SHAPE;
    if (m->n > 0 && m->row_stride > INT64_MAX / 8 / m->n) return FNN_E_SHAPE;
    if (!valid_type(m->dtype)) return FNN_E_DTYPE;
    if (m->n > 0 && m->d > 0 && !m->data) return FNN_E_NULL;
    return FNN_OK;
}
int64_t stride_of(const fnn_map* m) { return m->n > 1 ? m->row_stride : m->d; }

int32_t check_workspace(const void* workspace, size_t have, size_t need) {
    return need && (!workspace || ((uintptr_t)workspace & 255) || have < need) ? FNN_E_WORKSPACE : FNN_OK;
}
int32_t done(hipError_t e) { return e == hipSuccess ? FNN_OK : FNN_E_HIP; }


size_t aligned_to(size_t bytes, size_t to) { return (bytes + to - 1) / to * to; }
size_t aligned(size_t bytes) { return aligned_to(bytes, 256); }

// Sizes that the linear layers take: every dimension an int32, so that tiles and columns are.
bool linear_sizes(int64_t rows, int64_t inner, int64_t outer) {
    return rows >= 0 && rows <= MAX_SLOTS && inner >= 0 && inner <= MAX_SLOTS && outer >= 0 && outer <= MAX_SLOTS;
}
bool same_shape(const fnn_map* m, int64_t n, int64_t d) { return m->n == n && m->d == d; }

int64_t whole_runs(int64_t n, size_t es) { return (int64_t)aligned_to(n * es, 16) / (int64_t)es; }

// The workspace of a linear layer: copies of its operands where their rows do not end on 16-byte boundaries, and the shares of its product.
struct LinearLayout {
    size_t x, w, partial, total;  // offsets
    bool copies;
    int64_t stride;               // of the copies
};
LinearLayout linear_layout(int64_t rows, int64_t inner, int64_t outer, int32_t dtype) {
    LinearLayout L;
    const size_t es = dtype == FNN_F32 ? 4 : 2;
    L.stride = whole_runs(inner, es);
    L.copies = copies_pay(rows, outer, inner, inner, dtype, false);
    size_t at = 0;
    L.x = at;
    if (L.copies) at += aligned((size_t)rows * L.stride * es);
    L.w = at;
    if (L.copies) at += aligned((size_t)outer * L.stride * es);
    L.partial = at;
    L.total = at + gemm_workspace(rows, outer, inner, dtype, 0, 0);
    return L;
}

// That of its gradient: q (dy itself where it has no activation and its rows end well), the shares of dbias, copies of w and x, and one
// area that the two products use in turn.
struct LinearBackLayout {
    size_t q, sums, x, w, partial, total;  // offsets
    bool own_q, copies;
    int64_t q_stride, stride;
};
LinearBackLayout linear_back_layout(int64_t rows, int64_t inner, int64_t outer, int32_t dtype, int32_t act) {
    LinearBackLayout L;
    const size_t es = dtype == FNN_F32 ? 4 : 2;
    L.own_q = act != FNN_ACT_NONE || copies_pay(rows, inner, outer, outer, dtype, true);
    L.copies = copies_pay(rows, inner, outer, inner, dtype, true);
    L.q_stride = whole_runs(outer, es);
    L.stride = whole_runs(inner, es);
    size_t at = 0;
    L.q = at;
    if (L.own_q) at += aligned((size_t)rows * L.q_stride * es);
    L.sums = at;
    at += aligned((size_t)slope_strips(rows, outer) * outer * sizeof(float));
    L.x = at;
    if (L.copies) at += aligned((size_t)rows * L.stride * es);
    L.w = at;
    if (L.copies) at += aligned((size_t)outer * L.stride * es);
    L.partial = at;
    const size_t x = gemm_workspace(rows, inner, outer, dtype, 0, 1), w = gemm_workspace(outer, inner, rows, dtype, 1, 1);
    L.total = at + aligned(x > w ? x : w);
    return L;
}

int32_t check_heads(const fnn_heads* t) {
    if (!t) return FNN_E_NULL;
    if (t->n < 0 || t->n > MAX_SLOTS || t->heads < 1 || t->heads > 65535 || t->d < 1 || t->d > FNN_MAX_HEAD_DIM || t->reserved) return FNN_E_SHAPE;
    if ((t->n > 1 && t->row_stride < t->d) || (t->heads > 1 && t->head_stride < t->d)) return FNN_E_SHAPE;
    if ((t->n > 1 && t->row_stride > INT64_MAX / 8 / t->n) || (t->heads > 1 && t->head_stride > INT64_MAX / 8 / t->heads)) return FNN_E_SHAPE;
    if (t->dtype != FNN_F16 && t->dtype != FNN_BF16) return FNN_E_DTYPE;
    if (t->n > 0 && !t->data) return FNN_E_NULL;
    return FNN_OK;
}
// Rows (queries times heads) and keys times their heads are counted in 32 bits, with room for a tile beyond the last.
bool attention_sizes(int64_t tq, int64_t tk, int64_t batch, int64_t heads, int64_t groups, int64_t d) {
    return tq >= 0 && tk >= 0 && batch >= 1 && batch <= MAX_SLOTS / 2 && heads >= 1 && heads <= 65535 && groups >= 1 && heads % groups == 0 &&
           tq <= (MAX_SLOTS - 1024) / heads && tk <= (MAX_SLOTS - 1024) / groups && d >= 1 && d <= FNN_MAX_HEAD_DIM;
}
int64_t row_of(const fnn_heads* t) { return t->n > 1 ? t->row_stride : t->d; }
int64_t head_of(const fnn_heads* t) { return t->heads > 1 ? t->head_stride : t->d; }
bool same_heads(const fnn_heads* a, const fnn_heads* b) { return a->n == b->n && a->heads == b->heads && a->d == b->d; }
// Whether every vector starts on a 16-byte boundary, is whole runs of 16 bytes, and a tile's offsets fit 32 bits.
bool on_runs(const fnn_heads* t) {
    return ((uintptr_t)t->data & 15) == 0 && t->d % 8 == 0 && row_of(t) % 8 == 0 && head_of(t) % 8 == 0 && row_of(t) < ((int64_t)1 << 23);
}

// What the forward call and the gradient check alike, and the arguments that they share.
int32_t attention_args(const fnn_heads* q, const fnn_heads* k, const fnn_heads* v, int32_t batch, const int32_t* cu_q, const int32_t* cu_k,
                       int32_t causal, float scale, const fnn_heads* out, AttentionArgs& a) {
    FNN_CHECK(check_heads(q));
    FNN_CHECK(check_heads(k));
    FNN_CHECK(check_heads(v));
    FNN_CHECK(check_heads(out));
    if (batch < 1 || !(scale > 0.f) || isinf(scale)) return FNN_E_RANGE;
    if (k->n != v->n || k->heads != v->heads || out->n != q->n || out->heads != q->heads || k->d != q->d || v->d != q->d || out->d != q->d ||
        !attention_sizes(q->n, k->n, batch, q->heads, k->heads, q->d))
        return FNN_E_SHAPE;
    if (k->dtype != q->dtype || v->dtype != q->dtype || out->dtype != q->dtype) return FNN_E_DTYPE;
    if (!cu_q != !cu_k || (!cu_q && batch != 1)) return FNN_E_NULL;
    memset(&a, 0, sizeof(a));
    a.q = q->data;
    a.k = k->data;
    a.v = v->data;
    a.out = const_cast<void*>(out->data);
    a.cu_q = cu_q;
    a.cu_k = cu_k;
    a.q_row = row_of(q);
    a.q_head = head_of(q);
    a.k_row = row_of(k);
    a.k_head = head_of(k);
    a.v_row = row_of(v);
    a.v_head = head_of(v);
    a.out_row = row_of(out);
    a.out_head = head_of(out);
    a.tq = (int32_t)q->n;
    a.tk = (int32_t)k->n;
    a.batch = batch;
    a.heads = q->heads;
    a.groups = k->heads;
    a.share = q->heads / k->heads;
    a.d = q->d;
    a.causal = causal != 0;
    a.scale = scale;
    a.direct = on_runs(k) && on_runs(v);
    return FNN_OK;
}

// Shape, then pointers, of a matrix in 8 bits; the strides of what there is one of, and those of no scales, are not looked at.
int32_t check_scaled(const fnn_scaled* m) {
    if (!m) return FNN_E_NULL;
    // columns are counted in 32 bits, up to the end of a block
    if (m->n < 0 || m->n > MAX_SLOTS || m->d < 0 || m->d > MAX_SLOTS || (m->block_rows != 1 && m->block_rows != SCALED_BLOCK)) return FNN_E_SHAPE;
    const int64_t high = m->block_rows == 1 ? m->n : scaled_blocks(m->n), blocks = scaled_blocks(m->d);
    if (m->n > 1 && (m->row_stride < m->d || m->row_stride > INT64_MAX / 8 / m->n)) return FNN_E_SHAPE;
    if (high > 1 && blocks > 0 && (m->scale_row < 1 || m->scale_row > INT64_MAX / 16 / high)) return FNN_E_SHAPE;
    if (blocks > 1 && high > 0 && (m->scale_block < 1 || m->scale_block > INT64_MAX / 16 / blocks)) return FNN_E_SHAPE;
    if (m->n > 0 && m->d > 0 && (!m->data || !m->scale)) return FNN_E_NULL;
    return FNN_OK;
}
int64_t stride_of(const fnn_scaled* m) { return m->n > 1 ? m->row_stride : m->d; }
// A stride that is not looked at is 0: a product reads the scale of the first row, or block, in place of those behind the last.
int64_t scale_row_of(const fnn_scaled* m) { return m->d > 0 && (m->block_rows == 1 ? m->n : scaled_blocks(m->n)) > 1 ? m->scale_row : 0; }
int64_t scale_block_of(const fnn_scaled* m) { return m->n > 0 && m->d > SCALED_BLOCK ? m->scale_block : 0; }
CodesOut codes_of(const fnn_scaled* m) {
    return {(uint8_t*)const_cast<void*>(m->data), const_cast<float*>(m->scale), stride_of(m), scale_row_of(m), scale_block_of(m)};
}

// The workspace of the gradient of a layer in 8 bits: q by rows, w's transpose, q and x across, the shares of dbias, and one area that the two products use in turn.
struct E4m3BackLayout {
    size_t q, q_scale, w, q_across, q_across_scale, x, x_scale, sums, partial, total;  // offsets
    int64_t outer_stride, rows_stride;  // of codes along outer and along the rows
};
E4m3BackLayout e4m3_back_layout(int64_t rows, int64_t inner, int64_t outer, int32_t dtype) {
    E4m3BackLayout L;
    L.outer_stride = whole_runs(outer, 1);
    L.rows_stride = whole_runs(rows, 1);
    size_t at = 0;
    auto area = [&](size_t& place, int64_t bytes) {
        place = at;
        if (at < SIZE_MAX / 2) at += aligned((size_t)bytes);  // what no memory holds stays that large
    };
    area(L.q, rows * L.outer_stride);
    area(L.q_scale, rows * scaled_blocks(outer) * 4);
    area(L.w, inner * L.outer_stride);
    area(L.q_across, outer * L.rows_stride);
    area(L.q_across_scale, outer * scaled_blocks(rows) * 4);
    area(L.x, inner * L.rows_stride);
    area(L.x_scale, inner * scaled_blocks(rows) * 4);
    area(L.sums, scaled_blocks(rows) * outer * 4);
    L.partial = at;
    const size_t x = scaled_gemm_workspace(rows, inner, outer, dtype, false), w = scaled_gemm_workspace(outer, inner, rows, dtype, false);
    L.total = at + aligned(x > w ? x : w);
    return L;
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

int32_t fnn_layer_norm(const fnn_map* x, const void* weight, const void* bias, int32_t weight_dtype, float eps,
                       const fnn_map* y, float* mean, float* rstd, void* stream) {
    FNN_CHECK(check_matrix(x));
    FNN_CHECK(check_matrix(y));
    if (x->d < 1 || x->d > FNN_MAX_NORM_WIDTH || y->n != x->n || y->d != x->d) return FNN_E_SHAPE;
    if (y->dtype != x->dtype || (weight_dtype != x->dtype && weight_dtype != FNN_F32)) return FNN_E_DTYPE;
    if (!(eps >= 0.f) || isinf(eps)) return FNN_E_RANGE;
    if (x->n == 0) return FNN_OK;
    NormArgs a;
    memset(&a, 0, sizeof(a));
    a.x = x->data;
    a.weight = weight;
    a.bias = bias;
    a.y = const_cast<void*>(y->data);
    a.mean = mean;
    a.rstd = rstd;
    a.n = x->n;
    a.x_stride = stride_of(x);
    a.y_stride = stride_of(y);
    a.d = x->d;
    a.eps = eps;
    return done(launch_layer_norm(a, x->dtype, weight_dtype, (hipStream_t)stream));
}

size_t fnn_layer_norm_backward_workspace_bytes(int64_t n, int32_t d) {
    if (n < 0 || n > MAX_SLOTS || d < 1 || d > FNN_MAX_NORM_WIDTH) return 0;
    return (size_t)layer_norm_backward_groups(n, d) * 2 * d * sizeof(float);
}

int32_t fnn_layer_norm_backward(const fnn_map* dy, const fnn_map* x, const float* mean, const float* rstd, const void* weight,
                                int32_t weight_dtype, const fnn_map* dx, void* dweight, void* dbias,
                                void* workspace, size_t workspace_bytes, void* stream) {
    FNN_CHECK(check_matrix(dy));
    FNN_CHECK(check_matrix(x));
    if (x->d < 1 || x->d > FNN_MAX_NORM_WIDTH || dy->n != x->n || dy->d != x->d) return FNN_E_SHAPE;
    if (dy->dtype != x->dtype || (weight_dtype != x->dtype && weight_dtype != FNN_F32)) return FNN_E_DTYPE;
    if (dx) {
        FNN_CHECK(check_matrix(dx));
        if (dx->n != x->n || dx->d != x->d) return FNN_E_SHAPE;
        if (dx->dtype != x->dtype) return FNN_E_DTYPE;
    }
    if (x->n > 0 && (!mean || !rstd)) return FNN_E_NULL;
    const bool sums = dweight || dbias;
    if (sums) FNN_CHECK(check_workspace(workspace, workspace_bytes, fnn_layer_norm_backward_workspace_bytes(x->n, x->d)));
    if (!sums && (!dx || x->n == 0)) return FNN_OK;
    NormBackArgs a;
    memset(&a, 0, sizeof(a));
    a.dy = dy->data;
    a.x = x->data;
    a.mean = mean;
    a.rstd = rstd;
    a.weight = weight;
    a.dx = dx ? const_cast<void*>(dx->data) : nullptr;
    a.dweight = dweight;
    a.dbias = dbias;
    a.partial = sums ? (float*)workspace : nullptr;
    a.n = x->n;
    a.dy_stride = stride_of(dy);
    a.x_stride = stride_of(x);
    a.dx_stride = dx ? stride_of(dx) : 0;
    a.d = x->d;
    return done(launch_layer_norm_backward(a, x->dtype, weight_dtype, (hipStream_t)stream));
}

size_t fnn_linear_workspace_bytes(int64_t rows, int64_t inner, int64_t outer, int32_t dtype) {
    if (!linear_sizes(rows, inner, outer) || !valid_type(dtype)) return 0;
    return linear_layout(rows, inner, outer, dtype).total;
}

int32_t fnn_linear(const fnn_map* x, const fnn_map* w, const void* bias, int32_t act, const fnn_map* residual,
                   const fnn_map* y, const fnn_map* pre, void* workspace, size_t workspace_bytes, void* stream) {
    FNN_CHECK(check_matrix(x));
    FNN_CHECK(check_matrix(w));
    FNN_CHECK(check_matrix(y));
    if (residual) FNN_CHECK(check_matrix(residual));
    if (pre) FNN_CHECK(check_matrix(pre));
    const int64_t rows = x->n, inner = x->d, outer = w->n;
    if (w->d != inner || !same_shape(y, rows, outer) || (residual && !same_shape(residual, rows, outer)) || (pre && !same_shape(pre, rows, outer)))
        return FNN_E_SHAPE;
    if (w->dtype != x->dtype || y->dtype != x->dtype || (residual && residual->dtype != x->dtype) || (pre && pre->dtype != x->dtype))
        return FNN_E_DTYPE;
    if (act < FNN_ACT_NONE || act > FNN_ACT_SILU) return FNN_E_RANGE;
    const LinearLayout L = linear_layout(rows, inner, outer, x->dtype);
    FNN_CHECK(check_workspace(workspace, workspace_bytes, L.total));
    const hipStream_t s = (hipStream_t)stream;
    char* ws = (char*)workspace;
    GemmArgs a;
    memset(&a, 0, sizeof(a));
    a.a = x->data;
    a.b = w->data;
    a.lda = stride_of(x);
    a.ldb = stride_of(w);
    a.m = rows;
    a.n = (int32_t)outer;
    a.k = a.k_a = a.k_b = (int32_t)inner;
    if (L.copies) {
        if (launch_copy_rows(a.a, a.lda, rows, inner, ws + L.x, L.stride, x->dtype, TK_LINEAR, s) != hipSuccess ||
            launch_copy_rows(a.b, a.ldb, outer, inner, ws + L.w, L.stride, x->dtype, TK_LINEAR, s) != hipSuccess)
            return FNN_E_HIP;
        a.a = ws + L.x;
        a.b = ws + L.w;
        a.lda = a.ldb = L.stride;
        a.k_a = a.k_b = (int32_t)L.stride;
    }
    a.y = const_cast<void*>(y->data);
    a.bias = bias;
    a.residual = residual ? residual->data : nullptr;
    a.pre = pre ? const_cast<void*>(pre->data) : nullptr;
    a.ldy = stride_of(y);
    a.ldr = residual ? stride_of(residual) : 0;
    a.ldp = pre ? stride_of(pre) : 0;
    a.act = act;
    a.partial = (float*)(ws + L.partial);
    return done(launch_gemm(a, x->dtype, 0, 0, TK_LINEAR, s));
}

size_t fnn_linear_backward_workspace_bytes(int64_t rows, int64_t inner, int64_t outer, int32_t dtype, int32_t act) {
    if (!linear_sizes(rows, inner, outer) || !valid_type(dtype) || act < FNN_ACT_NONE || act > FNN_ACT_SILU) return 0;
    return linear_back_layout(rows, inner, outer, dtype, act).total;
}

int32_t fnn_linear_backward(const fnn_map* dy, const fnn_map* x, const fnn_map* w, const fnn_map* pre, int32_t act,
                            const fnn_map* dx, const fnn_map* dw, void* dbias, void* workspace, size_t workspace_bytes,
                            void* stream) {
    FNN_CHECK(check_matrix(dy));
    FNN_CHECK(check_matrix(x));
    FNN_CHECK(check_matrix(w));
    if (act < FNN_ACT_NONE || act > FNN_ACT_SILU) return FNN_E_RANGE;
    const bool slope = act != FNN_ACT_NONE;
    if (slope) FNN_CHECK(check_matrix(pre));
    if (dx) FNN_CHECK(check_matrix(dx));
    if (dw) FNN_CHECK(check_matrix(dw));
    const int64_t rows = x->n, inner = x->d, outer = w->n;
    if (w->d != inner || !same_shape(dy, rows, outer) || (slope && !same_shape(pre, rows, outer)) || (dx && !same_shape(dx, rows, inner)) ||
        (dw && !same_shape(dw, outer, inner)))
        return FNN_E_SHAPE;
    if (w->dtype != x->dtype || dy->dtype != x->dtype || (slope && pre->dtype != x->dtype) || (dx && dx->dtype != x->dtype) || (dw && dw->dtype != x->dtype))
        return FNN_E_DTYPE;
    if (!dx && !dw && !dbias) return FNN_OK;
    const LinearBackLayout L = linear_back_layout(rows, inner, outer, x->dtype, act);
    FNN_CHECK(check_workspace(workspace, workspace_bytes, L.total));
    const hipStream_t s = (hipStream_t)stream;
    char* ws = (char*)workspace;

    const void* q = dy->data;
    int64_t q_stride = stride_of(dy);
    const bool own_q = L.own_q && (dx || dw);
    if (outer > 0 && ((own_q && rows > 0) || dbias)) {
        SlopeArgs a;
        memset(&a, 0, sizeof(a));
        a.dy = dy->data;
        a.pre = slope ? pre->data : nullptr;
        a.p = own_q ? ws + L.q : nullptr;
        a.partial = dbias ? (float*)(ws + L.sums) : nullptr;
        a.m = rows;
        a.dy_stride = stride_of(dy);
        a.pre_stride = slope ? stride_of(pre) : 0;
        a.p_stride = L.q_stride;
        a.n = (int32_t)outer;
        a.act = act;
        if (launch_slope(a, x->dtype, s) != hipSuccess) return FNN_E_HIP;
        if (dbias && launch_column_sums(a.partial, slope_strips(rows, outer), outer, outer, dbias, nullptr, x->dtype, TK_LINEAR_BACKWARD, s) != hipSuccess)
            return FNN_E_HIP;
    }
    if (own_q) q = ws + L.q, q_stride = L.q_stride;
    const void* of_x = x->data;
    const void* of_w = w->data;
    int64_t x_stride = stride_of(x), w_stride = stride_of(w);
    if (L.copies) {
        if (dw && launch_copy_rows(of_x, x_stride, rows, inner, ws + L.x, L.stride, x->dtype, TK_LINEAR_BACKWARD, s) != hipSuccess) return FNN_E_HIP;
        if (dx && launch_copy_rows(of_w, w_stride, outer, inner, ws + L.w, L.stride, x->dtype, TK_LINEAR_BACKWARD, s) != hipSuccess) return FNN_E_HIP;
        of_x = ws + L.x;
        of_w = ws + L.w;
        x_stride = w_stride = L.stride;
    }
    GemmArgs a;
    memset(&a, 0, sizeof(a));
    a.partial = (float*)(ws + L.partial);
    if (dx) {
        a.a = q;
        a.lda = q_stride;
        a.b = of_w;
        a.ldb = w_stride;
        a.m = rows;
        a.n = (int32_t)inner;
        a.k = a.k_a = a.k_b = (int32_t)outer;
        if (own_q) a.k_a = (int32_t)L.q_stride;
        a.y = const_cast<void*>(dx->data);
        a.ldy = stride_of(dx);
        if (launch_gemm(a, x->dtype, 0, 1, TK_LINEAR_BACKWARD, s) != hipSuccess) return FNN_E_HIP;
    }
    if (dw) {
        a.a = q;
        a.lda = q_stride;
        a.b = of_x;
        a.ldb = x_stride;
        a.m = outer;
        a.n = (int32_t)inner;
        a.k = a.k_a = a.k_b = (int32_t)rows;
        a.y = const_cast<void*>(dw->data);
        a.ldy = stride_of(dw);
        if (launch_gemm(a, x->dtype, 1, 1, TK_LINEAR_BACKWARD, s) != hipSuccess) return FNN_E_HIP;
    }
    return FNN_OK;
}

size_t fnn_attention_workspace_bytes(int64_t tokens_q, int64_t tokens_k, int32_t batch, int32_t heads, int32_t key_heads, int32_t d) {
    if (!attention_sizes(tokens_q, tokens_k, batch, heads, key_heads, d)) return 0;
    return attention_workspace(tokens_q, tokens_k, batch, heads, key_heads, d);
}

int32_t fnn_attention(const fnn_heads* q, const fnn_heads* k, const fnn_heads* v, int32_t batch, const int32_t* cu_q,
                      const int32_t* cu_k, int32_t causal, float scale, const fnn_heads* out, float* lse,
                      void* workspace, size_t workspace_bytes, void* stream) {
    AttentionArgs a;
    FNN_CHECK(attention_args(q, k, v, batch, cu_q, cu_k, causal, scale, out, a));
    FNN_CHECK(check_workspace(workspace, workspace_bytes, attention_workspace(q->n, k->n, batch, q->heads, k->heads, q->d)));
    a.lse = lse;
    a.partial = (float*)workspace;
    return done(launch_attention(a, q->dtype, (hipStream_t)stream));
}

size_t fnn_attention_backward_workspace_bytes(int64_t tokens_q, int64_t tokens_k, int32_t batch, int32_t heads, int32_t key_heads, int32_t d) {
    if (!attention_sizes(tokens_q, tokens_k, batch, heads, key_heads, d)) return 0;
    return (size_t)tokens_q * heads * 2 * sizeof(float);
}

int32_t fnn_attention_backward(const fnn_heads* dout, const fnn_heads* q, const fnn_heads* k, const fnn_heads* v, const fnn_heads* out,
                               const float* lse, int32_t batch, const int32_t* cu_q, const int32_t* cu_k, int32_t causal, float scale,
                               const fnn_heads* dq, const fnn_heads* dk, const fnn_heads* dv, void* workspace, size_t workspace_bytes,
                               void* stream) {
    AttentionBackArgs a;
    memset(&a, 0, sizeof(a));
    FNN_CHECK(attention_args(q, k, v, batch, cu_q, cu_k, causal, scale, out, a.forward));
    FNN_CHECK(check_heads(dout));
    if (!same_heads(dout, q)) return FNN_E_SHAPE;
    if (dout->dtype != q->dtype) return FNN_E_DTYPE;
    const fnn_heads* grads[3] = {dq, dk, dv};
    for (int i = 0; i < 3; ++i) {
        if (!grads[i]) continue;
        FNN_CHECK(check_heads(grads[i]));
        if (!same_heads(grads[i], i ? k : q)) return FNN_E_SHAPE;
        if (grads[i]->dtype != q->dtype) return FNN_E_DTYPE;
    }
    if (q->n > 0 && !lse) return FNN_E_NULL;
    if (!dq && !dk && !dv) return FNN_OK;
    FNN_CHECK(check_workspace(workspace, workspace_bytes, (size_t)q->n * q->heads * 2 * sizeof(float)));
    a.forward.lse = const_cast<float*>(lse);
    a.dout = dout->data;
    a.dout_row = row_of(dout);
    a.dout_head = head_of(dout);
    a.dq = dq ? const_cast<void*>(dq->data) : nullptr;
    a.dk = dk ? const_cast<void*>(dk->data) : nullptr;
    a.dv = dv ? const_cast<void*>(dv->data) : nullptr;
    a.dq_row = dq ? row_of(dq) : 0;
    a.dq_head = dq ? head_of(dq) : 0;
    a.dk_row = dk ? row_of(dk) : 0;
    a.dk_head = dk ? head_of(dk) : 0;
    a.dv_row = dv ? row_of(dv) : 0;
    a.dv_head = dv ? head_of(dv) : 0;
    a.stats = (float*)workspace;
    // the heads of a group are reached from its first by 32-bit offsets too
    const int64_t apart = a.forward.share * (head_of(q) > head_of(dout) ? head_of(q) : head_of(dout));
    a.direct_rows = on_runs(q) && on_runs(dout) && apart < ((int64_t)1 << 28);
    return done(launch_attention_backward(a, q->dtype, (hipStream_t)stream));
}

int32_t fnn_quantize(const fnn_map* x, int32_t transposed, const fnn_scaled* q, void* stream) {
    FNN_CHECK(check_matrix(x));
    FNN_CHECK(check_scaled(q));
    if (transposed ? q->n != x->d || q->d != x->n : q->n != x->n || q->d != x->d) return FNN_E_SHAPE;
    if (x->n == 0 || x->d == 0) return FNN_OK;
    const hipStream_t s = (hipStream_t)stream;
    if (!transposed && q->block_rows == 1)
        return done(launch_quantize_rows(x->data, stride_of(x), x->n, x->d, codes_of(q), x->dtype, TK_QUANTIZE, s));
    QuantizeArgs a;
    memset(&a, 0, sizeof(a));
    a.x = x->data;
    (transposed ? a.across : a.rows) = codes_of(q);
    a.n = x->n;
    a.x_stride = stride_of(x);
    a.d = x->d;
    return done(launch_quantize_tiles(a, q->block_rows != 1, x->dtype, TK_QUANTIZE, s));
}

int32_t fnn_rms_norm(const fnn_map* x, const fnn_map* residual, const void* weight, int32_t weight_dtype, float eps,
                     const fnn_map* sum, const fnn_map* y, const fnn_scaled* codes, float* rstd, void* stream) {
    FNN_CHECK(check_matrix(x));
    if (x->d < 1 || x->d > FNN_MAX_NORM_WIDTH) return FNN_E_SHAPE;
    const fnn_map* others[3] = {residual, sum, y};
    for (const fnn_map* m : others) {
        if (!m) continue;
        FNN_CHECK(check_matrix(m));
        if (m->n != x->n || m->d != x->d) return FNN_E_SHAPE;
        if (m->dtype != x->dtype) return FNN_E_DTYPE;
    }
    if (codes) {
        FNN_CHECK(check_scaled(codes));
        // of one row the two are the same
        if (codes->n != x->n || codes->d != x->d || (codes->block_rows != 1 && x->n > 1)) return FNN_E_SHAPE;
    }
    if (weight_dtype != x->dtype && weight_dtype != FNN_F32) return FNN_E_DTYPE;
    if (!(eps >= 0.f) || isinf(eps)) return FNN_E_RANGE;
    if (x->n == 0 || (!sum && !y && !codes && !rstd)) return FNN_OK;
    RmsArgs a;
    memset(&a, 0, sizeof(a));
    a.x = x->data;
    a.residual = residual ? residual->data : nullptr;
    a.weight = weight;
    a.sum = sum ? const_cast<void*>(sum->data) : nullptr;
    a.y = y ? const_cast<void*>(y->data) : nullptr;
    if (codes) a.codes = codes_of(codes);
    a.rstd = rstd;
    a.n = x->n;
    a.x_stride = stride_of(x);
    a.residual_stride = residual ? stride_of(residual) : 0;
    a.sum_stride = sum ? stride_of(sum) : 0;
    a.y_stride = y ? stride_of(y) : 0;
    a.d = x->d;
    a.eps = eps;
    return done(launch_rms_norm(a, x->dtype, weight_dtype, (hipStream_t)stream));
}

size_t fnn_rms_norm_backward_workspace_bytes(int64_t n, int32_t d) {
    if (n < 0 || n > MAX_SLOTS || d < 1 || d > FNN_MAX_NORM_WIDTH) return 0;
    return (size_t)rms_norm_backward_groups(n, d) * d * sizeof(float);
}

int32_t fnn_rms_norm_backward(const fnn_map* dy, const fnn_map* sum, const float* rstd, const void* weight, int32_t weight_dtype, const fnn_map* dsum,
                              const fnn_map* dx, void* dweight, void* workspace, size_t workspace_bytes, void* stream) {
    FNN_CHECK(check_matrix(dy));
    FNN_CHECK(check_matrix(sum));
    if (sum->d < 1 || sum->d > FNN_MAX_NORM_WIDTH) return FNN_E_SHAPE;
    const fnn_map* others[3] = {dy, dsum, dx};
    for (const fnn_map* m : others) {
        if (!m) continue;
        FNN_CHECK(check_matrix(m));
        if (m->n != sum->n || m->d != sum->d) return FNN_E_SHAPE;
        if (m->dtype != sum->dtype) return FNN_E_DTYPE;
    }
    if (weight_dtype != sum->dtype && weight_dtype != FNN_F32) return FNN_E_DTYPE;
    if (sum->n > 0 && !rstd) return FNN_E_NULL;
    if (dweight) FNN_CHECK(check_workspace(workspace, workspace_bytes, fnn_rms_norm_backward_workspace_bytes(sum->n, sum->d)));
    if (!dweight && (!dx || sum->n == 0)) return FNN_OK;
    RmsBackArgs a;
    memset(&a, 0, sizeof(a));
    a.dy = dy->data;
    a.x = sum->data;
    a.dsum = dsum ? dsum->data : nullptr;
    a.rstd = rstd;
    a.weight = weight;
    a.dx = dx ? const_cast<void*>(dx->data) : nullptr;
    a.dweight = dweight;
    a.partial = dweight ? (float*)workspace : nullptr;
    a.n = sum->n;
    a.dy_stride = stride_of(dy);
    a.x_stride = stride_of(sum);
    a.dsum_stride = dsum ? stride_of(dsum) : 0;
    a.dx_stride = dx ? stride_of(dx) : 0;
    a.d = sum->d;
    return done(launch_rms_norm_backward(a, sum->dtype, weight_dtype, (hipStream_t)stream));
}

size_t fnn_linear_e4m3_workspace_bytes(int64_t rows, int64_t inner, int64_t outer, int32_t dtype) {
    if (!linear_sizes(rows, inner, outer) || !valid_type(dtype)) return 0;
    return scaled_gemm_workspace(rows, outer, inner, dtype, true);
}

int32_t fnn_linear_e4m3(const fnn_scaled* x, const fnn_scaled* w, const void* bias, int32_t act, const fnn_map* residual,
                        const fnn_map* y, const fnn_map* pre, void* workspace, size_t workspace_bytes, void* stream) {
    FNN_CHECK(check_scaled(x));
    FNN_CHECK(check_scaled(w));
    FNN_CHECK(check_matrix(y));
    const int64_t rows = x->n, inner = x->d, outer = w->n;
    if (w->d != inner || !same_shape(y, rows, outer)) return FNN_E_SHAPE;
    const fnn_map* others[2] = {residual, pre};
    for (const fnn_map* m : others) {
        if (!m) continue;
        FNN_CHECK(check_matrix(m));
        if (!same_shape(m, rows, outer)) return FNN_E_SHAPE;
        if (m->dtype != y->dtype) return FNN_E_DTYPE;
    }
    if (act < FNN_ACT_NONE || act > FNN_ACT_SILU) return FNN_E_RANGE;
    FNN_CHECK(check_workspace(workspace, workspace_bytes, scaled_gemm_workspace(rows, outer, inner, y->dtype, true)));
    ScaledGemmArgs a;
    memset(&a, 0, sizeof(a));
    a.g.a = x->data;
    a.g.b = w->data;
    a.g.lda = stride_of(x);
    a.g.ldb = stride_of(w);
    a.g.m = rows;
    a.g.n = (int32_t)outer;
    a.g.k = (int32_t)inner;
    a.g.y = const_cast<void*>(y->data);
    a.g.bias = bias;
    a.g.residual = residual ? residual->data : nullptr;
    a.g.pre = pre ? const_cast<void*>(pre->data) : nullptr;
    a.g.ldy = stride_of(y);
    a.g.ldr = residual ? stride_of(residual) : 0;
    a.g.ldp = pre ? stride_of(pre) : 0;
    a.g.act = act;
    a.g.partial = (float*)workspace;
    a.scale_a = x->scale;
    a.scale_b = w->scale;
    a.sa_row = scale_row_of(x);
    a.sa_block = scale_block_of(x);
    a.sb_row = scale_row_of(w);
    a.sb_block = scale_block_of(w);
    a.shift_a = x->block_rows == 1 ? 0 : 7;
    a.shift_b = w->block_rows == 1 ? 0 : 7;
    return done(launch_scaled_gemm(a, y->dtype, TK_LINEAR_E4M3, (hipStream_t)stream));
}

size_t fnn_linear_e4m3_backward_workspace_bytes(int64_t rows, int64_t inner, int64_t outer, int32_t dtype) {
    if (!linear_sizes(rows, inner, outer) || !valid_type(dtype)) return 0;
    return e4m3_back_layout(rows, inner, outer, dtype).total;
}

int32_t fnn_linear_e4m3_backward(const fnn_map* dy, const fnn_map* x, const fnn_scaled* w, const fnn_map* pre, int32_t act,
                                 const fnn_map* dx, const fnn_map* dw, void* dbias, void* workspace, size_t workspace_bytes, void* stream) {
    FNN_CHECK(check_matrix(dy));
    FNN_CHECK(check_matrix(x));
    FNN_CHECK(check_scaled(w));
    if (act < FNN_ACT_NONE || act > FNN_ACT_SILU) return FNN_E_RANGE;
    const bool slope = act != FNN_ACT_NONE;
    if (slope) FNN_CHECK(check_matrix(pre));
    if (dx) FNN_CHECK(check_matrix(dx));
    if (dw) FNN_CHECK(check_matrix(dw));
    const int64_t rows = x->n, inner = x->d, outer = w->n;
    if (w->d != inner || (w->block_rows != SCALED_BLOCK && outer > 1) || !same_shape(dy, rows, outer) || (slope && !same_shape(pre, rows, outer)) ||
        (dx && !same_shape(dx, rows, inner)) || (dw && !same_shape(dw, outer, inner)))
        return FNN_E_SHAPE;
    if (dy->dtype != x->dtype || (slope && pre->dtype != x->dtype) || (dx && dx->dtype != x->dtype) || (dw && dw->dtype != x->dtype)) return FNN_E_DTYPE;
    if (!dx && !dw && !dbias) return FNN_OK;
    const E4m3BackLayout L = e4m3_back_layout(rows, inner, outer, x->dtype);
    FNN_CHECK(check_workspace(workspace, workspace_bytes, L.total));
    const hipStream_t s = (hipStream_t)stream;
    char* ws = (char*)workspace;

    // q in one pass: by rows for dx, across for dw, the columns' sums for dbias
    GradientOperands o;
    memset(&o, 0, sizeof(o));
    if (rows > 0 && outer > 0) {
        o.q.x = dy->data;
        o.q.pre = slope ? pre->data : nullptr;
        if (dx) o.q.rows = {(uint8_t*)ws + L.q, (float*)(ws + L.q_scale), L.outer_stride, 1, rows};
        if (dw) o.q.across = {(uint8_t*)ws + L.q_across, (float*)(ws + L.q_across_scale), L.rows_stride, 1, outer};
        o.q.partial = dbias ? (float*)(ws + L.sums) : nullptr;
        o.q.n = rows;
        o.q.x_stride = stride_of(dy);
        o.q.pre_stride = slope ? stride_of(pre) : 0;
        o.q.d = (int32_t)outer;
        o.q.act = act;
    }
    if (dw && rows > 0 && inner > 0) {
        o.x.x = x->data;
        o.x.across = {(uint8_t*)ws + L.x, (float*)(ws + L.x_scale), L.rows_stride, 1, inner};
        o.x.n = rows;
        o.x.x_stride = stride_of(x);
        o.x.d = (int32_t)inner;
    }
    if (dx && inner > 0 && outer > 0) o.w = {(const uint8_t*)w->data, (uint8_t*)ws + L.w, stride_of(w), L.outer_stride, outer, (int32_t)inner};
    if (launch_gradient_operands(o, x->dtype, TK_LINEAR_E4M3_BACKWARD, s) != hipSuccess) return FNN_E_HIP;
    ScaledGemmArgs x_grad, w_grad;
    memset(&x_grad, 0, sizeof(x_grad));
    memset(&w_grad, 0, sizeof(w_grad));
    x_grad.g.partial = w_grad.g.partial = (float*)(ws + L.partial);
    if (dx) {
        ScaledGemmArgs& a = x_grad;
        a.g.a = ws + L.q;
        a.g.b = ws + L.w;
        a.g.lda = a.g.ldb = L.outer_stride;
        a.g.m = rows;
        a.g.n = (int32_t)inner;
        a.g.k = (int32_t)outer;
        a.g.y = const_cast<void*>(dx->data);
        a.g.ldy = stride_of(dx);
        a.scale_a = (float*)(ws + L.q_scale);
        a.sa_row = 1;
        a.sa_block = rows;
        a.scale_b = w->scale;          // of the transpose: rows and blocks change places
        a.sb_row = scale_block_of(w);
        a.sb_block = scale_row_of(w);
        a.shift_b = 7;
    }
    if (dw) {
        ScaledGemmArgs& a = w_grad;
        a.g.a = ws + L.q_across;
        a.g.b = ws + L.x;
        a.g.lda = a.g.ldb = L.rows_stride;
        a.g.m = outer;
        a.g.n = (int32_t)inner;
        a.g.k = (int32_t)rows;
        a.g.y = const_cast<void*>(dw->data);
        a.g.ldy = stride_of(dw);
        a.scale_a = (float*)(ws + L.q_across_scale);
        a.sa_row = 1;
        a.sa_block = outer;
        a.scale_b = (float*)(ws + L.x_scale);
        a.sb_row = 1;
        a.sb_block = inner;
    }
    return done(launch_scaled_gradient(x_grad, w_grad, o.q.partial, scaled_blocks(rows), outer, outer > 0 ? dbias : nullptr, x->dtype, TK_LINEAR_E4M3_BACKWARD, s));
}

}  // extern "C"
#pragma GCC visibility pop
