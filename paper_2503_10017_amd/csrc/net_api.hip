// C entry points of the network's operators (see include/fnn_net.h): argument checks and workspace carving.  Nothing here
// synchronises with the device or allocates memory.
#include <hip/hip_runtime.h>
#include <math.h>
#include <string.h>

#include "fnn_kernels.hpp"
#include "net_kernels.hpp"

using namespace fnn;

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

#define FNN_CHECK(call)                       \
    do {                                      \
        const int32_t status_ = (call);       \
        if (status_ != FNN_OK) return status_; \
    } while (0)

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

}  // extern "C"
#pragma GCC visibility pop
