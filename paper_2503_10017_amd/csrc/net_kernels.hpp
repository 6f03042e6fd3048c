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

}  // namespace fnn
