// Optional per-kernel timing: when a trace is open every kernel launch of the library is
// bracketed by a pair of HIP events attached to the dispatch itself, so the elapsed time of
// a pair is that kernel's own duration.  Closed (the default), launches are plain.
#pragma once
#include <hip/hip_ext.h>
#include <hip/hip_runtime.h>

namespace fnn {

enum TraceKind : int {
    TK_PREP = 0,
    TK_FILL = 1,
    TK_SEARCH = 2,
    TK_RESERVED_3 = 3,  // numbers are part of what fnn_trace_end reports: retired kinds keep theirs
    TK_RESERVED_4 = 4,
    TK_RECIP_STEP = 5,
    TK_RECIP_DEDUP = 6,
    TK_DENSE = 7,
    TK_DENSE_FINAL = 8,
    TK_RESOLVE = 9,
    TK_DENSE_RESOLVE = 10,
    TK_BLOCKED = 11,
    TK_PIXELS = 12,
    TK_RECIP_WALK = 13,
    TK_QUANTISE = 14,
    TK_COARSE = 15,
    TK_REFINE = 16,
    TK_DENSE_SELECT = 17,
    TK_RECIP_GROUPS = 18,
    TK_DENSE_SAMPLE = 19,
    TK_DENSE_ALIKE = 20,
    TK_RECIP_TAIL = 21,
    TK_LAYER_NORM = 22,
    TK_LAYER_NORM_BACKWARD = 23,
    TK_LINEAR = 24,
    TK_LINEAR_BACKWARD = 25,
    TK_ATTENTION = 26,
    TK_ATTENTION_BACKWARD = 27,
    TK_RMS_NORM = 28,
    TK_RMS_NORM_BACKWARD = 29,
    TK_QUANTIZE = 30,
    TK_LINEAR_E4M3 = 31,
    TK_LINEAR_E4M3_BACKWARD = 32,
    TK_COUNT = 33
};

// Returns false when no trace is open or it is full; otherwise hands out the next event pair.
// `detail` is a number the launcher wants reported with the kernel (the launch shape it chose).
bool trace_next(int kind, int detail, hipEvent_t* start, hipEvent_t* stop);

// A launch has fewer than 2^32 threads in each direction; the runtime takes one of more and leaves workgroups out without an error.
inline bool launch_fits(dim3 grid, dim3 block) {
    return (uint64_t)grid.x * block.x <= UINT32_MAX && (uint64_t)grid.y * block.y <= UINT32_MAX && (uint64_t)grid.z * block.z <= UINT32_MAX;
}
template <typename Kernel, typename... Args>
inline hipError_t launch_detail(int kind, int detail, Kernel kernel, dim3 grid, dim3 block, size_t lds_bytes,
                                hipStream_t s, Args... args) {
    if (!launch_fits(grid, block)) return hipErrorInvalidConfiguration;
    hipEvent_t e0, e1;
    if (trace_next(kind, detail, &e0, &e1)) {
        hipExtLaunchKernelGGL(kernel, grid, block, lds_bytes, s, e0, e1, 0, args...);
    } else {
        hipLaunchKernelGGL(kernel, grid, block, lds_bytes, s, args...);
    }
    return hipGetLastError();
}
template <typename Kernel, typename... Args>
inline hipError_t launch(int kind, Kernel kernel, dim3 grid, dim3 block, size_t lds_bytes, hipStream_t s, Args... args) {
    return launch_detail(kind, 0, kernel, grid, block, lds_bytes, s, args...);
}
// Calls f(first, grid) for one launch after the other of `groups` workgroups of `threads` threads, none of which has too many.
template <typename F>
inline hipError_t in_launches(int64_t groups, int threads, F f) {
    const int64_t most = ((int64_t)1 << 30) / threads;
    for (int64_t first = 0; first < groups; first += most) {
        const hipError_t e = f((uint32_t)first, dim3((unsigned)(groups - first < most ? groups - first : most)));
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace fnn
