// grad_clip.hpp -- the global norm of a list of tensors, and the clipping by it.
//
//   norm = sqrt(sum over every element of every tensor of g^2)
//   out  = g                              where norm + eps <= max_norm
//        = g max_norm / (norm + eps)      otherwise (a NaN norm makes every element NaN)
//
// Squares and their sums are fp64: the norm of any finite fp32 gradients neither
// overflows nor vanishes on the way.  Sums are taken in a fixed order.
#pragma once

#include <hip/hip_runtime.h>

#include "device_math.hpp"

namespace mbs {
namespace clip {

constexpr int kThreads = 256;
constexpr int kBlocks = 1024;      // workgroups of one tensor's pass, and partial sums of the norm

__device__ __forceinline__ double block_sum(double v, double *red) {
    red[threadIdx.x] = v;
    __syncthreads();
    for (int n = kThreads / 2; n > 0; n /= 2) {
        if ((int)threadIdx.x < n) red[threadIdx.x] += red[threadIdx.x + n];
        __syncthreads();
    }
    return red[0];
}

// One tensor's squares, added to the partial sums (`first`: written).
template <int DT>
__global__ __launch_bounds__(kThreads) void sum_squares(const void *g, int64_t n, double *part, int first) {
    __shared__ double red[kThreads];
    double sum = 0.0;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)kBlocks * kThreads) {
        const double v = Act<DT>::ld(g, i);
        sum += v * v;
    }
    sum = block_sum(sum, red);
    if (threadIdx.x == 0) part[blockIdx.x] = first ? sum : part[blockIdx.x] + sum;
}

// norm and the factor from the partial sums: out[0], out[1].
__global__ __launch_bounds__(kThreads) void finish_norm(const double *part, int nparts, float max_norm, float eps,
                                                        float *norm, float *factor) {
    __shared__ double red[kThreads];
    double sum = 0.0;
    for (int i = threadIdx.x; i < nparts; i += kThreads) sum += part[i];
    sum = block_sum(sum, red);
    if (threadIdx.x == 0) {
        const float v = (float)__builtin_sqrt(sum);
        *norm = v;
        if (factor) *factor = v + eps <= max_norm ? 1.0f : max_norm / (v + eps);
    }
}

template <int DT>
__global__ __launch_bounds__(kThreads) void scale_by(const void *g, void *out, int64_t n, const float *factor) {
    const float f = *factor;
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < n; i += (int64_t)kBlocks * kThreads)
        st_out<DT>(out, i, f * Act<DT>::ld(g, i));
}

}  // namespace clip
}  // namespace mbs
