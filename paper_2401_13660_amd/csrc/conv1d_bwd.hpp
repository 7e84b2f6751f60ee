// conv1d_bwd.hpp -- the gradient of the causal depthwise convolution (+ Swish) of conv1d.hpp.
//
// With ext = state_in followed by x (ext[t + j] is what tap j sees at time t, H = k - 1):
//
//   pre[t] = bias + sum_j w[j] ext[t + j],   y[t] = silu(pre[t]),   state_out = the last H of ext
//   g[t]   = dy[t] s (1 + pre (1 - s)),  s = sigmoid(pre[t])           (dy[t] without the Swish)
//   dext[m] = sum_j w[j] g[m - j]  over 0 <= m - j < L,  plus dstate_out[m - L] for m >= L
//   dstate_in = dext[0 .. H),  dx[t] = dext[t + H]
//   dw[j]  = sum over batch and t of g[t] ext[t + j],   dbias = sum of g[t]
//
// pre is computed again from x: storing it would cost a write and a read of the tensor.
#pragma once

#include <hip/hip_runtime.h>

#include "device_math.hpp"

namespace mbs {
namespace convbwd {

constexpr int kThreads = 256;

struct Params {
    int64_t batch, dim, seqlen;
    const void *x;                // (batch, dim, L) act
    const float *w, *bias;        // (dim, K), (dim) or null
    const float *state_in;        // (batch, dim, K-1) or null: zeros
    const void *dy;               // (batch, dim, L) out
    const float *dstate_out;      // (batch, dim, K-1) or null: zeros
    void *dx;                     // (batch, dim, L) out
    float *dw, *dbias;            // (dim, K), (dim) or null
    float *dstate_in;             // (batch, dim, K-1) or null
    float *part;                  // (batch, dim, K + 1): each row's share of dw and dbias
    int apply_silu;
};

// The slope of silu at pre: s (1 + pre (1 - s)).
__device__ __forceinline__ float silu_slope(float pre) {
    const float s = hw_rcp(1.0f + hw_exp2(-pre * kLog2e));
    return s * __builtin_fmaf(pre, 1.0f - s, 1.0f);
}

// One workgroup per row.
template <int IN, int OUT, int K>
__global__ __launch_bounds__(kThreads) void conv1d_bwd(Params p) {
    constexpr int H = K - 1;
    const int64_t L = p.seqlen, rows = p.batch * p.dim;
    __shared__ float red[kThreads];
    for (int64_t row = blockIdx.x; row < rows; row += gridDim.x) {
        const int64_t d = row % p.dim;
        float w[K];
        for (int j = 0; j < K; ++j) w[j] = p.w[d * K + j];
        const float b = p.bias ? p.bias[d] : 0.0f;
        auto ext = [&](int64_t m) {
            if (m < H) return p.state_in ? p.state_in[row * H + m] : 0.0f;
            return Act<IN>::ld(p.x, row * L + m - H);
        };
        auto grad = [&](int64_t t) {
            if (t < 0 || t >= L) return 0.0f;
            float pre = b;
            for (int j = 0; j < K; ++j) pre = __builtin_fmaf(w[j], ext(t + j), pre);
            const float dy = Act<OUT>::ld(p.dy, row * L + t);
            return p.apply_silu ? dy * silu_slope(pre) : dy;
        };
        float acc[K + 1] = {};
        for (int64_t m = threadIdx.x; m < L + H; m += kThreads) {
            float dext = m >= L && p.dstate_out ? p.dstate_out[row * H + m - L] : 0.0f;
            for (int j = 0; j < K; ++j) dext = __builtin_fmaf(w[j], grad(m - j), dext);
            if (m >= H) st_out<OUT>(p.dx, row * L + m - H, dext);
            else if (p.dstate_in) p.dstate_in[row * H + m] = dext;
            const float g = grad(m);
            if (m < L) {
                for (int j = 0; j < K; ++j) acc[j] = __builtin_fmaf(g, ext(m + j), acc[j]);
                acc[K] += g;
            }
        }
        for (int j = 0; j <= K; ++j) {
            red[threadIdx.x] = acc[j];
            __syncthreads();
            for (int n = kThreads / 2; n > 0; n /= 2) {
                if ((int)threadIdx.x < n) red[threadIdx.x] += red[threadIdx.x + n];
                __syncthreads();
            }
            if (threadIdx.x == 0) p.part[row * (K + 1) + j] = red[0];
            __syncthreads();
        }
    }
}

// dw and dbias from the rows' shares, in the order of the batch.
template <int K>
__global__ __launch_bounds__(kThreads) void conv1d_bwd_finish(Params p) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (i >= p.dim * (K + 1)) return;
    const int64_t d = i / (K + 1), j = i - d * (K + 1);
    float sum = 0.0f;
    for (int64_t b = 0; b < p.batch; ++b) sum += p.part[(b * p.dim + d) * (K + 1) + j];
    if (j < K) p.dw[d * K + j] = sum;
    else if (p.dbias) p.dbias[d] = sum;
}

}  // namespace convbwd
}  // namespace mbs
