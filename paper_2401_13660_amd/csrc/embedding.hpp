// embedding.hpp -- the embedding lookup with scaling, and its gradient.
//
//   y[i]  = scale * W[token_i]                (a negative token is padding: a row of zeros;
//                                              a token >= vocab is a mistake: a row of NaN)
//   dW[v] = scale * sum over i, token_i = v, of dy[i], in the order of i
//
// Tokens are bytes, int32 or int64.  Sums are fp32, rounded once to dW's type.
#pragma once

#include <hip/hip_runtime.h>

#include "device_math.hpp"

namespace mbs {
namespace embed {

constexpr int kThreads = 256;

struct FwdParams {
    int64_t ntokens, vocab, dim;
    const void *tokens, *weight;
    void *out;
    float scale;
};

struct BwdParams {
    int64_t ntokens, vocab, dim;
    const void *tokens, *dy;
    void *dweight;
    float scale;
};

// Tokens by mb_token_type.
template <int TOK> __device__ __forceinline__ int64_t token_at(const void *p, int64_t i) {
    if constexpr (TOK == 0) return static_cast<const uint8_t *>(p)[i];
    else if constexpr (TOK == 1) return static_cast<const int32_t *>(p)[i];
    else return static_cast<const int64_t *>(p)[i];
}

template <int TOK, int W, int OUT>
__global__ __launch_bounds__(kThreads) void embed_fwd(FwdParams p) {
    const int64_t elems = p.ntokens * p.dim, step = (int64_t)gridDim.x * kThreads;
    for (int64_t e = (int64_t)blockIdx.x * kThreads + threadIdx.x; e < elems; e += step) {
        const int64_t i = e / p.dim, t = token_at<TOK>(p.tokens, i);
        float v = t < 0 ? 0.0f : __builtin_nanf("");
        if (t >= 0 && t < p.vocab) v = p.scale * Act<W>::ld(p.weight, t * p.dim + (e - i * p.dim));
        st_out<OUT>(p.out, e, v);
    }
}

// One workgroup per 256 columns of a table row: it reads every token, and adds the rows of its own.
template <int TOK, int DY, int OUT>
__global__ __launch_bounds__(kThreads) void embed_bwd(BwdParams p) {
    const int64_t tiles = (p.dim + kThreads - 1) / kThreads;
    for (int64_t item = blockIdx.x; item < p.vocab * tiles; item += gridDim.x) {
        const int64_t v = item / tiles, col = (item - v * tiles) * kThreads + threadIdx.x;
        float sum = 0.0f;
        for (int64_t i = 0; i < p.ntokens; ++i)
            if (token_at<TOK>(p.tokens, i) == v && col < p.dim) sum += Act<DY>::ld(p.dy, i * p.dim + col);
        if (col < p.dim) st_out<OUT>(p.dweight, v * p.dim + col, p.scale * sum);
    }
}

}  // namespace embed
}  // namespace mbs
