// rms_norm.hpp -- the residual's addition and the root-mean-square norm, in one pass, and their gradients.
//
//   h = x + residual (rounded to the residual's type; x without one)
//   r = 1 / sqrt(mean(h^2) + eps),   y = h r w,   in 32 or 16 bits, or in 8 with a scale for each 128 columns
//
// With g = dy w, u = h r and dh what reaches h from behind:
//
//   d = r (g - u mean(g u)) + dh,    dx = d,  dresidual = d,    dw = sum over rows of dy u
//
// Bound by memory: every tensor passes once.  (32,768, 1792) in bf16 with a residual in fp32 takes 129 us, 5.4 TB/s, and its gradient
// 184 us, 5.1 TB/s, where a 1 GiB copy runs at 5.1; (2042, 1536) in fp32 the gradient 13 us, two launches that wait for chains of
// loads; 32 rows to 8 bits 6.7 us a call, of which the kernel is 3.2.  Streaming loads or stores cost the forward 6 to 17%.  A row stays in registers between its sum and its
// output: 8 columns per lane and span, J spans (1 to 4) per lane, a wave per row for narrow ones (no
// barrier; four rows per workgroup), several waves per row beyond, and a walk that reads its row twice past that.
// The gradient's waves keep dw's sums of their columns in registers from row to row; a workgroup's sums are
// joined in LDS, and a second launch joins the workgroups' in a fixed order.
#pragma once

#include <hip/hip_runtime.h>

#include "device_math.hpp"
#include "fp8.hpp"
#include "lanes.hpp"

namespace mbs {
namespace norm {

constexpr int kNone = 2;            // as RES: no residual
constexpr int kFp8 = 2;             // as OUT: 8 bits with scales
constexpr int kLoopWaves = 16;      // per row of any width

struct FwdParams {
    int64_t rows, dim;
    const void *x;
    const float *weight;            // (dim) or null: ones
    const void *residual;           // (rows, dim) or null
    void *y;
    float *scales;                  // (rows, ceil(dim / 128)) where y is in 8 bits
    void *residual_out;             // (rows, dim): h, may be residual
    float *rstd;                    // (rows) or null
    float eps;
};

struct BwdParams {
    int64_t rows, dim;
    const void *dy, *h;
    const float *rstd;              // (rows)
    const float *weight;            // (dim) or null: ones
    const void *dh;                 // (rows, dim) or null
    void *dx;
    void *dresidual;                // (rows, dim) or null
    float *dweight;                 // (dim) or null
    float *part;                    // (workgroups, dim), or dweight itself where there is one workgroup
};

// Spans of 8 columns, of which n are the row's.  CUT: the row may end within one; else n is 8 or 0.
template <bool CUT, int DT> __device__ __forceinline__ void load8(Span<DT, 8> &s, const void *p, int64_t at, int n) {
    if (n >= 8) s.load(p, at);
    else s.load_first(p, at, CUT ? n : 0);
}
template <bool CUT, int DT> __device__ __forceinline__ void store8(void *p, int64_t at, const float (&v)[8], int n) {
    if (n >= 8) store_span<DT, 8>(p, at, v);
    else if (CUT) store_first<DT, 8>(p, at, v, n);
}

// The sum over a row's W waves; `red` holds two rounds of W values, so that one barrier a row is enough.
template <int W> __device__ __forceinline__ float row_sum(float v, float *red, int round) {
    v = wave_sum(v);
    if constexpr (W > 1) {
        red += (round & 1) * W;
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        v = red[0];
#pragma unroll
        for (int w = 1; w < W; ++w) v += red[w];
    }
    return v;
}

// The columns of a span as the norm sees them.
template <int X, int RES, bool CUT> struct Sum8 {
    Span<X, 8> x;
    Span<RES == kNone ? X : RES, 8> res;
    __device__ __forceinline__ void load(const FwdParams &p, int64_t at, int n) {
        load8<CUT>(x, p.x, at, n);
        if constexpr (RES != kNone) load8<CUT>(res, p.residual, at, n);
    }
    // h, kept in residual_out
    __device__ __forceinline__ void add(const FwdParams &p, int64_t at, int n, float (&h)[8]) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            h[i] = x.get(i);
            if constexpr (RES != kNone) h[i] += res.get(i);
        }
        if constexpr (RES != kNone) {
            store8<CUT, RES>(p.residual_out, at, h, n);
            if constexpr (RES == 1) {
#pragma unroll
                for (int i = 0; i < 8; i += 2) {
                    const uint32_t r = bf16x2_pack(h[i], h[i + 1]);
                    h[i] = bf16_lo(r);
                    h[i + 1] = bf16_hi(r);
                }
            }
        }
    }
};

template <bool CUT> __device__ __forceinline__ void load_weight(const float *weight, int64_t col, int n, float (&w)[8]) {
    Span<0, 8> s;
    if (weight) load8<CUT>(s, weight, col, n);
#pragma unroll
    for (int i = 0; i < 8; ++i) w[i] = weight ? s.get(i) : 1.0f;
}

template <int OUT, bool CUT>
__device__ __forceinline__ void emit(const FwdParams &p, int64_t row, int64_t col, int n, const float (&h)[8], const float (&w)[8], float r) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = h[i] * r * w[i];
    if constexpr (OUT == kFp8) {
        float top = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = __builtin_fmaxf(top, __builtin_fabsf(CUT && i >= n ? 0.0f : y[i]));
        const float scale = fp8::scale_of(fp8::max_of_16(top));
        if (n > 0) {
            fp8::store8(static_cast<uint8_t *>(p.y) + row * p.dim + col, y, 1.0f / scale, CUT ? n : 8);
            if (col % fp8::kBlock == 0) p.scales[row * ((p.dim + fp8::kBlock - 1) / fp8::kBlock) + col / fp8::kBlock] = scale;
        }
    } else {
        if (n > 0) store8<CUT, OUT>(p.y, row * p.dim + col, y, n);
    }
}

__device__ __forceinline__ float inverse_length(float squares, const FwdParams &p) {
    return 1.0f / sqrtf(squares / (float)p.dim + p.eps);
}

// Columns of a span within the row: 8, fewer at its end, none past it.
template <bool CUT> __device__ __forceinline__ int within(int64_t dim, int64_t col) {
    return CUT ? (int)min((int64_t)8, max((int64_t)0, dim - col)) : col < dim ? 8 : 0;
}

template <int X, int RES, int OUT, int W, int J, bool CUT>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void rms_norm_rows(FwdParams p) {
    constexpr int kRows = W == 1 ? 4 : 1;
    __shared__ float red[2 * W];
    const int t = W == 1 ? threadIdx.x & 63 : threadIdx.x;
    const int64_t step = (int64_t)gridDim.x * kRows;
    int round = 0;
    for (int64_t row = (int64_t)blockIdx.x * kRows + (W == 1 ? threadIdx.x >> 6 : 0); row < p.rows; row += step, ++round) {
        Sum8<X, RES, CUT> in[J];
        float h[J][8], w[J][8];
        const int64_t at = row * p.dim;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int64_t col = 8 * (j * 64 * W + t);
            in[j].load(p, at + col, within<CUT>(p.dim, col));
            // ahead where the registers are there for it; rows of more spans hide its latency behind each other
            if (J == 1) load_weight<CUT>(p.weight, col, within<CUT>(p.dim, col), w[j]);
        }
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int64_t col = 8 * (j * 64 * W + t);
            in[j].add(p, at + col, within<CUT>(p.dim, col), h[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(h[j][i], h[j][i], sum);
        }
        float whole;
        if constexpr (W > 1) whole = row_sum<W>(sum, red, round);
        else whole = wave_sum(sum);
        const float r = inverse_length(whole, p);
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int64_t col = 8 * (j * 64 * W + t);
            if (J > 1) load_weight<CUT>(p.weight, col, within<CUT>(p.dim, col), w[j]);
            emit<OUT, CUT>(p, row, col, within<CUT>(p.dim, col), h[j], w[j], r);
        }
        if (p.rstd && t == 0) p.rstd[row] = r;
    }
}

// Rows of any width.  The second reading is of what the same thread wrote.
template <int X, int RES, int OUT>
__global__ __launch_bounds__(64 * kLoopWaves) void rms_norm_walk(FwdParams p) {
    __shared__ float red[2 * kLoopWaves];
    const int t = threadIdx.x;
    int round = 0;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, ++round) {
        const int64_t at = row * p.dim;
        float sum = 0.0f;
        for (int64_t first = 0; first < p.dim; first += 8 * 64 * kLoopWaves) {
            const int64_t col = first + 8 * t;
            const int n = within<true>(p.dim, col);
            Sum8<X, RES, true> in;
            float h[8];
            in.load(p, at + col, n);
            in.add(p, at + col, n, h);
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = __builtin_fmaf(h[i], h[i], sum);
        }
        const float r = inverse_length(row_sum<kLoopWaves>(sum, red, round), p);
        for (int64_t first = 0; first < p.dim; first += 8 * 64 * kLoopWaves) {
            const int64_t col = first + 8 * t;
            const int n = within<true>(p.dim, col);
            Span<RES == kNone ? X : RES, 8> s;
            float h[8], w[8];
            load8<true>(s, RES == kNone ? p.x : p.residual_out, at + col, n);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] = s.get(i);
            load_weight<true>(p.weight, col, n, w);
            emit<OUT, true>(p, row, col, n, h, w, r);
        }
        if (p.rstd && t == 0) p.rstd[row] = r;
    }
}

// One span of a row's gradient.
template <int DY, int H, bool CUT> struct Grad8 {
    Span<DY, 8> dy;
    Span<H, 8> h, dh;
    __device__ __forceinline__ void load(const BwdParams &p, int64_t at, int n) {
        load8<CUT>(dy, p.dy, at, n);
        load8<CUT>(h, p.h, at, n);
        if (p.dh) load8<CUT>(dh, p.dh, at, n);
    }
    template <int DX>
    __device__ __forceinline__ void store(const BwdParams &p, int64_t at, int n, const float (&w)[8], float r, float along) const {
        float d[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            d[i] = r * __builtin_fmaf(h.get(i) * r, -along, dy.get(i) * w[i]);
            if (p.dh) d[i] += dh.get(i);
        }
        if (n > 0) {
            store8<CUT, DX>(p.dx, at, d, n);
            if (p.dresidual) store8<CUT, H>(p.dresidual, at, d, n);
        }
    }
};

template <int DY, int H, int DX, int W, int J, bool CUT>
__global__ __launch_bounds__(W == 1 ? 256 : 64 * W) void rms_norm_bwd_rows(BwdParams p) {
    constexpr int kRows = W == 1 ? 4 : 1;
    __shared__ float red[2 * W];
    __shared__ float joined[W == 1 ? 64 * J * 8 : 1];
    const int t = W == 1 ? threadIdx.x & 63 : threadIdx.x, wave = threadIdx.x >> 6;
    const int64_t step = (int64_t)gridDim.x * kRows;
    float dw[J][8] = {};
    int round = 0;
    for (int64_t row = (int64_t)blockIdx.x * kRows + (W == 1 ? wave : 0); row < p.rows; row += step, ++round) {
        Grad8<DY, H, CUT> in[J];
        float w[J][8];
        const int64_t at = row * p.dim;
        const float r = p.rstd[row];
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int64_t col = 8 * (j * 64 * W + t);
            const int n = within<CUT>(p.dim, col);
            in[j].load(p, at + col, n);
            load_weight<CUT>(p.weight, col, n, w[j]);
        }
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < J; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float u = in[j].h.get(i) * r, g = in[j].dy.get(i);
                sum = __builtin_fmaf(g * w[j][i], u, sum);
                dw[j][i] = __builtin_fmaf(g, u, dw[j][i]);
            }
        const float along = row_sum<W>(sum, red, round) / (float)p.dim;
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int64_t col = 8 * (j * 64 * W + t);
            in[j].template store<DX>(p, at + col, within<CUT>(p.dim, col), w[j], r, along);
        }
    }
    if (!p.dweight) return;
    float *out = p.part + (int64_t)blockIdx.x * p.dim;
    if constexpr (W == 1) {
        for (int k = 3; k >= 0; --k) {                  // the waves' sums, one after the other
            if (wave == k) {
#pragma unroll
                for (int j = 0; j < J; ++j)
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float &s = joined[8 * (64 * j + t) + i];
                        if (k < 3) dw[j][i] += s;
                        s = dw[j][i];
                    }
            }
            __syncthreads();
        }
        if (wave != 0) return;
    }
#pragma unroll
    for (int j = 0; j < J; ++j) {
        const int64_t col = 8 * (j * 64 * W + t);
        const int n = within<CUT>(p.dim, col);
        if (n > 0) store8<CUT, 0>(out, col, dw[j], n);
    }
}

// Rows of any width: dw's sums are kept in the workgroup's part, where each column belongs to one thread.
template <int DY, int H, int DX>
__global__ __launch_bounds__(64 * kLoopWaves) void rms_norm_bwd_walk(BwdParams p) {
    __shared__ float red[2 * kLoopWaves];
    const int t = threadIdx.x;
    float *out = p.part + (int64_t)blockIdx.x * p.dim;
    int round = 0;
    for (int64_t row = blockIdx.x; row < p.rows; row += gridDim.x, ++round) {
        const int64_t at = row * p.dim;
        const float r = p.rstd[row];
        float sum = 0.0f;
        for (int64_t first = 0; first < p.dim; first += 8 * 64 * kLoopWaves) {
            const int64_t col = first + 8 * t;
            const int n = within<true>(p.dim, col);
            if (n <= 0) continue;
            Span<DY, 8> dy;
            Span<H, 8> h;
            float w[8], dw[8];
            load8<true>(dy, p.dy, at + col, n);
            load8<true>(h, p.h, at + col, n);
            load_weight<true>(p.weight, col, n, w);
            Span<0, 8> before;
            if (p.dweight && round > 0) load8<true>(before, out, col, n);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float u = h.get(i) * r, g = dy.get(i);
                sum = __builtin_fmaf(g * w[i], u, sum);
                dw[i] = round > 0 && p.dweight ? __builtin_fmaf(g, u, before.get(i)) : g * u;
            }
            if (p.dweight) store8<true, 0>(out, col, dw, n);
        }
        const float along = row_sum<kLoopWaves>(sum, red, round) / (float)p.dim;
        for (int64_t first = 0; first < p.dim; first += 8 * 64 * kLoopWaves) {
            const int64_t col = first + 8 * t;
            const int n = within<true>(p.dim, col);
            if (n <= 0) continue;
            Grad8<DY, H, true> in;
            float w[8];
            in.load(p, at + col, n);
            load_weight<true>(p.weight, col, n, w);
            in.template store<DX>(p, at + col, n, w, r, along);
        }
    }
}

constexpr int kJoinColumns = 16, kJoinShares = 64;

// dw from the workgroups' sums: kJoinShares threads take every kJoinShares-th part each of a column, and are joined as a tree.
__global__ __launch_bounds__(kJoinColumns * kJoinShares) void rms_norm_join(const float *part, int32_t parts, int64_t dim, float *dweight) {
    __shared__ float sums[kJoinShares][kJoinColumns];
    const int c = threadIdx.x % kJoinColumns, s = threadIdx.x / kJoinColumns;
    const int64_t col = (int64_t)blockIdx.x * kJoinColumns + c;
    float sum = 0.0f;
    if (col < dim)
        for (int i = s; i < parts; i += kJoinShares) sum += part[i * dim + col];
    sums[s][c] = sum;
    __syncthreads();
    for (int half = kJoinShares / 2; half > 0; half /= 2) {
        if (s < half) sums[s][c] += sums[s + half][c];
        __syncthreads();
    }
    if (s == 0 && col < dim) dweight[col] = sums[0][c];
}

}  // namespace norm
}  // namespace mbs
