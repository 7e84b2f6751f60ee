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
//
// A wave takes a stretch of one row and walks it from its end to its start in tiles of 64 spans, one
// span per lane.  A lane's H inputs before its span and the H values of g after it come from the
// lanes beside it; the g after a tile's last lane are those of the tile just done (or, at the
// stretch's end, computed there again), so x and dy are read once and dx is written once.  The next
// tile's loads are on their way while a tile is computed.
//
// Bound by HBM: 6 bytes and about 22 VALU instructions and 2 transcendentals per bf16 element.
// (4, 3584, 8192) bf16 takes 132 us, 5.3 TB/s, a little over the rate of a device copy (5.17); with
// ordinary instead of streaming loads and stores 147, with streaming stores alone 142, streaming loads
// alone 149.  One stretch per row there: with 2 (4) per row it took 150 (158), the waves' ends and the
// edges' second computation.
#pragma once

#include <hip/hip_runtime.h>

#include "device_math.hpp"
#include "lanes.hpp"

namespace mbs {
namespace convbwd {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;

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
    float *part;                  // (nseg, batch, dim, K + 1): each stretch's share of dw and dbias
    int64_t nseg;                 // stretches per row
    int32_t seg_tiles;            // tiles per stretch
    int apply_silu;
};

// Elements per lane: 16 bytes of the narrower of x and dy.
template <int IN, int OUT> constexpr int kSpan = IN == 0 && OUT == 0 ? 4 : 8;

// The slope of silu at pre: s (1 + pre (1 - s)).
__device__ __forceinline__ float silu_slope(float pre) {
    const float s = hw_rcp(1.0f + hw_exp2(-pre * kLog2e));
    return s * __builtin_fmaf(pre, 1.0f - s, 1.0f);
}

// CUT: L is no multiple of the span, so a row's last span is cut.
template <int IN, int OUT, int K, bool CUT>
__global__ __launch_bounds__(kThreads) void conv1d_bwd(Params p) {
    constexpr int H = K - 1, HH = H > 0 ? H : 1, S = kSpan<IN, OUT>, T = 64 * S;
    const int64_t L = p.seqlen, rows = p.batch * p.dim;
    const int64_t item = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    if (item >= rows * p.nseg) return;
    const int lane = threadIdx.x & 63;
    const int64_t seg = item / rows, row = item - seg * rows, d = row % p.dim, base = row * L;
    const int first = (int)(seg * p.seg_tiles);
    const int ntiles = (int)((L + T - 1) / T);
    const int last = min(first + p.seg_tiles, ntiles) - 1;     // below `first` only for L = 0

    float w[K];
#pragma unroll
    for (int j = 0; j < K; ++j) w[j] = p.w[d * K + j];
    const float bias = p.bias ? p.bias[d] : 0.0f;
    // the input at time t < 0 of the row's beginning, or of the tile before
    auto before = [&](int64_t t) -> float {
        if (t >= 0) return Act<IN>::ld(p.x, base + t);
        return p.state_in ? p.state_in[row * H + t + H] : 0.0f;
    };

    // g after the stretch
    float carry[HH] = {};
    if (H > 0 && last >= first) {
        const int64_t t = (int64_t)(last + 1) * T + lane;
        float g = 0.0f;
        if (lane < H && t < L) {
            float pre = bias;
#pragma unroll
            for (int j = 0; j < K; ++j) pre = __builtin_fmaf(w[j], before(t - H + j), pre);
            g = Act<OUT>::ld(p.dy, base + t);
            if (p.apply_silu) g *= silu_slope(pre);
        }
#pragma unroll
        for (int j = 0; j < H; ++j) carry[j] = lane_value(g, j);
    }

    Span<IN, S> xs;
    Span<OUT, S> ys;
    float halo = 0.0f;                                          // lane j < H: the input H - j before the tile
    auto load = [&](int tile) {
        const int64_t t = (int64_t)tile * T + lane * S;
        if (L >= S) {                                   // a span past the row's end: the last whole one, shifted below
            xs.template load<true>(p.x, base + min(t, L - S));
            ys.template load<true>(p.dy, base + min(t, L - S));
        } else {
            const int n = (int)max((int64_t)0, min(L - t, (int64_t)S));
            xs.load_first(p.x, base + t, n);
            ys.load_first(p.dy, base + t, n);
        }
        if (H > 0 && lane < H) halo = before((int64_t)tile * T - H + lane);
    };

    float acc[K + 1] = {};
    if (last >= first) load(last);
    for (int tile = last; tile >= first; --tile) {
        const int64_t t0 = (int64_t)tile * T + lane * S;
        float xin[H + S], g[S + HH];
        const bool whole = (int64_t)(tile + 1) * T <= L;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            xin[H + i] = xs.get(i);
            g[i] = ys.get(i);
        }
        if (!whole && L >= S) {
            // zeros past the end; a cut span, read where the row's last whole one lies, moves to its place
            const int64_t past = max(t0 + S - L, (int64_t)0);
#pragma unroll
            for (int i = 0; i < S; ++i) {
                float xi = 0.0f, gi = 0.0f;
#pragma unroll
                for (int k = i; k < (CUT ? S : i + 1); ++k) {
                    xi = past == k - i ? xin[H + k] : xi;
                    gi = past == k - i ? g[k] : gi;
                }
                xin[H + i] = xi;
                g[i] = gi;
            }
        }
#pragma unroll
        for (int j = 0; j < H; ++j) xin[j] = from_lane_before(xin[S + j], lane_value(halo, j));
        if (tile > first) load(tile - 1);

        if (p.apply_silu) {
#pragma unroll
            for (int i = 0; i < S; ++i) {
                float pre = bias;
#pragma unroll
                for (int j = 0; j < K; ++j) pre = __builtin_fmaf(w[j], xin[i + j], pre);
                g[i] *= silu_slope(pre);
            }
        }
        if (!whole) {                                   // nor does an infinity beside the end reach past it
#pragma unroll
            for (int i = 0; i < S; ++i) g[i] = t0 + i < L ? g[i] : 0.0f;
        }
#pragma unroll
        for (int i = 0; i < S; ++i) {
#pragma unroll
            for (int j = 0; j < K; ++j) acc[j] = __builtin_fmaf(g[i], xin[i + j], acc[j]);
            acc[K] += g[i];
        }
#pragma unroll
        for (int j = 0; j < H; ++j) {
            g[S + j] = from_lane_after(g[j], carry[j]);
            carry[j] = lane_value(g[j], 0);
        }
        float dx[S];
#pragma unroll
        for (int i = 0; i < S; ++i) {
            dx[i] = 0.0f;
#pragma unroll
            for (int j = 0; j < K; ++j) dx[i] = __builtin_fmaf(w[j], g[i + H - j], dx[i]);
        }
        if (H > 0 && p.dstate_out && (int64_t)(tile + 1) * T > L - H) {
#pragma unroll
            for (int i = 0; i < S; ++i)
                if (t0 + i >= L - H && t0 + i < L) dx[i] += p.dstate_out[row * H + t0 + i + H - L];
        }
        if (t0 + S <= L) store_span<OUT, S, true>(p.dx, base + t0, dx);
        else if (CUT) store_first<OUT, S>(p.dx, base + t0, dx, (int)max((int64_t)0, L - t0));
    }

    if (H > 0 && first == 0 && p.dstate_in && lane < H) {
        // dext[m], m < H: carry holds g[0 .. H), zeros past L
        float v = p.dstate_out && lane >= L ? p.dstate_out[row * H + lane - L] : 0.0f;
#pragma unroll
        for (int j = 0; j < H; ++j)
#pragma unroll
            for (int m = j; m < H; ++m) v = lane == m ? __builtin_fmaf(w[j], carry[m - j], v) : v;
        p.dstate_in[row * H + lane] = v;
    }
#pragma unroll
    for (int j = 0; j <= K; ++j) {
        const float s = wave_sum(acc[j]);
        if (lane == j) p.part[item * (K + 1) + j] = s;
    }
}

// dw and dbias from the stretches' shares, in the order of the stretches and of the batch.
template <int K>
__global__ __launch_bounds__(kThreads) void conv1d_bwd_finish(Params p) {
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x, n = p.dim * (K + 1);
    if (i >= n) return;
    const int64_t d = i / (K + 1), j = i - d * (K + 1);
    float sum = 0.0f;
#pragma unroll 8
    for (int64_t b = 0; b < p.nseg * p.batch; ++b) sum += p.part[b * n + i];
    if (j < K) p.dw[d * K + j] = sum;
    else if (p.dbias) p.dbias[d] = sum;
}

}  // namespace convbwd
}  // namespace mbs
