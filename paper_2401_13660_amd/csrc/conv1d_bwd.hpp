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
// A lane sums a tile's products, then the tiles', and so on: dw's rounding grows with the tiles of a row, not its timesteps.
//
// Bound by HBM: 6 bytes and 33 VALU instructions (two of them transcendental) per bf16 element.
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
    float *part;                  // (nseg, batch, dim, K + 1): each stretch's share of dw and dbias; null: nseg and batch are 1
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

// A span with the row's end in it or before it: zeros past the end.  It was read where the row's last whole span lies (L
// at least S), `past` elements early, and moves to its place; without CUT that is by all of S or not at all.
template <int S, bool CUT> __device__ __forceinline__ void end_span(float *v, int64_t past) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
        float r = 0.0f;
#pragma unroll
        for (int k = i; k < (CUT ? S : i + 1); ++k) r = past == k - i ? v[k] : r;
        v[i] = r;
    }
}

// g from dy, in place; xin: the H inputs before the span and the span's.
template <int S, int K> __device__ __forceinline__ void through_swish(float *g, const float *xin, const float *w, float bias) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
        float pre = bias;
#pragma unroll
        for (int j = 0; j < K; ++j) pre = __builtin_fmaf(w[j], xin[i + j], pre);
        g[i] *= silu_slope(pre);
    }
}

template <int S, int K> __device__ __forceinline__ void add_products(float *acc, const float *g, const float *xin) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
#pragma unroll
        for (int j = 0; j < K; ++j) acc[j] = __builtin_fmaf(g[i], xin[i + j], acc[j]);
        acc[K] += g[i];
    }
}

// dx of a span from its g and the H values after it.
template <int S, int K> __device__ __forceinline__ void back_through_taps(float (&dx)[S], const float *g, const float *w) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
        dx[i] = 0.0f;
#pragma unroll
        for (int j = 0; j < K; ++j) dx[i] = __builtin_fmaf(w[j], g[i + K - 1 - j], dx[i]);
    }
}

// The rows' ends.  Past a row's end the kernels below have g = 0, and take its products with the inputs and taps beside it as
// they take all others.  That adds nothing, unless such an input or tap is infinite or NaN: then the product is NaN, where by
// the definition there is no term.  With the Swish that changes nothing, since g beside the end, and all that it enters, is
// NaN then.  Without it, a wave that finds a NaN there, or a tap that is not finite, takes these sums, the last H of dx and
// dstate_in again from memory, timestep by timestep and only of what exists.  (Selecting the terms as they are taken cost 3 to
// 10% of the time of every call.)
template <int IN, int OUT, int K> struct Singly {
    static constexpr int H = K - 1;
    const Params &p;
    int64_t row;
    __device__ __forceinline__ float ext(int64_t m) const {
        if (m >= H) return Act<IN>::ld(p.x, row * p.seqlen + m - H);
        return p.state_in ? p.state_in[row * H + m] : 0.0f;
    }
    __device__ __forceinline__ float g(int64_t t) const { return Act<OUT>::ld(p.dy, row * p.seqlen + t); }
    // over every step-th timestep of [from, to)
    __device__ __forceinline__ void sums(float (&acc)[K + 1], int64_t from, int64_t to, int step) const {
#pragma unroll
        for (int j = 0; j <= K; ++j) acc[j] = 0.0f;
        for (int64_t t = from; t < to; t += step) {
            const float v = g(t);
#pragma unroll
            for (int j = 0; j < K; ++j) acc[j] = __builtin_fmaf(v, ext(t + j), acc[j]);
            acc[K] += v;
        }
    }
    __device__ __forceinline__ float dext(int64_t m) const {
        float v = p.dstate_out && m >= p.seqlen ? p.dstate_out[row * H + m - p.seqlen] : 0.0f;
#pragma unroll
        for (int j = 0; j < K; ++j)
            if (m >= j && m - j < p.seqlen) v = __builtin_fmaf(p.w[row % p.dim * K + j], g(m - j), v);
        return v;
    }
    // the first values were stored by other lanes, and are there before these follow; i < H
    __device__ __forceinline__ void ends(int64_t from, int64_t to, int i) const {
        const int64_t t = p.seqlen - H + i;
        if (t >= from && t < to) st_out<OUT>(p.dx, row * p.seqlen + t, dext(t + H));
        if (from == 0 && p.dstate_in) p.dstate_in[row * H + i] = dext(i);
    }
};

// A stretch's sum j: of dw's tap j, or (K) of dbias.  One sequence in one stretch per row: the result itself.
template <int K> __device__ __forceinline__ void put_sum(const Params &p, int64_t item, int j, float s) {
    if (p.part) p.part[item * (K + 1) + j] = s;
    else if (j < K) p.dw[item * K + j] = s;
    else if (p.dbias) p.dbias[item] = s;
}

// Rows of no timestep, or of more than 64 spans.  CUT: L is no multiple of the span, so a row's last span is cut.  The
// instantiations without need 91 to 97 registers, 5 waves per SIMD; with it up to 119, and 4.
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

    // for the row's end after the walk: the same in scalar registers, which costs the walk none of its own
    const int begin = __builtin_amdgcn_readfirstlane(first), end = __builtin_amdgcn_readfirstlane(last);
    const int row_at = __builtin_amdgcn_readfirstlane((int)row);    // rows are fewer than 2^26

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
        const int64_t t = min((int64_t)tile * T + lane * S, L - S);    // past the row's end: the last whole span, shifted below
        xs.template load<true>(p.x, base + t);
        ys.template load<true>(p.dy, base + t);
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
        if (!whole) {
            const int64_t past = max(t0 + S - L, (int64_t)0);
            end_span<S, CUT>(xin + H, past);
            end_span<S, CUT>(g, past);
        }
#pragma unroll
        for (int j = 0; j < H; ++j) xin[j] = from_lane_before(xin[S + j], lane_value(halo, j));
        if (tile > first) load(tile - 1);

        if (p.apply_silu) through_swish<S, K>(g, xin, w, bias);
        if (!whole) {                                   // what the Swish made of inputs beside the end
#pragma unroll
            for (int i = 0; i < S; ++i) g[i] = t0 + i < L ? g[i] : 0.0f;
        }
        float part[K + 1] = {};                         // a tile's sums of their own: a row's one running sum would round L / 64 times
        add_products<S, K>(part, g, xin);
#pragma unroll
        for (int j = 0; j <= K; ++j) acc[j] += part[j];
#pragma unroll
        for (int j = 0; j < H; ++j) {
            g[S + j] = from_lane_after(g[j], carry[j]);
            carry[j] = lane_value(g[j], 0);
        }
        float dx[S];
        back_through_taps<S, K>(dx, g, w);
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
    if (H > 0 && !p.apply_silu && (int64_t)(end + 1) * T > L - H) {
        float odd = 0.0f, taps = 0.0f;                  // NaN where there is something
#pragma unroll
        for (int j = 0; j < K; ++j) {
            odd += acc[j];
            taps = __builtin_fmaf(w[j], 0.0f, taps);
        }
        const bool beside = (int64_t)end * T + lane * S + S > L && odd != odd;
        if (__ballot(beside || taps != taps) != 0) {
            const Singly<IN, OUT, K> singly{p, row_at};
            const int64_t from = (int64_t)begin * T, to = min((int64_t)(end + 1) * T, L);
            wait_for_memory();
            singly.sums(acc, from + lane, to, 64);
            if (lane < H) singly.ends(from, to, lane);
        }
    }
#pragma unroll
    for (int j = 0; j <= K; ++j) {
        const float s = wave_sum(acc[j]);
        if (lane == j) put_sum<K>(p, item, j, s);
    }
}

// Rows of at most G spans: 64 / G of them side by side in a wave, each whole in its lanes.  (4, 4608, 64) bf16 takes 11
// us with the finish, a row in each wave took 19; (64, 3584, 16) 41 and 161; (4, 4608, 257), a row in each wave either
// way, 18 and 25 in the walk above, which has the edges of its stretches to look after.
template <int IN, int OUT, int K, int G>
__global__ __launch_bounds__(kThreads) void conv1d_bwd_short(Params p) {
    constexpr int H = K - 1, HH = H > 0 ? H : 1, S = kSpan<IN, OUT>;
    const int64_t L = p.seqlen, rows = p.batch * p.dim;
    const int lane = threadIdx.x & 63, l = lane & (G - 1);
    const int64_t asked = ((int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6)) * (64 / G) + lane / G;
    const bool active = asked < rows;                   // lanes without a row do the last one's work and write nothing
    const int64_t row = active ? asked : rows - 1, d = row % p.dim, base = row * L, t0 = (int64_t)l * S;
    Span<IN, S> xs;
    Span<OUT, S> ys;
    if (L >= S) {
        xs.load(p.x, base + min(t0, L - S));
        ys.load(p.dy, base + min(t0, L - S));
    } else {
        const int n = (int)max((int64_t)0, L - t0);
        xs.load_first(p.x, base + (n > 0 ? t0 : 0), n);
        ys.load_first(p.dy, base + (n > 0 ? t0 : 0), n);
    }
    float w[K], first[HH] = {};
#pragma unroll
    for (int j = 0; j < K; ++j) w[j] = p.w[d * K + j];
    const float bias = p.bias ? p.bias[d] : 0.0f;
    if (p.state_in) {
#pragma unroll
        for (int j = 0; j < H; ++j) first[j] = p.state_in[row * H + j];
    }
    float xin[H + S], g[S + HH], acc[K + 1] = {}, dx[S];
#pragma unroll
    for (int i = 0; i < S; ++i) {
        xin[H + i] = xs.get(i);
        g[i] = ys.get(i);
    }
    if (L >= S) {
        const int64_t past = max(t0 + S - L, (int64_t)0);
        end_span<S, true>(xin + H, past);
        end_span<S, true>(g, past);
    }
#pragma unroll
    for (int j = 0; j < H; ++j) {
        const float v = from_lane_before(xin[S + j], 0.0f);
        xin[j] = l == 0 ? first[j] : v;
    }
    if (p.apply_silu) through_swish<S, K>(g, xin, w, bias);
#pragma unroll
    for (int i = 0; i < S; ++i) g[i] = t0 + i < L ? g[i] : 0.0f;
    add_products<S, K>(acc, g, xin);
#pragma unroll
    for (int j = 0; j < H; ++j) {
        const float v = from_lane_after(g[j], 0.0f);
        g[S + j] = l == G - 1 ? 0.0f : v;
    }
    back_through_taps<S, K>(dx, g, w);
    if (H > 0 && p.dstate_out) {
#pragma unroll
        for (int i = 0; i < S; ++i)
            if (t0 + i >= L - H && t0 + i < L) dx[i] += p.dstate_out[row * H + t0 + i + H - L];
    }
    if (active && t0 < L) {
        if (t0 + S <= L) store_span<OUT, S>(p.dx, base + t0, dx);
        else store_first<OUT, S>(p.dx, base + t0, dx, (int)(L - t0));
    }
    if (H > 0 && p.dstate_in) {
        float v = p.dstate_out && l >= L && l < H ? p.dstate_out[row * H + l - L] : 0.0f;
#pragma unroll
        for (int k = 0; k < H; ++k) {
            const float gk = __shfl(g[k], lane & ~(G - 1), 64);
#pragma unroll
            for (int m = k; m < H; ++m) v = l == m ? __builtin_fmaf(w[m - k], gk, v) : v;
        }
        if (active && l < H) p.dstate_in[row * H + l] = v;
    }
    if (H > 0 && !p.apply_silu) {
        float odd = 0.0f;                               // NaN where there is something, or an infinite sum
#pragma unroll
        for (int j = 0; j < K; ++j) odd = __builtin_fmaf(acc[j], 0.0f, __builtin_fmaf(w[j], 0.0f, odd));
        const uint64_t where = __ballot(odd != odd);
        if (where != 0) {
            wait_for_memory();
            if (where >> (lane & ~(G - 1)) & (~0ull >> (64 - G))) {     // in this row
                const Singly<IN, OUT, K> singly{p, row};
                singly.sums(acc, l, L, G);
                if (active && l < H) singly.ends(0, L, l);
            }
        }
    }
#pragma unroll
    for (int j = 0; j <= K; ++j) {
        float s = acc[j];
#pragma unroll
        for (int off = 1; off < G; off *= 2) s += __shfl_xor(s, off, 64);
        if (active && l == j) put_sum<K>(p, row, j, s);
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
