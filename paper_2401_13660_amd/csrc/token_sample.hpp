// token_sample.hpp -- the next token by temperature, top-k, top-p and min-p, from given random numbers.
//
// In the order of falling logits, the lowest index first among equals, with e = exp((l - largest) / T):
//
//   top-k keeps the first k;   S = what they sum to
//   top-p keeps those before which less than p S lies (and the first);   min-p those of e >= min_p
//   token = the y of the largest e(y) / noise(y) of the kept, the lowest such y;   prob = e(token) / the kept sum
#pragma once

#include <hip/hip_runtime.h>

#include "device_math.hpp"
#include "lanes.hpp"

namespace mbs {
namespace pick {

constexpr int kThreads = 256;
constexpr int32_t kNobody = 0x7fffffff;

struct Params {
    int64_t batch, vocab;
    const void *logits;
    const float *noise;
    const float *temperatures, *top_ps, *min_ps;    // (batch) or null: the one for all
    const int32_t *top_ks;
    float temperature, top_p, min_p;
    int32_t top_k;
    int32_t *token;
    float *prob;                                    // (batch) or null
};

// A sequence's settings.
struct Filter {
    float inv_temp, top_p, min_p;
    int64_t top_k;                                  // vocab: no limit
    bool ok, greedy;
    __device__ __forceinline__ Filter(const Params &p, int64_t b) {
        const float t = p.temperatures ? p.temperatures[b] : p.temperature;
        top_p = p.top_ps ? p.top_ps[b] : p.top_p;
        min_p = p.min_ps ? p.min_ps[b] : p.min_p;
        const int64_t k = p.top_ks ? p.top_ks[b] : p.top_k;
        greedy = t == 0.0f;
        inv_temp = greedy ? 1.0f : 1.0f / t;
        top_k = greedy ? 1 : k <= 0 || k > p.vocab ? p.vocab : k;
        ok = t >= 0.0f && t < __builtin_inff() && inv_temp < __builtin_inff() && top_p == top_p && min_p <= 1.0f;
    }
};

// Logits as integers of the same order; both zeros are one value.
__device__ __forceinline__ uint32_t order_of(float l) {
    const uint32_t u = __float_as_uint(l + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

__device__ __forceinline__ double wave_sum64(double v) {
    for (int m = 1; m < 64; m *= 2) v += __shfl_xor(v, m);
    return v;
}

template <int DT> struct Block {
    const Params &p;
    double *red;
    int64_t row;
    float max, inv_temp;
    __device__ __forceinline__ float logit(int64_t y) const { return Act<DT>::ld(p.logits, row + y); }
    __device__ __forceinline__ double weight(float l) const { return exp(((double)l - (double)max) * (double)inv_temp); }
    __device__ double all(double v) const {
        v = wave_sum64(v);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
        __syncthreads();
        return (red[0] + red[1]) + (red[2] + red[3]);
    }
    template <class F> __device__ double sum(F f) const {
        double s = 0.0;
        for (int64_t y = threadIdx.x; y < p.vocab; y += kThreads) s += f(y);
        return all(s);
    }
};

template <int DT>
__global__ __launch_bounds__(kThreads) void sample_any(Params p) {
    __shared__ double red[kThreads / 64];
    __shared__ float scores[kThreads / 64];
    __shared__ int32_t who[kThreads / 64];
    const int64_t b = blockIdx.x, V = p.vocab;
    const Filter f(p, b);
    Block<DT> k{p, red, b * V, 0.0f, f.inv_temp};
    float m = -__builtin_inff();
    bool bad = !f.ok;
    for (int64_t y = threadIdx.x; y < V; y += kThreads) {
        const float l = k.logit(y);
        m = __builtin_fmaxf(m, l);
        bad |= !(l < __builtin_inff());
    }
    m = wave_max(m);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) scores[threadIdx.x >> 6] = m;
    __syncthreads();
    k.max = m = __builtin_fmaxf(__builtin_fmaxf(scores[0], scores[1]), __builtin_fmaxf(scores[2], scores[3]));
    if (k.all(bad ? 1.0 : 0.0) > 0.0 || m == -__builtin_inff()) {
        if (threadIdx.x == 0) {
            p.token[b] = -1;
            if (p.prob) p.prob[b] = 0.0f;
        }
        return;
    }
    // the last logit kept, and how many of its equals
    uint32_t last = 0;
    double ties = (double)V;
    if (f.top_k < V) {
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t c = last | 1u << bit;
            if (k.sum([&](int64_t y) { return order_of(k.logit(y)) >= c ? 1.0 : 0.0; }) >= (double)f.top_k) last = c;
        }
        ties = (double)f.top_k - k.sum([&](int64_t y) { return order_of(k.logit(y)) > last ? 1.0 : 0.0; });
    }
    if (f.top_p < 1.0f) {
        const uint32_t last_k = last;
        const double e_k = f.top_k < V ? k.weight(logit_of(last_k)) * ties : 0.0;
        auto from = [&](uint32_t c) {               // what the kept at or above c sum to
            const bool strict = f.top_k < V && c <= last_k;
            const double s = k.sum([&](int64_t y) {
                const uint32_t o = order_of(k.logit(y));
                return (strict ? o > last_k : o >= c) ? k.weight(k.logit(y)) : 0.0;
            });
            return strict ? s + e_k : s;
        };
        const double want = fmax((double)f.top_p * from(0), 4.9e-324);
        uint32_t at = 0;
        for (int bit = 31; bit >= 0; --bit)
            if (from(at | 1u << bit) >= want) at |= 1u << bit;
        const double above = at == 0xffffffffu ? 0.0 : from(at + 1);
        const double more = ceil((want - above) / k.weight(logit_of(at)));
        ties = at == last_k && f.top_k < V ? fmin(ties, more) : more;
        last = at;
    }
    // the index of the last equal that is kept
    int64_t upto = V - 1;
    if (k.sum([&](int64_t y) { return order_of(k.logit(y)) == last ? 1.0 : 0.0; }) > ties) {
        upto = 0;
        for (int bit = 30; bit >= 0; --bit) {       // the first index up to which there are `ties` of them
            const int64_t c = upto + (int64_t(1) << bit);
            if (k.sum([&](int64_t y) { return order_of(k.logit(y)) == last && y < c ? 1.0 : 0.0; }) < ties) upto = c;
        }
    }
    auto kept = [&](int64_t y) {
        const uint32_t o = order_of(k.logit(y));
        const double e = k.weight(k.logit(y));
        return (o > last || (o == last && y <= upto)) && e >= (double)f.min_p ? e : 0.0;
    };
    const double total = k.sum(kept);
    float best = 0.0f;
    int32_t at = kNobody;
    for (int64_t y = threadIdx.x; y < V; y += kThreads) {
        const float e = (float)kept(y), s = f.greedy ? e : e / p.noise[b * V + y];
        if (e > 0.0f && s > best) {
            best = s;
            at = (int32_t)y;
        }
    }
    const float w = wave_max(best);
    at = wave_min(best == w ? at : kNobody);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        scores[threadIdx.x >> 6] = w;
        who[threadIdx.x >> 6] = at;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        float s = 0.0f;
        at = kNobody;
        for (int i = 0; i < kThreads / 64; ++i)
            if (who[i] != kNobody && (scores[i] > s || (scores[i] == s && who[i] < at))) {
                s = scores[i];
                at = who[i];
            }
        p.token[b] = at == kNobody ? -1 : at;
        if (p.prob) p.prob[b] = at == kNobody ? 0.0f : (float)(kept(at) / total);
    }
}

}  // namespace pick
}  // namespace mbs
