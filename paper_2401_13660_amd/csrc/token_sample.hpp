// token_sample.hpp -- the next token by temperature, top-k, top-p and min-p, from given random numbers.
//
// In the order of falling logits, the lowest index first among equals, with e = exp((l - largest) / T):
//
//   top-k keeps the first k;   S = what they sum to
//   top-p keeps those before which less than p S lies (and the first);   min-p those of e >= min_p
//   token = the y of the largest e(y) / noise(y) of the kept, the lowest such y;   prob = e(token) / the kept sum
//
// The order is that of 64-bit ranks (the logit's bits in an order of integers, then the index from the last), and all that a
// filter does is to find the lowest rank that it keeps.  Nothing is sorted: tokens are counted into bins of falling logits with what
// they weigh, the bin in which the wanted count or weight is reached is found by a running sum over the bins, and its few
// tokens are ranked one by one.  A bin of more than kList of them (logits far apart from the rest, equals by the hundred) is
// counted once more into bins of its own, of ranks.  Weights are summed as integers of 2^-44: sums do not depend
// on the order of the atomics, and a border does not move from call to call.
//
// One workgroup per sequence, the row in registers from one load to the token drawn (up to 65,536 tokens; beyond, it is read
// again from the cache); random numbers are only read where a token is kept.  Bound by latency and, for large
// vocabularies, by one CU's instructions: about 30 per token for the weight and its bin.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "device_math.hpp"
#include "lanes.hpp"

namespace mbs {
namespace pick {

constexpr int32_t kNobody = 0x7fffffff;
constexpr int kList = 64;                           // tokens of a bin that are ranked one by one

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
    uint32_t top_k;                                 // vocab: no limit
    bool ok, greedy;
    __device__ __forceinline__ Filter(const Params &p, int64_t b) {
        const float t = p.temperatures ? p.temperatures[b] : p.temperature;
        top_p = p.top_ps ? p.top_ps[b] : p.top_p;
        min_p = p.min_ps ? p.min_ps[b] : p.min_p;
        const int64_t k = p.top_ks ? p.top_ks[b] : p.top_k;
        greedy = t == 0.0f;
        inv_temp = greedy ? 1.0f : 1.0f / t;
        top_k = greedy ? 1 : (uint32_t)(k <= 0 || k > p.vocab ? p.vocab : k);
        ok = t >= 0.0f && t < __builtin_inff() && inv_temp < __builtin_inff() && top_p == top_p && min_p <= 1.0f;
    }
};

// Logits as integers of the same order; both zeros are one value.
__device__ __forceinline__ uint32_t order_of(float l) {
    const uint32_t u = __float_as_uint(l + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t rank_of(float l, uint32_t y) { return (uint64_t)order_of(l) << 32 | (uint32_t)~y; }

// e in [0, 1] in units of 2^-44; what is below half of one counts as nothing.
__device__ __forceinline__ uint64_t units_of(float e) {
    const uint32_t u = __float_as_uint(e), down = 127 - (u >> 23);
    return ((uint64_t)((u & 0x7fffffu) | 0x800000u) << 21) >> min(down, 63u);
}
__device__ __forceinline__ uint64_t units_of(double e) {
    const double v = e * 17592186044416.0;          // 2^44
    const uint32_t high = (uint32_t)(v * (1.0 / 4294967296.0));
    return (uint64_t)high << 32 | (uint32_t)__builtin_fma((double)high, -4294967296.0, v);
}

// The sum over this lane and those before it.
template <class T> __device__ __forceinline__ T wave_running_sum(T v) {
    auto step = [&](auto ctrl, auto rows) {
        constexpr int C = decltype(ctrl)::value, R = decltype(rows)::value;
        if constexpr (sizeof(T) == 4) {
            v += (T)__builtin_amdgcn_update_dpp(0, (int)v, C, R, 0xf, false);
        } else {
            const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, C, R, 0xf, false);
            const uint32_t hi = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), C, R, 0xf, false);
            v += (T)hi << 32 | lo;
        }
    };
    using std::integral_constant;
    step(integral_constant<int, 0x111>{}, integral_constant<int, 0xf>{});   // rows of 16: 1, 2, 4 and 8 lanes on
    step(integral_constant<int, 0x112>{}, integral_constant<int, 0xf>{});
    step(integral_constant<int, 0x114>{}, integral_constant<int, 0xf>{});
    step(integral_constant<int, 0x118>{}, integral_constant<int, 0xf>{});
    step(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});   // rows 0 and 2 into 1 and 3
    step(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});   // both into the upper two
    return v;
}
__device__ __forceinline__ uint64_t last_lane(uint64_t v) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), 63) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, 63);
}

// What is computed of v is computed again from here on: a row's weights, bins and ranks, kept from one reading of it to the
// next, would not fit the registers.
template <class V> __device__ __forceinline__ void opaque(V &v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ void opaque(f32x4 (&v)[1]) { asm volatile("" : "+v"(v[0])); }

// T threads, S spans of 4 tokens each in registers (0: the row is read again each time).  Up to 1,024 tokens weights are exponentials in 64
// bits: a token next to a border is a thousandth of a short row's sum, and an error in 32 bits would move it oftener.
template <int DT, int T, int S> struct Row {
    using Weight = std::conditional_t<T == 256, double, float>;
    const void *logits;
    int64_t at;
    uint32_t vocab;
    float max, inv_temp;
    Span<DT, 4> s[S > 0 ? S : 1];

    __device__ __forceinline__ static uint32_t first_of(uint32_t k) { return (k * T + threadIdx.x) * 4; }
    __device__ __forceinline__ void load_span(Span<DT, 4> &to, uint32_t y) const {
        if (y + 4 <= vocab) to.load(logits, at + y);
        else to.load_first(logits, at + y, y < vocab ? (int)(vocab - y) : 0);
    }
    __device__ __forceinline__ void load() {
        if constexpr (S > 0) {
#pragma unroll
            for (int k = 0; k < S; ++k) load_span(s[k], first_of(k));
        }
    }
    // f(span k's first token, its logits), for all spans
    template <class F> __device__ __forceinline__ void spans(F f) {
        if constexpr (S > 0) {
#pragma unroll
            for (int k = 0; k < S; ++k) {
                opaque(s[k].v);
                f(first_of(k), s[k]);
                // span after span: the work of many side by side would not fit the registers
                if (S > 2 && k % 2 == 1) __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            for (uint32_t k = 0; first_of(k) < vocab; ++k) {
                load_span(s[0], first_of(k));
                f(first_of(k), s[0]);
            }
        }
    }
    // f(token, logit) for every token that -infinity does not mask
    template <class F> __device__ __forceinline__ void each(F f) {
        spans([&](uint32_t y, const Span<DT, 4> &v) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float l = v.get(i);
                if (y + i < vocab && l > -__builtin_inff()) f(y + i, l);
            }
        });
    }
    __device__ __forceinline__ Weight weight(float l) const {
        if constexpr (std::is_same_v<Weight, double>) {
            return exp(((double)l - (double)max) * (double)inv_temp);
        } else {
            // 2^(x log2 e), with what the product's rounding left over as a factor
            const float x = (l - max) * inv_temp, t = x * kLog2e;
            const float left = __builtin_fmaf(x, kLog2e, -t) + x * 1.925963033500547e-08f;      // log2 e - kLog2e
            const float e = hw_exp2(t);
            return x > -__builtin_inff() ? __builtin_fmaf(e, left * kLn2, e) : 0.0f;
        }
    }
};

template <int T> struct Shared {
    static constexpr int kBins = 4 * T, kWaves = T / 64;
    uint64_t weight[kBins];
    uint32_t count[kBins];
    uint64_t list[kList], list_weight[kList];
    uint64_t wave_weight[kWaves], low, high, border, border_sum, found_weight;
    uint32_t wave_count[kWaves], listed, found_bin, found_count, found_n;
    float tops[kWaves], lows[kWaves], scores[kWaves];
    int32_t who[kWaves];
    uint32_t bad;
};

template <int DT, int T, int S>
__global__ __launch_bounds__(T) void sample_rows(Params p) {
    using Sh = Shared<T>;
    constexpr int kBins = Sh::kBins, kWaves = Sh::kWaves;
    __shared__ Sh sh;
    const int64_t b = blockIdx.x;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const Filter f(p, b);
    Row<DT, T, S> row;
    row.logits = p.logits;
    row.at = b * p.vocab;
    row.vocab = (uint32_t)p.vocab;
    row.inv_temp = f.inv_temp;
    row.load();

    // the largest logit, the least one that is not -infinity, and whether the row is a distribution
    float top = -__builtin_inff(), low = __builtin_inff();
    bool bad = !f.ok;
    row.spans([&](uint32_t y, const Span<DT, 4> &v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float l = v.get(i);
            const bool in = y + i < row.vocab;
            top = __builtin_fmaxf(top, in ? l : top);
            low = __builtin_fminf(low, in && l > -__builtin_inff() ? l : low);
            bad |= in && !(l < __builtin_inff());
        }
    });
    auto clear = [&] {
#pragma unroll
        for (int i = 0; i < kBins / T; ++i) {
            sh.weight[i * T + t] = 0;
            sh.count[i * T + t] = 0;
        }
    };
    top = wave_max(top);
    low = -wave_max(-low);
    bad = __builtin_amdgcn_ballot_w64(bad) != 0;
    if (lane == 0) {
        sh.tops[wave] = bad ? __builtin_inff() : top;
        sh.lows[wave] = low;
    }
    clear();
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        top = __builtin_fmaxf(top, sh.tops[w]);
        low = __builtin_fminf(low, sh.lows[w]);
    }
    row.max = top;
    if (!(top < __builtin_inff()) || top == -__builtin_inff()) {            // the same in every thread
        if (t == 0) {
            p.token[b] = -1;
            if (p.prob) p.prob[b] = 0.0f;
        }
        return;
    }

    uint64_t border = 0;                            // the least rank kept
    const bool by_count = f.top_k < row.vocab, by_weight = f.top_p < 1.0f;
    if (by_count || by_weight) {
        // bins of equal width from the largest logit to the least; halves, so that no difference overflows
        const float half_top = 0.5f * top, width = half_top - 0.5f * low;
        const float per = __builtin_fminf((float)(kBins - 1) / width, 3.0e38f);
        auto bin_of = [&](float l) { return (uint32_t)min((int)((half_top - 0.5f * l) * per), kBins - 1); };
        auto count_all = [&] {
            row.each([&](uint32_t, float l) {
                const uint32_t at = bin_of(l);
                atomicAdd(&sh.count[at], 1u);
                if (by_weight) atomicAdd(reinterpret_cast<unsigned long long *>(&sh.weight[at]), (unsigned long long)units_of(row.weight(l)));
            });
        };
        // what lies before this thread's bins, and in all
        uint32_t before_count = 0;
        uint64_t before_weight = 0, all_weight = 0;
        auto run = [&] {
            uint32_t c = 0;
            uint64_t w = 0;
#pragma unroll
            for (int i = 0; i < kBins / T; ++i) {
                c += sh.count[t * (kBins / T) + i];
                w += sh.weight[t * (kBins / T) + i];
            }
            const uint32_t rc = wave_running_sum(c);
            const uint64_t rw = wave_running_sum(w);
            if (lane == 63) {
                sh.wave_count[wave] = rc;
                sh.wave_weight[wave] = rw;
            }
            __syncthreads();
            before_count = rc - c;
            before_weight = rw - w;
            all_weight = 0;
#pragma unroll
            for (int i = 0; i < kWaves; ++i) {
                if (i < wave) {
                    before_count += sh.wave_count[i];
                    before_weight += sh.wave_weight[i];
                }
                all_weight += sh.wave_weight[i];
            }
        };
        // the bin in which `wanted` tokens, or that much of their weight, are reached
        auto find = [&](bool weighs, uint64_t wanted) {
            uint32_t c = before_count;
            uint64_t w = before_weight;
#pragma unroll
            for (int i = 0; i < kBins / T; ++i) {
                const uint32_t at = t * (kBins / T) + i, n = sh.count[at];
                const uint64_t m = sh.weight[at];
                if (weighs ? w < wanted && w + m >= wanted : c < wanted && c + n >= wanted) {
                    sh.found_bin = at;
                    sh.found_n = n;
                    sh.found_count = c;
                    sh.found_weight = w;
                }
                c += n;
                w += m;
            }
            if (t == 0) {
                sh.listed = 0;
                sh.low = ~0ull;
                sh.high = 0;
                sh.border = 0;
            }
            __syncthreads();
        };
        // The least rank of those that reach `wanted`; what the ranks down to it weigh is left in border_sum.
        bool counted_anew = false;
        auto settle = [&](bool weighs, uint64_t wanted) {
            if (t == 0) sh.found_n = 0;
            __syncthreads();
            find(weighs, wanted);
            uint64_t low_rank = 0, high_rank = 0, above = 0;
            uint32_t bin = sh.found_bin, n = sh.found_n, shift = 0;
            if (n == 0) return (uint64_t)0;         // fewer tokens than top-k wants: all
            bool fine = false;
            wanted -= weighs ? sh.found_weight : sh.found_count;
            above += sh.found_weight;
            auto inside = [&](float l, uint64_t rank) {
                return fine ? rank >= low_rank && rank <= high_rank && (high_rank - rank) >> shift == bin : bin_of(l) == bin;
            };
            while (n > kList) {
                uint64_t least = ~0ull, most = 0;
                row.each([&](uint32_t y, float l) {
                    const uint64_t rank = rank_of(l, y);
                    if (inside(l, rank)) {
                        least = rank < least ? rank : least;
                        most = rank > most ? rank : most;
                    }
                });
                if (most) {
                    atomicMin(reinterpret_cast<unsigned long long *>(&sh.low), (unsigned long long)least);
                    atomicMax(reinterpret_cast<unsigned long long *>(&sh.high), (unsigned long long)most);
                }
                clear();
                __syncthreads();
                low_rank = sh.low;
                high_rank = sh.high;
                shift = (uint32_t)max(0, 64 - __builtin_clzll((high_rank - low_rank) | 1) - (31 - __builtin_clz(kBins)));
                fine = counted_anew = true;
                row.each([&](uint32_t y, float l) {
                    const uint64_t rank = rank_of(l, y);
                    if (rank < low_rank || rank > high_rank) return;
                    const uint32_t to = (uint32_t)((high_rank - rank) >> shift);
                    atomicAdd(&sh.count[to], 1u);
                    if (by_weight) atomicAdd(reinterpret_cast<unsigned long long *>(&sh.weight[to]), (unsigned long long)units_of(row.weight(l)));
                });
                __syncthreads();
                run();
                find(weighs, wanted);
                bin = sh.found_bin;
                n = sh.found_n;
                wanted -= weighs ? sh.found_weight : sh.found_count;
                above += sh.found_weight;
            }
            row.each([&](uint32_t y, float l) {
                const uint64_t rank = rank_of(l, y);
                if (!inside(l, rank)) return;
                const uint32_t at = atomicAdd(&sh.listed, 1u);
                sh.list[at] = rank;
                sh.list_weight[at] = by_weight ? units_of(row.weight(l)) : 0;
            });
            __syncthreads();
            if (wave == 0) {
                const uint64_t mine = lane < n ? sh.list[lane] : 0, weighs_mine = lane < n ? sh.list_weight[lane] : 0;
                uint64_t higher = 0;
                uint32_t places = 0;
                for (uint32_t i = 0; i < n; ++i) {
                    const uint64_t other = sh.list[i];
                    if (other > mine) {
                        ++places;
                        higher += sh.list_weight[i];
                    }
                }
                if (lane < n && (weighs ? higher < wanted && higher + weighs_mine >= wanted : places == wanted - 1)) {
                    sh.border = mine;
                    sh.border_sum = above + higher + weighs_mine;
                }
            }
            __syncthreads();
            return sh.border;
        };
        count_all();
        __syncthreads();
        run();
        uint64_t sum = all_weight;
        if (by_count) {
            border = settle(false, f.top_k);
            if (border) sum = sh.border_sum;
        }
        if (by_weight) {
            if (counted_anew) {
                clear();
                __syncthreads();
                count_all();
                __syncthreads();
                run();
            }
            // the first that reaches it is the last one kept; sums are whole numbers, and 1 keeps the first alone
            const double wanted = ceil((double)f.top_p * (double)sum);
            const uint64_t lowest = settle(true, wanted > 1.0 ? (uint64_t)wanted : 1);
            border = lowest > border ? lowest : border;
        }
    }

    // the race of the kept, and what they sum to
    float best = 0.0f;
    int32_t at = kNobody;
    uint64_t sum = 0;
    auto kept = [&](uint32_t y, float l, typename Row<DT, T, S>::Weight &e) {
        if (y >= row.vocab || !(l > -__builtin_inff()) || rank_of(l, y) < border) return false;
        e = row.weight(l);
        return e > 0 && e >= f.min_p;
    };
    row.spans([&](uint32_t y, const Span<DT, 4> &v) {
        typename Row<DT, T, S>::Weight e[4];
        bool in[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) in[i] = kept(y + i, v.get(i), e[i]);
        if (!(in[0] || in[1] || in[2] || in[3])) return;
        float noise[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) noise[i] = in[i] && !f.greedy ? p.noise[row.at + y + i] : 1.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (!in[i]) continue;
            sum += units_of(e[i]);
            const float s = (float)e[i] / noise[i];
            if (s > best) {
                best = s;
                at = (int32_t)(y + i);
            }
        }
    });
    const float won = wave_max(best);
    at = wave_min(best == won && at != kNobody ? at : kNobody);
    best = won;
    sum = last_lane(wave_running_sum(sum));
    __syncthreads();
    if (lane == 0) {
        sh.scores[wave] = won;
        sh.who[wave] = at;
        sh.wave_weight[wave] = sum;
    }
    __syncthreads();
    if (t == 0) {
        for (int w = 1; w < kWaves; ++w) {
            sum += sh.wave_weight[w];
            if (sh.who[w] != kNobody && (at == kNobody || sh.scores[w] > best || (sh.scores[w] == best && sh.who[w] < at))) {
                best = sh.scores[w];
                at = sh.who[w];
            }
        }
        p.token[b] = at == kNobody ? -1 : at;
        if (p.prob) p.prob[b] = at == kNobody ? 0.0f : (float)((double)row.weight(Act<DT>::ld(p.logits, row.at + at)) * 17592186044416.0 / (double)sum);
    }
}

}  // namespace pick
}  // namespace mbs
