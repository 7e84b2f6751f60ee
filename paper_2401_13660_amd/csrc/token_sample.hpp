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
// tokens are ranked one by one.  A bin of more than 256 of them (logits far apart from the rest, equals by the hundred) is
// counted once more into bins of its own, of ranks.  Weights are summed as integers of 2^-44: sums do not depend
// on the order of the atomics, and a border does not move from call to call.  2^20 tokens' weights could pass 64 bits of those: rows
// that long are summed once before, in 64-bit floats, and their unit is between 2^-63 and 2^-62 of that sum.
//
// One workgroup per sequence, the row in registers from one load to the token drawn (up to 8,192 tokens; beyond, it is read
// again from the cache); the kept tokens go to a list, and random numbers are only read for those.  The race divides, as verify_sample's does:
// times the hardware's reciprocal, (16, 131,072) without a filter took 52 us, but a noise below 2^-126 counted as 0.  Bound by latency and, for large vocabularies, by one CU's
// instructions: about 25 per token for the weight and its bin, 10 for the quotient.  Replayed from a graph, without a filter, with top-k, top-p and both:
// (32, 256) in fp32 3.8, 6.5, 6.4 and 8.4 us; (16, 32,000) in bf16 18, 23, 30 and 32; (16, 131,072) 57, 63, 129 and 91.  With a
// row's pieces among several workgroups, three launches, (16, 32,000) with top-p took 36.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "device_math.hpp"
#include "lanes.hpp"

namespace mbs {
namespace pick {

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
        ok = t >= 0.0f && t < __builtin_inff() && 2.0f * inv_temp < __builtin_inff() && top_p == top_p && min_p <= 1.0f;
    }
};

// Logits as integers of the same order; both zeros are one value.
__device__ __forceinline__ uint32_t order_of(float l) {
    const uint32_t u = __float_as_uint(l + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ uint64_t rank_of(float l, uint32_t y) { return (uint64_t)order_of(l) << 32 | (uint32_t)~y; }

// Tokens from which on a row's unit goes by its sum, and 2^-bits, the unit of all shorter rows.
constexpr int64_t kLongRow = int64_t(1) << 20;
constexpr int kBits = 44;

// e in [0, 1] in units of 2^-bits, cut: what is below one counts as nothing.
__device__ __forceinline__ uint64_t units_of(float e, int bits) {
    const uint32_t u = __float_as_uint(e), down = 127 - (u >> 23);
    return ((uint64_t)((u & 0x7fffffu) | 0x800000u) << (bits - 23)) >> min(down, 63u);
}
__device__ __forceinline__ uint64_t units_of(double e, int bits) {
    const double v = e * (double)(1ull << bits);
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
// What is computed of v is computed again from here on: a row's weights, bins and ranks, kept from one reading of it to the
// next, would not fit the registers.
template <class V> __device__ __forceinline__ void opaque(V &v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ void opaque(f32x4 (&v)[1]) { asm volatile("" : "+v"(v[0])); }

// T threads, S spans of 4 tokens each in registers (0: the row is read again each time).  W: up to 1,024 tokens weights are exponentials in
// 64 bits: a token next to a border is a thousandth of a short row's sum, and an error in 32 bits would move it oftener.
template <int DT, int T, int S, class W> struct Row {
    using Weight = W;
    const void *logits;
    int64_t at;
    uint32_t vocab;
    float max, inv_temp;
    // From T = 1 on differences of half logits are taken, as those of whole ones could overflow and yet weigh something.
    float scale, top;                               // 1 or 1/2, and the largest logit times it
    float per, per_rest, least;                     // log2 e / (T scale) and what it lacks, and the least difference told from others
    Span<DT, 4> s[S > 0 ? S : 1];

    __device__ __forceinline__ void set_temperature(float inv) {
        inv_temp = inv;
        scale = inv <= 1.0f ? 0.5f : 1.0f;
        const double exact = 1.4426950408889634 * (double)inv / (double)scale;
        per = (float)exact;                         // finite, as 2 / T is
        per_rest = (float)(exact - (double)per);
        least = -200.0f / per;
    }

    __device__ __forceinline__ void set_max(float m) {
        max = m;
        top = m * scale;
    }

    __device__ __forceinline__ static uint32_t first_of(uint32_t k) { return (k * T + threadIdx.x) * 4; }
    __device__ __forceinline__ void load_span(Span<DT, 4> &to, uint32_t y) const {
        if (y + 4 <= vocab) {
            to.load(logits, at + y);
            return;
        }
        // masked past the row's end
        const int n = y < vocab ? (int)(vocab - y) : 0;
        to.load_first(logits, at + y, n);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (DT == 0) to.v[0][i] = i < n ? to.v[0][i] : -__builtin_inff();
            else to.v[i / 2] |= i < n ? 0u : 0xff80u << 16 * (i % 2);
        }
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
                if (S > 1) opaque(s[k].v);
                f(first_of(k), s[k]);
                // span after span: the work of many side by side would not fit the registers
                if (S > 2 && k % 2 == 1) __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            constexpr int kAhead = 2;
#pragma unroll 1
            for (uint32_t k = 0; first_of(k) < vocab; k += kAhead) {
                Span<DT, 4> some[kAhead];
#pragma unroll
                for (int i = 0; i < kAhead; ++i) load_span(some[i], first_of(k + i));
#pragma unroll
                for (int i = 0; i < kAhead; ++i) f(first_of(k + i), some[i]);
            }
        }
    }
    // f(the first span's number, N spans), for all
    template <int N, class F> __device__ __forceinline__ void groups(F f) {
        if constexpr (S > 0) {
#pragma unroll
            for (int k = 0; k < S; k += N) {
                Span<DT, 4> some[N];
#pragma unroll
                for (int i = 0; i < N; ++i) {
                    if (S > 1) opaque(s[k + i].v);
                    some[i] = s[k + i];
                }
                f(k, some);
                if (S > 2) __builtin_amdgcn_sched_barrier(0);
            }
        } else {
            for (uint32_t k = 0; first_of(k) < vocab; k += N) {
                Span<DT, 4> some[N];
#pragma unroll
                for (int i = 0; i < N; ++i) load_span(some[i], first_of(k + i));
                f(k, some);
            }
        }
    }
    // f(token, logit) for every token that -infinity does not mask
    template <class F> __device__ __forceinline__ void each(F f) {
        spans([&](uint32_t y, const Span<DT, 4> &v) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float l = v.get(i);
                if (l > -__builtin_inff()) f(y + i, l);
            }
        });
    }
    __device__ __forceinline__ Weight weight(float l) const {
        if constexpr (std::is_same_v<Weight, double>) {
            return exp(((double)l - (double)max) * (double)inv_temp);
        } else {
            // 2^(d log2 e / T), with what the product's rounding left over as a factor; below 2^-200 all is alike
            const float d = __builtin_fmaxf(__builtin_fmaf(l, scale, -top), least), t = d * per;
            const float left = __builtin_fmaf(d, per_rest, __builtin_fmaf(d, per, -t)), e = hw_exp2(t);
            return __builtin_fmaf(e, left * kLn2, e);
        }
    }
};

// Bins of equal width from a row's largest logit to its least; halves, so that no difference overflows.
template <int N> struct Bins {
    float half_top, per;
    __device__ __forceinline__ Bins(float top, float low)
        : half_top(0.5f * top), per(__builtin_fminf((float)(N - 1) / (0.5f * top - 0.5f * low), 3.0e38f)) {}
    __device__ __forceinline__ uint32_t of(float l) const { return (uint32_t)min((int)((half_top - 0.5f * l) * per), N - 1); }
};

// The largest logit, the least one that is not -infinity; a row that is no distribution: infinity.
template <class R> __device__ __forceinline__ float2 wave_tops(R &row, bool ok) {
    float top = -__builtin_inff(), low = __builtin_inff();
    bool bad = !ok;
    row.spans([&](uint32_t, const auto &v) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float l = v.get(i);
            top = __builtin_fmaxf(top, l);
            low = __builtin_fminf(low, l > -__builtin_inff() ? l : low);
            bad |= !(l < __builtin_inff());
        }
    });
    top = wave_max(top);
    low = -wave_max(-low);
    return make_float2(__builtin_amdgcn_ballot_w64(bad) ? __builtin_inff() : top, low);
}

template <int T> struct Shared {
    static constexpr int kBins = 4 * T, kWaves = T / 64, kKept = 4 * T;
    static constexpr int kList = T == 64 ? 64 : 256;    // tokens of a bin that are ranked one by one
    union {
        struct {
            uint64_t weight[kBins];
            uint32_t count[kBins];
        };
        struct {
            uint32_t kept_at[kKept];
            float kept_logit[kKept];
        };
    };
    uint64_t list[kList], list_weight[kList], higher[kList];
    uint32_t places[kList], kept;
    uint64_t wave_weight[kWaves], low, high, border, border_sum, found_weight;
    uint32_t wave_count[kWaves], listed, found_bin, found_count;
    uint64_t sums[kWaves];
    double weights[kWaves];
    float tops[kWaves], lows[kWaves], scores[kWaves];
    int32_t who[kWaves];
    uint32_t bad;
};

// LONG: rows of kLongRow tokens and more.
template <int DT, int T, int S, bool LONG = false>
__global__ __launch_bounds__(T) void sample_rows(Params p) {
    using Sh = Shared<T>;
    constexpr int kBins = Sh::kBins, kWaves = Sh::kWaves, kList = Sh::kList;
    __shared__ Sh sh;
    const int64_t b = blockIdx.x;
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const Filter f(p, b);
    using R = Row<DT, T, S, std::conditional_t<T <= 256, double, float>>;
    R row;
    row.logits = p.logits;
    row.at = b * p.vocab;
    row.vocab = (uint32_t)p.vocab;
    row.set_temperature(f.inv_temp);
    row.load();

    auto clear = [&] {
#pragma unroll
        for (int i = 0; i < kBins / T; ++i) {
            sh.weight[i * T + t] = 0;
            sh.count[i * T + t] = 0;
        }
    };
    float2 ends = wave_tops(row, f.ok);
    if (lane == 0) {
        sh.tops[wave] = ends.x;
        sh.lows[wave] = ends.y;
    }
    if (t == 0) sh.kept = 0;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        ends.x = __builtin_fmaxf(ends.x, sh.tops[w]);
        ends.y = __builtin_fminf(ends.y, sh.lows[w]);
    }
    const float top = ends.x;
    row.set_max(top);
    if (!(top < __builtin_inff()) || top == -__builtin_inff()) {            // the same in every thread
        if (t == 0) {
            p.token[b] = -1;
            if (p.prob) p.prob[b] = 0.0f;
        }
        return;
    }

    int bits = kBits;
    if constexpr (LONG) {
        // so many that the sum, 2^x at least and less than 2^(x + 1), is below 2^63; x is 0 to 30
        double all = 0.0;
        row.each([&](uint32_t, float l) { all += (double)row.weight(l); });
#pragma unroll
        for (int m = 1; m < 64; m *= 2) all += __shfl_xor(all, m);
        if (lane == 0) sh.weights[wave] = all;
        __syncthreads();
        all = 0.0;
        for (int w = 0; w < kWaves; ++w) all += sh.weights[w];
        bits = 62 - ilogb(all);
    }

    uint64_t border = 0;                            // the least rank kept; 0: all are
    const bool by_count = f.top_k < row.vocab, by_weight = f.top_p < 1.0f;
    if (by_count || by_weight) {
        const Bins<kBins> bins(top, ends.y);
        // What the filter at hand narrows the row down to: tokens of one bin of logits, then (fine) of bins of ranks.
        bool fine = false;
        uint32_t bin = 0, shift = 0;
        uint64_t low_rank = 0, high_rank = 0;
        auto inside = [&](uint32_t y, float l) {
            if (!fine) return bins.of(l) == bin;
            const uint64_t rank = rank_of(l, y);
            return rank >= low_rank && rank <= high_rank && (high_rank - rank) >> shift == bin;
        };
        uint64_t sum = 0;                           // of the weights that top-k leaves
        bool counted = false;                       // the row's bins are there
        // top-k first (weighs = 0: so many tokens are wanted), then top-p (1: so much of their weight)
#pragma unroll 1
        for (int weighs = by_count ? 0 : 1; weighs < (by_weight ? 2 : 1); ++weighs) {
            uint64_t wanted = f.top_k, above = 0;
            fine = false;
#pragma unroll 1
            for (bool whole = true;; whole = false) {
                // tokens and weights of each bin: of the whole row, or of a bin's ranks
                if (!whole || !counted) {
                    clear();
                    __syncthreads();
                    row.each([&](uint32_t y, float l) {
                        uint32_t to;
                        if (whole) {
                            to = bins.of(l);
                        } else {
                            const uint64_t rank = rank_of(l, y);
                            if (rank < low_rank || rank > high_rank) return;
                            to = (uint32_t)((high_rank - rank) >> shift);
                        }
                        if (by_count) atomicAdd(&sh.count[to], 1u);
                        if (by_weight) atomicAdd(reinterpret_cast<unsigned long long *>(&sh.weight[to]), (unsigned long long)units_of(row.weight(l), bits));
                    });
                    counted = whole;
                }
                __syncthreads();
                // running sums over the bins: a thread's own, its wave's, the waves'
                constexpr int kOwn = kBins / T;
                uint32_t c = 0;
                uint64_t w = 0;
#pragma unroll
                for (int i = 0; i < kOwn; ++i) {
                    c += sh.count[t * kOwn + i];
                    w += sh.weight[t * kOwn + i];
                }
                const uint32_t run_c = wave_running_sum(c);
                const uint64_t run_w = wave_running_sum(w);
                if (lane == 63) {
                    sh.wave_count[wave] = run_c;
                    sh.wave_weight[wave] = run_w;
                }
                if (t == 0) {
                    sh.found_bin = kBins;
                    sh.listed = 0;
                    sh.low = ~0ull;
                    sh.high = 0;
                    sh.border = 0;
                }
                for (int i = t; i < kList; i += T) {
                    sh.places[i] = 0;
                    sh.higher[i] = 0;
                }
                __syncthreads();
                c = run_c - c;
                w = run_w - w;
                uint64_t all = 0;
                for (int i = 0; i < kWaves; ++i) {
                    if (i < wave) {
                        c += sh.wave_count[i];
                        w += sh.wave_weight[i];
                    }
                    all += sh.wave_weight[i];
                }
                if (whole && weighs) {
                    if (!by_count || border == 0) sum = all;
                    // the first that reaches it is the last one kept; sums are whole numbers, and 1 keeps the first alone
                    const double share = ceil((double)f.top_p * (double)sum);
                    wanted = share > 1.0 ? (uint64_t)share : 1;
                }
                // the bin in which what is wanted is reached
#pragma unroll
                for (int i = 0; i < kOwn; ++i) {
                    const uint32_t n = sh.count[t * kOwn + i];
                    const uint64_t m = sh.weight[t * kOwn + i];
                    if (weighs ? w < wanted && w + m >= wanted : c < wanted && c + n >= wanted) {
                        sh.found_bin = t * kOwn + i;
                        sh.found_count = c;
                        sh.found_weight = w;
                    }
                    c += n;
                    w += m;
                }
                __syncthreads();
                bin = sh.found_bin;
                if (bin == kBins) break;            // fewer tokens than top-k wants: all
                wanted -= weighs ? sh.found_weight : sh.found_count;
                above += sh.found_weight;
                // its tokens
                uint64_t least = ~0ull, most = 0;
                row.each([&](uint32_t y, float l) {
                    if (!inside(y, l)) return;
                    const uint64_t rank = rank_of(l, y);
                    least = rank < least ? rank : least;
                    most = rank > most ? rank : most;
                    const uint32_t at = atomicAdd(&sh.listed, 1u);
                    if (at >= kList) return;
                    sh.list[at] = rank;
                    sh.list_weight[at] = by_weight ? units_of(row.weight(l), bits) : 0;
                });
                if (most) {
                    atomicMin(reinterpret_cast<unsigned long long *>(&sh.low), (unsigned long long)least);
                    atomicMax(reinterpret_cast<unsigned long long *>(&sh.high), (unsigned long long)most);
                }
                __syncthreads();
                const uint32_t n = sh.listed;
                if (n > kList) {                    // too many to rank one by one
                    low_rank = sh.low;
                    high_rank = sh.high;
                    shift = (uint32_t)max(0, 64 - __builtin_clzll((high_rank - low_rank) | 1) - (31 - __builtin_clz(kBins)));
                    fine = true;
                    continue;
                }
                // each token of the list against every kWaves-th of them, wave by wave
                for (uint32_t k = lane; k < n; k += 64) {
                    const uint64_t mine = sh.list[k];
                    uint64_t higher = 0;
                    uint32_t places = 0;
                    for (uint32_t i = wave; i < n; i += kWaves)
                        if (sh.list[i] > mine) {
                            ++places;
                            higher += sh.list_weight[i];
                        }
                    if (places) {
                        atomicAdd(&sh.places[k], places);
                        atomicAdd(reinterpret_cast<unsigned long long *>(&sh.higher[k]), (unsigned long long)higher);
                    }
                }
                __syncthreads();
                for (uint32_t k = t; k < n; k += T) {
                    const uint32_t places = sh.places[k];
                    const uint64_t higher = sh.higher[k], mine = sh.list_weight[k];
                    if (weighs ? higher < wanted && higher + mine >= wanted : places == wanted - 1) {
                        sh.border = sh.list[k];
                        sh.border_sum = above + higher + mine;
                    }
                }
                __syncthreads();
                border = sh.border > border ? sh.border : border;
                sum = sh.border_sum;
                break;
            }
        }
    }

    // the race of the kept, and what they sum to
    float best = 0.0f;
    int32_t at = kNobody;
    uint64_t sum = 0;
    // the border as a logit and the last index that is kept of it
    const uint32_t border_bits = (uint32_t)(border >> 32), border_at = ~(uint32_t)border;
    const float border_logit = border ? __uint_as_float(border_bits & 0x80000000u ? border_bits & 0x7fffffffu : ~border_bits) : -__builtin_inff();
    auto kept = [&](uint32_t y, float l) { return l > border_logit || (l == border_logit && border && y <= border_at); };
    typename R::Weight weighs = 0;                  // of this thread's best
    auto run_race = [&](uint32_t y, float l, float noise) {
        const typename R::Weight e = row.weight(l);
        if (!(e > 0 && e >= f.min_p)) return;
        sum += units_of(e, bits);
        const float s = (float)e / noise;
        if (s > best || (s == best && s > 0.0f && (int32_t)y < at)) {
            best = s;
            at = (int32_t)y;
            weighs = e;
        }
    };
    // with a border, the kept in a list where it has room for them: few threads' work instead of everyone's
    bool listed = false;
    if (border) {
        __syncthreads();
        row.each([&](uint32_t y, float l) {
            if (!kept(y, l)) return;
            const uint32_t to = atomicAdd(&sh.kept, 1u);
            if (to >= Sh::kKept) return;
            sh.kept_at[to] = y;
            sh.kept_logit[to] = l;
        });
        __syncthreads();
        listed = sh.kept <= Sh::kKept;
        for (uint32_t i = t; listed && i < sh.kept; i += T) {
            const uint32_t y = sh.kept_at[i];
            run_race(y, sh.kept_logit[i], f.greedy ? 1.0f : p.noise[row.at + y]);
        }
    }
    // kSide spans side by side, so that their random numbers are asked for together
    constexpr int kSide = S > 0 ? S : 2;
    auto race = [&](uint32_t first, const Span<DT, 4> (&v)[kSide]) {
        Span<0, 4> noise[kSide];
#pragma unroll
        for (int k = 0; k < kSide; ++k) {
            const uint32_t y = row.first_of(first + k);
            if (y + 4 <= row.vocab) noise[k].load(p.noise, row.at + y);
            else noise[k].load_first(p.noise, row.at + y, y < row.vocab ? (int)(row.vocab - y) : 0);
        }
#pragma unroll
        for (int k = 0; k < kSide; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t y = row.first_of(first + k) + i;
                if (kept(y, v[k].get(i))) run_race(y, v[k].get(i), f.greedy ? 1.0f : noise[k].get(i));
            }
    };
    if (!listed) row.template groups<kSide>(race);
    const float won = wave_max(best);
    const int32_t first = wave_min(best == won ? at : kNobody);
    sum = wave_running_sum(sum);                    // whole numbers: the list's order does not show
    __syncthreads();
    if (lane == 63) {
        sh.scores[wave] = won;
        sh.who[wave] = first;
        sh.sums[wave] = sum;
    }
    if (at == first && at != kNobody) sh.weights[wave] = (double)weighs;
    __syncthreads();
    if (t == 0) {
        sum = 0;
        int winner = -1;
        for (int w = 0; w < kWaves; ++w) {
            sum += sh.sums[w];
            if (sh.who[w] == kNobody) continue;
            if (winner < 0 || sh.scores[w] > sh.scores[winner] || (sh.scores[w] == sh.scores[winner] && sh.who[w] < sh.who[winner])) winner = w;
        }
        p.token[b] = winner < 0 ? -1 : sh.who[winner];
        if (p.prob) p.prob[b] = winner < 0 ? 0.0f : (float)(sh.weights[winner] * (double)(1ull << bits) / (double)sum);
    }
}

}  // namespace pick
}  // namespace mbs
