// grad_clip.hpp -- the global norm of a list of tensors, and the clipping by it.
//
//   norm = sqrt(sum over every element of every tensor of g^2)
//   out  = g                              where norm + eps <= max_norm
//        = g max_norm / (norm + eps)      otherwise (a NaN norm makes every element NaN)
//
// Squares and their sums are fp64: the norm of any finite fp32 gradients neither
// overflows nor vanishes on the way.  Sums are taken in a fixed order.
//
// The tensors are cut into units of kUnit elements, numbered through the list, and a grid that fills
// the chip once takes equal runs of consecutive units.  One launch sums the squares, a second one
// adds up the first one's partial sums in every workgroup (the same bits in each) and scales: two
// passes over the gradients, the least that a global norm allows, in two launches whatever the
// number of tensors.  A short list travels in the kernels' arguments; a longer one is first written
// to memory, kFill tensors per launch, again from arguments, so that no host memory has to outlive
// the call.
//
// Bound by HBM, three times the gradients' bytes (two reads, one write).  The first pass's loads are
// streaming ones but for the last kCached bytes, which the second pass, walking every run backwards,
// reads first.  972M model in fp32: 574 us (6.8 TB/s) and 1,529 us (5.1), together 2.10 ms; with
// ordinary loads and stores 699 and 1,575, with streaming loads throughout 566 and 1,568.  353M model
// in bf16: 133 and 273 us, 406 together (178 and 281; 123 and 297).  2,048 workgroups, which do not
// all run at once, took 4% longer, units of half the size 2%.  fp64 squares cost nothing that shows:
// two conversions and two multiply-adds for 4 bytes of bf16.
#pragma once

#include <hip/hip_runtime.h>

#include "device_math.hpp"
#include "lanes.hpp"

namespace mbs {
namespace clip {

constexpr int kThreads = 256;
constexpr int kUnit = 8192;        // elements
constexpr int kBlocks = 1280;      // workgroups at most, and partial sums of the norm: 5 per CU, as their registers allow
constexpr int64_t kCached = int64_t(256) << 20;    // the Infinity Cache's bytes
constexpr int kInline = 64;        // tensors of a list that travels in the kernels' arguments
constexpr int kFill = 112;         // tensors per launch that writes the list

struct Entry {
    const void *in;
    void *out;
    int64_t n;
    uint32_t first;                // the tensor's first unit
    int32_t dtype;
};
template <int N> struct Table { Entry e[N]; };

struct Params {
    const Entry *table;            // null: in the arguments
    int32_t count;
    uint32_t units;
    uint32_t cached;               // units at the end of a workgroup's run that the second pass finds in the cache
    double *part;                  // (gridDim.x)
    float *norm;
    float max_norm, eps;
};

// Units start at 16-byte boundaries: a tensor's first one holds the elements before its first boundary
// too, so an element's place in its unit is its index plus this.
__host__ __device__ inline int lead(const void *p, int32_t dtype) {
    return (int)(reinterpret_cast<uintptr_t>(p) % 16) / (dtype == 1 ? 2 : 4);
}

__global__ void fill_table(Table<kFill> t, int n, Entry *to) {
    for (int i = threadIdx.x; i < n; i += blockDim.x) to[i] = t.e[i];
}

__device__ __forceinline__ double block_sum(double v) {
    __shared__ double red[kThreads / 64];
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int i = 0; i < kThreads / 64; ++i) s += red[i];
    return s;
}

// The entry that unit u lies in.
__device__ __forceinline__ int entry_of(const Entry *table, int count, uint32_t u) {
    int before = 0;
    for (int i = 0; i < count; i += kThreads) {
        const int k = i + threadIdx.x;
        before += __syncthreads_count(k < count && table[k].first <= u);
    }
    return before - 1;
}

// One unit of an entry.  f(vector) per whole 16-byte vector of the input, then, where the unit is cut by the
// tensor's beginning or end, e(element).
template <int DT, bool ONCE, class F, class E> __device__ __forceinline__ void for_unit(const Entry &t, uint32_t unit, F f, E e) {
    constexpr int V = DT == 1 ? 8 : 4, PER = kUnit / V / kThreads;
    const int64_t start = (int64_t)unit * kUnit - lead(t.in, DT);
    if (start >= 0 && start + kUnit <= t.n) {
        Span<DT, V> s[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) s[i].template load<ONCE>(t.in, start + (i * kThreads + (int)threadIdx.x) * V);
#pragma unroll
        for (int i = 0; i < PER; ++i) f(s[i], start + (i * kThreads + (int)threadIdx.x) * V);
    } else {
        for (int i = 0; i < PER; ++i) {
            const int64_t at = start + (i * kThreads + (int)threadIdx.x) * V;
            if (at >= 0 && at + V <= t.n) {
                Span<DT, V> s;
                s.load(t.in, at);
                f(s, at);
            } else {
                for (int64_t k = max(at, (int64_t)0); k < min(at + V, t.n); ++k) e(k);
            }
        }
    }
}

__device__ __forceinline__ void my_units(uint32_t units, uint32_t &from, uint32_t &to) {
    from = (uint32_t)((uint64_t)units * blockIdx.x / gridDim.x);
    to = (uint32_t)((uint64_t)units * (blockIdx.x + 1) / gridDim.x);
}

template <int DT, bool ONCE> __device__ __forceinline__ void unit_squares(const Entry &t, uint32_t unit, double (&acc)[4]) {
    constexpr int V = DT == 1 ? 8 : 4;
    for_unit<DT, ONCE>(t, unit,
        [&](const Span<DT, V> &s, int64_t) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const double v = s.get(i);
                acc[i & 3] = __builtin_fma(v, v, acc[i & 3]);
            }
        },
        [&](int64_t k) {
            const double v = Act<DT>::ld(t.in, k);
            acc[0] = __builtin_fma(v, v, acc[0]);
        });
}

template <int DT, bool ONCE> __device__ __forceinline__ void unit_scale(const Entry &t, uint32_t unit, float factor) {
    constexpr int V = DT == 1 ? 8 : 4;
    for_unit<DT, ONCE>(t, unit,
        [&](const Span<DT, V> &s, int64_t at) {
            float v[V];
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = factor * s.get(i);
            store_span<DT, V, true>(t.out, at, v);
        },
        [&](int64_t k) { st_out<DT>(t.out, k, factor * Act<DT>::ld(t.in, k)); });
}

__device__ __forceinline__ void sum_squares_of(const Params &p, const Entry *table) {
    uint32_t from, to;
    my_units(p.units, from, to);
    double acc[4] = {};
    if (from < to) {
        int at = __builtin_amdgcn_readfirstlane(entry_of(table, p.count, from));
        Entry t = table[at];
        for (uint32_t u = from; u < to; ++u) {
            while (at + 1 < p.count && table[at + 1].first <= u) t = table[++at];
            if (to - u > p.cached) {
                if (t.dtype == 1) unit_squares<1, true>(t, u - t.first, acc);
                else unit_squares<0, true>(t, u - t.first, acc);
            } else {
                if (t.dtype == 1) unit_squares<1, false>(t, u - t.first, acc);
                else unit_squares<0, false>(t, u - t.first, acc);
            }
        }
    }
    const double s = block_sum((acc[0] + acc[1]) + (acc[2] + acc[3]));
    if (threadIdx.x == 0) p.part[blockIdx.x] = s;
}

// norm from the partial sums, the same in every workgroup.
__device__ __forceinline__ float norm_of(const Params &p, int nparts) {
    double s = 0.0;
    for (int i = threadIdx.x; i < nparts; i += kThreads) s += p.part[i];
    return (float)__builtin_sqrt(block_sum(s));
}

// From the end of the run to its beginning: what the norm's pass read last may still be in a cache.
__device__ __forceinline__ void scale_of(const Params &p, const Entry *table) {
    const float norm = norm_of(p, gridDim.x);
    if (blockIdx.x == 0 && threadIdx.x == 0) *p.norm = norm;
    const bool keep = norm + p.eps <= p.max_norm;
    const float factor = keep ? 1.0f : p.max_norm / (norm + p.eps);
    uint32_t from, to;
    my_units(p.units, from, to);
    if (from >= to) return;
    int at = __builtin_amdgcn_readfirstlane(entry_of(table, p.count, to - 1));
    Entry t = table[at];
    for (uint32_t u = to; u-- > from;) {
        while (t.first > u) t = table[--at];
        if (keep && t.in == t.out) continue;
        if (to - u > p.cached) {
            if (t.dtype == 1) unit_scale<1, true>(t, u - t.first, factor);
            else unit_scale<0, true>(t, u - t.first, factor);
        } else {
            if (t.dtype == 1) unit_scale<1, false>(t, u - t.first, factor);
            else unit_scale<0, false>(t, u - t.first, factor);
        }
    }
}

__global__ __launch_bounds__(kThreads) void sum_squares_inline(Params p, Table<kInline> t) { sum_squares_of(p, t.e); }
__global__ __launch_bounds__(kThreads) void sum_squares(Params p) { sum_squares_of(p, p.table); }
__global__ __launch_bounds__(kThreads) void scale_inline(Params p, Table<kInline> t) { scale_of(p, t.e); }
__global__ __launch_bounds__(kThreads) void scale(Params p) { scale_of(p, p.table); }

__global__ __launch_bounds__(kThreads) void finish_norm(Params p, int nparts) {
    const float norm = norm_of(p, nparts);
    if (threadIdx.x == 0) *p.norm = norm;
}

}  // namespace clip
}  // namespace mbs
