// lanes.hpp -- spans of consecutive elements per lane, lane shifts and sums over a wave.
#pragma once

#include <hip/hip_runtime.h>

#include <type_traits>

#include "device_math.hpp"

namespace mbs {

// 16-byte and smaller vectors at any element's address: the hardware takes them.
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef u32x2 u32x2_any __attribute__((aligned(2)));
typedef f32x4 f32x4_any __attribute__((aligned(4)));

// ONCE: what is read or written once and is larger than the caches (their streaming policy).
template <bool ONCE> __device__ __forceinline__ u32x4 fetch(const u32x4_any *p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(p);
    else return *p;
}
template <bool ONCE> __device__ __forceinline__ void put(u32x4_any *p, u32x4 r) {
    if constexpr (ONCE) __builtin_nontemporal_store(r, p);
    else *p = r;
}
template <bool ONCE> __device__ __forceinline__ u32x2 fetch(const u32x2_any *p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(p);
    else return *p;
}
template <bool ONCE> __device__ __forceinline__ void put(u32x2_any *p, u32x2 r) {
    if constexpr (ONCE) __builtin_nontemporal_store(r, p);
    else *p = r;
}
template <bool ONCE> __device__ __forceinline__ f32x4 fetch(const f32x4_any *p) {
    if constexpr (ONCE) return __builtin_nontemporal_load(p);
    else return *p;
}
template <bool ONCE> __device__ __forceinline__ void put(f32x4_any *p, f32x4 r) {
    if constexpr (ONCE) __builtin_nontemporal_store(r, p);
    else *p = r;
}

// S consecutive elements as loaded; nothing is unpacked, so nothing is waited for, until get().
template <int DT, int S> struct Span;
template <> struct Span<1, 8> {
    u32x4 v;
    template <bool ONCE = false> __device__ __forceinline__ void load(const void *p, int64_t at) {
        v = fetch<ONCE>(reinterpret_cast<const u32x4_any *>(static_cast<const uint16_t *>(p) + at));
    }
    __device__ __forceinline__ void load_first(const void *p, int64_t at, int n) {   // the rest: zeros
        const uint16_t *e = static_cast<const uint16_t *>(p) + at;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            v[i] = (2 * i < n ? (uint32_t)e[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)e[2 * i + 1] << 16 : 0u);
    }
    __device__ __forceinline__ float get(int i) const { return i & 1 ? bf16_hi(v[i >> 1]) : bf16_lo(v[i >> 1]); }
};
template <> struct Span<1, 4> {
    u32x2 v;
    template <bool ONCE = false> __device__ __forceinline__ void load(const void *p, int64_t at) {
        v = fetch<ONCE>(reinterpret_cast<const u32x2_any *>(static_cast<const uint16_t *>(p) + at));
    }
    __device__ __forceinline__ void load_first(const void *p, int64_t at, int n) {
        const uint16_t *e = static_cast<const uint16_t *>(p) + at;
#pragma unroll
        for (int i = 0; i < 2; ++i)
            v[i] = (2 * i < n ? (uint32_t)e[2 * i] : 0u) | (2 * i + 1 < n ? (uint32_t)e[2 * i + 1] << 16 : 0u);
    }
    __device__ __forceinline__ float get(int i) const { return i & 1 ? bf16_hi(v[i >> 1]) : bf16_lo(v[i >> 1]); }
};
template <int S> struct SpanF32 {
    f32x4 v[S / 4];
    template <bool ONCE = false> __device__ __forceinline__ void load(const void *p, int64_t at) {
#pragma unroll
        for (int i = 0; i < S / 4; ++i)
            v[i] = fetch<ONCE>(reinterpret_cast<const f32x4_any *>(static_cast<const float *>(p) + at) + i);
    }
    __device__ __forceinline__ void load_first(const void *p, int64_t at, int n) {
#pragma unroll
        for (int i = 0; i < S; ++i) v[i / 4][i % 4] = i < n ? static_cast<const float *>(p)[at + i] : 0.0f;
    }
    __device__ __forceinline__ float get(int i) const { return v[i / 4][i % 4]; }
};

template <> struct Span<0, 4> : SpanF32<4> {};
template <> struct Span<0, 8> : SpanF32<8> {};

// One element: for rows shorter than a span.
template <int DT> struct Span<DT, 1> {
    float v;
    template <bool ONCE = false> __device__ __forceinline__ void load(const void *p, int64_t at) { v = Act<DT>::ld(p, at); }
    __device__ __forceinline__ float get(int) const { return v; }
};

template <int DT, int S, bool ONCE = false> __device__ __forceinline__ void store_span(void *p, int64_t at, const float (&v)[S]) {
    if constexpr (S == 1) {
        st_out<DT>(p, at, v[0]);
    } else if constexpr (DT == 0) {
#pragma unroll
        for (int i = 0; i < S / 4; ++i)
            put<ONCE>(reinterpret_cast<f32x4_any *>(static_cast<float *>(p) + at) + i,
                      f32x4{v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]});
    } else if constexpr (S == 8) {
        u32x4 r;
#pragma unroll
        for (int i = 0; i < 4; ++i) r[i] = bf16x2_pack(v[2 * i], v[2 * i + 1]);
        put<ONCE>(reinterpret_cast<u32x4_any *>(static_cast<uint16_t *>(p) + at), r);
    } else {
        u32x2 r;
#pragma unroll
        for (int i = 0; i < 2; ++i) r[i] = bf16x2_pack(v[2 * i], v[2 * i + 1]);
        put<ONCE>(reinterpret_cast<u32x2_any *>(static_cast<uint16_t *>(p) + at), r);
    }
}
template <int DT, int S> __device__ __forceinline__ void store_first(void *p, int64_t at, const float (&v)[S], int n) {
#pragma unroll
    for (int i = 0; i < S; ++i)
        if (i < n) st_out<DT>(p, at + i, v[i]);
}

// Everything asked of memory has arrived (vmcnt 0).  Loads and stores share that counter and a wait is for the oldest of
// both, so a wave that waited row by row would wait for each sum that it stored in between as well.
__device__ __forceinline__ void wait_for_memory() { __builtin_amdgcn_s_waitcnt(0x0f70); }

// Each lane's neighbour's value; the wave's first (last) lane takes `edge`.
__device__ __forceinline__ float from_lane_before(float v, float edge) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(edge), __float_as_int(v), 0x138, 0xf, 0xf, false));
}
__device__ __forceinline__ float from_lane_after(float v, float edge) {
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(edge), __float_as_int(v), 0x130, 0xf, 0xf, false));
}
__device__ __forceinline__ float lane_value(float v, int lane) {
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane));
}

// f over the 64 lanes' values (of 32 bits), the same in every lane: pairs, quads and rows of 16 by lane permutations,
// then the rows'.
template <class T, class F> __device__ __forceinline__ T wave_all(T v, F f) {
    auto moved = [&](auto ctrl) {
        return __builtin_bit_cast(T, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    v = f(v, moved(std::integral_constant<int, 0xB1>{}));    // lanes 1 0 3 2
    v = f(v, moved(std::integral_constant<int, 0x4E>{}));    // lanes 2 3 0 1
    v = f(v, moved(std::integral_constant<int, 0x141>{}));   // half rows mirrored
    v = f(v, moved(std::integral_constant<int, 0x140>{}));   // rows mirrored
    auto row = [&](int lane) { return __builtin_bit_cast(T, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), lane)); };
    return f(f(row(0), row(16)), f(row(32), row(48)));
}
__device__ __forceinline__ float wave_sum(float v) { return wave_all(v, [](float a, float b) { return a + b; }); }
__device__ __forceinline__ float wave_max(float v) { return wave_all(v, [](float a, float b) { return __builtin_fmaxf(a, b); }); }
__device__ __forceinline__ int32_t wave_min(int32_t v) { return wave_all(v, [](int32_t a, int32_t b) { return min(a, b); }); }

}  // namespace mbs
