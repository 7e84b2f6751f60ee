// fp8.hpp -- 8-bit floats (e4m3, largest 448, no infinities) with a scale for each block of 128 values.
//
// A block's scale is its largest magnitude over 448, and no less than the smallest normal float, so that a block of zeros
// has a finite inverse; values are multiplied by that inverse and rounded to nearest even (v_cvt_pk_fp8_f32).  A NaN stays
// one and leaves its block's others alone; an infinity makes its block's scale infinite and, with it, all of its values NaN.
#pragma once

#include <hip/hip_runtime.h>

#include "device_math.hpp"
#include "lanes.hpp"

namespace mbs {
namespace fp8 {

constexpr int kBlock = 128;
constexpr float kMost = 448.0f;
constexpr float kLeastScale = 1.17549435e-38f;      // 2^-126

// 8-bit rows may start at any byte.
typedef u32x2 u32x2_byte __attribute__((aligned(1)));
typedef u32x4 u32x4_byte __attribute__((aligned(1)));

__device__ __forceinline__ float scale_of(float amax) { return __builtin_fmaxf(amax / kMost, kLeastScale); }

__device__ __forceinline__ uint32_t pack4(float a, float b, float c, float d) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}

// The largest of 16 neighbouring lanes' values, in each of them.
__device__ __forceinline__ float max_of_16(float v) {
    auto moved = [&](auto ctrl) {
        return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), decltype(ctrl)::value, 0xf, 0xf, true));
    };
    v = __builtin_fmaxf(v, moved(std::integral_constant<int, 0xB1>{}));
    v = __builtin_fmaxf(v, moved(std::integral_constant<int, 0x4E>{}));
    v = __builtin_fmaxf(v, moved(std::integral_constant<int, 0x141>{}));
    return __builtin_fmaxf(v, moved(std::integral_constant<int, 0x140>{}));
}

// 8 values times `inv`, in 8 bits; the first n of them where a row ends within the span.
__device__ __forceinline__ void store8(uint8_t *q, const float (&v)[8], float inv, int n) {
    const u32x2 r = {pack4(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv), pack4(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv)};
    if (n >= 8) {
        *reinterpret_cast<u32x2_byte *>(q) = r;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) q[i] = (uint8_t)(r[i >> 2] >> (8 * (i & 3)));
    }
}

}  // namespace fp8
}  // namespace mbs
