// abi_checks.hpp -- argument checks and launching, shared by the C ABI's entry points.
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "mbscan.h"

namespace mbs {
namespace abi {

// Every element count the entry points form stays below 2^56, so that byte
// counts (at most 4 bytes per element, times the position count's factor
// already inside the count) and the address ranges of the alias checks stay far
// from overflow.  No device memory comes near it.
constexpr int64_t kMaxElems = int64_t(1) << 56;

inline bool valid_dtype(int32_t t) { return t == MB_F32 || t == MB_BF16; }
inline size_t dtype_size(int32_t t) { return t == MB_BF16 ? 2 : 4; }

inline bool aligned(const void *p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

// Does [a, a+na) overlap [b, b+nb)?  Null or empty ranges never overlap.
inline bool overlaps(const void *a, size_t na, const void *b, size_t nb) {
    if (!a || !b || na == 0 || nb == 0) return false;
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return x < y + nb && y < x + na;
}

// a * b without overflow past kMaxElems (both non-negative).
inline bool mul_ok(int64_t a, int64_t b, int64_t *out) {
    if (a != 0 && b > kMaxElems / a) return false;
    *out = a * b;
    return true;
}

inline hipError_t launch(const void *fn, dim3 grid, dim3 block, void *params, void *stream) {
    void *args[] = {params};
    return hipLaunchKernel(fn, grid, block, args, 0, static_cast<hipStream_t>(stream));
}

}  // namespace abi
}  // namespace mbs
