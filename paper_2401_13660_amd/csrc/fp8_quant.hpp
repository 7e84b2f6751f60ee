// fp8_quant.hpp -- matrices in 8 bits with a scale for each 128 columns of a row, or each 128 x 128 tile.
//
// Transposed, rows and columns are the output's: (channels, time) becomes (time, channels) with scales along the channels,
// as a product over the channels wants it.
//
// Bound by memory: one reading, one writing of half or a quarter of it.  (4, 3584, 8192) in bf16, turned, takes 69 us, 5.2 TB/s
// (79 with LDS lines of 33 words and every thread finding its columns' scales for itself); (7168, 1792) in fp32 by tiles 11.3 us, 5.7 TB/s.  Streaming loads or stores were no faster.  A workgroup takes a 128 x 128 piece of the input into
// registers, 8 columns per lane and span.  As it lies, 16 lanes hold a row's block and its largest value is theirs; transposed,
// the lanes of one column group join theirs in LDS, and the bytes pass through LDS, 4 rows of a column to a word, so
// that both sides of memory see whole lines.
#pragma once

#include <hip/hip_runtime.h>

#include "fp8.hpp"
#include "lanes.hpp"

namespace mbs {
namespace quant {

constexpr int kTile = fp8::kBlock;
constexpr int kThreads = 512;
constexpr int kSpans = kTile * kTile / 8 / kThreads;    // of a thread: 4 rows, 8 columns each

struct Params {
    int64_t rows, cols;             // of the input
    int32_t row_tiles, col_tiles;
    const void *x;                  // (batch, rows, cols)
    uint8_t *q;                     // as x, or (batch, cols, rows)
    float *scales;                  // (batch, rows or row tiles, column tiles); of the output's rows and columns
};

// Where word w of column c of a transposed piece lies.  A wave writes one column of each 8 and 4 words of it, and reads 8
// columns' 32 words: both are spread over all 64 banks.
__device__ __forceinline__ int place(int c, int w) { return (32 * c + ((w + 4 * (c >> 3)) & 31)) ^ (32 * (c >> 6)); }

// Thread t holds rows 4 (t / 16) to 4 (t / 16) + 3 of the piece, columns 8 (t % 16) on.
template <int X, bool TILE, bool TRANSPOSE>
__global__ __launch_bounds__(kThreads) void quantize(Params p) {
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int64_t tiles = (int64_t)p.row_tiles * p.col_tiles, b = blockIdx.x / tiles;
    const int in_batch = (int)(blockIdx.x - b * tiles), rt = in_batch / p.col_tiles, ct = in_batch - rt * p.col_tiles;
    const int64_t row0 = (int64_t)rt * kTile + 4 * (t / 16), col0 = (int64_t)ct * kTile + 8 * (t % 16);
    const int n = (int)min((int64_t)8, max((int64_t)0, p.cols - col0));
    Span<X, 8> s[kSpans];
#pragma unroll
    for (int k = 0; k < kSpans; ++k) {
        const int64_t at = (b * p.rows + row0 + k) * p.cols + col0;
        if (row0 + k < p.rows && n >= 8) s[k].load(p.x, at);
        else s[k].load_first(p.x, at, row0 + k < p.rows ? n : 0);
    }
    __shared__ float tops[kThreads / 64];
    __shared__ __align__(16) float by_col[TRANSPOSE && !TILE ? kThreads / 64 : 1][kTile];
    __shared__ __align__(16) uint32_t turned[TRANSPOSE ? kTile * kTile / 4 : 4];
    float top[kSpans];
#pragma unroll
    for (int k = 0; k < kSpans; ++k) {
        top[k] = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) top[k] = __builtin_fmaxf(top[k], __builtin_fabsf(s[k].get(i)));
    }
    float tile_scale = 0.0f;
    if constexpr (TILE) {
        const float m = wave_max(__builtin_fmaxf(__builtin_fmaxf(top[0], top[1]), __builtin_fmaxf(top[2], top[3])));
        if (lane == 0) tops[wave] = m;
        __syncthreads();
        float all = tops[0];
#pragma unroll
        for (int w = 1; w < kThreads / 64; ++w) all = __builtin_fmaxf(all, tops[w]);
        tile_scale = fp8::scale_of(all);
        if (t == 0)
            p.scales[b * tiles + (TRANSPOSE ? (int64_t)ct * p.row_tiles + rt : (int64_t)rt * p.col_tiles + ct)] = tile_scale;
    }
    if constexpr (!TRANSPOSE) {
#pragma unroll
        for (int k = 0; k < kSpans; ++k) {
            const float scale = TILE ? tile_scale : fp8::scale_of(fp8::max_of_16(top[k]));
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = s[k].get(i);
            if (row0 + k < p.rows && n > 0) {
                fp8::store8(p.q + (b * p.rows + row0 + k) * p.cols + col0, v, 1.0f / scale, n);
                if (!TILE && t % 16 == 0) p.scales[(b * p.rows + row0 + k) * p.col_tiles + ct] = scale;
            }
        }
    } else {
        float inv[8];
        if constexpr (TILE) {
#pragma unroll
            for (int i = 0; i < 8; ++i) inv[i] = 1.0f / tile_scale;
        } else {
            // a wave holds 16 rows: the 4 lanes of a column group, then the waves
            float m[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                m[i] = __builtin_fmaxf(__builtin_fmaxf(__builtin_fabsf(s[0].get(i)), __builtin_fabsf(s[1].get(i))),
                                       __builtin_fmaxf(__builtin_fabsf(s[2].get(i)), __builtin_fabsf(s[3].get(i))));
                m[i] = __builtin_fmaxf(m[i], __shfl_xor(m[i], 16));
                m[i] = __builtin_fmaxf(m[i], __shfl_xor(m[i], 32));
                if (lane < 16) by_col[wave][8 * lane + i] = m[i];
            }
            __syncthreads();
            if (t < kTile) {
                float all = by_col[0][t];
#pragma unroll
                for (int w = 1; w < kThreads / 64; ++w) all = __builtin_fmaxf(all, by_col[w][t]);
                const float scale = fp8::scale_of(all);
                by_col[0][t] = 1.0f / scale;            // column t is this thread's alone until the barrier
                const int64_t col = (int64_t)ct * kTile + t;
                if (col < p.cols) p.scales[(b * p.cols + col) * p.row_tiles + rt] = scale;
            }
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; ++i) inv[i] = by_col[0][8 * (t % 16) + i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            turned[place(8 * (t % 16) + i, t / 16)] =
                fp8::pack4(s[0].get(i) * inv[i], s[1].get(i) * inv[i], s[2].get(i) * inv[i], s[3].get(i) * inv[i]);
        __syncthreads();
        // 8 threads to a column's 128 bytes, 16 each
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const int c = k * 64 + t / 8, w = 4 * (t % 8);
            const int64_t col = (int64_t)ct * kTile + c, row = (int64_t)rt * kTile + 4 * w;
            if (col >= p.cols || row >= p.rows) continue;
            const u32x4 r = *reinterpret_cast<const u32x4 *>(&turned[place(c, w)]);
            uint8_t *to = p.q + (b * p.cols + col) * p.rows + row;
            if (row + 16 <= p.rows) {
                *reinterpret_cast<fp8::u32x4_byte *>(to) = r;
            } else {
                for (int i = 0; i < (int)(p.rows - row); ++i) to[i] = (uint8_t)(r[i / 4] >> (8 * (i % 4)));
            }
        }
    }
}

}  // namespace quant
}  // namespace mbs
