// embedding.hpp -- the embedding lookup with scaling, and its gradient.
//
//   y[i]  = scale * W[token_i]                (a negative token is padding: a row of zeros;
//                                              a token >= vocab is a mistake: a row of NaN)
//   dW[v] = scale * sum over i, token_i = v, of dy[i]
//
// Tokens are bytes, int32 or int64.  Sums are fp32, rounded once to dW's type.
//
// The gradient sorts the positions by token (a stable counting sort, 8 bits a pass: one pass for
// bytes) and cuts the sorted list into chunks of 64.  A wave adds up the rows of a chunk for a tile
// of columns, each row read once, and writes a token's sum where all of its rows lie in the chunk;
// the sums of a token that goes on into other chunks are joined afterwards in the order of the
// chunks.  No atomic adds floats: a result depends on the tokens and dy alone.
#pragma once

#include <hip/hip_runtime.h>

#include "device_math.hpp"
#include "lanes.hpp"

namespace mbs {
namespace embed {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 256;         // digits of one pass of the sort
constexpr int kChunk = 64;         // sorted positions per wave: one per lane
constexpr int kJoinWaves = 8;
constexpr int kNone = -1;

struct FwdParams {
    int64_t ntokens, vocab, dim;
    const void *tokens, *weight;
    void *out;
    float scale;
    int32_t rows;                  // per workgroup
};

struct Pair { uint32_t key, pos; };

struct BwdParams {
    int64_t ntokens, vocab, dim;
    const void *tokens, *dy;
    void *dweight;
    float scale;
    int32_t tile;                  // tokens per workgroup of the sort
    int32_t tiles;                 // workgroups of the sort, at most kBins
    int32_t shift;                 // bits below this pass's digit
    uint32_t *counts;              // (tiles, kBins)
    uint32_t *valid;               // tokens within the vocabulary
    const Pair *from;              // the pass's input after the first pass
    Pair *to;                      // the pass's output; the sorted list
    float *head, *tail;            // (chunks, dim): sums of the token that a chunk begins / ends with, where it
                                   // came from the chunk before / goes on into the next
};

// Tokens by mb_token_type.
template <int TOK> __device__ __forceinline__ int64_t token_at(const void *p, int64_t i) {
    if constexpr (TOK == 0) return static_cast<const uint8_t *>(p)[i];
    else if constexpr (TOK == 1) return static_cast<const int32_t *>(p)[i];
    else return static_cast<const int64_t *>(p)[i];
}

// Elements per lane: 16 bytes of the narrower type.
template <int A, int B> constexpr int kSpan = A == 0 && B == 0 ? 4 : 8;

// A workgroup takes p.rows rows, as spans side by side.
template <int TOK, int W, int OUT>
__global__ __launch_bounds__(kThreads) void embed_fwd(FwdParams p) {
    constexpr int S = kSpan<W, OUT>, PER = 4;
    const int64_t row0 = (int64_t)blockIdx.x * p.rows;
    const uint32_t spans = (uint32_t)((p.dim + S - 1) / S);
    const uint32_t items = (uint32_t)min((int64_t)p.rows, p.ntokens - row0) * spans;
    for (uint32_t i0 = threadIdx.x; i0 < items; i0 += PER * kThreads) {
        int64_t row[PER], t[PER];
        uint32_t col[PER];
        Span<W, S> s[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const uint32_t i = min(i0 + k * kThreads, items - 1);       // past the end: the last one again, not stored
            const uint32_t r = i / spans;
            row[k] = row0 + r;
            col[k] = (i - r * spans) * S;
            t[k] = token_at<TOK>(p.tokens, row[k]);
        }
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int64_t at = (t[k] >= 0 && t[k] < p.vocab ? t[k] : 0) * p.dim + col[k];
            if (p.vocab == 0) s[k].load_first(p.weight, 0, 0);
            else if (col[k] + S <= p.dim) s[k].load(p.weight, at);
            else s[k].load_first(p.weight, at, (int)(p.dim - col[k]));
        }
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            if (i0 + k * kThreads >= items) break;
            float v[S];
#pragma unroll
            for (int j = 0; j < S; ++j) v[j] = t[k] < 0 ? 0.0f : t[k] < p.vocab ? p.scale * s[k].get(j) : __builtin_nanf("");
            if (col[k] + S <= p.dim) store_span<OUT, S>(p.out, row[k] * p.dim + col[k], v);
            else store_first<OUT, S>(p.out, row[k] * p.dim + col[k], v, (int)(p.dim - col[k]));
        }
    }
}

// The key at place i of a pass's input, kNone for a token outside the vocabulary.
template <int TOK, bool FIRST> __device__ __forceinline__ int64_t key_at(const BwdParams &p, int64_t i) {
    if constexpr (FIRST) {
        const int64_t t = token_at<TOK>(p.tokens, i);
        return t >= 0 && t < p.vocab ? t : kNone;
    } else {
        return p.from[i].key;
    }
}

// Digits of the workgroup's places, counted; with the first pass the table is zeroed on the side (workgroups past the
// sort's do nothing else).
template <int TOK, int OUT, bool FIRST>
__global__ __launch_bounds__(kThreads) void count_digits(BwdParams p) {
    __shared__ uint32_t count[kBins];
    const int64_t n = FIRST ? p.ntokens : (int64_t)*p.valid;
    if ((int)blockIdx.x < p.tiles) {
        count[threadIdx.x] = 0;
        __syncthreads();
        const int64_t from = (int64_t)blockIdx.x * p.tile, to = min(from + p.tile, n);
        for (int64_t i = from + threadIdx.x; i < to; i += kThreads) {
            const int64_t key = key_at<TOK, FIRST>(p, i);
            if (key != kNone) atomicAdd(&count[(key >> p.shift) & (kBins - 1)], 1u);
        }
        __syncthreads();
        p.counts[blockIdx.x * kBins + threadIdx.x] = count[threadIdx.x];
    }
    if constexpr (FIRST) {
        constexpr int S = OUT == 1 ? 8 : 4;
        const int64_t elems = p.vocab * p.dim, step = (int64_t)gridDim.x * kThreads * S;
        const float zeros[S] = {};
        for (int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * S; i < elems; i += step) {
            if (i + S <= elems) store_span<OUT, S>(p.dweight, i, zeros);
            else store_first<OUT, S>(p.dweight, i, zeros, (int)(elems - i));
        }
    }
}

// Each place's key and position to the place that its digit gives it.  Every workgroup adds up the counts for itself:
// the digits below (over all workgroups), then the workgroups and the waves before, then the places before.
template <int TOK, bool FIRST>
__global__ __launch_bounds__(kThreads) void scatter(BwdParams p) {
    __shared__ uint32_t at[kWaves][kBins], scan[kBins];
    const int d = threadIdx.x, wave = d >> 6, lane = d & 63;
    const int64_t n = FIRST ? p.ntokens : (int64_t)*p.valid;
    uint32_t total = 0, before = 0;
#pragma unroll 8
    for (int g = 0; g < p.tiles; ++g) {
        const uint32_t c = p.counts[g * kBins + d];
        total += c;
        before += g < (int)blockIdx.x ? c : 0u;
    }
    scan[d] = total;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) at[w][d] = 0;
    __syncthreads();
#pragma unroll
    for (int off = 1; off < kBins; off *= 2) {
        const uint32_t v = d >= off ? scan[d - off] : 0u;
        __syncthreads();
        scan[d] += v;
        __syncthreads();
    }
    if (FIRST && blockIdx.x == 0 && d == kBins - 1) *p.valid = scan[d];
    before += scan[d] - total;
    // the wave's own places: a quarter of the workgroup's, in order
    const int64_t part = p.tile / kWaves, from = (int64_t)blockIdx.x * p.tile + wave * part, to = min(from + part, n);
    for (int64_t i = from + lane; i < to; i += 64) {
        const int64_t key = key_at<TOK, FIRST>(p, i);
        if (key != kNone) atomicAdd(&at[wave][(key >> p.shift) & (kBins - 1)], 1u);
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const uint32_t c = at[w][d];
        at[w][d] = before;
        before += c;
    }
    __syncthreads();
    for (int64_t i0 = from; i0 < to; i0 += 64) {
        const int64_t i = i0 + lane;
        const int64_t key = i < to ? key_at<TOK, FIRST>(p, i) : kNone;
        const uint32_t digit = (uint32_t)(key >> p.shift) & (kBins - 1);
        // the lanes of the same digit
        uint64_t same = __ballot(key != kNone);
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            const uint64_t set = __ballot((digit >> b) & 1);
            same &= (digit >> b) & 1 ? set : ~set;
        }
        if (key != kNone) {
            const int first = __ffsll((unsigned long long)same) - 1;
            uint32_t base = 0;
            if (lane == first) base = atomicAdd(&at[wave][digit], (uint32_t)__popcll(same));
            base = __shfl(base, first, 64);
            const uint32_t dest = base + __popcll(same & ((1ull << lane) - 1));
            p.to[dest] = Pair{(uint32_t)key, FIRST ? (uint32_t)i : p.from[i].pos};
        }
    }
}

template <int DY, int OUT> constexpr int kRowSpan = DY == 1 ? 8 : 4;

// Sums of one chunk's rows for one tile of columns.
template <int DY, int OUT>
__global__ __launch_bounds__(kThreads) void sum_chunks(BwdParams p, uint32_t col_tiles) {
    constexpr int S = kRowSpan<DY, OUT>, AHEAD = 8;
    const int64_t item = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
    const int64_t chunk = item / col_tiles, n = *p.valid, from = chunk * kChunk;
    if (from >= n) return;
    const int lane = threadIdx.x & 63;
    const int64_t col = (item - chunk * col_tiles) * (64 * S) + lane * S;
    const int cols = (int)max((int64_t)0, min((int64_t)S, p.dim - col));
    const int m = (int)min((int64_t)kChunk, n - from);
    const Pair mine = p.to[from + min(lane, m - 1)];
    const int64_t before = from > 0 ? (int64_t)p.to[from - 1].key : kNone;
    const int64_t after = from + m < n ? (int64_t)p.to[from + m].key : kNone;

    float acc[S] = {};
    uint32_t key = __builtin_amdgcn_readlane(mine.key, 0);
    bool first_run = true;
    auto store = [&](float *part) {
        if (cols == S) store_span<0, S>(part, chunk * p.dim + col, acc);
        else store_first<0, S>(part, chunk * p.dim + col, acc, cols);
    };
    auto flush = [&](bool goes_on) {
        if (first_run && before == (int64_t)key) {
            store(p.head);
        } else if (goes_on) {
            store(p.tail);
        } else {
            float v[S];
#pragma unroll
            for (int j = 0; j < S; ++j) v[j] = p.scale * acc[j];
            if (cols == S) store_span<OUT, S>(p.dweight, (int64_t)key * p.dim + col, v);
            else store_first<OUT, S>(p.dweight, (int64_t)key * p.dim + col, v, cols);
        }
    };
    for (int i0 = 0; i0 < m; i0 += AHEAD) {
        Span<DY, S> row[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int64_t at = (int64_t)(uint32_t)__builtin_amdgcn_readlane(mine.pos, min(i0 + k, m - 1)) * p.dim + col;
            if (cols == S) row[k].template load<true>(p.dy, at);
            else row[k].load_first(p.dy, at, cols);
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (i0 + k >= m) break;
            const uint32_t next = __builtin_amdgcn_readlane(mine.key, i0 + k);
            if (next != key) {
                flush(false);
                key = next;
                first_run = false;
#pragma unroll
                for (int j = 0; j < S; ++j) acc[j] = 0.0f;
            }
#pragma unroll
            for (int j = 0; j < S; ++j) acc[j] += row[k].get(j);
        }
    }
    flush(after == (int64_t)key);
}

// The tokens whose rows lie in more than one chunk: the chunk in which one begins joins its sums.
template <int OUT>
__global__ __launch_bounds__(64 * kJoinWaves) void join_chunks(BwdParams p, uint32_t col_tiles) {
    constexpr int S = 4;
    __shared__ f32x4 sums[kJoinWaves][64];
    const int64_t chunk = blockIdx.x / col_tiles, n = *p.valid, from = chunk * kChunk, next = from + kChunk;
    if (next >= n) return;                              // no chunk follows
    const uint32_t key = p.to[next - 1].key;
    if (p.to[next].key != key) return;                  // nothing goes on
    if (p.to[from].key == key && from > 0 && p.to[from - 1].key == key) return;      // it began before
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // the chunks after this one that begin with the token
    int64_t parts = 0;
    for (;;) {
        const int64_t at = next + (parts + lane) * kChunk;
        const uint64_t same = __ballot(at < n && p.to[min(at, n - 1)].key == key);
        const int run = ~same == 0 ? 64 : __ffsll((unsigned long long)~same) - 1;
        parts += run;
        if (run < 64) break;
    }
    const int64_t col = (blockIdx.x % col_tiles) * (64 * S) + lane * S;
    const int cols = (int)max((int64_t)0, min((int64_t)S, p.dim - col));
    // sum 0 is the tail of this chunk, the others the heads of the next; each wave takes a run of them
    const int64_t all = parts + 1, lo = all * wave / kJoinWaves, hi = all * (wave + 1) / kJoinWaves;
    f32x4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 8
    for (int64_t k = lo; k < hi; ++k) {
        const float *part = (k == 0 ? p.tail + chunk * p.dim : p.head + (chunk + k) * p.dim) + col;
        Span<0, S> s;
        if (cols == S) s.load(part, 0);
        else s.load_first(part, 0, cols);
        acc += s.v[0];
    }
    sums[wave][lane] = acc;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < kJoinWaves; ++w) acc += sums[w][lane];
    const float v[S] = {p.scale * acc[0], p.scale * acc[1], p.scale * acc[2], p.scale * acc[3]};
    if (cols == S) store_span<OUT, S>(p.dweight, (int64_t)key * p.dim + col, v);
    else store_first<OUT, S>(p.dweight, (int64_t)key * p.dim + col, v, cols);
}

}  // namespace embed
}  // namespace mbs
