// embedding.hpp -- the embedding lookup with scaling, and its gradient.
//
//   y[i]  = scale * W[token_i]                (a negative token is padding: a row of zeros;
//                                              a token >= vocab is a mistake: a row of NaN)
//   dW[v] = scale * sum over i, token_i = v, of dy[i]
//
// Tokens are bytes, int32 or int64.  Sums are fp32, rounded once to dW's type.
//
// Few tokens (sum_direct): a workgroup per row or per token looks for the row's tokens.  Otherwise the
// gradient sorts the positions by token (a stable counting sort, 8 bits a pass: one pass for bytes) and
// cuts the sorted list into chunks of 64.  A wave adds up the rows of a chunk for a tile of columns, each
// row read once, and writes a token's sum where all of its rows lie in the chunk; the sums of a token that
// goes on into other chunks are joined afterwards in the order of the chunks.  No atomic adds floats: a
// result depends on the tokens and dy alone.
//
// 32,768 bytes of a text, width 1792 in bf16: 34 us a call.  Kernel by kernel (a trace, where launches do not
// overlap, so that the parts come to 1.5 to 3 us more than a call): sums 22.9 (5.1 TB/s, the rate of a device
// copy), the sort 3.5 and 5.6, the joining 4.2, a chain of loads each.  16,384 tokens of a table of 32,000
// rows of 768 fp32: 41 us a call; in the trace the sort 5.6, 9.9 and 10.2 (a share of the table's 98 MB zeroed
// beside each), sums 13.8, joining 4.6.  With a launch of its own for each pass's counts the sort took four,
// 45 us a call; with the next pass's counts added in memory token by token instead of in LDS 49: equal
// tokens meet in one counter.
#pragma once

#include <hip/hip_runtime.h>

#include "device_math.hpp"
#include "lanes.hpp"

namespace mbs {
namespace embed {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / 64;
constexpr int kBins = 256;         // digits of one pass of the sort
constexpr int kWideBits = 10;      // of the one pass for tables a little larger
constexpr int kWideTiles = 64;     // workgroups of it at most
constexpr int kChunk = 64;         // sorted positions per wave at most: one per lane
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
    int32_t tiles;                 // workgroups of the sort, at most kBins (1: sort_small)
    int32_t chunk;                 // sorted positions per wave
    int64_t zero_from, zero_to;    // elements of dweight that the launch sets to zero on the side
    int32_t passes;                // 8 bits each
    int32_t shift;                 // bits below this pass's digit
    uint32_t *counts;              // (tiles, digits)
    uint32_t *next_counts;         // the next pass's, counted by this one, or null
    int32_t ahead;                 // passes after the first whose counts the first launch sets to zero
    uint32_t *valid;               // tokens within the vocabulary
    const Pair *from;              // the pass's input after the first pass
    Pair *to;                      // the pass's output; the sorted list
    float *head, *tail;            // (groups, dim): sums of the token that a group of chunks begins / ends with,
                                   // where it came from the group before / goes on into the next
};

// Tokens by mb_token_type.
template <int TOK> __device__ __forceinline__ int64_t token_at(const void *p, int64_t i) {
    if constexpr (TOK == 0) return static_cast<const uint8_t *>(p)[i];
    else if constexpr (TOK == 1) return static_cast<const int32_t *>(p)[i];
    else return static_cast<const int64_t *>(p)[i];
}

// Where the span of S columns that begins at `col` is read and written: a row's last span is moved back to end with the
// row, so that none is cut (what two spans share they both hold the same of).  Rows shorter than a span take spans of one.
template <int S> __device__ __forceinline__ int64_t span_at(int64_t col, int64_t dim) { return min(col, dim - S); }

// A workgroup takes p.rows rows at a time, as spans side by side.  Bound by the writes: 32,768 rows of 1,792 bf16 take
// 20.5 us, 5.8 TB/s with what the Infinity Cache takes of them; 32 rows 3 us, the chain of a token, its row and a store.
template <int TOK, int W, int OUT, int S>
__global__ __launch_bounds__(kThreads) void embed_fwd(FwdParams p) {
    constexpr int PER = 4;
    const uint32_t spans = (uint32_t)((p.dim + S - 1) / S);
    for (int64_t row0 = (int64_t)blockIdx.x * p.rows; row0 < p.ntokens; row0 += (int64_t)gridDim.x * p.rows) {
        const uint32_t items = (uint32_t)min((int64_t)p.rows, p.ntokens - row0) * spans;
        for (uint32_t i0 = threadIdx.x; i0 < items; i0 += PER * kThreads) {
            int64_t row[PER], t[PER], col[PER];
            Span<W, S> s[PER];
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const uint32_t i = min(i0 + k * kThreads, items - 1);   // past the end: the last one again, not stored
                const uint32_t r = i / spans;
                row[k] = row0 + r;
                col[k] = span_at<S>((int64_t)(i - r * spans) * S, p.dim);
                t[k] = token_at<TOK>(p.tokens, row[k]);
            }
#pragma unroll
            for (int k = 0; k < PER; ++k)
                s[k].load(p.weight, (t[k] >= 0 && t[k] < p.vocab ? t[k] : 0) * p.dim + col[k]);
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                if (i0 + k * kThreads >= items) break;
                float v[S];
#pragma unroll
                for (int j = 0; j < S; ++j)
                    v[j] = t[k] < 0 ? 0.0f : t[k] < p.vocab ? p.scale * s[k].get(j) : __builtin_nanf("");
                store_span<OUT, S>(p.out, row[k] * p.dim + col[k], v);
            }
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

// The places of a wave in a step of the sort: kPlaces per lane, 64 side by side, in order.
constexpr int kPlaces = 4;
constexpr int kStep = kThreads * kPlaces;

template <int TOK, bool FIRST> struct Keys {
    int64_t at[kPlaces];
    __device__ __forceinline__ void load(const BwdParams &p, int64_t from, int64_t n) {
        from += (threadIdx.x >> 6) * (64 * kPlaces) + (threadIdx.x & 63);
#pragma unroll
        for (int k = 0; k < kPlaces; ++k) at[k] = from + 64 * k < n ? key_at<TOK, FIRST>(p, from + 64 * k) : kNone;
    }
};

// A share of the table set to zero, by the workgroups of a launch past the sort's: the sort's few workgroups leave the
// chip to it.
template <int OUT> __device__ __forceinline__ void zero_share(const BwdParams &p) {
    constexpr int S = OUT == 1 ? 8 : 4;
    const int64_t step = (int64_t)(gridDim.x - p.tiles) * blockDim.x * S;
    const float zeros[S] = {};
    for (int64_t i = p.zero_from + ((int64_t)(blockIdx.x - p.tiles) * blockDim.x + threadIdx.x) * S; i < p.zero_to; i += step) {
        if (i + S <= p.zero_to) store_span<OUT, S>(p.dweight, i, zeros);
        else store_first<OUT, S>(p.dweight, i, zeros, (int)(p.zero_to - i));
    }
}

// The lanes whose digit is this lane's, of those that have one.
template <int BITS = 8> __device__ __forceinline__ uint64_t same_digit(uint32_t digit, bool has) {
    uint64_t same = __ballot(has);
#pragma unroll
    for (int b = 0; b < BITS; ++b) {
        const uint64_t set = __ballot((digit >> b) & 1);
        same &= (digit >> b) & 1 ? set : ~set;
    }
    return same;
}

// Digits of the workgroup's places, counted.
template <int TOK, int OUT, bool FIRST, int BITS>
__global__ __launch_bounds__(kThreads) void count_digits(BwdParams p) {
    constexpr int BINS = 1 << BITS;
    if ((int)blockIdx.x >= p.tiles) return zero_share<OUT>(p);
    __shared__ uint32_t count[BINS];
    const int64_t n = FIRST ? p.ntokens : (int64_t)*p.valid;
    const int64_t from = (int64_t)blockIdx.x * p.tile, to = min(from + p.tile, n);
#pragma unroll
    for (int d = threadIdx.x; d < BINS; d += kThreads) count[d] = 0;
    for (int k = 0; FIRST && k < p.ahead; ++k) p.next_counts[(k * p.tiles + blockIdx.x) * kBins + threadIdx.x] = 0;
    for (int64_t i = from; i < to || i == from; i += kStep) {
        Keys<TOK, FIRST> keys;
        keys.load(p, i, to);
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kPlaces; ++k)
            if (keys.at[k] != kNone) atomicAdd(&count[(keys.at[k] >> p.shift) & (BINS - 1)], 1u);
    }
    __syncthreads();
#pragma unroll
    for (int d = threadIdx.x; d < BINS; d += kThreads) p.counts[blockIdx.x * BINS + d] = count[d];
}

// Each place's key and position to the place that its digit gives it.  Every workgroup adds up the counts for itself:
// the digits below (over all workgroups), then the workgroups, steps and waves before, then the places before.
//
// NEXT (up to kNextTiles workgroups): it counts the next pass's digits too, by the workgroup that will find them, in LDS
// and then in memory: whole numbers, so the order of the atomics changes nothing, and a pass takes one launch.
//
// Tables of 257 to 1,024 rows (bytes and a few more) take one pass of 10 bits: 300 rows of 1,024 in bf16, 8,000 tokens 18 us in
// all, in two passes 25; 50,000 tokens 38 and 42; 131,000 77 and 75, since every workgroup adds up four times the counts,
// hence kWideTiles.  3,000 tokens 16 us, in two passes by one workgroup 17.6.
constexpr int kNextTiles = 32;

template <int TOK, int OUT, bool FIRST, bool NEXT, int BITS>
__global__ __launch_bounds__(kThreads) void scatter(BwdParams p) {
    constexpr int BINS = 1 << BITS, PER = BINS / kThreads;      // a thread's digits, side by side
    if ((int)blockIdx.x >= p.tiles) return zero_share<OUT>(p);
    __shared__ uint32_t next[NEXT ? kNextTiles : 1][kBins];
    __shared__ uint32_t at[kWaves][BINS], waves[kWaves];
    const int d = threadIdx.x, wave = d >> 6, lane = d & 63;
    const int64_t n = FIRST ? p.ntokens : (int64_t)*p.valid;
    const int64_t from = (int64_t)blockIdx.x * p.tile, to = min(from + p.tile, n);
    Keys<TOK, FIRST> keys;
    keys.load(p, from, to);
    if constexpr (NEXT)
        for (int g = 0; g < p.tiles; ++g) next[g][d] = 0;
    auto count_step = [&] {
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
#pragma unroll
            for (int j = 0; j < PER; ++j) at[w][d * PER + j] = 0;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kPlaces; ++k)
            if (keys.at[k] != kNone) atomicAdd(&at[wave][(keys.at[k] >> p.shift) & (BINS - 1)], 1u);
        __syncthreads();
    };
    count_step();
    uint32_t total[PER] = {}, before[PER] = {}, mine = 0;
#pragma unroll 16
    for (int g = 0; g < p.tiles; ++g) {
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            const uint32_t c = p.counts[g * BINS + d * PER + j];
            total[j] += c;
            before[j] += g < (int)blockIdx.x ? c : 0u;
        }
    }
#pragma unroll
    for (int j = 0; j < PER; ++j) mine += total[j];
    // the digits below: within the wave, then the waves before
    uint32_t below = mine;
#pragma unroll
    for (int off = 1; off < 64; off *= 2) {
        const uint32_t v = __shfl_up(below, off, 64);
        below += lane >= off ? v : 0u;
    }
    if (lane == 63) waves[wave] = below;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) below += w < wave ? waves[w] : 0u;
    if (FIRST && blockIdx.x == 0 && d == kThreads - 1) *p.valid = below;
    below -= mine;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        before[j] += below;
        below += total[j];
    }

    for (int64_t i0 = from; i0 < to; i0 += kStep) {
        if (i0 > from) {
            keys.load(p, i0, to);
            __syncthreads();                            // the last step's places are taken
            count_step();
        }
#pragma unroll
        for (int w = 0; w < kWaves; ++w)
#pragma unroll
            for (int j = 0; j < PER; ++j) {
                const uint32_t c = at[w][d * PER + j];
                at[w][d * PER + j] = before[j];
                before[j] += c;
            }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < kPlaces; ++k) {
            const int64_t key = keys.at[k];
            const uint32_t digit = (uint32_t)(key >> p.shift) & (BINS - 1);
            const uint64_t same = same_digit<BITS>(digit, key != kNone);
            if (key != kNone) {
                const int first = __ffsll((unsigned long long)same) - 1;
                uint32_t base = 0;
                if (lane == first) base = atomicAdd(&at[wave][digit], (uint32_t)__popcll(same));
                base = __shfl(base, first, 64);
                const int64_t i = i0 + wave * (64 * kPlaces) + 64 * k + lane;
                const uint32_t dest = base + __popcll(same & ((1ull << lane) - 1));
                p.to[dest] = Pair{(uint32_t)key, FIRST ? (uint32_t)i : p.from[i].pos};
                if constexpr (NEXT) atomicAdd(&next[dest / kStep][(key >> (p.shift + 8)) & (kBins - 1)], 1u);
            }
        }
    }
    if constexpr (NEXT) {
        __syncthreads();
        for (int g = 0; g < p.tiles; ++g)
            if (next[g][d] != 0) atomicAdd(&p.next_counts[g * kBins + d], next[g][d]);
    }
}

// The whole sort by one workgroup, for up to kSmallTokens: places in registers, moved through LDS between the passes.
// The other workgroups set the table to zero meanwhile.  In a kernel trace 4,096 bytes take 6.4 us, and as many tokens of
// 30,000 values 14.3 with the 92 MB of such a table of 768 columns zeroed beside them (10.4 with 24 columns); the launches
// above take about 9 and 21, and two or four times the host's time.  Up to 1,024 tokens, where sum_direct does not take them:
// 1,000 bytes of 4,352 columns 13.8 us a call with 256 threads and 15.0 with 1,024, 1,000 tokens of 200,000 rows of 64 19.2
// and 22.4.  16 places per thread took 21.5 us for 16,384 bytes: one CU's issue rate, where the launches above spread over many.
constexpr int kSmallThreads = 1024;
constexpr int kSmallPlaces = 4;
constexpr int kSmallTokens = kSmallThreads * kSmallPlaces;

template <int TOK, int OUT, int THREADS>
__global__ __launch_bounds__(THREADS) void sort_small(BwdParams p) {
    constexpr int PER = kSmallPlaces, WAVES = THREADS / 64;
    if (blockIdx.x >= 1) return zero_share<OUT>(p);
    __shared__ uint32_t keys[THREADS * PER];
    __shared__ uint16_t places[THREADS * PER];
    __shared__ uint32_t at[WAVES][kBins], waves[kBins / 64];
    const int tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const int mine = wave * (64 * PER) + lane;                  // the wave's places, 64 side by side
    int n = (int)p.ntokens;
    constexpr uint32_t kNoKey = ~0u;                            // keys are below 2^31
    uint32_t key[PER], pos[PER], rank[PER];
#pragma unroll
    for (int k = 0; k < PER; ++k) {
        pos[k] = mine + 64 * k;
        key[k] = (int)pos[k] < n ? (uint32_t)key_at<TOK, true>(p, pos[k]) : kNoKey;
    }
    for (int pass = 0; pass < p.passes; ++pass) {
        const int shift = 8 * pass;
        for (int i = lane; i < kBins; i += 64) at[wave][i] = 0;
        __builtin_amdgcn_wave_barrier();                        // a wave's own counts, in its own order
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const uint32_t digit = (key[k] >> shift) & (kBins - 1);
            const uint64_t same = same_digit(digit, key[k] != kNoKey);
            const int first = same ? __ffsll((unsigned long long)same) - 1 : lane;
            uint32_t base = 0;
            if (key[k] != kNoKey && lane == first) base = atomicAdd(&at[wave][digit], (uint32_t)__popcll(same));
            rank[k] = __shfl(base, first, 64) + __popcll(same & ((1ull << lane) - 1));
        }
        __syncthreads();
        // thread d: where digit d of each wave goes
        uint32_t total = 0, below = 0;
        if (tid < kBins) {
#pragma unroll
            for (int w = 0; w < WAVES; ++w) total += at[w][tid];
            below = total;
#pragma unroll
            for (int off = 1; off < 64; off *= 2) {
                const uint32_t v = __shfl_up(below, off, 64);
                below += lane >= off ? v : 0u;
            }
            if (lane == 63) waves[wave] = below;
        }
        __syncthreads();
        if (tid < kBins) {
#pragma unroll
            for (int w = 0; w < kBins / 64; ++w) below += w < wave ? waves[w] : 0u;
            if (pass == 0 && tid == kBins - 1) *p.valid = below;
            below -= total;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const uint32_t c = at[w][tid];
                at[w][tid] = below;
                below += c;
            }
        }
        __syncthreads();
        if (pass + 1 == p.passes) {
#pragma unroll
            for (int k = 0; k < PER; ++k)
                if (key[k] != kNoKey)
                    p.to[at[wave][(key[k] >> shift) & (kBins - 1)] + rank[k]] = Pair{key[k], pos[k]};
            return;
        }
        if (pass == 0) n = (int)(waves[0] + waves[1] + waves[2] + waves[3]);
#pragma unroll
        for (int k = 0; k < PER; ++k)
            if (key[k] != kNoKey) {
                const uint32_t dest = at[wave][(key[k] >> shift) & (kBins - 1)] + rank[k];
                keys[dest] = key[k];
                places[dest] = (uint16_t)pos[k];
            }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int i = mine + 64 * k;
            key[k] = i < n ? keys[i] : kNoKey;
            pos[k] = i < n ? places[i] : 0u;
        }
        __syncthreads();
    }
}

// Few tokens: a workgroup per row of the table (BY_ROW) or per token, the first of its value, and tile of 256 columns.  Each
// wave looks through its share of the tokens, lists the places of its row's, and adds those up; the waves' sums are joined
// in LDS.  One launch, no sort, no workspace; by token, workgroups of their own set the other rows to zero.
//
// Bound by latency: a token, a list, rows of dy, a store.  256 rows of 512 in bf16, 500 tokens of a text: 4.1 us, the sort
// and the sums 12; 2,000 tokens 8 and 14.  5,000 rows of 512, by token: 500 6.6 and 14.6, 32,000 rows 10.9 and 17.7.  A row's
// tokens are one compute unit's work, about 60 GB/s, so the worst is one value throughout: 13 (1,000 tokens) and 30 us
// (2,000) where sort and sums, which cut evenly, take 11 and 14; 4,000 tokens of a text take as long either way, hence
// kDirectTokens.  Every workgroup reads all tokens: 1,000 rows of 1,792 take 13 to 16 us, 4,000 of them 42 to 50, 1,000 tokens
// of 32,000 rows of 1,024 24 and sorted 20, hence the limits on workgroups.  16 waves, 16 rows ahead (registers) and tiles
// of 512 columns: all no faster.
constexpr int kDirectWaves = 8;
constexpr int kDirectTokens = 2048;
constexpr int kDirectRows = 4096;      // workgroups at most, by row
constexpr int kDirectPlaces = 2048;    // by token
constexpr int kDirectSteps = kDirectTokens / (64 * kDirectWaves);
constexpr int kZeroBlocks = 1024;
constexpr int kZeroRows = 128;         // per workgroup at most

// Rows of the table that no token names, set to zero by `blocks` workgroups.
template <int TOK, int OUT, int S> __device__ __forceinline__ void zero_unnamed(const BwdParams &p, int block, int blocks) {
    __shared__ uint32_t named[kZeroRows];
    const int64_t per = (p.vocab + blocks - 1) / blocks, lo = block * per;
    const int rows = (int)max((int64_t)0, min(per, p.vocab - lo));
    for (int i = threadIdx.x; i < rows; i += blockDim.x) named[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < (int)p.ntokens; i += blockDim.x) {
        const int64_t t = token_at<TOK>(p.tokens, i);
        if (t >= lo && t < lo + rows) named[t - lo] = 1;
    }
    __syncthreads();
    const uint32_t spans = (uint32_t)((p.dim + S - 1) / S);
    const float zeros[S] = {};
    for (uint32_t i = threadIdx.x; i < rows * spans; i += blockDim.x) {
        const uint32_t r = i / spans;
        if (!named[r]) store_span<OUT, S>(p.dweight, (lo + r) * p.dim + span_at<S>((int64_t)(i - r * spans) * S, p.dim), zeros);
    }
}

template <int TOK, int DY, int OUT, int S, bool BY_ROW>
__global__ __launch_bounds__(64 * kDirectWaves) void sum_direct(BwdParams p, uint32_t col_tiles) {
    constexpr int AHEAD = 8;
    const int n = (int)p.ntokens;
    int64_t v = blockIdx.x / col_tiles;
    const int own = BY_ROW ? 0 : (int)v;                // the place whose token's row it is
    if constexpr (!BY_ROW) {
        if (own >= n) return zero_unnamed<TOK, OUT, S>(p, (int)(blockIdx.x - n * col_tiles), (int)(gridDim.x - n * col_tiles));
        v = token_at<TOK>(p.tokens, own);
        if (v < 0 || v >= p.vocab) return;
    }
    __shared__ uint16_t list[kDirectWaves][64 * kDirectSteps];
    __shared__ float sums[kDirectWaves][64 * S];
    __shared__ int found[kDirectWaves];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int share = (n + kDirectWaves - 1) / kDirectWaves, from = wave * share, to = min(from + share, n);
    const int64_t tile0 = (int64_t)(blockIdx.x % col_tiles) * (64 * S), col = span_at<S>(tile0 + lane * S, p.dim);
    int64_t t[kDirectSteps];
#pragma unroll
    for (int k = 0; k < kDirectSteps; ++k) t[k] = from + 64 * k + lane < to ? token_at<TOK>(p.tokens, from + 64 * k + lane) : kNone;
    int m = 0;
#pragma unroll
    for (int k = 0; k < kDirectSteps; ++k) {
        const uint64_t same = __ballot(t[k] == v);
        if (t[k] == v) list[wave][m + __popcll(same & ((1ull << lane) - 1))] = (uint16_t)(from + 64 * k + lane);
        m += __popcll(same);
    }
    __builtin_amdgcn_wave_barrier();                    // a wave's own list, in its own order
    if constexpr (!BY_ROW) {                            // an earlier place has the token: that one's workgroup adds up
        if (__syncthreads_or(m > 0 && list[wave][0] < own)) return;
    }
    if (m > 0) {
        float acc[S] = {};
        for (int i = 0; i < m; i += AHEAD) {
            Span<DY, S> row[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) row[k].template load<true>(p.dy, (int64_t)list[wave][min(i + k, m - 1)] * p.dim + col);
            float part[S] = {};
#pragma unroll
            for (int k = 0; k < AHEAD; ++k)
#pragma unroll
                for (int j = 0; j < S; ++j) part[j] += i + k < m ? row[k].get(j) : 0.0f;
#pragma unroll
            for (int j = 0; j < S; ++j) acc[j] += part[j];
        }
#pragma unroll
        for (int j = 0; j < S; ++j) sums[wave][j * 64 + lane] = acc[j];
    }
    if (lane == 0) found[wave] = m;
    __syncthreads();
    if (wave != 0) return;
    float acc[S] = {};
#pragma unroll
    for (int w = 0; w < kDirectWaves; ++w)
        if (found[w] > 0) {
#pragma unroll
            for (int j = 0; j < S; ++j) acc[j] += sums[w][j * 64 + lane];
        }
#pragma unroll
    for (int j = 0; j < S; ++j) acc[j] *= p.scale;
    store_span<OUT, S>(p.dweight, v * p.dim + col, acc);
}

// Sums of the rows of a group of kWaves chunks, one chunk per wave, for one tile of columns.
template <int DY, int OUT, int S>
__global__ __launch_bounds__(kThreads) void sum_chunks(BwdParams p, uint32_t col_tiles) {
    constexpr int AHEAD = 8;
    __shared__ float piece[kWaves][2][64][S];           // a chunk's first run's sum, and its last one's
    __shared__ uint32_t piece_key[kWaves][2];
    __shared__ int piece_is[kWaves];
    constexpr int kHead = 1, kThrough = 2, kTail = 4;   // the first run came from before; it goes on after; the last one does
    const int64_t group = blockIdx.x / col_tiles, most = p.ntokens - 1;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t from = (group * kWaves + wave) * p.chunk;
    // All that the wave reads of the list, asked for at once; places past the valid ones hold nothing that counts.
    const Pair mine = p.to[min(from + lane, most)];
    const uint32_t key_before = p.to[min(max(from - 1, (int64_t)0), most)].key, key_after = p.to[min(from + p.chunk, most)].key;
    const int64_t n = *p.valid;
    if (group * kWaves * p.chunk >= n) return;
    const int64_t col = span_at<S>((int64_t)(blockIdx.x % col_tiles) * (64 * S) + lane * S, p.dim);
    const int m = (int)max((int64_t)0, min((int64_t)p.chunk, n - from));
    // The sum of a run that is whole, in dW's type.
    auto finish = [&](const float (&acc)[S], uint32_t key) {
        float v[S];
#pragma unroll
        for (int j = 0; j < S; ++j) v[j] = p.scale * acc[j];
        store_span<OUT, S>(p.dweight, (int64_t)key * p.dim + col, v);
    };
    int is = 0;
    if (m > 0) {
        const int64_t before = from > 0 ? (int64_t)key_before : kNone;
        const int64_t after = from + m < n ? (int64_t)key_after : kNone;
        float acc[S] = {};
        uint32_t key = __builtin_amdgcn_readlane(mine.key, 0);
        bool came = before == (int64_t)key;             // the run at hand began before the chunk
        auto keep = [&](int which) {
#pragma unroll
            for (int j = 0; j < S; ++j) piece[wave][which][lane][j] = acc[j];
            if (lane == 0) piece_key[wave][which] = key;
        };
        Span<DY, S> row[2][AHEAD];
        auto load = [&](Span<DY, S> (&r)[AHEAD], int i0) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const uint32_t pos = __builtin_amdgcn_readlane(mine.pos, min(i0 + k, m - 1));
                r[k].template load<true>(p.dy, pos * p.dim + col);
            }
        };
        auto add = [&](const Span<DY, S> (&r)[AHEAD], int i0) {
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (i0 + k >= m) break;
                const uint32_t next = __builtin_amdgcn_readlane(mine.key, i0 + k);
                if (next != key) {
                    if (came) {
                        keep(0);
                        is |= kHead;
                    } else {
                        finish(acc, key);
                    }
                    came = false;
                    key = next;
#pragma unroll
                    for (int j = 0; j < S; ++j) acc[j] = 0.0f;
                }
#pragma unroll
                for (int j = 0; j < S; ++j) acc[j] += r[k].get(j);
            }
        };
        // the next rows are on their way while a group is added up
        load(row[0], 0);
        for (int i0 = 0; i0 < m; i0 += 2 * AHEAD) {
            wait_for_memory();
            if (i0 + AHEAD < m) load(row[1], i0 + AHEAD);
            add(row[0], i0);
            wait_for_memory();
            if (i0 + 2 * AHEAD < m) load(row[0], i0 + 2 * AHEAD);
            add(row[1], i0 + AHEAD);
        }
        const bool goes_on = after == (int64_t)key;
        if (came) {
            keep(0);
            is |= kHead | (goes_on ? kThrough : 0);
        } else if (goes_on) {
            keep(1);
            is |= kTail;
        } else {
            finish(acc, key);
        }
    }
    if (lane == 0) piece_is[wave] = is;
    __syncthreads();
    if (wave != 0) return;

    // The runs that lie in more than one of the group's chunks, or go beyond it.
    float acc[S] = {};
    uint32_t key = 0;
    bool open = false, came = false;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        const int f = piece_is[w];
        if (f & kHead) {
            came = w == 0 || came;
            key = piece_key[w][0];
            open = true;
#pragma unroll
            for (int j = 0; j < S; ++j) acc[j] += piece[w][0][lane][j];
            if (!(f & kThrough)) {
                if (came) store_span<0, S>(p.head, group * p.dim + col, acc);
                else finish(acc, key);
                open = came = false;
#pragma unroll
                for (int j = 0; j < S; ++j) acc[j] = 0.0f;
            }
        }
        if (f & kTail) {
            key = piece_key[w][1];
            open = true;
#pragma unroll
            for (int j = 0; j < S; ++j) acc[j] = piece[w][1][lane][j];
        }
    }
    if (open) store_span<0, S>(came ? p.head : p.tail, group * p.dim + col, acc);
}

// The tokens whose rows lie in more than one group: the group in which one begins joins its sums.
template <int OUT, int S>
__global__ __launch_bounds__(64 * kJoinWaves) void join_groups(BwdParams p, uint32_t col_tiles) {
    __shared__ float sums[kJoinWaves][64][S];
    const int64_t size = (int64_t)kWaves * p.chunk, group = blockIdx.x / col_tiles, from = group * size, next = from + size;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // All that the decision reads, asked for at once; places past the valid ones hold nothing that counts.
    const int64_t most = p.ntokens - 1, n = *p.valid;
    const uint32_t first = p.to[from].key, before = p.to[max(from - 1, (int64_t)0)].key;
    const uint32_t key = p.to[min(next - 1, most)].key, after = p.to[min(next, most)].key;
    uint32_t begins = p.to[min(next + lane * size, most)].key;
    if (next >= n || after != key) return;                      // nothing goes on
    if (first == key && from > 0 && before == key) return;      // it began before
    // the groups after this one that begin with the token
    int64_t parts = 0;
    for (;;) {
        const uint64_t same = __ballot(next + (parts + lane) * size < n && begins == key);
        const int run = ~same == 0 ? 64 : __ffsll((unsigned long long)~same) - 1;
        parts += run;
        if (run < 64) break;
        begins = p.to[min(next + (parts + lane) * size, most)].key;
    }
    const int64_t col = span_at<S>((int64_t)(blockIdx.x % col_tiles) * (64 * S) + lane * S, p.dim);
    // sum 0 is the tail of this group, the others the heads of the next; each wave takes a run of them
    const int64_t all = parts + 1, lo = all * wave / kJoinWaves, hi = all * (wave + 1) / kJoinWaves;
    float acc[S] = {};
#pragma unroll 8
    for (int64_t k = lo; k < hi; ++k) {
        Span<0, S> s;
        s.load(k == 0 ? p.tail : p.head, (group + k) * p.dim + col);
#pragma unroll
        for (int j = 0; j < S; ++j) acc[j] += s.get(j);
    }
#pragma unroll
    for (int j = 0; j < S; ++j) sums[wave][lane][j] = acc[j];
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < kJoinWaves; ++w)
#pragma unroll
        for (int j = 0; j < S; ++j) acc[j] += sums[w][lane][j];
#pragma unroll
    for (int j = 0; j < S; ++j) acc[j] *= p.scale;
    store_span<OUT, S>(p.dweight, (int64_t)key * p.dim + col, acc);
}

}  // namespace embed
}  // namespace mbs
