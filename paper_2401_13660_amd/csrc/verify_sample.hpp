// verify_sample.hpp -- drafted tokens against the target's probabilities, from given random numbers.
//
// Row i of the target's logits scores drafted token x_i, and row len (the number of tokens drafted)
// the token after them all.  With p_i = softmax(logits_i / T) and q_i the drafter's distribution
// (softmax(draft_logits_i / T), or certainty of x_i without them):
//
//   token i passes when uniform_i q_i(x_i) < p_i(x_i);   accepted c = the leading tokens that pass
//   r = max(p_c - q_c, 0) for c < len (p_c where that is zero everywhere), r = p_len for c = len
//   next = the y of the largest r(y) / noise(y), the lowest such y
//
// With uniform numbers in [0, 1) and exponential noise of mean 1, the tokens kept and the next one
// are distributed as the target's own samples (the next one by a race of exponential clocks: the
// smallest noise(y) / r(y) falls on y with probability r(y) / sum r).  A race needs no running sum
// over the vocabulary, so its outcome hardly depends on how the probabilities round.
//
// exp((l - max) / T): the maximum is taken from the logits themselves, so that rows of the type's
// lowest values stay distributions.  A row that is none (a NaN or +infinity in it, or nothing above
// -infinity) accepts nothing, and no token follows it (-1).
//
// Up to kSmallVocab tokens (bytes): one workgroup per sequence, one wave per row, the row in
// registers from one load to the token drawn; the wave whose row stops the sequence draws, and the
// rows after it are only looked at where their probabilities are wanted.  Larger vocabularies: the
// rows are cut into pieces of kPiece tokens whose maxima and sums one launch finds; a second one
// joins them, decides, and races within each piece of the row that stops the sequence; a third one
// joins the pieces' winners.
//
// Bound by latency: in a kernel trace 16 drafts of 32 prompts over 256 bytes take 6.0 us for 1.1 MB (58 with
// one wave per sequence), one byte of one prompt 2.4; 4 drafts of 16 prompts over 32,000 tokens in bf16, 11 MB,
// 14.9 us a call and 5.7, 8.0 and 2.5 in the trace, where launches do not overlap.  With races of 8,192 tokens
// per workgroup instead of 2,048 the second launch took 16, and maxima and sums by 8,192 instead of 4,096
// took 0.6 us longer.
#pragma once

#include <hip/hip_runtime.h>

#include "device_math.hpp"
#include "lanes.hpp"

namespace mbs {
namespace sample {

constexpr int kSmallVocab = 1024;
constexpr int kMaxWaves = 16;
constexpr int kThreads = 256;      // of a piece
constexpr int kPieceSpans = 4;     // spans of 4 per thread where maxima and sums are found
constexpr int kRaceSpans = 2;      // and where the race is run, two exponentials and a division per token
constexpr int kPiece = kThreads * kPieceSpans * 4;
constexpr int kRacePiece = kThreads * kRaceSpans * 4;
constexpr int32_t kNobody = 0x7fffffff;

struct Best { float left, whole; int32_t left_at, whole_at; };

struct Params {
    int64_t batch, ndraft, vocab;
    const void *logits;           // (batch, ndraft + 1, vocab) act
    const void *draft_logits;     // (batch, ndraft, vocab) act or null
    const int32_t *draft;         // (batch, ndraft)
    const int32_t *lengths;       // (batch) or null: ndraft
    const float *uniform;         // (batch, ndraft)
    const float *noise;           // (batch, vocab)
    int32_t *accepted;            // (batch)
    int32_t *last_pos;            // (batch) or null: accepted - 1
    int32_t *next_token;          // (batch)
    float *probs;                 // (batch, ndraft) or null: the target's of the drafted tokens
    float inv_temp;
    int32_t pieces, race_pieces;  // per row, of a large vocabulary
    float2 *stats;                // (batch, 2 ndraft + 1, pieces): maximum and sum; the target's rows, then the drafter's
    Best *best;                   // (batch, race_pieces)
};

__device__ __forceinline__ int64_t length_of(const Params &p, int64_t b) {
    const int64_t len = p.lengths ? p.lengths[b] : p.ndraft;
    return len < 0 ? 0 : len > p.ndraft ? p.ndraft : len;
}

// e^((l - max) / T).  expf's own error is an ulp or so; a plain 2^x of the scaled argument would add the rounding of
// that argument, up to 40 ulp for the logits met here.
__device__ __forceinline__ float weight(float l, float max, float inv_temp) { return expf((l - max) * inv_temp); }

// Probabilities are rounded before anything is taken from them: fused into p - q the product would leave the rounding
// of q where p equals q.
__device__ __forceinline__ float rounded_product(float a, float b) {
#pragma clang fp contract(off)
    return a * b;
}

// A row's softmax.  ok: the row is a distribution.  The sum is 0 where nothing is above -infinity, and NaN with a NaN
// or +infinity in the row.
struct Row {
    float max = 0.0f, inv = 0.0f;
    bool ok = false;
    __device__ __forceinline__ void set(float m, float sum) {
        max = m;
        inv = 1.0f / sum;
        ok = sum > 0.0f && sum < __builtin_inff();
    }
    __device__ __forceinline__ float prob(float l, float inv_temp) const {
        return rounded_product(weight(l, max, inv_temp), inv);
    }
};

// The candidate with the largest score, the lowest of them; scores are above 0.
struct Race {
    float score = 0.0f;
    int32_t at = kNobody;
    __device__ __forceinline__ void run(float r, float noise, int32_t y) {
        const float s = r / noise;
        if (r > 0.0f && s > score) {
            score = s;
            at = y;
        }
    }
    __device__ __forceinline__ void join(float s, int32_t y) {
        if (y != kNobody && (s > score || (s == score && y < at))) {
            score = s;
            at = y;
        }
    }
    __device__ __forceinline__ void join_wave() {
        const float s = wave_max(score);
        at = wave_min(score == s ? at : kNobody);
        score = s;
    }
};

__device__ __forceinline__ void write_outcome(const Params &p, int64_t b, int64_t c) {
    p.accepted[b] = (int32_t)c;
    if (p.last_pos) p.last_pos[b] = (int32_t)c - 1;
}

// ---- small vocabularies ---------------------------------------------------------

// A row in a wave's registers: lane l holds tokens 256 j + 4 l + i.
template <int DT, int KPL> struct RowInLanes {
    Span<DT, 4> s[KPL / 4];
    float v[KPL];                                       // logits, then weights
    Row row;
    __device__ __forceinline__ void load(const void *base, int64_t at, int vocab, int lane) {
#pragma unroll
        for (int j = 0; j < KPL / 4; ++j) {
            const int y = 256 * j + 4 * lane;
            if (y + 4 <= vocab) s[j].load(base, at + y);
            else s[j].load_first(base, at + y, max(vocab - y, 0));
        }
    }
    __device__ __forceinline__ void softmax(int vocab, int lane, float inv_temp) {
        float m = -__builtin_inff();
#pragma unroll
        for (int k = 0; k < KPL; ++k) {
            v[k] = 256 * (k / 4) + 4 * lane + k % 4 < vocab ? s[k / 4].get(k % 4) : -__builtin_inff();
            m = __builtin_fmaxf(m, v[k]);
        }
        m = wave_max(m);
        // nothing above -infinity: weights of 0, not of NaN
        const float at = m == -__builtin_inff() ? 0.0f : m;
        float sum = 0.0f;
#pragma unroll
        for (int k = 0; k < KPL; ++k) {
            v[k] = weight(v[k], at, inv_temp);
            sum += v[k];
        }
        row.set(m, wave_sum(sum));
    }
    __device__ __forceinline__ float prob(int k) const { return rounded_product(v[k], row.inv); }
    // of one token, the same in every lane
    __device__ __forceinline__ float prob_of(int x) const {
        float r = 0.0f;
#pragma unroll
        for (int k = 0; k < KPL; ++k) r = 256 * (k / 4) + k % 4 == (x & ~255) + x % 4 ? prob(k) : r;
        return lane_value(r, (x & 255) >> 2);
    }
};

template <int DT, int KPL>
__global__ __launch_bounds__(64 * kMaxWaves) void verify_small(Params p) {
    __shared__ int stop;
    const int64_t b = blockIdx.x, n = p.ndraft;
    const int V = (int)p.vocab, lane = threadIdx.x & 63, waves = blockDim.x >> 6;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int len = (int)length_of(p, b);
    if (threadIdx.x == 0) stop = kNobody;
    if (p.probs)
        for (int64_t i = len + (int64_t)threadIdx.x; i < n; i += blockDim.x) p.probs[b * n + i] = 0.0f;
    RowInLanes<0, KPL> noise;
    noise.load(p.noise, b * V, V, lane);
    __syncthreads();
    int c = kNobody;                                    // the row that stops the sequence, once it is known
    for (int base = 0; base <= len; base += waves) {
        const int i = base + wave;
        const bool open = c == kNobody, here = i < len || (i == len && open);
        const bool have_q = open && i < len && p.draft_logits;
        RowInLanes<DT, KPL> t, q;
        int x = -1;
        if (here) {
            t.load(p.logits, (b * (n + 1) + i) * V, V, lane);
            if (have_q) q.load(p.draft_logits, (b * n + i) * V, V, lane);
            bool passes = false;
            if (i < len) {
                x = __builtin_amdgcn_readfirstlane(p.draft[b * n + i]);
                const float u = p.uniform[b * n + i];
                t.softmax(V, lane, p.inv_temp);
                const bool valid = x >= 0 && x < V && t.row.ok;
                const float px = valid ? t.prob_of(x) : 0.0f;
                float qx = 1.0f;
                if (have_q) q.softmax(V, lane, p.inv_temp);
                if (have_q && valid) qx = q.prob_of(x);
                passes = valid && (!have_q || q.row.ok) && u * qx < px;
                if (p.probs && lane == 0) p.probs[b * n + i] = px;
            } else {
                t.softmax(V, lane, p.inv_temp);
            }
            if (open && !passes && lane == 0) atomicMin(&stop, i);
        }
        __syncthreads();
        c = stop;
        if (open && here && i == c) {
            Race race;
            if (t.row.ok) {
                const bool less_q = have_q && q.row.ok;
#pragma unroll
                for (int k = 0; k < KPL; ++k) {
                    const int y = 256 * (k / 4) + 4 * lane + k % 4;
                    float left = t.prob(k);
                    if (less_q) left -= q.prob(k);
                    else if (!have_q && y == x) left = 0.0f;
                    race.run(y < V ? left : 0.0f, noise.s[k / 4].get(k % 4), y);
                }
                race.join_wave();
                if (race.at == kNobody) {
#pragma unroll
                    for (int k = 0; k < KPL; ++k) {
                        const int y = 256 * (k / 4) + 4 * lane + k % 4;
                        race.run(y < V ? t.prob(k) : 0.0f, noise.s[k / 4].get(k % 4), y);
                    }
                    race.join_wave();
                }
            }
            if (lane == 0) {
                write_outcome(p, b, c);
                p.next_token[b] = race.at == kNobody ? -1 : race.at;
            }
        }
        if (c != kNobody && !p.probs) break;
        __syncthreads();                                // every wave has read it before a later row may set it
    }
}

// ---- large vocabularies -----------------------------------------------------------

// A thread's share of a piece: spans of 4, 256 threads side by side.
template <int DT, int SPANS> struct PieceInLanes {
    Span<DT, 4> s[SPANS];
    __device__ __forceinline__ static int token(int piece, int k) {
        return (piece * SPANS + k) * (kThreads * 4) + (int)threadIdx.x * 4;
    }
    __device__ __forceinline__ void load(const void *base, int64_t at, int piece, int64_t vocab) {
#pragma unroll
        for (int k = 0; k < SPANS; ++k) {
            const int64_t y = token(piece, k);
            if (y + 4 <= vocab) s[k].load(base, at + y);
            else s[k].load_first(base, at + y, (int)max(vocab - y, (int64_t)0));
        }
    }
    __device__ __forceinline__ float get(int piece, int k, int i, int64_t vocab) const {
        return token(piece, k) + i < vocab ? s[k].get(i) : -__builtin_inff();
    }
};

__device__ __forceinline__ float block_all(float v, float *red, bool sum) {
    v = sum ? wave_sum(v) : wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return sum ? (red[0] + red[1]) + (red[2] + red[3])
               : __builtin_fmaxf(__builtin_fmaxf(red[0], red[1]), __builtin_fmaxf(red[2], red[3]));
}

template <int DT>
__global__ __launch_bounds__(kThreads) void piece_stats(Params p) {
    __shared__ float red[kThreads / 64];
    const int64_t rows = 2 * p.ndraft + 1, row = blockIdx.x / p.pieces, b = row / rows, i = row - b * rows;
    const int piece = (int)(blockIdx.x - row * p.pieces);
    const bool target = i <= p.ndraft;
    const int64_t at = target ? i : i - (p.ndraft + 1), len = length_of(p, b);
    if (target ? at > len : at >= len || !p.draft_logits) return;
    PieceInLanes<DT, kPieceSpans> v;
    v.load(target ? p.logits : p.draft_logits, (target ? b * (p.ndraft + 1) + at : b * p.ndraft + at) * p.vocab, piece, p.vocab);
    float m = -__builtin_inff();
#pragma unroll
    for (int k = 0; k < kPieceSpans; ++k)
#pragma unroll
        for (int j = 0; j < 4; ++j) m = __builtin_fmaxf(m, v.get(piece, k, j, p.vocab));
    m = block_all(m, red, false);
    const float from = m == -__builtin_inff() ? 0.0f : m;
    float sum = 0.0f;
#pragma unroll
    for (int k = 0; k < kPieceSpans; ++k) {
        float part = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) part += weight(v.get(piece, k, j, p.vocab), from, p.inv_temp);
        sum += part;
    }
    sum = block_all(sum, red, true);
    if (threadIdx.x == 0) p.stats[row * p.pieces + piece] = make_float2(m, sum);
}

// Row i of a sequence (the target's first, then the drafter's) from its pieces; a wave's lanes together.
__device__ __forceinline__ Row join_row(const Params &p, int64_t b, int64_t i) {
    const float2 *s = p.stats + (b * (2 * p.ndraft + 1) + i) * p.pieces;
    const int lane = threadIdx.x & 63;
    float m = -__builtin_inff(), sum = 0.0f;
    for (int k = lane; k < p.pieces; k += 64) m = __builtin_fmaxf(m, s[k].x);
    m = wave_max(m);
    // a piece with nothing above -infinity adds nothing; one that holds a NaN or +infinity adds NaN
    for (int k = lane; k < p.pieces; k += 64)
        sum += s[k].y == 0.0f ? 0.0f : rounded_product(s[k].y, weight(s[k].x, m, p.inv_temp));
    Row r;
    r.set(m, wave_sum(sum));
    return r;
}

template <int DT>
__global__ __launch_bounds__(kThreads) void decide_and_race(Params p) {
    __shared__ int stop;
    __shared__ float scores[kThreads / 64];
    __shared__ int32_t who[kThreads / 64];
    const int64_t b = blockIdx.x / p.race_pieces, n = p.ndraft, V = p.vocab;
    const int piece = (int)(blockIdx.x - b * p.race_pieces);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int len = (int)length_of(p, b);
    if (threadIdx.x == 0) stop = len;
    PieceInLanes<0, kRaceSpans> e;
    e.load(p.noise, b * V, piece, V);
    __syncthreads();
    const bool probs = p.probs && piece == 0;
    for (int i = wave; i < len; i += kThreads / 64) {   // a row per wave
        const int64_t x = p.draft[b * n + i];
        const bool in_range = x >= 0 && x < V;
        const float u = p.uniform[b * n + i];
        const float lx = in_range ? Act<DT>::ld(p.logits, (b * (n + 1) + i) * V + x) : 0.0f;
        const float mx = in_range && p.draft_logits ? Act<DT>::ld(p.draft_logits, (b * n + i) * V + x) : 0.0f;
        const Row t = join_row(p, b, i);
        bool ok = in_range && t.ok;
        const float px = ok ? t.prob(lx, p.inv_temp) : 0.0f;
        float qx = 1.0f;
        if (p.draft_logits) {
            const Row q = join_row(p, b, n + 1 + i);
            ok = ok && q.ok;
            if (ok) qx = q.prob(mx, p.inv_temp);
        }
        if (lane == 0) {
            if (!(ok && u * qx < px)) atomicMin(&stop, i);
            if (probs) p.probs[b * n + i] = px;
        }
    }
    if (probs)
        for (int64_t i = len + (int64_t)threadIdx.x; i < n; i += kThreads) p.probs[b * n + i] = 0.0f;
    __syncthreads();
    const int c = stop;
    if (piece == 0 && threadIdx.x == 0) write_outcome(p, b, c);

    const bool have_q = c < len && p.draft_logits;
    PieceInLanes<DT, kRaceSpans> tl, ql;
    tl.load(p.logits, (b * (n + 1) + c) * V, piece, V);
    if (have_q) ql.load(p.draft_logits, (b * n + c) * V, piece, V);
    const int64_t x = c < len && !p.draft_logits ? p.draft[b * n + c] : -1;
    const Row t = join_row(p, b, c);
    Row q;
    if (have_q) q = join_row(p, b, n + 1 + c);
    // the race of what is left of the target, or (second) of the target itself, within the workgroup
    auto race = [&](bool whole) {
        Race r;
        if (t.ok) {
#pragma unroll
            for (int k = 0; k < kRaceSpans; ++k)
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int y = PieceInLanes<DT, kRaceSpans>::token(piece, k) + j;
                    float left = t.prob(tl.s[k].get(j), p.inv_temp);
                    if (!whole && q.ok) left -= q.prob(ql.s[k].get(j), p.inv_temp);
                    if (!whole && y == x) left = 0.0f;
                    r.run(y < V ? left : 0.0f, e.s[k].get(j), y);
                }
        }
        r.join_wave();
        __syncthreads();
        if (lane == 0) {
            scores[wave] = r.score;
            who[wave] = r.at;
        }
        __syncthreads();
        for (int w = 0; w < kThreads / 64; ++w) r.join(scores[w], who[w]);
        return r;
    };
    const Race left = race(false);
    Race whole;
    if (left.at == kNobody) whole = race(true);         // needed only where no piece of the row has anything left
    if (threadIdx.x == 0) p.best[b * p.race_pieces + piece] = Best{left.score, whole.score, left.at, whole.at};
}

__global__ __launch_bounds__(64) void join_races(Params p) {
    const int64_t b = blockIdx.x;
    Race left, whole;
    for (int k = threadIdx.x; k < p.race_pieces; k += 64) {
        const Best o = p.best[b * p.race_pieces + k];
        left.join(o.left, o.left_at);
        whole.join(o.whole, o.whole_at);
    }
    left.join_wave();
    whole.join_wave();
    if (threadIdx.x == 0) p.next_token[b] = left.at != kNobody ? left.at : whole.at != kNobody ? whole.at : -1;
}

}  // namespace sample
}  // namespace mbs
