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
#pragma once

#include <hip/hip_runtime.h>

#include "device_math.hpp"

namespace mbs {
namespace sample {

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
};

// A row's softmax: e^((l - max) / T) times inv is a probability; ok: the row is a distribution.
struct Row {
    float max, inv;
    bool ok;
    // Rounded before anything is taken from it: fused into p - q it would leave the rounding of q where p equals q.
    __device__ __forceinline__ float prob(float l, float inv_temp) const {
#pragma clang fp contract(off)
        return expf((l - max) * inv_temp) * inv;
    }
};

// Maxima and sums of pieces of a row.  A piece with nothing above -infinity adds nothing.
struct Piece {
    float max = -__builtin_inff(), sum = 0.0f;
    __device__ __forceinline__ void add(float l, float inv_temp) { join(Piece{l, l == -__builtin_inff() ? 0.0f : 1.0f}, inv_temp); }
    __device__ __forceinline__ void join(Piece o, float inv_temp) {
        const float m = __builtin_fmaxf(max, o.max);
        // a piece without a sum stays out; infinities and NaN make a NaN of the sum
        float s = 0.0f;
        if (sum != 0.0f) s += sum * expf((max - m) * inv_temp);
        if (o.sum != 0.0f) s += o.sum * expf((o.max - m) * inv_temp);
        max = m;
        sum = s;
    }
    __device__ __forceinline__ Row row() const {
        const bool ok = sum > 0.0f && sum < __builtin_inff();
        return Row{max, 1.0f / sum, ok};
    }
};

template <int DT> __device__ Row row_of(const void *base, int64_t at, int64_t vocab, float inv_temp) {
    Piece a;
    for (int64_t y = threadIdx.x & 63; y < vocab; y += 64) a.add(Act<DT>::ld(base, at + y), inv_temp);
    for (int off = 32; off > 0; off >>= 1) {
        Piece o;
        o.max = __shfl_xor(a.max, off, 64);
        o.sum = __shfl_xor(a.sum, off, 64);
        a.join(o, inv_temp);
    }
    return a.row();
}

// One wave per sequence, row after row.
template <int DT>
__global__ __launch_bounds__(64) void verify_sample(Params p) {
    const int64_t b = blockIdx.x, V = p.vocab, n = p.ndraft;
    const int lane = threadIdx.x;
    int64_t len = p.lengths ? p.lengths[b] : n;
    len = len < 0 ? 0 : len > n ? n : len;
    int64_t c = -1;
    for (int64_t i = 0; i < n; ++i) {
        if (i >= len || (c >= 0 && !p.probs)) {
            if (p.probs && lane == 0) p.probs[b * n + i] = 0.0f;
            continue;
        }
        const int64_t at = (b * (n + 1) + i) * V, qat = (b * n + i) * V;
        const int64_t x = p.draft[b * n + i];
        const bool in_range = x >= 0 && x < V;
        const Row t = row_of<DT>(p.logits, at, V, p.inv_temp);
        const float px = in_range && t.ok ? t.prob(Act<DT>::ld(p.logits, at + x), p.inv_temp) : 0.0f;
        float qx = 1.0f;
        bool ok = in_range && t.ok;
        if (p.draft_logits) {
            const Row q = row_of<DT>(p.draft_logits, qat, V, p.inv_temp);
            ok = ok && q.ok;
            if (ok) qx = q.prob(Act<DT>::ld(p.draft_logits, qat + x), p.inv_temp);
        }
        if (lane == 0 && p.probs) p.probs[b * n + i] = px;
        if (c < 0 && !(ok && p.uniform[b * n + i] * qx < px)) c = i;
    }
    if (c < 0) c = len;
    const int64_t at = (b * (n + 1) + c) * V, qat = (b * n + c) * V;
    const Row t = row_of<DT>(p.logits, at, V, p.inv_temp);
    Row q{0.0f, 0.0f, false};
    int64_t x = -1;
    if (c < len) {
        x = p.draft[b * n + c];
        if (p.draft_logits) q = row_of<DT>(p.draft_logits, qat, V, p.inv_temp);
    }
    // the best of what is left of p, and of p itself
    float best = 0.0f, best_p = 0.0f;
    int64_t who = -1, who_p = -1;
    if (t.ok)
        for (int64_t y = lane; y < V; y += 64) {
            const float pr = t.prob(Act<DT>::ld(p.logits, at + y), p.inv_temp), e = p.noise[b * V + y];
            float left = pr;
            if (c < len && p.draft_logits) left = q.ok ? pr - q.prob(Act<DT>::ld(p.draft_logits, qat + y), p.inv_temp) : pr;
            else if (y == x) left = 0.0f;
            if (left > 0.0f && left / e > best) { best = left / e; who = y; }
            if (pr / e > best_p) { best_p = pr / e; who_p = y; }
        }
    auto reduce = [](float &v, int64_t &w) {
        for (int off = 32; off > 0; off >>= 1) {
            const float ov = __shfl_xor(v, off, 64);
            const int64_t ow = __shfl_xor(w, off, 64);
            if (ow >= 0 && (w < 0 || ov > v || (ov == v && ow < w))) { v = ov; w = ow; }
        }
    };
    reduce(best, who);
    reduce(best_p, who_p);
    if (lane == 0) {
        p.accepted[b] = (int32_t)c;
        if (p.last_pos) p.last_pos[b] = (int32_t)c - 1;
        p.next_token[b] = (int32_t)(who >= 0 ? who : who_p);
    }
}

}  // namespace sample
}  // namespace mbs
