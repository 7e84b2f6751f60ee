// model_ops.hip -- the C ABI of what surrounds the layers' scan in a model: the embedding and its
// gradient, the convolution's gradient, the gradients' norm and clipping, and the verification of
// drafted tokens by random numbers.  Argument checks and kernel dispatch; the contract is in
// include/mbscan.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdlib>

#include "abi_checks.hpp"
#include "conv1d_bwd.hpp"
#include "embedding.hpp"
#include "grad_clip.hpp"
#include "mbscan.h"
#include "verify_sample.hpp"

namespace {

using namespace mbs::abi;

struct Range { const void *p; size_t n; };

// Does any of the outputs overlap an input or another output?
template <int NO, int NI> bool any_overlap(const Range (&outs)[NO], const Range (&ins)[NI]) {
    for (int i = 0; i < NO; ++i) {
        for (const Range &r : ins)
            if (overlaps(outs[i].p, outs[i].n, r.p, r.n)) return true;
        for (int k = i + 1; k < NO; ++k)
            if (overlaps(outs[i].p, outs[i].n, outs[k].p, outs[k].n)) return true;
    }
    return false;
}

// Workgroups of a grid-stride launch: enough for `items`, at most 2^20.
unsigned blocks_for(int64_t items) { return (unsigned)std::min<int64_t>(std::max<int64_t>(items, 1), 1 << 20); }

int status(hipError_t e) { return e == hipSuccess ? MB_OK : MB_ERR_HIP; }

bool valid_token_type(int32_t t) { return t == MB_TOKEN_U8 || t == MB_TOKEN_I32 || t == MB_TOKEN_I64; }
size_t token_size(int32_t t) { return t == MB_TOKEN_U8 ? 1 : t == MB_TOKEN_I32 ? 4 : 8; }

template <int TOK, int A> const void *embed_fwd_fn(int32_t out) {
    return out == MB_F32 ? reinterpret_cast<const void *>(&mbs::embed::embed_fwd<TOK, A, 0>)
                         : reinterpret_cast<const void *>(&mbs::embed::embed_fwd<TOK, A, 1>);
}
template <int TOK> const void *embed_fwd_fn(int32_t in, int32_t out) {
    return in == MB_F32 ? embed_fwd_fn<TOK, 0>(out) : embed_fwd_fn<TOK, 1>(out);
}
template <int TOK, int A> const void *embed_bwd_fn(int32_t out) {
    return out == MB_F32 ? reinterpret_cast<const void *>(&mbs::embed::embed_bwd<TOK, A, 0>)
                         : reinterpret_cast<const void *>(&mbs::embed::embed_bwd<TOK, A, 1>);
}
template <int TOK> const void *embed_bwd_fn(int32_t in, int32_t out) {
    return in == MB_F32 ? embed_bwd_fn<TOK, 0>(out) : embed_bwd_fn<TOK, 1>(out);
}

// The checks that both directions share; the element counts of the tokens' and the table's rows.
int embed_checks(int64_t ntokens, int64_t vocab, int64_t dim, int32_t token_type, int32_t in_dtype, int32_t out_dtype,
                 int64_t *row_elems, int64_t *table_elems) {
    if (ntokens < 0 || vocab < 0 || dim < 0 || vocab >= (int64_t(1) << 31)) return MB_ERR_SHAPE;
    if (!valid_token_type(token_type) || !valid_dtype(in_dtype) || !valid_dtype(out_dtype)) return MB_ERR_DTYPE;
    if (ntokens >= kMaxElems || !mul_ok(ntokens, dim, row_elems) || !mul_ok(vocab, dim, table_elems)) return MB_ERR_SHAPE;
    return MB_OK;
}

template <int IN, int OUT, int K> hipError_t conv_bwd_k(mbs::convbwd::Params &p, hipStream_t st) {
    namespace C = mbs::convbwd;
    void *args[] = {&p};
    hipError_t e = hipSuccess;
    const int64_t waves = p.batch * p.dim * p.nseg;
    if (waves > 0)
        e = hipLaunchKernel(reinterpret_cast<const void *>(&C::conv1d_bwd<IN, OUT, K>),
                            dim3((unsigned)((waves + C::kWaves - 1) / C::kWaves)), dim3(C::kThreads), args, 0, st);
    if (e != hipSuccess) return e;
    return hipLaunchKernel(reinterpret_cast<const void *>(&C::conv1d_bwd_finish<K>),
                           dim3((unsigned)((p.dim * (K + 1) + C::kThreads - 1) / C::kThreads)), dim3(C::kThreads), args, 0, st);
}

// Stretches per row: as many as bring the waves to 16 per SIMD.
void conv_bwd_segments(mbs::convbwd::Params &p, int span) {
    const int64_t rows = p.batch * p.dim, tiles = std::max<int64_t>((p.seqlen + 64 * span - 1) / (64 * span), 1);
    const int64_t want = 4 * 256 * 16;
    const int64_t n = std::min(tiles, std::max<int64_t>(1, want / std::max<int64_t>(rows, 1)));
    p.seg_tiles = (int32_t)((tiles + n - 1) / n);
    p.nseg = (tiles + p.seg_tiles - 1) / p.seg_tiles;
}

template <int IN, int OUT> hipError_t conv_bwd_dispatch(mbs::convbwd::Params &p, int K, hipStream_t st) {
    switch (K) {
        case 1: return conv_bwd_k<IN, OUT, 1>(p, st);
        case 2: return conv_bwd_k<IN, OUT, 2>(p, st);
        case 3: return conv_bwd_k<IN, OUT, 3>(p, st);
        default: return conv_bwd_k<IN, OUT, 4>(p, st);
    }
}

// The checks of a list of tensors; *total: their elements.
int list_checks(int64_t count, const void *const *grads, const int64_t *sizes, const int32_t *dtypes, const float *norm) {
    if (count < 0) return MB_ERR_SHAPE;
    if (!norm || (count > 0 && (!grads || !sizes || !dtypes))) return MB_ERR_NULL;
    if (!aligned(norm, 4)) return MB_ERR_ALIGN;
    int64_t total = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (sizes[i] < 0 || sizes[i] > kMaxElems - total) return MB_ERR_SHAPE;
        total += sizes[i];
        if (!valid_dtype(dtypes[i])) return MB_ERR_DTYPE;
        if (sizes[i] > 0 && !grads[i]) return MB_ERR_NULL;
        const size_t e = dtype_size(dtypes[i]);
        if (!aligned(grads[i], e)) return MB_ERR_ALIGN;
        if (overlaps(norm, 4, grads[i], (size_t)sizes[i] * e)) return MB_ERR_ALIAS;
    }
    return MB_OK;
}

// Are the written tensors apart from each other, and, where they are others than the read ones, from those?
int list_alias(int64_t count, const void *const *grads, void *const *out, const int64_t *sizes, const int32_t *dtypes) {
    struct Span { uintptr_t lo, hi; };
    const void *const *written = out ? const_cast<const void *const *>(out) : grads;
    Span *s = static_cast<Span *>(std::malloc(sizeof(Span) * (size_t)std::max<int64_t>(count, 1)));
    if (!s) return MB_ERR_SHAPE;
    int64_t n = 0;
    bool sorted = true;
    for (int64_t i = 0; i < count; ++i) {
        if (sizes[i] == 0) continue;
        const uintptr_t lo = reinterpret_cast<uintptr_t>(written[i]);
        s[n] = {lo, lo + (uintptr_t)sizes[i] * dtype_size(dtypes[i])};
        if (n > 0 && s[n].lo < s[n - 1].lo) sorted = false;
        ++n;
    }
    if (!sorted) std::sort(s, s + n, [](const Span &a, const Span &b) { return a.lo < b.lo; });
    bool bad = false;
    for (int64_t i = 1; i < n; ++i) bad = bad || s[i].lo < s[i - 1].hi;
    for (int64_t i = 0; out && !bad && i < count; ++i) {
        if (sizes[i] == 0) continue;
        const uintptr_t lo = reinterpret_cast<uintptr_t>(grads[i]), hi = lo + (uintptr_t)sizes[i] * dtype_size(dtypes[i]);
        // the written spans are apart, so of those that start below hi the last one ends last
        const Span *after = std::lower_bound(s, s + n, hi, [](const Span &a, uintptr_t v) { return a.lo < v; });
        bad = after != s && (after - 1)->hi > lo;
    }
    std::free(s);
    return bad ? MB_ERR_ALIAS : MB_OK;
}

hipError_t norm_partials(int64_t count, const void *const *grads, const int64_t *sizes, const int32_t *dtypes, double *part,
                         hipStream_t st, int *nparts) {
    namespace C = mbs::clip;
    int first = 1;
    for (int64_t i = 0; i < count; ++i) {
        if (sizes[i] == 0) continue;
        const void *g = grads[i];
        int64_t n = sizes[i];
        void *args[] = {&g, &n, &part, &first};
        const hipError_t e = hipLaunchKernel(dtypes[i] == MB_F32 ? reinterpret_cast<const void *>(&C::sum_squares<0>)
                                                                 : reinterpret_cast<const void *>(&C::sum_squares<1>),
                                             dim3(C::kBlocks), dim3(C::kThreads), args, 0, st);
        if (e != hipSuccess) return e;
        first = 0;
    }
    *nparts = first ? 0 : C::kBlocks;
    return hipSuccess;
}

}  // namespace

extern "C" {

int mb_embedding_fwd(int64_t ntokens, int64_t vocab, int64_t dim, int32_t token_type, int32_t weight_dtype,
                     int32_t out_dtype, float scale, const void *tokens, const void *weight, void *out, void *stream) {
    int64_t row_elems, table_elems;
    const int st = embed_checks(ntokens, vocab, dim, token_type, weight_dtype, out_dtype, &row_elems, &table_elems);
    if (st != MB_OK) return st;
    if (row_elems == 0) return MB_OK;
    if (!tokens || !out || (!weight && table_elems > 0)) return MB_ERR_NULL;
    const size_t tsz = token_size(token_type), wsz = dtype_size(weight_dtype), osz = dtype_size(out_dtype);
    if (!aligned(tokens, tsz) || !aligned(weight, wsz) || !aligned(out, osz)) return MB_ERR_ALIGN;
    const Range outs[] = {{out, (size_t)row_elems * osz}};
    const Range ins[] = {{tokens, (size_t)ntokens * tsz}, {weight, (size_t)table_elems * wsz}};
    if (any_overlap(outs, ins)) return MB_ERR_ALIAS;
    mbs::embed::FwdParams p{ntokens, vocab, dim, tokens, weight, out, scale};
    const void *fn = token_type == MB_TOKEN_U8    ? embed_fwd_fn<0>(weight_dtype, out_dtype)
                     : token_type == MB_TOKEN_I32 ? embed_fwd_fn<1>(weight_dtype, out_dtype)
                                                  : embed_fwd_fn<2>(weight_dtype, out_dtype);
    return status(launch(fn, dim3(blocks_for((row_elems + mbs::embed::kThreads - 1) / mbs::embed::kThreads)),
                         dim3(mbs::embed::kThreads), &p, stream));
}

int mb_embedding_bwd(int64_t ntokens, int64_t vocab, int64_t dim, int32_t token_type, int32_t dy_dtype, int32_t out_dtype,
                     float scale, const void *tokens, const void *dy, void *dweight, void *stream) {
    int64_t row_elems, table_elems;
    const int st = embed_checks(ntokens, vocab, dim, token_type, dy_dtype, out_dtype, &row_elems, &table_elems);
    if (st != MB_OK) return st;
    if (ntokens >= (int64_t(1) << 31)) return MB_ERR_SHAPE;
    if (table_elems == 0) return MB_OK;
    if (!dweight || (ntokens > 0 && (!tokens || !dy))) return MB_ERR_NULL;
    const size_t tsz = token_size(token_type), ysz = dtype_size(dy_dtype), osz = dtype_size(out_dtype);
    if (!aligned(tokens, tsz) || !aligned(dy, ysz) || !aligned(dweight, osz)) return MB_ERR_ALIGN;
    const Range outs[] = {{dweight, (size_t)table_elems * osz}};
    const Range ins[] = {{tokens, (size_t)ntokens * tsz}, {dy, (size_t)row_elems * ysz}};
    if (any_overlap(outs, ins)) return MB_ERR_ALIAS;
    mbs::embed::BwdParams p{ntokens, vocab, dim, tokens, dy, dweight, scale};
    const void *fn = token_type == MB_TOKEN_U8    ? embed_bwd_fn<0>(dy_dtype, out_dtype)
                     : token_type == MB_TOKEN_I32 ? embed_bwd_fn<1>(dy_dtype, out_dtype)
                                                  : embed_bwd_fn<2>(dy_dtype, out_dtype);
    const int64_t tiles = (dim + mbs::embed::kThreads - 1) / mbs::embed::kThreads;
    return status(launch(fn, dim3(blocks_for(vocab * tiles)), dim3(mbs::embed::kThreads), &p, stream));
}

int mb_conv1d_bwd(const mb_conv_desc *desc, const void *x, const float *w, const float *bias, const float *state_in,
                  const void *dy, const float *dstate_out, void *dx, float *dw, float *dbias, float *dstate_in,
                  void *stream) {
    if (!desc) return MB_ERR_NULL;
    const int64_t B = desc->batch, D = desc->dim, L = desc->seqlen, K = desc->width;
    if (B < 0 || D < 0 || L < 0) return MB_ERR_SHAPE;
    if (!valid_dtype(desc->in_dtype) || !valid_dtype(desc->out_dtype)) return MB_ERR_DTYPE;
    if (K < 1 || K > 4 || desc->reserved != 0 || desc->reserved2 != 0) return MB_ERR_UNSUPPORTED;
    int64_t rows, elems, padded;
    if (!mul_ok(B, D, &rows) || !mul_ok(rows, L, &elems) || !mul_ok(rows, K + 1, &padded)) return MB_ERR_SHAPE;
    if (D >= (int64_t(1) << 31) || rows >= (int64_t(1) << 31) || L >= (int64_t(1) << 31)) return MB_ERR_SHAPE;
    if (D == 0) return MB_OK;
    if (!w || !dw || (bias && !dbias)) return MB_ERR_NULL;
    if (elems > 0 && (!x || !dy || !dx)) return MB_ERR_NULL;
    const size_t in_sz = dtype_size(desc->in_dtype), out_sz = dtype_size(desc->out_dtype);
    if (!aligned(x, in_sz) || !aligned(dy, out_sz) || !aligned(dx, out_sz)) return MB_ERR_ALIGN;
    const void *f32s[] = {w, bias, state_in, dstate_out, dw, dbias, dstate_in};
    for (const void *q : f32s)
        if (!aligned(q, 4)) return MB_ERR_ALIGN;
    const size_t w_b = (size_t)(D * K) * 4, b_b = (size_t)D * 4, st_b = (size_t)(rows * (K - 1)) * 4;
    const Range ins[] = {{x, (size_t)elems * in_sz}, {w, w_b}, {bias, b_b}, {state_in, st_b}, {dy, (size_t)elems * out_sz},
                         {dstate_out, st_b}};
    const Range outs[] = {{dx, (size_t)elems * out_sz}, {dw, w_b}, {dbias, bias ? b_b : 0}, {dstate_in, st_b}};
    if (any_overlap(outs, ins)) return MB_ERR_ALIAS;

    hipStream_t st = static_cast<hipStream_t>(stream);
    mbs::convbwd::Params p{};
    p.batch = B; p.dim = D; p.seqlen = L;
    p.x = x; p.w = w; p.bias = bias; p.state_in = state_in; p.dy = dy; p.dstate_out = dstate_out;
    p.dx = dx; p.dw = dw; p.dbias = bias ? dbias : nullptr; p.dstate_in = dstate_in;
    p.apply_silu = desc->apply_silu ? 1 : 0;
    conv_bwd_segments(p, desc->in_dtype == MB_F32 && desc->out_dtype == MB_F32 ? 4 : 8);
    hipError_t e = hipMallocAsync(reinterpret_cast<void **>(&p.part), (size_t)std::max<int64_t>(padded * p.nseg, 1) * 4, st);
    if (e != hipSuccess) return MB_ERR_HIP;
    if (desc->in_dtype == MB_F32)
        e = desc->out_dtype == MB_F32 ? conv_bwd_dispatch<0, 0>(p, (int)K, st) : conv_bwd_dispatch<0, 1>(p, (int)K, st);
    else
        e = desc->out_dtype == MB_F32 ? conv_bwd_dispatch<1, 0>(p, (int)K, st) : conv_bwd_dispatch<1, 1>(p, (int)K, st);
    const hipError_t f = hipFreeAsync(p.part, st);
    return status(e != hipSuccess ? e : f);
}

int mb_grad_norm(int64_t count, const void *const *grads, const int64_t *sizes, const int32_t *dtypes, float *norm,
                 void *stream) {
    namespace C = mbs::clip;
    const int bad = list_checks(count, grads, sizes, dtypes, norm);
    if (bad != MB_OK) return bad;
    hipStream_t st = static_cast<hipStream_t>(stream);
    double *part = nullptr;
    if (hipMallocAsync(reinterpret_cast<void **>(&part), sizeof(double) * C::kBlocks, st) != hipSuccess) return MB_ERR_HIP;
    int nparts = 0;
    hipError_t e = norm_partials(count, grads, sizes, dtypes, part, st, &nparts);
    float zero = 0.0f, *none = nullptr;
    void *args[] = {&part, &nparts, &zero, &zero, &norm, &none};
    if (e == hipSuccess)
        e = hipLaunchKernel(reinterpret_cast<const void *>(&C::finish_norm), dim3(1), dim3(C::kThreads), args, 0, st);
    const hipError_t f = hipFreeAsync(part, st);
    return status(e != hipSuccess ? e : f);
}

int mb_clip_grad_norm(int64_t count, const void *const *grads, void *const *out, const int64_t *sizes,
                      const int32_t *dtypes, float max_norm, float eps, float *norm, void *stream) {
    namespace C = mbs::clip;
    int bad = list_checks(count, grads, sizes, dtypes, norm);
    if (bad != MB_OK) return bad;
    if (!(max_norm >= 0.0f) || !(eps >= 0.0f) || std::isinf(max_norm) || std::isinf(eps)) return MB_ERR_UNSUPPORTED;
    for (int64_t i = 0; out && i < count; ++i) {
        if (sizes[i] > 0 && !out[i]) return MB_ERR_NULL;
        if (!aligned(out[i], dtype_size(dtypes[i]))) return MB_ERR_ALIGN;
        if (overlaps(norm, 4, out[i], (size_t)sizes[i] * dtype_size(dtypes[i]))) return MB_ERR_ALIAS;
    }
    bad = list_alias(count, grads, out, sizes, dtypes);
    if (bad != MB_OK) return bad;
    hipStream_t st = static_cast<hipStream_t>(stream);
    double *part = nullptr;
    if (hipMallocAsync(reinterpret_cast<void **>(&part), sizeof(double) * (C::kBlocks + 1), st) != hipSuccess)
        return MB_ERR_HIP;
    float *factor = reinterpret_cast<float *>(part + C::kBlocks);
    int nparts = 0;
    hipError_t e = norm_partials(count, grads, sizes, dtypes, part, st, &nparts);
    void *args[] = {&part, &nparts, &max_norm, &eps, &norm, &factor};
    if (e == hipSuccess)
        e = hipLaunchKernel(reinterpret_cast<const void *>(&C::finish_norm), dim3(1), dim3(C::kThreads), args, 0, st);
    for (int64_t i = 0; e == hipSuccess && i < count; ++i) {
        if (sizes[i] == 0) continue;
        const void *g = grads[i];
        void *o = out ? out[i] : const_cast<void *>(g);
        int64_t n = sizes[i];
        void *sargs[] = {&g, &o, &n, &factor};
        e = hipLaunchKernel(dtypes[i] == MB_F32 ? reinterpret_cast<const void *>(&C::scale_by<0>)
                                                : reinterpret_cast<const void *>(&C::scale_by<1>),
                            dim3(C::kBlocks), dim3(C::kThreads), sargs, 0, st);
    }
    const hipError_t f = hipFreeAsync(part, st);
    return status(e != hipSuccess ? e : f);
}

int mb_verify_sample(int64_t batch, int64_t ndraft, int64_t vocab, int32_t logit_dtype, float temperature,
                     const void *logits, const void *draft_logits, const int32_t *draft, const int32_t *lengths,
                     const float *uniform, const float *noise, int32_t *accepted, int32_t *last_pos,
                     int32_t *next_token, float *probs, void *stream) {
    if (batch < 0 || ndraft < 0 || vocab < 1) return MB_ERR_SHAPE;
    if (ndraft >= (int64_t(1) << 31) - 1 || vocab >= (int64_t(1) << 31) - 1 || batch >= (int64_t(1) << 31)) return MB_ERR_SHAPE;
    if (!valid_dtype(logit_dtype)) return MB_ERR_DTYPE;
    const float inv_temp = 1.0f / temperature;
    if (!(temperature > 0.0f) || std::isinf(temperature) || std::isinf(inv_temp)) return MB_ERR_UNSUPPORTED;
    int64_t rows, elems, pairs, noises;
    if (!mul_ok(batch, ndraft + 1, &rows) || !mul_ok(rows, vocab, &elems) || !mul_ok(batch, ndraft, &pairs) ||
        !mul_ok(batch, vocab, &noises))
        return MB_ERR_SHAPE;
    if (batch == 0) return MB_OK;
    if (!logits || !noise || !accepted || !next_token || (ndraft > 0 && (!draft || !uniform))) return MB_ERR_NULL;
    const size_t lsz = dtype_size(logit_dtype);
    if (!aligned(logits, lsz) || !aligned(draft_logits, lsz)) return MB_ERR_ALIGN;
    const void *words[] = {draft, lengths, uniform, noise, accepted, last_pos, next_token, probs};
    for (const void *q : words)
        if (!aligned(q, 4)) return MB_ERR_ALIGN;
    const size_t b_b = (size_t)batch * 4, p_b = (size_t)pairs * 4;
    const Range ins[] = {{logits, (size_t)elems * lsz}, {draft_logits, (size_t)(pairs * vocab) * lsz}, {draft, p_b},
                         {lengths, b_b}, {uniform, p_b}, {noise, (size_t)noises * 4}};
    const Range outs[] = {{accepted, b_b}, {last_pos, b_b}, {next_token, b_b}, {probs, p_b}};
    if (any_overlap(outs, ins)) return MB_ERR_ALIAS;
    mbs::sample::Params p{};
    p.batch = batch; p.ndraft = ndraft; p.vocab = vocab;
    p.logits = logits; p.draft_logits = ndraft > 0 ? draft_logits : nullptr; p.draft = draft; p.lengths = lengths;
    p.uniform = uniform; p.noise = noise;
    p.accepted = accepted; p.last_pos = last_pos; p.next_token = next_token; p.probs = probs;
    p.inv_temp = inv_temp;
    const void *fn = logit_dtype == MB_F32 ? reinterpret_cast<const void *>(&mbs::sample::verify_sample<0>)
                                           : reinterpret_cast<const void *>(&mbs::sample::verify_sample<1>);
    return status(launch(fn, dim3((unsigned)batch), dim3(64), &p, stream));
}

}  // extern "C"
