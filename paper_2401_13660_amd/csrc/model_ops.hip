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

int status(hipError_t e) { return e == hipSuccess ? MB_OK : MB_ERR_HIP; }

hipStream_t st_of(void *stream) { return static_cast<hipStream_t>(stream); }

// The caller's workspace, or memory allocated on the stream for the call (`at` null: it could not be).
struct Workspace {
    char *at;
    hipStream_t st;
    bool own;
    Workspace(void *given, size_t bytes, hipStream_t stream) : at(static_cast<char *>(given)), st(stream), own(!given) {
        if (own && hipMallocAsync(reinterpret_cast<void **>(&at), std::max<size_t>(bytes, 16), st) != hipSuccess) at = nullptr;
    }
    hipError_t done(hipError_t e) const {
        const hipError_t f = own ? hipFreeAsync(at, st) : hipSuccess;
        return e != hipSuccess ? e : f;
    }
};

bool valid_token_type(int32_t t) { return t == MB_TOKEN_U8 || t == MB_TOKEN_I32 || t == MB_TOKEN_I64; }
size_t token_size(int32_t t) { return t == MB_TOKEN_U8 ? 1 : t == MB_TOKEN_I32 ? 4 : 8; }

// Elements per lane: 16 bytes of the narrower type, or one where rows are shorter than that.
template <int A, int B> constexpr int kEmbedSpan = A == 0 && B == 0 ? 4 : 8;

template <int TOK, int W, int OUT> const void *embed_fwd_fn(int64_t dim, int64_t *span) {
    constexpr int S = kEmbedSpan<W, OUT>;
    *span = dim < S ? 1 : S;
    return dim < S ? reinterpret_cast<const void *>(&mbs::embed::embed_fwd<TOK, W, OUT, 1>)
                   : reinterpret_cast<const void *>(&mbs::embed::embed_fwd<TOK, W, OUT, S>);
}
template <int TOK> const void *embed_fwd_fn(int32_t in, int32_t out, int64_t dim, int64_t *span) {
    if (in == MB_F32) return out == MB_F32 ? embed_fwd_fn<TOK, 0, 0>(dim, span) : embed_fwd_fn<TOK, 0, 1>(dim, span);
    return out == MB_F32 ? embed_fwd_fn<TOK, 1, 0>(dim, span) : embed_fwd_fn<TOK, 1, 1>(dim, span);
}

// The workspace's areas, each on a 256-byte boundary.
struct Areas {
    size_t bytes = 0;
    size_t add(size_t n) {
        const size_t at = bytes;
        bytes += (n + 255) / 256 * 256;
        return at;
    }
};

// The sort of an embedding's gradient and its workspace.
struct EmbedPlan {
    int64_t tile, tiles, chunk, groups;
    int passes;
    bool merged;                                        // each pass counts the next one's digits
    bool wide;                                          // one pass of kWideBits
    bool direct, by_row;                                // no sort: sum_direct, without a workspace
    int64_t direct_blocks;
    size_t counts, valid, a, b, head, tail, bytes;
    EmbedPlan(int64_t ntokens, int64_t vocab, int64_t dim) {
        namespace E = mbs::embed;
        // few tokens: a workgroup per row of the table or per token, whichever are fewer, where either are few enough
        // (without tokens the rows are as wide: one workgroup counts a row's spans in 32 bits)
        const int64_t cols = (dim + 255) / 256, rows = vocab * cols, places = std::max<int64_t>(ntokens, 1) * cols;
        const bool few = ntokens <= E::kDirectTokens, row_ok = few && rows <= E::kDirectRows;
        const bool place_ok = few && places <= E::kDirectPlaces && vocab <= E::kZeroRows * E::kZeroBlocks;
        const int64_t place_blocks = ntokens * cols + std::min<int64_t>(vocab, E::kZeroBlocks);
        direct = row_ok || place_ok;
        by_row = row_ok && (!place_ok || rows <= place_blocks);
        direct_blocks = by_row ? rows : place_blocks;
        passes = 1;
        while (passes < 4 && (vocab - 1) >> (8 * passes)) ++passes;
        // tokens per workgroup: 1,024, or what keeps the workgroups at kBins (each reads the counts of all)
        tile = std::max<int64_t>(1024, ((ntokens + E::kBins - 1) / E::kBins + 1023) / 1024 * 1024);
        tiles = (ntokens + tile - 1) / tile;
        wide = passes == 2 && vocab <= 1 << E::kWideBits && ntokens > E::kDirectTokens && tiles <= E::kWideTiles;
        if (wide) passes = 1;
        if (!wide && ntokens > 0 && ntokens <= E::kSmallTokens) tiles = 1;  // sorted by one workgroup at once
        // sorted positions per wave: 64, or fewer where that leaves the SIMDs with less than two waves
        chunk = E::kChunk;
        while (chunk > 16 && ntokens / chunk * ((dim + 255) / 256) < 2048) chunk /= 2;
        groups = (ntokens + chunk * E::kWaves - 1) / (chunk * E::kWaves);
        Areas w;
        merged = tiles <= E::kNextTiles;                // tile is kStep then
        counts = w.add((size_t)(merged ? passes : 1) * (size_t)tiles * (wide ? 1 << E::kWideBits : E::kBins) * 4);
        valid = w.add(4);
        a = w.add((size_t)ntokens * sizeof(E::Pair));
        b = w.add(passes > 1 ? (size_t)ntokens * sizeof(E::Pair) : 0);
        head = w.add((size_t)groups * (size_t)dim * 4);
        tail = w.add((size_t)groups * (size_t)dim * 4);
        bytes = direct ? 0 : w.bytes;
    }
    // Do the sums' launches, of 256 and 512 threads per group and tile of columns, have less than 2^32 threads?
    bool launches(int64_t dim) const {
        const int64_t cols = (dim + 255) / 256;
        return direct || (groups * cols < int64_t(1) << 24 && (groups - 1) * cols < int64_t(1) << 23);
    }
};

template <int TOK, int OUT> hipError_t embed_sort(mbs::embed::BwdParams &p, const EmbedPlan &f, char *ws, hipStream_t st) {
    namespace E = mbs::embed;
    E::Pair *const ab[2] = {reinterpret_cast<E::Pair *>(ws + f.a), reinterpret_cast<E::Pair *>(ws + f.b)};
    // the table is set to zero in shares beside the launches of the sort.  A scatter takes twice a count's time and hides more: its
    // share is three times as large.  Equal ones took 44.4 us in all instead of 42.7 (16,384 tokens, 98 MB), 49.7 and 49.2
    // (135 MB), 75.9 and 77.4 (268 MB), 177 and 170 (604 MB); 65,536 tokens 84.2 and 84.7, 91.2 and 89.1, 129 and 130
    constexpr int kBeside = 3;
    const int64_t elems = p.vocab * p.dim;
    const int64_t parts = f.tiles <= 1 ? kBeside : f.passes * kBeside + (f.merged ? 1 : f.passes);
    const dim3 block(E::kThreads);
    int64_t part = 0, zeroing = 0;                      // workgroups of at least 4,096 elements
    dim3 grid;
    p.zero_from = p.zero_to = 0;
    auto next_share = [&](int weight) {
        part += weight;
        p.zero_from = p.zero_to;
        p.zero_to = part == parts ? elems : std::min(elems, elems / parts * part / 64 * 64);    // the stores stay aligned
        zeroing = std::min<int64_t>((p.zero_to - p.zero_from + 4095) / 4096, 2048);
        grid = dim3((unsigned)(f.tiles + zeroing));
    };
    void *args[] = {&p};
    if (f.tiles <= 1) {
        next_share(kBeside);
        p.to = ab[0];
        p.tiles = 1;
        // 256 threads where they do: fewer waves' counts to add up.  The larger workgroups zero four times as much each
        const bool quarter = p.ntokens <= E::kThreads * E::kSmallPlaces;
        const unsigned blocks = 1 + (unsigned)(quarter ? zeroing : (zeroing + 3) / 4);
        return hipLaunchKernel(quarter ? reinterpret_cast<const void *>(&E::sort_small<TOK, OUT, E::kThreads>)
                                       : reinterpret_cast<const void *>(&E::sort_small<TOK, OUT, E::kSmallThreads>),
                               dim3(blocks), dim3(quarter ? E::kThreads : E::kSmallThreads), args, 0, st);
    }
    for (int k = 0; k < f.passes; ++k) {
        const bool first = k == 0, next = f.merged && k + 1 < f.passes;
        uint32_t *const all = reinterpret_cast<uint32_t *>(ws + f.counts);
        p.shift = 8 * k;
        p.from = first ? nullptr : ab[(k - 1) & 1];
        p.to = ab[k & 1];
        p.counts = all + (f.merged ? (int64_t)k * f.tiles * E::kBins : 0);
        p.next_counts = next ? p.counts + f.tiles * E::kBins : nullptr;
        p.ahead = first && f.merged ? f.passes - 1 : 0;
        hipError_t e = hipSuccess;
        if (first || !f.merged) {
            next_share(1);
            // keys of later passes are no tokens: one instantiation for all token types
            e = hipLaunchKernel(f.wide  ? reinterpret_cast<const void *>(&E::count_digits<TOK, OUT, true, E::kWideBits>)
                                : first ? reinterpret_cast<const void *>(&E::count_digits<TOK, OUT, true, 8>)
                                        : reinterpret_cast<const void *>(&E::count_digits<0, OUT, false, 8>),
                                grid, block, args, 0, st);
            if (e != hipSuccess) return e;
        }
        next_share(kBeside);
        const void *fn = f.wide  ? reinterpret_cast<const void *>(&E::scatter<TOK, OUT, true, false, E::kWideBits>)
                         : first ? next ? reinterpret_cast<const void *>(&E::scatter<TOK, OUT, true, true, 8>)
                                        : reinterpret_cast<const void *>(&E::scatter<TOK, OUT, true, false, 8>)
                         : next  ? reinterpret_cast<const void *>(&E::scatter<0, OUT, false, true, 8>)
                                 : reinterpret_cast<const void *>(&E::scatter<0, OUT, false, false, 8>);
        e = hipLaunchKernel(fn, grid, block, args, 0, st);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <int DY, int OUT, int S> hipError_t embed_sum(mbs::embed::BwdParams &p, const EmbedPlan &f, hipStream_t st) {
    namespace E = mbs::embed;
    uint32_t cols = (uint32_t)((p.dim + 64 * S - 1) / (64 * S));
    void *args[] = {&p, &cols};
    hipError_t e = hipLaunchKernel(reinterpret_cast<const void *>(&E::sum_chunks<DY, OUT, S>),
                                   dim3((unsigned)(f.groups * cols)), dim3(E::kThreads), args, 0, st);
    if (e != hipSuccess || f.groups < 2) return e;
    constexpr int J = S == 1 ? 1 : 4;                               // the sums are fp32
    cols = (uint32_t)((p.dim + 64 * J - 1) / (64 * J));
    return hipLaunchKernel(reinterpret_cast<const void *>(&E::join_groups<OUT, J>), dim3((unsigned)((f.groups - 1) * cols)),
                           dim3(64 * E::kJoinWaves), args, 0, st);
}
template <int DY, int OUT> hipError_t embed_sum(mbs::embed::BwdParams &p, const EmbedPlan &f, hipStream_t st) {
    constexpr int S = DY == 1 ? 8 : 4;
    return p.dim < S ? embed_sum<DY, OUT, 1>(p, f, st) : embed_sum<DY, OUT, S>(p, f, st);
}

template <int TOK, int DY, int OUT> hipError_t embed_direct(mbs::embed::BwdParams &p, const EmbedPlan &f, hipStream_t st) {
    namespace E = mbs::embed;
    uint32_t cols = (uint32_t)((p.dim + 255) / 256);
    const void *fn = p.dim < 4  ? f.by_row ? reinterpret_cast<const void *>(&E::sum_direct<TOK, DY, OUT, 1, true>)
                                           : reinterpret_cast<const void *>(&E::sum_direct<TOK, DY, OUT, 1, false>)
                     : f.by_row ? reinterpret_cast<const void *>(&E::sum_direct<TOK, DY, OUT, 4, true>)
                                : reinterpret_cast<const void *>(&E::sum_direct<TOK, DY, OUT, 4, false>);
    void *args[] = {&p, &cols};
    return hipLaunchKernel(fn, dim3((unsigned)f.direct_blocks), dim3(64 * E::kDirectWaves), args, 0, st);
}
template <int DY, int OUT> hipError_t embed_direct(mbs::embed::BwdParams &p, const EmbedPlan &f, int32_t token_type, hipStream_t st) {
    return token_type == MB_TOKEN_U8    ? embed_direct<0, DY, OUT>(p, f, st)
           : token_type == MB_TOKEN_I32 ? embed_direct<1, DY, OUT>(p, f, st)
                                        : embed_direct<2, DY, OUT>(p, f, st);
}

template <int OUT> hipError_t embed_bwd(mbs::embed::BwdParams &p, const EmbedPlan &f, int32_t token_type, int32_t dy_dtype,
                                        char *ws, hipStream_t st) {
    if (f.direct) return dy_dtype == MB_F32 ? embed_direct<0, OUT>(p, f, token_type, st) : embed_direct<1, OUT>(p, f, token_type, st);
    const hipError_t e = token_type == MB_TOKEN_U8    ? embed_sort<0, OUT>(p, f, ws, st)
                         : token_type == MB_TOKEN_I32 ? embed_sort<1, OUT>(p, f, ws, st)
                                                      : embed_sort<2, OUT>(p, f, ws, st);
    if (e != hipSuccess || f.tiles == 0) return e;
    return dy_dtype == MB_F32 ? embed_sum<0, OUT>(p, f, st) : embed_sum<1, OUT>(p, f, st);
}

// The pieces of a large vocabulary's rows; none for a small one's.
struct SamplePlan {
    int64_t pieces = 0, race_pieces = 0, blocks = 0;
    size_t stats = 0, best = 0, bytes = 0;
    SamplePlan(int64_t batch, int64_t ndraft, int64_t vocab) {
        namespace S = mbs::sample;
        if (vocab <= S::kSmallVocab) return;
        pieces = (vocab + S::kPiece - 1) / S::kPiece;
        race_pieces = (vocab + S::kRacePiece - 1) / S::kRacePiece;
        blocks = batch * (2 * ndraft + 1) * pieces;
        Areas w;
        stats = w.add((size_t)blocks * sizeof(float2));
        best = w.add((size_t)(batch * race_pieces) * sizeof(S::Best));
        bytes = w.bytes;
    }
};

// The checks of its sizes, for the call and for its workspace.  Row and token numbers, and a last piece's tokens past the
// vocabulary, stay below 2^31, and a launch has less than 2^32 threads.
bool sample_sizes(int64_t batch, int64_t ndraft, int64_t vocab) {
    constexpr int64_t most = int64_t(1) << 31;
    if (batch < 0 || ndraft < 0 || vocab < 1) return false;
    if (batch >= most || ndraft >= most - mbs::sample::kMaxWaves || vocab >= most - mbs::sample::kPiece) return false;
    int64_t rows, elems;
    if (!mul_ok(batch, ndraft + 1, &rows) || !mul_ok(rows, vocab, &elems)) return false;
    if (vocab <= mbs::sample::kSmallVocab) return batch < most / (32 * mbs::sample::kMaxWaves);
    const SamplePlan f(batch, ndraft, vocab);
    return f.blocks < (int64_t(1) << 23) && batch * f.race_pieces < (int64_t(1) << 23);
}

template <int DT> hipError_t sample_launch(mbs::sample::Params &p, const SamplePlan &f, void *workspace, hipStream_t st) {
    namespace S = mbs::sample;
    void *args[] = {&p};
    if (f.pieces == 0) {
        // a wave per row, the row after the drafts included
        const int waves = (int)std::min<int64_t>(p.ndraft + 1, S::kMaxWaves);
        const void *fn = p.vocab <= 256 ? reinterpret_cast<const void *>(&S::verify_small<DT, 4>)
                                        : reinterpret_cast<const void *>(&S::verify_small<DT, 16>);
        return hipLaunchKernel(fn, dim3((unsigned)p.batch), dim3(64 * waves), args, 0, st);
    }
    Workspace ws(workspace, f.bytes, st);
    if (!ws.at) return hipErrorOutOfMemory;
    p.pieces = (int32_t)f.pieces;
    p.race_pieces = (int32_t)f.race_pieces;
    p.stats = reinterpret_cast<float2 *>(ws.at + f.stats);
    p.best = reinterpret_cast<S::Best *>(ws.at + f.best);
    // without the drafter's logits its rows' workgroups end at once
    hipError_t e = hipLaunchKernel(reinterpret_cast<const void *>(&S::piece_stats<DT>), dim3((unsigned)f.blocks),
                                   dim3(S::kThreads), args, 0, st);
    if (e == hipSuccess)
        e = hipLaunchKernel(reinterpret_cast<const void *>(&S::decide_and_race<DT>), dim3((unsigned)(p.batch * f.race_pieces)),
                            dim3(S::kThreads), args, 0, st);
    if (e == hipSuccess)
        e = hipLaunchKernel(reinterpret_cast<const void *>(&S::join_races), dim3((unsigned)p.batch), dim3(64), args, 0, st);
    return ws.done(e);
}

// The checks that both directions share; the element counts of the tokens' and the table's rows.
int embed_checks(int64_t ntokens, int64_t vocab, int64_t dim, int32_t token_type, int32_t in_dtype, int32_t out_dtype,
                 int64_t *row_elems, int64_t *table_elems) {
    if (ntokens < 0 || vocab < 0 || dim < 0 || vocab >= (int64_t(1) << 31)) return MB_ERR_SHAPE;
    if (!valid_token_type(token_type) || !valid_dtype(in_dtype) || !valid_dtype(out_dtype)) return MB_ERR_DTYPE;
    if (ntokens >= kMaxElems || !mul_ok(ntokens, dim, row_elems) || !mul_ok(vocab, dim, table_elems)) return MB_ERR_SHAPE;
    return MB_OK;
}

// Those of the gradient alone, before its plan is made.
int embed_bwd_checks(int64_t ntokens, int64_t vocab, int64_t dim, int32_t token_type, int32_t dy_dtype, int32_t out_dtype,
                     int64_t *row_elems, int64_t *table_elems) {
    const int st = embed_checks(ntokens, vocab, dim, token_type, dy_dtype, out_dtype, row_elems, table_elems);
    if (st != MB_OK) return st;
    if (ntokens >= (int64_t(1) << 31)) return MB_ERR_SHAPE;
    return *table_elems == 0 || EmbedPlan(ntokens, vocab, dim).launches(dim) ? MB_OK : MB_ERR_SHAPE;
}

template <int IN, int OUT, int K> hipError_t conv_bwd_k(mbs::convbwd::Params &p, hipStream_t st) {
    namespace C = mbs::convbwd;
    void *args[] = {&p};
    hipError_t e = hipSuccess;
    constexpr int S = C::kSpan<IN, OUT>;
    const int64_t rows = p.batch * p.dim, spans = (p.seqlen + S - 1) / S;
    // rows of one tile need no walk, and up to 32 (16) spans two (four) of them share a wave
    const int64_t lanes = spans == 0 || spans > 32 ? 64 : spans > 16 ? 32 : 16, waves = (rows * p.nseg * lanes + 63) / 64;
    const void *walk = p.seqlen % S ? reinterpret_cast<const void *>(&C::conv1d_bwd<IN, OUT, K, true>)
                                    : reinterpret_cast<const void *>(&C::conv1d_bwd<IN, OUT, K, false>);
    const void *fn = spans == 0 || spans > 64 ? walk
                     : lanes == 64            ? reinterpret_cast<const void *>(&C::conv1d_bwd_short<IN, OUT, K, 64>)
                     : lanes == 32            ? reinterpret_cast<const void *>(&C::conv1d_bwd_short<IN, OUT, K, 32>)
                                              : reinterpret_cast<const void *>(&C::conv1d_bwd_short<IN, OUT, K, 16>);
    if (waves > 0)
        e = hipLaunchKernel(fn, dim3((unsigned)((waves + C::kWaves - 1) / C::kWaves)), dim3(C::kThreads), args, 0, st);
    if (e != hipSuccess || (waves > 0 && !p.part)) return e;
    return hipLaunchKernel(reinterpret_cast<const void *>(&C::conv1d_bwd_finish<K>),
                           dim3((unsigned)((p.dim * (K + 1) + C::kThreads - 1) / C::kThreads)), dim3(C::kThreads), args, 0, st);
}

// Stretches per row: enough for 4 waves per SIMD.  (2, 1536, 1021) fp32 in one, two and four stretches per row took 13.6,
// 11.7 and 13.6 us, (1, 2048, 2047) in two, four and eight 14.7, 16.6 and 18.1 (with the finish): more waves hide more
// latency, but each computes its edge again and leaves partial sums.  One sequence in one stretch needs no finish (up to 4
// tiles, or one wave per SIMD for each 4 of them): (1, 3584, 1021) fp32 10.1 us instead of 12.4 in two stretches, (1, 512, 1021)
// 5.6 and 6.6, (1, 2048, 2048) 11.8 and 12.5; beyond, (1, 64, 2048) 7.6 and 5.3, (1, 1024, 4096) 19.2 and 13.8.
void conv_bwd_segments(mbs::convbwd::Params &p, int32_t in_dtype, int32_t out_dtype) {
    const int64_t span = in_dtype == MB_F32 && out_dtype == MB_F32 ? 4 : 8;
    const int64_t rows = p.batch * p.dim, tiles = std::max<int64_t>((p.seqlen + 64 * span - 1) / (64 * span), 1);
    const int64_t want = 4 * 256 * 4;
    const bool whole = p.batch == 1 && (tiles <= 4 || tiles * 256 <= rows);
    const int64_t n = whole ? 1 : std::min(tiles, (want + rows - 1) / std::max<int64_t>(rows, 1));
    p.seg_tiles = (int32_t)((tiles + n - 1) / std::max<int64_t>(n, 1));
    p.nseg = (tiles + p.seg_tiles - 1) / p.seg_tiles;
}

// The workspace: the stretches' sums, none where a row's one stretch has the channel's sums.
int64_t conv_bwd_bytes(const mbs::convbwd::Params &p, int64_t K) {
    return p.batch * p.nseg == 1 ? 0 : p.batch * p.dim * (K + 1) * p.nseg * 4;
}

// The checks of its sizes and types, for the call and for its workspace.  p: the sizes and stretches.
int conv_bwd_checks(const mb_conv_desc *desc, mbs::convbwd::Params &p, int64_t *elems) {
    if (!desc) return MB_ERR_NULL;
    const int64_t B = desc->batch, D = desc->dim, L = desc->seqlen, K = desc->width;
    if (B < 0 || D < 0 || L < 0) return MB_ERR_SHAPE;
    if (!valid_dtype(desc->in_dtype) || !valid_dtype(desc->out_dtype)) return MB_ERR_DTYPE;
    if (K < 1 || K > 4 || desc->reserved != 0 || desc->reserved2 != 0) return MB_ERR_UNSUPPORTED;
    int64_t rows, padded;
    if (!mul_ok(B, D, &rows) || !mul_ok(rows, L, elems) || !mul_ok(rows, K + 1, &padded)) return MB_ERR_SHAPE;
    if (D >= (int64_t(1) << 31) || rows >= (int64_t(1) << 31) || L >= (int64_t(1) << 31)) return MB_ERR_SHAPE;
    p.batch = B; p.dim = D; p.seqlen = L;
    conv_bwd_segments(p, desc->in_dtype, desc->out_dtype);
    // a wave per row and stretch, a thread per sum, and less than 2^32 threads in a launch
    return rows * p.nseg >= (int64_t(1) << 26) || D * (K + 1) >= int64_t(255) << 24 ? MB_ERR_SHAPE : MB_OK;
}

template <int IN, int OUT> hipError_t conv_bwd_dispatch(mbs::convbwd::Params &p, int K, hipStream_t st) {
    switch (K) {
        case 1: return conv_bwd_k<IN, OUT, 1>(p, st);
        case 2: return conv_bwd_k<IN, OUT, 2>(p, st);
        case 3: return conv_bwd_k<IN, OUT, 3>(p, st);
        default: return conv_bwd_k<IN, OUT, 4>(p, st);
    }
}

hipError_t conv_bwd_launch(mbs::convbwd::Params &p, const mb_conv_desc *desc, hipStream_t st) {
    if (desc->in_dtype == MB_F32)
        return desc->out_dtype == MB_F32 ? conv_bwd_dispatch<0, 0>(p, desc->width, st) : conv_bwd_dispatch<0, 1>(p, desc->width, st);
    return desc->out_dtype == MB_F32 ? conv_bwd_dispatch<1, 0>(p, desc->width, st) : conv_bwd_dispatch<1, 1>(p, desc->width, st);
}

// Partial sums, and the list where it does not fit the kernels' arguments.
size_t clip_workspace(int64_t count) {
    namespace C = mbs::clip;
    return sizeof(double) * C::kBlocks + (count <= C::kInline ? 0 : sizeof(C::Entry) * (size_t)count);
}

// The checks of a list of tensors.
int list_checks(int64_t count, const void *const *grads, const int64_t *sizes, const int32_t *dtypes, const float *norm,
                const void *workspace) {
    if (count < 0 || count >= (int64_t(1) << 31)) return MB_ERR_SHAPE;
    if (!norm || (count > 0 && (!grads || !sizes || !dtypes))) return MB_ERR_NULL;
    if (!aligned(norm, 4) || !aligned(workspace, 16)) return MB_ERR_ALIGN;
    const size_t ws_b = workspace ? clip_workspace(count) : 0;
    if (overlaps(norm, 4, workspace, ws_b)) return MB_ERR_ALIAS;
    int64_t total = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (sizes[i] < 0 || sizes[i] > kMaxElems - total) return MB_ERR_SHAPE;
        total += sizes[i];
        if (!valid_dtype(dtypes[i])) return MB_ERR_DTYPE;
        if (sizes[i] > 0 && !grads[i]) return MB_ERR_NULL;
        const size_t e = dtype_size(dtypes[i]);
        if (!aligned(grads[i], e)) return MB_ERR_ALIGN;
        if (overlaps(norm, 4, grads[i], (size_t)sizes[i] * e) || overlaps(workspace, ws_b, grads[i], (size_t)sizes[i] * e))
            return MB_ERR_ALIAS;
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

// The norm of a list and, where `scaled`, its clipping.
int norm_and_clip(int64_t count, const void *const *grads, void *const *out, const int64_t *sizes, const int32_t *dtypes,
                  bool scaled, float max_norm, float eps, float *norm, void *workspace, hipStream_t st) {
    namespace C = mbs::clip;
    int64_t used = 0, units = 0, bytes = 0;
    for (int64_t i = 0; i < count; ++i) {
        if (sizes[i] == 0) continue;
        bytes += sizes[i] * (int64_t)dtype_size(dtypes[i]);
        units += (sizes[i] + C::lead(grads[i], dtypes[i]) + C::kUnit - 1) / C::kUnit;
        ++used;
        if (units >= (int64_t(1) << 31) || used >= (int64_t(1) << 31)) return MB_ERR_SHAPE;
    }
    // the entries of the tensors from *i on, at most n of them, empty ones left out
    int64_t next = 0;
    uint32_t unit = 0;
    auto entries = [&](C::Entry *e, int n) {
        int k = 0;
        for (; next < count && k < n; ++next) {
            if (sizes[next] == 0) continue;
            const void *g = grads[next];
            e[k++] = {g, out ? out[next] : const_cast<void *>(g), sizes[next], unit, dtypes[next]};
            unit += (uint32_t)((sizes[next] + C::lead(g, dtypes[next]) + C::kUnit - 1) / C::kUnit);
        }
        return k;
    };
    const bool inlined = used <= C::kInline;
    Workspace ws(workspace, clip_workspace(used), st);
    if (!ws.at) return MB_ERR_HIP;
    hipError_t e = hipSuccess;
    C::Params p{};
    p.count = (int32_t)used;
    p.units = (uint32_t)units;
    p.part = reinterpret_cast<double *>(ws.at);
    p.norm = norm;
    p.max_norm = max_norm;
    p.eps = eps;
    const dim3 grid((unsigned)std::min<int64_t>(std::max<int64_t>(units, 1), C::kBlocks)), block(C::kThreads);
    // kCached bytes in units of the list's mean size, for each workgroup
    p.cached = (uint32_t)(scaled ? C::kCached / (std::max<int64_t>(bytes / std::max<int64_t>(units, 1), 1) * grid.x) : 0);
    C::Table<C::kInline> small{};
    void *args[] = {&p, &small};
    if (inlined) {
        entries(small.e, C::kInline);
    } else {
        C::Entry *table = reinterpret_cast<C::Entry *>(ws.at + sizeof(double) * C::kBlocks);
        p.table = table;
        while (e == hipSuccess && next < count) {
            C::Table<C::kFill> some{};
            int n = entries(some.e, C::kFill);
            void *fargs[] = {&some, &n, &table};
            if (n > 0)
                e = hipLaunchKernel(reinterpret_cast<const void *>(&C::fill_table), dim3(1), dim3(128), fargs, 0, st);
            table += n;
        }
    }
    if (e == hipSuccess)
        e = hipLaunchKernel(inlined ? reinterpret_cast<const void *>(&C::sum_squares_inline)
                                    : reinterpret_cast<const void *>(&C::sum_squares), grid, block, args, 0, st);
    if (e == hipSuccess && scaled)
        e = hipLaunchKernel(inlined ? reinterpret_cast<const void *>(&C::scale_inline)
                                    : reinterpret_cast<const void *>(&C::scale), grid, block, args, 0, st);
    if (e == hipSuccess && !scaled) {
        int nparts = (int)grid.x;
        void *nargs[] = {&p, &nparts};
        e = hipLaunchKernel(reinterpret_cast<const void *>(&C::finish_norm), dim3(1), block, nargs, 0, st);
    }
    return status(ws.done(e));
}

}  // namespace

extern "C" {

int mb_embedding_fwd(int64_t ntokens, int64_t vocab, int64_t dim, int32_t token_type, int32_t weight_dtype,
                     int32_t out_dtype, float scale, const void *tokens, const void *weight, void *out, void *stream) {
    int64_t row_elems, table_elems;
    const int st = embed_checks(ntokens, vocab, dim, token_type, weight_dtype, out_dtype, &row_elems, &table_elems);
    if (st != MB_OK) return st;
    if (row_elems == 0) return MB_OK;
    if (vocab == 0) return MB_ERR_SHAPE;                            // tokens, and no table to look them up in
    if (!tokens || !out || !weight) return MB_ERR_NULL;
    const size_t tsz = token_size(token_type), wsz = dtype_size(weight_dtype), osz = dtype_size(out_dtype);
    if (!aligned(tokens, tsz) || !aligned(weight, wsz) || !aligned(out, osz)) return MB_ERR_ALIGN;
    const Range outs[] = {{out, (size_t)row_elems * osz}};
    const Range ins[] = {{tokens, (size_t)ntokens * tsz}, {weight, (size_t)table_elems * wsz}};
    if (any_overlap(outs, ins)) return MB_ERR_ALIAS;
    int64_t span;
    const void *fn = token_type == MB_TOKEN_U8    ? embed_fwd_fn<0>(weight_dtype, out_dtype, dim, &span)
                     : token_type == MB_TOKEN_I32 ? embed_fwd_fn<1>(weight_dtype, out_dtype, dim, &span)
                                                  : embed_fwd_fn<2>(weight_dtype, out_dtype, dim, &span);
    // spans of a row, and rows per workgroup: 1,024 spans where that leaves 2,048 workgroups
    const int64_t spans = (dim + span - 1) / span;
    const int64_t rows = std::max<int64_t>(1, std::min(1024 / spans, ntokens / 2048));
    const int64_t blocks = std::min<int64_t>((ntokens + rows - 1) / rows, 1 << 20);
    if (spans >= (int64_t(1) << 30)) return MB_ERR_SHAPE;
    mbs::embed::FwdParams p{ntokens, vocab, dim, tokens, weight, out, scale, (int32_t)rows};
    return status(launch(fn, dim3((unsigned)blocks), dim3(mbs::embed::kThreads), &p, stream));
}

int mb_embedding_bwd(int64_t ntokens, int64_t vocab, int64_t dim, int32_t token_type, int32_t dy_dtype, int32_t out_dtype,
                     float scale, const void *tokens, const void *dy, void *dweight, void *workspace, void *stream) {
    int64_t row_elems, table_elems;
    const int st = embed_bwd_checks(ntokens, vocab, dim, token_type, dy_dtype, out_dtype, &row_elems, &table_elems);
    if (st != MB_OK) return st;
    if (table_elems == 0) return MB_OK;
    if (!dweight || (ntokens > 0 && (!tokens || !dy))) return MB_ERR_NULL;
    const size_t tsz = token_size(token_type), ysz = dtype_size(dy_dtype), osz = dtype_size(out_dtype);
    if (!aligned(tokens, tsz) || !aligned(dy, ysz) || !aligned(dweight, osz)) return MB_ERR_ALIGN;
    if (!aligned(workspace, 16)) return MB_ERR_ALIGN;
    const EmbedPlan f(ntokens, vocab, dim);
    const Range outs[] = {{dweight, (size_t)table_elems * osz},
                          {workspace, workspace ? std::max<size_t>(f.bytes, 16) : 0}};
    const Range ins[] = {{tokens, (size_t)ntokens * tsz}, {dy, (size_t)row_elems * ysz}};
    if (any_overlap(outs, ins)) return MB_ERR_ALIAS;
    mbs::embed::BwdParams p{};
    p.ntokens = ntokens; p.vocab = vocab; p.dim = dim;
    p.tokens = tokens; p.dy = dy; p.dweight = dweight; p.scale = scale;
    if (f.direct)
        return status(out_dtype == MB_F32 ? embed_bwd<0>(p, f, token_type, dy_dtype, nullptr, st_of(stream))
                                          : embed_bwd<1>(p, f, token_type, dy_dtype, nullptr, st_of(stream)));
    Workspace ws(workspace, f.bytes, st_of(stream));
    if (!ws.at) return MB_ERR_HIP;
    p.passes = f.passes;
    p.tile = (int32_t)f.tile; p.tiles = (int32_t)f.tiles; p.chunk = (int32_t)f.chunk;
    p.valid = reinterpret_cast<uint32_t *>(ws.at + f.valid);
    p.head = reinterpret_cast<float *>(ws.at + f.head);
    p.tail = reinterpret_cast<float *>(ws.at + f.tail);
    const hipError_t e = out_dtype == MB_F32 ? embed_bwd<0>(p, f, token_type, dy_dtype, ws.at, st_of(stream))
                                             : embed_bwd<1>(p, f, token_type, dy_dtype, ws.at, st_of(stream));
    return status(ws.done(e));
}

int64_t mb_embedding_bwd_workspace(int64_t ntokens, int64_t vocab, int64_t dim) {
    int64_t row_elems, table_elems;
    const int st = embed_bwd_checks(ntokens, vocab, dim, MB_TOKEN_U8, MB_F32, MB_F32, &row_elems, &table_elems);
    if (st != MB_OK) return st;
    return table_elems == 0 ? 0 : (int64_t)EmbedPlan(ntokens, vocab, dim).bytes;
}

int mb_conv1d_bwd(const mb_conv_desc *desc, const void *x, const float *w, const float *bias, const float *state_in,
                  const void *dy, const float *dstate_out, void *dx, float *dw, float *dbias, float *dstate_in,
                  void *workspace, void *stream) {
    mbs::convbwd::Params p{};
    int64_t elems;
    const int bad = conv_bwd_checks(desc, p, &elems);
    if (bad != MB_OK) return bad;
    const int64_t D = p.dim, K = desc->width, rows = p.batch * D;
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
    const size_t part_b = (size_t)conv_bwd_bytes(p, K);
    if (!aligned(workspace, 16)) return MB_ERR_ALIGN;
    const Range outs[] = {{dx, (size_t)elems * out_sz}, {dw, w_b}, {dbias, bias ? b_b : 0}, {dstate_in, st_b},
                          {workspace, workspace ? std::max<size_t>(part_b, 16) : 0}};
    if (any_overlap(outs, ins)) return MB_ERR_ALIAS;

    p.x = x; p.w = w; p.bias = bias; p.state_in = state_in; p.dy = dy; p.dstate_out = dstate_out;
    p.dx = dx; p.dw = dw; p.dbias = bias ? dbias : nullptr; p.dstate_in = dstate_in;
    p.apply_silu = desc->apply_silu ? 1 : 0;
    if (part_b == 0) return status(conv_bwd_launch(p, desc, st_of(stream)));
    Workspace ws(workspace, part_b, st_of(stream));
    if (!ws.at) return MB_ERR_HIP;
    p.part = reinterpret_cast<float *>(ws.at);
    return status(ws.done(conv_bwd_launch(p, desc, ws.st)));
}

int64_t mb_conv1d_bwd_workspace(const mb_conv_desc *desc) {
    mbs::convbwd::Params p{};
    int64_t elems;
    const int bad = conv_bwd_checks(desc, p, &elems);
    return bad != MB_OK ? bad : conv_bwd_bytes(p, desc->width);
}

int mb_grad_norm(int64_t count, const void *const *grads, const int64_t *sizes, const int32_t *dtypes, float *norm,
                 void *workspace, void *stream) {
    const int bad = list_checks(count, grads, sizes, dtypes, norm, workspace);
    if (bad != MB_OK) return bad;
    return norm_and_clip(count, grads, nullptr, sizes, dtypes, false, 0.0f, 0.0f, norm, workspace, st_of(stream));
}

int64_t mb_grad_norm_workspace(int64_t count) {
    return count < 0 || count >= (int64_t(1) << 31) ? MB_ERR_SHAPE : (int64_t)clip_workspace(count);
}

int mb_clip_grad_norm(int64_t count, const void *const *grads, void *const *out, const int64_t *sizes,
                      const int32_t *dtypes, float max_norm, float eps, float *norm, void *workspace,
                      void *stream) {
    int bad = list_checks(count, grads, sizes, dtypes, norm, workspace);
    if (bad != MB_OK) return bad;
    if (!(max_norm >= 0.0f) || !(eps >= 0.0f) || std::isinf(max_norm) || std::isinf(eps)) return MB_ERR_UNSUPPORTED;
    for (int64_t i = 0; out && i < count; ++i) {
        if (sizes[i] > 0 && !out[i]) return MB_ERR_NULL;
        if (!aligned(out[i], dtype_size(dtypes[i]))) return MB_ERR_ALIGN;
        const size_t bytes = (size_t)sizes[i] * dtype_size(dtypes[i]);
        if (overlaps(norm, 4, out[i], bytes) || (workspace && overlaps(workspace, clip_workspace(count), out[i], bytes)))
            return MB_ERR_ALIAS;
    }
    bad = list_alias(count, grads, out, sizes, dtypes);
    if (bad != MB_OK) return bad;
    return norm_and_clip(count, grads, out, sizes, dtypes, true, max_norm, eps, norm, workspace, st_of(stream));
}

int mb_verify_sample(int64_t batch, int64_t ndraft, int64_t vocab, int32_t logit_dtype, float temperature,
                     const void *logits, const void *draft_logits, const int32_t *draft, const int32_t *lengths,
                     const float *uniform, const float *noise, int32_t *accepted, int32_t *last_pos,
                     int32_t *next_token, float *probs, void *workspace, void *stream) {
    if (!sample_sizes(batch, ndraft, vocab)) return MB_ERR_SHAPE;
    if (!valid_dtype(logit_dtype)) return MB_ERR_DTYPE;
    const float inv_temp = 1.0f / temperature;
    if (!(temperature > 0.0f) || std::isinf(temperature) || std::isinf(inv_temp)) return MB_ERR_UNSUPPORTED;
    const int64_t elems = batch * (ndraft + 1) * vocab, pairs = batch * ndraft, noises = batch * vocab;
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
    const SamplePlan f(batch, ndraft, vocab);
    if (!aligned(workspace, 16)) return MB_ERR_ALIGN;
    const Range outs[] = {{accepted, b_b}, {last_pos, b_b}, {next_token, b_b}, {probs, p_b}, {workspace, f.bytes}};
    if (any_overlap(outs, ins)) return MB_ERR_ALIAS;
    mbs::sample::Params p{};
    p.batch = batch; p.ndraft = ndraft; p.vocab = vocab;
    p.logits = logits; p.draft_logits = ndraft > 0 ? draft_logits : nullptr; p.draft = draft; p.lengths = lengths;
    p.uniform = uniform; p.noise = noise;
    p.accepted = accepted; p.last_pos = last_pos; p.next_token = next_token; p.probs = probs;
    p.inv_temp = inv_temp;
    return status(logit_dtype == MB_F32 ? sample_launch<0>(p, f, workspace, st_of(stream))
                                        : sample_launch<1>(p, f, workspace, st_of(stream)));
}

int64_t mb_verify_sample_workspace(int64_t batch, int64_t ndraft, int64_t vocab) {
    return sample_sizes(batch, ndraft, vocab) ? (int64_t)SamplePlan(batch, ndraft, vocab).bytes : (int64_t)MB_ERR_SHAPE;
}

}  // extern "C"
