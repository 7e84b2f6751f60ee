// block_ops.hip -- the C ABI of what lies between a model's scans and after its last layer: the
// norm with the residual's addition and its gradient, matrices in 8 bits and their products, and the choice of the
// next token.  Argument checks and kernel dispatch; the contract is in include/mbscan.h.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "abi_checks.hpp"
#include "fp8_matmul.hpp"
#include "fp8_quant.hpp"
#include "mbscan.h"
#include "rms_norm.hpp"
#include "token_sample.hpp"

namespace {

using namespace mbs::abi;

int64_t blocks_of(int64_t n) { return n / mbs::fp8::kBlock + (n % mbs::fp8::kBlock != 0); }

// ---- norm -----------------------------------------------------------------------

// Waves per row and spans per lane for a row of this width, whole spans where it is made of them; a walk past the widest.
template <int X, int RES, int OUT> const void *norm_fn(int64_t dim, int *waves) {
    namespace N = mbs::norm;
    const int64_t spans = (dim + 7) / 8;
    const bool cut = dim % 8 != 0;
    *waves = 4;
    // to 8 bits, 4 waves instead of one: 32 rows of 1,792 2.6 and 4.1 us in a graph, 2,048 rows 7.6 and 9.3, 32,768 119.5 and 120.8;
    // of 1,024 (half of the waves have nothing) 32 rows 2.2 and 2.8, 2,048 rows 5.0 and 5.4, 32,768 67 and 70; but 32,768 rows of 640 40 and 36
    if (!cut && spans >= 128 && spans <= 256) return reinterpret_cast<const void *>(&N::rms_norm_rows<X, RES, OUT, 4, 1, false>);
    if (spans > 256 && spans <= 768)
        return cut ? reinterpret_cast<const void *>(&N::rms_norm_rows<X, RES, OUT, 4, 3, true>)
                   : reinterpret_cast<const void *>(&N::rms_norm_rows<X, RES, OUT, 4, 3, false>);
    *waves = 1;
    if (cut && spans <= 256) return reinterpret_cast<const void *>(&N::rms_norm_rows<X, RES, OUT, 1, 4, true>);
    if (spans <= 64) return reinterpret_cast<const void *>(&N::rms_norm_rows<X, RES, OUT, 1, 1, false>);
    if (spans < 128) return reinterpret_cast<const void *>(&N::rms_norm_rows<X, RES, OUT, 1, 2, false>);
    *waves = N::kLoopWaves;
    if (spans <= 2048) return reinterpret_cast<const void *>(&N::rms_norm_rows<X, RES, OUT, N::kLoopWaves, 2, true>);
    return reinterpret_cast<const void *>(&N::rms_norm_walk<X, RES, OUT>);
}
template <int X, int RES> const void *norm_fn(int32_t out, int64_t dim, int *waves) {
    return out == MB_F32    ? norm_fn<X, RES, 0>(dim, waves)
           : out == MB_BF16 ? norm_fn<X, RES, 1>(dim, waves)
                            : norm_fn<X, RES, mbs::norm::kFp8>(dim, waves);
}
template <int X> const void *norm_fn(int32_t res, int32_t out, int64_t dim, int *waves) {
    return res == MB_F32    ? norm_fn<X, 0>(out, dim, waves)
           : res == MB_BF16 ? norm_fn<X, 1>(out, dim, waves)
                            : norm_fn<X, mbs::norm::kNone>(out, dim, waves);
}

template <int DY, int H, int DX> const void *norm_bwd_fn(int64_t dim, int *waves) {
    namespace N = mbs::norm;
    const int64_t spans = (dim + 7) / 8;
    const bool cut = dim % 8 != 0;
    *waves = 1;
    if (cut && spans <= 256) return reinterpret_cast<const void *>(&N::rms_norm_bwd_rows<DY, H, DX, 1, 4, true>);
    if (spans <= 64) return reinterpret_cast<const void *>(&N::rms_norm_bwd_rows<DY, H, DX, 1, 1, false>);
    if (spans <= 128) return reinterpret_cast<const void *>(&N::rms_norm_bwd_rows<DY, H, DX, 1, 2, false>);
    if (spans <= 256) return reinterpret_cast<const void *>(&N::rms_norm_bwd_rows<DY, H, DX, 1, 4, false>);
    *waves = 4;
    if (spans <= 768)
        return cut ? reinterpret_cast<const void *>(&N::rms_norm_bwd_rows<DY, H, DX, 4, 3, true>)
                   : reinterpret_cast<const void *>(&N::rms_norm_bwd_rows<DY, H, DX, 4, 3, false>);
    *waves = N::kLoopWaves;
    if (spans <= 2048) return reinterpret_cast<const void *>(&N::rms_norm_bwd_rows<DY, H, DX, N::kLoopWaves, 2, true>);
    return reinterpret_cast<const void *>(&N::rms_norm_bwd_walk<DY, H, DX>);
}
template <int DY> const void *norm_bwd_fn(int32_t h, int32_t dx, int64_t dim, int *waves) {
    if (h == MB_F32) return dx == MB_F32 ? norm_bwd_fn<DY, 0, 0>(dim, waves) : norm_bwd_fn<DY, 0, 1>(dim, waves);
    return dx == MB_F32 ? norm_bwd_fn<DY, 1, 0>(dim, waves) : norm_bwd_fn<DY, 1, 1>(dim, waves);
}

// Sizes and the rows' elements.  A launch of dw's joining has less than 2^32 threads.
bool norm_sizes(int64_t rows, int64_t dim, int64_t *elems) {
    return rows >= 0 && dim >= 0 && dim < (int64_t(1) << 25) && rows < kMaxElems && mul_ok(rows, dim, elems);
}

// Workgroups of the gradient: what runs at once, 8 waves per CU.
int64_t norm_bwd_groups(int64_t rows, int64_t dim) {
    // at least two rows to a wave (or workgroup): (2042, 1536) fp32 16.9 us with one, 15.4 with two
    const int64_t per = dim <= 2048 ? 8 : 2, most = dim <= 6144 ? 512 : 256;
    return std::min(most, (rows + per - 1) / per);
}

int64_t norm_bwd_bytes(int64_t rows, int64_t dim) {
    const int64_t groups = norm_bwd_groups(rows, dim);
    return groups <= 1 ? 0 : groups * dim * 4;
}

// ---- matrices in 8 bits ------------------------------------------------------------

template <int X> const void *quant_fn(bool tile, bool transpose) {
    namespace Q = mbs::quant;
    if (tile)
        return transpose ? reinterpret_cast<const void *>(&Q::quantize<X, true, true>)
                         : reinterpret_cast<const void *>(&Q::quantize<X, true, false>);
    return transpose ? reinterpret_cast<const void *>(&Q::quantize<X, false, true>)
                     : reinterpret_cast<const void *>(&Q::quantize<X, false, false>);
}

// ---- sampling -----------------------------------------------------------------------

template <int DT> const void *sample_fn(int64_t vocab, unsigned *threads) {
    namespace S = mbs::pick;
    // one wave needs no barriers
    *threads = vocab <= 256 ? 64 : vocab <= 1024 ? 256 : 1024;
    if (vocab <= 256) return reinterpret_cast<const void *>(&S::sample_rows<DT, 64, 1>);
    if (vocab <= 1024) return reinterpret_cast<const void *>(&S::sample_rows<DT, 256, 1>);
    if (vocab <= 8192) return reinterpret_cast<const void *>(&S::sample_rows<DT, 1024, 2>);
    if (vocab < S::kLongRow) return reinterpret_cast<const void *>(&S::sample_rows<DT, 1024, 0>);
    return reinterpret_cast<const void *>(&S::sample_rows<DT, 1024, 0, true>);
}

// Which kernel takes a product, and its tiles.
struct MatmulPlan {
    const void *fn;
    int64_t tile_m, tile_n;
    unsigned threads;
    template <int OUT> void tiles(const mb_matmul_desc *d) {
        namespace M = mbs::matmul;
        fn = d->a_tile   ? reinterpret_cast<const void *>(&M::matmul_tiles<OUT, 1>)
             : d->b_tile ? reinterpret_cast<const void *>(&M::matmul_tiles<OUT, 2>)
                         : reinterpret_cast<const void *>(&M::matmul_tiles<OUT, 0>);
        tile_m = M::Tile128::kM; tile_n = M::Tile128::kN; threads = M::Tile128::kThreads;
    }
    void large(const mb_matmul_desc *d) {
        namespace M = mbs::matmul;
        fn = d->a_tile   ? reinterpret_cast<const void *>(&M::matmul_large<1>)
             : d->b_tile ? reinterpret_cast<const void *>(&M::matmul_large<2>)
                         : reinterpret_cast<const void *>(&M::matmul_large<0>);
        tile_m = tile_n = 256; threads = 512;
    }
    template <int OUT, int MI, int NJ> void split() {
        fn = reinterpret_cast<const void *>(&mbs::matmul::matmul_split<OUT, MI, NJ>);
        tile_m = 16 * MI; tile_n = 16 * NJ; threads = 64 * mbs::matmul::kSplit;
    }
    template <int OUT> void tiled(const mb_matmul_desc *d, const mbs::matmul::Params &p, bool whole) {
        const int64_t t128 = d->batch * ((p.m + 127) / 128) * ((p.n + 127) / 128), t256 = d->batch * ((p.m + 255) / 256) * ((p.n + 255) / 256);
        if (!whole) {
            fn = reinterpret_cast<const void *>(&mbs::matmul::matmul_any<OUT>);
            tile_m = tile_n = mbs::matmul::kAnyTile; threads = mbs::matmul::kAnyThreads;
        // tiles of 256 where those of 128 do not all run at once (two per CU) and the larger ones' places are mostly used: (2176, 4096, 1792)
        // 29.5 us against 36.5, (384, 30000, 1792) 31 and 36; but (2048, 4096, 1792) 30 and 27, 100 of (300, 300, 1792) 53 and 40, 600 of
        // (100, 100, 1792) 76 and 45
        } else if (OUT == 1 && t128 > 512 && 5 * t256 <= 2 * t128) large(d);
        else tiles<OUT>(d);
    }
    template <int OUT> void choose(const mb_matmul_desc *d, const mbs::matmul::Params &p, const void *a, const void *b) {
        // whole aligned pieces of 16 bytes, and a tile's rows within the 31 bits of a buffer's offsets
        const bool whole = p.k % 16 == 0 && aligned(a, 16) && aligned(b, 16) && p.k < (int64_t(1) << 22);
        const int64_t t16 = d->batch * ((p.m + 15) / 16) * ((p.n + 15) / 16);
        // past 2^23 of the smallest pieces a launch of theirs could have 2^32 threads
        if (t16 >= (int64_t(1) << 23)) tiled<OUT>(d, p, whole);
        else if (t16 < 512) split<OUT, 1, 1>();
        else if (p.m <= 16) t16 < 1024 ? split<OUT, 1, 2>() : split<OUT, 1, 4>();
        else if (p.n <= 16) t16 < 1024 ? split<OUT, 2, 1>() : split<OUT, 4, 1>();
        else if (t16 < 1024) split<OUT, 2, 2>();
        else if (p.m <= 32) split<OUT, 2, 4>();
        else if (p.n <= 32 || t16 < 2048) split<OUT, 4, 2>();
        else if (p.m <= 64 || p.n <= 64 || t16 < 5120) split<OUT, 4, 4>();
        else tiled<OUT>(d, p, whole);
    }
    MatmulPlan(const mb_matmul_desc *d, const mbs::matmul::Params &p, const void *a, const void *b) {
        if (d->out_dtype == MB_F32) choose<0>(d, p, a, b);
        else choose<1>(d, p, a, b);
    }
};

}  // namespace

extern "C" {

int mb_rms_norm_fwd(int64_t rows, int64_t dim, int32_t x_dtype, int32_t residual_dtype, int32_t out_dtype, float eps,
                    const void *x, const float *weight, const void *residual, void *y, float *scales, void *residual_out,
                    float *rstd, void *stream) {
    int64_t elems;
    if (!norm_sizes(rows, dim, &elems)) return MB_ERR_SHAPE;
    const bool fp8 = out_dtype == MB_FP8, adds = residual || residual_out;
    if (!valid_dtype(x_dtype) || (!valid_dtype(out_dtype) && !fp8) || (adds && !valid_dtype(residual_dtype))) return MB_ERR_DTYPE;
    if (!(eps >= 0.0f) || std::isinf(eps)) return MB_ERR_UNSUPPORTED;
    if (elems == 0 && (rows == 0 || !rstd)) return MB_OK;       // rows without columns have a rstd all the same
    if (elems > 0 && (!x || !y || (adds && (!residual || !residual_out)) || (fp8 && !scales))) return MB_ERR_NULL;
    const size_t xsz = dtype_size(x_dtype), rsz = dtype_size(residual_dtype), ysz = fp8 ? 1 : dtype_size(out_dtype);
    if (!aligned(x, xsz) || !aligned(y, ysz) || !aligned(residual, rsz) || !aligned(residual_out, rsz)) return MB_ERR_ALIGN;
    if (!aligned(weight, 4) || !aligned(scales, 4) || !aligned(rstd, 4)) return MB_ERR_ALIGN;
    const size_t n = (size_t)elems, s_b = fp8 ? (size_t)(rows * blocks_of(dim)) * 4 : 0;
    // h may take the residual's place
    const Range outs[] = {{y, n * ysz}, {scales, s_b}, {residual_out, n * rsz}, {rstd, (size_t)rows * 4}};
    const Range ins[] = {{x, n * xsz}, {weight, (size_t)dim * 4}, {residual == residual_out ? nullptr : residual, n * rsz}};
    if (any_overlap(outs, ins)) return MB_ERR_ALIAS;
    mbs::norm::FwdParams p{rows, dim, x, weight, residual, y, scales, residual_out, rstd, eps};
    const int32_t res = adds ? residual_dtype : -1;
    int waves;
    const void *fn = x_dtype == MB_F32 ? norm_fn<0>(res, out_dtype, dim, &waves) : norm_fn<1>(res, out_dtype, dim, &waves);
    const int64_t per = waves == 1 ? 4 : 1;
    const int64_t blocks = std::min<int64_t>((rows + per - 1) / per, 1 << 20);
    return status(launch(fn, dim3((unsigned)blocks), dim3(waves == 1 ? 256 : 64 * waves), &p, stream));
}

int mb_rms_norm_bwd(int64_t rows, int64_t dim, int32_t dy_dtype, int32_t h_dtype, int32_t dx_dtype, const void *dy,
                    const void *h, const float *rstd, const float *weight, const void *dh, void *dx, void *dresidual,
                    float *dweight, void *workspace, void *stream) {
    int64_t elems;
    if (!norm_sizes(rows, dim, &elems)) return MB_ERR_SHAPE;
    if (!valid_dtype(dy_dtype) || !valid_dtype(h_dtype) || !valid_dtype(dx_dtype)) return MB_ERR_DTYPE;
    if (dim == 0 || (rows == 0 && !dweight)) return MB_OK;
    if (rows > 0 && (!dy || !h || !rstd || !dx)) return MB_ERR_NULL;
    const size_t ysz = dtype_size(dy_dtype), hsz = dtype_size(h_dtype), xsz = dtype_size(dx_dtype);
    if (!aligned(dy, ysz) || !aligned(h, hsz) || !aligned(dh, hsz) || !aligned(dx, xsz) || !aligned(dresidual, hsz))
        return MB_ERR_ALIGN;
    if (!aligned(rstd, 4) || !aligned(weight, 4) || !aligned(dweight, 4) || !aligned(workspace, 16)) return MB_ERR_ALIGN;
    const size_t n = (size_t)elems, w_b = (size_t)dim * 4, part_b = dweight ? (size_t)norm_bwd_bytes(rows, dim) : 0;
    const Range outs[] = {{dx, n * xsz}, {dresidual, n * hsz}, {dweight, w_b}, {workspace, part_b}};
    const Range ins[] = {{dy, n * ysz}, {h, n * hsz}, {rstd, (size_t)rows * 4}, {weight, w_b}, {dh, n * hsz}};
    if (any_overlap(outs, ins)) return MB_ERR_ALIAS;
    mbs::norm::BwdParams p{rows, dim, dy, h, rstd, weight, dh, dx, dresidual, dweight, dweight};
    int waves;
    const void *fn = dy_dtype == MB_F32 ? norm_bwd_fn<0>(h_dtype, dx_dtype, dim, &waves) : norm_bwd_fn<1>(h_dtype, dx_dtype, dim, &waves);
    int32_t groups = (int32_t)norm_bwd_groups(rows, dim);
    const dim3 grid((unsigned)groups), block(waves == 1 ? 256 : 64 * waves);
    const dim3 jgrid((unsigned)((dim + mbs::norm::kJoinColumns - 1) / mbs::norm::kJoinColumns));
    const dim3 jblock(mbs::norm::kJoinColumns * mbs::norm::kJoinShares);
    void *args[] = {&p}, *jargs[] = {&p.part, &groups, &dim, &dweight};
    const void *join = reinterpret_cast<const void *>(&mbs::norm::rms_norm_join);
    if (rows == 0) return status(hipLaunchKernel(join, jgrid, jblock, jargs, 0, st_of(stream)));     // a sum of nothing: zeros
    if (part_b == 0) return status(hipLaunchKernel(fn, grid, block, args, 0, st_of(stream)));
    Workspace ws(workspace, part_b, st_of(stream));
    if (!ws.at) return MB_ERR_HIP;
    p.part = reinterpret_cast<float *>(ws.at);
    hipError_t e = hipLaunchKernel(fn, grid, block, args, 0, ws.st);
    if (e == hipSuccess) e = hipLaunchKernel(join, jgrid, jblock, jargs, 0, ws.st);
    return status(ws.done(e));
}

int64_t mb_rms_norm_bwd_workspace(int64_t rows, int64_t dim) {
    int64_t elems;
    return norm_sizes(rows, dim, &elems) ? norm_bwd_bytes(rows, dim) : (int64_t)MB_ERR_SHAPE;
}

int mb_quantize_fp8(int64_t batch, int64_t rows, int64_t cols, int32_t x_dtype, int32_t tile, int32_t transpose,
                    const void *x, void *q, float *scales, void *stream) {
    namespace Q = mbs::quant;
    int64_t elems, tiles;
    if (batch < 0 || rows < 0 || cols < 0 || rows >= (int64_t(1) << 37) || cols >= (int64_t(1) << 37)) return MB_ERR_SHAPE;
    if (!valid_dtype(x_dtype)) return MB_ERR_DTYPE;
    if (!mul_ok(batch, rows, &elems) || !mul_ok(elems, cols, &elems)) return MB_ERR_SHAPE;
    if (elems == 0) return MB_OK;
    // less than 2^32 threads in the launch
    if (!mul_ok(batch, blocks_of(rows), &tiles) || !mul_ok(tiles, blocks_of(cols), &tiles) || tiles >= int64_t(1) << 23) return MB_ERR_SHAPE;
    if (!x || !q || !scales) return MB_ERR_NULL;
    if (!aligned(x, dtype_size(x_dtype)) || !aligned(scales, 4)) return MB_ERR_ALIGN;
    const int64_t out_rows = transpose ? cols : rows, out_cols = transpose ? rows : cols;
    const size_t s_b = (size_t)(batch * (tile ? blocks_of(out_rows) : out_rows) * blocks_of(out_cols)) * 4;
    const Range outs[] = {{q, (size_t)elems}, {scales, s_b}};
    const Range ins[] = {{x, (size_t)elems * dtype_size(x_dtype)}};
    if (any_overlap(outs, ins)) return MB_ERR_ALIAS;
    Q::Params p{rows, cols, (int32_t)blocks_of(rows), (int32_t)blocks_of(cols), x, static_cast<uint8_t *>(q), scales};
    const void *fn = x_dtype == MB_F32 ? quant_fn<0>(tile, transpose) : quant_fn<1>(tile, transpose);
    return status(launch(fn, dim3((unsigned)tiles), dim3(Q::kThreads), &p, stream));
}

int mb_matmul_fp8(const mb_matmul_desc *desc, const void *a, const float *a_scales, const void *b, const float *b_scales,
                  void *c, void *stream) {
    namespace M = mbs::matmul;
    if (!desc) return MB_ERR_NULL;
    const int64_t batch = desc->batch, m = desc->m, n = desc->n, k = desc->k;
    if (batch < 0 || m < 0 || n < 0 || k < 0) return MB_ERR_SHAPE;
    if (!valid_dtype(desc->out_dtype)) return MB_ERR_DTYPE;
    if (desc->reserved != 0) return MB_ERR_UNSUPPORTED;
    // rows fit 31 bits with a tile more, blocks 23
    constexpr int64_t most = int64_t(1) << 30;
    if (m >= most || n >= most || k >= most) return MB_ERR_SHAPE;
    int64_t c_elems, a_elems, b_elems, tiles;
    const int64_t an = desc->a_batched ? batch : 1, bn = desc->b_batched ? batch : 1;
    if (!mul_ok(batch, m, &c_elems) || !mul_ok(c_elems, n, &c_elems)) return MB_ERR_SHAPE;
    if (!mul_ok(an, m, &a_elems) || !mul_ok(a_elems, k, &a_elems) || !mul_ok(bn, n, &b_elems) || !mul_ok(b_elems, k, &b_elems))
        return MB_ERR_SHAPE;
    if (c_elems == 0) return MB_OK;
    if (!c || (k > 0 && (!a || !a_scales || !b || !b_scales))) return MB_ERR_NULL;
    if (!aligned(c, dtype_size(desc->out_dtype)) || !aligned(a_scales, 4) || !aligned(b_scales, 4)) return MB_ERR_ALIGN;
    const int64_t blocks = blocks_of(k);
    const int64_t as_step = (desc->a_tile ? blocks_of(m) : m) * blocks, bs_step = (desc->b_tile ? blocks_of(n) : n) * blocks;
    const Range outs[] = {{c, (size_t)c_elems * dtype_size(desc->out_dtype)}};
    const Range ins[] = {{a, (size_t)a_elems}, {a_scales, (size_t)(an * as_step) * 4}, {b, (size_t)b_elems},
                         {b_scales, (size_t)(bn * bs_step) * 4}};
    if (any_overlap(outs, ins)) return MB_ERR_ALIAS;
    M::Params p{};
    p.m = m; p.n = n; p.k = k;
    p.a_step = desc->a_batched ? m * k : 0; p.b_step = desc->b_batched ? n * k : 0;
    p.as_step = desc->a_batched ? as_step : 0; p.bs_step = desc->b_batched ? bs_step : 0;
    p.blocks = (int32_t)blocks;
    p.a_shift = desc->a_tile ? 7 : 0; p.b_shift = desc->b_tile ? 7 : 0;
    p.a = static_cast<const uint8_t *>(a); p.b = static_cast<const uint8_t *>(b);
    p.as = a_scales; p.bs = b_scales; p.c = c;
    // less than 2^32 threads in the launch
    if (!mul_ok((m + 127) / 128, (n + 127) / 128, &tiles) || !mul_ok(tiles, batch, &tiles) || tiles >= int64_t(1) << 23) return MB_ERR_SHAPE;
    const MatmulPlan f(desc, p, a, b);
    p.m_tiles = (uint32_t)((m + f.tile_m - 1) / f.tile_m);
    p.n_tiles = (uint32_t)((n + f.tile_n - 1) / f.tile_n);
    return status(launch(f.fn, dim3((unsigned)(p.m_tiles * p.n_tiles * batch)), dim3(f.threads), &p, stream));
}

int mb_sample(int64_t batch, int64_t vocab, int32_t logit_dtype, float temperature, int32_t top_k, float top_p, float min_p,
              const float *temperatures, const int32_t *top_ks, const float *top_ps, const float *min_ps, const void *logits,
              const float *noise, int32_t *token, float *prob, void *stream) {
    namespace S = mbs::pick;
    int64_t elems;
    // less than 2^32 threads in the launch
    if (batch < 0 || vocab < 1 || vocab >= (int64_t(1) << 30) || batch >= int64_t(1) << 22 || !mul_ok(batch, vocab, &elems)) return MB_ERR_SHAPE;
    if (!valid_dtype(logit_dtype)) return MB_ERR_DTYPE;
    if (!temperatures && temperature != 0.0f &&
        (!(temperature > 0.0f) || std::isinf(temperature) || std::isinf(2.0f / temperature))) return MB_ERR_UNSUPPORTED;
    if ((!top_ps && std::isnan(top_p)) || (!min_ps && !(min_p <= 1.0f))) return MB_ERR_UNSUPPORTED;
    if (batch == 0) return MB_OK;
    if (!logits || !noise || !token) return MB_ERR_NULL;
    if (!aligned(logits, dtype_size(logit_dtype))) return MB_ERR_ALIGN;
    const void *words[] = {temperatures, top_ks, top_ps, min_ps, noise, token, prob};
    for (const void *q : words)
        if (!aligned(q, 4)) return MB_ERR_ALIGN;
    const size_t b_b = (size_t)batch * 4;
    const Range outs[] = {{token, b_b}, {prob, b_b}};
    const Range ins[] = {{logits, (size_t)elems * dtype_size(logit_dtype)}, {noise, (size_t)elems * 4}, {temperatures, b_b},
                         {top_ks, b_b}, {top_ps, b_b}, {min_ps, b_b}};
    if (any_overlap(outs, ins)) return MB_ERR_ALIAS;
    S::Params p{batch, vocab, logits, noise, temperatures, top_ps, min_ps, top_ks, temperature, top_p, min_p, top_k, token, prob};
    unsigned threads;
    const void *fn = logit_dtype == MB_F32 ? sample_fn<0>(vocab, &threads) : sample_fn<1>(vocab, &threads);
    return status(launch(fn, dim3((unsigned)batch), dim3(threads), &p, stream));
}

}  // extern "C"
