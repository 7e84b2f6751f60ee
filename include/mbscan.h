/*
 * mbscan.h -- C ABI of the MI355X (gfx950) selective-scan library libmbscan.so.
 *
 * The operation is the selective state-space scan that every MambaByte layer
 * runs over its byte sequence (MambaByte, Section 2, eq. (2), with the
 * discretisation of Appendix D and the output and gating rows of Table 8):
 *
 *   dlt_t  = softplus(delta_t + dt_bias)          (eq. (3); or delta_t + dt_bias when delta_softplus == 0)
 *   h_t[n] = exp(dlt_t A[n]) h_{t-1}[n] + dlt_t B_t[n] u_t    (ZOH on A, simplified Euler on B)
 *   y_t    = (sum_n C_t[n] h_t[n] + Dskip u_t) * z_t sigmoid(z_t)
 *
 * for every (batch b, channel d) row independently, starting from a carried
 * state h0 and optionally returning the final state: the resume capability
 * that speculative decoding needs to verify a drafted byte chunk from the
 * cached state and continue from it (Section 3 "Speculative decoding through
 * subword drafting"; Appendix F, Algorithm 1).  mb_scan_step is the
 * one-byte recurrent update used during generation (Section 2: the recurrence
 * is run directly at inference).
 *
 * Conventions shared by every entry point
 * ---------------------------------------
 * - All tensor pointers are DEVICE pointers (memory allocated with hipMalloc or
 *   by a framework on the GPU that is current for the calling thread), dense
 *   and row-major in the layouts stated below.  The caller owns every buffer;
 *   the library keeps no pointer after the call returns.
 * - Work is enqueued on `stream` (a hipStream_t; NULL means the default
 *   stream) and the call returns without waiting.  Argument errors are found
 *   on the host before anything is enqueued and return a negative mb_status;
 *   a launch failure returns MB_ERR_HIP.  Faults during execution surface at
 *   the caller's next synchronisation.  The library never prints or aborts.
 * - Element types: "act" tensors (u, delta, z, B, C and their step
 *   counterparts) share one type, in_dtype: MB_F32 (IEEE float) or MB_BF16
 *   (bfloat16).  A, Dskip, dt_bias, h0, h_last and the step state h are
 *   always float.  The output y has type out_dtype.  All arithmetic is fp32.
 * - Alignment: every pointer must be aligned to its element size.
 * - Sizes: batch, dim, seqlen >= 0 (an empty problem is valid and enqueues
 *   nothing, except that seqlen == 0 still writes h_last = h0, or zeros);
 *   dstate must be 16 (the n_state of every MambaByte model, Table 9), 8, 4,
 *   2 or 1.  Every element count an entry point derives from its sizes
 *   (batch * dim * seqlen, batch * dstate * seqlen, batch * dim * dstate and,
 *   with recorded positions, npos * batch * dim * dstate) must stay below
 *   2^56; a larger one returns MB_ERR_SHAPE.
 */
#ifndef MBSCAN_H
#define MBSCAN_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

/* Raised when an entry point changes; new ones beside the old leave it. */
#define MB_ABI_VERSION 6

typedef enum {
    MB_F32 = 0,
    MB_BF16 = 1,
    MB_FP8 = 2               /* e4m3 (largest 448, no infinities), where an entry point names it */
} mb_dtype;

typedef enum {
    MB_OK = 0,
    MB_ERR_NULL = -1,        /* a required pointer is NULL */
    MB_ERR_SHAPE = -2,       /* a size is negative or too large */
    MB_ERR_DTYPE = -3,       /* in_dtype or out_dtype is not an mb_dtype */
    MB_ERR_ALIGN = -4,       /* a pointer is not aligned to its element size */
    MB_ERR_UNSUPPORTED = -5, /* dstate not in {1, 2, 4, 8, 16}, a convolution width outside
                                1 .. 4, a reserved field is set, or a number (a temperature,
                                a bound of the norm) outside its range */
    MB_ERR_HIP = -6,         /* the HIP runtime reported an error when launching */
    MB_ERR_ALIAS = -7        /* an output overlaps an input it may not overlap */
} mb_status;

/* Problem description of mb_scan_fwd. */
typedef struct {
    int64_t batch;          /* B: independent sequences */
    int64_t dim;            /* D: channels (e * d in the paper's notation) */
    int64_t seqlen;         /* L: bytes in the sequence */
    int64_t dstate;         /* N: SSM state size per channel (n_state) */
    int32_t in_dtype;       /* mb_dtype of u, delta, z, Bmat, Cmat */
    int32_t out_dtype;      /* mb_dtype of y */
    int32_t delta_softplus; /* nonzero: dlt = softplus(delta + dt_bias); zero: dlt = delta + dt_bias */
    int32_t reserved;       /* must be 0 */
} mb_scan_desc;

/*
 * Forward selective scan over a whole sequence (Section 2, eq. (2); the
 * parallel-scan path of Section 2 "Implementation" that also verifies drafted
 * bytes in Algorithm 1).
 *
 *   u, delta     act   (B, D, L)  input x and the raw timestep, time contiguous
 *   A            float (D, N)     diagonal of A per channel (normally negative)
 *   Bmat, Cmat   act   (B, N, L)  input and output projections, shared by all
 *                                 channels of a batch element, time contiguous
 *   Dskip        float (D)        skip weight; NULL means 0
 *   dt_bias      float (D)        added to delta before softplus; NULL means 0
 *   z            act   (B, D, L)  gate input; NULL means no gate (y = C h + D u)
 *   h0           float (B, D, N)  initial state; NULL means zeros
 *   y            out   (B, D, L)  output; must not overlap any input
 *   h_last       float (B, D, N)  state after the last byte; NULL means not
 *                                 written.  It may be the same buffer as h0
 *                                 (each row reads its h0 before writing), but
 *                                 must not partially overlap it or any other
 *                                 argument.
 */
int mb_scan_fwd(const mb_scan_desc *desc,
                const void *u, const void *delta, const float *A,
                const void *Bmat, const void *Cmat,
                const float *Dskip, const float *dt_bias, const void *z,
                const float *h0, void *y, float *h_last, void *stream);

/*
 * mb_scan_fwd for callers that cannot allocate device memory: code under HIP
 * graph capture, tight serving loops, harnesses that forbid hipMalloc.  The
 * arguments, the results (the same bits as mb_scan_fwd's) and the errors are
 * those of mb_scan_fwd; the call itself allocates nothing.
 *
 * Where mb_scan_fwd cuts a sequence into time segments (few rows, long
 * sequences) it allocates a carry buffer on the stream: one plane of
 * batch x dim x 128 bytes per pre-pass piece (1, 2 or 4 per segment but the last)
 * and one for h0.  This entry point keeps that carry in a static device array of
 * 8 MiB instead: each GPU the library runs on holds its own copy until the
 * process ends.  A problem whose carry would exceed it returns MB_ERR_SHAPE
 * (on a 256-CU MI355X none does).  The array keeps the last
 * call's contents; nothing in it needs to start at zero (the segment pre-pass
 * writes every carry entry before the scan reads it).  Every call on one GPU
 * shares that GPU's array, so calls that may overlap in time on one GPU (other
 * streams, other threads) race: serialise them, or use mb_scan_fwd.
 */
int mb_scan_fwd_noalloc(const mb_scan_desc *desc,
                        const void *u, const void *delta, const float *A,
                        const void *Bmat, const void *Cmat,
                        const float *Dskip, const float *dt_bias, const void *z,
                        const float *h0, void *y, float *h_last, void *stream);

/*
 * mb_scan_fwd that also records the state at requested positions.  The
 * verifier of Algorithm 1 (Appendix F) scans the drafted bytes in parallel,
 * finds the bifurcation position c and continues byte by byte from h_c; the
 * resumable scan of Section 3 ("Speculative decoding through subword
 * drafting") restarts from that state instead of from the first byte.
 *
 *   pos    int32 (npos, B)        pos[k * B + b] is the k-th requested
 *                                 position of batch element b: a timestep
 *                                 0 <= p < L, or -1 for the state before the
 *                                 first byte.  Positions need not be sorted or
 *                                 distinct.  Device memory, read only.
 *   npos   >= 0                   0 disables recording (pos and h_pos are then
 *                                 ignored and may be NULL).
 *   h_pos  float (npos, B, D, N)  h_pos[k][b][d][n] = h_p[n] of row (b, d)
 *                                 after timestep p = pos[k * B + b] (h0, or
 *                                 zeros, for p = -1).  A position outside
 *                                 [-1, L-1] is not an error: its slot is
 *                                 filled with NaN.  h_pos[k] has the layout of
 *                                 h0, so it can be passed back as h0 to resume
 *                                 every row of the batch from its k-th
 *                                 position.  h_pos must not overlap any other
 *                                 argument; pos must not overlap y or h_last.
 *
 * Every other argument is as for mb_scan_fwd, and y and h_last are the same
 * bits as mb_scan_fwd's.  A recorded state equals the state the scan carries
 * at that timestep bit for bit.
 */
int mb_scan_fwd_states(const mb_scan_desc *desc,
                       const void *u, const void *delta, const float *A,
                       const void *Bmat, const void *Cmat,
                       const float *Dskip, const float *dt_bias, const void *z,
                       const float *h0, void *y, float *h_last,
                       const int32_t *pos, int64_t npos, float *h_pos, void *stream);

/*
 * mb_scan_fwd that also stores the checkpoints mb_scan_bwd recomputes its
 * chunks from: the training forward (Section 4, Appendix C), whose backward
 * then skips its own forward pass over the sequence.
 *
 *   ck     float (L/16, B, D, N)   ck[k][b][d][n] = h_{16k-1}[n] of row (b, d),
 *                                  the state before timestep 16k (h0, or zeros,
 *                                  for k = 0).  Required; must not overlap any
 *                                  other argument; 8-byte aligned.
 *
 * Every other argument is as for mb_scan_fwd, and y and h_last are the same
 * bits as mb_scan_fwd's (at L = 16, where mb_scan_fwd adds an output's terms in
 * another order, y may differ in its last bits).  Supported: dstate 16, L a multiple of 16 below 2^25
 * (MB_ERR_UNSUPPORTED otherwise), u, delta, z, Bmat, Cmat and y 16-byte
 * aligned (MB_ERR_ALIGN otherwise).
 */
int mb_scan_fwd_ckpt(const mb_scan_desc *desc,
                     const void *u, const void *delta, const float *A,
                     const void *Bmat, const void *Cmat,
                     const float *Dskip, const float *dt_bias, const void *z,
                     const float *h0, void *y, float *h_last, float *ck, void *stream);

/*
 * One recurrent step per row, the state updated in place (Section 2:
 * generation runs the recurrence directly; Algorithm 1's byte-level
 * correction loop).  Identical to mb_scan_fwd with L = 1, h0 = h_last = h.
 *
 *   u_t, delta_t   act   (B, D)     this byte's input and raw timestep
 *   A              float (D, N)
 *   B_t, C_t       act   (B, N)
 *   Dskip, dt_bias float (D)        NULL means 0
 *   z_t            act   (B, D)     NULL means no gate
 *   h              float (B, D, N)  state, read then overwritten; required
 *   y_t            out   (B, D)     output; must not overlap any input or h
 *
 * dim must stay below 2^36 (the launch covers 64 channels per workgroup along
 * one grid dimension); a larger one returns MB_ERR_SHAPE.
 */
int mb_scan_step(int64_t batch, int64_t dim, int64_t dstate,
                 int32_t in_dtype, int32_t out_dtype, int32_t delta_softplus,
                 const void *u_t, const void *delta_t, const float *A,
                 const void *B_t, const void *C_t,
                 const float *Dskip, const float *dt_bias, const void *z_t,
                 float *h, void *y_t, void *stream);

/*
 * The backward of mb_scan_fwd (training at the 8,192-byte context: Section 4,
 * Appendix C): the gradients of sum(dy * y) + sum(dh_last * h_last) with
 * respect to every input of the scan, by reverse-mode differentiation of eq. (2)
 * with the discretisation of Appendix D and Table 8's output and gating.
 *
 *   desc, u, delta, A, Bmat, Cmat, Dskip, dt_bias, z, h0   as for mb_scan_fwd
 *   dy        out-dtype (B, D, L)   gradient with respect to y (desc->out_dtype)
 *   dh_last   float (B, D, N)       gradient with respect to h_last; NULL means 0
 *   ck        float (L/16, B, D, N) checkpoints written by mb_scan_fwd_ckpt for
 *                                   the same inputs, read only; NULL: the call
 *                                   computes them itself (one more forward pass)
 *   du, ddelta, dz   out-dtype (B, D, L)   dz is required when z is given
 *   dA        float (D, N)          summed over batch and time
 *   dB, dC    float (B, N, L)       summed over the channels of each batch element
 *   dDskip, ddt_bias float (D)      required when Dskip / dt_bias are given
 *   dh0       float (B, D, N)       NULL means not written
 * Outputs are overwritten (not accumulated) and must not overlap any other
 * argument; with no row (batch 0) dA, dDskip and ddt_bias are set to zero.
 * Supported: dstate 16, L a multiple of 16 below 2^25, every activation
 * pointer 16-byte aligned and every float pointer 8-byte aligned
 * (MB_ERR_UNSUPPORTED / MB_ERR_ALIGN otherwise).  Results are deterministic.  The call allocates a
 * stream-ordered workspace (hipMallocAsync): state checkpoints every 16 bytes
 * (L/16 x B x D x 16 floats, only when ck is NULL) and per-8-channel dB/dC
 * partials (B x L x D/8 x 64 bytes), freed on the same stream.
 */
int mb_scan_bwd(const mb_scan_desc *desc,
                const void *u, const void *delta, const float *A,
                const void *Bmat, const void *Cmat,
                const float *Dskip, const float *dt_bias, const void *z,
                const float *h0, const void *dy, const float *dh_last, const float *ck,
                void *du, void *ddelta, void *dz, float *dA, float *dB, float *dC,
                float *dDskip, float *ddt_bias, float *dh0, void *stream);

/*
 * The causal depthwise convolution upstream of the scan.  In the Mamba block
 * the x branch is convolved per channel over time with a short kernel and a
 * bias, then passed through the Swish activation, and the result is the scan's
 * input u (Table 8, "Pre-SSM 1D convolution"; Fig. 5, right; kernel size
 * k = 4 in every MambaByte model, Table 9):
 *
 *   pre_t = bias[d] + sum_{i < k} w[d][i] x_{t-(k-1)+i}
 *   y_t   = pre_t * sigmoid(pre_t)     (apply_silu != 0), else pre_t
 *
 * The k - 1 inputs before the first byte come from a carried state, so that a
 * sequence continues exactly where the previous call stopped, and the call
 * returns the last k - 1 inputs as the next state (the convolution's part of
 * the resume that Algorithm 1 relies on).  Arithmetic is fp32.
 */
typedef struct {
    int64_t batch;          /* B */
    int64_t dim;            /* D: channels (e * d) */
    int64_t seqlen;         /* L */
    int32_t width;          /* k: taps per channel, 1 .. 4 */
    int32_t in_dtype;       /* mb_dtype of x */
    int32_t out_dtype;      /* mb_dtype of y */
    int32_t apply_silu;     /* nonzero: Swish after the convolution */
    int32_t reserved;       /* must be 0 */
    int32_t reserved2;      /* must be 0 */
} mb_conv_desc;

/*
 *   x          act   (B, D, L)    input, time contiguous
 *   w          float (D, k)       taps; w[d][k-1] multiplies the current byte
 *   bias       float (D)          NULL means 0
 *   state_in   float (B, D, k-1)  the k-1 inputs before x, oldest first; NULL
 *                                 means zeros (the start of a sequence)
 *   y          out   (B, D, L)    output; must not overlap any other argument
 *   state_out  float (B, D, k-1)  the last k-1 inputs (of state_in followed by
 *                                 x); NULL means not written.  It must not
 *                                 overlap any other argument, state_in
 *                                 included: alternate two buffers to chain
 *                                 calls.  With L = 0 it receives state_in.
 * Errors as for mb_scan_fwd; a width outside 1 .. 4 or a nonzero reserved
 * field is MB_ERR_UNSUPPORTED.
 */
int mb_conv1d_fwd(const mb_conv_desc *desc, const void *x, const float *w, const float *bias,
                  const float *state_in, void *y, float *state_out, void *stream);

/*
 * One byte per row, the convolution state updated in place (generation, and
 * Algorithm 1's byte-level correction loop).  Identical to mb_conv1d_fwd with
 * L = 1, state_in = the old state and state_out = the new one.
 *
 *   x_t    act   (B, D)        this byte's input
 *   w      float (D, k), bias float (D) (NULL means 0)
 *   state  float (B, D, k-1)   read then overwritten; required when k > 1
 *   y_t    out   (B, D)        must not overlap any other argument
 */
int mb_conv1d_step(int64_t batch, int64_t dim, int32_t width, int32_t in_dtype, int32_t out_dtype,
                   int32_t apply_silu, const void *x_t, const float *w, const float *bias,
                   float *state, void *y_t, void *stream);

/*
 * The top-beta check that ends a speculative verification (Section 3,
 * "Speculative decoding through subword drafting"; Appendix F, Algorithm 1;
 * beta = 3 in Table 6).  For drafted byte i of batch element b:
 *
 *   rank   = 1 + the number of candidates y with logits[b][i][y] > logits[b][i][x],
 *            x = draft[b][i]; vocab + 1 when x is outside [0, vocab) or its logit
 *            is NaN (such a byte is always rejected).  Ties do not count against x.
 *            Logits rank exactly like probabilities (a softmax is monotone).
 *   accepted[b] = the number of leading drafted bytes whose rank is <= beta, i.e.
 *            the bifurcation position c: bytes 1..c verified, byte c+1 not.
 *   last_pos[b] = accepted[b] - 1, the 0-based timestep of the last accepted byte
 *            in the verified chunk (-1: none), which can be passed on device, as
 *            pos, to mb_scan_fwd_states to recover the state there.
 *
 *   logits    act   (batch, ndraft, vocab)  next-byte scores; logits[b][i] scores
 *                                            drafted byte i
 *   draft     int32 (batch, ndraft)          the drafted bytes
 *   beta      any int32 (<= 0 accepts nothing)
 *   ranks     int32 (batch, ndraft)          output; NULL means not written
 *   accepted  int32 (batch)                  output; required
 *   last_pos  int32 (batch)                  output; NULL means not written
 * Outputs must not overlap each other or the inputs.  vocab >= 1, ndraft and
 * vocab below 2^31.
 */
int mb_verify_rank(int64_t batch, int64_t ndraft, int64_t vocab, int32_t logit_dtype, int32_t beta,
                   const void *logits, const int32_t *draft, int32_t *ranks, int32_t *accepted,
                   int32_t *last_pos, void *stream);

/* Integer types of the tokens of an embedding. */
typedef enum {
    MB_TOKEN_U8 = 0,         /* bytes */
    MB_TOKEN_I32 = 1,
    MB_TOKEN_I64 = 2
} mb_token_type;

/*
 * The embedding lookup with scaling: the byte model's inputs (256 byte values in
 * every MambaByte model), or a subword drafter's.
 *
 *   out[i][:] = scale * weight[tokens[i]][:]
 *
 * A negative token is padding: its row is zeros.  A token >= vocab is a mistake
 * that the host cannot see: its row is NaN.
 *
 *   tokens  token_type (ntokens)      any leading shape, flattened
 *   weight  weight_dtype (vocab, dim) vocab below 2^31, and not 0 where there are tokens; dim below 2^30
 *   out     out_dtype (ntokens, dim)  must not overlap an input
 * One fp32 product per element, rounded once to out_dtype.
 */
int mb_embedding_fwd(int64_t ntokens, int64_t vocab, int64_t dim, int32_t token_type, int32_t weight_dtype,
                     int32_t out_dtype, float scale, const void *tokens, const void *weight, void *out, void *stream);

/*
 * The gradient of mb_embedding_fwd's table:
 *
 *   dweight[v][:] = scale * sum of dy[i][:] over the i with tokens[i] == v
 *
 * Rows that no token names are zeros; tokens outside [0, vocab) add nothing.
 * Sums are fp32 in an order that the tokens alone fix (the same bits on every
 * call), rounded once to out_dtype.  dweight is overwritten, not accumulated.
 *
 *   tokens  token_type (ntokens)       ntokens below 2^31
 *   dy      dy_dtype (ntokens, dim)
 *   dweight out_dtype (vocab, dim)     must not overlap an input; with tokens, dim below 2^30 and ntokens * dim below 2^37
 *   workspace  device memory of mb_embedding_bwd_workspace(ntokens, vocab, dim) bytes (of a
 *              negative mb_status where the sizes are refused; 0: none is used), 16-byte aligned,
 *              that nothing else uses until the call's work is done; NULL: the call allocates it on the stream
 *              (hipMallocAsync) and frees it there, which costs the host about 8 us
 */
int mb_embedding_bwd(int64_t ntokens, int64_t vocab, int64_t dim, int32_t token_type, int32_t dy_dtype, int32_t out_dtype,
                     float scale, const void *tokens, const void *dy, void *dweight, void *workspace, void *stream);
int64_t mb_embedding_bwd_workspace(int64_t ntokens, int64_t vocab, int64_t dim);

/*
 * The backward of mb_conv1d_fwd: the gradients of sum(dy * y) + sum(dstate_out *
 * state_out) with respect to every input of the convolution.
 *
 *   desc, x, w, bias, state_in     as for mb_conv1d_fwd
 *   dy          out-dtype (B, D, L)   gradient with respect to y (desc->out_dtype)
 *   dstate_out  float (B, D, k-1)     gradient with respect to state_out; NULL means 0
 *   dx          out-dtype (B, D, L)
 *   dw          float (D, k)          summed over batch and time; required
 *   dbias       float (D)             required when bias is given, else ignored
 *   dstate_in   float (B, D, k-1)     NULL means not written
 * Outputs are overwritten (not accumulated) and must not overlap any other
 * argument; with no row or no timestep dw and dbias are zeros.  B * D below
 * 2^26, D * (k + 1) below 255 * 2^24, L below 2^31.  Arithmetic is fp32; results are deterministic.
 *   workspace   as for mb_embedding_bwd, of mb_conv1d_bwd_workspace(desc) bytes
 */
int mb_conv1d_bwd(const mb_conv_desc *desc, const void *x, const float *w, const float *bias, const float *state_in,
                  const void *dy, const float *dstate_out, void *dx, float *dw, float *dbias, float *dstate_in,
                  void *workspace, void *stream);
int64_t mb_conv1d_bwd_workspace(const mb_conv_desc *desc);

/*
 * The global norm of a list of tensors (the gradients of a model):
 *
 *   norm[0] = sqrt(sum of g^2 over every element of every tensor)
 *
 *   count          tensors; an empty one (size 0) may have a NULL address
 *   grads, sizes, dtypes   HOST arrays (count): device addresses, element counts, mb_dtype.
 *                  They are read before the call returns.
 *   norm           float, DEVICE memory, must not overlap a tensor
 *   workspace      as for mb_embedding_bwd, of mb_grad_norm_workspace(count) bytes
 * Squares and sums are fp64, in an order that the sizes and the addresses' places between
 * 16-byte boundaries fix; the result is rounded to fp32.  count below 2^31, and less than
 * about 2^44 elements in all.
 */
int mb_grad_norm(int64_t count, const void *const *grads, const int64_t *sizes, const int32_t *dtypes, float *norm,
                 void *workspace, void *stream);
int64_t mb_grad_norm_workspace(int64_t count);

/*
 * mb_grad_norm, then the tensors clipped by it:
 *
 *   out = g                            where norm + eps <= max_norm
 *       = g * (max_norm / (norm + eps))  otherwise
 *
 * A NaN norm makes every output NaN; an infinite one makes zeros (NaN where g is infinite).
 *
 *   out            HOST array (count) of device addresses of tensors of the same sizes and
 *                  types; NULL: in place, and nothing is written where nothing is clipped.
 *                  Written tensors overlap neither each other, norm nor (unless in place) grads.
 *   max_norm, eps  finite, >= 0 (MB_ERR_UNSUPPORTED otherwise)
 *   norm           the norm before clipping
 *   workspace      as for mb_grad_norm
 */
int mb_clip_grad_norm(int64_t count, const void *const *grads, void *const *out, const int64_t *sizes,
                      const int32_t *dtypes, float max_norm, float eps, float *norm, void *workspace,
                      void *stream);

/*
 * Verification of drafted tokens against the target's probabilities, from given
 * random numbers: the check of mb_verify_rank for sampled instead of greedy
 * generation, with the token that follows.  With ndraft = 0 it samples one token
 * per sequence.
 *
 *   p_i = softmax(logits[b][i] / temperature), q_i = softmax(draft_logits[b][i] / temperature),
 *   or, without draft_logits, certainty of the drafted token x_i
 *
 *   token i passes      uniform[b][i] * q_i(x_i) < p_i(x_i)
 *   accepted[b]   = c   the number of leading tokens that pass, of the len = lengths[b] drafted
 *   next_token[b]       the y with the largest r(y) / noise[b][y], the lowest such y, where
 *                       r = max(p_c - q_c, 0) for c < len (p_c if that is zero everywhere) and
 *                       r = p_len for c = len
 *
 * With uniform numbers in [0, 1) and exponential noise of mean 1 the tokens are
 * distributed as samples of the target.  A drafted token outside [0, vocab) does not
 * pass.  A row of logits that is no distribution (a NaN or +infinity in it, or nothing
 * above -infinity) passes nothing: in the target's row the next token is -1, in the
 * drafter's r = p_c.  -infinity masks a token.
 *
 *   logits        act (batch, ndraft + 1, vocab)
 *   draft_logits  act (batch, ndraft, vocab)   NULL: drafts without probabilities
 *   draft         int32 (batch, ndraft)
 *   lengths       int32 (batch)                tokens drafted, clamped to [0, ndraft]; NULL means ndraft
 *   uniform       float (batch, ndraft)
 *   noise         float (batch, vocab)
 *   accepted, next_token  int32 (batch)        required
 *   last_pos      int32 (batch)                accepted - 1, as mb_verify_rank's; NULL means not written
 *   probs         float (batch, ndraft)        p_i(x_i) for i < len (0 for a token outside [0, vocab) or
 *                                              a row that is no distribution), 0 for i >= len; NULL means
 *                                              not written
 *   temperature   > 0, it and its inverse finite (MB_ERR_UNSUPPORTED otherwise)
 *   workspace     as for mb_embedding_bwd, of mb_verify_sample_workspace(batch, ndraft, vocab) bytes
 *                 (none up to a vocabulary of 1,024)
 * Outputs must not overlap each other or the inputs.  vocab >= 1, below
 * 2^31 - 4096; batch below 2^22; batch * (2 ndraft + 1) * (vocab / 4096 + 1) below 2^23 where vocab
 * is above 1,024.  Probabilities are fp32.
 */
int mb_verify_sample(int64_t batch, int64_t ndraft, int64_t vocab, int32_t logit_dtype, float temperature,
                     const void *logits, const void *draft_logits, const int32_t *draft, const int32_t *lengths,
                     const float *uniform, const float *noise, int32_t *accepted, int32_t *last_pos,
                     int32_t *next_token, float *probs, void *workspace, void *stream);
int64_t mb_verify_sample_workspace(int64_t batch, int64_t ndraft, int64_t vocab);

/*
 * The residual's addition and the root-mean-square norm in front of a block:
 *
 *   h = x + residual, rounded to the residual's type (x itself without one)
 *   y = h * rstd * weight,   rstd = 1 / sqrt(mean over the row of h^2 + eps)
 *
 *   x            act (rows, dim)             x_dtype
 *   weight       float (dim)                 NULL means ones
 *   residual     (rows, dim)                 residual_dtype (fp32 or bf16, whatever x is); NULL: nothing is added,
 *                                            and residual_out is NULL too
 *   y            out_dtype (rows, dim)       fp32, bf16 or MB_FP8
 *   scales       float (rows, ceil(dim/128)) with MB_FP8 (required): those of y's blocks, as mb_quantize_fp8's
 *   residual_out (rows, dim)                 h, in residual's type; may be residual
 *   rstd         float (rows)                for the gradient, NaN where dim is 0; NULL means not written
 * Outputs overlap nothing else.  eps finite, >= 0 (MB_ERR_UNSUPPORTED otherwise); dim below 2^25.  Arithmetic is fp32,
 * squares included: a row of elements above 1e19 has rstd 0, and one of elements below 1e-23 that of a row of zeros.
 */
int mb_rms_norm_fwd(int64_t rows, int64_t dim, int32_t x_dtype, int32_t residual_dtype, int32_t out_dtype, float eps,
                    const void *x, const float *weight, const void *residual, void *y, float *scales, void *residual_out,
                    float *rstd, void *stream);

/*
 * The gradients of sum(dy * y) + sum(dh * h):
 *
 *   g = dy * weight,  d = rstd * (g - h rstd mean(g h rstd)) + dh
 *   dx = d,  dresidual = d,  dweight = sum over the rows of dy h rstd
 *
 *   dy         dy_dtype (rows, dim)
 *   h, dh      h_dtype (rows, dim)      h as the forward kept it (x without a residual); dh NULL means 0
 *   rstd       float (rows)             the forward's
 *   weight     float (dim)              NULL means ones
 *   dx         dx_dtype (rows, dim)
 *   dresidual  h_dtype (rows, dim)      NULL means not written
 *   dweight    float (dim)              summed over the rows; NULL means not written; zeros without rows
 *   workspace  as for mb_embedding_bwd, of mb_rms_norm_bwd_workspace(rows, dim) bytes; not used without dweight
 * Outputs are overwritten and overlap nothing else.  The same bits on every call.
 */
int mb_rms_norm_bwd(int64_t rows, int64_t dim, int32_t dy_dtype, int32_t h_dtype, int32_t dx_dtype, const void *dy,
                    const void *h, const float *rstd, const float *weight, const void *dh, void *dx, void *dresidual,
                    float *dweight, void *workspace, void *stream);
int64_t mb_rms_norm_bwd_workspace(int64_t rows, int64_t dim);

/*
 * Matrices in 8 bits (e4m3) with a scale for each 128 columns of a row, or each tile of 128 x 128:
 *
 *   scale = max(largest magnitude of the block / 448, 2^-126),   q = x * (1 / scale), rounded to nearest even
 *
 * so that q * scale stands for x.  A NaN stays one, and its block's scale is that of the others; an infinity makes its
 * block's scale infinite.
 *
 *   x       x_dtype (batch, rows, cols)
 *   q       e4m3 (batch, rows, cols), or with transpose (batch, cols, rows): blocks, rows and columns are then q's
 *   scales  float (batch, R, ceil(C/128)) for q of R rows and C columns; with tile (batch, ceil(R/128), ceil(C/128))
 * Outputs overlap nothing else.  batch * ceil(rows/128) * ceil(cols/128) below 2^23.
 */
int mb_quantize_fp8(int64_t batch, int64_t rows, int64_t cols, int32_t x_dtype, int32_t tile, int32_t transpose,
                    const void *x, void *q, float *scales, void *stream);

typedef struct {
    int64_t batch, m, n, k;
    int32_t a_batched, b_batched;   /* a (batch, m, k) or (m, k) for every product; b likewise */
    int32_t a_tile, b_tile;         /* scales per 128 x 128 tile instead of per row */
    int32_t out_dtype;              /* fp32 or bf16 */
    int32_t reserved;               /* 0 */
} mb_matmul_desc;

/*
 * Products of matrices in 8 bits with scales, as mb_quantize_fp8 and mb_rms_norm_fwd write them:
 *
 *   c[m][n] = sum over k of (a[m][k] * its scale) * (b[n][k] * its scale)
 *
 *   a         e4m3 (m, k) or (batch, m, k)     a_scales  float ([batch,] m or ceil(m/128), ceil(k/128))
 *   b         e4m3 (n, k) or (batch, n, k)     b_scales  likewise
 *   c         out_dtype (batch, m, n), overlaps nothing else
 * Scaling, by the product of a block's two scales, and the sum over blocks of 128 are fp32, rounded once to out_dtype.
 * Within a block: fp32 for an fp32 c; for a bf16 c the matrix unit first sums 8 neighbouring products at a time, each to
 * 2^-13 of the largest of the 8, and those sums in fp32.  The same bits on every call.  Nothing depends on the values of the
 * other rows, columns and products, but their numbers choose the kernel, and with it the order in which blocks are summed: past
 * k = 128 a product's bits may be others in a batch of another size.  k = 0 gives zeros.  m, n and k
 * below 2^30, batch * ceil(m/128) * ceil(n/128) below 2^23.
 */
int mb_matmul_fp8(const mb_matmul_desc *desc, const void *a, const float *a_scales, const void *b, const float *b_scales,
                  void *c, void *stream);

/*
 * The next token of each sequence, from given random numbers.  In the order of falling logits, the lowest index first
 * among equals, with e = exp((logit - largest) / temperature):
 *
 *   top-k keeps the first top_k tokens (all for top_k <= 0); S = what their e sum to
 *   top-p keeps those before which less than top_p * S lies (all for top_p >= 1), and always the first
 *   min-p keeps those with e >= min_p (all for min_p <= 0)
 *   token = the y with the largest e(y) / noise(y) of the kept, the lowest such y
 *   prob  = e(token) / the kept tokens' sum: the probability that it was drawn with
 *
 * The race is in fp32: an e below 2^-126 may count as 0 there and cannot win then, quotients past fp32's range are all infinite.
 * With exponential noise of mean 1 tokens are distributed as the filtered probabilities.  Temperature 0 takes the
 * largest logit, whatever the noise.  A row of logits that is no distribution (as for mb_verify_sample) gives token -1 and
 * prob 0; so does a row whose noise lets no token win.  -infinity masks a token.
 *
 *   temperature, top_k, top_p, min_p   for every sequence: temperature 0, or > 2^-127 and finite; top_p
 *                  not NaN; min_p <= 1 (MB_ERR_UNSUPPORTED otherwise)
 *   temperatures, top_ks, top_ps, min_ps   float (top_ks: int32) (batch) DEVICE memory: one for each sequence instead;
 *                  a sequence for which they are out of those ranges gives token -1 and prob 0.  NULL: the ones above
 *   logits         act (batch, vocab)
 *   noise          float (batch, vocab)
 *   token          int32 (batch)
 *   prob           float (batch)      NULL means not written
 * Outputs overlap nothing else.  vocab >= 1, below 2^30; batch below 2^22.
 */
int mb_sample(int64_t batch, int64_t vocab, int32_t logit_dtype, float temperature, int32_t top_k, float top_p, float min_p,
              const float *temperatures, const int32_t *top_ks, const float *top_ps, const float *min_ps, const void *logits,
              const float *noise, int32_t *token, float *prob, void *stream);

/* Static, NUL-terminated description of a status code (never NULL). */
const char *mb_status_string(int status);

/* MB_ABI_VERSION of the built library. */
int mb_abi_version(void);

#ifdef __cplusplus
}
#endif

#endif /* MBSCAN_H */
