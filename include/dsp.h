/*
 * dsp.h -- C ABI of libdsp: one GPU's share of a Dynamic Sequence Parallelism
 * (DSP) spatial-temporal transformer block on AMD MI355X (gfx950).
 *
 * The operations follow "DSP: Dynamic Sequence Parallelism for
 * Multi-Dimensional Transformers" (Zhao et al., ICML 2025):
 *   - the Switch primitive (primitive table, row s_i -> s_j; Eq. 10), here
 *     the local permute + pack of one GPU's shard that precedes the exchange;
 *   - scaled dot-product attention (Eq. 3), per head (Eq. 1-2), run along one
 *     sequence dimension of a multi-dimensional sequence (Eq. 7-8): spatial
 *     attention over S inside each frame, temporal attention over T at each
 *     spatial location;
 *   - the LayerNorm (Eq. 4, 6), linear maps and MLP (Eq. 5) of the block.
 *
 * Conventions shared by every entry point
 *   - All tensor arguments are DEVICE pointers owned by the caller.  The
 *     library allocates nothing, keeps no pointer after returning and holds no
 *     mutable global state; calls are thread-safe.  The one exception is
 *     dsp_attn_bwd_noalloc, whose scratch is a static per-device array (calls
 *     that overlap on one GPU race on it).
 *   - Work is enqueued asynchronously on `stream` (a hipStream_t passed as an
 *     opaque pointer; NULL means the default stream).  Device faults surface at
 *     the caller's next synchronisation.
 *   - Arguments are validated on the host before anything is launched; a
 *     failed check returns a nonzero dsp_status_t and launches nothing.  A
 *     launch failure returns DSP_ERR_HIP.  No C++ exception crosses the ABI.
 *   - Tensors are dense row-major.  Sequence tensors are [B, S_1, S_2, C]
 *     (C innermost); dimension numbers follow that order: 0 = batch,
 *     1 and 2 = the two sequence dimensions, 3 = hidden.
 *   - Weights of linear maps are stored [out][in] (row-major, the reduction
 *     index contiguous), i.e. y = x * W with W = stored^T.
 */
#ifndef DSP_H_
#define DSP_H_

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  DSP_OK = 0,
  DSP_ERR_NULL = 1,      /* a required pointer is NULL */
  DSP_ERR_DIM = 2,       /* bad ndim or dimension index */
  DSP_ERR_SHAPE = 3,     /* nonpositive / non-divisible / unsupported size */
  DSP_ERR_DTYPE = 4,     /* unknown or unsupported dtype */
  DSP_ERR_ALIGN = 5,     /* pointer or stride alignment the kernel requires */
  DSP_ERR_HIP = 6,       /* a HIP runtime call or kernel launch failed */
  DSP_ERR_WORKSPACE = 7, /* workspace missing or too small */
  DSP_ERR_ARG = 8        /* any other invalid argument (flags, eps, ...) */
} dsp_status_t;

/* DSP_E4M3: caches of dsp_kv_append and dsp_attn_paged only. */
typedef enum { DSP_F32 = 0, DSP_BF16 = 1, DSP_E4M3 = 2 } dsp_dtype_t;

/* Human-readable name of a status code (static string, never NULL). */
const char* dsp_status_str(int status);

/* Library version as MAJOR*10000 + MINOR*100 + PATCH. */
int dsp_version(void);

/* ------------------------------------------------------------------------
 * dsp_switch -- one GPU's share of DynamicSwitch(X, i, j)
 * (primitive table, row s_i -> s_j; Eq. 10; system overview figure).
 *
 * x:      [B, D1, D2, C] (ndim 4: K = 2 sequence dimensions) or
 *         [B, D1, D2, D3, C] (ndim 5: K = 3, the multi-dimensional form of
 *         Eq. 7), the local shard, currently sharded on `from_dim`.
 * y:      output, same number of elements as x, written as `n_chunks`
 *         contiguous per-destination chunks.  With from_dim=1, to_dim=2:
 *             y[n][b][j'][i][c] = x[b][i][n*D2/n_chunks + j'][c]
 *         (chunk n has shape [B, D2/n_chunks, D1, C]: the to-dim slice
 *         outermost, the from-dim -- the dimension the next stage computes
 *         over -- innermost before C).  With from_dim=2, to_dim=1:
 *             y[n][b][i'][j][c] = x[b][n*D1/n_chunks + i'][j][c].
 *         For (B,T,S,C) with T sharded, from=1 (T), to=2 (S) and n_chunks=1
 *         this is the permute to (B,S,T,C).  Chunk n is what rank n receives
 *         in the all-to-all; the exchange itself is not part of this call.
 *         For K = 3 the chunk keeps the other two sequence dimensions in
 *         their order (the to-dim cut to D_to/n_chunks) and puts the from-dim
 *         next to C, e.g. from=1, to=3:
 *             y[n][b][j][k'][i][c] = x[b][i][j][n*D3/n_chunks + k'][c].
 * from_dim == to_dim is the "no primitive" row of the table: y = copy of x.
 * Errors: DSP_ERR_NULL (shape NULL, or x / y NULL for a non-empty tensor;
 *   an empty tensor may come with NULL pointers), DSP_ERR_DIM (ndim not 4 or 5,
 *   or a dim not in 1..K), DSP_ERR_SHAPE (a size < 0, n_chunks < 1, the to-dim not
 *   divisible by n_chunks, or more than 2^31 rows / 16-byte vectors),
 *   DSP_ERR_DTYPE, DSP_ERR_ARG (x and y overlap).  A tensor with a zero size
 *   is accepted and launches nothing.
 * The data are moved as raw bits (bit-exact for any payload, NaNs included).
 * ------------------------------------------------------------------------ */
int dsp_switch(const void* x, void* y, const int64_t* shape, int ndim, int from_dim, int to_dim,
               int n_chunks, int dtype, void* stream);

/* Same as dsp_switch with an explicit kernel choice: 0 = automatic,
 * 1 = direct 128-bit row copy (requires 16-byte aligned pointers and rows),
 * 2 = LDS-staged tile transpose.  Any other value -> DSP_ERR_ARG.  K = 3
 * tensors (ndim 5) have one kernel: only variant 0 is accepted. */
int dsp_switch_variant(const void* x, void* y, const int64_t* shape, int ndim, int from_dim,
                       int to_dim, int n_chunks, int dtype, int variant, void* stream);

/* ------------------------------------------------------------------------
 * dsp_split -- the Split row of the primitive table (s^ -> s_i): a tensor
 * replicated on every rank becomes sharded on sequence dimension `dim`, with
 * no communication; rank `rank` keeps its slice.
 *
 * x:      [B, S_1, .., S_K, C] (ndim = K + 2, K = 2 or 3), replicated.
 * y:      [B, .., S_dim / n_chunks, .., C], dense:
 *             y[b][..][i'][..][c] = x[b][..][rank * S_dim/n_chunks + i'][..][c].
 * Errors: DSP_ERR_NULL, DSP_ERR_DIM (ndim not 4 or 5, dim not in 1..K),
 *   DSP_ERR_SHAPE (a negative size, n_chunks < 1, S_dim not divisible),
 *   DSP_ERR_DTYPE, DSP_ERR_ARG (rank not in [0, n_chunks), x and y overlap).
 * A bit copy; an empty result launches nothing.
 * ------------------------------------------------------------------------ */
int dsp_split(const void* x, void* y, const int64_t* shape, int ndim, int dim, int n_chunks,
              int rank, int dtype, void* stream);

/* ------------------------------------------------------------------------
 * dsp_gather -- the Gather row of the primitive table (s_i -> s^, an
 * all-gather): the receiver's concatenation of every rank's shard, run on
 * one GPU with one buffer per rank.
 *
 * shards:      host array of n_shards device pointers, each a dense
 *              [B, S_1, .., S_K, C] shard with the size shard_shape
 *              (ndim = K + 2, K = 2 or 3); they may alias each other.
 * y:           [B, .., n_shards * S_dim, .., C], dense:
 *                  y[b][..][m * S_dim + i][..][c] = shards[m][b][..][i][..][c].
 * n_shards:    1..64.
 * Errors: DSP_ERR_NULL, DSP_ERR_DIM, DSP_ERR_SHAPE (a negative size, n_shards
 *   out of range), DSP_ERR_DTYPE, DSP_ERR_ARG (y overlaps a shard).
 * A bit copy; an empty result launches nothing.
 * ------------------------------------------------------------------------ */
int dsp_gather(const void* const* shards, void* y, const int64_t* shard_shape, int ndim, int dim,
               int n_shards, int dtype, void* stream);

/* ------------------------------------------------------------------------
 * dsp_exchange_unpack -- the exchange of DynamicSwitch among N ranks (the
 * all-to-all of the primitive table's row s_i -> s_j, Eq. 10), run on one GPU
 * with one buffer per rank, fused with every receiver's unpack.
 *
 * packed: host array of N device pointers; packed[m] is rank m's dsp_switch
 *         output, shape [N][B][P][F][C] (P = D_to / N, F = rank m's length of
 *         the from-dimension; for K = 3, P is the product of the two other
 *         sequence dimensions of a chunk).  Read only; the N buffers may alias
 *         each other.
 * out:    host array of N device pointers; out[n] receives rank n's result,
 *         shape [B][P][N*F][C]:
 *             out[n][b][p][m*F + f][c] = packed[m][n][b][p][f][c]
 *         i.e. chunk n of every rank, concatenated along the from-dimension
 *         in rank order.  For the (B,T,S,C) -> (B,S,T,C) switch of T-shards
 *         this is S-shard n of the permuted tensor (Eq. 7-8, i = T).
 * shape:  {N, B, P, F, C}.  dtype: element type (only its size matters; the
 *         data move as raw bits).
 * The caller owns all buffers; N*(B*P*F*C) elements per buffer.
 * Errors: DSP_ERR_NULL (shape NULL, or a pointer array / pointer NULL for a
 *   non-empty exchange), DSP_ERR_SHAPE (N < 1, N > 64, a negative size, or a
 *   size overflow), DSP_ERR_DTYPE, DSP_ERR_ARG (an output buffer overlaps a
 *   packed buffer or another output buffer).  An empty exchange launches
 *   nothing.
 * ------------------------------------------------------------------------ */
int dsp_exchange_unpack(const void* const* packed, void* const* out, const int64_t* shape,
                        int dtype, void* stream);

/* ------------------------------------------------------------------------
 * Attention along one sequence dimension (Eq. 3 per head, Eq. 1-2; the
 * per-dimension reshape of Eq. 7-8).  Non-causal softmax(q k^T * scale) v.
 *
 * dsp_spatial_attn:  q, k, v, o laid out (B, T, S, *), attention over L = S
 *   inside each (b, t) frame, independently per head h.
 * dsp_temporal_attn: q, k, v, o laid out (B, S, T, *), attention over L = T at
 *   each (b, s) location, independently per head.
 *
 * Head h of a token occupies elements [h*D, (h+1)*D) of that token's row.
 * ld_in:  elements between consecutive token rows of q, k and v (C = H*D for
 *         separate tensors, 3C when q/k/v point into one packed [Q|K|V] buffer).
 * ld_out: elements between consecutive token rows of o (>= H*D).
 * scale:  softmax scale; scale <= 0 selects 1/sqrt(D) with the true D.
 * dtype:  DSP_BF16 (bf16 storage, bf16 MFMA, fp32 softmax and accumulation)
 *         or DSP_F32 (fp32 storage and fp32 arithmetic throughout).
 * Supported D: DSP_BF16 -- D in {16, 32, 64, 72, 80, 96}; DSP_F32 --
 *   1 <= D <= 256.  bf16 needs 16-byte aligned q/k/v/o and ld_in, ld_out
 *   multiples of 8 (DSP_ERR_ALIGN otherwise).
 * Errors: DSP_ERR_NULL, DSP_ERR_SHAPE (a size < 0, H < 1, D < 1, H*D > ld,
 *   unsupported D), DSP_ERR_DTYPE, DSP_ERR_ALIGN, DSP_ERR_ARG (scale NaN or
 *   infinite), DSP_ERR_HIP.  An empty input (B, T or S equal to 0) is
 *   accepted, may come with NULL pointers, and launches nothing.
 * ------------------------------------------------------------------------ */
int dsp_spatial_attn(const void* q, const void* k, const void* v, void* o, int64_t B, int64_t T,
                     int64_t S, int H, int D, int64_t ld_in, int64_t ld_out, float scale,
                     int dtype, void* stream);
int dsp_temporal_attn(const void* q, const void* k, const void* v, void* o, int64_t B, int64_t S,
                      int64_t T, int H, int D, int64_t ld_in, int64_t ld_out, float scale,
                      int dtype, void* stream);

/* Attention with explicit layouts: the same operation over L positions of
 * each (b, x, h) unit, element (b, x, l, h*D + d) of q/k/v at
 *     b*in_strides[0] + x*in_strides[1] + l*in_strides[2] + h*D + d
 * and of o at the same offsets with out_strides (strides in elements).  This
 * reads a layout the previous stage left behind without a switch, e.g.
 * temporal attention straight from (B, T, S, C): X = S, L = T, in_strides =
 * {T*S*C, C, S*C} (Eq. 7-8 with i = T, computed on the unswitched tensor).
 * dsp_spatial_attn and dsp_temporal_attn are this call with the strides of
 * their dense layouts.  Requirements and errors as for dsp_spatial_attn, plus:
 * strides must be >= 0 (DSP_ERR_SHAPE), the output rows must not overlap
 * (checked: DSP_ERR_ARG), and for DSP_BF16 every stride a multiple of 8
 * elements and min(L, 64) * in_strides[2] * 2 < 2^31 (DSP_ERR_ALIGN /
 * DSP_ERR_SHAPE).  o must not overlap q, k or v. */
int dsp_attn_strided(const void* q, const void* k, const void* v, void* o, int64_t B, int64_t X,
                     int64_t L, int H, int D, const int64_t* in_strides, const int64_t* out_strides,
                     float scale, int dtype, void* stream);

/* ------------------------------------------------------------------------
 * dsp_attn_fwd_lse -- dsp_attn_strided that also saves, for every query, the
 * natural-log log-sum-exp of its scaled scores,
 *     lse[u][i] = log sum_j exp(scale * q_i . k_j),
 * the row statistic of the softmax in Eq. 3 that the backward pass needs to
 * recompute the probabilities.  Used for training, which the paper's models
 * undergo (its weak-scaling runs are a training stage, with ZeRO-2).
 * lse: DEVICE fp32 [B * X * H][L], unit u = (b * X + x) * H + h, caller-owned,
 *   4-byte aligned (DSP_ERR_ALIGN), required unless the input is empty
 *   (DSP_ERR_NULL).  The bf16 kernels compute it from the same bf16-rounded
 *   scores and probabilities that produce o.
 * Everything else, including errors, as for dsp_attn_strided.
 * ------------------------------------------------------------------------ */
int dsp_attn_fwd_lse(const void* q, const void* k, const void* v, void* o, float* lse, int64_t B,
                     int64_t X, int64_t L, int H, int D, const int64_t* in_strides,
                     const int64_t* out_strides, float scale, int dtype, void* stream);

/* ------------------------------------------------------------------------
 * dsp_attn_bwd -- gradient of attention along one sequence dimension (Eq. 3
 * per head, Eq. 1-2; any layout as in dsp_attn_strided) by the chain rule
 * through the softmax.  With z = scale * q.k, P = softmax(z) per row and
 * Delta_i = sum_d dout[i][d] * o[i][d]:
 *     dv = P^T dout,  dz = P * (dout v^T - Delta),
 *     dq = scale * dz k,  dk = scale * dz^T q.
 * q, k, v: the forward's inputs; o, lse: its outputs (dsp_attn_fwd_lse);
 *   dout: the gradient of the loss with respect to o.
 * dq, dk, dv: outputs, same shapes and strides as q, k, v (qkv_strides), so
 *   gradients of a packed [Q|K|V] buffer land in a packed buffer.
 * o, dout: element (b, x, l, h*D + d) at b*o_strides[0] + x*o_strides[1] +
 *   l*o_strides[2] + h*D + d.
 * delta: DEVICE fp32 workspace [B * X * H][L]; on return it holds Delta.
 * All pointers are DEVICE pointers owned by the caller; dq, dk, dv must not
 *   overlap each other or any input, and delta must not overlap lse
 *   (checked: DSP_ERR_ARG).
 * dtype DSP_BF16: bf16 tensors, fp32 accumulation on the matrix cores; D in
 *   {16, 32, 64, 72, 80, 96}; 16-byte aligned tensors and strides that are
 *   multiples of 8 (DSP_ERR_ALIGN); 64 * qkv_strides[2] * 2 and
 *   64 * o_strides[2] * 2 below 2^31 (DSP_ERR_SHAPE).  Deterministic: no
 *   atomics, so repeated calls give identical bits.
 * dtype DSP_F32: fp32 products and accumulation throughout; 1 <= D <= 256.
 * scale <= 0 selects 1/sqrt(D).  An empty input launches nothing.
 * Errors: DSP_ERR_NULL, DSP_ERR_SHAPE, DSP_ERR_DTYPE, DSP_ERR_ALIGN,
 *   DSP_ERR_ARG (scale not finite, overlapping gradient rows), DSP_ERR_HIP.
 * ------------------------------------------------------------------------ */
int dsp_attn_bwd(const void* q, const void* k, const void* v, const void* o, const void* dout,
                 const float* lse, void* dq, void* dk, void* dv, float* delta, int64_t B, int64_t X,
                 int64_t L, int H, int D, const int64_t* qkv_strides, const int64_t* o_strides,
                 float scale, int dtype, void* stream);

/* ------------------------------------------------------------------------
 * dsp_attn_bwd_noalloc -- dsp_attn_bwd for callers that cannot allocate
 * device memory: code under HIP graph capture, tight serving loops, harnesses
 * that forbid hipMalloc.  It takes no `delta` workspace: the Delta rows live in
 * a library-owned static device array of dsp_attn_bwd_noalloc_max_rows()
 * fp32 values (4194304 values, 16 MiB), one copy per GPU, loaded with the
 * library's code and held until the process ends.  The call allocates nothing
 * (no hipMalloc, hipFree or allocating library routine); its first call on a
 * device looks up that device's copy (hipGetSymbolAddress).
 * Every call on one GPU uses that GPU's array, and its contents are those of
 * the last call: calls that overlap on one GPU (several streams or host
 * threads) race and must be serialised by the caller.  Delta is not returned.
 * B * X * H * L above the maximum: DSP_ERR_WORKSPACE, nothing launched.
 * Everything else -- arguments, layouts, dtypes, errors and the bits of dq,
 * dk, dv -- as dsp_attn_bwd.
 * ------------------------------------------------------------------------ */
int64_t dsp_attn_bwd_noalloc_max_rows(void);
int dsp_attn_bwd_noalloc(const void* q, const void* k, const void* v, const void* o, const void* dout,
                         const float* lse, void* dq, void* dk, void* dv, int64_t B, int64_t X, int64_t L, int H,
                         int D, const int64_t* qkv_strides, const int64_t* o_strides, float scale, int dtype,
                         void* stream);

/* ------------------------------------------------------------------------
 * dsp_attn_general / dsp_attn_general_bwd -- the attention variants the
 * paper states DSP is compatible with: multi-query and grouped-query attention
 * (Hkv key/value heads shared by H / Hkv query heads each) and cross-attention
 * (keys and values from another sequence, of their own length), on the same
 * per-(b, x) units as dsp_attn_strided.  For unit (b, x, h):
 *   queries: Lq positions, element (b, x, l, h*D + d) of q at
 *            b*q_strides[0] + x*q_strides[1] + l*q_strides[2] + h*D + d;
 *   keys, values: Lk positions of head h / (H / Hkv), at
 *            b*kv_strides[0] + x*kv_strides[1] + l*kv_strides[2] + (h/(H/Hkv))*D + d;
 *   output (and dout): o_strides, H heads, Lq positions.
 * Hkv == H, Lq == Lk and kv_strides == q_strides is dsp_attn_strided.  A
 * kv stride of 0 broadcasts keys and values (e.g. one text sequence shared
 * by every frame: kv_strides[1] = 0); the backward rejects it (its key and
 * value gradients would have no single owner: DSP_ERR_ARG).
 * lse (forward, optional: NULL skips it): fp32 [B * X * H][Lq].  The
 * backward's contract (lse, delta [B*X*H][Lq], dq with q's strides, dk and dv
 * with kv_strides -- the sums over each group's query heads) is otherwise
 * dsp_attn_bwd's.  H % Hkv != 0, or Lk == 0 with Lq > 0: DSP_ERR_SHAPE.
 * Everything else, including dtypes, alignment and errors, as for
 * dsp_attn_strided / dsp_attn_bwd.
 * ------------------------------------------------------------------------ */
int dsp_attn_general(const void* q, const void* k, const void* v, void* o, float* lse, int64_t B, int64_t X,
                     int64_t Lq, int64_t Lk, int H, int Hkv, int D, const int64_t* q_strides,
                     const int64_t* kv_strides, const int64_t* o_strides, float scale, int dtype, void* stream);
int dsp_attn_general_bwd(const void* q, const void* k, const void* v, const void* o, const void* dout,
                         const float* lse, void* dq, void* dk, void* dv, float* delta, int64_t B, int64_t X,
                         int64_t Lq, int64_t Lk, int H, int Hkv, int D, const int64_t* q_strides,
                         const int64_t* kv_strides, const int64_t* o_strides, float scale, int dtype,
                         void* stream);

/* ------------------------------------------------------------------------
 * dsp_qk_norm_rope -- queries and keys made ready for attention: the root mean
 * square norm of each head with a learned gain, and the rotation by position, in
 * one pass.  For each token (b, x, l) and head, u of width D:
 *     n = g * u / sqrt(mean(u^2) + eps),
 *     y = n with its first `rot` elements turned in pairs (n_a, n_b):
 *         y_a = n_a cos - n_b sin,  y_b = n_b cos + n_a sin,
 * cos and sin at row p of the table, column i for pair i < rot / 2.
 * q:      H heads, element (b, x, l, h*D + d) at b*q_strides[0] + x*q_strides[1]
 *         + l*q_strides[2] + h*D + d; k: Hkv heads with k_strides; yq, yk:
 *         outputs of the same shapes with strides of their own.  In place
 *         (yq == q or yk == k with equal strides) is allowed; k and yk may be
 *         columns of q's or yq's buffer ([Q | K | V]), any other overlap is
 *         DSP_ERR_ARG.  Hkv = 0: queries only (k, yk, gk unused); H = 0 keys only.
 * gq, gk: gains [D] of dtype, or NULL (1).
 * cos, sin: DEVICE fp32 [P][rot / 2]; unused when rot is 0.
 * pos:    DEVICE int32 [B][L], the table's row of each token, or NULL (row l,
 *         L <= P).  A token whose position has no row (outside 0 .. P - 1) gets
 *         NaN in the elements that turn; nothing outside the table is read.
 * rot:    even, 0 .. D.  flags: 0 pairs element i with i + rot/2,
 *         DSP_ROPE_ADJACENT pairs 2i with 2i + 1.
 * Arithmetic is fp32, each output is rounded once.  D is 1 .. 256 for both
 * dtypes at any alignment of an element; 16-byte aligned tensors and tables, with
 * strides, D and rot multiples of 16 bytes, are fastest.
 *
 * dsp_qk_norm_rope_bwd -- its gradient: with dn the turn back of dy and w = g dn,
 *     dg = sum over tokens and heads of dn * u * r,  r = 1/sqrt(mean(u^2) + eps),
 *     du = r (w - u r^2 mean(w u)).
 *   dq and dk may be in place of dyq and dyk, or of q and k (equal strides).  A token
 *   whose position has no row makes its rows of them and the sums dg NaN, whatever its dy:
 *   padding takes any row of the table.
 *   dgq, dgk: fp32 [D], or NULL.  workspace: at least
 *   dsp_qk_norm_rope_bwd_workspace_bytes(B, X, L, H, Hkv, D) bytes, 16-byte
 *   aligned, needed when dgq or dgk is given.  Deterministic.
 * Outputs and the workspace lie apart from gains, tables and positions too, and from one
 * another (DSP_ERR_ARG); dgq, dgk and the workspace may lie in gaps between rows.
 * Errors: DSP_ERR_NULL, DSP_ERR_SHAPE (a size < 0, D outside 1 .. 256, no heads,
 *   rot odd or past D, P < 1 or (pos NULL) P < L with rot > 0, 2^31 rows of
 *   B X L heads or more), DSP_ERR_DTYPE, DSP_ERR_ALIGN (off an element),
 *   DSP_ERR_ARG (eps < 0 or not finite, unknown flags, overlapping outputs),
 *   DSP_ERR_WORKSPACE, DSP_ERR_HIP.  An empty input launches nothing and may come
 *   with NULL pointers; the gradient then writes dgq = dgk = 0.
 * ------------------------------------------------------------------------ */
enum { DSP_ROPE_ADJACENT = 1 };
int dsp_qk_norm_rope(const void* q, const void* k, void* yq, void* yk, const void* gq, const void* gk,
                     const float* cos, const float* sin, const int32_t* pos, int64_t P, int rot, int flags, int64_t B,
                     int64_t X, int64_t L, int H, int Hkv, int D, const int64_t* q_strides, const int64_t* k_strides,
                     const int64_t* yq_strides, const int64_t* yk_strides, float eps, int dtype, void* stream);
size_t dsp_qk_norm_rope_bwd_workspace_bytes(int64_t B, int64_t X, int64_t L, int H, int Hkv, int D);
int dsp_qk_norm_rope_bwd(const void* q, const void* k, const void* dyq, const void* dyk, void* dq, void* dk,
                         float* dgq, float* dgk, const void* gq, const void* gk, const float* cos, const float* sin,
                         const int32_t* pos, int64_t P, int rot, int flags, void* workspace, size_t ws_bytes,
                         int64_t B, int64_t X, int64_t L, int H, int Hkv, int D, const int64_t* q_strides,
                         const int64_t* k_strides, const int64_t* dyq_strides, const int64_t* dyk_strides,
                         const int64_t* dq_strides, const int64_t* dk_strides, float eps, int dtype, void* stream);

/* ------------------------------------------------------------------------
 * dsp_attn_relpos -- attention with a learned relative position bias by buckets:
 *     s_ij = scale * q_i . k_j + bias[bucket(j - i - q_pos)][h],
 *     o_i = softmax over j (s_i) v,
 * on the units, heads and layouts of dsp_attn_general (Hkv key/value heads shared
 * by H / Hkv query heads each, lengths Lq and Lk, any strides, 0 to broadcast keys
 * and values; k and v have one layout, not one buffer: values may stay in a packed
 * projection while normalised keys lie in another buffer of its strides).
 * bias:    [n_buckets][H] of dtype.  A value of -1e30 or less (-inf, or the type's
 *          lowest) takes the keys of its distances out.
 * buckets: DEVICE int32 [2 * max_dist + 1], the bucket of each distance
 *          -max_dist .. max_dist (key position - query position); further
 *          distances take the nearest end's.  An entry outside
 *          0 .. n_buckets - 1 means no bias.  dsp_relpos_buckets fills the usual
 *          map.
 * q_pos:   DEVICE int32 [B], the key index of each sequence's first query (a new
 *          token's place in a cache), or NULL (0).
 * kv_len:  DEVICE int32 [B], the keys that each sequence has, 0 .. Lk (clamped),
 *          or NULL (Lk).  Keys and values past it are never used, whatever they
 *          hold; the others must be finite.
 * flags:   DSP_RELPOS_CAUSAL keeps the keys j <= i + q_pos only.
 * scale:   softmax scale; scale <= 0 selects 1/sqrt(D).
 * A query without keys (kv_len 0, or none before it) gives o = 0 and lse = -inf.  A
 * query that is not finite makes its own row of o and its lse NaN; a unit's gradients
 * are NaN where a query or a row of dout of theirs is not finite, no other unit's.
 * lse:     fp32 [B * X * H][Lq], the row log-sum-exp of s, or NULL.
 * dtype:   DSP_BF16 (fp32 scores, softmax and accumulation; probabilities are
 *          rounded to bf16 for the product with v), D a multiple of 8 up to 128,
 *          16-byte aligned tensors and strides multiples of 8; or DSP_F32, any D up
 *          to 128.  max_dist <= 1024, Lq and Lk below 2^30, and 64 rows of each tensor
 *          within 2^31 bytes.
 * workspace: dsp_attn_relpos_workspace_bytes(...) bytes, 16-byte aligned (0 except
 *          for a few queries against many keys: there the keys are cut among
 *          work-groups, whose sums are joined).
 *
 * dsp_attn_relpos_bwd -- the gradients dq, dk, dv (strides of q and k) and
 * dbias [n_buckets][H] of dtype, from the forward's o and lse and from dout (o's
 * strides; DSP_BF16 takes o's address but none of its values).  Deterministic: no sum
 * depends on timing.  Rows of dk and dv past kv_len
 * are 0, as is dbias where bias masks.  workspace:
 * dsp_attn_relpos_bwd_workspace_bytes(...) bytes, 16-byte aligned.  dq, dk and dv
 * may be columns of one buffer; broadcast keys are DSP_ERR_ARG.
 * In both calls every output, lse, dbias and the workspace among them, lies apart from
 * everything else that the call reads or writes (DSP_ERR_ARG); lse, dbias and the
 * workspace may lie in gaps between rows.
 *
 * dsp_relpos_buckets -- fills buckets[2 * max_dist + 1] in HOST memory: with
 * n = n_buckets (bidirectional: half of them for each direction, keys after the
 * query in the second half; otherwise keys after the query share bucket 0),
 * distances below n / 2 have a bucket each, and the other buckets divide
 * n / 2 .. max_dist evenly in the logarithm.
 * Errors: DSP_ERR_NULL, DSP_ERR_SHAPE (sizes < 0 or unsupported, H % Hkv,
 *   n_buckets < 1), DSP_ERR_DTYPE, DSP_ERR_ALIGN, DSP_ERR_ARG (scale not finite,
 *   unknown flags, overlapping outputs), DSP_ERR_WORKSPACE, DSP_ERR_HIP.  An empty
 *   input launches nothing and may come with NULL pointers (the gradient of no
 *   queries writes 0 into dk, dv and dbias).
 * ------------------------------------------------------------------------ */
enum { DSP_RELPOS_CAUSAL = 1 };
int dsp_relpos_buckets(int32_t* buckets, int max_dist, int n_buckets, int bidirectional);
size_t dsp_attn_relpos_workspace_bytes(int64_t B, int64_t X, int64_t Lq, int64_t Lk, int H, int Hkv, int D,
                                       int dtype);
int dsp_attn_relpos(const void* q, const void* k, const void* v, void* o, float* lse, const void* bias,
                    const int32_t* buckets, int n_buckets, int max_dist, const int32_t* q_pos,
                    const int32_t* kv_len, int flags, void* workspace, size_t ws_bytes, int64_t B, int64_t X,
                    int64_t Lq, int64_t Lk, int H, int Hkv, int D, const int64_t* q_strides,
                    const int64_t* kv_strides, const int64_t* o_strides, float scale, int dtype, void* stream);
size_t dsp_attn_relpos_bwd_workspace_bytes(int64_t B, int64_t X, int64_t Lq, int64_t Lk, int H, int Hkv, int D,
                                           int max_dist, int dtype);
int dsp_attn_relpos_bwd(const void* q, const void* k, const void* v, const void* o, const void* dout,
                        const float* lse, void* dq, void* dk, void* dv, void* dbias, const void* bias,
                        const int32_t* buckets, int n_buckets, int max_dist, const int32_t* q_pos,
                        const int32_t* kv_len, int flags, void* workspace, size_t ws_bytes, int64_t B, int64_t X,
                        int64_t Lq, int64_t Lk, int H, int Hkv, int D, const int64_t* q_strides,
                        const int64_t* kv_strides, const int64_t* o_strides, float scale, int dtype, void* stream);

/* ------------------------------------------------------------------------
 * dsp_attn_window -- attention with a window to either side of a query and first
 * tokens that stay visible (sinks), on the units, heads and layouts of
 * dsp_attn_general (any strides, 0 to broadcast keys and values; k and v have one
 * layout, not one buffer).  The query i of sequence b, at position p = i + q_pos[b],
 * sees the keys j < kv_len[b] with
 *     j <= p + right  (right < 0: no bound; 0: causal)  and
 *     j >= p - left   (left < 0: no bound)  or  j < sinks,
 * and o_i = softmax over those j (scale * q_i . k_j) v.
 * q_pos:   DEVICE int32 [B], the key index of each sequence's first query, or NULL (0).
 * kv_len:  DEVICE int32 [B], the keys that each sequence has, 0 .. Lk (clamped),
 *          or NULL (Lk).
 * A query that sees nothing gives o = 0 and lse = -inf.  Keys and values that no query
 * of their sequence sees are never used, whatever they hold; a key or value that is not
 * finite makes the queries that see it NaN and may make any other of its unit so (an infinite
 * key may also count as the softmax has it), a query that is not finite its own row.  A
 * unit's gradients may be NaN where a row of q or dout of theirs, or a key or value that is
 * seen, is not finite; no other unit's are.
 * lse:     fp32 [B * X * H][Lq], the row log-sum-exp of the scaled scores, or NULL.
 * scale:   softmax scale; scale <= 0 selects 1/sqrt(D).
 * dtype:   DSP_BF16 (fp32 scores, softmax and accumulation; probabilities are rounded to
 *          bf16 for the product with v, whose sums may be held at 2^-16 of their size:
 *          values below 2^-110 may lose bits), D a multiple of 8 up to 128, 16-byte aligned
 *          tensors and strides multiples of 8; or DSP_F32, any D up to 128.  Lq and Lk
 *          below 2^30, H / Hkv below 2^15, Lq * H / Hkv below 2^31, and 64 rows of each tensor within 2^31 bytes.
 * workspace: dsp_attn_window_workspace_bytes(...) bytes, 16-byte aligned (0 except for a
 *          few queries against many keys: there the keys are cut among work-groups, whose
 *          sums are joined).  Calls that may run at once, captured ones among them, have
 *          workspaces of their own.
 *
 * dsp_attn_window_bwd -- the gradients dq, dk, dv (strides of q and k) from the forward's
 * o and lse and from dout (o's strides).  Deterministic.  Rows of dk and dv that no query
 * sees are 0, as are rows of dq that see nothing.  workspace:
 * dsp_attn_window_bwd_workspace_bytes(...) bytes, 16-byte aligned.  dq, dk and dv may be
 * columns of one buffer; broadcast keys are DSP_ERR_ARG.
 * In both calls every output and the workspace lies apart from everything else that the
 * call reads or writes (DSP_ERR_ARG); lse and the workspace may lie in gaps between rows.
 * Errors: DSP_ERR_NULL, DSP_ERR_SHAPE (sizes < 0 or unsupported, H % Hkv),
 *   DSP_ERR_DTYPE, DSP_ERR_ALIGN, DSP_ERR_ARG (scale not finite, sinks < 0, overlapping
 *   outputs), DSP_ERR_WORKSPACE, DSP_ERR_HIP.  An empty input launches nothing and may
 *   come with NULL pointers (the gradient of no queries writes 0 into dk and dv).
 * ------------------------------------------------------------------------ */
size_t dsp_attn_window_workspace_bytes(int64_t B, int64_t X, int64_t Lq, int64_t Lk, int H, int Hkv, int D, int left,
                                       int right, int sinks, int dtype);
int dsp_attn_window(const void* q, const void* k, const void* v, void* o, float* lse, const int32_t* q_pos,
                    const int32_t* kv_len, int left, int right, int sinks, void* workspace, size_t ws_bytes, int64_t B,
                    int64_t X, int64_t Lq, int64_t Lk, int H, int Hkv, int D, const int64_t* q_strides,
                    const int64_t* kv_strides, const int64_t* o_strides, float scale, int dtype, void* stream);
size_t dsp_attn_window_bwd_workspace_bytes(int64_t B, int64_t X, int64_t Lq, int64_t Lk, int H, int Hkv, int D, int left,
                                           int right, int sinks, int dtype);
int dsp_attn_window_bwd(const void* q, const void* k, const void* v, const void* o, const void* dout, const float* lse,
                        void* dq, void* dk, void* dv, const int32_t* q_pos, const int32_t* kv_len, int left, int right,
                        int sinks, void* workspace, size_t ws_bytes, int64_t B, int64_t X, int64_t Lq, int64_t Lk, int H,
                        int Hkv, int D, const int64_t* q_strides, const int64_t* kv_strides, const int64_t* o_strides,
                        float scale, int dtype, void* stream);

/* ------------------------------------------------------------------------
 * A paged cache of keys and values: n_pages pages of `page` slots (a power of two, 16 ..
 * 1024), element (page, slot, head h, d) at page*cache_strides[0] + slot*cache_strides[1]
 * + h*cache_strides[2] + d of k_cache and of v_cache (one layout; the two may interleave
 * in one buffer).  Position j of sequence n lies in slot j % page of page
 * table[n][j / page].
 * table:    DEVICE int32 [N][max_pages].  An entry outside 0 .. n_pages - 1 is no page:
 *           its keys are not seen and tokens for it are dropped (a page given back, or not
 *           yet needed).  Nothing outside the caches is read or written.  A cache may have no
 *           pages at all (n_pages 0, NULL caches and scales).
 * q_start:  DEVICE int32 [N + 1], rising: rows q_start[n] .. q_start[n + 1] - 1 of the T
 *           packed rows are sequence n's new tokens.  Values outside 0 .. T are clamped.
 * kv_len:   DEVICE int32 [N], the positions of each sequence, the new tokens being the
 *           last of them: its row i is position kv_len[n] - (q_start[n+1] - q_start[n]) + i.
 * cache_dtype: dtype, or DSP_E4M3 where dtype is DSP_BF16: 8-bit codes (3 bits of mantissa,
 *           4 of exponent, no infinity) times k_scale[page][h] and v_scale[page][h] (DEVICE
 *           fp32 [n_pages][Hkv], powers of two; NULL otherwise).
 *
 * dsp_kv_append -- writes the new keys and values (k, v: T rows of Hkv heads, k_stride and
 * v_stride elements apart) into the cache, the first `rot` elements of each key turned by
 * its position as in dsp_qk_norm_rope (cos, sin, P, rot, flags; pos: DEVICE int32 [T], the
 * table's row of each token, or NULL: its position; a position without a row gives NaN in
 * the elements that turn), and, for H > 0, the queries q turned the same way into yq (T
 * rows; in place allowed with equal strides).
 *   DSP_E4M3: a page's scale for a head is the least power of two s, at least 2^-64, with
 *   |x| <= 448 s for every token that the page was given since its slot 0 was written;
 *   where new tokens make it grow, the slots before them are rounded again.  Elements that
 *   are not finite are held as NaN and do not count.  A page whose slot 0 is not among the
 *   new tokens must hold what earlier calls wrote (or scale 0: nothing).
 *   Slots other than the new tokens' (8 bits: and those before them in the page) and rows of
 *   no sequence are left as they were.  A page that is written belongs to one sequence and to one
 *   place of its table.
 *   D up to 256 (dsp_attn_paged: 128), H + 2 Hkv below 2048, at any alignment of an element;
 *   16-byte aligned tensors and tables, with D and rot multiples of 8, are fastest.
 *
 * dsp_attn_paged -- attention of the new tokens (q, o: T rows of H heads, q_stride and
 * o_stride elements apart) over their sequences' cached positions, with the visibility,
 * scale and precision of dsp_attn_window (left -1, right 0: causal without a window).
 * max_q:    no sequence has more new tokens (rows past it are left as they were); a small one
 *           lets the keys be cut among work-groups.
 * lse:      fp32 [T][H], or NULL.
 * Rows of no sequence are left as they were.  DSP_BF16: D a multiple of 8 up to 128,
 * 16-byte aligned q and o and bf16 caches (8-byte for DSP_E4M3) with strides multiples of 8;
 * DSP_F32: any D up to 128.  workspace: dsp_attn_paged_workspace_bytes(...) bytes,
 * 16-byte aligned, of each call's own.
 *
 * Outputs lie apart from everything that the call reads and from one another (DSP_ERR_ARG;
 * the caches: from first element to last).  N <= 2^20, H / Hkv below 2^15, T * H and max_pages * page
 * below 2^30, 64 slots of a page within 2^31 bytes.
 * Errors: DSP_ERR_NULL, DSP_ERR_SHAPE, DSP_ERR_DTYPE, DSP_ERR_ALIGN, DSP_ERR_ARG,
 *   DSP_ERR_WORKSPACE, DSP_ERR_HIP.  No sequences or no rows launch nothing.
 * ------------------------------------------------------------------------ */
int dsp_kv_append(const void* k, const void* v, const void* q, void* yq, void* k_cache, void* v_cache, float* k_scale,
                  float* v_scale, const int32_t* table, const int32_t* q_start, const int32_t* kv_len, const float* cos,
                  const float* sin, const int32_t* pos, int64_t P, int rot, int flags, int64_t N, int64_t T,
                  int64_t n_pages, int64_t max_pages, int page, int H, int Hkv, int D, int64_t k_stride, int64_t v_stride,
                  int64_t q_stride, int64_t yq_stride, const int64_t* cache_strides, int cache_dtype, int dtype,
                  void* stream);
size_t dsp_attn_paged_workspace_bytes(int64_t N, int64_t T, int64_t max_q, int64_t n_pages, int64_t max_pages, int page,
                                      int H, int Hkv, int D, int left, int right, int sinks, int dtype);
int dsp_attn_paged(const void* q, const void* k_cache, const void* v_cache, void* o, float* lse, const float* k_scale,
                   const float* v_scale, const int32_t* table, const int32_t* q_start, const int32_t* kv_len, int left,
                   int right, int sinks, void* workspace, size_t ws_bytes, int64_t N, int64_t T, int64_t max_q,
                   int64_t n_pages, int64_t max_pages, int page, int H, int Hkv, int D, int64_t q_stride,
                   const int64_t* cache_strides, int64_t o_stride, float scale, int cache_dtype, int dtype, void* stream);

/* ------------------------------------------------------------------------
 * dsp_layernorm -- per-row normalisation over C (Eq. 4, 6):
 *   y = (x - mean) / sqrt(var + eps), biased variance, no affine part,
 *   statistics in fp32.
 * x: [rows, C] of x_dtype; y: [rows, C] of y_dtype (DSP_F32 or DSP_BF16).
 * Errors: DSP_ERR_NULL, DSP_ERR_SHAPE (rows < 0, C < 1), DSP_ERR_DTYPE,
 *   DSP_ERR_ARG (eps < 0 or not finite).
 * ------------------------------------------------------------------------ */
int dsp_layernorm(const void* x, int x_dtype, void* y, int y_dtype, int64_t rows, int C, float eps,
                  void* stream);

/* ------------------------------------------------------------------------
 * dsp_layernorm_bwd -- gradient of dsp_layernorm with respect to its input
 * (Eq. 4, 6; used to train the block):
 *   dx = dres + (dy - mean(dy) - y * mean(dy * y)) / sqrt(var + eps),
 *   y = (x - mean) / sqrt(var + eps), statistics of x recomputed in fp32.
 * x: [rows, C] of x_dtype (the forward's input); dy: [rows, C] of dy_dtype;
 * dres: [rows, C] fp32 gradient already flowing into x (e.g. through a
 *   residual connection), or NULL; may equal dx (accumulate in place);
 * dx: [rows, C] fp32.  DEVICE pointers owned by the caller.
 * Errors: DSP_ERR_NULL, DSP_ERR_SHAPE, DSP_ERR_DTYPE, DSP_ERR_ARG (eps < 0
 *   or not finite; dx overlapping x, dy, or dres other than in place).
 * ------------------------------------------------------------------------ */
int dsp_layernorm_bwd(const void* x, int x_dtype, const void* dy, int dy_dtype, const float* dres, float* dx,
                      int64_t rows, int C, float eps, void* stream);

/* ------------------------------------------------------------------------
 * dsp_linear -- out = epilogue(a * W + bias)  (Eq. 1 W^O, Eq. 5 W_1/W_2)
 *
 * a:        [M, K] of dtype.
 * w:        [N, K] of dtype (stored [out][in]).
 * bias:     [N] of dtype at any element's address (4-byte aligned is fastest), or NULL.
 * residual: [M, N] fp32 or NULL; required iff DSP_EPI_RESID.  May equal out.
 * out:      [M, N]; dtype for DSP_EPI_NONE / DSP_EPI_GELU / DSP_EPI_RELU,
 *           fp32 for DSP_EPI_F32 (out = a*W + bias) and DSP_EPI_RESID
 *           (out = residual + a*W + bias).
 * epilogue: DSP_EPI_NONE, DSP_EPI_GELU (erf GELU: x*Phi(x)), DSP_EPI_RESID,
 *           DSP_EPI_F32, DSP_EPI_RELU (max(0, x): the FFN activation of Eq. 5).
 * dtype:    DSP_BF16 (bf16 MFMA, fp32 accumulation) or DSP_F32 (fp32
 *           products and accumulation).
 * bf16 needs K % 8 == 0 and 16-byte aligned a, w, out and residual
 * (DSP_ERR_ALIGN).  out must not overlap a, w or bias.
 * Errors: DSP_ERR_NULL, DSP_ERR_SHAPE (M < 0, N < 1, K < 1), DSP_ERR_DTYPE,
 *   DSP_ERR_ALIGN, DSP_ERR_ARG (unknown epilogue, residual missing).
 * ------------------------------------------------------------------------ */
enum { DSP_EPI_NONE = 0, DSP_EPI_GELU = 1, DSP_EPI_RESID = 2, DSP_EPI_F32 = 3, DSP_EPI_RELU = 4 };
int dsp_linear(const void* a, const void* w, const void* bias, const float* residual, void* out,
               int64_t M, int N, int K, int epilogue, int dtype, void* stream);

/* ------------------------------------------------------------------------
 * Gradients of dsp_linear, y = a * W + bias (W stored [N][K] = [out][in]),
 * for training the block (the paper trains its models; weak scaling is a
 * training stage with ZeRO-2).  Chain rule: da = dy * W^T-stored = dy W,
 * dW = dy^T a, dbias = the column sums of dy.
 *
 * dsp_linear_bwd_data -- dx[M][K] = epilogue(dy[M][N] * W[N][K]).
 *   dy: [M, N] of dtype;  w: [N, K] of dtype (the forward's weight);
 *   u:  [M, K] of dtype, the saved pre-activation for DSP_GRAD_EPI_GELU_BWD
 *       (dx = (dy W) * GELU'(u), GELU'(u) = Phi(u) + u phi(u): the backward
 *       through the MLP's activation, Eq. 5) and DSP_GRAD_EPI_RELU_BWD
 *       (dx = (dy W) where u > 0, else 0); NULL otherwise;
 *   dx: [M, K], fp32 for DSP_GRAD_EPI_F32, dtype otherwise.
 * dsp_linear_bwd_weight -- dw[N][K] = dy^T[N][M] * x[M][K] (fp32) and, when
 *   db is not NULL, db[N] = sum over m of dy[m][n] (fp32).
 *   dy: [M, N] of dtype; x: [M, K] of dtype (the forward's input).
 *   workspace: device memory of at least
 *   dsp_linear_bwd_weight_workspace_bytes(M, N, K, dtype) bytes (may be NULL
 *   when that is 0).  The reduction over M is split across work-groups, and
 *   their fp32 partial sums are added in a fixed order: the result is
 *   deterministic.
 * dtype DSP_BF16: bf16 operands on the matrix cores, fp32 accumulation;
 *   N % 8 == 0 and K % 8 == 0 and 16-byte aligned tensors (DSP_ERR_ALIGN).
 * dtype DSP_F32: fp32 products and accumulation.
 * All pointers are DEVICE pointers owned by the caller; outputs must not
 * overlap inputs (DSP_ERR_ARG).  M == 0: dsp_linear_bwd_data launches
 * nothing; dsp_linear_bwd_weight writes dw = 0 (and db = 0).
 * Errors: DSP_ERR_NULL, DSP_ERR_SHAPE (M < 0, N < 1, K < 1, sizes past the
 *   32-bit tile range), DSP_ERR_DTYPE, DSP_ERR_ALIGN, DSP_ERR_ARG (unknown
 *   epilogue, overlap), DSP_ERR_WORKSPACE, DSP_ERR_HIP.
 * ------------------------------------------------------------------------ */
enum { DSP_GRAD_EPI_F32 = 0, DSP_GRAD_EPI_BF16 = 1, DSP_GRAD_EPI_GELU_BWD = 2, DSP_GRAD_EPI_RELU_BWD = 3 };
int dsp_linear_bwd_data(const void* dy, const void* w, const void* u, void* dx, int64_t M, int N, int K,
                        int epilogue, int dtype, void* stream);
size_t dsp_linear_bwd_weight_workspace_bytes(int64_t M, int N, int K, int dtype);
int dsp_linear_bwd_weight(const void* dy, const void* x, float* dw, float* db, void* workspace,
                          size_t ws_bytes, int64_t M, int N, int K, int dtype, void* stream);

/* ------------------------------------------------------------------------
 * The spatial-temporal block: one GPU's share of one layer of the 2D
 * transformer of the model-details appendix (a spatial block, then a temporal
 * block), with one Switch between them.
 *
 *   x  += Wo_s * SpatialAttn(LN(x) * Wqkv_s)          x in (B,T,S,C)
 *   y   = Switch_{T->S}(x)                             y in (B,S,T,C)
 *   y  += Wo_t * TemporalAttn(LN(y) * Wqkv_t)
 *   y  += W2 * GELU(LN(y) * W1)
 *
 * Weights (dtype, stored [out][in]): wqkv_* [3C][C] with output columns
 * [Q | K | V], wo_* [C][C], w1 [F][C], w2 [C][F]; biases ([out], dtype) may be
 * NULL.  x_BTSC and y_BSTC are fp32 (the residual stream); they must not
 * overlap.  Flags:
 *   DSP_BLOCK_NO_MLP_LN -- no LayerNorm for the MLP;
 *   DSP_BLOCK_ATTN_ONLY -- projections and attention only: no LayerNorm, no
 *     residual adds and no MLP (w1/w2 unused):
 *       y = Wo_t * TemporalAttn(Switch(Wo_s * SpatialAttn(x * Wqkv_s)) * Wqkv_t);
 *   DSP_BLOCK_POST_LN -- every LayerNorm after its residual add, the form of
 *     Eq. 4 and Eq. 6:  x = LN(x + Wo_s * SpatialAttn(x * Wqkv_s)), ...,
 *     y = LN(y + W2 * act(y * W1));
 *   DSP_BLOCK_RELU -- the FFN activation is ReLU (Eq. 5) instead of GELU.
 *   DSP_BLOCK_POST_LN | DSP_BLOCK_RELU is the paper's own block.
 * workspace: device buffer of at least dsp_st_block_workspace_bytes(...)
 * bytes, 256-byte aligned, owned by the caller; contents are scratch.
 * dsp_st_block_workspace_bytes returns 0 for invalid sizes.
 * Errors: those of the pieces plus DSP_ERR_WORKSPACE and DSP_ERR_ARG.
 * ------------------------------------------------------------------------ */
typedef struct {
  const void *wqkv_s, *bqkv_s, *wo_s, *bo_s;
  const void *wqkv_t, *bqkv_t, *wo_t, *bo_t;
  const void *w1, *b1, *w2, *b2;
} dsp_block_weights_t;

enum { DSP_BLOCK_NO_MLP_LN = 1, DSP_BLOCK_ATTN_ONLY = 2, DSP_BLOCK_POST_LN = 4, DSP_BLOCK_RELU = 8 };

size_t dsp_st_block_workspace_bytes(int64_t B, int64_t T, int64_t S, int C, int H, int F,
                                    int dtype);
int dsp_st_block_forward(const float* x_BTSC, float* y_BSTC, const dsp_block_weights_t* w,
                         void* workspace, size_t ws_bytes, int64_t B, int64_t T, int64_t S, int C,
                         int H, int F, float ln_eps, int flags, int dtype, void* stream);

/* ------------------------------------------------------------------------
 * Training the block: a forward that keeps its activations, and the backward.
 * The paper trains its models (weak scaling as a training stage, ZeRO-2), so
 * every step of the block has a gradient: the chain rule through LayerNorm,
 * the linear maps and the MLP activation, attention along each sequence
 * dimension (Eq. 3 per head), and the Switch, whose adjoint is the switch
 * back (S -> T).
 *
 * dsp_st_block_forward_train -- dsp_st_block_forward (same x, y, w, sizes,
 *   eps and dtype) that writes the activations the backward needs into
 *   `saved`: DEVICE memory of at least dsp_st_block_train_saved_bytes(...)
 *   bytes for the same sizes, flags and dtype, 256-byte aligned, owned by the
 *   caller (1.7 GB at B1 T32 S1024 C1152 F4608 in bf16, pre-LN; post-LN with
 *   the MLP's LayerNorm keeps one more fp32 stream).  Flags: any combination
 *   of DSP_BLOCK_NO_MLP_LN, DSP_BLOCK_POST_LN (Eq. 4, 6: LN after each
 *   residual add) and DSP_BLOCK_RELU; the projection-only chain
 *   (DSP_BLOCK_ATTN_ONLY) gives DSP_ERR_ARG.  y has the bits
 *   dsp_st_block_forward writes for the same arguments (the MLP's first GEMM
 *   stores, from the same fp32 sum as the activation, what the activation's
 *   backward needs: the pre-activation, or GELU' there when the block is
 *   bf16 with GELU at sizes that fill every CU with 256-wide tiles).
 * dsp_st_block_backward -- given the forward's x (B,T,S,C), its saved
 *   activations, and dy (B,S,T,C) = dL/dy, writes dx = dL/dx (B,T,S,C, fp32)
 *   and the weight gradients into `grads`: fp32 arrays shaped like the weights
 *   (stored [out][in]), required for the six weights; bias gradients are
 *   written where the pointer is not NULL (whether or not the forward used a
 *   bias).  workspace: DEVICE scratch of at least
 *   dsp_st_block_backward_workspace_bytes(...) bytes, 256-byte aligned.
 *   Gradients are deterministic (no atomics).  bf16: the operands of every
 *   product are bf16 (gradients rounded to bf16 where they enter a product),
 *   accumulation and the residual-stream gradient are fp32.
 * Errors: as dsp_st_block_forward, plus DSP_ERR_WORKSPACE (saved or
 *   workspace missing or too small) and DSP_ERR_ARG (unsupported flags,
 *   overlapping buffers).
 * ------------------------------------------------------------------------ */
typedef struct {
  float *wqkv_s, *bqkv_s, *wo_s, *bo_s, *wqkv_t, *bqkv_t, *wo_t, *bo_t, *w1, *b1, *w2, *b2;
} dsp_block_grads_t;
size_t dsp_st_block_train_saved_bytes(int64_t B, int64_t T, int64_t S, int C, int H, int F, int flags,
                                      int dtype);
size_t dsp_st_block_backward_workspace_bytes(int64_t B, int64_t T, int64_t S, int C, int H, int F, int dtype);
int dsp_st_block_forward_train(const float* x_BTSC, float* y_BSTC, const dsp_block_weights_t* w, void* saved,
                               size_t saved_bytes, int64_t B, int64_t T, int64_t S, int C, int H, int F,
                               float ln_eps, int flags, int dtype, void* stream);
int dsp_st_block_backward(const float* x_BTSC, const float* dy_BSTC, const dsp_block_weights_t* w,
                          const void* saved, size_t saved_bytes, void* workspace, size_t ws_bytes, float* dx_BTSC,
                          const dsp_block_grads_t* grads, int64_t B, int64_t T, int64_t S, int C, int H, int F,
                          float ln_eps, int flags, int dtype, void* stream);

/* ------------------------------------------------------------------------
 * Measurement aid (not a step of the method): the bf16 MFMA rate the chip
 * sustains with every CU busy.  The published dense bf16 figure assumes the
 * peak engine clock; under a long all-CU MFMA load the clock settles lower.
 * A benchmark reports a kernel's fraction of the published peak, and this
 * rate beside it, measured in the same process and conditions.
 *
 * dsp_probe_mfma -- launches 2048 work-groups of 4 waves (two per SIMD), each
 *   wave issuing 8 * iters independent v_mfma_f32_32x32x16_bf16 on operands
 *   whose bits change every iteration; nothing else runs in its loop.  The
 *   caller times it (events on `stream`) and divides
 *   dsp_probe_mfma_flops(iters) by the time.  workspace: DEVICE memory of at
 *   least dsp_probe_mfma_workspace_bytes() bytes, 16-byte aligned (receives
 *   one float per thread, meaningless).  Errors: DSP_ERR_ARG (iters < 1),
 *   DSP_ERR_NULL, DSP_ERR_WORKSPACE, DSP_ERR_ALIGN.
 * ------------------------------------------------------------------------ */
size_t dsp_probe_mfma_workspace_bytes(void);
double dsp_probe_mfma_flops(int iters);
int dsp_probe_mfma(void* workspace, size_t ws_bytes, int iters, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* DSP_H_ */
