/*
 * ragged.h -- C ABI of the MI355X (gfx950) pack -> ragged attention -> unpack library.
 *
 * The three stages are the pack-attend-unpack pipeline of "Dispatch-Aware Ragged Attention for
 * Pruned Vision Transformers" (Section 4, "Method"): a keep mask produced by any token-pruning
 * method selects the surviving tokens of each image; they are packed into one flat buffer indexed
 * by cu_seqlens, attended per image, and scattered back.
 *
 * Conventions shared by every entry point
 *   - B images, N tokens per image before pruning, H heads, head dim D, row width C = H*D.
 *   - n_i = kept tokens of image i, T = sum_i n_i = cu_seqlens[B].
 *   - Every pointer except `stream` is a DEVICE pointer owned by the caller.  The library never
 *     allocates, frees or keeps a pointer, never synchronises and never copies to the host: each
 *     call enqueues exactly one kernel on `stream` (ragged_layernorm_backward and ragged_grad_clip:
 *     two) and returns, so all calls are legal inside a HIP stream capture.  The two calls that only
 *     prepare host data (ragged_rope_frequencies, ragged_grad_plan) enqueue nothing and take HOST pointers.  T is never read on the host; grids are sized by upper bounds and
 *     surplus work-groups exit on the device.
 *   - `stream` is a hipStream_t passed as void*; NULL is the default stream.
 *   - 16-bit floating rows are moved as raw words by pack / unpack (bit copy).
 *   - Return value: a ragged_status.  RAGGED_OK means "enqueued".  Arguments are validated on the
 *     host before anything is launched; a validation failure launches nothing.
 *   - x, packed, src, out, q, k, v, o must be 16-byte aligned; C must be a multiple of 8.
 *   - Calls on one stream are ordered; the caller orders calls across streams.
 */
#ifndef RAGGED_H
#define RAGGED_H

#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
    RAGGED_OK = 0,
    RAGGED_ERR_NULL = 1,         /* a required pointer is NULL                                   */
    RAGGED_ERR_SHAPE = 2,        /* a dimension is <= 0, overflows int32 row indexing, or a token
                                    stride is shorter than a row                                  */
    RAGGED_ERR_UNSUPPORTED = 3,  /* dtype pair, head dim, alignment or fill mode not supported    */
    RAGGED_ERR_CAPACITY = 4,     /* a row capacity is < 1 (ragged_pack_attn_unpack: < B*N)        */
    RAGGED_ERR_HIP = 5           /* the HIP runtime refused the launch                            */
} ragged_status;

typedef enum {
    RAGGED_F16 = 0,              /* IEEE binary16                                                 */
    RAGGED_BF16 = 1,             /* bfloat16                                                      */
    RAGGED_F32 = 2               /* IEEE binary32; attention output only                          */
} ragged_dtype;

/*
 * ragged_pack -- Section 4.1 "Fused Token Packing", both phases in ONE launch and without the
 * paper's host read of the total kept count.
 *
 *   x          [B, N, C]   16-bit rows (dt = RAGGED_F16 or RAGGED_BF16; only the width matters)
 *   keep       [B, N]      one byte per token, any nonzero value = keep
 *   packed     [cap_rows, C]  out: kept rows in stable order (images ascending, tokens ascending)
 *   cu_seqlens [B + 1]     out: cu[0] = 0, cu[i+1] = cu[i] + n_i
 *   gather_idx [cap_rows]  out: gather_idx[r] = flat source row i*N + t of packed row r
 *
 * Cost note: every work-group recounts the keep bytes in front of its chunk (no grid-wide scan, no second
 * launch, no workspace), i.e. O(B*N) mask bytes per work-group from L2.  That is free at ViT batch sizes (B*N up to
 * a few 10^4) and grows quadratically with the batch: around B*N = 10^6 the recount costs as much as the copy.
 * ragged_repack and ragged_pack_attn_unpack count the same way.
 *
 * cap_rows is the row capacity of `packed` and `gather_idx`.  B*N always suffices.  Rows whose
 * destination would be >= cap_rows are not written (cu_seqlens still holds the true counts, so the
 * caller can detect the overflow from cu_seqlens[B] afterwards).  Rows >= T are left untouched.
 */
int ragged_pack(const void* x, const uint8_t* keep, int B, int N, int C, ragged_dtype dt,
                void* packed, int64_t cap_rows, int32_t* cu_seqlens, int32_t* gather_idx,
                void* stream);

/*
 * ragged_attn -- Section 4.2 "Ragged Attention Kernel" (Algorithm 1): for every image i, head h
 * and query row r of that image,
 *     o[s+r, h, :] = softmax_j( scale * q[s+r, h, :] . k[s+j, h, :] ) v[s+j, h, :],
 *     s = cu_seqlens[i], j in [0, n_i)
 * bidirectional (no causal mask), no dropout, keys of other images never take part.
 *
 *   q, k, v    [T, H, D]   token-major, then head, then head dim contiguous (in_dt)
 *   o          [T, H, D]   out (out_dt); rows >= T are left untouched
 *   cu_seqlens [B + 1]     as written by ragged_pack
 *   max_seqlen             host-known upper bound on every n_i (N always works); it only sizes
 *                          the grid.  Query rows at positions >= max_seqlen inside an image are
 *                          NOT computed, so a bound that is too small loses rows (ragged_attn_checked
 *                          reports that case on the device).
 *   scale                  finite fp32 softmax scale (the paper uses 1/sqrt(D))
 *
 * Supported: D = 64; (in_dt, out_dt) in {F16->F16, F16->F32, BF16->BF16, BF16->F32}.
 * Limits of the launch (RAGGED_ERR_SHAPE beyond them; the same for every attention entry point, with N in
 * place of max_seqlen where the call has no bound): max_seqlen <= 64 * 65535, B * H <= 512 * 65535, and
 * ceil(B*H / 512) * 512 * ceil(max_seqlen / 64) < 2^31 work-groups.
 * Contractions run on MFMA with fp32 accumulation; the softmax runs in fp32.
 * Images with n_i = 0 produce no rows.  Results are bit-reproducible from run to run with the same arguments.
 * The launch shape follows B, H and max_seqlen (small launches split the keys of a sequence over the wavefronts
 * of a work-group and merge the partial results, large ones walk them in order), so the bits of a sequence
 * longer than 64 tokens may differ in the last place between calls with different B, H or max_seqlen; all the
 * entry points of this header take the same shape for the same (B, H, bound), so they stay bit-identical to
 * each other.
 */
int ragged_attn(const void* q, const void* k, const void* v, void* o,
                const int32_t* cu_seqlens, int B, int max_seqlen, int H, int D,
                float scale, ragged_dtype in_dt, ragged_dtype out_dt, void* stream);

/*
 * ragged_attn_strided -- ragged_attn on token rows that are not contiguous: token t of q, k, v
 * starts in_tok_stride elements after token t-1, token t of o out_tok_stride elements after its
 * predecessor; inside a token the layout stays [H, D].  This is what the late layers of Section 4.3
 * ("End-to-End Pipeline Integration", step 4: attention and MLP run on the packed buffer) need
 * between their linear layers: the QKV projection of packed rows writes one [T, 3, H, D] buffer, and
 * q = base, k = base + H*D, v = base + 2*H*D with in_tok_stride = 3*H*D attends on it in place,
 * without three de-interleaving copies.  ragged_attn is this call with both strides = H*D.
 *
 * Strides are in elements of the respective dtype, must be >= H*D (in_tok_stride also <= 2^23 and
 * out_tok_stride < 2^31, else RAGGED_ERR_SHAPE), and every token row must start
 * on a 16-byte boundary (in_tok_stride a multiple of 8; out_tok_stride a multiple of 8 for 16-bit
 * outputs, of 4 for F32).  Everything else as for ragged_attn; outputs are bit-identical to
 * ragged_attn on contiguous copies of the same rows.
 */
int ragged_attn_strided(const void* q, const void* k, const void* v, void* o,
                        const int32_t* cu_seqlens, int B, int max_seqlen, int H, int D,
                        int64_t in_tok_stride, int64_t out_tok_stride, float scale,
                        ragged_dtype in_dt, ragged_dtype out_dt, void* stream);

/*
 * ragged_attn_checked -- ragged_attn_strided that also reports a `max_seqlen` that was too small.
 * Section 4.2 sizes its grid from the host-known sequence bound; here that bound is an argument, a bound
 * below some n_i silently leaves query rows of that image uncomputed, and the host cannot see n_i without
 * the synchronisation this library avoids.  This entry point closes the gap on the device:
 *
 *   flags      [1]  int32, caller-zeroed.  Bit 0 (RAGGED_FLAG_SEQLEN_EXCEEDED) is OR-ed in when some image
 *                   has n_i > max_seqlen.  The library never clears it; the caller reads it whenever it
 *                   next synchronises (or never).
 *
 * Query rows at positions >= max_seqlen of an offending image may be left uncomputed (such a row of `o` then stays
 * untouched as a whole; rows at positions >= 64 * ceil(max_seqlen / 64) always do); every other row of the batch is
 * computed as by ragged_attn_strided with the same arguments, bit for bit.
 * ragged_pack_attn_unpack and ragged_attn_padded size their grids from N itself and can never lose a row.
 */
#define RAGGED_FLAG_SEQLEN_EXCEEDED 1
int ragged_attn_checked(const void* q, const void* k, const void* v, void* o,
                        const int32_t* cu_seqlens, int B, int max_seqlen, int H, int D,
                        int64_t in_tok_stride, int64_t out_tok_stride, float scale,
                        ragged_dtype in_dt, ragged_dtype out_dt, int32_t* flags, void* stream);

/*
 * ragged_unpack -- the inverse scatter of ragged_pack (the paper names the stage in its
 * "pack-attend-unpack pipeline", Sections 1 and 4, without describing it).
 *
 *   src        [T, C]      packed rows
 *   out        [B, N, C]   out: out[i, t, :] = src[cu[i] + rank(i, t), :] for kept tokens
 *   fill_mode  0: dropped rows of `out` are left untouched.  Reads gather_idx and cu_seqlens[B];
 *                 `keep` may be NULL.
 *              1: dropped rows are written with +0 words, so every byte of `out` is defined.
 *                 Reads keep and cu_seqlens; `gather_idx` may be NULL.
 */
int ragged_unpack(const void* src, const uint8_t* keep, const int32_t* cu_seqlens,
                  const int32_t* gather_idx, int B, int N, int C, ragged_dtype dt,
                  void* out, int fill_mode, void* stream);

/*
 * ragged_attn_padded -- the whole pack-attend-unpack pipeline of Section 4 for ONE attention layer
 * in ONE launch: the kernel turns each image's keep mask into its list of kept token positions and
 * reads / writes Q, K, V, O rows through that list, so no packed copy, no cu_seqlens and no gather
 * index exist.  Same arithmetic as ragged_attn on the packed rows (bit-identical outputs).  The
 * paper's argument (Section 3 and Section 4.2, "Why dispatch overhead is lower") is that at ViT sizes
 * the number of dispatches, not the arithmetic, sets the latency; this entry point removes two of
 * the three.
 *
 *   q, k, v    [B, N, H, D]  padded, token-major inside an image (in_dt); rows of dropped tokens are
 *                            never read
 *   o          [B, N, H, D]  out (out_dt): rows of kept tokens receive the attention output;
 *                            fill_mode 0 leaves rows of dropped tokens untouched, 1 writes +0
 *   keep       [B, N]        one byte per token, any nonzero value = keep
 *
 * Supported: D = 64, N <= 1536, the dtype pairs of ragged_attn.  Images with nothing kept produce no
 * attention rows.
 */
int ragged_attn_padded(const void* q, const void* k, const void* v, void* o, const uint8_t* keep,
                       int B, int N, int H, int D, float scale, ragged_dtype in_dt,
                       ragged_dtype out_dt, int fill_mode, void* stream);

/*
 * ragged_pack_attn_unpack -- ragged_pack, ragged_attn and ragged_unpack of one layer (the three
 * stages of Section 4) in ONE launch, with every output of the three calls produced and bit-identical
 * to theirs.  Section 3 and Section 4.2 ("Why dispatch overhead is lower") argue that at ViT sizes the
 * number of dispatches sets the latency; this entry point is that argument applied to the paper's
 * own pipeline.  Each work-group (image, head, 64-query tile) recounts the image's first packed row
 * and its kept-token list from the keep mask, so there is no dependency between work-groups.
 *
 *   x          [B, N, C]      padded features (dt), C = H*D
 *   keep       [B, N]         one byte per token, nonzero = keep
 *   q, k, v    [cap_rows, H, D]  ALREADY packed query / key / value rows (dt); rows [0, T) are read
 *   packed     [cap_rows, C]  out: as from ragged_pack(x, keep)
 *   cu_seqlens [B + 1]        out: as from ragged_pack
 *   gather_idx [cap_rows]     out: as from ragged_pack
 *   o          [cap_rows, H, D]  out (dt): as from ragged_attn(q, k, v, cu_seqlens)
 *   out        [B, N, C]      out: as from ragged_unpack(o, ..., fill_mode)
 *
 * Supported: D = 64, N <= 1536, dt = F16 or BF16 (o has the input dtype).  cap_rows must be >= B*N
 * (RAGGED_ERR_CAPACITY otherwise), so nothing can overflow.  x, packed, o, out must not overlap.
 */
int ragged_pack_attn_unpack(const void* x, const uint8_t* keep, const void* q, const void* k, const void* v,
                            int B, int N, int H, int D, float scale, ragged_dtype dt, void* packed,
                            int64_t cap_rows, int32_t* cu_seqlens, int32_t* gather_idx, void* o, void* out,
                            int fill_mode, void* stream);

/*
 * ragged_repack -- a second pruning decision applied to rows that are ALREADY packed.  Section 4.3
 * packs once and keeps every later layer on the packed buffer; pruning methods that drop tokens
 * at several depths (Section 2, "Token Pruning for ViTs": DynamicViT and EViT prune progressively)
 * then need a keep mask applied to packed rows, instead of an unpack -> pack round trip through
 * the padded tensor.  Equivalent to ragged_pack with the AND of both masks, in one launch:
 *
 *   packed_in  [cap_in, C]  packed rows; rows [0, T_in) are valid, T_in = cu_in[B] <= cap_in
 *   keep_rows  [cap_in]     one byte per packed row, nonzero = keep; bytes at rows >= T_in are ignored
 *   cu_in      [B + 1]      boundaries of packed_in
 *   packed_out [cap_out, C] out: kept rows in the same order
 *   cu_out     [B + 1]      out: cu_out[i] = number of kept rows before row cu_in[i]
 *   gather_out [cap_out]    out: gather_out[r] = row of packed_in that packed_out row r came from
 *                           (compose with the first gather_idx to get back to the padded tensor)
 *
 * Rows whose destination would be >= cap_out are not written (cu_out still holds the true counts).
 * packed_out must not overlap packed_in; cu_out must not alias cu_in.
 */
int ragged_repack(const void* packed_in, const uint8_t* keep_rows, const int32_t* cu_in, int B,
                  int64_t cap_in, int C, ragged_dtype dt, void* packed_out, int64_t cap_out,
                  int32_t* cu_out, int32_t* gather_out, void* stream);

/*
 * ragged_cls_extract -- step 5 of Section 4.3: the classifier reads each image's class token from
 * the packed buffer.  Packing keeps token order (Section 4.1), so a class token at position 0 that
 * the keep mask retains is the image's first packed row.
 *
 *   packed     [T, C]   packed rows
 *   cu_seqlens [B + 1]
 *   out        [B, C]   out: out[i, :] = packed[cu_seqlens[i], :]; +0 words for an image with no rows
 */
int ragged_cls_extract(const void* packed, const int32_t* cu_seqlens, int B, int C, ragged_dtype dt,
                       void* out, void* stream);

/*
 * ragged_linear -- a linear layer over packed rows, for the encoder blocks that Section 4.3 (item 4)
 * runs on the packed buffer after the pruning point (QKV projection, attention output projection and
 * the two MLP layers; Section 6, "Implications for pruning research", attributes most of the
 * realised speed-up of pruning to these, because their cost is linear in the number of kept tokens):
 *     y[m, n] = act( sum_k x[m, k] * w[n, k] + bias[n] ) + residual[m, n]
 *
 *   x        [rows_cap, K]  packed activations (dt)
 *   w        [N, K]         weights, one output feature per row (dt)
 *   bias     [N] or NULL    (dt)
 *   residual [rows_cap, N] or NULL (dt); may be the same buffer as y (each element is read before
 *                           it is written, by the same thread)
 *   y        [rows_cap, N]  out (dt); must not overlap x
 *   rows_dev                NULL, or a DEVICE pointer to the number of valid rows (for example
 *                           &cu_seqlens[B]); rows processed = min(rows_cap, *rows_dev), read on the
 *                           device, so the call stays capturable.  Rows beyond are left untouched.
 *   rows_hint               0, or the caller's estimate of the valid row count (1 <= rows_hint <=
 *                           rows_cap), e.g. keep ratio * B * N: it only chooses the launch shape (the
 *                           result and the rows written do not depend on it).  0 means rows_cap.
 *   act                     0: none, 1: GELU in its erf form t * Phi(t)
 *
 * Supported: dt = F16 or BF16, N and K multiples of 64, K <= 2^22.  MFMA with fp32
 * accumulation; bias, activation and residual are applied in fp32 before the single rounding to dt.
 */
int ragged_linear(const void* x, const void* w, const void* bias, const void* residual, void* y,
                  int64_t rows_cap, const int32_t* rows_dev, int64_t rows_hint, int N, int K, int act,
                  ragged_dtype dt, void* stream);

/*
 * ragged_layernorm -- LayerNorm over the feature dimension of packed rows (same blocks as above):
 *     y[m, :] = (x[m, :] - mean) / sqrt(var + eps) * gamma + beta,   var = biased variance of the row
 * x, y [rows_cap, C]; gamma, beta [C]; rows_dev as for ragged_linear.  y may be x.
 * Supported: dt = F16 or BF16, C a multiple of 8 and <= 2048, eps >= 0.  Statistics in fp32.
 */
int ragged_layernorm(const void* x, const void* gamma, const void* beta, void* y, int64_t rows_cap,
                     const int32_t* rows_dev, int C, float eps, ragged_dtype dt, void* stream);

/*
 * ragged_token_scores_l2 and ragged_keep_topk -- a keep-mask producer in front of ragged_pack.  The
 * pipeline takes its keep mask from any pruning method (Section 4.3 item 2); the paper's timings use
 * a threshold on the l2 norm of the token features at a fixed ratio (Section 5) and leave the method
 * undefined.  The definition taken here: score = squared l2 norm of the token's feature row; per
 * image the class token (position 0) is kept and, of the other tokens, the k-1 with the largest
 * score, equal scores ordered by position (lower first).  Every image then keeps min(k, N) tokens,
 * the uniform-length setting of the paper's kernel-latency tables.  ragged_keep_topk is independent
 * of how the scores were made (attention-based scores of other pruning methods fit as well).
 *
 *   x      [rows, C]   token features (dt), rows = B*N
 *   scores [rows]      out / in: fp64, 8-byte aligned.  Accumulated in fp64 (squares of 16-bit values
 *                      are exact there), so ranking does not depend on the summation order except
 *                      between scores that agree to the last bit of a rounded sum
 *   keep   [B, N]      out: 1 = keep, 0 = drop
 *
 * Supported: dt = F16 or BF16, C a multiple of 8; N <= 1536, k >= 1 (k >= N keeps everything).
 */
int ragged_token_scores_l2(const void* x, int64_t rows, int C, ragged_dtype dt, double* scores, void* stream);
int ragged_keep_topk(const double* scores, int B, int N, int k, uint8_t* keep, void* stream);

/*
 * ---- Training on packed rows ---------------------------------------------------------------------
 * What the encoder blocks of Section 4.3 (item 4) need on the way back, on the same packed rows: positions that survive packing,
 * attention with its gradients, LayerNorm's gradients, and the norm and clipping of a model's gradients.  Rows beyond the valid ones are
 * neither read nor written, as everywhere here.
 *
 * ragged_rope -- rotary positions: in every head the first 2 * pairs elements are rotated, two by two,
 *     y[a] = m (x[a] cos t - x[b] sin t),   y[b] = m (x[a] sin t + x[b] cos t),   t = coords[c, axis(p)] * freqs[p]
 * for pair p = 0 .. pairs - 1; the other elements of the head are passed on.  One launch for query and key rows.
 *
 *   q, q_out   [rows, Hq, D]  rows q_stride / q_out_stride elements apart, [Hq, D] contiguous inside a row (dt)
 *   k, k_out   [rows, Hk, D]  the same with k_stride / k_out_stride and their own number of heads; both NULL: no keys
 *              q_out may be q (then with the same stride) and k_out may be k; other overlaps are not allowed (q_out = k, k_out = q and
 *              q_out = k_out are refused, RAGGED_ERR_UNSUPPORTED)
 *   rows_cap, rows_dev        as for ragged_linear
 *   coords     [n_coords, axes]  fp32 positions; row r has those of line  u mod n_coords,  u = index[r] as an unsigned number
 *                             (index NULL: r itself).  Packed rows of images pass gather_idx and the N tokens' coordinates, text passes
 *                             its positions and the numbers 0 .. n_coords - 1
 *   freqs      [pairs]        fp64 radians per unit (see ragged_rope_frequencies); axis(p) = p / (pairs / axes): with two
 *                             axes the first half of the pairs turns with coords[., 0], the second with coords[., 1]
 *   layout     0: half, a = p, b = pairs + p;  1: interleaved, a = 2 p, b = 2 p + 1
 *   amplitude  m; inverse 1: t negated.  The rotation's transpose, which takes gradients back, is inverse 1 with the same m
 *
 * Angles are formed and brought to one turn in fp64, sines, cosines and the rotation are fp32, one rounding to dt.
 * Supported: dt = F16 or BF16, D a multiple of 8 and <= 512, 1 <= pairs <= D / 2, pairs a multiple of axes, (Hq + Hk) * D <= 2^22,
 * strides multiples of 8 that hold a row and < 2^31, finite amplitude.
 */
int ragged_rope(const void* q, const void* k, void* q_out, void* k_out, int64_t rows_cap, const int32_t* rows_dev, int Hq, int Hk, int D,
                int64_t q_stride, int64_t k_stride, int64_t q_out_stride, int64_t k_out_stride, const float* coords, int64_t n_coords,
                int axes, const int32_t* index, const double* freqs, int pairs, int layout, float amplitude, int inverse,
                ragged_dtype dt, void* stream);

/*
 * ragged_rope_frequencies -- the frequencies of one axis, P pairs, into HOST memory (an axis' part of freqs above):
 *     f[p] = base^(-p / P)
 *   scaling 0: as they are;  1: f / factor (positions interpolated);  2: with base * factor^(P / (P - 1)) for base: the highest
 *   frequency stays, the lowest is divided by factor (P = 1: stays);  3: by parts: with r = original_length * f / (2 pi) turns over the
 *   original length and g = (r - slow) / (fast - slow) held to [0, 1],  f * g + f / factor * (1 - g): what turns often stays, what turns
 *   seldom is interpolated.
 * base, factor > 0; scaling 3: original_length > 0, fast > slow.  The last three are not looked at otherwise.
 */
int ragged_rope_frequencies(double* freqs, int pairs, double base, int scaling, double factor, double original_length, double fast, double slow);

/*
 * ragged_attn_lse -- ragged_attn_strided that also writes what the backward pass needs of it:
 *   lse        [T, H]   fp32 out: lse[s + r, h] = ln sum_j exp( scale * q[s+r, h, :] . k[s+j, h, :] ); rows >= T are left untouched, and so
 *                        may be, as in o, rows at positions >= max_seqlen of a sequence that is longer than this bound
 * o has the dtype of the inputs and is bit-identical to ragged_attn_strided's with the same arguments.
 */
int ragged_attn_lse(const void* q, const void* k, const void* v, void* o, float* lse, const int32_t* cu_seqlens, int B, int max_seqlen, int H,
                    int D, int64_t in_tok_stride, int64_t out_tok_stride, float scale, ragged_dtype dt, void* stream);

/*
 * ragged_attn_backward -- the gradients of q, k and v of ragged_attn_lse, given that of o, in one launch:
 *     P = exp(scale q k^T - lse),  dS = P * (dO v^T - rowsum(dO * o)),  dv = P^T dO,  dq = scale dS k,  dk = scale dS^T q
 *
 *   q, k, v    [T, H, D]  as given to ragged_attn_lse, in_tok_stride elements between tokens
 *   o, d_o     [T, H, D]  its output and that output's gradient, out_tok_stride elements between tokens
 *   lse        [T, H]     as it wrote them
 *   dq, dk, dv [T, H, D]  out (dt), grad_tok_stride elements between tokens (for example the slices of a fused [T, 3, H, D] buffer);
 *                         they must not overlap any input or each other (the same address is refused, RAGGED_ERR_UNSUPPORTED).  Rows >= T
 *                         are left untouched
 *   max_seqlen            an upper bound on every n_i.  Of a sequence that is longer all the same, gradients of rows at positions >= max_seqlen may be
 *                         left uncomputed (such a row then stays untouched as a whole); dq of the rows below is right, and dk and dv, sums over all
 *                         of its queries, are right only where o and lse hold all of its rows.  A forward call with the same bound has left the
 *                         last ones unwritten, and these dk and dv then mean nothing (ragged_attn_checked tells whether a bound holds).  Other
 *                         sequences are right either way
 *
 * Supported: D = 64, dt = F16 or BF16; every token row on a 16-byte boundary; strides as for ragged_attn_strided (grad_tok_stride as
 * out_tok_stride).  max_seqlen <= 64 * 32767 and half of the work-groups of ragged_attn's limit.  Products on MFMA with fp32 sums;
 * P and dS are rounded to dt in between; with fp16 as 2^15 P and F dS, where F is a power of two that the kernel takes from dO and v, 1 or more unless
 * dS would overflow with it: neither leaves the type's range, F dS loses bits below 2^-14 only, and a gradient is infinite only where its own value is.
 * In sequences of up to 32 rows rowsum(dO * o) is formed as rowsum(P * dO v^T) in fp32 (the rounding of o does not tell), and a sequence of
 * one row gets dq = dk = 0.
 * No atomics: results are bit-reproducible, and those of a sequence do not depend on the other sequences or, as long as it holds, on max_seqlen.
 */
int ragged_attn_backward(const void* q, const void* k, const void* v, const void* o, const void* d_o, const float* lse, void* dq, void* dk,
                         void* dv, const int32_t* cu_seqlens, int B, int max_seqlen, int H, int D, int64_t in_tok_stride,
                         int64_t out_tok_stride, int64_t grad_tok_stride, float scale, ragged_dtype dt, void* stream);

/*
 * ragged_layernorm_backward -- the gradients of ragged_layernorm.  With xh = (x - mean) / sqrt(var + eps) and w = gamma * dy, row by row:
 *     dx = (w - mean(w) - xh mean(w xh)) / sqrt(var + eps)  [+ residual_grad],   dgamma = sum_rows dy xh,   dbeta = sum_rows dy
 *
 *   x, dy, dx      [rows_cap, C] (dt); gamma [C] (dt); dx may be dy or residual_grad (each element is read before it is written, by
 *                  the same thread), and must not be x; other overlaps of what is written (workspace among it) are not allowed
 *   residual_grad  [rows_cap, C] (dt) or NULL: the gradient that reaches x past the LayerNorm (x + f(LN(x)))
 *   dgamma, dbeta  [C] fp32 out (0 where there are no rows)
 *   workspace      ragged_layernorm_backward_workspace(rows_cap, C) bytes, 16-byte aligned; its contents before and after the call mean
 *                  nothing, and calls that may run at the same time (other streams, other captured graphs) need one each
 *   rows_dev       as for ragged_linear
 * Nothing of the forward pass is needed but x.  Types and widths as for ragged_layernorm; two kernels; sums in one order (bit-reproducible).
 */
int64_t ragged_layernorm_backward_workspace(int64_t rows_cap, int C);      /* bytes; 0 for sizes that are not supported */
int ragged_layernorm_backward(const void* x, const void* gamma, const void* dy, const void* residual_grad, void* dx, float* dgamma,
                              float* dbeta, void* workspace, int64_t rows_cap, const int32_t* rows_dev, int C, float eps, ragged_dtype dt,
                              void* stream);

/*
 * ragged_grad_plan and ragged_grad_clip -- the norm over the gradients of a whole model, and the gradients clipped by it:
 *     norm = |scale| * sqrt( sum over all tensors of g^2 ),   dst = g * scale * min(1, max_norm / (norm + 1e-6))
 * scale undoes a loss scale (1 otherwise).  A norm that is infinite or no number clips nothing (dst = g * scale): it is written all the
 * same, and whoever steps the weights looks at it there.
 *
 * ragged_grad_plan lays the tensors out once, as a table of equal pieces in HOST memory, which the caller copies to the device:
 *   tensors    [n]  host array: src and dst are DEVICE pointers (aligned to their own values), numel >= 0; src_dt F16, BF16 or F32, dst_dt
 *                   the same or F32.  dst may be src (then of the same dtype) or NULL (the tensor counts for the norm only); other
 *                   overlaps are not allowed
 *   table      host memory of capacity bytes, or NULL to learn the size;  chunks: out, host: RAGGED_GRAD_CHUNK_BYTES of table each
 * ragged_grad_clip runs it (two kernels):
 *   table      the table in DEVICE memory, 16-byte aligned, chunks as given back
 *   workspace  RAGGED_GRAD_WORKSPACE bytes, 16-byte aligned; calls that may run at the same time need one each
 *   norm       [1] fp64 out, 8-byte aligned
 *   max_norm   > 0, may be infinite (no clipping);  scale finite
 * Squares and their sums are fp64, in one order (bit-reproducible).  With dst = src and a factor of 1 nothing is rewritten.
 */
#define RAGGED_GRAD_CHUNK_BYTES 32
#define RAGGED_GRAD_WORKSPACE 16384
typedef struct {
    const void* src;
    void* dst;
    int64_t numel;
    int32_t src_dt, dst_dt;      /* ragged_dtype */
} ragged_grad_tensor;
int ragged_grad_plan(const ragged_grad_tensor* tensors, int n, void* table, int64_t capacity, int64_t* chunks);
int ragged_grad_clip(const void* table, int64_t chunks, float scale, float max_norm, void* workspace, double* norm, void* stream);

/*
 * ragged_noop -- enqueue an empty kernel of `grid` work-groups of 256 threads on `stream`.
 * It exists to measure the launch floor that Section 3 ("The Dispatch Overhead") is about,
 * separately from the time the real kernels spend on the GPU.
 */
int ragged_noop(int grid, void* stream);

/* Text for a ragged_status (static storage; never free it).  Unknown codes give "unknown". */
const char* ragged_status_string(int status);

/* Library version: major * 10000 + minor * 100 + patch. */
int ragged_version(void);

#ifdef __cplusplus
}
#endif
#endif /* RAGGED_H */
